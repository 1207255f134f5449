"""Pins of the MXFP4 and expert-order oracle (CPU)."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import mx_moe_oracle as mx


def test_e2m1_is_sign_two_exponent_bits_one_mantissa_bit():
    for code in range(16):
        e, m = (code >> 1) & 3, code & 1
        v = m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        assert mx.e2m1_decode(code) == (-v if code & 8 else v)
        assert np.signbit(mx.e2m1_decode(code)) == bool(code & 8)


def test_rounding_is_to_nearest_with_ties_to_even():
    grid = mx.E2M1
    for i in range(7):
        mid = (grid[i] + grid[i + 1]) / 2
        even = i if i % 2 == 0 else i + 1
        for sign in (1, -1):
            s = 8 if sign < 0 else 0
            assert mx.e2m1_nearest(sign * mid) == even + s
            assert mx.e2m1_nearest(sign * np.nextafter(mid, 9)) == i + 1 + s
            assert mx.e2m1_nearest(sign * np.nextafter(mid, -9)) == i + s
    assert mx.e2m1_nearest(np.array([0.0, -0.0])).tolist() == [0, 8]


@pytest.mark.parametrize("seed", range(4))
def test_scale_is_the_smallest_power_of_two_that_keeps_elements_below_six(seed):
    rng = np.random.default_rng(seed)
    a = np.abs(rng.standard_normal(200)).astype(np.float32) * np.float32(2.0) ** rng.integers(-130, 125, 200).astype(np.float32)
    a = np.concatenate([a, np.float32([1.0, 1.5, 6.0, np.nextafter(np.float32(6), np.float32(7)), 3.0, 2.0 ** -149, 3.0e38, 12.0])])
    for v in a[a > 0]:
        e, x = mx.scale_exponent(float(v)), Fraction(float(v))
        assert 6 * Fraction(2) ** e >= x and e >= -127
        assert e == -127 or 6 * Fraction(2) ** (e - 1) < x


def test_quantizer_round_trip_packing_and_ragged_rows():
    rng = np.random.default_rng(5)
    # values that the format holds come back as they are, whatever their group's scale
    e = rng.integers(-20, 20, (5, 9))
    c = rng.integers(0, 16, (5, 9, 32))
    c[:, :, 0] = 7                                       # (a six fixes the scale)
    x = (mx.e2m1_decode(c) * np.ldexp(1.0, e)[..., None]).reshape(5, -1)[:, : 8 * 32 + 20].astype(np.float32)
    q, s = mx.quant_mxfp4(x)
    assert q.shape == (5, 138) and s.shape == (5, 12)
    assert np.array_equal(mx.dequant_mxfp4(q, s, 276), x.astype(np.float64))
    assert np.array_equal(s[:, :9], (e + 127).astype(np.uint8)) and (s[:, 9:] == 127).all()
    assert np.array_equal(q[:, 0] & 15, c[:, 0, 0]) and np.array_equal(q[:, 0] >> 4, c[:, 0, 1])
    assert mx.words(s)[0, 0] == int.from_bytes(bytes(s[0, :4]), "little", signed=True)
    odd, so = mx.quant_mxfp4(x[:, :33])
    assert odd.shape == (5, 17) and (odd[:, 16] >> 4 == 0).all()


def test_error_is_at_most_half_a_step_and_bad_groups_are_nan():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((16, 256)).astype(np.float32)
    x[3, 40], x[4, 70], x[5, :32] = np.nan, -np.inf, 0
    q, s = mx.quant_mxfp4(x)
    v = mx.dequant_mxfp4(q, s)
    assert s[3, 1] == 255 and s[4, 2] == 255 and s[5, 0] == 127 and np.isnan(v[3, 32:64]).all() and (v[5, :32] == 0).all()
    assert (q[3, 16:32] == 0).all()
    fine = np.isfinite(v)
    scale = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, axis=1)
    y = np.abs(x / scale)
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    assert (np.abs(v - x)[fine] <= (step * scale / 2)[fine]).all()


def test_sort_orders_by_expert_then_token_then_slot():
    ids = np.array([[3, 1], [1, 1], [0, 9], [-1, 3], [2, 1]])
    off, rows = mx.moe_sort(ids, 3, 1)                   # experts 1, 2, 3
    assert off.tolist() == [0, 4, 5, 7]
    assert rows.tolist() == [[5, 0], [1, 2], [-1, -1], [-1, 6], [4, 3]]


def test_combine_gradients_against_differences():
    rng = np.random.default_rng(7)
    _, rows = mx.moe_sort(rng.integers(0, 6, (5, 3)), 4, 0)
    n = int(rows.max()) + 1
    y, w, d = rng.standard_normal((n, 7)), rng.random((5, 3)), rng.standard_normal((5, 7))
    dy, dw = mx.combine_bwd(d, y, rows, w)
    f = lambda: float((mx.combine(y, rows, w) * d).sum())  # noqa: E731
    for arr, grad in ((y, dy), (w, dw)):
        for at in np.ndindex(arr.shape):
            keep, h = arr[at], 1e-3
            arr[at] = keep + h
            up = f()
            arr[at] = keep - h
            down = f()
            arr[at] = keep
            # (the function is linear in each: differences are off by rounding alone)
            assert abs((up - down) / (2 * h) - grad[at]) < 1e-9
