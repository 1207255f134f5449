"""An expert layer's rows into expert order and back."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce

pytestmark = pytest.mark.gpu


def chosen(rng, tokens, k, experts, padded=0):
    ids = rng.integers(0, experts, (tokens, k)).astype(np.int32)     # (the same expert twice is allowed)
    ids[tokens - padded :] = -1
    return ids


def sort_by_keys(ids, groups, first):
    """The order in numpy's stable sort, for what the oracle takes too long for."""
    e = ids.reshape(-1).astype(np.int64) - first
    here = (e >= 0) & (e < groups)
    order = np.argsort(np.where(here, e, groups), kind="stable")[: here.sum()]
    rows = np.full(e.size, -1, np.int32)
    rows[order] = np.arange(order.size)
    return np.concatenate([[0], np.cumsum(np.bincount(e[here], minlength=groups))]).astype(np.int32), rows.reshape(ids.shape)


@pytest.mark.parametrize("tokens,k,experts,groups,first,padded", [
    (0, 4, 8, 8, 0, 0), (1, 1, 1, 1, 0, 0), (1, 8, 256, 256, 0, 0), (7, 3, 16, 4, 8, 2), (64, 64, 60, 60, 0, 0), (33, 6, 1023, 1023, 0, 3),
    (200, 8, 256, 32, 64, 10), (130, 8, 64, 64, 0, 130), (1000, 2, 5, 3, 1, 0), (300, 7, 40, 0, 0, 0), (2048, 8, 256, 256, 0, 100)])
def test_sort(ds3, tokens, k, experts, groups, first, padded):
    ids = chosen(np.random.default_rng(tokens + k), tokens, k, experts, padded)
    off, rows = ds3.ds3_moe_sort(torch.from_numpy(ids).to(DEV), groups, first_expert=first)
    woff, wrows = mx.moe_sort(ids, groups, first)
    assert off.cpu().numpy().tolist() == woff.tolist() and np.array_equal(rows.cpu().numpy(), wrows)


@pytest.mark.parametrize("n", [1023, 1024, 1025, 4095, 4097, 65535, 65536, 65537, 69632, 69633, 200_001, 1_000_000])
@pytest.mark.parametrize("k,experts,groups,first", [(1, 300, 300, 0), (1, 1100, 1023, 40), (8, 64, 8, 16)])
def test_sort_of_many_choices(ds3, n, k, experts, groups, first):
    rng = np.random.default_rng(n)
    ids = chosen(rng, -(-n // k), k, experts, padded=n // 50)
    ids.reshape(-1)[rng.integers(0, ids.size, 20)] = np.array([-5, 2**31 - 1, -(2**31), 1 << 20] * 5, np.int32)
    wide = torch.full((ids.shape[0], k + 3), 2, dtype=torch.int32, device=DEV)      # columns that are nobody's choices
    wide[:, :k] = torch.from_numpy(ids).to(DEV)
    for t in (torch.from_numpy(ids).to(DEV), wide[:, :k]):
        off, rows = ds3.ds3_moe_sort(t, groups, first_expert=first)
        woff, wrows = sort_by_keys(ids, groups, first)
        assert np.array_equal(off.cpu().numpy(), woff) and np.array_equal(rows.cpu().numpy(), wrows)


def test_sort_of_the_last_numbers_and_at_the_longest_single_launch(ds3):
    """Experts up to 2^31 - 1: the lowest numbers are not theirs.  A packed list, its copy that begins on another border, and
    one choice more."""
    first = 2**31 - 7
    for n in (40, 9000, 131072, 131073):
        ids = np.random.default_rng(n).choice(np.array([first - 1, first, first + 3, 2**31 - 1, -(2**31), -(2**31) + 2, -1, 0], np.int64), (n, 1)).astype(np.int32)
        off_border = torch.zeros(n + 1, dtype=torch.int32, device=DEV)[1:].view(n, 1)
        off_border.copy_(torch.from_numpy(ids))
        for t in (torch.from_numpy(ids).to(DEV), off_border):
            off, rows = ds3.ds3_moe_sort(t, 7, first_expert=first)
            woff, wrows = sort_by_keys(ids, 7, first)
            assert np.array_equal(off.cpu().numpy(), woff) and np.array_equal(rows.cpu().numpy(), wrows)
    with pytest.raises(RuntimeError):
        ds3.ds3_moe_sort(t, 8, first_expert=first)


CASES = [(1, 1, 8, 8, 0), (1, 8, 16, 128, 0), (5, 2, 4, 40, 1), (17, 3, 8, 136, 0), (40, 6, 60, 2048, 4), (33, 8, 32, 2056, 0), (9, 64, 7, 264, 0),
         (6, 4, 8, 8200, 0), (70, 5, 64, 1000, 10)]


def layout(ds3, tokens, k, experts, padded, seed, spare=5):
    rng = np.random.default_rng(seed)
    ids = chosen(rng, tokens, k, experts, padded)
    groups = max(1, experts * 3 // 4)
    _, rows = ds3.ds3_moe_sort(torch.from_numpy(ids).to(DEV), groups)
    return rng, rows, rows.cpu().numpy(), int(rows.max()) + 1 + spare


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,k,experts,cols,padded", CASES)
def test_dispatch(ds3, tokens, k, experts, cols, padded, dtype):
    announce(f"dispatch {tokens}x{k} of {experts}, {cols} columns, {dtype}")
    rng, rows, hrows, total = layout(ds3, tokens, k, experts, padded, tokens + cols)
    wide = torch.full((tokens, cols + 16), float("nan"), dtype=dtype, device=DEV)
    wide[:, :cols] = torch.from_numpy(rng.standard_normal((tokens, cols)).astype(np.float32)).to(DEV).to(dtype)
    x = wide[:, :cols]
    for limit in (total, max(1, total // 2)):                        # (rows beyond the output are dropped)
        named = (hrows >= 0) & (hrows < limit)
        src = np.full(limit, -1)
        src[hrows[named]] = np.nonzero(named)[0]
        at = torch.from_numpy(src).to(DEV)
        out = torch.full((limit, cols + 16), 7.0, dtype=dtype, device=DEV)
        y = ds3.ds3_moe_dispatch(x, rows, out=out[:, :cols])
        want = torch.where((at >= 0)[:, None], x[at.clamp(min=0)], torch.full_like(y, 7.0))
        assert torch.equal(y, want) and (out[:, cols:] == 7).all()
        for name in ("1x128", "1x128_pow2", "mxfp4"):
            quant = {"1x128": ds3.ds3_quant_act_1x128, "1x128_pow2": ds3.ds3_quant_act_1x128_pow2, "mxfp4": ds3.ds3_quant_mxfp4}[name]
            q0, s0 = quant(x)
            for k_major in (True, False):
                lead = -(-q0.shape[1] // 16) * 16 + 16
                q = torch.full((limit, lead), 0x3C, dtype=torch.uint8, device=DEV)
                kb = s0.shape[1]
                s = torch.full((kb, limit) if k_major else (limit, kb), 9, dtype=s0.dtype, device=DEV)
                s = s.t() if k_major else s
                got = getattr(ds3, "ds3_moe_dispatch_quant_" + name)(x, rows, out=(q[:, : q0.shape[1]], s))
                assert torch.equal(got[0], torch.where((at >= 0)[:, None], q0[at.clamp(min=0)], 0x3C)), name
                assert torch.equal(got[1], torch.where((at >= 0)[:, None], s0[at.clamp(min=0)], 9)), name
                assert (q[:, q0.shape[1] :] == 0x3C).all()
    # outputs made by the call
    y = ds3.ds3_moe_dispatch(x, rows)
    assert y.shape == (tokens * k, cols)
    q, s = ds3.ds3_moe_dispatch_quant_mxfp4(x, rows, rows=total)
    assert q.shape == (total, cols // 2) and s.shape == (total, -(-cols // 128))


def test_dispatch_of_fp32_rows_that_end_after_four(ds3):
    rows = torch.tensor([[2, 0], [-1, 1]], dtype=torch.int32, device=DEV)
    x = torch.randn((2, 132), device=DEV)
    y = ds3.ds3_moe_dispatch(x, rows, rows=3)
    assert torch.equal(y, x[torch.tensor([0, 1, 0], device=DEV)])
    for call, quant in ((ds3.ds3_moe_dispatch_quant_1x128, ds3.ds3_quant_act_1x128), (ds3.ds3_moe_dispatch_quant_mxfp4, ds3.ds3_quant_mxfp4)):
        q, s = call(x, rows, rows=3)
        q0, s0 = quant(x)
        assert torch.equal(q, q0[torch.tensor([0, 1, 0], device=DEV)]) and torch.equal(s, s0[torch.tensor([0, 1, 0], device=DEV)])


EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}          # half a step, relative


@pytest.mark.parametrize("yt,ot", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16),
                                   (torch.float32, torch.float32)])
@pytest.mark.parametrize("tokens,k,experts,cols,padded", CASES)
def test_combine_and_its_gradients(ds3, tokens, k, experts, cols, padded, yt, ot):
    """An FP32 sum of n terms, each addition and product rounded once, is within n * 2^-24 of the sum of the magnitudes (a
    little more: the factor 1.01 covers the products of such terms); then the output's rounding."""
    announce(f"combine {tokens}x{k} of {experts}, {cols} columns, {yt} -> {ot}")
    rng, rows, hrows, total = layout(ds3, tokens, k, experts, padded, tokens * 3 + cols)
    y = torch.full((total, cols + 16), float("nan"), dtype=yt, device=DEV)
    y[:, :cols] = torch.from_numpy(rng.standard_normal((total, cols)).astype(np.float32)).to(DEV).to(yt)
    nobody = np.setdiff1d(np.arange(total), hrows)
    y[torch.from_numpy(nobody).to(DEV)] = float("nan")               # nothing may come from rows that nobody names
    y = y[:, :cols]
    w = rng.random((tokens, k)).astype(np.float32) - 0.3
    dout = torch.from_numpy(rng.standard_normal((tokens, cols)).astype(np.float32)).to(DEV).to(ot)
    hy = np.nan_to_num(y.double().cpu().numpy())
    hd = dout.double().cpu().numpy()
    for limit in (total, max(1, total // 2)):
        for weights in (w, None):
            wd = None if weights is None else torch.from_numpy(weights).to(DEV)
            got = ds3.ds3_moe_combine(y[:limit], rows, wd, out_dtype=ot)
            assert got.dtype == ot and got.shape == (tokens, cols)
            want = mx.combine(hy[:limit], hrows, weights)
            near = 1.01 * k * 2.0 ** -24 * mx.combine(np.abs(hy[:limit]), hrows, None if weights is None else np.abs(weights))
            assert (np.abs(got.double().cpu().numpy() - want) <= near + EPS[ot] * (np.abs(want) + near)).all()
            dyd = torch.full((limit, cols + 16), 11.0, dtype=yt, device=DEV)
            dy, dw = ds3.ds3_moe_combine_bwd(dout, y[:limit], rows, wd, dy=dyd[:, :cols])
            wdy, wdw = mx.combine_bwd(hd, hy[:limit], hrows, weights)
            kept = np.isnan(wdy)
            hdy = dy.double().cpu().numpy()
            assert (hdy[kept] == 11).all() and (dyd[:, cols:] == 11).all()
            # one FP32 product, then y's type
            assert (np.abs(hdy - wdy)[~kept] <= 1.01 * (2.0 ** -24 + EPS[yt]) * np.abs(wdy)[~kept] + 2.0 ** -133).all()
            # a lane's columns one after the other, eight of every 512, then 6 steps over the lanes
            terms = 8 * -(-cols // 512) + 6
            _, mag = mx.combine_bwd(np.abs(hd), np.abs(hy[:limit]), hrows)
            assert dw.dtype == torch.float32 and (np.abs(dw.double().cpu().numpy() - wdw) <= 1.01 * terms * 2.0 ** -24 * mag).all()
            assert (dw.cpu().numpy()[(hrows < 0) | (hrows >= limit)] == 0).all()


def test_gradients_against_differences(ds3):
    """Both gradients of sum(dout * combine(y, w)) against the function itself, which is linear in each: the difference of
    two FP32 outputs of magnitude c is off by two roundings, 2 * 2^-24 * c each column."""
    rng, rows, hrows, total = layout(ds3, 6, 3, 6, 1, 5, spare=0)
    cols = 64
    y, w = torch.randn((total, cols), device=DEV), torch.rand((6, 3), device=DEV)
    dout = torch.randn((6, cols), device=DEV)
    dy, dw = ds3.ds3_moe_combine_bwd(dout, y, rows, w)
    base = ds3.ds3_moe_combine(y, rows, w).double()
    slack = 8 * 2.0 ** -24 * float(((base.abs() + 16) * dout.double().abs()).sum())
    for t, j in zip(*np.nonzero(hrows >= 0)):
        other = w.clone()
        other[t, j] += 1.0
        diff = float(((ds3.ds3_moe_combine(y, rows, other).double() - base) * dout.double()).sum())
        assert abs(diff - float(dw[t, j])) <= slack
        moved = y.clone()
        moved[hrows[t, j], 7] += 1.0
        diff = float(((ds3.ds3_moe_combine(moved, rows, w).double() - base) * dout.double()).sum())
        assert abs(diff - float(dy[hrows[t, j], 7])) <= slack


def test_combine_without_columns_or_rows(ds3):
    """Sums over nothing are zeros, in what the gradients write too."""
    rng, rows, hrows, total = layout(ds3, 9, 3, 6, 1, 5, spare=0)
    for cols, held in ((0, total), (64, 0)):
        y, d = torch.ones((held, cols), device=DEV), torch.ones((9, cols), device=DEV)
        dw = torch.full((9, 3), 5.0, device=DEV)               # (so that what the call allocates next holds no zeros yet)
        del dw
        dy, dw = ds3.ds3_moe_combine_bwd(d, y, rows, torch.rand((9, 3), device=DEV))
        assert dy.shape == y.shape and torch.equal(dw, torch.zeros((9, 3), device=DEV))
        out = ds3.ds3_moe_combine(y, rows, torch.rand((9, 3), device=DEV))
        assert out.shape == (9, cols) and (out == 0).all()


def test_combine_without_weights_is_the_gradient_of_dispatch(ds3):
    rng, rows, hrows, total = layout(ds3, 50, 4, 12, 3, 8, spare=0)
    x, g = torch.randn((50, 72), device=DEV), torch.randn((total, 72), device=DEV)
    y = ds3.ds3_moe_dispatch(x, rows, rows=total)
    dx = ds3.ds3_moe_combine(g, rows)
    left, right = float((y.double() * g.double()).sum()), float((x.double() * dx.double()).sum())
    # <dispatch(x), g> = <x, dx>: dx has four FP32 additions an element
    assert abs(left - right) <= 4 * 2.0 ** -24 * float((y.double() * g.double()).abs().sum())


def test_rows_past_32_bits(ds3):
    """Rows and tokens whose bytes lie beyond 2^32."""
    tokens, cols = 300_000, 7168
    x = torch.empty((tokens, cols), dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(4))
    rows = torch.arange(tokens - 1, -1, -1, dtype=torch.int32, device=DEV)[:, None].contiguous()
    at = torch.tensor([0, 1, 150_000, 299_998, 299_999], device=DEV)
    y = ds3.ds3_moe_dispatch(x, rows)
    assert torch.equal(y[at], x[tokens - 1 - at])
    back = ds3.ds3_moe_combine(y, rows)
    assert torch.equal(back[at], x[at])
    dy, dw = ds3.ds3_moe_combine_bwd(x, y, rows, dy=back)
    assert torch.equal(dy[at], x[tokens - 1 - at])
    want = x[at].double().square().sum(1)
    assert ((dw[at, 0].double() - want).abs() <= (8 * 14 + 6) * 2.0 ** -24 * want).all()     # (7168 = 14 * 512 columns)
    q, s = ds3.ds3_moe_dispatch_quant_1x128(x, rows)
    q0, s0 = ds3.ds3_quant_act_1x128(x[at])
    assert torch.equal(q[tokens - 1 - at], q0) and torch.equal(s[tokens - 1 - at], s0)
