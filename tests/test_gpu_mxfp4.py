"""MXFP4 quantizers and dequantizer against the oracle, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce

pytestmark = pytest.mark.gpu


def bytes_of(s):
    """Scale words, logical [rows][kb], as bytes [rows][4 * kb]."""
    return np.ascontiguousarray(s.cpu().contiguous().numpy()).view(np.uint8)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().float().numpy()


def sample(rows, cols, seed, hard=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)).astype(np.float32) * np.float32(2.0) ** rng.integers(-12, 12, (rows, 1)).astype(np.float32)
    if hard:
        for i in range(rows * cols // 97 + 1):           # zeros, signs of zero, far magnitudes, values that no group may hold
            r, c = rng.integers(rows), rng.integers(cols)
            v = [0.0, -0.0, 2.0 ** -149, -(2.0 ** -130), 2.0 ** -126, 3.3e38, -1e30, np.inf, -np.inf, np.nan, 6.0, 0.25, 5.0][rng.integers(13)]
            x[r, c] = v
        x[rng.integers(rows), : min(cols, 64)] = 0
    return x


def check_quant(ds3, x, t, k_major=True):
    q, s = ds3.ds3_quant_mxfp4(t, k_major)
    wq, ws = mx.quant_mxfp4(x)
    assert q.shape == wq.shape and s.shape == (x.shape[0], -(-x.shape[1] // 128))
    assert np.array_equal(bytes_of(s), ws)
    assert np.array_equal(q.cpu().numpy(), wq)
    qt, st = ds3.ds3_quant_mxfp4_t(t, k_major)
    wq, ws = mx.quant_mxfp4(np.ascontiguousarray(x.T))
    assert np.array_equal(bytes_of(st), ws)
    assert np.array_equal(qt.cpu().numpy(), wq)
    return (q, s), (qt, st)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 128), (2, 32), (3, 40), (17, 136), (31, 1000), (33, 2056), (255, 72), (257, 64), (513, 200), (1030, 24)])
def test_codes_and_scales_equal_the_oracle(ds3, rows, cols, dtype):
    announce(f"mxfp4 {rows}x{cols} {dtype}")
    for seed in range(2):
        x = sample(rows, cols, 100 * rows + cols + seed)
        if dtype == torch.bfloat16:
            x = bf16(x)
        check_quant(ds3, x, torch.from_numpy(x).to(DEV).to(dtype), k_major=seed == 0)


def test_fp32_rows_that_end_after_four(ds3):
    for rows, cols in ((5, 4), (3, 132), (40, 36)):
        x = sample(rows, cols, cols)
        check_quant(ds3, x, torch.from_numpy(x).to(DEV))


def test_every_border_of_the_rounding(ds3):
    """Every value of the grid, every midpoint and the floats around them, both signs, in groups whose scale is 1 and others."""
    g = mx.E2M1.astype(np.float32)
    at = np.concatenate([g, (g[1:] + g[:-1]) / 2]).astype(np.float32)
    near = [at]
    for towards in (np.float32(0), np.float32(100)):
        v = at
        for _ in range(3):
            v = np.nextafter(v, towards)
            near.append(v)
    v = np.unique(np.concatenate(near))
    v = np.concatenate([v, -v])
    v = v[np.abs(v) <= 6]
    groups = -(-v.size // 31)
    x = np.zeros((groups, 32), np.float32)
    x[:, 0] = 6
    x[:, 1:].reshape(-1)[: v.size] = v
    for e in (0, -100, 100, -126, 125):
        check_quant(ds3, np.ldexp(x, e).astype(np.float32), torch.from_numpy(np.ldexp(x, e).astype(np.float32)).to(DEV))


def test_strides_guards_and_other_streams(ds3):
    rows, cols = 70, 264
    x = bf16(sample(rows, cols, 9))
    wide = torch.full((rows, cols + 24), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :cols] = torch.from_numpy(x).to(DEV)
    t = wide[:, :cols]
    L, st = ds3._L(), torch.cuda.current_stream().cuda_stream
    for transposed in (False, True):
        n, k = (cols, rows) if transposed else (rows, cols)
        ldq, kw = 176, -(-k // 128)
        q = torch.full((n + 2, ldq), 0xA5, dtype=torch.uint8, device=DEV)
        s = torch.full((n + 2, kw + 1), 0x5A5A5A5A, dtype=torch.int32, device=DEV)
        f = L.ds3_quant_mxfp4_t if transposed else L.ds3_quant_mxfp4
        assert f(t.data_ptr(), 1, rows, cols, t.stride(0), q[1].data_ptr(), ldq, s[1].data_ptr(), kw + 1, 1, st) == 0
        wq, ws = mx.quant_mxfp4(np.ascontiguousarray(x.T) if transposed else x)
        w = wq.shape[1]
        assert np.array_equal(q[1:-1, :w].cpu().numpy(), wq) and np.array_equal(bytes_of(s[1:-1, :kw]), ws)
        assert (q[1:-1, w:] == 0xA5).all() and (q[0] == 0xA5).all() and (q[-1] == 0xA5).all()
        assert (s[1:-1, kw] == 0x5A5A5A5A).all() and (s[0] == 0x5A5A5A5A).all() and (s[-1] == 0x5A5A5A5A).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check_quant(ds3, x, t)
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2), (3, 33), (17, 127), (20, 128), (5, 250), (34, 1025)])
def test_dequantizer_is_exact(ds3, rows, cols):
    rng = np.random.default_rng(rows + cols)
    w, kw = (cols + 1) // 2, -(-cols // 128)
    q = rng.integers(0, 256, (rows, w)).astype(np.uint8)
    s = rng.integers(0, 252, (rows, 4 * kw)).astype(np.uint8)     # (6 * 2^124 is BF16's last step but one)
    s[rng.random(s.shape) < 0.05] = 255
    s[rng.random(s.shape) < 0.05] = 0
    lead = (w + 15) // 16 * 16
    qd = torch.full((rows, lead), 0x77, dtype=torch.uint8, device=DEV)
    qd[:, :w] = torch.from_numpy(q).to(DEV)
    sd = torch.from_numpy(mx.words(s).copy()).to(DEV)
    for words in (sd, sd.t().contiguous().t()):
        y = ds3.ds3_dequant_mxfp4(qd[:, :w], words, cols=cols)
        assert y.shape == (rows, cols) and y.dtype == torch.bfloat16
        want = mx.dequant_mxfp4(q, s, cols)
        got = y.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


def test_round_trip_of_large_tensors_on_sampled_rows(ds3):
    """Past 2^32 bytes of input: the last rows and columns are what they should be."""
    rows, cols = 300_000, 7168                                       # 4.3 GB of BF16
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(3))
    q, s = ds3.ds3_quant_mxfp4(x)
    at = torch.tensor([0, 1, 149_999, 299_990, 299_999], device=DEV)
    wq, ws = mx.quant_mxfp4(x[at].float().cpu().numpy())
    assert np.array_equal(q[at].cpu().numpy(), wq) and np.array_equal(bytes_of(s[at]), ws)
    qt, st = ds3.ds3_quant_mxfp4_t(x)
    cols_at = torch.tensor([0, 63, 64, 7167], device=DEV)
    wq, ws = mx.quant_mxfp4(x[rows - 352 :, cols_at].float().cpu().numpy().T)   # (299648 = 2341 * 128)
    assert np.array_equal(qt[cols_at, (rows - 352) // 2 :].cpu().numpy(), wq)
    assert np.array_equal(bytes_of(st[cols_at, (rows - 352) // 128 :]), ws)
