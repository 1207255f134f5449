"""MXFP4 products, dense and grouped, against 64 bits.

Tolerance: every matrix instruction adds four groups' products to the FP32 sum; each of its additions is taken to be off
by at most one unit in the last place of what the sum's terms can reach, so an output is within (K / 128 + 4) * 2^-23 of
the sum of the products' magnitudes, and a BF16 output by another half step, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce

pytestmark = pytest.mark.gpu


def operand(rng, rows, k, spread=12, lead=0):
    """Random codes and scales: (oracle's values, codes on the device with garbage behind each row, scale bytes)."""
    q = rng.integers(0, 256, (rows, k // 2)).astype(np.uint8)
    s = rng.integers(127 - spread // 2, 128 + spread // 2, (rows, k // 32)).astype(np.uint8)
    wide = torch.full((rows + 1, (k // 2 + 15) // 16 * 16 + 16 * lead), 0x77, dtype=torch.uint8, device=DEV)
    wide[:rows, : k // 2] = torch.from_numpy(q).to(DEV)
    return mx.dequant_mxfp4(q, s), wide[:rows, : k // 2], s


def words(s, k_major=True):
    w = torch.from_numpy(mx.words(s).copy()).to(DEV)
    return w.t().contiguous().t() if k_major else w


def allowed(a, b, want, k, bf16):
    t = (k / 128 + 4) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    return t + 2.0 ** -8 * (np.abs(want) + t) if bf16 else t


SHAPES = [(1, 1, 128), (1, 16, 256), (3, 5, 384), (16, 64, 512), (17, 33, 128), (32, 100, 1152), (33, 128, 256), (64, 200, 640), (65, 129, 384),
          (127, 257, 512), (128, 128, 7168), (129, 300, 2048), (200, 72, 896), (256, 256, 256), (257, 513, 1280), (300, 1000, 512), (1, 4096, 1536),
          (40, 2304, 2048), (600, 640, 128), (1025, 384, 384)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_dense(ds3, M, N, K):
    announce(f"mxfp4 gemm {M}x{N}x{K}")
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    a, qa, sa = operand(rng, M, K)
    b, qb, sb = operand(rng, N, K, lead=2)
    want = a @ b.T
    for k_major in (True, False):
        y = ds3.ds3_gemm_mxfp4(qa, words(sa, k_major), qb, words(sb, k_major), out_dtype=torch.float32)
        assert (np.abs(y.double().cpu().numpy() - want) <= allowed(a, b, want, K, False)).all()
    y = ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb))
    assert y.dtype == torch.bfloat16
    assert (np.abs(y.double().cpu().numpy() - want) <= allowed(a, b, want, K, True)).all()
    # accumulated into a wider output whose other columns stay
    c = torch.full((M, (N + 3) // 4 * 4 + 8), 3.0, device=DEV)
    ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), c=c[:, :N], accumulate=True)
    got = c[:, :N].double().cpu().numpy() - 3.0
    assert (np.abs(got - want) <= allowed(a, b, want, K, False) + 2.0 ** -23 * (np.abs(want) + 3)).all()
    assert (c[:, N:] == 3.0).all()


def compute_units():
    return torch.cuda.get_device_properties(0).multi_processor_count


# a shape (or several) for every tile configuration of the dense call, with ragged edges and K-steps that end in a half
DENSE = {0: [(20, 1500, 2688)], 1: [(30, 12000, 1408), (120, 4001, 2176)], 2: [(16, 18431, 7168), (3529, 67, 640)],
         3: [(9, 24001, 2176), (300, 2100, 1920)], 4: [(450, 2001, 896), (4451, 33, 384)], 5: [(333, 4001, 640)],
         6: [(65, 16794, 384), (2048, 2304, 896)], 7: [(5000, 9216, 384), (265, 21812, 384)]}


@pytest.mark.parametrize("config", sorted(DENSE))
def test_every_dense_configuration(ds3, config):
    for M, N, K in DENSE[config]:
        announce(f"mxfp4 gemm {M}x{N}x{K}, configuration {config}")
        assert compute_units() != 256 or ds3._L().ds3_gemm_mxfp4_config(0, M, N, K, 256) == config
        rng = np.random.default_rng(config)
        a, qa, sa = operand(rng, M, K, lead=1)
        b, qb, sb = operand(rng, N, K, lead=2)
        da, db = torch.from_numpy(a).to(DEV), torch.from_numpy(b).to(DEV)      # (the products in 64 bits on the device: large)
        want, mag = da @ db.t(), da.abs() @ db.abs().t()
        near = (K / 128 + 4) * 2.0 ** -23 * mag
        y = ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), out_dtype=torch.float32)
        assert bool(((y.double() - want).abs() <= near).all())
        y = ds3.ds3_gemm_mxfp4(qa, words(sa, False), qb, words(sb))
        assert bool(((y.double() - want).abs() <= near + 2.0 ** -8 * (want.abs() + near)).all())
        c = torch.full((M, (N + 3) // 4 * 4 + 4), -2.0, device=DEV)
        ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), c=c[:, :N], accumulate=True)
        assert bool(((c[:, :N].double() + 2 - want).abs() <= near + 2.0 ** -23 * (want.abs() + 2)).all()) and bool((c[:, N:] == -2).all())


# experts' rows (with some empty, some uneven), N, K for every configuration of the grouped call
GROUPED = {8: ((3, 0, 40, 1, 17, 0, 2, 8), 300, 896), 9: ((40, 0, 33, 60, 31, 47, 1, 100), 260, 640), 10: ((70, 0, 55, 130, 64, 60, 80, 50), 264, 2688),
           11: ((120, 90, 0, 200, 64, 65, 129, 300), 2056, 384), 12: ((60, 0, 129, 90, 64, 257, 31, 1) * 4, 4104, 384),
           13: ((250, 100, 0, 300, 257, 129, 1, 256) * 4, 4104, 384)}


@pytest.mark.parametrize("config", sorted(GROUPED))
def test_every_grouped_configuration(ds3, config):
    sizes, N, K = GROUPED[config]
    G, rows = len(sizes), sum(sizes) + 5
    announce(f"mxfp4 grouped {G} experts, {rows} rows, {N}x{K}, configuration {config}")
    assert compute_units() != 256 or ds3._L().ds3_gemm_mxfp4_config(G, rows, N, K, 256) == config
    rng = np.random.default_rng(config)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    a, qa, sa = operand(rng, rows, K, lead=1)
    b, qb, sb = operand(rng, G * N, K)
    w = words(sb, False).view(G, N, K // 128).transpose(1, 2).contiguous().transpose(1, 2)
    qb = qb.contiguous().view(G, N, K // 2)
    offd = torch.from_numpy(off).to(DEV)
    for dtype in (torch.float32, torch.bfloat16):
        c = torch.full((rows, (N + 7) // 8 * 8), 5.0, dtype=dtype, device=DEV)
        y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), offd, qb, w, c=c[:, :N])
        assert bool((c[:, N:] == 5).all()) and bool((y[off[-1] :] == 5).all())
        for g in range(G):
            at = slice(int(off[g]), int(off[g + 1]))
            da, db = torch.from_numpy(a[at]).to(DEV), torch.from_numpy(b[g * N : (g + 1) * N]).to(DEV)
            want = da @ db.t()
            near = (K / 128 + 4) * 2.0 ** -23 * (da.abs() @ db.abs().t())
            tol = near + 2.0 ** -8 * (want.abs() + near) if dtype == torch.bfloat16 else near
            assert bool(((y[at].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M,N,K", [(5, 40, 256), (48, 96, 384), (130, 260, 1024), (512, 512, 896)])
def test_equal_scales_are_exact(ds3, M, N, K):
    """With one scale everything is a multiple of 1/4 below 2^22: FP32 sums in any order are exact."""
    rng = np.random.default_rng(K)
    a, qa, sa = operand(rng, M, K, spread=0)
    b, qb, sb = operand(rng, N, K, spread=0)
    y = ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), out_dtype=torch.float32)
    assert np.array_equal(y.double().cpu().numpy(), a @ b.T)


@pytest.mark.parametrize("M,N,K", [(19, 44, 640), (300, 716, 384), (530, 2300, 896)])
def test_output_rows_that_begin_on_eight_bytes(ds3, M, N, K):
    """A leading dimension of four elements more than a multiple of eight: BF16 rows are not 16-byte aligned."""
    rng = np.random.default_rng(N)
    a, qa, sa = operand(rng, M, K)
    b, qb, sb = operand(rng, N, K)
    want = a @ b.T
    ld = N // 8 * 8 + 12
    c = torch.full((M, ld), 1.5, dtype=torch.bfloat16, device=DEV)
    ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), c=c[:, :N])
    assert (np.abs(c[:, :N].double().cpu().numpy() - want) <= allowed(a, b, want, K, True)).all() and (c[:, N:] == 1.5).all()
    off = torch.tensor([0, M // 3, M], dtype=torch.int32, device=DEV)
    c.fill_(1.5)
    ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), off, qb.contiguous().view(1, N, K // 2).repeat(2, 1, 1), words(sb, False)[None].repeat(2, 1, 1), c=c[:, :N])
    assert (np.abs(c[:, :N].double().cpu().numpy() - want) <= allowed(a, b, want, K, True)).all() and (c[:, N:] == 1.5).all()


@pytest.mark.parametrize("M,N,K", [(20, 48, 384), (300, 264, 1152)])
def test_nan_scales_stay_in_their_rows_and_columns(ds3, M, N, K):
    rng = np.random.default_rng(1)
    a, qa, sa = operand(rng, M, K)
    b, qb, sb = operand(rng, N, K)
    sa[3, 1] = 255
    sb[7, K // 32 - 1] = 255
    y = ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), out_dtype=torch.float32).cpu().numpy()
    nan = np.zeros((M, N), bool)
    nan[3], nan[:, 7] = True, True
    assert np.array_equal(np.isnan(y), nan)


def test_empty_sums_and_extreme_scales(ds3):
    c = torch.full((6, 8), 2.0, device=DEV)
    e, se = torch.empty((6, 0), dtype=torch.uint8, device=DEV), torch.empty((6, 0), dtype=torch.int32, device=DEV)
    e8, se8 = torch.empty((8, 0), dtype=torch.uint8, device=DEV), torch.empty((8, 0), dtype=torch.int32, device=DEV)
    assert (ds3.ds3_gemm_mxfp4(e, se, e8, se8, c=c, accumulate=True) == 2).all()
    assert (ds3.ds3_gemm_mxfp4(e, se, e8, se8, c=c) == 0).all()
    # 2^-127 and 2^127 are scales like others; their product leaves FP32's range on neither side
    q = torch.full((16, 128), 0x22, dtype=torch.uint8, device=DEV)               # ones
    lo, hi = torch.zeros((16, 2), dtype=torch.int32, device=DEV), torch.full((16, 2), -0x01010102, dtype=torch.int32, device=DEV)
    y = ds3.ds3_gemm_mxfp4(q, lo, q, hi, out_dtype=torch.float32)
    assert (y == 256.0).all()


@pytest.mark.parametrize("M,N", [(3, 40), (40, 700), (300, 400), (1100, 2100)])
@pytest.mark.parametrize("K", [128, 384, 1024, 1664])
def test_zeros_under_the_largest_scales(ds3, M, N, K):
    """0 * 2^127 * 2^127 is 0, in a half K-step's empty half too; a one among them is 2^254, an infinity."""
    qa, qb = torch.zeros((M, K // 2), dtype=torch.uint8, device=DEV), torch.full((N, K // 2), 0x22, dtype=torch.uint8, device=DEV)
    sa, sb = (torch.full((n, K // 128), -0x01010102, dtype=torch.int32, device=DEV) for n in (M, N))
    assert (ds3.ds3_gemm_mxfp4(qa, sa, qb, sb, out_dtype=torch.float32) == 0).all()
    qa[M // 2, K // 2 - 1] = 0x20
    y = ds3.ds3_gemm_mxfp4(qa, sa, qb, sb, out_dtype=torch.float32)
    assert (y[M // 2] == float("inf")).all() and (y == 0).sum() == (M - 1) * N


@pytest.mark.parametrize("sizes", [(2, 0, 9), (30, 50, 41), (150, 100, 0, 130), (256, 700)])
def test_groups_that_begin_behind_the_first_row(ds3, sizes):
    rng = np.random.default_rng(sum(sizes))
    G, N, K, rows = len(sizes), 1032, 640, sum(sizes) + 20
    off = (7 + np.concatenate([[0], np.cumsum(sizes)])).astype(np.int32)
    a, qa, sa = operand(rng, rows, K)
    b, qb, sb = operand(rng, G * N, K)
    c = torch.full((rows, N), 5.0, device=DEV)
    y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), torch.from_numpy(off).to(DEV), qb.contiguous().view(G, N, K // 2), words(sb, False).view(G, N, K // 128),
                                   c=c).double().cpu().numpy()
    assert (y[:7] == 5).all() and (y[off[-1]:] == 5).all()
    for g in range(G):
        at, bg = slice(off[g], off[g + 1]), b[g * N : (g + 1) * N]
        want = a[at] @ bg.T
        assert (np.abs(y[at] - want) <= allowed(a[at], bg, want, K, False)).all()


@pytest.mark.parametrize("M,N,K", [(5, 96, 512), (200, 640, 384), (1200, 2304, 640)])
def test_captured(ds3, M, N, K):
    """Quantizers, products (one adding to what is there) and the way back in a graph, replayed on other values between eager work."""
    gen = torch.Generator(device=DEV).manual_seed(N)
    make = lambda *s: torch.randn(s, generator=gen, device=DEV)
    x, w, c = make(M, K).bfloat16(), make(K, N), make(M, N)

    def step(c):
        q, s = ds3.ds3_quant_mxfp4(x)
        qw, sw = ds3.ds3_quant_mxfp4_t(w)
        return ds3.ds3_gemm_mxfp4(q, s, qw, sw), ds3.ds3_gemm_mxfp4(q, s, qw, sw, c=c, accumulate=True), ds3.ds3_dequant_mxfp4(q, s), qw, sw

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c.clone())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step(c)
    for i in range(4):
        x.copy_(make(M, K))
        w.copy_(make(K, N) * 2.0 ** i)
        c.copy_(make(M, N))
        want = step(c.clone())
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, v) for o, v in zip(outs, want))
        make(64, 64).sum().item()


@pytest.mark.parametrize("sizes,N,K", [((0, 5, 0, 1, 40, 0), 200, 384), ((130, 0, 257, 3), 264, 512), ((1,) * 70 + (0,) * 3 + (20,), 64, 256),
                                       ((0, 0, 0), 32, 128), ((33, 90, 64, 300, 12), 1024, 1152), ((700, 1, 500), 384, 256)])
def test_grouped(ds3, sizes, N, K):
    announce(f"mxfp4 grouped {len(sizes)} experts, {sum(sizes)} rows, {N}x{K}")
    rng = np.random.default_rng(N + K)
    G, rows = len(sizes), sum(sizes) + 9                              # nine rows belong to nobody
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    a, qa, sa = operand(rng, rows, K, lead=1)
    b, qb, sb = operand(rng, G * N, K)
    kw = K // 128
    wb = words(sb, False).view(G, N, kw)
    forms = [wb, wb.transpose(1, 2).contiguous().transpose(1, 2)]
    qb = qb.contiguous().view(G, N, K // 2)
    want = np.full((rows, N), 5.0)
    tol = np.zeros((rows, N))
    tol16 = np.zeros((rows, N))
    for g in range(G):
        at = slice(off[g], off[g + 1])
        bg = b[g * N : (g + 1) * N]
        want[at] = a[at] @ bg.T
        tol[at] = allowed(a[at], bg, want[at], K, False)
        tol16[at] = allowed(a[at], bg, want[at], K, True)
    offd = torch.from_numpy(off).to(DEV)
    for form in forms:
        c = torch.full((rows, (N + 7) // 8 * 8), 5.0, device=DEV)
        y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), offd, qb, form, c=c[:, :N])
        assert (np.abs(y.double().cpu().numpy() - want) <= tol).all() and (c[:, N:] == 5.0).all()
    c = torch.full((rows, (N + 7) // 8 * 8), 5.0, dtype=torch.bfloat16, device=DEV)[:, :N]
    y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa, False), offd, qb, forms[1], c=c)
    assert (np.abs(y.double().cpu().numpy() - want) <= tol16).all()


def test_most_experts_and_one_row_each(ds3):
    G, N, K = 1023, 40, 128
    rng = np.random.default_rng(2)
    sizes = (rng.random(G) < 0.5).astype(int)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    a, qa, sa = operand(rng, int(off[-1]), K)
    b, qb, sb = operand(rng, G * N, K)
    y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), torch.from_numpy(off).to(DEV), qb.contiguous().view(G, N, K // 2),
                                   words(sb, False).view(G, N, 1), out_dtype=torch.float32).double().cpu().numpy()
    for g in np.nonzero(sizes)[0]:
        bg = b[g * N : (g + 1) * N]
        want = a[off[g] : off[g] + 1] @ bg.T
        assert (np.abs(y[off[g]] - want) <= allowed(a[off[g] : off[g] + 1], bg, want, K, False)).all()


def test_offsets_past_32_bits(ds3):
    """An output of more than 2^32 bytes and an operand of more than 2^31: the last rows and columns."""
    M, N, K = 80_000, 16_384, 256
    rng = np.random.default_rng(3)
    b, qb, sb = operand(rng, N, K)
    ra, rq, rs = operand(rng, 16, K)
    qa = torch.zeros((M, 28_672), dtype=torch.uint8, device=DEV)[:, : K // 2]    # 2.3 GB between the first row and the last
    sa = torch.full((2, M), 0x7F7F7F7F, dtype=torch.int32, device=DEV).t()
    at = torch.tensor([0, 1, 255, 256, 37_449, 37_450, 65_535, 65_536, 74_898, 74_899, 79_990, 79_991, 79_996, 79_997, 79_998, 79_999], device=DEV)
    qa[at] = rq
    sa[at] = words(rs, False)
    y = ds3.ds3_gemm_mxfp4(qa, sa, qb, words(sb))
    got, want = y[at].double().cpu().numpy(), ra @ b.T
    assert (np.abs(got - want) <= allowed(ra, b, want, K, True)).all()
    other = torch.ones(M, dtype=torch.bool, device=DEV)
    other[at] = False
    assert not y[other].any()


def test_results_do_not_depend_on_timing(ds3):
    rng = np.random.default_rng(4)
    _, qa, sa = operand(rng, 200, 3584)
    _, qb, sb = operand(rng, 700, 3584)
    first = ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), out_dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(first, ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), out_dtype=torch.float32))
