"""MXFP4 products whose persistent workgroups take several tiles, over several K-steps: a tile's stores in flight under the
next tile's first K-steps, what is there fetched under the next tile's loads, and last rounds whose tiles are cut into halves.

Tolerance as in test_gpu_gemm_mxfp4.py: (K / 128 + 4) * 2^-23 of the sum of the products' magnitudes, a BF16 output another half
step.  Where the result is added to c the sum is rounded once more, half a step of it: 2^-24 of |result| + |c|, doubled for the
result's own error."""
import numpy as np
import pytest
import torch

from tests._gpu_util import DEV, announce
from tests.test_gpu_gemm_mxfp4 import compute_units, operand, words

pytestmark = pytest.mark.gpu


def walk(M, N, bm, bn, per_cu, cus=256):
    """(full rounds, tiles left, whether those are cut into halves) of each of the eight parts of the tile list."""
    tiles = -(-M // bm) * -(-N // bn)
    slots = min(-(-tiles // 8) * 8, cus * per_cu) // 8
    part = -(-tiles // 8)
    out = []
    for x in range(8):
        mine = max(0, min(part, tiles - x * part))
        rounds, left = divmod(mine, slots)
        out.append((rounds, left, rounds > 0 and left > 0 and 2 * left <= slots and M % bm == 0))
    return out


# configuration, M, N, K, whether a last round is cut: 256x256 and 128x128 tiles, K-steps that end in a half and whole ones,
# columns that end inside a tile, rows that do
ROUNDS = [(7, 2304, 14676, 1152, True), (7, 2300, 14680, 1152, False), (6, 2048, 9216, 640, True), (6, 1920, 9220, 896, True),
          (6, 3000, 7168, 1536, False)]


@pytest.mark.parametrize("config,M,N,K,cut", ROUNDS)
def test_dense_over_several_rounds(ds3, config, M, N, K, cut):
    announce(f"mxfp4 gemm {M}x{N}x{K}, configuration {config}, several rounds")
    if compute_units() == 256:
        assert ds3._L().ds3_gemm_mxfp4_config(0, M, N, K, 256) == config
        parts = walk(M, N, *((256, 256, 1) if config == 7 else (128, 128, 2)))
        assert max(r for r, _, _ in parts) >= 2 and any(h for _, _, h in parts) == cut and all(left for _, left, _ in parts)
    rng = np.random.default_rng(M + N + K)
    a, qa, sa = operand(rng, M, K, lead=1)
    b, qb, sb = operand(rng, N, K, lead=2)
    da, db = torch.from_numpy(a).to(DEV), torch.from_numpy(b).to(DEV)          # (the products in 64 bits on the device: large)
    want, near = da @ db.t(), (K / 128 + 4) * 2.0 ** -23 * (da.abs() @ db.abs().t())
    ld = (N + 7) // 8 * 8 + 8
    for dtype in (torch.float32, torch.bfloat16):
        c = torch.full((M, ld), 5.0, dtype=dtype, device=DEV)
        ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), c=c[:, :N])
        tol = near + 2.0 ** -8 * (want.abs() + near) if dtype == torch.bfloat16 else near
        assert bool(((c[:, :N].double() - want).abs() <= tol).all()) and bool((c[:, N:] == 5).all())
    c0 = torch.randn((M, N), generator=torch.Generator(device=DEV).manual_seed(K), device=DEV) * 30
    c = torch.full((M, ld), 5.0, device=DEV)
    c[:, :N] = c0
    ds3.ds3_gemm_mxfp4(qa, words(sa), qb, words(sb), c=c[:, :N], accumulate=True)
    full = want + c0.double()
    assert bool(((c[:, :N].double() - full).abs() <= near + 2.0 ** -23 * (want.abs() + c0.double().abs())).all()) and bool((c[:, N:] == 5).all())


# configuration, an expert's rows, N, K: more tiles than workgroups at once (512 of 128x128, 256 of the others)
GROUPED = [(11, (129,) * 32, 1280, 1152), (12, (60, 0, 129, 90, 64, 257, 31, 1) * 4, 4104, 1664), (13, (250, 100, 0, 300, 257, 129, 1, 256) * 4, 4104, 1152)]


@pytest.mark.parametrize("config,sizes,N,K", GROUPED)
def test_grouped_over_several_rounds(ds3, config, sizes, N, K):
    G, rows = len(sizes), sum(sizes) + 5
    announce(f"mxfp4 grouped {G} experts, {rows} rows, {N}x{K}, configuration {config}, several rounds")
    if compute_units() == 256:
        bm, bn, slots = {11: (128, 128, 512), 12: (128, 256, 256), 13: (256, 256, 256)}[config]
        assert ds3._L().ds3_gemm_mxfp4_config(G, rows, N, K, 256) == config
        assert sum(-(-n // bm) for n in sizes) * -(-N // bn) > slots
    rng = np.random.default_rng(config + K)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    a, qa, sa = operand(rng, rows, K, lead=1)
    b, qb, sb = operand(rng, G * N, K)
    w = words(sb, False).view(G, N, K // 128).transpose(1, 2).contiguous().transpose(1, 2)
    qb, offd = qb.contiguous().view(G, N, K // 2), torch.from_numpy(off).to(DEV)
    got = {}
    for dtype in (torch.float32, torch.bfloat16):
        c = torch.full((rows, (N + 7) // 8 * 8), 5.0, dtype=dtype, device=DEV)
        got[dtype] = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), offd, qb, w, c=c[:, :N])
        assert bool((c[:, N:] == 5).all()) and bool((c[off[-1] :] == 5).all())
    for g in range(G):
        at = slice(int(off[g]), int(off[g + 1]))
        da, db = torch.from_numpy(a[at]).to(DEV), torch.from_numpy(b[g * N : (g + 1) * N]).to(DEV)
        want, near = da @ db.t(), (K / 128 + 4) * 2.0 ** -23 * (da.abs() @ db.abs().t())
        assert bool(((got[torch.float32][at].double() - want).abs() <= near).all())
        assert bool(((got[torch.bfloat16][at].double() - want).abs() <= near + 2.0 ** -8 * (want.abs() + near)).all())
