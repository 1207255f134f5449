"""A grouped MXFP4 product of few rows with more tiles of 64x32 than a grid holds workgroups: 61 GB of weights."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce
from tests.test_gpu_gemm_mxfp4 import allowed, operand, words

pytestmark = pytest.mark.gpu


def test_more_tiles_than_a_grid_holds(ds3):
    G, M, N, K = 64, 256, 14_950_016, 128
    announce(f"mxfp4 grouped {G} experts, {M} rows, {N}x{K}")
    rng = np.random.default_rng(8)
    sizes = [4] * G
    sizes[3], sizes[4] = 0, 8
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    a, qa, sa = operand(rng, M, K)
    gen = torch.Generator(device=DEV).manual_seed(2)
    qb = torch.randint(0, 256, (G, N, K // 2), dtype=torch.uint8, device=DEV, generator=gen)
    sb = torch.randint(120, 134, (G, N, 4), dtype=torch.uint8, device=DEV, generator=gen).view(torch.int32)
    y = ds3.ds3_grouped_gemm_mxfp4(qa, words(sa), torch.from_numpy(off).to(DEV), qb, sb)
    at = torch.cat([torch.arange(0, 130), torch.arange(N // 2 - 70, N // 2 + 70), torch.randint(0, N, (300,), generator=torch.Generator().manual_seed(1)),
                    torch.arange(N - 130, N)]).to(DEV)
    for g in range(G):
        rows = slice(int(off[g]), int(off[g + 1]))
        b = mx.dequant_mxfp4(qb[g, at].cpu().numpy(), sb[g, at].contiguous().cpu().numpy().view(np.uint8))
        want = a[rows] @ b.T
        assert (np.abs(y[rows][:, at].double().cpu().numpy() - want) <= allowed(a[rows], b, want, K, True)).all()
