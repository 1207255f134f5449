"""Dispatch, combine and its gradients at the sizes of a training batch, where a wave takes two or four times 512 columns of a
token and where large results are written past the caches: every form, type and ragged end, all rows compared."""
import numpy as np
import pytest
import torch

from tests import test_gpu_moe as small
from tests._gpu_util import DEV, announce

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def waves(tokens, cols):
    return tokens * -(-cols // 512)


# tokens, choices a token, experts, columns, padding: from 4096 waves of 512 columns on a wave takes four (from 1025 columns on) or
# two (from 513) of them
BATCHES = [(1100, 6, 64, 2056, 10), (2100, 2, 16, 1000, 0), (1400, 1, 8, 1544, 3), (4200, 3, 12, 264, 7), (300, 20, 24, 7176, 0)]


@pytest.mark.parametrize("dtype,less", [(BF16, 0), (F32, 0), (F32, 4)])
@pytest.mark.parametrize("tokens,k,experts,cols,padded", BATCHES)
def test_dispatch(ds3, tokens, k, experts, cols, padded, dtype, less):
    """Rows, FP8 with both kinds of scales, MXFP4: equal to the quantizers' on the token's row; FP32 rows that end after four."""
    assert waves(tokens, cols - less) >= 4096
    small.test_dispatch(ds3, tokens, k, experts, cols - less, padded, dtype)


@pytest.mark.parametrize("yt,ot,less", [(BF16, BF16, 0), (BF16, F32, 0), (F32, BF16, 0), (F32, F32, 0), (F32, F32, 4)])
@pytest.mark.parametrize("tokens,k,experts,cols,padded", BATCHES)
def test_combine_and_its_gradients(ds3, tokens, k, experts, cols, padded, yt, ot, less):
    assert waves(tokens, cols - less) >= 4096
    small.test_combine_and_its_gradients(ds3, tokens, k, experts, cols - less, padded, yt, ot)


# at least 64 MiB of sums (by out's type) and of gradients (by y's)
LARGE = [(2400, 2, 8, 7172, F32, F32), (4700, 2, 8, 7176, BF16, BF16), (4700, 2, 8, 7176, BF16, F32), (4700, 2, 8, 7176, F32, BF16),
         (1500, 9, 16, 5004, F32, F32)]


@pytest.mark.parametrize("tokens,k,experts,cols,yt,ot", LARGE)
@pytest.mark.parametrize("weighted", [True, False])
def test_large_results(ds3, tokens, k, experts, cols, yt, ot, weighted):
    """The sums in 64 bits on the device, tolerances as in test_gpu_moe.py: k * 2^-24 of the sum of the magnitudes (1.01: the
    products of such terms), then the output's rounding; a lane's columns, eight of every 512, then six steps over the lanes."""
    announce(f"combine {tokens}x{k} of {experts}, {cols} columns, {yt} -> {ot}, weights {weighted}")
    rng, rows, hrows, total = small.layout(ds3, tokens, k, experts, 9, tokens + cols)
    size = {BF16: 2, F32: 4}
    sums, grads = tokens * cols * size[ot], min(total, tokens * k) * cols * size[yt]
    assert max(sums, grads) >= 64 << 20
    gen = torch.Generator(device=DEV).manual_seed(cols)
    y = torch.full((total, cols + 16), float("nan"), dtype=yt, device=DEV)
    y[:, :cols] = torch.randn((total, cols), generator=gen, device=DEV).to(yt)
    nobody = torch.from_numpy(np.setdiff1d(np.arange(total), hrows)).to(DEV)
    y[nobody] = float("nan")                                         # nothing may come from rows that nobody names
    y = y[:, :cols]
    w = torch.rand((tokens, k), generator=gen, device=DEV) - 0.3 if weighted else None
    dout = torch.randn((tokens, cols), generator=gen, device=DEV).to(ot)
    wd = torch.ones((tokens, k), dtype=torch.float64, device=DEV) if w is None else w.double()
    want, mag = (torch.zeros((tokens, cols), dtype=torch.float64, device=DEV) for _ in range(2))
    wdy = torch.full((total, cols), 11.0, dtype=torch.float64, device=DEV)
    wdw, wdm = (torch.zeros((tokens, k), dtype=torch.float64, device=DEV) for _ in range(2))
    for j in range(k):
        t = torch.from_numpy(np.nonzero(hrows[:, j] >= 0)[0]).to(DEV)
        r = rows[t, j].long()
        term = y[r].double()
        want[t] += wd[t, j, None] * term
        mag[t] += (wd[t, j, None] * term).abs()
        wdy[r] = wd[t, j, None] * dout[t].double()
        wdw[t, j] = (dout[t].double() * term).sum(1)
        wdm[t, j] = (dout[t].double() * term).abs().sum(1)
    out = torch.full((tokens, cols + 16), 7.0, dtype=ot, device=DEV)
    got = ds3.ds3_moe_combine(y, rows, w, out=out[:, :cols])
    near = 1.01 * k * 2.0 ** -24 * mag
    assert bool(((got.double() - want).abs() <= near + small.EPS[ot] * (want.abs() + near)).all()) and bool((out[:, cols:] == 7).all())
    dyd = torch.full((total, cols + 16), 11.0, dtype=yt, device=DEV)
    dy, dw = ds3.ds3_moe_combine_bwd(dout, y, rows, w, dy=dyd[:, :cols])
    kept = torch.ones(total, dtype=torch.bool, device=DEV)
    kept[torch.from_numpy(hrows[hrows >= 0]).to(DEV).long()] = False
    assert bool((dy[kept] == 11).all()) and bool((dyd[:, cols:] == 11).all())
    slack = 1.01 * (2.0 ** -24 + small.EPS[yt]) * wdy.abs() + 2.0 ** -133
    assert bool(((dy.double() - wdy).abs() <= slack)[~kept].all())
    assert bool(((dw.double() - wdw).abs() <= 1.01 * (8 * -(-cols // 512) + 6) * 2.0 ** -24 * wdm).all())
    assert not dw[rows < 0].any()
