"""The MXFP4 quantizers and the calls around expert order at the largest sizes that the header gives."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce
from tests.test_gpu_mxfp4 import bytes_of

pytestmark = pytest.mark.gpu


def values(rows, cols, seed):
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    return x.normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


def test_most_rows_along_a_row_and_back(ds3):
    rows = 16 * (2**24 - 1)
    announce(f"mxfp4 {rows}x8")
    x = values(rows, 8, 1)
    q, s = ds3.ds3_quant_mxfp4(x)
    y = ds3.ds3_dequant_mxfp4(q, s)
    at = torch.tensor([0, 1, 2**27 - 1, 2**27, 2**27 + 1, rows - 17, rows - 2, rows - 1], device=DEV)
    wq, ws = mx.quant_mxfp4(x[at].float().cpu().numpy())
    assert np.array_equal(q[at].cpu().numpy(), wq) and np.array_equal(bytes_of(s[at]), ws)
    assert np.array_equal(y[at].double().cpu().numpy(), mx.dequant_mxfp4(wq, ws, 8))
    # all of it against itself, moved by half the rows
    half = rows // 2
    q2, s2 = ds3.ds3_quant_mxfp4(x[half:])
    assert torch.equal(q[half:], q2) and torch.equal(s[half:], s2)


def test_most_rows_transposed(ds3):
    """Equal to the quantizer along a row on the transposed matrix."""
    rows = 65535 * 256
    announce(f"mxfp4, transposed, {rows}x8")
    x = values(rows, 8, 2)
    qt, st = ds3.ds3_quant_mxfp4_t(x)
    q, s = ds3.ds3_quant_mxfp4(x.t().contiguous())
    assert torch.equal(qt, q) and torch.equal(st, s)


def test_most_tokens_dispatched_and_combined(ds3):
    tokens = 2**26 - 4
    announce(f"dispatch, combine and gradients of {tokens} tokens")
    x = values(tokens, 8, 3)
    rows = torch.arange(tokens - 1, -1, -1, dtype=torch.int32, device=DEV)[:, None].contiguous()
    y = ds3.ds3_moe_dispatch(x, rows)
    assert torch.equal(y, x.flip(0))
    assert torch.equal(ds3.ds3_moe_combine(y, rows), x)
    dy, dw = ds3.ds3_moe_combine_bwd(x, y, rows)
    assert torch.equal(dy, y)
    want = x.double().square().sum(1)
    assert bool(((dw[:, 0].double() - want).abs() <= 1.01 * (8 + 6) * 2.0 ** -24 * want).all())
    del dy, dw, want
    q, s = ds3.ds3_moe_dispatch_quant_mxfp4(x, rows)
    q0, s0 = ds3.ds3_quant_mxfp4(y)
    assert torch.equal(q, q0) and torch.equal(s, s0)
    q, s = ds3.ds3_moe_dispatch_quant_1x128(x, rows)
    q0, s0 = ds3.ds3_quant_act_1x128(y)
    assert torch.equal(q, q0) and torch.equal(s, s0)


def test_most_choices_sorted(ds3):
    """Experts in turn, so that the row of choice i is known: the first row of its expert and i / experts."""
    n, experts, held = 2**31 - 8192, 6, 5
    announce(f"sort of {n} choices")
    ids = torch.arange(n, dtype=torch.int32, device=DEV).remainder_(experts)[:, None]
    off, rows = ds3.ds3_moe_sort(ids, held)
    counts = [(n - e + experts - 1) // experts for e in range(held)]
    first = np.concatenate([[0], np.cumsum(counts)])
    assert off.cpu().numpy().tolist() == first.tolist()
    starts = torch.from_numpy(np.append(first[:held], 0)).to(DEV)
    for at in range(0, n, 1 << 28):
        i = torch.arange(at, min(at + (1 << 28), n), device=DEV)
        e = i % experts
        want = torch.where(e < held, starts[e] + i // experts, -1)
        assert torch.equal(rows[at : at + (1 << 28), 0].long(), want)
