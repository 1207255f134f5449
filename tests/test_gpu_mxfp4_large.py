"""The MXFP4 dequantizer where its values are written past the caches (from 48 MiB on) and past 32 bits."""
import numpy as np
import pytest
import torch

from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce
from tests.test_gpu_mxfp4 import bytes_of

pytestmark = pytest.mark.gpu


def equal_with_nan(got, want):
    return np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


@pytest.mark.parametrize("rows,cols", [(6200, 4099), (6145, 4096), (25_000, 1030), (1_700_000, 15)])
def test_values_written_past_the_caches(ds3, rows, cols):
    """Every value, random codes and scales with NaN scales among them; rows that end inside eight, in padding left as it was."""
    announce(f"dequant {rows}x{cols}")
    assert rows * cols * 2 >= 48 << 20
    rng = np.random.default_rng(cols)
    w, kw = (cols + 1) // 2, -(-cols // 128)
    q = rng.integers(0, 256, (rows, w), dtype=np.uint8)
    s = rng.integers(0, 252, (rows, 4 * kw)).astype(np.uint8)        # (6 * 2^124 is BF16's last step but one)
    s[rng.random(s.shape) < 0.01] = 255
    qd = torch.full((rows, (w + 15) // 16 * 16), 0x77, dtype=torch.uint8, device=DEV)
    qd[:, :w] = torch.from_numpy(q).to(DEV)
    sd = torch.from_numpy(mx.words(s).copy()).to(DEV)
    # the values by the format's definition, in 64 bits on the device; sampled rows are compared with the oracle's as well
    table = torch.from_numpy(mx.e2m1_decode(np.arange(16))).to(DEV)
    code = torch.stack((qd[:, :w] & 15, qd[:, :w] >> 4), -1).flatten(1)[:, :cols].long()
    power = np.ldexp(1.0, np.arange(256) - 127)
    power[255] = np.nan
    scale = torch.from_numpy(power).to(DEV)[torch.from_numpy(s).to(DEV).long()].repeat_interleave(32, 1)[:, :cols]
    want = table[code] * scale
    lead = (cols + 7) // 8 * 8
    for words in (sd, sd.t().contiguous().t()):
        y = torch.full((rows + 1, lead), 3.0, dtype=torch.bfloat16, device=DEV)
        st = torch.cuda.current_stream().cuda_stream
        assert ds3._L().ds3_dequant_mxfp4(qd.data_ptr(), rows, cols, qd.stride(0), words.data_ptr(), words.stride(0), words.stride(1),
                                          y.data_ptr(), lead, st) == 0
        got = y[:rows, :cols].double()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
        assert bool((y[rows] == 3).all()) and bool((y[:, cols:] == 3).all())
    at = np.array([0, 1, rows // 2, rows - 2, rows - 1])
    assert equal_with_nan(want[torch.from_numpy(at).to(DEV)].cpu().numpy(), mx.dequant_mxfp4(q[at], s[at], cols))


def test_rows_past_32_bits(ds3):
    """Codes of 2.2 GB and values of 8.6 GB: sampled rows and the last columns."""
    rows, cols = 600_000, 7168
    gen = torch.Generator(device=DEV).manual_seed(6)
    q = torch.randint(0, 256, (rows, cols // 2), dtype=torch.uint8, device=DEV, generator=gen)
    s = torch.randint(100, 150, (cols // 128, rows, 4), dtype=torch.uint8, device=DEV, generator=gen).view(torch.int32)[..., 0].t()
    y = ds3.ds3_dequant_mxfp4(q, s)
    at = torch.tensor([0, 1, 299_593, 299_594, 599_186, 599_187, rows - 2, rows - 1], device=DEV)
    want = mx.dequant_mxfp4(q[at].cpu().numpy(), bytes_of(s[at]))
    assert np.array_equal(y[at].double().cpu().numpy(), want)
