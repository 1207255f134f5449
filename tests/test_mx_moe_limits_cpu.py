"""The sizes that the header gives for the MXFP4 quantizers and the calls around expert order: one more is refused on the host
(the pointers are host memory that nothing reads).  That the last ones run is tested on the GPU (test_gpu_mx_moe_limits.py)."""
import ctypes

import pytest

import paper_2412_19437_amd as pkg

UNSUPPORTED = 5


@pytest.fixture(scope="module")
def mem():
    buf = (ctypes.c_uint8 * 4096)()
    yield (ctypes.addressof(buf) + 15) & ~15
    del buf


def test_quantizers(mem):
    L = pkg._L()
    rows = 16 * (2**24 - 1) + 1
    assert L.ds3_quant_mxfp4(mem, 1, rows, 8, 8, mem, 16, mem, 1, rows, None) == UNSUPPORTED
    assert L.ds3_quant_mxfp4(mem, 1, 2**20 * 16 - 15, 16 * 256, 16 * 256, mem, 2048, mem, 16, 1, None) == UNSUPPORTED
    assert L.ds3_dequant_mxfp4(mem, rows, 8, 16, mem, 1, rows, mem, 8, None) == UNSUPPORTED
    assert L.ds3_quant_mxfp4_t(mem, 1, 16776961, 8, 8, mem, 8388496, mem, 1, 8, None) == UNSUPPORTED
    assert L.ds3_quant_mxfp4_t(mem, 1, 32, 2**30 - 56, 2**30 - 56, mem, 16, mem, 1, 2**30 - 56, None) == UNSUPPORTED


def test_expert_order(mem):
    L = pkg._L()
    t = 2**26 - 3
    assert L.ds3_moe_sort(mem, 2**31 - 8191, 1, 1, 0, 4, mem, mem, None) == UNSUPPORTED
    for dispatch in (L.ds3_moe_dispatch_quant_1x128, L.ds3_moe_dispatch_quant_1x128_pow2, L.ds3_moe_dispatch_quant_mxfp4):
        assert dispatch(mem, 1, t, 8, 8, mem, 1, t, mem, 16, mem, 1, t, None) == UNSUPPORTED
    assert L.ds3_moe_dispatch(mem, 1, t, 8, 8, mem, 1, t, mem, 8, None) == UNSUPPORTED
    assert L.ds3_moe_combine(mem, 1, t, 8, 8, mem, mem, t, 1, mem, 1, 8, None) == UNSUPPORTED
    assert L.ds3_moe_combine_bwd(mem, 1, 8, mem, 1, t, 8, 8, mem, mem, t, 1, mem, 8, mem, None) == UNSUPPORTED
    # the gradients go by choices, the sums by tokens
    assert L.ds3_moe_combine_bwd(mem, 1, 8, mem, 1, t, 8, 8, mem, mem, 2**20, 64, mem, 8, mem, None) == UNSUPPORTED


def test_products(mem):
    L = pkg._L()
    n = 2**40 // (1023 * 64) + 1
    assert L.ds3_grouped_gemm_mxfp4(1023, mem, 16, n, 128, mem, 64, mem, 1, 16, mem, 64, mem, 1, n, mem, 1, n + 3 & ~3, None) == UNSUPPORTED
