"""Refusals of the MXFP4 calls and of the calls around expert order: found on the host, before any launch, so they need no
GPU (the pointers are host memory that nothing reads)."""
import ctypes
import os

import pytest
import torch

NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def pkg():
    import paper_2412_19437_amd as p
    if not (os.path.exists(p.LIB_PATH) and os.path.exists(p.NATIVE_PATH)):
        from paper_2412_19437_amd.build import build_library
        build_library(verbose=False)
    return p


@pytest.fixture(scope="module")
def mem():
    buf = (ctypes.c_uint8 * 4096)()
    yield (ctypes.addressof(buf) + 15) & ~15
    del buf


def _try(fn, good, **changes):
    args = dict(good)
    args.update(changes)
    return fn(*args.values())


def test_quantizers(pkg, mem):
    for name in ("ds3_quant_mxfp4", "ds3_quant_mxfp4_t"):
        fn = getattr(pkg._L(), name)
        good = dict(x=mem, xt=1, rows=64, cols=128, ldx=128, q=mem, ldq=64, s=mem, s0=1, s1=64, st=None)
        for key in ("x", "q", "s"):
            assert _try(fn, good, **{key: None}) == NULL
        assert _try(fn, good, xt=7) == DTYPE
        assert _try(fn, good, rows=-1) == SHAPE and _try(fn, good, cols=-8) == SHAPE and _try(fn, good, ldx=120) == SHAPE
        assert _try(fn, good, cols=124) == ALIGN and _try(fn, good, ldx=132) == ALIGN and _try(fn, good, x=mem + 8) == ALIGN
        assert _try(fn, good, xt=0, cols=126, ldx=128) == ALIGN
        assert _try(fn, good, q=mem + 4) == ALIGN and _try(fn, good, ldq=72) == ALIGN and _try(fn, good, s=mem + 2) == ALIGN
        assert _try(fn, good, ldq=16) == SHAPE                       # 128 (transposed: 64) elements take more
        assert _try(fn, good, rows=0, x=None, q=None, s=None) == 0 and _try(fn, good, cols=0, x=None) == 0
        assert _try(fn, good, rows=1 << 31) in (SHAPE, UNSUPPORTED)
    assert _try(pkg._L().ds3_quant_mxfp4_t, good, rows=1 << 25, ldq=1 << 24) == UNSUPPORTED
    fn = pkg._L().ds3_dequant_mxfp4
    good = dict(q=mem, rows=4, cols=33, ldq=32, s=mem, s0=2, s1=1, y=mem, ldy=40, st=None)
    for key in ("q", "s", "y"):
        assert _try(fn, good, **{key: None}) == NULL
    assert _try(fn, good, cols=65) == SHAPE and _try(fn, good, ldy=32) == SHAPE and _try(fn, good, rows=-1) == SHAPE
    assert _try(fn, good, ldy=36) == ALIGN and _try(fn, good, y=mem + 8) == ALIGN and _try(fn, good, ldq=24) == ALIGN
    assert _try(fn, good, rows=0, q=None) == 0


def test_products(pkg, mem):
    fn = pkg._L().ds3_gemm_mxfp4
    good = dict(M=16, N=24, K=256, a=mem, lda=128, sa=mem, sar=1, sak=16, b=mem, ldb=128, sb=mem, sbr=1, sbk=24, c=mem, ct=1, ldc=24,
                acc=0, st=None)
    for key in ("a", "sa", "b", "sb", "c"):
        assert _try(fn, good, **{key: None}) == NULL
    assert _try(fn, good, ct=3) == DTYPE and _try(fn, good, acc=1) == DTYPE
    for bad in (dict(K=192), dict(M=-1), dict(lda=112), dict(ldb=112), dict(ldc=20)):
        assert _try(fn, good, **bad) == SHAPE, bad
    for bad in (dict(a=mem + 8), dict(b=mem + 8), dict(c=mem + 8), dict(lda=136), dict(ldb=136), dict(ldc=26), dict(sa=mem + 2)):
        assert _try(fn, good, **bad) == ALIGN, bad
    for bad in (dict(sar=-1), dict(sbk=-1), dict(sak=1 << 29), dict(sar=0, sak=(1 << 29) - 1), dict(sbr=1 << 26), dict(lda=1 << 23), dict(ldb=1 << 23), dict(M=1 << 31),
                dict(lda=1 << 31)):
        assert _try(fn, good, **bad) == UNSUPPORTED, bad
    for big in ((1 << 31) - 1, (1 << 31) - 255):                     # tiles of 256 of them would pass 32 bits
        assert _try(fn, good, M=big, sar=0) == UNSUPPORTED and _try(fn, good, N=big, ldc=1 << 31, sbr=0) == UNSUPPORTED
        assert pkg._L().ds3_gemm_mxfp4_config(0, big, 64, 128, 256) == -1 and pkg._L().ds3_gemm_mxfp4_config(8, 64, big, 128, 256) == -1
    assert _try(fn, good, M=0, a=None, c=None) == 0 and _try(fn, good, N=0) == 0
    assert _try(fn, good, K=0, ct=0, acc=1, a=None) == 0             # C += an empty sum
    fn = pkg._L().ds3_grouped_gemm_mxfp4
    good = dict(G=2, off=mem, M=16, N=24, K=256, a=mem, lda=128, sa=mem, sar=1, sak=16, b=mem, ldb=128, sb=mem, sbr=1, sbk=24, c=mem,
                ct=1, ldc=24, st=None)
    for key in ("off", "a", "sa", "b", "sb", "c"):
        assert _try(fn, good, **{key: None}) == NULL
    assert _try(fn, good, G=-1) == SHAPE and _try(fn, good, G=1024) == UNSUPPORTED and _try(fn, good, K=0) == UNSUPPORTED
    assert _try(fn, good, G=0, off=None) == 0 and _try(fn, good, M=0, off=None) == 0
    assert _try(fn, good, off=mem + 2) == ALIGN
    assert _try(fn, good, G=1023, N=1 << 24, ldb=128, ldc=1 << 24, sbk=1 << 24) == UNSUPPORTED


def test_configuration_query(pkg):
    f = pkg._L().ds3_gemm_mxfp4_config
    for bad in ((0, 0, 64, 128, 256), (0, 16, 0, 128, 256), (0, 16, 64, 0, 256), (0, 16, 64, 100, 256), (0, 16, 64, 128, 4), (-1, 16, 64, 128, 256),
                (1024, 16, 64, 128, 256), (0, 1 << 31, 64, 128, 256)):
        assert f(*bad) == -1
    seen = {f(0, m, n, k, 256) for m in (1, 16, 100, 450, 2048, 4096) for n in (576, 2001, 18432) for k in (128, 896, 2176, 7168)}
    seen |= {f(0, 333, 4001, 640, 256)} | {f(8, 8 * m, n, 384, 256) for m in (4, 40, 60, 128, 200, 600) for n in (64, 264, 2056, 8192)}
    assert seen == set(range(14))
    # the groups of waves of a tile never outnumber the K-steps of 256
    assert f(0, 1, 512, 128, 256) == 5 and f(0, 1, 512, 512, 256) != 0


def test_expert_order(pkg, mem):
    L = pkg._L()
    good = dict(ids=mem, tokens=8, k=2, ld=2, first=0, G=4, off=mem, rows=mem, st=None)
    for key in ("ids", "off", "rows"):
        assert _try(L.ds3_moe_sort, good, **{key: None}) == NULL
    for bad in (dict(tokens=-1), dict(k=0), dict(ld=1), dict(first=-1), dict(G=-1), dict(first=(1 << 31) - 3)):
        assert _try(L.ds3_moe_sort, good, **bad) == SHAPE, bad
    assert _try(L.ds3_moe_sort, good, k=65, ld=65) == UNSUPPORTED and _try(L.ds3_moe_sort, good, G=1024) == UNSUPPORTED
    assert _try(L.ds3_moe_sort, good, tokens=1 << 30) == UNSUPPORTED
    assert _try(L.ds3_moe_sort, good, ids=mem + 2) == ALIGN
    plain = dict(x=mem, xt=1, tokens=8, cols=128, ldx=128, rows=mem, k=2, total=16, y=mem, ldy=128, st=None)
    quant = dict(x=mem, xt=1, tokens=8, cols=128, ldx=128, rows=mem, k=2, total=16, q=mem, ldq=128, s=mem, s0=1, s1=16, st=None)
    for fn, good, out in ((L.ds3_moe_dispatch, plain, "y"), (L.ds3_moe_dispatch_quant_1x128, quant, "q"),
                          (L.ds3_moe_dispatch_quant_1x128_pow2, quant, "q"), (L.ds3_moe_dispatch_quant_mxfp4, quant, "q")):
        for key in ("x", "rows", out) + (("s",) if out == "q" else ()):
            assert _try(fn, good, **{key: None}) == NULL
        assert _try(fn, good, xt=2) == DTYPE
        for bad in (dict(tokens=-1), dict(cols=-8), dict(k=0), dict(total=-1), dict(ldx=120), {"ld" + out: 48}):
            assert _try(fn, good, **bad) == SHAPE, bad
        for bad in (dict(x=mem + 8), {out: mem + 8}, dict(cols=124), dict(ldx=132), {"ld" + out: 132}, dict(rows=mem + 1)):
            assert _try(fn, good, **bad) == ALIGN, bad
        assert _try(fn, good, k=65) == UNSUPPORTED and _try(fn, good, total=1 << 31) == UNSUPPORTED
        assert _try(fn, good, tokens=0, x=None) == 0 and _try(fn, good, total=0, x=None) == 0 and _try(fn, good, cols=0) == 0
        assert _try(fn, good, tokens=1 << 27, cols=8) == UNSUPPORTED           # more workgroups than a grid holds
    good = dict(y=mem, yt=1, total=16, cols=128, ldy=128, rows=mem, w=mem, tokens=8, k=2, out=mem, ot=1, ldo=128, st=None)
    fn = L.ds3_moe_combine
    for key in ("y", "rows", "out"):
        assert _try(fn, good, **{key: None}) == NULL
    assert _try(fn, good, yt=2) == DTYPE and _try(fn, good, ot=-1) == DTYPE
    for bad in (dict(ldy=120), dict(ldo=120), dict(k=0), dict(tokens=-1), dict(total=-1)):
        assert _try(fn, good, **bad) == SHAPE, bad
    for bad in (dict(y=mem + 8), dict(out=mem + 8), dict(w=mem + 2), dict(cols=124), dict(ldy=132), dict(ldo=132)):
        assert _try(fn, good, **bad) == ALIGN, bad
    assert _try(fn, good, k=65) == UNSUPPORTED and _try(fn, good, tokens=0, y=None) == 0 and _try(fn, good, cols=0, y=None) == 0
    good = dict(d=mem, ot=1, ldo=128, y=mem, yt=1, total=16, cols=128, ldy=128, rows=mem, w=mem, tokens=8, k=2, dy=mem, lddy=128, dw=mem,
                st=None)
    fn = L.ds3_moe_combine_bwd
    for key in ("d", "y", "rows", "dy", "dw"):
        assert _try(fn, good, **{key: None}) == NULL
    assert _try(fn, good, yt=2) == DTYPE and _try(fn, good, lddy=120) == SHAPE and _try(fn, good, lddy=132) == ALIGN
    assert _try(fn, good, cols=0, d=None, y=None, dy=None, dw=None) == NULL       # (zeros are written there)
    assert _try(fn, good, dy=mem + 8) == ALIGN and _try(fn, good, dw=mem + 2) == ALIGN and _try(fn, good, tokens=1 << 27) == UNSUPPORTED


def test_python_calls_ask_for_tensors_of_the_current_device(pkg):
    x, ids = torch.zeros((8, 128)), torch.zeros((8, 2), dtype=torch.int32)
    q, s = torch.zeros((8, 64), dtype=torch.uint8), torch.zeros((8, 1), dtype=torch.int32)
    calls = [lambda: pkg.ds3_quant_mxfp4(x), lambda: pkg.ds3_quant_mxfp4_t(x), lambda: pkg.ds3_dequant_mxfp4(q, s),
             lambda: pkg.ds3_gemm_mxfp4(q, s, q, s), lambda: pkg.ds3_grouped_gemm_mxfp4(q, s, ids, q, s), lambda: pkg.ds3_moe_sort(ids, 4),
             lambda: pkg.ds3_moe_dispatch(x, ids), lambda: pkg.ds3_moe_dispatch_quant_1x128(x, ids),
             lambda: pkg.ds3_moe_dispatch_quant_1x128_pow2(x, ids), lambda: pkg.ds3_moe_dispatch_quant_mxfp4(x, ids),
             lambda: pkg.ds3_moe_combine(x, ids), lambda: pkg.ds3_moe_combine_bwd(x, x, ids)]
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    for call in (lambda: pkg.ds3_quant_mxfp4([1]), lambda: pkg.ds3_moe_sort(None, 4), lambda: pkg.ds3_gemm_mxfp4(q, s, q, s, out_dtype=torch.float16),
                 lambda: pkg.ds3_moe_combine(x, ids, out_dtype=torch.int32)):
        with pytest.raises(TypeError):
            call()
