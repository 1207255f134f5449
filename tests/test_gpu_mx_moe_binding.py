"""What the Python calls of the MXFP4 operators and of expert order refuse, and that they launch nothing then."""
import pytest
import torch

from tests._gpu_util import DEV

pytestmark = pytest.mark.gpu


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device=DEV)


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device=DEV)


def test_mxfp4_calls(ds3):
    x = bf16(4, 128)
    for f in (ds3.ds3_quant_mxfp4, ds3.ds3_quant_mxfp4_t):
        with pytest.raises(TypeError):
            f(x.half())
        with pytest.raises(ValueError):
            f(x.T)
        with pytest.raises(ValueError):
            f(x[0])
    with pytest.raises(TypeError, match="uint8"):
        ds3.ds3_dequant_mxfp4(x, i32(4, 2))
    for cols in (126, 129):
        with pytest.raises(ValueError, match="two columns a byte"):
            ds3.ds3_dequant_mxfp4(u8(4, 64), i32(4, 1), cols=cols)
    with pytest.raises(ValueError, match="int32"):
        ds3.ds3_dequant_mxfp4(u8(4, 64), i32(4, 2))
    a, sa, b, sb = u8(4, 128), i32(4, 2), u8(8, 128), i32(8, 2)
    assert (ds3.ds3_gemm_mxfp4(a, sa, b, sb) == 0).all()
    for bad in (dict(b=u8(8, 64)), dict(sa=i32(4, 1)), dict(sb=i32(4, 2)), dict(sb=sb.float()), dict(c=bf16(4, 4)), dict(c=bf16(8, 8).T[:4]), dict(accumulate=True)):
        with pytest.raises(ValueError):
            ds3.ds3_gemm_mxfp4(**{**dict(a=a, sa=sa, b=b, sb=sb), **bad})
    for bad in (dict(a=x), dict(out_dtype=torch.float16), dict(c=bf16(4, 8).half())):
        with pytest.raises(TypeError):
            ds3.ds3_gemm_mxfp4(**{**dict(a=a, sa=sa, b=b, sb=sb), **bad})
    with pytest.raises(RuntimeError):
        ds3.ds3_gemm_mxfp4(a, sa, b, sb, c=bf16(4, 8), accumulate=True)      # (FP32 only)
    off, bg, sbg = i32(3), u8(2, 8, 128), i32(2, 8, 2)
    ds3.ds3_grouped_gemm_mxfp4(a, sa, off, bg, sbg)
    for bad in (dict(group_offsets=i32(2)), dict(group_offsets=off.long()), dict(b=bg[0]), dict(b=u8(2, 8, 256)[..., ::2]), dict(sa=i32(3, 2)),
                dict(sb=i32(2, 8, 3)), dict(sb=i32(2, 9, 2)[:, :8]), dict(c=bf16(3, 8))):
        with pytest.raises(ValueError):
            ds3.ds3_grouped_gemm_mxfp4(**{**dict(a=a, sa=sa, group_offsets=off, b=bg, sb=sbg), **bad})


def test_expert_order(ds3):
    ids = i32(6, 2)
    for bad in ((ids, 1024), (ids, -1), (ids, 4, -1), (ids, 2**40), (ids, 4, 2**31), (ids[0], 4)):
        with pytest.raises(ValueError):
            ds3.ds3_moe_sort(*bad)
    with pytest.raises(TypeError):
        ds3.ds3_moe_sort(ids.long(), 4)
    with pytest.raises(RuntimeError):
        ds3.ds3_moe_sort(i32(6, 65), 4)
    _, rows = ds3.ds3_moe_sort(ids, 1)
    x, w = bf16(6, 128), torch.ones((6, 2), device=DEV)
    q, s = ds3.ds3_moe_dispatch_quant_1x128(x, rows)
    calls = [(ds3.ds3_moe_dispatch, dict(x=x, row_of_slot=rows), bf16(12, 128)), (ds3.ds3_moe_dispatch_quant_1x128, dict(x=x, row_of_slot=rows), (q, s)),
             (ds3.ds3_moe_dispatch_quant_1x128_pow2, dict(x=x, row_of_slot=rows), (q, s)),
             (ds3.ds3_moe_dispatch_quant_mxfp4, dict(x=x, row_of_slot=rows), (u8(12, 64), i32(12, 1)))]
    for f, good, out in calls:
        assert f(**good, out=out) is out
        for bad in (dict(row_of_slot=rows[:5]), dict(row_of_slot=rows.long()), dict(row_of_slot=i32(6, 4)[:, ::2]), dict(rows=-1), dict(rows=11, out=out),
                    dict(x=x[:5]), dict(out=bf16(12, 64) if out is calls[0][2] else (out[0], out[1][:11]))):
            with pytest.raises(ValueError):
                f(**{**good, **bad})
        with pytest.raises(TypeError):
            f(**{**good, "x": x.half()})
    with pytest.raises(TypeError):
        ds3.ds3_moe_dispatch_quant_1x128(x, rows, out=[q, s])
    with pytest.raises(ValueError, match="overlap"):
        ds3.ds3_moe_dispatch_quant_1x128(x, rows, out=(q, s[:1].expand(12, 1)))
    y, out = bf16(12, 128), bf16(6, 128)
    for bad in (dict(weights=w.double()), dict(weights=w[:5]), dict(weights=torch.ones((6, 4), device=DEV)[:, ::2]), dict(out=bf16(5, 128)), dict(out=bf16(6, 64))):
        with pytest.raises(ValueError):
            ds3.ds3_moe_combine(**{**dict(y=y, row_of_slot=rows, weights=w), **bad})
    for bad in (dict(dout=bf16(5, 128)), dict(dout=bf16(6, 64)), dict(dy=bf16(11, 128)), dict(dy=y.float()), dict(weights=w.T)):
        with pytest.raises(ValueError):
            ds3.ds3_moe_combine_bwd(**{**dict(dout=out, y=y, row_of_slot=rows, weights=w), **bad})
    with pytest.raises(TypeError):
        ds3.ds3_moe_combine(y, rows, w, out_dtype=torch.float16)
