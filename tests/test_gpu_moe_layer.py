"""The expert layer as it is used: choices sorted, tokens dispatched with the cast on the way, the experts' products,
combine, and the gradients; eager, on another stream and captured into a graph."""
import numpy as np
import pytest
import torch

from oracle import ds3_oracle as orc
from oracle import mx_moe_oracle as mx
from tests._gpu_util import DEV, announce
from tests.test_gpu_mxfp4 import bytes_of

pytestmark = pytest.mark.gpu

T, K, E, G, FIRST, H, I = 150, 4, 16, 8, 4, 512, 256


def setup(seed):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(E)[:K] for _ in range(T)]).astype(np.int32)
    ids[T - 7 :] = -1
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).to(DEV).bfloat16()
    w = torch.from_numpy(rng.random((T, K)).astype(np.float32)).to(DEV)
    w13 = torch.from_numpy((rng.standard_normal((G, 2 * I, H)) * 0.05).astype(np.float32)).to(DEV).bfloat16()
    w2 = torch.from_numpy((rng.standard_normal((G, H, I)) * 0.05).astype(np.float32)).to(DEV).bfloat16()
    return torch.from_numpy(ids).to(DEV), x, w, w13, w2


def per_expert(q, s, g):
    """One quantized [G * N][K] weight as [G][N] of codes and of scale words, K-block-major within an expert."""
    n = q.shape[0] // g
    return q.contiguous().view(g, n, -1), s.contiguous().view(g, n, -1).transpose(1, 2).contiguous().transpose(1, 2)


def test_four_bit_layer_step_by_step(ds3):
    announce("expert layer, MXFP4")
    ids, x, w, w13, w2 = setup(1)
    off, rows = ds3.ds3_moe_sort(ids, G, first_expert=FIRST)
    woff, wrows = mx.moe_sort(ids.cpu().numpy(), G, FIRST)
    assert np.array_equal(off.cpu().numpy(), woff) and np.array_equal(rows.cpu().numpy(), wrows)
    total = T * K
    q, s = ds3.ds3_moe_dispatch_quant_mxfp4(x, rows, rows=total)
    n = int(off[-1])
    tok = np.zeros(n, int)
    tok[wrows[wrows >= 0]] = np.nonzero(wrows >= 0)[0]
    wq, ws = mx.quant_mxfp4(x.float().cpu().numpy()[tok])
    assert np.array_equal(q[:n].cpu().numpy(), wq) and np.array_equal(bytes_of(s[:n]), ws)
    kept13, kept2 = per_expert(*ds3.ds3_quant_mxfp4(w13.view(-1, H)), G), per_expert(*ds3.ds3_quant_mxfp4(w2.view(-1, I)), G)

    def product(a_q, a_s, kept, got, k):
        for g in range(G):
            at = slice(int(woff[g]), int(woff[g + 1]))
            a, b = mx.dequant_mxfp4(a_q[at].cpu().numpy(), bytes_of(a_s[at])), mx.dequant_mxfp4(kept[0][g].cpu().numpy(), bytes_of(kept[1][g]))
            want, near = a @ b.T, (k / 128 + 4) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
            assert (np.abs(got[at].double().cpu().numpy() - want) <= near + 2.0 ** -8 * (np.abs(want) + near)).all()

    h = ds3.ds3_grouped_gemm_mxfp4(q, s, off, *kept13)
    product(q, s, kept13, h, H)
    act = ds3.ds3_swiglu(h)
    qa, sa = ds3.ds3_quant_mxfp4(act)
    wq, ws = mx.quant_mxfp4(act[:n].float().cpu().numpy())
    assert np.array_equal(qa[:n].cpu().numpy(), wq) and np.array_equal(bytes_of(sa[:n]), ws)
    y = ds3.ds3_grouped_gemm_mxfp4(qa, sa, off, *kept2)
    product(qa, sa, kept2, y, I)
    out = ds3.ds3_moe_combine(y, rows, w)
    hy, hw = np.nan_to_num(y.double().cpu().numpy()), w.cpu().numpy()
    want = mx.combine(hy, wrows, hw)
    near = 1.01 * K * 2.0 ** -24 * mx.combine(np.abs(hy), wrows, hw)
    assert (np.abs(out.double().cpu().numpy() - want) <= near + 2.0 ** -8 * (np.abs(want) + near)).all()
    assert not out[T - 7 :].any()


def test_eight_bit_layer_reads_the_dispatched_codes(ds3):
    """The FP8 grouped product on codes and scales that dispatch wrote is that on quantized rows in expert order."""
    ids, x, w, w13, _ = setup(2)
    off, rows = ds3.ds3_moe_sort(ids, G, first_expert=FIRST)
    n = int(off[-1])
    qw, sw = ds3.ds3_quant_w_128x128(w13.view(-1, H))
    qw, sw = qw.view(G, 2 * I, H), sw.view(G, 2 * I // 128, H // 128)
    q, s = ds3.ds3_moe_dispatch_quant_1x128(x, rows, rows=n)
    sorted_x = ds3.ds3_moe_dispatch(x, rows, rows=n)
    q0, s0 = ds3.ds3_quant_act_1x128(sorted_x)
    assert torch.equal(q, q0) and torch.equal(s, s0)
    qr, sr = orc.quant_act_1x128(sorted_x.float().cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), qr) and np.array_equal(s.cpu().numpy(), sr)
    assert torch.equal(ds3.ds3_grouped_gemm_fp8_bs(q, s, off, qw, sw), ds3.ds3_grouped_gemm_fp8_bs(q0, s0, off, qw, sw))


def test_weight_gradients_of_a_dense_layer(ds3):
    """Forward, input gradient and weight gradient of one layer in 4 bits: each operand quantized along what is contracted."""
    rng = np.random.default_rng(3)
    t, n, k = 256, 384, 512
    x = torch.from_numpy(rng.standard_normal((t, k)).astype(np.float32)).to(DEV).bfloat16()
    w = torch.from_numpy((rng.standard_normal((n, k)) * 0.05).astype(np.float32)).to(DEV).bfloat16()
    dy = torch.from_numpy(rng.standard_normal((t, n)).astype(np.float32)).to(DEV).bfloat16()
    y = ds3.ds3_gemm_mxfp4(*ds3.ds3_quant_mxfp4(x), *ds3.ds3_quant_mxfp4(w), out_dtype=torch.float32)
    dx = ds3.ds3_gemm_mxfp4(*ds3.ds3_quant_mxfp4(dy), *ds3.ds3_quant_mxfp4_t(w), out_dtype=torch.float32)
    dw = ds3.ds3_gemm_mxfp4(*ds3.ds3_quant_mxfp4_t(dy), *ds3.ds3_quant_mxfp4_t(x), out_dtype=torch.float32)
    hx, hw, hd = (a.float().cpu().numpy() for a in (x, w, dy))
    for got, a, b, c in ((y, hx, hw, k), (dx, hd, hw.T, n), (dw, hd.T, hx.T, t)):
        va, vb = (mx.dequant_mxfp4(*mx.quant_mxfp4(np.ascontiguousarray(m))) for m in (a, b))
        assert (np.abs(got.double().cpu().numpy() - va @ vb.T) <= (c / 128 + 4) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)).all()


def step(ds3, ids, x, w, kept13, kept2, dout, bufs):
    off, rows = ds3.ds3_moe_sort(ids, G, first_expert=FIRST)
    q, s = ds3.ds3_moe_dispatch_quant_mxfp4(x, rows, out=bufs["in"])
    h = ds3.ds3_grouped_gemm_mxfp4(q, s, off, *kept13, c=bufs["h"])
    y = ds3.ds3_grouped_gemm_mxfp4(*ds3.ds3_quant_mxfp4(ds3.ds3_swiglu(h)), off, *kept2, c=bufs["y"])
    out = ds3.ds3_moe_combine(y, rows, w)
    dy, dw = ds3.ds3_moe_combine_bwd(dout, y, rows, w, dy=bufs["dy"])
    q8, s8 = ds3.ds3_moe_dispatch_quant_1x128(x, rows, out=bufs["in8"])
    dx = ds3.ds3_moe_combine(ds3.ds3_moe_dispatch(x, rows, out=bufs["rows"]), rows)
    return off, rows, q, s, h, y, out, dy, dw, q8, s8, dx


def buffers():
    z = lambda c, t: torch.zeros((T * K, c), dtype=t, device=DEV)  # noqa: E731
    return {"in": (z(H // 2, torch.uint8), z(H // 128, torch.int32)), "h": z(2 * I, torch.bfloat16), "y": z(H, torch.bfloat16),
            "dy": z(H, torch.bfloat16), "rows": z(H, torch.bfloat16), "in8": (z(H, torch.uint8), z(H // 128, torch.float32))}


def test_captured_and_on_another_stream(ds3):
    """Replays between eager work, each against the eager step's results bit for bit; two graphs in flight on two streams
    share nothing that either writes."""
    ids, x, w, w13, w2 = setup(4)
    kept13, kept2 = per_expert(*ds3.ds3_quant_mxfp4(w13.view(-1, H)), G), per_expert(*ds3.ds3_quant_mxfp4(w2.view(-1, I)), G)
    dout = torch.randn((T, H), device=DEV).bfloat16()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs, outs, xs = [], [], [x.clone(), x.clone()]
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(side[i]):
            bufs = buffers()
            step(ds3, ids, xs[i], w, kept13, kept2, dout, bufs)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side[i]):
            outs.append(step(ds3, ids, xs[i], w, kept13, kept2, dout, bufs))
        graphs.append((g, bufs))
    for it in range(4):
        want = []
        for i in range(2):
            xs[i].normal_()
            want.append([t.clone() for t in step(ds3, ids, xs[i], w, kept13, kept2, dout, buffers())])
        _ = float((x.float() @ x.float().t()).sum())
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(side[i]):
                graphs[i][0].replay()
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(outs[i], want[i]):
                assert torch.equal(a, b), (it, i)
