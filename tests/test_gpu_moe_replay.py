"""An expert layer captured once and replayed for other choices: the groups' sizes, which the host never sees, change from replay
to replay, from even loads to all tokens at one expert and to none here."""
import pytest
import torch

from tests._gpu_util import DEV, announce

pytestmark = pytest.mark.gpu


# tokens, choices a token, experts in all, experts here, first, width, products' columns; the last sorts in three launches
@pytest.mark.parametrize("T,K,E,G,first,H,N", [(6, 2, 8, 4, 2, 256, 72), (700, 4, 16, 16, 0, 384, 520), (3000, 4, 32, 16, 8, 512, 2056), (18_000, 8, 64, 48, 0, 128, 136)])
def test_other_choices(ds3, T, K, E, G, first, H, N):
    announce(f"replayed expert layer, {T}x{K} of {E}, {G} here, {H} -> {N}")
    gen = torch.Generator(device=DEV).manual_seed(T)
    x, dout = (torch.randn((T, c), generator=gen, device=DEV).bfloat16() for c in (H, N))
    w = torch.rand((T, K), generator=gen, device=DEV)
    q, s = ds3.ds3_quant_mxfp4(torch.randn((G * N, H), generator=gen, device=DEV), k_major_scales=False)
    kept = q.contiguous().view(G, N, H // 2), s.view(G, N, H // 128)
    ids = torch.randint(0, E, (T, K), dtype=torch.int32, generator=gen, device=DEV)
    room = T * K

    def buffers():
        z = lambda r, c, t: torch.zeros((r, c), dtype=t, device=DEV)  # noqa: E731
        return (z(room, H // 2, torch.uint8), z(room, H // 128, torch.int32)), z(room, N, torch.bfloat16), z(room, N, torch.bfloat16)

    def step(bufs):
        off, rows = ds3.ds3_moe_sort(ids, G, first_expert=first)
        a = ds3.ds3_moe_dispatch_quant_mxfp4(x, rows, out=bufs[0])
        y = ds3.ds3_grouped_gemm_mxfp4(*a, off, *kept, c=bufs[1])
        return off, rows, y, ds3.ds3_moe_combine(y, rows, w), *ds3.ds3_moe_combine_bwd(dout, y, rows, w, dy=bufs[2])

    bufs = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(bufs)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(bufs)
    for i in range(6):
        ids.copy_([torch.randint(0, E, (T, K), generator=gen, device=DEV), torch.full((T, K), first + G - 1, device=DEV),
                   torch.full((T, K), -1, device=DEV), torch.randint(first, first + 2, (T, K), generator=gen, device=DEV),
                   torch.randint(-3, 2 * E, (T, K), generator=gen, device=DEV), torch.randint(0, E, (T, K), generator=gen, device=DEV)][i])
        x.normal_(generator=gen)
        fresh = buffers()
        want = step(fresh)
        for b in (*bufs[0], *bufs[1:]):
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, v) for o, v in zip(outs, want)), i
        n = int(outs[0][-1])
        assert n == int((outs[1] >= 0).sum()) and not outs[2][n:].any() and not outs[4][n:].any()
        torch.randn((64, 64), device=DEV).sum().item()
