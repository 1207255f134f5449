"""Operators around and below the expert products, as training and serving programs call them: rows taken into expert
order and back, and the 4-bit (MXFP4) quantizers and products.

A case's `kind` is one of
  dispatch  the chosen experts of a batch sorted, and the tokens' rows written in expert order.
              tokens, top_k, experts   tokens, experts a token, experts in all;  hidden: width of a row
              local, first             experts held here: [first, first + local); choices of others leave no row
              padded                   the last sixteenth of the batch is padding, which chose nothing
              to                       "bf16" / "f32": rows as they are; "fp8" / "fp8_pow2": quantized 1x128 on the way;
                                       "mxfp4": quantized to 4 bits on the way
  combine   experts' outputs summed per token with the router's weights (`weights`; without: the gradient of dispatch),
              and with `backward` the gradients of the experts' outputs and of the weights
  quantise  a matrix to MXFP4 and its values back; `along`: "rows", "columns" (written transposed: the operand of the
              other gradient) or "both"
  linear    input quantized, product with a weight kept in MXFP4
  wgrad     both operands quantized along the tokens, dW += dY^T X in FP32
  experts   rows in expert order quantized, each expert's product with its own MXFP4 weight
MXFP4: groups of 32 elements share a power of two (the smallest with which none exceeds 6, a byte with bias 127; 127 for a
group of zeros), elements are E2M1 (0, .5, 1, 1.5, 2, 3, 4, 6) rounded to nearest even, two in a byte, the first in the low
half; the bytes of four groups are one 32-bit word, words stored by K-block, then row.
"""
from __future__ import annotations

import random

import torch

own = False

DEVICE = "cuda"
HIDDEN, DENSE_INTER, MOE_INTER, N_ROUTED, TOP_K = 7168, 18432, 2048, 256, 8
LARGEST = 4096 * DENSE_INTER * HIDDEN                    # m * n * k of the largest product


def _dispatch(tokens, top_k, experts, local, hidden, to, first=0, padded=False):
    return dict(kind="dispatch", tokens=tokens, top_k=top_k, experts=experts, local=local, first=first, hidden=hidden, to=to,
                padded=padded)


def _combine(tokens, top_k, experts, local, hidden, type="bf16", weights=True, backward=False, first=0, padded=False):
    return dict(kind="combine", tokens=tokens, top_k=top_k, experts=experts, local=local, first=first, hidden=hidden,
                type=type, weights=weights, backward=backward, padded=padded)


def _quantise(rows, cols, along, x="bf16"):
    return dict(kind="quantise", rows=rows, cols=cols, along=along, x=x)


def _linear(m, n, k, out="bf16"):
    return dict(kind="linear", m=m, n=n, k=k, out=out)


def _wgrad(tokens, n, k):
    return dict(kind="wgrad", tokens=tokens, n=n, k=k)


def _experts(rows, experts, n, k, out="bf16"):
    return dict(kind="experts", rows=rows, experts=experts, n=n, k=k, out=out)


def listed():
    return [
        # a decode step with every expert at hand: launches and host work
        dict(_dispatch(4, TOP_K, N_ROUTED, N_ROUTED, HIDDEN, "bf16"), name="dispatch_decode"),
        # a training batch, one GPU's 32 of 256 experts, cast to FP8 on the way to the grouped product
        dict(_dispatch(8192, TOP_K, N_ROUTED, 32, HIDDEN, "fp8", first=64), name="dispatch_train_fp8"),
        # a small model's ragged, padded batch, all experts here, cast to 4 bits
        dict(_dispatch(1333, 6, 64, 64, 1536, "mxfp4", padded=True), name="dispatch_ragged_mxfp4"),
        # the way back of a decode batch of the whole model, FP32 sums of an odd batch of narrow rows with gradients, ...
        dict(_combine(33, 2, 16, 16, 1000, "f32", backward=True, padded=True), name="combine_small_f32"),
        # ... and of the training batch above with its gradients
        dict(_combine(8192, TOP_K, N_ROUTED, 32, HIDDEN, backward=True, first=64), name="combine_train"),
        # a small FP32 activation of odd height
        dict(_quantise(257, 1024, "rows", "f32"), name="quantise_small_f32"),
        # a layer's new weights after an optimizer step, for the forward pass and for the input's gradient
        dict(_quantise(HIDDEN, 4096, "both"), name="quantise_weights"),
        # a decode step of the dense FFN: the weights' stream
        dict(_linear(16, DENSE_INTER, HIDDEN), name="linear_decode"),
        # the dense FFN over a training batch: the largest product
        dict(_linear(4096, DENSE_INTER, HIDDEN), name="linear_ffn_up"),
        # gradient of the MLA query projection's weight, odd width
        dict(_wgrad(2048, 1536, 1000), name="wgrad_odd"),
        # one GPU's experts: gate | up of a training batch, down of a decode batch (4 rows an expert)
        dict(_experts(8192, 32, 2 * MOE_INTER, HIDDEN), name="experts_train"),
        dict(_experts(128, 32, HIDDEN, MOE_INTER), name="experts_decode"),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng: random.Random):
    kind = rng.choice(["dispatch", "dispatch", "combine", "combine", "quantise", "linear", "linear", "wgrad", "experts", "experts"])
    if kind in ("dispatch", "combine"):
        experts, hidden = rng.choice([8, 16, 60, 64, 160, 256]), 8 * _log(rng, 16, HIDDEN // 8)
        parts = rng.choice([1, 1, 2, 4])
        local = max(1, experts // parts)
        at = dict(tokens=_log(rng, 1, 8192), top_k=rng.randint(1, 8), experts=experts, local=local, hidden=hidden,
                  first=local * rng.randrange(experts // local), padded=rng.random() < 0.3)
        if at["tokens"] * at["top_k"] * hidden > 8192 * HIDDEN * 2:
            at["tokens"] = max(1, 8192 * HIDDEN * 2 // (at["top_k"] * hidden))
        if kind == "dispatch":
            return _dispatch(to=rng.choice(["bf16", "f32", "fp8", "fp8_pow2", "mxfp4", "mxfp4"]), **at)
        weights = rng.random() < 0.75
        return _combine(type=rng.choice(["bf16", "bf16", "f32"]), weights=weights, backward=weights and rng.random() < 0.6, **at)
    if kind == "quantise":
        return _quantise(_log(rng, 1, 8192), 8 * _log(rng, 4, 896), rng.choice(["rows", "columns", "both"]), rng.choice(["bf16", "bf16", "f32"]))
    while True:
        n, k, out = _log(rng, 64, 24576), 128 * _log(rng, 1, 144), rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.5:
            n = n // 64 * 64
        if kind == "linear":
            m = _log(rng, 1, 8192)
            if m * n * k <= LARGEST and n * k <= DENSE_INTER * HIDDEN:
                return _linear(m, n, k, out)
        elif kind == "wgrad":
            m, n, k = 128 * _log(rng, 1, 64), 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)
            if m * n * k <= LARGEST // 4:
                return _wgrad(m, n, k)
        else:
            g, m = rng.choice([4, 8, 16, 32]), _log(rng, 8, 8192)
            n = min(n, 8192)
            if m * n * k <= LARGEST // 2 and g * n * k <= 32 * 2 * MOE_INTER * HIDDEN:
                return _experts(m, g, n, k, out)


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _randn(gen, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEVICE).mul_(std).to(dtype)


def _activations(gen, m, k, dtype=torch.bfloat16):
    """N(0, 1) with one channel in a hundred 50 times as large."""
    x = torch.randn((m, k), generator=gen, device=DEVICE)
    cols = torch.randperm(k, generator=gen, device=DEVICE)[: max(1, k // 100)]
    x[:, cols] *= 50.0
    return x.to(dtype)


def _capacity(case):
    """Rows that the program keeps room for: half as many again as even loads bring, and at most every choice."""
    every = case["tokens"] * case["top_k"]
    return min(every, every * case["local"] * 3 // (case["experts"] * 2) + 256)


def _chosen(gen, case):
    """Distinct experts a token, uneven loads (a quarter of the mean either way and more); -1 in padding."""
    t, e = case["tokens"], case["experts"]
    load = 0.3 * torch.randn(e, generator=gen, device=DEVICE)
    u = torch.rand((t, e), generator=gen, device=DEVICE).clamp_(1e-6, 1 - 1e-6)
    ids = (load - (-u.log()).log()).topk(case["top_k"], dim=1).indices.int()
    if case["padded"]:
        ids[t - t // 16 :] = -1
    return ids.contiguous()


# ---- MXFP4 in elementary operations ---------------------------------------------------

def _groups(x):
    """[rows][cols] as [rows][cols / 32 rounded up to whole words][32], padded with zeros, in 32 bits."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 32)


def _mx(x):
    """(codes 0 .. 15, one a byte [rows][groups][32]; exponents with their bias [rows][groups]) of groups along a row."""
    g = _groups(x)
    m, e = torch.frexp(g.abs().amax(2))                  # amax = m 2^e, m in [1/2, 1);  6 = 3/4 2^3
    e = torch.where(m == 0, 0, torch.where(m <= 0.75, e - 3, e - 2)).clamp(-127, 127)
    y = torch.ldexp(g, -e[..., None])
    a = y.abs()
    code = (a > 0.25).byte()
    for border, tie_up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if tie_up else (a > border)
    return code + torch.signbit(y).byte() * 8, (e + 127).to(torch.uint8)


def _values(code, e):
    """What codes [rows][groups][32] and exponents [rows][groups] stand for, [rows][groups * 32] in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return torch.ldexp(table[code.int()], (e.int() - 127)[..., None]).flatten(1)


def _words(e):
    """Scale bytes [rows][groups] as 32-bit words, logical [rows][groups / 4], stored by K-block."""
    return e.clone(memory_format=torch.contiguous_format).view(torch.int32).t().contiguous().t()


def _packed(code):
    c = code.flatten(1)
    return c[:, 0::2] | (c[:, 1::2] << 4)


def _unpacked(q, s):
    """Values of packed codes [rows][K / 2] and scale words [rows][K / 128], in 32 bits."""
    c = torch.stack((q & 15, q >> 4), -1).view(q.shape[0], -1, 32)
    return _values(c, s.clone(memory_format=torch.contiguous_format).view(torch.uint8))


def _kept(gen, n, k):
    """A weight as a program keeps it: (packed codes, scale words)."""
    code, e = _mx(_randn(gen, (n, k), 0.02))
    return _packed(code), _words(e)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind in ("dispatch", "combine"):
        s["ids"], cap, h = _chosen(gen, case), _capacity(case), case["hidden"]
        zeros = lambda cols, t: torch.zeros((cap, cols), dtype=t, device=DEVICE)  # noqa: E731  (rows nobody chose stay so)
        if kind == "dispatch":
            to = case["to"]
            s["x"] = _activations(gen, case["tokens"], h, torch.float32 if to == "f32" else torch.bfloat16)
            kb = (h + 127) // 128
            if to in _TYPES:
                s["out"] = zeros(h, _TYPES[to])
            elif to == "mxfp4":
                s["out"] = zeros(-(-h // 32) * 16, torch.uint8)[:, : h // 2], torch.zeros((kb, cap), dtype=torch.int32, device=DEVICE).t()
            else:
                s["out"] = zeros(-(-h // 16) * 16, torch.uint8)[:, :h], torch.zeros((kb, cap), device=DEVICE).t()
            return s
        t = _TYPES[case["type"]]
        s["rows"] = _sorted(s["ids"], case)[1]
        s["y"] = _randn(gen, (cap, h), 1.0, t)
        w = torch.rand((case["tokens"], case["top_k"]), generator=gen, device=DEVICE) + 0.05
        s["w"] = 2.5 * w / w.sum(1, keepdim=True) if case["weights"] else None
        if case["backward"]:
            s["dout"], s["dy"] = _randn(gen, (case["tokens"], h), 0.01, t), zeros(h, t)
        return s
    if kind == "quantise":
        x = _TYPES[case["x"]]
        s["x"] = _activations(gen, case["rows"], case["cols"], x) if case["along"] == "rows" else _randn(gen, (case["rows"], case["cols"]), 0.02, x)
        return s
    n, k = case["n"], case["k"]
    if kind == "wgrad":
        s["dy"], s["x"] = _randn(gen, (case["tokens"], n), 0.01), _activations(gen, case["tokens"], k)
        s["dw"] = torch.zeros((n, -(-k // 8) * 8), device=DEVICE)[:, :k]
        return s
    if kind == "linear":
        s["x"], s["w"] = _activations(gen, case["m"], k), _kept(gen, n, k)
        return s
    g, rows, rng = case["experts"], case["rows"], random.Random(seed)
    sizes, loads = [0] * g, [rng.lognormvariate(0.0, 0.3) for _ in range(g)]
    for e in rng.choices(range(g), loads, k=rows):
        sizes[e] += 1
    s["off"] = torch.tensor([sum(sizes[:e]) for e in range(g + 1)], dtype=torch.int32, device=DEVICE)
    s["most"] = max(sizes)
    cap = rows + rows // 8                               # the rows behind the last group belong to nobody
    s["x"] = _activations(gen, cap, k)
    q, sc = zip(*(_kept(gen, n, k) for _ in range(g)))
    s["w"] = torch.stack(q), torch.stack([t.t() for t in sc]).transpose(1, 2)
    s["c"] = torch.zeros((cap, -(-n // 8) * 8), dtype=_TYPES[case["out"]], device=DEVICE)[:, :n]
    return s


# ---- plain forms -------------------------------------------------------------------------

def _sorted(ids, case):
    """(row offsets of the experts held here, row of every choice or -1): by expert, then token, then choice."""
    e = ids.flatten().long() - case["first"]
    one = torch.nn.functional.pad((e[:, None] == torch.arange(case["local"], device=ids.device)).int(), (1, 0))
    before = one.cumsum(0, dtype=torch.int32)
    off = before[-1].cumsum(0, dtype=torch.int32)
    here = (e >= 0) & (e < case["local"])
    at = e.clamp(0, case["local"] - 1)
    rank = before.gather(1, at[:, None] + 1)[:, 0] - 1
    return off, torch.where(here, off[at] + rank, -1).int().view_as(ids)


def _spread(values, rows, cap):
    """`values` [tokens][...] written to the rows of their choices, zeros elsewhere."""
    out = values.new_zeros((cap + 1, *values.shape[1:]))
    at = torch.where((rows < 0) | (rows >= cap), cap, rows).long()
    out[at] = values[:, None].expand(*rows.shape, *values.shape[1:])
    return out[:cap]


def _fp8(x, pow2):
    """1x128 tiles: (E4M3 values, scales)."""
    rows, cols = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 128)
    amax = g.abs().amax(2)
    most = torch.full_like(amax, 448.0)                  # (a division by a number may be a product with its reciprocal)
    if pow2:
        m, e = torch.frexp(amax / most)
        sc = torch.ldexp(torch.ones_like(amax), torch.where(m == 0.5, e - 1, e))
        r = 1.0 / sc
    else:
        sc, r = amax / most, most / amax
    sc, r = torch.where(amax == 0, 1.0, sc), torch.where(amax == 0, 0.0, r)
    return (g * r[..., None]).flatten(1)[:, :cols].to(torch.float8_e4m3fn), sc


def _plain_dispatch(s, case):
    off, rows = _sorted(s["ids"], case)
    x, cap, to = s["x"], _capacity(case), case["to"]
    if to in _TYPES:
        return off, rows, _spread(x, rows, cap)
    if to == "mxfp4":
        code, e = _mx(x)
        q, sc = _values(code, e)[:, : x.shape[1]].bfloat16(), _words(e)
    else:
        q, sc = _fp8(x, to == "fp8_pow2")
        return off, rows, _spread(q.view(torch.uint8), rows, cap).view(torch.float8_e4m3fn), _spread(sc, rows, cap)
    return off, rows, _spread(q, rows, cap), _spread(sc, rows, cap)


def _plain_combine(s, case):
    y, rows, w = s["y"], s["rows"], s["w"]
    cap = y.shape[0]
    here = (rows >= 0) & (rows < cap)
    at = rows.clamp(0, cap - 1).long()
    picked = torch.where(here[..., None], y[at].float(), 0.0)
    out = (picked if w is None else picked * w[..., None]).sum(1).to(y.dtype)
    if not case["backward"]:
        return out
    d = s["dout"].float()
    dy = torch.zeros((cap + 1, y.shape[1]), device=y.device)
    dy[torch.where(here, at, cap)] = w[..., None] * d[:, None]
    return out, dy[:cap].to(y.dtype), (picked * d[:, None]).sum(2)


def _plain_quantise(s, case):
    got = []
    for x in ([s["x"]] if case["along"] != "columns" else []) + ([s["x"].t()] if case["along"] != "rows" else []):
        code, e = _mx(x)
        got += [_values(code, e)[:, : x.shape[1]].bfloat16(), _words(e)]
    return got


def _plain_experts(s, case):
    k, cap, off, most = case["k"], s["x"].shape[0], s["off"].long(), max(1, s["most"])
    x = _values(*_mx(s["x"]))[:, :k]
    at = off[:-1, None] + torch.arange(most, device=x.device)            # rows of each expert, padded to the most
    valid = at < off[1:, None]
    q, sc = s["w"]
    w = _unpacked(q.flatten(0, 1), sc.flatten(0, 1)).view(*q.shape[:2], k)
    y = torch.bmm(x[at.clamp(max=cap - 1)], w.transpose(1, 2).contiguous())
    c = torch.zeros((cap + 1, case["n"]), device=x.device)
    c[torch.where(valid, at, cap)] = y
    return c[:cap].to(s["c"].dtype)


def _plain(s, case):
    kind = case["kind"]
    if kind == "dispatch":
        return _plain_dispatch(s, case)
    if kind == "combine":
        return _plain_combine(s, case)
    if kind == "quantise":
        return _plain_quantise(s, case)
    if kind == "linear":
        return (_values(*_mx(s["x"])) @ _unpacked(*s["w"]).t()).to(_TYPES[case["out"]])
    if kind == "wgrad":
        s["dw"] += _values(*_mx(s["dy"].t())) @ _values(*_mx(s["x"].t())).t()
        return s["dw"]
    return _plain_experts(s, case)


# ---- the framework's calls ---------------------------------------------------------------

def _own_dispatch(ds3, s, case):
    off, rows = ds3.ds3_moe_sort(s["ids"], case["local"], first_expert=case["first"])
    to = case["to"]
    if to in _TYPES:
        return off, rows, ds3.ds3_moe_dispatch(s["x"], rows, out=s["out"])
    if to == "mxfp4":
        q, sc = ds3.ds3_moe_dispatch_quant_mxfp4(s["x"], rows, out=s["out"])
        return off, rows, ds3.ds3_dequant_mxfp4(q, sc), sc
    call = ds3.ds3_moe_dispatch_quant_1x128_pow2 if to == "fp8_pow2" else ds3.ds3_moe_dispatch_quant_1x128
    q, sc = call(s["x"], rows, out=s["out"])
    return off, rows, q.view(torch.float8_e4m3fn), sc


def _own_combine(ds3, s, case):
    out = ds3.ds3_moe_combine(s["y"], s["rows"], s["w"])
    if not case["backward"]:
        return out
    dy, dw = ds3.ds3_moe_combine_bwd(s["dout"], s["y"], s["rows"], s["w"], dy=s["dy"])
    return out, dy, dw


def _own_quantise(ds3, s, case):
    got = []
    for call in ([ds3.ds3_quant_mxfp4] if case["along"] != "columns" else []) + ([ds3.ds3_quant_mxfp4_t] if case["along"] != "rows" else []):
        q, sc = call(s["x"])
        got += [ds3.ds3_dequant_mxfp4(q, sc, cols=case["cols"] if call is ds3.ds3_quant_mxfp4 else case["rows"]), sc]
    return got


def _own(s, case):
    import paper_2412_19437_amd as ds3

    kind = case["kind"]
    if kind == "dispatch":
        return _own_dispatch(ds3, s, case)
    if kind == "combine":
        return _own_combine(ds3, s, case)
    if kind == "quantise":
        return _own_quantise(ds3, s, case)
    if kind == "linear":
        return ds3.ds3_gemm_mxfp4(*ds3.ds3_quant_mxfp4(s["x"]), *s["w"], out_dtype=_TYPES[case["out"]])
    if kind == "wgrad":
        return ds3.ds3_gemm_mxfp4(*ds3.ds3_quant_mxfp4_t(s["dy"]), *ds3.ds3_quant_mxfp4_t(s["x"]), c=s["dw"], accumulate=True)
    return ds3.ds3_grouped_gemm_mxfp4(*ds3.ds3_quant_mxfp4(s["x"]), s["off"], *s["w"], c=s["c"])


def run(state):
    if own:
        return _own(state, state["case"])
    return _plain(state, state["case"])


# ---- definitions in 64 bits --------------------------------------------------------------

def _even(y, steps):
    """y rounded to the nearest multiple of `steps`, ties to the even one."""
    return torch.round(y / steps) * steps


def _exact_mx(x):
    """Values of x [rows][cols] in MXFP4 along its rows, by the definition."""
    rows, cols = x.shape
    g = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    amax = g.abs().amax(2, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(amax == 0, 6.0, amax) / 6.0)).clamp(-127, 127)
    e = torch.where(torch.exp2(e - 1) * 6.0 >= amax, e - 1, e)           # (a logarithm may be off next to a whole number)
    scale = torch.where(amax == 0, 1.0, torch.exp2(torch.where(torch.exp2(e) * 6.0 < amax, e + 1, e).clamp(-127, 127)))
    y = g / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (_even(y, step) * scale).view(rows, -1)[:, :cols]


def _exact_kept(q, sc):
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=q.device)
    c = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.float64, device=q.device)
    for half, n in ((0, q & 15), (1, q >> 4)):
        c[:, half::2] = value[(n & 7).int()] * (1.0 - 2.0 * (n >> 3).double())
    e = torch.stack([(sc.contiguous() >> (8 * i)) & 255 for i in range(4)], -1).flatten(1)
    return c * torch.exp2(e.double() - 127.0).repeat_interleave(32, 1)[:, : c.shape[1]]


def _exact_fp8(x, pow2):
    rows, cols = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 128)
    amax = g.abs().amax(2, keepdim=True)
    if pow2:
        s = torch.exp2(torch.ceil(torch.log2(torch.where(amax == 0, 448.0, amax).double() / 448.0)))
        r = (1.0 / s).float()
    else:                                                # the factors and the product are 32-bit numbers by definition
        s, r = (amax / torch.full_like(amax, 448.0)).double(), torch.full_like(amax, 448.0) / amax
    y = torch.where(amax == 0, 0.0, g * r).double()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0**-6))) - 3.0)
    return _even(y, step).clamp(-448, 448).view(rows, -1)[:, :cols], torch.where(amax == 0, 1.0, s)[..., 0]


def _exact_rows(s, case):
    """(row, token, choice) of every choice that has a row, in lists made one by one on the host."""
    ids, cap = s["ids"].cpu().tolist(), _capacity(case)
    of = [[] for _ in range(case["local"])]
    for t, row in enumerate(ids):
        for j, e in enumerate(row):
            if case["first"] <= e < case["first"] + case["local"]:
                of[e - case["first"]].append((t, j))
    flat = [p for e in of for p in e][:cap]
    return torch.tensor([p[0] for p in flat], dtype=torch.long, device=DEVICE), torch.tensor([p[1] for p in flat], dtype=torch.long, device=DEVICE)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "dispatch":
        x, to, (tok, _) = s["x"], case["to"], _exact_rows(s, case)
        v, sc = {"fp8": lambda: _exact_fp8(x, False), "fp8_pow2": lambda: _exact_fp8(x, True), "mxfp4": lambda: (_exact_mx(x), None)}.get(to, lambda: (x.double(), None))()
        full = lambda v: torch.cat((v[tok], v.new_zeros((_capacity(case) - len(tok), v.shape[1]))))  # noqa: E731
        return (None, None, full(v)) + (() if to in _TYPES else (None if sc is None else full(sc),))
    if kind == "combine":
        tok, j = _exact_rows(s, case)
        y = s["y"][: len(tok)].double()
        w = torch.ones(len(tok), dtype=torch.float64, device=DEVICE) if s["w"] is None else s["w"][tok, j].double()
        out = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device=DEVICE).index_add_(0, tok, y * w[:, None])
        if not case["backward"]:
            return out
        d = s["dout"][tok].double()
        dy, dw = torch.zeros(s["y"].shape, dtype=torch.float64, device=DEVICE), torch.zeros(s["w"].shape, dtype=torch.float64, device=DEVICE)
        dy[: len(tok)] = d * w[:, None]
        dw[tok, j] = (d * y).sum(1)
        return out, dy, dw
    if kind == "quantise":
        got = []
        if case["along"] != "columns":
            got += [_exact_mx(s["x"]), None]
        if case["along"] != "rows":
            got += [_exact_mx(s["x"].t()), None]
        return got
    if kind == "linear":
        return _exact_mx(s["x"]) @ _exact_kept(*s["w"]).t()
    if kind == "wgrad":
        return _exact_mx(s["dy"].t()) @ _exact_mx(s["x"].t()).t()
    off, x = s["off"].tolist(), _exact_mx(s["x"])
    c = torch.zeros((x.shape[0], case["n"]), dtype=torch.float64, device=DEVICE)
    for e in range(case["experts"]):
        c[off[e] : off[e + 1]] = x[off[e] : off[e + 1]] @ _exact_kept(s["w"][0][e], s["w"][1][e]).t()
    return c


def _mx_bytes(rows, cols):
    return rows * cols // 2 + rows * -(-cols // 32)


def work(case):
    kind = case["kind"]
    if kind in ("dispatch", "combine"):
        t, h, held = case["tokens"], case["hidden"], case["local"] / case["experts"]
        if case["padded"]:
            t -= t // 16
        rows = t * case["top_k"] * held                  # rows here, and tokens that have any
        some = t * (1 - (1 - held) ** case["top_k"])
        index = 4 * t * case["top_k"]
        if kind == "dispatch":
            es = 4 if case["to"] == "f32" else 2
            row = {"bf16": 2 * h, "f32": 4 * h, "mxfp4": 2 * h + -(-h // 32)}.get(case["to"], h + 4 * -(-h // 128))
            return {"bytes": some * h * es + rows * row + 2 * index, "flops": rows * h}
        es = 2 if case["type"] == "bf16" else 4
        moved = rows * h * es + case["tokens"] * h * es + 2 * index
        if case["backward"]:
            moved += (rows + some) * h * es + index      # the experts' outputs are read once for both
        return {"bytes": moved, "flops": rows * h * (5 if case["backward"] else 2)}
    if kind == "quantise":
        r, c = case["rows"], case["cols"]
        out = sum(2 * r * c + a * -(-b // 32) for a, b, on in ((r, c, "rows"), (c, r, "columns")) if case["along"] in (on, "both"))
        return {"bytes": r * c * (2 if case["x"] == "bf16" else 4) + out, "flops": 3 * r * c}
    n, k = case["n"], case["k"]
    if kind == "wgrad":
        return {"bytes": case["tokens"] * (n + k) * 2 + n * k * 8, "flops": 2 * case["tokens"] * n * k}
    m, out = case["m"] if kind == "linear" else case["rows"], 2 if case["out"] == "bf16" else 4
    weights = 1 if kind == "linear" else min(m, case["experts"])
    return {"bytes": m * k * 2 + weights * _mx_bytes(n, k) + m * n * out, "flops": 2 * m * n * k}
