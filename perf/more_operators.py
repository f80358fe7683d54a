"""The norm in front of a layer, expert products on rows in 8 bits, and a whole layer for a few tokens, as measurable cases.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one pass: with
`own` false in elementary torch operations, with `own` true through the library's entry points.  `exact` gives the same
outputs from the definitions in 64 bits.

Definitions
  norm      h = x + delta, rounded to the type (without delta: x); n = h * weight / sqrt(mean of h^2 over the row + eps).
  rows8     the same with n in 8 bits: 32 neighbours of a row share a power of two, the least one with which the largest
            magnitude is at most 448; a value is the nearest e4m3 number times it, ties to the even code.
  backward  gradients of n and h -> gradient of x (and of delta, which is the same) and of the weight.
  experts8  rows r of expert e: y = W_down a, a = silu(W_gate x) * (W_up x) rounded to 8 bits as above; x in 8 bits, weights
            in 4 bits (groups of 32, a power of two each, times +-{0, .5, 1, 1.5, 2, 3, 4, 6}); shared experts see every token.
  layer     h and n as in norm (n rounded to the type; without a norm both are x); logits z = W_router n, rounded to fp32 once;
            each token's k experts of largest key (softmax: z; sigmoid: score + bias, from the best groups), gates c * score
            over their sum; out = h + sum of the shared experts + sum of gate * expert, each a silu-gated product of n.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                                           # values that share a scale, of rows and of weights
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)      # magnitudes of the eight 4-bit codes; codes 8..15 are their negatives
TOP8 = 448.0                                         # the largest e4m3 number
EPS = 1e-6
# d_model, experts, d_ffn, shared experts, top-k for text, for visual tokens: the layer shapes of the library's workloads
SHAPES = {
    "small": (1280, 64, 896, 2, 6, 3),
    "medium": (2048, 64, 1408, 2, 6, 3),
    "wide": (2048, 128, 768, 0, 8, 4),
}


def _named(name, c):
    return c if name is None else dict(c, name=name)


def _norm(name, op, T, d, dtype, delta):
    return _named(name, {"op": op, "T": T, "d": d, "dtype": dtype, "delta": delta})


def _experts(name, T, d, E, F, shared, k_text, k_visual):
    return _named(name, {"op": "experts8", "T": T, "d": d, "E": E, "F": F, "shared": shared, "k_text": k_text, "k_visual": k_visual})


def _layer(name, T, d, E, F, shared, k_text, k_visual, weights, norm, score="softmax", groups=1, topk_groups=1, scale=1.0):
    return _named(name, {"op": "layer", "T": T, "d": d, "E": E, "F": F, "shared": shared, "k_text": k_text, "k_visual": k_visual,
                         "weights": weights, "norm": norm, "score": score, "groups": groups, "topk_groups": topk_groups,
                         "scale": scale})


def listed():
    return [
        # One decoding step of eight conversations: nothing but latency.
        _norm("norm_8x2048", "norm", 8, 2048, "bf16", True),
        # A picture in fp32, odd sizes, the first norm of a stack (nothing to add yet).
        _norm("norm_1601x1288_f32", "norm", 1601, 1288, "f32", False),
        # The packed batch of several large pictures.
        _norm("norm_22016x2048", "norm", 22016, 2048, "bf16", True),
        # Rows in 8 bits, the last group of each shorter than the others.
        _norm("rows8_903x1288", "rows8", 903, 1288, "bf16", False),
        # A picture in 31 tiles on its way to products on 8-bit rows.
        _norm("rows8_8192x2048", "rows8", 8192, 2048, "bf16", True),
        # Training on one picture in fp32.
        _norm("backward_1600x1280_f32", "backward", 1600, 1280, "f32", True),
        # The training batch.
        _norm("backward_22016x2048", "backward", 22016, 2048, "bf16", True),
        # One small picture and a short question.
        _experts("experts8_416_small", 416, *SHAPES["small"]),
        # A picture in 31 tiles.
        _experts("experts8_8192_wide", 8192, *SHAPES["wide"]),
        # One token of one conversation on 4-bit weights: launches and latencies.
        _layer("layer_1_medium_4bit", 1, *SHAPES["medium"], "4bit", True),
        # A decoding step of eight conversations on bf16 weights, without a norm.
        _layer("layer_8_wide_bf16", 8, *SHAPES["wide"], "bf16", False),
        # The largest step, a router with sigmoid scores, a balance bias and groups.
        _layer("layer_16_medium_4bit_groups", 16, *SHAPES["medium"], "4bit", True, "sigmoid", 8, 4, 2.5),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "rows8", "backward", "experts8", "experts8", "layer", "layer"])
    if op in ("norm", "rows8", "backward"):
        d = 8 * _log_uniform(rng, 2, 1024)
        T = _log_uniform(rng, 1, 22016)
        T = min(T, 22016 * 2048 // d)
        return _norm(None, op, T, d, rng.choice(["bf16", "bf16", "f32"]) if T * d <= 1 << 24 else "bf16", rng.random() < 0.6)
    most = work(listed()[8])
    if op == "experts8":
        E = _log_uniform(rng, 4, 128)
        k_text = rng.randint(1, min(8, E))
        c = _experts(None, _log_uniform(rng, 1, 8192), 32 * _log_uniform(rng, 2, 64), E, 32 * _log_uniform(rng, 2, 44),
                     rng.randint(0, 2), k_text, rng.randint(0, k_text))
        while work(c)["flops"] > most["flops"] or work(c)["bytes"] > most["bytes"]:
            c["T"], c["F"] = max(1, c["T"] // 2), max(64, c["F"] // 64 * 32)
            c["E"] = max(c["k_text"], c["E"] * 3 // 4)
        return c
    groups = rng.choice([1, 1, 2, 4])
    E = groups * _log_uniform(rng, 8 // groups, 256 // groups)
    topk_groups = rng.randint(1, groups)
    k_text = rng.randint(1, min(8, topk_groups * (E // groups)))
    c = _layer(None, rng.randint(1, 16), 8 * _log_uniform(rng, 8, 256), E, 8 * _log_uniform(rng, 8, 176), rng.randint(0, 2), k_text,
               rng.randint(0, k_text), rng.choice(["bf16", "4bit"]), rng.random() < 0.6,
               "softmax" if groups == 1 and rng.random() < 0.6 else "sigmoid", groups, topk_groups, round(rng.uniform(0.5, 3.0), 2))
    most = work(listed()[11])
    while work(c)["bytes"] > most["bytes"]:
        c["F"] = max(64, c["F"] // 16 * 8)
        c["d"] = max(64, c["d"] // 16 * 8)
    return c


# ---------------------------------------------------------------------------------------------- the state of a program


def _visual_mask(T):
    """Visual tokens first, one text token in sixteen behind them."""
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[T - (T + 15) // 16:] = 0
    return mask


def _quantized(w):
    """What a checkpoint of 4-bit weights holds: codes, two to a byte (even positions in the low half), and scale bytes."""
    K = w.shape[-1]
    pad = -K % GROUP
    v = torch.nn.functional.pad(w.float(), (0, pad)).view(*w.shape[:-1], -1, GROUP)
    big = v.abs().amax(-1, keepdim=True)
    e = torch.where(big > 0, (torch.frexp(big).exponent - 3).clamp(-126, 127), torch.zeros_like(big, dtype=torch.int32))
    t = torch.ldexp(v, -e)
    a = t.abs()
    q = torch.where(a < 2, torch.round(a * 2), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4)).clamp(max=7.0)
    code = (q.to(torch.uint8) + (torch.signbit(t).to(torch.uint8) << 3)).reshape(*w.shape[:-1], K + pad)[..., :K]
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), (e[..., 0] + 127).to(torch.uint8)


class _State:
    pass


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    T, d = c["T"], c["d"]
    if c["op"] in ("norm", "rows8", "backward"):
        dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        # tokens of unequal size, a few dimensions that stand out
        s.x = (normal(T, d) * torch.exp(0.5 * normal(T, 1)) * (1.0 + 8.0 * (normal(d) > 2.5))).to(dtype)
        s.delta = (0.3 * normal(T, d)).to(dtype) if c["delta"] else None
        s.weight = (1.0 + 0.2 * normal(d)).to(dtype)
        if c["op"] == "backward":
            s.d_n, s.d_h = normal(T, d).to(dtype), s.delta
        return s
    E, F, shared, k = c["E"], c["F"], c["shared"], c["k_text"]
    weights = [(E, F, d), (E, F, d), (E, d, F)] + ([(shared, F, d), (shared, F, d), (shared, d, F)] if shared else [])
    weights = [(0.02 * normal(*shape)).to(torch.bfloat16) for shape in weights]
    if c["op"] == "layer":
        s.x = normal(T, d).to(torch.bfloat16)
        s.delta = (0.3 * normal(T, d)).to(torch.bfloat16) if c["norm"] else None
        s.weight = (1.0 + 0.2 * normal(d)).to(torch.bfloat16) if c["norm"] else None
        s.router = (normal(E, d) / math.sqrt(d)).to(torch.bfloat16)
        s.bias = 0.1 * normal(E) if c["score"] == "sigmoid" else None
        s.is_visual = _visual_mask(T)
        s.weights = [_quantized(w) for w in weights] if c["weights"] == "4bit" else weights
    else:
        s.codes, s.scales = _rows8(normal(T, d) * torch.exp(0.3 * normal(T, 1)))
        s.weights = [_quantized(w) for w in weights]
        # the rows of each expert, in the order the dispatch leaves them in: experts ascending, tokens ascending
        order = torch.argsort(normal(T, E) + 0.7 * normal(E), dim=1, descending=True)[:, :k]
        limit = torch.where(_visual_mask(T) > 0, c["k_visual"], k)
        taken = torch.arange(k, device="cuda")[None] < limit[:, None]
        chosen = torch.zeros(E, T, dtype=torch.bool, device="cuda")
        token = torch.arange(T, device="cuda")[:, None].expand(T, k)
        chosen[order[taken], token[taken]] = True
        s.expert_of_row, src = torch.nonzero(chosen, as_tuple=True)
        counts = chosen.sum(1)
        s.rows, s.most = int(counts.sum()), int(counts.max())
        s.offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s.perm_src = torch.zeros(max(T * k, 1), dtype=torch.int32, device="cuda")
        s.perm_src[:s.rows] = src.to(torch.int32)
    if own:
        from paper_2511_17885_amd import binding
        s.moe = binding.FMoE(d_model=d, n_experts=E, d_ffn=F, n_shared=shared, d_ffn_shared=F if shared else 0, k_text=k,
                             k_visual=c["k_visual"], dtype="bf16")
        if c["op"] == "experts8":
            s.moe.set_weights_quant_rows(*s.weights)
        elif c["weights"] == "4bit":
            s.moe.set_weights_quant(s.router, None, *s.weights)
        else:
            s.moe.set_weights(s.router, None, *s.weights)
        if c["op"] == "layer" and c["score"] == "sigmoid":
            s.params = binding.select_params("sigmoid", c["groups"], c["topk_groups"], 1, c["scale"])
        elif c["op"] == "layer":
            s.params = binding.select_params(gate_scale=c["scale"])
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms


def _rows8(v):
    """Rows in 8 bits: (codes [T, d] e4m3, scale bytes [T, 4 * ceil(d / 128)]: the last word's unused ones are 127)."""
    T, d = v.shape
    p = torch.nn.functional.pad(v, (0, -d % GROUP)).view(T, -1, GROUP)
    big = p.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(big)                              # big = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875)
    e = torch.where(big > 0, e.clamp(-126, 127), torch.zeros_like(e))
    t = torch.ldexp(p, -e)
    step = torch.ldexp(torch.ones_like(t), (torch.frexp(t).exponent - 1).clamp(min=-6) - 3)
    codes = (torch.round(t / step) * step).view(T, -1)[:, :d].to(torch.float8_e4m3fn)
    scales = torch.nn.functional.pad(e[..., 0] + 127, (0, -e.shape[1] % 4), value=127).to(torch.uint8)
    return codes, scales


def _of_rows8(codes, scales, dtype):
    d = codes.shape[1]
    power = torch.ldexp(torch.ones((), dtype=dtype, device=codes.device), scales.int() - 127)
    return codes.to(dtype) * power.repeat_interleave(GROUP, dim=1)[:, :d]


def _plain_norm(s, dtype):
    """(h rounded to the type, n in `dtype`)."""
    h = s.x if s.delta is None else (s.x.to(dtype) + s.delta.to(dtype)).to(s.x.dtype)
    v = h.to(dtype)
    return h, v * (1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)) * s.weight.to(dtype)


def _plain_backward(s):
    h, g = s.x.float(), s.d_n.float()
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    c = h * r
    gw = g * s.weight.float()
    d_x = r * (gw - c * (gw * c).mean(1, keepdim=True))
    if s.d_h is not None:
        d_x = d_x + s.d_h.float()
    return [d_x.to(s.x.dtype), (g * c).sum(0)]


def _dense(w, dtype):
    if torch.is_tensor(w):
        return w.to(dtype)
    codes, scales = w
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=dtype, device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    scale = torch.ldexp(torch.ones((), dtype=dtype, device=codes.device), scales.int() - 127)
    return grid[code.int()] * scale.repeat_interleave(GROUP, dim=-1)[..., :code.shape[-1]]


def _at(w, e):
    return w[e] if torch.is_tensor(w) else (w[0][e], w[1][e])


def _swiglu(x, gate, up, down, eight):
    """x [g, r, d] times the weights of its group [g, ., .]."""
    g = torch.bmm(x, gate.transpose(1, 2).contiguous())
    a = g / (1.0 + torch.exp(-g)) * torch.bmm(x, up.transpose(1, 2).contiguous())
    if eight:
        a = _of_rows8(*_rows8(a.flatten(0, 1)), a.dtype).view(a.shape)
    return torch.bmm(a, down.transpose(1, 2).contiguous())


def _plain_experts8(s):
    c = s.case
    f32, E, d = torch.float32, c["E"], c["d"]
    x, src, e = _of_rows8(s.codes, s.scales, f32), s.perm_src[:s.rows].long(), s.expert_of_row
    if s.rows == 0:
        y = x.new_zeros(0, d)
    elif s.rows <= E:   # fewer rows than experts: each row with the weights of its own
        y = _swiglu(x[src][:, None], *[_dense(_at(w, e), f32) for w in s.weights[:3]], True)[:, 0]
    else:               # all experts side by side, as many rows each as the fullest has
        at = torch.arange(s.rows, device=x.device) - s.offsets[:-1].long()[e]
        padded = x.new_zeros(E, s.most, d)
        padded[e, at] = x[src]
        y = _swiglu(padded, *[_dense(w, f32) for w in s.weights[:3]], True)[e, at]
    y = y.to(torch.bfloat16)
    if not c["shared"]:
        return [y]
    many = x[None].expand(c["shared"], -1, -1).contiguous()
    return [y, _swiglu(many, *[_dense(w, f32) for w in s.weights[3:]], True).to(torch.bfloat16)]


def _choice(s, z):
    """(idx [T, k], -1 in empty places; gate in 64 bits) from fp32 logits z; keys in 64 bits, as neighbours decide."""
    c, z = s.case, z.double()
    E, G = c["E"], c["groups"]
    key = z
    if c["score"] == "sigmoid":
        key = 1.0 / (1.0 + torch.exp(-z)) + s.bias.double()
        if G > 1:
            top = torch.sort(key.view(-1, G, E // G), dim=-1, descending=True).values[..., :2].sum(-1)
            stay = torch.sort(top, dim=1, descending=True, stable=True).indices[:, :c["topk_groups"]]
            group = torch.zeros_like(top, dtype=torch.bool).scatter_(1, stay, True)
            key = torch.where(group.repeat_interleave(E // G, dim=1), key, torch.full_like(key, -math.inf))
    at = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :c["k_text"]]
    limit = torch.where(s.is_visual > 0, c["k_visual"], c["k_text"])[:, None]
    there = torch.arange(c["k_text"], device=z.device)[None] < limit
    score = torch.gather(z, 1, at)
    score = 1.0 / (1.0 + torch.exp(-score)) if c["score"] == "sigmoid" else torch.exp(score - z.max(1, keepdim=True).values)
    score = torch.where(there, score, torch.zeros_like(score))
    gate = c["scale"] * score / score.sum(1, keepdim=True).clamp(min=1e-300)
    return torch.where(there, at, torch.full_like(at, -1)).to(torch.int32), gate


def _plain_layer(s):
    c, f32 = s.case, torch.float32
    h, n = (s.x, s.x) if s.weight is None else _plain_norm(s, torch.float64)   # in 64 bits: n is rounded before it decides
    n = n.to(torch.bfloat16)
    idx, gate = _choice(s, (n.double() @ s.router.double().T).float())
    e = idx.clamp(min=0).long().flatten()
    x = n.to(f32).repeat_interleave(c["k_text"], dim=0)[:, None]
    y = _swiglu(x, *[_dense(_at(w, e), f32) for w in s.weights[:3]], False).view(c["T"], c["k_text"], c["d"])
    out = h.to(f32) + (gate.to(f32)[..., None] * y).sum(1)
    if c["shared"]:
        many = n.to(f32)[None].expand(c["shared"], -1, -1).contiguous()
        out = out + _swiglu(many, *[_dense(w, f32) for w in s.weights[3:]], False).sum(0)
    return [out.to(torch.bfloat16), idx, gate.to(f32)]


# ------------------------------------------------------------------------------------------------------ one pass


def _own(s):
    from paper_2511_17885_amd import binding
    c = s.case
    if c["op"] == "norm":
        return list(binding.rms_norm(s.x, s.weight, EPS, delta=s.delta))
    if c["op"] == "rows8":
        h, codes, scales = binding.rms_norm_quant(s.x, s.weight, EPS, delta=s.delta)
        return [h, codes, scales]
    if c["op"] == "backward":
        return list(binding.rms_norm_backward(s.x, s.weight, EPS, s.d_n, d_h=s.d_h))
    if c["op"] == "layer":
        norm = None if s.weight is None else (s.weight, EPS)
        return list(s.moe.layer_decode(s.x, s.is_visual, norm=norm, delta=s.delta, params=s.params, select_bias=s.bias))
    y, y_shared = s.moe.expert_ffn_quant_rows(s.codes, s.scales, None, c["T"], s.offsets, s.perm_src)
    return [y[:s.rows]] if y_shared is None else [y[:s.rows], y_shared]


def run(state):
    if own:
        return _own(state)
    op = state.case["op"]
    if op == "norm":
        h, n = _plain_norm(state, torch.float32)
        return [h, n.to(state.x.dtype)]
    if op == "rows8":
        h, n = _plain_norm(state, torch.float64)   # in 64 bits: values next to a border of two codes
        return [h, *_rows8(n)]
    if op == "backward":
        return _plain_backward(state)
    return _plain_layer(state) if op == "layer" else _plain_experts8(state)


# -------------------------------------------------------------------------------------------- what a pass cannot avoid


def work(case):
    c = case
    T, d = c["T"], c["d"]
    if c["op"] in ("norm", "rows8", "backward"):
        size = 2 if c["dtype"] == "bf16" else 4
        delta = 1 if c["delta"] else 0
        if c["op"] == "backward":
            return {"bytes": (3 + delta) * T * d * size + d * (size + 4), "flops": 14 * T * d}
        out = T * d * size if c["op"] == "norm" else T * d + 4 * T * -(-d // 128)
        return {"bytes": (2 + delta) * T * d * size + d * size + out, "flops": (5 if c["op"] == "norm" else 9) * T * d}
    E, F, shared, k = c["E"], c["F"], c["shared"], c["k_text"]
    text = (T + 15) // 16
    rows = text * k + (T - text) * c["k_visual"]
    touched = E * (1.0 - (1.0 - 1.0 / E) ** rows) + shared
    products = 6 * (rows + shared * T) * d * F
    if c["op"] == "layer":
        size = 2 if c["weights"] == "bf16" else 17 / 32
        return {"bytes": touched * 3 * F * d * size + E * d * 2 + T * d * 2 * (3 if c["norm"] else 2) + T * k * 8,
                "flops": products + 2 * T * E * d}
    return {"bytes": touched * 3 * F * d * 17 / 32 + T * d * 33 / 32 + (rows + shared * T) * d * 2 + rows * 4, "flops": products}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits


def _nearest8(v):
    """v rounded to 8 bits, by the list of all e4m3 numbers."""
    T, d = v.shape
    p = torch.nn.functional.pad(v, (0, -d % GROUP)).unflatten(1, (-1, GROUP))
    big = p.abs().amax(2, keepdim=True)
    power = torch.floor(torch.log2(big / TOP8))
    power = torch.where(torch.exp2(power) * TOP8 < big, power + 1, power)
    power = torch.where(torch.exp2(power - 1) * TOP8 >= big, power - 1, power)
    power = torch.where(big > 0, power.clamp(-126, 127), torch.zeros_like(power))
    table = torch.arange(127, dtype=torch.uint8, device=v.device).view(torch.float8_e4m3fn).double()
    middle = (table[1:] + table[:-1]) / 2
    a = p.abs() / torch.exp2(power)
    low, high = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)   # apart only on a middle
    code = torch.sign(p) * table[torch.where(low % 2 == 0, low, high)]
    return code.flatten(1)[:, :d], power[..., 0]


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    c = case
    if c["op"] in ("norm", "rows8", "layer"):
        h = s.x.double() if s.delta is None else (s.x.double() + s.delta.double()).to(s.x.dtype).double()
        if s.weight is not None:
            n = h / torch.sqrt(h.square().sum(1, keepdim=True) / c["d"] + EPS) * s.weight.double()
        if c["op"] == "norm":
            return [h, n]
        if c["op"] == "rows8":
            return [h, _nearest8(n)[0], None]
    if c["op"] == "backward":
        # by differentiation of the definition, some rows at a time
        d_x, d_w = [], 0.0
        for i in range(0, c["T"], 4096):
            h = s.x[i:i + 4096].double().requires_grad_()
            w = s.weight.double().requires_grad_()
            n = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * w
            total = (n * s.d_n[i:i + 4096].double()).sum()
            if s.d_h is not None:
                total = total + (h * s.d_h[i:i + 4096].double()).sum()
            g = torch.autograd.grad(total, (h, w))
            d_x.append(g[0])
            d_w = d_w + g[1]
        return [torch.cat(d_x), d_w]

    def ffn(x, w, at, eight):
        gate, up, down = (_dense(_at(m, at), torch.float64) for m in w)
        a = torch.nn.functional.silu(x @ gate.T) * (x @ up.T)
        if eight and a.shape[0]:
            code, power = _nearest8(a)
            a = code * torch.exp2(power).repeat_interleave(GROUP, dim=1)[:, :a.shape[1]]
        return a @ down.T

    if c["op"] == "layer":
        n = h if s.weight is None else n.to(torch.bfloat16).double()
        idx, gate = _choice(s, (n @ s.router.double().T).float())
        out = h.clone()
        for e in range(c["shared"]):
            out = out + ffn(n, s.weights[3:], e, False)
        for e in sorted(set(idx.flatten().tolist()) - {-1}):
            out = out + (gate * (idx == e)).sum(1, keepdim=True) * ffn(n, s.weights[:3], e, False)
        return [out, None, gate]
    offsets, src = s.offsets.tolist(), s.perm_src[:s.rows].long()
    x = _of_rows8(s.codes, s.scales, torch.float64)
    y = torch.cat([ffn(x[src[offsets[e]:offsets[e + 1]]], s.weights[:3], e, True) for e in range(c["E"])])
    return [y] if not c["shared"] else [y, torch.stack([ffn(x, s.weights[3:], e, True) for e in range(c["shared"])])]
