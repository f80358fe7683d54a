"""Routing by scores, groups and a balance bias, its gradient, and expert products with 4-bit weights, as measurable cases.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one pass: with
`own` false in elementary torch operations, with `own` true through the library's entry points.  `exact` gives the same
outputs from the definitions in 64 bits.

Definitions
  select    logits z [T, E].  Experts with z = -inf or NaN are masked, z = +inf counts as the largest fp32 number.
            score: softmax over the unmasked experts, or sigmoid.  Key: score + bias in 64 bits; without a bias the
            order of z itself.  The experts form G groups of neighbours; a group's score is its largest key, or the
            sum of its two largest; the best `topk_groups` stay.  A token lists its k largest keys (ties: lower index).
            Gates: c times the softmax over the list of log(score) (renormalised), or c times the score.
  backward  gradients of gates and scores -> gradient of z for the list that was chosen.
  quantize  groups of 32 values along a row share a power of two; a value is one of +-{0, .5, 1, 1.5, 2, 3, 4, 6} times
            it, the nearest, ties to the even code.  The values are returned, as the quantized weights stand for them.
  experts   rows r of expert e: y = W_down (silu(W_gate x) * (W_up x)) with such weights; shared experts see every token.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                                          # weights that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)      # magnitudes of the eight codes; codes 8..15 are their negatives
# d_model, experts, d_ffn, shared experts, top-k for text: the layer shapes of the library's workloads
SHAPES = {
    "small": (1280, 64, 896, 2, 6),
    "medium": (2048, 64, 1408, 2, 6),
    "wide": (2048, 128, 768, 0, 8),
}
FLT_MAX = torch.finfo(torch.float32).max


def _select(name, op, T, E, k_text, k_visual, *, dtype="f32", score="softmax", bias=False, groups=1, topk_groups=1,
            group_score=0, renormalize=True, scale=1.0, scores=False):
    c = {"op": op, "T": T, "E": E, "k_text": k_text, "k_visual": k_visual, "dtype": dtype, "score": score, "bias": bias,
         "groups": groups, "topk_groups": topk_groups, "group_score": group_score, "renormalize": renormalize,
         "scale": scale, "scores": scores}
    return c if name is None else dict(c, name=name)


def _quantize(name, rows, K, dtype, saturate):
    c = {"op": "quantize", "rows": rows, "K": K, "dtype": dtype, "saturate": saturate}
    return c if name is None else dict(c, name=name)


def _experts(name, T, d, E, F, shared, k_text, k_visual):
    c = {"op": "experts", "T": T, "d": d, "E": E, "F": F, "shared": shared, "k_text": k_text, "k_visual": k_visual}
    return c if name is None else dict(c, name=name)


def _experts_of(name, shape, T, k_visual):
    d, E, F, shared, k_text = SHAPES[shape]
    return _experts(name, T, d, E, F, shared, k_text, k_visual)


def listed():
    return [
        # One decoding step of eight conversations: nothing but latency.
        _select("select_8x64", "select", 8, 64, 6, 3),
        # A large picture with logits kept in bf16; the scores are wanted for the pruning that follows.
        _select("select_4097x128_bf16_scores", "select", 4097, 128, 8, 4, dtype="bf16", scores=True),
        # A training batch, 256 experts in eight groups, a balance bias on sigmoid scores.
        _select("select_22016x256_groups", "select", 22016, 256, 8, 8, score="sigmoid", bias=True, groups=8, topk_groups=4,
                group_score=1, scale=2.5),
        # One picture, softmax scores with the gradient of a balance loss on them.
        _select("backward_1600x64_scores", "backward", 1600, 64, 6, 3, scores=True),
        # The training batch: gates only.
        _select("backward_22016x256", "backward", 22016, 256, 8, 8, score="sigmoid", bias=True, groups=8, topk_groups=4,
                group_score=1, scale=2.5),
        # One expert matrix, odd sizes, from fp32 master weights.
        _quantize("quantize_903x1288_f32", 903, 1288, "f32", False),
        # The gate weights of a whole layer.
        _quantize("quantize_layer", 64 * 1408, 2048, "bf16", True),
        # One token of one conversation: eight experts' weights stream past one row.
        _experts_of("experts_1_medium", "medium", 1, 3),
        # A decoding step of eight conversations.
        _experts_of("experts_8_medium", "medium", 8, 3),
        # One small picture and a short question, odd sizes.
        _experts_of("experts_416_small", "small", 416, 3),
        # A large picture.
        _experts_of("experts_4096_medium", "medium", 4096, 3),
        # A picture in 31 tiles.
        _experts_of("experts_8192_wide", "wide", 8192, 4),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "select", "backward", "quantize", "experts", "experts", "experts"])
    if op in ("select", "backward"):
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _log_uniform(rng, max(2, 8 // groups), 256 // groups)
        topk_groups = rng.randint(1, groups)
        most = min(16, topk_groups * (E // groups))
        k_text = rng.randint(1, most)
        return _select(None, op, _log_uniform(rng, 1, 22016), E, k_text, rng.randint(0, k_text),
                       dtype=rng.choice(["f32", "f32", "bf16"]), score=rng.choice(["softmax", "sigmoid"]),
                       bias=rng.random() < 0.5, groups=groups, topk_groups=topk_groups, group_score=rng.randint(0, 1),
                       renormalize=rng.random() < 0.7, scale=round(rng.uniform(0.5, 3.0), 2), scores=rng.random() < 0.5)
    if op == "quantize":
        return _quantize(None, _log_uniform(rng, 1, 64 * 1024), 8 * _log_uniform(rng, 4, 256), rng.choice(["f32", "bf16"]),
                         rng.random() < 0.5)
    E = _log_uniform(rng, 4, 128)
    k_text = rng.randint(1, min(8, E))
    shared = rng.randint(0, 2)
    d, F, T = 8 * _log_uniform(rng, 16, 256), 8 * _log_uniform(rng, 16, 176), _log_uniform(rng, 1, 8192)
    c = _experts(None, T, d, E, F, shared, k_text, rng.randint(0, k_text))
    most = work(dict(listed()[-1]))
    while work(c)["flops"] > most["flops"] or work(c)["bytes"] > most["bytes"]:
        c["T"], c["F"] = max(1, c["T"] // 2), max(128, c["F"] // 16 * 8)
        c["E"] = max(c["k_text"], c["E"] * 3 // 4)
    return c


# ---------------------------------------------------------------------------------------------- the state of a program


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _visual_mask(T):
    """Visual tokens first, one text token in sixteen behind them."""
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[T - (T + 15) // 16:] = 0
    return mask


def _quantized(w, saturate=True):
    """What a checkpoint of 4-bit weights holds: codes, two to a byte (even positions in the low half), and scale bytes."""
    value, scale = _nearest(w, saturate)
    grid = torch.tensor(GRID, device=w.device)
    code = torch.searchsorted(grid, value.abs()).to(torch.uint8) + (torch.signbit(value).to(torch.uint8) << 3)
    exponent = (torch.frexp(scale).exponent + 126).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), exponent


class _State:
    pass


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    if c["op"] in ("select", "backward"):
        T, E = c["T"], c["E"]
        # logits as a router makes them: experts of unequal popularity
        s.logits = (normal(T, E) + 0.7 * normal(E)).to(_dtype(c))
        s.is_visual = _visual_mask(T)
        s.bias = 0.1 * normal(E) if c["bias"] else None
        if c["op"] == "backward":
            _, s.idx, _ = _plain_select(s)
            s.d_gate = normal(*s.idx.shape)
            s.d_scores = normal(T, E) / E if c["scores"] else None
        if own:
            from paper_2511_17885_amd import binding
            s.moe = binding.FMoE(d_model=64, n_experts=E, d_ffn=64, k_text=c["k_text"], k_visual=c["k_visual"], dtype="bf16",
                                 renormalize=c["renormalize"])
            s.params = binding.select_params(score=c["score"], n_groups=c["groups"], topk_groups=c["topk_groups"],
                                             group_score=c["group_score"], gate_scale=c["scale"])
        return s
    if c["op"] == "quantize":
        # rows of unequal size, as the columns of a trained matrix have
        s.w = (0.02 * normal(c["rows"], c["K"]) * torch.exp(0.5 * normal(c["rows"], 1))).to(_dtype(c))
        return s
    T, d, E, F, shared, k = c["T"], c["d"], c["E"], c["F"], c["shared"], c["k_text"]
    s.x = normal(T, d).to(torch.bfloat16)
    weights = [(E, F, d), (E, F, d), (E, d, F)] + ([(shared, F, d), (shared, F, d), (shared, d, F)] if shared else [])
    s.weights = [_quantized((0.02 * normal(*shape)).to(torch.bfloat16)) for shape in weights]
    # the rows of each expert, in the order the dispatch leaves them in: experts ascending, tokens ascending
    order = torch.argsort(normal(T, E) + 0.7 * normal(E), dim=1, descending=True)[:, :k]
    limit = torch.where(_visual_mask(T) > 0, c["k_visual"], k)
    listed_ = torch.arange(k, device="cuda")[None] < limit[:, None]
    chosen = torch.zeros(E, T, dtype=torch.bool, device="cuda")
    token = torch.arange(T, device="cuda")[:, None].expand(T, k)
    chosen[order[listed_], token[listed_]] = True
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
        s.moe.set_weights_quant(torch.zeros(E, d, dtype=torch.bfloat16, device="cuda"), None, *s.weights)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms


def _two_largest(key):
    """Sum of the two largest keys of each group; masked ones (-inf) add nothing beside another."""
    top = torch.sort(key, dim=-1, descending=True).values[..., :2]
    if top.shape[-1] == 1:
        return top[..., 0]
    return top[..., 0] + torch.where(top[..., 1] > -math.inf, top[..., 1], torch.zeros_like(top[..., 1]))


def _logits(s, dtype):
    z = s.logits.to(dtype).clamp(max=FLT_MAX)
    return torch.where(z > -math.inf, z, torch.full_like(z, -math.inf))


def _scores(z, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    return e / e.sum(1, keepdim=True).clamp(min=torch.finfo(z.dtype).tiny)


def _log_sigmoid(z):
    return torch.where(z > 0, -torch.log1p(torch.exp(-z.abs())), z - torch.log1p(torch.exp(-z.abs())))


def _share(z, idx, score):
    """Softmax over the list of log(score); 0 in empty places."""
    there = idx >= 0
    l = torch.gather(z, 1, idx.clamp(min=0).long())
    l = _log_sigmoid(l) if score == "sigmoid" else l
    l = torch.where(there, l, torch.full_like(l, -math.inf))
    top = l.max(1, keepdim=True).values
    e = torch.where(there, torch.exp(l - torch.where(top > -math.inf, top, torch.zeros_like(top))), torch.zeros_like(l))
    return e / e.sum(1, keepdim=True).clamp(min=torch.finfo(z.dtype).tiny)


def _plain_select(s):
    c = s.case
    E, G, K = c["E"], c["groups"], max(c["k_text"], c["k_visual"])
    z = _logits(s, torch.float32)
    z64 = z.double()
    score64 = _scores(z64, c["score"])   # in 64 bits: keys next to each other decide
    by_key = s.bias is not None
    key = score64 + s.bias.double() if by_key else z64
    masked = torch.full_like(key, -math.inf)
    key = torch.where((z64 > -math.inf) & (key > -math.inf), key, masked)
    if G > 1:
        if c["group_score"] == 1:
            best = _two_largest((key if by_key else torch.where(z64 > -math.inf, score64, masked)).view(-1, G, E // G))
        else:
            best = key.view(-1, G, E // G).max(-1).values
        stay = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["topk_groups"]]
        group = torch.zeros_like(best, dtype=torch.bool).scatter_(1, stay, True)
        key = torch.where(group[:, :, None].expand(-1, G, E // G).reshape(key.shape), key, masked)
    top = torch.sort(key, dim=1, descending=True, stable=True)
    k = torch.where(s.is_visual > 0, c["k_visual"], c["k_text"])[:, None]
    there = (torch.arange(K, device=z.device)[None] < k) & (top.values[:, :K] > -math.inf)
    idx = torch.where(there, top.indices[:, :K], torch.full_like(top.indices[:, :K], -1)).to(torch.int32)
    score = _scores(z, c["score"])
    if c["renormalize"]:
        gate = _share(z, idx, c["score"])
    else:
        gate = torch.where(there, torch.gather(score, 1, idx.clamp(min=0).long()), torch.zeros((), device=z.device))
    return (score if c["scores"] else None), idx, gate * c["scale"]


def _plain_backward(s):
    c = s.case
    z = _logits(s, torch.float32)
    there = s.idx >= 0
    at = s.idx.clamp(min=0).long()
    a = torch.where(there, s.d_gate, torch.zeros_like(s.d_gate)) * c["scale"]
    score = _scores(z, c["score"])
    d_score = s.d_scores if s.d_scores is not None else torch.zeros_like(z)
    d_z = torch.zeros_like(z)
    if c["renormalize"]:
        p = _share(z, s.idx, c["score"])
        d_l = p * (a - (p * a).sum(1, keepdim=True))
        if c["score"] == "sigmoid":
            d_l = d_l / (1.0 + torch.exp(torch.gather(z, 1, at)))
        d_z = d_z.scatter_add(1, at, torch.where(there, d_l, torch.zeros_like(d_l)))
    else:
        d_score = d_score.scatter_add(1, at, a)
    if c["score"] == "sigmoid":
        d_z = d_z + score * (1.0 / (1.0 + torch.exp(z))) * d_score
    else:
        d_z = d_z + score * (d_score - (score * d_score).sum(1, keepdim=True))
    return torch.where(z > -math.inf, d_z, torch.zeros_like(d_z)).to(s.logits.dtype)


def _nearest(w, saturate):
    """(value / scale on the grid of the codes, scale of each group) of the rows of w."""
    K = w.shape[-1]
    pad = -K % GROUP
    v = torch.nn.functional.pad(w.float(), (0, pad)).view(*w.shape[:-1], -1, GROUP)
    big = v.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(big)                        # big = m * 2^e, m in [0.5, 1)
    e = e - 3 if saturate else e - 3 + (m > 0.75)  # 2^floor(log2 big) / 4; or the least power with big <= 6 of it
    e = torch.where(big > 0, e.clamp(-126, 127), torch.zeros_like(e))
    scale = torch.ldexp(torch.ones_like(big), e)
    t = v / scale
    a = t.abs()
    q = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2)).clamp(max=6.0)
    return torch.copysign(q, t).reshape(*w.shape[:-1], K + pad)[..., :K], scale[..., 0]


def _plain_quantize(s):
    q, scale = _nearest(s.w, s.case["saturate"])
    return (q * scale.repeat_interleave(GROUP, dim=-1)[..., :q.shape[-1]]).to(s.w.dtype)


def _dense(codes, scales, dtype):
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=dtype, device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    scale = torch.ldexp(torch.ones((), dtype=dtype, device=codes.device), scales.int() - 127)
    return grid[code.int()] * scale.repeat_interleave(GROUP, dim=-1)[..., :code.shape[-1]]


def _swiglu(x, gate, up, down):
    """x [g, r, d] times the weights of its group [g, ., .]."""
    g = torch.bmm(x, gate.transpose(1, 2).contiguous())
    u = torch.bmm(x, up.transpose(1, 2).contiguous())
    return torch.bmm(g / (1.0 + torch.exp(-g)) * u, down.transpose(1, 2).contiguous())


def _plain_experts(s):
    c = s.case
    f32, E, d = torch.float32, c["E"], c["d"]
    x, src, e = s.x.to(f32), s.perm_src[:s.rows].long(), s.expert_of_row
    if s.rows == 0:
        y = x.new_zeros(0, d)
    elif s.rows <= E:   # fewer rows than experts: each row with the weights of its own
        y = _swiglu(x[src][:, None], *[_dense(codes[e], scales[e], f32) for codes, scales in s.weights[:3]])[:, 0]
    else:               # all experts side by side, as many rows each as the fullest has
        at = torch.arange(s.rows, device=x.device) - s.offsets[:-1].long()[e]
        padded = x.new_zeros(E, s.most, d)
        padded[e, at] = x[src]
        y = _swiglu(padded, *[_dense(codes, scales, f32) for codes, scales in s.weights[:3]])[e, at]
    y = y.to(torch.bfloat16)
    if not c["shared"]:
        return [y]
    many = x[None].expand(c["shared"], -1, -1).contiguous()
    return [y, _swiglu(many, *[_dense(codes, scales, f32) for codes, scales in s.weights[3:]]).to(torch.bfloat16)]


# ------------------------------------------------------------------------------------------------------ one pass


def _own(s):
    from paper_2511_17885_amd import binding
    c = s.case
    if c["op"] == "select":
        return list(s.moe.select_experts(s.params, s.logits, s.is_visual, select_bias=s.bias, want_scores=c["scores"]))
    if c["op"] == "backward":
        return [s.moe.select_experts_backward(s.params, s.logits, s.idx, s.d_gate, d_scores=s.d_scores)]
    if c["op"] == "quantize":
        return [binding.dequantize_weights(*binding.quantize_weights(s.w, saturate=c["saturate"]), dtype=s.w.dtype)]
    y, y_shared = s.moe.expert_ffn(s.x, None, c["T"], s.offsets, s.perm_src)
    return [y[:s.rows]] if y_shared is None else [y[:s.rows], y_shared]


def run(state):
    if own:
        return _own(state)
    op = state.case["op"]
    if op == "select":
        return list(_plain_select(state))
    if op == "backward":
        return [_plain_backward(state)]
    if op == "quantize":
        return [_plain_quantize(state)]
    return _plain_experts(state)


# -------------------------------------------------------------------------------------------- what a pass cannot avoid


def work(case):
    c = case
    if c["op"] in ("select", "backward"):
        T, E, K = c["T"], c["E"], max(c["k_text"], c["k_visual"])
        size = 2 if c["dtype"] == "bf16" else 4
        if c["op"] == "select":
            return {"bytes": T * E * size + T + T * K * 8 + (T * E * 4 if c["scores"] else 0) + (E * 4 if c["bias"] else 0),
                    "flops": 8 * T * E}
        dense = c["scores"] or not (c["renormalize"] or c["score"] == "sigmoid")   # needs every logit
        read = T * E * size if dense else T * K * size
        return {"bytes": read + T * K * 8 + (T * E * 4 if c["scores"] else 0) + T * E * size, "flops": 8 * T * (E if dense else K)}
    if c["op"] == "quantize":
        n, size = c["rows"] * c["K"], 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * size * 2 + 2 * (n // 2 + c["rows"] * -(-c["K"] // GROUP)), "flops": 4 * n}
    T, d, E, F, shared, k = c["T"], c["d"], c["E"], c["F"], c["shared"], c["k_text"]
    text = (T + 15) // 16
    rows = text * k + (T - text) * c["k_visual"]
    touched = E * (1.0 - (1.0 - 1.0 / E) ** rows) + shared
    return {"bytes": touched * 3 * F * d * 17 / 32 + T * d * 2 + (rows + shared * T) * d * 2 + rows * 4,
            "flops": 6 * (rows + shared * T) * d * F}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    c = case
    if c["op"] in ("select", "backward"):
        z = s.logits.double()
        z = torch.where(z == math.inf, torch.full_like(z, FLT_MAX), z)
        out = z.isnan() | (z == -math.inf)
        l = torch.nn.functional.logsigmoid(z) if c["score"] == "sigmoid" else torch.log_softmax(z.masked_fill(out, -math.inf), 1)
        l = l.masked_fill(out, -math.inf).nan_to_num(nan=-math.inf, neginf=-math.inf)
        idx = s.idx if c["op"] == "backward" else _plain_select(s)[1]
        hit = torch.zeros_like(z).scatter_add_(1, idx.clamp(min=0).long(), (idx >= 0).double()) > 0
        if c["op"] == "backward":
            # by differentiation of the definition
            z = z.masked_fill(out, 0.0).requires_grad_()
            l = torch.nn.functional.logsigmoid(z) if c["score"] == "sigmoid" else torch.log_softmax(z.masked_fill(out, -math.inf), 1)
        score = torch.exp(l)
        weight = torch.softmax(l.masked_fill(~hit, -1e300), 1) * hit if c["renormalize"] else score
        gate = torch.gather(weight, 1, idx.clamp(min=0).long()) * (idx >= 0) * c["scale"]
        if c["op"] == "select":
            return [score if c["scores"] else None, None, gate]
        total = (gate * s.d_gate.double()).sum()
        if s.d_scores is not None:
            total = total + (score.masked_fill(out, 0.0) * s.d_scores.double()).sum()
        (grad,) = torch.autograd.grad(total, z)
        return [grad.masked_fill(out, 0.0)]
    if c["op"] == "quantize":
        grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
        middle = (grid[1:] + grid[:-1]) / 2
        done = []
        for w in s.w.double().split(8192):   # some rows at a time
            v = torch.nn.functional.pad(w, (0, -w.shape[1] % GROUP)).unflatten(1, (-1, GROUP))
            big = v.abs().amax(2, keepdim=True)
            power = torch.floor(torch.log2(big)) - 2
            power = torch.where(torch.exp2(power + 3) <= big, power + 1, torch.where(torch.exp2(power + 2) > big, power - 1, power))
            if not c["saturate"]:
                power = power + (big > 6 * torch.exp2(power))
            scale = torch.exp2(torch.where(big > 0, power.clamp(-126, 127), torch.zeros_like(power)))
            a = v.abs() / scale
            low, high = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)   # apart only on a middle
            code = torch.where(low % 2 == 0, low, high)
            done.append((torch.sign(v) * grid[code] * scale).flatten(1)[:, :w.shape[1]])
        return [torch.cat(done)]
    offsets = s.offsets.tolist()
    ys, src = [], s.perm_src[:s.rows].long()
    for e in range(c["E"] + c["shared"]):
        routed = e < c["E"]
        rows = src[offsets[e]:offsets[e + 1]] if routed else torch.arange(c["T"], device="cuda")
        w = s.weights[:3] if routed else s.weights[3:]
        at = e if routed else e - c["E"]
        gate, up, down = (_dense(codes[at], scales[at], torch.float64) for codes, scales in w)
        x = s.x[rows].double()
        ys.append((torch.nn.functional.silu(x @ gate.T) * (x @ up.T)) @ down.T)
    y = torch.cat(ys[:c["E"]])
    return [y] if not c["shared"] else [y, torch.stack(ys[c["E"]:])]
