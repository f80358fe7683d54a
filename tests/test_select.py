"""Routing from logits (fmoe_select_experts) and its gradient against plain implementations in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2511_17885_amd import binding

U = 2.0 ** -24                     # half a step of fp32, relative
FLT_MAX = float(np.finfo(np.float32).max)
HALF_BF16 = 2.0 ** -8


# ------------------------------------------------------------------------------------ the definitions, in 64 bits


def _clean(z):
    z = np.asarray(z, np.float64)
    z = np.where(z > -np.inf, z, -np.inf)          # NaN is masked
    return np.minimum(z, FLT_MAX)


def _scores(z, sigmoid):
    if sigmoid:
        with np.errstate(over="ignore"):
            return np.where(z > -np.inf, 1.0 / (1.0 + np.exp(-z)), 0.0)
    m = z.max()
    if m == -np.inf:
        return np.zeros_like(z)
    e = np.exp(z - m)
    return e / e.sum()


def _log_sigmoid(z):
    return np.minimum(z, 0.0) - np.log1p(np.exp(-np.abs(z)))


def _choose(z, bias, k, sigmoid, groups, topk_groups, group_score):
    """One token's list: plain loops over the definition."""
    E = len(z)
    s = _scores(z, sigmoid)
    usable = [e for e in range(E) if z[e] > -np.inf and (bias is None or bias[e] > -np.inf)]
    key = {e: (s[e] + float(bias[e]) if bias is not None else z[e]) for e in usable}
    if groups > 1:
        size, score = E // groups, []
        for g in range(groups):
            members = [e for e in usable if e // size == g]
            if group_score == 0:
                score.append(max([key[e] for e in members], default=-np.inf))
            else:
                u = sorted([key[e] if bias is not None else s[e] for e in members], reverse=True)[:2]
                score.append(sum(u) if u else -np.inf)
        best = sorted(range(groups), key=lambda g: (-score[g], g))[:topk_groups]
        usable = [e for e in usable if e // size in best]
    return sorted(usable, key=lambda e: (-key[e], e))[:k]


def _gates(z, chosen, sigmoid, renorm, scale):
    if not chosen:
        return np.zeros(0)
    if not renorm:
        return scale * _scores(z, sigmoid)[chosen]
    l = (_log_sigmoid(z) if sigmoid else z)[chosen]
    p = np.exp(l - l.max())
    return scale * p / p.sum()


def _reference(z, vis, bias, cfg):
    z = _clean(z)
    T = len(z)
    idx = np.full((T, cfg["kmax"]), -1, np.int32)
    gate = np.zeros((T, cfg["kmax"]))
    score = np.zeros(z.shape)
    for t in range(T):
        k = cfg["k_visual"] if vis is not None and vis[t] else cfg["k_text"]
        chosen = _choose(z[t], bias, k, cfg["sigmoid"], cfg["groups"], cfg["topk_groups"], cfg["group_score"])
        idx[t, :len(chosen)] = chosen
        gate[t, :len(chosen)] = _gates(z[t], chosen, cfg["sigmoid"], cfg["renorm"], cfg["scale"])
        score[t] = _scores(z[t], cfg["sigmoid"])
    return score, idx, gate


def _objective(z, idx, d_gate, d_scores, cfg):
    total = 0.0
    chosen = [int(e) for e in idx if e >= 0]
    total += float(np.dot(_gates(z, chosen, cfg["sigmoid"], cfg["renorm"], cfg["scale"]), d_gate[:len(chosen)]))
    if d_scores is not None:
        live = z > -np.inf
        total += float(np.dot(_scores(z, cfg["sigmoid"])[live], d_scores[live]))
    return total


def _gradient(z, idx, d_gate, d_scores, cfg):
    """The formula, one token."""
    z = _clean(z)
    s = _scores(z, cfg["sigmoid"])
    live = z > -np.inf
    out = np.zeros_like(z)
    ds = np.where(live, 0.0 if d_scores is None else d_scores, 0.0)
    n = int((idx >= 0).sum())
    chosen, a = idx[:n].astype(int), cfg["scale"] * np.asarray(d_gate[:n], np.float64)
    with np.errstate(over="ignore"):
        slope = np.where(live, 1.0 / (1.0 + np.exp(np.where(live, z, 0.0))), 0.0)   # 1 - sigmoid
    if cfg["renorm"]:
        p = _gates(z, list(chosen), cfg["sigmoid"], True, 1.0)
        dl = p * (a - (p * a).sum())
        np.add.at(out, chosen, dl * (slope[chosen] if cfg["sigmoid"] else 1.0))
    else:
        np.add.at(ds, chosen, a)
    out += s * slope * ds if cfg["sigmoid"] else s * (ds - (s * ds).sum())
    return np.where(live, out, 0.0)


# ------------------------------------------------------------------------------------------------- derived bounds


def _gate_bound(z, cfg):
    """Relative error of a gate.  exp and log1p are good to 2 steps (4 U).  Renormalised: l is off by 6 U |l| and the
    difference to the largest by 2 such and one rounding, 13 U max|l| in the exponent; exp 4 U, a sum of 16 terms 4 U and
    its terms' own, quotient and scale 2 U.  Not renormalised: exponent |z - m| U, exp 4 U, sum of E terms (16 in a lane
    and 4 steps) 20 U with its terms' own, reciprocal, product and scale 4 U."""
    live = np.abs(z[np.isfinite(z)])
    big = float(live.max()) if live.size else 0.0
    return (2 * (13 * big + 8) + 16 if cfg["renorm"] else 2 * (2 * big + 8) + 40) * U


def _score_bound(z):
    live = np.abs(z[np.isfinite(z)])
    return (2 * (2 * float(live.max() if live.size else 0.0) + 8) + 40) * U


# ---------------------------------------------------------------------------------------------------------- cases


def _cfg(E, k_text, k_visual, sigmoid=False, renorm=True, groups=1, topk_groups=1, group_score=0, scale=1.0):
    return dict(E=E, k_text=k_text, k_visual=k_visual, kmax=max(k_text, k_visual), sigmoid=sigmoid, renorm=renorm,
                groups=groups, topk_groups=topk_groups, group_score=group_score, scale=scale)


CASES = [
    # T, config, with bias
    (1, _cfg(1, 1, 1), False),
    (1, _cfg(8, 2, 1), False),
    (5, _cfg(7, 7, 3, sigmoid=True), False),
    (17, _cfg(64, 6, 3), False),
    (33, _cfg(64, 6, 0, renorm=False), False),
    (40, _cfg(65, 5, 5, sigmoid=True, renorm=False, scale=1.7), True),
    (16, _cfg(96, 8, 4, groups=3, topk_groups=2), False),
    (16, _cfg(96, 8, 4, groups=3, topk_groups=2, group_score=1), False),
    (50, _cfg(128, 8, 4, sigmoid=True, groups=8, topk_groups=3, group_score=1, scale=2.5), True),
    (50, _cfg(256, 16, 7, sigmoid=True, groups=8, topk_groups=4, group_score=1, scale=2.5), True),
    (31, _cfg(255, 12, 12, groups=15, topk_groups=7, group_score=0), True),
    (31, _cfg(250, 16, 1, renorm=False, groups=10, topk_groups=10, group_score=1), True),
    (19, _cfg(16, 4, 2, groups=16, topk_groups=5, group_score=1), True),       # one expert a group
    (19, _cfg(32, 16, 2, groups=16, topk_groups=3), False),                    # fewer experts stay than are asked for
    (257, _cfg(130, 3, 3, sigmoid=True), True),
    (3, _cfg(20, 0, 0), False),                                                # nothing listed
]


def _make(T, cfg, with_bias, seed, dtype=np.float32, spread=2.0):
    rng = np.random.default_rng(seed)
    z = (spread * rng.standard_normal((T, cfg["E"]))).astype(np.float32)
    if dtype == "bf16":
        z = torch.from_numpy(z).to(torch.bfloat16).float().numpy()
    bias = (0.2 * rng.standard_normal(cfg["E"])).astype(np.float32) if with_bias else None
    vis = (rng.random(T) < 0.6).astype(np.uint8)
    return z, bias, vis


def _context(cfg):
    return binding.FMoE(d_model=64, n_experts=cfg["E"], d_ffn=64, k_text=cfg["k_text"], k_visual=cfg["k_visual"],
                        dtype="f32", renormalize=cfg["renorm"])


def _params(cfg):
    return binding.select_params("sigmoid" if cfg["sigmoid"] else "softmax", cfg["groups"], cfg["topk_groups"],
                                 cfg["group_score"], cfg["scale"])


def _gpu(a, dtype=None):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(dtype) if dtype is not None else t


def _check_forward(z, bias, vis, cfg, torch_type, got):
    scores, idx, gate = got
    want_s, want_i, want_g = _reference(z, vis, bias, cfg)
    assert np.array_equal(idx.cpu().numpy(), want_i)
    g = gate.double().cpu().numpy()
    assert (np.abs(g - want_g) <= _gate_bound(_clean(z), cfg) * np.abs(want_g) + 2.0 ** -126 * cfg["scale"]).all()
    assert (g[want_i < 0] == 0).all()
    s = scores.double().cpu().numpy()
    # below the normal range a score has an absolute error
    assert (np.abs(s - want_s) <= _score_bound(_clean(z)) * want_s + 2.0 ** -126).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_select(case, dtype):
    T, cfg, with_bias = CASES[case]
    z, bias, vis = _make(T, cfg, with_bias, 100 + case, dtype)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    m = _context(cfg)
    got = m.select_experts(_params(cfg), _gpu(z, tt), _gpu(vis), _gpu(bias), want_scores=True)
    _check_forward(z, bias, vis, cfg, tt, got)
    # the scores are optional, and so is the mask
    s, idx, gate = m.select_experts(_params(cfg), _gpu(z, tt), None, _gpu(bias))
    assert s is None
    want = _reference(z, None, bias, cfg)
    assert np.array_equal(idx.cpu().numpy(), want[1])


def _special_rows(E, rng):
    """Rows where a mask, an infinity, NaN or equal keys decide."""
    lowest = -FLT_MAX
    rows = [np.full(E, -np.inf), np.full(E, np.nan), np.full(E, lowest), np.full(E, np.inf), np.full(E, -200.0),
            np.full(E, 0.0)]
    r = np.full(E, -np.inf); r[E - 1] = 1.0; rows.append(r)                     # a single expert is left
    r = np.full(E, -np.inf); r[0] = lowest; rows.append(r)
    r = rng.standard_normal(E); r[::2] = -np.inf; rows.append(r)
    r = rng.standard_normal(E); r[1::3] = np.nan; rows.append(r)
    r = rng.standard_normal(E); r[2] = np.inf; r[E - 2] = np.inf; rows.append(r)
    r = rng.standard_normal(E); r[: E // 2] = lowest; rows.append(r)
    r = np.round(rng.standard_normal(E)); rows.append(r)                        # many equal ones
    r = np.where(np.arange(E) % 2 == 0, 0.0, -0.0); rows.append(r)
    rows.append(50.0 * rng.standard_normal(E))                                  # scores that underflow or saturate
    return np.stack(rows).astype(np.float32)


SPECIAL = [_cfg(24, 5, 2), _cfg(24, 5, 2, sigmoid=True), _cfg(24, 5, 2, renorm=False), _cfg(24, 5, 2, sigmoid=True, renorm=False),
           _cfg(24, 6, 3, groups=4, topk_groups=2), _cfg(24, 6, 3, groups=4, topk_groups=2, group_score=1),
           _cfg(24, 6, 3, sigmoid=True, groups=4, topk_groups=2, group_score=1), _cfg(130, 6, 3, sigmoid=True, groups=2)]


@pytest.mark.gpu
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("case", range(len(SPECIAL)))
def test_select_masked_infinite_and_equal_logits(case, with_bias):
    cfg = SPECIAL[case]
    rng = np.random.default_rng(case)
    z = _special_rows(cfg["E"], rng)
    bias = None
    if with_bias:
        bias = np.zeros(cfg["E"], np.float32)          # equal keys stay equal
        bias[3], bias[5], bias[7], bias[11] = -np.inf, np.nan, 0.5, np.inf
    got = _context(cfg).select_experts(_params(cfg), _gpu(z), None, _gpu(bias), want_scores=True)
    scores, idx, gate = got
    want_s, want_i, want_g = _reference(z, None, bias, cfg)
    assert np.array_equal(idx.cpu().numpy(), want_i)
    g, s = gate.double().cpu().numpy(), scores.double().cpu().numpy()
    assert np.isfinite(g).all() and np.isfinite(s).all()
    for t in range(len(z)):
        zt = _clean(z[t])
        fine = zt[np.abs(zt) < 1e6]                    # rows of huge logits: shares and scores there are 0 or 1 / n
        bound = _gate_bound(fine, cfg)
        assert (np.abs(g[t] - want_g[t]) <= bound * np.abs(want_g[t]) + 2.0 ** -126).all(), t
        assert (np.abs(s[t] - want_s[t]) <= _score_bound(fine) * want_s[t] + 2.0 ** -126).all(), t


@pytest.mark.gpu
def test_select_decides_by_keys_that_are_equal_in_32_bits():
    """Logits whose sigmoid is the same fp32 number, in descending and ascending order of index: the larger logit is first."""
    E = 40
    base = np.float32(6.0)
    z = np.zeros((2, E), np.float32)
    for i in range(E):
        z[0, i] = base + np.float32(i) * np.float32(2.0 ** -21)
        z[1, i] = base - np.float32(i) * np.float32(2.0 ** -21)
    assert len(np.unique((1.0 / (1.0 + np.exp(-z[0].astype(np.float32)))).astype(np.float32))) < E // 2
    for bias in (None, np.full(E, 0.25, np.float32)):
        cfg = _cfg(E, 16, 16, sigmoid=True)
        idx = _context(cfg).select_experts(_params(cfg), _gpu(z), None, _gpu(bias))[1].cpu().numpy()
        assert list(idx[0]) == list(range(E - 1, E - 17, -1)) and list(idx[1]) == list(range(16))


@pytest.mark.gpu
@pytest.mark.parametrize("sigmoid", [False, True])
def test_select_biases_of_any_size(sigmoid):
    """Keys whose size hides the scores in 32 bits (they differ by a score's last bits at 1000), groups whose two largest keys
    cancel, and keys further apart than a list's integers span."""
    rng = np.random.default_rng(77)
    E = 64
    z = rng.standard_normal((40, E)).astype(np.float32)
    for k, groups, bias in ((6, 1, np.full(E, 1000.0)), (8, 8, np.where(np.arange(E) % 2 == 0, 300.0, -300.0)),
                            (8, 32 // 2, np.where(np.arange(E) % 4 == 0, 1e4, np.where(np.arange(E) % 4 == 1, -1e4, -3e4))),
                            (16, 1, rng.choice([-9.0, 0.0, 9.0], size=E)), (5, 1, np.zeros(E)), (3, 4, np.full(E, -1e6))):
        cfg = _cfg(E, k, k, sigmoid=sigmoid, groups=groups, topk_groups=max(1, groups // 2), group_score=1)
        b = bias.astype(np.float32)
        idx = _context(cfg).select_experts(_params(cfg), _gpu(z), None, _gpu(b))[1].cpu().numpy()
        assert np.array_equal(idx, _reference(z, None, b, cfg)[1]), (k, groups)


@pytest.mark.gpu
def test_select_large_logits():
    rng = np.random.default_rng(78)
    for scale, offset in ((1.0, 1e4), (100.0, 0.0), (1e5, -1e6), (1e-3, 0.0), (1e-3, 5e3)):
        z = (scale * rng.standard_normal((50, 96)) + offset).astype(np.float32)
        for cfg in (_cfg(96, 8, 8), _cfg(96, 8, 8, sigmoid=True, groups=6, topk_groups=2)):
            idx = _context(cfg).select_experts(_params(cfg), _gpu(z))[1].cpu().numpy()
            assert np.array_equal(idx, _reference(z, None, None, cfg)[1]), (scale, offset)


@pytest.mark.gpu
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("E", [40, 100, 256])
def test_select_fewer_usable_experts_than_are_asked_for(E, with_bias):
    """Rows with none to ten usable experts of which eight are asked for, near, equal and further apart than integers span."""
    rng = np.random.default_rng(E)
    z = np.full((66, E), -np.inf, np.float32)
    for t in range(66):
        n = t % 11
        where = rng.choice(E, size=n, replace=False)
        kind = t // 11
        values = rng.standard_normal(n) * (1.0, 1e-6, 0.0, 40.0, 400.0, 1e5)[kind]
        z[t, where] = values.astype(np.float32)
    bias = rng.choice([-9.0, -3.9, -4.1, 0.0, 0.1], size=E).astype(np.float32) if with_bias else None
    for sigmoid in (False, True):
        for groups, topk in ((1, 1), (4, 2)):
            cfg = _cfg(E, 8, 8, sigmoid=sigmoid, groups=groups, topk_groups=topk)
            idx, gate = _context(cfg).select_experts(_params(cfg), _gpu(z), None, _gpu(bias))[1:]
            want = _reference(z, None, bias, cfg)[1]
            assert np.array_equal(idx.cpu().numpy(), want), (sigmoid, groups)
            assert (gate.cpu().numpy()[want < 0] == 0).all()


@pytest.mark.gpu
def test_select_many_rows_and_replay():
    """More rows than blocks run at once; the same from a captured graph, three times, with other work between."""
    T, cfg = 40000, _cfg(256, 8, 4, sigmoid=True, groups=8, topk_groups=4, group_score=1, scale=2.5)
    gen = torch.Generator(device="cuda"); gen.manual_seed(5)
    z = torch.randn(T, 256, generator=gen, device="cuda")
    bias = 0.1 * torch.randn(256, generator=gen, device="cuda")
    vis = (torch.arange(T, device="cuda") % 3 > 0).to(torch.uint8)
    m, p = _context(cfg), _params(cfg)
    scores, idx, gate = m.select_experts(p, z, vis, bias, want_scores=True)
    for t in list(range(0, 40)) + list(range(T - 40, T)):
        row = _clean(z[t].cpu().numpy())
        chosen = _choose(row, bias.cpu().numpy(), 4 if t % 3 else 8, True, 8, 4, 1)
        assert idx[t].tolist() == chosen + [-1] * (8 - len(chosen))
    d_gate = torch.randn(T, 8, generator=gen, device="cuda")
    d_z = m.select_experts_backward(p, z, idx, d_gate, scores)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(2):
            m.select_experts_backward(p, z, m.select_experts(p, z, vis, bias, want_scores=True)[1], d_gate, scores)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.select_experts(p, z, vis, bias, want_scores=True)
        out_d = m.select_experts_backward(p, z, out[1], d_gate, out[0])
    for _ in range(3):
        for o in (*out, out_d):
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, (scores, idx, gate))) and torch.equal(out_d, d_z)
        m.select_experts(p, -z, vis, bias)
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------- gradient


def _backward_bound(z, d_gate, d_scores, cfg):
    """Absolute, per token.  List part: p is off by the gate bound and at most 1, the difference a - sum p a by the same and
    by a sum's 16 roundings, and is at most 2 max|a|.  Score part: s off by the score bound, the sum over the experts by
    that and 20 roundings, the difference at most 2 max|ds|."""
    a = cfg["scale"] * (np.abs(d_gate).max(initial=0.0))
    ds = (np.abs(d_scores).max(initial=0.0) if d_scores is not None else 0.0) + (0.0 if cfg["renorm"] else a)
    rel = _gate_bound(z, dict(cfg, renorm=True)) + _score_bound(z)
    return 2 * a * (2 * rel + 40 * U) + 2 * ds * (2 * _score_bound(z) + 60 * U)


@pytest.mark.gpu
@pytest.mark.parametrize("with_scores", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_select_backward(case, dtype, with_scores):
    T, cfg, with_bias = CASES[case]
    z, bias, vis = _make(T, cfg, with_bias, 300 + case, dtype)
    rng = np.random.default_rng(case)
    _, idx, _ = _reference(z, vis, bias, cfg)
    d_gate = rng.standard_normal((T, cfg["kmax"])).astype(np.float32)
    d_gate[idx < 0] = np.nan                                  # not looked at
    d_scores = rng.standard_normal((T, cfg["E"])).astype(np.float32) if with_scores else None
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    got = _context(cfg).select_experts_backward(_params(cfg), _gpu(z, tt), _gpu(idx), _gpu(d_gate), _gpu(d_scores))
    assert got.dtype == tt
    got = got.double().cpu().numpy()
    for t in range(T):
        used = np.where(idx[t] >= 0, d_gate[t], 0.0)
        want = _gradient(z[t], idx[t], used, None if d_scores is None else d_scores[t].astype(np.float64), cfg)
        bound = _backward_bound(_clean(z[t]), used, None if d_scores is None else d_scores[t], cfg)
        allowed = bound + (HALF_BF16 * np.abs(want) if dtype == "bf16" else 0.0)
        assert (np.abs(got[t] - want) <= allowed).all(), (t, np.abs(got[t] - want).max(), bound)


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(SPECIAL)))
def test_select_backward_of_masked_logits(case):
    cfg = SPECIAL[case]
    rng = np.random.default_rng(40 + case)
    z = _special_rows(cfg["E"], rng)
    _, idx, _ = _reference(z, None, None, cfg)
    d_gate = rng.standard_normal(idx.shape).astype(np.float32)
    d_scores = rng.standard_normal(z.shape).astype(np.float32)
    d_scores[~(z > -np.inf)] = np.nan                          # gradients of masked scores are not looked at
    for ds in (None, d_scores):
        got = _context(cfg).select_experts_backward(_params(cfg), _gpu(z), _gpu(idx), _gpu(d_gate), _gpu(ds))
        got = got.double().cpu().numpy()
        assert (got[~(z > -np.inf)] == 0).all()
        for t in range(len(z)):
            zt = _clean(z[t])
            live = None if ds is None else np.where(zt > -np.inf, np.nan_to_num(ds[t]), 0.0).astype(np.float64)
            want = _gradient(z[t], idx[t], d_gate[t], live, cfg)
            bound = _backward_bound(zt[np.abs(zt) < 1e6], d_gate[t], live, cfg)
            assert (np.abs(got[t] - want) <= bound).all(), (t, np.abs(got[t] - want).max(), bound)


@pytest.mark.gpu
@pytest.mark.parametrize("sigmoid,renorm", [(False, True), (True, True), (False, False), (True, False)])
def test_select_backward_against_differences(sigmoid, renorm):
    """Central differences of the objective in 64 bits, step 1e-5: their error is 1e-10 |third derivative| and 2e-16 / 1e-5 of
    the objective, both far below the kernel's own bound."""
    cfg = _cfg(20, 5, 2, sigmoid=sigmoid, renorm=renorm, scale=1.3)
    z, _, vis = _make(6, cfg, False, 9)
    rng = np.random.default_rng(2)
    _, idx, _ = _reference(z, vis, None, cfg)
    d_gate = rng.standard_normal(idx.shape).astype(np.float32)
    d_scores = rng.standard_normal(z.shape).astype(np.float32)
    got = _context(cfg).select_experts_backward(_params(cfg), _gpu(z), _gpu(idx), _gpu(d_gate), _gpu(d_scores)).double().cpu().numpy()
    step = 1e-5
    for t in range(len(z)):
        bound = _backward_bound(_clean(z[t]), d_gate[t], d_scores[t], cfg) + 1e-8
        for e in range(cfg["E"]):
            up, down = z[t].astype(np.float64), z[t].astype(np.float64)
            up[e] += step
            down[e] -= step
            f = lambda v: _objective(v, idx[t], d_gate[t], d_scores[t].astype(np.float64), cfg)  # noqa: E731
            assert abs((f(up) - f(down)) / (2 * step) - got[t, e]) <= bound


@pytest.mark.gpu
def test_select_backward_keeps_a_nan_gradient():
    cfg = _cfg(8, 2, 2)
    z = np.zeros((1, 8), np.float32)
    idx = np.array([[0, 1]], np.int32)
    d_gate = np.array([[np.nan, 1.0]], np.float32)
    for tt in (torch.float32, torch.bfloat16):
        got = _context(cfg).select_experts_backward(_params(cfg), _gpu(z, tt), _gpu(idx), _gpu(d_gate)).float().cpu().numpy()
        assert np.isnan(got[0, :2]).all() and (got[0, 2:] == 0).all()


@pytest.mark.gpu
def test_select_empty_batch():
    cfg = _cfg(8, 2, 2)
    m = _context(cfg)
    z = torch.empty(0, 8, device="cuda")
    s, idx, gate = m.select_experts(_params(cfg), z, want_scores=True)
    assert s.shape == (0, 8) and idx.shape == (0, 2) and gate.shape == (0, 2)
    assert m.select_experts_backward(_params(cfg), z, idx, gate).shape == (0, 8)


@pytest.mark.gpu
def test_select_on_two_streams_at_once_and_on_rows_inside_a_larger_tensor():
    cfgs = (_cfg(256, 8, 4, sigmoid=True, groups=8, topk_groups=4, group_score=1), _cfg(64, 6, 3, renorm=False))
    jobs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    gen = torch.Generator(device="cuda"); gen.manual_seed(9)
    for cfg in cfgs:
        z = torch.randn(3010, cfg["E"], generator=gen, device="cuda")[10:]     # contiguous, not at the start
        bias = 0.1 * torch.randn(cfg["E"], generator=gen, device="cuda")
        m, p = _context(cfg), _params(cfg)
        want = m.select_experts(p, z, None, bias, want_scores=True)
        d_gate = torch.randn(3000, cfg["kmax"], generator=gen, device="cuda")
        jobs.append((m, p, z, bias, d_gate, want, m.select_experts_backward(p, z, want[1], d_gate, want[0])))
        head = _reference(z[:20].cpu().numpy(), None, bias.cpu().numpy(), cfg)[1]
        assert np.array_equal(want[1][:20].cpu().numpy(), head)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (m, p, z, bias, d_gate, want, want_d) in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                out = m.select_experts(p, z, None, bias, want_scores=True)
                got[i].append((*out, m.select_experts_backward(p, z, out[1], d_gate, out[0])))
    torch.cuda.synchronize()
    for i, job in enumerate(jobs):
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, (*job[5], job[6])))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_offsets_past_32_bits(dtype):
    """4.4 and 2.2 GB of logits: rows far behind come out as they do alone."""
    E, T = 256, 4_300_000 * (1 if dtype == torch.float32 else 2)
    cfg = _cfg(E, 4, 4, sigmoid=True)
    m, p = _context(cfg), _params(cfg)
    z = torch.zeros(T, E, dtype=dtype, device="cuda")
    gen = torch.Generator(device="cuda"); gen.manual_seed(1)
    z[-100:] = torch.randn(100, E, generator=gen, device="cuda").to(dtype)
    _, idx, gate = m.select_experts(p, z)
    d_gate = torch.ones(T, 4, device="cuda")
    d_gate[:, 1] = -2.0
    d = m.select_experts_backward(p, z, idx, d_gate)
    tail = z[-100:].clone()
    _, i, g = m.select_experts(p, tail)
    assert torch.equal(idx[-100:], i) and torch.equal(gate[-100:], g)
    assert torch.equal(d[-100:], m.select_experts_backward(p, tail, i, d_gate[-100:].contiguous()))
    assert (idx[:-100] == torch.arange(4, dtype=torch.int32, device="cuda")).all()


@pytest.mark.gpu
def test_select_backward_of_lists_that_were_not_chosen_here():
    """Any distinct experts may be listed, in any order and with gaps; places outside 0 .. E-1 are empty."""
    rng = np.random.default_rng(31)
    for sigmoid in (False, True):
        for renorm in (False, True):
            cfg = _cfg(20, 5, 5, sigmoid=sigmoid, renorm=renorm, scale=0.7)
            z = rng.standard_normal((30, 20)).astype(np.float32)
            idx = np.stack([rng.choice(20, size=5, replace=False) for _ in range(30)]).astype(np.int32)
            idx[rng.random(idx.shape) < 0.3] = -1
            idx[0, 2], idx[1, 0], idx[2] = 20, 2 ** 31 - 1, -7
            d_gate = rng.standard_normal(idx.shape).astype(np.float32)
            got = _context(cfg).select_experts_backward(_params(cfg), _gpu(z), _gpu(idx), _gpu(d_gate)).double().cpu().numpy()
            for t in range(30):
                on = (idx[t] >= 0) & (idx[t] < 20)
                want = _gradient(z[t], np.concatenate([idx[t][on], np.full(5 - on.sum(), -1)]), d_gate[t][on], None, cfg)
                assert (np.abs(got[t] - want) <= _backward_bound(_clean(z[t]), d_gate[t], None, cfg)).all(), t


# ------------------------------------------------------------------------- row maxima of any size, rows beside each other


def _lists(z, bias, cfg):
    """Lists [T, kmax] of rows without masked logits, all of them at once: the definition by stable sorts in 64 bits."""
    z = z.astype(np.float64)
    T, E = z.shape
    if cfg["sigmoid"]:
        s = 1.0 / (1.0 + np.exp(-z))
    else:
        s = np.exp(z - z.max(1, keepdims=True))
        s = s / s.sum(1, keepdims=True)
    key = z if bias is None else s + bias.astype(np.float64)
    if cfg["groups"] > 1:
        members = (s if bias is None and cfg["group_score"] else key).reshape(T, cfg["groups"], -1)
        score = np.sort(members, axis=2)[:, :, -2:].sum(2) if cfg["group_score"] else members.max(2)
        best = np.argsort(-score, axis=1, kind="stable")[:, :cfg["topk_groups"]]
        stays = np.zeros(score.shape, bool)
        np.put_along_axis(stays, best, True, 1)
        key = np.where(np.repeat(stays, E // cfg["groups"], axis=1), key, -np.inf)
    return np.argsort(-key, axis=1, kind="stable")[:, :cfg["kmax"]].astype(np.int32)


def _maxima(reach):
    """fp32 numbers between -reach and reach: evenly spread, 300 neighbours at either side of every place where reach / 8
    less the number comes to another binade, and neighbours all through the last sixteenth below."""
    half = np.float32(reach)
    parts = [np.linspace(-reach, reach, 6000).astype(np.float32),
             np.linspace(-reach, -reach * 15 / 16, 2000).astype(np.float32)]
    for n in range(-3, 4):
        edge = np.float32(reach / 8 * (1 - 2.0 ** n))
        bits = np.arange(-300, 300) * np.spacing(np.abs(edge) + np.float32(1e-3))
        parts.append((edge + bits).astype(np.float32))
    for at in (-reach * 239.5 / 256, -reach * 239.004 / 256):
        parts.append((np.float32(at) + np.arange(64) * np.spacing(half / 2)).astype(np.float32))
    return np.concatenate(parts)


@pytest.mark.gpu
@pytest.mark.parametrize("group_score", [0, 1])
@pytest.mark.parametrize("groups", [1, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_row_maxima_of_any_size(dtype, groups, group_score):
    """The list compares keys by their distance to the row's largest: rows whose largest logit is any number from -512 to 512
    and beyond, on and beside the places where that distance is rounded to another step."""
    rng = np.random.default_rng(groups)
    top = np.concatenate([_maxima(512.0), np.linspace(-700, 700, 500).astype(np.float32)])
    z = (top[:, None] - 3.0 * rng.random((len(top), 64))).astype(np.float32)
    z[np.arange(len(top)), rng.integers(0, 64, size=len(top))] = top
    if dtype == "bf16":
        z = torch.from_numpy(z).to(torch.bfloat16).float().numpy()
    for sigmoid in (False, True):
        cfg = _cfg(64, 6, 6, sigmoid=sigmoid, groups=groups, topk_groups=max(1, groups // 2), group_score=group_score)
        idx = _context(cfg).select_experts(_params(cfg), _gpu(z, torch.bfloat16 if dtype == "bf16" else None))[1].cpu().numpy()
        wrong = (idx != _lists(z, None, cfg)).any(1)
        assert not wrong.any(), (sigmoid, int(wrong.sum()), top[wrong][:5])


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [1, 8])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_select_biased_maxima_of_any_size(sigmoid, groups):
    """The same for keys with a bias, whose size is the bias's: from -32 to 32 and beyond, closely from -31 to -29."""
    rng = np.random.default_rng(5 + groups)
    z = rng.standard_normal((400, 64)).astype(np.float32)
    cfg = _cfg(64, 6, 6, sigmoid=sigmoid, groups=groups, topk_groups=max(1, groups // 2), group_score=1)
    m, p, zg = _context(cfg), _params(cfg), _gpu(z)
    for size in np.concatenate([np.linspace(-40.0, 40.0, 81), np.linspace(-31.0, -29.0, 81), [4 - 2.0 ** n for n in range(-2, 6)]]):
        bias = (size + 0.01 * rng.standard_normal(64)).astype(np.float32)
        idx = m.select_experts(p, zg, None, _gpu(bias))[1].cpu().numpy()
        wrong = (idx != _lists(z, bias, cfg)).any(1)
        assert not wrong.any(), (size, int(wrong.sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_select_of_a_row_does_not_depend_on_the_rows_beside_it(sigmoid, renorm):
    """Rows alone, and each beside rows whose scores underflow, whose logits are all masked, or whose keys are equal: the same
    bits; so is the gradient."""
    rng = np.random.default_rng(6)
    E, T = 64, 45
    z = (3.0 * rng.standard_normal((T, E))).astype(np.float32)
    low = (rng.standard_normal((T, E)) - 70.0).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    others = [low, np.full((T, E), -np.inf, np.float32), np.zeros((T, E), np.float32)]
    mixed = np.stack([z] + others, 1).reshape(4 * T, E)
    for groups in (1, 8):
        for b in (None, bias):
            cfg = _cfg(E, 6, 6, sigmoid=sigmoid, renorm=renorm, groups=groups, topk_groups=max(1, groups // 2), group_score=1, scale=2.5)
            m, p = _context(cfg), _params(cfg)
            together = m.select_experts(p, _gpu(mixed), None, _gpu(b), want_scores=True)
            d_gate = torch.randn(4 * T, 6, device="cuda")
            d_z = m.select_experts_backward(p, _gpu(mixed), together[1], d_gate, together[0])
            for i, rows in enumerate([z] + others):
                alone = m.select_experts(p, _gpu(rows), None, _gpu(b), want_scores=True)
                assert all(torch.equal(x, y[i::4]) for x, y in zip(alone, together)), (groups, i)
                d = m.select_experts_backward(p, _gpu(rows), alone[1], d_gate[i::4].contiguous(), alone[0])
                assert torch.equal(d, d_z[i::4]), (groups, i)
                one = m.select_experts(p, _gpu(rows[7:8]), None, _gpu(b), want_scores=True)
                assert all(torch.equal(x, y[7:8]) for x, y in zip(one, alone)), (groups, i)


@pytest.mark.gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("lowest", [-FLT_MAX, -3e38, -1.8e38, 3e38, FLT_MAX])
def test_select_groups_whose_two_largest_keys_overflow_in_32_bits(lowest, sigmoid):
    """Biases of the type's lowest or largest value: the sum of a group's two largest keys does not fit in fp32, and still is
    the score of a group that has usable experts, not of one that has none."""
    rng = np.random.default_rng(8)
    for E, groups, topk_groups in ((16, 2, 1), (48, 8, 3), (64, 16, 5), (200, 4, 2)):
        z = rng.standard_normal((60, E)).astype(np.float32)
        z[rng.random(z.shape) < 0.6] = -np.inf
        size = E // groups
        for t in range(60):      # one or more groups without any usable expert, the others with few
            g = rng.choice(groups, size=rng.integers(1, groups), replace=False)
            z[t, (g[:, None] * size + np.arange(size)).ravel()] = -np.inf
        bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
        bias[rng.random(E) < 0.8] = lowest
        for b in (bias, np.full(E, lowest, np.float32)):
            cfg = _cfg(E, 6, 6, sigmoid=sigmoid, groups=groups, topk_groups=topk_groups, group_score=1)
            idx = _context(cfg).select_experts(_params(cfg), _gpu(z), None, _gpu(b))[1].cpu().numpy()
            assert np.array_equal(idx, _reference(z, None, b, cfg)[1]), (E, groups)


# --------------------------------------------------------------------------------------------------------- refusals


def test_select_refuses_bad_arguments():
    lib = binding.load()
    cfg = binding.FmoeConfig(64, 24, 32, 0, 0, 4, 2, 1, binding.FMOE_F32)
    ctx = C.c_void_p()
    assert lib.fmoe_create(C.byref(ctx), C.byref(cfg), 0) == 0
    ok, d = binding.select_params("sigmoid", 4, 2, 1, 2.5), C.c_void_p(0x1000)
    odd = C.c_void_p(0x1004)
    fwd = lambda p=ok, z=d, t=0, T=4, bias=None, s=None, i=d, g=d: lib.fmoe_select_experts(  # noqa: E731
        ctx, None if p is None else C.byref(p), z, t, None, bias, T, s, i, g, None)
    bwd = lambda p=ok, z=d, t=0, i=d, dg=d, ds=None, T=4, o=d: lib.fmoe_select_experts_backward(  # noqa: E731
        ctx, None if p is None else C.byref(p), z, t, i, dg, ds, T, o, None)
    for call in (fwd, bwd):
        assert call(p=None) == -2
        for bad, code in [(dict(score=2), -1), (dict(n_groups=5), -1), (dict(n_groups=0), -1), (dict(n_groups=24), -5),
                          (dict(n_groups=4, topk_groups=5), -1), (dict(n_groups=4, topk_groups=0), -1), (dict(group_score=2), -1),
                          (dict(gate_scale=math.inf), -1), (dict(gate_scale=math.nan), -1)]:
            assert call(p=binding.select_params(**bad)) == code, bad
            assert lib.fmoe_last_error() != b""
        assert call(t=2) == -1 and call(T=-1) == -1 and call(T=1 << 24) == -5
        assert call(z=None) == -2 and call(z=odd) == -1
        assert call(z=None, T=0) == 0                       # nothing to do
    assert fwd(i=None) == -2 and fwd(g=None) == -2 and fwd(s=odd) == -1 and fwd(bias=odd) == -1
    assert bwd(i=None) == -2 and bwd(dg=None) == -2 and bwd(o=None) == -2 and bwd(o=odd) == -1 and bwd(ds=odd) == -1
    assert lib.fmoe_select_experts(None, C.byref(ok), d, 0, None, None, 4, None, d, d, None) == -2
    assert lib.fmoe_select_experts_backward(None, C.byref(ok), d, 0, d, d, None, 4, d, None) == -2
    lib.fmoe_destroy(ctx)


@pytest.mark.gpu
def test_select_binding_refuses_tensors_of_other_shapes():
    cfg = _cfg(8, 2, 1)
    m, p = _context(cfg), _params(cfg)
    z = torch.zeros(4, 8, device="cuda")
    idx = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for call in (lambda: m.select_experts(p, z[:, :7]), lambda: m.select_experts(p, z.t().contiguous()),
                 lambda: m.select_experts(p, z, torch.zeros(3, dtype=torch.uint8, device="cuda")),
                 lambda: m.select_experts(p, z, None, torch.zeros(7, device="cuda")),
                 lambda: m.select_experts(p, torch.zeros(8, 8, device="cuda")[::2]),
                 lambda: m.select_experts_backward(p, z, idx[:3], torch.zeros(4, 2, device="cuda")),
                 lambda: m.select_experts_backward(p, z, idx, torch.zeros(4, 2, device="cuda", dtype=torch.float64)),
                 lambda: m.select_experts_backward(p, z, idx, torch.zeros(4, 2, device="cuda"), torch.zeros(4, 7, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        m.select_experts(p, z.double())


@pytest.mark.gpu
def test_select_binding_refuses_tensors_on_the_host():
    cfg = _cfg(8, 2, 1)
    m, p = _context(cfg), _params(cfg)
    z, idx, dg = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for call in (lambda: m.select_experts(p, z.cpu()), lambda: m.select_experts(p, z, torch.zeros(4, dtype=torch.uint8)),
                 lambda: m.select_experts(p, z, None, torch.zeros(8)), lambda: m.select_experts_backward(p, z, idx.cpu(), dg),
                 lambda: m.select_experts_backward(p, z, idx, dg.cpu()), lambda: m.select_experts_backward(p, z, idx, dg, z.cpu())):
        with pytest.raises(ValueError, match="on cuda:0"):
            call()
