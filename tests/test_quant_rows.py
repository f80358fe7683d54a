"""Expert products on rows in 8 bits with weights in 4 bits, against plain implementations in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_17885_amd import binding
from test_norm import E4M3, _quantize
from test_quant_weights import GRID, _pack, _rows, _silu

U = 2.0 ** -24
HALF_BF16 = 2.0 ** -8


def _values8(codes, scales):
    return _unscaled(codes) * np.repeat(np.exp2(scales.astype(np.float64) - 127.0), 32, axis=-1)[..., :codes.shape[-1]]


def _exact_rows(rng, T, d):
    """Rows whose products with _exact_weights add up without any rounding in fp32: quarters up to 7.5, scales 1/2, 1, 2."""
    q = rng.integers(0, 16, (T, d)) * 0.5
    codes = (np.searchsorted(E4M3, q) | (rng.integers(0, 2, (T, d)) << 7)).astype(np.uint8)
    scales = np.full((T, binding.row_scales(d)), 127, np.uint8)
    scales[:, :-(-d // 32)] = rng.integers(126, 129, (T, -(-d // 32)))
    return codes, scales


def _exact_weights(rng, G, n, K, small):
    """Codes and scales: powers of two within a factor of four, small enough for sums of the order of one."""
    codes = rng.integers(0, 16, (G, n, K)).astype(np.uint8)
    return codes, (127 - small + rng.integers(0, 3, (G, n, -(-K // 32)))).astype(np.uint8)


def _matrix(codes, scales):
    """(numbers, scales) of 4-bit codes"""
    return np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7], np.exp2(scales.astype(np.float64) - 127.0)


def _as_rows(codes, scales):
    return _unscaled(codes), np.exp2(scales[:, :-(-codes.shape[1] // 32)].astype(np.float64) - 127.0)


class _Layer:
    def __init__(self, rng, d, E, F, shared=0, F_shared=0, k=2):
        shapes = [(E, F, d), (E, F, d), (E, d, F)] + ([(shared, F_shared, d)] * 2 + [(shared, d, F_shared)] if shared else [])
        small = int(round(np.log2(d) / 2)) + 4   # products of the order of 10, sqrt(d) of them
        host = [_exact_weights(rng, *s, small) for s in shapes]
        self.w = [[_matrix(c[g], s[g]) for g in range(len(c))] for c, s in host]
        self.pairs = [(torch.from_numpy(_pack(c)).cuda(), torch.from_numpy(s).cuda()) for c, s in host]
        self.m = binding.FMoE(d_model=d, n_experts=E, d_ffn=F, n_shared=shared, d_ffn_shared=F_shared, k_text=k, k_visual=k, dtype="bf16")
        self.m.set_weights_quant_rows(*self.pairs)


def _unscaled(codes):
    """e4m3 numbers of codes, without their scales"""
    return np.where(codes & 0x80, -1.0, 1.0) * E4M3[np.minimum(codes & 0x7f, 126)]


def _products(x, x_scales, w, w_scales, cuts=True):
    """x @ w.T of numbers [., K] times powers of two [., K/32], and how far the matrix instruction may be off: it cuts the products of
    eight neighbours (towards zero) at 2^-13 of the largest power of two among them (exponents of the factors added, those of
    subnormal codes as they are stored), and adds the eights up in fp32: as many roundings of at most the sum of magnitudes, twice
    for what is rounded inside."""
    K = x.shape[1]
    v = np.abs(x) * np.repeat(x_scales, 32, 1)[:, :K], np.abs(w) * np.repeat(w_scales, 32, 1)[:, :K]
    want = (np.sign(x) * v[0]) @ (np.sign(w) * v[1]).T
    cut = np.zeros(want.shape)
    if not cuts:
        return want, 2 * 2 * (K / 8) * U * (v[0] @ v[1].T)   # large and small codes apart: twice as many sums
    with np.errstate(divide="ignore"):
        ex = np.where(x == 0, -np.inf, np.maximum(np.floor(np.log2(np.abs(x))), -6))
        ew = np.where(w == 0, -np.inf, np.maximum(np.floor(np.log2(np.abs(w))), 0))
    for k in range(0, K, 8):
        b = slice(k, k + 8)
        unit = np.exp2((ex[:, None, b] + ew[None, :, b]).max(2, keepdims=True) - 13.0)   # 0 where all products are
        t = np.abs(x[:, None, b] * w[None, :, b])
        part = (t - np.floor(t / np.where(unit > 0, unit, 1.0)) * unit).sum(2)
        cut += part * x_scales[:, k // 32, None] * w_scales[None, :, k // 32]
    return want, cut + 2 * (K / 8) * U * (v[0] @ v[1].T)


def _slack(a, err):
    """(a in 8 bits, how far a kernel may be off whose values are within err of a): both ends, with both scales they allow."""
    codes, scales = _quantize(a)
    want = _values8(codes, scales)
    off = np.zeros_like(a)
    for end in (np.abs(a) - err, np.abs(a) + err):
        end = np.copysign(np.maximum(end, 0.0), a)
        off = np.maximum(off, np.abs(_values8(*_quantize(end)) - want))
    return want, off


def _ffn(x, xs, gate, up, down):
    """y and how far a correct kernel may be from it, per element; matrices as (numbers, scales).  Gate and up as above.  silu:
    2^-20 (1 + |g|) relative (exponential and reciprocal of the hardware); then the rounding to 8 bits, which may fall to either
    side where that reaches a border; the down product as above; y in bf16."""
    g, eg = _products(x, xs, *gate)
    u, eu = _products(x, xs, *up)
    a = _silu(g) * u
    ea = 1.1 * np.abs(u) * eg + np.abs(_silu(g)) * eu + 1.1 * eg * eu + 2.0 ** -20 * (1 + np.abs(g)) * np.abs(a)
    _, eh = _slack(a, ea)
    codes, scales = _quantize(a)
    scales = np.exp2(scales[:, :-(-a.shape[1] // 32)].astype(np.float64) - 127.0)
    y, ey = _products(_unscaled(codes), scales, *down)
    wide = np.abs(down[0]) * np.repeat(down[1], 32, 1)[:, :down[0].shape[1]]
    ey = ey + 1.01 * eh @ wide.T   # what the other codes add to the sums, to their cuts and roundings
    return y, ey + HALF_BF16 * (np.abs(y) + ey) + 2.0 ** -133


def _gpu(a):
    return torch.from_numpy(a).cuda()


def _check(layer, rng, T, E, k, shared, skew=0.0):
    d = layer.m.d
    codes, scales = _exact_rows(rng, T, d)
    x, xs = _as_rows(codes, scales)
    offsets, src = _rows(rng, T, E, k, skew)
    args = (_gpu(codes).view(torch.float8_e4m3fn), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
    first = None
    for shape in (0, 1, 2):
        layer.m.set_ffn_shape(shape)
        y, ysh = layer.m.expert_ffn_quant_rows(*args)
        torch.cuda.synchronize()
        if first is None:
            first = (y, ysh)
            for e in range(E):
                if offsets[e] == offsets[e + 1]:
                    continue
                some = np.arange(offsets[e], offsets[e + 1])
                some = some if len(some) <= 40 else np.r_[some[:3], np.sort(rng.choice(some, 30, replace=False)), some[-3:]]
                want, bound = _ffn(x[src[some]], xs[src[some]], *[w[e] for w in layer.w[:3]])
                assert (np.abs(y[some].double().cpu().numpy() - want) <= bound).all(), e
            for i in range(shared):
                some = np.arange(T) if T <= 40 else np.r_[0:3, np.sort(rng.choice(T, 30, replace=False)), T - 3:T]
                want, bound = _ffn(x[some], xs[some], *[w[i] for w in layer.w[3:]])
                assert (np.abs(ysh[i][some].double().cpu().numpy() - want) <= bound).all(), i
        else:   # these sums are exact in every form
            assert torch.equal(y[:len(src)], first[0][:len(src)]), shape
            assert ysh is None or torch.equal(ysh, first[1]), shape
    layer.m.set_ffn_shape(0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 33, 64, 129, 300])
@pytest.mark.parametrize("d,E,F,shared,F_shared,k", [(64, 4, 32, 0, 0, 2), (160, 5, 96, 2, 64, 3), (32, 1, 32, 1, 32, 1),
                                                     (288, 8, 224, 1, 160, 2), (128, 3, 256, 3, 32, 1)])
def test_experts_on_8_bit_rows(T, d, E, F, shared, F_shared, k):
    rng = np.random.default_rng(T * 1000 + d)
    _check(_Layer(rng, d, E, F, shared, F_shared, k), rng, T, E, k, shared)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [32, 64, 96, 128, 160, 256, 288, 384, 512, 544, 640, 672, 768, 896, 1024, 1056])
@pytest.mark.parametrize("T", [3, 40, 200])
def test_every_length_of_the_k_loop(T, K):
    rng = np.random.default_rng(T * 10000 + K)
    _check(_Layer(rng, K, 3, 64, k=2), rng, T, 3, 2, 0)
    _check(_Layer(rng, 64, 3, K, 1, K, k=2), rng, T, 3, 2, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("E,T", [(130, 3), (130, 200), (256, 16), (256, 900)])
def test_more_than_one_wavefront_of_groups(E, T):
    rng = np.random.default_rng(E + T)
    _check(_Layer(rng, 64, E, 32, 1, 32, 3), rng, T, E, 3, 1, skew=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 700, 3000])
def test_at_a_layer_shape(T):
    rng = np.random.default_rng(T)
    _check(_Layer(rng, 1280, 8, 896, 2, 896, 3), rng, T, 8, 3, 2, skew=0.7)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(1, 512), (3, 2048), (20, 1056), (200, 288)])
def test_few_rows_lose_nothing_before_they_are_rounded(T, d):
    """Fewer rows than for the wide tiles: nothing is cut off the products of gate and up, so the hidden codes are those of the 64-bit
    values but where these lie within fp32 sums of a border.  The down matrix hands them out: ones, one a row."""
    rng = np.random.default_rng(d)
    F, E = 256, 3
    v = rng.standard_normal((T, d)) * np.exp(0.3 * rng.standard_normal((T, 1)))
    codes, scales = _quantize(v)
    x, xs = _as_rows(codes, scales)
    small = int(round(np.log2(d) / 2)) + 1
    host = [_exact_weights(rng, E, F, d, small) for _ in range(2)]
    down = np.zeros((E, d, F), np.uint8)
    place = rng.permutation(d)[:F]
    down[:, place, np.arange(F)] = 2
    host.append((down, np.full((E, d, F // 32), 127, np.uint8)))
    shared = [(c[:1], s[:1]) for c, s in host]
    m = binding.FMoE(d_model=d, n_experts=E, d_ffn=F, n_shared=1, d_ffn_shared=F, k_text=2, k_visual=2, dtype="bf16")
    m.set_weights_quant_rows(*[(_gpu(_pack(c)), _gpu(s)) for c, s in host + shared])
    offsets, src = _rows(rng, T, E, 2)
    y, ysh = m.expert_ffn_quant_rows(_gpu(codes).view(torch.float8_e4m3fn), _gpu(scales), None, T, _gpu(offsets), _gpu(src))

    def check(rows, got, e):
        gate, up = [_matrix(c[e], s[e]) for c, s in host[:2]]
        (g, eg), (u, eu) = _products(x[rows], xs[rows], *gate, cuts=False), _products(x[rows], xs[rows], *up, cuts=False)
        a = _silu(g) * u
        ea = 1.1 * np.abs(u) * eg + np.abs(_silu(g)) * eu + 1.1 * eg * eu + 2.0 ** -20 * (1 + np.abs(g)) * np.abs(a)
        want, off = _slack(a, ea)
        got = got.double().cpu().numpy()[:, place]
        assert (np.abs(got - want) <= off).all()

    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        check(src[r], y[r], e)
    check(np.arange(T), ysh[0], 0)


@pytest.mark.gpu
def test_every_code_and_scale():
    """A single product per output: every e4m3 number with scales over the range, times every 4-bit code with its own."""
    rng = np.random.default_rng(3)
    d, E, F, T = 128, 1, 32, 254
    codes = np.zeros((T, d), np.uint8)
    numbers = np.r_[0:127, 128:255].astype(np.uint8)
    codes[np.arange(T), 37] = numbers
    gate, up, down = (np.zeros(s, np.uint8) for s in ((E, F, d), (E, F, d), (E, d, F)))
    sg, su, sd = (np.full(s, 127, np.uint8) for s in ((E, F, 4), (E, F, 4), (E, d, 1)))
    gate[:, :, 37] = 2
    up[:, :, 37] = np.arange(F) % 16
    su[:, :, 1] = 127 - 8 + np.arange(F) // 2
    down[0, np.arange(F), np.arange(F)] = np.arange(F) % 8 + 8 * (np.arange(F) // 8 % 2)
    m = binding.FMoE(d_model=d, n_experts=E, d_ffn=F, k_text=1, k_visual=1, dtype="bf16")
    w = [_matrix(c[0], s[0]) for c, s in ((gate, sg), (up, su), (down, sd))]
    m.set_weights_quant_rows(*[(_gpu(_pack(c)), _gpu(s)) for c, s in ((gate, sg), (up, su), (down, sd))])
    offsets, src = np.array([0, T], np.int32), np.arange(T, dtype=np.int32)
    for byte in (127, 100, 117, 130, 133):
        scales = np.full((T, 4), 127, np.uint8)
        scales[:, 1] = byte
        scales[:, [0, 2, 3]] = rng.integers(1, 254, (T, 3))   # of groups that are zero
        y, _ = m.expert_ffn_quant_rows(_gpu(codes), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
        want, bound = _ffn(*_as_rows(codes, scales), *w)
        assert (np.abs(y[:T].double().cpu().numpy() - want) <= bound).all(), byte


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 100])
def test_nan_reaches_its_own_rows_and_experts_only(T):
    rng = np.random.default_rng(9)
    layer = _Layer(rng, 160, 4, 96, 1, 64, 2)
    codes, scales = _exact_rows(rng, T, 160)
    offsets, src = _rows(rng, T, 4, 2)
    clean, clean_sh = layer.m.expert_ffn_quant_rows(_gpu(codes), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
    scales[1, 4] = 255
    codes[1, 128:] = 0
    codes[3, 7] = 0x7f
    y, ysh = layer.m.expert_ffn_quant_rows(_gpu(codes), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
    bad = torch.from_numpy(np.isin(src, [1, 3])).cuda()
    rows = y[:len(src)]
    assert rows[bad].isnan().all() and torch.equal(rows[~bad], clean[:len(src)][~bad])
    keep = [t for t in range(T) if t not in (1, 3)]
    assert ysh[0, [1, 3]].isnan().all() and torch.equal(ysh[0, keep], clean_sh[0, keep])
    c, s = layer.pairs[1]
    s = s.clone()
    s[2, 5, 1] = 255
    layer.m.set_weights_quant_rows(layer.pairs[0], (c, s), *layer.pairs[2:])
    codes, scales = _exact_rows(np.random.default_rng(10), T, 160)
    y, ysh = layer.m.expert_ffn_quant_rows(_gpu(codes), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
    expert = np.repeat(np.arange(4), np.diff(offsets))
    nan = y[:len(src)].isnan().cpu().numpy()
    assert nan[expert == 2].all() and not nan[expert != 2].any() and not ysh.isnan().any()


# The first product of the form for many rows an expert takes each code in one piece, and cuts (see _products)


def _real_layer(rng, d, E, F, shared, F_shared, k):
    """Random weights of the usual sizes: what they and the rows add up to, and what is cut, is not exact."""
    shapes = [(E, F, d), (E, F, d), (E, d, F)] + ([(shared, F_shared, d)] * 2 + [(shared, d, F_shared)] if shared else [])
    host = [(rng.integers(0, 16, s).astype(np.uint8), (125 - int(round(np.log2(s[2]) / 2)) + rng.integers(-1, 2, (*s[:2], -(-s[2] // 32)))).astype(np.uint8))
            for s in shapes]
    m = binding.FMoE(d_model=d, n_experts=E, d_ffn=F, n_shared=shared, d_ffn_shared=F_shared, k_text=k, k_visual=k, dtype="bf16")
    m.set_weights_quant_rows(*[(_gpu(_pack(c)), _gpu(s)) for c, s in host])
    return m, [[_matrix(c[g], s[g]) for g in range(len(c))] for c, s in host]


def _check_real(m, w, rng, T, E, k, codes, scales, skew=0.0, most=24):
    x, xs = _as_rows(codes, scales)
    offsets, src = _rows(rng, T, E, k, skew)
    y, ysh = m.expert_ffn_quant_rows(_gpu(codes).view(torch.float8_e4m3fn), _gpu(scales), None, T, _gpu(offsets), _gpu(src))
    torch.cuda.synchronize()
    pick = lambda n: np.arange(n) if n <= most else np.unique(np.r_[:2, rng.choice(n, most - 4, replace=False), n - 2:n])  # noqa: E731
    for e in range(E):
        r = offsets[e] + pick(offsets[e + 1] - offsets[e])
        want, bound = _ffn(x[src[r]], xs[src[r]], *[v[e] for v in w[:3]])
        assert (np.abs(y[r].double().cpu().numpy() - want) <= bound).all(), e
    for i in range(len(w[3]) if len(w) > 3 else 0):
        r = pick(T)
        want, bound = _ffn(x[r], xs[r], *[v[i] for v in w[3:]])
        assert (np.abs(ysh[i][r].double().cpu().numpy() - want) <= bound).all(), i


def _force(monkeypatch, shape):
    """Every layer that is made from now on takes the form for few (1) or for many rows an expert (2)."""
    made = binding.FMoE

    def of_shape(**kw):
        m = made(**kw)
        m.set_ffn_shape(shape)
        return m

    monkeypatch.setattr(binding, "FMoE", of_shape)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("T,d,F", [(3, 64, 32), (130, 288, 96), (40, 1056, 224), (300, 512, 160)])
def test_rows_of_all_sizes_in_either_form(T, d, F, shape):
    """Rows as the norm rounds them, with groups and elements of very different sizes among neighbours, so that products are cut."""
    rng = np.random.default_rng(T + d + shape)
    m, w = _real_layer(rng, d, 3, F, 1, 64, 2)
    m.set_ffn_shape(shape)
    v = rng.standard_normal((T, d)) * np.exp(0.5 * rng.standard_normal((T, 1))) * np.exp2(-rng.integers(0, 12, (T, d)) * (rng.random((T, d)) < 0.5))
    _check_real(m, w, rng, T, 3, 2, *_quantize(v))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [1, 2])
def test_every_code_and_scale_in_either_form(shape, monkeypatch):
    _force(monkeypatch, shape)
    test_every_code_and_scale()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [1, 2])
@pytest.mark.parametrize("T", [5, 300])
def test_nan_reaches_its_own_rows_and_experts_only_in_either_form(T, shape, monkeypatch):
    _force(monkeypatch, shape)
    test_nan_reaches_its_own_rows_and_experts_only(T)


@pytest.mark.gpu
def test_many_rows_reach_their_form_unforced():
    """Sizes that the rule gives to the form for many rows: 300 items of 128 rows and more, 64 rows an expert and more."""
    rng = np.random.default_rng(77)
    T, d, E, F, k = 9000, 512, 24, 1408, 2
    assert T * k >= 64 * E and (E + T * k // 128) * min(-(-F // 128), -(-d // 256)) >= 300
    m, w = _real_layer(rng, d, E, F, 1, 96, k)
    codes, scales = _quantize(rng.standard_normal((T, d)))
    _check_real(m, w, rng, T, E, k, codes, scales, skew=0.5, most=8)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("T,k", [(700, 0), (1500, 1)])
def test_shared_experts_see_far_more_rows_than_the_others(T, k, shape):
    """Shared experts alone, and beside 64 experts that have a few rows each."""
    rng = np.random.default_rng(T + shape)
    m, w = _real_layer(rng, 160, 64, 64, 2, 96, max(k, 1))
    m.set_ffn_shape(shape)
    codes, scales = _quantize(rng.standard_normal((T, 160)))
    if k:
        _check_real(m, w, rng, T, 64, k, codes, scales, most=6)
        return
    m.set_topk(0, 0)
    x, xs = _as_rows(codes, scales)
    _, ysh = m.expert_ffn_quant_rows(_gpu(codes), _gpu(scales), None, T, None, None)
    r = np.r_[0:10, T // 2:T // 2 + 10, T - 10:T]
    for i in range(2):
        want, bound = _ffn(x[r], xs[r], *[v[i] for v in w[3:]])
        assert (np.abs(ysh[i][r].double().cpu().numpy() - want) <= bound).all(), i


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [1, 2])
def test_norm_router_experts_and_combine_together_in_either_form(shape, monkeypatch):
    _force(monkeypatch, shape)
    test_norm_router_experts_and_combine_together(300)


@pytest.mark.gpu
def test_indexes_counts_and_rows_behind():
    """Kept tokens by index, a device count below the capacity, experts without rows, and rows behind the last left alone."""
    rng = np.random.default_rng(8)
    T, E, d, F = 150, 6, 96, 64
    layer = _Layer(rng, d, E, F, 1, 32, 2)
    codes, scales = _exact_rows(rng, 400, d)
    x, xs = _as_rows(codes, scales)
    kept = np.sort(rng.choice(400, size=T, replace=False)).astype(np.int32)
    offsets, src = _rows(rng, 90, E, 2)
    lib, m = binding.load(), layer.m
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    cg, scg, kept_g, n_dev = _gpu(codes), _gpu(scales), _gpu(kept), torch.tensor([90], dtype=torch.int32, device="cuda")
    og, sg = _gpu(offsets), torch.zeros(2 * T, dtype=torch.int32, device="cuda")
    sg[:len(src)] = _gpu(src)
    for shape in (0, 1, 2):
        m.set_ffn_shape(shape)
        y = torch.full((2 * T, d), 9.0, dtype=torch.bfloat16, device="cuda")
        ysh = torch.full((1, T, d), 9.0, dtype=torch.bfloat16, device="cuda")
        need = m.workspace_bytes(T, 1)
        ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        assert lib.fmoe_expert_ffn_quant_rows(m._ctx, p(cg), p(scg), p(kept_g), T, p(n_dev), p(og), p(sg), p(y), p(ysh), p(ws),
                                              need, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        assert (y[len(src):] == 9.0).all() and (ysh[0, 90:] == 9.0).all() and (ws[need:] == 0xA5).all()
        for e in range(E):
            r = slice(offsets[e], offsets[e + 1])
            want, bound = _ffn(x[kept[src[r]]], xs[kept[src[r]]], *[w[e] for w in layer.w[:3]])
            assert (np.abs(y[r].double().cpu().numpy() - want) <= bound).all(), e
        want, bound = _ffn(x[kept[:90]], xs[kept[:90]], *[w[0] for w in layer.w[3:]])
        assert (np.abs(ysh[0, :90].double().cpu().numpy() - want) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [8, 120])
def test_malformed_offsets_and_lists(T):
    """Experts with malformed offsets are left out; the same token many times in a list; shared experts alone need no lists."""
    rng = np.random.default_rng(T)
    layer = _Layer(rng, 96, 4, 64, 1, 32, 2)
    codes, scales = _exact_rows(rng, T, 96)
    cg, sg = _gpu(codes), _gpu(scales)
    src = rng.integers(0, T, 2 * T).astype(np.int32)
    src[:T] = 3
    good = np.array([0, T, T, 2 * T - 1, 2 * T], np.int32)
    y, ysh = layer.m.expert_ffn_quant_rows(cg, sg, None, T, _gpu(good), _gpu(src))
    x, xs = _as_rows(codes, scales)
    for e in range(4):
        r = slice(good[e], good[e + 1])
        want, bound = _ffn(x[src[r]], xs[src[r]], *[w[e] for w in layer.w[:3]])
        assert (np.abs(y[r].double().cpu().numpy() - want) <= bound).all(), e
    bad = np.array([0, -5, T, 3 * T, 2 * T], np.int32)
    layer.m.expert_ffn_quant_rows(cg, sg, None, T, _gpu(bad), _gpu(src))
    torch.cuda.synchronize()
    layer.m.set_topk(0, 0)
    lib, m = binding.load(), layer.m
    out = torch.empty_like(ysh)
    ws = m.workspace(T, 1)
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.fmoe_expert_ffn_quant_rows(m._ctx, p(cg), p(sg), None, T, None, None, None, None, p(out), p(ws), ws.numel(),
                                          C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, ysh)


@pytest.mark.gpu
def test_two_streams_and_a_graph():
    """One context, two workspaces of the caller, two streams at once; a captured call replayed with other rows."""
    rng = np.random.default_rng(58)
    layer = _Layer(rng, 160, 8, 96, 1, 64, 2)
    lib, m = binding.load(), layer.m
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    jobs = []
    for T in (5, 300):
        codes, scales = (_gpu(v) for v in _exact_rows(rng, T, 160))
        offsets, src = (_gpu(v) for v in _rows(rng, T, 8, 2))
        ws = torch.empty(m.workspace_bytes(T, 1), dtype=torch.uint8, device="cuda")
        want = m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)
        out = [(torch.zeros_like(want[0]), torch.zeros_like(want[1])) for _ in range(6)]
        jobs.append((torch.cuda.Stream(), T, codes, scales, offsets, src, ws, out, want))
    torch.cuda.synchronize()
    for turn in range(6):
        for stream, T, codes, scales, offsets, src, ws, out, _ in jobs:
            y, ysh = out[turn]
            assert lib.fmoe_expert_ffn_quant_rows(m._ctx, p(codes), p(scales), None, T, None, p(offsets), p(src), p(y), p(ysh),
                                                  p(ws), ws.numel(), C.c_void_p(stream.cuda_stream)) == 0
    torch.cuda.synchronize()
    for *_, out, want in jobs:
        for y, ysh in out:
            assert torch.equal(y, want[0]) and torch.equal(ysh, want[1])
    stream, T, codes, scales, offsets, src, *_ = jobs[1]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        y, ysh = m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)
    for turn in range(3):
        new = _exact_rows(rng, T, 160)
        codes.copy_(torch.from_numpy(new[0]))
        scales.copy_(torch.from_numpy(new[1]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)
        assert torch.equal(y, want[0]) and torch.equal(ysh, want[1])


@pytest.mark.gpu
def test_both_registrations_side_by_side():
    """Weights for 8-bit rows leave those in force for the other calls alone, and the other way round."""
    rng = np.random.default_rng(4)
    layer = _Layer(rng, 96, 4, 64, 0, 0, 2)
    m, T = layer.m, 40
    codes, scales = (_gpu(v) for v in _exact_rows(rng, T, 96))
    offsets, src = (_gpu(v) for v in _rows(rng, T, 4, 2))
    y8, _ = m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)
    m.set_weights_quant(torch.zeros(4, 96, dtype=torch.bfloat16, device="cuda"), None, *layer.pairs)
    x = torch.randn(T, 96, device="cuda").to(torch.bfloat16)
    y16, _ = m.expert_ffn(x, None, T, offsets, src)
    assert torch.equal(m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)[0][:2 * T], y8[:2 * T])
    m.set_weights_quant_rows(*layer.pairs)
    assert torch.equal(m.expert_ffn(x, None, T, offsets, src)[0][:2 * T], y16[:2 * T])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 9, 260])
def test_norm_router_experts_and_combine_together(T):
    """A pre-norm layer on 8-bit rows as it is used: norm, routing, dispatch, products, combine with the residual; against the same
    steps in 64 bits on what the steps before gave."""
    rng = np.random.default_rng(T)
    d, E, F, k = 192, 8, 96, 3
    layer = _Layer(rng, d, E, F, 1, 64, k)
    m = layer.m
    to = lambda a, t=torch.bfloat16: torch.from_numpy(a.astype(np.float32)).to(t).cuda()  # noqa: E731
    x, delta, w = to(rng.standard_normal((T, d))), to(0.3 * rng.standard_normal((T, d))), to(1 + 0.2 * rng.standard_normal(d))
    h, n = binding.rms_norm(x, w, 1e-6, delta=delta)
    h2, codes, scales = binding.rms_norm_quant(x, w, 1e-6, delta=delta)
    assert torch.equal(h, h2)
    z = (n.float() @ to(rng.standard_normal((E, d)) / 14, torch.float32).T).contiguous()
    _, idx, gate = m.select_experts(binding.select_params(), z)
    offsets, src, inv = m.permute(idx, None, T)
    y, ysh = m.expert_ffn_quant_rows(codes, scales, None, T, offsets, src)
    out = m.combine(y, ysh, inv, gate, None, T, residual=h)
    v = _as_rows(codes.view(torch.uint8).cpu().numpy(), scales.cpu().numpy())
    idx, gate = idx.cpu().numpy(), gate.double().cpu().numpy()
    want, slack = _ffn(*v, *[q[0] for q in layer.w[3:]])
    sizes = np.abs(want)
    for e in range(E):
        y_e, s_e = _ffn(*v, *[q[e] for q in layer.w[:3]])
        g_e = (gate * (idx == e)).sum(1, keepdims=True)
        want, slack, sizes = want + g_e * y_e, slack + g_e * s_e, sizes + np.abs(g_e * y_e)
    want = want + h.double().cpu().numpy()
    slack = slack + 6 * U * (sizes + np.abs(want))   # six additions in fp32
    assert (np.abs(out[:T].double().cpu().numpy() - want) <= slack + HALF_BF16 * (np.abs(want) + slack)).all()


# ------------------------------------------------------------------------------------------------------------- refusals


def test_set_weights_quant_rows_refuses_bad_arguments():
    lib = binding.load()

    def ctx(**kw):
        base = dict(d_model=64, n_experts=4, d_ffn=32, n_shared=0, d_ffn_shared=0, k_text=2, k_visual=1, renormalize=1, dtype=1)
        base.update(kw)
        cfg = binding.FmoeConfig(*[base[f[0]] for f in binding.FmoeConfig._fields_])
        c = C.c_void_p()
        assert lib.fmoe_create(C.byref(c), C.byref(cfg), 0) == 0
        return c

    q = C.byref(binding.FmoeQuantTensor(0x1000, 0x2000))
    odd, none = C.byref(binding.FmoeQuantTensor(0x1008, 0x2000)), C.byref(binding.FmoeQuantTensor(0x1000, None))
    reg = lambda c, a=q, b=q, w=q, sa=None, sb=None, sw=None: lib.fmoe_set_weights_quant_rows(c, a, b, w, sa, sb, sw, None)  # noqa: E731
    c = ctx()
    assert reg(None) == -2 and reg(c, a=None) == -2 and reg(c, b=odd) == -1 and reg(c, w=none) == -2 and reg(c, sa=q) == -3
    for bad in (dict(dtype=0), dict(d_model=72), dict(d_ffn=40), dict(n_shared=1, d_ffn_shared=24), dict(d_model=1 << 17, d_ffn=1 << 15)):
        assert reg(ctx(**bad), sa=q if "n_shared" in bad else None, sb=q if "n_shared" in bad else None,
                   sw=q if "n_shared" in bad else None) == -5, bad
        assert lib.fmoe_last_error() != b""
    assert reg(ctx(n_shared=1, d_ffn_shared=32)) == -2
    d = C.c_void_p(0x1000)
    run = lambda c=c, x=d, s=d, T=4, o=d, p=d, y=d, ws=d: lib.fmoe_expert_ffn_quant_rows(c, x, s, None, T, None, o, p, y, None, ws, 1 << 30, None)  # noqa: E731
    assert run(c=None) == -2 and run(T=-1) == -1 and run(T=1 << 24) == -5
    assert run() == -1 and b"fmoe_set_weights_quant_rows" in lib.fmoe_last_error()   # nothing registered


def test_build_check_catches_operands_written_just_before(tmp_path):
    from paper_2511_17885_amd import build
    mfma = "\t;;#ASMSTART\n\tv_mfma_f32_16x16x32_bf16 a[0:3], v[8:11], v[4:7], a[0:3]\n\t;;#ASMEND\n"
    good = ["\tv_mov_b32_e32 v12, v1\n", "\tv_add_u32_e32 v5, v1, v2\n\ts_nop 1\n", "\tds_read_b128 v[4:7], v1\n",
            "\tv_mov_b32_e32 v9, v1\n\ts_nop 0\n\ts_add_i32 s1, s1, s2\n"]
    bad = ["\tv_mov_b32_e32 v9, v1\n", "\tv_add_u32_e32 v5, v1, v2\n\ts_nop 0\n", "\tv_mov_b32_e32 v4, v1\n.LBB0_1:\n\ts_add_i32 s1, s1, s2\n"]
    p = tmp_path / "a.s"
    for before in good:
        p.write_text(before + mfma)
        assert build.check_matrix_operands(str(p)) == 1
    for before in bad:
        p.write_text(before + mfma)
        with pytest.raises(RuntimeError, match="written just before"):
            build.check_matrix_operands(str(p))


def test_build_check_follows_branches_and_exchanges(tmp_path):
    """Both operands of an exchange are written; what a block is entered with by a branch counts, over one or two of them."""
    from paper_2511_17885_amd import build
    mfma = ("\t;;#ASMSTART\n\tv_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[4:7], v[8:15], a[0:3], v16, v17 cbsz:4\n\t;;#ASMEND\n\ts_endpgm\n")
    good = ["\tv_permlane32_swap_b32_e32 v1, v2\n", "\tv_permlane32_swap_b32_e32 v1, v9\n\ts_nop 1\n",
            "\tv_mov_b32_e32 v9, v1\n\ts_nop 0\n\ts_cbranch_scc0 .L1\n\ts_nop 1\n.L1:\n",
            "\tv_mov_b32_e32 v9, v1\n\ts_branch .L2\n.L1:\n",                 # leads elsewhere
            "\tv_mov_b32_e32 v9, v1\n\ts_endpgm\n.L1:\n",
            ".L1:\n\tv_mov_b32_e32 v9, v1\n\ts_nop 1\n"]
    bad = ["\tv_permlane32_swap_b32_e32 v1, v9\n", "\tv_permlane16_swap_b32_e32 v9, v1\n\ts_nop 0\n", "\tv_swap_b32 v1, v17\n",
           "\tv_mov_b32_e32 v9, v1\n\ts_cbranch_scc0 .L1\n\ts_nop 1\n.L1:\n",
           "\tv_mov_b32_e32 v9, v1\n\ts_branch .L1\n\ts_nop 1\n.L1:\n",
           "\ts_branch .L3\n.L1:\n\ts_branch .L2\n.L3:\n\tv_mov_b32_e32 v16, v1\n.L4:\n\ts_branch .L2\n\ts_nop 1\n.L2:\n",
           "\ts_cbranch_vccnz .L1\n\ts_nop 1\n.L2:\n" + mfma + ".L1:\n\tv_mov_b32_e32 v9, v1\n\ts_branch .L2\n"]   # backwards
    p = tmp_path / "a.s"
    for before in good:
        p.write_text(before + mfma)
        assert build.check_matrix_operands(str(p)) == 1
    for before in bad:
        p.write_text(before + mfma)
        with pytest.raises(RuntimeError, match="written just before"):
            build.check_matrix_operands(str(p))


def test_rows_past_32_bit_offsets_are_refused():
    m = binding.FMoE(d_model=64, n_experts=2, d_ffn=64, k_text=1, k_visual=1, dtype="bf16")
    codes = torch.empty((1 << 26, 64), dtype=torch.uint8, device="meta")
    with pytest.raises(ValueError, match="32-bit"):
        m.expert_ffn_quant_rows(codes, codes, codes, 1, codes, codes)


def test_indexes_of_other_types_and_sizes_are_refused(monkeypatch):
    """Offsets as cumsum gives them (int64) are not pairs of int32 numbers, and a list is not read past its end."""
    m = object.__new__(binding.FMoE)
    m._ctx, m.device = None, torch.device("cpu")
    m.cfg = binding.FmoeConfig(64, 4, 32, 0, 0, 2, 1, 1, 1)
    m.lib = type("Lib", (), {"fmoe_expert_ffn_quant_rows": None, "fmoe_expert_ffn": staticmethod(lambda *a: 0)})
    m.workspace = lambda *a: torch.empty(256, dtype=torch.uint8)
    calls = []
    monkeypatch.setattr(binding, "_call", lambda *a: calls.append(a))
    monkeypatch.setattr(binding, "_stream", lambda: None)
    m.torch_dtype = torch.bfloat16
    codes, scales, x = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8), torch.zeros(8, 64, dtype=torch.bfloat16)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    good = {"kept_idx": i32(6), "n_kept": 6, "expert_offsets": i32(5), "perm_src": i32(12), "n_kept_dev": i32(1)}
    m.expert_ffn_quant_rows(codes, scales, **good)
    m.expert_ffn_quant_rows(codes, scales, **dict(good, kept_idx=None, n_kept_dev=None))
    m.expert_ffn(x, **good)
    assert len(calls) == 2
    for name, least in (("kept_idx", 6), ("expert_offsets", 5), ("perm_src", 12), ("n_kept_dev", 1)):
        for bad in (i32(least).long(), i32(least).float(), i32(2 * least + 2)[::2], i32(least).to("meta"), i32(least - 1)):
            with pytest.raises(ValueError, match=name):
                m.expert_ffn_quant_rows(codes, scales, **dict(good, **{name: bad}))
            if name != "perm_src" or bad.numel() >= least:   # (there the offsets say how many)
                with pytest.raises(ValueError, match=name):
                    m.expert_ffn(x, **dict(good, **{name: bad}))
    assert len(calls) == 2
    m.cfg.k_text = m.cfg.k_visual = 0                        # shared experts alone need no lists
    m.expert_ffn_quant_rows(codes, scales, None, 6, None, None)
    assert len(calls) == 3


@pytest.mark.gpu
def test_expert_ffn_quant_rows_refuses_bad_arguments():
    rng = np.random.default_rng(1)
    layer = _Layer(rng, 64, 4, 32, 1, 32, 2)
    lib, m = binding.load(), layer.m
    d, odd = 0x1000, 0x1002
    run = lambda x=d, s=d, T=4, o=d, p=d, y=d, ysh=d, ws=0x10000, nb=1 << 30: lib.fmoe_expert_ffn_quant_rows(  # noqa: E731
        m._ctx, x, s, None, T, None, o, p, y, ysh, ws, nb, None)
    assert run(x=None) == -2 and run(s=None) == -2 and run(o=None) == -2 and run(p=None) == -2 and run(y=None) == -2 and run(ysh=None) == -2
    assert run(x=odd) == -1 and run(s=odd) == -1 and run(y=odd) == -1 and run(ysh=odd) == -1
    assert run(ws=None) == -4 and run(ws=0x10010) == -4 and run(nb=16) == -4 and run(T=0, x=None) == 0
    codes, scales = (_gpu(v) for v in _exact_rows(rng, 4, 64))
    offsets, src = (_gpu(v) for v in _rows(rng, 4, 4, 2))
    for bad in ((codes[:, :32], scales), (codes, scales[:, :2]), (codes, scales[:3]), (codes.cpu(), scales), (codes, scales.cpu())):
        with pytest.raises(ValueError):
            m.expert_ffn_quant_rows(*bad, None, 4, offsets, src)
    with pytest.raises(ValueError):
        m.expert_ffn_quant_rows(codes, scales, None, 5, offsets, src)
    with pytest.raises(TypeError):
        m.expert_ffn_quant_rows(codes.float(), scales, None, 4, offsets, src)
    with pytest.raises(ValueError):
        m.set_weights_quant_rows(layer.pairs[1][:1] + layer.pairs[2][1:], *layer.pairs[1:])
