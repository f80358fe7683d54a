"""Weights in 4 bits: the conversions, the expert products with them, and a layer that routes from logits and runs on them,
against plain implementations in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_17885_amd import binding

U = 2.0 ** -24
HALF_BF16 = 2.0 ** -8
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# --------------------------------------------------------------------------------------------------- the definition


def _group_scale(a, saturate):
    """Scale byte of a group whose largest magnitude is a (numbers as they are defined, no bits)."""
    if not np.isfinite(a):
        return 255
    if a == 0.0:
        return 127
    n = int(np.floor(np.log2(a)))
    while 2.0 ** (n + 1) <= a:
        n += 1
    while 2.0 ** n > a:
        n -= 1
    e = n - 2
    if not saturate and a > 6.0 * 2.0 ** e:
        e += 1
    return max(e, -126) + 127


def _nearest_code(v, scale):
    t = abs(float(v)) / scale
    best = min(range(8), key=lambda c: (abs(t - GRID[c]) if t < 16 else 8 - c, c % 2))
    return best | (8 if np.signbit(v) else 0)


def _quantize(w, saturate):
    rows, K = w.shape
    groups = -(-K // 32)
    codes = np.zeros((rows, K), np.uint8)
    scales = np.zeros((rows, groups), np.uint8)
    for r in range(rows):
        for g in range(groups):
            part = w[r, 32 * g:32 * g + 32].astype(np.float64)
            scales[r, g] = _group_scale(np.abs(part).max() if np.isfinite(part).all() else np.inf, saturate)
            if scales[r, g] != 255:
                codes[r, 32 * g:32 * g + 32] = [_nearest_code(v, 2.0 ** (int(scales[r, g]) - 127)) for v in part]
    return codes, scales


def _values(codes, scales):
    """float64 [.., K] of unpacked codes [.., K] and scale bytes [.., groups]."""
    sign = np.where(codes & 8, -1.0, 1.0)
    scale = np.exp2(scales.astype(np.float64) - 127.0)
    return sign * GRID[codes & 7] * np.repeat(scale, 32, axis=-1)[..., :codes.shape[-1]]


def _unpack(codes):
    codes = codes.cpu().numpy()
    return np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)


def _pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


# -------------------------------------------------------------------------------------------------------- conversions


@pytest.mark.gpu
@pytest.mark.parametrize("saturate", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,K", [(1, 8), (3, 40), (5, 32), (2, 24), (7, 64), (4, 1288 // 8 * 8), (65, 96)])
def test_quantize(rows, K, dtype, saturate):
    rng = np.random.default_rng(rows * 1000 + K)
    w = torch.from_numpy((0.02 * rng.standard_normal((rows, K)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)).to(dtype)
    codes, scales = binding.quantize_weights(w.cuda(), saturate=saturate)
    assert codes.shape == (rows, K // 2) and scales.shape == (rows, -(-K // 32))
    want_c, want_s = _quantize(w.float().numpy(), saturate)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(_unpack(codes), want_c)
    for out in (torch.bfloat16, torch.float32):
        back = binding.dequantize_weights(codes, scales, dtype=out)
        assert back.dtype == out and np.array_equal(back.double().cpu().numpy(), _values(want_c, want_s))


@pytest.mark.gpu
@pytest.mark.parametrize("saturate", [False, True])
def test_quantize_edges_of_the_codes(saturate):
    """Values on and beside every middle of two codes, at scales over fp32's whole range, subnormals among them; zeros,
    infinities, NaN, signs of zero."""
    rows = []
    for n in (-149, -140, -127, -126, -125, -60, 0, 60, 124, 125):
        top = np.float32(2.0 ** n) * np.float32(4.0) if n <= 125 else np.float32(2.0 ** n)
        mids = [(GRID[i] + GRID[i + 1]) / 2 * 2.0 ** n for i in range(7)]
        vals = []
        for v in mids:
            f = np.float32(v)
            vals += [f, np.nextafter(f, np.float32(np.inf)), np.nextafter(f, np.float32(0)), -f]
        rows.append(np.array((vals + [top] * 4)[:32], np.float32))
    for big in (1.0, 1.5, np.nextafter(np.float32(1.5), np.float32(2)), 1.75, np.nextafter(np.float32(2), np.float32(0)), 2.0):
        r = np.zeros(32, np.float32)
        r[5], r[6], r[7] = big, -big, np.float32(big) / 8
        rows.append(r)
    rows += [np.zeros(32, np.float32), -np.zeros(32, np.float32), np.full(32, np.finfo(np.float32).max, np.float32),
             np.full(32, 2.0 ** -149, np.float32)]
    for v in (np.inf, -np.inf, np.nan):
        r = np.linspace(-1, 1, 32).astype(np.float32)
        r[31] = v
        rows.append(r)
    w = np.stack(rows)
    codes, scales = binding.quantize_weights(torch.from_numpy(w).cuda(), saturate=saturate)
    want_c, want_s = _quantize(w, saturate)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(_unpack(codes), want_c)
    back = binding.dequantize_weights(codes, scales, dtype=torch.float32).cpu().numpy()
    with np.errstate(over="ignore"):
        want = _values(want_c, want_s).astype(np.float32)
    assert np.isnan(back[-3:]).all() and np.array_equal(back[:-3], want[:-3])


@pytest.mark.gpu
def test_every_code_with_every_scale_and_every_bf16_value():
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None].repeat(255, 0)
    scales = np.arange(255, dtype=np.uint8)[:, None]
    with np.errstate(over="ignore"):
        want = _values(codes, scales).astype(np.float32)
    for dtype in (torch.bfloat16, torch.float32):
        got = binding.dequantize_weights(torch.from_numpy(_pack(codes)).cuda(), torch.from_numpy(scales).cuda(), dtype=dtype)
        assert np.array_equal(got.float().cpu().numpy(), want)
    # each of 2^16 bf16 values beside a group's largest 5 * 2^n, which fixes the scale at 2^n, where it is not larger itself
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16)
    v = v[torch.isfinite(v)]
    for n in (-20, 0, 90):
        w = torch.zeros(len(v), 32, dtype=torch.bfloat16)
        w[:, 0], w[:, 7] = v, 5.0 * 2.0 ** n
        codes, scales = binding.quantize_weights(w.cuda(), saturate=True)
        got = binding.dequantize_weights(codes, scales).double().cpu().numpy()[:, 0]
        a = v.double().numpy()
        scale = np.exp2(scales.cpu().numpy()[:, 0].astype(np.float64) - 127)
        t = np.abs(a) / scale
        grid = np.where(t < 2, np.round(t * 2) / 2, np.where(t < 4, np.round(t), np.minimum(np.round(t / 2) * 2, 6)))
        inside = np.abs(a) <= 5.0 * 2.0 ** n
        assert (scale[inside] == 2.0 ** n).all()
        assert np.array_equal(got, np.copysign(grid * scale, a))


@pytest.mark.gpu
def test_quantize_writes_nothing_past_its_outputs():
    lib = binding.load()
    rows, K = 9, 40
    w = torch.randn(rows, K, device="cuda")
    codes = torch.full((rows * K // 2 + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * 2 + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.fmoe_quantize_weights(p(w), 0, rows, K, 1, p(codes), p(scales), stream) == 0
    back = torch.full((rows * K + 64,), 7.0, device="cuda")
    assert lib.fmoe_dequantize_weights(p(codes), p(scales), rows, K, 0, p(back), stream) == 0
    torch.cuda.synchronize()
    assert (codes[rows * K // 2:] == 0xAB).all() and (scales[rows * 2:] == 0xAB).all() and (back[rows * K:] == 7.0).all()


@pytest.mark.gpu
def test_quantize_shapes_of_a_layer_and_no_rows():
    w = torch.randn(3, 5, 48, device="cuda")
    codes, scales = binding.quantize_weights(w)
    assert codes.shape == (3, 5, 24) and scales.shape == (3, 5, 2)
    flat = binding.quantize_weights(w.view(15, 48))
    assert torch.equal(codes.view(15, 24), flat[0]) and torch.equal(scales.view(15, 2), flat[1])
    none = binding.quantize_weights(torch.empty(0, 48, device="cuda"))
    assert none[0].shape == (0, 24) and binding.dequantize_weights(*none).shape == (0, 48)


# ---------------------------------------------------------------------------------------------------- expert products


def _random_quant(rng, *shape, spread=1.0):
    """Codes of all kinds and scales over some octaves around 0.02 / 3."""
    *lead, K = shape
    codes = rng.integers(0, 16, size=shape).astype(np.uint8)
    scales = (127 - 8 + rng.integers(0, 1 + int(3 * spread), size=(*lead, -(-K // 32)))).astype(np.uint8)
    return codes, scales


class _Layer:
    """A layer with 4-bit weights on the GPU, its matrices in 64 bits, and the same layer with dequantized bf16 weights."""

    def __init__(self, rng, d, E, F, shared=0, F_shared=0, k_text=2, k_visual=2, router=None, plain=True):
        shapes = [(E, F, d), (E, F, d), (E, d, F)] + ([(shared, F_shared, d)] * 2 + [(shared, d, F_shared)] if shared else [])
        host = [_random_quant(rng, *s) for s in shapes]
        self.w = [_values(*h) for h in host]
        self.pairs = [(torch.from_numpy(_pack(c)).cuda(), torch.from_numpy(s).cuda()) for c, s in host]
        self.router = (0.05 * torch.from_numpy(rng.standard_normal((E, d)).astype(np.float32))).to(torch.bfloat16).cuda() if router is None else router
        kw = dict(d_model=d, n_experts=E, d_ffn=F, n_shared=shared, d_ffn_shared=F_shared, k_text=k_text, k_visual=k_visual, dtype="bf16")
        self.m = binding.FMoE(**kw)
        self.m.set_weights_quant(self.router, None, *self.pairs)
        if plain:
            self.bf16 = binding.FMoE(**kw)
            dense = [binding.dequantize_weights(*p) for p in self.pairs]
            self.bf16.set_weights(self.router, None, *dense)


def _silu(v):
    return v / (1.0 + np.exp(-v))


def _ffn(x, gate, up, down):
    """y and how far a correct kernel may be from it, per element.  Sums of K products in fp32: K roundings of at most the sum
    of magnitudes, and one each for what the matrix instruction adds inside.  silu: 2^-20 (1 + |g|) relative (exponential and
    reciprocal of the hardware).  h is rounded to bf16 (half a step), then y."""
    g, u = x @ gate.T, x @ up.T
    eg = 2 * gate.shape[1] * U * (np.abs(x) @ np.abs(gate).T)
    eu = 2 * gate.shape[1] * U * (np.abs(x) @ np.abs(up).T)
    h = _silu(g) * u
    eh = 1.1 * np.abs(u) * eg + np.abs(_silu(g)) * eu + 2.0 ** -20 * (1 + np.abs(g)) * np.abs(h) + eg * eu
    eh = eh + HALF_BF16 * (np.abs(h) + eh) + 2.0 ** -133
    y = h @ down.T
    ey = eh @ np.abs(down).T + 2 * down.shape[1] * U * (np.abs(h) @ np.abs(down).T)
    return y, ey + HALF_BF16 * (np.abs(y) + ey) + 2.0 ** -133


def _rows(rng, T, E, k, skew=0.0):
    """Rows by expert, tokens ascending: (offsets [E+1], perm_src [T*k], rows)."""
    pop = np.exp(skew * rng.standard_normal(E))
    lists = [[] for _ in range(E)]
    for t in range(T):
        for e in rng.choice(E, size=k, replace=False, p=pop / pop.sum()):
            lists[e].append(t)
    offsets = np.concatenate([[0], np.cumsum([len(v) for v in lists])]).astype(np.int32)
    src = np.concatenate([np.array(v, np.int32) for v in lists] + [np.zeros(0, np.int32)])
    return offsets, src.astype(np.int32)


def _bf16(rng, *shape):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def _check_experts(layer, rng, T, E, k, shared, skew=0.0, shapes=(0, 1, 2)):
    x, x64 = _bf16(rng, T, layer.m.d)
    offsets, src = _rows(rng, T, E, k, skew)
    og, sg = torch.from_numpy(offsets).cuda(), torch.from_numpy(src).cuda()
    first = None
    for shape in shapes:
        layer.m.set_ffn_shape(shape)
        y, ysh = layer.m.expert_ffn(x, None, T, og, sg)
        torch.cuda.synchronize()
        if first is None:
            first = (y, ysh)
            for e in range(E):
                r = slice(offsets[e], offsets[e + 1])
                if offsets[e] == offsets[e + 1]:
                    continue
                want, bound = _ffn(x64[src[r]], *[w[e] for w in layer.w[:3]])
                diff = np.abs(y[r].double().cpu().numpy() - want)
                assert (diff <= bound).all(), (e, (diff / bound).max())
            for i in range(shared):
                want, bound = _ffn(x64, *[w[i] for w in layer.w[3:]])
                assert (np.abs(ysh[i].double().cpu().numpy() - want) <= bound).all(), i
        else:   # every form adds in the same order
            assert torch.equal(y[:len(src)], first[0][:len(src)]), shape
            assert ysh is None or torch.equal(ysh, first[1]), shape
    layer.m.set_ffn_shape(0)
    if hasattr(layer, "bf16"):
        want, want_sh = layer.bf16.expert_ffn(x, None, T, og, sg)
        assert torch.equal(first[0][:len(src)], want[:len(src)])
        assert want_sh is None or torch.equal(first[1], want_sh)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 33, 64, 129, 300])
@pytest.mark.parametrize("d,E,F,shared,F_shared,k", [(64, 4, 32, 0, 0, 2), (136, 5, 72, 2, 40, 3), (8, 1, 8, 1, 8, 1),
                                                     (264, 8, 200, 1, 96, 2)])
def test_experts(T, d, E, F, shared, F_shared, k):
    rng = np.random.default_rng(T * 7 + d)
    _check_experts(_Layer(rng, d, E, F, shared, F_shared, k, k), rng, T, E, k, shared, skew=0.7)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [8, 24, 32, 40, 64, 72, 128, 192, 256, 264, 320, 384, 448, 512, 520, 576, 640, 704, 768, 1032])
@pytest.mark.parametrize("T", [3, 40, 200])
def test_experts_every_length_of_the_k_loop(T, K):
    """Reductions of one to seventeen k tiles, ragged ends among them, in either product."""
    rng = np.random.default_rng(K * 3 + T)
    _check_experts(_Layer(rng, K, 2, 48, 0, 0, 1, 1), rng, T, 2, 1, 0)
    _check_experts(_Layer(rng, 56, 2, K, 1, K, 1, 1), rng, T, 2, 1, 1)


@pytest.mark.gpu
def test_experts_scales_far_apart_and_the_smallest():
    """Scale bytes over the whole range a bf16 context holds without overflow, codes 0 with every one of them."""
    rng = np.random.default_rng(3)
    layer = _Layer(rng, 64, 2, 32, 0, 0, 1, 1)
    x = torch.ones(8, 64, dtype=torch.bfloat16, device="cuda")
    offsets, src = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    for low, high in ((0, 3), (100, 150), (1, 140)):
        pairs = []
        for c, s in layer.pairs:
            pairs.append((c, torch.from_numpy(rng.integers(low, high, size=tuple(s.shape)).astype(np.uint8)).cuda()))
        layer.m.set_weights_quant(layer.router, None, *pairs)
        layer.bf16.set_weights(layer.router, None, *[binding.dequantize_weights(*p) for p in pairs])
        a, b = (m.expert_ffn(x, None, 8, offsets, src)[0] for m in (layer.m, layer.bf16))
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.gpu
def test_experts_nan_scale_reaches_its_own_expert_only():
    rng = np.random.default_rng(4)
    layer = _Layer(rng, 64, 2, 32, 0, 0, 1, 1, plain=False)
    pairs = [(c, s.clone()) for c, s in layer.pairs]
    pairs[0][1][1, 5, 0] = 255
    layer.m.set_weights_quant(layer.router, None, *pairs)
    x, _ = _bf16(rng, 8, 64)
    offsets, src = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    y = layer.m.expert_ffn(x, None, 8, offsets, src)[0].float()
    assert torch.isfinite(y[:4]).all() and torch.isnan(y[4:]).all()


@pytest.mark.gpu
def test_experts_indexes_counts_and_rows_behind():
    """Kept tokens by index, a device count below the capacity, experts without rows, and rows behind the last left alone."""
    rng = np.random.default_rng(8)
    T, E, d, F = 150, 6, 72, 40
    layer = _Layer(rng, d, E, F, 1, 24, 2, 2)
    x, x64 = _bf16(rng, 400, d)
    kept = np.sort(rng.choice(400, size=T, replace=False)).astype(np.int32)
    offsets, src = _rows(rng, 90, E, 2)
    lib, m = binding.load(), layer.m
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    kept_g, n_dev = torch.from_numpy(kept).cuda(), torch.tensor([90], dtype=torch.int32, device="cuda")
    og, sg = torch.from_numpy(offsets).cuda(), torch.zeros(2 * T, dtype=torch.int32, device="cuda")
    sg[:len(src)] = torch.from_numpy(src).cuda()
    for shape in (0, 1, 2):
        m.set_ffn_shape(shape)
        y = torch.full((2 * T, d), 9.0, dtype=torch.bfloat16, device="cuda")
        ysh = torch.full((1, T, d), 9.0, dtype=torch.bfloat16, device="cuda")
        ws = m.workspace(T, 1)
        assert lib.fmoe_expert_ffn(m._ctx, p(x), p(kept_g), T, p(n_dev), p(og), p(sg), p(y), p(ysh), p(ws), ws.numel(),
                                   C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        assert (y[len(src):] == 9.0).all() and (ysh[0, 90:] == 9.0).all()
        for e in range(E):
            r = slice(offsets[e], offsets[e + 1])
            want, bound = _ffn(x64[kept[src[r]]], *[w[e] for w in layer.w[:3]])
            assert (np.abs(y[r].double().cpu().numpy() - want) <= bound).all(), e
        want, bound = _ffn(x64[kept[:90]], *[w[0] for w in layer.w[3:]])
        assert (np.abs(ysh[0, :90].double().cpu().numpy() - want) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 700])
def test_experts_at_the_layer_shapes(T):
    """d 1280, 64 experts of 896 and two shared ones: against the bf16 kernels, bit for bit, in every form."""
    rng = np.random.default_rng(T)
    E, d, F = 64, 1280, 896
    pairs = []
    for s in [(E, F, d), (E, F, d), (E, d, F), (2, F, d), (2, F, d), (2, d, F)]:
        w = 0.02 * torch.randn(s, device="cuda")
        pairs.append(binding.quantize_weights(w))
    kw = dict(d_model=d, n_experts=E, d_ffn=F, n_shared=2, d_ffn_shared=F, k_text=6, k_visual=6, dtype="bf16")
    a, b = binding.FMoE(**kw), binding.FMoE(**kw)
    router = torch.zeros(E, d, dtype=torch.bfloat16, device="cuda")
    a.set_weights_quant(router, None, *pairs)
    b.set_weights(router, None, *[binding.dequantize_weights(*p) for p in pairs])
    x, _ = _bf16(rng, T, d)
    offsets, src = _rows(rng, T, E, 6, skew=1.0)
    og, sg = torch.from_numpy(offsets).cuda(), torch.from_numpy(src).cuda()
    want, want_sh = b.expert_ffn(x, None, T, og, sg)
    for shape in (0, 1, 2):
        a.set_ffn_shape(shape)
        y, ysh = a.expert_ffn(x, None, T, og, sg)
        assert torch.equal(y, want) and torch.equal(ysh, want_sh), shape


@pytest.mark.gpu
def test_weights_can_be_registered_again_in_either_form():
    rng = np.random.default_rng(12)
    layer = _Layer(rng, 64, 4, 32, 0, 0, 2, 2)
    x, _ = _bf16(rng, 20, 64)
    offsets, src = (torch.from_numpy(v).cuda() for v in _rows(rng, 20, 4, 2))
    quant = layer.m.expert_ffn(x, None, 20, offsets, src)[0]
    other = [torch.randn(s, device="cuda").mul_(0.1).to(torch.bfloat16) for s in ((4, 32, 64), (4, 32, 64), (4, 64, 32))]
    layer.m.set_weights(layer.router, None, *other)
    layer.bf16.set_weights(layer.router, None, *other)
    assert torch.equal(layer.m.expert_ffn(x, None, 20, offsets, src)[0], layer.bf16.expert_ffn(x, None, 20, offsets, src)[0])
    layer.m.set_weights_quant(layer.router, None, *layer.pairs)
    for c, s in layer.pairs:      # the context has copies
        torch.cuda.synchronize()
        c.zero_(); s.zero_()
    assert torch.equal(layer.m.expert_ffn(x, None, 20, offsets, src)[0], quant)


@pytest.mark.gpu
@pytest.mark.parametrize("E,T", [(130, 3), (130, 200), (256, 16), (256, 500)])
def test_experts_of_more_than_one_wavefront_of_groups(E, T):
    rng = np.random.default_rng(E + T)
    _check_experts(_Layer(rng, 40, E, 24, 1, 16, 4, 4), rng, T, E, 4, 1, skew=1.5)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [8, 24, 64, 72, 128, 192, 256, 264, 320, 384, 448, 520])
def test_experts_of_many_tiles_with_short_reductions(K):
    """Many experts of some tens of rows: either product with reductions of one to nine k tiles, against the bf16 kernels."""
    rng = np.random.default_rng(K)
    E, T, k = 256, 1300, 8
    for d, F in ((K, 48), (56, K)):
        layer = _Layer(rng, d, E, F, 1, F, k, k)
        x, _ = _bf16(rng, T, d)
        offsets, src = (torch.from_numpy(v).cuda() for v in _rows(rng, T, E, k, skew=0.8))
        want, want_sh = layer.bf16.expert_ffn(x, None, T, offsets, src)
        for shape in (0, 1, 2):
            layer.m.set_ffn_shape(shape)
            for _ in range(10):   # (a wait that is too short shows now and then)
                y, ysh = layer.m.expert_ffn(x, None, T, offsets, src)
                assert torch.equal(y, want) and torch.equal(ysh, want_sh), (d, F, shape)


@pytest.mark.gpu
def test_experts_of_row_lists_with_the_same_token_many_times():
    """Sixteen tokens, 32 rows of one expert: the form for a few tokens takes several turns; the row lists are the caller's."""
    rng = np.random.default_rng(55)
    layer = _Layer(rng, 72, 3, 40, 1, 24, 2, 2)
    x, _ = _bf16(rng, 16, 72)
    src = torch.from_numpy(rng.integers(0, 16, size=32).astype(np.int32)).cuda()
    src[:20] = 7
    for bounds in ([0, 0, 32, 32], [0, 17, 17, 32], [3, 3, 3, 32]):
        offsets = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        want = layer.bf16.expert_ffn(x, None, 16, offsets, src)
        for shape in (0, 1, 2):
            layer.m.set_ffn_shape(shape)
            got = layer.m.expert_ffn(x, None, 16, offsets, src)
            assert torch.equal(got[0][bounds[0]:], want[0][bounds[0]:]) and torch.equal(got[1], want[1]), (bounds, shape)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 16, 17, 200])
@pytest.mark.parametrize("d,shared,F_shared", [(72, 1, 40), (136, 2, 40), (264, 3, 136), (8, 1, 8)])
def test_shared_experts_alone_need_no_offsets(T, d, shared, F_shared):
    """No expert is listed (k 0): offsets, rows and y may be null.  The shared experts' column units (3 and 3, 5 and 10, 26 and
    27, 1 and 1 in the two products) are not whole eights, as a launch's workgroups are."""
    rng = np.random.default_rng(T + d)
    layer = _Layer(rng, d, 4, 32, shared, F_shared, 0, 0)
    x, x64 = _bf16(rng, T, d)
    _, want = layer.bf16.expert_ffn(x, None, T, None, None)
    lib, m = binding.load(), layer.m
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    for shape in (0, 1, 2):
        m.set_ffn_shape(shape)
        assert torch.equal(m.expert_ffn(x, None, T, None, None)[1], want), shape
        out = torch.full((shared, T, d), 9.0, dtype=torch.bfloat16, device="cuda")
        ws = m.workspace(T, 1)
        assert lib.fmoe_expert_ffn(m._ctx, p(x), None, T, None, None, None, None, p(out), p(ws), ws.numel(),
                                   C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        assert torch.equal(out, want), shape
    for i in range(shared):
        want64, bound = _ffn(x64, *[w[i] for w in layer.w[3:]])
        assert (np.abs(want[i].double().cpu().numpy() - want64) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [8, 120])
def test_experts_with_malformed_offsets_are_left_out(T):
    """Offsets below 0, past the room for rows or descending: the expert has no rows, the others are what they are."""
    rng = np.random.default_rng(56)
    layer = _Layer(rng, 64, 4, 32, 0, 0, 2, 2)
    x, _ = _bf16(rng, T, 64)
    src = torch.arange(2 * T, dtype=torch.int32, device="cuda") % T
    good = torch.tensor([0, 3, 6, 9, 12], dtype=torch.int32, device="cuda")
    for shape in (0, 1, 2):
        layer.m.set_ffn_shape(shape)
        want = layer.m.expert_ffn(x, None, T, good, src)[0][:12].clone()
        for bad, rows in (([0, 3, 6, 9, 2 * T + 1], slice(0, 9)), ([-5, 3, 6, 9, 12], slice(3, 12)), ([0, 3, 6, 1, 1], slice(0, 6))):
            got = layer.m.expert_ffn(x, None, T, torch.tensor(bad, dtype=torch.int32, device="cuda"), src)[0]
            assert torch.equal(got[rows], want[rows]), (shape, bad)


@pytest.mark.gpu
def test_scales_at_any_address_and_weights_inside_a_larger_tensor():
    rng = np.random.default_rng(57)
    layer = _Layer(rng, 64, 2, 32, 0, 0, 1, 1)
    x, _ = _bf16(rng, 9, 64)
    offsets, src = (torch.from_numpy(v).cuda() for v in _rows(rng, 9, 2, 1))
    want = layer.m.expert_ffn(x, None, 9, offsets, src)[0]
    moved = []
    for c, s in layer.pairs:
        room = torch.zeros(s.numel() + 3, dtype=torch.uint8, device="cuda")
        room[3:] = s.flatten()
        moved.append((c, room[3:].view(s.shape)))
        w = binding.dequantize_weights(c, moved[-1][1])
        assert torch.equal(w, binding.dequantize_weights(c, s))
    other = binding.FMoE(d_model=64, n_experts=2, d_ffn=32, k_text=1, k_visual=1, dtype="bf16")
    other.set_weights_quant(layer.router, None, *moved)
    assert torch.equal(other.expert_ffn(x, None, 9, offsets, src)[0], want)


@pytest.mark.gpu
def test_quantize_offsets_past_32_bits():
    """2.2 billion weights: the last rows come out as they do alone."""
    rows, K = 2_200_000, 1000
    w = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    w[-50:] = torch.randn(50, K, generator=gen, device="cuda").to(torch.bfloat16)
    codes, scales = binding.quantize_weights(w)
    c, s = binding.quantize_weights(w[-50:].clone())
    assert torch.equal(codes[-50:], c) and torch.equal(scales[-50:], s)
    assert (scales[:-50] == 127).all()
    back = binding.dequantize_weights(codes, scales)
    assert torch.equal(back[-50:], binding.dequantize_weights(c, s)) and not back[:-50].any()


@pytest.mark.gpu
def test_experts_on_two_streams_at_once():
    """Two contexts; one context with two workspaces of the caller."""
    rng = np.random.default_rng(58)
    layers = [_Layer(rng, 136, 8, 72, 1, 40, 2, 2, plain=False) for _ in range(2)]
    lib = binding.load()
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    streams, jobs = [torch.cuda.Stream() for _ in range(4)], []
    for i, T in enumerate((5, 90, 300, 16)):
        m = layers[i % 2].m
        x, _ = _bf16(rng, T, 136)
        offsets, src = (torch.from_numpy(v).cuda() for v in _rows(rng, T, 8, 2))
        ws = torch.empty(m.workspace_bytes(T, 1), dtype=torch.uint8, device="cuda")
        out = [(torch.zeros(2 * T, 136, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 136, dtype=torch.bfloat16, device="cuda"))
               for _ in range(6)]
        jobs.append((m, T, x, offsets, src, ws, out, m.expert_ffn(x, None, T, offsets, src)))
    torch.cuda.synchronize()
    for turn in range(6):
        for stream, (m, T, x, offsets, src, ws, out, _) in zip(streams, jobs):
            y, ysh = out[turn]
            assert lib.fmoe_expert_ffn(m._ctx, p(x), None, T, None, p(offsets), p(src), p(y), p(ysh), p(ws), ws.numel(),
                                       C.c_void_p(stream.cuda_stream)) == 0
    torch.cuda.synchronize()
    for *_, out, want in jobs:
        for y, ysh in out:
            assert torch.equal(y, want[0]) and torch.equal(ysh, want[1].view_as(ysh))


# --------------------------------------------------------------------------------------------------------- whole layers


@pytest.mark.gpu
@pytest.mark.parametrize("T_v,T_t", [(0, 3), (40, 9), (500, 20)])
def test_layer_and_stack_on_4_bit_weights_equal_the_dequantized_ones(T_v, T_t):
    rng = np.random.default_rng(T_v)
    layers = [_Layer(rng, 128, 8, 96, 1, 64, 3, 2) for _ in range(2)]
    T = T_v + T_t
    x, _ = _bf16(rng, T, 128)
    vis = torch.cat([torch.ones(T_v, dtype=torch.uint8), torch.zeros(T_t, dtype=torch.uint8)]).cuda()
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    for pp in (None, binding.prune_params(retention=0.5, window=3), binding.prune_params(retention=0.5, window=3, gamma=0.2)):
        (a, ka, ca, _), (b, kb, cb, _) = (m.layer_forward(x, vis, cu, pp, add_residual=True) for m in (layers[0].m, layers[0].bf16))
        n = int(ca[-1])
        assert torch.equal(ca, cb) and torch.equal(ka[:n], kb[:n]) and torch.equal(a[:n], b[:n])
    sched = [(3, 3), (3, 2)]
    outs = []
    for form in ("m", "bf16"):
        stack = binding.FMoEStack([getattr(l, form) for l in layers], sched, prune_after_layer=1, params=binding.prune_params(retention=0.5, window=3))
        outs.append(stack.forward(x, vis, cu, [T_v], [T_t]))
    assert all(torch.equal(p, q) for p, q in zip(*outs))


def _run_together(m, params, x, logits, vis, bias, T):
    scores, idx, gate = m.select_experts(params, logits, vis, select_bias=bias, want_scores=True)
    offsets, perm, inv = m.permute(idx, None, T)
    y, ysh = m.expert_ffn(x, None, T, offsets, perm)
    return m.combine(y, ysh, inv, gate, None, T, residual=x), scores, idx, gate


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 16, 77, 400])
def test_router_experts_and_combine_together(T):
    """Logits -> experts -> permutation -> 4-bit products -> combine, against the whole layer in 64 bits; then captured into
    a graph and replayed three times with eager work between."""
    rng = np.random.default_rng(T)
    E, d, F, k = 16, 136, 72, 4
    layer = _Layer(rng, d, E, F, 1, 48, k, 2)
    x, x64 = _bf16(rng, T, d)
    router = 0.1 * rng.standard_normal((E, d))
    logits = torch.from_numpy((x64 @ router.T).astype(np.float32)).cuda()
    bias = torch.from_numpy((0.1 * rng.standard_normal(E)).astype(np.float32)).cuda()
    vis = torch.from_numpy((rng.random(T) < 0.5).astype(np.uint8)).cuda()
    p = binding.select_params("sigmoid", n_groups=4, topk_groups=2, group_score=1, gate_scale=2.5)
    out, scores, idx, gate = _run_together(layer.m, p, x, logits, vis, bias, T)
    shared, shared_bound = _ffn(x64, *[w[0] for w in layer.w[3:]])
    g64, i64 = gate.double().cpu().numpy(), idx.cpu().numpy()
    want, bound = x64 + shared, shared_bound.copy()
    for t in range(T):
        for s in range(k):
            if i64[t, s] >= 0:
                y, ey = _ffn(x64[t:t + 1], *[w[i64[t, s]] for w in layer.w[:3]])
                want[t] += g64[t, s] * y[0]
                bound[t] += g64[t, s] * ey[0] + 8 * U * np.abs(g64[t, s] * y[0])
    bound = bound + 8 * U * np.abs(want) + HALF_BF16 * (np.abs(want) + bound)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _run_together(layer.m, p, x, logits, vis, bias, T)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run_together(layer.m, p, x, logits, vis, bias, T)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, scores, idx, gate)))
        _run_together(layer.m, p, 2 * x, -logits, vis, bias, T)
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_sigmoid_scores_feed_the_pruning():
    rng = np.random.default_rng(21)
    layer = _Layer(rng, 64, 8, 32, 0, 0, 2, 2, plain=False)
    logits = torch.from_numpy(rng.standard_normal((60, 8)).astype(np.float32)).cuda()
    scores, _, _ = layer.m.select_experts(binding.select_params("sigmoid"), logits, want_scores=True)
    vis = torch.ones(60, dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, 60], dtype=torch.int32, device="cuda")
    kept, new_cu, c = layer.m.prune(binding.prune_params(retention=0.5, window=3), scores, vis, cu, want_scores=True)
    assert int(new_cu[-1]) == 30
    s = scores.double().cpu().numpy().reshape(20, 3, 8)
    mean = s.mean(1, keepdims=True)
    want = ((s * mean).sum(2) / np.linalg.norm(s, axis=2) / np.linalg.norm(mean, axis=2)).mean(1)
    assert np.abs(c[:20].double().cpu().numpy() - want).max() <= 64 * U   # eight products, norms, three terms


# ------------------------------------------------------------------------------------------------------------- refusals


def _ctx(dtype=binding.FMOE_BF16, shared=0):
    ctx = C.c_void_p()
    cfg = binding.FmoeConfig(64, 4, 32, shared, 16 if shared else 0, 2, 1, 1, dtype)
    assert binding.load().fmoe_create(C.byref(ctx), C.byref(cfg), 0) == 0
    return ctx


def test_set_weights_quant_refuses_bad_arguments():
    lib = binding.load()
    d = C.c_void_p(0x1000)
    q = lambda codes=0x1000, scales=0x1001: C.byref(binding.FmoeQuantTensor(codes, scales))  # noqa: E731
    ctx = _ctx()
    call = lambda *w, router=d, bias=None, c=None: lib.fmoe_set_weights_quant(c or ctx, router, bias, *w, None)  # noqa: E731
    none = (None, None, None)
    assert call(q(), q(), None, *none) == -2 and call(q(), q(None), q(), *none) == -2 and call(q(), q(), q(0x1000, None), *none) == -2
    assert call(q(), q(), q(), *none, router=None) == -2
    assert call(q(), q(0x1004), q(), *none) == -1                                  # codes not aligned
    assert call(q(), q(), q(), *none, router=C.c_void_p(0x1008)) == -1
    assert call(q(), q(), q(), *none, bias=C.c_void_p(0x1004)) == -1
    assert call(q(), q(), q(), q(), None, None) == -3                              # shared weights without shared experts
    assert lib.fmoe_set_weights_quant(None, d, None, q(), q(), q(), *none, None) == -2
    # nothing was registered
    assert lib.fmoe_expert_ffn(ctx, d, None, 4, None, d, d, d, None, d, 0, None) == -1
    lib.fmoe_destroy(ctx)
    ctx = _ctx(shared=1)
    assert call(q(), q(), q(), *none) == -2 and call(q(), q(), q(), q(), q(), None) == -2
    lib.fmoe_destroy(ctx)
    ctx = _ctx(dtype=binding.FMOE_F32)
    assert call(q(), q(), q(), *none) == -5 and b"bf16" in lib.fmoe_last_error()
    lib.fmoe_destroy(ctx)
    # offsets inside a packed matrix are 32 bits wide
    for d_model, d_ffn, shared, d_shared in ((65536, 65536, 0, 0), (65536, 64, 2, 32768)):
        ctx = C.c_void_p()
        cfg = binding.FmoeConfig(d_model, 4, d_ffn, shared, d_shared, 2, 1, 1, binding.FMOE_BF16)
        assert lib.fmoe_create(C.byref(ctx), C.byref(cfg), 0) == 0
        assert call(*([q()] * (6 if shared else 3)), *(none if not shared else ())) == -5
        lib.fmoe_destroy(ctx)


def test_quantize_refuses_bad_arguments():
    lib = binding.load()
    d, odd = C.c_void_p(0x1000), C.c_void_p(0x1008)
    qu = lambda w=d, t=0, rows=4, K=64, c=d, s=d: lib.fmoe_quantize_weights(w, t, rows, K, 1, c, s, None)  # noqa: E731
    de = lambda w=d, t=0, rows=4, K=64, c=d, s=d: lib.fmoe_dequantize_weights(c, s, rows, K, t, w, None)  # noqa: E731
    for call in (qu, de):
        assert call(t=2) == -1 and call(rows=-1) == -1 and call(K=0) == -1 and call(K=-8) == -1
        assert call(K=60) == -5 and call(K=(1 << 24) + 8) == -5 and call(rows=1 << 36) == -5
        assert call(w=None) == -2 and call(c=None) == -2 and call(s=None) == -2
        assert call(w=odd) == -1 and call(c=odd) == -1
        assert call(rows=0, w=None, c=None, s=None) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    w = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        binding.quantize_weights(w.double())
    with pytest.raises(ValueError):
        binding.quantize_weights(torch.zeros(64, 4).t())
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    with pytest.raises(ValueError):
        binding.dequantize_weights(codes, scales[:, :1])
    with pytest.raises(ValueError):
        binding.dequantize_weights(codes, scales.int())
    with pytest.raises(ValueError):
        binding.dequantize_weights(codes.t(), scales)
    m = binding.FMoE(d_model=64, n_experts=4, d_ffn=32, k_text=2, k_visual=1, dtype="bf16")
    router = torch.zeros(4, 64, dtype=torch.bfloat16)
    pair = lambda *s: (torch.zeros(*s[:-1], s[-1] // 2, dtype=torch.uint8), torch.zeros(*s[:-1], s[-1] // 32, dtype=torch.uint8))  # noqa: E731
    good = [pair(4, 32, 64), pair(4, 32, 64), pair(4, 64, 32)]
    for i in range(3):
        bad = list(good)
        bad[i] = (good[i][0][:3].contiguous(), good[i][1])
        with pytest.raises(ValueError):
            m.set_weights_quant(router, None, *bad)
        bad[i] = (good[i][0], good[i][1][:, :-1].contiguous())
        with pytest.raises(ValueError):
            m.set_weights_quant(router, None, *bad)
    with pytest.raises(ValueError):
        m.set_weights_quant(router.float(), None, *good)
    with pytest.raises(ValueError):
        m.set_weights_quant(router, torch.zeros(3), *good)


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit_or_are_on_the_host():
    m = binding.FMoE(d_model=64, n_experts=4, d_ffn=32, k_text=2, k_visual=1, dtype="bf16")
    router = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    pair = lambda *s: (torch.zeros(*s[:-1], s[-1] // 2, dtype=torch.uint8, device="cuda"), torch.zeros(*s[:-1], s[-1] // 32, dtype=torch.uint8, device="cuda"))  # noqa: E731
    good = [pair(4, 32, 64), pair(4, 32, 64), pair(4, 64, 32)]
    m.set_weights_quant(router, None, *good)
    for i in range(3):
        c, s = good[i]
        for bad in ((c[:3].contiguous(), s), (c, s[:, :-1].contiguous()), (c.cpu(), s), (c, s.cpu()), (c.int(), s)):
            with pytest.raises(ValueError):
                m.set_weights_quant(router, None, *good[:i], bad, *good[i + 1:])
    for args in ((router.float(), None), (router.cpu(), None), (router, torch.zeros(3, device="cuda")), (router, torch.zeros(4))):
        with pytest.raises(ValueError):
            m.set_weights_quant(*args, *good)
    with pytest.raises(ValueError):
        binding.dequantize_weights(good[0][0], good[0][1].cpu())
    with pytest.raises(ValueError):
        binding.quantize_weights(torch.zeros(4, 64))


def test_a_refused_registration_keeps_the_tensors_of_the_one_in_force(monkeypatch):
    """The context goes on borrowing the tensors that it was given before, so the binding has to hold on to them."""
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    m = binding.FMoE(d_model=64, n_experts=4, d_ffn=32, k_text=2, k_visual=1, dtype="f32")
    m.device = torch.device("cpu")
    pair = lambda *s: (torch.zeros(*s[:-1], s[-1] // 2, dtype=torch.uint8), torch.zeros(*s[:-1], s[-1] // 32, dtype=torch.uint8))  # noqa: E731
    held = m._weights = (torch.zeros(4, 64), None)
    with pytest.raises(binding.FmoeError, match="bf16 context"):
        m.set_weights_quant(torch.zeros(4, 64), None, pair(4, 32, 64), pair(4, 32, 64), pair(4, 64, 32))
    assert m._weights is held
    odd = torch.zeros(4 * 64 + 1)[1:].view(4, 64)
    with pytest.raises(binding.FmoeError, match="16-byte aligned"):
        m.set_weights(odd, None, torch.zeros(4, 32, 64), torch.zeros(4, 32, 64), torch.zeros(4, 64, 32))
    assert m._weights is held


def test_build_check_catches_registers_used_before_an_lds_read_has_landed(tmp_path):
    from paper_2511_17885_amd import build
    issue = "\t;;#ASMSTART\n\tds_read_b128 v[4:7], v1 offset:64\n\t;;#ASMEND\n"
    wait = "\t;;#ASMSTART\n\ts_waitcnt lgkmcnt(0)\n\t;;#ASMEND\n"
    use = "\tv_mov_b32_e32 v9, v6\n"
    p = tmp_path / "a.s"
    p.write_text("k:\n" + issue + "\tv_add_u32 v8, v3, v10\n\tv_mfma_f32_16x16x32_bf16 a[4:7], v[12:15], v[16:19], 0\n" + wait + use)
    assert build.check_pending_reads(str(p)) == 1
    for early in (use, "\tv_mfma_f32_16x16x32_bf16 a[0:3], v[2:5], v[16:19], 0\n", "\tglobal_load_dwordx4 v[7:10], v[20:21], off\n"):
        p.write_text("k:\n" + issue + early + wait)
        with pytest.raises(RuntimeError, match="has not reached"):
            build.check_pending_reads(str(p))
