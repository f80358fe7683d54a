"""Root-mean-square norms with the addition in front of them, their output in 8 bits, and their gradient, against plain
implementations in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2511_17885_amd import binding

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
SIZES = [(1, 8), (1, 16), (3, 24), (5, 40), (2, 128), (7, 136), (4, 1288), (2, 2048), (1, 4096), (2, 4104), (3, 6152), (1, 16384),
         (1025, 64), (1026, 520), (1027, 1032), (1030, 2048), (1025, 2568), (1026, 4096)]
EPS = 1e-6


# --------------------------------------------------------------------------------------------------- the definition


def _to_bf16(v):
    """float64 -> the nearest bfloat16 number, ties to even (values in its normal range, zeros, infinities, NaN)."""
    m, e = np.frexp(v)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(v), np.ldexp(np.rint(np.ldexp(m, 8)), e - 8), v)


def _rounded(v, dtype):
    return _to_bf16(v) if dtype == torch.bfloat16 else v.astype(np.float32).astype(np.float64)


def _norm(x, delta, w, eps, dtype):
    h = x if delta is None else _rounded(x + delta, dtype)
    with np.errstate(all="ignore"):
        r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + np.float64(np.float32(eps)))
        return h, h * r * w


E4M3 = np.array([(m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127])


def _quantize(v):
    """(codes, scale bytes) of rows v in float64."""
    T, d = v.shape
    codes, scales = np.zeros((T, d), np.uint8), np.full((T, 4 * -(-d // 128)), 127, np.uint8)
    for t in range(T):
        for g in range(-(-d // 32)):
            p = v[t, 32 * g:32 * g + 32]
            if not np.isfinite(p).all():
                scales[t, g] = 255
                continue
            big = np.abs(p).max()
            n = 0
            if big > 0:
                n = max(-126, math.frexp(big)[1] - 11)
                while big > 448 * 2.0 ** n:
                    n += 1
            scales[t, g] = n + 127
            a = np.abs(p) / 2.0 ** n
            lo = np.clip(np.searchsorted(E4M3, a, side="right") - 1, 0, 126)
            hi = np.minimum(lo + 1, 126)
            up = (E4M3[hi] - a < a - E4M3[lo]) | ((E4M3[hi] - a == a - E4M3[lo]) & (hi % 2 == 0))
            codes[t, 32 * g:32 * g + 32] = np.where(up, hi, lo) | np.where(np.signbit(p), 0x80, 0)
    return codes, scales


def _inputs(T, d, dtype, weight_dtype, delta, seed=0):
    rng = np.random.default_rng(seed + 1000 * T + d)
    t = lambda a, ty: torch.from_numpy(a.astype(np.float32)).to(ty)  # noqa: E731
    x = t(rng.standard_normal((T, d)) * np.exp(rng.standard_normal((T, 1))), dtype)
    dl = t(0.4 * rng.standard_normal((T, d)), dtype) if delta else None
    return x, dl, t(1.0 + 0.3 * rng.standard_normal(d), weight_dtype)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _cuda(t):
    return None if t is None else t.cuda()


def _assert_norm(n, want, dtype):
    got = _np(n)
    if dtype == torch.bfloat16:
        with np.errstate(over="ignore"):   # the nearest fp32 number, rounded
            assert np.array_equal(got, _to_bf16(want.astype(np.float32).astype(np.float64)))
    else:   # one rounding, of a value that is off by far less than 2^-34 of itself
        assert (np.abs(got - want) <= U * (1 + 2.0 ** -10) * np.abs(want) + 2.0 ** -149).all()


# ------------------------------------------------------------------------------------------------------------- forward


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weight_dtype,delta", [(torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False),
                                                      (torch.float32, torch.float32, True), (torch.float32, torch.bfloat16, False)])
@pytest.mark.parametrize("T,d", SIZES)
def test_norm(T, d, dtype, weight_dtype, delta):
    x, dl, w = _inputs(T, d, dtype, weight_dtype, delta)
    h, n = binding.rms_norm(x.cuda(), w.cuda(), EPS, delta=_cuda(dl))
    want_h, want_n = _norm(_np(x), _np(dl), _np(w), EPS, dtype)
    assert h.dtype == n.dtype == dtype and n.shape == x.shape
    assert np.array_equal(_np(h), want_h)
    _assert_norm(n, want_n, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weight_dtype,delta", [(torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False),
                                                      (torch.float32, torch.float32, True), (torch.float32, torch.bfloat16, False)])
@pytest.mark.parametrize("T,d", SIZES)
def test_norm_in_8_bits(T, d, dtype, weight_dtype, delta):
    x, dl, w = _inputs(T, d, dtype, weight_dtype, delta, seed=1)
    h, codes, scales = binding.rms_norm_quant(x.cuda(), w.cuda(), EPS, delta=_cuda(dl))
    want_h, want_n = _norm(_np(x), _np(dl), _np(w), EPS, dtype)
    assert np.array_equal(_np(h), want_h)
    rows = np.arange(T) if T < 100 else np.unique(np.r_[0:3, T // 2, T - 5:T])
    want_c, want_s = _quantize(want_n[rows])
    assert codes.dtype == torch.float8_e4m3fn and scales.shape == (T, binding.row_scales(d))
    assert np.array_equal(scales.cpu().numpy()[rows], want_s)
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy()[rows], want_c)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 1100])
def test_8_bits_at_the_borders_of_codes_and_scales(rows):
    """A row of ones without eps has the norm one: the outputs are the weights themselves.  Every middle of two codes, the numbers
    beside it, at several scales down to the smallest; largest magnitudes at and beside 448 scales; zeros."""
    groups = []
    mids = (E4M3[1:] + E4M3[:-1]) / 2
    for n in (0, -20, 60, 118, -100, -126):
        for part in np.array_split(mids, 5):
            f = (part * 2.0 ** n).astype(np.float32)
            for v in (f, np.nextafter(f, np.float32(np.inf)), np.nextafter(f, np.float32(0)), -f):
                groups.append(np.r_[v, np.full(31 - len(v), 0.0), np.float32(448 * 2.0 ** n)])
    for big in (448.0, np.nextafter(np.float32(448), np.float32(512)), np.nextafter(np.float32(448), np.float32(0)), 512.0, 256.0, 255.99, 1e-38, 3e38):
        groups.append(np.r_[np.linspace(-1, 1, 31) * big, big])
    groups += [np.zeros(32), -np.zeros(32), np.r_[np.full(31, 0.0), np.float32(2.0 ** -149)]]
    w = np.concatenate(groups).astype(np.float32)
    w = np.r_[w, np.zeros(-len(w) % 4096, np.float32)].reshape(-1, 4096)
    for part in w:
        x = torch.ones(rows, 4096, dtype=torch.float32, device="cuda")
        x[:, ::3] = -1.0
        _, codes, scales = binding.rms_norm_quant(x, torch.from_numpy(part).cuda(), 0.0)
        want_c, want_s = _quantize(_np(x[:1]) * part.astype(np.float64))
        got_c, got_s = codes.view(torch.uint8).cpu().numpy(), scales.cpu().numpy()
        # below 2^-149 scales there are no fp32 numbers to tell zeros from, and the sign of a zero is not compared
        same = (got_c == want_c) | ((got_c & 0x7f) + (want_c & 0x7f) == 0)
        assert same.all() and np.array_equal(got_s, np.repeat(want_s, rows, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [8, 1100])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_rows_that_are_no_ordinary_numbers(T, dtype):
    d = 264
    x, dl, w = _inputs(T, d, dtype, torch.float32, True, seed=2)
    x[0] = 0.0
    dl[0] = 0.0
    x[1, 5] = math.inf
    x[2, 7], dl[2, 7] = math.inf, -math.inf
    x[3, 100] = math.nan
    x[4] *= 2.0 ** 120          # squares past fp32
    x[5] *= 2.0 ** -80          # squares below it
    dl[5] *= 2.0 ** -80
    x[6] = torch.finfo(dtype).max
    dl[6] = 0.0
    for eps in (EPS, 0.0):
        h, n = binding.rms_norm(x.cuda(), w.cuda(), eps, delta=dl.cuda())
        want_h, want_n = _norm(_np(x), _np(dl), _np(w), eps, dtype)
        got, bad = _np(n), ~np.isfinite(want_n)
        assert np.array_equal(_np(h), want_h, equal_nan=True)
        assert np.array_equal(np.isnan(got), np.isnan(want_n))
        _assert_norm(torch.where(torch.from_numpy(bad), 0.0, n.cpu()), np.where(bad, 0.0, want_n), dtype)
        _, codes, scales = binding.rms_norm_quant(x.cuda(), w.cuda(), eps, delta=dl.cuda())
        want_c, want_s = _quantize(want_n[:8])
        assert np.array_equal(scales.cpu().numpy()[:8], want_s)
        got_c = codes.view(torch.uint8).cpu().numpy()[:8]
        assert ((got_c == want_c) | ((got_c & 0x7f) + (want_c & 0x7f) == 0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(5, 72), (1100, 200), (1030, 4096), (3, 16384)])
def test_norm_in_place_without_h_and_nothing_past_the_rows(T, d):
    """h over x and n over delta; h not wanted; a guard behind every output."""
    lib = binding.load()
    x, dl, w = _inputs(T, d, torch.bfloat16, torch.bfloat16, True, seed=3)
    h0, n0 = binding.rms_norm(x.cuda(), w.cuda(), EPS, delta=dl.cuda())
    guard = lambda t: torch.cat([t.flatten(), torch.full((64,), 7.0, dtype=t.dtype)]).cuda()  # noqa: E731
    wg = w.cuda()
    for first in (True, False):
        a, b = guard(x), guard(dl)
        n_to, h_to = (b, a) if first else (a, b)
        assert lib.fmoe_rms_norm(a.data_ptr(), b.data_ptr(), wg.data_ptr(), 1, 1, T, d, EPS, h_to.data_ptr(), n_to.data_ptr(), None) == 0
        torch.cuda.synchronize()
        assert torch.equal(h_to[:-64].view(T, d), h0) and torch.equal(n_to[:-64].view(T, d), n0)
        assert (a[-64:] == 7).all() and (b[-64:] == 7).all()
    a, b = guard(x), guard(dl)
    assert lib.fmoe_rms_norm(a.data_ptr(), b.data_ptr(), wg.data_ptr(), 1, 1, T, d, EPS, None, b.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(b[:-64].view(T, d), n0)
    a, b = guard(x), guard(dl)
    stride = binding.row_scales(d)
    codes = torch.full((T * d + 64,), 9, dtype=torch.uint8, device="cuda")
    scales = torch.full((T * stride + 64,), 9, dtype=torch.uint8, device="cuda")
    assert lib.fmoe_rms_norm_quant(a.data_ptr(), b.data_ptr(), wg.data_ptr(), 1, 1, T, d, EPS, a.data_ptr(), codes.data_ptr(),
                                   scales.data_ptr(), None) == 0
    torch.cuda.synchronize()
    _, c0, s0 = binding.rms_norm_quant(x.cuda(), wg, EPS, delta=dl.cuda())
    assert torch.equal(a[:-64].view(T, d), h0) and torch.equal(codes[:-64].view(T, d), c0.view(torch.uint8))
    assert torch.equal(scales[:-64].view(T, stride), s0) and (codes[-64:] == 9).all() and (scales[-64:] == 9).all()


@pytest.mark.gpu
def test_a_row_does_not_depend_on_how_many_there_are():
    x, dl, w = _inputs(1500, 1288, torch.bfloat16, torch.bfloat16, True, seed=4)
    x, dl, w = x.cuda(), dl.cuda(), w.cuda()
    h, n = binding.rms_norm(x, w, EPS, delta=dl)
    _, c, s = binding.rms_norm_quant(x, w, EPS, delta=dl)
    for part in (slice(0, 1), slice(700, 709), slice(1499, 1500)):
        h1, n1 = binding.rms_norm(x[part], w, EPS, delta=dl[part])
        _, c1, s1 = binding.rms_norm_quant(x[part], w, EPS, delta=dl[part])
        assert torch.equal(h[part], h1) and torch.equal(n[part], n1)
        assert torch.equal(c[part].view(torch.uint8), c1.view(torch.uint8)) and torch.equal(s[part], s1)


@pytest.mark.gpu
def test_norm_of_more_than_4_gib():
    T, d = 1100000, 2048
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(3, d, device="cuda").to(torch.bfloat16)
    x[-3:] = tail
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    _, n = binding.rms_norm(x, w, EPS)
    assert torch.equal(n[-3:], binding.rms_norm(tail, w, EPS)[1]) and not n[0].any()
    del n
    _, codes, scales = binding.rms_norm_quant(x, w, EPS)
    _, c1, s1 = binding.rms_norm_quant(tail, w, EPS)
    assert torch.equal(codes[-3:].view(torch.uint8), c1.view(torch.uint8)) and torch.equal(scales[-3:], s1)
    del codes, scales
    g = torch.zeros_like(x)
    g[-3:] = 1.0
    dx, dw = binding.rms_norm_backward(x, w, EPS, g)
    dx1, dw1 = binding.rms_norm_backward(tail, w, EPS, g[-3:].contiguous())
    assert torch.equal(dx[-3:], dx1) and not dx[:-3].any()
    assert torch.allclose(dw, dw1, rtol=0, atol=8 * U * 3 * 6)   # three terms of at most 6, in another order


@pytest.mark.gpu
def test_no_rows():
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    assert binding.rms_norm(x, w)[1].shape == (0, 64)
    assert binding.rms_norm_quant(x, w)[1].shape == (0, 64)
    dx, dw = binding.rms_norm_backward(x, w, EPS, x)
    assert dx.shape == (0, 64) and not dw.any()


# ------------------------------------------------------------------------------------------------------------ backward


def _backward(h, w, eps, dn, dh):
    """The formula's gradients, and the sizes of the terms that fp32 adds up."""
    d = h.shape[1]
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + np.float64(np.float32(eps)))
    c, g = h * r, dn * w
    m = (g * c).mean(1, keepdims=True)
    dx = r * (g - c * m)
    # relative roundings: g, c, their difference and the two factors 8; the mean: a chain of at most 64 + 16, its terms 3
    size = r * (8 * (np.abs(g) + np.abs(c * m)) + np.abs(c) * 83 * np.abs(g * c).mean(1, keepdims=True))
    if dh is not None:
        dx, size = dx + dh, size + np.abs(dh) + np.abs(dx)
    return dx, size, (dn * c).sum(0), np.abs(dn * c).sum(0), d


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weight_dtype,residual", [(torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False),
                                                         (torch.float32, torch.float32, True), (torch.float32, torch.bfloat16, False)])
@pytest.mark.parametrize("T,d", SIZES + [(5000, 72), (2500, 2048)])
def test_backward(T, d, dtype, weight_dtype, residual):
    h, dh, w = _inputs(T, d, dtype, weight_dtype, residual, seed=5)
    dn = _inputs(T, d, dtype, weight_dtype, False, seed=6)[0]
    dx, dw = binding.rms_norm_backward(h.cuda(), w.cuda(), EPS, dn.cuda(), d_h=_cuda(dh))
    want, size, want_w, size_w, _ = _backward(_np(h), _np(w), EPS, _np(dn), _np(dh))
    assert dx.dtype == dtype and dw.dtype == torch.float32 and dw.shape == (d,)
    assert (np.abs(_np(dx) - want) <= HALF[dtype] * (np.abs(want) + U * size) + U * size).all()
    rows = -(-T // 2048) if T > 1024 else -(-T // 512)   # that a wavefront adds up in fp32, then three sums, then 64 bits
    assert (np.abs(_np(dw) - want_w) <= U * (rows + 3 + 5) * size_w).all()
    again = binding.rms_norm_backward(h.cuda(), w.cuda(), EPS, dn.cuda(), d_h=_cuda(dh))
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    alone, none = binding.rms_norm_backward(h.cuda(), w.cuda(), EPS, dn.cuda(), d_h=_cuda(dh), want_weight=False)
    assert none is None and torch.equal(alone, dx)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(3, 64), (1100, 40)])
def test_backward_against_differences(T, d):
    """Along random directions: the outputs of two forward calls, a small step apart to either side."""
    x, dl, w = (t.cuda() for t in _inputs(T, d, torch.float32, torch.float32, True, seed=7))
    dn, dh, _ = (t.cuda() for t in _inputs(T, d, torch.float32, torch.float32, True, seed=8))
    h, _ = binding.rms_norm(x, w, EPS, delta=dl)
    dx, dw = binding.rms_norm_backward(h, w, EPS, dn, d_h=dh)
    loss = lambda x, w, dl: sum((a.double() * b.double()).sum() for a, b in zip(binding.rms_norm(x, w, EPS, delta=dl), (dh, dn)))  # noqa: E731
    s = 2.0 ** -7
    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(3):
        v = torch.randn(T, d, generator=gen, device="cuda") * h.abs().mean(1, keepdim=True)
        u = torch.randn(d, generator=gen, device="cuda")
        h_n = [t.double() for t in binding.rms_norm(x, w, EPS, delta=dl)]
        # one rounding of n and of h on either side, over the step; third derivatives of a row of unit size are of the order of
        # its gradient, so s^2 of the sizes, with a factor of 4
        noise = U * sum((a.abs() * b.abs().double()).sum() for a, b in zip(h_n, (dh, dn))) / s * 2
        for got, part, size in ((dx, lambda k: loss(x + k * s * v, w, dl), (dx.abs().double() * v.abs()).sum()),
                                (dx, lambda k: loss(x, w, dl + k * s * v), (dx.abs().double() * v.abs()).sum()),
                                (dw, lambda k: loss(x, w + k * s * u, dl), (dw.abs().double() * u.abs()).sum())):
            along = (got.double() * (v if got is dx else u)).sum()
            assert abs((part(1) - part(-1)) / (2 * s) - along) <= noise + 4 * s * s * size


@pytest.mark.gpu
def test_backward_of_rows_far_from_one_and_in_place():
    lib = binding.load()
    T, d = 6, 128
    h, dh, w = _inputs(T, d, torch.float32, torch.float32, True, seed=10)
    dn = _inputs(T, d, torch.float32, torch.float32, False, seed=11)[0]
    h[1] *= 2.0 ** 70
    h[2] *= 2.0 ** -70
    h[3] = 0.0
    want, size, want_w, size_w, _ = _backward(_np(h), _np(w), EPS, _np(dn), _np(dh))
    hg, wg = h.cuda(), w.cuda()
    for over in ("dn", "dh"):
        g, r = dn.cuda(), dh.cuda()
        ws = torch.empty(lib.fmoe_rms_norm_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")
        dw = torch.empty(d, device="cuda")
        out = g if over == "dn" else r
        assert lib.fmoe_rms_norm_backward(hg.data_ptr(), wg.data_ptr(), g.data_ptr(), r.data_ptr(), 0, 0, T, d, EPS, out.data_ptr(),
                                          dw.data_ptr(), ws.data_ptr(), ws.numel(), None) == 0
        torch.cuda.synchronize()
        assert (np.abs(_np(out) - want) <= U * (np.abs(want) + 2 * size)).all()
        assert (np.abs(_np(dw) - want_w) <= U * 9 * size_w).all()


# Up to 4096 rows of more than 1024 elements have four wavefronts a row, from 4097 on one (up to 4096 elements).  From 100 MB of tensors
# on, one wavefront's rows pass the caches by.
TYPES = [(torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False), (torch.float32, torch.float32, True),
         (torch.float32, torch.bfloat16, False)]
ONE_WAVEFRONT = [(4097, 1032), (4098, 1288), (4097, 1544), (4099, 2048), (4097, 2056), (4098, 2568), (4097, 4096)]
PAST_CACHES = [(6401, 2048, torch.bfloat16), (4097, 4096, torch.bfloat16), (6403, 1024, torch.float32), (4097, 2048, torch.float32),
               (52001, 256, torch.bfloat16)]


def _sample(T):
    return np.unique(np.r_[0:4, 62:66, T // 2 + np.arange(8), T - 5:T])


def _check_norms(T, d, dtype, weight_dtype, delta, seed):
    x, dl, w = _inputs(T, d, dtype, weight_dtype, delta, seed=seed)
    rows = _sample(T)
    h, n = binding.rms_norm(x.cuda(), w.cuda(), EPS, delta=_cuda(dl))
    h8, codes, scales = binding.rms_norm_quant(x.cuda(), w.cuda(), EPS, delta=_cuda(dl))
    want_h, want_n = _norm(_np(x[rows]), None if dl is None else _np(dl[rows]), _np(w), EPS, dtype)
    assert np.array_equal(_np(h[rows]), want_h) and torch.equal(h8, h)
    _assert_norm(n[rows], want_n, dtype)
    want_c, want_s = _quantize(want_n)
    assert np.array_equal(codes.view(torch.uint8)[rows].cpu().numpy(), want_c) and np.array_equal(scales[rows].cpu().numpy(), want_s)
    # and rows here and there as in calls of 64, which pass no cache by and have four wavefronts a row of more than 1024
    for i in range(0, T, 997):
        part = slice(i, i + 64)
        h1, n1 = binding.rms_norm(x[part].cuda(), w.cuda(), EPS, delta=_cuda(None if dl is None else dl[part]))
        _, c1, s1 = binding.rms_norm_quant(x[part].cuda(), w.cuda(), EPS, delta=_cuda(None if dl is None else dl[part]))
        assert torch.equal(n[part], n1) and torch.equal(h[part], h1)
        assert torch.equal(codes[part].view(torch.uint8), c1.view(torch.uint8)) and torch.equal(scales[part], s1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weight_dtype,delta", TYPES)
@pytest.mark.parametrize("T,d", ONE_WAVEFRONT)
def test_norms_of_many_rows_with_one_wavefront_each(T, d, dtype, weight_dtype, delta):
    _check_norms(T, d, dtype, weight_dtype, delta, 20)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", PAST_CACHES)
def test_norms_whose_rows_pass_the_caches(T, d, dtype):
    _check_norms(T, d, dtype, dtype, True, 21)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", PAST_CACHES + [(3203, 2048, torch.float32), (700, 8200, torch.bfloat16)])
def test_backward_whose_rows_pass_the_caches(T, d, dtype):
    """Gradients of rows as in calls of 64, the weight's against 64 bits."""
    h, dh, w = _inputs(T, d, dtype, dtype, True, seed=22)
    dn = _inputs(T, d, dtype, dtype, False, seed=23)[0]
    dx, dw = binding.rms_norm_backward(h.cuda(), w.cuda(), EPS, dn.cuda(), d_h=dh.cuda())
    rows = _sample(T)
    want, size, _, _, _ = _backward(_np(h[rows]), _np(w), EPS, _np(dn[rows]), _np(dh[rows]))
    assert (np.abs(_np(dx[rows]) - want) <= HALF[dtype] * (np.abs(want) + U * size) + U * size).all()
    for i in range(0, T, 997):
        part = slice(i, i + 64)
        assert torch.equal(dx[part], binding.rms_norm_backward(h[part].cuda(), w.cuda(), EPS, dn[part].cuda(), d_h=dh[part].cuda())[0])
    want_w, size_w = 0.0, 0.0
    for i in range(0, T, 4096):
        part = slice(i, i + 4096)
        _, _, a, b, _ = _backward(_np(h[part]), _np(w), EPS, _np(dn[part]), None)
        want_w, size_w = want_w + a, size_w + b
    in_a_row = -(-T // 2048) if d <= 4096 else -(-T // 512)   # that a wavefront, or four, add up in fp32, then three sums, then 64 bits
    assert (np.abs(_np(dw) - want_w) <= U * (in_a_row + 3 + 5) * size_w).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(4096, 1288), (4097, 1288), (4096, 4096), (4097, 4096), (4097, 8192)])
def test_a_row_is_the_same_on_both_sides_of_the_line(T, d):
    x, dl, w = (t.cuda() for t in _inputs(4097, d, torch.bfloat16, torch.bfloat16, True, seed=24))
    h, n = binding.rms_norm(x[:T], w, EPS, delta=dl[:T])
    _, c, s = binding.rms_norm_quant(x[:T], w, EPS, delta=dl[:T])
    for part in (slice(0, 1), slice(2000, 2009), slice(4095, 4096)):
        h1, n1 = binding.rms_norm(x[part], w, EPS, delta=dl[part])
        _, c1, s1 = binding.rms_norm_quant(x[part], w, EPS, delta=dl[part])
        assert torch.equal(h[part], h1) and torch.equal(n[part], n1)
        assert torch.equal(c[part].view(torch.uint8), c1.view(torch.uint8)) and torch.equal(s[part], s1)


@pytest.mark.gpu
def test_8_bits_at_the_borders_of_codes_and_scales_with_one_wavefront_a_row():
    test_8_bits_at_the_borders_of_codes_and_scales(4097)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(8, 1288), (8, 4104), (4097, 1288), (4097, 2056)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_are_no_ordinary_numbers_in_either_form(T, d, dtype):
    x, dl, w = _inputs(T, d, dtype, torch.float32, True, seed=25)
    x[0], dl[0] = 0.0, 0.0
    x[1, 5] = -math.inf
    x[2, 7], dl[2, 7] = math.inf, -math.inf
    x[3, d - 1] = math.nan
    x[4] *= 2.0 ** 120
    x[5] *= 2.0 ** -80
    dl[5] *= 2.0 ** -80
    x[6], dl[6] = torch.finfo(dtype).max, 0.0
    with np.errstate(all="ignore"):
        for eps in (EPS, 0.0):
            h, n = binding.rms_norm(x.cuda(), w.cuda(), eps, delta=dl.cuda())
            want_h, want_n = _norm(_np(x[:8]), _np(dl[:8]), _np(w), eps, dtype)
            got, odd = _np(n[:8]), ~np.isfinite(want_n)
            assert np.array_equal(_np(h[:8]), want_h, equal_nan=True) and np.array_equal(np.isnan(got), np.isnan(want_n))
            _assert_norm(torch.where(torch.from_numpy(odd), 0.0, n[:8].cpu()), np.where(odd, 0.0, want_n), dtype)
            assert np.isfinite(got[4:]).all() and np.isnan(got[1:4]).any(1).all()
            _, codes, scales = binding.rms_norm_quant(x.cuda(), w.cuda(), eps, delta=dl.cuda())
            want_c, want_s = _quantize(want_n)
            assert np.array_equal(scales.cpu().numpy()[:8], want_s)
            got_c = codes.view(torch.uint8).cpu().numpy()[:8]
            assert ((got_c == want_c) | ((got_c & 0x7f) + (want_c & 0x7f) == 0)).all()


# -------------------------------------------------------------------------------------------------- streams and graphs


@pytest.mark.gpu
def test_norms_captured_and_replayed_on_another_stream():
    T, d = 1200, 520
    x, dl, w = (t.cuda() for t in _inputs(T, d, torch.bfloat16, torch.bfloat16, True, seed=12))
    dn = torch.randn(T, d, device="cuda").to(torch.bfloat16)

    def step():
        h, n = binding.rms_norm(x, w, EPS, delta=dl)
        _, c, s = binding.rms_norm_quant(x, w, EPS, delta=dl)
        return [h, n, c.view(torch.uint8), s, *binding.rms_norm_backward(h, w, EPS, dn, d_h=dl)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = step()
    for turn in range(4):
        x.copy_(torch.randn(T, d, device="cuda"))
        dn.copy_(torch.randn(T, d, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b), turn


# ------------------------------------------------------------------------------------------------------------- refusals


def test_norm_refuses_bad_arguments():
    lib = binding.load()
    p, odd = 0x1000, 0x1008
    fwd = lambda x=p, dl=None, w=p, t=0, wt=0, T=4, d=64, eps=1e-6, h=None, n=0x2000: lib.fmoe_rms_norm(  # noqa: E731
        x, dl, w, t, wt, T, d, eps, h, n, None)
    qnt = lambda x=p, dl=None, w=p, t=0, wt=0, T=4, d=64, eps=1e-6, h=None, n=0x2000, s=0x3000: lib.fmoe_rms_norm_quant(  # noqa: E731
        x, dl, w, t, wt, T, d, eps, h, n, s, None)
    bwd = lambda x=p, dl=None, w=p, t=0, wt=0, T=4, d=64, eps=1e-6, n=p, dx=p, dw=None, ws=0x4000, nb=1 << 20: lib.fmoe_rms_norm_backward(  # noqa: E731
        x, w, n, dl, t, wt, T, d, eps, dx, dw, ws, nb, None)
    for call in (fwd, qnt, bwd):
        assert call(t=2) == -1 and call(wt=-1) == -1 and call(d=0) == -1 and call(d=-8) == -1
        assert call(d=12) == -5 and call(d=16392) == -5 and call(T=-1) == -1 and call(T=1 << 24) == -5
        assert call(eps=-1e-6) == -1 and call(eps=math.nan) == -1 and call(eps=math.inf) == -1
        assert call(x=None) == -2 and call(w=None) == -2 and call(n=None) == -2
        assert call(x=odd) == -1 and call(w=odd) == -1 and call(n=odd) == -1 and call(dl=odd) == -1
        assert lib.fmoe_last_error() != b""
    assert fwd(T=0, x=None) == 0 and qnt(T=0, x=None) == 0 and bwd(T=0, x=None) == 0
    assert fwd(h=odd) == -1 and fwd(h=0x2000) == -1 and qnt(h=odd) == -1 and qnt(s=None) == -2 and qnt(s=odd) == -1
    assert bwd(dx=None) == -2 and bwd(dx=odd) == -1 and bwd(dw=odd) == -1
    need = lib.fmoe_rms_norm_workspace_bytes(4, 64)
    assert need >= 64 * 4
    assert bwd(dw=p, ws=None) == -4 and bwd(dw=p, ws=0x4010) == -4 and bwd(dw=p, nb=need - 1) == -4


def test_norm_sizes_past_32_bits_are_refused(monkeypatch):
    """2^32 + 4 rows are not four, nor a row of 2^32 + 8 elements one of eight."""
    monkeypatch.setattr(binding, "_call", lambda *a: None)
    empty = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="meta")  # noqa: E731
    for x, w in ((empty((1 << 32) + 4, 8), empty(8)), (empty(1 << 16, (1 << 15) + 1, 16), empty(16)), (empty(1, (1 << 32) + 8), empty((1 << 32) + 8))):
        for call in (lambda: binding.rms_norm(x, w), lambda: binding.rms_norm_quant(x, w), lambda: binding.rms_norm_backward(x, w, EPS, x)):
            with pytest.raises(ValueError, match="32 bits"):
                call()


@pytest.mark.gpu
def test_norm_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for call in (lambda: binding.rms_norm(x[:, ::2], w), lambda: binding.rms_norm(x, w[:32]), lambda: binding.rms_norm(x, w.cpu()),
                 lambda: binding.rms_norm(x, w, delta=x[:3]), lambda: binding.rms_norm(x, w, delta=x.to(torch.bfloat16)),
                 lambda: binding.rms_norm_quant(x.t(), w), lambda: binding.rms_norm_backward(x, w, EPS, x[:2]),
                 lambda: binding.rms_norm_backward(x, w, EPS, x, d_h=x.cpu())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        binding.rms_norm(x.double(), w)
