"""The operators of a head that answers on the GPU against plain implementations in 64 bits: root-mean-square norm of the residual
stream, rows in 8 bits and their product, words drawn from logits.

Tolerances follow from the arithmetic.  A result is rounded once to its type: off by half a step, finfo(type).eps / 2 of its value.  Sums
are binary32: with m the additions that a value passes through, a sum is off by m 2^-24 of the sum of magnitudes.  8-bit values, steps and
words are equal, not close."""
import math

import numpy as np
import pytest
import torch

import paper_1610_02496_amd as pk

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {t: torch.finfo(t).eps / 2 for t in (F32, F16, BF16)}
TINY = {F32: 1e-37, F16: 2.0 ** -25, BF16: 1e-37}      # half a step of what is not a normal number, and the flush of what is tiny
E = 2.0 ** -24


def dev(a, dtype=None):
    return torch.as_tensor(a).to(device="cuda", dtype=dtype)


def make(seed, *shape, dtype=F32, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale + shift).to(dtype)


def within(got, want, bound, what):
    got, want, bound = got.double().cpu(), want.double().cpu(), torch.as_tensor(bound).double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%s: %d of %d values, worst %.3g against a bound of %.3g" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound.expand_as(off)[bad].min()))


# ---- root-mean-square norm --------------------------------------------------------------------------------------------

EPS = 1e-6


def rms64(s, w):
    s = s.double()
    r = 1 / (s.square().mean(-1, keepdim=True) + EPS).sqrt()
    return s * r * w, r, s * r


def steps64(t):
    """(whole numbers, step) of every row of t: the step is a 127th of the largest magnitude in binary32, ties go to even."""
    step = (t.double().abs().amax(-1, keepdim=True) / 127).float().double()
    return torch.where(step > 0, (t.double() / step).round(), 0.0).clamp(-127, 127), step


SHAPES = [(1, 1), (1, 1000), (3, 7), (5, 128), (130, 129), (64, 512), (67, 513), (33, 1000), (21, 1025), (9, 2048), (10, 2049), (7, 4096),
          (5, 4099), (6, 8192), (3, 8193), (2, 20001), (2100, 96), (4099, 40), (8195, 520), (2051, 1030)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,rtype,wtype,pad", [(F32, F32, F32, 0), (BF16, BF16, BF16, 3), (F16, F32, F32, 8), (BF16, F32, F16, 0), (F32, F32, BF16, 5),
                                                   (F16, F16, F16, 1), (BF16, None, F32, 0), (F32, None, None, 1)])
def test_rms_norm_both_passes(rows, cols, dtype, rtype, wtype, pad):
    print("rms", rows, cols, dtype, rtype, wtype, pad, flush=True)
    x = make(1, rows, cols + pad, dtype=dtype, scale=1.3, shift=0.2)
    res = None if rtype is None else make(2, rows, cols + pad, dtype=rtype, scale=2.0)
    w = None if wtype is None else make(3, cols, dtype=wtype, scale=0.3, shift=1.0)
    dy, stype = make(4, rows, cols + pad, dtype=dtype), rtype or dtype
    dsum = make(5, rows, cols + pad, dtype=stype, scale=0.5)
    cut = lambda a: None if a is None else dev(a)[:, :cols]  # noqa: E731
    y, saved = pk.ops.rms_norm_forward(cut(x), None if w is None else dev(w), cut(res), EPS)
    x, dy, dsum = x[:, :cols], dy[:, :cols], dsum[:, :cols]
    s = x if res is None else (x.float() + res[:, :cols].float()).to(stype)
    assert saved.x.dtype == stype and torch.equal(saved.x.cpu(), s), "the sum"
    w64 = 1.0 if w is None else w.double()
    y64, r64, h64 = rms64(s, w64)
    # a sum of squares passes through 16 additions in a lane (wide rows: one per 1,024 columns), 6 between lanes, 16 between wavefronts
    adds = 40.0 + cols / 1024
    rel = (adds / 2 + 4) * E            # of r: half of the sum's, the square root's, the division's
    within(saved.rstd[:, None], r64, rel * r64, "rstd")
    within(y, y64, HALF[dtype] * y64.abs() + TINY[dtype] + (rel + 2 * E) * y64.abs() * (1 + HALF[dtype]), "y")

    dx, dres, dw = pk.ops.rms_norm_backward(dev(make(4, rows, cols + pad, dtype=dtype))[:, :cols], saved, dev(dsum))
    g = dy.double() * w64
    mgh = (g * h64).mean(1, keepdim=True)
    ds64 = r64 * (g - h64 * mgh) + dsum.double()
    # h is off by rel, the mean by its additions and by h's error in each term, then three roundings each
    err = (rel + 4 * E) * r64 * (g.abs() + h64.abs() * mgh.abs()) + r64 * h64.abs() * (adds + 4) * E * 3 * (g * h64).abs().mean(1, keepdim=True) + 2 * E * (ds64.abs() + dsum.double().abs())
    within(dx, ds64, HALF[dtype] * ds64.abs() + TINY[dtype] + err * (1 + HALF[dtype]), "dx")
    if res is None:
        assert dres is None
    elif stype == dtype:
        assert dres is dx
    else:
        within(dres, ds64, HALF[stype] * ds64.abs() + err * (1 + E), "dresidual")
    if w is None:
        assert dw is None
    else:
        size = (dy.double() * h64).abs().sum(0)
        dw64 = (dy.double() * h64).sum(0)
        lines = rows / 4 + 64           # additions: a lane's rows, a workgroup's wavefronts, the partial rows
        within(dw, dw64, HALF[wtype] * dw64.abs() + TINY[wtype] + (lines * E + rel + 2 * E) * size * (1 + HALF[wtype]), "dweight")


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,rtype,wtype", [(F32, F32, F32), (BF16, BF16, BF16), (F16, F32, F32), (BF16, None, F32), (F32, None, None)])
def test_rms_norm_in_8_bits(rows, cols, dtype, rtype, wtype):
    print("rms8", rows, cols, dtype, rtype, wtype, flush=True)
    x = make(1, rows, cols + 3, dtype=dtype, scale=1.3)
    res = None if rtype is None else make(2, rows, cols, dtype=rtype, scale=2.0)
    w = None if wtype is None else make(3, cols, dtype=wtype, scale=0.3, shift=1.0)
    c, total = pk.ops.rms_norm8(dev(x)[:, :cols], None if w is None else dev(w), None if res is None else dev(res), EPS)
    x = x[:, :cols]
    s = x if res is None else (x.float() + res.float()).to(rtype)
    assert torch.equal(total.cpu(), s)
    t = s.float() * (1.0 if w is None else w.float())
    q64, step = steps64(t)
    assert torch.equal(c.q.cpu().double(), q64)
    _, r64, _ = rms64(s, 1.0)
    adds = 40.0 + cols / 1024
    within(c.scale[:, None], step * r64, ((adds / 2 + 4) * E + 2 * E) * step * r64, "scale")
    wide = c.q.as_strided((rows, c._stride), (c._stride, 1)).cpu()
    assert int(wide[:, cols:(cols + 15) // 16 * 16].abs().sum()) == 0, "zeros up to the next multiple of 16"
    assert torch.equal(c.restore(F32).cpu(), c.q.cpu().float() * c.scale.cpu()[:, None])


def test_rms_norm_values_at_the_edge():
    """Rows of zeros, rows whose squares do not fit binary32, and rows that are not finite: they stay by themselves."""
    for cols in (300, 1500, 9000):
        x = torch.zeros(7, cols)
        x[1] = 1e30 * make(1, cols)
        x[2] = 1e-30 * make(2, cols)
        x[3, 5] = float("nan")
        x[4, 6] = float("inf")
        x[5, 7] = torch.finfo(F32).max
        x[6] = make(3, cols)
        y, saved = pk.ops.rms_norm_forward(dev(x))
        y64, r64, _ = rms64(x, 1.0)
        for i in (0, 1, 2, 6):
            within(y[i], y64[i], 64 * E * y64[i].abs() + 1e-37, "row %d" % i)
        # (r is not a normal number here: half a step of it is 2^-150)
        within(y[5], y64[5], 64 * E * y64[5].abs() + 2.0 ** -150 * float(torch.finfo(F32).max), "row 5")
        assert bool(y[3].isnan().all()) and bool(y[4, 6].isnan()) and float(y[4, :6].abs().max()) == 0
        c, _ = pk.ops.rms_norm8(dev(x))
        back = c.restore()
        assert float(back[0].abs().max()) == 0 and bool(back[3].isnan().all()) and bool(back[4].isnan().all())
        for i in (1, 2, 5, 6):
            q, step = steps64(x[i:i + 1])
            assert torch.equal(c.q[i].cpu().double(), q[0])
        dy = make(5, 7, cols)
        _, _, dw = pk.ops.rms_norm_backward(dev(dy)[6:], pk.ops.rms_norm_forward(dev(x)[6:], dev(torch.ones(cols)))[1])
        assert bool(dw.isfinite().all())


def test_rms_norm_parts_and_no_rows():
    x, res, w, dy, dsum = make(1, 37, 300), make(2, 37, 300), make(3, 300), make(4, 37, 300), make(5, 37, 300)
    _, saved = pk.ops.rms_norm_forward(dev(x), dev(w), dev(res))
    full = pk.ops.rms_norm_backward(dev(dy), saved, dev(dsum))
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        got = pk.ops.rms_norm_backward(dev(dy), saved, dev(dsum), *need)
        for n, a, f in zip(need, got, full):
            assert torch.equal(a, f) if n else a is None
    without = pk.ops.rms_norm_backward(dev(dy), saved)
    zero = pk.ops.rms_norm_backward(dev(dy), saved, torch.zeros(37, 300, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(without, zero))
    none = torch.empty(0, 300, device="cuda")
    y, saved = pk.ops.rms_norm_forward(none, dev(w), none)
    dx, _, dw = pk.ops.rms_norm_backward(none, saved)
    assert y.shape == dx.shape == (0, 300) and float(dw.abs().sum()) == 0
    c, total = pk.ops.rms_norm8(none, dev(w), none)
    assert c.shape == total.shape == (0, 300) and c.restore().shape == (0, 300)
    a, b = make(2, 3, 5, 64), make(3, 3, 5, 64)
    y, s = pk.ops.rms_norm(dev(a).transpose(0, 1), None, dev(b).transpose(0, 1))
    flat, t = pk.ops.rms_norm(dev(a).transpose(0, 1).reshape(15, 64), None, dev(b).transpose(0, 1).reshape(15, 64))
    assert torch.equal(y.reshape(15, 64), flat) and torch.equal(s.reshape(15, 64), t)


def test_rms_norm_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    x, res, w = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 33), (5, 33), (33,)))
    a, b = torch.randn(5, 33, generator=g, dtype=torch.float64), torch.randn(5, 33, generator=g, dtype=torch.float64)

    def f(x, res, w):
        s = x + res
        return float((a * s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * w).sum() + (b * s.square()).sum())

    t = [dev(v, F32).requires_grad_() for v in (x, res, w)]
    y, s = pk.ops.rms_norm(t[0], t[2], t[1], EPS)
    loss = (dev(a, F32) * y).sum() + (dev(b, F32) * s * s).sum()
    loss.backward()
    h = 1e-5
    for k, v in enumerate((x, res, w)):
        flat = v.view(-1)
        for i in range(0, flat.numel(), 7):
            keep = float(flat[i])
            flat[i] = keep + h
            up = f(x, res, w)
            flat[i] = keep - h
            down = f(x, res, w)
            flat[i] = keep
            assert abs(float(t[k].grad.view(-1)[i]) - (up - down) / (2 * h)) < 2e-4, (k, i)
    # only the sum is used, only the norm is used, the stream in 32 bits
    u = [dev(v, F32).requires_grad_() for v in (x, res)]
    pk.ops.rms_norm(u[0], None, u[1])[1].sum().backward()
    assert torch.equal(u[0].grad, torch.ones_like(u[0])) and torch.equal(u[1].grad, torch.ones_like(u[1]))
    v = [dev(x, BF16).requires_grad_(), dev(res, F32).requires_grad_()]
    y, s = pk.ops.rms_norm(v[0], None, v[1])
    assert y.dtype == BF16 and s.dtype == F32
    y.float().sum().backward()
    assert v[0].grad.dtype == BF16 and v[1].grad.dtype == F32 and torch.equal(v[0].grad, v[1].grad.to(BF16))


# ---- rows in 8 bits and their product -----------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,pad", [(F32, 0), (F16, 3), (BF16, 8)])
def test_rows8(rows, cols, dtype, pad):
    print("rows8", rows, cols, dtype, pad, flush=True)
    x = make(1, rows, cols + pad, dtype=dtype, scale=1.3)
    c = pk.ops.rows8(dev(x)[:, :cols])
    q64, step = steps64(x[:, :cols].float())
    assert torch.equal(c.q.cpu().double(), q64) and torch.equal(c.scale.cpu().double()[:, None], step)
    wide = c.q.as_strided((rows, c._stride), (c._stride, 1)).cpu()
    assert int(wide[:, cols:(cols + 15) // 16 * 16].abs().sum()) == 0
    assert torch.equal(c.restore().cpu(), (c.q.cpu().float() * c.scale.cpu()[:, None]).to(dtype))


def test_rows8_of_quotients_next_to_a_half():
    """x / step that binary32 rounds to a half but is not one: the whole number is that of the quotient itself."""
    found = 0
    g = torch.Generator().manual_seed(1)
    for k in range(200):
        top = float(torch.rand(1, generator=g) + 0.5)
        step = np.float32(np.float32(top) / np.float32(127))
        x = [np.float32(top)]
        for n in range(0, 126, 2):
            a = np.float32((n + 0.5) * float(step))
            x += [np.nextafter(a, np.float32(-9)), a, np.nextafter(a, np.float32(9))]
        x = torch.from_numpy(np.array(x, dtype=np.float32))[None]
        q64, step64 = steps64(x)
        c = pk.ops.rows8(dev(x))
        assert torch.equal(c.q.cpu().double(), q64)
        found += int(((x / step64.float()).round() != q64).sum())
    assert found > 0   # (the inputs hold such quotients)


def test_rows8_edges():
    x = torch.zeros(5, 100)
    x[1, 3] = torch.finfo(F32).max
    x[1, 4] = -torch.finfo(F32).max
    x[2, 5] = 1e-44
    x[3, 6] = float("inf")
    x[4, 7] = float("nan")
    c = pk.ops.rows8(dev(x))
    back = c.restore().cpu()
    assert float(back[0].abs().max()) == 0 and bool(back[1].isfinite().all()) and float(back[1, 3]) > 3.4e38
    assert bool(back[3].isnan().all()) and bool(back[4].isnan().all()) and bool(back[2].isfinite().all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,words,cols", [(1, 1, 1), (1, 1000, 777), (2, 33, 16), (16, 4097, 64), (17, 300, 65), (61, 3001, 777), (64, 64, 128), (65, 255, 129),
                                             (130, 1030, 1000), (300, 2500, 300), (515, 9000, 256), (1, 20000, 8200), (5, 70, 131071), (2100, 5003, 100),
                                             (1000, 12003, 272)])
def test_linear8(rows, words, cols, dtype):
    print("linear8", rows, words, cols, dtype, flush=True)
    g = torch.Generator().manual_seed(rows + cols)
    q, w = (torch.randint(-127, 128, (n, cols), generator=g, dtype=torch.int8) for n in (rows, words))
    q[0], w[0] = -128, -128            # the largest sums
    sx, sw = torch.rand(rows, generator=g) + 0.01, torch.rand(words, generator=g) / cols
    a, b = pk.ops.Rows8.of(dev(q), dev(sx), dtype), pk.ops.Rows8.of(dev(w), dev(sw))
    out = pk.ops.linear8(a, b)
    assert out.shape == (rows, words) and out.dtype == dtype
    sums = q.double() @ w.double().t()
    want = (sums.float() * sx[:, None] * sw[None]).to(dtype)      # sums are exact, the rest is defined step by step
    assert torch.equal(out.cpu(), want)


def test_linear8_of_features_and_shapes():
    x, w = make(1, 3, 7, 200, dtype=BF16), make(2, 500, 200, dtype=BF16, scale=0.1)
    w8 = pk.ops.rows8(dev(w))
    out = pk.ops.linear8(dev(x), w8)
    assert out.shape == (3, 7, 500) and out.dtype == BF16
    again = pk.ops.linear8(pk.ops.rows8(dev(x).view(21, 200)), w8, F32)
    q, s = steps64(x.view(21, 200).float())
    qw, sw = steps64(w.float())
    within(again, (q @ qw.t()) * s * sw.t(), 3 * E * ((q @ qw.t()) * s * sw.t()).abs(), "logits")
    assert torch.equal(again.to(BF16), out.view(21, 500))
    assert pk.ops.linear8(torch.empty(0, 200, device="cuda", dtype=BF16), w8).shape == (0, 500)
    # a row that is not finite stays by itself
    x = dev(make(3, 4, 200))
    x[1, 5] = float("nan")
    x[2, 7] = float("inf")
    out = pk.ops.linear8(x, w8)
    assert bool(out[1:3].isnan().all()) and bool(out[0].isfinite().all()) and bool(out[3].isfinite().all())


# ---- words drawn from logits -----------------------------------------------------------------------------------------------

def draw64(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row, from the definition in 64 bits, with sorting."""
    l = np.asarray(l, dtype=np.float64)
    u, temperature, top_p, min_p = (float(np.float32(v)) for v in (u, temperature, top_p, min_p))
    if np.isnan(l).any():
        return -1, math.nan
    top = l.max()
    if top == -math.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(l.argmax()), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(l == top, 0.0, (l - top) / temperature)
    z[l == -math.inf] = -math.inf
    e = np.exp(z)
    bits = max(len(l) - 1, 0).bit_length()
    e[e * 2.0 ** (45 if bits <= 17 else 62 - bits) < 0.5] = 0   # (no mass, as documented: what a random number of exactly 0 would find otherwise)
    order = np.argsort(-l, kind="stable")
    n = len(l) if top_k <= 0 else min(top_k, len(l))
    if top_p < 1:
        sums = np.cumsum(e[order[:n]])
        n = min(n, int(np.searchsorted(sums, top_p * sums[-1], side="left")) + 1)
    keep = np.zeros(len(l), dtype=bool)
    keep[order[:max(n, 1)]] = True
    if min_p > 0:
        keep &= z >= math.log(min(min_p, 1.0))
    e = np.where(keep, e, 0.0)
    sums = np.cumsum(e)
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    word = int(np.searchsorted(sums, u * sums[-1], side="right"))
    return word, e[word] / sums[-1]


def check_draws(logits, u, **limits):
    """Every row against draw64; limits are numbers or tensors with a value per row."""
    rows = logits.shape[0]
    on = {k: dev(v) if isinstance(v, torch.Tensor) else v for k, v in limits.items()}
    word, p = pk.ops.sample(logits if logits.is_cuda else dev(logits), dev(u), **on)
    l = logits.double().cpu().numpy()
    for i in range(rows):
        one = {k: v[i].item() if isinstance(v, torch.Tensor) else v for k, v in limits.items()}
        want, share = draw64(l[i], float(u[i]), **one)
        assert int(word[i]) == want, (i, one, float(u[i]), int(word[i]), want, float(p[i]), share)
        assert (math.isnan(share) and math.isnan(float(p[i]))) or abs(float(p[i]) - share) <= 2 * E * share, (i, float(p[i]), share)


LIMITS = [{}, {"temperature": 0.7}, {"top_k": 5}, {"top_k": 50, "temperature": 1.5}, {"top_p": 0.9}, {"top_p": 0.3, "temperature": 2.0}, {"min_p": 0.05},
          {"top_k": 300, "top_p": 0.8}, {"top_k": 40, "top_p": 0.95, "min_p": 0.1, "temperature": 0.8}, {"top_p": 0.999}, {"top_k": 1}, {"temperature": 0.0},
          {"top_p": 0.0}, {"min_p": 1.0}, {"top_k": 100000}, {"temperature": 0.01}, {"temperature": 30.0, "top_p": 0.5}, {"top_k": 3000, "top_p": 0.99}]


def natural(seed, rows, words, dtype, masked=0.02):
    g = torch.Generator().manual_seed(seed)
    rank = torch.randperm(words, generator=g).double()
    l = 4 - torch.log1p(rank) + 1.7 * torch.randn(rows, words, generator=g, dtype=torch.float64)
    l[:, torch.rand(words, generator=g) < masked] = -math.inf
    l[:, int(rank.argmin())] = 5.0
    return l.to(dtype)


@pytest.mark.parametrize("words", [1, 2, 7, 511, 512, 513, 3000, 8192, 8193, 30011, 100000])
@pytest.mark.parametrize("dtype,pad", [(F32, 0), (F16, 5), (BF16, 0), (F32, 3)])
def test_sample(words, dtype, pad):
    print("sample", words, dtype, pad, flush=True)
    rows = 5 if words > 10000 else 20
    l = natural(words, rows, words + pad, dtype)
    g = torch.Generator().manual_seed(words + 1)
    for limits in LIMITS:
        check_draws(dev(l)[:, :words], torch.rand(rows, generator=g), **limits)


@pytest.mark.parametrize("words", [300, 20000])
def test_sample_equal_logits(words):
    """Logits that are all equal, or of few values: ties go to the lowest number."""
    g = torch.Generator().manual_seed(1)
    u = torch.cat([torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24]), torch.rand(5, generator=g)])
    flat = torch.full((10, words), 1.25)
    few = torch.randint(0, 3, (10, words), generator=g).float() * 0.5
    signs = torch.where(torch.rand(10, words, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0))
    for l in (flat, few, signs):
        for dtype in (F32, BF16):
            for limits in LIMITS:
                check_draws(l.to(dtype), u, **limits)


@pytest.mark.parametrize("spread", [1e-6, 1e-3, 0.01])
def test_sample_logits_that_are_close(spread):
    """All logits in a few bins of a histogram, more of them than the list of a bin holds, at several magnitudes and around zero."""
    g = torch.Generator().manual_seed(5)
    u = torch.rand(4, generator=g)
    for shift in (0.0, 100.0, -0.3):
        l = (torch.randn(4, 9000, generator=g, dtype=torch.float64) * spread + shift).float()
        for limits in LIMITS:
            check_draws(l, u, **limits)


def test_sample_rows_with_limits_of_their_own():
    rows, words = 64, 12000
    l = natural(3, rows, words, F32)
    l[5] = -math.inf
    l[6, 100] = math.nan
    l[7, 50] = l[7, 9000] = math.inf
    l[8] = torch.finfo(F32).min
    l[9, :-1] = -math.inf
    l[10] = torch.where(torch.arange(words) % 3 == 0, torch.tensor(3e38), torch.tensor(-3e38))
    g = torch.Generator().manual_seed(4)
    rand = lambda: torch.rand(rows, generator=g)  # noqa: E731
    for again in range(3):
        temperature, top_k = torch.where(rand() < 0.2, 0.0, 0.3 + rand()), torch.where(rand() < 0.5, 0, (rand() * 2000)).to(torch.int64)
        top_p, min_p = torch.where(rand() < 0.5, 1.0, rand()), torch.where(rand() < 0.5, 0.0, 0.2 * rand())
        check_draws(l, rand(), temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
        check_draws(l, rand(), temperature=temperature, top_k=top_k.to(torch.int32), min_p=min_p, top_p=0.7)


def test_sample_odd_numbers():
    """Random numbers outside of [0, 1), and values per row that are no limits: what the header says of them."""
    l = natural(8, 6, 1000, F32)
    u = torch.tensor([-0.5, 1.0, 7.0, math.nan, math.inf, -math.inf])
    check_draws(l, u)
    nan = torch.full((6,), math.nan)
    word, p = pk.ops.sample(dev(l), dev(u), top_p=dev(nan), min_p=dev(nan), top_k=dev(torch.full((6,), -3)))
    plain, q = pk.ops.sample(dev(l), dev(u))
    assert torch.equal(word, plain) and torch.equal(p, q)
    word, p = pk.ops.sample(dev(l), dev(u), temperature=dev(nan))
    assert torch.equal(word.cpu(), l.argmax(1)) and bool((p == 1).all())
    inf = pk.ops.sample(dev(l), dev(torch.rand(6)), temperature=math.inf)[0]
    assert bool((l[torch.arange(6), inf.cpu()] > -math.inf).all())
    check_draws(l, torch.rand(6), top_p=torch.tensor([-1.0, 2.0, 0.5, 1.0, 0.0, 0.9]).clamp(0, 1))
    below = pk.ops.sample(dev(l), dev(torch.rand(6)), top_p=dev(torch.full((6,), -1.0)))[0]
    assert torch.equal(below.cpu(), l.argmax(1))


def test_sample_of_many_words():
    """More words than tiles of 512 in LDS, and rows that the workgroups take in turn."""
    words = (1 << 20) + 700
    l = natural(9, 2, words, BF16)
    for limits in ({}, {"top_k": 70}, {"top_p": 0.9}, {"min_p": 0.01, "top_k": 100000, "top_p": 0.7}):
        check_draws(l, torch.tensor([0.3, 0.9999]), **limits)
    l = natural(10, 9001, 40, F16)
    check_draws(l, torch.rand(9001, generator=torch.Generator().manual_seed(1)), top_p=0.9, top_k=20)


def test_sample_follows_the_distribution():
    """Numbers spread evenly over [0, 1) take every word as often as its share says, to one."""
    l = natural(11, 1, 50, F32)
    n = 4096
    u = ((torch.arange(n) + 0.5) / n).float()
    word, p = pk.ops.sample(dev(l).expand(n, 50), dev(u), temperature=0.9, top_p=0.95)
    count = torch.bincount(word.cpu(), minlength=50)
    share = torch.zeros(50, dtype=torch.float64)
    share[word.cpu()] = p.double().cpu()
    assert abs(float(share.sum()) - 1) < 1e-6 and bool(((count - share * n).abs() <= 1).all())


def test_sample_shapes():
    l = dev(natural(12, 6, 100, F32))
    u = torch.rand(6, device="cuda")
    flat = pk.ops.sample(l, u, top_k=7)
    cube = pk.ops.sample(l.view(2, 3, 100), u.view(2, 3), top_k=7)
    assert torch.equal(cube[0].view(6), flat[0]) and torch.equal(cube[1].view(6), flat[1])
    one = pk.ops.sample(l[2], u[2])
    assert one[0].shape == () and int(one[0]) == int(pk.ops.sample(l, u)[0][2])
    none = pk.ops.sample(l[:0], u[:0])
    assert none[0].shape == none[1].shape == (0,)


# ---- together ---------------------------------------------------------------------------------------------------------------

def answer(x, res, w, w8, u, limits):
    y, total = pk.ops.rms_norm8(x, w, res)
    logits = pk.ops.linear8(y, w8)
    word, p = pk.ops.sample(logits, u, **limits)
    return total, logits, word, p


@pytest.mark.parametrize("rows,words,cols,dtype", [(1, 5000, 333, BF16), (40, 9001, 512, F16), (300, 1200, 1000, F32)])
def test_from_the_stream_to_a_word(rows, words, cols, dtype):
    x, res, w = make(1, rows, cols, dtype=dtype), make(2, rows, cols, dtype=F32), make(3, cols, scale=0.1, shift=1.0)
    proj = make(4, words, cols, scale=2.0 / math.sqrt(cols))
    u = torch.rand(rows, generator=torch.Generator().manual_seed(5))
    limits = {"temperature": 0.8, "top_k": 200, "top_p": 0.9, "min_p": 0.001}
    total, logits, word, p = answer(dev(x), dev(res), dev(w), pk.ops.rows8(dev(proj)), dev(u), limits)
    s = x.float() + res
    assert torch.equal(total.cpu(), s)
    q, step = steps64(s * w)
    qw, sw = steps64(proj)
    want = (q @ qw.t()) * (step * rms64(s, 1.0)[1]) * sw.t()
    within(logits, want, (HALF[dtype] + 40 * E) * want.abs() + TINY[dtype], "logits")
    for i in range(rows):
        at, share = draw64(logits[i].double().cpu().numpy(), float(u[i]), **limits)
        assert int(word[i]) == at and abs(float(p[i]) - share) <= 2 * E * share


def test_captured_and_replayed():
    """The calls in a graph, with other inputs in every replay and eager work in between; two graphs at once."""
    w, w8 = dev(make(3, 512, scale=0.1, shift=1.0)), pk.ops.rows8(dev(make(4, 9000, 512, scale=0.1)))
    limits = {"temperature": 0.8, "top_k": 100, "top_p": 0.9}
    held = []
    for k in range(2):
        x, res, u = dev(make(k, 20, 512, dtype=BF16)), dev(make(k + 9, 20, 512)), torch.rand(20, device="cuda")
        answer(x, res, w, w8, u, limits)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = answer(x, res, w, w8, u, limits)
        held.append((graph, x, res, u, out))
    for again in range(4):
        for graph, x, res, u, out in held:
            x.copy_(dev(make(100 + again, 20, 512, dtype=BF16)))
            u.uniform_()
            graph.replay()
        torch.cuda.synchronize()
        for graph, x, res, u, out in held:
            want = answer(x, res, w, w8, u, limits)
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_training_step_captured():
    """Forward and backward pass of the norm in a graph while an eager step of the same sizes ran before and runs between."""
    x, res, w = dev(make(1, 300, 777)), dev(make(2, 300, 777)), dev(make(3, 777))
    dy, ds = dev(make(4, 300, 777)), dev(make(5, 300, 777))

    def step():
        y, saved = pk.ops.rms_norm_forward(x, w, res)
        return (y,) + pk.ops.rms_norm_backward(dy, saved, ds)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for again in range(4):
        dy.copy_(dev(make(20 + again, 300, 777)))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_on_another_stream():
    x, res, w = dev(make(1, 2000, 777)), dev(make(2, 2000, 777)), dev(make(3, 777))
    w8, u = pk.ops.rows8(dev(make(4, 3000, 777, scale=0.1))), torch.rand(2000, device="cuda")
    want = answer(x, res, w, w8, u, {"top_p": 0.8})
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = answer(x, res, w, w8, u, {"top_p": 0.8})
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x, w8, u = dev(make(1, 4, 64)), pk.ops.rows8(dev(make(2, 100, 64))), torch.rand(4, device="cuda")
    ops = pk.ops
    l = ops.linear8(x, w8)
    for call, error in [
            (lambda: ops.rms_norm_forward(x.cpu()), ValueError), (lambda: ops.rms_norm_forward(x, residual=x[:2]), ValueError),
            (lambda: ops.rms_norm_forward(x, residual=x.half()), TypeError), (lambda: ops.rms_norm_forward(x, dev(make(1, 63))), ValueError),
            (lambda: ops.rms_norm_forward(x, eps=-1.0), pk.SaberError), (lambda: ops.rms_norm_forward(x.double()), TypeError),
            (lambda: ops.rms_norm_backward(x.half(), ops.rms_norm_forward(x)[1]), TypeError),
            (lambda: ops.rms_norm_backward(x[:2], ops.rms_norm_forward(x)[1]), ValueError),
            (lambda: ops.rms_norm_backward(x, ops.rms_norm_forward(x)[1], x[:2]), ValueError),
            (lambda: ops.rms_norm_backward(x, ops.rms_norm_forward(x)[1], x.half()), TypeError),
            (lambda: ops.rms_norm8(x.clone().requires_grad_()), ValueError), (lambda: ops.linear8(x.clone().requires_grad_(), w8), ValueError),
            (lambda: ops.rows8(torch.empty(3, 0, device="cuda")), ValueError), (lambda: ops.rows8(x.long()), TypeError),
            (lambda: ops.Rows8.of(x, u), TypeError), (lambda: ops.Rows8.of(w8.q, u), ValueError), (lambda: ops.Rows8.of(w8.q.cpu(), u), ValueError),
            (lambda: ops.Rows8.of(w8.q, w8.scale, torch.float64), TypeError),
            (lambda: ops.linear8(x, x), TypeError), (lambda: ops.linear8(x[:, :63], w8), ValueError), (lambda: ops.linear8(x, w8, torch.float64), TypeError),
            (lambda: ops.sample(l.cpu(), u), ValueError), (lambda: ops.sample(l, u.cpu()), ValueError), (lambda: ops.sample(l, u.double()), TypeError),
            (lambda: ops.sample(l, u[:3]), ValueError), (lambda: ops.sample(l, u, temperature=-1.0), pk.SaberError),
            (lambda: ops.sample(l, u, top_p=1.5), pk.SaberError), (lambda: ops.sample(l, u, min_p=-0.1), pk.SaberError),
            (lambda: ops.sample(l, u, top_k=-1), pk.SaberError), (lambda: ops.sample(l, u, temperature=math.nan), pk.SaberError),
            (lambda: ops.sample(l, u, top_k=u), TypeError), (lambda: ops.sample(l, u, top_p=u.double()), TypeError),
            (lambda: ops.sample(l, u, min_p=u[:2]), ValueError), (lambda: ops.sample(l, u, temperature=u.cpu()), ValueError),
            (lambda: ops.sample(l[:, :0], u), ValueError)]:
        with pytest.raises(error):
            call()
    with torch.no_grad():
        assert ops.linear8(x.clone().requires_grad_(), w8).shape == (4, 100)
