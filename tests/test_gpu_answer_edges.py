"""The operators of a head that answers where their calls are unusual: norms of tiny rows without eps, gradients in memory of their own,
logits whose largest comes late, whose first are masked or that are nearly all masked, lists that overflow, more rows than one launch takes,
two streams at once.  Tolerances as in test_gpu_answer.py: half a step of the result's type and 2^-24 of the magnitudes per addition."""
import math

import pytest
import torch

import paper_1610_02496_amd as pk
from tests.test_gpu_answer import BF16, E, F16, F32, HALF, LIMITS, TINY, answer, check_draws, dev, make, natural, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [5, 300, 1500, 9000])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-32])
def test_rms_norm_of_tiny_rows(cols, eps):
    """Squares that binary32 does not hold; eps that is nothing or next to them."""
    x = make(1, 6, cols, scale=1.0)
    x[1] *= 1e-16
    x[2] *= 1e-19
    x[3] *= 1e-25
    x[4] *= 1e-37
    x[5] = 0
    y, saved = pk.ops.rms_norm_forward(dev(x), eps=eps)
    eps32 = float(torch.tensor(eps, dtype=F32))
    ms = x.double().square().mean(1, keepdim=True)
    r64 = 1 / (ms + eps32).sqrt()
    rel = ((40.0 + cols / 1024) / 2 + 6) * E
    within(saved.rstd[:5, None], r64[:5], rel * r64[:5], "rstd")
    within(y[:5], (x.double() * r64)[:5], (rel + 2 * E) * (x.double() * r64)[:5].abs() + 1e-37, "y")
    assert float(y[5].abs().max()) == 0
    c, _ = pk.ops.rms_norm8(dev(x), eps=eps)
    back = c.restore()
    assert float(back[5].abs().max()) == 0
    for i in range(4):   # (steps of row 4 are no normal numbers)
        want = (x[i].double() * r64[i]).abs().max()
        within(back[i], x[i].double() * r64[i], float(want) * (0.5 / 127 + 64 * E), "row %d in 8 bits" % i)


def test_rms_norm_gradients_are_tensors_of_their_own():
    x, res, w = (dev(make(i, *s)).requires_grad_() for i, s in ((1, (20, 64)), (2, (20, 64)), (3, (64,))))
    y, s = pk.ops.rms_norm(x, w, res)
    (y.square().sum() + s.sum()).backward()
    assert torch.equal(x.grad, res.grad) and x.grad.data_ptr() != res.grad.data_ptr()
    before = res.grad.clone()
    x.grad.zero_()
    assert torch.equal(res.grad, before)
    y, s = pk.ops.rms_norm(x, w, res)
    s += 1                                     # what the backward pass reads
    with pytest.raises(RuntimeError):
        y.sum().backward()
    # one tensor as both
    a = dev(make(4, 10, 64)).requires_grad_()
    y, _ = pk.ops.rms_norm(a, None, a)
    y.square().sum().backward()
    b = a.detach().double().requires_grad_()
    t = 2 * b
    (t / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()).square().sum().backward()
    # dx is 2 r (g - h mean(g h)) with g = 2 h, so a difference of nearly equal numbers: off by their roundings
    within(a.grad, b.grad, 200 * E * 2 * float((2 / t.detach().square().mean(1).sqrt()).max()) * 8, "gradient of both")


@pytest.mark.parametrize("words", [3000, 9000, 30011, 141000])
def test_sample_largest_logit_comes_late(words):
    """The first logits say nothing of the largest: masked, tiny, or far below (further than a histogram reaches)."""
    g = torch.Generator().manual_seed(words)
    l = natural(words, 8, words, F32)
    l[0, :-7] = -math.inf
    l[1, : words // 2] = -math.inf
    l[2, : words // 2] -= 20.0
    l[3, : words // 2] -= 40.0
    l[4, -1] = 100.0
    l[5, -3:] = 1e30
    l[6, words // 2:] += 3e5
    l[7, : words - words // 8] = torch.finfo(F32).min
    u = torch.rand(8, generator=g)
    for limits in LIMITS + [{"top_p": 0.9, "temperature": 0.05}, {"top_k": 2500, "temperature": 0.05}, {"top_p": 0.9, "temperature": 1e4}, {"top_p": 0.9, "temperature": 1e-30},
                            {"top_p": 0.5, "temperature": 1e30}]:
        check_draws(l, u, **limits)


@pytest.mark.parametrize("words", [700, 20000])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_sample_mostly_masked(words, dtype):
    g = torch.Generator().manual_seed(2)
    l = natural(1, 6, words, dtype)
    l[:, torch.rand(words, generator=g) < 0.99] = -math.inf
    l[1, 5:] = -math.inf
    l[2] = -math.inf
    l[2, words // 2] = -3.0
    for limits in LIMITS:
        check_draws(l, torch.rand(6, generator=g), **limits)


def test_sample_lists_that_overflow():
    """Few values, so that a bin, or the words among which the top_k are, holds more than a list; the same result every time."""
    g = torch.Generator().manual_seed(3)
    l = (torch.randint(0, 40, (6, 60000), generator=g).float() / 8).to(BF16)
    u = torch.rand(6, generator=g)
    for limits in LIMITS + [{"top_p": 0.95, "temperature": 5.0}, {"top_k": 900, "top_p": 0.5, "min_p": 0.3}, {"top_k": 20000, "top_p": 0.7, "min_p": 0.6}]:
        check_draws(l, u, **limits)
        a, b = (pk.ops.sample(dev(l), dev(u), **limits) for _ in range(2))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_sample_rows_of_several_launches():
    rows = (1 << 21) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    l = torch.randn(rows, 2, device="cuda", generator=g)
    u = torch.rand(rows, device="cuda", generator=g)
    word, p = pk.ops.sample(l, u)
    share = torch.softmax(l.double(), 1)
    clear = (share[:, 0] - u.double()).abs() > 1e-9
    assert bool(((word == (u.double() >= share[:, 0])) | ~clear).all())
    want = share.gather(1, word[:, None])[:, 0]
    assert bool(((p.double() - want).abs() <= 2 * E * want + 1e-12).all())


def test_two_streams_at_once():
    sets = []
    for k in range(2):
        sets.append((dev(make(k, 500, 777, dtype=BF16)), dev(make(k + 5, 500, 777)), dev(make(k + 9, 777)), pk.ops.rows8(dev(make(k + 4, 9000, 777, scale=0.1))),
                     torch.rand(500, device="cuda"), {"top_p": 0.8, "top_k": 3000 * k}))
    want = [answer(*s) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for again in range(3):
        for k, (s, stream) in enumerate(zip(sets, streams)):
            with torch.cuda.stream(stream):
                got[k].append(answer(*s))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))


def test_sample_limits_of_other_kinds():
    l, u = dev(natural(1, 4, 500, F32)), torch.rand(4, device="cuda")
    for bad in ({"top_k": 2.5}, {"top_k": "5"}, {"temperature": None}, {"top_p": [0.5]}):
        with pytest.raises(TypeError):
            pk.ops.sample(l, u, **bad)
    want = pk.ops.sample(l, u, top_k=7, top_p=0.5)
    import numpy as np
    got = pk.ops.sample(l, u, top_k=np.int64(7), top_p=np.float32(0.5), temperature=1)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    assert torch.equal(pk.ops.sample(l, u, top_k=1 << 70)[0], pk.ops.sample(l, u)[0])


def test_logits_of_strided_features():
    """Features and stream that are slices, transposed or expanded."""
    x = dev(make(1, 40, 24, dtype=F16))
    w8 = pk.ops.rows8(dev(make(2, 300, 40)))
    assert torch.equal(pk.ops.linear8(x.t(), w8), pk.ops.linear8(x.t().contiguous(), w8))
    one = dev(make(3, 1, 64))
    y, s = pk.ops.rms_norm_forward(one.expand(9, 64), residual=dev(make(4, 64, 9)).t())
    z, t = pk.ops.rms_norm_forward(one.repeat(9, 1), residual=dev(make(4, 64, 9)).t().contiguous())
    assert torch.equal(y, z) and torch.equal(s.x, t.x)
    dx, dres, _ = pk.ops.rms_norm_backward(one.expand(9, 64), s, one.expand(9, 64))
    ex, eres, _ = pk.ops.rms_norm_backward(one.repeat(9, 1), t, one.repeat(9, 1))
    assert torch.equal(dx, ex) and torch.equal(dres, eres)
    wide = dev(make(5, 700))[::2][:300]
    words = pk.ops.Rows8.of(w8.q.t().contiguous().t(), wide.abs())
    assert torch.equal(pk.ops.linear8(x.t(), words), pk.ops.linear8(x.t(), pk.ops.Rows8.of(w8.q.contiguous(), wide.abs().contiguous())))
    assert HALF[F16] == 2.0 ** -11


@pytest.mark.parametrize("rows,cols,dtype,rtype", [(16390, 1030, BF16, F32), (16385, 2048, F32, F32), (65540, 2048, BF16, F32), (65600, 2047, F16, F16)])
def test_rms_norm_of_many_rows(rows, cols, dtype, rtype):
    """So many rows that those of up to 2,048 columns belong to a wavefront; the reference in 64 bits on the device, some rows at a time."""
    print("rms", rows, cols, dtype, rtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda t, *s: torch.randn(*s, device="cuda", generator=g).to(t)  # noqa: E731
    x, res, dy, dsum, w = rand(dtype, rows, cols), rand(rtype, rows, cols), rand(dtype, rows, cols), rand(rtype, rows, cols), 1 + 0.2 * rand(F32, cols)
    y, saved = pk.ops.rms_norm_forward(x, w, res)
    dx, dres, dw = pk.ops.rms_norm_backward(dy, saved, dsum)
    rel, dw64, size = 30 * E, torch.zeros(cols, device="cuda", dtype=torch.float64), torch.zeros(cols, device="cuda", dtype=torch.float64)
    for lo in range(0, rows, 8192):
        part = slice(lo, min(rows, lo + 8192))
        s = (x[part].float() + res[part].float()).to(rtype)
        assert torch.equal(saved.x[part], s)
        s = s.double()
        r = 1 / (s.square().mean(1, keepdim=True) + 1e-6).sqrt()
        h, gw = s * r, dy[part].double() * w.double()
        y64 = h * w.double()
        assert bool(((y[part].double() - y64).abs() <= HALF[dtype] * y64.abs() + TINY[dtype] + rel * y64.abs() * (1 + HALF[dtype])).all())
        mean = (gw * h).mean(1, keepdim=True)
        d = r * (gw - h * mean) + dsum[part].double()
        err = rel * r * (gw.abs() + h.abs() * mean.abs()) + r * h.abs() * 50 * E * 3 * (gw * h).abs().mean(1, keepdim=True) + 2 * E * (d.abs() + dsum[part].double().abs())
        assert bool(((dx[part].double() - d).abs() <= HALF[dtype] * d.abs() + TINY[dtype] + err * (1 + HALF[dtype])).all())
        assert bool(((dres[part].double() - d).abs() <= HALF[rtype] * d.abs() + TINY[rtype] + err * (1 + HALF[rtype])).all())
        dw64 += (dy[part].double() * h).sum(0)
        size += (dy[part].double() * h).abs().sum(0)
    # a lane adds up the rows of its wavefront (a workgroup: of 2,048 wavefronts; else of 768 or 1,024 workgroups), the rest is joined in some 100 additions
    lines = rows / 768 + 100
    assert bool(((dw.double() - dw64).abs() <= HALF[F32] * dw64.abs() + (lines + 40) * E * size).all())
    c, total = pk.ops.rms_norm8(x, w, res)
    assert torch.equal(total, saved.x)
    s = saved.x[-100:].float() * w
    step = (s.double().abs().amax(1, keepdim=True) / 127).float().double()
    assert torch.equal(c.q[-100:].double(), (s.double() / step).round().clamp(-127, 127))
