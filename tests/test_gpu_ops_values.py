"""The head's operators on the GPU over the values that a program may bring: rows of mixed magnitudes, infinities, gradients of very
different size, sizes at which every loop takes a second turn.  Against plain implementations in 64 bits."""
import pytest
import torch

import paper_1610_02496_amd as pk

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ROUND = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
E = 2.0 ** -24


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def words(seed, rows, vocab):
    return torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(seed))


def within(got, want, bound, what):
    got, want = got.double().cpu(), want.double().cpu()
    bound = (bound if isinstance(bound, torch.Tensor) else torch.tensor(float(bound))).double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%s: %d of %d values, worst %.3g against a bound of %.3g" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound.expand_as(off)[bad].min()))


def xent64(x, w, t, g):
    """On the operands' device, which is where sizes are large."""
    x, w = x.double(), w.double()
    logits = torch.mm(x, w.t())
    lse = torch.logsumexp(logits, 1)
    i, has, to = torch.arange(len(t), device=x.device), t >= 0, t.clamp(min=0)
    loss = torch.where(has, lse - logits[i, to], 0.0)
    d = (logits - lse[:, None]).exp()
    d[i, to] -= 1
    d *= torch.where(has, g.double(), 0.0)[:, None]
    return loss, lse, d, logits


def rounding(x, w, logits):
    """What a logit in binary32 may be off: the roundings of its sum walk at random, so that four standard deviations of
    sqrt(columns) steps of 2^-24 of the sum of magnitudes hold, and the exponentials add 2^-22 of the logit's size."""
    mag = torch.mm(x.double().abs(), w.double().abs().t())
    return 4 * (x.shape[1] + 8) ** 0.5 * E * mag.amax(1) + 2 ** -22 * (1 + logits.abs().amax(1))


def both_passes32(x, w, t, g):
    """Forward and backward pass in binary32 on the GPU against 64 bits."""
    x, w, t, g = x.to("cuda", F32), w.to("cuda", F32), t.cuda(), g.to("cuda", F32)
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    loss64, lse64, d, logits = xent64(x, w, t, g)
    off = rounding(x, w, logits)
    within(lse, lse64, off, "lse")
    within(loss, loss64, 2 * off, "loss")
    dx, dw = pk.ops.linear_cross_entropy_backward(g, x, w, t, lse)
    p = d.abs()
    p[torch.arange(len(t), device="cuda"), t.clamp(min=0)] += torch.where(t >= 0, g.double(), 0.0)
    d_err = p * (4 * off[:, None] + 2 ** -20)
    x64, w64 = x.double(), w.double()
    for got, d64, err, other, what in ((dx, d, d_err, w64, "dx"), (dw, d.t().contiguous(), d_err.t().contiguous(), x64, "dweight")):
        want, sums = torch.mm(d64, other), torch.mm(d64.abs(), other.abs())
        within(got, want, torch.mm(err, other.abs()) + 4 * (d64.shape[1] + 8) ** 0.5 * E * sums + E * want.abs() + 1e-37, what)


MIXED = {
    "one magnitude": lambda x, w: None,
    "a large column without weight": lambda x, w: (x[:, 3].mul_(1e8), w[:, 3].zero_()),
    "a large column of small weight": lambda x, w: (x[:, 3].mul_(1e8), w[:, 3].mul_(1e-8)),
    "a very large column without weight": lambda x, w: (x[:, 3].mul_(1e10), w[:, 3].zero_()),
    "an unused column that hides all others": lambda x, w: (x[:, 3].fill_(1e30), w[:, 3].zero_()),
    "a large column of the weights": lambda x, w: (w[:, 5].mul_(1e9), x[:, 5].mul_(1e-9)),
    "two columns against each other, 2^16": lambda x, w: (x[:, 3].mul_(2.0 ** 16), w[:, 3].mul_(2.0 ** -16), x[:, 4].mul_(2.0 ** -16), w[:, 4].mul_(2.0 ** 16)),
    "two columns against each other, 2^20": lambda x, w: (x[:, 3].mul_(2.0 ** 20), w[:, 3].mul_(2.0 ** -20), x[:, 4].mul_(2.0 ** -20), w[:, 4].mul_(2.0 ** 20)),
    "sparse rows, 2^30": lambda x, w: (x[:, 2:].mul_(normal(9, *x[:, 2:].shape) > 2), x[:, 0].fill_(1), x[:, 1].mul_(2.0 ** -30),
                                       w.mul_(torch.arange(w.shape[1]) < 2), w[:, 1].mul_(2.0 ** 30)),
    "single rows of counts": lambda x, w: (x[::7, 3].mul_(3e6), w[:, 3].mul_(1e-7)),
}


@pytest.mark.parametrize("rows,vocab,cols", [(20, 1000, 512), (90, 700, 513), (300, 9000, 512), (300, 22001, 500)])
@pytest.mark.parametrize("what", MIXED)
def test_binary32_rows_of_mixed_magnitudes(what, rows, vocab, cols):
    print("mixed magnitudes:", what, rows, vocab, cols, flush=True)
    x, w = normal(1, rows, cols), normal(2, vocab, cols) * (4.0 / cols ** 0.5)
    MIXED[what](x, w)
    t = words(3, rows, vocab)
    t[rows // 2] = -1
    both_passes32(x, w, t, normal(4, rows).abs() + 0.1)


def test_binary32_tiles_of_either_kind_side_by_side():
    """Only some words and some rows are of mixed magnitudes: tiles beside and below each other are of either kind."""
    rows, vocab, cols = 700, 5000, 200
    x, w = normal(1, rows, cols), normal(2, vocab, cols) * (3.0 / cols ** 0.5)
    x[100:130, 7] *= 1e9
    w[2100:2300, 8] *= 1e9
    x[:, 8] *= 1e-9
    w[:, 7] *= 1e-9
    both_passes32(x, w, words(3, rows, vocab), normal(4, rows).abs() + 0.1)


@pytest.mark.parametrize("rows", [3, 40, 90, 300])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_words_of_infinite_weight(rows, dtype):
    """A word whose logit is minus infinity takes no part: the others' loss and gradients are those of a vocabulary without it."""
    vocab, cols = 900, 96
    x, w = normal(1, rows, cols).to("cuda", dtype), (normal(2, vocab, cols) * 0.3).to("cuda", dtype)
    x[:, 5] = x[:, 5].abs() + 0.125
    x[:, 6:9] = 1.0                       # (a value of few bits: nothing of it is left for a second plane)
    masked = torch.tensor([0, 17, 255, 256, 899], device="cuda")
    w[masked, 5] = float("-inf")
    w[masked, 6] = float("-inf")
    kept = torch.ones(vocab, dtype=torch.bool, device="cuda")
    kept[masked] = False
    t = words(3, rows, vocab - 5)
    t[2] = -1
    at = torch.arange(vocab, device="cuda")[kept][t.clamp(min=0).cuda()]
    at[2] = -1
    g = torch.ones(rows, device="cuda")
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, at)
    loss64, lse64, d, logits = xent64(x, w[kept], t.cuda(), g)
    off = rounding(x, w[kept], logits) + 2 ** -20
    within(lse, lse64, off, "lse")
    within(loss, loss64, 2 * off, "loss")
    _, dw = pk.ops.linear_cross_entropy_backward(g, x, w, at, lse, need_x=False)
    assert bool(torch.isfinite(dw).all()) and float(dw[masked].abs().sum()) == 0
    want = torch.mm(d.t().contiguous(), x.double())
    assert float((dw[kept].double() - want).norm() / want.norm()) < {F32: 2.0 ** -18, F16: 2.0 ** -10, BF16: 2.0 ** -7}[dtype]


def spread(dtype, rows=200, vocab=9000, cols=128):
    """A batch whose dloss spans 2^26: sizes at which binary16 holds dx and dweight themselves, and a projection with a common part, so that
    the softmax' many small probabilities make up much of dx."""
    x, w = (normal(1, rows, cols) * 0.3).to("cuda", dtype), (normal(2, vocab, cols) * 0.3 + 0.5).to("cuda", dtype)
    t = words(3, rows, vocab)
    t[5] = -1
    g = (1 + normal(4, rows).abs().clamp(max=0.9)) * 2.0 ** (12 - torch.arange(rows) % 27).double()
    return x, w, t.cuda(), g.to("cuda", F32)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rows_of_small_gradient_keep_their_precision(dtype):
    x, w, t, g = spread(dtype)
    rows, cols = x.shape
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    dx, dw = pk.ops.linear_cross_entropy_backward(g, x, w, t, lse)
    _, _, d, logits = xent64(x, w, t, g)
    x64, w64, has = x.double(), w.double(), t >= 0
    hold = {F32: 2.0 ** -22, F16: 2.0 ** -11, BF16: 2.0 ** -8}[dtype]
    size = torch.where(has, g.double(), 0.0)
    p = d.abs()
    p[torch.arange(rows, device="cuda"), t.clamp(min=0)] += size
    # d is rounded relative to its row's dloss; binary16's steps end at 2^-24 after 2^14
    d_err = hold * d.abs() + p * (4 * rounding(x, w, logits)[:, None] + 2 ** -20) + size[:, None] * 2.0 ** -38
    tiny = 2.0 ** -25 if dtype is F16 else 1e-37
    want = torch.mm(d, w64)
    within(dx, want, ROUND[dtype] * want.abs() * 1.01 + tiny + torch.mm(d_err, w64.abs()) + (len(w) + 8) * E * torch.mm(p, w64.abs()), "dx")
    want = torch.mm(d.t().contiguous(), x64)
    # the features of a row of small dloss are brought to it: 2^-39 of the largest feature times the largest dloss, in binary16
    moved = (p / size.clamp(min=1e-300)[:, None]).sum(0)[:, None] * float(g.max()) * float(x64.abs().max()) * 2.0 ** -38
    within(dw, want, ROUND[dtype] * want.abs() * 1.01 + tiny + torch.mm(d_err.t().contiguous(), x64.abs()) + (rows + 8) * E * torch.mm(p.t().contiguous(), x64.abs()) + moved, "dweight")


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_a_gradient_that_is_not_finite_stays_in_its_row(dtype, value):
    x, w, t, g = spread(dtype, vocab=3000)
    g[17] = value
    lse = pk.ops.linear_cross_entropy_forward(x, w, t)[1]
    dx = pk.ops.linear_cross_entropy_backward(g, x, w, t, lse, need_weight=False)[0]
    assert not bool(torch.isfinite(dx[17]).any())
    left, t2, g2 = torch.arange(200) != 17, t.clone(), g.clone()
    t2[17], g2[17] = -1, 0.0
    want = pk.ops.linear_cross_entropy_backward(g2, x, w, t2, lse, need_weight=False)[0]
    assert torch.equal(dx[left], want[left])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_no_gradient_at_all(dtype):
    x, w, t, _ = spread(dtype, rows=70, vocab=300)
    lse = pk.ops.linear_cross_entropy_forward(x, w, t)[1]
    dx, dw = pk.ops.linear_cross_entropy_backward(torch.zeros(70, device="cuda"), x, w, t, lse)
    assert float(dx.abs().sum()) == 0 and float(dw.abs().sum()) == 0


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab,cols", [(1, 1), (777, 33), (9000, 520)])
def test_cross_entropy_of_no_rows(dtype, vocab, cols):
    x, w, t = torch.empty(0, cols, device="cuda", dtype=dtype), normal(2, vocab, cols).to("cuda", dtype), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    dx, dw = pk.ops.linear_cross_entropy_backward(torch.empty(0, device="cuda"), x, w, t, lse)
    assert loss.shape == lse.shape == (0,) and dx.shape == (0, cols) and dw.shape == (vocab, cols) and bool((dw == 0).all())
    w.requires_grad_()
    loss = pk.ops.linear_cross_entropy(x, w, t)
    loss.backward()
    assert float(loss) == 0 and bool((w.grad == 0).all())


def test_a_loss_may_be_changed_in_place():
    x, w, t = normal(1, 90, 64).to("cuda", BF16), normal(2, 700, 64).mul(0.2).to("cuda", BF16), words(3, 90, 700).cuda()
    weight, left_out = torch.rand(90, device="cuda"), torch.arange(90, device="cuda") % 9 == 7
    grads = []
    for in_place in (False, True):
        xs, ws = x.clone().requires_grad_(), w.clone().requires_grad_()
        loss = pk.ops.linear_cross_entropy(xs, ws, t, "none")
        if in_place:
            loss.mul_(weight)
            loss[left_out] = 0
        else:
            loss = torch.where(left_out, 0.0, loss * weight)
        loss.sum().backward()
        grads.append((xs.grad, ws.grad))
    assert torch.equal(grads[0][0], grads[1][0]) and torch.equal(grads[0][1], grads[1][1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_checkpoints_of_the_largest_numbers_are_finite(dtype):
    """The type's largest and lowest value, as masks hold them, come back within half a step."""
    most = torch.finfo(dtype).max
    x = normal(1, 9, 300).to(dtype)
    x[0, 5], x[1, 7], x[2, :] = most, -most, most
    x[3, 100] = -most * (1 - 2.0 ** -8)
    x[4, 200], x[4, 201] = most, most / 2
    for c in (pk.ops.checkpoint8(x.cuda()), pk.ops.layer_norm_forward(x.cuda(), checkpoint=True)[1].checkpoint):
        got = c.restore().double().cpu()
        step = c.scale.double().cpu().repeat_interleave(128, 1)[:, :300]
        assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(c.scale).all())
        assert bool(((got - x.double()).abs() <= step * (0.5 + 2.0 ** -15) + ROUND[dtype] * x.double().abs()).all())


def test_features_without_a_dimension_are_refused():
    w, t = torch.zeros(10, 1, device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")
    for x in (torch.tensor(1.0, device="cuda"), torch.zeros((), device="cuda")):
        for call in (lambda: pk.ops.linear_cross_entropy(x, w, t), lambda: pk.ops.linear_cross_entropy_backward(x, x, w, t, x), lambda: pk.ops.layer_norm(x),
                     lambda: pk.ops.checkpoint8(x)):
            with pytest.raises(ValueError):
                call()
    loss, lse = pk.ops.linear_cross_entropy_forward(torch.ones(1, device="cuda"), w, t)   # a single row, of one column
    assert loss.shape == () and abs(float(lse) - 2.302585) < 1e-6
