"""The operators of a head that answers in the corners of what they accept: temperatures and logits at the ends of binary32, shares that
fall on a border of whole masses, norms of one tensor as both inputs and of many rows, gradients that
a call does not have."""
import math

import pytest
import torch

import paper_1610_02496_amd as pk
from tests.test_gpu_answer import BF16, E, F16, F32, HALF, TINY, check_draws, dev, make, natural, within

pytestmark = pytest.mark.gpu

MOST = float(torch.finfo(F32).max)


# ---- temperatures and logits at the ends of binary32 ------------------------------------------------------------------------

@pytest.mark.parametrize("temperature", [9.5e-38, 9e-38, 5e-38, float(torch.finfo(F32).tiny), 1e-38, 1e-41, 2.0 ** -149])
@pytest.mark.parametrize("words", [1000, 9000])
def test_sample_least_temperatures(words, temperature):
    """32 / T ends at the largest number of binary32 and so do the bins of a histogram; logits of zeros, of both signs, natural ones
    with 0 as their largest, and some that differ by a few T."""
    print("sample", words, temperature, flush=True)
    g = torch.Generator().manual_seed(words)
    l = torch.zeros(5, words)
    l[1] = torch.where(torch.rand(words, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0))
    n = natural(words, 2, words, F32)
    l[2:4] = n - n.amax(1, keepdim=True)
    l[3] *= 1e-38
    l[4] = -torch.floor(torch.rand(words, generator=g) * 8) * torch.tensor(temperature, dtype=F32)
    u = torch.rand(5, generator=g)
    for limits in ({}, {"top_p": 0.5}, {"top_p": 0.9}, {"top_k": 7}, {"top_k": 600}, {"top_k": 2500, "top_p": 0.7}, {"top_k": 300, "top_p": 0.6, "min_p": 0.1}, {"min_p": 0.3}):
        check_draws(l, u, temperature=temperature, **limits)


@pytest.mark.parametrize("temperature", [1e36, 2.0 ** 122, 6e36, 1e37, 2e37, 1e38, MOST, math.inf])
@pytest.mark.parametrize("words", [1000, 9000])
def test_sample_differences_beyond_binary32(words, temperature):
    """Logits whose difference is no number of binary32, at temperatures where the lower ones have mass."""
    print("sample", words, temperature, flush=True)
    g = torch.Generator().manual_seed(words)
    upper = torch.rand(words, generator=g) < 0.5
    l = torch.empty(4, words)
    l[0] = torch.where(upper, 3e38, -3e38)
    l[1] = torch.where(upper, MOST, -MOST)
    l[2] = (torch.rand(words, generator=g, dtype=torch.float64) * 2 - 1).float() * 3.2e38
    l[3] = torch.where(upper, -1e38, l[2].abs())
    l[3, ::7] = -math.inf
    u = torch.rand(4, generator=g)
    half = int(upper.sum())
    for limits in ({}, {"top_p": 0.999}, {"top_p": 0.6}, {"top_k": half + 70}, {"top_k": half + 70, "top_p": 0.9}, {"top_k": 4000, "top_p": 0.99}, {"min_p": 1e-4}):
        check_draws(l, u, temperature=temperature, **limits)


# ---- a share of the whole, where it falls on a border -------------------------------------------------------------------------

@pytest.mark.parametrize("words,deep", [(100000, -31.95), (131072, -31.9), ((1 << 22) + 5, -27.9)])
def test_sample_share_of_whole_masses(words, deep):
    """Two words that share all of the mass: half of it is the first one's.  The others are too deep to have a mass (they round to none), but
    there are so many of them that what is left out would move the border.  Wherever the two are, and at every temperature."""
    print("sample", words, deep, flush=True)
    places = [(3, 900), (5, words - 2), (words - 9, words - 5), (words // 2, words // 2 + 1)]
    l = torch.full((len(places), words), deep)
    for i, at in enumerate(places):
        l[i, list(at)] = 0.0
    for temperature in (1.0, 0.25, 8.0):
        for u, share, which, p in ((0.75, 0.5, 0, 1.0), (0.75, 0.501, 1, 0.5), (0.25, 0.501, 0, 0.5), (0.999, 0.0, 0, 1.0)):
            word, got = pk.ops.sample(dev(l * temperature), torch.full((len(places),), u, device="cuda"), temperature=temperature, top_p=share, min_p=0.4 * (share == 0.5))
            assert word.tolist() == [at[which] for at in places], (temperature, u, share)
            assert bool((got - p).abs().max() <= 2 * E)


@pytest.mark.parametrize("deep,units", [(-31.95, 0.0), (-31.7, 1.0)])
@pytest.mark.parametrize("min_p", [0.0, 0.2])
def test_sample_share_between_two_bins(deep, units, min_p):
    """Two words of different logits, the share such that the first one's mass is just enough, or just not, by what the masses of 100,000 deep words
    are rounded by, to none or to one unit of 2^-45: which words are left is decided by whole masses, wherever the two are."""
    words, unit, found = 100000, 2.0 ** -45, 0
    z = float(torch.tensor(deep, dtype=F32))
    tail, whole = (words - 2) * math.exp(z), (words - 2) * units * unit
    places = [(3, 900), (900, 3), (words - 9, words - 5), (7, words - 1)]
    for i in range(4000):
        share = float(torch.tensor(0.52 + i * 1e-5, dtype=F32))
        low = float(torch.tensor(math.log(1 / share - 1), dtype=F32))
        two = 1 + math.exp(low)
        exact, rough = (share - 2.0 ** -40) * (two + whole), (share - 2.0 ** -40) * (two + tail)
        if not min(exact, rough) < 1 - 2e-11 or not max(exact, rough) > 1 + 2e-11:
            continue
        found += 1
        l = torch.full((len(places), words), deep)
        for k, (a, b) in enumerate(places):
            l[k, a], l[k, b] = 0.0, low
        u = torch.where(torch.tensor([a < b for a, b in places]), 0.99, 0.1)
        word, p = pk.ops.sample(dev(l), dev(u), top_p=share, min_p=min_p)
        left = 2 if exact > 1 else 1
        assert word.tolist() == [at[left - 1] for at in places], (share, low, exact - 1, rough - 1)
        assert bool((p.cpu().double() - (1.0 if left == 1 else math.exp(low) / two)).abs().max() <= 2 * E)
        if found == 6:
            break
    assert found == 6


@pytest.mark.parametrize("words", [64, 1024, 8192, 65536])
def test_sample_share_of_equal_logits(words):
    """Of n equal words an exact share of n are left, at any temperature and magnitude: p is 1 / (share n)."""
    shares = [0.5, 0.75, 0.875, 0.9375, 0.96875, 0.984375]
    rows = 400 * len(shares)
    print("sample", words, rows, flush=True)
    g = torch.Generator().manual_seed(words)
    temperature = torch.exp(torch.rand(rows, generator=g) * 8 - 4)
    top_p = torch.tensor(shares).repeat(400)
    level = torch.randn(rows, 1, generator=g) * 3
    for some in range(0, rows, 600):
        part = slice(some, some + 600)
        word, p = pk.ops.sample(dev(level[part]).repeat(1, words), torch.full((600,), 1 - 2.0 ** -24, device="cuda"), temperature=dev(temperature[part]), top_p=dev(top_p[part]))
        left = (top_p[part] * words).to(torch.int64)
        last = torch.floor((1 - 2.0 ** -24) * left.double()).to(torch.int64)
        bad = (word.cpu() != last).nonzero()[:, 0]
        assert not len(bad), (len(bad), word.cpu()[bad][:5], last[bad][:5], temperature[part][bad][:5], top_p[part][bad][:5])
        assert bool((p.cpu().double() * left - 1).abs().max() <= 2 * E)


@pytest.mark.parametrize("equal", [2, 4096])
def test_sample_no_share_of_very_many_words(equal):
    """top_p of 0, and less than the 2^-40 that a share may lack, leave the likeliest word; where masses are as coarse as they get, too."""
    words = (1 << 30) + 8
    l = torch.full((1, words), -math.inf, dtype=torch.bfloat16, device="cuda")
    at = [5 + i * (words // equal) for i in range(equal)]
    l[0, torch.tensor(at, device="cuda")] = 2.0
    for share, left in ((0.0, 1), (1e-13, 1), (0.5, equal // 2), (0.75, (3 * equal + 3) // 4)):
        print("sample", words, equal, share, flush=True)
        word, p = pk.ops.sample(l, torch.tensor([0.999], device="cuda"), top_p=share)
        assert int(word) == at[int(0.999 * left)] and abs(float(p) * left - 1) <= 2 * E, share


# ---- norms: one tensor as both inputs, many rows ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(10, 64), (33, 1000), (5, 2500), (3, 9000)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rms_norm_gradient_of_one_tensor_as_both(rows, cols, dtype):
    """x as features and as residual: twice the gradient of the sum, of a loss in which half of it, none, or one of the other sign is far off."""
    print("rms", rows, cols, dtype, flush=True)
    x, a, b = (make(i, rows, cols, dtype=dtype) for i in (4, 5, 6))
    leaf = dev(x).requires_grad_()
    y, s = pk.ops.rms_norm(leaf, None, leaf)
    ((y * dev(a)).float().sum() + (s * dev(b)).float().sum()).backward()
    t = 2 * x.double()
    r = 1 / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()
    h, g = t * r, a.double()
    mgh = (g * h).mean(1, keepdim=True)
    ds = r * (g - h * mgh) + b.double()
    # as in test_rms_norm_both_passes: h by rel, the mean by its additions and h's error in each term, then three roundings each; both gradients are
    # rounded to the type and their sum, of equal numbers, is not
    adds = 40.0 + cols / 1024
    rel = (adds / 2 + 4) * E
    err = (rel + 4 * E) * r * (g.abs() + h.abs() * mgh.abs()) + r * h.abs() * (adds + 4) * E * 3 * (g * h).abs().mean(1, keepdim=True) + 2 * E * (ds.abs() + b.double().abs())
    bound = 2 * (HALF[dtype] * ds.abs() + TINY[dtype] + err * (1 + HALF[dtype]))
    assert bool((bound < 0.1 * ds.abs().mean()).all())
    within(leaf.grad, 2 * ds, bound, "gradient of both")


@pytest.mark.parametrize("rows,cols,dtype,rtype", [(39999, 1600, F16, F32), (40000, 1600, F16, F32), (40003, 1599, F16, F32), (40001, 2045, BF16, BF16), (40002, 1777, F32, F32)])
def test_rms_norm_around_the_choice_of_a_variant(rows, cols, dtype, rtype):
    """Both sides of the sizes from which on a row belongs to a wavefront: every row as the same row by itself, the weight's gradient in 64 bits."""
    print("rms", rows, cols, dtype, rtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda t, *s: torch.randn(*s, device="cuda", generator=g).to(t)  # noqa: E731
    x, res, dy, dsum, w = rand(dtype, rows, cols), rand(rtype, rows, cols), rand(dtype, rows, cols), rand(rtype, rows, cols), 1 + 0.2 * rand(F32, cols)
    y, saved = pk.ops.rms_norm_forward(x, w, res)
    dx, dres, dw = pk.ops.rms_norm_backward(dy, saved, dsum)
    adds = 40.0 + cols / 1024
    for part in (slice(0, 9), slice(rows // 2, rows // 2 + 9), slice(rows - 9, rows)):
        z, one = pk.ops.rms_norm_forward(x[part], w, res[part])
        ex, eres, _ = pk.ops.rms_norm_backward(dy[part], one, dsum[part])
        assert torch.equal(saved.x[part], one.x)
        # sums of a row in another order: r is off by half of that, y by it and a step of its type, the gradient's mean by that of the terms
        rel = (adds + 8) * E
        step = 2 * HALF[dtype]
        within(y[part], z, (step + rel) * z.double().abs() + TINY[dtype], "y")
        s, r = one.x.double(), one.rstd.double()[:, None]
        h, gw = s * r, dy[part].double() * w.double()
        size = r * (gw.abs() + h.abs() * (gw * h).abs().mean(1, keepdim=True)) * 3 * rel + 4 * E * eres.double().abs()
        within(dx[part], ex, step * ex.double().abs() + TINY[dtype] + size, "dx")
        within(dres[part], eres, 2 * HALF[rtype] * eres.double().abs() + TINY[rtype] + size, "dresidual")
    dw64, size = (torch.zeros(cols, device="cuda", dtype=torch.float64) for _ in range(2))
    for lo in range(0, rows, 8192):
        part = slice(lo, min(rows, lo + 8192))
        t = dy[part].double() * saved.x[part].double() * saved.rstd[part].double()[:, None]
        dw64 += t.sum(0)
        size += t.abs().sum(0)
    # a lane adds up the rows of its wavefront or workgroup, 512 or 1,024 of these; the rest is joined in some 100 additions
    within(dw, dw64, HALF[F32] * dw64.abs() + (rows / 512 + 140) * E * size, "dweight")


# ---- gradients that a call does not have -----------------------------------------------------------------------------------------

def test_calls_without_gradients_refuse_to_lose_one():
    """Logits, temperatures and features that ask for a gradient, or that carry one of forward mode."""
    ops, x, w8 = pk.ops, dev(make(1, 4, 64)), pk.ops.rows8(dev(make(2, 100, 64)))
    l, u, t = ops.linear8(x, w8), torch.rand(4, device="cuda"), torch.full((4,), 0.7, device="cuda")
    want = ops.sample(l, u, temperature=t, top_p=0.9)
    asks = lambda a: a.clone().requires_grad_()  # noqa: E731
    calls = [lambda f: ops.sample(f(l), u, temperature=t, top_p=0.9), lambda f: ops.sample(l, u, temperature=f(t)), lambda f: ops.linear8(f(x), w8),
             lambda f: ops.rms_norm8(f(x)), lambda f: ops.rms_norm8(x, residual=f(x)), lambda f: ops.rms_norm8(x, f(x[0]))]
    for call in calls:
        with pytest.raises(ValueError, match="no gradient"):
            call(asks)
        with torch.no_grad():
            call(asks)
        call(lambda a: asks(a).detach())
        with torch.autograd.forward_ad.dual_level():
            dual = lambda a: torch.autograd.forward_ad.make_dual(a, torch.ones_like(a))  # noqa: E731
            with pytest.raises(ValueError, match="forward mode"):
                call(dual)
            with torch.no_grad(), pytest.raises(ValueError, match="forward mode"):
                call(dual)
            call(lambda a: dual(a).detach())
            call(lambda a: a)
    with torch.no_grad():
        got = ops.sample(asks(l), u, temperature=asks(t), top_p=0.9)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[1].requires_grad
    # numbers and limits that only choose words carry nothing to lose
    got = ops.sample(l, asks(u), temperature=t, top_p=asks(torch.full((4,), 0.9, device="cuda")))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with torch.inference_mode():
        ops.sample(l, u)
