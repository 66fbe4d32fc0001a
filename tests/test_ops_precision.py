"""That the tests of binary32 gradients would see a missing product of planes: the planes' arithmetic on the CPU, the mistake planted there."""
import torch

E = 2.0 ** -24


def planes(v):
    """Three numbers of bfloat16, cut off, whose sum is the value."""
    out = []
    for _ in range(3):
        cut = (v.view(torch.int32) & -65536).view(torch.float32)
        out.append(cut.double())
        v = v - cut
    assert bool((v == 0).all())
    return out


ALL = [(2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0)]


def error_of(segments, rows=120, vocab=700, cols=90):
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(rows, cols, generator=g), torch.randn(vocab, cols, generator=g) * 2 / cols ** 0.5
    d = torch.softmax(x.double() @ w.double().T, 1)
    d[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] -= 1
    d = d.float()
    pd, pw = planes(d), planes(w)
    got = sum(pd[a] @ pw[b] for a, b in segments)
    want = d.double() @ w.double()
    return float((got - want).norm() / want.norm())


def test_a_missing_product_of_planes_is_seen():
    """The bound of the GPU tests is 2^-18 of the whole gradient's norm."""
    assert error_of(ALL) < 2.0 ** -21
    assert error_of(ALL[3:]) > 2.0 ** -18          # without the three smallest
    assert error_of(ALL[:3] + ALL[4:]) > 2.0 ** -18 and error_of(ALL[:4] + ALL[5:]) > 2.0 ** -18
