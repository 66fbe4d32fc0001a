"""The head's operators on the GPU at sizes where every loop over rows, words, blocks or pieces takes a second turn, the last of them ragged.
Against plain implementations in 64 bits on the GPU."""
import pytest
import torch

import paper_1610_02496_amd as pk
from tests.test_gpu_ops_values import BF16, E, F16, F32, ROUND, within, xent64

pytestmark = pytest.mark.gpu


def normal(seed, *shape):
    """On the GPU: these tests are of millions of values."""
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def held64(x):
    """What an 8-bit checkpoint stands for; steps are binary32."""
    n, h = x.shape
    out = torch.empty(n, h, dtype=torch.float64, device=x.device)
    for a in range(0, h, 128):
        p = x[:, a:a + 128].float()
        c = p.abs().amax(1, keepdim=True) / torch.full((1,), 127.0, device=x.device)
        out[:, a:a + 128] = (torch.where(c > 0, torch.round(p / c), 0.0).clamp(-127, 127) * c).double()
    return out


# a wavefront, a workgroup of 256 and one of 512 per row; rows beyond 2,048 workgroups forward, 768, 1,024 and 512 backward; rows too wide for
# registers: 16,384 workgroups, 256 parts of the column sums
@pytest.mark.parametrize("rows,cols", [(9001, 100), (9001, 1000), (2500, 1500), (2311, 3333), (1100, 5000), (2077, 8192), (300, 9000), (16_500, 8200)])
@pytest.mark.parametrize("dtype,wtype,held", [(F32, F32, False), (BF16, F32, True), (F16, F16, False)])
def test_norm_of_many_rows(rows, cols, dtype, wtype, held):
    print("norm", rows, cols, dtype, held, flush=True)
    x = (normal(1, rows, cols) * (1 + torch.arange(rows, device="cuda")[:, None] % 7) + torch.arange(rows, device="cuda")[:, None] % 3).to(dtype)
    w, b, dy = (1 + 0.3 * normal(2, cols)).to(wtype), (0.2 * normal(3, cols)).to(wtype), normal(4, rows, cols).to(dtype)
    y, saved = pk.ops.layer_norm_forward(x, w, b, checkpoint=held)
    dx, dw, db = pk.ops.layer_norm_backward(dy, saved)
    tiny = {F32: 1e-37, F16: 2.0 ** -24, BF16: 1e-37}[dtype]
    adds = 64.0 + cols / 512         # additions that a value of a row passes through
    dw64 = db64 = dw_off = db_off = 0
    for lo in range(0, rows, 4096):
        s = slice(lo, min(rows, lo + 4096))
        v, g = x[s].double(), dy[s].double()
        m = v.mean(1, keepdim=True)
        r = 1 / ((v - m).square().mean(1, keepdim=True) + 1e-5).sqrt()
        h = (v - m) * r
        most = v.abs().amax(1, keepdim=True)
        rel = 4 * adds * E * (1 + most * r)
        within(saved.mean[s, None], m, adds * E * most, "mean")
        within(saved.rstd[s, None], r, rel * r, "rstd")
        y64 = h * w.double() + b.double()
        h_err = rel * (1 + h.abs())
        within(y[s], y64, ROUND[dtype] * y64.abs() * 1.01 + tiny + h_err * w.double().abs() + 4 * E * (h.abs() * w.double().abs() + b.double().abs()), "y")
        if held:
            v = held64(x[s])
            assert torch.equal(pk.ops.Checkpoint8(saved.checkpoint.q[s], saved.checkpoint.scale[s], dtype).restore(F32).double(), v)
            h = (v - m) * r
            h_err = rel * (1 + h.abs())
        gw = g * w.double()
        mgh = (gw * h).mean(1, keepdim=True)
        want = r * (gw - gw.mean(1, keepdim=True) - h * mgh)
        size = gw.abs() + gw.abs().mean(1, keepdim=True) + h.abs() * (gw * h).abs().mean(1, keepdim=True)
        err = r * ((rel + 2 * adds * E) * size + h_err * mgh.abs() + h.abs() * (gw.abs() * h_err).mean(1, keepdim=True))
        within(dx[s], want, ROUND[dtype] * want.abs() * 1.01 + tiny + err, "dx")
        dw64, db64 = dw64 + (g * h).sum(0), db64 + g.sum(0)
        n = (rows / 256 + 64) * E
        dw_off, db_off = dw_off + n * (g * h).abs().sum(0) + (g.abs() * h_err).sum(0), db_off + n * g.abs().sum(0)
    wtiny = {F32: 1e-37, F16: 2.0 ** -24}[wtype]
    within(dw, dw64, ROUND[wtype] * dw64.abs() * 1.01 + wtiny + dw_off, "dweight")
    within(db, db64, ROUND[wtype] * db64.abs() * 1.01 + wtiny + db_off, "dbias")


@pytest.mark.parametrize("rows,cols,pad", [(40_001, 300, 0), (70_003, 128, 3), (3001, 4100, 8)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_checkpoints_of_many_blocks(rows, cols, pad, dtype):
    """More than the 65,536 blocks that one turn takes."""
    x = (normal(1, rows, cols + pad) * (1 + torch.arange(rows, device="cuda")[:, None] % 5)).to(dtype)[:, :cols]
    c = pk.ops.checkpoint8(x)
    want = held64(x)
    assert torch.equal(c.restore(F32).double(), want)
    assert torch.equal(c.restore(), want.float().to(dtype))


@pytest.mark.parametrize("rows,vocab,cols", [(40, 140_001, 777), (3, 140_001, 64), (20, 140_003, 500), (64, 70_001, 1100)])
@pytest.mark.parametrize("dtype,pad", [(F16, 0), (BF16, 5), (F32, 3)])
def test_few_rows_of_many_words(rows, vocab, cols, dtype, pad):
    """A wavefront takes several tiles of 16 words: the largest logit of a row lies in its first, in its last, or in one between."""
    print("few rows", rows, vocab, cols, dtype, flush=True)
    x = normal(1, rows, cols + pad).to(dtype)[:, :cols]
    w = (normal(2, vocab, cols + pad) * (1.0 / cols ** 0.5)).to(dtype)[:, :cols]
    place = torch.tensor([0, 5, vocab // 2, vocab - 20, vocab - 1, 65_000, 65_540], device="cuda")[torch.arange(rows, device="cuda") % 7]
    place = place + torch.where(place < vocab // 2, 17, -17) * (torch.arange(rows, device="cuda") // 7)   # (a word of its own for every row)
    w[place] = (x.float() * (30.0 / x.float().square().sum(1, keepdim=True))).to(dtype)   # a logit of 30
    t = torch.where(torch.arange(rows, device="cuda") % 2 == 0, place, torch.arange(rows, device="cuda") * 1999 % vocab)
    t[rows // 2] = -1
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    loss64, lse64, _, logits = xent64(x, w, t, torch.ones(rows, device="cuda"))
    assert bool((logits.argmax(1) == place).all())
    mag = torch.mm(x.double().abs(), w.double().abs().t()).amax(1)
    off = 4 * (cols + 8) ** 0.5 * E * mag + 2 ** -21 * (1 + logits.abs().amax(1))
    within(lse, lse64, off, "lse")
    within(loss, loss64, 2 * off, "loss")


def borders(rows, vocab, seed):
    """Targets on both sides of every 256th word, where pieces and tiles meet, then random ones; some rows have none."""
    at = torch.arange(256, vocab, 256)
    edge = torch.stack([at - 1, at], 1).reshape(-1)[:rows]
    rest = torch.randint(0, vocab, (max(0, rows - len(edge)),), generator=torch.Generator().manual_seed(seed))
    t = torch.cat([edge, rest])[torch.randperm(rows, generator=torch.Generator().manual_seed(seed))]
    t[::17] = -1
    return t.cuda()


# rows, words, columns, type, elements between rows; words of a piece: forward / backward (of the last one fewer)
@pytest.mark.parametrize("rows,vocab,cols,dtype,pad", [
    (600, 70_001, 1000, F32, 0),      # 65,280 / 21,760, filled to whole rounds
    (100, 70_001, 1000, F32, 3),      # 65,536 / 23,552, even
    (3000, 40_001, 100, F32, 0),      # all / 10,752, filled
    (2100, 60_001, 250, F32, 1),      # all / 20,224, even
    (90, 141_000, 1001, F16, 0),      # 131,072 / 131,072 (rows that are not aligned)
    (600, 100_001, 1500, BF16, 5),    # 87,040 / 87,040
    (6000, 50_001, 75, F16, 5),       # all / 20,480, filled
    (9000, 30_000, 64, BF16, 0),      # all / 14,336, filled
    (20_000, 14_001, 40, BF16, 3),    # all / 4,864, even
])
def test_cross_entropy_of_several_pieces(rows, vocab, cols, dtype, pad):
    print("pieces", rows, vocab, cols, dtype, pad, flush=True)
    x = normal(1, rows, cols + pad).to(dtype)[:, :cols]
    w = (normal(2, vocab, cols + pad) * (2.0 / cols ** 0.5)).to(dtype)[:, :cols]
    t = borders(rows, vocab, 3)
    g = normal(4, rows).abs() + 0.1
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    loss64, lse64, d, logits = xent64(x, w, t, g)
    off = torch.zeros(rows, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 2000):
        off[lo:lo + 2000] = 4 * (cols + 8) ** 0.5 * E * torch.mm(x[lo:lo + 2000].double().abs(), w.double().abs().t()).amax(1)
    off += (2 ** -20 if dtype is not F32 else 2 ** -22) * (1 + logits.abs().amax(1))
    del logits
    within(lse, lse64, off, "lse")
    within(loss, loss64, 2 * off, "loss")
    dx, dw = pk.ops.linear_cross_entropy_backward(g, x, w, t, lse)
    assert float(dx[t < 0].abs().sum()) == 0
    compare_gradients(dx, dw, d, x, w, dtype)


def compare_gradients(dx, dw, d, x, w, dtype):
    """By the norm of every row, and of all: the roundings of the type (of d, and of the result) are independent of each other, and
    binary32 has those of the planes, 2^-21 of a product, and of its sums, which walk at random: sqrt(k) 2^-24, k up to 2^15 here."""
    each = {F32: 2.0 ** -15, F16: 2.0 ** -9, BF16: 2.0 ** -6}[dtype]
    whole = {F32: 2.0 ** -18, F16: 2.0 ** -10.5, BF16: 2.0 ** -7.5}[dtype]
    for got, want, what in ((dx, torch.mm(d, w.double()), "dx"), (dw, torch.mm(d.t().contiguous(), x.double()), "dweight")):
        off, size = (got.double() - want).norm(dim=1), want.norm(dim=1)
        assert float(off.norm() / size.norm()) < whole, (what, float(off.norm() / size.norm()))
        bad = ~(off <= each * size + each * float(size.max()) * 2.0 ** -10)
        assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:5].flatten().tolist(), float((off / size)[bad].max()))


# binary32 keeps its 24 bits through the products: tiles of 64, 128 and 256, one split and many
@pytest.mark.parametrize("rows,vocab,cols", [(70, 500, 40), (250, 5000, 256), (500, 9000, 300), (300, 22_001, 500), (2048, 30_000, 512), (65, 20_000, 1000)])
def test_binary32_gradients_are_of_binary32(rows, vocab, cols):
    x, w = normal(1, rows, cols), normal(2, vocab, cols) * (2.0 / cols ** 0.5)
    t, g = borders(rows, vocab, 5), normal(4, rows).abs() + 0.1
    lse = pk.ops.linear_cross_entropy_forward(x, w, t)[1]
    d = xent64(x, w, t, g)[2]
    dx, dw = pk.ops.linear_cross_entropy_backward(g, x, w, t, lse)
    compare_gradients(dx, dw, d, x, w, F32)


def test_score_of_more_parts_than_a_turn_joins():
    """The join of a row's partial sums takes 512 at a time."""
    rows, vocab, cols = 90, 150_001, 64
    x, w, t = normal(1, rows, cols).to(BF16), (normal(2, vocab, cols) * 0.4).to(BF16), borders(rows, vocab, 3)
    w[torch.tensor([3, 70_000, 140_000, 150_000], device="cuda")] *= 4
    loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
    loss64, lse64, _, logits = xent64(x, w, t, torch.ones(rows, device="cuda"))
    off = 2 ** -20 * (1 + logits.abs().amax(1)) + 4 * 72 ** 0.5 * E * torch.mm(x.double().abs(), w.double().abs().t()).amax(1)
    within(lse, lse64, off, "lse")
    within(loss, loss64, 2 * off, "loss")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows", [40, 200])
def test_captured_steps_of_every_type(dtype, rows):
    """Replays with other inputs (in binary32 such as change which tiles the planes hold) between eager work, against the eager step."""
    x, w, t = normal(1, rows, 96).to(dtype), (normal(2, 1500, 96) * 0.2).to(dtype), torch.arange(rows, device="cuda") * 7 % 1500
    g = torch.full((rows,), 0.01, device="cuda")

    def step():
        loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
        return (loss, lse) + pk.ops.linear_cross_entropy_backward(g, x, w, t, lse)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(normal(10 + k, rows, 96))
        if dtype is F32 and k % 2:
            x[:, 3] *= 1e8
        w[:, 3] = 0
        g.copy_(torch.rand(rows, device="cuda") * 2.0 ** -k)
        graph.replay()
        got = [o.clone() for o in out]
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_the_same_bits_every_time_in_the_largest_tiles(dtype):
    rows, vocab, cols = 1500, 21_500, 1000
    x, w, t = normal(1, rows, cols).to(dtype), (normal(2, vocab, cols) * 0.05).to(dtype), borders(rows, vocab, 3)
    g = torch.rand(rows, device="cuda")
    runs = []
    for _ in range(4):
        loss, lse = pk.ops.linear_cross_entropy_forward(x, w, t)
        runs.append((loss, lse) + pk.ops.linear_cross_entropy_backward(g, x, w, t, lse))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
