"""Operators of a head that answers: from the residual stream to a word, and the training of its norm.

The head as it serves: what a layer adds to the residual stream -> root-mean-square norm of the sum, held in 8 bits with a
step per row -> logits over the vocabulary by a product of 8-bit integers -> a word drawn from them.  ``listed()`` names
the standing cases, ``draw(rng)`` gives further ones of the same ranges; ``prepare`` makes what a program holds before the
call, ``run`` is one pass (the plain form in elementary torch operations, or with ``own`` the framework's kernels),
``work`` the bytes and operations that no implementation can do without, ``exact`` the results in 64 bits.

Kinds of pass:
  rms        norm of x + residual, forward: the sum, its norm, 1 / root mean square
  rms_train  the same and its backward pass, with the sum of the weight's gradient
  rms8       norm of x + residual held in 8 bits, one step per row, and taken back
  linear8    logits of features: the features rounded to 8 bits with a step per row, times 8-bit weights with a step per word
  head8      rms8 and linear8 in a row, as a server calls them
  sample     a word per row of logits for given random numbers: temperature, top-k, top-p and min-p
"""
import math

import torch

own = False

EPS = 1e-6

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _case(name, kind, rows, width, dtype, vocab=0, rtype="", wtype="", pad=0, rule=""):
    """rows x width features of a type (a sample has no width, only rows x vocab logits); rtype, wtype: types of the residual
    stream and of the norm's weight (the features' own if not given); pad: elements between rows (a slice of a wider
    array); rule: what limits a sample's words, see _rules()."""
    c = {"kind": kind, "rows": rows, "width": width, "dtype": dtype, "vocab": vocab, "rtype": rtype or dtype, "wtype": wtype or dtype,
         "pad": pad, "rule": rule}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token's topic features (K = 1,000) in a server: nothing but latency.
        _case("rms_token", "rms", 1, 1000, "bf16"),
        # A training step of the norm on a batch of short texts, an odd number of topics cut out of a wider array.
        _case("rms_train_odd", "rms_train", 5003, 777, "f32", pad=23),
        # A large training batch: 16-bit features, residual stream and weight kept in 32 bits.
        _case("rms_train_large", "rms_train", 65_536, 2048, "bf16", rtype="f32", wtype="f32"),
        # A large batch's norm in 8 bits.
        _case("rms8_large", "rms8", 32_768, 4096, "f16"),
        # One token from the residual stream to its logits over the news-sized vocabulary.
        _case("head8_token", "head8", 1, 1024, "bf16", vocab=100_000),
        # A first experiment: a small batch and vocabulary in 32 bits.
        _case("linear8_small", "linear8", 250, 256, "f32", vocab=5000),
        # The tokens of a short document, newsgroup-sized vocabulary, odd sizes throughout.
        _case("linear8_text", "linear8", 61, 777, "f16", vocab=30_011, pad=5),
        # Logits of a held-out batch over the abstracts' vocabulary, on 1,000 topic features.
        _case("linear8_large", "linear8", 8192, 1000, "bf16", vocab=141_000),
        # The next word of one text, all limits at once.
        _case("sample_token", "sample", 1, 0, "f32", vocab=100_000, rule="all"),
        # A word for every place of a short document, rows that start at odd addresses.
        _case("sample_text", "sample", 61, 0, "f16", vocab=30_011, pad=5, rule="top_p"),
        # Requests of a server in one batch, each with a temperature and limits of its own.
        _case("sample_batch", "sample", 1024, 0, "bf16", vocab=100_000, rule="rows"),
        # Synthetic documents: a word for every token of a large batch, logits in 32 bits.
        _case("sample_large", "sample", 2048, 0, "f32", vocab=141_000, rule="top_p"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rms", "rms_train", "rms_train", "rms8", "head8", "linear8", "linear8", "sample", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 8, 5])
    if kind == "sample":
        vocab = _log_uniform(rng, 1000, 141_000)
        rows = min(_log_uniform(rng, 1, 4096), 2048 * 141_000 // vocab)
        return _case("", kind, rows, 0, dtype, vocab=vocab, pad=pad, rule=rng.choice(["none", "top_k", "top_p", "min_p", "all", "rows"]))
    if kind in ("head8", "linear8"):
        vocab = _log_uniform(rng, 1000, 141_000)
        width = _log_uniform(rng, 64, 4096)
        most = min(1e12 / (vocab * width), (5e8 if dtype == "f32" else 1e9) / vocab)
        rows = min(_log_uniform(rng, 1, 8192), max(1, int(most)))
        if rng.random() < 0.5:
            width = -(-width // 8) * 8
        return _case("", kind, rows, width, dtype, vocab=vocab, pad=pad)
    width = _log_uniform(rng, 48, 8192)
    if rng.random() < 0.5:
        width = -(-width // 8) * 8
    rows = min(_log_uniform(rng, 1, 65_536), 120_000_000 // width)
    return _case("", kind, rows, width, dtype, rtype=rng.choice([dtype, "f32"]), wtype=rng.choice([dtype, "f32"]), pad=pad)


def _slice(n, h, pad, t):
    wide = torch.ones((n, h + pad), device="cuda", dtype=t)
    return wide[:, :h]


def _step(most):
    """The step of a row whose largest magnitude is `most`, held in 32 bits."""
    return most / torch.full_like(most, 127.0)


def _in_steps(x, step):
    """Whole numbers of steps, ties to even; divided in 64 bits, as in 32 a quotient next to a half may become that half."""
    return torch.where(step > 0, torch.round(x.double() / step.double()), 0.0).clamp_(-127, 127).float()


def _rules(c, g):
    """Temperature, top_k, top_p and min_p: numbers for the whole batch, or a value per row."""
    off = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}
    rule, n = c["rule"], c["rows"]
    if rule == "none":
        return dict(off, temperature=0.9)
    if rule == "top_k":
        return dict(off, temperature=0.7, top_k=50)
    if rule == "top_p":
        return dict(off, top_p=0.95)
    if rule == "min_p":
        return dict(off, temperature=1.3, min_p=0.05)
    if rule == "all":
        return {"temperature": 0.8, "top_k": 400, "top_p": 0.9, "min_p": 0.01}

    def some(share, value, otherwise):
        chosen = torch.rand(n, device="cuda", generator=g) < share
        return torch.where(chosen, value, torch.full_like(value, otherwise))

    u = lambda: torch.rand(n, device="cuda", generator=g)  # noqa: E731
    temperature = some(0.9, 0.5 + u(), 0.0)   # every tenth row takes its likeliest word
    top_k = some(0.4, torch.exp(u() * math.log(1000.0)).floor(), 0.0).to(torch.int32)
    return {"temperature": temperature, "top_k": top_k, "top_p": some(0.5, 0.5 + 0.499 * u(), 1.0), "min_p": some(0.3, 0.2 * u(), 0.0)}


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, h, v, t = c["rows"], c["width"], c["vocab"], TYPES[c["dtype"]]
    s = {"case": c}
    randn = lambda *size: torch.randn(size, device="cuda", generator=g)  # noqa: E731
    if c["kind"] == "sample":
        # words by rank as in a text (frequency about 1/rank, in another order), sharpened by a context; some words are masked
        rank = torch.argsort(torch.rand(v, device="cuda", generator=g)).float()
        s["logits"] = _slice(n, v, c["pad"], t)
        s["logits"].copy_(4.0 - torch.log1p(rank) + 1.7 * randn(n, v))
        s["logits"].masked_fill_((torch.rand(v, device="cuda", generator=g) < 0.02), -math.inf)
        if c["rule"] == "rows" and n > 1:
            s["logits"][n // 2] = -math.inf   # a row whose mask leaves nothing
        s["u"] = torch.rand(n, device="cuda", generator=g)
        s.update(_rules(c, g))
        return s
    if c["kind"] == "linear8":
        s["x"] = _slice(n, h, c["pad"], t)
        s["x"].copy_(randn(n, h) * torch.exp(0.3 * randn(h)))
    else:
        # the stream: columns with a scale of their own, rows that have grown to different lengths; x: what a layer adds to it
        r = TYPES[c["rtype"]]
        s["residual"] = (randn(n, h) * torch.exp(0.5 * randn(h)) * torch.exp(0.3 * randn(n, 1))).to(r)
        s["x"] = _slice(n, h, c["pad"], t)
        s["x"].copy_(0.5 * randn(n, h))
        s["weight"] = (1 + 0.2 * randn(h)).to(TYPES[c["wtype"]])
        if c["kind"] == "rms_train":
            s["dy"] = (randn(n, h) / 8).to(t)
            s["dsum"] = (randn(n, h) / 8).to(r)
    if v:   # a model's output weights, rounded to 8 bits once
        words = randn(v, h) * (1.5 / math.sqrt(h))
        s["words_step"] = _step(words.abs().amax(1))
        s["words"] = _in_steps(words, s["words_step"][:, None]).to(torch.int8)
        if own:
            from paper_1610_02496_amd import ops
            s["words8"] = ops.Rows8.of(s["words"], s["words_step"])
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _plain_sum(x, residual):
    """The stream as it is held, which is what the norm is of."""
    return (x.float() + residual.float()).to(residual.dtype)


def _plain_rms(total, weight, dtype):
    f = total.float()
    rstd = torch.rsqrt((f * f).mean(1, keepdim=True) + EPS)
    return (f * rstd * weight.float()).to(dtype), rstd


def _plain_rms_backward(dy, dsum, total, rstd, weight, dtype):
    g = dy.float()
    hat = total.float() * rstd
    gw = g * weight.float()
    d = rstd * (gw - hat * (gw * hat).mean(1, keepdim=True)) + dsum.float()
    return d.to(dtype), d.to(total.dtype), (g * hat).sum(0).to(weight.dtype)


def _plain_rows8(x):
    step = _step(x.abs().amax(1, keepdim=True))
    return _in_steps(x, step), step


def _plain_rms8(total, weight):
    """Steps of total * weight (in 32 bits), which 1 / root mean square only scales."""
    f = total.float()
    rstd = torch.rsqrt((f * f).mean(1, keepdim=True) + EPS)
    q, step = _plain_rows8(f * weight.float())
    return q, step * rstd


def _plain_linear8(q, step, words, words_step, dtype):
    return (q @ words.float().t() * step * words_step).to(dtype)


def _per_row(value, n, t):
    """A number or a value per row, as a column in 64 bits of what it is in type t."""
    return torch.as_tensor(value, device="cuda").to(t).to(torch.float64).expand(n)[:, None]


def _plain_sample(logits, u, temperature, top_k, top_p, min_p):
    n, v = logits.shape
    temperature, top_p, min_p = (_per_row(a, n, torch.float32) for a in (temperature, top_p, min_p))
    top_k = _per_row(top_k, n, torch.int64)
    down, order = torch.sort(logits.float(), dim=1, descending=True, stable=True)   # equal ones by their index
    top = down[:, :1].double()
    greedy = temperature <= 0
    z = (down.double() - top) / torch.where(greedy, torch.ones_like(temperature), temperature)
    e = z.exp()
    place = torch.arange(v, device=logits.device)
    e *= torch.where(greedy, place == 0, (top_k <= 0) | (place < top_k))
    mass = e.cumsum(1)
    # up to the first word at which the words before it and it hold the share
    e *= (mass - e < top_p * mass[:, -1:]) | (top_p >= 1) | (place == 0)
    e *= z >= min_p.log()
    by_word = torch.zeros_like(e).scatter_(1, order, e)
    mass = by_word.cumsum(1)
    total = mass[:, -1:].contiguous()
    word = torch.searchsorted(mass, u.double()[:, None] * total, right=True).clamp_(max=v - 1)
    p = by_word.gather(1, word) / total
    some = top > -math.inf
    return torch.where(some, word, torch.full_like(word, -1))[:, 0], torch.where(some, p, torch.zeros_like(p))[:, 0].float()


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "sample":
        word, p = _plain_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return {"word": word, "p": p}
    x = s["x"]
    if kind == "linear8":
        q, step = _plain_rows8(x.float())
        return {"logits": _plain_linear8(q, step, s["words"], s["words_step"], x.dtype)}
    total = _plain_sum(x, s["residual"])
    out = {"sum": total}
    if kind in ("rms8", "head8"):
        q, step = _plain_rms8(total, s["weight"])
        if kind == "rms8":
            out["y"] = (q * step).to(x.dtype)
        else:
            out["logits"] = _plain_linear8(q, step, s["words"], s["words_step"], x.dtype)
        return out
    out["y"], rstd = _plain_rms(total, s["weight"], x.dtype)
    out["rstd"] = rstd.squeeze(1)
    if kind == "rms_train":
        out["dx"], out["dresidual"], out["dweight"] = _plain_rms_backward(s["dy"], s["dsum"], total, rstd, s["weight"], x.dtype)
    return out


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _run_own(s):
    from paper_1610_02496_amd import ops
    c = s["case"]
    kind = c["kind"]
    if kind == "sample":
        word, p = ops.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"word": word, "p": p}
    if kind == "linear8":
        return {"logits": ops.linear8(s["x"], s["words8"])}
    if kind in ("rms8", "head8"):
        y, total = ops.rms_norm8(s["x"], s["weight"], s["residual"], EPS)
        if kind == "rms8":
            return {"sum": total, "y": y.restore()}
        return {"sum": total, "logits": ops.linear8(y, s["words8"])}
    y, saved = ops.rms_norm_forward(s["x"], s["weight"], s["residual"], EPS)
    out = {"sum": saved.x, "y": y, "rstd": saved.rstd}
    if kind == "rms_train":
        out["dx"], out["dresidual"], out["dweight"] = ops.rms_norm_backward(s["dy"], saved, s["dsum"])
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once, each output written once, and what the backward pass or the next operator takes read once more;
    operations of the definition."""
    c = case
    n, h, v, e, r, w = c["rows"], c["width"], c["vocab"], SIZE[c["dtype"]], SIZE[c["rtype"]], SIZE[c["wtype"]]
    kind = c["kind"]
    if kind == "sample":
        return {"bytes": n * v * e + 16 * n, "flops": 5 * n * v}
    if kind == "linear8":
        return {"bytes": n * h * e + v * (h + 4) + n * v * e, "flops": 2 * n * v * h}
    norm = n * h * (e + 2 * r) + h * w   # x and residual read, their sum written
    if kind == "rms":
        return {"bytes": norm + n * (h * e + 4), "flops": 6 * n * h}
    if kind == "rms8":
        return {"bytes": norm + n * (2 * h + h * e + 8), "flops": 9 * n * h}
    if kind == "head8":
        return {"bytes": norm + n * (2 * h + 8) + v * (h + 4) + n * v * e, "flops": 2 * n * v * h}
    # y written; dy, dsum and the sum read, the gradients of residual and (of another type) x written
    back = n * h * (e + 3 * r + (e if c["rtype"] != c["dtype"] else 0)) + 2 * h * w
    return {"bytes": norm + n * (h * e + 8) + back, "flops": 16 * n * h}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------

def _exact_steps(a):
    """(whole numbers, step) of every row: the step is a 127th of the largest magnitude in 32 bits, ties go to even."""
    step = (a.abs().max(1).values / 127).float().double()[:, None]
    return torch.where(step > 0, a / step, 0.0).round().clamp(min=-127.0, max=127.0), step


def _exact_norm(s, lo, hi):
    """The rows lo .. hi-1 of every output of a norm."""
    c = s["case"]
    kind, h = c["kind"], c["width"]
    x, res, w = s["x"][lo:hi].double(), s["residual"][lo:hi].double(), s["weight"].double()
    held = (x + res).to(s["residual"].dtype)
    a = held.double()
    sigma = torch.sqrt(torch.einsum("nh,nh->n", a, a) / h + EPS)[:, None]
    part = {"sum": held}
    if kind in ("rms8", "head8"):
        q, step = _exact_steps((a * w).float().double())
        part["y"] = q * step / sigma
        return part
    z = a / sigma
    part["y"], part["rstd"] = z * w, 1 / sigma[:, 0]
    if kind == "rms_train":
        dy = s["dy"][lo:hi].double()
        dz = dy * w
        d = (dz - z * ((dz * z).sum(1) / h)[:, None]) / sigma + s["dsum"][lo:hi].double()
        part["dx"], part["dresidual"], part["dweight"] = d, d, (dy * z).sum(0)
    return part


def _exact_words(logits, u, temperature, top_k, top_p, min_p):
    """Words of some rows by their border: all logits above it take part, and of those equal to it the first few."""
    n, v = logits.shape
    l = logits.double()
    best, first = l.max(1)
    empty = best == -math.inf
    t = torch.where(temperature > 0, temperature, 1.0)
    z = torch.where(empty[:, None], 0.0, (l - best[:, None]) / t[:, None])
    by_size = z.sort(1, descending=True).values
    k = torch.where(top_k > 0, top_k.clamp(max=v), v)
    w = by_size.exp()
    w[torch.arange(v, device=w.device)[None] >= k[:, None]] = 0
    sums = torch.cumsum(w, 1)
    goal = (top_p * sums[:, -1])[:, None]
    count = torch.where(top_p < 1, 1 + (sums < goal).sum(1).clamp(max=v - 1), v)
    count = torch.minimum(torch.minimum(count, k), (by_size >= torch.log(min_p)[:, None]).sum(1)).clamp(min=1)
    border = by_size.gather(1, count[:, None] - 1)
    above, equal = z > border, z == border
    keep = above | (equal & (equal.cumsum(1) <= (count - above.sum(1))[:, None]))
    part = torch.where(keep, z.exp(), 0.0)
    sums = torch.cumsum(part, 1)
    word = (sums <= (u.double() * sums[:, -1])[:, None]).sum(1).clamp(max=v - 1)
    word = torch.where(temperature > 0, word, first)
    p = torch.where(temperature > 0, part.gather(1, word[:, None])[:, 0] / sums[:, -1], 1.0)
    return torch.where(empty, -1, word), torch.where(empty, 0.0, p)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    n, h, v, kind = c["rows"], c["width"], c["vocab"], c["kind"]
    if kind == "sample":
        row = lambda a, t: torch.as_tensor(a, device="cuda").to(t).expand(n)  # noqa: E731
        limits = [row(s["temperature"], torch.float32).double(), row(s["top_k"], torch.int64), row(s["top_p"], torch.float32).double(),
                  row(s["min_p"], torch.float32).double()]
        some = max(1, 30_000_000 // v)
        parts = [_exact_words(s["logits"][i:i + some], s["u"][i:i + some], *(a[i:i + some] for a in limits)) for i in range(0, n, some)]
        return {"word": torch.cat([a for a, _ in parts]), "p": torch.cat([b for _, b in parts])}
    words = s["words"].double() * s["words_step"].double()[:, None] if v else None
    some = max(1, min(50_000_000 // h, 200_000_000 // v if v else n))
    parts = []
    for lo in range(0, n, some):
        hi = min(n, lo + some)
        if kind == "linear8":
            q, step = _exact_steps(s["x"][lo:hi].double())
            parts.append({"logits": torch.mm(q * step, words.t())})
            continue
        part = _exact_norm(s, lo, hi)
        if kind == "head8":
            part["logits"] = torch.mm(part.pop("y"), words.t())
        parts.append(part)
    return {k: sum(p[k] for p in parts) if k == "dweight" else torch.cat([p[k] for p in parts]) for k in parts[0]}
