"""The operators of a head that is trained on a topic model's features, as calls of their public entry points.

The head: features of every token -> layer norm -> logits over the vocabulary -> softmax cross entropy with the token's
word.  ``listed()`` names the standing cases, ``draw(rng)`` gives further ones of the same ranges; ``prepare`` makes what a
program holds before the call, ``run`` is one pass (the plain form in elementary torch operations, or with ``own`` the
framework's kernels), ``work`` the bytes and operations that no implementation can do without, ``exact`` the results in
64 bits.

Kinds of pass:
  norm        layer norm, forward
  norm_train  layer norm, forward and backward, with the sums of the weight's and bias's gradients
  norm8_train the same with the input held as an 8-bit checkpoint between the two
  checkpoint  an activation saved in 8 bits and restored
  score       log-likelihood of given words: projection onto the vocabulary and softmax cross entropy, forward
  head_train  the same with the gradients of features and projection
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128   # columns that share one scale of a checkpoint

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _case(name, kind, rows, width, dtype, vocab=0, wtype="", pad=0):
    """rows x width features of a type; vocab: words of the projection; wtype: type of a norm's weight and bias (the
    features' own if not given); pad: elements between the rows of the features (a slice of a wider array)."""
    c = {"kind": kind, "rows": rows, "width": width, "dtype": dtype, "vocab": vocab, "wtype": wtype or dtype, "pad": pad}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token's topic features (K = 1,000) in a server: nothing but latency.
        _case("norm_token", "norm", 1, 1000, "bf16"),
        # A training step of the norm on a batch of short texts whose features are an odd number of topics, cut out of a
        # wider array.
        _case("norm_train_odd", "norm_train", 5003, 777, "f32", pad=23),
        # A large training batch of wide features, weights kept in 32 bits.
        _case("norm_train_large", "norm_train", 65_536, 2048, "f16", wtype="f32"),
        # The same step with the norm's input held in 8 bits, at the head's ordinary batch and width ...
        _case("norm8_train", "norm8_train", 16_384, 1024, "bf16"),
        # ... and on an odd number of topics in 32 bits.
        _case("norm8_train_odd", "norm8_train", 2261, 777, "f32"),
        # Activations of a large batch put away and taken back.
        _case("checkpoint_large", "checkpoint", 32_768, 4096, "bf16"),
        # One token scored over the news-sized vocabulary.
        _case("score_token", "score", 1, 1024, "bf16", vocab=100_000),
        # The tokens of a short document, newsgroup-sized vocabulary, odd sizes throughout.
        _case("score_text", "score", 61, 777, "f16", vocab=30_011),
        # Log-likelihood of a held-out batch over the abstracts' vocabulary, on 1,000 topic features.
        _case("score_large", "score", 8192, 1000, "bf16", vocab=141_000),
        # A first experiment: a small batch and vocabulary.
        _case("head_train_small", "head_train", 250, 256, "f32", vocab=5000),
        # A training step of the head over the news-sized vocabulary.
        _case("head_train", "head_train", 4096, 1024, "bf16", vocab=100_000),
        # The same in 32 bits on a streamed corpus' vocabulary.
        _case("head_train_f32", "head_train", 2048, 512, "f32", vocab=60_000),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm8_train", "checkpoint", "score", "score", "head_train", "head_train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("score", "head_train"):
        vocab = _log_uniform(rng, 1000, 141_000)
        width = _log_uniform(rng, 64, 2048)
        most = (2e11 if dtype == "f32" else 4e11) / (vocab * width)
        rows = min(_log_uniform(rng, 1, 8192), max(1, int(most)))
        if rng.random() < 0.5:
            width = -(-width // 8) * 8
        return _case("", kind, rows, width, dtype, vocab=vocab, pad=rng.choice([0, 0, 8, 5]))
    width = _log_uniform(rng, 48, 8192)
    if rng.random() < 0.5:
        width = -(-width // 8) * 8
    rows = min(_log_uniform(rng, 1, 65_536), 134_000_000 // width)
    wtype = rng.choice([dtype, "f32"])
    return _case("", kind, rows, width, dtype, wtype=wtype, pad=rng.choice([0, 0, 8, 5]))


def _features(c, g):
    """Activations as they come out of a sum of embeddings: every column with an offset and a scale of its own, some of
    them large."""
    n, h = c["rows"], c["width"]
    wide = torch.empty((n, h + c["pad"]), device="cuda", dtype=TYPES[c["dtype"]])
    scale = torch.exp(0.5 * torch.randn(h, device="cuda", generator=g))
    shift = 0.3 * torch.randn(h, device="cuda", generator=g)
    wide[:, :h] = torch.randn((n, h), device="cuda", generator=g) * scale + shift
    wide[:, h:] = 1.0
    return wide[:, :h]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, h, t = c["rows"], c["width"], TYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] in ("norm", "norm_train", "norm8_train"):
        w = TYPES[c["wtype"]]
        s["x"] = _features(c, g)
        s["weight"] = (1 + 0.2 * torch.randn(h, device="cuda", generator=g)).to(w)
        s["bias"] = (0.1 * torch.randn(h, device="cuda", generator=g)).to(w)
        if c["kind"] != "norm":
            s["dy"] = (torch.randn((n, h), device="cuda", generator=g) / 8).to(t)
    elif c["kind"] == "checkpoint":
        s["x"] = _features(c, g)
    else:
        v = c["vocab"]
        wide = torch.randn((n, h + c["pad"]), device="cuda", generator=g).to(t)   # what a norm gives
        s["x"] = wide[:, :h]
        s["weight"] = (torch.randn((v, h), device="cuda", generator=g) * (1.5 / math.sqrt(h))).to(t)
        # words by rank as in a text (frequency about 1/rank), a few places without a target (padding of a batch)
        u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
        word = (torch.exp(u * math.log(v + 1.0)) - 1).long().clamp_(0, v - 1)
        s["target"] = torch.where(torch.rand(n, device="cuda", generator=g) < 0.03, torch.full_like(word, -1), word)
        s["target"][0] = word[0]
        if c["kind"] == "head_train":   # gradient of the mean; in 16-bit floats with a loss scale, as such steps are run
            count = (s["target"] >= 0).sum()
            s["dloss"] = (torch.full((n,), 65536.0 if c["dtype"] == "f16" else 1.0, device="cuda") / count).float()
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _plain_norm(x, weight, bias):
    xf = x.float()
    mean = xf.mean(1, keepdim=True)
    xc = xf - mean
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    y = xc * rstd * weight.float() + bias.float()
    return y.to(x.dtype), mean, rstd


def _plain_norm_backward(dy, xf, mean, rstd, weight, dtype):
    g = dy.float()
    hat = (xf - mean) * rstd
    gw = g * weight.float()
    dx = rstd * (gw - gw.mean(1, keepdim=True) - hat * (gw * hat).mean(1, keepdim=True))
    return dx.to(dtype), (g * hat).sum(0).to(weight.dtype), g.sum(0).to(weight.dtype)


def _plain_save(x):
    n, h = x.shape
    full = -(-h // BLOCK) * BLOCK
    blocks = torch.zeros((n, full), device=x.device, dtype=torch.float32)
    blocks[:, :h] = x
    blocks = blocks.view(n, full // BLOCK, BLOCK)
    most = blocks.abs().amax(2, keepdim=True)
    scale = most / torch.full_like(most, 127.0)
    q = torch.where(scale > 0, torch.round(blocks / scale), torch.zeros_like(blocks)).clamp_(-127, 127)
    return q.to(torch.int8), scale


def _plain_restore(q, scale, h):
    return (q.float() * scale).view(q.shape[0], -1)[:, :h]


def _plain_score(x, weight, target):
    logits = x.float() @ weight.float().t()
    top = logits.amax(1, keepdim=True)
    lse = (top + (logits - top).exp().sum(1, keepdim=True).log()).squeeze(1)
    at = logits.gather(1, target.clamp(min=0)[:, None]).squeeze(1)
    return torch.where(target >= 0, lse - at, torch.zeros_like(lse)), lse, logits


def _plain_score_backward(dloss, x, weight, target, lse, logits):
    d = (logits - lse[:, None]).exp()
    d.scatter_add_(1, target.clamp(min=0)[:, None], torch.full_like(lse, -1.0)[:, None])
    d *= torch.where(target >= 0, dloss, torch.zeros_like(dloss))[:, None]
    return (d @ weight.float()).to(x.dtype), (d.t() @ x.float()).to(weight.dtype)


def _run_plain(s):
    c, x = s["case"], s["x"]
    kind = c["kind"]
    if kind in ("norm", "norm_train", "norm8_train"):
        y, mean, rstd = _plain_norm(x, s["weight"], s["bias"])
        out = {"y": y, "mean": mean.squeeze(1), "rstd": rstd.squeeze(1)}
        if kind != "norm":
            xf = _plain_restore(*_plain_save(x), c["width"]) if kind == "norm8_train" else x.float()
            out["dx"], out["dweight"], out["dbias"] = _plain_norm_backward(s["dy"], xf, mean, rstd, s["weight"], x.dtype)
        return out
    if kind == "checkpoint":
        return {"x": _plain_restore(*_plain_save(x), c["width"]).to(x.dtype)}
    loss, lse, logits = _plain_score(x, s["weight"], s["target"])
    out = {"loss": loss, "lse": lse}
    if kind == "head_train":
        out["dx"], out["dweight"] = _plain_score_backward(s["dloss"], x, s["weight"], s["target"], lse, logits)
    return out


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _run_own(s):
    from paper_1610_02496_amd import ops
    c, x = s["case"], s["x"]
    kind = c["kind"]
    if kind in ("norm", "norm_train", "norm8_train"):
        y, saved = ops.layer_norm_forward(x, s["weight"], s["bias"], EPS, checkpoint=kind == "norm8_train")
        out = {"y": y, "mean": saved.mean, "rstd": saved.rstd}
        if kind != "norm":
            out["dx"], out["dweight"], out["dbias"] = ops.layer_norm_backward(s["dy"], saved)
        return out
    if kind == "checkpoint":
        return {"x": ops.checkpoint8(x).restore()}
    loss, lse = ops.linear_cross_entropy_forward(x, s["weight"], s["target"])
    out = {"loss": loss, "lse": lse}
    if kind == "head_train":
        out["dx"], out["dweight"] = ops.linear_cross_entropy_backward(s["dloss"], x, s["weight"], s["target"], lse)
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once, each output written once; of a product's operations those of the definition (three products
    for a training step of the head)."""
    c = case
    n, h, v, e = c["rows"], c["width"], c["vocab"], SIZE[c["dtype"]]
    w = SIZE[c["wtype"]]
    kind = c["kind"]
    if kind == "norm":
        return {"bytes": 2 * n * h * e + 8 * n + 2 * h * w, "flops": 8 * n * h}
    if kind == "norm_train":
        return {"bytes": 5 * n * h * e + 16 * n + 5 * h * w, "flops": 20 * n * h}
    if kind == "norm8_train":
        scales = 4 * n * (-(-h // BLOCK))
        return {"bytes": 4 * n * h * e + 2 * (n * h + scales) + 16 * n + 5 * h * w, "flops": 24 * n * h}
    if kind == "checkpoint":
        return {"bytes": 2 * n * h * e + 2 * n * h + 8 * n * (-(-h // BLOCK)), "flops": 5 * n * h}
    if kind == "score":
        return {"bytes": (n + v) * h * e + 16 * n, "flops": 2 * n * v * h}
    return {"bytes": 2 * (n + v) * h * e + 20 * n, "flops": 6 * n * v * h}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------

def _exact_rows(s, lo, hi):
    """Layer norm (and its backward pass) of the rows lo .. hi-1, from the definition in 64 bits."""
    c = s["case"]
    h, kind = c["width"], c["kind"]
    x, w, b = s["x"][lo:hi].double(), s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    sigma = torch.sqrt(var + EPS)
    part = {"y": (x - mean[:, None]) / sigma[:, None] * w + b, "mean": mean, "rstd": 1 / sigma}
    if kind == "norm":
        return part
    held = _exact_checkpoint(x, h) if kind == "norm8_train" else x
    z = (held - mean[:, None]) / sigma[:, None]
    dy = s["dy"][lo:hi].double()
    dz = dy * w
    part["dx"] = (dz - (dz.sum(1) / h)[:, None] - z * ((dz * z).sum(1) / h)[:, None]) / sigma[:, None]
    part["dweight"], part["dbias"] = (dy * z).sum(0), dy.sum(0)
    return part


def _exact_checkpoint(x, h):
    """Values that a checkpoint of x stands for: per block of columns a step of a 127th of the largest magnitude, held in
    32 bits; whole numbers of steps, ties to even."""
    out = torch.empty_like(x)
    for a in range(0, h, BLOCK):
        piece = x[:, a:a + BLOCK]
        step = (piece.abs().max(1).values / 127).float().double()[:, None]
        steps = torch.where(step > 0, piece / step, 0.0).round()
        out[:, a:a + BLOCK] = torch.maximum(torch.minimum(steps, torch.full_like(steps, 127.0)), torch.full_like(steps, -127.0)) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    n, kind = c["rows"], c["kind"]
    if kind in ("norm", "norm_train", "norm8_train", "checkpoint"):
        rows = max(1, 50_000_000 // c["width"])
        parts = []
        for lo in range(0, n, rows):
            hi = min(n, lo + rows)
            parts.append({"x": _exact_checkpoint(s["x"][lo:hi].double(), c["width"])} if kind == "checkpoint" else _exact_rows(s, lo, hi))
        return {k: sum(p[k] for p in parts) if k in ("dweight", "dbias") else torch.cat([p[k] for p in parts]) for k in parts[0]}
    w = s["weight"].double()
    rows = max(1, min(n, 100_000_000 // c["vocab"]))
    out = {"loss": [], "lse": []}
    if kind == "head_train":
        out["dx"], dweight = [], torch.zeros_like(w)
    for lo in range(0, n, rows):
        hi = min(n, lo + rows)
        x, t = s["x"][lo:hi].double(), s["target"][lo:hi]
        logits = torch.mm(x, w.t())
        lse = torch.logsumexp(logits, 1)
        i = torch.arange(hi - lo, device=x.device)
        has = t >= 0
        at = logits[i, t.clamp(min=0)]
        out["lse"].append(lse)
        out["loss"].append(torch.where(has, lse - at, 0.0))
        if kind == "head_train":
            p = torch.softmax(logits, 1)
            p[i, t.clamp(min=0)] -= 1
            p *= (s["dloss"][lo:hi].double() * has)[:, None]
            out["dx"].append(torch.mm(p, w))
            dweight += torch.mm(p.t(), x)
    out = {k: torch.cat(v) for k, v in out.items()}
    if kind == "head_train":
        out["dweight"] = dweight
    return out
