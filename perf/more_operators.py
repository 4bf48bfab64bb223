"""Workloads for timing the operators that train a token encoder from its tokens: table, layers and loss.

The search engine scores tokens that an encoder made. Training that encoder on a collection starts at a table of
tokens, goes through linear layers, and ends at a softmax over the same table (tokens that were masked are
predicted). A case is a dict of plain values; ``kind`` names the operator:

* ``embed``: ``tokens`` rows of a table [``vocabulary``, ``cols``], scaled; with ``train`` the table's gradient too.
  ``padding`` is the share of tokens that are padding (id -1)
* ``loss``: softmax cross entropy of ``tokens`` hidden rows over the table; with ``train`` the gradients of rows and
  table too. ``kept`` is the share of rows that are predicted (the others' target is -100); ``weights``: every
  predicted row counts alike ("mean") or by a weight of its own ("tokens")
* ``linear``: ``rows`` by a weight [``n``, ``cols``]; with ``train`` also the input in 8 bits, which is what is kept of
  it, and the gradients of input, weight and bias, the weight's from the 8-bit rows

``run`` computes a case in its plain form where ``own`` is false and calls the library where it is true.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
IDS = {"int64": torch.int64, "int32": torch.int32}
IGNORED = -100  # the target of a row that is not predicted


def _embed(name, tokens, vocabulary, cols, dtype, ids, padding, train):
    return _named(name, {"kind": "embed", "tokens": tokens, "vocabulary": vocabulary, "cols": cols, "dtype": dtype,
                         "ids": ids, "padding": padding, "train": train})


def _loss(name, tokens, vocabulary, cols, dtype, kept, weights, train):
    return _named(name, {"kind": "loss", "tokens": tokens, "vocabulary": vocabulary, "cols": cols, "dtype": dtype,
                         "kept": kept, "weights": weights, "train": train})


def _linear(name, rows, cols, n, dtype, bias, train):
    return _named(name, {"kind": "linear", "rows": rows, "cols": cols, "n": n, "dtype": dtype, "bias": bias,
                         "train": train})


def _named(name, c):
    return {"name": name, **c} if name else c


def listed():
    return [
        # the 32 tokens of one query: a single launch's latency
        _embed("embed_query", 32, 32_128, 768, "bfloat16", "int64", 0.0, False),
        # a training step at an odd width in full precision
        _embed("embed_train_odd", 4099, 9973, 771, "float32", "int64", 0.1, True),
        # a training step over a batch of passages (1,024 of 128 tokens), the shorter ones padded
        _embed("embed_train_large", 131_072, 32_128, 1024, "bfloat16", "int64", 0.3, True),
        # a table of many languages, of which a small batch touches few rows
        _embed("embed_vocabulary", 8192, 250_001, 768, "float16", "int32", 0.0, True),
        # scoring a handful of tokens: the table's bytes
        _loss("loss_query", 5, 32_128, 768, "bfloat16", 1.0, "mean", False),
        # a ragged batch in full precision, every size odd
        _loss("loss_ragged", 1771, 9973, 771, "float32", 0.8, "tokens", True),
        # masked tokens: 15% of a batch's rows are predicted
        _loss("loss_masked", 16_384, 32_128, 1024, "bfloat16", 0.15, "mean", True),
        # every row of a batch is predicted
        _loss("loss_large", 16_384, 32_128, 1024, "bfloat16", 1.0, "mean", True),
        # one token through a square layer: the weight's bytes and the launches
        _linear("linear_token", 1, 1024, 1024, "bfloat16", True, False),
        # 77 queries of 23 tokens, ragged in every size
        _linear("linear_train_odd", 1771, 771, 1003, "float16", True, True),
        # the projection to the 128 columns that are searched, over a batch of passages
        _linear("linear_train_head", 65_536, 1024, 128, "bfloat16", False, True),
        # a large square layer
        _linear("linear_train_large", 32_768, 4096, 4096, "bfloat16", True, True),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm; above a thousand odd, as a batch of texts has no round number of tokens."""
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n if n <= 1000 else (n - 1) | 1


def _width(rng, lo, hi):
    """Odd widths, multiples of 16 and powers of two."""
    w, u = _log_int(rng, lo, hi), rng.random()
    return w | 1 if u < 0.4 else max(80, w // 80 * 80) if u < 0.7 else 1 << int(math.log2(w))


def draw(rng):
    kind = rng.choice(["embed", "loss", "linear"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    train = rng.random() < 0.7
    if kind == "embed":
        cols = _width(rng, 64, 4096)
        vocabulary = _log_int(rng, 100, min(262_144, 192_000_000 // cols))
        tokens = 1 if rng.random() < 0.1 else _log_int(rng, 1, min(131_072, 134_000_000 // cols))
        return _embed(None, tokens, vocabulary, cols, dtype, rng.choice(["int64", "int32"]),
                      rng.choice([0.0, round(rng.uniform(0, 0.6), 3)]), train)
    if kind == "loss":
        cols = _width(rng, 64, 4096)
        vocabulary = _log_int(rng, 100, 262_144)
        most = min(16_384, 16_384 * 32_128 // vocabulary, 16_384 * 32_128 * 1024 // (vocabulary * cols))
        tokens = 1 if rng.random() < 0.1 else _log_int(rng, 1, max(1, most))
        return _loss(None, tokens, vocabulary, cols, dtype, rng.choice([1.0, 0.15, round(rng.uniform(0.05, 1), 3)]),
                     rng.choice(["mean", "tokens"]), train)
    cols, n = _width(rng, 64, 4096), rng.choice([128, _width(rng, 64, 4096), _width(rng, 64, 4096)])
    rows = 1 if rng.random() < 0.1 else _log_int(rng, 1, min(65_536, 65_536 * 2048 // max(cols, n)))
    return _linear(None, rows, cols, n, dtype, rng.random() < 0.5, train)


# ---------------------------------------------------------------------------- inputs

def _kept(case):
    return min(case["tokens"], max(1, round(case["kept"] * case["tokens"])))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    t = TYPES[case["dtype"]]
    if case["kind"] == "linear":
        rows, cols, n = case["rows"], case["cols"], case["n"]
        # hidden states: channels of different spread, a few of them large, and an offset
        spread = torch.exp(0.5 * randn(cols)) * torch.where(rand(cols) < 0.01, 10.0, 1.0)
        return {"case": case, "x": (randn(rows, cols) * spread + 0.5 * randn(cols)).to(t),
                "w": (randn(n, cols) / math.sqrt(cols)).to(t), "b": (0.1 * randn(n)).to(t) if case["bias"] else None,
                "dy": (0.01 * randn(rows, n)).to(t) if case["train"] else None}
    tokens, vocabulary, cols = case["tokens"], case["vocabulary"], case["cols"]
    # tokens as texts have them: the frequency of the r-th falls like 1 / r; common ones anywhere in the table
    ranks = torch.exp(rand(tokens).double() * math.log(vocabulary + 1)).floor().clamp(1, vocabulary).long() - 1
    ids = torch.randperm(vocabulary, generator=gen, device="cuda")[ranks]
    table = (0.5 * randn(vocabulary, cols)).to(t)
    s = {"case": case, "table": table}
    if case["kind"] == "embed":
        ids = torch.where(rand(tokens) < case["padding"], -1, ids)
        s["ids"], s["scale"] = ids.to(IDS[case["ids"]]), math.sqrt(cols) / 8
        s["dy"] = (0.01 * randn(tokens, cols)).to(t) if case["train"] else None
        return s
    # some rows know their token, some do not
    sure = rand(tokens, 1) ** 2 * 10
    s["hidden"] = (randn(tokens, cols) + sure * table[ids].float() / (0.25 * math.sqrt(cols))).to(t)
    s["scale"] = 2 / math.sqrt(cols)
    left = torch.randperm(tokens, generator=gen, device="cuda")[_kept(case):]
    ids[left] = IGNORED
    s["targets"] = ids
    # the loss's gradient for each row; in float16 losses are scaled up
    dloss = torch.full((tokens,), (65536.0 if t == torch.float16 else 1.0) / _kept(case), device="cuda")
    s["dloss"] = dloss * (0.5 + rand(tokens)) if case["weights"] == "tokens" else dloss
    return s


# ---------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2501_17788_amd as warp

    case = s["case"]
    if case["kind"] == "embed":
        out = warp.embedding(s["ids"], s["table"], s["scale"])
        if not case["train"]:
            return out
        return out, warp.embedding_backward(s["dy"], s["ids"], case["vocabulary"], s["scale"])
    if case["kind"] == "loss":
        loss, lse = warp.cross_entropy(s["hidden"], s["table"], s["targets"], s["scale"])
        if not case["train"]:
            return loss
        return (loss, *warp.cross_entropy_backward(s["dloss"], s["hidden"], s["table"], s["targets"], loss, lse,
                                                   s["scale"]))
    y = warp.linear(s["x"], s["w"], s["b"])
    if not case["train"]:
        return y
    kept = warp.quantize_rows(s["x"])
    return (y, *warp.linear_backward(s["dy"], kept, s["w"]))


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "embed":
        t, there = s["table"].dtype, s["ids"] >= 0
        ids = s["ids"].long().clamp(min=0)
        out = torch.where(there[:, None], s["table"][ids].float() * s["scale"], 0.0).to(t)
        if not case["train"]:
            return out
        sums = torch.zeros(case["vocabulary"], case["cols"], device="cuda")
        sums.index_add_(0, ids, torch.where(there[:, None], s["dy"].float(), 0.0))
        return out, (sums * s["scale"]).to(t)
    if case["kind"] == "loss":
        return _loss_plain(s)
    x, w, t = s["x"].float(), s["w"].float(), s["x"].dtype
    y = x @ w.t()
    y = (y if s["b"] is None else y + s["b"].float()).to(t)
    if not case["train"]:
        return y
    q, scale = _to_int8(x)
    dy = s["dy"].float()
    return y, (dy @ w).to(t), (dy.t() @ (q * scale)).to(t), dy.sum(0).to(t)


def _loss_plain(s):
    h, table, t = s["hidden"].float(), s["table"].float(), s["table"].dtype
    there = s["targets"] >= 0
    targets = s["targets"].clamp(min=0)[:, None]
    logits = (h @ table.t()) * s["scale"]
    top = logits.amax(1, keepdim=True)
    of_target = logits.gather(1, targets)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    loss = torch.where(there, (top + torch.log(total) - of_target)[:, 0], 0.0)
    if not s["case"]["train"]:
        return loss
    g = torch.where(there, s["dloss"] * s["scale"], 0.0)[:, None]
    d = e * (g / total)
    # at the target p - 1, with no difference of close numbers: minus the sum of the others' shares
    others = (total - e.gather(1, targets)) / total
    small = e.scatter(1, targets, 0.0).sum(1, keepdim=True) / total
    d.scatter_(1, targets, -g * torch.where(others < 0.1, small, others))
    return loss, (d @ table).to(t), (d.t() @ torch.where(there[:, None], h, 0.0)).to(t)


def _to_int8(x):
    """Rows of whole numbers of at most 127, and the scale of each: x is about q * scale."""
    top = x.abs().amax(1, keepdim=True)
    inv = torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)
    return torch.round(x * inv), top * (1.0 / 127.0)


# ---------------------------------------------------------------------------- bounds and 64-bit values

def work(case):
    t = TYPES[case["dtype"]].itemsize
    if case["kind"] == "linear":
        rows, cols, n = case["rows"], case["cols"], case["n"]
        forward = (rows * cols + n * cols + rows * n + (n if case["bias"] else 0)) * t
        if not case["train"]:
            return {"bytes": forward, "flops": 2 * rows * cols * n}
        # the 8-bit rows with their scales, written and read; dy read, the three gradients written
        back = 2 * rows * (cols + 4) + (rows * n + rows * cols + n * cols + n) * t
        return {"bytes": forward + back, "flops": 6 * rows * cols * n}
    tokens, vocabulary, cols = case["tokens"], case["vocabulary"], case["cols"]
    if case["kind"] == "embed":
        there = round(tokens * (1 - case["padding"]))
        # distinct rows of the table that a batch reads, at frequencies of 1 / rank
        log = math.log(vocabulary + 1)
        at = [math.exp((i + 0.5) * log / 64) for i in range(64)]
        rows = min(there, sum((1 - (1 - min(1.0, 1 / (log * r))) ** there) * r * log / 64 for r in at))
        size = IDS[case["ids"]].itemsize
        forward = int(rows) * cols * t + tokens * cols * t + tokens * size
        back = there * cols * t + vocabulary * cols * t + tokens * size if case["train"] else 0
        return {"bytes": forward + back, "flops": (2 if case["train"] else 1) * there * cols}
    kept = _kept(case)
    both = (kept + vocabulary) * cols * t
    forward = both + tokens * 12
    if not case["train"]:
        return {"bytes": forward, "flops": 2 * kept * vocabulary * cols}
    return {"bytes": forward + (tokens + vocabulary) * cols * t + tokens * 4, "flops": 6 * kept * vocabulary * cols}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "embed":
        ids = s["ids"].long()
        there = torch.nonzero(ids >= 0)[:, 0]
        out = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
        out[there] = s["scale"] * s["table"].double()[ids[there]]
        if not case["train"]:
            return out
        grad = torch.zeros(case["vocabulary"], case["cols"], dtype=torch.float64, device="cuda")
        grad.index_put_((ids[there],), s["scale"] * s["dy"][there].double(), accumulate=True)
        return out, grad
    if case["kind"] == "loss":
        return _loss_exact(s)
    x, w = s["x"].double(), s["w"].double()
    y = x @ w.t() + (0 if s["b"] is None else s["b"].double())
    if not case["train"]:
        return y
    # the whole numbers are defined by 32-bit arithmetic: the factor 127 / max and its product are rounded
    top = x.abs().amax(1, keepdim=True)
    factor = (127.0 / top).float().double()
    q = torch.round((x * factor).float().double())
    dy = s["dy"].double()
    return y, dy @ w, dy.t() @ (q * (top / 127.0)), dy.sum(0)


def _loss_exact(s):
    """Row by row group over the predicted rows alone."""
    case = s["case"]
    rows = torch.nonzero(s["targets"] >= 0)[:, 0]
    table = s["table"].double()
    loss = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
    dh = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
    dt = torch.zeros_like(table)
    for part in rows.split(max(1, (1 << 28) // case["vocabulary"])):
        h, y = s["hidden"][part].double(), s["targets"][part]
        logits = s["scale"] * (h @ table.t())
        lse = torch.logsumexp(logits, 1)
        at = torch.arange(len(part), device="cuda")
        loss[part] = lse - logits[at, y]
        if not case["train"]:
            continue
        p = torch.exp(logits - lse[:, None])
        p[at, y] -= 1
        p *= s["scale"] * s["dloss"][part].double()[:, None]
        dh[part] = p @ table
        dt += p.t() @ h
    return (loss, dh, dt) if case["train"] else loss
