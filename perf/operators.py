"""Workloads for timing the operators of a token encoder's head: training and serving.

The search engine scores 128-wide token embeddings; an encoder's last layers make them. A case is a
dict of plain values; ``kind`` names the call:

* ``norm``: layer norm of ``rows`` token rows of ``cols`` columns; with ``train`` its backward too
* ``linear``: token rows to int8, then the int8 product with a weight of ``n`` output channels
* ``encode``: layer norm straight to int8 rows, then the product (the serving form of both)
* ``adamw``: one step over all tensors of an encoder of ``layers`` layers of ``width`` columns,
  moments in 32 or 8 ``bits``; ``packed``: the tensors lie back to back, at any alignment

``run`` computes a case in its plain form where ``own`` is false and calls the library where it is true.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 100
BLOCK = 256  # elements of a tensor that share a scale of 8-bit moments
PAD = 128    # int8 rows are padded with zeros to a multiple of this width
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _norm(name, rows, cols, dtype, train, params="float32"):
    return _named(name, {"kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "params": params,
                         "train": train})


def _linear(name, kind, rows, cols, n, dtype, out, bias):
    return _named(name, {"kind": kind, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "out": out,
                         "bias": bias})


def _adamw(name, layers, width, wide, tokens, dtype, grads, bits, packed):
    return _named(name, {"kind": "adamw", "layers": layers, "width": width, "wide": wide, "tokens": tokens,
                         "dtype": dtype, "grads": grads, "bits": bits, "packed": packed})


def _named(name, c):
    return {"name": name, **c} if name else c


def listed():
    return [
        # the 32 tokens of one query through a norm of a small encoder: a single launch's latency
        _norm("norm_query", 32, 768, "bfloat16", False),
        # a training step's norm at an odd width in full precision
        _norm("norm_train_odd", 4099, 771, "float32", True),
        # a training step over a batch of passages (1,024 of 128 tokens), half-precision parameters
        _norm("norm_train_large", 131_072, 1024, "bfloat16", True, "bfloat16"),
        # serving: a batch of passages, wide rows
        _norm("norm_wide", 8192, 4096, "float16", False),
        # one token through a square layer: the weight's bytes and the launches
        _linear("linear_token", "linear", 1, 1024, 1024, "bfloat16", "bfloat16", True),
        # 77 queries of 23 tokens, ragged in every size, full precision out
        _linear("linear_ragged", "linear", 1771, 771, 1003, "float16", "float32", True),
        # encoding a collection: many passages through a large square layer
        _linear("linear_large", "linear", 32_768, 4096, 4096, "bfloat16", "bfloat16", False),
        # one query's 32 tokens: last norm and the projection to 128 columns
        _linear("encode_query", "encode", 32, 768, 128, "bfloat16", "bfloat16", True),
        # a batch of passages through the same head
        _linear("encode_passages", "encode", 65_536, 1024, 128, "bfloat16", "bfloat16", True),
        # fine-tuning a small head: two layers, tensors back to back, 8-bit moments
        _adamw("adamw8_small", 2, 250, 1000, 1001, "float32", "float32", 8, True),
        # an encoder of 12 layers in full precision, 32-bit moments
        _adamw("adamw32_base", 12, 768, 2048, 32_128, "float32", "float32", 32, False),
        # an encoder of 24 layers in half precision, 8-bit moments
        _adamw("adamw8_large", 24, 1024, 2816, 32_128, "bfloat16", "bfloat16", 8, False),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm; above a thousand odd, as a batch of texts has no round number of tokens."""
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n if n <= 1000 else (n - 1) | 1


def _width(rng, lo, hi):
    """Odd widths, multiples of 16 and powers of two."""
    w, u = _log_int(rng, lo, hi), rng.random()
    return w | 1 if u < 0.45 else max(80, w // 80 * 80) if u < 0.75 else 1 << int(math.log2(w))


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "encode", "adamw", "adamw"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    if kind == "norm":
        cols = _width(rng, 64, 8192)
        rows = _log_int(rng, 1, min(131_072, 131_072 * 1024 // (cols * (2 if dtype == "float32" else 1))))
        return _norm(None, rows, cols, dtype, rng.random() < 0.6, rng.choice([dtype, "float32"]))
    if kind in ("linear", "encode"):
        cols = _width(rng, 64, 4096)
        n = _width(rng, 64, 4096) if kind == "linear" else rng.choice([128, 128, _width(rng, 64, 1024)])
        rows = 1 if rng.random() < 0.15 else _log_int(rng, 1, 32_768 if kind == "linear" else 65_536)
        out = rng.choice(["bfloat16", "float16", "float32"]) if kind == "linear" else rng.choice(["bfloat16", "float16"])
        if kind == "encode":  # the rows of the largest listed batch
            rows = min(rows, 65_536 * 1024 // cols)
        return _linear(None, kind, rows, cols, n, dtype, out, rng.random() < 0.5)
    dtype = rng.choice(["float32", "bfloat16"])
    width = _width(rng, 64, 1024)
    return _adamw(None, _log_int(rng, 1, 24), width, _width(rng, width, int(2.75 * width)),
                  _log_int(rng, 100, 32_128), dtype, rng.choice([dtype, "float32"]), rng.choice([32, 8]),
                  rng.random() < 0.4)


# ---------------------------------------------------------------------------- inputs

def _tensor_sizes(case):
    """Element counts of an encoder's tensors: a token table, then per layer four square matrices, two
    between width and the wide middle, their biases and two norms; at the end the 128-column projection."""
    w, f = case["width"], case["wide"]
    layer = [w * w, w] * 4 + [w * f, f, w * f, w] + [w] * 4
    return [case["tokens"] * w] + layer * case["layers"] + [w, w, 128 * w]


def _ceil(n, m):
    return -(-n // m) * m


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["kind"] == "adamw":
        return _prepare_adamw(case, randn, rand)
    rows, cols, t = case["rows"], case["cols"], TYPES[case["dtype"]]
    # hidden states: channels of different spread, a few of them large, and an offset
    spread = torch.exp(0.5 * randn(cols)) * torch.where(rand(cols) < 0.01, 10.0, 1.0)
    s = {"case": case, "x": (randn(rows, cols) * spread + 0.5 * randn(cols)).to(t)}
    if case["kind"] != "linear":
        p = TYPES[case.get("params", "float32")]
        s["weight"] = (1 + 0.1 * randn(cols)).to(p)
        s["bias"] = (0.1 * randn(cols)).to(p)
    if case["kind"] == "norm":
        s["dy"] = (0.01 * randn(rows, cols)).to(t) if case["train"] else None
        return s
    # the quantised weight that a serving program keeps: int8 rows, padded, a scale for each channel
    n = case["n"]
    w = randn(n, cols) / math.sqrt(cols)
    top = w.abs().amax(1)
    wq = torch.zeros(n, _ceil(cols, PAD), dtype=torch.int8, device="cuda")
    wq[:, :cols] = torch.round(w * (127.0 / top)[:, None]).to(torch.int8)
    s["w"], s["w_scale"] = wq, top / 127.0
    s["b"] = 0.1 * randn(n) if case["bias"] else None
    return s


def _prepare_adamw(case, randn, rand):
    sizes = _tensor_sizes(case)
    starts, total = [], 0  # of each tensor's moments: at multiples of BLOCK
    for n in sizes:
        starts.append(total)
        total += _ceil(n, BLOCK)
    places = starts
    if case["packed"]:  # of each tensor's values and gradients
        places = [sum(sizes[:i]) for i in range(len(sizes))]
    length = places[-1] + sizes[-1] if case["packed"] else total
    scale = torch.zeros(total, device="cuda")  # spread of each element's gradients; 0 between the tensors
    where = torch.empty(sum(sizes), dtype=torch.int64, device="cuda") if case["packed"] else None
    done = 0
    for i, n in enumerate(sizes):
        scale[starts[i]:starts[i] + n] = 1e-3 * 10.0 ** (-(i % 3))
        if where is not None:
            where[done:done + n] = torch.arange(starts[i], starts[i] + n, device="cuda")
        done += n
    scale *= torch.exp(randn(total))
    inside = scale > 0
    flat_g, flat_p = scale * randn(total), torch.where(inside, 0.05 * randn(total), 0.0)
    if case["packed"]:
        flat_g, flat_p = flat_g[where], flat_p[where]
    s = {"case": case, "sizes": sizes, "places": places, "starts": starts, "where": where, "step": STEP,
         "p": flat_p.to(TYPES[case["dtype"]]), "g": flat_g.to(TYPES[case["grads"]])}
    assert s["p"].numel() == length
    m, v = 0.3 * scale * randn(total), 0.1 * scale.square() * (0.25 + rand(total))
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_codes(m, 127, 2)
        s["v"], s["v_scale"] = _to_codes(v, 255, 4)
    else:
        s["m"], s["v"] = m, v
    if own:  # the optimizer that a training program keeps
        import paper_2501_17788_amd as warp

        def views(flat):
            return [flat[a:a + n] for a, n in zip(places, sizes)]

        s["params"], s["grads"] = views(s["p"]), views(s["g"])
        s["opt"] = warp.AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
                              bits=case["bits"])
        state = {k: s.pop(k) for k in ("m", "v", "m_scale", "v_scale") if k in s}
        s["opt"].load_state_dict({"step": STEP, "bits": case["bits"], **state})
    return s


# ---------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2501_17788_amd as warp

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        y, mean, rstd = warp.layer_norm(s["x"], s["weight"], s["bias"], EPS)
        if not case["train"]:
            return y
        return (y, *warp.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd))
    if kind in ("linear", "encode"):
        a = warp.quantize_rows(s["x"]) if kind == "linear" else warp.layer_norm_int8(s["x"], s["weight"], s["bias"],
                                                                                     EPS)
        w = warp.QuantizedRows(s["w"], s["w_scale"], case["cols"])
        return warp.linear_int8(a, w, s["b"], TYPES[case["out"]])
    s["opt"].step(s["grads"])
    return (s["p"], *s["opt"].moments())


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].float()
        mean, rstd = _stats(x)
        h = (x - mean) * rstd
        y = (h * s["weight"].float() + s["bias"].float()).to(s["x"].dtype)
        if not case["train"]:
            return y
        dy = s["dy"].float()
        c = dy * s["weight"].float()
        dx = rstd * (c - c.mean(1, keepdim=True) - h * (c * h).mean(1, keepdim=True))
        dw, db = (dy * h).sum(0), dy.sum(0)
        return y, dx.to(s["x"].dtype), dw.to(s["weight"].dtype), db.to(s["bias"].dtype)
    if kind in ("linear", "encode"):
        x = s["x"].float()
        if kind == "encode":
            mean, rstd = _stats(x)
            x = (x - mean) * rstd * s["weight"].float() + s["bias"].float()
        q, scale = _to_int8(x)
        out = (q @ s["w"][:, :case["cols"]].float().t()) * s["w_scale"] * scale
        if s["b"] is not None:
            out = out + s["b"]
        return out.to(TYPES[case["out"]])
    return _adamw_plain(s)


def _stats(x):
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    return mean, 1.0 / torch.sqrt(var + EPS)


def _to_int8(x):
    """Rows of whole numbers of at most 127, and the scale of each: x is about q * scale."""
    top = x.abs().amax(1, keepdim=True)
    inv = torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)
    return torch.round(x * inv), top * (1.0 / 127.0)


def _cutoffs(levels, power):
    j = torch.arange(1, levels + 1, device="cuda", dtype=torch.float32)
    t = (j - 0.5) * (1.0 / levels)
    t = t * t
    return t * t if power == 4 else t


def _to_codes(x, levels, power):
    """Moments as 8-bit codes, with a scale for each block: a code counts the cutoffs that the magnitude
    over the block's largest reaches. A second moment (power 4) above zero has a code above zero."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1).clamp(min=torch.finfo(torch.float32).tiny)
    c = torch.bucketize(b.abs() * (torch.ones_like(top) / top)[:, None], _cutoffs(levels, power), right=True)
    if power == 4:
        return torch.maximum(c, (b > 0).to(c.dtype)).to(torch.uint8).view(-1), top
    return torch.where(b < 0, -c, c).to(torch.int8).view(-1), top


def _from_codes(code, scale, levels, power):
    c = code.view(-1, BLOCK).float()
    t = c.abs() * (1.0 / levels)
    t = t * t
    t = t * t if power == 4 else t
    return (torch.where(c < 0, -t, t) * scale[:, None]).view(-1)


def _adamw_plain(s):
    case, eight = s["case"], s["case"]["bits"] == 8
    s["step"] += 1
    t = s["step"]
    m = _from_codes(s["m"], s["m_scale"], 127, 2) if eight else s["m"]
    v = _from_codes(s["v"], s["v_scale"], 255, 4) if eight else s["v"]
    p, g = s["p"].float(), s["g"].float()
    if case["packed"]:  # to the moments' places
        p, g = (torch.zeros_like(m).index_copy_(0, s["where"], x) for x in (p, g))
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    denom = torch.sqrt(v) / math.sqrt(1 - BETA2 ** t) + ADAM_EPS
    p = p * (1 - LR * DECAY) - (LR / (1 - BETA1 ** t)) * m / denom
    s["p"].copy_(p[s["where"]] if case["packed"] else p)
    if eight:
        s["m"], s["m_scale"] = _to_codes(m, 127, 2)
        s["v"], s["v_scale"] = _to_codes(v, 255, 4)
        m, v = _from_codes(s["m"], s["m_scale"], 127, 2), _from_codes(s["v"], s["v_scale"], 255, 4)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        m, v = s["m"], s["v"]
    return s["p"], m, v


# ---------------------------------------------------------------------------- bounds and 64-bit values

def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = sum(_tensor_sizes(case))
        p, g = (TYPES[case[k]].itemsize for k in ("dtype", "grads"))
        if case["bits"] == 32:
            return {"bytes": n * (2 * p + g + 16), "flops": 16 * n}
        # the 8-bit moments and, as the pass returns them, their 32-bit values
        return {"bytes": n * (2 * p + g + 4 + 8 + 16 / BLOCK), "flops": 40 * n}
    rows, cols, t = case["rows"], case["cols"], TYPES[case["dtype"]].itemsize
    if kind == "norm":
        p = TYPES[case["params"]].itemsize
        if case["train"]:
            return {"bytes": rows * cols * 4 * t + cols * 4 * p, "flops": 20 * rows * cols}
        return {"bytes": rows * cols * 2 * t + cols * 2 * p, "flops": 8 * rows * cols}
    n = case["n"]
    out = TYPES[case["out"]].itemsize
    extra = cols * 8 if kind == "encode" else 0
    return {"bytes": rows * cols * t + n * cols + 4 * n + rows * n * out + extra, "flops": 2 * rows * cols * n}


def exact(case, seed):
    s = _plain_state(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    x = s["x"].double()
    if case["kind"] != "linear":
        g, b = s["weight"].double(), s["bias"].double()
        mean = x.sum(1, keepdim=True) / case["cols"]
        std = torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / case["cols"] + EPS)
        h = (x - mean) / std
        x = h * g + b
    if case["kind"] == "norm":
        if not case["train"]:
            return x
        dy = s["dy"].double()
        c = dy * g
        along = (c * h).sum(1, keepdim=True) / case["cols"]
        dx = (c - c.sum(1, keepdim=True) / case["cols"] - h * along) / std
        return x, dx, (dy * h).sum(0), dy.sum(0)
    # the whole numbers are defined by 32-bit arithmetic: the factor 127 / max and its product are rounded
    top = x.abs().amax(1, keepdim=True)
    factor = (127.0 / top.float().double()).float().double()
    q = torch.round((x.float().double() * factor).float().double())
    out = (q @ s["w"][:, :case["cols"]].double().t()) * (top / 127.0) * s["w_scale"].double()
    return out + s["b"].double() if s["b"] is not None else out


def _plain_state(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_adamw(s):
    case = s["case"]
    t = s["step"] + 1
    p, g = s["p"].double(), s["g"].double()
    if case["bits"] == 8:
        m = s["m"].double().abs().div(127.0).pow(2) * s["m"].double().sign()
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = s["v"].double().div(255.0).pow(4) * s["v_scale"].double().repeat_interleave(BLOCK)
    else:
        m, v = s["m"].double(), s["v"].double()
    if case["packed"]:
        whole = torch.zeros_like(m)
        whole[s["where"]] = g
        g = whole
    m += (1 - BETA1) * (g - m)
    v += (1 - BETA2) * (g ** 2 - v)
    step = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    step = step[s["where"]] if case["packed"] else step
    p = p - LR * (DECAY * p + step)
    # 8-bit moments are a choice among 256 values: they have none in 64 bits
    return (p, None, None) if case["bits"] == 8 else (p, m, v)
