"""The operators that train a token encoder from its tokens (table lookup, linear layers with 8-bit inputs, softmax cross
entropy over a table) against their definitions in 64 bits (run on an MI355X).

Bounds. U = 2^-24 is fp32's unit roundoff; a result is rounded once to its type, by eps / 2 of its value (and half a
subnormal step). Products of two 16-bit elements are exact in fp32. The matrix cores' sums are counted as
rounded at every product by 2 U of the sum of magnitudes so far: k products are within 2 U k sum |a b|. A float32
product is six products of planes, and what it leaves out is below 2^-23 |a b|: within (12 k + 2) U sum |a b|. Sums of whole
numbers below 2^24 have no error at all, in any order: they find a term that is missing, doubled or misplaced at any
size.
"""
from __future__ import annotations

import gc
import math

import numpy as np
import pytest

import product_plans

torch = pytest.importorskip("torch")
w = pytest.importorskip("paper_2501_17788_amd")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}  # smallest above zero
ALL = pytest.mark.parametrize("dtype", list(TYPES.values()), ids=list(TYPES))


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def whole(g, most, *shape):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()


def rounding(v, dtype):
    return torch.finfo(dtype).eps / 2 * v.abs() + STEP[dtype] / 2


def close(got, want, tol, what):
    """Within tol; NaN for NaN; and an infinity of the right sign where a value within tol rounds to it: from 65,520 on in
    float16, whose largest number is 65,504 in steps of 32."""
    half = got.dtype == torch.float16
    got, want = got.detach().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= tol) & ~(got.isnan() & want.isnan())
    if half:
        bad &= ~(got.isinf() & (got.sign() == want.sign()) & (want.abs() + tol >= 65_520))
    if bad.any():
        i = torch.nonzero(bad.reshape(-1))[0].item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values are off, the first at {i}: "
                             f"{got.reshape(-1)[i].item()!r} for {want.reshape(-1)[i].item()!r}, bound "
                             f"{tol.expand_as(want).reshape(-1)[i].item():.3g}")


def shifted(t, by=1):
    """The same values at an address that suits one element and no more, rows an odd number of elements apart."""
    rows, cols = t.shape
    room = torch.full((rows * (cols + 3) + by,), 99.0, dtype=t.dtype, device=t.device)
    v = room[by:].view(rows, cols + 3)[:, :cols]
    v.copy_(t)
    return v


# ---------------------------------------------------------------------------- table lookup

def embed64(ids, table, scale):
    ids = ids.long()
    inside = (ids >= 0) & (ids < table.shape[0])
    out = table.double()[ids.clamp(0, table.shape[0] - 1)] * scale
    return torch.where(inside[..., None], out, torch.where(ids < 0, 0.0, math.nan)[..., None].to(out))


@ALL
@pytest.mark.parametrize("cols", [1, 3, 7, 8, 9, 64, 255, 512, 513, 771, 1024, 1030, 2049, 5000])
def test_embedding(cols, dtype):
    g = gen(cols)
    for vocabulary, shape in ((1, (3,)), (37, (5, 7)), (1000, (501,)), (50, ()), (50, (0,)), (20, (2, 1, 3))):
        table = randn(g, vocabulary, cols).to(dtype)
        ids = torch.randint(-2, vocabulary + 2, shape, generator=g, device="cuda")
        for i, t in ((ids, table), (ids.int(), shifted(table))):
            out = w.embedding(i, t, 1.7)
            assert out.dtype == dtype and out.shape == (*shape, cols)
            want = embed64(ids, table, float(np.float32(1.7)))
            close(out, want, torch.nan_to_num(U * want.abs() + rounding(want, dtype)), (vocabulary, shape))
    ids = torch.arange(24, device="cuda").view(4, 6).t()  # not in one piece
    table = randn(g, 24, cols).to(dtype)
    assert torch.equal(w.embedding(ids, table), table[ids])


def embed_back64(dy, ids, vocabulary, scale):
    """The gradient and its bound: n terms in any order are within n U of their magnitudes' sum."""
    dtype, dy, ids = dy.dtype, dy.double().reshape(-1, dy.shape[-1]), ids.long().reshape(-1)
    there = (ids >= 0) & (ids < vocabulary)
    sums, sizes = (torch.zeros(vocabulary, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids[there], v[there])
                   for v in (dy, dy.abs()))
    n = torch.bincount(ids[there], minlength=vocabulary)[:, None]
    want = sums * scale
    return want, abs(scale) * n * U * sizes + U * want.abs() + rounding(want, dtype)


@ALL
@pytest.mark.parametrize("cols", [1, 5, 8, 100, 513, 771, 1024, 2050])
def test_embedding_gradient(cols, dtype):
    g = gen(100 + cols)
    for vocabulary, shape in ((1, (700,)), (37, (9, 77)), (1000, (1,)), (3, (0,)), (5000, (300,)), (513, (4097,)),
                              (600, (5, 1900))):
        ids = torch.randint(-1, vocabulary + 1, shape, generator=g, device="cuda")
        if len(shape) == 1 and shape[0] > 500:  # a common token, whose sorted place starts anywhere
            ids[torch.rand(shape, generator=g, device="cuda") < 0.4] = vocabulary // 3
        dy = randn(g, *shape, cols).to(dtype)
        got = w.embedding_backward(dy, ids, vocabulary, 0.3)
        assert got.dtype == dtype and got.shape == (vocabulary, cols)
        close(got, *embed_back64(dy, ids, vocabulary, float(np.float32(0.3))), (vocabulary, shape))
        assert torch.equal(got, w.embedding_backward(dy, ids.int(), vocabulary, 0.3))
        if len(shape) == 1:
            assert torch.equal(got, w.embedding_backward(shifted(dy), ids, vocabulary, 0.3))


@pytest.mark.parametrize("count", [1, 2, 62, 63, 64, 65, 127, 128, 129, 191, 192, 193, 320, 4000, 4096, 4097, 9000])
def test_embedding_gradient_of_common_tokens(count):
    """A token that comes `count` times, with every number of smaller ones before it that moves it against the chunks of
    64 sorted tokens; exact in whole numbers."""
    g = gen(count)
    for before in (0, 1, 63, 64, 65, 100):
        ids = torch.cat([torch.full((before,), 2), torch.full((count,), 5), torch.arange(6, 40)]).cuda()
        ids = ids[torch.randperm(len(ids), generator=g, device="cuda")]
        dy = whole(g, 50, len(ids), 96)
        want = torch.zeros(41, 96, device="cuda").double().index_add_(0, ids, dy.double())
        assert torch.equal(w.embedding_backward(dy, ids, 41).double(), want), before


@pytest.mark.parametrize("tokens,vocabulary,cols", [
    (4096, 260_000, 8), (4097, 260_000, 8), (70_001, 300_000, 16), (131_072, 32_128, 64), (524_289, 511, 9),
    (600_001, 100_000, 8), (1_100_000, 2, 8), (4099, 1 << 19, 3), (65_537, 1, 4), (200_000, 512, 8), (200_000, 513, 8)])
def test_embedding_gradient_larger(tokens, vocabulary, cols):
    """Sorting in one to three passes and tiles of one to several units: exact in whole numbers."""
    g = gen(tokens)
    rare = torch.randint(-1, vocabulary, (tokens,), generator=g, device="cuda")
    ids = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.2, vocabulary // 2, rare)
    dy = whole(g, 3, tokens, cols)
    want = torch.zeros(vocabulary, cols, device="cuda").double().index_add_(0, ids.clamp(min=0), torch.where(
        ids[:, None] >= 0, dy, 0.0).double())
    say("embedding gradient", tokens, vocabulary, cols)
    got = w.embedding_backward(dy, ids, vocabulary)
    assert torch.equal(got.double(), want)


def test_embedding_gradient_is_the_same_every_time():
    g = gen(3)
    ids = (torch.rand(50_000, generator=g, device="cuda") ** 4 * 3000).long()
    dy = randn(g, 50_000, 200)
    first = w.embedding_backward(dy, ids, 3000)
    for _ in range(3):
        assert torch.equal(w.embedding_backward(dy, ids, 3000), first)


def test_embedding_past_32_bits():
    """Tables and rows of more than 2^31 elements."""
    g = gen(4)
    table = torch.empty(560_001, 4096, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ids = torch.tensor([0, 524_287, 524_288, 560_000, 1, 560_000], device="cuda")
    say("embedding from", table.numel(), "elements")
    assert torch.equal(w.embedding(ids, table), table[ids])
    many = torch.randint(0, 100, (560_001,), generator=g, device="cuda")
    out = w.embedding(many, table[:100])
    assert torch.equal(out[-50:], table[many[-50:]]) and torch.equal(out[524_280:524_300], table[many[524_280:524_300]])
    del out
    # gradients of rows behind 2^31 elements, and into them
    many[-1], many[-2] = 200, 201
    d = w.embedding_backward(table, many, 202)
    assert torch.equal(d[200], table[-1]) and torch.equal(d[201], table[-2])
    d = w.embedding_backward(table[:6].contiguous(), ids, 560_001)
    assert torch.equal(d[560_000], (table[3].float() + table[5].float()).bfloat16()) and torch.equal(d[524_288], table[2])
    assert int((d != 0).any(1).sum()) == 5


# ---------------------------------------------------------------------------- linear layers

def linear_tol(a, b, dtype, extra=0.0):
    """a [m, k] by b [n, k] in 64 bits and the bound of the kernels' errors before the last rounding."""
    k = a.shape[1]
    sizes = a.abs() @ b.abs().t()
    return ((12 * k + 2) if dtype == torch.float32 else 2 * k) * U * sizes + extra * sizes


SIZES = [(1, 1, 1), (1, 8, 8), (2, 3, 5), (5, 64, 64), (17, 100, 33), (64, 72, 128), (65, 771, 100), (130, 129, 257),
         (333, 1000, 70), (1, 2000, 1003), (700, 24, 3), (300, 520, 264)]


@ALL
@pytest.mark.parametrize("rows,cols,n", SIZES)
def test_linear(rows, cols, n, dtype):
    g = gen(rows * cols + n)
    x, weight, bias = randn(g, rows, cols).to(dtype), randn(g, n, cols).to(dtype), randn(g, n)
    dy = randn(g, rows, n).to(dtype)
    x64, w64, dy64 = x.double(), weight.double(), dy.double()
    want = x64 @ w64.t() + bias.double()
    tol = linear_tol(x64, w64, dtype) + 2 * U * (want.abs() + bias.double().abs()) + rounding(want, dtype)
    y = w.linear(x, weight, bias)
    assert y.dtype == dtype
    close(y, want, tol, "y")
    close(w.linear(x.view(rows, 1, cols), weight, bias.to(dtype)).view(rows, n), x64 @ w64.t() + bias.to(dtype).double(),
          tol + 2 * U * bias.double().abs() + rounding(want, dtype), "y of a bias of x's type")
    kept = w.quantize_rows(x)
    got = w.linear_backward(dy, kept, weight)
    for a, b in zip(got, w.linear_backward(shifted(dy), kept, shifted(weight))):
        # other layouts take copies of the operands: the same sums
        assert torch.equal(a, b)
    assert torch.equal(w.linear(shifted(x), shifted(weight), bias), y)
    dx, dw, db = got
    close(dx, dy64 @ w64, linear_tol(dy64, w64.t(), dtype) + rounding(dy64 @ w64, dtype), "dx")
    # q * s in 64 bits; rounded to the type for the product, of float32 once
    back = kept.values[:, :cols].double() * kept.scale.double()[:, None]
    want = dy64.t() @ back
    off = U if dtype == torch.float32 else torch.finfo(dtype).eps / 2 + U
    slip = STEP[dtype] / 2 * dy64.abs().sum(0)[:, None]
    close(dw, want, linear_tol(dy64.t(), back.t(), dtype, off) + slip + rounding(want, dtype), "dweight")
    sizes = dy64.abs().sum(0)
    close(db, dy64.sum(0), rows * U * sizes + rounding(dy64.sum(0), dtype), "dbias")


@ALL
@pytest.mark.parametrize("rows,cols,n", product_plans.SIZES + product_plans.FEW)
def test_linear_of_whole_numbers(rows, cols, n, dtype):
    """Every sum is exact, and so is its rounding."""
    g = gen(rows + cols + n)
    x, weight, dy = whole(g, 3, rows, cols).to(dtype), whole(g, 2, n, cols).to(dtype), whole(g, 2, rows, n).to(dtype)
    bias = whole(g, 100, n)
    say("linear", rows, cols, n, dtype)
    assert torch.equal(w.linear(x, weight, bias), (x.double() @ weight.double().t() + bias.double()).to(dtype))
    kept = w.QuantizedRows.from_int8(x.to(torch.int8), 2.0 ** torch.randint(-1, 2, (rows,), generator=g, device="cuda"))
    dx, dw, db = w.linear_backward(dy, kept, weight)
    assert torch.equal(dx, (dy.double() @ weight.double()).to(dtype))
    assert torch.equal(dw, (dy.double().t() @ (x.double() * kept.scale.double()[:, None])).to(dtype))
    assert torch.equal(db, dy.double().sum(0).to(dtype))


def test_linear_of_no_rows():
    for dtype in TYPES.values():
        x, weight = torch.zeros(0, 70, device="cuda", dtype=dtype), torch.ones(33, 70, device="cuda", dtype=dtype)
        y = w.linear(x, weight, torch.ones(33, device="cuda"))
        assert y.shape == (0, 33)
        dx, dw, db = w.linear_backward(y, w.quantize_rows(x), weight)
        assert dx.shape == (0, 70) and dw.shape == (33, 70) and not dw.any() and db.shape == (33,) and not db.any()


@ALL
def test_linear_of_spoilt_values(dtype):
    """An infinity or a NaN in a row of x or dy spoils what it enters and nothing else."""
    g = gen(9)
    x, weight, dy = randn(g, 200, 136).to(dtype), randn(g, 72, 136).to(dtype), randn(g, 200, 72).to(dtype)
    clean = w.linear(x, weight)
    x[7, 3], x[190, 100] = math.inf, math.nan
    y = w.linear(x, weight)
    rows = [i for i in range(200) if i not in (7, 190)]
    assert torch.equal(y[rows], clean[rows]) and not y[[7, 190]].isfinite().any()
    kept = w.quantize_rows(torch.nan_to_num(x, nan=0.0, posinf=1.0))
    clean = w.linear_backward(dy, kept, weight)
    dy[11, 5] = math.nan
    dx, dw, db = w.linear_backward(dy, kept, weight)
    rows = [i for i in range(200) if i != 11]
    cols = [i for i in range(72) if i != 5]
    assert torch.equal(dx[rows], clean[0][rows]) and dx[11].isnan().all()
    assert torch.equal(dw[cols], clean[1][cols]) and dw[5].isnan().all()
    assert torch.equal(db[cols], clean[2][cols]) and db[5].isnan()


def test_float32_products_keep_their_digits():
    """Elements with 24 bits set, in sums of one to eight products: nothing of a plane is lost. And magnitudes from the
    smallest normal numbers to those near the largest."""
    g = gen(10)
    for k in (1, 2, 3, 8):
        x = (torch.randint(2 ** 23, 2 ** 24, (130, k), generator=g, device="cuda") | 1).float() * 2.0 ** -23
        weight = (torch.randint(2 ** 23, 2 ** 24, (70, k), generator=g, device="cuda") | 1).float() * -2.0 ** -23
        for by in (1.0, 2.0 ** 120, 2.0 ** -100):
            want = (x.double() * by) @ weight.double().t()
            close(w.linear(x * by, weight), want, linear_tol(x.double() * by, weight.double(), torch.float32) +
                  rounding(want, torch.float32), (k, by))


@pytest.mark.parametrize("rows", [1, 20, 40, 300, 500, 3000])
def test_float32_products_of_tiny_values(rows):
    """Subnormal operands: in planes each loses less than 2^-133."""
    g = gen(rows)
    x, weight = 1e-40 * randn(g, rows, 64), 1e10 * randn(g, 72, 64)
    want, sizes = x.double() @ weight.double().t(), x.double().abs() @ weight.double().abs().t()
    lost = 0.0 if rows <= 300 else 2.0 ** -133
    close(w.linear(x, weight), want, (12 * 64 + 3) * U * sizes + lost * weight.double().abs().sum(1), "y")
    dy = 1e-40 * randn(g, rows, 72)
    want, sizes = dy.double() @ weight.double(), dy.double().abs() @ weight.double().abs()
    dx, _, _ = w.linear_backward(dy, w.quantize_rows(torch.ones(rows, 64, device="cuda")), weight)
    close(dx, want, (12 * 72 + 3) * U * sizes + lost * weight.double().abs().sum(0), "dx")


def test_linear_past_32_bits():
    """x and y of more than 2^31 elements: the last rows equal those of a call on them alone."""
    g = gen(12)
    weight = whole(g, 2, 1024, 64).bfloat16()
    x = torch.randint(-3, 4, (2_200_001, 64), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    say("linear of", x.shape[0] * 1024, "results")
    y = w.linear(x, weight)
    at = [slice(0, 5), slice(2_097_100, 2_097_200), slice(2_199_990, 2_200_001)]
    for s in at:
        assert torch.equal(y[s], (x[s].double() @ weight.double().t()).bfloat16())
    kept = w.QuantizedRows.from_int8(x.to(torch.int8), torch.ones(2_200_001, device="cuda"))
    y.clamp_(-1, 1)
    dx, dw, db = w.linear_backward(y, kept, weight)
    for s in at:
        assert torch.equal(dx[s], (y[s].double() @ weight.double()).bfloat16())
    assert torch.equal(db, y.double().sum(0).bfloat16())
    want = torch.zeros(1024, 64, dtype=torch.float64, device="cuda")
    for part in range(0, 2_200_001, 200_000):
        want += y[part:part + 200_000].double().t() @ x[part:part + 200_000].double()
    assert torch.equal(dw, want.bfloat16())


# ---------------------------------------------------------------------------- softmax cross entropy

class Loss64:
    """The loss in 64 bits, with bounds of the kernels' errors. A logit is off by the product's error and 3 U of its value
    (its factor, the product with it, its rounding in units of log 2); a sum of v exponentials by v U and 24 U (three
    levels of sums, each with exponentials that are off by 2 U or more); so p = exp(l - lse) by twice the largest logit's
    error and those, relative. Exponentials below 2^-126 are zero. loss = log(1 + S) moves by S / (1 + S) times S's relative
    error, 1 - p by that times p; the logarithms and expm1 are off by up to 4 U."""

    def __init__(self, hidden, table, targets, scale):
        self.h, self.t, self.scale, self.dtype = hidden.double(), table.double(), scale, hidden.dtype
        self.v = table.shape[0]
        self.y = targets.long()
        self.keep = (self.y >= 0) & (self.y < self.v)
        self.outside = self.y >= self.v
        y = self.y.clamp(0, self.v - 1)
        logits = scale * (self.h @ self.t.t())
        self.lse = torch.logsumexp(logits, 1)
        off = abs(scale) * linear_tol(self.h, self.t, self.dtype) + 3 * U * logits.abs()
        self.rel = 2 * off.amax(1) + (self.v + 24) * U + 4 * U * self.lse.abs()
        self.p = torch.exp(logits - self.lse[:, None])
        others = self.p.scatter(1, y[:, None], 0.0).sum(1)  # 1 - p without a difference
        self.loss = torch.where(self.p.gather(1, y[:, None])[:, 0] > 0.5, -torch.log1p(-others),
                                self.lse - logits.gather(1, y[:, None])[:, 0])
        self.e_loss = others * self.rel + 8 * U * self.loss + self.v * 2.0 ** -126
        self.others, self.at = others, y
        nan = torch.full_like(self.loss, math.nan)
        self.want_loss = torch.where(self.keep, self.loss, torch.where(self.outside, nan, 0.0))
        self.want_lse = torch.where(self.keep, self.lse, torch.where(self.outside, nan, 0.0))
        self.e_lse = self.rel + 2 * U * self.lse.abs()

    def backward(self, dloss):
        g = torch.where(self.keep, dloss.double(), 0.0)[:, None]
        half = 0.0 if self.dtype == torch.float32 else torch.finfo(self.dtype).eps / 2
        G = self.p.scatter(1, self.at[:, None], -self.others[:, None]) * g
        # G's own error, its rounding, and in float16 a subnormal step of the largest |dloss| / 2^15
        off = self.p * self.rel[:, None]
        off.scatter_(1, self.at[:, None], (self.others * self.rel * 2 + 16 * U * self.others)[:, None])
        off = g.abs() * (off + 4 * U * self.p) + (half + 2 * U) * G.abs()
        off = off + torch.where(g != 0, 2.0 ** -124 * g.abs().max(), 0.0)
        if self.dtype == torch.float16:
            off = off + torch.where(g != 0, 2.0 ** -25 * 2.0 ** -15 * g.abs().max(), 0.0)
        h = torch.where(self.keep[:, None], self.h, 0.0)
        out = []
        for a, e, b, k in ((G, off, self.t, self.v), (G.t(), off.t(), h, len(h))):
            want = self.scale * (a @ b)
            chain = (12 * k + 2) if self.dtype == torch.float32 else 2 * k
            tol = abs(self.scale) * (e @ b.abs() + chain * U * ((a.abs() + e) @ b.abs())) + 8 * U * want.abs()
            out.append((want, tol + rounding(want, self.dtype)))
        out[0] = (torch.where(self.outside[:, None], math.nan, out[0][0]), out[0][1])
        return out


def scores(g, tokens, vocabulary, cols, dtype, sharp=1.0):
    table = randn(g, vocabulary, cols).to(dtype)
    targets = torch.randint(0, vocabulary, (tokens,), generator=g, device="cuda")
    sure = torch.rand(tokens, 1, generator=g, device="cuda") * 3 * sharp
    hidden = (randn(g, tokens, cols) + sure * table[targets].float()).to(dtype)
    return hidden, table, targets


def check_loss(hidden, table, targets, scale, dloss, what):
    scale = float(np.float32(scale))
    r = Loss64(hidden, table, targets, scale)
    loss, lse = w.cross_entropy(hidden, table, targets, scale)
    assert loss.dtype == lse.dtype == torch.float32
    close(loss, r.want_loss, r.e_loss, (what, "loss"))
    close(lse, r.want_lse, r.e_lse, (what, "lse"))
    dh, dt = w.cross_entropy_backward(dloss, hidden, table, targets, loss, lse, scale)
    for name, got, (want, tol) in zip(("dhidden", "dtable"), (dh, dt), r.backward(dloss)):
        assert got.dtype == hidden.dtype
        close(got, want, tol, (what, name))
    return loss, lse, dh, dt


LOSSES = [(1, 1, 1), (1, 5, 3), (3, 2, 8), (7, 64, 64), (33, 65, 100), (64, 300, 72), (65, 1003, 771), (130, 257, 40),
          (300, 520, 264), (1, 2000, 128), (2, 70, 1000)]


@ALL
@pytest.mark.parametrize("tokens,vocabulary,cols", LOSSES)
def test_cross_entropy(tokens, vocabulary, cols, dtype):
    g = gen(tokens + vocabulary + cols)
    hidden, table, targets = scores(g, tokens, vocabulary, cols, dtype)
    dloss = (0.5 + torch.rand(tokens, generator=g, device="cuda")) * (1000 if dtype == torch.float16 else 1)
    a = check_loss(hidden, table, targets, cols ** -0.5, dloss, "all")
    # rows left out, and one target outside the vocabulary; other layouts
    some = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.4, -100, targets)
    some[tokens // 2] = vocabulary + 3
    check_loss(hidden, table, some, cols ** -0.5, dloss, "some")
    b = check_loss(shifted(hidden), shifted(table), targets.int(), cols ** -0.5, dloss, "shifted")
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@ALL
@pytest.mark.parametrize("tokens", [1, 15, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257])
def test_cross_entropy_of_few_tokens(tokens, dtype):
    """On both sides of the numbers of tokens that choose between the kernels; vocabularies of both of their widths."""
    for vocabulary, cols in ((5, 1), (33, 260), (300, 1030), (8200, 129), (16_500, 64), (17_000, 33)):
        g = gen(tokens + vocabulary)
        hidden, table, targets = scores(g, tokens, vocabulary, cols, dtype)
        if tokens > 2:
            targets[1], targets[2] = -1, vocabulary
        dloss = torch.full((tokens,), 1000.0 if dtype == torch.float16 else 1.0, device="cuda")
        say("cross entropy of few", tokens, vocabulary, cols, dtype)
        a = check_loss(hidden, table, targets, cols ** -0.5, dloss, (tokens, vocabulary))
        b = check_loss(shifted(hidden), shifted(table), targets.int(), -cols ** -0.5, dloss, (tokens, vocabulary, "negative"))
        assert torch.isfinite(a[0]).sum() == torch.isfinite(b[0]).sum() >= tokens - 1
        if tokens > 2:  # what a row that is left out holds is in no result
            hidden[1] = math.nan
            loss, lse = w.cross_entropy(hidden, table, targets, cols ** -0.5)
            c = (loss, lse, *w.cross_entropy_backward(dloss, hidden, table, targets, loss, lse, cols ** -0.5))
            assert all(torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in zip(a, c))


@ALL
def test_cross_entropy_of_larger_sizes(dtype):
    """Tiles of 128 and 256, many parts of a sum."""
    for tokens, vocabulary, cols in ((2100, 3001, 136), (400, 30_011, 72), (5000, 130, 64), (9, 100_003, 24), (140_001, 50, 8)):
        g = gen(tokens)
        hidden, table, targets = scores(g, tokens, vocabulary, cols, dtype)
        targets[::3] = -1
        dloss = torch.full((tokens,), 1000.0 if dtype == torch.float16 else 1.0, device="cuda")
        say("cross entropy", tokens, vocabulary, cols, dtype)
        check_loss(hidden, table, targets, cols ** -0.5, dloss, (tokens, vocabulary))


def test_cross_entropy_in_pieces():
    """A vocabulary in several pieces: of float32 rows G's three planes, and the packed table."""
    g = gen(31)
    hidden, table, targets = scores(g, 8191, 24_007, 9, torch.float32)
    say("cross entropy in pieces")
    check_loss(hidden, table, targets, 0.3, torch.ones(8191, device="cuda"), "pieces of G")
    # more tiles than the statistics of one piece have room for
    hidden, table, targets = scores(g, 140_001, 65_000, 8, torch.bfloat16)
    targets[targets % 16 != 3] = -100
    loss, lse = w.cross_entropy(hidden, table, targets, 0.3)
    rows = torch.nonzero(targets >= 0)[:, 0]
    r = Loss64(hidden[rows], table, targets[rows], float(np.float32(0.3)))
    close(loss[rows], r.want_loss, r.e_loss, "pieces of statistics")
    assert not loss[targets < 0].any() and not lse[targets < 0].any()
    # a table that is packed piece by piece, whose rows are no whole pieces of 16 bytes
    hidden, table, targets = scores(g, 70, 300_001, 1025, torch.bfloat16)
    targets[:5] = torch.tensor([0, 300_000, 150_015, 150_016, -1], device="cuda")
    check_loss(hidden, table, targets, 0.02, torch.ones(70, device="cuda"), "pieces of a packed table")


@ALL
def test_cross_entropy_left_out_rows(dtype):
    """What lies in rows without a target does not count, be it infinite or NaN; all rows may be such."""
    g = gen(32)
    hidden, table, targets = scores(g, 90, 300, 72, dtype)
    dloss = 0.5 + torch.rand(90, generator=g, device="cuda")
    targets[::2] = -1
    want = check_loss(hidden, table, targets, 0.1, dloss, "clean")
    hidden[::4], hidden[2::4], dloss[::2] = math.nan, math.inf, math.nan
    for a, b in zip(want, w.cross_entropy(hidden, table, targets, 0.1)):
        assert torch.equal(a, b)
    for a, b in zip(want[2:], w.cross_entropy_backward(dloss, hidden, table, targets, *want[:2], 0.1)):
        assert torch.equal(a, b)
    targets[:] = -7
    loss, lse = w.cross_entropy(hidden, table, targets, 0.1)
    dh, dt = w.cross_entropy_backward(dloss, hidden, table, targets, loss, lse, 0.1)
    assert not loss.any() and not lse.any() and not dh.any() and not dt.any()
    loss, lse = w.cross_entropy(hidden[:0], table, targets[:0])
    dh, dt = w.cross_entropy_backward(dloss[:0], hidden[:0], table, targets[:0], loss, lse)
    assert loss.shape == (0,) and dh.shape == (0, 72) and dt.shape == table.shape and not dt.any()


def test_cross_entropy_hard_values():
    g = gen(33)
    for dtype in TYPES.values():
        # tokens that are all but sure, right or wrong; logits of hundreds
        hidden, table, targets = scores(g, 60, 130, 64, dtype, sharp=4)
        targets[::3] = (targets[::3] + 1) % 130
        for scale in (1.0, 3.0, -1.0, 0.0):
            check_loss(hidden, table, targets, scale, torch.ones(60, device="cuda"), scale)
        # a token without doubt keeps the digits of a tiny loss
        hidden, table = torch.zeros(2, 64, device="cuda").to(dtype), torch.zeros(5, 64, device="cuda").to(dtype)
        hidden[:, 0], table[1, 0] = 4.0, 6.0
        loss, _ = w.cross_entropy(hidden, table, torch.tensor([1, 0], device="cuda"))
        want = torch.tensor([math.log1p(4 * math.exp(-24)), 24 + math.log1p(4 * math.exp(-24))], device="cuda").double()
        close(loss, want, want * 40 * U, "sure")
        # a spoilt row spoils its own loss and gradient and no other row's
        hidden, table, targets = scores(g, 70, 200, 72, dtype)
        clean = w.cross_entropy(hidden, table, targets, 0.1)
        hidden[9, 4], hidden[50] = math.nan, math.inf
        loss, lse = w.cross_entropy(hidden, table, targets, 0.1)
        rows = [i for i in range(70) if i not in (9, 50)]
        assert torch.equal(loss[rows], clean[0][rows]) and not loss[[9, 50]].isfinite().any()
        dh, dt = w.cross_entropy_backward(torch.ones(70, device="cuda"), hidden, table, targets, loss, lse, 0.1)
        assert dh[rows].isfinite().all() and not dh[[9, 50]].isfinite().any()
        # a gradient that overflowed in one row
        hidden, table, targets = scores(g, 70, 200, 72, dtype)
        clean = w.cross_entropy(hidden, table, targets, 0.1)
        dloss = torch.ones(70, device="cuda")
        a = w.cross_entropy_backward(dloss, hidden, table, targets, *clean, 0.1)[0]
        dloss[3] = math.inf
        b = w.cross_entropy_backward(dloss, hidden, table, targets, *clean, 0.1)[0]
        assert torch.equal(a[4:], b[4:]) and not b[3].isfinite().any()


def test_cross_entropy_weights_of_every_size():
    """dloss of many magnitudes, among them zeros; a gradient far below float16's smallest number comes back scaled."""
    g = gen(34)
    for dtype in TYPES.values():
        hidden, table, targets = scores(g, 120, 500, 64, dtype)
        dloss = 10.0 ** torch.randint(-3, 4, (120,), generator=g, device="cuda").float()
        dloss[::5], dloss[1::5] = 0.0, -dloss[1::5]
        check_loss(hidden, table, targets, 0.125, dloss, "sizes")
        loss, lse = w.cross_entropy(hidden, table, targets, 0.125)
        dh, dt = w.cross_entropy_backward(torch.zeros_like(dloss), hidden, table, targets, loss, lse, 0.125)
        assert not dh.any() and not dt.any()


def test_cross_entropy_gradients_against_differences():
    """Central differences of sum(dloss * loss) in 64 bits: their own error is h^2 / 6 of a third derivative of a few units
    (h = 1e-4) and 1e-15 / h of rounding: 1e-7 bounds both."""
    g = gen(35)
    hidden, table, targets = scores(g, 4, 9, 6, torch.float32)
    targets[2] = -1
    dloss, h = 0.5 + torch.rand(4, generator=g, device="cuda"), 1e-4
    keep = targets >= 0

    def total(a, b):
        logits = 0.5 * (a @ b.t())
        each = torch.logsumexp(logits, 1) - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
        return (dloss.double() * torch.where(keep, each, 0.0)).sum()

    loss, lse = w.cross_entropy(hidden, table, targets, 0.5)
    got = w.cross_entropy_backward(dloss, hidden, table, targets, loss, lse, 0.5)
    bounds = [tol for _, tol in Loss64(hidden, table, targets, 0.5).backward(dloss)]
    args = [hidden.double(), table.double()]
    for i in range(2):
        slopes = []
        for at in range(args[i].numel()):
            step = torch.zeros_like(args[i]).view(-1)
            step[at] = h
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + step.view_as(args[i]), args[i] - step.view_as(args[i])
            slopes.append((total(*up) - total(*down)) / (2 * h))
        want = torch.stack(slopes).view_as(args[i])
        close(got[i], want, bounds[i] + 1e-7 * (1 + want.abs()), i)


def test_cross_entropy_past_32_bits():
    """A table of more than 2^31 elements, targets on both sides."""
    g = gen(36)
    table = torch.empty(280_003, 8192, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    targets = torch.tensor([0, 262_143, 262_144, 280_002, 5], device="cuda")
    hidden = table[targets] * 0.125
    say("cross entropy over", table.numel(), "elements")
    scale = 2.0 ** -8
    loss, lse = w.cross_entropy(hidden, table, targets, scale)
    logits = torch.cat([scale * (hidden.double() @ t.double().t()) for t in table.split(20_000)], 1)
    want = torch.logsumexp(logits, 1) - logits.gather(1, targets[:, None])[:, 0]
    # products: 2 k U sum |a b| of about 8192 * 0.125 * 0.64; exponentials' sums as in Loss64
    tol = torch.full_like(want, 2 * (scale * 2 * 8192 * U * 8192 * 0.125 + 3 * U * 8) + 280_011 * U)
    close(loss, want, tol, "loss")
    dh, dt = w.cross_entropy_backward(torch.ones(5, device="cuda"), hidden, table, targets, loss, lse, scale)
    p = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))
    p[torch.arange(5, device="cuda"), targets] -= 1
    for rows in (slice(0, 9), slice(262_140, 262_150), slice(279_993, 280_003)):
        want = scale * (p[:, rows].t() @ hidden.double())
        size = scale * (p[:, rows].abs().t() @ hidden.double().abs())
        close(dt[rows], want, size * (2.0 ** -8 + 2 * tol[0]) + rounding(want, torch.bfloat16), rows)


# ---------------------------------------------------------------------------- as they are used

def test_autograd():
    """Gradients reach what they should, as the backward calls give them; none under no_grad, and no second ones."""
    g = gen(40)
    for dtype in TYPES.values():
        ids = torch.randint(-1, 50, (3, 20), generator=g, device="cuda")
        table = randn(g, 50, 72).to(dtype).requires_grad_()
        weight, bias = randn(g, 40, 72).to(dtype).requires_grad_(), randn(g, 40).requires_grad_()
        x = w.embedding(ids, table, 2.0)
        dy = randn(g, 3, 20, 72).to(dtype)
        assert torch.equal(torch.autograd.grad(x, table, dy)[0], w.embedding_backward(dy, ids, 50, 2.0))
        expanded, = torch.autograd.grad(w.embedding(ids, table).sum(), table)
        assert torch.equal(expanded, w.embedding_backward(torch.ones_like(dy), ids, 50))
        x = randn(g, 3, 20, 72).to(dtype).requires_grad_()
        y = w.linear(x, weight, bias)
        dy = randn(g, 3, 20, 40).to(dtype)
        kept = w.quantize_rows(x.detach())
        want = w.linear_backward(dy, kept, weight.detach())
        got = torch.autograd.grad(y, [x, weight, bias], dy)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert got[2].dtype == torch.float32 and torch.equal(got[2].to(dtype), want[2])
        # shared rows; one gradient alone; a broadcast gradient; no bias
        got, = torch.autograd.grad(w.linear(x.detach(), weight, None, kept), [weight], dy)
        assert torch.equal(got, want[1])
        got, = torch.autograd.grad(w.linear(x, weight.detach()), [x], dy)
        assert torch.equal(got, want[0])
        got, = torch.autograd.grad(w.linear(x.detach(), weight.detach(), bias).sum(), [bias])
        assert torch.equal(got, torch.full((40,), 60.0, device="cuda"))
        targets = torch.randint(-1, 50, (3, 20), generator=g, device="cuda")
        loss, lse = w.cross_entropy(x, table, targets, 0.1)
        assert loss.requires_grad and not lse.requires_grad
        ones = torch.full((3, 20), 1 / 60, device="cuda")
        want = w.cross_entropy_backward(ones, x.detach(), table.detach(), targets, loss.detach(), lse, 0.1)
        mean = loss.mean()
        loss.detach().zero_()  # the node keeps its own
        got = torch.autograd.grad(mean, [x, table], retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for i, leaf in enumerate((x, table)):
            args = [x.detach(), table.detach()]
            args[i] = leaf
            got, = torch.autograd.grad(w.cross_entropy(*args, targets, 0.1)[0].mean(), [leaf])
            assert torch.equal(got, want[i])
        with torch.no_grad():
            for out in (w.embedding(ids, table), w.linear(x, weight, bias), w.cross_entropy(x, table, targets)[0]):
                assert not out.requires_grad
    x, weight, table = (randn(g, 8, 16).requires_grad_() for _ in range(3))
    ids = torch.arange(8, device="cuda")
    for out in (w.linear(x, weight).square().sum(), w.embedding(ids, table).square().sum(),
                w.cross_entropy(x, table, ids)[0].square().sum()):
        leaf = next(t for t in (x, table) if torch.autograd.grad(out, [t], allow_unused=True, retain_graph=True)[0] is not None)
        first, = torch.autograd.grad(out, [leaf], create_graph=True)
        with pytest.raises(RuntimeError):
            first.sum().backward()


def test_linear_keeps_8_bits():
    """What autograd holds of a layer's input between the passes is its 8-bit rows."""
    x = randn(gen(41), 8192, 1024).bfloat16()
    weight = randn(gen(42), 512, 1024).bfloat16().requires_grad_()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = w.linear(x, weight)
    held = torch.cuda.memory_allocated() - before - y.numel() * 2
    assert 8192 * 1024 <= held <= 8192 * (1024 + 8) + 4096


def encoder64(ids, targets, table, norm, weight, bias, rounded):
    """The chain of the next test in 64 bits; `rounded`: the rows that the linear layer keeps, for its weight's gradient."""
    x = table[ids.clamp(min=0)] * 4.0 * (ids >= 0)[:, None]
    d = x - x.mean(1, keepdim=True)
    n = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * norm
    y = n @ weight.t() + bias
    y = y - (n - rounded).detach() @ weight.t() + ((n - rounded).detach() @ weight.detach().t())
    logits = y @ table.t() * 0.125
    each = torch.logsumexp(logits, 1) - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    return torch.where(targets >= 0, each, 0.0).sum() / (targets >= 0).sum()


def test_a_training_step_of_all():
    """Table, lookup, layer norm, linear layer, loss over the same table, AdamW: gradients against 64 bits, and steps."""
    g = gen(43)
    ids = torch.randint(-1, 301, (700,), generator=g, device="cuda")
    targets = torch.where(torch.rand(700, generator=g, device="cuda") < 0.3, ids, -100)
    table, weight = 0.3 * randn(g, 301, 64), randn(g, 64, 64) / 8
    norm, bias = 1 + 0.1 * randn(g, 64), 0.1 * randn(g, 64)
    leaves = [t.requires_grad_() for t in (table, norm, weight, bias)]
    opt = w.AdamW(leaves, lr=1e-2, bits=32)
    first = None
    for step in range(4):
        x = w.embedding(ids, table, 4.0)
        n = w.layer_norm(x, norm)[0]
        loss, _ = w.cross_entropy(w.linear(n, weight, bias), table, targets, 0.125)
        total = loss.sum() / (targets >= 0).sum()
        grads = torch.autograd.grad(total, leaves)
        q = w.quantize_rows(n.detach())
        wide = [t.detach().double().requires_grad_() for t in leaves]
        total64 = encoder64(ids, targets, *wide, q.values[:, :64].double() * q.scale.double()[:, None])
        assert abs(total.item() - total64.item()) < 1e-5 * total64.item()
        for a, b in zip(grads, torch.autograd.grad(total64, wide)):
            # relative to the largest: fp32 chains of at most 700 terms, 2 U each, through four operators
            assert (a.double() - b).abs().max() <= 4 * 2 * 700 * U * b.abs().max() + 1e-6 * b.abs().max()
        opt.step([t.contiguous() for t in grads])
        first = first if first is not None else total.item()
    assert total.item() < first


def calls(g, dtype=torch.bfloat16):
    """One call of each kind, as a function of its inputs, and a function that gives them new values."""
    ids = torch.randint(-1, 3000, (6000,), generator=g, device="cuda")
    targets = torch.randint(-1, 3000, (6000,), generator=g, device="cuda")
    targets[::2] = -1
    table, x, dy = (randn(g, n, 136).to(dtype) for n in (3000, 6000, 6000))
    weight, bias = randn(g, 100, 136).to(dtype), randn(g, 100)
    dz, dloss = randn(g, 6000, 100).to(dtype), torch.rand(6000, generator=g, device="cuda")

    def renew():
        for t, n in ((ids, 3000), (targets, 3000)):
            t.copy_(torch.randint(-1, n, t.shape, generator=g, device="cuda"))
        for t in (table, x, dy, weight, bias, dz, dloss):
            t.copy_(randn(g, *t.shape))

    def work(stream=None):
        out = [w.embedding(ids, table, 1.5, stream=stream), w.embedding_backward(dy, ids, 3000, 1.5, stream=stream),
               w.linear(x, weight, bias, stream=stream)]
        kept = w.quantize_rows(x, stream=stream)
        out += w.linear_backward(dz, kept, weight, stream=stream)
        loss, lse = w.cross_entropy(x, table, targets, 0.1, stream=stream)
        return [*out, loss, lse, *w.cross_entropy_backward(dloss, x, table, targets, loss, lse, 0.1, stream=stream)]

    return work, renew


@ALL
def test_another_stream(dtype):
    work, renew = calls(gen(44), dtype)
    want = work()
    s = torch.cuda.Stream()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        got = work(s)
        torch.full((4_000_000,), 3.0, device="cuda")  # other work that may take freed memory
        torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got


@ALL
def test_captured_in_two_graphs(dtype):
    """Two graphs of the same calls on inputs of their own, replayed in turn, side by side and with eager work between."""
    made = [calls(gen(45 + i), dtype) for i in range(2)]
    graphs, outs = [], []
    for work, _ in made:
        work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(work())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in range(4):
        for _, renew in made:
            renew()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for (work, _), out in zip(made, outs):
            for i, (a, b) in enumerate(zip(out, work())):
                assert torch.equal(a, b), (k, i)


@pytest.mark.parametrize("name", ["embedding", "linear", "cross_entropy", "layer_norm"])
def test_captured_backward_of_leaves_in_use(name):
    """A backward pass under capture is refused while an eager graph of its leaves lives; afterwards it is captured, and
    replays give what eager passes give."""
    g = gen(60)
    leaf = randn(g, 97, 64).requires_grad_() if name != "layer_norm" else (1 + 0.1 * randn(g, 64)).requires_grad_()
    x, ids = randn(g, 70, 64), torch.randint(-1, 97, (70,), generator=g, device="cuda")
    out = {"embedding": lambda: w.embedding(ids, leaf), "linear": lambda: w.linear(x, leaf),
           "cross_entropy": lambda: w.cross_entropy(x, leaf, ids)[0], "layer_norm": lambda: w.layer_norm(x, leaf)[0]}[name]
    dy = torch.randn(out().shape, generator=g, device="cuda")
    lives = out()
    torch.cuda.synchronize()
    say("refused capture of", name)
    with pytest.raises(RuntimeError, match="cannot be captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            out().backward(dy)
    assert leaf.grad is None
    lives.backward(dy)  # the eager graph is whole
    assert leaf.grad is not None
    leaf.grad = None
    del lives
    gc.collect()  # the refused graph, which the error's traceback held
    torch.cuda.synchronize()
    say("capture of", name)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out().backward(dy)
    got = leaf.grad
    for k in range(3):
        x.copy_(randn(g, 70, 64))
        dy.copy_(torch.randn(dy.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.no_grad():
            kept = got.clone()
        assert torch.equal(kept, torch.autograd.grad(out(), leaf, dy)[0]), k


def test_products_side_by_side():
    """Products on two streams at once, whose workgroups share compute units: the same bits as alone. Loads into LDS that
    came before another wave's reads showed here, in one call of ten."""
    g = gen(50)
    x = [randn(g, 6000, 136) for _ in range(2)]
    weight = randn(g, 3000, 136)
    q, wq = [w.quantize_rows(t) for t in x], w.quantize_rows(weight)
    targets = torch.randint(0, 3000, (6000,), generator=g, device="cuda")
    dy = randn(g, 6000, 3000)

    def work(i):
        out = [w.linear_int8(q[i], wq), w.linear(x[i], weight), *w.cross_entropy(x[i], weight, targets, 0.1)]
        out += w.linear_backward(dy, q[i], weight)[:2]
        return out + list(w.cross_entropy_backward(targets.float(), x[i], weight, targets, *out[2:4], 0.1))

    want = [work(i) for i in range(2)]
    graphs, outs = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(work(i))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in range(40):
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b)), k


def test_outputs_alone_are_written():
    """C calls into the middle of larger buffers: what lies around the results stays."""
    lib, g = w.lib, gen(47)
    stream = torch.cuda.current_stream().cuda_stream
    ids = torch.randint(0, 30, (5,), generator=g, device="cuda")
    for cols in (5, 64, 100):
        table, x = randn(g, 30, cols), randn(g, 5, cols)
        room = torch.full((40, cols + 7), 7.0, device="cuda")
        scratch = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        at = room[4:, 3:].data_ptr()
        P = lambda t: t.data_ptr()  # noqa: E731

        def check(rows, wide, want):
            assert torch.equal(room[4:4 + rows, 3:3 + wide], want)
            room[4:4 + rows, 3:3 + wide] = 7.0
            assert (room == 7.0).all()

        assert not lib.warp_embedding(P(ids), 8, 5, P(table), cols, 30, cols, 0, 1.0, at, cols + 7, stream)
        check(5, cols, table[ids])
        assert not lib.warp_embedding_backward(P(x), cols, P(ids), 8, 5, 30, cols, 0, 1.0, at, cols + 7, P(scratch), 1 << 28,
                                               stream)
        check(30, cols, w.embedding_backward(x, ids, 30))
        weight = randn(g, cols, cols)
        assert not lib.warp_linear(P(x), cols, 5, cols, 0, P(weight), cols, cols, None, 0, at, cols + 7, P(scratch), 1 << 28,
                                   stream)
        check(5, cols, w.linear(x, weight))
        kept = w.quantize_rows(x)
        back = w.linear_backward(x, kept, weight)
        for part, rows in ((0, 5), (1, cols)):
            if rows > 36:
                continue
            to = [(None, 0), (None, 0)]
            to[part] = (at, cols + 7)
            assert not lib.warp_linear_backward(P(x), cols, 5, cols, 0, P(kept.values), kept.values.stride(0), P(kept.scale),
                                                cols, P(weight), cols, *to[0], *to[1], None, 0, P(scratch), 1 << 28, stream)
            check(rows, cols, back[part])
        loss, lse = w.cross_entropy(x, table, ids)
        dloss = torch.ones(5, device="cuda")
        want = w.cross_entropy_backward(dloss, x, table, ids, loss, lse)
        for part, rows in ((0, 5), (1, 30)):
            to = [(None, 0), (None, 0)]
            to[part] = (at, cols + 7)
            assert not lib.warp_cross_entropy_backward(P(dloss), P(x), cols, 5, cols, 0, P(table), cols, 30, P(ids), 8, 1.0,
                                                       P(loss), P(lse), *to[0], *to[1], P(scratch), 1 << 28, stream)
            check(rows, cols, want[part])


@ALL
def test_scratch_is_written_before_it_is_read(dtype):
    """C calls whose scratch holds NaN (bytes of 255) or zeros give the same bits; without tokens or rows, gradients of zeros."""
    lib, g, code = w.lib, gen(48), {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}[dtype]
    stream = torch.cuda.current_stream().cuda_stream
    room = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    P = lambda t: t.data_ptr()  # noqa: E731

    def both(call, *shapes):
        got = []
        for fill in (0, 255):
            room.fill_(fill)
            out = [torch.full(s, 7.0, dtype=t, device="cuda") for s, t in shapes]
            assert not call(*out), w.last_error()
            got.append(out)
        for a, b in zip(*got):
            assert torch.equal(a, b)
        return got[0]

    for tokens, vocabulary, cols in ((0, 300, 72), (0, 9, 5), (1, 300, 72), (20, 40, 24), (90, 300, 72), (700, 2000, 136)):
        say("scratch", tokens, vocabulary, cols, dtype)
        x, table, dloss = randn(g, tokens, cols).to(dtype), randn(g, vocabulary, cols).to(dtype), randn(g, tokens)
        for kept in (True, False):
            ids = torch.randint(-1, vocabulary, (tokens,), generator=g, device="cuda") if kept else torch.full((tokens,), -1).cuda()
            loss, lse = both(lambda a, b: lib.warp_cross_entropy(P(x), cols, tokens, cols, code, P(table), cols, vocabulary, P(ids),
                                                                 8, 0.1, P(a), P(b), P(room), 1 << 26, stream),
                             ((tokens,), torch.float32), ((tokens,), torch.float32))
            dh, dt = both(lambda a, b: lib.warp_cross_entropy_backward(
                P(dloss), P(x), cols, tokens, cols, code, P(table), cols, vocabulary, P(ids), 8, 0.1, P(loss), P(lse), P(a), cols, P(b),
                cols, P(room), 1 << 26, stream), ((tokens, cols), dtype), ((vocabulary, cols), dtype))
            de, = both(lambda a: lib.warp_embedding_backward(P(x), cols, P(ids), 8, tokens, vocabulary, cols, code, 1.0, P(a), cols,
                                                             P(room), 1 << 26, stream), ((vocabulary, cols), dtype))
            if not tokens or not kept:
                assert not dh.any() and not dt.any() and not de.any()
        dy, q = randn(g, tokens, vocabulary).to(dtype), w.quantize_rows(x)
        both(lambda a: lib.warp_linear(P(x), cols, tokens, cols, code, P(table), cols, vocabulary, None, 0, P(a), vocabulary, P(room),
                                       1 << 26, stream), ((tokens, vocabulary), dtype))
        dx, dw, db = both(lambda a, b, c: lib.warp_linear_backward(
            P(dy), vocabulary, tokens, vocabulary, code, P(q.values), q.values.stride(0), P(q.scale), cols, P(table), cols, P(a), cols,
            P(b), cols, P(c), code, P(room), 1 << 26, stream), ((tokens, cols), dtype), ((vocabulary, cols), dtype), ((vocabulary,), dtype))
        assert tokens or not (dw.any() or db.any())


def differentiable(g):
    """Calls that autograd follows, and their differentiable inputs."""
    ids = torch.randint(-1, 30, (8,), generator=g, device="cuda")
    x, table, weight = (randn(g, n, 16) for n in (8, 30, 24))
    return {"embedding": (lambda t: w.embedding(ids, t, 2.0), [table]),
            "layer_norm": (lambda a, b, c: w.layer_norm(a, b, c)[0], [x, randn(g, 16), randn(g, 16)]),
            "linear": (lambda a, b, c: w.linear(a, b, c), [x, weight, randn(g, 24)]),
            "cross_entropy": (lambda a, b: w.cross_entropy(a, b, ids, 0.1)[0], [x, table])}


@pytest.mark.parametrize("name", ["embedding", "layer_norm", "linear", "cross_entropy"])
def test_forward_mode_is_refused(name):
    """A tangent is refused and not dropped, whichever input has it, with gradients off too; without one nothing is."""
    from torch.autograd import forward_ad

    call, inputs = differentiable(gen(70))[name]
    want = call(*inputs)
    with forward_ad.dual_level():
        assert torch.equal(call(*inputs), want)
        for i, t in enumerate(inputs):
            args = list(inputs)
            args[i] = forward_ad.make_dual(t, torch.ones_like(t))
            with pytest.raises(NotImplementedError):
                call(*args)
            with torch.no_grad(), pytest.raises(NotImplementedError):
                call(*args)
    leaves = [t.clone().requires_grad_() for t in inputs]
    out = call(*leaves)
    with forward_ad.dual_level(), pytest.raises(NotImplementedError):
        torch.autograd.grad(out, leaves, forward_ad.make_dual(torch.ones_like(out), torch.ones_like(out)), retain_graph=True)
    assert all(t is not None for t in torch.autograd.grad(out, leaves, torch.ones_like(out)))


@pytest.mark.parametrize("grads", [False, True])
@pytest.mark.parametrize("name", ["embedding", "layer_norm", "linear", "cross_entropy"])
def test_traced_calls_follow_their_inputs(name, grads):
    """What torch.jit.trace recorded gives other inputs' results, and their gradients."""
    call, inputs = differentiable(gen(71))[name]
    traced = torch.jit.trace(lambda *a: call(*a) * 2.0, tuple(t.clone().requires_grad_(grads) for t in inputs))
    others = [(t * 0.5 + 0.25).requires_grad_(grads) for t in inputs]
    for _ in range(3):  # the executor rewrites a graph in its first runs
        got, want = traced(*others), call(*others) * 2.0
        assert torch.equal(got, want)
        if grads:
            for a, b in zip(torch.autograd.grad(got.sum(), others), torch.autograd.grad(want.sum(), others)):
                assert torch.equal(a, b)


def test_traced_tokens_and_targets_are_inputs():
    g = gen(72)
    table, ids = randn(g, 30, 16), torch.randint(-1, 30, (2, 8), generator=g, device="cuda")

    def call(i, y):
        return w.cross_entropy(w.embedding(i, table), table, y, 0.5)

    traced = torch.jit.trace(call, (ids[0], ids[1]))
    for i, y in ((ids[1], ids[0]), (ids[0, :5], ids[1, 3:])):
        for a, b in zip(traced(i, y), call(i, y)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [130, 500])
def test_float32_products_of_full_mantissas(rows):
    """Elements with 24 bits set, of either sign, in results of one to eight products, on both sides of the number of rows from which on
    operands go in planes: each of the six products of planes is above the bound where it is left out, (1, 1), (0, 2) and (2, 0), the
    smallest, for half of all pairs."""
    g = gen(80 + rows)

    def full(*shape):
        m = (torch.randint(2 ** 23, 2 ** 24, shape, generator=g, device="cuda") | 1).float() * 2.0 ** -23
        return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.5, -m, m)

    def bound(a, b, k):  # of sums whose other products are zeros, which round nothing
        sizes = a.double().abs() @ b.double().abs()
        return (12 * k + 2) * U * sizes + rounding(a.double() @ b.double(), torch.float32)

    for k in (1, 2, 3, 8):
        say("full mantissas", rows, k)
        x, weight = full(rows, k), full(70, k)
        for by in (1.0, 2.0 ** 110, 2.0 ** -100):
            close(w.linear(x * by, weight), (x * by).double() @ weight.double().t(), bound(x * by, weight.t(), k), ("y", k, by))
        dy, weight = full(rows, k), full(k, 72)
        dx, _, _ = w.linear_backward(dy, w.quantize_rows(full(rows, 72)), weight)
        close(dx, dy.double() @ weight.double(), bound(dy, weight, k), ("dx", k))
        dy, kept = full(rows, 70), w.quantize_rows(full(rows, 72))
        dy[torch.randperm(rows, generator=g, device="cuda")[k:]] = 0.0
        _, dw, _ = w.linear_backward(dy, kept, full(70, 72))
        back = kept.values[:, :72].double() * kept.scale.double()[:, None]  # rounded to float32 once
        close(dw, dy.double().t() @ back, bound(dy.t(), back, k) + U * (dy.double().abs().t() @ back.abs()), ("dweight", k))
        # a vocabulary of one: lse is the logit; its factor, the product with it, and back from units of log 2
        table = full(1, k)
        loss, lse = w.cross_entropy(x, table, torch.zeros(rows, dtype=torch.int64, device="cuda"), 0.5)
        want = 0.5 * (x.double() @ table.double().t())
        close(lse[:, None], want, 0.5 * bound(x, table.t(), k) + 8 * U * want.abs(), ("lse", k))
        assert not loss.any()


@pytest.mark.parametrize("name", ["embedding", "linear", "cross_entropy", "layer_norm"])
def test_captured_backward_of_cast_leaves_in_use(name):
    """The same where a leaf of 32 bits is cast for the call, as master weights are: refused while an eager graph of it lives, then
    captured, and replays give what eager passes give."""
    g = gen(61)
    leaf = randn(g, 97, 64).requires_grad_() if name != "layer_norm" else (1 + 0.1 * randn(g, 64)).requires_grad_()
    x, ids = randn(g, 70, 64).bfloat16(), torch.randint(-1, 97, (70,), generator=g, device="cuda")
    call = {"embedding": lambda t: w.embedding(ids, t), "linear": lambda t: w.linear(x, t),
            "cross_entropy": lambda t: w.cross_entropy(x, t, ids)[0], "layer_norm": lambda t: w.layer_norm(x, t)[0]}[name]
    out = lambda: call(leaf.to(torch.bfloat16)).float()  # noqa: E731
    dy = torch.randn(out().shape, generator=g, device="cuda")
    lives = out()
    torch.cuda.synchronize()
    say("refused capture of a cast leaf:", name)
    with pytest.raises(RuntimeError, match="cannot be captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            out().backward(dy)
    assert leaf.grad is None
    lives.backward(dy)
    assert leaf.grad is not None
    leaf.grad = None
    del lives
    gc.collect()
    torch.cuda.synchronize()
    say("capture of a cast leaf:", name)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out().backward(dy)
    got = leaf.grad
    for k in range(3):
        x.copy_(randn(g, 70, 64))
        dy.copy_(torch.randn(dy.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.no_grad():
            kept = got.clone()
        assert torch.equal(kept, torch.autograd.grad(out(), leaf, dy)[0]), k
