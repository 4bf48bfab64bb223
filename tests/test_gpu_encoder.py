"""The operators of the token encoder's head against their definitions in 64 bits (run on an MI355X).

Bounds. The kernels compute in fp32 (unit roundoff U = 2^-24) and round once to the output's type (half an
ulp: 2^-9 of a bfloat16, 2^-12 of a float16 relative to the power of two above, here 2^-11 of the value, plus
its subnormal step). A sum of n products in a chain of d roundings is within d U sum |terms| of its value; a
row's sums have chains of at most 32 elements of a lane, 6 steps over lanes and 16 over waves: d <= 64 with
room. Errors of intermediate values are carried through the formulas element by element below.
"""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
w = pytest.importorskip("paper_2501_17788_amd")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CHAIN = 64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # relative, with room
STEP = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def f64(t):
    return t.detach().double().cpu()


def rounding(t, dtype):
    """Bound of rounding the 64-bit values t once to dtype (nothing for float32: its roundings are counted)."""
    return torch.zeros_like(t) if dtype == torch.float32 else HALF[dtype] * t.abs() + STEP[dtype]


def close(got, want, tol, what):
    got, want = f64(got), want
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= tol)
    if bad.any():
        i = torch.nonzero(bad.reshape(-1))[0].item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values are off, the first at {i}: "
                             f"{got.reshape(-1)[i].item()!r} for {want.reshape(-1)[i].item()!r}, bound "
                             f"{tol.expand_as(want).reshape(-1)[i].item():.3g}")


# ---------------------------------------------------------------------------- layer norm

class Norm64:
    """Layer norm in 64 bits, with bounds of the kernels' errors."""

    def __init__(self, x, weight, bias, eps):
        self.x = f64(x)
        n = self.x.shape[-1]
        self.w = f64(weight) if weight is not None else torch.ones(n, dtype=torch.float64)
        self.b = f64(bias) if bias is not None else torch.zeros(n, dtype=torch.float64)
        self.mean = self.x.mean(-1, keepdim=True)
        d = self.x - self.mean
        self.rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
        self.h = d * self.rstd
        self.y = self.h * self.w + self.b
        # the mean's error, and with it those of x - mean, of the variance (relative) and of h
        self.e_mean = CHAIN * U * self.x.abs().mean(-1, keepdim=True)
        e_d = self.e_mean + U * d.abs()
        e_var = CHAIN * U + 2 * (d.abs() * e_d).mean(-1, keepdim=True) * self.rstd ** 2
        self.e_rstd = self.rstd * (0.5 * e_var + 4 * U)
        self.e_h = self.rstd * e_d + self.h.abs() * (0.5 * e_var + 6 * U)
        self.e_y = self.w.abs() * (self.e_h + U * self.h.abs()) + 2 * U * (self.y.abs() + self.b.abs())

    def backward(self, dy, rows_chain):
        dy = f64(dy)
        c = dy * self.w
        s1, s2 = c.mean(-1, keepdim=True), (c * self.h).mean(-1, keepdim=True)
        dx = self.rstd * (c - s1 - self.h * s2)
        e_s1 = CHAIN * U * c.abs().mean(-1, keepdim=True)
        e_s2 = CHAIN * U * (c * self.h).abs().mean(-1, keepdim=True) + (c.abs() * self.e_h).mean(-1, keepdim=True)
        inner = 4 * U * (c.abs() + s1.abs() + (self.h * s2).abs()) + e_s1 + self.h.abs() * e_s2 + self.e_h * s2.abs()
        e_dx = self.rstd * inner + (self.e_rstd + 2 * U * self.rstd) * (dx / self.rstd).abs()
        flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        terms, dyf = flat(dy * self.h), flat(dy)
        e_dw = flat(dy.abs() * self.e_h).sum(0) + rows_chain * U * terms.abs().sum(0)
        return (dx, e_dx), (terms.sum(0), e_dw), (dyf.sum(0), rows_chain * U * dyf.abs().sum(0))


def hidden(g, rows, cols, dtype, offset=0.5):
    spread = torch.exp(0.5 * randn(g, cols))
    return (randn(g, rows, cols) * spread + offset * randn(g, cols)).to(dtype)


# a lane's vectors hold 8 (or 4) elements and a wave's 512 (256): both sides of each limit, single columns and rows
COLS = [1, 2, 3, 5, 7, 8, 9, 63, 64, 65, 127, 128, 255, 257, 511, 512, 513, 771, 1023, 1024, 1025, 2047, 2048, 2049,
        4096, 4099, 8191, 8192, 8193, 16383, 16384]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", list(TYPES), ids=list(TYPES))
def test_layer_norm_and_gradients(cols, dtype):
    t = TYPES[dtype]
    g = gen(cols)
    for rows, params in ((1, torch.float32), (5, t), (37, torch.float32)):
        say(f"layer norm {rows} x {cols} {dtype}, params {params}")
        x = hidden(g, rows, cols, t)
        weight, bias = (1 + 0.2 * randn(g, cols)).to(params), (0.2 * randn(g, cols)).to(params)
        dy = randn(g, rows, cols).to(t)
        y, mean, rstd = w.layer_norm(x, weight, bias, 1e-5)
        dx, dw, db = w.layer_norm_backward(dy, x, weight, mean, rstd)
        assert y.dtype == dx.dtype == t and dw.dtype == db.dtype == params and mean.dtype == torch.float32
        r = Norm64(x, weight, bias, 1e-5)
        close(y, r.y, r.e_y + rounding(r.y, t), "y")
        close(mean, r.mean[:, 0], r.e_mean[:, 0] + U * r.mean[:, 0].abs(), "mean")
        close(rstd, r.rstd[:, 0], r.e_rstd[:, 0], "rstd")
        (rdx, e_dx), (rdw, e_dw), (rdb, e_db) = r.backward(dy, CHAIN)
        close(dx, rdx, e_dx + rounding(rdx, t), "dx")
        close(dw, rdw, e_dw + rounding(rdw, params), "dweight")
        close(db, rdb, e_db + rounding(rdb, params), "dbias")


@pytest.mark.parametrize("rows,cols", [(4099, 96), (2500, 1027), (70_001, 8), (600, 8200)])
def test_layer_norm_of_many_rows(rows, cols):
    """More rows than the grid has places for: every workgroup takes several."""
    g = gen(rows)
    x, dy = hidden(g, rows, cols, torch.bfloat16), randn(g, rows, cols).bfloat16()
    weight = 1 + 0.2 * randn(g, cols)
    y, mean, rstd = w.layer_norm(x, weight, None)
    dx, dw, db = w.layer_norm_backward(dy, x, weight, mean, rstd)
    r = Norm64(x, weight, None, 1e-5)
    (rdx, e_dx), (rdw, e_dw), (rdb, e_db) = r.backward(dy, CHAIN + rows // 256)
    close(y, r.y, r.e_y + rounding(r.y, y.dtype), "y")
    close(dx, rdx, e_dx + rounding(rdx, y.dtype), "dx")
    close(dw, rdw, e_dw, "dweight")
    close(db, rdb, e_db, "dbias")
    again = w.layer_norm_backward(dy, x, weight, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again)), "the same call twice"


@pytest.mark.parametrize("dtype", list(TYPES), ids=list(TYPES))
@pytest.mark.parametrize("cols", [1, 6, 8, 100, 777, 2056])
def test_layer_norm_strides_and_alignment(cols, dtype):
    """Rows cut from a wider tensor, at every alignment of their start, and leading dimensions."""
    t = TYPES[dtype]
    g = gen(3)
    wide = hidden(g, 6, cols + 13, t)
    grads = randn(g, 6, cols + 13).to(t)
    for at in (0, 1, 3, 8):
        x, dy = wide[:, at:at + cols], grads[:, 13 - at:13 - at + cols]
        y, mean, rstd = w.layer_norm(x)
        dx, dw, db = w.layer_norm_backward(dy, x, None, mean, rstd)
        cx, cdy = x.contiguous(), dy.contiguous()
        y2, mean2, rstd2 = w.layer_norm(cx)
        same = (y, mean, rstd, dx, dw, db)
        for a, b in zip(same, (y2, mean2, rstd2, *w.layer_norm_backward(cdy, cx, None, mean2, rstd2))):
            assert torch.equal(a, b), (cols, at)
        q, q2 = w.layer_norm_int8(x), w.layer_norm_int8(cx)
        assert torch.equal(q.values, q2.values) and torch.equal(q.scale, q2.scale)
    cube = hidden(g, 6, cols, t).view(2, 3, cols)
    y, mean, rstd = w.layer_norm(cube)
    assert y.shape == cube.shape and mean.shape == rstd.shape == (2, 3)
    assert torch.equal(y.view(6, cols), w.layer_norm(cube.view(6, cols))[0])
    turned = cube.transpose(0, 1)  # rows of another order
    assert torch.equal(w.layer_norm(turned)[0], y.transpose(0, 1))
    line = cube[0, 0]
    assert torch.equal(w.layer_norm(line)[0], y[0, 0])


def test_layer_norm_writes_only_its_rows():
    g = gen(9)
    from paper_2501_17788_amd import lib

    for cols in (5, 8, 100, 771, 2100):
        out = torch.full((4, cols + 24), 7.0, device="cuda")
        x = hidden(g, 4, cols, torch.float32)
        rc = lib.warp_layer_norm(x.data_ptr(), cols, 4, cols, 0, None, None, 0, 1e-5, out[0, 8:].data_ptr(), cols + 24,
                                 None, None, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        assert torch.equal(out[:, 8:8 + cols], w.layer_norm(x)[0])
        assert (out[:, :8] == 7).all() and (out[:, 8 + cols:] == 7).all()


def test_layer_norm_in_place():
    g = gen(10)
    from paper_2501_17788_amd import lib

    for cols in (8, 100, 771, 3000, 5001, 9001):
        x = hidden(g, 9, cols, torch.bfloat16)
        want = w.layer_norm(x)[0]
        assert lib.warp_layer_norm(x.data_ptr(), cols, 9, cols, 2, None, None, 0, 1e-5, x.data_ptr(), cols, None, None,
                                   torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(x, want), cols


def test_layer_norm_hard_values():
    """Rows far from zero, constant rows (eps alone), huge and tiny values, a NaN and infinities in one row."""
    g = gen(4)
    for cols in (64, 300, 5000):
        x = randn(g, 8, cols)
        x[0] = x[0] * 1e-3 + 1000
        x[1] = 3.5
        x[2] *= 1e15
        x[3] *= 1e-18
        x[4] = 0
        y, mean, rstd = w.layer_norm(x, None, None, 1e-5)
        r = Norm64(x, None, None, 1e-5)
        close(y, r.y, r.e_y + U * (r.mean.abs() * r.rstd), "y")
        assert (y[4] == 0).all()
        x[6, cols // 2] = float("nan")
        x[7, 3], x[7, 5] = float("inf"), float("-inf")
        again = w.layer_norm(x)[0]
        assert torch.equal(again[:6], w.layer_norm(x[:6])[0])
        assert again[6:].isnan().all()
        dy = randn(g, 8, cols)
        dx = w.layer_norm_backward(dy, x, None, *w.layer_norm(x)[1:])[0]
        assert dx[:6].isfinite().all() and dx[6:].isnan().all()


def test_layer_norm_gradients_against_differences():
    """Central differences of sum(dy * y) in 64 bits. Their own error is h^2 / 6 of a third derivative of a few
    units (h = 1e-4) and 1e-16 / h of rounding: 1e-7 bounds both."""
    g = gen(5)
    rows, cols, h = 3, 11, 1e-4
    x, dy = randn(g, rows, cols), randn(g, rows, cols)
    weight, bias = 1 + 0.2 * randn(g, cols), 0.2 * randn(g, cols)
    _, mean, rstd = w.layer_norm(x, weight, bias)
    dx, dw, db = (f64(t) for t in w.layer_norm_backward(dy, x, weight, mean, rstd))
    x64, w64, b64, dy64 = f64(x), f64(weight), f64(bias), f64(dy)

    def loss(x, weight, bias):
        d = x - x.mean(1, keepdim=True)
        return (dy64 * (d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * weight + bias)).sum()

    def slope(i, at):
        args = [x64, w64, b64]
        up, down = args[i].clone(), args[i].clone()
        up.view(-1)[at] += h
        down.view(-1)[at] -= h
        return (loss(*args[:i], up, *args[i + 1:]) - loss(*args[:i], down, *args[i + 1:])) / (2 * h)

    r = Norm64(x, weight, bias, 1e-5)
    bounds = [e for _, e in r.backward(dy, CHAIN)]
    for i, (got, e) in enumerate(zip((dx, dw, db), bounds)):
        want = torch.stack([slope(i, at) for at in range(got.numel())]).view_as(got)
        assert ((got - want).abs() <= e + 1e-7 * (1 + want.abs())).all(), i


def test_layer_norm_of_no_rows():
    x = torch.empty(0, 40, device="cuda")
    y, mean, rstd = w.layer_norm(x)
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = w.layer_norm_backward(x, x, torch.ones(40, device="cuda"), mean, rstd)
    assert dx.shape == (0, 40) and (dw == 0).all() and (db == 0).all() and dw.shape == (40,)
    q = w.layer_norm_int8(x)
    assert q.values.shape == (0, 128) and w.quantize_rows(x).scale.shape == (0,)
    assert w.linear_int8(q, w.quantize_rows(torch.ones(3, 40, device="cuda"))).shape == (0, 3)


# ---------------------------------------------------------------------------- 8-bit rows and their products

def quantised(x):
    """The definition's whole numbers and scales, in fp32 operations one by one."""
    x = x.detach().float().cpu().numpy()
    top = np.abs(x).max(1)
    some = (top >= 2.0 ** -120) & np.isfinite(top)
    with np.errstate(all="ignore"):
        f = np.where(some, np.float32(127) / top, np.float32(0)).astype(np.float32)
        q = np.where(some[:, None], np.rint(x * f[:, None]), 0).astype(np.int8)
    return q, np.where(np.isfinite(top), top * np.float32(1.0 / 127.0), np.float32(np.nan)).astype(np.float32)


@pytest.mark.parametrize("dtype", list(TYPES), ids=list(TYPES))
def test_quantize_rows(dtype):
    t = TYPES[dtype]
    g = gen(6)
    for cols in COLS:
        for rows in (1, 9):
            x = hidden(g, rows, cols, t)
            if rows == 9:
                x[2] = 0
                x[3] *= 2.0 ** -10
                x[4] = x[4].abs().max()
                x[5, cols // 2] = float("nan")
                x[6, cols - 1] = float("-inf")
                if t != torch.float16:
                    x[7] *= 2.0 ** -125
            r = w.quantize_rows(x)
            q, scale = quantised(x)
            assert r.cols == cols and r.values.shape[1] % 128 == 0
            np.testing.assert_array_equal(r.values[:, :cols].cpu().numpy(), q, err_msg=f"{rows} x {cols}")
            assert not r.values[:, cols:].any()
            np.testing.assert_array_equal(r.scale.cpu().numpy(), scale)


@pytest.mark.parametrize("cols", COLS)
def test_layer_norm_int8(cols):
    """Within half a step of the 64-bit norm, plus what its values and the factor 127 / max are off."""
    g = gen(cols)
    for t in TYPES.values():
        x = hidden(g, 7, cols, t)
        weight, bias = 1 + 0.2 * randn(g, cols), 0.2 * randn(g, cols)
        q = w.layer_norm_int8(x, weight, bias)
        r = Norm64(x, weight, bias, 1e-5)
        scale = f64(q.scale)[:, None]
        top = r.y.abs().amax(1, keepdim=True)
        assert ((scale * 127 - top).abs() <= r.e_y.amax(1, keepdim=True) + 4 * U * top).all()
        got = f64(q.values[:, :cols]) * scale
        off = scale * 0.5 + r.e_y + r.e_y.amax(1, keepdim=True) + 8 * U * top
        assert ((got - r.y).abs() <= off).all() and not q.values[:, cols:].any()


def int8_rows(g, rows, cols, full=False):
    v = torch.randint(-127, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
    if full:
        v = torch.where(v < 0, -127, 127).to(torch.int8)
    return v, torch.rand(rows, generator=g, device="cuda") * 0.02 + 1e-4


def product(a, sa, b, sb, bias):
    """(value, bound of the fp32 epilogue: the sum's conversion, two products and the bias)."""
    acc = (a.cpu().double() @ b.cpu().double().t())  # exact: below 2^53
    scaled = acc * f64(sb) * f64(sa)[:, None]
    out = scaled + (f64(bias) if bias is not None else 0)
    return out, 4 * U * scaled.abs() + U * out.abs()


# one token, a query's tokens, both sides of the tile sizes; channels and columns of every kind
@pytest.mark.parametrize("rows", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 400])
def test_linear_int8(rows):
    g = gen(rows)
    for n, cols in ((1, 1), (3, 64), (16, 127), (17, 128), (128, 129), (100, 771), (128, 768), (255, 1024),
                    (257, 300), (1030, 513), (640, 4096)):
        a, sa = int8_rows(g, rows, cols)
        b, sb = int8_rows(g, n, cols)
        bias = randn(g, n) if n % 2 else None
        qa, qb = w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb)
        want, tol = product(a, sa, b, sb, bias)
        for t in TYPES.values():
            out = w.linear_int8(qa, qb, bias, t)
            assert out.dtype == t
            close(out, want, tol + rounding(want, t), f"{rows} x {cols} by {n} {t}")


@pytest.mark.parametrize("rows,n,cols", [(2000, 1003, 771), (1025, 2049, 1000), (4096, 512, 256), (300, 5000, 640),
                                         (33_000, 128, 192), (1, 9001, 2500), (64, 4096, 9000),
                                         (1990, 3999, 530), (2040, 4000, 100), (4090, 4083, 900), (5000, 3900, 1100),
                                         (4081, 4096, 65)])
def test_linear_int8_larger(rows, n, cols):
    g = gen(n)
    a, sa = int8_rows(g, rows, cols)
    b, sb = int8_rows(g, n, cols)
    bias = randn(g, n)
    qa, qb = w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb)
    acc = a.double() @ b.double().t()  # exact, on the GPU in 64 bits
    scaled = acc * sb.double() * sa.double()[:, None]
    want = scaled + bias.double()
    for t in (torch.float32, torch.bfloat16):
        out = w.linear_int8(qa, qb, bias, t)
        tol = 4 * U * scaled.abs() + U * want.abs() + rounding(want, t)
        bad = ~((out.double() - want).abs() <= tol)
        assert not bad.any(), (rows, n, cols, t, int(bad.sum()))


@pytest.mark.parametrize("rows,n,cols", [(1, 16_384, 300), (1, 16_385, 300), (16, 16_384, 1000), (17, 8192, 129),
                                         (5, 10_007, 4096), (16_384, 16, 129), (16_001, 1, 2000), (10_001, 15, 1025),
                                         (500, 512, 1024), (500, 509, 1025), (33, 4999, 2048)])
def test_linear_int8_one_side_short(rows, n, cols):
    """Few tokens by many channels and the reverse, and the sizes where one kind of tiles gives way to the next."""
    g = gen(rows + n)
    a, sa = int8_rows(g, rows, cols)
    b, sb = int8_rows(g, n, cols)
    qa, qb = w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb)
    for bias in (None, randn(g, n)):
        want, tol = product(a, sa, b, sb, bias)
        for t in TYPES.values():
            close(w.linear_int8(qa, qb, bias, t), want, tol + rounding(want, t), f"{rows} x {cols} by {n} {t}")


def test_linear_int8_longest_sum():
    """k at its limit with every product at its largest: the sums need all 32 bits."""
    g = gen(1)
    cols = 131_071
    a, sa = int8_rows(g, 3, cols, full=True)
    b, sb = int8_rows(g, 18, cols, full=True)
    a[0], b[0], b[1] = 127, 127, -127
    want, tol = product(a, sa, b, sb, None)
    out = w.linear_int8(w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb), None, torch.float32)
    close(out, want, tol, "longest")


def test_linear_int8_strides_and_bounds():
    """Operands cut from wider rows; an output inside a larger one keeps what lies around it."""
    from paper_2501_17788_amd import lib

    g = gen(2)
    for rows, n, cols in ((5, 20, 100), (70, 130, 256), (300, 257, 400)):
        pad = -(-cols // 128) * 128
        a, sa = int8_rows(g, rows, cols)
        b, sb = int8_rows(g, n, cols)
        wide_a = torch.full((rows, pad + 48), 99, dtype=torch.int8, device="cuda")
        wide_b = torch.full((n, pad + 16), -99, dtype=torch.int8, device="cuda")
        for wide, v in ((wide_a, a), (wide_b, b)):
            wide[:, 16:16 + pad if wide is wide_a else 16 + pad] = 0
            wide[:, 16:16 + cols] = v
        want = w.linear_int8(w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb), None, torch.float32)
        out = torch.full((rows + 2, n + 9), 5.0, device="cuda")
        rc = lib.warp_linear_int8(wide_a[:, 16:].data_ptr(), wide_a.stride(0), sa.data_ptr(), rows,
                                  wide_b[:, 16:].data_ptr(), wide_b.stride(0), sb.data_ptr(), n, cols, None,
                                  out[1, 3:].data_ptr(), n + 9, 0, torch.cuda.current_stream().cuda_stream)
        assert rc == 0, w.last_error()
        assert torch.equal(out[1:-1, 3:3 + n], want)
        out[1:-1, 3:3 + n] = 5.0
        assert (out == 5).all()


def test_linear_int8_of_a_spoilt_row():
    g = gen(8)
    x = randn(g, 40, 200)
    x[7, 3] = float("nan")
    x[9, 0] = float("inf")
    out = w.linear_int8(w.quantize_rows(x), w.quantize_rows(randn(g, 70, 200)))
    spoilt = out.isnan().all(1)
    assert spoilt[7] and spoilt[9] and int(spoilt.sum()) == 2 and out[~spoilt].isfinite().all()


# ---------------------------------------------------------------------------- AdamW

LR, B1, B2, EPS, DECAY = 1e-2, 0.9, 0.999, 1e-8, 0.1


def reference_step(p, g, m, v, t):
    """(p, m, v) in 64 bits with bounds of the kernel's errors; the constants too are rounded to fp32."""
    m1 = B1 * m + (1 - B1) * g
    v1 = B2 * v + (1 - B2) * g * g
    e_m = 3 * U * (abs(B1 * m) + abs((1 - B1) * g))
    e_v = 4 * U * v1
    denom = np.sqrt(v1) / np.sqrt(1 - B2 ** t) + EPS
    move = LR / (1 - B1 ** t) * m1 / denom
    p1 = p * (1 - LR * DECAY) - move
    e_p = 3 * U * (abs(p) + abs(p1)) + LR / (1 - B1 ** t) * e_m / denom + 12 * U * abs(move)
    return (p1, e_p), (m1, e_m), (v1, e_v)


SIZES = [1, 2, 3, 7, 8, 255, 256, 257, 1000, 2047, 2048, 2049, 5000, 0, 40_001]


def tensors(g, sizes, dtype, scale, shift=0):
    """Tensors of these sizes; with `shift` they lie back to back in one, from that element on."""
    if not shift:
        return [(randn(g, n) * scale).to(dtype) for n in sizes]
    flat = (randn(g, sum(sizes) + shift) * scale).to(dtype)
    out = []
    for n in sizes:
        out.append(flat[shift:shift + n])
        shift += n
    return out


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "packed"])
@pytest.mark.parametrize("grads", list(TYPES), ids=list(TYPES))
@pytest.mark.parametrize("params", list(TYPES), ids=list(TYPES))
def test_adamw_32(params, grads, shift):
    g = gen(11)
    pt = TYPES[params]
    p = tensors(g, SIZES, pt, 1.0, shift)
    opt = w.AdamW(p, LR, (B1, B2), EPS, DECAY)
    m = [np.zeros(n) for n in SIZES]
    v = [np.zeros(n) for n in SIZES]
    e_m, e_v = [0 * x for x in m], [0 * x for x in v]
    for t in range(1, 4):
        grad = tensors(g, SIZES, TYPES[grads], 10.0 ** -t, shift)
        before = [f64(x).numpy() for x in p]
        say(f"adamw 32 {params} {grads} step {t}")
        opt.step(grad)
        fm, fv = (f64(x).numpy() for x in opt.moments())
        at = 0
        for i, n in enumerate(SIZES):
            gi = f64(grad[i]).numpy()
            (p1, e_p), (m1, d_m), (v1, d_v) = reference_step(before[i], gi, m[i], v[i], t)
            # the moments' own errors so far are carried along
            e_m[i], e_v[i] = B1 * e_m[i] + d_m, B2 * e_v[i] + d_v
            assert (abs(fm[at:at + n] - m1) <= e_m[i]).all() and (abs(fv[at:at + n] - v1) <= e_v[i]).all()
            with np.errstate(invalid="ignore"):
                share = np.where(v1 > 0, e_v[i] / np.maximum(v1, 1e-300), 0)
            denom = np.sqrt(v1) / np.sqrt(1 - B2 ** t) + EPS
            e_p = e_p + LR / (1 - B1 ** t) * (e_m[i] + abs(m1) * share) / denom
            tol = e_p + rounding(torch.from_numpy(p1), pt).numpy()
            assert (abs(f64(p[i]).numpy() - p1) <= tol).all(), (i, n, t)
            m[i], v[i] = m1, v1
            assert not fm[at + n:at + -(-n // 256) * 256].any()
            at += -(-n // 256) * 256


def cutoffs(levels, power):
    t = (np.arange(1, levels + 1, dtype=np.float32) - np.float32(0.5)) * np.float32(1 / levels)
    t = t * t
    return t * t if power == 4 else t


def coded(x, levels, power):
    """Codes and scales of fp32 moments by the definition, in fp32 operations."""
    b = np.zeros(-(-len(x) // 256) * 256, np.float32)
    b[:len(x)] = x
    b = b.reshape(-1, 256)
    top = np.maximum(np.abs(b).max(1), np.float32(2.0 ** -126)).astype(np.float32)
    c = np.searchsorted(cutoffs(levels, power), np.abs(b) * (np.float32(1) / top)[:, None], side="right")
    if power == 4:
        c = np.maximum(c, b > 0)
    return (np.where(b < 0, -c, c).reshape(-1), top)


def values(c, top, levels, power):
    t = np.abs(c).astype(np.float32) * np.float32(1 / levels)
    t = t * t
    t = t * t if power == 4 else t
    return (np.where(c < 0, -t, t).reshape(-1, 256) * top[:, None]).reshape(-1).astype(np.float32)


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "packed"])
@pytest.mark.parametrize("grads", list(TYPES), ids=list(TYPES))
@pytest.mark.parametrize("params", list(TYPES), ids=list(TYPES))
def test_adamw_8(params, grads, shift):
    """Codes and scales equal those of the definition's fp32 operations, step after step."""
    g = gen(12)
    pt = TYPES[params]
    p = tensors(g, SIZES, pt, 1.0, shift)
    opt = w.AdamW(p, LR, (B1, B2), EPS, DECAY, bits=8)
    f = np.float32
    m = [np.zeros(n, f) for n in SIZES]
    v = [np.zeros(n, f) for n in SIZES]
    for t in range(1, 5):
        spread = [torch.exp(3 * randn(g, n)) for n in SIZES]
        grad = [(a.float() * s).to(a.dtype).clamp(-60000, 60000) if not shift else a
                for a, s in zip(tensors(g, SIZES, TYPES[grads], 10.0 ** -t, shift), spread)]
        before = [f64(x).numpy() for x in p]
        say(f"adamw 8 {params} {grads} step {t}")
        opt.step(grad)
        cm, cv = opt.m.cpu().numpy().astype(np.int32), opt.v.cpu().numpy().astype(np.int32)
        sm, sv = opt.m_scale.cpu().numpy(), opt.v_scale.cpu().numpy()
        fm, fv = (x.cpu().numpy() for x in opt.moments())
        at = 0
        for i, n in enumerate(SIZES):
            gi = grad[i].float().cpu().numpy()
            (p1, e_p), _, _ = reference_step(before[i], gi.astype(np.float64), m[i].astype(np.float64),
                                             v[i].astype(np.float64), t)
            tol = e_p + rounding(torch.from_numpy(p1), pt).numpy()
            assert (abs(f64(p[i]).numpy() - p1) <= tol).all(), (i, n, t)
            m32 = m[i] * f(B1) + gi * f(1 - B1)
            v32 = v[i] * f(B2) + (gi * gi) * f(1 - B2)
            room = -(-n // 256) * 256
            for codes, scales, flat, x, levels, power, keep in ((cm, sm, fm, m32, 127, 2, m), (cv, sv, fv, v32, 255, 4, v)):
                c, top = coded(x, levels, power)
                np.testing.assert_array_equal(codes[at:at + room], c)
                np.testing.assert_array_equal(scales[at // 256:(at + room) // 256], top)
                val = values(c, top, levels, power)
                np.testing.assert_array_equal(flat[at:at + room], val)
                keep[i] = val[:n]
            at += room


def test_adamw_8_code_boundaries():
    """Magnitudes at, just below and just above every cutoff, and one that is far smaller than its block's largest."""
    f = np.float32
    for levels, power in ((127, 2), (255, 4)):
        cut = cutoffs(levels, power)
        for x in (cut, np.nextafter(cut, f(0)), np.nextafter(cut, f(1))):
            x = x[x < 1]
            g = np.concatenate([[f(1)], x[:254], [f(1e-12)]]).astype(f)
            # one step from zero moments with betas that make the moment the gradient itself (m) or its square (v)
            opt = w.AdamW([torch.zeros(len(g), device="cuda")], bits=8, betas=(0.0, 0.0))
            opt.step([torch.from_numpy(g if power == 2 else np.sqrt(g)).cuda()])
            got = (opt.m if power == 2 else opt.v).cpu().numpy().astype(np.int32)
            value = g if power == 2 else np.sqrt(g) * np.sqrt(g)
            want, top = coded(value, levels, power)
            np.testing.assert_array_equal(got, want)
            assert got[len(g) - 1] == (0 if power == 2 else 1)  # a second moment above zero is not lost


def test_adamw_many_tensors_and_skipped_ones():
    """More tensors than one launch takes; those without a gradient keep their values and moments."""
    g = gen(13)
    sizes = [int(n) for n in np.random.default_rng(0).integers(1, 3000, 203)]
    for bits in (32, 8):
        p = tensors(g, sizes, torch.float32, 1.0)
        alone = [x.clone() for x in p]
        grad = tensors(g, sizes, torch.float32, 0.1)
        skipped = {0, 63, 64, 100, 202}
        opt = w.AdamW(p, LR, (B1, B2), EPS, DECAY, bits)
        for _ in range(2):
            opt.step([None if i in skipped else x for i, x in enumerate(grad)])
        fm = opt.moments()[0]
        at = 0
        for i, n in enumerate(sizes):
            if i in skipped:
                assert torch.equal(p[i], alone[i]) and not fm[at:at + n].any()
            else:
                one = w.AdamW([alone[i]], LR, (B1, B2), EPS, DECAY, bits)
                one.step([grad[i]])
                one.step([grad[i]])
                assert torch.equal(p[i], alone[i]) and torch.equal(one.moments()[0][:n], fm[at:at + n]), i
            at += -(-n // 256) * 256
        opt.step([None] * len(p))
        assert torch.equal(p[0], alone[0]) and opt.steps == 3


def test_adamw_gradient_scale_and_checkpoint():
    g = gen(14)
    for bits in (32, 8):
        p = tensors(g, [700, 33], torch.float32, 1.0)
        q = [x.clone() for x in p]
        grad = tensors(g, [700, 33], torch.float32, 0.1)
        a, b = w.AdamW(p, bits=bits), w.AdamW(q, bits=bits)
        a.step(grad, grad_scale=torch.tensor([0.25], device="cuda"))
        b.step([0.25 * x for x in grad])  # a power of two: the same bits
        assert all(torch.equal(x, y) for x, y in zip(p, q))
        c = w.AdamW([x.clone() for x in p], bits=bits)
        c.load_state_dict(a.state_dict())
        assert c.steps == 1
        a.step(grad)
        c.step(grad)
        assert all(torch.equal(x, y) for x, y in zip(p, c.params)) and torch.equal(a.v, c.v)
        with pytest.raises(ValueError):
            c.load_state_dict(w.AdamW(p, bits=40 - bits).state_dict())


def test_adamw_on_another_stream():
    g = gen(17)
    for bits in (32, 8):
        p = tensors(g, [70_000, 300], torch.float32, 1.0)
        q = [x.clone() for x in p]
        grads = [tensors(g, [70_000, 300], torch.float32, 0.1) for _ in range(3)]
        a, b = w.AdamW(p, bits=bits), w.AdamW(q, bits=bits)
        for x in grads:
            a.step(x)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for x in grads:
            b.step(x, stream=s)
        moments = b.moments(stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(x, y) for x, y in zip(p, q))
        assert all(torch.equal(x, y) for x, y in zip(a.moments(), moments))


def test_adamw_refuses_what_changed_underneath():
    """Parameters, gradients and moments that no longer fit are refused before anything is launched."""
    p = [torch.ones(300, device="cuda"), torch.ones(5, device="cuda")]
    grads = [torch.ones_like(x) for x in p]
    for bits in (32, 8):
        opt = w.AdamW(p, bits=bits)
        before = [x.clone() for x in p]

        def refused(match, *args, **kw):
            with pytest.raises(ValueError, match=match):
                opt.step(*args, **kw)
            assert opt.steps == 0 and all(torch.equal(a, b) for a, b in zip(before, p))

        refused("gradients for", grads[:1])
        refused("gradient 1", [grads[0], grads[1][:4]])
        refused("gradient 0", [torch.ones(600, device="cuda")[::2], grads[1]])
        refused("gradient 1", [grads[0], grads[1].half()])
        refused("gradient 0", [grads[0].cpu(), grads[1]])
        refused("no tensor", [1.0, grads[1]])
        refused("float32, float16", [x.double() for x in grads])
        refused("grad_scale", grads, grad_scale=torch.ones(2, device="cuda"))
        opt.params.append(torch.ones(7, device="cuda"))
        refused("when the optimizer was made", grads + [torch.ones(7, device="cuda")])
        opt.params.pop()
        kept = opt.params[1]
        opt.params[1] = torch.ones(6, device="cuda")
        refused("parameter 1", grads)
        opt.params[1] = kept
        m = opt.m
        opt.m = m[:256]
        refused("moments", grads)
        opt.m = m
        if bits == 8:
            scale, opt.v_scale = opt.v_scale, None
            refused("scales", grads)
            opt.v_scale = scale
        opt.step(grads)
        assert opt.steps == 1 and not torch.equal(before[0], p[0])


def test_adamw_spoilt_gradients():
    """A NaN or an infinity reaches its element (32 bits) or its block's moments (8 bits), no other."""
    for bits in (32, 8):
        for bad in (float("nan"), float("inf")):
            p = [torch.ones(2000, device="cuda")]
            grad = torch.full((2000,), 0.5, device="cuda")
            grad[300] = bad
            opt = w.AdamW(p, bits=bits)
            opt.step([grad])
            assert p[0][300].isnan() and p[0].isnan().sum() == 1
            fm, fv = opt.moments()
            hit = slice(300, 301) if bits == 32 else slice(256, 512)
            assert not fv[hit].isfinite().any()
            rest = torch.ones(2048, dtype=torch.bool, device="cuda")
            rest[hit] = False
            assert fm[rest].isfinite().all() and fv[rest].isfinite().all()


# ---------------------------------------------------------------------------- streams, graphs

def test_calls_on_another_stream():
    """Work on a stream of its own, with inputs that need a copy (not contiguous) and memory that is freed at once."""
    g = gen(15)
    x = hidden(g, 900, 1000, torch.bfloat16)
    weight, bias = 1 + 0.1 * randn(g, 1000), 0.1 * randn(g, 1000)
    wq = w.quantize_rows(randn(g, 300, 1000))
    dy = randn(g, 1000, 900).bfloat16().t()
    y, mean, rstd = w.layer_norm(x, weight, bias)
    want = [y, *w.layer_norm_backward(dy, x, weight, mean, rstd), w.linear_int8(w.layer_norm_int8(x, weight, bias), wq),
            w.linear_int8(w.quantize_rows(dy), wq)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        y, mean, rstd = w.layer_norm(x, weight, bias, stream=s)
        got = [y, *w.layer_norm_backward(dy, x, weight, mean, rstd, stream=s)]
        a = w.layer_norm_int8(x, weight, bias, stream=s)
        got.append(w.linear_int8(a, wq, stream=s))
        b = w.quantize_rows(dy, stream=s)
        got.append(w.linear_int8(b, wq, stream=s))
        del a, b, mean, rstd, y
        torch.full((4_000_000,), 3.0, device="cuda")  # other work that may take freed memory
        torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got


def test_capture_in_a_graph():
    """One training step's operators and one encoding, replayed with new inputs, against the eager calls."""
    g = gen(16)
    x, dy = hidden(g, 500, 768, torch.bfloat16), randn(g, 500, 768).bfloat16()
    weight, bias = torch.ones(768, device="cuda"), torch.zeros(768, device="cuda")
    wq = w.quantize_rows(randn(g, 128, 768))

    def work():
        y, mean, rstd = w.layer_norm(x, weight, bias)
        return (y, *w.layer_norm_backward(dy, x, weight, mean, rstd),
                w.linear_int8(w.layer_norm_int8(x, weight, bias), wq))

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for k in range(4):
        x.copy_(hidden(g, 500, 768, torch.bfloat16))
        weight.copy_(1 + 0.1 * randn(g, 768))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, work()):
            assert torch.equal(a, b), k


# ---------------------------------------------------------------------------- sizes past 32 bits

def test_layer_norm_past_32_bits():
    """More than 2^31 elements: the last rows equal those of a call on them alone."""
    rows, cols = 2_100_003, 1024
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen(20))
    weight = 1 + 0.1 * randn(gen(21), cols)
    say("layer norm of", x.numel(), "elements")
    y, mean, rstd = w.layer_norm(x, weight, None)
    at = [slice(0, 3), slice(2_097_150, 2_097_155), slice(rows - 3, rows)]
    for s in at:
        assert torch.equal(y[s], w.layer_norm(x[s], weight, None)[0])
    dx = w.layer_norm_backward(y, x, weight, mean, rstd)[0]
    for s in at:
        alone = w.layer_norm_backward(y[s], x[s], weight, mean[s].contiguous(), rstd[s].contiguous())[0]
        assert torch.equal(dx[s], alone)
    del dx, y
    q = w.quantize_rows(x)
    for s in at:
        alone = w.quantize_rows(x[s])
        assert torch.equal(q.values[s], alone.values) and torch.equal(q.scale[s], alone.scale)


def test_linear_int8_past_32_bits():
    """More than 2^31 results, and operands of more than 2^31 bytes."""
    g = gen(22)
    for rows, n, cols in ((70_001, 32_768, 128), (2_200_001, 33, 1000), (33, 2_097_000, 1100)):
        a, sa = int8_rows(g, rows, cols)
        b, sb = int8_rows(g, n, cols)
        qa, qb = w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb)
        del a, b
        say("int8 product", rows, n, cols)
        out = w.linear_int8(qa, qb)
        last = w.QuantizedRows(qa.values[-20:].contiguous(), sa[-20:].contiguous(), cols)
        assert torch.equal(out[-20:], w.linear_int8(last, qb))
        few = w.QuantizedRows(qb.values[-20:].contiguous(), sb[-20:].contiguous(), cols)
        assert torch.equal(out[:, -20:], w.linear_int8(qa, few))
        del out, qa, qb, last, few


def test_adamw_past_32_bits():
    """A tensor of more than 2^31 elements: its last ones move as they do alone."""
    n = (1 << 31) + 5000
    for bits in (8, 32):
        p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        tail = slice(n - n % 256 - 2560, n)  # whole blocks and the last, partial one
        grad[tail].normal_(generator=gen(23))
        say("adamw", bits, n)
        opt = w.AdamW([p], LR, (B1, B2), EPS, DECAY, bits)
        opt.step([grad])
        small = torch.zeros(n - tail.start, dtype=torch.bfloat16, device="cuda")
        alone = w.AdamW([small], LR, (B1, B2), EPS, DECAY, bits)
        alone.step([grad[tail].clone()])
        assert torch.equal(p[tail], small) and not p[:5000].any()
        assert torch.equal(opt.m[tail.start:], alone.m) and torch.equal(opt.v[tail.start:], alone.v)
        del opt, p, grad


def test_adamw_copies_step_on_their_own():
    """A deep copy and an unpickled optimizer go on as the original does, also after that is gone."""
    import copy
    import io

    g = gen(24)
    grad = tensors(g, [700, 0, 33], torch.float32, 0.1)
    for bits in (32, 8):
        opt = w.AdamW(tensors(g, [700, 0, 33], torch.float32, 1.0), bits=bits)
        opt.step(grad)
        file = io.BytesIO()
        torch.save(opt, file)
        file.seek(0)
        twins = [copy.deepcopy(opt), torch.load(file, weights_only=False)]
        opt.step(grad)
        want = [x.clone() for x in (*opt.params, *opt.moments())]
        del opt
        for twin in twins:
            twin.step(grad)
            assert all(torch.equal(a, b) for a, b in zip(want, (*twin.params, *twin.moments())))


def test_adamw_refuses_parameters_that_share_memory():
    flat = torch.ones(1000, device="cuda")
    for shared in ([flat, flat], [flat[:600], torch.ones(3, device="cuda"), flat[599:]]):
        for bits in (32, 8):
            with pytest.raises(ValueError, match="share memory"):
                w.AdamW(shared, bits=bits)
    w.AdamW([flat[600:], flat[:600], flat[:0], flat[:0]]).step([flat[600:].clone(), flat[:600].clone(), None, None])
    assert (flat < 1).all()


def test_adamw_refuses_gradients_of_another_shape():
    """As many elements in another shape (a transposed weight's gradient) would move the wrong ones."""
    p = [torch.ones(30, 7, device="cuda"), torch.ones(8, device="cuda")]
    ones = [torch.ones_like(x) for x in p]
    for bits in (32, 8):
        opt = w.AdamW(p, bits=bits)
        for bad in (torch.ones(7, 30, device="cuda"), torch.ones(210, device="cuda"), torch.ones(1, 30, 7, device="cuda")):
            with pytest.raises(ValueError, match="gradient 0"):
                opt.step([bad, ones[1]])
        with pytest.raises(ValueError, match="gradient 1"):
            opt.step([ones[0], torch.ones(2, 4, device="cuda")])
        assert opt.steps == 0 and all((x == 1).all() for x in p)
        opt.step(ones)
        p = [torch.ones_like(x) for x in p]


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-21, EPS])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_tiny_gradients(bits, eps):
    """Second moments below the smallest normal number divide as any other: with an eps below their root, the step
    is the formula's. Alone, and in one block with ordinary gradients. The moments before a step are read back, the new
    ones follow from them in single fp32 operations; bounds as in reference_step."""
    f = np.float32
    tiny = (10.0 ** np.linspace(-20.5, -15, 250) * np.where(np.arange(250) % 3, 1, -1)).astype(f)
    usual = (10.0 ** np.linspace(-12, 0, 256)).astype(f)
    mixed = np.where(np.arange(256) % 5, usual, f(2e-20))
    g = np.concatenate([tiny, np.full(6, 1e-19, f), usual, mixed, tiny[:99]])
    grad = torch.from_numpy(g).cuda()
    p = torch.linspace(-1, 1, len(g), device="cuda") * 1e-3
    opt = w.AdamW([p], LR, (B1, B2), eps, DECAY, bits)
    for t in (1, 2):
        m, v = (x.cpu().numpy()[:len(g)].copy() for x in opt.moments())
        before = f64(p).numpy()
        opt.step([grad])
        m = (m * f(B1) + g * f(1 - B1)).astype(np.float64)
        v = (v * f(B2) + (g * g) * f(1 - B2)).astype(np.float64)
        assert (v > 0).all() and (v < 2.0 ** -126).any()
        move = LR / (1 - B1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - B2 ** t) + eps)
        want = before * (1 - LR * DECAY) - move
        tol = 3 * U * (abs(before) + abs(want)) + 12 * U * abs(move)
        off = abs(f64(p).numpy() - want) <= tol
        assert off.all(), (t, int((~off).sum()), int(np.argmin(off)), p[int(np.argmin(off))].item())


def test_layer_norm_in_autograd():
    """Gradients reach x, weight and bias, as the backward call gives them; none under no_grad."""
    g = gen(25)
    for t in TYPES.values():
        for shape, params in (((5, 100), torch.float32), ((2, 3, 777), t), ((64,), t)):
            cols = shape[-1]
            x = hidden(g, 6, cols, t).flatten()[:int(np.prod(shape))].view(shape).requires_grad_()
            weight, bias = ((1 + 0.2 * randn(g, cols)).to(params).requires_grad_() for _ in range(2))
            dy = randn(g, *shape).to(t)
            y, mean, rstd = w.layer_norm(x, weight, bias)
            assert y.requires_grad and not mean.requires_grad and not rstd.requires_grad
            y.backward(dy)
            with torch.no_grad():
                plain, m, r = w.layer_norm(x, weight, bias)
            assert not plain.requires_grad and torch.equal(plain, y) and torch.equal(m, mean) and torch.equal(r, rstd)
            want = w.layer_norm_backward(dy, x.detach(), weight.detach(), mean, rstd)
            for got, ref in zip((x.grad, weight.grad, bias.grad), want):
                assert got.dtype == ref.dtype and torch.equal(got, ref)
            # one of them alone; a broadcast gradient; without weight or bias
            fixed = x.detach()
            alone, = torch.autograd.grad(w.layer_norm(fixed, weight.detach(), bias)[0].sum(), [bias])
            assert torch.equal(alone, w.layer_norm_backward(torch.ones_like(fixed), fixed, weight.detach(), m, r)[2])
            alone, = torch.autograd.grad(w.layer_norm(fixed, None, bias)[0], [bias], dy)
            assert alone.dtype == params
            assert torch.equal(alone, w.layer_norm_backward(dy, fixed, None, m, r)[2].to(params))
            alone, = torch.autograd.grad(w.layer_norm(x)[0], [x], dy)
            assert torch.equal(alone, w.layer_norm_backward(dy, fixed, None, m, r)[0])
    # a second derivative is refused, not left out
    x = randn(g, 4, 32).requires_grad_()
    first, = torch.autograd.grad(w.layer_norm(x)[0].square().sum(), [x], create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()


def test_layer_norm_in_autograd_on_another_stream():
    g = gen(26)
    x, dy = hidden(g, 900, 1000, torch.bfloat16), randn(g, 900, 1000).bfloat16()
    weight = 1 + 0.1 * randn(g, 1000)
    y, mean, rstd = w.layer_norm(x, weight)
    want = w.layer_norm_backward(dy, x, weight, mean, rstd)[:2]
    torch.cuda.synchronize()
    x.requires_grad_()
    weight.requires_grad_()
    s = torch.cuda.Stream()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        out = w.layer_norm(x, weight, stream=s)[0]
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(out, y)
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, [x, weight], dy), want))


def test_adamw_is_seen_by_autograd():
    """A backward pass over parameters that a step has changed since is refused, as after any change in place."""
    for bits in (32, 8):
        p, still = torch.ones(4, 8, device="cuda", requires_grad=True), torch.ones(8, device="cuda", requires_grad=True)
        other = torch.ones(5, device="cuda")
        with torch.inference_mode():
            apart = torch.ones(5, device="cuda")  # counts no versions
        opt = w.AdamW([p, still, other, apart], bits=bits)
        x = torch.ones(2, 4, device="cuda", requires_grad=True)
        stale, fine = (x @ p).sum(), (x.sum() * still).sum()
        before = [t._version for t in (p, still, other)]
        opt.step([torch.ones_like(p), None, torch.ones_like(other), torch.ones(5, device="cuda")])
        assert [t._version > b for t, b in zip((p, still, other), before)] == [True, False, True]
        assert (apart < 1).all()
        fine.backward()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            stale.backward()
        # a view's change is the whole tensor's
        flat = torch.ones(20, device="cuda")
        seen = flat._version
        w.AdamW([flat[3:9]], bits=bits).step([torch.ones(6, device="cuda")])
        assert flat._version > seen


def _product_cases():
    import product_sizes

    return [pytest.param(kernel, size, id=f"{kernel}: {size[0]} x {size[1]} x {size[2]}".replace(" ", ""))
            for kernel, sizes in product_sizes.SIZES.items() for size in sizes]


@pytest.mark.parametrize("kernel,size", _product_cases())
def test_linear_int8_kernels(kernel, size):
    """Every kernel of the product at sizes that are no multiples of its tiles, in every type, with a bias and without."""
    rows, n, cols = size
    g = gen(n)
    a, sa = int8_rows(g, rows, cols)
    b, sb = int8_rows(g, n, cols)
    qa, qb = w.QuantizedRows.from_int8(a, sa), w.QuantizedRows.from_int8(b, sb)
    acc = a.double() @ b.double().t()  # exact: below 2^53
    scaled = acc * sb.double() * sa.double()[:, None]
    del acc
    for bias in (randn(g, n), None):
        want = scaled if bias is None else scaled + bias.double()
        for t in TYPES.values():
            say("int8 product", kernel, size, t)
            out = w.linear_int8(qa, qb, bias, t)
            off = (out.double() - want).abs() - (4 * U * scaled.abs() + U * want.abs() + rounding(want, t))
            assert out.shape == want.shape and not (off > 0).any(), (t, int((off > 0).sum()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(37, 3), (5000, 100), (37, 101), (37, 256), (2100, 771), (9, 1024), (37, 2047),
                                       (9, 3000), (700, 5001), (9, 8200), (600, 9001), (9, 16_383), (9, 16_384)])
def test_layer_norm_backward_in_place_and_in_part(rows, cols, dtype):
    """dx over x or over dy, either sum left out, and neither with no scratch: the bits of the ordinary call. Rows of
    16 lanes, a wave, four and eight waves, even and ragged."""
    from paper_2501_17788_amd import lib

    t = TYPES[dtype]
    code = {torch.float32: 0, torch.bfloat16: 2}[t]
    g = gen(rows + cols)
    x, dy, weight = hidden(g, rows, cols, t), randn(g, rows, cols).to(t), 1 + 0.2 * randn(g, cols)
    _, mean, rstd = w.layer_norm(x, weight)
    want = w.layer_norm_backward(dy, x, weight, mean, rstd)
    need = np.zeros(1, np.int64)
    assert lib.warp_layer_norm_backward_scratch(rows, cols, code, need.ctypes.data) == 0
    scratch = torch.empty(int(need[0]), dtype=torch.uint8, device="cuda")
    for place in ("x", "dy", "apart"):
        for sums in ("both", "dw", "db", "none"):
            say("backward", rows, cols, dtype, place, sums)
            a, d = x.clone(), dy.clone()
            dx = {"x": a, "dy": d, "apart": torch.empty_like(x)}[place]
            dw, db = torch.full((2, cols), 7.0, device="cuda")
            rc = lib.warp_layer_norm_backward(
                d.data_ptr(), cols, a.data_ptr(), cols, rows, cols, code, weight.data_ptr(), 0, mean.data_ptr(),
                rstd.data_ptr(), dx.data_ptr(), cols, dw.data_ptr() if sums in ("both", "dw") else None,
                db.data_ptr() if sums in ("both", "db") else None, scratch.data_ptr() if sums != "none" else None,
                int(need[0]) if sums != "none" else 0, torch.cuda.current_stream().cuda_stream)
            assert rc == 0, w.last_error()
            assert torch.equal(dx, want[0])
            assert torch.equal(dw, want[1]) if sums in ("both", "dw") else (dw == 7).all()
            assert torch.equal(db, want[2]) if sums in ("both", "db") else (db == 7).all()
            if place != "x":
                assert torch.equal(a, x)
            if place != "dy":
                assert torch.equal(d, dy)
