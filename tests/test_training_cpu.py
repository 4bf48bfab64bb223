"""Refusals and sizes of the operators that train a token encoder, before a device is touched."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
w = pytest.importorskip("paper_2501_17788_amd")

lib = w.lib
P = 1 << 20  # an aligned address that no call below reads
BIG = 1 << 40


def refused(rc, code, needle):
    assert rc == code, (rc, w.last_error())
    assert needle in w.last_error(), w.last_error()


def embed(**over):
    a = dict(ids=P, id_bytes=8, tokens=4, table=P, table_stride=64, vocabulary=9, cols=64, dtype=0, scale=1.0, out=P,
             out_stride=64, stream=None)
    a.update(over)
    return lib.warp_embedding(*a.values())


def embed_back(**over):
    a = dict(dy=P, dy_stride=64, ids=P, id_bytes=8, tokens=4, vocabulary=9, cols=64, dtype=0, scale=1.0, dtable=P,
             dtable_stride=64, scratch=P, bytes=BIG, stream=None)
    a.update(over)
    return lib.warp_embedding_backward(*a.values())


@pytest.mark.parametrize("call", [embed, embed_back])
@pytest.mark.parametrize("over,code,needle", [
    (dict(tokens=-1), w.EINVAL, "tokens"), (dict(vocabulary=0), w.EINVAL, "vocabulary"), (dict(cols=0), w.EINVAL, "cols"),
    (dict(tokens=(1 << 25) + 1), w.ENOTSUP, "2^25"), (dict(vocabulary=(1 << 25) + 1), w.ENOTSUP, "2^25"),
    (dict(cols=(1 << 20) + 1), w.ENOTSUP, "2^20"), (dict(id_bytes=2), w.EINVAL, "ids of 4 or 8"),
    (dict(tokens=1 << 25, cols=1 << 13), w.ENOTSUP, "2^37"), (dict(vocabulary=1 << 25, cols=1 << 13), w.ENOTSUP, "2^37"),
    (dict(dtype=3), w.EINVAL, "dtype"), (dict(scale=float("nan")), w.EINVAL, "scale"),
    (dict(scale=float("inf")), w.EINVAL, "scale"), (dict(ids=None), w.EINVAL, "null"), (dict(ids=P + 4), w.EINVAL, "misaligned"),
])
def test_embedding_refusals(call, over, code, needle):
    refused(call(**over), code, needle)


@pytest.mark.parametrize("over,needle", [(dict(table=None), "null"), (dict(out=None), "null"), (dict(table=P + 2), "misaligned"),
                                         (dict(out=P + 1), "misaligned"), (dict(table_stride=63), "stride"),
                                         (dict(out_stride=-64), "stride")])
def test_lookup_refusals(over, needle):
    refused(embed(**over), w.EINVAL, needle)


@pytest.mark.parametrize("over,needle", [(dict(dy=None), "null"), (dict(dtable=None), "null"), (dict(dy=P + 2), "misaligned"),
                                         (dict(dy_stride=0), "stride"), (dict(dtable_stride=63), "stride"),
                                         (dict(scratch=None), "scratch"), (dict(bytes=100), "scratch"),
                                         (dict(scratch=P + 8), "scratch")])
def test_embedding_backward_refusals(over, needle):
    refused(embed_back(**over), w.EINVAL, needle)


def loss(**over):
    a = dict(hidden=P, hidden_stride=64, tokens=4, cols=64, dtype=0, table=P, table_stride=64, vocabulary=9, targets=P,
             target_bytes=8, scale=1.0, loss=P, lse=P, scratch=P, bytes=BIG, stream=None)
    a.update(over)
    return lib.warp_cross_entropy(*a.values())


def loss_back(**over):
    a = dict(dloss=P, hidden=P, hidden_stride=64, tokens=4, cols=64, dtype=0, table=P, table_stride=64, vocabulary=9,
             targets=P, target_bytes=8, scale=1.0, loss=P, lse=P, dhidden=P, dhidden_stride=64, dtable=P, dtable_stride=64,
             scratch=P, bytes=BIG, stream=None)
    a.update(over)
    return lib.warp_cross_entropy_backward(*a.values())


@pytest.mark.parametrize("call", [loss, loss_back])
@pytest.mark.parametrize("over,code,needle", [
    (dict(tokens=-1), w.EINVAL, "tokens"), (dict(vocabulary=0), w.EINVAL, "vocabulary"), (dict(cols=0), w.EINVAL, "cols"),
    (dict(tokens=(1 << 22) + 1), w.ENOTSUP, "2^22"), (dict(vocabulary=(1 << 25) + 1), w.ENOTSUP, "2^25"),
    (dict(cols=(1 << 14) + 1), w.ENOTSUP, "2^14"), (dict(dtype=-1), w.EINVAL, "dtype"),
    (dict(hidden=None), w.EINVAL, "null"), (dict(table=None), w.EINVAL, "null"), (dict(targets=None), w.EINVAL, "null"),
    (dict(loss=None), w.EINVAL, "null"), (dict(lse=None), w.EINVAL, "null"), (dict(hidden_stride=63), w.EINVAL, "stride"),
    (dict(table_stride=1), w.EINVAL, "stride"), (dict(hidden=P + 2), w.EINVAL, "misaligned"),
    (dict(table=P + 1), w.EINVAL, "misaligned"), (dict(targets=P + 4), w.EINVAL, "misaligned"),
    (dict(loss=P + 2), w.EINVAL, "misaligned"), (dict(target_bytes=1), w.EINVAL, "targets of 4 or 8"),
    (dict(scale=float("nan")), w.EINVAL, "scale"), (dict(scratch=None), w.EINVAL, "scratch"),
    (dict(bytes=1000), w.EINVAL, "scratch"), (dict(scratch=P + 4), w.EINVAL, "scratch"),
])
def test_cross_entropy_refusals(call, over, code, needle):
    refused(call(**over), code, needle)


@pytest.mark.parametrize("over,needle", [(dict(dloss=None), "null"), (dict(dloss=P + 1), "misaligned"),
                                         (dict(dhidden=P + 2), "misaligned"), (dict(dtable=P + 2), "misaligned"),
                                         (dict(dhidden_stride=8), "stride"), (dict(dtable_stride=8), "stride")])
def test_cross_entropy_backward_refusals(over, needle):
    refused(loss_back(**over), w.EINVAL, needle)


def linear(**over):
    a = dict(x=P, x_stride=64, rows=4, cols=64, dtype=0, weight=P, weight_stride=64, n=9, bias=None, bias_dtype=0, y=P,
             y_stride=9, scratch=P, bytes=BIG, stream=None)
    a.update(over)
    return lib.warp_linear(*a.values())


def linear_back(**over):
    a = dict(dy=P, dy_stride=9, rows=4, n=9, dtype=0, q=P, q_stride=128, q_scale=P, cols=64, weight=P, weight_stride=64, dx=P,
             dx_stride=64, dw=P, dw_stride=64, db=P, db_dtype=0, scratch=P, bytes=BIG, stream=None)
    a.update(over)
    return lib.warp_linear_backward(*a.values())


@pytest.mark.parametrize("call", [linear, linear_back])
@pytest.mark.parametrize("over,code,needle", [
    (dict(rows=-1), w.EINVAL, "rows"), (dict(n=0), w.EINVAL, "n and cols"), (dict(cols=0), w.EINVAL, "n and cols"),
    (dict(rows=(1 << 24) + 1), w.ENOTSUP, "2^24"), (dict(n=(1 << 20) + 1), w.ENOTSUP, "2^20"),
    (dict(rows=1 << 24, n=1 << 14), w.ENOTSUP, "2^36"), (dict(cols=1 << 18, n=1 << 17), w.ENOTSUP, "2^34"),
    (dict(dtype=9), w.EINVAL, "dtype"), (dict(weight=None), w.EINVAL, "null"), (dict(weight=P + 2), w.EINVAL, "misaligned"),
    (dict(weight_stride=63), w.EINVAL, "stride"), (dict(rows=400, scratch=None), w.EINVAL, "scratch"),
    (dict(rows=400, bytes=8), w.EINVAL, "scratch"), (dict(rows=400, scratch=P + 1), w.EINVAL, "scratch"),
])
def test_linear_refusals(call, over, code, needle):
    refused(call(**over), code, needle)


@pytest.mark.parametrize("over,needle", [(dict(x=None), "null"), (dict(y=None), "null"), (dict(x=P + 2), "misaligned"),
                                         (dict(x_stride=63), "stride"), (dict(y_stride=8), "stride"),
                                         (dict(bias=P, bias_dtype=1), "bias"), (dict(bias=P, bias_dtype=7), "bias"),
                                         (dict(bias=P + 2), "misaligned")])
def test_linear_forward_refusals(over, needle):
    refused(linear(**over), w.EINVAL, needle)


@pytest.mark.parametrize("over,needle", [(dict(dy=None), "null"), (dict(dy=P + 2), "misaligned"), (dict(dy_stride=8), "stride"),
                                         (dict(dx_stride=63), "stride"), (dict(dw_stride=63), "stride"),
                                         (dict(dx=P + 1), "misaligned"), (dict(q=None), "null"), (dict(q_scale=None), "null"),
                                         (dict(q_stride=64), "int8 rows"), (dict(q_stride=130), "int8 rows"),
                                         (dict(q=P + 8), "int8 rows"), (dict(q_scale=P + 2), "int8 rows"),
                                         (dict(db_dtype=2), "dbias"), (dict(db=P + 2), "misaligned")])
def test_linear_backward_refusals(over, needle):
    refused(linear_back(**over), w.EINVAL, needle)


def test_scratch_sizes():
    """Many rows of 16-bit operands of ordinary alignment take none; other operands a copy; more rows never take less."""
    n = ctypes.c_int64()
    assert not lib.warp_linear_scratch(P, 1024, 65_536, 1024, 2, P, 1024, 1024, ctypes.byref(n)) and n.value == 0
    assert not lib.warp_linear_scratch(P + 2, 1024, 65_536, 1024, 2, P, 1024, 1024, ctypes.byref(n))
    assert 65_536 * 1024 * 2 <= n.value < 65_536 * 1024 * 2 + 4096
    assert not lib.warp_linear_scratch(P, 1024, 4096, 1024, 0, P, 1024, 1024, ctypes.byref(n))
    assert n.value >= (4096 + 1024) * 1024 * 6
    assert lib.warp_linear_scratch(P, 1024, 4096, 1024, 0, P, 1024, 1024, None) == w.EINVAL
    assert lib.warp_linear_backward_scratch(P, 64, -1, 64, 0, 64, P, 64, ctypes.byref(n)) == w.EINVAL
    assert lib.warp_embedding_backward_scratch(1, 0, 1, ctypes.byref(n)) == w.EINVAL
    assert lib.warp_embedding_backward_scratch(1, 1 << 60, 1, ctypes.byref(n)) == w.ENOTSUP
    assert lib.warp_cross_entropy_scratch(1, 1, 0, P, 1, 0, ctypes.byref(n), None) == w.EINVAL
    # G is never larger than a piece, whatever the vocabulary
    sizes = []
    for vocabulary in (100, 1000, 30_000, 250_001, 1 << 24):
        m = ctypes.c_int64()
        assert not lib.warp_cross_entropy_scratch(16_384, 1024, 2, P, 1024, vocabulary, ctypes.byref(n), ctypes.byref(m))
        sizes.append(m.value)
        assert n.value < 600 << 20
    assert max(sizes) < 1000 << 20
    last = 0
    for tokens in (0, 1, 100, 16_384, 100_000):
        assert not lib.warp_cross_entropy_scratch(tokens, 64, 1, P, 64, 5000, ctypes.byref(n), None)
        assert n.value >= last
        last = n.value


def test_host_tensors_are_refused():
    x, ids = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64)
    rows = w.QuantizedRows(torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3), 8)
    for call in (lambda: w.embedding(ids, x), lambda: w.embedding_backward(x, ids, 3), lambda: w.linear(x, x),
                 lambda: w.linear_backward(torch.zeros(3, 3), rows, x), lambda: w.cross_entropy(x, x, ids),
                 lambda: w.cross_entropy_backward(ids.float(), x, x, ids, ids.float(), ids.float())):
        with pytest.raises(ValueError, match="device tensors"):
            call()
    with pytest.raises(ValueError, match="columns"):
        w.linear_backward(torch.zeros(3, 3), rows._replace(cols=9), x)


def test_product_sizes_reach_their_kernels():
    """The sizes of the GPU tests choose the products that they are listed under: a change of the choice that leaves one
    without a test fails here."""
    import product_plans

    choose = lib["_ZN4warp14product_choiceElllib"]  # int warp::product_choice(int64_t m, int64_t n, int64_t k, int dtype, bool bytes)
    choose.argtypes, choose.restype = [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_bool], ctypes.c_int
    seen = set()
    for rows, cols, n in product_plans.SIZES:
        for dtype in (0, 1, 2):
            few, whole, outer = rows <= 32, dtype == 0 and rows <= 384, dtype == 0 and rows <= 32
            seen.add(("y", "few" if few else "whole" if whole else choose(rows, n, cols, dtype, False)))
            seen.add(("dx", "few" if rows <= (64 if dtype == 0 else 32) else "whole" if whole else choose(rows, cols, n, dtype, False)))
            packed, direct = choose(n, cols, rows, dtype, False), choose(n, cols, rows, dtype, True)
            seen.add(("dweight", "outer" if outer else "whole" if whole else direct + 10 if direct >= 0 else packed))
    want = {(name, tile + 4 * split) for name in ("y", "dx", "dweight") for tile in range(3) for split in (0, 1)}
    want |= {("y", "few"), ("y", "whole"), ("dx", "few"), ("dx", "whole"), ("dweight", "outer"), ("dweight", "whole")} | {("dweight", 10 + tile + 4 * split) for tile in range(2) for split in (0, 1)}
    assert want <= seen, sorted(want - seen, key=str)


@pytest.mark.parametrize("name", ["quantize_rows", "layer_norm_int8", "linear_int8", "layer_norm_backward", "embedding_backward",
                                  "cross_entropy_backward", "linear_backward", "linear"])
def test_calls_that_a_trace_cannot_hold_are_refused(name):
    ids, stats = torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    rows = w.QuantizedRows(torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3), 8)
    call = {"quantize_rows": lambda x: w.quantize_rows(x).values, "layer_norm_int8": lambda x: w.layer_norm_int8(x).values,
            "linear_int8": lambda x: w.linear_int8(rows, rows, x[0]), "linear": lambda x: w.linear(x, x, None, rows),
            "layer_norm_backward": lambda x: w.layer_norm_backward(x, x, None, stats, stats)[0],
            "embedding_backward": lambda x: w.embedding_backward(x, ids, 3),
            "cross_entropy_backward": lambda x: w.cross_entropy_backward(stats, x, x, ids, stats, stats)[0],
            "linear_backward": lambda x: w.linear_backward(x[:, :3], rows, x)[0]}[name]
    with pytest.raises(RuntimeError, match=name + ".* cannot be traced"):
        torch.jit.trace(call, torch.zeros(3, 8))


def planes_of(x):
    """The three bfloat16 planes that float32 products are made of, as 64-bit numbers [3, n]."""
    split = lib["_ZN4warp12split_planesEPKflPt"]  # void warp::split_planes(const float* x, int64_t n, uint16_t* planes)
    split.argtypes, split.restype = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p], None
    x = np.ascontiguousarray(x, np.float32)
    out = np.empty((3, len(x)), np.uint16)
    split(x.ctypes.data, len(x), out.ctypes.data)
    return (out.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def hard_operands(rng):
    """Mantissas at which a plane is as large as it gets, and others; near one, by signs."""
    some = [0x800000, 0x800001, 0x807fff, 0x808000, 0x808001, 0x80ffff, 0x810000, 0x8080ff, 0x80807f, 0x808080, 0x80ff80, 0xff7fff,
            0xff8000, 0xff8080, 0xffffff, 0xffff00, 0xfffe80, 0x817f7f, 0x80fffe]
    x = np.concatenate([np.array(some), rng.integers(1 << 23, 1 << 24, 3000)]).astype(np.float64) * 2.0 ** -23
    return (x * rng.choice([-1.0, 1.0], len(x))).astype(np.float32)


def test_planes_of_a_float32():
    """Their sum is the number, to the last bit down to 2^-110 and within half of 2^-133 below; up to the largest one."""
    rng = np.random.default_rng(1)
    x = hard_operands(rng)
    for by in (0, 40, -60, -110, 126):
        a = x * np.float32(2.0 ** by)
        assert np.isfinite(a).all() and (planes_of(a).sum(0) == a).all(), by
    top = np.finfo(np.float32).max
    near = np.array([top, -top, np.nextafter(np.float32(top), np.float32(0)), 0.998 * top, 0.0, -0.0], np.float32)
    p = planes_of(near)
    assert np.isfinite(p).all() and (p.sum(0) == near).all()
    small = np.concatenate([(rng.standard_normal(3000) * 10.0 ** rng.uniform(-45, -33, 3000)), [1e-45, 2.0 ** -133]]).astype(np.float32)
    p = planes_of(small)
    assert (abs(p.sum(0) - small) <= 2.0 ** -134).all()
    p = planes_of(np.array([np.inf, -np.inf, np.nan], np.float32))
    assert p[0, 0] == np.inf and p[0, 1] == -np.inf and np.isnan(p[0, 2]) and not p[1:].any()


def test_what_products_of_planes_leave_out():
    """A product is six of nine products of planes: high, middle and low by each other but for middle by low and low by low. With
    |middle| <= 2^-8 and |low| <= 2^-17 of an operand's power of two these are at most 2 x 2^-25 + 2^-34 of the operands', on either
    side of zero: the mean of a million of them lies within 6 standard deviations, of at most 2^-24 / 1000 each."""
    rng = np.random.default_rng(2)

    def left_out(a, b):  # exact: each product has 16 bits
        p, q = planes_of(a), planes_of(b)
        return p[1] * q[2] + p[2] * q[1] + p[2] * q[2]

    x = hard_operands(rng)
    a, b = (t.reshape(-1) for t in np.meshgrid(x[:500], x[:500]))
    for other in (b, b * np.float32(2.0 ** -100), rng.permutation(b)):
        both = abs(a.astype(np.float64) * other)
        assert (abs(left_out(a, other)) <= (2.0 ** -24 + 2.0 ** -34) * both).all()
    # an operand near the largest number, whose first plane is cut off and not rounded up to infinity
    top = x[:19] * np.float32(2.0 ** 127)
    a, b = (t.reshape(-1) for t in np.meshgrid(np.concatenate([top, np.float32([3.4028235e38, 3.4e38])]), x[:200] * np.float32(0.25)))
    assert (abs(left_out(a, b)) <= 2.0 ** -23 * abs(a.astype(np.float64) * b)).all()
    a, b = (rng.standard_normal(1_000_000).astype(np.float32) for _ in range(2))
    assert abs((left_out(a, b) / (a.astype(np.float64) * b)).mean()) <= 6 * 2.0 ** -24 / 1000


def test_leaves_behind_other_operations_are_seen(monkeypatch):
    """A captured backward pass is refused by the leaves that it leads to, whatever lies between; on the host, since trying such a capture
    ends the process."""
    from paper_2501_17788_amd import encoder

    leaf, other = torch.ones(4, 4, requires_grad=True), torch.ones(4, 4, requires_grad=True)

    class Named(torch.autograd.Function):  # whose context holds something under an accumulator's name
        @staticmethod
        def forward(ctx, x):
            ctx.variable = other
            return x * 2

        @staticmethod
        def backward(ctx, dy):
            return dy * 2

    cast = leaf.to(torch.bfloat16)
    behind = [cast.t() * 2, cast.view(2, 8)[:1], (cast.float() @ other).sum(), Named.apply(leaf.t()), torch.cat([other, leaf.t()]) + 1,
              sum(leaf * i for i in range(3000))]
    monkeypatch.setattr(encoder._native, "adds_on_default_stream", lambda t: t is leaf)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    for out in behind:
        encoder._refuse_capture(out.grad_fn)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for out in behind:
        with pytest.raises(RuntimeError, match="cannot be captured"):
            encoder._refuse_capture(out.grad_fn)
    for out in (other * 2, Named.apply(other), (leaf.detach() * other).sum()):
        encoder._refuse_capture(out.grad_fn)
