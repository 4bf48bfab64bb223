// The Python binding of the token encoder's operators: checks torch tensors, allocates outputs and calls the C
// functions of warp.h on the current stream of the tensors' device. Native because a small call's time is the host's:
// layer norm of 32 rows takes 10.2 us through ctypes and 6 us through this, 3.5 us of either being the launch.
#include <ATen/TracerMode.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/extension.h>

#include <sstream>
#include <stdexcept>

#include "warp.h"

namespace py = pybind11;
using at::Tensor;
using MaybeTensor = std::optional<Tensor>;

namespace {

constexpr int64_t kPad = 128, kBlock = 256;

template <typename... A>
[[noreturn]] void refuse(const A&... parts) {  // a ValueError
    std::ostringstream s;
    (s << ... << parts);
    throw std::invalid_argument(s.str());
}

// WarpError with the library's message
void check(int rc) {
    if (rc != WARP_OK) py::module_::import("paper_2501_17788_amd.warp").attr("_check")(rc);
}

bool known(at::ScalarType t) { return t == at::kFloat || t == at::kHalf || t == at::kBFloat16; }
int32_t code(at::ScalarType t) { return t == at::kFloat ? WARP_F32 : t == at::kHalf ? WARP_F16 : WARP_BF16; }

void on_device(const Tensor& first) {
    if (!first.is_cuda()) refuse("expected device tensors, got ", first.device());
}
void on_device(const Tensor& first, const MaybeTensor& t) {
    if (t && t->device() != first.device()) refuse("expected tensors on ", first.device(), ", got ", t->device());
}

void* stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

const void* ptr(const MaybeTensor& t) { return t ? t->const_data_ptr() : nullptr; }

// A tensor [..., cols] as rows whose elements lie one after the other: itself, or a copy.
struct Rows {
    Tensor t;
    int64_t rows, stride;
    int32_t cols;
};
Rows rows_of(const Tensor& x, const char* name) {
    if (!known(x.scalar_type())) refuse(name, " must be float32, float16 or bfloat16, got ", x.dtype());
    if (x.dim() == 0) refuse(name, " must have at least one dimension");
    const int64_t cols = x.size(-1);
    if (cols < 1 || cols > INT32_MAX) refuse(name, " has rows of ", cols, " columns");
    if (x.dim() == 2 && (x.stride(1) == 1 || cols == 1) && (x.stride(0) >= cols || x.size(0) <= 1))
        return {x, x.size(0), x.stride(0), (int32_t)cols};
    return {x.contiguous(), x.numel() / cols, cols, (int32_t)cols};
}

// weight and bias [cols], contiguous, and their common type
struct Params {
    MaybeTensor weight, bias;
    at::ScalarType type = at::kFloat;
};
Params params_of(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias) {
    Params p;
    for (const auto* t : {&weight, &bias}) {
        if (!*t) continue;
        const char* name = t == &weight ? "weight" : "bias";
        if ((*t)->dim() != 1 || (*t)->size(0) != x.size(-1))
            refuse(name, " must have shape (", x.size(-1), ",), got ", (*t)->sizes());
        if (p.weight && (*t)->scalar_type() != p.type)
            refuse("weight and bias must be of one type, got ", p.type, " and ", (*t)->scalar_type());
        p.type = (*t)->scalar_type();
        (t == &weight ? p.weight : p.bias) = (*t)->contiguous();
    }
    if (p.type != at::kFloat && p.type != x.scalar_type())
        refuse("weight and bias must be float32 or ", x.scalar_type(), ", got ", p.type);
    return p;
}

Tensor like(const Tensor& x) { return x.is_contiguous() ? at::empty_like(x) : at::empty(x.sizes(), x.options()); }

bool tracked(const MaybeTensor& t) { return t && t->requires_grad(); }
// Whether forward-mode differentiation follows t: by a tangent, which a tensor without a gradient can have too.
bool has_tangent(const MaybeTensor& t) {
    return t && c10::AutogradState::get_tls_state().get_fw_grad_mode() && t->_fw_grad(0).defined();
}
// Whether torch.jit.trace records, which knows torch's own operations only: of a call it would keep the empty results.
bool traced() { return at::tracer::impl::is_dispatch_enabled(); }
void not_traced(const char* name) {  // a RuntimeError
    if (traced()) throw std::runtime_error(std::string(name) + " cannot be traced: its results would not be recorded");
}
// Calls that autograd follows go through its node, which refuses tangents and is recorded as a whole; it calls the function of
// the same name with _forward, which looks at none of these.
template <typename... T>
bool followed(const T&... tensors) {
    return traced() || (at::GradMode::is_enabled() && (tracked(tensors) || ...)) || (has_tangent(tensors) || ...);
}
py::object node(const char* name) {
    return py::module_::import("paper_2501_17788_amd.encoder").attr(name).attr("apply");
}

py::tuple layer_norm_forward(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x");
    const Params p = params_of(x, weight, bias);
    const auto stats = x.sizes().slice(0, x.dim() - 1);
    Tensor y = like(r.t);
    const auto f32 = x.options().dtype(at::kFloat);
    Tensor mean = at::empty(stats, f32), rstd = at::empty(stats, f32);
    check(warp_layer_norm(r.t.const_data_ptr(), r.stride, r.rows, r.cols, code(x.scalar_type()), ptr(p.weight),
                          ptr(p.bias), code(p.type), (float)eps, y.data_ptr(), r.cols, mean.data_ptr<float>(),
                          rstd.data_ptr<float>(), stream_of(x)));
    return py::make_tuple(y, mean, rstd);
}

py::tuple layer_norm(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
    on_device(x);
    on_device(x, weight);
    on_device(x, bias);
    if (followed(x, weight, bias))
        return node("_LayerNorm")(x, weight, bias, eps);
    return layer_norm_forward(x, weight, bias, eps);
}

py::tuple layer_norm_backward(const Tensor& dy, const Tensor& x, const MaybeTensor& weight, const Tensor& mean,
                              const Tensor& rstd) {
    not_traced("layer_norm_backward");
    if (dy.sizes() != x.sizes() || dy.scalar_type() != x.scalar_type())
        refuse("dy must be like x (", x.sizes(), ", ", x.scalar_type(), "), got ", dy.sizes(), ", ", dy.scalar_type());
    if (x.dim() == 0) refuse("x must have at least one dimension");
    const auto stats = x.sizes().slice(0, x.dim() - 1);
    for (const Tensor* t : {&mean, &rstd})
        if (t->sizes() != stats || t->scalar_type() != at::kFloat || !t->is_contiguous())
            refuse(t == &mean ? "mean" : "rstd", " must be what layer_norm gave: contiguous float32 ", stats);
    on_device(x);
    for (const Tensor* t : {&dy, &mean, &rstd}) on_device(x, *t);
    on_device(x, weight);
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x"), d = rows_of(dy, "dy");
    const Params p = params_of(x, weight, std::nullopt);
    int64_t need = 0;
    check(warp_layer_norm_backward_scratch(r.rows, r.cols, code(x.scalar_type()), &need));
    Tensor dx = like(r.t);
    const auto pt = x.options().dtype(p.type);
    Tensor dw = at::empty({r.cols}, pt), db = at::empty({r.cols}, pt);
    Tensor scratch = at::empty({need}, x.options().dtype(at::kByte));
    check(warp_layer_norm_backward(d.t.const_data_ptr(), d.stride, r.t.const_data_ptr(), r.stride, r.rows, r.cols,
                                   code(x.scalar_type()), ptr(p.weight), code(p.type), mean.const_data_ptr<float>(),
                                   rstd.const_data_ptr<float>(), dx.data_ptr(), r.cols, dw.data_ptr(), db.data_ptr(),
                                   scratch.data_ptr(), need, stream_of(x)));
    return py::make_tuple(dx, dw, db);
}

std::pair<Tensor, Tensor> int8_rows(const Rows& r) {
    return {at::empty({r.rows, (r.cols + kPad - 1) / kPad * kPad}, r.t.options().dtype(at::kChar)),
            at::empty({r.rows}, r.t.options().dtype(at::kFloat))};
}

py::tuple quantize_rows_forward(const Tensor& x) {
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x");
    auto [q, scale] = int8_rows(r);
    check(warp_quantize_rows(r.t.const_data_ptr(), r.stride, r.rows, r.cols, code(x.scalar_type()),
                             (int8_t*)q.data_ptr(), q.size(1), scale.data_ptr<float>(), stream_of(x)));
    return py::make_tuple(q, scale, r.cols);
}

py::tuple quantize_rows(const Tensor& x) {
    not_traced("quantize_rows");
    on_device(x);
    return quantize_rows_forward(x);
}

py::tuple layer_norm_int8(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
    not_traced("layer_norm_int8");
    on_device(x);
    on_device(x, weight);
    on_device(x, bias);
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x");
    const Params p = params_of(x, weight, bias);
    auto [q, scale] = int8_rows(r);
    check(warp_layer_norm_int8(r.t.const_data_ptr(), r.stride, r.rows, r.cols, code(x.scalar_type()), ptr(p.weight),
                               ptr(p.bias), code(p.type), (float)eps, (int8_t*)q.data_ptr(), q.size(1),
                               scale.data_ptr<float>(), stream_of(x)));
    return py::make_tuple(q, scale, r.cols);
}

// what the kernels read of a row must lie inside the tensor
void check_int8(const char* name, const Tensor& v, const Tensor& s, int64_t padded) {
    if (v.scalar_type() != at::kChar || v.dim() != 2 || v.stride(1) != 1)
        refuse(name, ": int8 rows of contiguous elements are needed");
    if (s.scalar_type() != at::kFloat || s.dim() != 1 || s.size(0) != v.size(0) || !s.is_contiguous())
        refuse(name, ": a contiguous float32 scale for each row is needed");
    if (v.size(1) < padded)
        refuse(name, ": rows of ", v.size(1), " columns are not padded to a multiple of ", kPad,
               "; see QuantizedRows.from_int8");
}

Tensor linear_int8(const Tensor& av, const Tensor& sa, int64_t cols, const Tensor& wv, const Tensor& sw,
                   int64_t w_cols, const MaybeTensor& bias, at::ScalarType dtype) {
    not_traced("linear_int8");
    if (!known(dtype)) refuse("dtype must be float32, float16 or bfloat16, got ", dtype);
    if (cols != w_cols) refuse("tokens of ", cols, " columns against a weight of ", w_cols);
    if (cols < 1 || cols > INT32_MAX - kPad) refuse("rows of ", cols, " columns");
    const int64_t padded = (cols + kPad - 1) / kPad * kPad;
    check_int8("a", av, sa, padded);
    check_int8("w", wv, sw, padded);
    const int64_t rows = av.size(0), n = wv.size(0);
    if (n > INT32_MAX) refuse("a weight of ", n, " channels");
    if (bias && (bias->scalar_type() != at::kFloat || bias->dim() != 1 || bias->size(0) != n))
        refuse("bias must be float32 (", n, ",), got ", bias->scalar_type(), " ", bias->sizes());
    on_device(av);
    for (const Tensor* t : {&sa, &wv, &sw}) on_device(av, *t);
    on_device(av, bias);
    const c10::DeviceGuard guard(av.device());
    const MaybeTensor b = bias ? MaybeTensor(bias->contiguous()) : std::nullopt;
    Tensor out = at::empty({rows, n}, av.options().dtype(dtype));
    check(warp_linear_int8((const int8_t*)av.const_data_ptr(), av.stride(0), sa.const_data_ptr<float>(), rows,
                           (const int8_t*)wv.const_data_ptr(), wv.stride(0), sw.const_data_ptr<float>(), (int32_t)n,
                           (int32_t)cols, (const float*)ptr(b), out.data_ptr(), n, code(dtype), stream_of(av)));
    return out;
}

// Whether a leaf's gradients are added on the default stream, where a graph that was made there lives.
bool adds_on_default_stream(const Tensor& leaf) {
    const auto node = torch::autograd::impl::try_get_grad_accumulator(leaf);
    const auto stream = node ? node->stream() : std::nullopt;
    return stream && stream->id() == c10::hip::getDefaultHIPStream(leaf.get_device()).id();
}

Tensor scratch_of(const Tensor& like, int64_t bytes) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

// Whole numbers, one for each row, in one piece.
Tensor whole_numbers(const Tensor& t, const char* name) {
    if (t.scalar_type() != at::kLong && t.scalar_type() != at::kInt)
        refuse(name, " must be int64 or int32, got ", t.scalar_type());
    return t.contiguous();
}
int32_t bytes_of(const Tensor& t) { return (int32_t)t.element_size(); }

Rows matrix_of(const Tensor& t, const char* name, int64_t cols) {
    if (t.dim() != 2) refuse(name, " must have two dimensions, got ", t.sizes());
    if (cols >= 0 && t.size(1) != cols) refuse(name, " has rows of ", t.size(1), " columns, ", cols, " are needed");
    return rows_of(t, name);
}

void same_type(const Tensor& a, const Tensor& b, const char* name, const char* other) {
    if (a.scalar_type() != b.scalar_type()) refuse(name, " must be of ", other, "'s type ", b.scalar_type(), ", got ", a.scalar_type());
}

// leading sizes followed by one more
std::vector<int64_t> with_last(at::IntArrayRef lead, int64_t last) {
    std::vector<int64_t> s(lead.begin(), lead.end());
    s.push_back(last);
    return s;
}

Tensor embedding_forward(const Tensor& ids, const Tensor& table, double scale) {
    const c10::DeviceGuard guard(table.device());
    const Rows t = matrix_of(table, "table", -1);
    const Tensor i = whole_numbers(ids, "ids");
    Tensor out = at::empty(with_last(ids.sizes(), t.cols), table.options());
    check(warp_embedding(i.const_data_ptr(), bytes_of(i), i.numel(), t.t.const_data_ptr(), t.stride, t.rows, t.cols,
                         code(table.scalar_type()), (float)scale, out.data_ptr(), t.cols, stream_of(table)));
    return out;
}

Tensor embedding(const Tensor& ids, const Tensor& table, double scale) {
    on_device(table);
    on_device(table, ids);
    if (followed(table))
        return node("_Embedding")(ids, table, scale).cast<Tensor>();
    return embedding_forward(ids, table, scale);
}

Tensor embedding_backward(const Tensor& dy, const Tensor& ids, int64_t vocabulary, double scale) {
    not_traced("embedding_backward");
    on_device(dy);
    on_device(dy, ids);
    if (dy.dim() < 1 || dy.sizes().slice(0, dy.dim() - 1) != ids.sizes())
        refuse("dy must have a row for each of the ids ", ids.sizes(), ", got ", dy.sizes());
    const c10::DeviceGuard guard(dy.device());
    const Rows d = rows_of(dy, "dy");
    const Tensor i = whole_numbers(ids, "ids");
    int64_t need = 0;
    check(warp_embedding_backward_scratch(i.numel(), vocabulary, d.cols, &need));
    Tensor out = at::empty({vocabulary, d.cols}, dy.options()), scratch = scratch_of(dy, need);
    check(warp_embedding_backward(d.t.const_data_ptr(), d.stride, i.const_data_ptr(), bytes_of(i), i.numel(), vocabulary,
                                  d.cols, code(dy.scalar_type()), (float)scale, out.data_ptr(), d.cols, scratch.data_ptr(),
                                  need, stream_of(dy)));
    return out;
}

// hidden rows, table and targets that fit
struct Scores {
    Rows h, t;
    Tensor y;
    Scores(const Tensor& hidden, const Tensor& table, const Tensor& targets)
        : h(rows_of(hidden, "hidden")), t(matrix_of(table, "table", h.cols)), y(whole_numbers(targets, "targets")) {
        same_type(table, hidden, "table", "hidden");
        if (hidden.sizes().slice(0, hidden.dim() - 1) != targets.sizes())
            refuse("targets must have a number for each row of hidden ", hidden.sizes(), ", got ", targets.sizes());
    }
};

py::tuple cross_entropy_forward(const Tensor& hidden, const Tensor& table, const Tensor& targets, double scale) {
    const c10::DeviceGuard guard(hidden.device());
    const Scores s(hidden, table, targets);
    const int32_t type = code(hidden.scalar_type());
    int64_t need = 0;
    check(warp_cross_entropy_scratch(s.h.rows, s.h.cols, type, s.t.t.const_data_ptr(), s.t.stride, s.t.rows, &need, nullptr));
    const auto f32 = hidden.options().dtype(at::kFloat);
    Tensor loss = at::empty(targets.sizes(), f32), lse = at::empty(targets.sizes(), f32), scratch = scratch_of(hidden, need);
    check(warp_cross_entropy(s.h.t.const_data_ptr(), s.h.stride, s.h.rows, s.h.cols, type, s.t.t.const_data_ptr(), s.t.stride,
                             s.t.rows, s.y.const_data_ptr(), bytes_of(s.y), (float)scale, loss.data_ptr<float>(),
                             lse.data_ptr<float>(), scratch.data_ptr(), need, stream_of(hidden)));
    return py::make_tuple(loss, lse);
}

py::tuple cross_entropy(const Tensor& hidden, const Tensor& table, const Tensor& targets, double scale) {
    on_device(hidden);
    on_device(hidden, table);
    on_device(hidden, targets);
    if (followed(hidden, table))
        return node("_CrossEntropy")(hidden, table, targets, scale);
    return cross_entropy_forward(hidden, table, targets, scale);
}

py::tuple cross_entropy_backward(const Tensor& dloss, const Tensor& hidden, const Tensor& table, const Tensor& targets,
                                 const Tensor& loss, const Tensor& lse, double scale, bool want_hidden, bool want_table) {
    not_traced("cross_entropy_backward");
    on_device(hidden);
    for (const Tensor* t : {&dloss, &table, &targets, &loss, &lse}) on_device(hidden, *t);
    const c10::DeviceGuard guard(hidden.device());
    const Scores s(hidden, table, targets);
    for (const Tensor* t : {&dloss, &loss, &lse})
        if (t->sizes() != targets.sizes() || t->scalar_type() != at::kFloat)
            refuse(t == &dloss ? "dloss" : t == &loss ? "loss" : "lse", " must be float32 ", targets.sizes(), ", got ",
                   t->scalar_type(), " ", t->sizes());
    const int32_t type = code(hidden.scalar_type());
    int64_t need = 0;
    check(warp_cross_entropy_scratch(s.h.rows, s.h.cols, type, s.t.t.const_data_ptr(), s.t.stride, s.t.rows, nullptr, &need));
    const Tensor g = dloss.contiguous(), l = loss.contiguous(), e = lse.contiguous();
    MaybeTensor dh, dt;
    if (want_hidden) dh = at::empty(hidden.sizes(), hidden.options());
    if (want_table) dt = at::empty({s.t.rows, s.t.cols}, table.options());
    Tensor scratch = scratch_of(hidden, need);
    check(warp_cross_entropy_backward(g.const_data_ptr<float>(), s.h.t.const_data_ptr(), s.h.stride, s.h.rows, s.h.cols, type,
                                      s.t.t.const_data_ptr(), s.t.stride, s.t.rows, s.y.const_data_ptr(), bytes_of(s.y),
                                      (float)scale, l.const_data_ptr<float>(), e.const_data_ptr<float>(),
                                      dh ? dh->data_ptr() : nullptr, s.h.cols, dt ? dt->data_ptr() : nullptr, s.h.cols,
                                      scratch.data_ptr(), need, stream_of(hidden)));
    return py::make_tuple(dh, dt);
}

Tensor linear_forward(const Tensor& x, const Tensor& weight, const MaybeTensor& bias) {
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x"), w = matrix_of(weight, "weight", r.cols);
    same_type(weight, x, "weight", "x");
    if (w.rows < 1 || w.rows > INT32_MAX) refuse("a weight of ", w.rows, " channels");
    if (bias && (bias->dim() != 1 || bias->size(0) != w.rows ||
                 (bias->scalar_type() != at::kFloat && bias->scalar_type() != x.scalar_type())))
        refuse("bias must be float32 or ", x.scalar_type(), " (", w.rows, ",), got ", bias->scalar_type(), " ", bias->sizes());
    const int32_t type = code(x.scalar_type());
    int64_t need = 0;
    check(warp_linear_scratch(r.t.const_data_ptr(), r.stride, r.rows, r.cols, type, w.t.const_data_ptr(), w.stride,
                              (int32_t)w.rows, &need));
    const MaybeTensor b = bias ? MaybeTensor(bias->contiguous()) : std::nullopt;
    Tensor y = at::empty(with_last(x.sizes().slice(0, x.dim() - 1), w.rows), x.options()), scratch;
    if (need) scratch = scratch_of(x, need);
    check(warp_linear(r.t.const_data_ptr(), r.stride, r.rows, r.cols, type, w.t.const_data_ptr(), w.stride, (int32_t)w.rows,
                      ptr(b), bias ? code(bias->scalar_type()) : WARP_F32, y.data_ptr(), w.rows,
                      need ? scratch.data_ptr() : nullptr, need, stream_of(x)));
    return y;
}

Tensor linear(const Tensor& x, const Tensor& weight, const MaybeTensor& bias, const py::object& rows) {
    if (!rows.is_none()) not_traced("linear of given rows");
    on_device(x);
    on_device(x, weight);
    on_device(x, bias);
    if (followed(x, weight, bias))
        return node("_Linear")(x, weight, bias, rows).cast<Tensor>();
    return linear_forward(x, weight, bias);
}

// dy [..., n] for the rows `values * scale` and the weight [n, cols]
py::tuple linear_backward(const Tensor& dy, const MaybeTensor& values, const MaybeTensor& scale, const Tensor& weight,
                          bool want_x, bool want_weight, bool want_bias, at::ScalarType bias_type) {
    not_traced("linear_backward");
    on_device(dy);
    on_device(dy, weight);
    on_device(dy, values);
    on_device(dy, scale);
    const c10::DeviceGuard guard(dy.device());
    const Rows d = rows_of(dy, "dy"), w = matrix_of(weight, "weight", -1);
    same_type(weight, dy, "weight", "dy");
    if (d.cols != w.rows) refuse("dy has rows of ", d.cols, " columns for a weight of ", w.rows, " channels");
    if (want_weight) {
        check_int8("rows", *values, *scale, ((int64_t)w.cols + kPad - 1) / kPad * kPad);
        if (values->size(0) != d.rows) refuse(values->size(0), " rows in 8 bits for ", d.rows, " of dy");
    }
    if (bias_type != at::kFloat && bias_type != dy.scalar_type())
        refuse("dbias must be float32 or ", dy.scalar_type(), ", got ", bias_type);
    const int32_t type = code(dy.scalar_type());
    int64_t need = 0;
    check(warp_linear_backward_scratch(d.t.const_data_ptr(), d.stride, d.rows, d.cols, type, w.cols, w.t.const_data_ptr(),
                                       w.stride, &need));
    MaybeTensor dx, dw, db;
    if (want_x) dx = at::empty(with_last(dy.sizes().slice(0, dy.dim() - 1), w.cols), dy.options());
    if (want_weight) dw = at::empty({w.rows, w.cols}, weight.options());
    if (want_bias) db = at::empty({w.rows}, dy.options().dtype(bias_type));
    Tensor scratch;
    if (need) scratch = scratch_of(dy, need);
    check(warp_linear_backward(d.t.const_data_ptr(), d.stride, d.rows, d.cols, type,
                               want_weight ? (const int8_t*)values->const_data_ptr() : nullptr,
                               want_weight ? values->stride(0) : 0, want_weight ? scale->const_data_ptr<float>() : nullptr,
                               w.cols, w.t.const_data_ptr(), w.stride, dx ? dx->data_ptr() : nullptr, w.cols,
                               dw ? dw->data_ptr() : nullptr, w.cols, db ? db->data_ptr() : nullptr, code(bias_type),
                               need ? scratch.data_ptr() : nullptr, need, stream_of(dy)));
    return py::make_tuple(dx, dw, db);
}

// The optimizer's records (warp_adamw_tensor) in a buffer that it owns, held for one call.
struct Records {
    Py_buffer view;
    explicit Records(const py::object& table) {
        if (PyObject_GetBuffer(table.ptr(), &view, PyBUF_WRITABLE | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            refuse("the optimizer's records must be a writable array in one piece");
        }
    }
    ~Records() { PyBuffer_Release(&view); }
    Records(const Records&) = delete;
    Records& operator=(const Records&) = delete;
};

// `table`: the optimizer's records for its parameters, with sizes and moments filled in
void adamw_step(const py::list& params, const py::sequence& grads, const py::object& table, at::ScalarType dtype,
                int32_t bits, const Tensor& m, const MaybeTensor& m_scale, const Tensor& v, const MaybeTensor& v_scale,
                double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                const MaybeTensor& grad_scale) {
    not_traced("AdamW.step");
    const size_t n = params.size();
    const Records held(table);
    const size_t bytes = (size_t)held.view.len;
    if (bytes != n * sizeof(warp_adamw_tensor))
        refuse(n, " parameters, and records of ", bytes / sizeof(warp_adamw_tensor), " when the optimizer was made");
    if (py::len(grads) != n) refuse(py::len(grads), " gradients for ", n, " parameters");
    auto* records = static_cast<warp_adamw_tensor*>(held.view.buf);
    const auto device = m.device();
    const int64_t size = n ? records[n - 1].moment + (records[n - 1].n + kBlock - 1) / kBlock * kBlock : 0;
    const bool eight = bits == 8;
    for (const Tensor* t : {&m, &v})
        if (t->numel() != size || !t->is_contiguous() || !t->is_cuda() || t->device() != device ||
            t->scalar_type() != (!eight ? at::kFloat : t == &m ? at::kChar : at::kByte))
            refuse("the moments are no longer the ones that the optimizer made");
    for (const MaybeTensor* t : {&m_scale, &v_scale})
        if (eight && (!*t || (*t)->numel() != size / kBlock || !(*t)->is_contiguous() || (*t)->device() != device ||
                      (*t)->scalar_type() != at::kFloat))
            refuse("the moments' scales are no longer the ones that the optimizer made");
    at::ScalarType grad_type = at::kFloat;
    bool any = false;
    const py::object fast = py::reinterpret_steal<py::object>(PySequence_Fast(grads.ptr(), "grads must be a sequence"));
    if (!fast) throw py::error_already_set();
    for (size_t i = 0; i < n; ++i) {
        PyObject* po = PyList_GET_ITEM(params.ptr(), (Py_ssize_t)i);
        PyObject* go = PySequence_Fast_GET_ITEM(fast.ptr(), (Py_ssize_t)i);
        records[i].grad = nullptr;
        if (!THPVariable_Check(po)) refuse("parameter ", i, " is no tensor");
        const Tensor& p = THPVariable_Unpack(po);
        if (p.scalar_type() != dtype || p.device() != device || !p.is_contiguous() || p.numel() != records[i].n)
            refuse("parameters must stay contiguous tensors of their type, size and device (parameter ", i, ")");
        records[i].param = p.data_ptr();
        if (go == Py_None) continue;
        if (!THPVariable_Check(go)) refuse("gradient ", i, " is no tensor");
        const Tensor& g = THPVariable_Unpack(go);
        if (!any) grad_type = g.scalar_type();
        any = true;
        if (!known(grad_type)) refuse("gradients must be float32, float16 or bfloat16, got ", grad_type);
        if (g.scalar_type() != grad_type || g.device() != device || !g.is_contiguous() || g.sizes() != p.sizes())
            refuse("gradients must be contiguous tensors of one type and of their parameters' shapes, on ", device,
                   " (gradient ", i, ")");
        records[i].grad = g.const_data_ptr();
    }
    if (grad_scale && (grad_scale->scalar_type() != at::kFloat || grad_scale->numel() != 1 ||
                       grad_scale->device() != device))
        refuse("grad_scale must be a float32 device tensor of one element");
    const c10::DeviceGuard guard(device);
    check(warp_adamw_step(records, (int32_t)n, code(dtype), code(grad_type), bits, m.data_ptr(),
                          m_scale ? m_scale->data_ptr<float>() : nullptr, v.data_ptr(),
                          v_scale ? v_scale->data_ptr<float>() : nullptr, lr, beta1, beta2, eps, weight_decay, step,
                          (const float*)ptr(grad_scale), stream_of(m)));
    // for autograd: what was changed in place
    for (size_t i = 0; i < n; ++i) {
        const Tensor& p = THPVariable_Unpack(PyList_GET_ITEM(params.ptr(), (Py_ssize_t)i));
        if (records[i].grad && !p.is_inference()) p.unsafeGetTensorImpl()->bump_version();
    }
}

py::tuple adamw_moments(const Tensor& m, const Tensor& m_scale, const Tensor& v, const Tensor& v_scale) {
    not_traced("AdamW.moments");
    on_device(m);
    for (const Tensor* t : {&m_scale, &v, &v_scale}) on_device(m, *t);
    if (m.scalar_type() != at::kChar || v.scalar_type() != at::kByte || m_scale.scalar_type() != at::kFloat ||
        v_scale.scalar_type() != at::kFloat || v.numel() != m.numel() || m_scale.numel() * kBlock != m.numel() ||
        v_scale.numel() * kBlock != m.numel() || !m.is_contiguous() || !v.is_contiguous() || !m_scale.is_contiguous() ||
        !v_scale.is_contiguous())
        refuse("the moments are no longer the ones that the optimizer made");
    const c10::DeviceGuard guard(m.device());
    const auto f32 = m_scale.options();
    Tensor out_m = at::empty({m.numel()}, f32), out_v = at::empty({m.numel()}, f32);
    check(warp_adamw_moments((const int8_t*)m.const_data_ptr(), m_scale.const_data_ptr<float>(),
                             (const uint8_t*)v.const_data_ptr(), v_scale.const_data_ptr<float>(), m.numel(),
                             out_m.data_ptr<float>(), out_v.data_ptr<float>(), stream_of(m)));
    return py::make_tuple(out_m, out_v);
}

}  // namespace

PYBIND11_MODULE(_encoder, mod) {
    mod.def("layer_norm", &layer_norm);
    mod.def("layer_norm_forward", &layer_norm_forward);
    mod.def("layer_norm_backward", &layer_norm_backward);
    mod.def("quantize_rows", &quantize_rows);
    mod.def("quantize_rows_forward", &quantize_rows_forward);
    mod.def("layer_norm_int8", &layer_norm_int8);
    mod.def("linear_int8", &linear_int8);
    mod.def("has_tangent", [](const Tensor& t) { return has_tangent(t); });
    mod.def("adds_on_default_stream", &adds_on_default_stream);
    mod.def("embedding", &embedding);
    mod.def("embedding_forward", &embedding_forward);
    mod.def("embedding_backward", &embedding_backward);
    mod.def("cross_entropy", &cross_entropy);
    mod.def("cross_entropy_forward", &cross_entropy_forward);
    mod.def("cross_entropy_backward", &cross_entropy_backward);
    mod.def("linear", &linear);
    mod.def("linear_forward", &linear_forward);
    mod.def("linear_backward", &linear_backward);
    mod.def("adamw_step", &adamw_step);
    mod.def("adamw_moments", &adamw_moments);
}
