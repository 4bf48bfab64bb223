// The Python binding of the token encoder's operators: checks torch tensors, allocates outputs and calls the C
// functions of warp.h on the current stream of the tensors' device. Native because a small call's time is the host's:
// layer norm of 32 rows takes 10.2 us through ctypes and 6 us through this, 3.5 us of either being the launch.
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

py::tuple layer_norm(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
    on_device(x);
    on_device(x, weight);
    on_device(x, bias);
    // autograd's node, which calls this again with gradients off
    if (at::GradMode::is_enabled() && (x.requires_grad() || tracked(weight) || tracked(bias)))
        return py::module_::import("paper_2501_17788_amd.encoder").attr("_LayerNorm").attr("apply")(x, weight, bias, eps);
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

py::tuple layer_norm_backward(const Tensor& dy, const Tensor& x, const MaybeTensor& weight, const Tensor& mean,
                              const Tensor& rstd) {
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

py::tuple quantize_rows(const Tensor& x) {
    on_device(x);
    const c10::DeviceGuard guard(x.device());
    const Rows r = rows_of(x, "x");
    auto [q, scale] = int8_rows(r);
    check(warp_quantize_rows(r.t.const_data_ptr(), r.stride, r.rows, r.cols, code(x.scalar_type()),
                             (int8_t*)q.data_ptr(), q.size(1), scale.data_ptr<float>(), stream_of(x)));
    return py::make_tuple(q, scale, r.cols);
}

py::tuple layer_norm_int8(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
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
    mod.def("layer_norm_backward", &layer_norm_backward);
    mod.def("quantize_rows", &quantize_rows);
    mod.def("layer_norm_int8", &layer_norm_int8);
    mod.def("linear_int8", &linear_int8);
    mod.def("adamw_step", &adamw_step);
    mod.def("adamw_moments", &adamw_moments);
}
