// The operators on token states for torch tensors: checks of arguments, results and workspaces from torch's allocator, descriptors for the C ABI.
//
// A call on a short sentence lasts as long as the host needs for it: attention of one sentence took 10.8 us with all of this in Python, and takes 6.0;
// layer norm 10.0 and 6.1, the mean 7.5 and 4.5, of which a launch is 2 to 3.  Functions take (context, device, stream, ...); they raise ValueError for tensors that do not fit, and return the status of a library call
// that refuses the rest.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <limits>

#include "he.h"

namespace {

using at::Tensor;

struct Refusal {
    std::string text;
};
template <class... A> [[noreturn]] void refuse(const A &...a) { throw Refusal{c10::str(a...)}; }

template <class F> PyObject *guarded(F f)
{
    HANDLE_TH_ERRORS
    try {
        at::AutoDispatchBelowADInplaceOrView raw; // results have no history: the differentiable functions are elsewhere
        return f();
    } catch (const Refusal &r) {
        PyErr_SetString(PyExc_ValueError, r.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// The arguments of a call, in order.
struct Args {
    PyObject *const *at;
    he_ctx *ctx;
    int device;
    void *stream;
    Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want)
    {
        if (n != want) refuse(n, " arguments, want ", want);
        ctx = (he_ctx *)PyLong_AsVoidPtr(args[0]);
        device = (int)PyLong_AsLong(args[1]);
        stream = PyLong_AsVoidPtr(args[2]);
        at = args + 3;
        if (PyErr_Occurred()) throw python_error();
    }
};
bool none(PyObject *o) { return o == Py_None; }
double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
const Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) refuse(what, ": want a tensor");
    return THPVariable_Unpack(o);
}

int32_t type_of(at::ScalarType t)
{
    if (t == at::kFloat) return HE_F32;
    if (t == at::kHalf) return HE_F16;
    if (t == at::kBFloat16) return HE_BF16;
    refuse(t, ": rows are float32, float16 or bfloat16");
}

void placed(const Args &a, const Tensor &t, const char *what, at::ScalarType type)
{
    if (t.layout() != at::kStrided || t.is_neg()) refuse(what, ": want a strided tensor that holds its values as they are");
    if (a.device < 0 || !t.is_cuda() || t.get_device() != a.device) refuse(what, ": on ", t.device(), ", the context is on device ", a.device);
    if (t.scalar_type() != type) refuse(what, ": ", t.scalar_type(), ", want ", type);
}

// [rows][width], dense along the width
he_rows rows_of(const Args &a, const Tensor &t, const char *what, at::IntArrayRef shape, at::ScalarType type)
{
    if (shape.size() != 2 || t.sizes() != shape) refuse(what, ": ", t.sizes(), ", want [rows][width]", shape.size() == 2 ? c10::str(" = ", shape) : "");
    placed(a, t, what, type);
    if (t.stride(1) != 1 && shape[1] > 1) refuse(what, ": want rows that are dense along the width");
    return {t.data_ptr(), shape[0] > 1 ? t.stride(0) : shape[1]};
}
void *vector_of(const Args &a, const Tensor &t, const char *what, int64_t n, at::ScalarType type)
{
    if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) refuse(what, ": ", t.sizes(), ", want a dense vector of ", n);
    placed(a, t, what, type);
    return t.data_ptr();
}
// [rows][heads][dim] with a dense last dimension, at multiples of 16 bytes; the stride of one row or one head, which may be any number, is none
he_heads heads_of(const Args &a, const Tensor &t, const char *what, at::IntArrayRef shape, at::ScalarType type)
{
    if (shape.size() != 3 || t.sizes() != shape) refuse(what, ": ", t.sizes(), ", want [rows][heads][dim]", shape.size() == 3 ? c10::str(" = ", shape) : "");
    placed(a, t, what, type);
    if (t.stride(2) != 1 && shape[2] > 1) refuse(what, ": the last dimension is not dense");
    void *const p = t.data_ptr();
    const int64_t row = shape[0] > 1 ? t.stride(0) : 0, head = shape[1] > 1 ? t.stride(1) : 0;
    if ((((int64_t)p | (row | head) * (int64_t)t.element_size()) & 15) && t.numel())
        refuse(what, ": address ", p, " or strides ", t.strides(), " not in multiples of 16 bytes");
    return {p, row, head};
}
// a vector of count + 1 offsets, or a pair of vectors (begin, end)
he_spans spans_of(const Args &a, PyObject *o, int64_t rows, const char *what)
{
    constexpr int64_t most = std::numeric_limits<int32_t>::max();
    const auto count_of = [&](const Tensor &t, int64_t less) {
        if (t.dim() != 1 || t.size(0) < less || t.size(0) > most) refuse(what, ": want a vector of count + 1 offsets, or a pair of vectors (begin, end)");
        return t.size(0) - less;
    };
    if (PyTuple_Check(o) || PyList_Check(o)) {
        if (PySequence_Size(o) != 2) refuse(what, ": want a pair (begin, end)");
        const Tensor &b = tensor(PyTuple_Check(o) ? PyTuple_GET_ITEM(o, 0) : PyList_GET_ITEM(o, 0), what);
        const Tensor &e = tensor(PyTuple_Check(o) ? PyTuple_GET_ITEM(o, 1) : PyList_GET_ITEM(o, 1), what);
        const int64_t n = count_of(b, 0);
        return {(const int32_t *)vector_of(a, b, what, n, at::kInt), (const int32_t *)vector_of(a, e, what, n, at::kInt), (int32_t)n, rows};
    }
    const Tensor &t = tensor(o, what);
    const int64_t n = count_of(t, 1);
    const int32_t *p = (const int32_t *)vector_of(a, t, what, n + 1, at::kInt);
    return {p, p + 1, (int32_t)n, rows};
}

// A buffer of the caller's to write to: autograd has no part in that, so one that it tracks is refused where it is switched on, ..
const Tensor &out_of(PyObject *o, const char *what)
{
    const Tensor &t = tensor(o, what);
    if (t.requires_grad() && c10::GradMode::is_enabled()) refuse(what, ": buffers to write to must not require gradients");
    return t;
}
// .. and one that it may have saved gets another version, so that it notices.
void written(const Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// What a call reads or writes: n[0] x n[1] pieces of `bytes`, step[0] and step[1] apart.
struct Part {
    int64_t at, bytes, n[2], step[2];
    // the last dimension is one piece; a step that is never taken is 0
    explicit Part(const Tensor &t) : at((int64_t)t.data_ptr()), bytes(t.element_size()), n{1, 1}, step{0, 0}
    {
        const int64_t size = t.element_size(), d = t.dim();
        bytes = t.numel() ? t.size(d - 1) * size : 0;
        for (int64_t i = 0; i + 1 < d; i++)
            if (t.size(i) > 1 && t.stride(i)) n[i] = t.size(i), step[i] = t.stride(i) * size;
    }
    int64_t end() const { return at + (n[0] - 1) * step[0] + (n[1] - 1) * step[1] + bytes; }
};
// Whether two of them share an address.  Rows of the same step, as the parts of one buffer have, are looked at head by head; rows of different steps
// in one place are taken to overlap.
bool overlap(const Part &a, const Part &b)
{
    if (!a.bytes || !b.bytes || a.end() <= b.at || b.end() <= a.at) return false;
    const int64_t step = a.step[0] ? a.step[0] : b.step[0], lowest = 1 - b.n[0], highest = a.n[0] - 1; // of the row of a minus the row of b
    if (a.step[0] && b.step[0] && a.step[0] != b.step[0]) return true;
    const auto near = [&](int64_t d) { // a row d bytes from its place in b's rows: d + i step in (-a.bytes, b.bytes) for some i
        if (!step) return d > -a.bytes && d < b.bytes;
        const int64_t low = -a.bytes + 1 - d, i = std::max(low >= 0 ? (low + step - 1) / step : -(-low / step), lowest);
        return i <= highest && d + i * step < b.bytes;
    };
    const int64_t d = a.at - b.at;
    if (a.step[1] == b.step[1] || !a.step[1] || !b.step[1]) { // heads of one step: by their differences
        const int64_t head = a.step[1] ? a.step[1] : b.step[1];
        for (int64_t j = 1 - b.n[1]; j < a.n[1]; j++)
            if (near(d + j * head)) return true;
        return false;
    }
    for (int64_t i = 0; i < a.n[1]; i++)
        for (int64_t j = 0; j < b.n[1]; j++)
            if (near(d + i * a.step[1] - j * b.step[1])) return true;
    return false;
}
// A buffer of the caller's and what the same call reads, or writes as well.  (One that repeats itself is for the library to refuse.)
void apart(const Tensor &out, const char *what, std::initializer_list<PyObject *> others)
{
    for (int64_t i = 0; i < out.dim(); i++)
        if (out.size(i) > 1 && !out.stride(i)) return;
    const Part p(out);
    for (PyObject *o : others)
        if (!none(o) && overlap(p, Part(THPVariable_Unpack(o)))) refuse(what, ": the buffer overlaps another tensor of the call");
}

Tensor dense(at::IntArrayRef shape, const Tensor &like, at::ScalarType type) { return at::empty(shape, like.options().dtype(type)); }
// A workspace of this call's own, from torch's allocator: calls on other streams and captured graphs have theirs.
Tensor scratch(const Tensor &like, size_t bytes) { return bytes ? dense({(int64_t)(bytes + 3) / 4}, like, at::kFloat) : Tensor(); }
void *address(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

PyObject *status(int32_t rc) { return PyLong_FromLong(rc); }
template <class... P> PyObject *pack(P... p)
{
    PyObject *const items[] = {p...}, *const t = PyTuple_New(sizeof...(p));
    for (size_t i = 0; i < sizeof...(p); i++) PyTuple_SET_ITEM(t, i, items[i]);
    return t;
}
PyObject *wrap(Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *same(PyObject *o)
{
    Py_INCREF(o);
    return o;
}

// x, weight, bias, residual, eps, out
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 9);
        const Tensor &x = tensor(a.at[0], "x"), &w = tensor(a.at[1], "weight"), &b = tensor(a.at[2], "bias");
        const at::ScalarType type = x.scalar_type();
        he_norm n{type_of(type), 0, 0, 0, number(a.at[4])};
        const he_rows xr = rows_of(a, x, "x", x.sizes(), type);
        const int64_t rows = x.size(0), width = x.size(1);
        if (width > INT32_MAX) refuse("x: ", x.sizes(), ", rows are too wide");
        n.weight_type = type_of(w.scalar_type()), n.rows = rows, n.width = (int32_t)width;
        const void *wp = vector_of(a, w, "weight", width, w.scalar_type()), *bp = vector_of(a, b, "bias", width, w.scalar_type());
        he_rows rr{}, sr{}, yr;
        Tensor s, y;
        const bool residual = !none(a.at[3]);
        if (residual) {
            rr = rows_of(a, tensor(a.at[3], "residual"), "residual", x.sizes(), type);
            s = dense(x.sizes(), x, type);
            sr = {s.data_ptr(), width};
        }
        if (none(a.at[5])) {
            y = dense(x.sizes(), x, type);
            yr = {y.data_ptr(), width};
        } else {
            const Tensor &out = out_of(a.at[5], "out");
            yr = rows_of(a, out, "out", x.sizes(), type);
            apart(out, "out", {a.at[0], a.at[1], a.at[2], a.at[3]});
        }
        Tensor mean = dense({rows}, x, at::kFloat), rstd = dense({rows}, x, at::kFloat);
        const int32_t rc = he_layer_norm(a.ctx, &n, &xr, residual ? &rr : nullptr, wp, bp, &yr, residual ? &sr : nullptr, (float *)mean.data_ptr(),
                                         (float *)rstd.data_ptr(), a.stream);
        if (rc != HE_OK) return status(rc);
        if (!y.defined()) written(tensor(a.at[5], "out"));
        return pack(y.defined() ? wrap(y) : same(a.at[5]), residual ? wrap(s) : same(a.at[0]), wrap(mean), wrap(rstd));
    });
}

// dy, s, weight, mean, rstd, ds
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 9);
        const Tensor &s = tensor(a.at[1], "s"), &w = tensor(a.at[2], "weight");
        const at::ScalarType type = s.scalar_type(), wt = w.scalar_type();
        he_norm n{type_of(type), type_of(wt), 0, 0, 0.0};
        const he_rows sr = rows_of(a, s, "s", s.sizes(), type), dyr = rows_of(a, tensor(a.at[0], "dy"), "dy", s.sizes(), type);
        const int64_t rows = s.size(0), width = s.size(1);
        if (width > INT32_MAX) refuse("s: ", s.sizes(), ", rows are too wide");
        n.rows = rows, n.width = (int32_t)width;
        he_rows ar{};
        if (!none(a.at[5])) ar = rows_of(a, tensor(a.at[5], "ds"), "ds", s.sizes(), type);
        const void *wp = vector_of(a, w, "weight", width, wt);
        const float *mean = (const float *)vector_of(a, tensor(a.at[3], "mean"), "mean", rows, at::kFloat);
        const float *rstd = (const float *)vector_of(a, tensor(a.at[4], "rstd"), "rstd", rows, at::kFloat);
        size_t need = 0;
        if (const int32_t rc = he_layer_norm_workspace_bytes(a.ctx, &n, &need)) return status(rc);
        Tensor dx = dense(s.sizes(), s, type), dw = dense({width}, w, wt), db = dense({width}, w, wt);
        const Tensor ws = scratch(s, need);
        const he_rows xr{dx.data_ptr(), width};
        const int32_t rc = he_layer_norm_grad(a.ctx, &n, &dyr, &sr, wp, mean, rstd, none(a.at[5]) ? nullptr : &ar, &xr, dw.data_ptr(), db.data_ptr(),
                                              address(ws), need, a.stream);
        if (rc != HE_OK) return status(rc);
        return pack(wrap(dx), wrap(dw), wrap(db));
    });
}

// x, weight, residual and eps, as both forms of the root-mean-square norm take them; the residual sum
struct Rms {
    he_norm n;
    he_rows x, r, sum;
    const void *w;
    bool residual;
    Tensor s;
    at::ScalarType type;
    Rms(const Args &a, PyObject *const *in) : r{}, sum{}
    {
        const Tensor &tx = tensor(in[0], "x"), &tw = tensor(in[1], "weight");
        type = tx.scalar_type();
        n = {type_of(type), 0, 0, 0, number(in[3])};
        x = rows_of(a, tx, "x", tx.sizes(), type);
        if (tx.size(1) > INT32_MAX) refuse("x: ", tx.sizes(), ", rows are too wide");
        n.weight_type = type_of(tw.scalar_type()), n.rows = tx.size(0), n.width = (int32_t)tx.size(1);
        w = vector_of(a, tw, "weight", n.width, tw.scalar_type());
        residual = !none(in[2]);
        if (residual) {
            r = rows_of(a, tensor(in[2], "residual"), "residual", tx.sizes(), type);
            s = dense(tx.sizes(), tx, type);
            sum = {s.data_ptr(), n.width};
        }
    }
    PyObject *kept(PyObject *x) { return residual ? wrap(s) : same(x); }
};
// 8-bit rows that begin at multiples of 64 bytes, so that products read them by whole lines, and their scales: two views of one allocation, which takes 0.7 us
// less than two.
struct Eight {
    Tensor rows, scale;
    he_rows8 d;
    Eight(const Tensor &like, int64_t n, int64_t width)
    {
        const int64_t stride = (width + 63) / 64 * 64;
        const Tensor all = dense({n * (stride + 4)}, like, at::kChar);
        const auto part = [&](at::IntArrayRef sizes, at::IntArrayRef strides, at::ScalarType type, int64_t offset) {
            Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(type));
            t.unsafeGetTensorImpl()->set_sizes_and_strides(sizes, strides, offset);
            return t;
        };
        rows = part({n, width}, {stride, 1}, at::kChar, 0);
        scale = part({n}, {1}, at::kFloat, n * stride / 4);
        d = {(int8_t *)rows.data_ptr(), stride, (float *)scale.data_ptr()};
    }
};
// 8-bit rows that a product reads, by pieces of 16 bytes
he_rows8 eight_of(const Args &a, const Tensor &t, const char *what, const Tensor &scale, const char *what_scale)
{
    if (t.dim() != 2) refuse(what, ": ", t.sizes(), ", want [rows][width]");
    const he_rows r = rows_of(a, t, what, t.sizes(), at::kChar);
    const int64_t rows = t.size(0), width = t.size(1), stride = rows > 1 ? r.stride : (width + 15) / 16 * 16;
    if (((int64_t)r.d & 15 || stride % 16) && t.numel()) refuse(what, ": address ", r.d, " or stride ", stride, " is not a multiple of 16");
    if (t.numel() && t.storage().nbytes() < (size_t)(t.storage_offset() + (rows - 1) * stride + (width + 15) / 16 * 16))
        refuse(what, ": the buffer ends inside a piece of 16 bytes of the last row");
    return {(int8_t *)r.d, stride, (float *)vector_of(a, scale, what_scale, rows, at::kFloat)};
}

// x, weight, residual, eps, out
PyObject *rms_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 8);
        Rms t(a, a.at);
        const Tensor &x = tensor(a.at[0], "x");
        Tensor y;
        he_rows yr;
        if (none(a.at[4])) {
            y = dense(x.sizes(), x, t.type);
            yr = {y.data_ptr(), t.n.width};
        } else {
            const Tensor &out = out_of(a.at[4], "out");
            yr = rows_of(a, out, "out", x.sizes(), t.type);
            apart(out, "out", {a.at[0], a.at[1], a.at[2]});
        }
        Tensor rstd = dense({t.n.rows}, x, at::kFloat);
        const int32_t rc = he_rms_norm(a.ctx, &t.n, &t.x, t.residual ? &t.r : nullptr, t.w, &yr, t.residual ? &t.sum : nullptr, (float *)rstd.data_ptr(), a.stream);
        if (rc != HE_OK) return status(rc);
        if (!y.defined()) written(tensor(a.at[4], "out"));
        return pack(y.defined() ? wrap(y) : same(a.at[4]), t.kept(a.at[0]), wrap(rstd));
    });
}

// dy, s, weight, rstd, ds
PyObject *rms_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 8);
        const Tensor &s = tensor(a.at[1], "s"), &w = tensor(a.at[2], "weight");
        const at::ScalarType type = s.scalar_type(), wt = w.scalar_type();
        he_norm n{type_of(type), type_of(wt), 0, 0, 0.0};
        const he_rows sr = rows_of(a, s, "s", s.sizes(), type), dyr = rows_of(a, tensor(a.at[0], "dy"), "dy", s.sizes(), type);
        const int64_t rows = s.size(0), width = s.size(1);
        if (width > INT32_MAX) refuse("s: ", s.sizes(), ", rows are too wide");
        n.rows = rows, n.width = (int32_t)width;
        he_rows ar{};
        if (!none(a.at[4])) ar = rows_of(a, tensor(a.at[4], "ds"), "ds", s.sizes(), type);
        const void *wp = vector_of(a, w, "weight", width, wt);
        const float *rstd = (const float *)vector_of(a, tensor(a.at[3], "rstd"), "rstd", rows, at::kFloat);
        size_t need = 0;
        if (const int32_t rc = he_rms_norm_workspace_bytes(a.ctx, &n, &need)) return status(rc);
        Tensor dx = dense(s.sizes(), s, type), dw = dense({width}, w, wt);
        const Tensor ws = scratch(s, need);
        const he_rows xr{dx.data_ptr(), width};
        const int32_t rc = he_rms_norm_grad(a.ctx, &n, &dyr, &sr, wp, rstd, none(a.at[4]) ? nullptr : &ar, &xr, dw.data_ptr(), address(ws), need, a.stream);
        if (rc != HE_OK) return status(rc);
        return pack(wrap(dx), wrap(dw));
    });
}

// x, weight, residual, eps
PyObject *rms_norm8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 7);
        Rms t(a, a.at);
        Eight y(tensor(a.at[0], "x"), t.n.rows, t.n.width);
        const int32_t rc = he_rms_norm8(a.ctx, &t.n, &t.x, t.residual ? &t.r : nullptr, t.w, &y.d, t.residual ? &t.sum : nullptr, a.stream);
        if (rc != HE_OK) return status(rc);
        return pack(wrap(y.rows), wrap(y.scale), t.kept(a.at[0]));
    });
}

// x, gelu
PyObject *quantize8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 5);
        const Tensor &x = tensor(a.at[0], "x");
        const int gelu = PyObject_IsTrue(a.at[1]);
        if (gelu < 0) throw python_error();
        const int32_t type = type_of(x.scalar_type());
        const he_rows xr = rows_of(a, x, "x", x.sizes(), x.scalar_type());
        if (x.size(1) > INT32_MAX) refuse("x: ", x.sizes(), ", rows are too wide");
        Eight y(x, x.size(0), x.size(1));
        const int32_t rc = he_quantize8(a.ctx, type, x.size(0), (int32_t)x.size(1), gelu, &xr, &y.d, a.stream);
        if (rc != HE_OK) return status(rc);
        return pack(wrap(y.rows), wrap(y.scale));
    });
}

// x8, scale, w8, w_scale, bias, dtype, out
PyObject *linear8(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 10);
        const Tensor &x = tensor(a.at[0], "x8"), &w = tensor(a.at[2], "w8");
        const he_rows8 xr = eight_of(a, x, "x8", tensor(a.at[1], "scale"), "scale"), wr = eight_of(a, w, "w8", tensor(a.at[3], "w_scale"), "w_scale");
        const int64_t rows = x.size(0), width = x.size(1), channels = w.size(0), shape[2] = {rows, channels};
        if (w.size(1) != width) refuse("w8: ", w.sizes(), ", want [channels][", width, "]");
        if (width > INT32_MAX || channels > INT32_MAX) refuse("w8: ", w.sizes(), " is too large");
        if (!none(a.at[5]) && !THPDtype_Check(a.at[5])) refuse("dtype: want a torch.dtype");
        const at::ScalarType dtype = !none(a.at[5]) ? ((THPDtype *)a.at[5])->scalar_type : none(a.at[6]) ? at::kBFloat16 : tensor(a.at[6], "out").scalar_type();
        he_product8 p{type_of(dtype), HE_F32, rows, (int32_t)width, (int32_t)channels};
        const void *bias = nullptr;
        if (!none(a.at[4])) {
            const Tensor &b = tensor(a.at[4], "bias");
            p.bias_type = type_of(b.scalar_type());
            bias = vector_of(a, b, "bias", channels, b.scalar_type());
        }
        Tensor o;
        he_rows orows;
        if (none(a.at[6])) {
            o = dense(shape, x, dtype);
            orows = {o.data_ptr(), channels};
        } else {
            const Tensor &out = out_of(a.at[6], "out");
            orows = rows_of(a, out, "out", shape, dtype);
            apart(out, "out", {a.at[0], a.at[1], a.at[2], a.at[3], a.at[4]});
        }
        const int32_t rc = he_linear8(a.ctx, &p, &xr, &wr, bias, &orows, a.stream);
        if (rc != HE_OK) return status(rc);
        if (o.defined()) return wrap(o);
        written(tensor(a.at[6], "out"));
        return same(a.at[6]);
    });
}

// x, offsets, out
PyObject *pool_mean(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 6);
        const Tensor &x = tensor(a.at[0], "x");
        const int32_t type = type_of(x.scalar_type());
        const he_rows xr = rows_of(a, x, "x", x.sizes(), x.scalar_type());
        const int64_t width = x.size(1);
        if (width > INT32_MAX) refuse("x: ", x.sizes(), ", rows are too wide");
        const he_spans sp = spans_of(a, a.at[1], x.size(0), "offsets");
        Tensor e;
        if (none(a.at[2]))
            e = dense({sp.count, width}, x, at::kFloat);
        else {
            e = out_of(a.at[2], "out");
            if (e.dim() != 2 || e.size(0) != sp.count || e.size(1) != width || !e.is_contiguous())
                refuse("out: ", e.sizes(), ", want a dense [", sp.count, "][", width, "]");
            placed(a, e, "out", at::kFloat);
            apart(e, "out", {a.at[0]});
        }
        // most calls take no workspace, and one that does says so before it enqueues anything
        int32_t rc = he_pool(a.ctx, type, &sp, (int32_t)width, &xr, (float *)e.data_ptr(), nullptr, 0, a.stream);
        if (rc == HE_EWORKSPACE) {
            size_t need = 0;
            if (const int32_t bad = he_pool_workspace_bytes(a.ctx, &sp, (int32_t)width, &need)) return status(bad);
            const Tensor ws = scratch(x, need);
            rc = he_pool(a.ctx, type, &sp, (int32_t)width, &xr, (float *)e.data_ptr(), address(ws), need, a.stream);
        }
        if (rc != HE_OK) return status(rc);
        if (none(a.at[2])) return wrap(e);
        written(e);
        return same(a.at[2]);
    });
}

// de, offsets, rows, dtype, out
PyObject *pool_mean_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 8);
        const Tensor &de = tensor(a.at[0], "de");
        const int64_t rows = PyLong_AsLongLong(a.at[2]);
        if (PyErr_Occurred()) throw python_error();
        if (rows < 0) refuse("rows: ", rows);
        if (!THPDtype_Check(a.at[3])) refuse("dtype: want a torch.dtype");
        const at::ScalarType dtype = ((THPDtype *)a.at[3])->scalar_type;
        const int32_t type = type_of(dtype);
        const he_spans sp = spans_of(a, a.at[1], rows, "offsets");
        if (de.dim() != 2 || de.size(0) != sp.count || !de.is_contiguous() || de.size(1) > INT32_MAX)
            refuse("de: ", de.sizes(), ", want a dense [", sp.count, "][width]");
        placed(a, de, "de", at::kFloat);
        const int64_t width = de.size(1), shape[2] = {rows, width};
        Tensor dx;
        he_rows xr;
        const bool fill = none(a.at[4]);
        if (fill) {
            dx = dense(shape, de, dtype);
            if (!sp.count) dx.zero_(); // the library writes nothing without sequences
            xr = {dx.data_ptr(), width};
        } else {
            const Tensor &out = out_of(a.at[4], "out");
            xr = rows_of(a, out, "out", shape, dtype);
            apart(out, "out", {a.at[0]});
        }
        const int32_t rc = he_pool_grad(a.ctx, type, &sp, (int32_t)width, (const float *)de.data_ptr(), &xr, fill, a.stream);
        if (rc != HE_OK) return status(rc);
        if (fill) return wrap(dx);
        written(tensor(a.at[4], "out"));
        return same(a.at[4]);
    });
}

// What both passes of attention take: q, k, v; offsets, offsets_k, scale, cap, slopes.
struct Attention {
    he_attn s;
    he_heads q, k, v;
    at::ScalarType type;
    Attention(const Args &a, PyObject *const *qkv, PyObject *const *rest)
    {
        const Tensor &tq = tensor(qkv[0], "q"), &tk = tensor(qkv[1], "k"), &tv = tensor(qkv[2], "v");
        memset(&s, 0, sizeof(s));
        type = tq.scalar_type();
        s.type = type_of(type);
        q = heads_of(a, tq, "q", tq.sizes(), type);
        const int64_t rows = tq.size(0), heads = tq.size(1), dim = tq.size(2);
        if (tk.dim() != 3 || tk.size(2) != dim) refuse("k: ", tk.sizes(), ", want [rows][heads][", dim, "]");
        k = heads_of(a, tk, "k", tk.sizes(), type);
        v = heads_of(a, tv, "v", tk.sizes(), type);
        const int64_t rows_k = tk.size(0), kv = tk.size(1);
        if (kv == 0 || heads % kv) refuse(heads, " query heads on ", kv, " key heads");
        if (heads > INT32_MAX || dim > INT32_MAX) refuse("q: ", tq.sizes(), " is too large");
        s.heads = (int32_t)heads, s.kv_heads = (int32_t)kv, s.dim = (int32_t)dim;
        s.q = spans_of(a, rest[0], rows, "offsets");
        s.k = s.q, s.k.rows = rows_k;
        if (!none(rest[1])) {
            s.k = spans_of(a, rest[1], rows_k, "offsets_k");
            if (s.k.count != s.q.count) refuse("offsets and offsets_k: another number of sequences");
        } else if (rows_k != rows)
            refuse("keys of another length than the queries need offsets_k");
        s.scale = none(rest[2]) ? 1.0 / std::sqrt((double)dim) : number(rest[2]);
        s.cap = number(rest[3]);
        if (!none(rest[4])) s.d_slopes = (const float *)vector_of(a, tensor(rest[4], "slopes"), "slopes", heads, at::kFloat);
    }
};
he_heads dense_heads(const Tensor &t) { return {t.data_ptr(), t.size(1) * t.size(2), t.size(2)}; }

// q, k, v, offsets, offsets_k, scale, cap, slopes, out
PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 12);
        Attention t(a, a.at, a.at + 3);
        const Tensor &q = tensor(a.at[0], "q");
        const bool made = none(a.at[8]);
        t.s.fill = made;
        Tensor lse = dense({q.size(1), q.size(0)}, q, at::kFloat), o;
        he_heads oh;
        if (made) {
            o = dense(q.sizes(), q, t.type);
            oh = dense_heads(o);
        } else {
            const Tensor &out = out_of(a.at[8], "out");
            oh = heads_of(a, out, "out", q.sizes(), t.type);
            apart(out, "out", {a.at[0], a.at[1], a.at[2], a.at[7]});
        }
        if (!made || !t.s.q.count) lse.fill_(-std::numeric_limits<float>::infinity()); // rows that the library leaves as they are
        if (made && !t.s.q.count) o.zero_();
        // most calls take no workspace, and one that does says so before it enqueues anything
        int32_t rc = he_attention(a.ctx, &t.s, &t.q, &t.k, &t.v, &oh, (float *)lse.data_ptr(), nullptr, 0, a.stream);
        if (rc == HE_EWORKSPACE) {
            size_t need = 0;
            if (const int32_t bad = he_attention_workspace_bytes(a.ctx, &t.s, 0, &need)) return status(bad);
            const Tensor ws = scratch(q, need);
            rc = he_attention(a.ctx, &t.s, &t.q, &t.k, &t.v, &oh, (float *)lse.data_ptr(), address(ws), need, a.stream);
        }
        if (rc != HE_OK) return status(rc);
        if (!made) written(tensor(a.at[8], "out"));
        return pack(made ? wrap(o) : same(a.at[8]), wrap(lse));
    });
}

// do, q, k, v, o, lse, offsets, offsets_k, scale, cap, slopes, out (a tuple of three or None), fill
PyObject *attention_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded([&]() -> PyObject * {
        const Args a(args, nargs, 16);
        Attention t(a, a.at + 1, a.at + 6);
        const Tensor &q = tensor(a.at[1], "q"), &k = tensor(a.at[2], "k"), &lse = tensor(a.at[5], "lse");
        const bool made = none(a.at[11]);
        const int fill = PyObject_IsTrue(a.at[12]);
        if (fill < 0) throw python_error();
        t.s.fill = fill;
        const he_heads gh = heads_of(a, tensor(a.at[0], "do"), "do", q.sizes(), t.type), oh = heads_of(a, tensor(a.at[4], "o"), "o", q.sizes(), t.type);
        if (lse.dim() != 2 || lse.size(0) != q.size(1) || lse.size(1) != q.size(0) || !lse.is_contiguous())
            refuse("lse: ", lse.sizes(), ", want a dense [heads][rows]");
        placed(a, lse, "lse", at::kFloat);
        static const char *const names[3] = {"dq", "dk", "dv"};
        Tensor d[3];
        he_heads g[3];
        if (!made && (!PyTuple_Check(a.at[11]) || PyTuple_GET_SIZE(a.at[11]) != 3)) refuse("out: want dq, dk and dv");
        for (int i = 0; i < 3; i++) {
            const Tensor &like = i ? k : q;
            d[i] = made ? dense(like.sizes(), like, t.type) : out_of(PyTuple_GET_ITEM(a.at[11], i), names[i]);
            g[i] = made ? dense_heads(d[i]) : heads_of(a, d[i], names[i], like.sizes(), t.type);
        }
        if (!made)
            for (int i = 0; i < 3; i++) {
                apart(d[i], names[i], {a.at[0], a.at[1], a.at[2], a.at[3], a.at[4], a.at[5], a.at[10]});
                for (int j = 0; j < i; j++) apart(d[i], names[i], {PyTuple_GET_ITEM(a.at[11], j)});
            }
        if (fill && !t.s.q.count) // the library writes nothing without sequences
            for (Tensor &x : d) x.zero_();
        size_t need = 0;
        if (const int32_t rc = he_attention_workspace_bytes(a.ctx, &t.s, 1, &need)) return status(rc);
        const Tensor ws = scratch(q, need);
        const int32_t rc = he_attention_grad(a.ctx, &t.s, &gh, &t.q, &t.k, &t.v, &oh, (const float *)lse.data_ptr(), &g[0], &g[1], &g[2], address(ws), need,
                                             a.stream);
        if (rc != HE_OK) return status(rc);
        if (!made)
            for (const Tensor &x : d) written(x);
        return made ? pack(wrap(d[0]), wrap(d[1]), wrap(d[2])) : same(a.at[11]);
    });
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(layer_norm), ENTRY(layer_norm_backward), ENTRY(pool_mean), ENTRY(pool_mean_backward),
                         ENTRY(attention),  ENTRY(attention_backward),  ENTRY(rms_norm), ENTRY(rms_norm_backward),
                         ENTRY(rms_norm8),  ENTRY(quantize8),           ENTRY(linear8),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "he_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit_he_tensors(void) { return PyModule_Create(&module); }
