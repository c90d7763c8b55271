// Python calls of the operators around the masked layers (layer norm, 8-bit copies, the nonlinearity, 4-bit and 8-bit products,
// what stands between two blocks):
// checks of torch tensors, allocation of the outputs, the C ABI call.  No computation here.
//
// These calls are made per layer and per token on arrays of a few microseconds' work, so their cost on the host counts:
// the same steps written in Python took 14 to 22 us a call, more than most of the kernels.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <utility>

#include "lrbi.h"

namespace {

PyObject *g_error = nullptr;   // the binding's exception for a status of the C ABI: called with (status, what)

struct BadType : std::runtime_error { using std::runtime_error::runtime_error; };
struct BadValue : std::runtime_error { using std::runtime_error::runtime_error; };
struct BadStatus { int code; const char *what; };

// A Python exception that a Python call has already set.
struct Raised {};

template <class F>
PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const BadType &e) { PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const BadValue &e) { PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Raised &) {
    } catch (const BadStatus &e) {
        PyObject *args = Py_BuildValue("(is)", e.code, e.what);
        if (args && g_error) PyErr_SetObject(g_error, args);
        Py_XDECREF(args);
    } catch (const c10::OutOfMemoryError &e) {
        PyObject *torch = PyImport_ImportModule("torch"), *type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
    } catch (const std::exception &e) { PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

int type_code(at::ScalarType t) { return t == at::kBFloat16 ? LRBI_Y_BF16 : t == at::kFloat ? LRBI_Y_F32 : -1; }

at::ScalarType dtype_of(PyObject *o, at::ScalarType other, const char *what)
{
    if (o == Py_None) return other;
    if (!THPDtype_Check(o) || type_code(reinterpret_cast<THPDtype *>(o)->scalar_type) < 0)
        throw BadType(std::string(what) + " must be torch.bfloat16 or torch.float32");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

const at::Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) throw BadType(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}

// A [rows, cols] CUDA matrix with unit column stride.
struct Matrix {
    void *data;
    int dtype, rows, cols;
    int64_t stride;
    at::Device device{at::kCPU};
    at::ScalarType type;
};

Matrix matrix(const at::Tensor &t, const char *what)
{
    Matrix m;
    m.type = t.scalar_type();
    m.dtype = type_code(m.type);
    if (t.dim() != 2 || !t.is_cuda() || m.dtype < 0 || t.layout() != at::kStrided) throw BadType(std::string(what) + " must be a [rows, cols] CUDA tensor of bfloat16 or float32");
    const int64_t rows = t.size(0), cols = t.size(1);
    m.stride = rows > 1 ? t.stride(0) : cols;
    if (cols < 1 || (cols > 1 && t.stride(1) != 1) || m.stride < cols) throw BadValue(std::string(what) + " must have unit column stride and rows that do not overlap");
    if (rows > INT_MAX || cols > LRBI_MAX_ROW_COLS) throw BadValue(std::string(what) + " is too large");
    m.rows = (int)rows;
    m.cols = (int)cols;
    m.data = t.data_ptr();
    m.device = t.device();
    return m;
}

Matrix matrix_like(PyObject *o, const char *what, const Matrix &like)
{
    const Matrix m = matrix(tensor(o, what), what);
    if (m.rows != like.rows || m.cols != like.cols || m.device != like.device) throw BadValue(std::string(what) + " must have the shape and device of the call's input");
    return m;
}

// The stream of a call: the current one, or the torch.cuda.Stream that was given.
struct Call {
    c10::cuda::CUDAStream current, stream;
    at::Device device;

    Call(const at::Device &d, PyObject *s) : current(c10::cuda::getCurrentCUDAStream(d.index())), stream(current), device(d)
    {
        if (d.index() != c10::cuda::current_device()) throw BadValue("the call's tensors must be on the current CUDA device");
        if (s == Py_None) return;
        int64_t v[3];
        const char *names[3] = {"stream_id", "device_index", "device_type"};
        for (int i = 0; i < 3; ++i) {
            PyObject *a = PyObject_GetAttrString(s, names[i]);
            if (!a) throw Raised();
            v[i] = PyLong_AsLongLong(a);
            Py_DECREF(a);
            if (v[i] == -1 && PyErr_Occurred()) throw Raised();
        }
        if (v[2] != (int64_t)c10::DeviceType::CUDA || v[1] != d.index()) throw BadValue("stream must be a stream of the tensors' device");
        stream = c10::cuda::CUDAStream::unpack3(v[0], (c10::DeviceIndex)v[1], (c10::DeviceType)v[2]);
    }
    // Memory that this call alone uses, out of the pool of the call's stream: what was freed there is through with before the
    // call's kernels begin.  (The current stream may still be reading what was freed to its own pool.)
    at::Tensor scratch(at::IntArrayRef sizes, at::ScalarType type) const
    {
        if (stream == current) return at::detail::empty_cuda(sizes, type, device, std::nullopt);
        const c10::cuda::CUDAStreamGuard guard(stream);
        return at::detail::empty_cuda(sizes, type, device, std::nullopt);
    }
    // A new tensor for the caller, whose own stream will use it too: its memory is kept until that stream is through with it.
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type) const
    {
        at::Tensor t = scratch(sizes, type);
        if (stream != current) t.record_stream(current.unwrap());
        return t;
    }
    // Two new arrays out of one allocation, the second on a 16-byte boundary (allocations cost more than the checks of a call).
    std::pair<at::Tensor, at::Tensor> make_two(at::IntArrayRef a, at::ScalarType a_type, at::IntArrayRef b, at::ScalarType b_type) const
    {
        const int64_t a_bytes = c10::multiply_integers(a) * (int64_t)c10::elementSize(a_type), at_b = (a_bytes + 15) / 16 * 16;
        const at::Tensor all = make({at_b + c10::multiply_integers(b) * (int64_t)c10::elementSize(b_type)}, at::kByte);
        return {part(all, 0, a, a_type), part(all, at_b / (int64_t)c10::elementSize(b_type), b, b_type)};
    }
    static at::Tensor part(const at::Tensor &all, int64_t offset, at::IntArrayRef sizes, at::ScalarType type)
    {
        at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(type));
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        t.unsafeGetTensorImpl()->set_storage_offset(offset);
        return t;
    }
    // New arrays: out of one allocation where they are small (allocations cost more than the checks of a call), else each its own.
    struct Wanted { at::Tensor &tensor; at::DimVector sizes; at::ScalarType type; };
    void make_all(std::initializer_list<Wanted> wanted) const
    {
        int64_t total = 0;
        for (const Wanted &w : wanted) total += room(w);
        if (total > SMALL) {
            for (const Wanted &w : wanted) w.tensor = make(w.sizes, w.type);
            return;
        }
        const at::Tensor all = make({total}, at::kByte);
        int64_t at_byte = 0;
        for (const Wanted &w : wanted) {
            w.tensor = part(all, at_byte / (int64_t)c10::elementSize(w.type), w.sizes, w.type);
            at_byte += room(w);
        }
    }
    static constexpr int64_t SMALL = 1 << 18;
    static int64_t room(const Wanted &w) { return (c10::multiply_integers(w.sizes) * (int64_t)c10::elementSize(w.type) + 31) / 32 * 32; }      // rows in vectors start on 32-byte boundaries
    void *handle() const { return stream.stream(); }
};

struct Params { const void *gamma, *beta; int dtype; };

const at::Tensor &param(PyObject *o, const char *what, const Matrix &x)
{
    const at::Tensor &t = tensor(o, what);
    if (type_code(t.scalar_type()) < 0 || !t.is_contiguous() || t.device() != x.device) throw BadType(std::string(what) + " must be a contiguous bfloat16 or float32 tensor on the call's device");
    if (t.numel() != x.cols) throw BadValue(std::string(what) + " must hold one value per column");
    return t;
}

Params params(PyObject *gamma, PyObject *beta, const Matrix &x)
{
    const at::Tensor &g = param(gamma, "gamma", x);
    Params p = {g.data_ptr(), nullptr, type_code(g.scalar_type())};
    if (beta != Py_None) {
        const at::Tensor &b = param(beta, "beta", x);
        if (b.scalar_type() != g.scalar_type()) throw BadValue("beta must have gamma's type");
        p.beta = b.data_ptr();
    }
    return p;
}

const float *statistics(PyObject *o, const char *what, const Matrix &x)
{
    const at::Tensor &t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.device() != x.device || t.numel() != x.rows)
        throw BadType(std::string(what) + " must be a contiguous float32 tensor with one value per row");
    return static_cast<const float *>(t.data_ptr());
}

// An 8-bit copy: made for a call, or read by one.
struct Copy {
    at::Tensor q, scale;
    int8_t *bytes() const { return q.defined() ? static_cast<int8_t *>(q.data_ptr()) : nullptr; }
    float *scales() const { return scale.defined() ? static_cast<float *>(scale.data_ptr()) : nullptr; }
};

Copy make_copy(const Call &c, int rows, int cols)
{
    auto both = c.make_two({rows, lrbi_checkpoint_pitch(cols)}, at::kChar, {rows, lrbi_checkpoint_groups(cols)}, at::kFloat);
    return {std::move(both.first), std::move(both.second)};
}

// The copy of a [rows, cols] matrix that a call reads.
Copy read_copy(PyObject *q, PyObject *scale, int64_t rows, int64_t cols, const at::Device &device)
{
    Copy k = {tensor(q, "q"), tensor(scale, "scale")};
    if (!k.q.is_cuda() || k.q.device() != device || k.scale.device() != device) throw BadValue("the 8-bit copy must be on the call's device");
    if (k.q.scalar_type() != at::kChar || k.scale.scalar_type() != at::kFloat || !k.q.is_contiguous() || !k.scale.is_contiguous())
        throw BadType("an 8-bit copy is contiguous int8 and its scales contiguous float32");
    if (rows < 0 || rows > INT_MAX || cols < 1 || cols > LRBI_MAX_ROW_COLS || k.q.numel() != rows * lrbi_checkpoint_pitch((int)cols) || k.scale.numel() != rows * lrbi_checkpoint_groups((int)cols))
        throw BadValue("the 8-bit copy does not have the size of its matrix");
    return k;
}

int64_t whole_number(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

void check(int rc, const char *what)
{
    if (rc != LRBI_OK) throw BadStatus{rc, what};
}

// A tuple of new tensors.
template <class... T>
PyObject *tuple(T &&...t)
{
    PyObject *items[] = {THPVariable_Wrap(std::forward<T>(t))...};
    constexpr Py_ssize_t n = sizeof...(T);
    PyObject *r = PyTuple_New(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (r) PyTuple_SET_ITEM(r, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    return r;
}

#define CALL(name, count)                                                                          \
    if (n != count) { PyErr_SetString(PyExc_TypeError, name ": wrong number of arguments"); return nullptr; } \
    return guarded([&]() -> PyObject *

// checkpoint_store(x, stream) -> (q, scale)
PyObject *checkpoint_store(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("checkpoint_store", 2) {
        const Matrix x = matrix(tensor(a[0], "x"), "x");
        const Call c(x.device, a[1]);
        Copy k = make_copy(c, x.rows, x.cols);
        check(lrbi_checkpoint_store(x.data, x.dtype, x.stride, x.rows, x.cols, k.bytes(), k.scales(), c.handle()), "lrbi_checkpoint_store");
        return tuple(std::move(k.q), std::move(k.scale));
    });
}

// checkpoint_load(q, scale, rows, cols, dtype, stream) -> x
PyObject *checkpoint_load(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("checkpoint_load", 6) {
        const at::Device device = tensor(a[0], "q").device();
        const int64_t rows = whole_number(a[2]), cols = whole_number(a[3]);
        const Copy k = read_copy(a[0], a[1], rows, cols, device);
        const at::ScalarType type = dtype_of(a[4], at::kBFloat16, "dtype");
        const Call c(device, a[5]);
        at::Tensor x = c.make({rows, cols}, type);
        check(lrbi_checkpoint_load(k.bytes(), k.scales(), (int)rows, (int)cols, x.data_ptr(), type_code(type), cols, c.handle()), "lrbi_checkpoint_load");
        return THPVariable_Wrap(std::move(x));
    });
}

// layer_norm(x, gamma, beta, eps, y_dtype, checkpoint, stream) -> (y, mean, rstd[, q, scale])
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("layer_norm", 7) {
        const Matrix x = matrix(tensor(a[0], "x"), "x");
        const Params p = params(a[1], a[2], x);
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1.0 && PyErr_Occurred()) throw Raised();
        const at::ScalarType type = dtype_of(a[4], x.type, "y_dtype");
        const int keep = PyObject_IsTrue(a[5]);
        if (keep < 0) throw Raised();
        const Call c(x.device, a[6]);
        at::Tensor y = c.make({x.rows, x.cols}, type);
        auto [mean, rstd] = c.make_two({x.rows}, at::kFloat, {x.rows}, at::kFloat);
        Copy k;
        if (keep) k = make_copy(c, x.rows, x.cols);
        check(lrbi_layer_norm(x.data, x.dtype, x.stride, x.rows, x.cols, p.gamma, p.beta, p.dtype, (float)eps, y.data_ptr(), type_code(type), x.cols,
                              static_cast<float *>(mean.data_ptr()), static_cast<float *>(rstd.data_ptr()), k.bytes(), k.scales(), c.handle()),
              "lrbi_layer_norm");
        if (keep) return tuple(std::move(y), std::move(mean), std::move(rstd), std::move(k.q), std::move(k.scale));
        return tuple(std::move(y), std::move(mean), std::move(rstd));
    });
}

// layer_norm_backward(dy, x or None, q, scale, gamma, mean, rstd, beta, dres, restore, dx_dtype, stream) -> (dx, dgamma, dbeta[, y])
PyObject *layer_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("layer_norm_backward", 12) {
        const Matrix dy = matrix(tensor(a[0], "dy"), "dy");
        Matrix x = {nullptr, LRBI_Y_BF16, dy.rows, dy.cols, dy.cols, dy.device, dy.type};
        Copy k;
        if (a[1] != Py_None) x = matrix_like(a[1], "x", dy);
        else k = read_copy(a[2], a[3], dy.rows, dy.cols, dy.device);
        const Params p = params(a[4], a[7], dy);
        const float *mean = statistics(a[5], "mean", dy), *rstd = statistics(a[6], "rstd", dy);
        const at::ScalarType type = dtype_of(a[10], x.type, "dx_dtype");
        Matrix dres = {nullptr, 0, 0, 0, dy.cols, dy.device, type};
        if (a[8] != Py_None) {
            dres = matrix_like(a[8], "dres", dy);
            if (dres.type != type) throw BadValue("dres must have dx's type");
        }
        const int restore = PyObject_IsTrue(a[9]);
        if (restore < 0) throw Raised();
        const Call c(dy.device, a[11]);
        at::Tensor dx = c.make({dy.rows, dy.cols}, type), y;
        auto [dgamma, dbeta] = c.make_two({dy.cols}, at::kFloat, {dy.cols}, at::kFloat);
        if (restore) y = c.make({dy.rows, dy.cols}, dy.type);
        const size_t need = lrbi_layer_norm_backward_workspace(dy.rows, dy.cols);
        const at::Tensor work = c.scratch({(int64_t)need}, at::kByte);
        check(lrbi_layer_norm_backward(dy.data, dy.dtype, dy.stride, x.data, x.dtype, x.stride, k.bytes(), k.scales(), dy.rows, dy.cols, p.gamma, p.beta,
                                       p.dtype, mean, rstd, dres.data, dres.stride, dx.data_ptr(), type_code(type), dy.cols,
                                       restore ? y.data_ptr() : nullptr, dy.cols, static_cast<float *>(dgamma.data_ptr()),
                                       static_cast<float *>(dbeta.data_ptr()), work.data_ptr(), need, c.handle()),
              "lrbi_layer_norm_backward");
        if (restore) return tuple(std::move(dx), std::move(dgamma), std::move(dbeta), std::move(y));
        return tuple(std::move(dx), std::move(dgamma), std::move(dbeta));
    });
}

// activation(h, act, a_dtype, checkpoint, stream) -> a, or (a, q, scale)
PyObject *activation(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("activation", 5) {
        const Matrix h = matrix(tensor(a[0], "h"), "h");
        const int act = (int)PyLong_AsLong(a[1]);
        const at::ScalarType type = dtype_of(a[2], h.type, "a_dtype");
        const int keep = PyObject_IsTrue(a[3]);
        if (keep < 0) throw Raised();
        const Call c(h.device, a[4]);
        at::Tensor out = c.make({h.rows, h.cols}, type);
        Copy k;
        if (keep) k = make_copy(c, h.rows, h.cols);
        check(lrbi_activation(h.data, h.dtype, h.stride, h.rows, h.cols, act, out.data_ptr(), type_code(type), h.cols, k.bytes(), k.scales(), c.handle()),
              "lrbi_activation");
        if (keep) return tuple(std::move(out), std::move(k.q), std::move(k.scale));
        return THPVariable_Wrap(std::move(out));
    });
}

// activation_backward(da, h or None, q, scale, act, restore, dh_dtype, stream) -> dh, or (dh, a)
PyObject *activation_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("activation_backward", 8) {
        const Matrix da = matrix(tensor(a[0], "da"), "da");
        Matrix h = {nullptr, LRBI_Y_BF16, da.rows, da.cols, da.cols, da.device, da.type};
        Copy k;
        if (a[1] != Py_None) h = matrix_like(a[1], "h", da);
        else k = read_copy(a[2], a[3], da.rows, da.cols, da.device);
        const int act = (int)PyLong_AsLong(a[4]);
        const int restore = PyObject_IsTrue(a[5]);
        if (restore < 0) throw Raised();
        const at::ScalarType type = dtype_of(a[6], da.type, "dh_dtype");
        const Call c(da.device, a[7]);
        at::Tensor dh = c.make({da.rows, da.cols}, type), again;
        if (restore) again = c.make({da.rows, da.cols}, da.type);
        check(lrbi_activation_backward(da.data, da.dtype, da.stride, h.data, h.dtype, h.stride, k.bytes(), k.scales(), da.rows, da.cols, act, dh.data_ptr(),
                                       type_code(type), da.cols, restore ? again.data_ptr() : nullptr, da.cols, c.handle()),
              "lrbi_activation_backward");
        if (restore) return tuple(std::move(dh), std::move(again));
        return THPVariable_Wrap(std::move(dh));
    });
}

// w4_gemv(packed, meta, rows, cols, group, X, y_dtype, stream) -> Y
PyObject *w4_gemv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("w4_gemv", 8) {
        const at::Tensor &packed = tensor(a[0], "packed"), &meta = tensor(a[1], "meta"), &X = tensor(a[5], "X");
        const int64_t rows = whole_number(a[2]), cols = whole_number(a[3]), group = whole_number(a[4]);
        if (packed.scalar_type() != at::kInt || meta.scalar_type() != at::kInt || !packed.is_cuda() || !packed.is_contiguous() || !meta.is_contiguous())
            throw BadType("4-bit weights are contiguous CUDA tensors of int32");
        if (rows < 1 || rows > INT_MAX || cols < 1 || cols > LRBI_MAX_ROW_COLS || group < 1 || group > INT_MAX || meta.device() != packed.device() ||
            (size_t)packed.numel() != lrbi_w4_packed_words((int)rows, (int)cols) || (size_t)meta.numel() != lrbi_w4_meta_words((int)rows, (int)cols, (int)group))
            throw BadValue("the 4-bit weights do not have the size of their layer");
        if (!X.is_cuda() || X.scalar_type() != at::kBFloat16 || !X.is_contiguous()) throw BadType("X must be a contiguous CUDA tensor of dtype torch.bfloat16");
        if (X.dim() != 2 || X.size(1) != cols || X.device() != packed.device() || X.size(0) > INT_MAX) throw BadValue("X must be [batch, cols] on the weights' device");
        const at::ScalarType type = dtype_of(a[6], at::kBFloat16, "y_dtype");
        const int batch = (int)X.size(0);
        const Call c(X.device(), a[7]);
        at::Tensor Y = c.make({batch, rows}, type);
        check(lrbi_w4_gemv(static_cast<const uint32_t *>(packed.data_ptr()), static_cast<const uint32_t *>(meta.data_ptr()), (int)rows, (int)cols, (int)group,
                           static_cast<const uint16_t *>(X.data_ptr()), batch, Y.data_ptr(), type_code(type), c.handle()),
              "lrbi_w4_gemv");
        return THPVariable_Wrap(std::move(Y));
    });
}

// Rows in 8-bit integers that a call reads: [rows, pitch] int8 and a scale each.
struct Rows8 { const int8_t *q; const float *scale; };
Rows8 rows8(PyObject *q, PyObject *scale, int64_t rows, int64_t cols, const at::Device &device, const char *what)
{
    const at::Tensor &t = tensor(q, what), &s = tensor(scale, what);
    if (!t.is_cuda() || t.device() != device || s.device() != device) throw BadValue(std::string(what) + " must be on the call's device");
    if (t.scalar_type() != at::kChar || s.scalar_type() != at::kFloat || !t.is_contiguous() || !s.is_contiguous())
        throw BadType(std::string(what) + ": 8-bit rows are contiguous int8 and their scales contiguous float32");
    if (rows < 0 || rows > INT_MAX || cols < 1 || cols > LRBI_I8_MAX_COLS || t.numel() != rows * lrbi_i8_pitch((int)cols) || s.numel() != rows)
        throw BadValue(std::string(what) + " does not have the size of its rows");
    return {static_cast<const int8_t *>(t.data_ptr()), static_cast<const float *>(s.data_ptr())};
}

std::pair<at::Tensor, at::Tensor> make_rows8(const Call &c, int rows, int cols)
{
    if (cols > LRBI_I8_MAX_COLS) throw BadValue("rows in 8 bits have at most 131072 columns");
    return c.make_two({rows, lrbi_i8_pitch(cols)}, at::kChar, {rows}, at::kFloat);
}

// i8_tokens(x, act, stream) -> (q, scale, rows, cols)
PyObject *i8_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("i8_tokens", 3) {
        const Matrix x = matrix(tensor(a[0], "x"), "x");
        const int act = (int)whole_number(a[1]);
        const Call c(x.device, a[2]);
        auto [q, scale] = make_rows8(c, x.rows, x.cols);
        check(lrbi_i8_tokens(x.data, x.dtype, x.stride, x.rows, x.cols, act, static_cast<int8_t *>(q.data_ptr()), static_cast<float *>(scale.data_ptr()), c.handle()),
              "lrbi_i8_tokens");
        PyObject *r = PyTuple_New(4), *items[] = {THPVariable_Wrap(std::move(q)), THPVariable_Wrap(std::move(scale)), PyLong_FromLong(x.rows), PyLong_FromLong(x.cols)};
        for (int i = 0; i < 4; ++i) {
            if (r) PyTuple_SET_ITEM(r, i, items[i]);
            else Py_XDECREF(items[i]);
        }
        return r;
    });
}

// i8_gemm(w_q, w_scale, rows, cols, x_q, x_scale, batch, y_dtype, stream) -> Y
PyObject *i8_gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("i8_gemm", 9) {
        const at::Device device = tensor(a[0], "weights").device();
        const int64_t rows = whole_number(a[2]), cols = whole_number(a[3]), batch = whole_number(a[6]);
        const Rows8 w = rows8(a[0], a[1], rows, cols, device, "weights"), x = rows8(a[4], a[5], batch, cols, device, "tokens");
        const at::ScalarType type = dtype_of(a[7], at::kBFloat16, "y_dtype");
        const Call c(device, a[8]);
        at::Tensor Y = c.make({batch, rows}, type);
        check(lrbi_i8_gemm(w.q, w.scale, (int)rows, (int)cols, x.q, x.scale, (int)batch, Y.data_ptr(), type_code(type), c.handle()), "lrbi_i8_gemm");
        return THPVariable_Wrap(std::move(Y));
    });
}

// The vectors and numbers of a call between two blocks: a[0 ..] = gamma, beta, post_gamma, post_beta, gate.
lrbi_residual residual(PyObject *const *a, const Matrix &x, const Matrix &f, double scale, double eps, int kind)
{
    lrbi_residual h = {x.rows, x.cols, kind, x.dtype, f.dtype, LRBI_Y_F32, (float)scale, (float)eps, nullptr, nullptr, nullptr, nullptr, nullptr};
    if (x.cols > LRBI_MAX_RESIDUAL_COLS) throw BadValue("the residual stream has at most 32768 columns");
    if (x.dtype == LRBI_Y_BF16 && f.dtype != LRBI_Y_BF16) throw BadType("f must be bfloat16 where x is");
    const char *names[5] = {"gamma", "beta", "post_gamma", "post_beta", "gate"};
    const void **at[5] = {&h.gamma, &h.beta, &h.post_gamma, &h.post_beta, &h.gate};
    int type = -1;
    for (int i = 0; i < 5; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor &t = param(a[i], names[i], x);
        const int code = type_code(t.scalar_type());
        if (type >= 0 && code != type) throw BadValue(std::string(names[i]) + " must have the type of the other vectors");
        h.param_dtype = type = code;
        *at[i] = t.data_ptr();
    }
    if (h.beta && !h.gamma) throw BadValue("beta comes with gamma");
    if (h.post_beta && !h.post_gamma) throw BadValue("post_beta comes with post_gamma");
    return h;
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

PyObject *or_none(at::Tensor t)
{
    if (t.defined()) return THPVariable_Wrap(std::move(t));
    Py_RETURN_NONE;
}

template <int N>
PyObject *tuple_of(at::Tensor (&t)[N])
{
    PyObject *r = PyTuple_New(N);
    for (int i = 0; r && i < N; ++i) {
        PyObject *item = or_none(std::move(t[i]));
        if (!item) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i, item);
    }
    return r;
}

// residual_norm(x, f, gamma, beta, post_gamma, post_beta, gate, residual_scale, eps, kind, tokens, stream) -> (out, u, stats, q, scale): None for what the call does not make
PyObject *residual_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("residual_norm", 12) {
        const Matrix x = matrix(tensor(a[0], "x"), "x"), f = matrix_like(a[1], "f", x);
        const lrbi_residual how = residual(a + 2, x, f, number(a[7]), number(a[8]), (int)whole_number(a[9]));
        const int tokens = PyObject_IsTrue(a[10]);
        if (tokens < 0) throw Raised();
        if (tokens && !how.gamma) throw BadValue("tokens come from the second norm: give gamma");
        const Call c(x.device, a[11]);
        at::Tensor t[5];      // out, u, stats, q, scale
        if (tokens) c.make_all({{t[0], {x.rows, x.cols}, x.type}, {t[3], {x.rows, lrbi_i8_pitch(x.cols)}, at::kChar}, {t[4], {x.rows}, at::kFloat}});
        else if (how.gamma) c.make_all({{t[0], {x.rows, x.cols}, x.type}, {t[1], {x.rows, x.cols}, f.type}, {t[2], {4, x.rows}, at::kFloat}});
        else c.make_all({{t[0], {x.rows, x.cols}, x.type}, {t[2], {4, x.rows}, at::kFloat}});
        auto at = [](const at::Tensor &v) { return v.defined() ? v.data_ptr() : nullptr; };
        check(lrbi_residual_norm(&how, x.data, x.stride, f.data, f.stride, at(t[0]), x.cols, at(t[1]), x.cols, static_cast<int8_t *>(at(t[3])),
                                 static_cast<float *>(at(t[4])), static_cast<float *>(at(t[2])), c.handle()),
              "lrbi_residual_norm");
        return tuple_of(t);
    });
}

// residual_norm_backward(du, dout, out, f, gamma, beta, post_gamma, post_beta, gate, residual_scale, stats, kind, stream)
//     -> (dx, df, dgamma, dbeta, dpost_gamma, dpost_beta, dgate): None for vectors that the call does not have
PyObject *residual_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    CALL("residual_norm_backward", 13) {
        const Matrix f = matrix(tensor(a[3], "f"), "f");
        Matrix x = f, du = {nullptr, f.dtype, f.rows, f.cols, f.cols, f.device, f.type}, dout = du;
        if (a[2] != Py_None) x = matrix_like(a[2], "out", f);
        if (a[1] != Py_None) dout = matrix_like(a[1], "dout", f);
        if (a[2] == Py_None) { if (a[1] == Py_None) throw BadValue("out or dout must be given"); x = dout; }
        if (a[1] != Py_None && dout.type != x.type) throw BadValue("dout must have out's type");
        const lrbi_residual how = residual(a + 4, x, f, number(a[9]), 0., (int)whole_number(a[11]));
        if (how.gamma) {
            if (a[2] == Py_None) throw BadValue("out must be given where gamma is");
            du = matrix_like(a[0], "du", f);
            if (du.type != f.type) throw BadValue("du must have f's type");
        } else if (a[0] != Py_None) throw BadValue("du comes with gamma");
        const float *stats = nullptr;
        if (how.gamma || how.post_gamma) {
            const at::Tensor &t = tensor(a[10], "stats");
            if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.device() != f.device || t.numel() != 4 * (int64_t)f.rows)
                throw BadType("stats must be the contiguous float32 tensor [4, rows] of the forward pass");
            stats = static_cast<const float *>(t.data_ptr());
        }
        const Call c(f.device, a[12]);
        at::Tensor t[7];      // dx, df, and the vectors' gradients out of one allocation
        const void *vectors[5] = {how.gamma, how.beta, how.post_gamma, how.post_beta, how.gate};
        float *to[5] = {};
        int count = 0;
        for (const void *v : vectors) count += v != nullptr;
        const int64_t pitch = (f.cols + 3) / 4 * 4;
        at::Tensor all;
        c.make_all({{t[0], {f.rows, f.cols}, x.type}, {t[1], {f.rows, f.cols}, f.type}, {all, {count * pitch}, at::kFloat}});
        if (count) {
            for (int i = 0, k = 0; i < 5; ++i) {
                if (!vectors[i]) continue;
                t[2 + i] = Call::part(all, all.storage_offset() + k++ * pitch, {f.cols}, at::kFloat);
                to[i] = static_cast<float *>(t[2 + i].data_ptr());
            }
        }
        const size_t need = lrbi_residual_norm_backward_workspace(f.rows, f.cols);
        const at::Tensor work = c.scratch({(int64_t)need}, at::kByte);
        check(lrbi_residual_norm_backward(&how, du.data, du.stride, a[1] != Py_None ? dout.data : nullptr, dout.stride, how.gamma ? x.data : nullptr, x.stride,
                                          f.data, f.stride, stats, t[0].data_ptr(), f.cols, t[1].data_ptr(), f.cols, to[0], to[1], to[2], to[3], to[4],
                                          work.data_ptr(), need, c.handle()),
              "lrbi_residual_norm_backward");
        return tuple_of(t);
    });
}

PyObject *set_error(PyObject *, PyObject *error)
{
    Py_INCREF(error);
    Py_XDECREF(g_error);
    g_error = error;
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(checkpoint_store), FAST(checkpoint_load), FAST(layer_norm), FAST(layer_norm_backward), FAST(activation),
                         FAST(activation_backward), FAST(w4_gemv), FAST(i8_tokens), FAST(i8_gemm), FAST(residual_norm), FAST(residual_norm_backward), {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lrbi_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lrbi_torch() { return PyModule_Create(&module); }
