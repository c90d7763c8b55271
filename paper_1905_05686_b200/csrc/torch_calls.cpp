// Python calls of the operators around the masked layers (layer norm, 8-bit copies, the nonlinearity, 4-bit products):
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

PyObject *set_error(PyObject *, PyObject *error)
{
    Py_INCREF(error);
    Py_XDECREF(g_error);
    g_error = error;
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(checkpoint_store), FAST(checkpoint_load), FAST(layer_norm), FAST(layer_norm_backward), FAST(activation),
                         FAST(activation_backward), FAST(w4_gemv), {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lrbi_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lrbi_torch() { return PyModule_Create(&module); }
