// What paper_1803_03288_amd/layers.py calls: checks of tensors, their outputs and workspaces, and the C calls of libtictac.so (include/tictac.h).
// A call of the layers' operators on few rows takes the GPU 3 to 10 us; the same steps in Python take the host 13 us and more, here 6.
// Plain CPython functions on torch's C++ tensors: no arithmetic, no HIP call but the current stream and device.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>
#include <vector>

#include "tictac.h"

namespace {

using at::Tensor;

constexpr int64_t kGroup = 128;

// the C calls, by the addresses that init() is given
decltype(&tictac_quantize_rows) g_quantize_rows;
decltype(&tictac_dequantize_rows) g_dequantize_rows;
decltype(&tictac_layer_norm) g_layer_norm;
decltype(&tictac_layer_norm_backward_workspace) g_layer_norm_backward_workspace;
decltype(&tictac_layer_norm_backward) g_layer_norm_backward;
decltype(&tictac_linear_q8_workspace) g_linear_q8_workspace;
decltype(&tictac_linear_q8) g_linear_q8;
decltype(&tictac_linear_q8_backward_workspace) g_linear_q8_backward_workspace;
decltype(&tictac_linear_q8_backward) g_linear_q8_backward;
PyObject *g_fail;               // raises the error of a status
PyObject *g_out_of_memory;      // torch's exception

struct Refused {                // a wrong argument: the Python exception to be raised
    PyObject *type;
    std::string what;
};
struct Status { int code; };    // what the library refused

[[noreturn]] void value_error(std::string what) { throw Refused{PyExc_ValueError, std::move(what)}; }
[[noreturn]] void type_error(std::string what) { throw Refused{PyExc_TypeError, std::move(what)}; }
std::string str(int64_t v) { return std::to_string(v); }

int dtype_code(at::ScalarType t)
{
    switch (t) {
        case at::kFloat: return TICTAC_F32;
        case at::kHalf: return TICTAC_F16;
        case at::kBFloat16: return TICTAC_BF16;
        default: return -1;
    }
}

const Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) type_error(std::string(name) + " is no tensor");
    return THPVariable_Unpack(o);
}

at::ScalarType dtype(PyObject *o, const char *name)
{
    if (!THPDtype_Check(o) || dtype_code(reinterpret_cast<THPDtype *>(o)->scalar_type) < 0) type_error(std::string(name) + ": expected float32, float16 or bfloat16");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

void check_device(const Tensor &t, const char *name)
{
    if (!t.is_cuda()) value_error(std::string(name) + " is on " + t.device().str() + ": the operators take CUDA tensors");
    if (t.get_device() != c10::hip::current_device())
        value_error(std::string(name) + " is on " + t.device().str() + ", the current device is cuda:" + str(c10::hip::current_device()));
}

// The tensor itself, or a copy where it is a view of another's values with their signs turned (the imaginary part of a conjugate): what lies in memory then
// are the others.
Tensor own_sign(const Tensor &t) { return t.is_neg() ? t.resolve_neg() : t; }

// Rows of floats: [rows][cols] with the elements of a row next to each other (copied where they are not).
struct Rows {
    Tensor t;                   // keeps a copy alive
    int dtype;
    int64_t rows, cols, ld;
    void *data() const { return t.data_ptr(); }
};
Rows float_rows(const Tensor &x, const char *name)
{
    check_device(x, name);
    const int dt = dtype_code(x.scalar_type());
    if (dt < 0) type_error(std::string(name) + " is " + toString(x.scalar_type()) + ": expected float32, float16 or bfloat16");
    const int64_t dim = x.dim();
    if (dim == 0) value_error(std::string(name) + " has no dimension");
    const int64_t cols = x.size(dim - 1);
    if (cols == 0) value_error(std::string(name) + " has rows of no columns");
    Tensor t = own_sign(dim == 2 ? x : x.reshape({-1, cols}));
    if ((t.stride(1) != 1 && cols > 1) || t.stride(0) < 0) t = t.contiguous();
    const int64_t rows = t.size(0);
    return Rows{t, dt, rows, cols, rows > 1 ? t.stride(0) : cols};
}

// A parameter of n values in float32 or `type`, or None.
struct Vector {
    Tensor t;
    void *data = nullptr;
    int dtype = TICTAC_F32;
};
Vector vector(PyObject *o, const char *name, int64_t n, at::ScalarType type, const Tensor &like)
{
    Vector v;
    if (o == Py_None) return v;
    const Tensor &t = tensor(o, name);
    if (t.dim() != 1 || t.size(0) != n) value_error(std::string(name) + " has another shape than (" + str(n) + ",)");
    if (t.scalar_type() != at::kFloat && t.scalar_type() != type) type_error(std::string(name) + " is " + toString(t.scalar_type()) + ": expected float32 or " + toString(type));
    if (t.device() != like.device()) value_error(std::string(name) + " is on " + t.device().str() + ", expected " + like.device().str());
    v.t = own_sign(t.is_contiguous() ? t : t.contiguous());
    v.data = v.t.data_ptr();
    v.dtype = dtype_code(t.scalar_type());
    return v;
}
Tensor statistic(PyObject *o, const char *name, int64_t rows, const Tensor &like)
{
    const Tensor &t = tensor(o, name);
    if (t.scalar_type() != at::kFloat || t.numel() != rows || t.device() != like.device())
        value_error(std::string(name) + ": expected " + str(rows) + " float32 values on " + like.device().str());
    return own_sign(t.is_contiguous() ? t : t.contiguous());
}

int64_t padded(int64_t cols) { return (cols + 127) / 128 * 128; }

// 8-bit rows, a tuple (q, scale, cols, group).
struct Rows8 {
    const Tensor *q;
    Tensor scale;
    int64_t rows, cols, group, ld;
    const int8_t *data() const { return (const int8_t *)q->data_ptr(); }
    const float *scales() const { return (const float *)scale.data_ptr(); }
};
bool is_rows8(PyObject *o) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4; }
Rows8 rows8(PyObject *o, const char *name, int64_t group, const at::Device *device)       // group -1: any
{
    if (!is_rows8(o)) type_error(std::string(name) + ": expected Rows8");
    Rows8 r;
    r.q = &tensor(PyTuple_GET_ITEM(o, 0), name);
    r.scale = own_sign(tensor(PyTuple_GET_ITEM(o, 1), name));
    r.cols = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
    r.group = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 3));
    if (PyErr_Occurred()) { PyErr_Clear(); type_error(std::string(name) + ": cols and group are whole numbers"); }
    if (r.group != 0 && r.group != kGroup) value_error(std::string(name) + ": a group of " + str(r.group) + ", expected 0 or " + str(kGroup));
    if (group >= 0 && r.group != group) value_error(std::string(name) + " has a scale per " + (r.group ? str(r.group) : "row") + ", expected one per " + (group ? str(group) : "row"));
    if (r.q->scalar_type() != at::kChar || r.q->dim() != 2 || r.scale.scalar_type() != at::kFloat) type_error(std::string(name) + ": expected int8 rows and float32 scales");
    if (!device) check_device(*r.q, name);
    if (r.q->device() != (device ? *device : r.scale.device()) || r.scale.device() != r.q->device()) value_error(std::string(name) + " is on another device");
    r.rows = r.q->size(0);
    if (r.cols < 1 || r.q->size(1) < padded(r.cols) || r.q->stride(1) != 1 || !r.scale.is_contiguous())
        value_error(std::string(name) + ": rows of " + str(r.cols) + " columns are padded to " + str(padded(r.cols)) + ", contiguous, and so are their scales");
    if (r.scale.numel() != r.rows * (r.group ? (r.cols + kGroup - 1) / kGroup : 1)) value_error(std::string(name) + ": " + str(r.scale.numel()) + " scales for " + str(r.rows) + " rows");
    r.ld = r.rows > 1 ? r.q->stride(0) : padded(r.q->size(1));
    return r;
}

Tensor empty(at::IntArrayRef size, at::ScalarType type, const Tensor &like) { return at::empty(size, like.options().dtype(type).requires_grad(false).memory_format(c10::nullopt)); }

Tensor workspace(size_t bytes, const Tensor &like) { return bytes ? empty({(int64_t)bytes}, at::kByte, like) : Tensor(); }
void *ptr(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
void check(int rc) { if (rc != TICTAC_OK) throw Status{rc}; }
tictac_stream stream() { return (tictac_stream)c10::hip::getCurrentHIPStream().stream(); }

PyObject *wrap(const Tensor &t) { if (!t.defined()) Py_RETURN_NONE; return THPVariable_Wrap(t); }
// a tensor of the shape of `like` but for the last dimension
Tensor shaped(const Tensor &t, const Tensor &like, int64_t last)
{
    if (like.dim() == 2) return t;
    std::vector<int64_t> shape(like.sizes().begin(), like.sizes().end());
    shape.back() = last;
    return t.view(shape);
}
PyObject *tuple(std::initializer_list<Tensor> all)
{
    PyObject *out = PyTuple_New((Py_ssize_t)all.size());
    Py_ssize_t i = 0;
    for (const Tensor &t : all) PyTuple_SET_ITEM(out, i++, wrap(t));
    return out;
}

void take(Py_ssize_t n, Py_ssize_t want) { if (n != want) type_error("expected " + str(want) + " arguments"); }

// (x, group) -> (q, scale)
PyObject *quantize_rows(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 2);
    const Rows x = float_rows(tensor(arg[0], "x"), "x");
    const int64_t group = PyLong_AsLongLong(arg[1]), ld = padded(x.cols);
    if (group != 0 && group != kGroup) {
        PyErr_Clear();
        value_error("group: expected 0 or " + str(kGroup));
    }
    const Tensor q = empty({x.rows, ld}, at::kChar, x.t), scale = empty({x.rows, group ? (x.cols + kGroup - 1) / kGroup : 1}, at::kFloat, x.t);
    check(g_quantize_rows(x.dtype, x.rows, x.cols, x.data(), x.ld, (int32_t)group, (int8_t *)q.data_ptr(), ld, (float *)scale.data_ptr(), stream()));
    return tuple({q, scale});
}

// (rows8, dtype) -> x
PyObject *dequantize_rows(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 2);
    const at::ScalarType type = dtype(arg[1], "dtype");
    const Rows8 r = rows8(arg[0], "r", -1, nullptr);
    const Tensor x = empty({r.rows, r.cols}, type, *r.q);
    check(g_dequantize_rows(dtype_code(type), r.rows, r.cols, r.data(), r.ld, r.scales(), (int32_t)r.group, x.data_ptr(), r.cols, stream()));
    return wrap(x);
}

// (x, weight, bias, eps, y8, save) -> (y, mean, rstd[, xq, xs]), or with y8 (yq, ys, mean, rstd[, xq, xs])
PyObject *layer_norm(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 6);
    const Tensor &given = tensor(arg[0], "x");
    const Rows x = float_rows(given, "x");
    const at::ScalarType type = given.scalar_type();
    const Vector w = vector(arg[1], "weight", x.cols, type, x.t), b = vector(arg[2], "bias", x.cols, type, x.t);
    if (w.data && b.data && w.dtype != b.dtype) type_error("weight and bias are of two types");
    const double eps = PyFloat_AsDouble(arg[3]);
    if (PyErr_Occurred()) { PyErr_Clear(); type_error("eps is no number"); }
    const bool y8 = arg[4] == Py_True, save = arg[5] == Py_True;
    const int64_t ld = padded(x.cols);
    Tensor y, yq, ys, xq, xs;
    if (y8) {
        yq = empty({x.rows, ld}, at::kChar, x.t);
        ys = empty({x.rows, 1}, at::kFloat, x.t);
    } else {
        y = empty({x.rows, x.cols}, type, x.t);
    }
    if (save) {
        xq = empty({x.rows, ld}, at::kChar, x.t);
        xs = empty({x.rows, (x.cols + kGroup - 1) / kGroup}, at::kFloat, x.t);
    }
    const Tensor mean = empty({x.rows}, at::kFloat, x.t), rstd = empty({x.rows}, at::kFloat, x.t);
    check(g_layer_norm(x.dtype, x.rows, x.cols, x.data(), x.ld, w.data ? w.dtype : b.dtype, w.data, b.data, (float)eps, ptr(y), x.cols, (float *)mean.data_ptr(),
                       (float *)rstd.data_ptr(), (int8_t *)ptr(yq), ld, (float *)ptr(ys), (int8_t *)ptr(xq), ld, (float *)ptr(xs), stream()));
    if (y8) return save ? tuple({yq, ys, mean, rstd, xq, xs}) : tuple({yq, ys, mean, rstd});
    y = shaped(y, given, x.cols);
    return save ? tuple({y, mean, rstd, xq, xs}) : tuple({y, mean, rstd});
}

// (dy, x, weight, mean, rstd) -> (dx, dweight, dbias)
PyObject *layer_norm_backward(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 5);
    const Tensor &given = tensor(arg[0], "dy");
    const Rows dy = float_rows(given, "dy");
    const at::Device device = dy.t.device();
    Rows x{};
    Rows8 saved{};
    const bool kept = is_rows8(arg[1]);
    if (kept) {
        saved = rows8(arg[1], "x", kGroup, &device);
    } else {
        x = float_rows(tensor(arg[1], "x"), "x");
        if (x.dtype != dy.dtype) type_error("x and dy are of two types");
    }
    if ((kept ? saved.rows : x.rows) != dy.rows || (kept ? saved.cols : x.cols) != dy.cols)
        value_error("x has " + str(kept ? saved.rows : x.rows) + " rows of " + str(kept ? saved.cols : x.cols) + ", dy " + str(dy.rows) + " of " + str(dy.cols));
    const Vector w = vector(arg[2], "weight", dy.cols, given.scalar_type(), dy.t);
    const Tensor mean = statistic(arg[3], "mean", dy.rows, dy.t), rstd = statistic(arg[4], "rstd", dy.rows, dy.t);
    const at::ScalarType of = w.data ? w.t.scalar_type() : at::kFloat;
    const Tensor dx = empty({dy.rows, dy.cols}, given.scalar_type(), dy.t), dw = empty({dy.cols}, of, dy.t), db = empty({dy.cols}, of, dy.t);
    size_t bytes = 0;
    check(g_layer_norm_backward_workspace(dy.rows, dy.cols, &bytes));
    const Tensor room = workspace(bytes, dy.t);
    check(g_layer_norm_backward(dy.dtype, dy.rows, dy.cols, dy.data(), dy.ld, kept ? nullptr : x.data(), x.ld, kept ? saved.data() : nullptr, saved.ld,
                                kept ? saved.scales() : nullptr, w.dtype, w.data, (const float *)mean.data_ptr(), (const float *)rstd.data_ptr(), dx.data_ptr(), dy.cols, dw.data_ptr(),
                                db.data_ptr(), ptr(room), bytes, stream()));
    return tuple({shaped(dx, given, dy.cols), dw, db});
}

// (x, w, bias, dtype) -> y
PyObject *linear_q8(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 4);
    Rows x{};
    Rows8 x8{};
    const bool ready = is_rows8(arg[0]);
    at::ScalarType type = at::kFloat;
    if (ready) {
        x8 = rows8(arg[0], "x", 0, nullptr);
        if (arg[3] != Py_None) type = dtype(arg[3], "dtype");
    } else {
        x = float_rows(tensor(arg[0], "x"), "x");
        type = x.t.scalar_type();
        if (arg[3] != Py_None && dtype(arg[3], "dtype") != type) type_error("dtype is not that of x");
    }
    const Tensor &like = ready ? *x8.q : x.t;
    const at::Device device = like.device();
    const Rows8 w = rows8(arg[1], "w", 0, &device);
    const int64_t rows = ready ? x8.rows : x.rows, cols = ready ? x8.cols : x.cols;
    if (w.cols != cols) value_error("x has " + str(cols) + " columns, w " + str(w.cols));
    const Vector bias = vector(arg[2], "bias", w.rows, type, like);
    const Tensor y = empty({rows, w.rows}, type, like);
    size_t bytes = 0;
    check(g_linear_q8_workspace(!ready, rows, cols, w.rows, &bytes));
    const Tensor room = workspace(bytes, like);
    check(g_linear_q8(dtype_code(type), rows, cols, w.rows, ready ? nullptr : x.data(), x.ld, ready ? x8.data() : nullptr, x8.ld, ready ? x8.scales() : nullptr, w.data(), w.ld, w.scales(),
                      bias.dtype, bias.data, y.data_ptr(), w.rows, ptr(room), bytes, stream()));
    return wrap(ready ? y : shaped(y, tensor(arg[0], "x"), w.rows));
}

// (dy, x, w) -> (dx, dw, db)
PyObject *linear_q8_backward(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 3);
    const Tensor &given = tensor(arg[0], "dy");
    const Rows dy = float_rows(given, "dy");
    const at::Device device = dy.t.device();
    const Rows8 x = rows8(arg[1], "x", 0, &device), w = rows8(arg[2], "w", 0, &device);
    if (x.rows != dy.rows || w.rows != dy.cols || w.cols != x.cols)
        value_error("dy is " + str(dy.rows) + " x " + str(dy.cols) + ", x " + str(x.rows) + " x " + str(x.cols) + ", w " + str(w.rows) + " x " + str(w.cols));
    const at::ScalarType type = given.scalar_type();
    const Tensor dx = empty({dy.rows, x.cols}, type, dy.t), dw = empty({dy.cols, x.cols}, type, dy.t), db = empty({dy.cols}, type, dy.t);
    size_t bytes = 0;
    check(g_linear_q8_backward_workspace(dy.dtype, dy.rows, x.cols, dy.cols, &bytes));
    const Tensor room = workspace(bytes, dy.t);
    check(g_linear_q8_backward(dy.dtype, dy.rows, x.cols, dy.cols, dy.data(), dy.ld, x.data(), x.ld, x.scales(), w.data(), w.ld, w.scales(), dx.data_ptr(), x.cols, dw.data_ptr(), x.cols,
                               db.data_ptr(), ptr(room), bytes, stream()));
    return tuple({shaped(dx, given, x.cols), dw, db});
}

// No C++ exception leaves: wrong arguments and what torch raises become Python exceptions, a status what `fail` raises for it.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *arg, Py_ssize_t n)
{
    try {
        const at::NoGradGuard no_grad;
        return F(arg, n);
    } catch (const Refused &e) {
        PyErr_SetString(e.type, e.what.c_str());
    } catch (const Status &e) {
        PyObject *r = PyObject_CallFunction(g_fail, "i", e.code);
        if (r) {
            Py_DECREF(r);
            PyErr_Format(PyExc_RuntimeError, "status %d", e.code);
        }
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(g_out_of_memory, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// (addresses of the nine C calls, the function that raises the error of a status, torch.OutOfMemoryError)
PyObject *init(PyObject *, PyObject *args)
{
    unsigned long long a[9];
    PyObject *fail, *out_of_memory;
    if (!PyArg_ParseTuple(args, "(KKKKKKKKK)OO", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8, &fail, &out_of_memory)) return nullptr;
    const auto set = [](auto &f, unsigned long long p) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p); };
    set(g_quantize_rows, a[0]);
    set(g_dequantize_rows, a[1]);
    set(g_layer_norm, a[2]);
    set(g_layer_norm_backward_workspace, a[3]);
    set(g_layer_norm_backward, a[4]);
    set(g_linear_q8_workspace, a[5]);
    set(g_linear_q8, a[6]);
    set(g_linear_q8_backward_workspace, a[7]);
    set(g_linear_q8_backward, a[8]);
    Py_INCREF(fail);
    Py_XSETREF(g_fail, fail);
    Py_INCREF(out_of_memory);
    Py_XSETREF(g_out_of_memory, out_of_memory);
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr}, ENTRY(quantize_rows), ENTRY(dequantize_rows), ENTRY(layer_norm), ENTRY(layer_norm_backward), ENTRY(linear_q8),
                         ENTRY(linear_q8_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers(void) { return PyModule_Create(&module); }
