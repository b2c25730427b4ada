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

#include <cmath>
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
decltype(&tictac_quantize_f8) g_quantize_f8;
decltype(&tictac_dequantize_f8) g_dequantize_f8;
decltype(&tictac_linear_f8_workspace) g_linear_f8_workspace;
decltype(&tictac_linear_f8) g_linear_f8;
decltype(&tictac_linear_f8_backward_workspace) g_linear_f8_backward_workspace;
decltype(&tictac_linear_f8_backward) g_linear_f8_backward;
decltype(&tictac_gradient_norm_workspace) g_gradient_norm_workspace;
decltype(&tictac_gradient_norm) g_gradient_norm;
decltype(&tictac_adamw_step) g_adamw_step;
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

// ---- 8-bit floats in blocks, a tuple (q, scale, cols, block) ----
int f8_format(at::ScalarType t) { return t == at::kFloat8_e4m3fn ? TICTAC_E4M3 : t == at::kFloat8_e5m2 ? TICTAC_E5M2 : -1; }
int f8_format(PyObject *o, const char *name)
{
    const int f = THPDtype_Check(o) ? f8_format(reinterpret_cast<THPDtype *>(o)->scalar_type) : -1;
    if (f < 0) type_error(std::string(name) + ": expected float8_e4m3fn or float8_e5m2");
    return f;
}
int64_t scales_of(int64_t cols) { return (cols + 511) / 512 * 4; }       // bytes of a row of scales

struct Float8 {
    Tensor q, scale;
    int64_t rows, cols;
    tictac_float8 c;
};
// scales whose rows do not start on 4-byte boundaries, end before the next or lie on each other (one row for all) are copied, but where they will be written
Float8 float8(PyObject *o, const char *name, const at::Device *device, bool written = false)
{
    if (!is_rows8(o)) type_error(std::string(name) + ": expected Float8");
    Float8 r;
    r.q = tensor(PyTuple_GET_ITEM(o, 0), name);
    r.scale = tensor(PyTuple_GET_ITEM(o, 1), name);
    r.cols = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
    const int64_t block = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 3));
    if (PyErr_Occurred()) { PyErr_Clear(); type_error(std::string(name) + ": cols and block are whole numbers"); }
    if (block != 1 && block != kGroup) value_error(std::string(name) + ": blocks of " + str(block) + " rows, expected 1 or " + str(kGroup));
    const int format = f8_format(r.q.scalar_type());
    if (format < 0 || r.q.dim() != 2 || r.scale.dim() != 2 || r.scale.scalar_type() != at::kFloat8_e8m0fnu) type_error(std::string(name) + ": expected rows of float8_e4m3fn or float8_e5m2 and rows of float8_e8m0fnu scales");
    if (!device) check_device(r.q, name);
    if (r.q.device() != (device ? *device : r.scale.device()) || r.scale.device() != r.q.device()) value_error(std::string(name) + " is on another device");
    r.rows = r.q.size(0);
    if (r.cols < 1 || r.q.size(1) < padded(r.cols) || r.q.stride(1) != 1) value_error(std::string(name) + ": rows of " + str(r.cols) + " columns are padded to " + str(padded(r.cols)));
    const int64_t up = (r.rows + block - 1) / block, along = padded(r.cols) / kGroup;
    if (r.scale.size(0) != up || r.scale.size(1) < along)
        value_error(std::string(name) + ": scales of " + str(r.scale.size(0)) + " x " + str(r.scale.size(1)) + " blocks, expected " + str(up) + " x " + str(along));
    const bool as_is = r.scale.stride(1) == 1 && r.scale.size(1) >= scales_of(r.cols) && (up <= 1 || (r.scale.stride(0) % 4 == 0 && r.scale.stride(0) >= scales_of(r.cols))) && ((uintptr_t)r.scale.data_ptr() & 3) == 0;
    if (!as_is) {
        if (written) value_error(std::string(name) + ": scales lie on 4-byte boundaries, " + str(scales_of(r.cols)) + " of them");
        Tensor to = at::zeros({up, scales_of(r.cols)}, r.scale.options().dtype(at::kByte));
        to.narrow(1, 0, along).copy_(r.scale.narrow(1, 0, along).view(at::kByte));
        r.scale = to;
    }
    r.c = tictac_float8{r.q.data_ptr(), r.rows > 1 ? r.q.stride(0) : padded(r.q.size(1)), (uint8_t *)r.scale.data_ptr(), up > 1 ? r.scale.stride(0) : scales_of(r.cols), format, (int32_t)block};
    return r;
}

// (x, block, dtype) -> (q, scale)
PyObject *quantize_f8(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 3);
    const Rows x = float_rows(tensor(arg[0], "x"), "x");
    const int64_t block = PyLong_AsLongLong(arg[1]), ld = padded(x.cols);
    if (block != 1 && block != kGroup) {
        PyErr_Clear();
        value_error("block: expected 1 or " + str(kGroup));
    }
    const int format = f8_format(arg[2], "dtype");
    const Tensor q = empty({x.rows, ld}, reinterpret_cast<THPDtype *>(arg[2])->scalar_type, x.t), scale = empty({(x.rows + block - 1) / block, scales_of(x.cols)}, at::kFloat8_e8m0fnu, x.t);
    const tictac_float8 to{q.data_ptr(), ld, (uint8_t *)scale.data_ptr(), scales_of(x.cols), format, (int32_t)block};
    check(g_quantize_f8(x.dtype, x.rows, x.cols, x.data(), x.ld, &to, stream()));
    return tuple({q, scale});
}

// (float8, dtype) -> x
PyObject *dequantize_f8(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 2);
    const at::ScalarType type = dtype(arg[1], "dtype");
    const Float8 r = float8(arg[0], "r", nullptr);
    const Tensor x = empty({r.rows, r.cols}, type, r.q);
    check(g_dequantize_f8(dtype_code(type), r.rows, r.cols, &r.c, x.data_ptr(), r.cols, stream()));
    return wrap(x);
}

// (x, w, bias, dtype) -> y
PyObject *linear_f8(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 4);
    Rows x{};
    Float8 x8{};
    const bool ready = is_rows8(arg[0]);
    at::ScalarType type = at::kFloat;
    if (ready) {
        x8 = float8(arg[0], "x", nullptr);
        if (arg[3] != Py_None) type = dtype(arg[3], "dtype");
    } else {
        x = float_rows(tensor(arg[0], "x"), "x");
        type = x.t.scalar_type();
        if (arg[3] != Py_None && dtype(arg[3], "dtype") != type) type_error("dtype is not that of x");
    }
    const Tensor &like = ready ? x8.q : x.t;
    const at::Device device = like.device();
    const Float8 w = float8(arg[1], "w", &device);
    const int64_t rows = ready ? x8.rows : x.rows, cols = ready ? x8.cols : x.cols;
    if (w.cols != cols) value_error("x has " + str(cols) + " columns, w " + str(w.cols));
    const Vector bias = vector(arg[2], "bias", w.rows, type, like);
    const Tensor y = empty({rows, w.rows}, type, like);
    size_t bytes = 0;
    check(g_linear_f8_workspace(dtype_code(type), !ready, rows, cols, w.rows, &bytes));
    const Tensor room = workspace(bytes, like);
    check(g_linear_f8(dtype_code(type), rows, cols, w.rows, ready ? nullptr : x.data(), x.ld, ready ? &x8.c : nullptr, &w.c, bias.dtype, bias.data, y.data_ptr(), w.rows, ptr(room), bytes,
                      stream()));
    return wrap(ready ? y : shaped(y, tensor(arg[0], "x"), w.rows));
}

// (dy, x, w, dtype) -> (dx, dw, db)
PyObject *linear_f8_backward(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 4);
    const Tensor &given = tensor(arg[0], "dy");
    const Rows dy = float_rows(given, "dy");
    const at::Device device = dy.t.device();
    const Float8 x = float8(arg[1], "x", &device), w = float8(arg[2], "w", &device);
    const int format = f8_format(arg[3], "grad_dtype");
    if (x.rows != dy.rows || w.rows != dy.cols || w.cols != x.cols)
        value_error("dy is " + str(dy.rows) + " x " + str(dy.cols) + ", x " + str(x.rows) + " x " + str(x.cols) + ", w " + str(w.rows) + " x " + str(w.cols));
    const at::ScalarType type = given.scalar_type();
    const Tensor dx = empty({dy.rows, x.cols}, type, dy.t), dw = empty({dy.cols, x.cols}, type, dy.t), db = empty({dy.cols}, type, dy.t);
    size_t bytes = 0;
    check(g_linear_f8_backward_workspace(dy.dtype, dy.rows, x.cols, dy.cols, &bytes));
    const Tensor room = workspace(bytes, dy.t);
    check(g_linear_f8_backward(dy.dtype, dy.rows, x.cols, dy.cols, dy.data(), dy.ld, format, &x.c, &w.c, dx.data_ptr(), x.cols, dw.data_ptr(), x.cols, db.data_ptr(), ptr(room), bytes, stream()));
    return tuple({shaped(dx, given, x.cols), dw, db});
}

// ---- the update ----
struct Sequence {               // a list or tuple
    PyObject *fast;
    Sequence(PyObject *o, const char *name) : fast(PyList_Check(o) || PyTuple_Check(o) ? PySequence_Fast(o, "") : nullptr)
    {
        if (!fast) { PyErr_Clear(); type_error(std::string(name) + ": expected a list or tuple"); }
    }
    Sequence(const Sequence &) = delete;
    ~Sequence() { Py_DECREF(fast); }
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};
void same_length(const Sequence &s, const char *name, Py_ssize_t n)
{
    if (s.size() != n) value_error(std::string(name) + ": " + str(s.size()) + " of them for " + str(n) + " params");
}
std::string nth(const char *name, Py_ssize_t i) { return std::string(name) + "[" + str(i) + "]"; }
double real(PyObject *o, const char *name)
{
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) { PyErr_Clear(); type_error(std::string(name) + " is no number"); }
    return v;
}
// one number on the device
const void *one(PyObject *o, const char *name, at::ScalarType type)
{
    const Tensor &t = tensor(o, name);
    check_device(t, name);
    if (t.scalar_type() != type || t.numel() != 1 || t.is_neg()) value_error(std::string(name) + ": expected one " + toString(type) + " value");
    return t.data_ptr();
}
int float_code(const Tensor &t, const char *name, Py_ssize_t i)
{
    const int dt = dtype_code(t.scalar_type());
    if (dt < 0) type_error(nth(name, i) + " is " + toString(t.scalar_type()) + ": expected float32, float16 or bfloat16");
    return dt;
}
// tensor i of many on the current device, which `here` (-1 at first) remembers
const Tensor &one_of(PyObject *from, const char *name, Py_ssize_t i, c10::DeviceIndex &here)
{
    if (!THPVariable_Check(from)) type_error(nth(name, i) + " is no tensor");
    const Tensor &t = THPVariable_Unpack(from);
    if (!t.is_cuda() || t.get_device() != here) {
        check_device(t, nth(name, i).c_str());
        here = (c10::DeviceIndex)t.get_device();
    }
    return t;
}

// (gradients, scale) -> norm
PyObject *gradient_norm(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 2);
    const Sequence grads(arg[0], "grads");
    const float scale = (float)real(arg[1], "scale");
    if (grads.size() == 0) value_error("grads: none");
    std::vector<Tensor> kept;
    std::vector<tictac_gradient> all;
    all.reserve(grads.size());
    c10::DeviceIndex here = -1;
    for (Py_ssize_t i = 0; i < grads.size(); ++i) {
        const Tensor &t = one_of(grads[i], "grads", i, here);
        const int dt = float_code(t, "grads", i);
        const Tensor *at = &t;                                          // (signs turned lazily, and the order of elements, do not matter)
        if (!t.is_non_overlapping_and_dense()) {
            kept.push_back(t.contiguous());
            at = &kept.back();
        }
        all.push_back({at->data_ptr(), at->numel(), dt});
    }
    const Tensor &like = tensor(grads[0], "a gradient");
    const Tensor norm = empty({}, at::kFloat, like);
    size_t bytes = 0;
    check(g_gradient_norm_workspace((int32_t)all.size(), &bytes));
    const Tensor room = workspace(bytes, like);
    check(g_gradient_norm((int32_t)all.size(), all.data(), scale, (float *)norm.data_ptr(), ptr(room), bytes, stream()));
    return wrap(norm);
}

// what is written in place: the version that autograd sees goes up
void written(c10::TensorImpl *t)
{
    if (!t->is_inference()) t->bump_version();
}

// (params, grads, moments, step, lr, (beta1, beta2), eps, weight_decay, grad_scale, norm, max_norm, copies, seed)
PyObject *adamw_step(PyObject *const *arg, Py_ssize_t n)
{
    take(n, 13);
    const Sequence params(arg[0], "params"), grads(arg[1], "grads"), moments(arg[2], "moments");
    const Py_ssize_t count = params.size();
    same_length(grads, "grads", count);
    same_length(moments, "moments", count);
    c10::optional<Sequence> copies;
    if (arg[11] != Py_None) {
        copies.emplace(arg[11], "copies");
        same_length(*copies, "copies", count);
    }
    tictac_adamw_options o{};
    if (THPVariable_Check(arg[3])) {
        o.step_at = (const int64_t *)one(arg[3], "step", at::kLong);
        o.step = 1;
    } else {
        o.step = PyLong_AsLongLong(arg[3]);
        if (PyErr_Occurred()) { PyErr_Clear(); type_error("step is no whole number"); }
        if (o.step < 1) value_error("step counts from 1");
    }
    if (THPVariable_Check(arg[4])) o.lr_at = (const float *)one(arg[4], "lr", at::kFloat);
    else o.lr = real(arg[4], "lr");
    const Sequence betas(arg[5], "betas");
    if (betas.size() != 2) value_error("betas: expected two");
    o.beta1 = real(betas[0], "betas");
    o.beta2 = real(betas[1], "betas");
    o.eps = real(arg[6], "eps");
    o.weight_decay = real(arg[7], "weight_decay");
    o.grad_scale = (float)real(arg[8], "grad_scale");
    if (arg[9] != Py_None) o.norm = (const float *)one(arg[9], "norm", at::kFloat);
    o.max_norm = INFINITY;
    if (arg[10] != Py_None) {
        if (!o.norm) value_error("max_norm without norm");
        o.max_norm = (float)real(arg[10], "max_norm");
        if (!(o.max_norm > 0)) value_error("max_norm: expected more than zero");
    }
    o.seed = PyLong_AsUnsignedLongLongMask(arg[12]);
    if (PyErr_Occurred()) { PyErr_Clear(); type_error("seed is no whole number"); }
    std::vector<tictac_adamw_tensor> all;
    std::vector<Tensor> kept;
    std::vector<c10::TensorImpl *> outputs;                              // (which the arguments keep alive)
    all.reserve(count);
    outputs.reserve(count * 4);
    c10::DeviceIndex here = -1;
    for (Py_ssize_t i = 0; i < count; ++i) {
        const auto a_tensor = [&](PyObject *from, const char *name) -> const Tensor & { return one_of(from, name, i, here); };
        tictac_adamw_tensor u{};
        const Tensor &p = a_tensor(params[i], "params");
        u.dtype = float_code(p, "params", i);
        if (!p.is_non_overlapping_and_dense() || p.is_neg()) value_error(nth("params", i) + " has gaps or overlaps, or its signs turned lazily: it is changed in place");
        u.p = p.data_ptr();
        u.numel = p.numel();
        outputs.push_back(p.unsafeGetTensorImpl());
        const Tensor &g = a_tensor(grads[i], "grads");
        u.grad_dtype = float_code(g, "grads", i);
        if (g.sizes() != p.sizes()) value_error(nth("grads", i) + " has another shape than its parameter");
        if (g.strides() == p.strides() && !g.is_neg()) {
            u.g = g.data_ptr();
        } else {                                                        // in the order in which the parameter's elements lie
            kept.push_back(at::empty_strided(p.sizes(), p.strides(), g.options().requires_grad(false)).copy_(g));
            u.g = kept.back().data_ptr();
        }
        if (copies && (*copies)[i] != Py_None) {
            const Tensor &c = a_tensor((*copies)[i], "copies");
            u.copy_dtype = float_code(c, "copies", i);
            if (c.sizes() != p.sizes() || c.strides() != p.strides() || c.is_neg()) value_error(nth("copies", i) + " has another shape or other strides than its parameter");
            u.copy = c.data_ptr();
            outputs.push_back(c.unsafeGetTensorImpl());
        }
        if (!PyTuple_Check(moments[i]) || PyTuple_GET_SIZE(moments[i]) != 2) type_error(nth("moments", i) + ": expected Moments");
        for (int k = 0; k < 2; ++k) {
            PyObject *const from = PyTuple_GET_ITEM(moments[i], k);
            void *&to = k ? u.v : u.m;
            if (PyTuple_Check(from)) {
                const Float8 f = float8(from, "moments", nullptr, true);
                if (f.rows != 1 || f.cols != u.numel || f.c.block != 1 || f.c.format != TICTAC_E4M3) value_error(nth("moments", i) + ": expected one row of " + str(u.numel) + " columns of float8_e4m3fn in blocks of one row");
                to = f.c.q;
                (k ? u.v_scale : u.m_scale) = f.c.scale;
                outputs.push_back(f.q.unsafeGetTensorImpl());
                outputs.push_back(f.scale.unsafeGetTensorImpl());
            } else {
                const Tensor &t = a_tensor(from, "moments");
                if (t.scalar_type() != at::kFloat) type_error(nth("moments", i) + ": expected float32 or Float8");
                if (t.numel() != u.numel || t.is_neg() || !(t.dim() == 1 ? t.is_contiguous() : t.sizes() == p.sizes() && t.strides() == p.strides()))
                    value_error(nth("moments", i) + ": expected " + str(u.numel) + " elements, in one row or with the strides of its parameter");
                to = t.data_ptr();
                outputs.push_back(t.unsafeGetTensorImpl());
            }
        }
        if (!u.m_scale != !u.v_scale) value_error(nth("moments", i) + ": one in 8 bits, one in 32");
        all.push_back(u);
    }
    check(g_adamw_step((int32_t)all.size(), all.data(), &o, stream()));
    for (c10::TensorImpl *const t : outputs) written(t);
    Py_RETURN_NONE;
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

// (addresses of the C calls, the function that raises the error of a status, torch.OutOfMemoryError)
PyObject *init(PyObject *, PyObject *args)
{
    PyObject *calls, *fail, *out_of_memory;
    if (!PyArg_ParseTuple(args, "O!OO", &PyTuple_Type, &calls, &fail, &out_of_memory)) return nullptr;
    constexpr Py_ssize_t kCalls = 18;
    if (PyTuple_GET_SIZE(calls) != kCalls) {
        PyErr_SetString(PyExc_TypeError, "init: another number of calls");
        return nullptr;
    }
    unsigned long long a[kCalls];
    for (Py_ssize_t i = 0; i < kCalls; ++i) a[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(calls, i));
    if (PyErr_Occurred()) return nullptr;
    const unsigned long long *next = a;
    const auto set = [&](auto &f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(*next++); };
    set(g_quantize_rows);
    set(g_dequantize_rows);
    set(g_layer_norm);
    set(g_layer_norm_backward_workspace);
    set(g_layer_norm_backward);
    set(g_linear_q8_workspace);
    set(g_linear_q8);
    set(g_linear_q8_backward_workspace);
    set(g_linear_q8_backward);
    set(g_quantize_f8);
    set(g_dequantize_f8);
    set(g_linear_f8_workspace);
    set(g_linear_f8);
    set(g_linear_f8_backward_workspace);
    set(g_linear_f8_backward);
    set(g_gradient_norm_workspace);
    set(g_gradient_norm);
    set(g_adamw_step);
    Py_INCREF(fail);
    Py_XSETREF(g_fail, fail);
    Py_INCREF(out_of_memory);
    Py_XSETREF(g_out_of_memory, out_of_memory);
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr}, ENTRY(quantize_rows), ENTRY(dequantize_rows), ENTRY(layer_norm), ENTRY(layer_norm_backward), ENTRY(linear_q8),
                         ENTRY(linear_q8_backward), ENTRY(quantize_f8), ENTRY(dequantize_f8), ENTRY(linear_f8), ENTRY(linear_f8_backward), ENTRY(gradient_norm), ENTRY(adamw_step),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers(void) { return PyModule_Create(&module); }
