// Entry points of the layers' operators: checks of sizes, strides and pointers, then the launches of k7_*.hip and k8_*.hip.
#include <hip/hip_runtime.h>

#include <exception>

#include "internal.h"

using namespace tictac;

namespace {

constexpr int64_t kMostCols = 131072;           // |q| <= 128: sums of the products of so many int8 values fit int32, but for one (exact_sum)
constexpr int64_t kMostRows = 1 << 21;          // of the products (offsets inside a tile are 32 bits)
constexpr int64_t kMostStride = 1 << 24;        // bytes between 8-bit rows of the products, for the same reason

int check_dtype(const char *what, int32_t dt)
{
    if (dt == TICTAC_F32 || dt == TICTAC_F16 || dt == TICTAC_BF16) return TICTAC_OK;
    set_error("%s = %d is no tictac_dtype", what, dt);
    return TICTAC_ERR_UNSUPPORTED;
}
int check_sizes(int64_t rows, int64_t cols)
{
    if (rows >= 0 && cols >= 1 && rows <= INT64_C(1) << 40 && cols <= INT64_C(1) << 30) return TICTAC_OK;
    set_error("%lld rows of %lld columns: expected no fewer than none of at least one (at most 2^40 of 2^30)", (long long)rows, (long long)cols);
    return TICTAC_ERR_UNSUPPORTED;
}
int check_group(int32_t group)
{
    if (group == 0 || group == kRows8Group) return TICTAC_OK;
    set_error("group = %d, expected 0 (a scale per row) or %d", group, kRows8Group);
    return TICTAC_ERR_UNSUPPORTED;
}
// rows that are read may lie on each other (a stride of zero: one row for all), rows that are written may not
int check_read(const char *what, const void *p, int32_t dt, int64_t rows, int64_t ld)
{
    if (!p) { set_error("%s is NULL", what); return TICTAC_ERR_NULL; }
    if (ld < 0 || ld > INT64_C(1) << 40) { set_error("stride of %s = %lld", what, (long long)ld); return TICTAC_ERR_UNSUPPORTED; }
    if ((uintptr_t)p % (dt == TICTAC_F32 ? 4 : 2)) { set_error("%s does not lie on a boundary of its elements", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_write(const char *what, const void *p, int32_t dt, int64_t rows, int64_t cols, int64_t ld)
{
    if (const int rc = check_read(what, p, dt, rows, ld); rc != TICTAC_OK) return rc;
    if (rows > 1 && ld < cols) { set_error("stride of %s = %lld, rows hold %lld", what, (long long)ld, (long long)cols); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_rows8(const char *what, const int8_t *q, const float *scale, int64_t rows, int64_t cols, int64_t ld, int64_t most = INT64_C(1) << 40)
{
    if (!q || !scale) { set_error("%s or its scales are NULL", what); return TICTAC_ERR_NULL; }
    const int64_t padded = (cols + 127) / 128 * 128;
    if (ld % 128 || ld < padded || ld > most) {
        set_error("stride of %s = %lld, expected a multiple of 128 from %lld to %lld", what, (long long)ld, (long long)padded, (long long)most);
        return TICTAC_ERR_UNSUPPORTED;
    }
    if ((uintptr_t)q & 15 || (uintptr_t)scale & 3) { set_error("%s: rows lie on 16-byte boundaries, scales on 4-byte ones", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_floats(const char *what, const void *p, int32_t dt, bool needed)
{
    if (!p && needed) { set_error("%s is NULL", what); return TICTAC_ERR_NULL; }
    if ((uintptr_t)p % (dt == TICTAC_F32 ? 4 : 2)) { set_error("%s does not lie on a boundary of its elements", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_workspace(const void *p, size_t have, size_t need)
{
    if (need && !p) { set_error("workspace is NULL, %zu bytes are needed", need); return TICTAC_ERR_NULL; }
    if (have < need) { set_error("workspace of %zu bytes, %zu are needed", have, need); return TICTAC_ERR_NO_MEM; }
    if ((uintptr_t)p & 255) { set_error("workspace does not lie on a 256-byte boundary"); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_product(int64_t rows, int64_t cols, int64_t outs)
{
    // (the last: tiles of a product, whose threads a grid counts in 32 bits)
    if (rows >= 0 && outs >= 0 && cols >= 1 && rows <= kMostRows && outs <= kMostRows && cols <= kMostCols && (rows + 255) / 256 * ((outs + 255) / 256) < 1 << 22)
        return TICTAC_OK;
    set_error("%lld rows, %lld columns, %lld outputs: the products take at most 2^21 rows and outputs of 1 to 2^17 columns", (long long)rows, (long long)cols, (long long)outs);
    return TICTAC_ERR_UNSUPPORTED;
}

#define TT_CHECK(expr)                               \
    do {                                             \
        const int rc_ = (expr);                      \
        if (rc_ != TICTAC_OK) return rc_;            \
    } while (0)

}  // namespace

extern "C" {

int tictac_quantize_rows(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ld_x, int32_t group, int8_t *q, int64_t ld_q, float *scale, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_sizes(rows, cols));
    TT_CHECK(check_group(group));
    if (rows == 0) return TICTAC_OK;
    TT_CHECK(check_read("x", x, dtype, rows, ld_x));
    TT_CHECK(check_rows8("q", q, scale, rows, cols, ld_q));
    QuantizeArgs a{};
    a.dtype = dtype; a.rows = rows; a.cols = cols; a.x = x; a.ld_x = ld_x; a.group = group; a.q = q; a.ld_q = ld_q; a.scale = scale;
    HIP_TRY(launch_quantize_rows(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_dequantize_rows(int32_t dtype, int64_t rows, int64_t cols, const int8_t *q, int64_t ld_q, const float *scale, int32_t group, void *x, int64_t ld_x, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_sizes(rows, cols));
    TT_CHECK(check_group(group));
    if (rows == 0) return TICTAC_OK;
    TT_CHECK(check_rows8("q", q, scale, rows, cols, ld_q));
    TT_CHECK(check_write("x", x, dtype, rows, cols, ld_x));
    QuantizeArgs a{};
    a.dtype = dtype; a.rows = rows; a.cols = cols; a.out = x; a.ld_x = ld_x; a.group = group;
    a.q = const_cast<int8_t *>(q); a.ld_q = ld_q; a.scale = const_cast<float *>(scale);
    HIP_TRY(launch_dequantize_rows(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_layer_norm(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ld_x, int32_t param_dtype, const void *weight, const void *bias, float eps,
                      void *y, int64_t ld_y, float *mean, float *rstd, int8_t *yq, int64_t ld_yq, float *y_scale, int8_t *xq, int64_t ld_xq, float *x_scale,
                      tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_dtype("param_dtype", param_dtype));
    TT_CHECK(check_sizes(rows, cols));
    if (!(eps >= 0.0f)) { set_error("eps = %g", (double)eps); return TICTAC_ERR_UNSUPPORTED; }
    if (rows == 0) return TICTAC_OK;
    TT_CHECK(check_read("x", x, dtype, rows, ld_x));
    TT_CHECK(check_floats("weight", weight, param_dtype, false));
    TT_CHECK(check_floats("bias", bias, param_dtype, false));
    TT_CHECK(check_floats("mean", mean, TICTAC_F32, true));
    TT_CHECK(check_floats("rstd", rstd, TICTAC_F32, true));
    if (y) TT_CHECK(check_write("y", y, dtype, rows, cols, ld_y));
    if (yq || y_scale) TT_CHECK(check_rows8("yq", yq, y_scale, rows, cols, ld_yq));
    if (xq || x_scale) TT_CHECK(check_rows8("xq", xq, x_scale, rows, cols, ld_xq));
    NormArgs a{};
    a.dtype = dtype; a.param_dtype = param_dtype; a.rows = rows; a.cols = cols; a.x = x; a.ld_x = ld_x; a.weight = weight; a.bias = bias; a.eps = eps;
    a.y = y; a.ld_y = ld_y; a.mean = mean; a.rstd = rstd; a.yq = yq; a.ld_yq = ld_yq; a.ys = y_scale; a.xq = xq; a.ld_xq = ld_xq; a.xs = x_scale;
    HIP_TRY(launch_layer_norm(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_layer_norm_backward_workspace(int64_t rows, int64_t cols, size_t *bytes)
try {
    TT_CHECK(check_sizes(rows, cols));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = layer_norm_backward_workspace(rows, cols);
    return TICTAC_OK;
} TT_CATCH

int tictac_layer_norm_backward(int32_t dtype, int64_t rows, int64_t cols, const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const int8_t *xq, int64_t ld_xq,
                               const float *x_scale, int32_t param_dtype, const void *weight, const float *mean, const float *rstd, void *dx, int64_t ld_dx, void *dweight,
                               void *dbias, void *workspace, size_t workspace_bytes, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_dtype("param_dtype", param_dtype));
    TT_CHECK(check_sizes(rows, cols));
    if (!dx && !dweight && !dbias) return TICTAC_OK;
    TT_CHECK(check_floats("weight", weight, param_dtype, false));
    TT_CHECK(check_floats("dweight", dweight, param_dtype, false));
    TT_CHECK(check_floats("dbias", dbias, param_dtype, false));
    const bool params = dweight || dbias;
    if (rows) {
        if (x && xq) { set_error("x and xq: expected one of them"); return TICTAC_ERR_UNSUPPORTED; }
        TT_CHECK(check_read("dy", dy, dtype, rows, ld_dy));
        if (xq) TT_CHECK(check_rows8("xq", xq, x_scale, rows, cols, ld_xq));
        else TT_CHECK(check_read("x", x, dtype, rows, ld_x));
        TT_CHECK(check_floats("mean", mean, TICTAC_F32, true));
        TT_CHECK(check_floats("rstd", rstd, TICTAC_F32, true));
        if (dx) TT_CHECK(check_write("dx", dx, dtype, rows, cols, ld_dx));
        if (params) TT_CHECK(check_workspace(workspace, workspace_bytes, layer_norm_backward_workspace(rows, cols)));
    }
    NormArgs a{};
    a.dtype = dtype; a.param_dtype = param_dtype; a.rows = rows; a.cols = cols; a.x = x; a.ld_x = ld_x; a.weight = weight;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.xq = const_cast<int8_t *>(xq); a.ld_xq = ld_xq; a.xs = const_cast<float *>(x_scale);
    a.dy = dy; a.ld_dy = ld_dy; a.dx = dx; a.ld_dx = ld_dx; a.dweight = dweight; a.dbias = dbias;
    a.workspace = params && layer_norm_backward_workspace(rows, cols) ? workspace : nullptr;
    HIP_TRY(launch_layer_norm_backward(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_q8_workspace(int32_t from_floats, int64_t rows, int64_t cols, int64_t outs, size_t *bytes)
try {
    TT_CHECK(check_product(rows, cols, outs));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = linear_q8_workspace(from_floats, rows, cols, outs);
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_q8(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, const void *x, int64_t ld_x, const int8_t *xq, int64_t ld_xq, const float *x_scale,
                     const int8_t *wq, int64_t ld_w, const float *w_scale, int32_t bias_dtype, const void *bias, void *y, int64_t ld_y, void *workspace, size_t workspace_bytes,
                     tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_dtype("bias_dtype", bias_dtype));
    TT_CHECK(check_product(rows, cols, outs));
    if (rows == 0 || outs == 0) return TICTAC_OK;
    if (x && xq) { set_error("x and xq: expected one of them"); return TICTAC_ERR_UNSUPPORTED; }
    if (xq) TT_CHECK(check_rows8("xq", xq, x_scale, rows, cols, ld_xq, kMostStride));
    else TT_CHECK(check_read("x", x, dtype, rows, ld_x));
    TT_CHECK(check_rows8("wq", wq, w_scale, outs, cols, ld_w, kMostStride));
    TT_CHECK(check_floats("bias", bias, bias_dtype, false));
    TT_CHECK(check_write("y", y, dtype, rows, outs, ld_y));
    TT_CHECK(check_workspace(workspace, workspace_bytes, linear_q8_workspace(x != nullptr, rows, cols, outs)));
    LinearArgs a{};
    a.dtype = dtype; a.bias_dtype = bias_dtype; a.rows = rows; a.cols = cols; a.outs = outs; a.x = x; a.ld_x = ld_x; a.xq = xq; a.ld_xq = ld_xq; a.xs = x_scale;
    a.w = wq; a.ld_w = ld_w; a.ws = w_scale; a.bias = bias; a.y = y; a.ld_y = ld_y; a.workspace = workspace;
    HIP_TRY(launch_linear_q8(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_q8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, size_t *bytes)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_product(rows, cols, outs));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = linear_q8_backward_workspace(dtype, rows, cols, outs);
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_q8_backward(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, const void *dy, int64_t ld_dy, const int8_t *xq, int64_t ld_xq, const float *x_scale,
                              const int8_t *wq, int64_t ld_w, const float *w_scale, void *dx, int64_t ld_dx, void *dw, int64_t ld_dw, void *db, void *workspace,
                              size_t workspace_bytes, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_product(rows, cols, outs));
    if (!dx && !dw && !db) return TICTAC_OK;
    if (rows && outs) {
        TT_CHECK(check_read("dy", dy, dtype, rows, ld_dy));
        if (dw) TT_CHECK(check_rows8("xq", xq, x_scale, rows, cols, ld_xq, kMostStride));
        if (dx) TT_CHECK(check_rows8("wq", wq, w_scale, outs, cols, ld_w, kMostStride));
        TT_CHECK(check_workspace(workspace, workspace_bytes, linear_q8_backward_workspace(dtype, rows, cols, outs)));
    }
    if (dx && rows) TT_CHECK(check_write("dx", dx, dtype, rows, cols, ld_dx));
    if (dw && outs) TT_CHECK(check_write("dw", dw, dtype, outs, cols, ld_dw));
    TT_CHECK(check_floats("db", db, dtype, false));
    LinearArgs a{};
    a.dtype = dtype; a.rows = rows; a.cols = cols; a.outs = outs; a.dy = dy; a.ld_dy = ld_dy; a.xq = xq; a.ld_xq = ld_xq; a.xs = x_scale;
    a.w = wq; a.ld_w = ld_w; a.ws = w_scale; a.dx = dx; a.ld_dx = ld_dx; a.dw = dw; a.ld_dw = ld_dw; a.db = db; a.workspace = workspace;
    HIP_TRY(launch_linear_q8_backward(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

}  // extern "C"
