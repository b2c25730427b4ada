// Entry points of products in 8-bit floats and of the update: checks of sizes, strides and pointers, then the launches of k9_*.hip and k10_update.hip.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <exception>
#include <utility>
#include <vector>

#include "api_checks.h"
#include "f8.h"
#include "update.h"

using namespace tictac;

namespace {

int check_format(const char *what, int32_t format)
{
    if (format == TICTAC_E4M3 || format == TICTAC_E5M2) return TICTAC_OK;
    set_error("%s = %d is no tictac_f8", what, format);
    return TICTAC_ERR_UNSUPPORTED;
}
int check_float8(const char *what, const tictac_float8 *f, int64_t rows, int64_t cols, int64_t most = INT64_C(1) << 40)
{
    if (!f) { set_error("%s is NULL", what); return TICTAC_ERR_NULL; }
    TT_CHECK(check_format(what, f->format));
    if (f->block != 1 && f->block != kF8Block) { set_error("%s: blocks of %d rows, expected 1 or %d", what, f->block, kF8Block); return TICTAC_ERR_UNSUPPORTED; }
    if (!f->q || !f->scale) { set_error("%s or its scales are NULL", what); return TICTAC_ERR_NULL; }
    const int64_t padded = f8_blocks(cols) * kF8Block, least = f8_scale_stride(cols);
    if (f->ld % kF8Block || f->ld < padded || f->ld > most) {
        set_error("stride of %s = %lld, expected a multiple of 128 from %lld to %lld", what, (long long)f->ld, (long long)padded, (long long)most);
        return TICTAC_ERR_UNSUPPORTED;
    }
    if (f->ld_scale % 4 || f->ld_scale < least || f->ld_scale > most) {
        set_error("stride of the scales of %s = %lld, expected a multiple of 4 from %lld to %lld", what, (long long)f->ld_scale, (long long)least, (long long)most);
        return TICTAC_ERR_UNSUPPORTED;
    }
    if ((uintptr_t)f->q & 15 || (uintptr_t)f->scale & 3) { set_error("%s: rows lie on 16-byte boundaries, scales on 4-byte ones", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
int check_weights(const tictac_float8 *w)
{
    if (w->format == TICTAC_E4M3) return TICTAC_OK;
    set_error("w: weights are e4m3");
    return TICTAC_ERR_UNSUPPORTED;
}
F8Rows rows_of(const tictac_float8 *f)
{
    if (!f) return F8Rows{};
    return F8Rows{(const uint8_t *)f->q, f->ld, f->scale, f->ld_scale, f->format, f->block == 1 ? 0 : 7};
}
F8QuantizeArgs quantize_args(int32_t dtype, int64_t rows, int64_t cols, const tictac_float8 *f, int64_t ld_x)
{
    F8QuantizeArgs a{};
    a.dtype = dtype; a.format = f->format; a.block = f->block; a.rows = rows; a.cols = cols; a.ld_x = ld_x;
    a.q = (uint8_t *)f->q; a.ld_q = f->ld; a.scale = f->scale; a.ld_scale = f->ld_scale;
    return a;
}
int check_count(int32_t n)
{
    if (n >= 0 && n < 1 << 24) return TICTAC_OK;
    set_error("n = %d tensors, expected fewer than 2^24", n);
    return TICTAC_ERR_UNSUPPORTED;
}
int check_backward(int64_t rows, int64_t cols, int64_t outs)
{
    TT_CHECK(check_product(rows, cols, outs));
    if (f8_blocks(rows) * f8_blocks(outs) + (f8_blocks(rows) + f8_blocks(outs)) * f8_blocks(cols) < 1 << 24) return TICTAC_OK;
    set_error("%lld rows, %lld columns, %lld outputs: more than 2^24 blocks of 128 x 128", (long long)rows, (long long)cols, (long long)outs);
    return TICTAC_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

int tictac_quantize_f8(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ld_x, const tictac_float8 *to, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_sizes(rows, cols));
    if (rows == 0) return TICTAC_OK;
    TT_CHECK(check_read("x", x, dtype, rows, ld_x));
    TT_CHECK(check_float8("to", to, rows, cols));
    if (to->block != 1 && f8_blocks(rows) * f8_blocks(cols) >= 1 << 23) { set_error("%lld rows of %lld columns: more than 2^23 blocks of 128 x 128", (long long)rows, (long long)cols); return TICTAC_ERR_UNSUPPORTED; }
    F8QuantizeArgs a = quantize_args(dtype, rows, cols, to, ld_x);
    a.x = x;
    HIP_TRY(launch_quantize_f8(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_dequantize_f8(int32_t dtype, int64_t rows, int64_t cols, const tictac_float8 *from, void *x, int64_t ld_x, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_sizes(rows, cols));
    if (rows == 0) return TICTAC_OK;
    TT_CHECK(check_float8("from", from, rows, cols));
    TT_CHECK(check_write("x", x, dtype, rows, cols, ld_x));
    F8QuantizeArgs a = quantize_args(dtype, rows, cols, from, ld_x);
    a.out = x;
    HIP_TRY(launch_dequantize_f8(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_f8_workspace(int32_t dtype, int32_t from_floats, int64_t rows, int64_t cols, int64_t outs, size_t *bytes)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_product(rows, cols, outs));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = linear_f8_workspace(dtype, from_floats, rows, cols, outs);
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_f8(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, const void *x, int64_t ld_x, const tictac_float8 *x8, const tictac_float8 *w,
                     int32_t bias_dtype, const void *bias, void *y, int64_t ld_y, void *workspace, size_t workspace_bytes, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_dtype("bias_dtype", bias_dtype));
    TT_CHECK(check_product(rows, cols, outs));
    if (rows == 0 || outs == 0) return TICTAC_OK;
    if (x && x8) { set_error("x and x8: expected one of them"); return TICTAC_ERR_UNSUPPORTED; }
    if (x8) TT_CHECK(check_float8("x8", x8, rows, cols, kMostStride));
    else TT_CHECK(check_read("x", x, dtype, rows, ld_x));
    TT_CHECK(check_float8("w", w, outs, cols, kMostStride));
    TT_CHECK(check_weights(w));
    TT_CHECK(check_floats("bias", bias, bias_dtype, false));
    TT_CHECK(check_write("y", y, dtype, rows, outs, ld_y));
    TT_CHECK(check_workspace(workspace, workspace_bytes, linear_f8_workspace(dtype, x != nullptr, rows, cols, outs)));
    LinearF8Args a{};
    a.dtype = dtype; a.bias_dtype = bias_dtype; a.rows = rows; a.cols = cols; a.outs = outs; a.x = x; a.ld_x = ld_x; a.x8 = rows_of(x8); a.w = rows_of(w);
    a.bias = bias; a.y = y; a.ld_y = ld_y; a.workspace = workspace;
    HIP_TRY(launch_linear_f8(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_f8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, size_t *bytes)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_backward(rows, cols, outs));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = rows && outs ? linear_f8_backward_workspace(dtype, rows, cols, outs) : 0;
    return TICTAC_OK;
} TT_CATCH

int tictac_linear_f8_backward(int32_t dtype, int64_t rows, int64_t cols, int64_t outs, const void *dy, int64_t ld_dy, int32_t format, const tictac_float8 *x8,
                              const tictac_float8 *w, void *dx, int64_t ld_dx, void *dw, int64_t ld_dw, void *db, void *workspace, size_t workspace_bytes, tictac_stream stream)
try {
    TT_CHECK(check_dtype("dtype", dtype));
    TT_CHECK(check_format("format", format));
    TT_CHECK(check_backward(rows, cols, outs));
    if (!dx && !dw && !db) return TICTAC_OK;
    if (rows && outs) {
        TT_CHECK(check_read("dy", dy, dtype, rows, ld_dy));
        if (dw) TT_CHECK(check_float8("x8", x8, rows, cols, kMostStride));
        if (dx) {
            TT_CHECK(check_float8("w", w, outs, cols, kMostStride));
            TT_CHECK(check_weights(w));
        }
        TT_CHECK(check_workspace(workspace, workspace_bytes, linear_f8_backward_workspace(dtype, rows, cols, outs)));
    }
    if (dx && rows) TT_CHECK(check_write("dx", dx, dtype, rows, cols, ld_dx));
    if (dw && outs) TT_CHECK(check_write("dw", dw, dtype, outs, cols, ld_dw));
    TT_CHECK(check_floats("db", db, dtype, false));
    LinearF8Args a{};
    a.dtype = dtype; a.format = format; a.rows = rows; a.cols = cols; a.outs = outs; a.dy = dy; a.ld_dy = ld_dy;
    if (dw) a.x8 = rows_of(x8);
    if (dx) a.w = rows_of(w);
    a.dx = dx; a.ld_dx = ld_dx; a.dw = dw; a.ld_dw = ld_dw; a.db = db; a.workspace = workspace;
    HIP_TRY(launch_linear_f8_backward(a, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_gradient_norm_workspace(int32_t n, size_t *bytes)
try {
    TT_CHECK(check_count(n));
    if (!bytes) { set_error("bytes is NULL"); return TICTAC_ERR_NULL; }
    *bytes = gradient_norm_workspace(n);
    return TICTAC_OK;
} TT_CATCH

int tictac_gradient_norm(int32_t n, const tictac_gradient *gradients, float scale, float *norm, void *workspace, size_t workspace_bytes, tictac_stream stream)
try {
    TT_CHECK(check_count(n));
    if (n && !gradients) { set_error("gradients is NULL"); return TICTAC_ERR_NULL; }
    TT_CHECK(check_floats("norm", norm, TICTAC_F32, true));
    if (!(fabsf(scale) < INFINITY)) { set_error("scale = %g", (double)scale); return TICTAC_ERR_UNSUPPORTED; }
    for (int32_t i = 0; i < n; ++i) {
        TT_CHECK(check_dtype("dtype of a gradient", gradients[i].dtype));
        if (gradients[i].numel < 0 || gradients[i].numel > INT64_C(1) << 37) { set_error("gradient %d of %lld elements", i, (long long)gradients[i].numel); return TICTAC_ERR_UNSUPPORTED; }
        TT_CHECK(check_floats("a gradient", gradients[i].g, gradients[i].dtype, gradients[i].numel > 0));
    }
    TT_CHECK(check_workspace(workspace, workspace_bytes, gradient_norm_workspace(n)));
    HIP_TRY(launch_gradient_norm(n, gradients, fabsf(scale), norm, (double *)workspace, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

int tictac_adamw_step(int32_t n, const tictac_adamw_tensor *tensors, const tictac_adamw_options *options, tictac_stream stream)
try {
    TT_CHECK(check_count(n));
    if ((n && !tensors) || !options) { set_error("tensors or options is NULL"); return TICTAC_ERR_NULL; }
    const tictac_adamw_options &o = *options;
    const auto number = [](double v) { return fabs(v) < INFINITY; };
    if (!(o.beta1 >= 0.0 && o.beta1 < 1.0 && o.beta2 >= 0.0 && o.beta2 < 1.0)) { set_error("beta1 = %g, beta2 = %g: expected 0 <= beta < 1", o.beta1, o.beta2); return TICTAC_ERR_UNSUPPORTED; }
    if (!(o.eps >= 0.0) || !number(o.eps) || !number(o.lr) || !number(o.weight_decay) || !number(o.grad_scale)) {
        set_error("lr = %g, eps = %g, weight_decay = %g, grad_scale = %g", o.lr, o.eps, o.weight_decay, (double)o.grad_scale);
        return TICTAC_ERR_UNSUPPORTED;
    }
    if (!o.step_at && o.step < 1) { set_error("step = %lld counts from 1", (long long)o.step); return TICTAC_ERR_UNSUPPORTED; }
    if (o.norm && !(o.max_norm > 0.0f)) { set_error("max_norm = %g", (double)o.max_norm); return TICTAC_ERR_UNSUPPORTED; }
    TT_CHECK(check_floats("norm", o.norm, TICTAC_F32, false));
    TT_CHECK(check_floats("lr_at", o.lr_at, TICTAC_F32, false));
    if ((uintptr_t)o.step_at & 7) { set_error("step_at does not lie on a boundary of its elements"); return TICTAC_ERR_UNSUPPORTED; }
    // what is read and written: begins, and ends of which the lowest bit says whether it is written
    std::vector<std::pair<uint64_t, uint64_t>> ranges;
    ranges.reserve((size_t)n * 7 + 3);
    const auto add = [&](const void *p, int64_t bytes, bool written) { ranges.emplace_back((uint64_t)(uintptr_t)p, ((uint64_t)(uintptr_t)p + (uint64_t)bytes) << 1 | written); };
    // (every workgroup reads these when it starts, behind others' ends)
    if (o.norm) add(o.norm, sizeof(*o.norm), false);
    if (o.lr_at) add(o.lr_at, sizeof(*o.lr_at), false);
    if (o.step_at) add(o.step_at, sizeof(*o.step_at), false);
    for (int32_t i = 0; i < n; ++i) {
        const tictac_adamw_tensor &t = tensors[i];
        TT_CHECK(check_dtype("dtype", t.dtype));
        TT_CHECK(check_dtype("grad_dtype", t.grad_dtype));
        if (t.copy) TT_CHECK(check_dtype("copy_dtype", t.copy_dtype));
        if (t.numel < 0 || t.numel > INT64_C(1) << 32) { set_error("tensor %d of %lld elements", i, (long long)t.numel); return TICTAC_ERR_UNSUPPORTED; }
        if (t.numel == 0) continue;
        TT_CHECK(check_floats("p", t.p, t.dtype, true));
        TT_CHECK(check_floats("g", t.g, t.grad_dtype, true));
        if (t.copy) TT_CHECK(check_floats("copy", t.copy, t.copy_dtype, true));
        const auto size = [](int32_t dtype) { return (int64_t)elem_size(dtype); };
        if (!t.m_scale != !t.v_scale) { set_error("tensor %d: one moment in 8 bits, one in 32", i); return TICTAC_ERR_UNSUPPORTED; }
        if (t.m_scale) {
            const tictac_float8 m{t.m, (t.numel + 127) / 128 * 128, t.m_scale, f8_scale_stride(t.numel), TICTAC_E4M3, 1}, v{t.v, m.ld, t.v_scale, m.ld_scale, TICTAC_E4M3, 1};
            TT_CHECK(check_float8("m", &m, 1, t.numel));
            TT_CHECK(check_float8("v", &v, 1, t.numel));
            add(t.m, m.ld, true);
            add(t.v, m.ld, true);
            add(t.m_scale, f8_blocks(t.numel), true);
            add(t.v_scale, f8_blocks(t.numel), true);
        } else {
            TT_CHECK(check_floats("m", t.m, TICTAC_F32, true));
            TT_CHECK(check_floats("v", t.v, TICTAC_F32, true));
            add(t.m, t.numel * 4, true);
            add(t.v, t.numel * 4, true);
        }
        add(t.p, t.numel * size(t.dtype), true);
        add(t.g, t.numel * size(t.grad_dtype), false);
        if (t.copy) add(t.copy, t.numel * size(t.copy_dtype), true);
    }
    std::sort(ranges.begin(), ranges.end());
    uint64_t end = 0, written_end = 0;
    for (const auto &[at, last] : ranges) {
        const bool written = last & 1;
        if (at < written_end || (written && at < end)) { set_error("tensors overlap: what one element writes is another's"); return TICTAC_ERR_UNSUPPORTED; }
        end = std::max(end, last >> 1);
        if (written) written_end = std::max(written_end, last >> 1);
    }
    HIP_TRY(launch_adamw_step(n, tensors, o, (hipStream_t)stream));
    return TICTAC_OK;
} TT_CATCH

}  // extern "C"
