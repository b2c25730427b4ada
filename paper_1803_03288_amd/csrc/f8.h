// 8-bit floats in blocks of 128 with a power of two as scale: the format of the k9_* kernels and of the moments of k10_update.hip.
//   A block is 128 columns of one row, or of 128 rows.  scale = 2^e, e the least from -126 on with amax <= 0.875 2^TOP 2^e (the largest value of the type:
//   448 or 57344); held as the byte e + 127.  q = x 2^-e rounded to the type, ties to even.
// A power of two loses nothing beside a scale of amax / 448 but half of the type's subnormal range: the values are floats.  Scaling then is exact, so q does not depend on the
// precision it is formed in; a block of 128 x 128 cut into blocks of one column keeps its values; and the matrix instruction takes such scales for nothing.
// Finite values read back finite: what rounding would take to 2^128 gets the type's value below that.  A NaN or an infinity in a block makes all of it NaN: the scale's byte is 255, and so are the values that lie in the tensor.
#pragma once

#include "rows8.h"

namespace tictac {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

constexpr int kF8Block = 128;

__device__ __forceinline__ int f8_top(int format) { return format == TICTAC_E5M2 ? 16 : 9; }

// the scale's byte for a largest magnitude, given by its bits: adding what lies above 1.75 carries into the exponent
__device__ __forceinline__ uint32_t f8_scale(uint32_t amax, int format)
{
    if (amax >= 0x7f800000u) return 255;
    return (uint32_t)max(1, (int32_t)((amax + 0x1fffffu) >> 23) + 1 - f8_top(format));
}
__device__ __forceinline__ float f8_inverse(uint32_t scale) { return __builtin_bit_cast(float, (254u - min(scale, 254u)) << 23); }
__device__ __forceinline__ float f8_factor(uint32_t scale)
{
    return __builtin_bit_cast(float, scale == 255 ? 0x7fc00000u : scale == 0 ? 0x00400000u : scale << 23);
}

template <int FORMAT>
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d)
{
    if (FORMAT == TICTAC_E5M2) return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ void f8_values4(uint32_t w, int format, float *v)
{
    const auto put = [&](auto lo, auto hi) { v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1]; };
    if (format == TICTAC_E5M2) put(__builtin_amdgcn_cvt_pk_f32_bf8((int)w, false), __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true));
    else put(__builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true));
}

// What eight values of a block that is NaN become: `left` of them lie before the row's end.
__device__ __forceinline__ uint2 f8_nans(int64_t left)
{
    const uint64_t all = left <= 0 ? 0 : 0x7f7f7f7f7f7f7f7full >> (8 * (8 - (left < 8 ? left : 8)));
    return uint2{(uint32_t)all, (uint32_t)(all >> 32)};
}
// Values of a block in 8 bits, without a branch: the kernels that turn operands round hold dozens of these, and what they wait for is their code.
template <int FORMAT>
__device__ __forceinline__ uint32_t f8_quantized4(const float *v, uint32_t scale, uint32_t nans)
{
    constexpr uint32_t kTop = FORMAT == TICTAC_E5M2 ? 16 : 9;
    const float inv = f8_inverse(scale), most = scale >= 256 - kTop ? (FORMAT == TICTAC_E5M2 ? 28672.0f : 240.0f) : (FORMAT == TICTAC_E5M2 ? 57344.0f : 448.0f);
    float u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_fmed3f(v[i] * inv, -most, most);        // (2^128 is out of float32's range)
    const uint32_t q = f8_pack4<FORMAT>(u[0], u[1], u[2], u[3]);
    return scale == 255 ? nans : q;
}
template <int FORMAT>
__device__ __forceinline__ uint2 f8_quantized8(const float *v, uint32_t scale, uint2 nans)
{
    return uint2{f8_quantized4<FORMAT>(v, scale, nans.x), f8_quantized4<FORMAT>(v + 4, scale, nans.y)};
}
__device__ __forceinline__ void f8_values8(uint2 q, uint32_t scale, int format, float *v)
{
    const float s = f8_factor(scale);
    f8_values4(q.x, format, v);
    f8_values4(q.y, format, v + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
}

// Values of an 8-bit type times a power of two as bf16: exact (what falls below bf16's range becomes zero).
__device__ __forceinline__ uint2 f8_bf16_4(const float *v)
{
    const auto two = [](float a, float b) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302); };
    return uint2{two(v[0], v[1]), two(v[2], v[3])};
}
__device__ __forceinline__ i32x4 f8_bf16(const float *v)
{
    const uint2 lo = f8_bf16_4(v), hi = f8_bf16_4(v + 4);
    return i32x4{(int32_t)lo.x, (int32_t)lo.y, (int32_t)hi.x, (int32_t)hi.y};
}

// An operand: blocks of `1 << shift` rows.
struct F8Rows {
    const uint8_t *q;
    int64_t ld;
    const uint8_t *scale;
    int64_t ld_scale;
    int32_t format, shift;
};

__host__ __device__ inline int64_t f8_blocks(int64_t n) { return (n + kF8Block - 1) / kF8Block; }
inline int64_t f8_scale_stride(int64_t cols) { return (f8_blocks(cols) + 3) / 4 * 4; }

// ---- k9_blocks.hip ----
struct F8QuantizeArgs {
    int32_t dtype, format, block;       // block: 1 or 128 rows
    int64_t rows, cols;
    const void *x;                      // to 8 bits
    void *out;                          // and back
    int64_t ld_x;
    uint8_t *q;
    int64_t ld_q;
    uint8_t *scale;
    int64_t ld_scale;
};
hipError_t launch_quantize_f8(const F8QuantizeArgs &a, hipStream_t s);
hipError_t launch_dequantize_f8(const F8QuantizeArgs &a, hipStream_t s);
// x (of float32, or where x.x is NULL of 8-bit floats) and w as bf16, [rows][padded], to `out`: ld_q of an x of float32; else cols is ld_x, the padded width
hipError_t launch_widen_f8(const F8QuantizeArgs &x, const F8QuantizeArgs &w, hipStream_t s);

// The operands of a backward pass: k contiguous and padded with zeros to whole blocks of 128; 8-bit floats with their scales, or where the gradients are float32 the values
// as bf16.  `dy` in blocks of its columns and (turned round) of its rows, x and w turned round.
struct F8Operand {
    void *q;                            // NULL: not needed
    int64_t ld;                         // elements
    uint8_t *scale;
    int64_t ld_scale;
};
struct F8TurnArgs {
    int32_t dtype, format;              // of dy, and what it is rounded to
    int64_t rows, cols, outs;
    const void *dy;
    int64_t ld_dy;
    F8Rows x, w;
    F8Operand dy_rows, dy_cols, x_cols, w_cols;
    float *sums;                        // [blocks of rows][outs]: sums of dy, may be NULL
};
hipError_t launch_turn_f8(const F8TurnArgs &a, hipStream_t s);

// ---- k9_linear.hip ----
struct LinearF8Args {
    int32_t dtype, bias_dtype, format;  // format: that dy is rounded to
    int64_t rows, cols, outs;
    const void *x;                      // float rows, rounded to e4m3, or NULL: x8
    int64_t ld_x;
    F8Rows x8, w;
    const void *bias;                   // may be NULL
    void *y;
    int64_t ld_y;
    void *workspace;
    // backward pass (dtype: of dy, dx, dw, db)
    const void *dy;
    int64_t ld_dy;
    void *dx, *dw, *db;                 // each may be NULL
    int64_t ld_dx, ld_dw;
};
hipError_t launch_linear_f8(const LinearF8Args &a, hipStream_t s);
size_t linear_f8_workspace(int32_t dtype, int32_t from_floats, int64_t rows, int64_t cols, int64_t outs);
hipError_t launch_linear_f8_backward(const LinearF8Args &a, hipStream_t s);
size_t linear_f8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs);

}  // namespace tictac
