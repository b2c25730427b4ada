// Rows of eight elements at a time: loads, stores and reductions shared by the kernels on layers' activations (k7_*, k8_*).
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "internal.h"

namespace tictac {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// A float32 value as it is: the compiler would take a product and its conversion to float16 as one operation in some kernels and not in others.
__device__ __forceinline__ float settled(float v)
{
    asm("" : "+v"(v));
    return v;
}

// The element types of activations.  `raw` holds eight of them as they lie in memory; a load and its conversion are apart so that a
// kernel can have the next row's loads under way.
template <int DT>
struct Elem;

template <>
struct Elem<TICTAC_F32> {
    typedef float type;
    struct raw { f32x4 a, b; };
    static __device__ __forceinline__ raw load(const float *p) { return {*(const f32x4 *)p, *(const f32x4 *)(p + 4)}; }
    static __device__ __forceinline__ void floats(const raw &r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
    }
    static __device__ __forceinline__ raw pack(const float *v)
    {
        return {f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]}};
    }
    static __device__ __forceinline__ void store(float *p, const raw &r) { *(f32x4 *)p = r.a; *(f32x4 *)(p + 4) = r.b; }
    static __device__ __forceinline__ float to_float(float x) { return x; }
    static __device__ __forceinline__ float from_float(float x) { return x; }
};

template <>
struct Elem<TICTAC_F16> {
    typedef _Float16 type;
    struct raw { f16x2 a[4]; };
    static __device__ __forceinline__ raw load(const _Float16 *p) { return __builtin_bit_cast(raw, *(const i32x4 *)p); }
    static __device__ __forceinline__ void floats(const raw &r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)r.a[i >> 1][i & 1];
    }
    static __device__ __forceinline__ raw pack(const float *v)
    {
        raw r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.a[i >> 1][i & 1] = (_Float16)settled(v[i]);
        return r;
    }
    static __device__ __forceinline__ void store(_Float16 *p, const raw &r) { *(i32x4 *)p = __builtin_bit_cast(i32x4, r); }
    static __device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }
    static __device__ __forceinline__ _Float16 from_float(float x) { return (_Float16)settled(x); }
};

template <>
struct Elem<TICTAC_BF16> {
    typedef __bf16 type;
    struct raw { bf16x2 a[4]; };
    static __device__ __forceinline__ raw load(const __bf16 *p) { return __builtin_bit_cast(raw, *(const i32x4 *)p); }
    static __device__ __forceinline__ void floats(const raw &r, float *v)
    {
        const i32x4 w = __builtin_bit_cast(i32x4, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            v[2 * i + 1] = __builtin_bit_cast(float, (int32_t)(w[i] & 0xffff0000));
        }
    }
    static __device__ __forceinline__ raw pack(const float *v)
    {
        raw r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.a[i] = __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2);
        return r;
    }
    static __device__ __forceinline__ void store(__bf16 *p, const raw &r) { *(i32x4 *)p = __builtin_bit_cast(i32x4, r); }
    static __device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }
    static __device__ __forceinline__ __bf16 from_float(float x) { return (__bf16)x; }
};

// Eight elements anywhere in memory: the same loads and stores, which this GPU does at any boundary of an element.
template <int DT>
__device__ __forceinline__ typename Elem<DT>::raw load_anywhere(const typename Elem<DT>::type *p)
{
    typename Elem<DT>::raw r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <int DT>
__device__ __forceinline__ void store_anywhere(typename Elem<DT>::type *p, const typename Elem<DT>::raw &r) { __builtin_memcpy(p, &r, sizeof(r)); }

// Elements `col` .. `col` + 7 of a row of `cols`, zeros behind its end.  WIDE: rows start on 16-byte boundaries and hold a multiple of
// eight elements.
template <int DT, bool WIDE>
__device__ __forceinline__ typename Elem<DT>::raw load8(const typename Elem<DT>::type *row, int64_t col, int64_t cols)
{
    using E = Elem<DT>;
    if (WIDE) {
        if (col < cols) return E::load(row + col);
        return typename E::raw{};
    }
    if (col + 8 <= cols) return load_anywhere<DT>(row + col);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = E::to_float(row[min(col + i, cols - 1)]);          // (eight loads without a branch)
        v[i] = col + i < cols ? x : 0.0f;
    }
    return E::pack(v);              // (the values of the type: nothing is rounded)
}

// The same where a caller makes zeros of what lies behind the end: the row's last elements come again, without a branch.
template <int DT, bool WIDE>
__device__ __forceinline__ typename Elem<DT>::raw load8_or_last(const typename Elem<DT>::type *row, int64_t col, int64_t cols)
{
    if (WIDE) return Elem<DT>::load(row + min(col, cols - 8));
    return load8<DT, false>(row, col, cols);
}

template <int DT, bool WIDE>
__device__ __forceinline__ void store8(typename Elem<DT>::type *row, int64_t col, int64_t cols, const float *v)
{
    using E = Elem<DT>;
    if (WIDE) {
        if (col < cols) E::store(row + col, E::pack(v));
        return;
    }
    if (col + 8 <= cols) {
        store_anywhere<DT>(row + col, E::pack(v));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) row[col + i] = E::from_float(v[i]);
}

// Element i of a vector of parameters, float32 or of the activations' type (`dt` is the same for all threads).
__device__ __forceinline__ float param(const void *p, int dt, int64_t i)
{
    if (dt == TICTAC_F32) return ((const float *)p)[i];
    return dt == TICTAC_F16 ? (float)((const _Float16 *)p)[i] : (float)((const __bf16 *)p)[i];
}

__device__ __forceinline__ void put_param(void *p, int dt, int64_t i, float v)
{
    if (dt == TICTAC_F32) ((float *)p)[i] = v;
    else if (dt == TICTAC_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// Eight parameters from `col` on, zeros behind the end.
__device__ __forceinline__ void params8(const void *p, int dt, int64_t col, int64_t cols, float *v)
{
    if (col + 8 <= cols) {
        if (dt == TICTAC_F32) Elem<TICTAC_F32>::floats(load_anywhere<TICTAC_F32>((const float *)p + col), v);
        else if (dt == TICTAC_F16) Elem<TICTAC_F16>::floats(load_anywhere<TICTAC_F16>((const _Float16 *)p + col), v);
        else Elem<TICTAC_BF16>::floats(load_anywhere<TICTAC_BF16>((const __bf16 *)p + col), v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? param(p, dt, col + i) : 0.0f;
}

// Eight parameters from each of NC columns on, THREADS * 8 apart, zeros behind the end: all loads before the first conversion, those of a row's
// last columns too (forward, 4165 x 916 bfloat16: 7.4 us, 9.0 one chunk after the other; backward, 16000 x 2276: float32 114, 125, but 16-bit types 96, 80).
template <int PT, int THREADS, int NC>
__device__ __forceinline__ void params_of(const void *p, int64_t col, int64_t cols, float (&v)[NC][8])
{
    typename Elem<PT>::raw raw[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) raw[j] = load8<PT, false>((const typename Elem<PT>::type *)p, col + j * THREADS * 8, cols);
#pragma unroll
    for (int j = 0; j < NC; ++j) Elem<PT>::floats(raw[j], v[j]);
}
template <int THREADS, int NC>
__device__ __forceinline__ void params_at_once(const void *p, int dt, int64_t col, int64_t cols, float (&v)[NC][8])
{
    if (dt == TICTAC_F32) params_of<TICTAC_F32, THREADS, NC>(p, col, cols, v);
    else if (dt == TICTAC_F16) params_of<TICTAC_F16, THREADS, NC>(p, col, cols, v);
    else params_of<TICTAC_BF16, THREADS, NC>(p, col, cols, v);
}

// ---- reductions ----
template <int CTRL>
__device__ __forceinline__ float dpp0_f32(float v)              // a lane without a source gets zero
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_f32(float v)               // a lane without a source, or in another row, gets zero
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROW_MASK, 0xf, false));
}
// A maximum that keeps NaN (fmaxf drops it): magnitudes as integers, NaN's bits lie above infinity's.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp0_u32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// all 16 lanes of a row get its maximum (row_ror)
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
    v = max(v, dpp0_u32<0x121>(v));
    v = max(v, dpp0_u32<0x122>(v));
    v = max(v, dpp0_u32<0x124>(v));
    return max(v, dpp0_u32<0x128>(v));
}
__device__ __forceinline__ float wave_sum_f32(float v)           // all lanes get the sum
{
    v += dpp0_f32<0x111>(v);
    v += dpp0_f32<0x112>(v);
    v += dpp0_f32<0x114>(v);
    v += dpp0_f32<0x118>(v);
    v += dpp_f32<0x142, 0xa>(v);
    v += dpp_f32<0x143, 0xc>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    v = row16_max(v);
    v = max(max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16)),
            max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
    return v;
}

// ---- 8-bit rows ----
// amax is the largest magnitude of a row (or of a group of its columns), as bits.  scale = amax / 127 and q = round(x * (127 / amax)), ties
// to even.  What is below 2^-116 is stored as zeros (127 / amax would leave the range of float32, and amax / 127 its normal numbers).  A row with
// a NaN or an infinity gets a scale of NaN: all of it reads as NaN, so that the value that spoilt it is not lost.  The largest scale is the one
// whose product with 127 is finite (the next float would read back as infinity).
struct RowScale { float scale, inv; };
__device__ __forceinline__ RowScale row_scale(uint32_t amax)
{
    const float a = __builtin_bit_cast(float, amax);
    if (amax >= 0x7f800000u) return {__builtin_nanf(""), 0.0f};
    if (amax < 0x05800000u) return {0.0f, 0.0f};                // 2^-116
    return {fminf(a / 127.0f, 0x1.020406p+121f), 127.0f / a};
}
__device__ __forceinline__ uint2 quantized8(const float *v, const RowScale &s)
{
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = rintf(v[i] * s.inv);                    // |t| <= 127: |x| <= amax, and 127 rounds to itself
        const int32_t k = s.inv != 0.0f ? (int32_t)t : 0;       // (a row of zeros, or with a NaN)
        w[i >> 2] |= ((uint32_t)k & 0xffu) << (8 * (i & 3));
    }
    return uint2{w[0], w[1]};
}
__device__ __forceinline__ float whole8(uint2 q, int i)          // the i-th of eight
{
    return (float)(((int32_t)(i < 4 ? q.x : q.y) << (24 - 8 * (i & 3))) >> 24);
}
__device__ __forceinline__ void values8(uint2 q, float scale, float *v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = whole8(q, i) * scale;
}

inline int64_t rows8_stride(int64_t cols) { return (cols + 127) / 128 * 128; }
inline size_t elem_size(int dt) { return dt == TICTAC_F32 ? 4 : 2; }
// whether rows can be taken sixteen bytes at a time (load8, store8)
inline bool wide_rows(const void *p, int dt, int64_t ld, int64_t cols)
{
    return ((uintptr_t)p & 15) == 0 && (ld * elem_size(dt)) % 16 == 0 && cols % 8 == 0;
}

// f<type, wide>(...)
#define BY_TYPE(dt, wide, f, ...)                                                                               \
    ((dt) == TICTAC_F32    ? ((wide) ? f<TICTAC_F32, true>(__VA_ARGS__) : f<TICTAC_F32, false>(__VA_ARGS__))    \
     : (dt) == TICTAC_F16  ? ((wide) ? f<TICTAC_F16, true>(__VA_ARGS__) : f<TICTAC_F16, false>(__VA_ARGS__))    \
                           : ((wide) ? f<TICTAC_BF16, true>(__VA_ARGS__) : f<TICTAC_BF16, false>(__VA_ARGS__)))

}  // namespace tictac
