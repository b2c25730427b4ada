// AdamW over many tensors at once, and the norm of their gradients.
//   c  = grad_scale min(1, max_norm / norm),  g = c gradient
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g g
//   p' = p (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
// all in float32, each product and sum rounded by itself, so that moments in 8 bits do not depend on what a compiler contracts.  Moments in 8 bits are rows of e4m3 (f8.h) of m and
// of r = sqrt(v), which the update needs anyway: the range of r is half of v's in powers of two.  They are rounded at random, up with a probability of the part that is cut off: with
// b2 = 0.999 v decays by 0.1 % a step, and to nearest would never leave a value whose neighbours are 6 to 12 % away.  A positive r is a step of the type at least: it divides, and where it became zero
// the next step would have only 1 - b2 of a gradient's square under an m of up to a whole step (elements 2^-17 of their block's largest moved by up to 500 lr in a step; now by up to 4).
// Bound by memory: an element is read and written once.  67 million parameters with moments in 8 bits: 196 to 227 us, 4.8 to 5.5 TB/s (0.7 % of it for the least root, both in turn).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "f8.h"
#include "update.h"

namespace tictac {

// ---- the norm ----
// Squares and sums in float64: squares of float32 leave its range.  (176 tensors of 2^37 elements at most have fewer than 2^32 chunks.)  A workgroup's sum goes to the workspace, one workgroup adds those up: a fixed order, the same bits at every run.  Up to
// kNormOnce chunks one workgroup is all there is, and one launch (16 384 elements: 3.1 us, in two 4.4; 24 571 in three tensors 5.9 and 5.1).
constexpr int kNormTensors = 176, kNormBlocks = 2048, kNormOnce = 2, kNormChunk = 8192;

struct NormTable {
    const void *g[kNormTensors];
    int64_t numel[kNormTensors];
    uint32_t first[kNormTensors + 1];   // chunks before tensor i
    uint8_t dtype[kNormTensors];
    int32_t n;
};

// The tensor that has a chunk: the last whose first is no larger.  All of them are compared at once, by the lanes of a wave: a search by halves takes eight trips to the arguments, one behind
// the other.
template <class T>
__device__ __forceinline__ int32_t tensor_of(const T &table, uint32_t chunk)
{
    constexpr int kMost = (int)(sizeof(table.first) / sizeof(table.first[0])) - 1;
    const int lane = threadIdx.x & 63;
    int32_t before = 0;
#pragma unroll
    for (int k = 0; k < kMost; k += 64) {
        const int at = min(k + lane, kMost);
        before += __popcll(__ballot(k + lane < table.n && table.first[at] <= chunk));
    }
    return __builtin_amdgcn_readfirstlane(before) - 1;
}

// Eight elements of a vector as they lie in memory: loads and their conversion are apart, so that a branch on the type does not wait for each.
struct Raw8 {
    i32x4 a, b;
};
__device__ __forceinline__ Raw8 raw8(const void *p, int dt, int64_t at)
{
    Raw8 r;
    if (dt == TICTAC_F32) {
        const float *const q = (const float *)p + at;
        __builtin_memcpy(&r.a, q, 16);
        __builtin_memcpy(&r.b, q + 4, 16);
    } else {
        __builtin_memcpy(&r.a, (const uint16_t *)p + at, 16);
    }
    return r;
}
// the same where the vector may end among them, or before: zeros behind its end
__device__ __forceinline__ Raw8 raw8_within(const void *p, int dt, int64_t at, int64_t n)
{
    if (dt == TICTAC_F32) {
        const auto r = load8<TICTAC_F32, false>((const float *)p, at, n);
        return Raw8{__builtin_bit_cast(i32x4, r.a), __builtin_bit_cast(i32x4, r.b)};
    }
    if (dt == TICTAC_F16) return Raw8{__builtin_bit_cast(i32x4, load8<TICTAC_F16, false>((const _Float16 *)p, at, n)), i32x4{}};
    return Raw8{__builtin_bit_cast(i32x4, load8<TICTAC_BF16, false>((const __bf16 *)p, at, n)), i32x4{}};
}
__device__ __forceinline__ void raw_floats(const Raw8 &r, int dt, float *v)
{
    if (dt == TICTAC_F32) Elem<TICTAC_F32>::floats({__builtin_bit_cast(f32x4, r.a), __builtin_bit_cast(f32x4, r.b)}, v);
    else if (dt == TICTAC_F16) Elem<TICTAC_F16>::floats(__builtin_bit_cast(Elem<TICTAC_F16>::raw, r.a), v);
    else Elem<TICTAC_BF16>::floats(__builtin_bit_cast(Elem<TICTAC_BF16>::raw, r.a), v);
}

// the squares of a chunk that lies within its tensor, all loads under way at once
template <int DT>
__device__ __forceinline__ void add_squares(const void *g, int64_t at, double &sum)
{
    constexpr int kEach = kNormChunk / 2048;
    typename Elem<DT>::raw raw[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) raw[k] = load_anywhere<DT>((const typename Elem<DT>::type *)g + at + k * 2048);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        float v[8];
        Elem<DT>::floats(raw[k], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (double)v[e] * (double)v[e];
    }
}

// A workgroup has a run of chunks, which a walk through the table finds the tensors of.  67 million bfloat16 values: 26 us, 5 TB/s; 33 to 48 behind a
// step, whose writes are still on their way.
__global__ __launch_bounds__(256) void gradient_norm_kernel(NormTable table, double *parts, float scale, float *norm)
{
    __shared__ double part[4];
    const uint32_t chunks = table.first[table.n];
    uint32_t chunk = (uint32_t)((uint64_t)chunks * blockIdx.x / gridDim.x);
    const uint32_t last = (uint32_t)((uint64_t)chunks * (blockIdx.x + 1) / gridDim.x);
    int32_t i = tensor_of(table, chunk);
    double sum = 0.0;
    for (; chunk < last; ++chunk) {
        while (i + 1 < table.n && table.first[i + 1] <= chunk) ++i;
        const int64_t start = (int64_t)(chunk - table.first[i]) * kNormChunk, at = start + threadIdx.x * 8, n = table.numel[i];
        const void *const g = table.g[i];
        const int dt = table.dtype[i];
        if (start + kNormChunk <= n) {
            if (dt == TICTAC_F32) add_squares<TICTAC_F32>(g, at, sum);
            else if (dt == TICTAC_F16) add_squares<TICTAC_F16>(g, at, sum);
            else add_squares<TICTAC_BF16>(g, at, sum);
            continue;
        }
        for (int64_t k = at; k < n; k += 2048) {
            float v[8];
            params8(g, dt, k, n, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (double)v[e] * (double)v[e];
        }
    }
    sum = wave_sum_f64(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    if (norm) *norm = (float)(sqrt(sum) * (double)scale);               // (the only workgroup)
    else parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void gradient_norm_join_kernel(const double *parts, int32_t n, float scale, float *norm)
{
    __shared__ double part[4];
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < n; i += 256) sum += parts[i];
    sum = wave_sum_f64(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) *norm = (float)(sqrt((part[0] + part[1]) + (part[2] + part[3])) * (double)scale);
}

size_t gradient_norm_workspace(int32_t n) { return (size_t)std::max(1, (n + kNormTensors - 1) / kNormTensors) * kNormBlocks * sizeof(double); }

hipError_t launch_gradient_norm(int32_t n, const tictac_gradient *g, float scale, float *norm, double *workspace, hipStream_t s)
{
    int32_t parts = 0, i = 0;
    while (i < n) {
        NormTable table{};
        for (; i < n && table.n < kNormTensors; ++i) {
            if (g[i].numel == 0) continue;
            const int64_t chunks = (g[i].numel + kNormChunk - 1) / kNormChunk;
            table.g[table.n] = g[i].g;
            table.numel[table.n] = g[i].numel;
            table.dtype[table.n] = (uint8_t)g[i].dtype;
            table.first[table.n + 1] = table.first[table.n] + (uint32_t)chunks;
            ++table.n;
        }
        if (table.n == 0) break;
        const uint32_t blocks = std::min<uint32_t>(table.first[table.n], kNormBlocks);
        const bool once = blocks <= kNormOnce && parts == 0 && i == n;
        hipLaunchKernelGGL(gradient_norm_kernel, dim3(once ? 1 : blocks), dim3(256), 0, s, table, workspace + parts, scale, once ? norm : nullptr);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess || once) return e;
        parts += (int32_t)blocks;
    }
    hipLaunchKernelGGL(gradient_norm_join_kernel, dim3(1), dim3(256), 0, s, workspace, parts, scale, norm);
    return hipGetLastError();
}

// ---- the update ----
// A launch costs its start and its end, so descriptions are short.
constexpr int kUpdateChunk = 4096;

struct UpdateScales {
    uint8_t *m_scale, *v_scale;
};
struct NoScales {};
template <int BITS>
struct UpdateTensor : std::conditional_t<BITS == 8, UpdateScales, NoScales> {
    void *p, *m, *v, *copy;
    const void *g;
    uint64_t numel : 34, dtype : 2, grad_dtype : 2, copy_dtype : 2, number : 24;        // number: among all of the call
};
struct UpdateRates {
    float lr, beta1, beta2, rest1, rest2, eps, weight_decay, grad_scale, max_norm;
    float step_size, root;              // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), where lr and t are the host's
    double log1, log2;                  // of b1 and b2
    const float *norm, *lr_at;          // may be NULL
    const int64_t *step_at;             // may be NULL
    int64_t step;
    uint32_t seed_lo, seed_hi;
};
template <int BITS>
struct UpdateTable {
    static constexpr int kMost = (4096 - (int)sizeof(UpdateRates) - 16) / ((int)sizeof(UpdateTensor<BITS>) + 4);
    UpdateTensor<BITS> t[kMost];
    UpdateRates rates;
    uint32_t first[kMost + 1];          // chunks before tensor i
    int32_t n;
};

__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x9E3779B9u;
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    return x ^ (x >> 16);
}

// What all elements of a launch share.
struct UpdateFactors {
    float scale, keep, step_size, root;
    uint32_t key;
};

// `x` (a moment) in e4m3 under the scale of its block, up or down by 16 random bits: how many steps it is from zero, plus a part of a step, cut off; no fewer than `least`.
__device__ __forceinline__ float f8_at_random(float x, float inv, uint32_t bits, float least)
{
#pragma clang fp contract(off)
    const float y = x * inv, a = fabsf(y);
    // the exponent of the step: that of a, from -6 on, less 3
    const int32_t e = max((int32_t)(__builtin_bit_cast(uint32_t, a) >> 23) - 127, -6) - 3;
    const float k = fmaxf(floorf(a * __builtin_bit_cast(float, (uint32_t)(127 - e) << 23) + (float)bits * 0x1p-16f), least);
    return copysignf(k * __builtin_bit_cast(float, (uint32_t)(127 + e) << 23), y);
}

// Eight elements from `at` on: what they are, and what becomes of them.  FULL: none lies behind the end.
template <int BITS>
struct Elements {
    Raw8 g, p, m, v;
    uint32_t m_scale, v_scale;
    template <bool FULL>
    __device__ __forceinline__ void load(const UpdateTensor<BITS> &t, int64_t at)
    {
        const auto raw = [&](const void *from, int dt) { return FULL ? raw8(from, dt, at) : raw8_within(from, dt, at, t.numel); };
        g = raw(t.g, t.grad_dtype);
        p = raw(t.p, t.dtype);
        if constexpr (BITS == 32) {
            m = raw(t.m, TICTAC_F32);
            v = raw(t.v, TICTAC_F32);
        } else {                                                // (rows of moments go on to the next multiple of 128)
            __builtin_memcpy(&m.a, (const uint8_t *)t.m + at, 8);
            __builtin_memcpy(&v.a, (const uint8_t *)t.v + at, 8);
            m_scale = t.m_scale[at >> 7];
            v_scale = t.v_scale[at >> 7];
        }
    }
};

template <int BITS, bool FULL>
__device__ __forceinline__ void update8(const UpdateRates &table, const UpdateTensor<BITS> &t, const UpdateFactors &f, int64_t at, const Elements<BITS> &x)
{
#pragma clang fp contract(off)
    float p[8], g[8], m[8], v[8];
    raw_floats(x.g, t.grad_dtype, g);
    raw_floats(x.p, t.dtype, p);
    if constexpr (BITS == 32) {
        raw_floats(x.m, TICTAC_F32, m);
        raw_floats(x.v, TICTAC_F32, v);
    } else {
        f8_values8(uint2{(uint32_t)x.m.a[0], (uint32_t)x.m.a[1]}, x.m_scale, TICTAC_E4M3, m);
        f8_values8(uint2{(uint32_t)x.v.a[0], (uint32_t)x.v.a[1]}, x.v_scale, TICTAC_E4M3, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * v[i];
    }
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = g[i] * f.scale;
        m[i] = m[i] * table.beta1 + d * table.rest1;
        v[i] = v[i] * table.beta2 + (d * d) * table.rest2;
        r[i] = sqrtf(v[i]);
        p[i] = p[i] * f.keep - f.step_size * (m[i] / (r[i] * f.root + table.eps));
    }
    const auto put_as = [&](auto dt, void *to, const float *y) {
        constexpr int DT = decltype(dt)::value;
        typename Elem<DT>::type *const row = (typename Elem<DT>::type *)to;
        if constexpr (FULL) store_anywhere<DT>(row + at, Elem<DT>::pack(y));
        else store8<DT, false>(row, at, t.numel, y);
    };
    const auto put = [&](void *to, int dt, const float *y) {
        if (dt == TICTAC_F32) put_as(std::integral_constant<int, TICTAC_F32>(), to, y);
        else if (dt == TICTAC_F16) put_as(std::integral_constant<int, TICTAC_F16>(), to, y);
        else put_as(std::integral_constant<int, TICTAC_BF16>(), to, y);
    };
    put(t.p, t.dtype, p);
    if (t.copy) put(t.copy, t.copy_dtype, p);
    if constexpr (BITS == 32) {
        put(t.m, TICTAC_F32, m);
        put(t.v, TICTAC_F32, v);
    } else {
        uint32_t am = 0, ar = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { am = max(am, magnitude(m[i])); ar = max(ar, magnitude(r[i])); }
        const uint32_t sm = f8_scale(row16_max(am), TICTAC_E4M3), sr = f8_scale(row16_max(ar), TICTAC_E4M3);
        const float im = f8_inverse(sm), ir = f8_inverse(sr);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = mixed(f.key + (uint32_t)(at + i));
            m[i] = f8_at_random(m[i], im, bits & 0xffff, 0.0f);
            r[i] = f8_at_random(r[i], ir, bits >> 16, r[i] > 0.0f ? 1.0f : 0.0f);
        }
        const auto put8 = [&](void *to, uint8_t *scales, uint32_t scale, const float *y) {
            uint2 q{f8_pack4<TICTAC_E4M3>(y[0], y[1], y[2], y[3]), f8_pack4<TICTAC_E4M3>(y[4], y[5], y[6], y[7])};
            if (scale == 255) q = f8_nans(t.numel - at);
            *(uint2 *)((uint8_t *)to + at) = q;
            if ((threadIdx.x & 15) == 0) scales[at >> 7] = (uint8_t)scale;
        };
        put8(t.m, t.m_scale, sm, m);
        put8(t.v, t.v_scale, sr, r);
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(UpdateTable<BITS> table)
{
    const UpdateRates &rates = table.rates;
    UpdateFactors f;
    f.scale = rates.grad_scale;
    if (rates.norm) {
        const float norm = *rates.norm;
        if (!(norm < INFINITY)) return;                     // (no step with gradients that are not finite)
        f.scale = f.scale * fminf(rates.max_norm / norm, 1.0f);
    }
    const int32_t i = tensor_of(table, blockIdx.x);
    const UpdateTensor<BITS> &t = table.t[i];
    // (behind the loads: what it takes is not waited for before them)
    const auto factors = [&] {
        const float lr = rates.lr_at ? *rates.lr_at : rates.lr;
        const int64_t step = rates.step_at ? *rates.step_at : rates.step;
        f.keep = 1.0f - lr * rates.weight_decay;
        f.step_size = rates.step_size;
        f.root = rates.root;
        if (rates.lr_at || rates.step_at) {
            f.step_size = (float)((double)lr / -expm1((double)step * rates.log1));
            f.root = (float)(1.0 / sqrt(-expm1((double)step * rates.log2)));
        }
        f.key = mixed(mixed(mixed(mixed(rates.seed_lo) + rates.seed_hi) + (uint32_t)step) + t.number);
    };
    const int64_t start = (int64_t)(blockIdx.x - table.first[i]) * kUpdateChunk, at = start + threadIdx.x * 8;
    constexpr int kEach = kUpdateChunk / 2048;
    static_assert(kEach == 2, "two turns");
    Elements<BITS> x[kEach];
    if (start + kUpdateChunk <= (int64_t)t.numel) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) x[k].template load<true>(t, at + k * 2048);
        factors();
#pragma unroll
        for (int k = 0; k < kEach; ++k) update8<BITS, true>(rates, t, f, at + k * 2048, x[k]);
        return;
    }
    // the last of a tensor: all loads under way at once here too, one code for both turns (6 tensors of 1668 elements 5.4 us, with loads by turns 6.0)
    const int64_t end = BITS == 8 ? ((int64_t)t.numel + 127) / 128 * 128 : (int64_t)t.numel;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (at + k * 2048 < end) x[k].template load<false>(t, at + k * 2048);
    factors();
#pragma unroll 1
    for (int k = 0; k < kEach; ++k) {
        if (at + k * 2048 < end) update8<BITS, false>(rates, t, f, at + k * 2048, x[0]);
        x[0] = x[1];
    }
}

// the tensors with moments in BITS bits
template <int BITS>
static hipError_t launch_adamw(int32_t n, const tictac_adamw_tensor *t, const UpdateRates &rates, hipStream_t s)
{
    UpdateTable<BITS> table{};
    static_assert(sizeof(table) <= 4096, "a kernel's arguments");
    table.rates = rates;
    const auto launch = [&] {
        if (table.n == 0) return hipSuccess;
        hipLaunchKernelGGL(adamw_kernel<BITS>, dim3(table.first[table.n]), dim3(256), 0, s, table);
        table.n = 0;
        return hipGetLastError();
    };
    for (int32_t i = 0; i < n; ++i) {
        if ((t[i].m_scale != nullptr) != (BITS == 8) || t[i].numel == 0) continue;
        const int64_t chunks = (t[i].numel + kUpdateChunk - 1) / kUpdateChunk;
        if (table.n == table.kMost || (table.n && table.first[table.n] + chunks > INT32_MAX / 256))         // (a grid counts its threads in 32 bits)
            if (const hipError_t e = launch(); e != hipSuccess) return e;
        UpdateTensor<BITS> &u = table.t[table.n];
        u.p = t[i].p; u.m = t[i].m; u.v = t[i].v; u.copy = t[i].copy; u.g = t[i].g;
        if constexpr (BITS == 8) { u.m_scale = t[i].m_scale; u.v_scale = t[i].v_scale; }
        u.numel = (uint64_t)t[i].numel; u.dtype = (uint64_t)t[i].dtype; u.grad_dtype = (uint64_t)t[i].grad_dtype; u.copy_dtype = t[i].copy ? (uint64_t)t[i].copy_dtype : 0; u.number = (uint64_t)i;
        table.first[table.n + 1] = table.first[table.n] + (uint32_t)chunks;
        ++table.n;
    }
    return launch();
}

hipError_t launch_adamw_step(int32_t n, const tictac_adamw_tensor *t, const tictac_adamw_options &o, hipStream_t s)
{
    UpdateRates r{};
    r.lr = (float)o.lr;
    r.beta1 = (float)o.beta1;
    r.beta2 = (float)o.beta2;
    r.rest1 = (float)(1.0 - o.beta1);
    r.rest2 = (float)(1.0 - o.beta2);
    r.eps = (float)o.eps;
    r.weight_decay = (float)o.weight_decay;
    r.grad_scale = o.grad_scale;
    r.max_norm = o.max_norm;
    r.log1 = log(o.beta1);
    r.log2 = log(o.beta2);
    r.step_size = (float)(o.lr / -expm1((double)o.step * r.log1));
    r.root = (float)(1.0 / sqrt(-expm1((double)o.step * r.log2)));
    r.norm = o.norm;
    r.lr_at = o.lr_at;
    r.step_at = o.step_at;
    r.step = o.step;
    r.seed_lo = (uint32_t)o.seed;
    r.seed_hi = (uint32_t)(o.seed >> 32);
    if (const hipError_t e = launch_adamw<32>(n, t, r, s); e != hipSuccess) return e;
    return launch_adamw<8>(n, t, r, s);
}

}  // namespace tictac
