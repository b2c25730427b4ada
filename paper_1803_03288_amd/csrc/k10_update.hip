// AdamW over many tensors at once, and the norm of their gradients.
//   c  = grad_scale min(1, max_norm / norm),  g = c gradient
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g g
//   p' = p (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
// all in float32, each product and sum rounded by itself, so that moments in 8 bits do not depend on what a compiler contracts.  Moments in 8 bits are rows of e4m3 (f8.h) of m and
// of r = sqrt(v), which the update needs anyway: the range of r is half of v's in powers of two.  They are rounded at random, up with a probability of the part that is cut off: with
// b2 = 0.999 v decays by 0.1 % a step, and to nearest would never leave a value whose neighbours are 6 to 12 % away.
// Bound by memory: an element is read and written once.
#include <math.h>

#include <algorithm>

#include "device_utils.h"
#include "f8.h"
#include "update.h"

namespace tictac {

// ---- the norm ----
// Squares and sums in float64: squares of float32 leave its range.  A workgroup's sum goes to the workspace, one workgroup adds those up: a fixed order, the same bits at every run.
constexpr int kNormTensors = 128, kNormBlocks = 1024, kNormChunk = 4096;

struct NormTable {
    const void *g[kNormTensors];
    int64_t numel[kNormTensors];
    uint32_t first[kNormTensors + 1];   // chunks before tensor i
    uint8_t dtype[kNormTensors];
    int32_t n;
};

// the tensor that has a chunk: the last whose first is no larger
template <class T>
__device__ __forceinline__ int32_t tensor_of(const T &table, uint32_t chunk)
{
    int32_t lo = 0, hi = table.n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (table.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// eight elements from `at` on of a vector, zeros behind its end
__device__ __forceinline__ void floats8(const void *p, int dt, int64_t at, int64_t n, float *v) { params8(p, dt, at, n, v); }

__global__ __launch_bounds__(256) void gradient_norm_kernel(NormTable table, double *parts)
{
    __shared__ double part[4];
    double sum = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < table.first[table.n]; chunk += gridDim.x) {
        const int32_t i = tensor_of(table, chunk);
        const int64_t at = (int64_t)(chunk - table.first[i]) * kNormChunk + threadIdx.x * 8, n = table.numel[i];
        float v[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (at + k * 2048 < n) floats8(table.g[i], table.dtype[i], at + k * 2048, n, v[k]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (double)v[k][e] * (double)v[k][e];
    }
    sum = wave_sum_f64(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) parts[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
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
            if (table.first[table.n] + chunks > UINT32_MAX) break;
            table.g[table.n] = g[i].g;
            table.numel[table.n] = g[i].numel;
            table.dtype[table.n] = (uint8_t)g[i].dtype;
            table.first[table.n + 1] = table.first[table.n] + (uint32_t)chunks;
            ++table.n;
        }
        if (table.n == 0) break;
        const uint32_t blocks = std::min<uint32_t>(table.first[table.n], kNormBlocks);
        hipLaunchKernelGGL(gradient_norm_kernel, dim3(blocks), dim3(256), 0, s, table, workspace + parts);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        parts += (int32_t)blocks;
    }
    hipLaunchKernelGGL(gradient_norm_join_kernel, dim3(1), dim3(256), 0, s, workspace, parts, scale, norm);
    return hipGetLastError();
}

// ---- the update ----
constexpr int kUpdateTensors = 40, kUpdateChunk = 4096;

struct UpdateTensor {
    void *p, *m, *v, *copy;
    const void *g;
    uint8_t *m_scale, *v_scale;
    int64_t numel;
    uint32_t number;                    // among all of the call
    uint8_t dtype, grad_dtype, copy_dtype;
};
struct UpdateTable {
    UpdateTensor t[kUpdateTensors];
    uint32_t first[kUpdateTensors + 1]; // chunks before tensor i
    int32_t n;
    float lr, beta1, beta2, rest1, rest2, eps, weight_decay, grad_scale, max_norm;
    float step_size, root;              // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), where lr and t are the host's
    double log1, log2;                  // of b1 and b2
    const float *norm, *lr_at;          // may be NULL
    const int64_t *step_at;             // may be NULL
    int64_t step;
    uint32_t seed_lo, seed_hi;
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

// `x` (a moment) in e4m3 under the scale of its block, up or down by 16 random bits: how many steps it is from zero, plus a part of a step, cut off.
__device__ __forceinline__ float f8_at_random(float x, float inv, uint32_t bits)
{
#pragma clang fp contract(off)
    const float y = x * inv, a = fabsf(y);
    // the exponent of the step: that of a, from -6 on, less 3
    const int32_t e = max((int32_t)(__builtin_bit_cast(uint32_t, a) >> 23) - 127, -6) - 3;
    const float k = floorf(a * __builtin_bit_cast(float, (uint32_t)(127 - e) << 23) + (float)bits * 0x1p-16f);
    return copysignf(k * __builtin_bit_cast(float, (uint32_t)(127 + e) << 23), y);
}

template <int BITS>
__device__ __forceinline__ void update8(const UpdateTable &table, const UpdateTensor &t, const UpdateFactors &f, int64_t at)
{
#pragma clang fp contract(off)
    float p[8], g[8], m[8], v[8];
    floats8(t.g, t.grad_dtype, at, t.numel, g);
    floats8(t.p, t.dtype, at, t.numel, p);
    if constexpr (BITS == 32) {
        floats8(t.m, TICTAC_F32, at, t.numel, m);
        floats8(t.v, TICTAC_F32, at, t.numel, v);
    } else {
        f8_values8(*(const uint2 *)((const uint8_t *)t.m + at), t.m_scale[at >> 7], TICTAC_E4M3, m);
        f8_values8(*(const uint2 *)((const uint8_t *)t.v + at), t.v_scale[at >> 7], TICTAC_E4M3, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * v[i];
    }
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = g[i] * f.scale;
        m[i] = m[i] * table.beta1 + x * table.rest1;
        v[i] = v[i] * table.beta2 + (x * x) * table.rest2;
        r[i] = sqrtf(v[i]);
        p[i] = p[i] * f.keep - f.step_size * (m[i] / (r[i] * f.root + table.eps));
    }
    const auto put = [&](void *to, int dt, const float *x) {
        if (dt == TICTAC_F32) store8<TICTAC_F32, false>((float *)to, at, t.numel, x);
        else if (dt == TICTAC_F16) store8<TICTAC_F16, false>((_Float16 *)to, at, t.numel, x);
        else store8<TICTAC_BF16, false>((__bf16 *)to, at, t.numel, x);
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
            m[i] = f8_at_random(m[i], im, bits & 0xffff);
            r[i] = f8_at_random(r[i], ir, bits >> 16);
        }
        const auto put8 = [&](void *to, uint8_t *scales, uint32_t scale, const float *x) {
            uint2 q{f8_pack4<TICTAC_E4M3>(x[0], x[1], x[2], x[3]), f8_pack4<TICTAC_E4M3>(x[4], x[5], x[6], x[7])};
            if (scale == 255) q = f8_nans(t.numel - at);
            *(uint2 *)((uint8_t *)to + at) = q;
            if ((threadIdx.x & 15) == 0) scales[at >> 7] = (uint8_t)scale;
        };
        put8(t.m, t.m_scale, sm, m);
        put8(t.v, t.v_scale, sr, r);
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(UpdateTable table)
{
    UpdateFactors f;
    f.scale = table.grad_scale;
    if (table.norm) {
        const float norm = *table.norm;
        if (!(norm < INFINITY)) return;                     // (no step with gradients that are not finite)
        f.scale = f.scale * fminf(table.max_norm / norm, 1.0f);
    }
    const float lr = table.lr_at ? *table.lr_at : table.lr;
    const int64_t step = table.step_at ? *table.step_at : table.step;
    f.keep = 1.0f - lr * table.weight_decay;
    f.step_size = table.step_size;
    f.root = table.root;
    if (table.lr_at || table.step_at) {
        f.step_size = (float)((double)lr / -expm1((double)step * table.log1));
        f.root = (float)(1.0 / sqrt(-expm1((double)step * table.log2)));
    }
    const int32_t i = tensor_of(table, blockIdx.x);
    const UpdateTensor &t = table.t[i];
    f.key = mixed(mixed(mixed(mixed(table.seed_lo) + table.seed_hi) + (uint32_t)step) + t.number);
    const int64_t chunk = (int64_t)(blockIdx.x - table.first[i]) * kUpdateChunk + threadIdx.x * 8, end = BITS == 8 ? (t.numel + 127) / 128 * 128 : t.numel;
#pragma unroll
    for (int k = 0; k < kUpdateChunk / 2048; ++k)
        if (chunk + k * 2048 < end) update8<BITS>(table, t, f, chunk + k * 2048);
}

hipError_t launch_adamw_step(int32_t n, const tictac_adamw_tensor *t, const tictac_adamw_options &o, hipStream_t s)
{
    UpdateTable table{};
    static_assert(sizeof(UpdateTable) <= 4096, "a kernel's arguments");
    table.lr = (float)o.lr;
    table.beta1 = (float)o.beta1;
    table.beta2 = (float)o.beta2;
    table.rest1 = (float)(1.0 - o.beta1);
    table.rest2 = (float)(1.0 - o.beta2);
    table.eps = (float)o.eps;
    table.weight_decay = (float)o.weight_decay;
    table.grad_scale = o.grad_scale;
    table.max_norm = o.max_norm;
    table.log1 = log(o.beta1);
    table.log2 = log(o.beta2);
    table.step_size = (float)(o.lr / -expm1((double)o.step * table.log1));
    table.root = (float)(1.0 / sqrt(-expm1((double)o.step * table.log2)));
    table.norm = o.norm;
    table.lr_at = o.lr_at;
    table.step_at = o.step_at;
    table.step = o.step;
    table.seed_lo = (uint32_t)o.seed;
    table.seed_hi = (uint32_t)(o.seed >> 32);
    // tensors with moments in 32 bits, then those in 8
    for (int bits = 32; bits >= 8; bits -= 24) {
        table.n = 0;
        const auto launch = [&] {
            if (table.n == 0) return hipSuccess;
            if (bits == 32) hipLaunchKernelGGL(adamw_kernel<32>, dim3(table.first[table.n]), dim3(256), 0, s, table);
            else hipLaunchKernelGGL(adamw_kernel<8>, dim3(table.first[table.n]), dim3(256), 0, s, table);
            table.n = 0;
            return hipGetLastError();
        };
        for (int32_t i = 0; i < n; ++i) {
            if ((t[i].m_scale != nullptr) != (bits == 8) || t[i].numel == 0) continue;
            const int64_t chunks = (t[i].numel + kUpdateChunk - 1) / kUpdateChunk;
            if (table.n == kUpdateTensors || (table.n && table.first[table.n] + chunks > INT32_MAX / 256))
                if (const hipError_t e = launch(); e != hipSuccess) return e;
            UpdateTensor &u = table.t[table.n];
            u.p = t[i].p; u.m = t[i].m; u.v = t[i].v; u.copy = t[i].copy; u.g = t[i].g; u.m_scale = t[i].m_scale; u.v_scale = t[i].v_scale; u.numel = t[i].numel;
            u.number = (uint32_t)i; u.dtype = (uint8_t)t[i].dtype; u.grad_dtype = (uint8_t)t[i].grad_dtype; u.copy_dtype = (uint8_t)t[i].copy_dtype;
            table.first[table.n + 1] = table.first[table.n] + (uint32_t)chunks;
            ++table.n;
        }
        if (const hipError_t e = launch(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tictac
