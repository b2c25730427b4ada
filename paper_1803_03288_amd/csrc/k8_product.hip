// See k8_product.h.  A workgroup has a tile of the output, its waves a part of that each; the operands come through LDS in steps of 128
// bytes of k, two buffers in turn: while one is computed from, the next step is under way into the other, straight from memory to LDS.
#include "k8_product.h"

namespace tictac {

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

struct OpI8 {
    typedef i32x4 acc;
    static __device__ __forceinline__ acc mma(i32x4 a, i32x4 b, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};
struct OpBf16 {
    typedef f32x4 acc;
    static __device__ __forceinline__ acc mma(i32x4 a, i32x4 b, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ void put4(void *out, int dt, int64_t at, const float *v, int n)
{
    // (four outputs from `at` on; whole ones on an 8-byte boundary in one store)
    if (dt == TICTAC_F32) {
        float *o = (float *)out + at;
        if (n == 4 && ((uintptr_t)o & 15) == 0) { *(f32x4 *)o = f32x4{v[0], v[1], v[2], v[3]}; return; }
        for (int i = 0; i < n; ++i) o[i] = v[i];
        return;
    }
    uint2 w;
    if (dt == TICTAC_F16) {
        const f16x2 a{(_Float16)v[0], (_Float16)v[1]}, b{(_Float16)v[2], (_Float16)v[3]};
        w = uint2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    } else {
        w = uint2{__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2)),
                  __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2], v[3]}), bf16x2))};
    }
    uint16_t *o = (uint16_t *)out + at;
    if (n == 4 && ((uintptr_t)o & 7) == 0) { *(uint2 *)o = w; return; }
    for (int i = 0; i < n; ++i) o[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
}

// outputs r .. r + 3 of column c from their sums
template <typename ACC>
__device__ __forceinline__ void finish4(const ProductArgs &a, int32_t r, int32_t c, const ACC &sum)
{
    const int n = min(4, a.R - r);
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)sum[i];
    if (a.p_scale) {
        const float qs = a.q_scale[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= n) continue;
            v[i] *= qs * a.p_scale[r + i];
            if (a.bias) v[i] += param(a.bias, a.bias_dtype, r + i);
        }
    }
    put4(a.out, a.dtype, (int64_t)c * a.ld_out + r, v, n);
}

// TR x TC outputs per workgroup, WR x WC waves, FR x FC blocks of 16 x 16 per wave.
template <class OP, int WR, int WC, int FR, int FC>
__global__ __launch_bounds__(WR *WC * 64) void product_kernel(ProductArgs a, int32_t tiles_r, int32_t tiles_c)
{
    constexpr int TR = WR * FR * 16, TC = WC * FC * 16, kWaves = WR * WC;
    constexpr int LP = TR / 8 / kWaves, LQ = TC / 8 / kWaves;           // loads of 8 rows x 128 bytes per wave and step
    extern __shared__ char lds[];                                       // [2][TR + TC][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn; each XCD gets a run of consecutive tiles, and a run goes down eight columns of tiles
    // side by side, so that what an XCD's L2 holds is used again.
    const int32_t tiles = tiles_r * tiles_c;
    int32_t at = blockIdx.x % tiles;
    const int32_t split = blockIdx.x / tiles;
    {
        const int32_t xcd = at & 7, whole = tiles >> 3, more = tiles & 7;
        at = xcd * whole + min(xcd, more) + (at >> 3);
    }
    const int32_t band = at / (8 * tiles_r), in_band = at - band * 8 * tiles_r, width = min(8, tiles_c - band * 8);
    const int32_t r0 = in_band / width * TR, c0 = (band * 8 + in_band % width) * TC;

    const int32_t first = (int32_t)((int64_t)a.steps * split / a.splits), last = (int32_t)((int64_t)a.steps * (split + 1) / a.splits);
    // A load brings 8 rows of 128 bytes, lane l the sixteen bytes that belong at place l % 8 of row l / 8.  Place j of row i holds the
    // bytes 16 (j ^ i % 8) ..: eight rows of one k then lie in all banks.
    const int lrow = lane >> 3, lcol = ((lane & 7) ^ lrow) * 16;
    uint32_t off_p[LP], off_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) off_p[i] = (uint32_t)min(a.R - 1 - r0, (i * kWaves + wave) * 8 + lrow) * (uint32_t)a.ld_p + lcol;
#pragma unroll
    for (int i = 0; i < LQ; ++i) off_q[i] = (uint32_t)min(a.C - 1 - c0, (i * kWaves + wave) * 8 + lrow) * (uint32_t)a.ld_q + lcol;
    const char *base_p = a.p + (int64_t)r0 * a.ld_p, *base_q = a.q + (int64_t)c0 * a.ld_q;

    auto request = [&](int32_t step, int buffer) {
        char *to = lds + buffer * (TR + TC) * 128;
        const char *p = base_p + (int64_t)(step % a.p_steps) * 128, *q = base_q + (int64_t)step * 128;
#pragma unroll
        for (int i = 0; i < LP; ++i)
            __builtin_amdgcn_global_load_lds((global_void *)(p + off_p[i]), (lds_void *)(to + (i * kWaves + wave) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < LQ; ++i)
            __builtin_amdgcn_global_load_lds((global_void *)(q + off_q[i]), (lds_void *)(to + TR * 128 + (i * kWaves + wave) * 1024), 16, 0, 0);
    };

    const int wr = wave % WR, wc = wave / WR;
    typename OP::acc acc[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = typename OP::acc{};

    const int frow = lane & 15, fk = lane >> 4;
    if (first < last) request(first, 0);
    for (int32_t step = first; step < last; ++step) {
        const int buffer = (step - first) & 1;
        __syncthreads();                    // this step has come, and nobody reads the other buffer any more
        if (step + 1 < last) request(step + 1, buffer ^ 1);
        const char *tp = lds + buffer * (TR + TC) * 128 + (wr * FR * 16 + frow) * 128;
        const char *tq = lds + buffer * (TR + TC) * 128 + TR * 128 + (wc * FC * 16 + frow) * 128;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int place = ((k * 4 + fk) ^ (frow & 7)) * 16;
            i32x4 fp[FR], fq[FC];
#pragma unroll
            for (int j = 0; j < FC; ++j) fq[j] = *(const i32x4 *)(tq + j * 2048 + place);
#pragma unroll
            for (int i = 0; i < FR; ++i) fp[i] = *(const i32x4 *)(tp + i * 2048 + place);
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j) acc[i][j] = OP::mma(fp[i], fq[j], acc[i][j]);
        }
    }
    // lane l of a block of 16 x 16 holds rows 4 (l / 16) .. + 3 of column l % 16
#pragma unroll
    for (int j = 0; j < FC; ++j) {
        const int32_t c = c0 + (wc * FC + j) * 16 + frow;
        if (c >= a.C) continue;
#pragma unroll
        for (int i = 0; i < FR; ++i) {
            const int32_t r = r0 + (wr * FR + i) * 16 + fk * 4;
            if (r >= a.R) continue;
            if (a.splits == 1) {
                finish4(a, r, c, acc[i][j]);
            } else {
                uint32_t *part = (uint32_t *)a.parts + ((int64_t)split * a.C + c) * a.R + r;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const auto sum = acc[i][j][e];          // (a bit cast of a vector's element itself takes its first element)
                    if (r + e < a.R) part[e] = __builtin_bit_cast(uint32_t, sum);
                }
            }
        }
    }
}

// Adds up the splits in their order.
template <class OP>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, int32_t quads)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)quads * a.C) return;
    const int32_t c = (int32_t)(at / quads), r = (int32_t)(at % quads) * 4;
    typename OP::acc sum{};
    for (int32_t k = 0; k < a.splits; ++k) {
        const uint32_t *part = (const uint32_t *)a.parts + ((int64_t)k * a.C + c) * a.R + r;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r + e < a.R) sum[e] += __builtin_bit_cast(typename std::remove_reference<decltype(sum[0] + sum[0])>::type, part[e]);
    }
    finish4(a, r, c, sum);
}

constexpr int32_t kSmallTile = 128;

int32_t product_splits(int32_t R, int32_t C, int32_t steps)
{
    const int64_t tiles = (int64_t)((R + kSmallTile - 1) / kSmallTile) * ((C + kSmallTile - 1) / kSmallTile);
    if (tiles == 0 || tiles >= 256) return 1;
    int64_t n = 512 / tiles;                            // two workgroups of small tiles per compute unit
    if (n > steps / 4) n = steps / 4;                   // four steps at least for each
    return (int32_t)(n < 1 ? 1 : n > 16 ? 16 : n);
}

template <class OP>
static hipError_t launch(const ProductArgs &a, hipStream_t s)
{
    if (a.R == 0 || a.C == 0) return hipSuccess;
    const int64_t big = (int64_t)((a.R + 255) / 256) * ((a.C + 255) / 256);
    if (a.splits == 1 && big >= 192) {
        constexpr int lds = 2 * 512 * 128;
        const auto kernel = product_kernel<OP, 2, 4, 8, 4>;
        if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)big), dim3(512), lds, s, a, (a.R + 255) / 256, (a.C + 255) / 256);
        return hipGetLastError();
    }
    constexpr int lds = 2 * 256 * 128;
    const int32_t tr = (a.R + kSmallTile - 1) / kSmallTile, tc = (a.C + kSmallTile - 1) / kSmallTile;
    const auto kernel = product_kernel<OP, 2, 2, 4, 4>;
    if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tr * tc * a.splits), dim3(256), lds, s, a, tr, tc);
    if (a.splits > 1) {
        const int32_t quads = (a.R + 3) / 4;
        hipLaunchKernelGGL((product_join_kernel<OP>), dim3((unsigned)(((int64_t)quads * a.C + 255) / 256)), dim3(256), 0, s, a, quads);
    }
    return hipGetLastError();
}

hipError_t launch_product_i8(const ProductArgs &a, hipStream_t s) { return launch<OpI8>(a, s); }
hipError_t launch_product_bf16(const ProductArgs &a, hipStream_t s) { return launch<OpBf16>(a, s); }

}  // namespace tictac
