// What the tiled products share (k8_product.hip: int8 and bf16; k9_product.hip: 8-bit floats): which tile a workgroup has, the loads that bring its operands to LDS, and
// how outputs leave the registers.
#pragma once

#include "device_utils.h"
#include "k8_product.h"

namespace tictac {

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// ---- outputs ----
// What becomes of an operation's sums: scales of rows and columns and the bias, the bias alone, or nothing.
template <class OP>
struct Scaled { static constexpr bool value = false; };
template <class OP>
struct Biased { static constexpr bool value = false; };

// Eight outputs r .. r + 7 of a column from their sums.  The scales and the bias of r are the same for all columns of a thread.
template <bool SCALED, bool BIASED>
struct Finish8 {
    float scale[8], bias[8];
    __device__ __forceinline__ void init(const ProductArgs &a, int32_t r)
    {
        if (!SCALED && !BIASED) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (SCALED) scale[i] = r + i < a.R ? a.p_scale[r + i] : 0.0f;
            bias[i] = a.bias && r + i < a.R ? param(a.bias, a.bias_dtype, r + i) : 0.0f;
        }
    }
    template <int DT>
    __device__ __forceinline__ void store(const ProductArgs &a, int32_t r, int32_t c, const float *sum, bool wide) const
    {
        float v[8];
        if (SCALED) {
            const float qs = a.q_scale[c];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = sum[i] * (qs * scale[i]) + bias[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = BIASED ? sum[i] + bias[i] : sum[i];
        }
        typename Elem<DT>::type *row = (typename Elem<DT>::type *)a.out + (int64_t)c * a.ld_out;
        if (wide) store8<DT, true>(row, r, a.R, v);
        else store8<DT, false>(row, r, a.R, v);
    }
};

constexpr int kParts = 3;           // in the place of an output type: sums of a split, as they are

// What a wave holds, FR x FC blocks of 16 x 16 from (r, c) on, goes column by column through its own part of LDS, so that a thread has eight
// consecutive outputs.  Lane l of a block holds rows 4 (l / 16) .. + 3 of column l % 16.
template <class OP, int OUT, int FR, int FC>
__device__ __forceinline__ void put_blocks(const ProductArgs &a, const typename OP::acc (&acc)[FR][FC], int32_t r, int32_t c, int32_t split, char *room)
{
    typedef typename OP::acc A;
    constexpr int kStride = FR * 16 + 4, kThreads = FR * 2, kColumns = 64 / kThreads;       // words; threads per column; columns at a time
    const int lane = threadIdx.x & 63, part = lane % kThreads, first = lane / kThreads;
    A *to = (A *)room + ((lane & 15) * kStride + (lane >> 4) * 4) / 4;
    const A *from = (const A *)room + (first * kStride + part * 8) / 4;
    const int32_t mine = r + part * 8;
    Finish8<Scaled<OP>::value && OUT != kParts, Biased<OP>::value && OUT != kParts> finish;
    finish.init(a, mine);
    const bool wide = OUT != kParts && (a.ld_out * (OUT == TICTAC_F32 ? 4 : 2)) % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.R % 8 == 0;
#pragma unroll
    for (int j = 0; j < FC; ++j) {
#pragma unroll
        for (int i = 0; i < FR; ++i) to[i * 4] = acc[i][j];
        wave_sync();
#pragma unroll
        for (int k = 0; k < 16 / kColumns; ++k) {
            const A lo = from[k * kColumns * kStride / 4], hi = from[k * kColumns * kStride / 4 + 1];
            const int32_t column = c + j * 16 + k * kColumns + first;
            if (column >= a.C || mine >= a.R) continue;
            if constexpr (OUT == kParts) {
                A *out = (A *)((uint32_t *)a.parts + ((int64_t)split * a.C + column) * a.R + mine);
                if (a.R % 8 == 0) {
                    out[0] = lo;
                    out[1] = hi;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const auto sum = e < 4 ? lo[e & 3] : hi[e & 3];         // (a bit cast of a vector's element itself takes its first element)
                        if (mine + e < a.R) ((uint32_t *)out)[e] = __builtin_bit_cast(uint32_t, sum);
                    }
                }
            } else {
                float sum[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) { sum[e] = OP::value(lo[e]); sum[4 + e] = OP::value(hi[e]); }
                finish.template store<OUT>(a, mine, column, sum, wide);
            }
        }
        wave_sync();
    }
}

// ---- tiles ----
// What one launch does: up to two products, a run of workgroups each, and the sums of columns.
template <class ARGS>
struct ProductsOf {
    ARGS a[2];
    int32_t tiles_r[2], tiles_c[2];
    int32_t first[3];                   // tiles (times splits) from first[i] on: product 0, product 1, none
    int32_t sum_blocks;                 // the last workgroups: sums
    ColumnSums sums;
};
typedef ProductsOf<ProductArgs> Products;

__device__ __forceinline__ void column_sums(const ColumnSums &c, int32_t block, float *room)        // 64 columns per workgroup
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int64_t at = (int64_t)block * 64 + lane, per = (c.parts + waves - 1) / waves;
    float sum = 0.0f;
    if (at < c.n)
        for (int64_t k = wave * per; k < min(c.parts, (wave + 1) * per); ++k) sum += c.sums[k * c.n + at];
    room[wave * 64 + lane] = sum;
    __syncthreads();
    if (wave || at >= c.n) return;
    sum = 0.0f;
    for (int k = 0; k < waves; ++k) sum += room[k * 64 + lane];
    put_param(c.out, c.dtype, at, sum);
}

// Workgroups go to the eight XCDs in turn; each XCD gets a run of consecutive tiles, and a run goes down eight columns of tiles side by side,
// so that what an XCD's L2 holds is used again.
__device__ __forceinline__ void tile_of(int32_t block, int32_t tiles_r, int32_t tiles_c, int32_t &split, int32_t &tr, int32_t &tc)
{
    const int32_t tiles = tiles_r * tiles_c;
    int32_t at = block % tiles;
    split = block / tiles;
    const int32_t xcd = at & 7, whole = tiles >> 3, more = tiles & 7;
    at = xcd * whole + min(xcd, more) + (at >> 3);
    const int32_t band = at / (8 * tiles_r), in_band = at - band * 8 * tiles_r, width = min(8, tiles_c - band * 8);
    tr = in_band / width;
    tc = band * 8 + in_band % width;
}

// The loads of a tile.  A load brings 8 rows of 128 bytes to LDS, lane l the sixteen bytes that belong at place l % 8 of row l / 8.  Place j of row i
// holds the bytes 16 (j ^ i % 8) ..: eight rows of one k then lie in all banks.  Rows behind the end are the last row again; nobody
// stores what comes of them.
// ORDER 1: rows of p go to the places that suit the reads of the tiles of 256 x 256 (both types'), j ^ (i % 4 + 4 (i / 8 % 2)).  LDS serves sixteen-byte reads sixteen lanes at a time, from 64
// banks: lanes 0-3, 12-15, 20-23 and 24-27, then 4-7, 8-11, 16-19 and 28-31.  Where the first 32 lanes read 32 rows (the blocks of 32 x 32 of product_f8_kernel, ORDER 2), places
// j ^ (i / 2 % 8) have all of them apart, and j ^ i % 8 half.
template <int TR, int TC, int WAVES, int ORDER>
struct TileLoads {
    static constexpr int LP = TR / 8 / WAVES, LQ = TC / 8 / WAVES;      // per wave and step
    uint32_t off_p[LP], off_q[LQ];
    const char *p, *q;
    int32_t p_left;                     // steps until p starts again
    __device__ __forceinline__ void init(const ProductArgs &a, int32_t r0, int32_t c0, int32_t first, int wave)
    {
        static_assert(WAVES % 4 == 0, "rows 8 (i WAVES + wave) .. + 7: bits 3 and 4 are those of the wave");
        const int lane = threadIdx.x & 63, row = lane >> 3, key = ORDER < 2 ? row : (row >> 1) | (wave & 1) << 2;
        const int key_p = ORDER == 1 ? (row & 3) | (wave & 1) << 2 : key;
        const int col = ((lane & 7) ^ key) * 16, col_p = ((lane & 7) ^ key_p) * 16;
#pragma unroll
        for (int i = 0; i < LP; ++i) off_p[i] = (uint32_t)min(a.R - 1 - r0, (i * WAVES + wave) * 8 + row) * (uint32_t)a.ld_p + col_p;
#pragma unroll
        for (int i = 0; i < LQ; ++i) off_q[i] = (uint32_t)min(a.C - 1 - c0, (i * WAVES + wave) * 8 + row) * (uint32_t)a.ld_q + col;
        const int32_t at = a.p_steps ? first % a.p_steps : 0;
        p = a.p + (int64_t)r0 * a.ld_p + (int64_t)at * 128;
        q = a.q + (int64_t)c0 * a.ld_q + (int64_t)first * 128;
        p_left = a.p_steps - at;
    }
    // the next step, to `to`: [TR + TC][128]
    __device__ __forceinline__ void request(const ProductArgs &a, char *to, int wave)
    {
#pragma unroll
        for (int i = 0; i < LP; ++i)
            __builtin_amdgcn_global_load_lds((global_void *)(p + off_p[i]), (lds_void *)(to + (i * WAVES + wave) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < LQ; ++i)
            __builtin_amdgcn_global_load_lds((global_void *)(q + off_q[i]), (lds_void *)(to + TR * 128 + (i * WAVES + wave) * 1024), 16, 0, 0);
        next(a);
    }
    // one of its LP + LQ loads; next() when all have been asked for
    __device__ __forceinline__ void request_one(const ProductArgs &a, char *to, int wave, int i)
    {
        if (i < LP) __builtin_amdgcn_global_load_lds((global_void *)(p + off_p[i % LP]), (lds_void *)(to + (i * WAVES + wave) * 1024), 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((global_void *)(q + off_q[(i - LP) % LQ]), (lds_void *)(to + TR * 128 + ((i - LP) * WAVES + wave) * 1024), 16, 0, 0);
    }
    __device__ __forceinline__ void next(const ProductArgs &a)
    {
        q += 128;
        p += 128;
        if (--p_left == 0) {
            p_left = a.p_steps;
            p -= (int64_t)a.p_steps * 128;
        }
    }
};

__device__ __forceinline__ i32x4 i32x4_of(const float *v) { return __builtin_bit_cast(i32x4, (f32x4{v[0], v[1], v[2], v[3]})); }

// Lanes 16 g + n hold, of column `column` (n on from a multiple of 16), sixteen bytes `lo` at row `row` and sixteen `hi` STEP rows behind, the four g making
// up 64 bytes, or every other sixteen of 128.  Columns n and n + 8 exchange a half, so that each store brings eight lanes' 128 bytes of a column: whole
// lines, which stores past the caches need.  Through the caches the outputs (25 MB at least, where tiles of this size are taken) would drive out what
// they hold of the operands: 8192 x 4096 x 16384 int8 to bf16, all values alike: 435 us through the caches, 400 past them in parts, 374 in lines;
// with random values 494 and 465.
template <int STEP, typename T>
__device__ __forceinline__ void put_lines(T *out, int32_t row, int32_t column, int64_t ld, i32x4 lo, i32x4 hi)
{
    const bool first = (threadIdx.x & 8) == 0;
    i32x4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = __builtin_amdgcn_update_dpp(lo[e], hi[e], 0x128, 0xf, 0xc, false);       // row_ror:8, to columns n + 8
        b[e] = __builtin_amdgcn_update_dpp(hi[e], lo[e], 0x128, 0xf, 0x3, false);       // to columns n
    }
    i32x4 *const to = (i32x4 *)(out + (int64_t)(first ? column : column - 8) * ld + row + (first ? 0 : STEP)), *const next = (i32x4 *)((T *)to + 8 * ld);
    __builtin_nontemporal_store(a, to);
    __builtin_nontemporal_store(b, next);
}

// Adds up the splits in their order, four outputs per thread (one where rows of the sums do not start on 16-byte boundaries), the loads of
// four splits under way.  32 x 25088 from two splits: 5 us.
struct Joins {
    ProductArgs a[2];
    uint32_t first1;                    // workgroups from here on: product 1
};

template <class OP, int OUT, int VEC>
__device__ __forceinline__ void join_part(const ProductArgs &a, int64_t at)
{
    typedef typename OP::sum N;
    typedef N NV __attribute__((ext_vector_type(VEC)));
    const int32_t pieces = a.R / VEC;
    if (at >= (int64_t)pieces * a.C) return;
    const int32_t c = (int32_t)(at / pieces), r = (int32_t)(at % pieces) * VEC;
    const NV *part = (const NV *)((const N *)a.parts + (int64_t)c * a.R + r);
    const int64_t step = (int64_t)a.C * a.R / VEC;
    NV sum = {};
    int32_t k = 0;
    for (; k + 4 <= a.splits; k += 4) {
        NV v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = part[(k + i) * step];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += v[i];
    }
    for (; k < a.splits; ++k) sum += part[k * step];
    typename Elem<OUT>::type *out = (typename Elem<OUT>::type *)a.out + (int64_t)c * a.ld_out + r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        float v = OP::value(sum[i]);
        if (Scaled<OP>::value) {
            v *= a.q_scale[c] * a.p_scale[r + i];
            if (a.bias) v += param(a.bias, a.bias_dtype, r + i);
        } else if (Biased<OP>::value && a.bias) {
            v += param(a.bias, a.bias_dtype, r + i);
        }
        out[i] = Elem<OUT>::from_float(v);
    }
}

template <class OP, int OUT>
__global__ __launch_bounds__(256) void product_join_kernel(Joins all)
{
    const int which = blockIdx.x >= all.first1;
    const ProductArgs &a = all.a[which];
    const int64_t at = (int64_t)(blockIdx.x - (which ? all.first1 : 0)) * 256 + threadIdx.x;
    if (a.R % 4 == 0) join_part<OP, OUT, 4>(a, at);
    else join_part<OP, OUT, 1>(a, at);
}

template <class OP, int OUT>
static hipError_t join_as(const ProductArgs *const *a, int n, hipStream_t s)
{
    Joins all{};
    uint32_t blocks = 0;
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (a[i]->splits <= 1) continue;
        all.a[m] = *a[i];
        if (m == 1) all.first1 = blocks;
        blocks += (uint32_t)(((int64_t)(a[i]->R % 4 ? a[i]->R : a[i]->R / 4) * a[i]->C + 255) / 256);
        ++m;
    }
    if (m == 0) return hipSuccess;
    if (m == 1) all.first1 = UINT32_MAX;
    hipLaunchKernelGGL((product_join_kernel<OP, OUT>), dim3(blocks), dim3(256), 0, s, all);
    return hipGetLastError();
}

}  // namespace tictac
