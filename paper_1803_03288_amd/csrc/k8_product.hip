// See k8_product.h.  A workgroup has a tile of the output, its waves a part of that each; the operands come through LDS in steps of 128
// bytes of k, two buffers in turn: while one is computed from, the next step is under way into the other, straight from memory to LDS.
#include "device_utils.h"
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

// ---- outputs ----
// Eight outputs r .. r + 7 of a column from their sums.  The scales and the bias of r are the same for all columns of a thread.
template <bool SCALED>
struct Finish8 {
    float scale[8], bias[8];
    __device__ __forceinline__ void init(const ProductArgs &a, int32_t r)
    {
        if (!SCALED) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            scale[i] = r + i < a.R ? a.p_scale[r + i] : 0.0f;
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
            for (int i = 0; i < 8; ++i) v[i] = sum[i];
        }
        typename Elem<DT>::type *row = (typename Elem<DT>::type *)a.out + (int64_t)c * a.ld_out;
        if (wide) store8<DT, true>(row, r, a.R, v);
        else store8<DT, false>(row, r, a.R, v);
    }
};
template <class OP>
struct Scaled { static constexpr bool value = false; };
template <>
struct Scaled<OpI8> { static constexpr bool value = true; };

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
    Finish8<Scaled<OP>::value && OUT != kParts> finish;
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
                for (int e = 0; e < 4; ++e) { sum[e] = (float)lo[e]; sum[4 + e] = (float)hi[e]; }
                finish.template store<OUT>(a, mine, column, sum, wide);
            }
        }
        wave_sync();
    }
}

// ---- tiles ----
// What one launch does: up to two products, a run of workgroups each, and the sums of columns.
struct Products {
    ProductArgs a[2];
    int32_t tiles_r[2], tiles_c[2];
    int32_t first[3];                   // workgroups from first[i] on: product 0, product 1, sums
    ColumnSums sums;
};

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
template <int TR, int TC, int WAVES>
struct TileLoads {
    static constexpr int LP = TR / 8 / WAVES, LQ = TC / 8 / WAVES;      // per wave and step
    uint32_t off_p[LP], off_q[LQ];
    const char *p, *q;
    int32_t p_left;                     // steps until p starts again
    __device__ __forceinline__ void init(const ProductArgs &a, int32_t r0, int32_t c0, int32_t first, int wave)
    {
        const int lane = threadIdx.x & 63, row = lane >> 3, col = ((lane & 7) ^ row) * 16;
#pragma unroll
        for (int i = 0; i < LP; ++i) off_p[i] = (uint32_t)min(a.R - 1 - r0, (i * WAVES + wave) * 8 + row) * (uint32_t)a.ld_p + col;
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
        q += 128;
        p += 128;
        if (--p_left == 0) {
            p_left = a.p_steps;
            p -= (int64_t)a.p_steps * 128;
        }
    }
};

// A tile of 32 FR x 32 FC outputs by four waves, several workgroups per compute unit.
template <class OP, int OUT, int FR, int FC>
__global__ __launch_bounds__(256) void product_kernel(Products all)
{
    constexpr int TR = FR * 32, TC = FC * 32;
    extern __shared__ char lds[];                                       // [2][TR + TC][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int32_t)blockIdx.x >= all.first[2]) {
        column_sums(all.sums, blockIdx.x - all.first[2], (float *)lds);
        return;
    }
    const int which = (int32_t)blockIdx.x >= all.first[1];
    const ProductArgs &a = all.a[which];
    int32_t split, tr, tc;
    tile_of(blockIdx.x - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
    const int32_t r0 = tr * TR, c0 = tc * TC;
    const int32_t first = (int32_t)((int64_t)a.steps * split / a.splits), last = (int32_t)((int64_t)a.steps * (split + 1) / a.splits);
    TileLoads<TR, TC, 4> loads;
    loads.init(a, r0, c0, first, wave);
    const int wr = wave & 1, wc = wave >> 1;
    typename OP::acc acc[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = typename OP::acc{};
    const int frow = lane & 15, fk = lane >> 4;
    if (first < last) loads.request(a, lds, wave);
    for (int32_t step = first; step < last; ++step) {
        const int buffer = (step - first) & 1;
        __syncthreads();                    // this step has come, and nobody reads the other buffer any more
        if (step + 1 < last) loads.request(a, lds + (buffer ^ 1) * (TR + TC) * 128, wave);
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
    __syncthreads();
    char *room = lds + wave * 16 * (FR * 16 + 4) * 4;
    if (a.splits > 1) put_blocks<OP, kParts, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
    else put_blocks<OP, OUT, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
}

// A tile of 256 x 256 outputs by eight waves, two per SIMD: while one of the two computes, the other reads its next operands from LDS.  The waves of the
// second half run one slot behind (a barrier ends a slot); a step has four slots of reading and four of sixteen matrix instructions each.
// Slots of step t, for the first half: 8t read, 8t + 1 compute, ...; for the second: 8t + 1 read, 8t + 2 compute, ...
//   - The other buffer is free from slot 8t on: the second half's last reads of step t - 1 are over at the barrier behind slot 8t - 1
//     (they are waited for before it).  So each wave asks for step t + 1 in its first reading slot of step t.
//   - Step t + 1 is read from slot 8t + 8 on: every wave has waited for its loads at the end of slot 8t + 7.
template <class OP, int OUT>
__global__ __launch_bounds__(512, 2) void product_kernel_256(Products all)
{
    constexpr int TR = 256, TC = 256, FR = 8, FC = 4;
    extern __shared__ char lds[];                                       // [2][TR + TC][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave >> 2;
    if ((int32_t)blockIdx.x >= all.first[2]) {
        column_sums(all.sums, blockIdx.x - all.first[2], (float *)lds);
        return;
    }
    const int which = (int32_t)blockIdx.x >= all.first[1];
    const ProductArgs &a = all.a[which];
    int32_t split, tr, tc;
    tile_of(blockIdx.x - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
    const int32_t r0 = tr * TR, c0 = tc * TC;
    TileLoads<TR, TC, 8> loads;
    loads.init(a, r0, c0, 0, wave);
    const int wr = wave & 1, wc = wave >> 1;
    typename OP::acc acc[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = typename OP::acc{};
    const int frow = lane & 15, fk = lane >> 4;
    if (a.steps) loads.request(a, lds, wave);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    if (half) __builtin_amdgcn_s_barrier();
    for (int32_t step = 0; step < a.steps; ++step) {
        char *const here = lds + (step & 1) * (TR + TC) * 128;
        const char *tp = here + (wr * FR * 16 + frow) * 128, *tq = here + TR * 128 + (wc * FC * 16 + frow) * 128;
        i32x4 fp[FR / 2], fq[FC];
#pragma unroll
        for (int slot = 0; slot < 4; ++slot) {
            const int k = slot >> 1, at = (slot & 1) * (FR / 2), place = ((k * 4 + fk) ^ (frow & 7)) * 16;
            if (at == 0) {
#pragma unroll
                for (int j = 0; j < FC; ++j) fq[j] = *(const i32x4 *)(tq + j * 2048 + place);
            }
#pragma unroll
            for (int i = 0; i < FR / 2; ++i) fp[i] = *(const i32x4 *)(tp + (at + i) * 2048 + place);
            if (slot == 0 && step + 1 < a.steps) loads.request(a, lds + ((step & 1) ^ 1) * (TR + TC) * 128, wave);
            if (slot == 3 && half) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < FR / 2; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j) acc[at + i][j] = OP::mma(fp[i], fq[j], acc[at + i][j]);
            __builtin_amdgcn_s_setprio(0);
            if (slot == 3 && !half) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (!half) __builtin_amdgcn_s_barrier();
    __syncthreads();
    put_blocks<OP, OUT, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, 0, lds + wave * 16 * (FR * 16 + 4) * 4);
}

// Adds up the splits in their order, four outputs per thread (one where rows of the sums do not start on 16-byte boundaries), the loads of
// four splits under way.
struct Joins {
    ProductArgs a[2];
    uint32_t first1;                    // workgroups from here on: product 1
};

template <class OP, int OUT, int VEC>
__device__ __forceinline__ void join_part(const ProductArgs &a, int64_t at)
{
    typedef typename std::remove_reference<decltype(typename OP::acc{}[0] + typename OP::acc{}[0])>::type N;
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
        float v = (float)sum[i];
        if (Scaled<OP>::value) {
            v *= a.q_scale[c] * a.p_scale[r + i];
            if (a.bias) v += param(a.bias, a.bias_dtype, r + i);
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
static hipError_t join_as(const ProductArgs *a, int n, hipStream_t s)
{
    Joins all{};
    uint32_t blocks = 0;
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (a[i].splits <= 1) continue;
        all.a[m] = a[i];
        if (m == 1) all.first1 = blocks;
        blocks += (uint32_t)(((int64_t)(a[i].R % 4 ? a[i].R : a[i].R / 4) * a[i].C + 255) / 256);
        ++m;
    }
    if (m == 0) return hipSuccess;
    if (m == 1) all.first1 = UINT32_MAX;
    hipLaunchKernelGGL((product_join_kernel<OP, OUT>), dim3(blocks), dim3(256), 0, s, all);
    return hipGetLastError();
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

template <class OP, int OUT>
static hipError_t launch_as(const ProductArgs *a, int n, const ColumnSums &c, hipStream_t s)
{
    Products all{};
    int64_t big = 0;
    bool whole = true;
    for (int i = 0; i < n; ++i) {
        big += (int64_t)((a[i].R + 255) / 256) * ((a[i].C + 255) / 256);
        whole &= a[i].splits <= 1;
    }
    whole &= big >= 192;
    const int32_t tile = whole ? 256 : kSmallTile;
    int32_t blocks = 0;
    for (int i = 0; i < 2; ++i) {
        all.first[i] = blocks;
        if (i >= n) continue;
        all.a[i] = a[i];
        all.tiles_r[i] = (a[i].R + tile - 1) / tile;
        all.tiles_c[i] = (a[i].C + tile - 1) / tile;
        blocks += all.tiles_r[i] * all.tiles_c[i] * a[i].splits;
    }
    all.first[2] = blocks;
    all.sums = c;
    if (c.out) blocks += (int32_t)((c.n + 63) / 64);
    if (n == 1) all.first[1] = all.first[2];
    if (blocks == 0) return hipSuccess;
    const auto kernel = whole ? product_kernel_256<OP, OUT> : product_kernel<OP, OUT, 4, 4>;
    const int lds = 2 * 2 * tile * 128;
    if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(whole ? 512 : 256), lds, s, all);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return join_as<OP, OUT>(a, n, s);
}

template <class OP>
static hipError_t launch(const ProductArgs *a, int n, const ColumnSums &c, hipStream_t s)
{
    const int32_t dt = n ? a[0].dtype : c.dtype;
    if (dt == TICTAC_F32) return launch_as<OP, TICTAC_F32>(a, n, c, s);
    return dt == TICTAC_F16 ? launch_as<OP, TICTAC_F16>(a, n, c, s) : launch_as<OP, TICTAC_BF16>(a, n, c, s);
}

template <class OP>
static hipError_t join(const ProductArgs &a, hipStream_t s)
{
    if (a.dtype == TICTAC_F32) return join_as<OP, TICTAC_F32>(&a, 1, s);
    return a.dtype == TICTAC_F16 ? join_as<OP, TICTAC_F16>(&a, 1, s) : join_as<OP, TICTAC_BF16>(&a, 1, s);
}

hipError_t launch_product_join_i8(const ProductArgs &a, hipStream_t s) { return join<OpI8>(a, s); }
hipError_t launch_product_join_bf16(const ProductArgs &a, hipStream_t s) { return join<OpBf16>(a, s); }
hipError_t launch_product_i8(const ProductArgs &a, hipStream_t s) { return launch<OpI8>(&a, 1, ColumnSums{}, s); }
hipError_t launch_products_bf16(const ProductArgs *a, int n, const ColumnSums &c, hipStream_t s) { return launch<OpBf16>(a, n, c, s); }

}  // namespace tictac
