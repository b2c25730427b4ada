// See k8_product.h.  A workgroup has a tile of the output, its waves a part of that each; the operands come through LDS in steps of 128
// bytes of k, several buffers in turn: while one is computed from, the next steps are under way into the others, straight from memory to LDS.
#include <algorithm>

#include "device_utils.h"
#include "k8_product.h"

namespace tictac {

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

struct OpI8 {
    typedef i32x4 acc;
    typedef uint32_t sum;               // (adding up wraps, defined)
    static __device__ __forceinline__ float value(int32_t s) { return (float)s; }
    static __device__ __forceinline__ acc mma(i32x4 a, i32x4 b, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ void mma_in_place(i32x4 a, i32x4 b, acc &c) { asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
struct OpI8Widest : OpI8 {              // of kWidest columns
    static __device__ __forceinline__ float value(int32_t s) { return exact_sum(s); }
};
struct OpBf16 {
    typedef f32x4 acc;
    typedef float sum;
    static __device__ __forceinline__ float value(float s) { return s; }
    static __device__ __forceinline__ acc mma(i32x4 a, i32x4 b, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void mma_in_place(i32x4 a, i32x4 b, acc &c) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
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
template <>
struct Scaled<OpI8Widest> { static constexpr bool value = true; };

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
                for (int e = 0; e < 4; ++e) { sum[e] = OP::value(lo[e]); sum[4 + e] = OP::value(hi[e]); }
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
    int32_t first[3];                   // tiles (times splits) from first[i] on: product 0, product 1, none
    int32_t sum_blocks;                 // the last workgroups: sums
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
// PAIRED: rows of p go to the places that suit the reads of product_kernel_256, j ^ (i % 4 + 4 (i / 8 % 2)).
template <int TR, int TC, int WAVES, bool PAIRED>
struct TileLoads {
    static constexpr int LP = TR / 8 / WAVES, LQ = TC / 8 / WAVES;      // per wave and step
    uint32_t off_p[LP], off_q[LQ];
    const char *p, *q;
    int32_t p_left;                     // steps until p starts again
    __device__ __forceinline__ void init(const ProductArgs &a, int32_t r0, int32_t c0, int32_t first, int wave)
    {
        static_assert(WAVES % 2 == 0, "rows 8 (i WAVES + wave) .. + 7: bit 3 is that of the wave");
        const int lane = threadIdx.x & 63, row = lane >> 3, col = ((lane & 7) ^ row) * 16;
        const int col_p = PAIRED ? ((lane & 7) ^ ((row & 3) | (wave & 1) << 2)) * 16 : col;
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

// A tile of 32 FR x 32 FC outputs by four waves, STAGES buffers in turn, two workgroups per compute unit where they fit (kTiles).  A step has two halves; under the
// matrix instructions of each the operands of the next are read:
//   - half 0 of step t reads the rest of step t; then a barrier, before which each wave has waited for its reads and for its loads of step t + 1;
//   - half 1 of step t reads the first half of step t + 1 and asks for step t + STAGES, into the buffer of step t.
template <class OP, int OUT, int FR, int FC, int STAGES>
__global__ __launch_bounds__(256, STAGES * (FR + FC) > 20 ? 1 : 2) void product_kernel(Products all)
{
    constexpr int TR = FR * 32, TC = FC * 32, kBuffer = (TR + TC) * 128, kMma = FR * FC, kReads = FR + FC;
    extern __shared__ char lds[];                                       // [STAGES][TR + TC][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int32_t)blockIdx.x >= all.first[2]) {                          // (a workgroup per tile)
        column_sums(all.sums, blockIdx.x - all.first[2], (float *)lds);
        return;
    }
    const int which = (int32_t)blockIdx.x >= all.first[1];
    const ProductArgs &a = all.a[which];
    int32_t split, tr, tc;
    tile_of(blockIdx.x - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
    const int32_t r0 = tr * TR, c0 = tc * TC;
    const int32_t first = (int32_t)((int64_t)a.steps * split / a.splits), last = (int32_t)((int64_t)a.steps * (split + 1) / a.splits);
    typedef TileLoads<TR, TC, 4, false> Loads;
    constexpr int kLoads = Loads::LP + Loads::LQ;
    Loads loads;
    loads.init(a, r0, c0, first, wave);
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 15, fk = lane >> 4, swizzle = frow & 7;
    const char *const tp = lds + (wr * FR * 16 + frow) * 128, *const tq = lds + TR * 128 + (wc * FC * 16 + frow) * 128;
    typename OP::acc acc[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = typename OP::acc{};
    i32x4 fp[2][FR], fq[2][FC];
    const auto read_one = [&](int half, int n, int place) {
        if (n < FC) fq[half][n] = *(const i32x4 *)(tq + n * 2048 + place);
        else fp[half][n - FC] = *(const i32x4 *)(tp + (n - FC) * 2048 + place);
    };
    // the wait for a step's loads, with `later` steps' behind them under way
    const auto arrived = [&](int32_t later) {
        if (STAGES > 3 && later >= 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kLoads) : "memory");
        else if (STAGES > 2 && later == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");                                  // (nothing is read before the barrier)
    };
    const auto run = [&](int half, int place, bool read, bool ask, char *to) {
#pragma unroll
        for (int m = 0; m < kMma; ++m) {
            if (read)
#pragma unroll
                for (int n = m * kReads / kMma; n < (m + 1) * kReads / kMma; ++n) read_one(half ^ 1, n, place);
            if (ask)
#pragma unroll
                for (int n = m * kLoads / kMma; n < (m + 1) * kLoads / kMma; ++n) loads.request_one(a, to, wave, n);
            acc[m / FC][m % FC] = OP::mma(fp[half][m / FC], fq[half][m % FC], acc[m / FC][m % FC]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (ask) loads.next(a);
    };
    if (first < last) {
        for (int32_t step = first; step < last && step < first + STAGES; ++step) loads.request(a, lds + (step - first) * kBuffer, wave);
        const int32_t later = min(last - 1 - first, STAGES - 1);
        if (STAGES > 3 && later >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * kLoads) : "memory");
        else if (STAGES > 2 && later >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
        else if (later >= 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < kReads; ++n) read_one(0, n, (fk ^ swizzle) * 16);
    }
    int buffer = 0;
    for (int32_t step = first; step < last; ++step) {
        const int next = buffer + 1 < STAGES ? buffer + 1 : 0;
        run(0, buffer * kBuffer + ((4 + fk) ^ swizzle) * 16, true, false, nullptr);
        arrived(min(last - 2 - step, STAGES - 2));
        const int place = next * kBuffer + (fk ^ swizzle) * 16;
        if (step + STAGES < last) run(1, place, true, true, lds + buffer * kBuffer);
        else run(1, place, step + 1 < last, false, nullptr);
        buffer = next;
    }
    __syncthreads();
    char *room = lds + wave * 16 * (FR * 16 + 4) * 4;
    if (a.splits > 1) put_blocks<OP, kParts, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
    else put_blocks<OP, OUT, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
}

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
        const int32_t mine = first ? hi[e] : lo[e], other = __builtin_amdgcn_update_dpp(0, mine, 0x128, 0xf, 0xf, true);     // row_ror:8
        a[e] = first ? lo[e] : other;
        b[e] = first ? other : hi[e];
    }
    i32x4 *const to = (i32x4 *)(out + (int64_t)(first ? column : column - 8) * ld + row + (first ? 0 : STEP)), *const next = (i32x4 *)((T *)to + 8 * ld);
    __builtin_nontemporal_store(a, to);
    __builtin_nontemporal_store(b, next);
}

// Tiles of 256 x 256 outputs by four waves, one per SIMD, of 128 x 128 each.  A step of 128 bytes has two halves of 64 matrix instructions; under
// each half the operands of the next are read:
//   - half 0 of step t reads the rest of step t; then a barrier, before which each wave has waited for its reads and for its loads of step t + 1:
//     all of step t + 1 is there, and nobody reads the buffer of step t any more;
//   - half 1 of step t reads the first half of step t + 1 and asks for step t + 2, into the buffer of step t.
// The accumulators fill the 256 accumulation registers, hence the matrix instructions in assembly.  One workgroup per compute unit goes from tile to tile:
// behind the last barrier of a tile LDS is free, and the first two steps of the next tile are asked for before this one's outputs are formed.
// Two blocks of 16 rows share 32 rows of p in turns of four (row 4 n + e of block 2 m + h is row 32 m + 8 n + 4 h + e of the tile), so that a lane has
// eight outputs next to each other and stores sixteen bytes of bf16 straight from its registers.
// 8192 x 4096 x 16384 int8: a step takes 1.45 us of a workgroup (2.9 POP/s while it lasts), 464 to 499 us in all, by the clock that the
// power limit leaves (2.04 to 1.98 GHz).
template <class OP, int OUT>
__global__ __launch_bounds__(256, 1) void product_kernel_256(Products all)
{
    constexpr int TR = 256, TC = 256, FR = 8, FC = 8, kBuffer = (TR + TC) * 128;
    extern __shared__ char lds[];                                       // [2][TR + TC][128], scales of rows, bias, scales of columns
    float *const scales = (float *)(lds + 2 * kBuffer);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t workers = gridDim.x - all.sum_blocks;
    if ((int32_t)blockIdx.x >= workers) {
        column_sums(all.sums, blockIdx.x - workers, (float *)lds);
        return;
    }
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 15, fk = lane >> 4, swizzle = frow & 7;
    const char *const tp = lds + (wr * FR * 16 + (frow >> 2) * 8 + (frow & 3)) * 128, *const tq = lds + TR * 128 + (wc * FC * 16 + frow) * 128;
    constexpr bool kScaled = Scaled<OP>::value;
    TileLoads<TR, TC, 4, true> loads;
    typename OP::acc acc[FR][FC];
    i32x4 fp[2][FR], fq[2][FC];
    int32_t r0, c0, which;
    const auto begin = [&](int32_t tile) {
        which = tile >= all.first[1];
        const ProductArgs &a = all.a[which];
        int32_t split, tr, tc;
        tile_of(tile - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
        r0 = tr * TR;
        c0 = tc * TC;
        loads.init(a, r0, c0, 0, wave);
        if (a.steps) loads.request(a, lds, wave);
        if (a.steps > 1) loads.request(a, lds + kBuffer, wave);
    };
    const auto read_one = [&](int half, int n, int place) {
        if (n < FC) fq[half][n] = *(const i32x4 *)(tq + n * 2048 + place);
        else fp[half][n - FC] = *(const i32x4 *)(tp + ((n - FC) >> 1) * 4096 + ((n - FC) & 1) * 512 + place);
    };
    // One half of a step: its 64 matrix instructions, after every fourth a read of the operands of the next half and a load of a later step
    const auto run = [&](const ProductArgs &a, int half, int32_t step, bool read, bool ask) {
        const int buffer = (step + half) & 1;                           // (half 1 reads the next step)
        const int place = buffer * kBuffer + (((half ^ 1) * 4 + fk) ^ swizzle) * 16;
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            if (read) read_one(half ^ 1, n, place);
            if (ask) loads.request_one(a, lds + (step & 1) * kBuffer, wave, n);
            const int i = n >> 1, j0 = (n & 1) * 4;
#pragma unroll
            for (int j = j0; j < j0 + 4; ++j) OP::mma_in_place(fp[half][i], fq[half][j], acc[i][j]);
        }
        if (ask) loads.next(a);
    };
    const auto barrier = [] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");                                  // (nothing is read before the barrier)
    };
    int32_t tile = blockIdx.x, after = 0;                               // after: stores that surely were issued behind the loads under way
    begin(tile);
    while (true) {
        const ProductArgs &a = all.a[which];
        const int32_t steps = a.steps, row0 = r0, col0 = c0, t = threadIdx.x;
        float row_scale = 0.0f, row_bias = 0.0f, col_scale = 0.0f;
        if (kScaled) {
            if (row0 + t < a.R) row_scale = a.p_scale[row0 + t];
            if (a.bias && row0 + t < a.R) row_bias = param(a.bias, a.bias_dtype, row0 + t);
            if (col0 + t < a.C) col_scale = a.q_scale[col0 + t];
        }
#pragma unroll
        for (int i = 0; i < FR; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j) acc[i][j] = typename OP::acc{};
        // (of what was issued behind the loads, the stores of the tile before may go on)
        if (after >= 32) asm volatile("s_waitcnt vmcnt(32)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        barrier();
        if (steps) {
#pragma unroll
            for (int n = 0; n < 16; ++n) read_one(0, n, (fk ^ swizzle) * 16);
        }
        const auto meet = [&] {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            barrier();
        };
        int32_t step = 0;
        for (; step + 2 < steps; ++step) {
            run(a, 0, step, true, false);
            meet();
            run(a, 1, step, true, true);
        }
        for (; step < steps; ++step) {
            run(a, 0, step, true, false);
            meet();
            run(a, 1, step, step + 1 < steps, false);
        }
        if (kScaled) {
            scales[t] = row_scale;
            scales[256 + t] = row_bias;
            scales[512 + t] = col_scale;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            barrier();
        }
        tile += workers;
        const bool more = tile < all.first[2];
        if (more) begin(tile);
        // the compiler does not know that matrix instructions wrote these, and their results take a while
#pragma unroll
        for (int i = 0; i < FR; ++i)
            asm volatile("s_nop 15" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]), "+a"(acc[i][3]), "+a"(acc[i][4]), "+a"(acc[i][5]), "+a"(acc[i][6]), "+a"(acc[i][7]));
        typedef typename Elem<OUT>::type T;
        const bool wide = (a.ld_out * sizeof(T)) % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.R % 8 == 0;
        const bool whole = wide && row0 + TR <= a.R && col0 + TC <= a.C;
        const int32_t r = wr * FR * 16 + fk * 8, c = wc * FC * 16 + frow;
        T *const out = (T *)a.out;
        i32x4 held[FC];                                                 // 16-bit outputs of the block before
#pragma unroll
        for (int i = 0; i < FR / 2; ++i) {
            float s[8], b[8];
            if (kScaled)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 u = *(const f32x4 *)(scales + r + i * 32 + h * 4), v = *(const f32x4 *)(scales + 256 + r + i * 32 + h * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { s[h * 4 + e] = u[e]; b[h * 4 + e] = v[e]; }
                }
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                const float qs = kScaled ? scales[512 + c + j * 16] : 0.0f;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = OP::value(acc[2 * i + (e >> 2)][j][e & 3]);
                    if (kScaled) v[e] = v[e] * (qs * s[e]) + b[e];
                }
                const int32_t row = row0 + r + i * 32, column = col0 + c + j * 16;
                if (!whole) {
                    if (column >= a.C) continue;
                    if (wide) store8<OUT, true>(out + (int64_t)column * a.ld_out, row, a.R, v);
                    else store8<OUT, false>(out + (int64_t)column * a.ld_out, row, a.R, v);
                } else if constexpr (OUT == TICTAC_F32) {
                    put_lines<4>(out, row, column, a.ld_out, i32x4_of(v), i32x4_of(v + 4));
                } else {
                    const auto packed = Elem<OUT>::pack(v);
                    if (i & 1) put_lines<32>(out, row - 32, column, a.ld_out, held[j], __builtin_bit_cast(i32x4, packed));
                    else held[j] = __builtin_bit_cast(i32x4, packed);
                }
            }
        }
        if (!more) return;
        after = whole ? 32 : 0;
        if (kScaled) barrier();                                         // (the scales are read before the next tile's are written)
    }
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

// The tiles by rows x columns of 32, and what a workgroup takes, in us: `fixed`, and per step with one workgroup per compute unit and (both of them
// together) with two.  Measured with int8 on 256, 512 and 1024 workgroups of 2 to 64 steps: 128 x 128 on 256 workgroups 8.7 us for two steps and 39.5 for 64,
// 128 x 64 6.8 and 26.6, 64 x 64 5.6 and 21.6; on 512 11.1 and 63.6, 8.7 and 43.1, 6.2 and 29.2.  Full, all of them come to what the L2 gives LDS (18 to
// 21 TB/s).
struct Tile { int32_t r, c; float fixed, step, step2; };
constexpr Tile kTiles[] = {{4, 4, 7.6f, 0.5f, 0.85f}, {4, 2, 6.0f, 0.33f, 0.56f}, {2, 2, 5.1f, 0.26f, 0.37f}};
constexpr int32_t kTile256 = 3;

ProductPlan plan_products(const ProductShape *shapes, int n)
{
    ProductPlan best{0, {1, 1}};
    float least = 1e30f;
    const auto take = [&](int32_t tile, const int32_t (&splits)[2], float us) {
        if (us >= least) return;
        least = us;
        best.tile = tile;
        best.splits[0] = splits[0];
        best.splits[1] = splits[1];
    };
    for (int32_t tile = 0; tile < kTile256; ++tile) {
        const Tile &t = kTiles[tile];
        int64_t tiles[2] = {0, 0};
        for (int i = 0; i < n; ++i) tiles[i] = (int64_t)((shapes[i].R + 32 * t.r - 1) / (32 * t.r)) * ((shapes[i].C + 32 * t.c - 1) / (32 * t.c));
        for (int32_t most = 1 << 30; most >= 2; most = most > 64 ? 64 : most / 2) {         // steps of a workgroup
            int32_t splits[2] = {1, 1};
            int64_t blocks = 0;
            float steps = 0.0f, all_steps = 0.0f, us = 0.0f;
            for (int i = 0; i < n; ++i) {
                splits[i] = std::min(16, std::max(1, (shapes[i].steps + most - 1) / most));
                blocks += tiles[i] * splits[i];
                steps = std::max(steps, (float)shapes[i].steps / (float)splits[i]);
                all_steps += (float)tiles[i] * (float)shapes[i].steps;
                if (splits[i] > 1) us += 1.0f + (float)splits[i] * (float)shapes[i].R * (float)shapes[i].C * (8.0f / 4.5e6f);       // written and read again
            }
            for (int i = 0; i < n; ++i)
                if (splits[i] > 1) { us += 2.0f; break; }                                   // the launch that adds them up
            const float per_cu = (float)((blocks + 255) / 256);
            if (per_cu <= 1.0f) {
                us += t.fixed + t.step * steps;
            } else {                                            // the longest of them begin at once where they are the first product's, and else may come last
                const float mean = std::min(all_steps / (float)blocks, steps), work = t.step2 * 0.5f * mean * per_cu, one = t.step2 * steps;
                us += t.fixed * (0.5f + 0.35f * per_cu) + (shapes[0].steps * splits[n - 1] >= shapes[n - 1].steps * splits[0] ? std::max(work, one) : work + t.step2 * (steps - mean));
            }
            take(tile, splits, us);
        }
    }
    // tiles of 256 x 256, one workgroup per compute unit from tile to tile, those of the first product first: 1.45 us a step with all compute units busy, 1.0 with
    // half of them, 6 us for a first tile besides and 11 for each behind it; the longest of the workgroups that begin with the second product's tiles one turn earlier or later
    float each[2] = {0.0f, 0.0f};
    int64_t tiles[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
        tiles[i] = (int64_t)((shapes[i].R + 255) / 256) * ((shapes[i].C + 255) / 256);
    }
    const float step = std::min(1.45f, std::max(1.0f, (float)(tiles[0] + tiles[1]) * (1.45f / 256.0f)));
    for (int i = 0; i < n; ++i) each[i] = 6.0f + step * (float)shapes[i].steps;
    const int64_t turns = (tiles[0] + tiles[1] + 255) / 256, early = tiles[0] / 256, late = (tiles[0] + 255) / 256;
    const float us = 4.0f + 5.0f * (float)(turns - 1) + std::max((float)early * each[0] + (float)(turns - early) * each[1], (float)late * each[0] + (float)(turns - late) * each[1]);
    take(kTile256, {1, 1}, us);
    return best;
}

template <class OP, int OUT>
static hipError_t launch_as(const ProductArgs *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    Products all{};
    const bool large = tile == kTile256;
    const int32_t tr = large ? 256 : 32 * kTiles[tile].r, tc = large ? 256 : 32 * kTiles[tile].c;
    int32_t blocks = 0;
    for (int i = 0; i < 2; ++i) {
        all.first[i] = blocks;
        if (i >= n) continue;
        all.a[i] = a[i];
        all.tiles_r[i] = (a[i].R + tr - 1) / tr;
        all.tiles_c[i] = (a[i].C + tc - 1) / tc;
        blocks += all.tiles_r[i] * all.tiles_c[i] * a[i].splits;
    }
    all.first[2] = blocks;
    all.sums = c;
    all.sum_blocks = c.out ? (int32_t)((c.n + 63) / 64) : 0;
    if (n == 1) all.first[1] = all.first[2];
    if (blocks + all.sum_blocks == 0) return hipSuccess;
    if (large) {
        int device = 0;
        if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
        blocks = std::min(blocks, (int32_t)device_cu_count(device));
    }
    blocks += all.sum_blocks;
    // LDS: the buffers of a step's operands; for the outputs they are enough too.  Four buffers of the largest tile leave room for one workgroup only.
    const bool alone = blocks <= 256;
    const auto kernel = large       ? product_kernel_256<OP, OUT>
                        : tile == 0 ? (alone ? product_kernel<OP, OUT, 4, 4, 4> : product_kernel<OP, OUT, 4, 4, 2>)
                        : tile == 1 ? product_kernel<OP, OUT, 4, 2, 3>
                                    : product_kernel<OP, OUT, 2, 2, 4>;
    const int lds = large ? 2 * 512 * 128 + 768 * 4 : (tile == 0 ? (alone ? 4 : 2) : tile == 1 ? 3 : 4) * (tr + tc) * 128;
    if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), lds, s, all);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return join_as<OP, OUT>(a, n, s);
}

template <class OP>
static hipError_t launch(const ProductArgs *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    const int32_t dt = n ? a[0].dtype : c.dtype;
    if (dt == TICTAC_F32) return launch_as<OP, TICTAC_F32>(a, n, tile, c, s);
    return dt == TICTAC_F16 ? launch_as<OP, TICTAC_F16>(a, n, tile, c, s) : launch_as<OP, TICTAC_BF16>(a, n, tile, c, s);
}

template <class OP>
static hipError_t join(const ProductArgs &a, hipStream_t s)
{
    if (a.dtype == TICTAC_F32) return join_as<OP, TICTAC_F32>(&a, 1, s);
    return a.dtype == TICTAC_F16 ? join_as<OP, TICTAC_F16>(&a, 1, s) : join_as<OP, TICTAC_BF16>(&a, 1, s);
}

hipError_t launch_product_join_i8(const ProductArgs &a, hipStream_t s) { return join<OpI8Widest>(a, s); }
hipError_t launch_product_join_bf16(const ProductArgs &a, hipStream_t s) { return join<OpBf16>(a, s); }
hipError_t launch_product_i8(const ProductArgs &a, int32_t tile, hipStream_t s)
{
    return a.steps < kWidest / 128 ? launch<OpI8>(&a, 1, tile, ColumnSums{}, s) : launch<OpI8Widest>(&a, 1, tile, ColumnSums{}, s);
}
hipError_t launch_products_bf16(const ProductArgs *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s) { return launch<OpBf16>(a, n, tile, c, s); }

}  // namespace tictac
