// See k9_product.h.  A step of 128 bytes of k is two matrix instructions of 32 x 32 x 64 for each block of outputs, in tiles of 256 x 256 one of 16 x 16 x 128; they take the scales of their
// operands' rows too.  The instruction aligns eight neighbouring products to the largest and cuts the rest off at about 2^-13 of it (measured: 1.4e-5 of the result's norm for normal values, 5e-5
// where values are spread over many powers of two); outputs here have 16 bits, and their own rounding is off by 2^-9 or 2^-12 of the norm.  float32 outputs take bf16 instructions, whose sums
// are float32.
#include "k9_product.h"

#include <algorithm>

#include "k8_tiles.h"

namespace tictac {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int QF>                       // format of q
struct OpF8 {
    typedef f32x4 acc;
    typedef float sum;
    static __device__ __forceinline__ float value(float s) { return s; }
    // In assembly, so that the compiler neither moves accumulators nor multiplies ahead of a branch.  It does not know that this is a matrix instruction: one that reads a register right
    // behind a vector instruction that wrote it would be too early (hence the s_nop, which a matrix instruction under way hides), and results take a while (results_settled).
    static __device__ __forceinline__ void mma(i32x8 a, i32x8 b, f32x16 &c, int ea, int eb)
    {
        asm volatile("s_nop 1\n\tv_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] blgp:%5" : "+a"(c) : "v"(a), "v"(b), "v"(ea), "v"(eb), "n"(QF));
    }
};
template <int QF>
struct Biased<OpF8<QF>> { static constexpr bool value = true; };

// what the matrix instructions wrote can be read behind this
template <int BR, int BC>
__device__ __forceinline__ void results_settled(f32x16 (&acc)[BR][BC])
{
#pragma unroll
    for (int i = 0; i < BR; ++i)
#pragma unroll
        for (int j = 0; j < BC; ++j) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[i][j]));
}

typedef ProductsOf<ProductF8Args> ProductsF8;

// The loads of the scales of a step: the four bytes that hold it, of TR rows of p and TC of q, 64 rows a load.  A wave makes NS of them, the same number in every wave and at every
// step, so that loads can be counted; where there are less than that, the last rows come again, to a place that nobody reads.
template <int TR, int TC, int WAVES>
struct ScaleLoads {
    static constexpr int kRuns = (TR + TC) / 64, NS = (kRuns + WAVES - 1) / WAVES, kBytes = NS * WAVES * 256;
    const uint8_t *base[NS];
    uint32_t off[NS];
    __device__ __forceinline__ void init(const ProductF8Args &a, int32_t r0, int32_t c0, int wave)
    {
        const int lane = threadIdx.x & 63;
        const uint8_t *const p_e = a.p_e, *const q_e = a.q_e;
        const int64_t ld_pe = a.ld_pe, ld_qe = a.ld_qe;
        const int32_t p_shift = a.p_shift, q_shift = a.q_shift;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int run = min(i * WAVES + wave, kRuns - 1), row = run * 64 + lane;
            const bool is_p = run < TR / 64;
            const int32_t shift = is_p ? p_shift : q_shift, from = is_p ? r0 : c0, at = (is_p ? min(r0 + row, a.R - 1) : min(c0 + row - TR, a.C - 1)) >> shift, first = from >> shift;
            const int64_t ld = is_p ? ld_pe : ld_qe;
            base[i] = (is_p ? p_e : q_e) + (int64_t)first * ld;
            off[i] = (uint32_t)(at - first) * (uint32_t)ld;
        }
    }
    __device__ __forceinline__ void request(int32_t step, char *to, int wave)
    {
#pragma unroll
        for (int i = 0; i < NS; ++i) request_one(step, to, wave, i);
    }
    __device__ __forceinline__ void request_one(int32_t step, char *to, int wave, int i)
    {
        __builtin_amdgcn_global_load_lds((global_void *)(base[i] + (step & ~3) + off[i]), (lds_void *)(to + (i * WAVES + wave) * 256), 4, 0, 0);
    }
};

// What a wave holds, BR x BC blocks of 32 x 32 from (r, c) on, goes column by column through its own part of LDS, so that a thread has eight consecutive outputs.  Lane l of a block holds
// rows 8 n + 4 (l / 32) .. + 3, n = 0 .. 3, of column l % 32.
template <class OP, int OUT, int BR, int BC>
__device__ __forceinline__ void put_blocks32(const ProductArgs &a, const f32x16 (&acc)[BR][BC], int32_t r, int32_t c, int32_t split, char *room)
{
    constexpr int kStride = BR * 32 + 4, kThreads = BR * 4, kColumns = 64 / kThreads;       // words; threads per column; columns at a time
    const int lane = threadIdx.x & 63, part = lane % kThreads, first = lane / kThreads;
    f32x4 *const to = (f32x4 *)room + ((lane & 31) * kStride + (lane >> 5) * 4) / 4;
    const f32x4 *const from = (const f32x4 *)room + (first * kStride + part * 8) / 4;
    const int32_t mine = r + part * 8;
    Finish8<false, OUT != kParts> finish;
    finish.init(a, mine);
    const bool wide = OUT != kParts && (a.ld_out * (OUT == TICTAC_F32 ? 4 : 2)) % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.R % 8 == 0;
#pragma unroll
    for (int j = 0; j < BC; ++j) {
#pragma unroll
        for (int i = 0; i < BR; ++i)
#pragma unroll
            for (int n = 0; n < 4; ++n) to[i * 8 + n * 2] = f32x4{acc[i][j][4 * n], acc[i][j][4 * n + 1], acc[i][j][4 * n + 2], acc[i][j][4 * n + 3]};
        wave_sync();
#pragma unroll
        for (int k = 0; k < 32 / kColumns; ++k) {
            const f32x4 lo = from[k * kColumns * kStride / 4], hi = from[k * kColumns * kStride / 4 + 1];
            const int32_t column = c + j * 32 + k * kColumns + first;
            if (column >= a.C || mine >= a.R) continue;
            const float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if constexpr (OUT == kParts) {
                float *const out = (float *)a.parts + ((int64_t)split * a.C + column) * a.R;
                if (a.R % 8 == 0) store8<TICTAC_F32, true>(out, mine, a.R, sum);
                else store8<TICTAC_F32, false>(out, mine, a.R, sum);
            } else {
                finish.template store<OUT>(a, mine, column, sum, wide);
            }
        }
        wave_sync();
    }
}

// A tile of 64 BR x 64 BC outputs by four waves, STAGES buffers in turn, two workgroups per compute unit where they fit.  A step has two halves of 64 bytes of k, a matrix instruction for each
// block of 32 x 32; under those of each half the operands of the next are read:
//   - half 0 of step t reads the rest of step t; then a barrier, before which each wave has waited for its reads and for its loads of step t + 1;
//   - half 1 of step t reads the first half of step t + 1 and asks for step t + STAGES, into the buffer of step t.
// 1024 x 4096 -> 4096: 23.5 us, 1.46 PFLOP/s; bound by what the L2 gives LDS, and small ones by their start.
template <int QF, int OUT, int BR, int BC, int STAGES>
__global__ __launch_bounds__(256, STAGES * (BR + BC) > 10 ? 1 : 2) void product_f8_kernel(ProductsF8 all)
{
    using OP = OpF8<QF>;
    constexpr int TR = BR * 64, TC = BC * 64, kMma = BR * BC, kReads = BR + BC;
    typedef TileLoads<TR, TC, 4, 2> Loads;
    typedef ScaleLoads<TR, TC, 4> Scales;
    constexpr int kBuffer = (TR + TC) * 128 + Scales::kBytes, kOperands = Loads::LP + Loads::LQ, kLoads = kOperands + Scales::NS;
    extern __shared__ char lds[];                                       // [STAGES]{[TR + TC][128], scales}
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int32_t)blockIdx.x >= all.first[2]) {                          // (a workgroup per tile)
        column_sums(all.sums, blockIdx.x - all.first[2], (float *)lds);
        return;
    }
    const int which = (int32_t)blockIdx.x >= all.first[1];
    const ProductF8Args &a = all.a[which];
    int32_t split, tr, tc;
    tile_of(blockIdx.x - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
    const int32_t r0 = tr * TR, c0 = tc * TC;
    const int32_t first = (int32_t)((int64_t)a.steps * split / a.splits), last = (int32_t)((int64_t)a.steps * (split + 1) / a.splits);
    Loads loads;
    Scales scales;
    loads.init(a, r0, c0, first, wave);
    scales.init(a, r0, c0, wave);
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 31, fk = lane >> 5, swizzle = frow >> 1 & 7;
    const int row_p = wr * BR * 32 + frow, row_q = TR + wc * BC * 32 + frow;
    f32x16 acc[BR][BC];
#pragma unroll
    for (int i = 0; i < BR; ++i)
#pragma unroll
        for (int j = 0; j < BC; ++j) acc[i][j] = f32x16{};
    i32x8 fp[2][BR], fq[2][BC];
    int ep[2][BR], eq[2][BC];
    // operand n of a half: columns first
    const auto read_one = [&](int half, int n, int32_t step, int buffer) {
        const char *const from = lds + buffer * kBuffer;
        const int lo = ((half * 4 + fk * 2) ^ swizzle) * 16, hi = ((half * 4 + fk * 2 + 1) ^ swizzle) * 16, row = n < BC ? row_q + n * 32 : row_p + (n - BC) * 32;
        const i32x4 u = *(const i32x4 *)(from + row * 128 + lo), v = *(const i32x4 *)(from + row * 128 + hi);
        const i32x8 w{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
        const int e = *(const uint8_t *)(from + (TR + TC) * 128 + row * 4 + (step & 3));
        if (n < BC) { fq[half][n] = w; eq[half][n] = e; }
        else { fp[half][n - BC] = w; ep[half][n - BC] = e; }
    };
    const auto request = [&](int32_t step, char *to) {
        loads.request(a, to, wave);
        scales.request(step, to + (TR + TC) * 128, wave);
    };
    // the wait for a step's loads, with `later` steps' behind them under way
    const auto arrived = [&](int32_t later) {
        if (STAGES > 3 && later >= 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kLoads) : "memory");
        else if (STAGES > 2 && later >= 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");                                  // (nothing is read before the barrier)
    };
    const auto run = [&](int half, int32_t step, int buffer, bool ask, char *to) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < kMma; ++m) {
            OP::mma(fp[half][m / BC], fq[half][m % BC], acc[m / BC][m % BC], ep[half][m / BC], eq[half][m % BC]);
#pragma unroll
            for (int n = m * kReads / kMma; n < (m + 1) * kReads / kMma; ++n) read_one(half ^ 1, n, step, buffer);
            if (ask)
#pragma unroll
                for (int n = m * kOperands / kMma; n < (m + 1) * kOperands / kMma; ++n) loads.request_one(a, to, wave, n);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (first < last) {
        for (int32_t step = first; step < last && step < first + STAGES; ++step) request(step, lds + (step - first) * kBuffer);
        const int32_t later = min(last - 1 - first, STAGES - 1);
        if (STAGES > 3 && later >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * kLoads) : "memory");
        else if (STAGES > 2 && later >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
        else if (later >= 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < kReads; ++n) read_one(0, n, first, 0);
    }
    int buffer = 0;
    int32_t step = first;
    for (; step + STAGES < last; ++step) {
        const int next = buffer + 1 < STAGES ? buffer + 1 : 0;
        char *const to = lds + buffer * kBuffer;
        run(0, step, buffer, false, nullptr);
        arrived(STAGES - 2);
        run(1, step + 1, next, true, to);
        scales.request(step + STAGES, to + (TR + TC) * 128, wave);
        loads.next(a);
        buffer = next;
    }
    for (; step < last; ++step) {
        const int next = buffer + 1 < STAGES ? buffer + 1 : 0;
        run(0, step, buffer, false, nullptr);
        arrived(min(last - 2 - step, STAGES - 2));
        run(1, step + 1, next, false, nullptr);                         // (behind the last step what is read is not used)
        buffer = next;
    }
    results_settled(acc);
    __syncthreads();
    char *room = lds + wave * 32 * (BR * 32 + 4) * 4;
    if (a.splits > 1) put_blocks32<OP, kParts, BR, BC>(a, acc, r0 + wr * BR * 32, c0 + wc * BC * 32, split, room);
    else put_blocks32<OP, OUT, BR, BC>(a, acc, r0 + wr * BR * 32, c0 + wc * BC * 32, split, room);
}

// Tiles of 256 x 256 outputs by four waves, one per SIMD, of 128 x 128 each: 8 x 8 blocks of 16 x 16, whose matrix instruction takes a whole step.  (Blocks of 32 x 32 take half a step each, and
// 5 to 7 % more power for the same values, by which large products are bound: 8192 x 4096 -> 16384 492 us, now 460 to 470, 2.35 PFLOP/s, where a library product of 8-bit floats without
// such scales takes 446 to 466.)  The accumulators fill the 256 accumulation registers, the operands of one step
// half of the others; the next step's go to the same registers, as they become free:
//   - the first half of step t multiplies rows 0-3 of the blocks by all columns, and reads rows 4-7; then a barrier, before which each wave has waited for its reads and for its loads of
//     step t + 1: nobody reads the buffer of step t any more;
//   - the second half multiplies rows 4-7, column by column, and reads rows 0-3 of step t + 1 and, behind each column, that column of step t + 1, while loads of step t + 2 go to the
//     buffer of step t.
// One workgroup per compute unit goes from tile to tile, and the first two steps of the next tile are asked for before this one's outputs are formed.  Rows of p lie in the order that gives a
// lane eight outputs next to each other, as in product_kernel_256.
template <int QF, int OUT>
__global__ __launch_bounds__(256, 1) void product_f8_kernel_256(ProductsF8 all)
{
    constexpr int TR = 256, TC = 256, FR = 8, FC = 8;
    typedef TileLoads<TR, TC, 4, 1> Loads;
    typedef ScaleLoads<TR, TC, 4> Scales;
    constexpr int kScales = (TR + TC) * 128, kBuffer = kScales + Scales::kBytes;
    extern __shared__ char lds[];                                       // [2]{[TR + TC][128], scales}, bias
    float *const biases = (float *)(lds + 2 * kBuffer);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t workers = gridDim.x - all.sum_blocks;
    if ((int32_t)blockIdx.x >= workers) {
        column_sums(all.sums, blockIdx.x - workers, (float *)lds);
        return;
    }
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 15, fk = lane >> 4, swizzle = frow & 7;
    const int row_p = wr * FR * 16 + (frow >> 2) * 8 + (frow & 3), row_q = TR + wc * FC * 16 + frow, lo = (fk ^ swizzle) * 16, hi = ((4 + fk) ^ swizzle) * 16;
    Loads loads;
    Scales scales;
    f32x4 acc[FR][FC];
    i32x8 p[FR], q[FC];
    int ep[FR], eq[FC];
    int32_t r0, c0, which;
    float bias;                                                         // of row r0 + the thread's number
    const auto begin = [&](int32_t tile) __attribute__((always_inline)) {
        which = tile >= all.first[1];
        const ProductF8Args &a = all.a[which];
        int32_t split, tr, tc;
        tile_of(tile - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
        r0 = tr * TR;
        c0 = tc * TC;
        loads.init(a, r0, c0, 0, wave);
        scales.init(a, r0, c0, wave);
        loads.request(a, lds, wave);
        scales.request(0, lds + kScales, wave);
        if (a.steps > 1) {
            loads.request(a, lds + kBuffer, wave);
            scales.request(1, lds + kBuffer + kScales, wave);
        }
        bias = a.bias && r0 + (int32_t)threadIdx.x < a.R ? param(a.bias, a.bias_dtype, r0 + (int32_t)threadIdx.x) : 0.0f;
    };
    // Where a lane's reads of a step begin, in bytes of LDS: blocks lie at constant distances from there.
    typedef const __attribute__((address_space(3))) char *At;
    struct Places {
        At lo, hi, e;
    };
    const auto places = [&](int32_t step, int row) __attribute__((always_inline)) {
        const At from = (At)lds + (step & 1) * kBuffer;
        Places at{from + (row * 128 + lo), from + (row * 128 + hi), from + (kScales + (step & 3) + row * 4)};
        asm("" : "+v"(at.lo), "+v"(at.hi), "+v"(at.e));                 // (what is added to them stays an offset of the reads)
        return at;
    };
    const auto operand = [&](const Places &at, int row, i32x8 &to, int &e) __attribute__((always_inline)) {
        typedef const __attribute__((address_space(3))) i32x4 *Quad;
        const i32x4 u = *(Quad)(at.lo + row * 128), v = *(Quad)(at.hi + row * 128);
        to = i32x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
        e = *(const __attribute__((address_space(3))) uint8_t *)(at.e + row * 4);
    };
    const auto read_p = [&](const Places &at, int i) __attribute__((always_inline)) { operand(at, (i >> 1) * 32 + (i & 1) * 4, p[i], ep[i]); };
    const auto read_q = [&](const Places &at, int j) __attribute__((always_inline)) { operand(at, j * 16, q[j], eq[j]); };
    const auto mma = [&](int i, int j) __attribute__((always_inline)) {
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] blgp:%5" : "+a"(acc[i][j]) : "v"(p[i]), "v"(q[j]), "v"(ep[i]), "v"(eq[j]), "n"(QF));
    };
    // what the matrix instructions wrote can be read, or moved, behind this: the compiler does not know that they wrote it, and that it takes a while
    const auto settled = [&]() __attribute__((always_inline)) {
        asm volatile("s_nop 15");
#pragma unroll
        for (int i = 0; i < FR; ++i)
            asm volatile("" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]), "+a"(acc[i][3]), "+a"(acc[i][4]), "+a"(acc[i][5]), "+a"(acc[i][6]), "+a"(acc[i][7]));
    };
    const auto barrier = [] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");                                  // (nothing is read before the barrier)
    };
    // the loads of step + 2, two behind each column from kFirst on of the first half
    constexpr int kFirst = 5;
    const auto request_two = [&](const ProductF8Args &a, int32_t step, int k) __attribute__((always_inline)) {
        char *const to = lds + (step & 1) * kBuffer;
        if (k < 8) {
            loads.request_one(a, to, wave, 2 * k);
            loads.request_one(a, to, wave, 2 * k + 1);
        } else if (k == 8) {
            scales.request_one(step + 2, to + kScales, wave, 0);
            scales.request_one(step + 2, to + kScales, wave, 1);
            loads.next(a);
        }
    };
    // the halves of a step
    const auto first_half = [&](const ProductF8Args &a, int32_t step, bool ask) __attribute__((always_inline)) {
        const Places at_p = places(step, row_p);
#pragma unroll
        for (int j = 0; j < FC; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mma(i, j);
            if (j < 4) read_p(at_p, 4 + j);
            if (j == kFirst - 1 && ask) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                barrier();
            }
            if (j >= kFirst && ask) request_two(a, step, j - kFirst);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (ask) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (FC - kFirst)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        barrier();
    };
    const auto second_half = [&](const ProductF8Args &a, int32_t step, bool read, bool ask) __attribute__((always_inline)) {
        const Places at_p = places(step + 1, row_p), at_q = places(step + 1, row_q);
#pragma unroll
        for (int j = 0; j < FC; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mma(4 + i, j);
            if (read) read_q(at_q, j);
            if (read && j < 4) read_p(at_p, j);
            if (ask) request_two(a, step, j + FC - kFirst);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int32_t tile = blockIdx.x, after = 0;                               // after: stores that surely were issued behind the loads under way
    begin(tile);
    while (true) {
        const ProductF8Args &a = all.a[which];
        const int32_t steps = a.steps, row0 = r0, col0 = c0, r = wr * FR * 16 + fk * 8, c = wc * FC * 16 + frow;
        // (of what was issued behind the loads, the stores of the tile before may go on)
        biases[threadIdx.x] = bias;
        if (after >= 32) asm volatile("s_waitcnt vmcnt(32) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        barrier();
        // sums begin with the bias
#pragma unroll
        for (int i = 0; i < FR; ++i) {
            const f32x4 b = *(const f32x4 *)(biases + r + (i >> 1) * 32 + (i & 1) * 4);
#pragma unroll
            for (int j = 0; j < FC; ++j) acc[i][j] = b;
        }
        {
            const Places at_p = places(0, row_p), at_q = places(0, row_q);
#pragma unroll
            for (int i = 0; i < 4; ++i) read_p(at_p, i);
#pragma unroll
            for (int j = 0; j < FC; ++j) read_q(at_q, j);
        }
        int32_t step = 0;
        if (steps > 2) {
            do {
                first_half(a, step, true);
                second_half(a, step, true, true);
            } while (++step + 2 < steps);
            settled();                                                  // (between the loops some move to other registers)
        }
        for (; step < steps; ++step) {
            first_half(a, step, false);
            second_half(a, step, true, false);                          // (behind the last step what is read is not used)
        }
        // (what the last step needed was read before its last barrier: LDS is free)
        tile += workers;
        const bool more = tile < all.first[2];
        if (more) begin(tile);
        settled();
        typedef typename Elem<OUT>::type T;
        const bool wide = (a.ld_out * sizeof(T)) % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.R % 8 == 0;
        const bool whole = wide && row0 + TR <= a.R && col0 + TC <= a.C;
        T *const out = (T *)a.out;
#pragma unroll
        for (int j = 0; j < FC; ++j) {
            const int32_t column = col0 + c + j * 16;
            if (whole) {
                i32x4 piece[FR / 2];
#pragma unroll
                for (int i = 0; i < FR / 2; ++i) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[2 * i + (e >> 2)][j][e & 3];
                    piece[i] = __builtin_bit_cast(i32x4, Elem<OUT>::pack(v));
                }
#pragma unroll
                for (int i = 0; i < FR / 2; i += 2) put_lines<32>(out, row0 + r + i * 32, column, a.ld_out, piece[i], piece[i + 1]);
            } else if (column < a.C) {
#pragma unroll
                for (int i = 0; i < FR / 2; ++i) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[2 * i + (e >> 2)][j][e & 3];
                    if (wide) store8<OUT, true>(out + (int64_t)column * a.ld_out, row0 + r + i * 32, a.R, v);
                    else store8<OUT, false>(out + (int64_t)column * a.ld_out, row0 + r + i * 32, a.R, v);
                }
            }
        }
        if (!more) return;
        after = whole ? 32 : 0;
    }
}

// Measured on 128 to 1024 workgroups of 1 to 196 steps: 128 x 128 on 256 workgroups 7.8 us for two steps and 41.3 for 64, 128 x 64 5.8 and 28.2, 64 x 64 5.0 and 24.7; on 512 10.6 and 68.5,
// 7.5 and 46.2, 5.6 and 34.9; 256 x 256 12.0 and 98.9, on 512 24.5 and 196.  Over 61 forward and backward calls the choice takes up to 1.06 of the best one's time, and 1.12
// in two of them; by the costs of int8 up to 1.24 (512 x 25088 -> 4096: 82 us, now 66).
constexpr ProductCosts kCostsF8{{{4, 4, 6.6f, 0.56f, 0.98f}, {4, 2, 4.9f, 0.36f, 0.66f}, {2, 2, 4.6f, 0.31f, 0.47f}}, 128, true, 4e6f, 4.6f, 4.5f, 3.0f, 1.4f, 1.12f};

ProductPlan plan_products_f8(const ProductShape *shapes, int n) { return plan_products(shapes, n, kCostsF8); }

template <int QF, int OUT>
static hipError_t launch_as(const ProductF8Args *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    ProductsF8 all{};
    const bool large = tile == kTile256;
    const int32_t tr = large ? 256 : 32 * kCostsF8.tiles[tile].r, tc = large ? 256 : 32 * kCostsF8.tiles[tile].c;
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
    const bool alone = blocks <= 256;                                   // (1024 x 4096 -> 4096, 256 workgroups: four buffers 29.9 us, two 35.8; 2048 x 2048 -> 4096, 512: 35.4 and 29.4)
    const auto kernel = large       ? product_f8_kernel_256<QF, OUT>
                        : tile == 0 ? (alone ? product_f8_kernel<QF, OUT, 2, 2, 4> : product_f8_kernel<QF, OUT, 2, 2, 2>)
                        : tile == 1 ? product_f8_kernel<QF, OUT, 2, 1, 3>
                                    : product_f8_kernel<QF, OUT, 1, 1, 4>;
    const int stages = large ? 2 : tile == 0 ? (alone ? 4 : 2) : tile == 1 ? 3 : 4, scales = ((tr + tc) / 64 + 3) / 4 * 1024;
    const int lds = stages * ((tr + tc) * 128 + scales) + (large ? 1024 : 0);
    if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), lds, s, all);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const ProductArgs *const joined[2] = {a, n > 1 ? a + 1 : a};
    return join_as<OpF8<QF>, OUT>(joined, n, s);
}

hipError_t launch_products_f8(const ProductF8Args *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    const int32_t dt = n ? a[0].dtype : c.dtype, format = n ? a[0].q_format : TICTAC_E4M3;
    if (format == TICTAC_E5M2) return dt == TICTAC_F16 ? launch_as<TICTAC_E5M2, TICTAC_F16>(a, n, tile, c, s) : launch_as<TICTAC_E5M2, TICTAC_BF16>(a, n, tile, c, s);
    return dt == TICTAC_F16 ? launch_as<TICTAC_E4M3, TICTAC_F16>(a, n, tile, c, s) : launch_as<TICTAC_E4M3, TICTAC_BF16>(a, n, tile, c, s);
}

}  // namespace tictac
