// See k9_product.h.  A step of 128 bytes of k is two matrix instructions of 32 x 32 x 64 for each block of outputs, which take the scales of their operands' rows too.
// The instruction adds the 128 products with what they exceed about 2^-13 of the largest by (measured: 1.4e-5 of the result's norm for normal values, 5e-5 where values
// are spread over many powers of two); outputs here have 16 bits, and their own rounding is off by 2^-9 or 2^-12.  float32 outputs take bf16 instructions, whose sums are float32.
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

// Sixteen-byte pieces of outputs, four of a line of 128 bytes of column n in lane n + 32 g, to whole lines: the lanes of columns n, n + 8, n + 16 and n + 24 exchange them (a square of four by
// four is turned round), so that each of four stores brings eight lanes' 128 bytes of eight columns.
template <typename T>
__device__ __forceinline__ void put_lines32(T *line, int64_t ld, i32x4 (&piece)[4])
{
    const int lane = threadIdx.x & 63;
    const bool first = (lane & 8) == 0;
    i32x4 out[2][2];                    // [column + 16 ..][+ 8 ..]
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)piece[k][e], (uint32_t)piece[k + 2][e], false, false);
            piece[k][e] = (int32_t)r[0];
            piece[k + 2][e] = (int32_t)r[1];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t lo = piece[2 * h][e], hi = piece[2 * h + 1][e], other = __builtin_amdgcn_update_dpp(0, first ? hi : lo, 0x128, 0xf, 0xf, true);       // row_ror:8
            out[h][0][e] = first ? lo : other;
            out[h][1][e] = first ? other : hi;
        }
    }
    T *const to = line + (int64_t)(lane & 7) * ld + (lane & 16) * 2 + (lane >> 5) * 16 + (lane & 8);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k) __builtin_nontemporal_store(out[h][k], (i32x4 *)(to + (int64_t)(h * 16 + k * 8) * ld));
}

// Tiles of 256 x 256 outputs by four waves, one per SIMD, of 128 x 128 each: 4 x 4 blocks of 32 x 32, whose matrix instruction takes half a step (64 bytes of k).  A step has two halves of
// sixteen of them; under each half the operands of the next are read:
//   - half 0 of step t reads the rest of step t; then a barrier, before which each wave has waited for its reads and for its loads of step t + 1;
//   - half 1 of step t reads the first half of step t + 1 and asks for step t + 2, into the buffer of step t.
// The accumulators fill the 256 accumulation registers, hence the matrix instructions in assembly.  (Blocks of 16 x 16 take a whole step at once: operands of two steps do not
// fit beside them.)  One workgroup per compute unit goes from tile to tile, and the first two steps of the next tile are asked for before this one's outputs are formed.
// Row m of a block of rows of p is row 16 (m / 4 % 2) + 4 (m / 8) + m % 4 of 32, so that a lane has sixteen outputs next to each other.
template <int QF, int OUT>
__global__ __launch_bounds__(256, 1) void product_f8_kernel_256(ProductsF8 all)
{
    constexpr int TR = 256, TC = 256, FR = 4, FC = 4;
    typedef TileLoads<TR, TC, 4, 3> Loads;
    typedef ScaleLoads<TR, TC, 4> Scales;
    constexpr int kBuffer = (TR + TC) * 128 + Scales::kBytes;
    extern __shared__ char lds[];                                       // [2]{[TR + TC][128], scales}, bias
    float *const biases = (float *)(lds + 2 * kBuffer);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t workers = gridDim.x - all.sum_blocks;
    if ((int32_t)blockIdx.x >= workers) {
        column_sums(all.sums, blockIdx.x - workers, (float *)lds);
        return;
    }
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 31, fk = lane >> 5;
    const int row_p = wr * 128 + (frow >> 2 & 1) * 16 + (frow >> 3) * 4 + (frow & 3), row_q = TR + wc * 128 + frow, swizzle = frow >> 1 & 7;     // (of both)
    Loads loads;
    Scales scales;
    f32x16 acc[FR][FC];
    i32x8 fp[2][FR], fq[2][FC];
    int ep[2][FR], eq[2][FC];
    int32_t r0, c0, which;
    const auto begin = [&](int32_t tile) {
        which = tile >= all.first[1];
        const ProductF8Args &a = all.a[which];
        int32_t split, tr, tc;
        tile_of(tile - all.first[which], all.tiles_r[which], all.tiles_c[which], split, tr, tc);
        r0 = tr * TR;
        c0 = tc * TC;
        loads.init(a, r0, c0, 0, wave);
        scales.init(a, r0, c0, wave);
        loads.request(a, lds, wave);
        scales.request(0, lds + (TR + TC) * 128, wave);
        if (a.steps > 1) {
            loads.request(a, lds + kBuffer, wave);
            scales.request(1, lds + kBuffer + (TR + TC) * 128, wave);
        }
    };
    // operand n of a half: columns first
    const auto read_one = [&](int half, int n, int32_t step) {
        const char *const from = lds + (step & 1) * kBuffer;
        const int lo = ((half * 4 + fk * 2) ^ swizzle) * 16, hi = ((half * 4 + fk * 2 + 1) ^ swizzle) * 16, row = n < FC ? row_q + n * 32 : row_p + (n - FC) * 32;
        const i32x4 u = *(const i32x4 *)(from + row * 128 + lo), v = *(const i32x4 *)(from + row * 128 + hi);
        const i32x8 w{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
        const int e = *(const uint8_t *)(from + (TR + TC) * 128 + row * 4 + (step & 3));
        if (n < FC) { fq[half][n] = w; eq[half][n] = e; }
        else { fp[half][n - FC] = w; ep[half][n - FC] = e; }
    };
    // One half of a step: its sixteen matrix instructions, behind the first eight of them an operand of the next half is read, and in half 1 loads of a later step are asked for
    const auto run = [&](const ProductF8Args &a, int half, int32_t step, bool read, bool ask) {
        char *const to = lds + (step & 1) * kBuffer;
#pragma unroll
        for (int n = 0; n < FR * FC; ++n) {
            OpF8<QF>::mma(fp[half][n / FC], fq[half][n % FC], acc[n / FC][n % FC], ep[half][n / FC], eq[half][n % FC]);
            if (read && n < FR + FC) read_one(half ^ 1, n, step + half);        // (half 1 reads the next step)
            if (ask) loads.request_one(a, to, wave, n);
            if (ask && n % 8 == 7) scales.request_one(step + 2, to + (TR + TC) * 128, wave, n / 8);
            __builtin_amdgcn_sched_barrier(0);
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
        const ProductF8Args &a = all.a[which];
        const int32_t steps = a.steps, row0 = r0, col0 = c0, t = threadIdx.x;
        float bias = 0.0f;
        if (a.bias && row0 + t < a.R) bias = param(a.bias, a.bias_dtype, row0 + t);
#pragma unroll
        for (int i = 0; i < FR; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j) acc[i][j] = f32x16{};
        // (of what was issued behind the loads, the stores of the tile before may go on)
        if (after >= 32) asm volatile("s_waitcnt vmcnt(32)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        barrier();
#pragma unroll
        for (int n = 0; n < FR + FC; ++n) read_one(0, n, 0);
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
        // (the last reads of a step lie before its barrier: LDS is free)
        biases[t] = bias;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
        tile += workers;
        const bool more = tile < all.first[2];
        if (more) begin(tile);
        results_settled(acc);
        typedef typename Elem<OUT>::type T;
        const bool wide = (a.ld_out * sizeof(T)) % 16 == 0 && ((uintptr_t)a.out & 15) == 0 && a.R % 8 == 0;
        const bool whole = wide && row0 + TR <= a.R && col0 + TC <= a.C;
        T *const out = (T *)a.out;
#pragma unroll
        for (int line = 0; line < 2; ++line) {
            float b[2][16];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const f32x4 v = *(const f32x4 *)(biases + wr * 128 + line * 64 + h * 32 + fk * 16 + k * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[h][k * 4 + e] = v[e];
                }
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                i32x4 piece[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[line * 2 + (k >> 1)][j][(k & 1) * 8 + e] + b[k >> 1][(k & 1) * 8 + e];
                    if (whole) {
                        piece[k] = __builtin_bit_cast(i32x4, Elem<OUT>::pack(v));
                        continue;
                    }
                    const int32_t row = row0 + wr * 128 + line * 64 + (k >> 1) * 32 + fk * 16 + (k & 1) * 8, column = col0 + wc * 128 + j * 32 + frow;
                    if (column >= a.C) continue;
                    if (wide) store8<OUT, true>(out + (int64_t)column * a.ld_out, row, a.R, v);
                    else store8<OUT, false>(out + (int64_t)column * a.ld_out, row, a.R, v);
                }
                if (whole) put_lines32(out + (int64_t)(col0 + wc * 128 + j * 32) * a.ld_out + row0 + wr * 128 + line * 64, a.ld_out, piece);
            }
        }
        if (!more) return;
        after = whole ? 32 : 0;
        barrier();                                                      // (the biases are read before the next tile's are written)
    }
}

struct TileF8 { int32_t r, c; };
constexpr TileF8 kTilesF8[] = {{2, 2}, {2, 1}, {1, 1}, {4, 4}};
constexpr int32_t kLargest = 3;

ProductPlan plan_products_f8(const ProductShape *shapes, int n) { return plan_products(shapes, n); }

template <int QF, int OUT>
static hipError_t launch_as(const ProductF8Args *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    ProductsF8 all{};
    const int32_t tr = 64 * kTilesF8[tile].r, tc = 64 * kTilesF8[tile].c;
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
    const bool large = tile == kLargest;
    if (large) {
        int device = 0;
        if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
        blocks = std::min(blocks, (int32_t)device_cu_count(device));
    }
    blocks += all.sum_blocks;
    const bool alone = blocks <= 256;
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
