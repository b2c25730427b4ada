// See k9_product.h.  A step of 128 bytes of k is one matrix instruction of 16 x 16 x 128 for each block of outputs, which takes the scales of its operands' rows too.
// The instruction adds the 128 products with what they exceed about 2^-13 of the largest by (measured: 1.4e-5 of the result's norm for normal values, 5e-5 where values
// are spread over many powers of two); outputs here have 16 bits, and their own rounding is off by 2^-9 or 2^-12.  float32 outputs take bf16 instructions, whose sums are float32.
#include "k9_product.h"

#include <algorithm>

#include "k8_tiles.h"

namespace tictac {

template <int QF>                       // format of q
struct OpF8 {
    typedef f32x4 acc;
    typedef float sum;
    static __device__ __forceinline__ float value(float s) { return s; }
    static __device__ __forceinline__ acc mma(i32x8 a, i32x8 b, acc c, int ea, int eb)
    {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, TICTAC_E4M3, QF, 0, ea, 0, eb);
    }
};
template <int QF>
struct Biased<OpF8<QF>> { static constexpr bool value = true; };

typedef ProductsOf<ProductF8Args> ProductsF8;
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// A tile of 32 FR x 32 FC outputs by four waves, STAGES buffers in turn.  While a step is multiplied from registers, the operands of the next are read from LDS; then a barrier, before
// which each wave has waited for its reads and for its loads of the step behind that, and the buffer of the step that was read is asked to take the one STAGES on.
template <int QF, int OUT, int FR, int FC, int STAGES>
__global__ __launch_bounds__(256, STAGES * (FR + FC) > 20 ? 1 : 2) void product_f8_kernel(ProductsF8 all)
{
    using OP = OpF8<QF>;
    constexpr int TR = FR * 32, TC = FC * 32;
    typedef TileLoads<TR, TC, 4, 0> Loads;
    typedef ScaleLoads<TR, TC, 4> Scales;
    constexpr int kBuffer = (TR + TC) * 128 + Scales::kBytes, kLoads = Loads::LP + Loads::LQ + Scales::NS;
    extern __shared__ char lds[];                                       // [STAGES]{[TR + TC][128], scales}
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int32_t)blockIdx.x >= all.first[2]) {
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
    const int wr = wave & 1, wc = wave >> 1, frow = lane & 15, fk = lane >> 4, swizzle = frow & 7;
    const int lo = (fk ^ swizzle) * 16, hi = ((4 + fk) ^ swizzle) * 16, row_p = wr * FR * 16 + frow, row_q = wc * FC * 16 + frow;
    f32x4 acc[FR][FC];
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = f32x4{};
    struct Operands {
        i32x8 p[FR], q[FC];
        int ep[FR], eq[FC];
    };
    const auto request = [&](int32_t step) {
        char *to = lds + (step - first) % STAGES * kBuffer;
        loads.request(a, to, wave);
        scales.request(step, to + (TR + TC) * 128, wave);
    };
    const auto two = [&](const char *row) {
        const i32x4 u = *(const i32x4 *)(row + lo), v = *(const i32x4 *)(row + hi);
        return i32x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
    };
    const auto read = [&](int32_t step, Operands &o) {
        const char *from = lds + (step - first) % STAGES * kBuffer, *e = from + (TR + TC) * 128 + (step & 3);
#pragma unroll
        for (int i = 0; i < FR; ++i) { o.p[i] = two(from + (row_p + i * 16) * 128); o.ep[i] = *(const uint8_t *)(e + (row_p + i * 16) * 4); }
#pragma unroll
        for (int j = 0; j < FC; ++j) { o.q[j] = two(from + (TR + row_q + j * 16) * 128); o.eq[j] = *(const uint8_t *)(e + (TR + row_q + j * 16) * 4); }
    };
    const auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int i = 0; i < FR; ++i)
#pragma unroll
            for (int j = 0; j < FC; ++j) acc[i][j] = OP::mma(o.p[i], o.q[j], acc[i][j], o.ep[i], o.eq[j]);
    };
    // waits until all but the loads of the last `later` steps that were asked for have arrived, and for the wave's reads
    const auto arrived = [&](int32_t later) {
        if (STAGES > 3 && later >= 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(3 * kLoads) : "memory");
        else if (STAGES > 2 && later >= 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kLoads) : "memory");
        else if (later >= 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    Operands now, next;
    if (first < last) {
        for (int32_t step = first; step < last && step < first + STAGES; ++step) request(step);
        arrived(min(last - 1 - first, STAGES - 1));                     // the first step
        read(first, now);
        arrived(min(max(last - 2 - first, 0), STAGES - 2));             // the second; nobody reads the first any more
    }
    for (int32_t step = first; step < last; ++step) {
        if (step + STAGES < last) request(step + STAGES);
        if (step + 1 < last) read(step + 1, next);
        multiply(now);
        if (step + 1 < last) {
            // what was asked for behind step + 2: up to step + STAGES, or to the last
            arrived(min(max(last - 3 - step, 0), STAGES - 2));
            now = next;
        }
    }
    __syncthreads();
    char *room = lds + wave * 16 * (FR * 16 + 4) * 4;
    if (a.splits > 1) put_blocks<OP, kParts, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
    else put_blocks<OP, OUT, FR, FC>(a, acc, r0 + wr * FR * 16, c0 + wc * FC * 16, split, room);
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
    typedef TileLoads<TR, TC, 4, 2> Loads;
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
    const int row_p = wr * 128 + (frow >> 2 & 1) * 16 + (frow >> 3) * 4 + (frow & 3), row_q = TR + wc * 128 + frow, swizzle = frow & 7;     // (of both)
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
            asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] blgp:%5"
                         : "+a"(acc[n / FC][n % FC]) : "v"(fp[half][n / FC]), "v"(fq[half][n % FC]), "v"(ep[half][n / FC]), "v"(eq[half][n % FC]), "n"(QF));
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
        // the compiler does not know that matrix instructions wrote these, and their results take a while
#pragma unroll
        for (int i = 0; i < FR; ++i) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]), "+a"(acc[i][3]));
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
constexpr TileF8 kTilesF8[] = {{4, 4}, {4, 2}, {2, 2}, {8, 8}};
constexpr int32_t kLargest = 3;

ProductPlan plan_products_f8(const ProductShape *shapes, int n) { return plan_products(shapes, n); }

template <int QF, int OUT>
static hipError_t launch_as(const ProductF8Args *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s)
{
    ProductsF8 all{};
    const int32_t tr = 32 * kTilesF8[tile].r, tc = 32 * kTilesF8[tile].c;
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
                        : tile == 0 ? (alone ? product_f8_kernel<QF, OUT, 4, 4, 4> : product_f8_kernel<QF, OUT, 4, 4, 2>)
                        : tile == 1 ? product_f8_kernel<QF, OUT, 4, 2, 3>
                                    : product_f8_kernel<QF, OUT, 2, 2, 4>;
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
