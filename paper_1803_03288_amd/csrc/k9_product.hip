// See k9_product.h.  A step of 128 bytes of k is one matrix instruction of 16 x 16 x 128 for each block of outputs, which takes the scales of its operands' rows too.
// The instruction adds the 128 products with what they exceed about 2^-13 of the largest by (measured: 1.4e-5 of the result's norm for normal values, 5e-5 where values
// are spread over many powers of two); outputs here have 16 bits, and their own rounding is off by 2^-9 or 2^-12.  float32 outputs take bf16 instructions, whose sums are float32.
#include "k9_product.h"
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
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int run = min(i * WAVES + wave, kRuns - 1), row = run * 64 + lane;
            const bool is_p = run < TR / 64;
            const int32_t at = is_p ? min(r0 + row, a.R - 1) >> a.p_shift : min(c0 + row - TR, a.C - 1) >> a.q_shift;
            const int32_t first = is_p ? r0 >> a.p_shift : c0 >> a.q_shift;
            base[i] = is_p ? a.p_e + (int64_t)first * a.ld_pe : a.q_e + (int64_t)first * a.ld_qe;
            off[i] = (uint32_t)(at - first) * (uint32_t)(is_p ? a.ld_pe : a.ld_qe);
        }
    }
    __device__ __forceinline__ void request(int32_t step, char *to, int wave)
    {
#pragma unroll
        for (int i = 0; i < NS; ++i)
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
    typedef TileLoads<TR, TC, 4, false> Loads;
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

struct TileF8 { int32_t r, c; };
constexpr TileF8 kTilesF8[] = {{4, 4}, {4, 2}, {2, 2}};

ProductPlan plan_products_f8(const ProductShape *shapes, int n)
{
    ProductPlan plan = plan_products(shapes, n);
    if (plan.tile > 2) plan.tile = 0;
    return plan;
}

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
    blocks += all.sum_blocks;
    const bool alone = blocks <= 256;
    const auto kernel = tile == 0   ? (alone ? product_f8_kernel<QF, OUT, 4, 4, 4> : product_f8_kernel<QF, OUT, 4, 4, 2>)
                        : tile == 1 ? product_f8_kernel<QF, OUT, 4, 2, 3>
                                    : product_f8_kernel<QF, OUT, 2, 2, 4>;
    const int stages = tile == 0 ? (alone ? 4 : 2) : tile == 1 ? 3 : 4, scales = ((tr + tc) / 64 + 3) / 4 * 1024;
    const int lds = stages * ((tr + tc) * 128 + scales);
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
