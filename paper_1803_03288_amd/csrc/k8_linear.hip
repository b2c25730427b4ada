// A layer with 8-bit weights, y[t][o] = xs[t] ws[o] sum_i xq[t][i] w[o][i] + bias[o], and its gradients
//   dx[t][i] = sum_o (dy[t][o] ws[o]) w[o][i],   dw[o][i] = sum_t (dy[t][o] xs[t]) xq[t][i],   db[o] = sum_t dy[t][o]
// Forward: sums exact in int32.  Backward: int8 values are exact in bf16; dy times a scale, a float32 value, is cut into as many bf16
// pieces as dy's type has bits to give (bf16 one, rounded once as dy itself was; float16 two; float32 three, exact), and the pieces go side by
// side along k through the one product of k8_product.hip (with many rows of bf16 the scale goes to the 8-bit value instead, also rounded once);
// sums in float32.
#include "k8_product.h"

namespace tictac {

// ---- few rows: bound by the bytes of the weights ----
// A workgroup has 16 FB outputs and a part of k, its eight waves an eighth of that each: weights go from memory to the matrix instruction without
// LDS, sixteen bytes per lane, the next unit of 128 bytes under way while one is computed.  TB blocks of 16 rows of x come from the caches.  The
// sums of the waves meet in LDS, those of several workgroups along k in the workspace.
// Alone the weights of 4096 x 25088 stream at 5.1 TB/s (20 us).  Through the L2 go 7.4 TB/s in all, so x, read again for each 16 FB outputs, has to
// stay well below the weights: rows / (16 FB) of their bytes.  32 rows with FB = 1: 41 us, with FB = 4 26.
constexpr int kFewWaves = 8;

template <int TB, int FB>
__global__ __launch_bounds__(kFewWaves * 64) void linear_few_kernel(LinearArgs p, const int8_t *xq, int64_t ld_xq, const float *xs, int32_t splits, int32_t *parts)
{
    __shared__ i32x4 sums[kFewWaves][TB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, fk = (lane >> 4) * 16;
    const int64_t blocks = gridDim.x / splits, o0 = blockIdx.x % blocks * (16 * FB);
    const int32_t split = (int32_t)(blockIdx.x / blocks), all = (int32_t)((p.cols + 127) / 128);
    const int32_t first = (int32_t)((int64_t)all * split / splits), units = (int32_t)((int64_t)all * (split + 1) / splits);
    const int8_t *w[FB], *x[TB];
#pragma unroll
    for (int f = 0; f < FB; ++f) w[f] = p.w + min(o0 + f * 16 + row, p.outs - 1) * p.ld_w + fk;
#pragma unroll
    for (int b = 0; b < TB; ++b) x[b] = xq + min((int64_t)b * 16 + row, p.rows - 1) * ld_xq + fk;
    i32x4 acc[FB][TB] = {}, now[FB][2], next[FB][2];
    const auto request = [&](int32_t u) {
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int k = 0; k < 2; ++k) next[f][k] = *(const i32x4 *)(w[f] + (int64_t)u * 128 + k * 64);
    };
    if (first + wave < units) request(first + wave);
    for (int32_t u = first + wave; u < units; u += kFewWaves) {
        i32x4 fx[2][TB];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int b = 0; b < TB; ++b) fx[k][b] = *(const i32x4 *)(x[b] + (int64_t)u * 128 + k * 64);
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int k = 0; k < 2; ++k) now[f][k] = next[f][k];
        if (u + kFewWaves < units) request(u + kFewWaves);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int b = 0; b < TB; ++b) acc[f][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[f][k], fx[k][b], acc[f][b], 0, 0, 0);
    }
#pragma unroll
    for (int f = 0; f < FB; ++f) {
        if (f) __syncthreads();
#pragma unroll
        for (int b = 0; b < TB; ++b) sums[wave][b][lane] = acc[f][b];
        __syncthreads();
        // lane l of a block holds outputs 4 (l / 16) .. + 3 of row l % 16; a thread finishes one output
        for (int i = threadIdx.x; i < TB * 256; i += kFewWaves * 64) {
            const int b = i >> 8, o = i & 15, t = (i >> 4) & 15;
            uint32_t sum = 0;
#pragma unroll
            for (int k = 0; k < kFewWaves; ++k) sum += (uint32_t)sums[k][b][(o >> 2) * 16 + t][o & 3];
            const int64_t at = (int64_t)b * 16 + t, out = o0 + f * 16 + o;
            if (at >= p.rows || out >= p.outs) continue;
            if (splits > 1) {
                parts[((int64_t)split * p.rows + at) * p.outs + out] = (int32_t)sum;
                continue;
            }
            float v = exact_sum((int32_t)sum) * (xs[at] * p.ws[out]);
            if (p.bias) v += param(p.bias, p.bias_dtype, out);
            put_param(p.y, p.dtype, at * p.ld_y + out, v);
        }
    }
}

// Up to sixteen rows of floats, rounded to 8 bits here: every workgroup takes the largest magnitudes of the rows again (they come from the caches, under the
// first loads of the weights), which costs less than a launch before it (2.6 us, and what lies between two) while all rows are at most 64 KB (kOnceBytes).
// 1 x 4096 x 4096: 8 us.  The 8-bit values are those of quantize_rows_kernel.
constexpr int kOnceWaves = 16, kOnceRows = 16;
constexpr int64_t kOnceBytes = 64 << 10;

template <int DT, bool WIDE>
__global__ __launch_bounds__(kOnceWaves * 64) void linear_once_kernel(LinearArgs p)
{
    using E = Elem<DT>;
    using T = typename E::type;
    constexpr int kUnits = 2;                               // of weights under way
    __shared__ uint32_t part[kOnceRows][kOnceWaves];
    __shared__ i32x4 sums[kOnceWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, fk = (lane >> 4) * 16;
    const int64_t o0 = (int64_t)blockIdx.x * 16;
    const int32_t units = (int32_t)((p.cols + 127) / 128), rows = (int32_t)p.rows;
    const int8_t *w = p.w + min(o0 + row, p.outs - 1) * p.ld_w + fk;
    i32x4 next[kUnits][2];
    const auto request = [&](int32_t u) {
#pragma unroll
        for (int n = 0; n < kUnits; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                next[n][k] = u + n * kOnceWaves < units ? *(const i32x4 *)(w + (int64_t)(u + n * kOnceWaves) * 128 + k * 64) : i32x4{};
    };
    request(wave);
    // each row's largest magnitude by 16 / rows waves
    const int each = rows <= 1 ? 16 : rows <= 2 ? 8 : rows <= 4 ? 4 : rows <= 8 ? 2 : 1, of = wave / each, piece = wave % each;
    if (of < rows) {
        uint32_t m = 0;
        for (int64_t col = piece * 512 + lane * 8; col < p.cols; col += each * 512) {
            float v[8];
            E::floats(load8<DT, WIDE>((const T *)p.x + of * p.ld_x, col, p.cols), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
        }
        m = wave_max_u32(m);
        if (lane == 0) part[of][piece] = m;
    }
    __syncthreads();
    const int mine = min(row, rows - 1);
    uint32_t m = 0;
    for (int i = 0; i < each; ++i) m = max(m, part[mine][i]);
    const RowScale scale = row_scale(m);
    const T *x = (const T *)p.x + mine * p.ld_x;
    i32x4 acc{};
    for (int32_t u = wave; u < units; u += kUnits * kOnceWaves) {
        i32x4 now[kUnits][2], fx[kUnits][2];
#pragma unroll
        for (int n = 0; n < kUnits; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                now[n][k] = next[n][k];
                const int64_t col = (int64_t)(u + n * kOnceWaves) * 128 + k * 64 + fk;
                float v[16];
                E::floats(load8<DT, WIDE>(x, col, p.cols), v);
                E::floats(load8<DT, WIDE>(x, col + 8, p.cols), v + 8);
                const uint2 lo = quantized8(v, scale), hi = quantized8(v + 8, scale);
                fx[n][k] = i32x4{(int32_t)lo.x, (int32_t)lo.y, (int32_t)hi.x, (int32_t)hi.y};
            }
        request(u + kUnits * kOnceWaves);
#pragma unroll
        for (int n = 0; n < kUnits; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[n][k], fx[n][k], acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    const int o = threadIdx.x & 15, t = threadIdx.x >> 4;
    if (t >= rows || o0 + o >= p.outs) return;
    int32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kOnceWaves; ++k) sum += sums[k][(o >> 2) * 16 + t][o & 3];
    m = 0;
    for (int i = 0; i < each; ++i) m = max(m, part[t][i]);
    float v = (float)sum * (row_scale(m).scale * p.ws[o0 + o]);
    if (p.bias) v += param(p.bias, p.bias_dtype, o0 + o);
    put_param(p.y, p.dtype, t * p.ld_y + o0 + o, v);
}

static bool once(const LinearArgs &p)
{
    return p.x && p.rows <= kOnceRows && p.rows * p.cols * (int64_t)elem_size(p.dtype) <= kOnceBytes;
}

template <int DT, bool WIDE>
static hipError_t launch_once(const LinearArgs &p, hipStream_t s)
{
    hipLaunchKernelGGL((linear_once_kernel<DT, WIDE>), dim3((unsigned)((p.outs + 15) / 16)), dim3(kOnceWaves * 64), 0, s, p);
    return hipGetLastError();
}

// Into how many parts along k the work of `blocks` workgroups is cut, at most `most`, where `room` workgroups run at a time: rounds times the length of a
// part, an eighth of the whole added for what each part costs by itself.
static int32_t parts_along_k(int64_t blocks, int64_t most, int64_t room)
{
    int32_t best = 1;
    float least = 1e30f;
    for (int32_t n = 1; n <= 16 && n <= most; ++n) {
        const float cost = (float)((blocks * n + room - 1) / room) * (1.0f / (float)n + 0.125f);
        if (cost < least) { least = cost; best = n; }
    }
    return best;
}

constexpr int64_t kFewRows = 64;
// FB: x at most half of the weights' bytes, up to 32 rows; with few outputs a workgroup for each 16 (x then is read few times, and the chip is idle)
static int32_t few_blocks_of(int64_t rows, int64_t outs) { return rows <= 8 || outs <= 2048 ? 1 : rows <= 16 ? 2 : 4; }
static int32_t few_splits(int64_t rows, int64_t cols, int64_t outs)
{
    const int64_t each = 16 * few_blocks_of(rows, outs), blocks = (outs + each - 1) / each, units = (cols + 127) / 128;
    return parts_along_k(blocks, units / kFewWaves, 256);                   // a unit for each wave at least
}

static ProductPlan forward_plan(int64_t rows, int64_t cols, int64_t outs)
{
    if (rows <= kFewRows) return {0, {few_splits(rows, cols, outs), 1}};
    const ProductShape shape{(int32_t)outs, (int32_t)rows, (int32_t)(rows8_stride(cols) / 128)};
    return plan_products(&shape, 1);
}
size_t linear_q8_workspace(int32_t from_floats, int64_t rows, int64_t cols, int64_t outs)
{
    return (from_floats ? (size_t)rows * rows8_stride(cols) + ((size_t)rows * 4 + 255) / 256 * 256 : 0) +
           product_parts_bytes(forward_plan(rows, cols, outs).splits[0], (int32_t)outs, (int32_t)rows);
}

hipError_t launch_linear_q8(const LinearArgs &p, hipStream_t s)
{
    if (once(p)) return BY_TYPE(p.dtype, wide_rows(p.x, p.dtype, p.ld_x, p.cols), launch_once, p, s);
    const int8_t *xq = p.xq;
    const float *xs = p.xs;
    int64_t ld_xq = p.ld_xq;
    char *room = (char *)p.workspace;
    if (p.x) {
        ld_xq = rows8_stride(p.cols);
        float *scale = (float *)room;
        room += ((size_t)p.rows * 4 + 255) / 256 * 256;
        QuantizeArgs q{};
        q.dtype = p.dtype; q.rows = p.rows; q.cols = p.cols; q.x = p.x; q.ld_x = p.ld_x; q.q = (int8_t *)room; q.ld_q = ld_xq; q.scale = scale;
        if (const hipError_t e = launch_quantize_rows(q, s); e != hipSuccess) return e;
        xq = (const int8_t *)room;
        xs = scale;
        room += (size_t)p.rows * ld_xq;
    }
    ProductArgs a{};
    a.p = (const char *)p.w; a.ld_p = p.ld_w;
    a.q = (const char *)xq; a.ld_q = ld_xq;
    a.R = (int32_t)p.outs; a.C = (int32_t)p.rows;
    a.steps = a.p_steps = (int32_t)(rows8_stride(p.cols) / 128);
    a.out = p.y; a.ld_out = p.ld_y; a.dtype = p.dtype;
    a.p_scale = p.ws; a.q_scale = xs; a.bias = p.bias; a.bias_dtype = p.bias_dtype;
    a.parts = room;
    const ProductPlan plan = forward_plan(p.rows, p.cols, p.outs);
    a.splits = plan.splits[0];
    if (p.rows > kFewRows) return launch_product_i8(a, plan.tile, s);
    const int32_t fb = few_blocks_of(p.rows, p.outs), outs = 16 * fb;
    const dim3 grid((unsigned)((p.outs + outs - 1) / outs * a.splits)), block(kFewWaves * 64);
    const auto kernel = p.rows <= 16   ? (fb == 1 ? linear_few_kernel<1, 1> : linear_few_kernel<1, 2>)
                        : p.rows <= 32 ? (fb == 1 ? linear_few_kernel<2, 1> : linear_few_kernel<2, 4>)
                                       : (fb == 1 ? linear_few_kernel<4, 1> : linear_few_kernel<4, 4>);
    hipLaunchKernelGGL(kernel, grid, block, 0, s, p, xq, ld_xq, xs, a.splits, (int32_t *)room);
    return a.splits > 1 ? launch_product_join_i8(a, s) : hipGetLastError();
}

// dy times a scale in PIECES bf16 values that add up to it: all but the last cut off, which leaves the rest exact, the last rounded.  An infinity
// leaves NaN, for which the median of three takes the smallest number, zero: the other pieces then are zeros, and their products add nothing to the
// infinity's.
template <int PIECES>
__device__ __forceinline__ void cut(float v, uint16_t *piece)
{
#pragma unroll
    for (int k = 0; k < PIECES - 1; ++k) {
        const uint32_t high = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
        piece[k] = (uint16_t)(high >> 16);
        v -= __builtin_bit_cast(float, high);
        v = __builtin_amdgcn_fmed3f(v, v, 0.0f);
    }
    const __bf16 last = (__bf16)v;
    piece[PIECES - 1] = __builtin_bit_cast(uint16_t, last);
}
__device__ __forceinline__ int32_t pair(uint16_t lo, uint16_t hi) { return lo | (int32_t)((uint32_t)hi << 16); }

// Byte `b` of eight words as eight bf16 values (exact: eight bits).
__device__ __forceinline__ i32x4 bytes_bf16(const int32_t *w, int b)
{
    uint32_t f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(uint32_t, (float)((w[e] << (24 - 8 * b)) >> 24));
    i32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (int32_t)__builtin_amdgcn_perm(f[2 * e + 1], f[2 * e], 0x07060302);
    return r;
}
__device__ __forceinline__ f32x4 mma_bf16(i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
static int pieces_of(int32_t dtype) { return dtype == TICTAC_F32 ? 3 : dtype == TICTAC_F16 ? 2 : 1; }
template <int DT>
struct Pieces { static constexpr int value = DT == TICTAC_F32 ? 3 : DT == TICTAC_F16 ? 2 : 1; };

// ---- backward with few rows: bound by the weights read for dx, and by dw written ----
// dx: the weights have k (the outputs o) as rows, and the matrix instruction wants eight of k per lane.  A lane reads 4 ND bytes of each of eight
// rows and turns this block of 8 x 4 ND round in registers: byte j of the eight words is an operand whose row r is the column
// i = 4 ND r + j of the block, so 4 ND instructions take what one round of loads brought.  The result has, per lane, 4 ND columns next to each
// other.  A workgroup has 64 ND columns and a part of k, its eight waves blocks of 32 of k in turn; their sums meet in LDS, in fixed order.
// 32 rows, 4096 x 25088 float16: 30 us by itself, 39 in turn with dw, whose 205 MB are still on their way out of the caches.
constexpr int kBackWaves = 8;

// what eight of k bring for dx besides the weights: dy of TB blocks of 16 rows, and the weights' scales
template <int DT, bool WIDE, int TB>
struct GradientRows {
    using E = Elem<DT>;
    typename E::raw dy[TB];
    Elem<TICTAC_F32>::raw scale;
    __device__ __forceinline__ void load(const LinearArgs &p, int64_t row, int64_t o)
    {
#pragma unroll
        for (int b = 0; b < TB; ++b)
            dy[b] = load8_or_last<DT, WIDE>((const typename E::type *)p.dy + min(b * 16 + row, p.rows - 1) * p.ld_dy, o, p.outs);
        scale = load8_or_last<TICTAC_F32, WIDE>(p.ws, o, p.outs);
    }
    template <int PIECES>
    __device__ __forceinline__ void operands(int64_t o, int64_t outs, i32x4 (&q)[TB][PIECES]) const
    {
        float s[8];
        Elem<TICTAC_F32>::floats(scale, s);
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            float v[8];
            uint16_t cuts[8][PIECES];
            E::floats(dy[b], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= s[e];
            if (o + 8 > outs)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = o + e < outs ? v[e] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) cut<PIECES>(v[e], cuts[e]);
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) q[b][k][e] = pair(cuts[2 * e][k], cuts[2 * e + 1][k]);
        }
    }
};

template <int DT, bool WIDE, int TB, int ND>
__global__ __launch_bounds__(kBackWaves * 64) void linear_dx_few_kernel(LinearArgs p, int32_t splits, float *parts)
{
    using T = typename Elem<DT>::type;
    constexpr int PIECES = Pieces<DT>::value, NJ = 4 * ND;
    extern __shared__ float room[];                             // [waves][NJ][64 lanes][4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int64_t blocks = gridDim.x / splits, i0 = blockIdx.x % blocks * (16 * NJ), padded = (p.cols + 127) / 128 * 128;
    const int32_t split = (int32_t)(blockIdx.x / blocks), all = (int32_t)((p.outs + 31) / 32);
    const int32_t first = (int32_t)((int64_t)all * split / splits), last = (int32_t)((int64_t)all * (split + 1) / splits);
    // rows g * 8 .. + 7 of a block of 32 of the weights, the same for all blocks (columns behind the end: any will do)
    const uint32_t at = (uint32_t)(g * 8) * (uint32_t)p.ld_w + (uint32_t)(i0 + c * NJ < padded ? i0 + c * NJ : 0);
    typedef int32_t Words __attribute__((ext_vector_type(ND)));
    Words now[8], next[8];
    GradientRows<DT, WIDE, TB> dy;
    const auto request = [&](int32_t kb) {
        const int8_t *block = p.w + (int64_t)kb * 32 * p.ld_w;
        if ((int64_t)kb * 32 + 32 <= p.outs) {
#pragma unroll
            for (int e = 0; e < 8; ++e) next[e] = *(const Words *)(block + e * p.ld_w + at);
        } else {                                                // the last block: its last row again
            const int32_t rows = (int32_t)(p.outs - (int64_t)kb * 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) next[e] = *(const Words *)(block + (at - (uint32_t)(g * 8) * (uint32_t)p.ld_w) + min(g * 8 + e, rows - 1) * p.ld_w);
        }
        dy.load(p, c, (int64_t)kb * 32 + g * 8);
    };
    f32x4 acc[NJ][TB] = {};
    // Each workgroup starts at another block: rows of dy often lie a power of two apart, and what all ask for at a time would be in few channels.
    const int32_t count = last - first, turn = count ? blockIdx.x * 5 % count : 0;
    const auto block_of = [&](int32_t n) { return first + (n + turn < count ? n + turn : n + turn - count); };
    if (wave < count) request(block_of(wave));
    for (int32_t n = wave; n < count; n += kBackWaves) {
        i32x4 q[TB][PIECES];
        dy.template operands<PIECES>((int64_t)block_of(n) * 32 + g * 8, p.outs, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) now[e] = next[e];
        if (n + kBackWaves < count) request(block_of(n + kBackWaves));
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            int32_t words[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) words[e] = now[e][j >> 2];
            const i32x4 f = bytes_bf16(words, j & 3);
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int k = 0; k < PIECES; ++k) acc[j][b] = mma_bf16(f, q[b][k], acc[j][b]);
        }
    }
    // A thread adds up eight columns of one row over the waves, in their order: element e of lane l, halves of the NJ operands by threads.
    constexpr int kParts = NJ / 8, kThreads = 256 * kParts;
    const int le = threadIdx.x & 255, part = threadIdx.x >> 8, from = le >> 2;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        if (b) __syncthreads();
#pragma unroll
        for (int j = 0; j < NJ; ++j) *(f32x4 *)(room + ((wave * NJ + j) * 64 + lane) * 4) = acc[j][b];
        __syncthreads();
        const int64_t t = b * 16 + (from & 15), i = i0 + NJ * (4 * (from >> 4) + (le & 3)) + part * 8;
        if ((int)threadIdx.x >= kThreads || t >= p.rows) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0.0f;
#pragma unroll
            for (int k = 0; k < kBackWaves; ++k) v[j] += room[(k * NJ + part * 8 + j) * 256 + le];
        }
        if (splits > 1) {
            float *to = parts + ((int64_t)split * p.rows + t) * p.cols;
            if (p.cols % 8 == 0) store8<TICTAC_F32, true>(to, i, p.cols, v);
            else store8<TICTAC_F32, false>(to, i, p.cols, v);
        } else {
            store8<DT, WIDE>((T *)p.dx + t * p.ld_dx, i, p.cols, v);
        }
    }
}

// dw: all of k (the rows t, up to 32 KB) is at hand.  The activations are turned round in registers as the weights above, four bytes per lane, and stay
// there; the pieces of dy times scale lie in LDS.  A workgroup has 64 outputs and 512 columns, a wave 64 columns.  db rides along with the first columns, and
// is all there is where dw is not asked for: xq and xs may be NULL then.
// 32 rows, 4096 x 25088 float16: 47 us, 4.4 TB/s; with stores past the caches 64.
template <int DT, bool WIDE, int KB>
__global__ __launch_bounds__(512) void linear_dw_few_kernel(LinearArgs p)
{
    using E = Elem<DT>;
    using T = typename E::type;
    constexpr int PIECES = Pieces<DT>::value, kOuts = 64, kStride = KB * 32 * PIECES + 8;       // (sixteen bytes more: rows start in other banks)
    __shared__ __align__(16) uint16_t q[kOuts * kStride];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int64_t o0 = (int64_t)blockIdx.y * kOuts, i0 = (int64_t)blockIdx.x * 512 + wave * 64;
    const int o = threadIdx.x & 63;
    for (int t = threadIdx.x >> 6; t < (p.dw ? KB * 32 : 0); t += 8) {
        uint16_t cuts[PIECES];
        cut<PIECES>(t < p.rows && o0 + o < p.outs ? E::to_float(((const T *)p.dy)[t * p.ld_dy + o0 + o]) * p.xs[t] : 0.0f, cuts);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) q[o * kStride + k * KB * 32 + t] = cuts[k];
    }
    if (p.db && blockIdx.x == 0 && threadIdx.x < kOuts && o0 + o < p.outs) {
        float sum = 0.0f;
        for (int64_t t = 0; t < p.rows; ++t) sum += E::to_float(((const T *)p.dy)[t * p.ld_dy + o0 + o]);
        ((T *)p.db)[o0 + o] = E::from_float(sum);
    }
    __syncthreads();
    if (!p.dw || i0 >= p.cols) return;
    // row r of an operand is the column at(r) + j: a lane's results (rows 4 g + e) then are eight next to each other at 8 g, and eight at 32 + 8 g, and
    // four lanes store 64 bytes in a row
    const int64_t column = i0 + ((c & 2) << 4) + ((c >> 2) << 3) + ((c & 1) << 2);
    i32x4 f[KB][4];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        int32_t words[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) words[e] = *(const int32_t *)(p.xq + min((int64_t)b * 32 + g * 8 + e, p.rows - 1) * p.ld_xq + column);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[b][j] = bytes_bf16(words, j);
    }
#pragma unroll
    for (int block = 0; block < kOuts / 16; ++block) {
        f32x4 acc[4] = {};
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const i32x4 fq = *(const i32x4 *)(q + (block * 16 + c) * kStride + k * KB * 32 + b * 32 + g * 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = mma_bf16(f[b][j], fq, acc[j]);
            }
        const int64_t out = o0 + block * 16 + c;
        if (out >= p.outs) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] = acc[n & 3][h * 2 + (n >> 2)];
            store8<DT, WIDE>((T *)p.dw + out * p.ld_dw, i0 + h * 32 + g * 8, p.cols, v);
        }
    }
}

static int32_t dx_few_words(int64_t rows) { return rows <= 32 ? 4 : 2; }
static int32_t dx_few_splits(int64_t rows, int64_t cols, int64_t outs)
{
    const int64_t wide = 64 * dx_few_words(rows), blocks = (cols + wide - 1) / wide, units = (outs + 31) / 32;
    return parts_along_k(blocks, units / kBackWaves, 256);                  // a block of k for each wave at least
}

// ---- backward with more rows: operands with k contiguous, for the tiles of k8_product.hip ----
// A wave turns 64 rows of 128 bytes round in registers: lane l has eight rows, 8 (l % 8) .. + 7, and sixteen bytes of each, 16 (l / 8) ..; it stores for
// each column eight values next to each other, and eight lanes store 128 bytes.  Reads and writes are whole lines, and nothing goes through LDS.
// Bound by memory: 8192 x 4096 -> 4096 bfloat16 50 us, 272 MB at 5.4 TB/s.
//   weights, activations: int8 -> bf16, out[c][r] = q[r][c], times the scale of row r where dy is bf16 (SCALED: rounded once; dy then is an
//   operand as it is)
//   dy: out[o][piece][t] = pieces of dy[t][o] xs[t] and out[t][piece][o] = pieces of dy[t][o] ws[o]; where dy is bf16, dy[t][o] itself (and the second only
//   if its rows are no operands as they are); sums of dy over each 64 rows
template <bool SCALED>
__device__ __forceinline__ void turn_rows8(int64_t rows, int64_t cols, const int8_t *q, int64_t ld, const float *scale, uint16_t *out, int64_t padded, int64_t r0, int64_t c0)
{
    const int lane = threadIdx.x & 63;
    const int64_t r = r0 + (lane & 7) * 8, c = c0 + (lane >> 3) * 16;
    i32x4 w[8];
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = *(const i32x4 *)(q + min(r + e, rows - 1) * ld + c);          // (c + 16 <= ld: rows are padded to 128)
        s[e] = r + e < rows ? (SCALED ? scale[min(r + e, rows - 1)] : 1.0f) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        int32_t words[8];
        i32x4 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) words[e] = w[e][j >> 2];
        if (SCALED) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = r + e < rows ? (float)((words[e] << (24 - 8 * (j & 3))) >> 24) * s[e] : 0.0f;
            v = __builtin_bit_cast(i32x4, Elem<TICTAC_BF16>::pack(f));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) words[e] = r + e < rows ? words[e] : 0;
            v = bytes_bf16(words, j & 3);
        }
        if (c + j < cols) *(i32x4 *)(out + (c + j) * padded + r) = v;
    }
}

struct Operands {
    int64_t units[4];                   // waves: up to here weights, activations, rows of dy, columns of dy
    uint16_t *p_x, *p_w, *q_x, *q_w;    // NULL: not needed
    float *sums;                        // [rows / 64][outs], may be NULL
    int64_t padded_o, padded_t;
};

// half of what load8 brings
template <int DT, bool WIDE>
__device__ __forceinline__ void load_half(const typename Elem<DT>::type *row, int64_t col, int64_t cols, float *v)
{
    typename Elem<DT>::type r[4];
    if (WIDE ? col < cols : col + 4 <= cols) {
        __builtin_memcpy(r, row + col, sizeof(r));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = Elem<DT>::to_float(r[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = Elem<DT>::to_float(row[min(col + i, cols - 1)]);
        v[i] = col + i < cols ? x : 0.0f;
    }
}

// N: rows, or columns, of dy that a lane cuts to pieces.  Eight are whole lines for 16-bit types; with float32, and with float16 where there are less than four
// waves per compute unit, four are better: a chain of a thousand instructions is cut in half (101 x 777 -> 1001 float32: 22.0 us, 19.4; 300 x 153 -> 587
// float16: 18.6, 16.1; but 4096 x 4096 -> 4096: 388.8, 393.3).
template <int DT, bool WIDE, int N>
__global__ __launch_bounds__(256) void linear_operands_kernel(LinearArgs p, Operands to)
{
    using E = Elem<DT>;
    using T = typename E::type;
    constexpr int PIECES = Pieces<DT>::value;
    const int lane = threadIdx.x & 63;
    int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t wide = (p.cols + 127) / 128;
    if (unit < to.units[0]) {
        turn_rows8<PIECES == 1>(p.outs, p.cols, p.w, p.ld_w, p.ws, to.p_x, to.padded_o, unit / wide * 64, unit % wide * 128);
        return;
    }
    if (unit < to.units[1]) {
        unit -= to.units[0];
        turn_rows8<PIECES == 1>(p.rows, p.cols, p.xq, p.ld_xq, p.xs, to.p_w, to.padded_t, unit / wide * 64, unit % wide * 128);
        return;
    }
    if (unit >= to.units[3]) return;
    // rows and columns of dy by waves of their own
    const bool rows_only = unit < to.units[2];
    unit -= rows_only ? to.units[1] : to.units[2];
    const int part = (int)(unit % (8 / N)) * N;
    unit /= 8 / N;
    const int64_t tiles = (p.outs + 63) / 64, t0 = unit / tiles * 64, t = t0 + (lane & 7) * 8 + (rows_only ? part : 0), o = unit % tiles * 64 + (lane >> 3) * 8 + (rows_only ? 0 : part);
    if (rows_only) {
        float v[N][8], s[8];
#pragma unroll
        for (int e = 0; e < N; ++e) E::floats(load8<DT, WIDE>((const T *)p.dy + min(t + e, p.rows - 1) * p.ld_dy, o, p.outs), v[e]);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = PIECES > 1 && o + i < p.outs ? p.ws[o + i] : 1.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            uint16_t cuts[8][PIECES];
#pragma unroll
            for (int i = 0; i < 8; ++i) cut<PIECES>(PIECES > 1 ? v[e][i] * s[i] : v[e][i], cuts[i]);
            if (t + e >= p.rows) continue;
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
                *(i32x4 *)(to.q_x + ((t + e) * PIECES + k) * to.padded_o + o) = i32x4{pair(cuts[0][k], cuts[1][k]), pair(cuts[2][k], cuts[3][k]), pair(cuts[4][k], cuts[5][k]), pair(cuts[6][k], cuts[7][k])};
        }
        return;
    }
    float v[8][N], s[8];                                        // [row][column]
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const T *const row = (const T *)p.dy + min(t + e, p.rows - 1) * p.ld_dy;
        if constexpr (N == 8) E::floats(load8<DT, WIDE>(row, o, p.outs), v[e]);
        else load_half<DT, WIDE>(row, o, p.outs, v[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] = PIECES > 1 && to.q_w ? p.xs[min(t + e, p.rows - 1)] : 1.0f;      // (without dw there may be no xs)
#pragma unroll
        for (int i = 0; i < N; ++i) v[e][i] = t + e < p.rows ? v[e][i] : 0.0f;
    }
    if (to.sums) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[e][i];
#pragma unroll
            for (int k = 1; k < 8; k <<= 1) sum += __shfl_xor(sum, k);
            if ((lane & 7) == 0 && o + i < p.outs) to.sums[t0 / 64 * p.outs + o + i] = sum;
        }
    }
    if (!to.q_w) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint16_t cuts[8][PIECES];
#pragma unroll
        for (int e = 0; e < 8; ++e) cut<PIECES>(PIECES > 1 ? (t + e < p.rows ? v[e][i] * s[e] : 0.0f) : v[e][i], cuts[e]);
        if (o + i >= p.outs) continue;
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
            *(i32x4 *)(to.q_w + ((o + i) * PIECES + k) * to.padded_t + t) = i32x4{pair(cuts[0][k], cuts[1][k]), pair(cuts[2][k], cuts[3][k]), pair(cuts[4][k], cuts[5][k]), pair(cuts[6][k], cuts[7][k])};
    }
}

// The workspace of one backward call.
struct BackwardRoom {
    int64_t padded_o, padded_t;
    ProductPlan plan;                                       // dx, dw
    size_t sums, p_x, p_w, q_x, q_w, parts_x, parts_w, bytes;           // offsets
};
static BackwardRoom backward_room(int32_t dtype, int64_t rows, int64_t cols, int64_t outs)
{
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const int pieces = pieces_of(dtype);
    BackwardRoom r{};
    if (rows <= kFewRows) {
        r.bytes = up(product_parts_bytes(dx_few_splits(rows, cols, outs), (int32_t)cols, (int32_t)rows));
        return r;
    }
    r.padded_o = (outs + 63) / 64 * 64;
    r.padded_t = (rows + 63) / 64 * 64;
    const ProductShape shapes[2] = {{(int32_t)cols, (int32_t)rows, (int32_t)(r.padded_o / 64 * pieces)}, {(int32_t)cols, (int32_t)outs, (int32_t)(r.padded_t / 64 * pieces)}};
    r.plan = plan_products(shapes, 2);
    r.p_x = r.sums + up((size_t)(r.padded_t / 64) * outs * 4);
    r.p_w = r.p_x + up((size_t)cols * r.padded_o * 2);
    r.q_x = r.p_w + up((size_t)cols * r.padded_t * 2);
    r.q_w = r.q_x + up((size_t)rows * r.padded_o * pieces * 2);
    r.parts_x = r.q_w + up((size_t)outs * r.padded_t * pieces * 2);
    r.parts_w = r.parts_x + up(product_parts_bytes(r.plan.splits[0], (int32_t)cols, (int32_t)rows));
    r.bytes = r.parts_w + up(product_parts_bytes(r.plan.splits[1], (int32_t)cols, (int32_t)outs));
    return r;
}
size_t linear_q8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs) { return backward_room(dtype, rows, cols, outs).bytes; }

template <int DT, bool WIDE>
static hipError_t backward_few(const LinearArgs &p, hipStream_t s)
{
    if (p.dx && p.rows) {
        const int32_t splits = dx_few_splits(p.rows, p.cols, p.outs), wide = 64 * dx_few_words(p.rows);
        const auto kernel = p.rows <= 16 ? linear_dx_few_kernel<DT, WIDE, 1, 4> : p.rows <= 32 ? linear_dx_few_kernel<DT, WIDE, 2, 4> : linear_dx_few_kernel<DT, WIDE, 4, 2>;
        const size_t lds = (size_t)kBackWaves * wide * 64;
        if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.cols + wide - 1) / wide * splits)), dim3(kBackWaves * 64), lds, s, p, splits, (float *)p.workspace);
        if (splits > 1) {
            ProductArgs a{};
            a.R = (int32_t)p.cols; a.C = (int32_t)p.rows; a.splits = splits; a.out = p.dx; a.ld_out = p.ld_dx; a.dtype = DT; a.parts = p.workspace;
            if (const hipError_t e = launch_product_join_bf16(a, s); e != hipSuccess) return e;
        }
    }
    if ((p.dw || p.db) && p.outs) {
        const dim3 grid((unsigned)(p.dw ? (p.cols + 511) / 512 : 1), (unsigned)((p.outs + 63) / 64));
        const auto kernel = p.rows <= 32 ? linear_dw_few_kernel<DT, WIDE, 1> : linear_dw_few_kernel<DT, WIDE, 2>;
        hipLaunchKernelGGL(kernel, grid, dim3(512), 0, s, p);
    }
    return hipGetLastError();
}

template <int DT, bool WIDE>
static hipError_t backward(const LinearArgs &p, hipStream_t s)
{
    constexpr int PIECES = Pieces<DT>::value;
    const BackwardRoom room = backward_room(DT, p.rows, p.cols, p.outs);
    char *at = (char *)p.workspace;
    // rows of bf16 that are whole steps of 128 bytes are operands as they are
    const bool as_is = PIECES == 1 && WIDE && p.outs % 64 == 0 && p.ld_dy * 2 <= 1 << 24;         // (offsets inside a tile are 32 bits)
    Operands to{};
    to.padded_o = room.padded_o;
    to.padded_t = room.padded_t;
    if (p.dx) to.p_x = (uint16_t *)(at + room.p_x);
    if (p.dw) to.p_w = (uint16_t *)(at + room.p_w);
    if (p.dx && !as_is) to.q_x = (uint16_t *)(at + room.q_x);
    if (p.dw) to.q_w = (uint16_t *)(at + room.q_w);
    if (p.db) to.sums = (float *)(at + room.sums);
    to.units[0] = p.dx ? (p.cols + 127) / 128 * (room.padded_o / 64) : 0;
    to.units[1] = to.units[0] + (p.dw ? (p.cols + 127) / 128 * (room.padded_t / 64) : 0);
    int64_t tiles = (p.outs + 63) / 64 * (room.padded_t / 64);
    const bool halves = PIECES == 3 || (PIECES == 2 && tiles <= 512);
    if (halves) tiles *= 2;
    to.units[2] = to.units[1] + (to.q_x ? tiles : 0);
    to.units[3] = to.units[2] + (to.q_w || to.sums ? tiles : 0);
    if (to.units[3]) {
        const auto kernel = PIECES == 3 || halves ? linear_operands_kernel<DT, WIDE, PIECES == 1 ? 8 : 4> : linear_operands_kernel<DT, WIDE, PIECES == 3 ? 4 : 8>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((to.units[3] + 3) / 4)), dim3(256), 0, s, p, to);
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    ProductArgs a[2] = {};
    int n = 0;
    if (p.dx) {
        ProductArgs &x = a[n++];
        x.p = at + room.p_x;
        x.ld_p = room.padded_o * 2;
        x.q = as_is ? (const char *)p.dy : at + room.q_x;
        x.ld_q = as_is ? p.ld_dy * 2 : room.padded_o * 2 * PIECES;
        x.R = (int32_t)p.cols;
        x.C = (int32_t)p.rows;
        x.p_steps = (int32_t)(room.padded_o / 64);
        x.splits = room.plan.splits[0];
        x.out = p.dx;
        x.ld_out = p.ld_dx;
        x.parts = at + room.parts_x;
    }
    if (p.dw) {
        ProductArgs &w = a[n++];
        w.p = at + room.p_w;
        w.ld_p = room.padded_t * 2;
        w.q = at + room.q_w;
        w.ld_q = room.padded_t * 2 * PIECES;
        w.R = (int32_t)p.cols;
        w.C = (int32_t)p.outs;
        w.p_steps = (int32_t)(room.padded_t / 64);
        w.splits = room.plan.splits[1];
        w.out = p.dw;
        w.ld_out = p.ld_dw;
        w.parts = at + room.parts_w;
    }
    for (int i = 0; i < n; ++i) {
        a[i].steps = a[i].p_steps * PIECES;
        a[i].dtype = DT;
    }
    const ColumnSums c{(const float *)(at + room.sums), room.padded_t / 64, p.outs, p.db, DT};
    return launch_products_bf16(a, n, room.plan.tile, c, s);
}

// No rows, or no outputs: what there is of the gradients is zero.
static hipError_t backward_nothing(const LinearArgs &p, hipStream_t s)
{
    ProductArgs a{};
    a.splits = 1;
    a.R = (int32_t)p.cols;
    a.dtype = p.dtype;
    a.C = (int32_t)(p.rows ? p.rows : p.outs);
    a.out = p.rows ? p.dx : p.dw;
    a.ld_out = p.rows ? p.ld_dx : p.ld_dw;
    const ColumnSums c{nullptr, 0, p.outs, p.outs ? p.db : nullptr, p.dtype};
    return launch_products_bf16(&a, a.out && a.C ? 1 : 0, 0, c, s);
}

hipError_t launch_linear_q8_backward(const LinearArgs &p, hipStream_t s)
{
    if (p.rows == 0 || p.outs == 0) return backward_nothing(p, s);
    const bool few = p.rows <= kFewRows, wide = wide_rows(p.dy, p.dtype, p.ld_dy, p.outs);
    if (!few) return BY_TYPE(p.dtype, wide, backward, p, s);
    const bool all = wide && ((uintptr_t)p.ws & 15) == 0 && (!p.dx || wide_rows(p.dx, p.dtype, p.ld_dx, p.cols)) && (!p.dw || wide_rows(p.dw, p.dtype, p.ld_dw, p.cols));
    return BY_TYPE(p.dtype, all, backward_few, p, s);
}

}  // namespace tictac
