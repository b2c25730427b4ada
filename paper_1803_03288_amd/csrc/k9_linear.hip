// A layer with weights in 8-bit floats, y[t][o] = sum_i x[t][i] w[o][i] + bias[o], and its gradients
//   dx[t][i] = sum_o dy'[t][o] w'[o][i],   dw[o][i] = sum_t dy"[t][o] x"[t][i],   db[o] = sum_t dy[t][o]
// dy' is dy in blocks of 128 outputs, dy" and x" are dy and x in blocks of 128 rows, w' is w in blocks of 128 outputs: an operand's blocks lie along what is summed over.
// Outputs of 16 bits come from the matrix instructions for 8-bit floats (k9_product.hip says what those cut off); float32 ones from those for bf16, in which the
// operands' values are exact, with sums in float32.
#include <algorithm>

#include "device_utils.h"
#include "k8_tiles.h"
#include "k9_product.h"

namespace tictac {

__device__ __forceinline__ f32x4 mma_bf16(i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// ---- few rows: bound by the bytes of the weights ----
// A workgroup has 16 FB outputs and a part of k, its eight waves blocks of 128 of that in turn: weights go from memory to the matrix instruction without LDS, 32 bytes per lane, the next
// block under way while one is computed.  TB blocks of 16 rows of x come from the caches.  The sums of the waves meet in LDS, those of several workgroups along k in the
// workspace.  EXACT: bf16 instructions.  A lane's 32 bytes of a block lie next to each other: the order of k is free, where both operands have it.
// x is asked for together with the weights (float32 outputs, 16 x 16384 -> 16384: 64.5 us, 4.2 TB/s; without that 68.8), but where its bf16 values leave no registers for that
// (64 x 25088 -> 4096: 43 us, with it 70).
constexpr int kFewWaves = 8;

// sixteen 8-bit floats times a power of two as operands of two bf16 instructions
__device__ __forceinline__ void widen(i32x4 q, float s, int format, i32x4 (&to)[2])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float v[8];
        f8_values4((uint32_t)q[2 * h], format, v);
        f8_values4((uint32_t)q[2 * h + 1], format, v + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s;
        to[h] = f8_bf16(v);
    }
}

template <bool EXACT, int QF, int TB, int FB>
__global__ __launch_bounds__(kFewWaves * 64) void linear_f8_few_kernel(LinearF8Args p, F8Rows xq, int32_t splits, float *parts)
{
    constexpr bool kAhead = !(EXACT && TB == 4);
    __shared__ f32x4 sums[kFewWaves][TB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, fk = (lane >> 4) * 32;
    const int64_t blocks = gridDim.x / splits, o0 = blockIdx.x % blocks * (16 * FB);
    const int32_t split = (int32_t)(blockIdx.x / blocks), all = (int32_t)((p.cols + 127) / 128);
    const int32_t first = (int32_t)((int64_t)all * split / splits), units = (int32_t)((int64_t)all * (split + 1) / splits);
    const uint8_t *w[FB], *x[TB], *we[FB], *xe[TB];
#pragma unroll
    for (int f = 0; f < FB; ++f) {
        const int64_t o = min(o0 + f * 16 + row, p.outs - 1);
        w[f] = p.w.q + o * p.w.ld + fk;
        we[f] = p.w.scale + (o >> p.w.shift) * p.w.ld_scale;
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int64_t t = min((int64_t)b * 16 + row, p.rows - 1);
        x[b] = xq.q + t * xq.ld + fk;
        xe[b] = xq.scale + (t >> xq.shift) * xq.ld_scale;
    }
    struct Operands {
        i32x4 q[FB][2], x[TB][2];
        int e[FB], ex[TB];
    } now, next;
    f32x4 acc[FB][TB] = {};
    const auto request_x = [&](int32_t u) {
#pragma unroll
        for (int b = 0; b < TB; ++b) {
#pragma unroll
            for (int k = 0; k < 2; ++k) next.x[b][k] = *(const i32x4 *)(x[b] + (int64_t)u * 128 + k * 16);
            next.ex[b] = xe[b][u];
        }
    };
    const auto request = [&](int32_t u) {
#pragma unroll
        for (int f = 0; f < FB; ++f) {
#pragma unroll
            for (int k = 0; k < 2; ++k) next.q[f][k] = *(const i32x4 *)(w[f] + (int64_t)u * 128 + k * 16);
            next.e[f] = we[f][u];
        }
        if (kAhead) request_x(u);
    };
    if (first + wave < units) request(first + wave);
    for (int32_t u = first + wave; u < units; u += kFewWaves) {
        if (!kAhead) request_x(u);
        now = next;
        if (u + kFewWaves < units) request(u + kFewWaves);
        if constexpr (EXACT) {
            i32x4 wide_x[TB][2][2];
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int k = 0; k < 2; ++k) widen(now.x[b][k], f8_factor(now.ex[b]), QF, wide_x[b][k]);
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    i32x4 wide_w[2];
                    widen(now.q[f][k], f8_factor(now.e[f]), TICTAC_E4M3, wide_w);
#pragma unroll
                    for (int b = 0; b < TB; ++b)
#pragma unroll
                        for (int h = 0; h < 2; ++h) acc[f][b] = mma_bf16(wide_w[h], wide_x[b][k][h], acc[f][b]);
                }
        } else {
            const auto whole = [](const i32x4 (&v)[2]) { return i32x8{v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]}; };
#pragma unroll
            for (int f = 0; f < FB; ++f)
#pragma unroll
                for (int b = 0; b < TB; ++b)
                    acc[f][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(now.q[f]), whole(now.x[b]), acc[f][b], TICTAC_E4M3, QF, 0, now.e[f], 0, now.ex[b]);
        }
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
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kFewWaves; ++k) sum += sums[k][b][(o >> 2) * 16 + t][o & 3];
            const int64_t at = (int64_t)b * 16 + t, out = o0 + f * 16 + o;
            if (at >= p.rows || out >= p.outs) continue;
            if (splits > 1) {
                parts[((int64_t)split * p.rows + at) * p.outs + out] = sum;
                continue;
            }
            if (p.bias) sum += param(p.bias, p.bias_dtype, out);
            put_param(p.y, p.dtype, at * p.ld_y + out, sum);
        }
    }
}

// Up to sixteen rows of floats, rounded to 8 bits here: every workgroup does that again, into LDS, under its first loads of the weights, which costs less than a launch before it while there
// are few elements to round, of a workgroup and of all (once).  A workgroup has 16 outputs, its eight waves blocks of 128 of k in turn, kOnceUnits of them under way.  The 8-bit values are
// those of quantize_f8_kernel.  1 x 4096 -> 16384 bfloat16: 13.6 us, 4.9 TB/s.
constexpr int kOnceRows = 16, kOnceUnits = 4, kOnceWaves = 8;

template <int DT, bool WIDE>
__global__ __launch_bounds__(kOnceWaves * 64) void linear_f8_once_kernel(LinearF8Args p)
{
    using E = Elem<DT>;
    constexpr bool EXACT = DT == TICTAC_F32;
    extern __shared__ __align__(16) uint8_t held[];             // [rows][stride] 8-bit values, [rows][blocks] scales; then [waves][64] sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, fk = (lane >> 4) * 16;
    const int32_t units = (int32_t)((p.cols + 127) / 128), rows = (int32_t)p.rows, stride = units * 128 + 16;
    const int64_t o0 = (int64_t)blockIdx.x * 16, o = min(o0 + row, p.outs - 1);
    const uint8_t *const w = p.w.q + o * p.w.ld + fk, *const we = p.w.scale + (o >> p.w.shift) * p.w.ld_scale;
    uint8_t *const scales = held + rows * stride;
    struct Unit {
        i32x4 q[2];
        int e;
    } unit[kOnceUnits];
    const auto request = [&](int n, int32_t u) {
        u = min(u, units - 1);
#pragma unroll
        for (int k = 0; k < 2; ++k) unit[n].q[k] = *(const i32x4 *)(w + (int64_t)u * 128 + k * 64);
        unit[n].e = we[u];
    };
#pragma unroll
    for (int n = 0; n < kOnceUnits; ++n) request(n, wave + n * kOnceWaves);
    for (int32_t at = (int32_t)threadIdx.x >> 4; at < rows * units; at += kOnceWaves * 4) {
        const int32_t t = at / units, b = at - t * units, part = (int32_t)threadIdx.x & 15, col = b * 128 + part * 8;
        float v[8];
        E::floats(load8<DT, WIDE>((const typename E::type *)p.x + t * p.ld_x, col, p.cols), v);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
        const uint32_t scale = f8_scale(row16_max(m), TICTAC_E4M3);
        *(uint2 *)(held + t * stride + col) = f8_quantized8<TICTAC_E4M3>(v, scale, f8_nans(p.cols - col));
        if (part == 0) scales[at] = (uint8_t)scale;
    }
    __syncthreads();
    const int mine = min(row, rows - 1);
    const uint8_t *const x = held + mine * stride + fk, *const xe = scales + mine * units;
    f32x4 acc{};
    for (int32_t u0 = wave; u0 < units; u0 += kOnceUnits * kOnceWaves) {
#pragma unroll
        for (int n = 0; n < kOnceUnits; ++n) {
            const int32_t u = u0 + n * kOnceWaves;
            if (u >= units) break;
            const Unit now = unit[n];
            if (u + kOnceUnits * kOnceWaves < units) request(n, u + kOnceUnits * kOnceWaves);
            const i32x4 lo = *(const i32x4 *)(x + u * 128), hi = *(const i32x4 *)(x + u * 128 + 64);
            const int e = xe[u];
            if constexpr (EXACT) {
                i32x4 a[2], b[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    widen(now.q[k], f8_factor(now.e), TICTAC_E4M3, a);
                    widen(k ? hi : lo, f8_factor(e), TICTAC_E4M3, b);
#pragma unroll
                    for (int h = 0; h < 2; ++h) acc = mma_bf16(a[h], b[h], acc);
                }
            } else {
                const i32x8 a{now.q[0][0], now.q[0][1], now.q[0][2], now.q[0][3], now.q[1][0], now.q[1][1], now.q[1][2], now.q[1][3]};
                const i32x8 b{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, TICTAC_E4M3, TICTAC_E4M3, 0, now.e, 0, e);
            }
        }
    }
    __syncthreads();
    f32x4 *const sums = (f32x4 *)held;
    sums[threadIdx.x] = acc;
    __syncthreads();
    const int out = threadIdx.x & 15, t = threadIdx.x >> 4;
    if (t >= rows || o0 + out >= p.outs) return;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kOnceWaves; ++k) sum += sums[k * 64 + (out >> 2) * 16 + t][out & 3];
    if (p.bias) sum += param(p.bias, p.bias_dtype, o0 + out);
    put_param(p.y, p.dtype, t * p.ld_y + o0 + out, sum);
}

// (microseconds, here and by a launch for the rounding and the better of the others, outputs of 16 bits: 1 x 4096 -> 4096 5.6 and 9.1, 8 rows 9.5 and 9.8, 12 rows 11.9 and 10.1;
// 2 x 4096 -> 16384 14.1 and 16.5, 4 rows 17.4 and 16.6; float32, whose operands are widened in every workgroup too: 2 x 4096 -> 4096 8.1 and 9.5, 8 rows 11.6 and 10.2)
static bool once(bool exact, int64_t rows, int64_t cols, int64_t outs)
{
    const int64_t elements = rows * rows8_stride(cols);
    return rows <= kOnceRows && elements <= 1 << 15 && elements * ((outs + 15) / 16) <= (exact ? 1 << 22 : 1 << 23);
}

template <int DT, bool WIDE>
static hipError_t launch_once(const LinearF8Args &p, hipStream_t s)
{
    const int64_t units = f8_blocks(p.cols);
    const size_t lds = std::max<size_t>((size_t)(p.rows * (units * 128 + 16 + units)), kOnceWaves * 1024);
    hipLaunchKernelGGL((linear_f8_once_kernel<DT, WIDE>), dim3((unsigned)((p.outs + 15) / 16)), dim3(kOnceWaves * 64), (lds + 15) / 16 * 16, s, p);
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

// Few rows, by linear_f8_few_kernel: float32 outputs up to 64, where tiles want all weights as bf16 first (64 x 4096 -> 4096: 19 us, 25 in tiles; 17 rows 11.6 and 25).  In 16 bits tiles read the
// weights as fast and x less often, and what is left are small products and, up to 16 rows, medium ones (microseconds, here and in tiles: 16 x 4096 -> 4096 10.7 and 12.4, 16 x 4096 ->
// 16384 19.2 and 17.0; 32 x 1024 -> 4096 8.2 and 9.7, 32 x 4096 -> 4096 13.0 and 12.7, 32 x 25088 -> 4096 31.9 and 28.4).
static bool few_rows(bool exact, int64_t rows, int64_t cols, int64_t outs)
{
    const int64_t weights = cols * outs;
    return exact ? rows <= 64 : rows <= 16 ? weights < 1 << 26 : rows <= 64 && weights <= 1 << 22;
}
// Blocks of 16 outputs of a workgroup: more of them read x less often, but leave fewer workgroups.  (16 x 2048 -> 16384: one 14.0 us, two 12.3; 16 x 4096 -> 4096 10.7 and 12.2; float32, 64 x 2048 ->
// 16384: one 34, four 21; 32 x 4096 -> 4096 13.3 and 14.2.)
static int32_t few_blocks_of(int64_t rows, int64_t cols, int64_t outs) { return cols * outs < 1 << 25 ? 1 : rows <= 16 ? 2 : 4; }
static int32_t few_splits(int64_t rows, int64_t cols, int64_t outs)
{
    const int64_t each = 16 * few_blocks_of(rows, cols, outs), blocks = (outs + each - 1) / each, units = (cols + 127) / 128;
    return parts_along_k(blocks, units / kFewWaves, 256);
}

static size_t up(size_t n) { return (n + 255) / 256 * 256; }

// The workspace of a forward call.
struct ForwardRoom {
    ProductPlan plan;
    size_t x, xe, w, parts, bytes;          // offsets: x in 8 bits and its scales, or as bf16; w as bf16; sums of splits
};
static ForwardRoom forward_room(int32_t dtype, int32_t from_floats, int64_t rows, int64_t cols, int64_t outs)
{
    ForwardRoom r{};
    const int64_t ld = rows8_stride(cols);
    const bool exact = dtype == TICTAC_F32, few = few_rows(exact, rows, cols, outs);
    if (from_floats && once(exact, rows, cols, outs)) return r;
    if (few) {
        r.plan = {0, {few_splits(rows, cols, outs), 1}};
    } else {
        const ProductShape shape{(int32_t)outs, (int32_t)rows, (int32_t)(exact ? ld / 64 : ld / 128)};
        r.plan = exact ? plan_products(&shape, 1) : plan_products_f8(&shape, 1);
    }
    const bool wide = exact && !few;
    r.xe = r.x + up(wide ? (size_t)rows * ld * 2 : from_floats ? (size_t)rows * ld : 0);
    r.w = r.xe + up(from_floats && !wide ? (size_t)rows * f8_scale_stride(cols) : 0);
    r.parts = r.w + up(wide ? (size_t)outs * ld * 2 : 0);
    r.bytes = r.parts + up(product_parts_bytes(r.plan.splits[0], (int32_t)outs, (int32_t)rows));
    return r;
}
size_t linear_f8_workspace(int32_t dtype, int32_t from_floats, int64_t rows, int64_t cols, int64_t outs) { return forward_room(dtype, from_floats, rows, cols, outs).bytes; }

// 8-bit floats whose values go to `to` as bf16, [rows][padded]
static F8QuantizeArgs widened(const F8Rows &r, int64_t rows, int64_t padded, void *to)
{
    F8QuantizeArgs a{};
    a.dtype = TICTAC_BF16; a.format = r.format; a.block = 1 << r.shift; a.rows = rows; a.cols = padded; a.out = to; a.ld_x = padded;
    a.q = const_cast<uint8_t *>(r.q); a.ld_q = r.ld; a.scale = const_cast<uint8_t *>(r.scale); a.ld_scale = r.ld_scale;
    return a;
}

template <bool EXACT, int QF>
static auto few_kernel(int64_t rows, int32_t fb)
{
    if (rows <= 16) return fb == 1 ? linear_f8_few_kernel<EXACT, QF, 1, 1> : linear_f8_few_kernel<EXACT, QF, 1, 2>;
    if constexpr (EXACT)
        if (fb != 1) return rows <= 32 ? linear_f8_few_kernel<EXACT, QF, 2, 4> : linear_f8_few_kernel<EXACT, QF, 4, 4>;
    return rows <= 32 ? linear_f8_few_kernel<EXACT, QF, 2, 1> : linear_f8_few_kernel<EXACT, QF, 4, 1>;
}

hipError_t launch_linear_f8(const LinearF8Args &p, hipStream_t s)
{
    const bool exact = p.dtype == TICTAC_F32, few = few_rows(exact, p.rows, p.cols, p.outs), wide = exact && !few;
    if (p.x && once(exact, p.rows, p.cols, p.outs)) return BY_TYPE(p.dtype, wide_rows(p.x, p.dtype, p.ld_x, p.cols), launch_once, p, s);
    const ForwardRoom room = forward_room(p.dtype, p.x != nullptr, p.rows, p.cols, p.outs);
    const int64_t ld = rows8_stride(p.cols);
    char *at = (char *)p.workspace;
    F8Rows x = p.x8;
    F8QuantizeArgs q{};
    if (p.x) {
        q.dtype = p.dtype; q.format = TICTAC_E4M3; q.block = 1; q.rows = p.rows; q.cols = p.cols; q.x = p.x; q.ld_x = p.ld_x; q.ld_q = ld;
        if (wide) {
            q.out = at + room.x;
        } else {
            q.q = (uint8_t *)at + room.x;
            q.scale = (uint8_t *)at + room.xe;
            q.ld_scale = f8_scale_stride(p.cols);
            if (const hipError_t e = launch_quantize_f8(q, s); e != hipSuccess) return e;
            x = F8Rows{q.q, ld, q.scale, q.ld_scale, TICTAC_E4M3, 0};
        }
    } else if (wide) {
        q = widened(p.x8, p.rows, ld, at + room.x);
    }
    const int32_t splits = room.plan.splits[0];
    ProductF8Args a{};
    a.R = (int32_t)p.outs; a.C = (int32_t)p.rows; a.splits = splits;
    a.out = p.y; a.ld_out = p.ld_y; a.dtype = p.dtype; a.bias = p.bias; a.bias_dtype = p.bias_dtype; a.parts = at + room.parts;
    if (few) {
        const int32_t fb = few_blocks_of(p.rows, p.cols, p.outs), outs = 16 * fb;
        const auto kernel = exact ? (x.format == TICTAC_E5M2 ? few_kernel<true, TICTAC_E5M2>(p.rows, fb) : few_kernel<true, TICTAC_E4M3>(p.rows, fb))
                                  : (x.format == TICTAC_E5M2 ? few_kernel<false, TICTAC_E5M2>(p.rows, fb) : few_kernel<false, TICTAC_E4M3>(p.rows, fb));
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.outs + outs - 1) / outs * splits)), dim3(kFewWaves * 64), 0, s, p, x, splits, (float *)a.parts);
        return splits > 1 ? launch_product_join_biased(a, s) : hipGetLastError();
    }
    if (wide) {
        if (const hipError_t e = launch_widen_f8(q, widened(p.w, p.outs, ld, at + room.w), s); e != hipSuccess) return e;
        a.p = at + room.w; a.ld_p = ld * 2;
        a.q = at + room.x; a.ld_q = ld * 2;
        a.steps = a.p_steps = (int32_t)(ld / 64);
        return launch_product_bf16_biased(a, room.plan.tile, s);
    }
    a.p = (const char *)p.w.q; a.ld_p = p.w.ld; a.p_e = p.w.scale; a.ld_pe = p.w.ld_scale; a.p_shift = p.w.shift;
    a.q = (const char *)x.q; a.ld_q = x.ld; a.q_e = x.scale; a.ld_qe = x.ld_scale; a.q_shift = x.shift; a.q_format = x.format;
    a.steps = a.p_steps = (int32_t)(ld / 128);
    return launch_products_f8(&a, 1, room.plan.tile, ColumnSums{}, s);
}

// ---- dx with few rows: bound by the bytes of the weights ----
// The weights, in blocks of 128 x 128, have k (the outputs o) as rows, and the matrix instruction wants 32 of k per lane.  A lane reads eight bytes of each of 32 rows, a wave 128 rows of
// 128 columns, one block; squares of 4 x 4 bytes are turned round in registers, and byte j of the eight is an operand whose row r is column 8 r + j, so that a lane's results are columns
// next to each other.  A workgroup has 128 columns and a part of k, its eight waves blocks of that in turn; their sums meet in LDS, in fixed order.  The 16 KB that each wave
// has under way are more than memory's latency asks for.  32 x 4096 -> 25088 float16: 27 us, 3.9 TB/s.
constexpr int kBackWaves = 8;

// four rows of four bytes to four columns
__device__ __forceinline__ void turn4(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d)
{
    const uint32_t ab_lo = __builtin_amdgcn_perm(b, a, 0x05010400), ab_hi = __builtin_amdgcn_perm(b, a, 0x07030602);       // a0 b0 a1 b1, a2 b2 a3 b3
    const uint32_t cd_lo = __builtin_amdgcn_perm(d, c, 0x05010400), cd_hi = __builtin_amdgcn_perm(d, c, 0x07030602);
    a = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100);
    b = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302);
    c = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100);
    d = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302);
}

template <int QF, int TB>
__global__ __launch_bounds__(kBackWaves * 64) void linear_f8_dx_few_kernel(LinearF8Args p, F8Operand dy, int32_t splits, float *parts)
{
    extern __shared__ float room[];                             // [waves][8][64 lanes][4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int64_t strips = gridDim.x / splits, strip = blockIdx.x % strips, i0 = strip * 128;
    const int32_t split = (int32_t)(blockIdx.x / strips), all = (int32_t)((p.outs + 127) / 128);
    const int32_t first = (int32_t)((int64_t)all * split / splits), last = (int32_t)((int64_t)all * (split + 1) / splits);
    f32x4 acc[8][TB] = {};
    for (int32_t u = first + wave; u < last; u += kBackWaves) {
        const int64_t o0 = (int64_t)u * 128 + g * 32, rest = p.outs - o0;       // (rows behind the end: the last again, times zeros)
        const uint8_t *const w = p.w.q + i0 + r * 8;
        uint32_t v[2][32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const uint2 two = *(const uint2 *)(w + (e < rest ? o0 + e : p.outs - 1) * p.w.ld);
            v[0][e] = two.x;
            v[1][e] = two.y;
        }
        const int we = p.w.scale[(int64_t)u * p.w.ld_scale + strip];
        i32x8 q[TB];
        int qe[TB];
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            const int64_t t = min((int64_t)b * 16 + r, p.rows - 1);
            const i32x4 *const from = (const i32x4 *)((const uint8_t *)dy.q + t * dy.ld + o0);
            const i32x4 lo = from[0], hi = from[1];
            q[b] = i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            qe[b] = dy.scale[t * dy.ld_scale + u];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) turn4(v[h][e], v[h][e + 1], v[h][e + 2], v[h][e + 3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                i32x8 f;
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (int32_t)v[h][e * 4 + j];
#pragma unroll
                for (int b = 0; b < TB; ++b)
                    acc[h * 4 + j][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f, q[b], acc[h * 4 + j][b], TICTAC_E4M3, QF, 0, we, 0, qe[b]);
            }
        }
    }
    // A thread adds up eight columns of one row over the waves, in their order: element e of lane l.
    const int le = threadIdx.x & 255, from = le >> 2;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        if (b) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) *(f32x4 *)(room + ((wave * 8 + j) * 64 + lane) * 4) = acc[j][b];
        __syncthreads();
        const int64_t t = b * 16 + (from & 15), i = i0 + 8 * (4 * (from >> 4) + (le & 3));
        if (threadIdx.x >= 256 || t >= p.rows) continue;
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[j] = 0.0f;
#pragma unroll
            for (int k = 0; k < kBackWaves; ++k) sum[j] += room[(k * 8 + j) * 256 + le];
        }
        if (splits > 1) {
            store8<TICTAC_F32, false>(parts + ((int64_t)split * p.rows + t) * p.cols, i, p.cols, sum);
        } else if (p.dtype == TICTAC_F16) {
            store8<TICTAC_F16, false>((_Float16 *)p.dx + t * p.ld_dx, i, p.cols, sum);
        } else {
            store8<TICTAC_BF16, false>((__bf16 *)p.dx + t * p.ld_dx, i, p.cols, sum);
        }
    }
}

// dw where the rows are one block: a matrix instruction is all that an output takes, and dw's bytes are what bounds it.  A wave has 64 columns, whose operands (turned round before, 128
// bytes of k each, of which those behind the last row are not read) stay in registers, and 128 outputs, a workgroup 512 columns.  Row r of operand j is the column at(r) + j: a lane's results (rows 4 g + e) then are eight next to each other at
// 8 g, and eight at 32 + 8 g, and four lanes store 64 bytes in a row.  25088 x 4096 float16: 51 us, 4.7 TB/s; workgroups of 256 outputs take 3 us more.
constexpr int kDwOuts = 128;

template <int QF, int DT, bool WIDE>
__global__ __launch_bounds__(512) void linear_f8_dw_few_kernel(LinearF8Args p, F8Operand x, F8Operand dy, ColumnSums sums)
{
    using T = typename Elem<DT>::type;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int64_t o0 = (int64_t)blockIdx.y * kDwOuts, i0 = (int64_t)blockIdx.x * 512 + wave * 64;
    if (sums.out && blockIdx.x == 0 && (int)threadIdx.x < kDwOuts && o0 + threadIdx.x < p.outs) put_param(sums.out, DT, o0 + threadIdx.x, sums.sums[o0 + threadIdx.x]);
    if (i0 >= p.cols) return;
    const auto operand = [&](const F8Operand &from, int64_t row) {
        const i32x4 *const at = (const i32x4 *)((const uint8_t *)from.q + row * from.ld + g * 32);
        i32x4 lo{}, hi{};
        if (g * 32 < p.rows) { lo = at[0]; hi = at[1]; }
        return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    const int64_t column = i0 + ((c & 2) << 4) + ((c >> 2) << 3) + ((c & 1) << 2);
    const bool whole = WIDE && i0 + 64 <= p.cols;
    i32x8 f[4], q;
    int fe[4], qe;
    const auto request = [&](int b) {
        const int64_t o = min(o0 + b * 16 + c, p.outs - 1);
        q = operand(dy, o);
        qe = dy.scale[o * dy.ld_scale];
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = min(column + j, p.cols - 1);
        f[j] = operand(x, i);
        fe[j] = x.scale[i * x.ld_scale];
    }
    request(0);
#pragma unroll 2
    for (int b = 0; b < kDwOuts / 16; ++b) {
        const i32x8 now = q;
        const int e = qe;
        if (b + 1 < kDwOuts / 16) request(b + 1);
        f32x4 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f[j], now, f32x4{}, TICTAC_E4M3, QF, 0, fe[j], 0, e);
        const int64_t out = o0 + b * 16 + c;
        if (whole && o0 + b * 16 + 16 <= p.outs) {
            i32x4 piece[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) v[n] = acc[n & 3][h * 2 + (n >> 2)];
                piece[h] = __builtin_bit_cast(i32x4, Elem<DT>::pack(v));
            }
            put_lines<32>((T *)p.dw + i0, g * 8, (int32_t)out, p.ld_dw, piece[0], piece[1]);
            continue;
        }
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

template <int DT, bool WIDE>
static hipError_t launch_dw_few(const LinearF8Args &p, const F8Operand &x, const F8Operand &dy, const ColumnSums &sums, hipStream_t s)
{
    const auto kernel = p.format == TICTAC_E5M2 ? linear_f8_dw_few_kernel<TICTAC_E5M2, DT, WIDE> : linear_f8_dw_few_kernel<TICTAC_E4M3, DT, WIDE>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.cols + 511) / 512), (unsigned)((p.outs + kDwOuts - 1) / kDwOuts)), dim3(512), 0, s, p, x, dy, sums);
    return hipGetLastError();
}

static int32_t dx_few_splits(int64_t cols, int64_t outs) { return parts_along_k(f8_blocks(cols), f8_blocks(outs) / kBackWaves, 256); }     // a block for each wave at least

template <int QF>
static hipError_t launch_dx_few(const LinearF8Args &p, const F8Operand &dy, void *parts, hipStream_t s)
{
    const int32_t splits = dx_few_splits(p.cols, p.outs);
    const auto kernel = p.rows <= 16 ? linear_f8_dx_few_kernel<QF, 1> : linear_f8_dx_few_kernel<QF, 2>;
    const size_t lds = (size_t)kBackWaves * 8 * 64 * 16;
    if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(f8_blocks(p.cols) * splits)), dim3(kBackWaves * 64), lds, s, p, dy, splits, (float *)parts);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || splits == 1) return e;
    ProductArgs a{};
    a.R = (int32_t)p.cols; a.C = (int32_t)p.rows; a.splits = splits; a.out = p.dx; a.ld_out = p.ld_dx; a.dtype = p.dtype; a.parts = parts;
    return launch_product_join_bf16(a, s);
}

// ---- backward ----
// Both products in tiles are one launch; by themselves those of few rows leave the weights as they lie and write dw past the caches, which pays where there are many weights (microseconds,
// outputs of 16 bits, dx and dw by themselves, dw alone, none: 32 x 1024 -> 4096 25, 24, 20; 32 x 4096 -> 4096 29, 35, 36; 64 x 4096 -> 4096 42, 35, 36; 32 x 25088 -> 4096 83, 109, 127;
// 64 x 25088 -> 4096 120, 113, 129; 128 x 4096 -> 4096 41 and 35, 128 x 4096 -> 16384 94 and 103 for the last two).
constexpr int64_t kDxFewRows = 32;
static bool dw_by_itself(bool exact, int64_t rows, int64_t cols, int64_t outs) { return !exact && rows <= kF8Block && cols * outs >= (rows <= kDxFewRows ? 1 << 23 : 1 << 25); }
struct BackwardRoom {
    int64_t padded_o, padded_t;
    ProductPlan plan;                       // dx, dw
    size_t sums, w, we, x, xe, dy_rows, dy_rows_e, dy_cols, dy_cols_e, parts_x, parts_w, bytes;
};
static BackwardRoom backward_room(int32_t dtype, int64_t rows, int64_t cols, int64_t outs)
{
    const bool exact = dtype == TICTAC_F32;
    const size_t size = exact ? 2 : 1;
    BackwardRoom r{};
    r.padded_o = rows8_stride(outs);
    r.padded_t = rows8_stride(rows);
    const int64_t step = exact ? 64 : 128;
    const ProductShape shapes[2] = {{(int32_t)cols, (int32_t)rows, (int32_t)(r.padded_o / step)}, {(int32_t)cols, (int32_t)outs, (int32_t)(r.padded_t / step)}};
    const bool alone = dw_by_itself(exact, rows, cols, outs), few = alone && rows <= kDxFewRows;       // (few: dx may come from the weights as they lie)
    // where dw is by itself, the tiles are dx's alone
    r.plan = exact ? plan_products(shapes, 2) : plan_products_f8(shapes, alone ? 1 : 2);
    const size_t e = exact ? 0 : 1;         // (values as bf16 have no scales)
    r.w = r.sums + up((size_t)f8_blocks(rows) * outs * 4);
    r.we = r.w + up((size_t)cols * r.padded_o * size);
    r.x = r.we + up(e * cols * f8_scale_stride(outs));
    r.xe = r.x + up((size_t)cols * r.padded_t * size);
    r.dy_rows = r.xe + up(e * cols * f8_scale_stride(rows));
    r.dy_rows_e = r.dy_rows + up((size_t)rows * r.padded_o * size);
    r.dy_cols = r.dy_rows_e + up(e * rows * f8_scale_stride(outs));
    r.dy_cols_e = r.dy_cols + up((size_t)outs * r.padded_t * size);
    r.parts_x = r.dy_cols_e + up(e * outs * f8_scale_stride(rows));
    r.parts_w = r.parts_x + up(product_parts_bytes(few ? std::max(r.plan.splits[0], dx_few_splits(cols, outs)) : r.plan.splits[0], (int32_t)cols, (int32_t)rows));
    r.bytes = r.parts_w + up(product_parts_bytes(r.plan.splits[1], (int32_t)cols, (int32_t)outs));
    return r;
}
size_t linear_f8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs) { return backward_room(dtype, rows, cols, outs).bytes; }

// No rows, or no outputs: what there is of the gradients is zero.
static hipError_t backward_nothing(const LinearF8Args &p, hipStream_t s)
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

hipError_t launch_linear_f8_backward(const LinearF8Args &p, hipStream_t s)
{
    if (p.rows == 0 || p.outs == 0) return backward_nothing(p, s);
    const BackwardRoom room = backward_room(p.dtype, p.rows, p.cols, p.outs);
    const bool exact = p.dtype == TICTAC_F32, alone = dw_by_itself(exact, p.rows, p.cols, p.outs);
    const int64_t size = exact ? 2 : 1, step = exact ? 64 : 128;
    char *at = (char *)p.workspace;
    F8TurnArgs t{};
    t.dtype = p.dtype; t.format = p.format; t.rows = p.rows; t.cols = p.cols; t.outs = p.outs; t.dy = p.dy; t.ld_dy = p.ld_dy; t.x = p.x8; t.w = p.w;
    const bool dx_few = p.dx && alone && p.rows <= kDxFewRows && p.w.shift;
    if (p.dx) {
        if (!dx_few) t.w_cols = {at + room.w, room.padded_o, (uint8_t *)at + room.we, f8_scale_stride(p.outs)};
        t.dy_rows = {at + room.dy_rows, room.padded_o, (uint8_t *)at + room.dy_rows_e, f8_scale_stride(p.outs)};
    }
    if (p.dw) {
        t.x_cols = {at + room.x, room.padded_t, (uint8_t *)at + room.xe, f8_scale_stride(p.rows)};
        t.dy_cols = {at + room.dy_cols, room.padded_t, (uint8_t *)at + room.dy_cols_e, f8_scale_stride(p.rows)};
    }
    if (p.db) t.sums = (float *)(at + room.sums);
    if (const hipError_t e = launch_turn_f8(t, s); e != hipSuccess) return e;
    ProductF8Args a[2] = {};
    int n = 0;
    const auto add = [&](const F8Operand &rows_p, const F8Operand &rows_q, int64_t padded, int64_t outputs, void *out, int64_t ld, int32_t splits, size_t parts) {
        ProductF8Args &x = a[n++];
        x.p = (const char *)rows_p.q; x.ld_p = rows_p.ld * size; x.p_e = rows_p.scale; x.ld_pe = rows_p.ld_scale;
        x.q = (const char *)rows_q.q; x.ld_q = rows_q.ld * size; x.q_e = rows_q.scale; x.ld_qe = rows_q.ld_scale; x.q_format = p.format;
        x.R = (int32_t)p.cols; x.C = (int32_t)outputs; x.steps = x.p_steps = (int32_t)(padded / step);
        x.splits = splits; x.out = out; x.ld_out = ld; x.parts = at + parts; x.dtype = p.dtype;
    };
    if (dx_few) {
        if (const hipError_t e = p.format == TICTAC_E5M2 ? launch_dx_few<TICTAC_E5M2>(p, t.dy_rows, at + room.parts_x, s) : launch_dx_few<TICTAC_E4M3>(p, t.dy_rows, at + room.parts_x, s); e != hipSuccess) return e;
    }
    if (p.dx && !dx_few) add(t.w_cols, t.dy_rows, room.padded_o, p.rows, p.dx, p.ld_dx, room.plan.splits[0], room.parts_x);
    const ColumnSums c{t.sums, f8_blocks(p.rows), p.outs, p.db, p.dtype};
    if (p.dw && alone) {
        const bool wide = wide_rows(p.dw, p.dtype, p.ld_dw, p.cols);
        const hipError_t e = p.dtype == TICTAC_F16 ? (wide ? launch_dw_few<TICTAC_F16, true>(p, t.x_cols, t.dy_cols, c, s) : launch_dw_few<TICTAC_F16, false>(p, t.x_cols, t.dy_cols, c, s))
                                                   : (wide ? launch_dw_few<TICTAC_BF16, true>(p, t.x_cols, t.dy_cols, c, s) : launch_dw_few<TICTAC_BF16, false>(p, t.x_cols, t.dy_cols, c, s));
        if (e != hipSuccess || !n) return e;
        return launch_products_f8(a, n, room.plan.tile, ColumnSums{}, s);
    }
    if (p.dw) add(t.x_cols, t.dy_cols, room.padded_t, p.outs, p.dw, p.ld_dw, room.plan.splits[1], room.parts_w);
    if (!exact) return launch_products_f8(a, n, room.plan.tile, c, s);
    const ProductArgs wide[2] = {a[0], a[1]};
    return launch_products_bf16(wide, n, room.plan.tile, c, s);
}

}  // namespace tictac
