// Rows in 8 bits: activations and weights as int8 with float32 scales, one per row (the operands of the products) or one per
// kRows8Group columns (activations kept for the backward pass), and back.
//   scale = amax / 127,  q = round(x * (127 / amax)),  x ~ q * scale
// Bound by memory: an element is read once and written as one byte (back: the other way round), eight of a row per thread.
#include "rows8.h"

namespace tictac {

// A scale per 128 columns.  128 columns are eight elements of each of 16 lanes, a row of the data-parallel primitives, so the maximum takes four
// steps without LDS.  A group of lanes has kTurns groups of columns at hand at once, to have as many loads under way.  16384 x 4096 bfloat16: 47 us,
// 4.3 TB/s.
constexpr int kTurns = 4;

template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void quantize_groups_kernel(QuantizeArgs p, int64_t groups, int64_t total)
{
    using E = Elem<DT>;
    const int lane = threadIdx.x & 15;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 16, step = (int64_t)gridDim.x * 16;
    for (int64_t at = first; at < total; at += kTurns * step) {
        typename E::raw raw[kTurns];
        int64_t row[kTurns];
        int32_t g[kTurns];
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int64_t i = at + k * step;
            if (i >= total) continue;
            row[k] = total < (1ll << 31) ? (int64_t)((uint32_t)i / (uint32_t)groups) : i / groups;
            g[k] = (int32_t)(i - row[k] * groups);
            raw[k] = load8<DT, WIDE>((const typename E::type *)p.x + row[k] * p.ld_x, (int64_t)g[k] * 128 + lane * 8, p.cols);
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            if (at + k * step >= total) continue;
            float v[8];
            E::floats(raw[k], v);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
            const RowScale s = row_scale(row16_max(m));
            *(uint2 *)(p.q + row[k] * p.ld_q + (int64_t)g[k] * 128 + lane * 8) = quantized8(v, s);      // (also the zeros behind the end)
            if (lane == 0) p.scale[row[k] * groups + g[k]] = s.scale;
        }
    }
}

// A scale per row, a workgroup per row, which stays in registers: NC pieces of eight elements per thread.  Longer rows (NC = 0) are read twice.
// 16384 x 4096 bfloat16: 34 us, 5.9 TB/s; 1024 x 65536, read twice: 53.
template <int DT, bool WIDE, int THREADS, int NC>
__global__ __launch_bounds__(THREADS) void quantize_rows_kernel(QuantizeArgs p)
{
    using E = Elem<DT>;
    __shared__ uint32_t part[2][THREADS / 64];          // (two sets in turn: one barrier a row)
    const int64_t padded = (p.cols + 127) / 128 * 128;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        const typename E::type *x = (const typename E::type *)p.x + row * p.ld_x;
        typename E::raw raw[NC ? NC : 1];
        uint32_t m = 0;
        const auto largest = [&](const typename E::raw &r) {
            float v[8];
            E::floats(r, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
        };
        if (NC) {
#pragma unroll
            for (int j = 0; j < NC; ++j) raw[j] = load8<DT, WIDE>(x, (int64_t)(j * THREADS + threadIdx.x) * 8, p.cols);
#pragma unroll
            for (int j = 0; j < NC; ++j) largest(raw[j]);
        } else {
            for (int64_t col = threadIdx.x * 8; col < p.cols; col += THREADS * 8) largest(load8<DT, WIDE>(x, col, p.cols));
        }
        m = wave_max_u32(m);
        if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) m = max(m, part[turn][i]);
        const RowScale s = row_scale(m);
        const auto put = [&](const typename E::raw &r, int64_t col) {
            float v[8];
            E::floats(r, v);
            if (col < padded) *(uint2 *)(p.q + row * p.ld_q + col) = quantized8(v, s);
        };
        if (NC) {
#pragma unroll
            for (int j = 0; j < NC; ++j) put(raw[j], (int64_t)(j * THREADS + threadIdx.x) * 8);
        } else {
            for (int64_t col = threadIdx.x * 8; col < padded; col += THREADS * 8) put(load8<DT, WIDE>(x, col, p.cols), col);
        }
        if (threadIdx.x == 0) p.scale[row] = s.scale;
    }
}

// Back: eight values a thread.  16384 x 4096 to bfloat16: 35 us, 5.9 TB/s.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void dequantize_kernel(QuantizeArgs p, int64_t chunks, int64_t total, int64_t scales)
{
    using E = Elem<DT>;
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t at = first; at < total; at += kTurns * step) {
        uint2 q[kTurns];
        float s[kTurns];
        int64_t row[kTurns], col[kTurns];
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int64_t i = at + k * step;
            if (i >= total) continue;
            row[k] = total < (1ll << 31) ? (int64_t)((uint32_t)i / (uint32_t)chunks) : i / chunks;
            col[k] = (i - row[k] * chunks) * 8;
            q[k] = *(const uint2 *)(p.q + row[k] * p.ld_q + col[k]);
            s[k] = p.scale[row[k] * scales + (scales > 1 ? col[k] >> 7 : 0)];
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            if (at + k * step >= total) continue;
            float v[8];
            values8(q[k], s[k], v);
            store8<DT, WIDE>((typename E::type *)p.out + row[k] * p.ld_x, col[k], p.cols, v);
        }
    }
}

static unsigned elementwise_blocks(int64_t per_block_units)
{
    return (unsigned)(per_block_units < 1 ? 1 : per_block_units > 256 * 16 ? 256 * 16 : per_block_units);
}

template <int DT, bool WIDE>
static hipError_t quantize(const QuantizeArgs &p, hipStream_t s)
{
    if (p.group) {
        const int64_t groups = (p.cols + 127) / 128, total = groups * p.rows;
        hipLaunchKernelGGL((quantize_groups_kernel<DT, WIDE>), dim3(elementwise_blocks((total + 16 * kTurns - 1) / (16 * kTurns))), dim3(256), 0, s, p, groups, total);
    } else {
        const dim3 grid((unsigned)(p.rows < (1 << 20) ? p.rows : (1 << 20)));
        // few long rows leave most of the chip idle: as many threads for each as a workgroup can have
        const int64_t c = p.cols;
        if (c <= 2048) hipLaunchKernelGGL((quantize_rows_kernel<DT, WIDE, 256, 1>), grid, dim3(256), 0, s, p);
        else if (c <= 8192 && p.rows <= 512) hipLaunchKernelGGL((quantize_rows_kernel<DT, WIDE, 1024, 1>), grid, dim3(1024), 0, s, p);
        else if (c <= 8192) hipLaunchKernelGGL((quantize_rows_kernel<DT, WIDE, 256, 4>), grid, dim3(256), 0, s, p);
        else if (c <= 32768) hipLaunchKernelGGL((quantize_rows_kernel<DT, WIDE, 1024, 4>), grid, dim3(1024), 0, s, p);
        else hipLaunchKernelGGL((quantize_rows_kernel<DT, WIDE, 1024, 0>), grid, dim3(1024), 0, s, p);
    }
    return hipGetLastError();
}

template <int DT, bool WIDE>
static hipError_t dequantize(const QuantizeArgs &p, hipStream_t s)
{
    const int64_t chunks = (p.cols + 7) / 8, total = chunks * p.rows;
    hipLaunchKernelGGL((dequantize_kernel<DT, WIDE>), dim3(elementwise_blocks((total + 256 * kTurns - 1) / (256 * kTurns))), dim3(256), 0, s, p, chunks, total,
                       p.group ? (p.cols + 127) / 128 : (int64_t)1);
    return hipGetLastError();
}

hipError_t launch_quantize_rows(const QuantizeArgs &p, hipStream_t s)
{
    return BY_TYPE(p.dtype, wide_rows(p.x, p.dtype, p.ld_x, p.cols), quantize, p, s);
}

hipError_t launch_dequantize_rows(const QuantizeArgs &p, hipStream_t s)
{
    return BY_TYPE(p.dtype, wide_rows(p.out, p.dtype, p.ld_x, p.cols), dequantize, p, s);
}

}  // namespace tictac
