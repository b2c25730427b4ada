// Rounding to 8-bit floats in blocks (f8.h), back, and the operands of a backward pass.
#include <algorithm>

#include "device_utils.h"
#include "f8.h"

namespace tictac {

// Blocks of 128 columns of one row: eight elements of each of 16 lanes, a row of the data-parallel primitives, so the maximum takes four steps without LDS.  kTurns blocks of a
// group of lanes are under way at once.  Bound by memory: 8192 x 4096 bfloat16 25 us, 4.1 TB/s; back 33 us for 16384 x 4096, 6.0 TB/s.
constexpr int kTurns = 4;

// A block's scale; behind the last of a row, zeros up to the next multiple of four.  `lane` counts the lanes that have the block.
__device__ __forceinline__ void put_scale(uint8_t *row, int64_t at, int64_t blocks, int lane, uint32_t scale)
{
    if (lane == 0 || (lane < 4 && at == blocks - 1 && at + lane < (blocks + 3) / 4 * 4)) row[at + lane] = lane ? (uint8_t)0 : (uint8_t)scale;
}

// The blocks of one row that workgroup `group` of `groups` has.  BF16: the values that 8 bits keep, as bf16.
template <int DT, bool WIDE, int FORMAT, bool BF16>
__device__ __forceinline__ void quantize_blocks(const F8QuantizeArgs &p, int64_t blocks, int64_t total, uint32_t group, uint32_t groups)
{
    using E = Elem<DT>;
    const int lane = threadIdx.x & 15;
    const int64_t first = ((int64_t)group * 256 + threadIdx.x) / 16, step = (int64_t)groups * 16;
    for (int64_t at = first; at < total; at += kTurns * step) {
        typename E::raw raw[kTurns];
        int64_t row[kTurns], col[kTurns];
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int64_t i = at + k * step;
            if (i >= total) continue;
            row[k] = total < (1ll << 31) ? (int64_t)((uint32_t)i / (uint32_t)blocks) : i / blocks;
            col[k] = (i - row[k] * blocks) * 128 + lane * 8;
            raw[k] = load8<DT, WIDE>((const typename E::type *)p.x + row[k] * p.ld_x, col[k], p.cols);
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            if (at + k * step >= total) continue;
            float v[8];
            E::floats(raw[k], v);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
            const uint32_t scale = f8_scale(row16_max(m), FORMAT);
            const uint2 q = f8_quantized8<FORMAT>(v, scale, f8_nans(p.cols - col[k]));      // (also the zeros behind the end)
            if constexpr (BF16) {
                f8_values8(q, scale, FORMAT, v);
                *(i32x4 *)((uint16_t *)p.out + row[k] * p.ld_q + col[k]) = f8_bf16(v);
            } else {
                *(uint2 *)(p.q + row[k] * p.ld_q + col[k]) = q;
                put_scale(p.scale + row[k] * p.ld_scale, col[k] >> 7, blocks, lane, scale);
            }
        }
    }
}

template <int DT, bool WIDE, int FORMAT>
__global__ __launch_bounds__(256) void quantize_f8_kernel(F8QuantizeArgs p, int64_t blocks, int64_t total)
{
    quantize_blocks<DT, WIDE, FORMAT, false>(p, blocks, total, blockIdx.x, gridDim.x);
}

// The tile of 128 x 128 that a workgroup has: thread t has rows N (t / 16) .. + N - 1 and columns 8 (t % 16) .. + 7 of it.
template <int N>
struct Tile128 {
    static constexpr int kThreads = 128 / N * 16;
    int lane, group;
    int64_t r, c;               // of the thread's first element
    __device__ __forceinline__ Tile128(int64_t tile_r, int64_t tile_c) : lane(threadIdx.x & 15), group(threadIdx.x >> 4), r(tile_r * 128 + group * N), c(tile_c * 128 + lane * 8) {}
};

// (rows and, with WIDE, columns behind the end: the last again, made zeros, so that all loads are under way at once)
template <int DT, bool WIDE, int N>
__device__ __forceinline__ void load_tile(const void *x, int64_t ld, int64_t rows, int64_t cols, const Tile128<N> &t, typename Elem<DT>::raw (&raw)[N])
{
    using E = Elem<DT>;
    const typename E::type *const from = (const typename E::type *)x;
    if (WIDE || t.c + 8 <= cols) {
        const int64_t c = WIDE ? min(t.c, cols - 8) : t.c;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const typename E::type *const at = from + min(t.r + e, rows - 1) * ld + c;
            raw[e] = WIDE ? E::load(at) : load_anywhere<DT>(at);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) raw[e] = load8<DT, false>(from + min(t.r + e, rows - 1) * ld, t.c, cols);
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (t.r + e >= rows || (WIDE && t.c >= cols)) raw[e] = typename E::raw{};
}

// Blocks of 128 x 128: a workgroup each, which stays in registers between its maximum and its rounding.  16384 x 4096 bfloat16: 40 us, 5.0 TB/s.
template <int DT, bool WIDE, int FORMAT>
__global__ __launch_bounds__(256) void quantize_f8_tiles_kernel(F8QuantizeArgs p, uint32_t across)
{
    using E = Elem<DT>;
    __shared__ uint32_t part[4];
    const uint32_t tile_r = blockIdx.x / across, tile_c = blockIdx.x % across;
    const Tile128<8> t(tile_r, tile_c);
    typename E::raw raw[8];
    load_tile<DT, WIDE, 8>(p.x, p.ld_x, p.rows, p.cols, t, raw);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float v[8];
        E::floats(raw[e], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
    }
    m = wave_max_u32(m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    const uint32_t scale = f8_scale(max(max(part[0], part[1]), max(part[2], part[3])), FORMAT);
    const uint2 nans = f8_nans(p.cols - t.c);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (t.r + e >= p.rows) continue;
        float v[8];
        E::floats(raw[e], v);
        *(uint2 *)(p.q + (t.r + e) * p.ld_q + t.c) = f8_quantized8<FORMAT>(v, scale, nans);
    }
    put_scale(p.scale + tile_r * p.ld_scale, tile_c, across, threadIdx.x, scale);
}

// Back: eight values a thread.
template <int DT, bool WIDE>
__device__ __forceinline__ void dequantize_chunks(const F8QuantizeArgs &p, int64_t chunks, int64_t total, uint32_t group, uint32_t groups)
{
    const int64_t first = (int64_t)group * 256 + threadIdx.x, step = (int64_t)groups * 256;
    const int shift = p.block == 1 ? 0 : 7;
    for (int64_t at = first; at < total; at += kTurns * step) {
        uint2 q[kTurns];
        uint32_t s[kTurns];
        int64_t row[kTurns], col[kTurns];
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int64_t i = at + k * step;
            if (i >= total) continue;
            row[k] = total < (1ll << 31) ? (int64_t)((uint32_t)i / (uint32_t)chunks) : i / chunks;
            col[k] = (i - row[k] * chunks) * 8;
            q[k] = *(const uint2 *)(p.q + row[k] * p.ld_q + col[k]);
            s[k] = p.scale[(row[k] >> shift) * p.ld_scale + (col[k] >> 7)];
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            if (at + k * step >= total) continue;
            float v[8];
            f8_values8(q[k], s[k], p.format, v);
            store8<DT, WIDE>((typename Elem<DT>::type *)p.out + row[k] * p.ld_x, col[k], p.cols, v);
        }
    }
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void dequantize_f8_kernel(F8QuantizeArgs p, int64_t chunks, int64_t total)
{
    dequantize_chunks<DT, WIDE>(p, chunks, total, blockIdx.x, gridDim.x);
}

// The operands of a product in float32 as bf16, in one launch: x of floats (rounded to e4m3) or of 8-bit floats, and w.  (333 x 1001 -> 777: 13.7 us; in two launches with a quarter
// of the workgroups 17.9, in one with so few 16.6.)
template <bool FLOATS, bool WIDE>
__global__ __launch_bounds__(256) void widen_f8_kernel(F8QuantizeArgs x, F8QuantizeArgs w, uint32_t x_groups)
{
    if (blockIdx.x >= x_groups) {
        const int64_t chunks = w.cols / 8;
        dequantize_chunks<TICTAC_BF16, true>(w, chunks, chunks * w.rows, blockIdx.x - x_groups, gridDim.x - x_groups);
    } else if constexpr (FLOATS) {
        const int64_t blocks = f8_blocks(x.cols);
        quantize_blocks<TICTAC_F32, WIDE, TICTAC_E4M3, true>(x, blocks, blocks * x.rows, blockIdx.x, x_groups);
    } else {
        const int64_t chunks = x.cols / 8;
        dequantize_chunks<TICTAC_BF16, true>(x, chunks, chunks * x.rows, blockIdx.x, x_groups);
    }
}

// Workgroups for `n` times what one has at once: a turn each while few of them run, then kTurns, then more turns for all.  (333 x 1001: a turn each 4.4 us, four 7.6.)
static unsigned groups_of(int64_t n)
{
    constexpr int64_t kFew = 1024, kMost = 256 * 16;
    return (unsigned)std::min(kMost, std::max<int64_t>({1, (n + kTurns - 1) / kTurns, std::min(n, kFew)}));
}

template <int DT, bool WIDE>
static hipError_t quantize(const F8QuantizeArgs &p, hipStream_t s)
{
    const int64_t blocks = f8_blocks(p.cols);
    const bool e5 = p.format == TICTAC_E5M2;
    if (p.block == 1) {
        const int64_t total = blocks * p.rows;
        const auto kernel = e5 ? quantize_f8_kernel<DT, WIDE, TICTAC_E5M2> : quantize_f8_kernel<DT, WIDE, TICTAC_E4M3>;
        hipLaunchKernelGGL(kernel, dim3(groups_of((total + 15) / 16)), dim3(256), 0, s, p, blocks, total);
    } else {
        const auto kernel = e5 ? quantize_f8_tiles_kernel<DT, WIDE, TICTAC_E5M2> : quantize_f8_tiles_kernel<DT, WIDE, TICTAC_E4M3>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks * f8_blocks(p.rows))), dim3(256), 0, s, p, (uint32_t)blocks);
    }
    return hipGetLastError();
}

template <int DT, bool WIDE>
static hipError_t dequantize(const F8QuantizeArgs &p, hipStream_t s)
{
    const int64_t chunks = (p.cols + 7) / 8, total = chunks * p.rows;
    hipLaunchKernelGGL((dequantize_f8_kernel<DT, WIDE>), dim3(groups_of((total + 255) / 256)), dim3(256), 0, s, p, chunks, total);
    return hipGetLastError();
}

hipError_t launch_quantize_f8(const F8QuantizeArgs &p, hipStream_t s)
{
    return BY_TYPE(p.dtype, wide_rows(p.x, p.dtype, p.ld_x, p.cols), quantize, p, s);
}
hipError_t launch_dequantize_f8(const F8QuantizeArgs &p, hipStream_t s) { return BY_TYPE(p.dtype, wide_rows(p.out, p.dtype, p.ld_x, p.cols), dequantize, p, s); }

hipError_t launch_widen_f8(const F8QuantizeArgs &x, const F8QuantizeArgs &w, hipStream_t s)
{
    const unsigned x_groups = groups_of(x.x ? (f8_blocks(x.cols) * x.rows + 15) / 16 : (x.cols / 8 * x.rows + 255) / 256), w_groups = groups_of((w.cols / 8 * w.rows + 255) / 256);
    const auto kernel = !x.x ? widen_f8_kernel<false, true> : wide_rows(x.x, TICTAC_F32, x.ld_x, x.cols) ? widen_f8_kernel<true, true> : widen_f8_kernel<true, false>;
    hipLaunchKernelGGL(kernel, dim3(x_groups + w_groups), dim3(256), 0, s, x, w, x_groups);
    return hipGetLastError();
}

// ---- the operands of a backward pass ----
// A workgroup has a tile of 128 x 128 of dy, of x or of w as floats in registers; blocks of its rows are maxima over 16 lanes, those of its columns meet in LDS, through which they are
// turned round too, so that reads and writes are whole lines.  BF16: the values that 8 bits keep, as bf16.  Bound by memory where there is much: the operands of 8192 x 4096 -> 16384
// bfloat16 take 139 us, 5.4 TB/s; small ones by one trip there and three barriers, 7 us.
template <int N>
struct TurnRoom {
    uint32_t part[128 / N][128];        // maxima, sums
    uint8_t scale[128];
};

// v: N x 8 of a tile; the blocks of its columns go to `to`, [columns][ld], in the format
template <bool BF16, int FORMAT, int N>
__device__ __forceinline__ void put_columns(const Tile128<N> &t, const float (&v)[N][8], int64_t rows, int64_t cols, int64_t tile_r, int64_t tile_c, const F8Operand &to,
                                            TurnRoom<N> &room, char *turned)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) m = max(m, magnitude(v[e][i]));
        room.part[t.group][t.lane * 8 + i] = m;
    }
    __syncthreads();
    if (threadIdx.x < 128) {
        uint32_t m = 0;
#pragma unroll
        for (int g = 0; g < 128 / N; ++g) m = max(m, room.part[g][threadIdx.x]);
        const uint32_t scale = f8_scale(m, FORMAT);
        room.scale[threadIdx.x] = (uint8_t)scale;
        const int64_t c = tile_c * 128 + threadIdx.x;
        if (!BF16 && c < cols) to.scale[c * to.ld_scale + tile_r] = (uint8_t)scale;
    }
    __syncthreads();
    const uint2 nans = f8_nans(rows - t.r);
    // Eight rows of a column are one piece; piece g of column c lies at place g ^ c / 8 of its 16: a wave's stores and loads then meet all banks alike.
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float u[N];
        const uint32_t scale = room.scale[t.lane * 8 + i];
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = v[e][i];
        const int at = (t.lane * 8 + i) * 16 + ((t.group * N / 8) ^ t.lane);
        if constexpr (N == 8) {
            const uint2 q = f8_quantized8<FORMAT>(u, scale, nans);
            if (BF16) {
                f8_values8(q, scale, FORMAT, u);
                *(i32x4 *)(turned + at * 16) = f8_bf16(u);
            } else {
                *(uint2 *)(turned + at * 8) = q;
            }
        } else {                                                        // (half a piece)
            const uint32_t q = f8_quantized4<FORMAT>(u, scale, nans.x);
            if (BF16) {
                f8_values4(q, FORMAT, u);
                const float s = f8_factor(scale);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] *= s;
                *(uint2 *)(turned + at * 16 + (t.group & 1) * 8) = f8_bf16_4(u);
            } else {
                *(uint32_t *)(turned + at * 8 + (t.group & 1) * 4) = q;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < (BF16 ? N : N / 2); ++k) {
        const int n = k * Tile128<N>::kThreads + threadIdx.x, c = n / (BF16 ? 16 : 8), piece = n % (BF16 ? 16 : 8), lane = c >> 3;
        if (tile_c * 128 + c >= cols) continue;
        if (BF16) {
            *(i32x4 *)((uint16_t *)to.q + (tile_c * 128 + c) * to.ld + tile_r * 128 + piece * 8) = *(const i32x4 *)(turned + (c * 16 + (piece ^ lane)) * 16);
        } else {
            const i32x4 two = *(const i32x4 *)(turned + (c * 16 + ((2 * piece ^ lane) & ~1)) * 8);
            *(i32x4 *)((uint8_t *)to.q + (tile_c * 128 + c) * to.ld + tile_r * 128 + piece * 16) = lane & 1 ? i32x4{two[2], two[3], two[0], two[1]} : two;
        }
    }
}

template <int DT, bool WIDE, int FORMAT, int N>
__global__ __launch_bounds__(Tile128<N>::kThreads) void turn_f8_kernel(F8TurnArgs p, uint32_t dy_tiles, uint32_t x_tiles)
{
    using E = Elem<DT>;
    constexpr bool BF16 = DT == TICTAC_F32;
    __shared__ TurnRoom<N> room;
    __shared__ __align__(16) char turned[128 * 16 * (BF16 ? 16 : 8)];
    uint32_t unit = blockIdx.x;
    float v[N][8];
    if (unit < dy_tiles) {
        const uint32_t across = (uint32_t)((p.outs + 127) / 128), tile_r = unit / across, tile_c = unit % across;
        const Tile128<N> t(tile_r, tile_c);
        {
            typename E::raw raw[N];
            load_tile<DT, WIDE, N>(p.dy, p.ld_dy, p.rows, p.outs, t, raw);
#pragma unroll
            for (int e = 0; e < N; ++e) E::floats(raw[e], v[e]);
        }
        if (p.dy_rows.q) {
            const uint2 nans = f8_nans(p.outs - t.c);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[e][i]));
                const uint32_t scale = f8_scale(row16_max(m), FORMAT);
                if (t.r + e >= p.rows) continue;
                const uint2 q = f8_quantized8<FORMAT>(v[e], scale, nans);
                const int64_t at = (t.r + e) * p.dy_rows.ld + t.c;
                if (BF16) {
                    float u[8];
                    f8_values8(q, scale, FORMAT, u);
                    *(i32x4 *)((uint16_t *)p.dy_rows.q + at) = f8_bf16(u);
                } else {
                    *(uint2 *)((uint8_t *)p.dy_rows.q + at) = q;
                    if (t.lane == 0) p.dy_rows.scale[(t.r + e) * p.dy_rows.ld_scale + tile_c] = (uint8_t)scale;
                }
            }
        }
        if (p.sums) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) sum += v[e][i];
                room.part[t.group][t.lane * 8 + i] = __builtin_bit_cast(uint32_t, sum);
            }
            __syncthreads();
            const int64_t c = tile_c * 128 + threadIdx.x;
            if (threadIdx.x < 128 && c < p.outs) {
                float sum = 0.0f;
#pragma unroll
                for (int g = 0; g < 128 / N; ++g) sum += __builtin_bit_cast(float, room.part[g][threadIdx.x]);
                p.sums[tile_r * p.outs + c] = sum;
            }
            __syncthreads();
        }
        if (p.dy_cols.q) put_columns<BF16, FORMAT, N>(t, v, p.rows, p.outs, tile_r, tile_c, p.dy_cols, room, turned);
        return;
    }
    unit -= dy_tiles;
    const bool is_x = unit < x_tiles;
    if (!is_x) unit -= x_tiles;
    const F8Rows &from = is_x ? p.x : p.w;
    const int64_t rows = is_x ? p.rows : p.outs;
    const uint32_t across = (uint32_t)((p.cols + 127) / 128), tile_r = unit / across, tile_c = unit % across;
    const Tile128<N> t(tile_r, tile_c);
    uint2 q[N];
    uint32_t scale[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int64_t row = min(t.r + e, rows - 1);
        q[e] = *(const uint2 *)(from.q + row * from.ld + t.c);
        scale[e] = from.scale[(row >> from.shift) * from.ld_scale + tile_c];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const bool in = t.r + e < rows;
        f8_values8(uint2{in ? q[e].x : 0, in ? q[e].y : 0}, in ? scale[e] : 127, from.format, v[e]);
    }
    put_columns<BF16, TICTAC_E4M3, N>(t, v, rows, p.cols, tile_r, tile_c, is_x ? p.x_cols : p.w_cols, room, turned);
}

// Up to a tile per compute unit by workgroups of 512: what bounds them is each wave's own code.  (us of a gradient by 512 and by 256: 30 x 300 -> 200 bfloat16 9.7 and 10.5, 64 x 1024 -> 1000 11.9 and
// 12.5, 8192 x 4096 -> 4096 247 and 243.)
constexpr int64_t kFewTurns = 256;

template <int DT, bool WIDE>
static hipError_t turn(const F8TurnArgs &p, hipStream_t s)
{
    const int64_t dy = p.dy_rows.q || p.dy_cols.q || p.sums ? f8_blocks(p.rows) * f8_blocks(p.outs) : 0, x = p.x_cols.q ? f8_blocks(p.rows) * f8_blocks(p.cols) : 0,
                  w = p.w_cols.q ? f8_blocks(p.outs) * f8_blocks(p.cols) : 0;
    if (dy + x + w == 0) return hipSuccess;
    const bool few = dy + x + w <= kFewTurns;
    const auto kernel = p.format == TICTAC_E5M2 ? (few ? turn_f8_kernel<DT, WIDE, TICTAC_E5M2, 4> : turn_f8_kernel<DT, WIDE, TICTAC_E5M2, 8>)
                                                : (few ? turn_f8_kernel<DT, WIDE, TICTAC_E4M3, 4> : turn_f8_kernel<DT, WIDE, TICTAC_E4M3, 8>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(dy + x + w)), dim3(few ? 512 : 256), 0, s, p, (uint32_t)dy, (uint32_t)x);
    return hipGetLastError();
}
hipError_t launch_turn_f8(const F8TurnArgs &p, hipStream_t s) { return BY_TYPE(p.dtype, wide_rows(p.dy, p.dtype, p.ld_dy, p.outs), turn, p, s); }

}  // namespace tictac
