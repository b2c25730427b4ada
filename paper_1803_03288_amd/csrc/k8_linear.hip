// A layer with 8-bit weights, y[t][o] = xs[t] ws[o] sum_i xq[t][i] w[o][i] + bias[o], and its gradients
//   dx[t][i] = sum_o (dy[t][o] ws[o]) w[o][i],   dw[o][i] = sum_t (dy[t][o] xs[t]) xq[t][i],   db[o] = sum_t dy[t][o]
// Forward: sums exact in int32.  Backward: int8 values are exact in bf16; dy times a scale, a float32 value, is cut into as many bf16
// pieces as dy's type has bits to give (bf16 one, rounded once as dy itself was; float16 two; float32 three, exact), and the pieces go side by
// side along k through the one product of k8_product.hip; sums in float32.
#include "k8_product.h"

namespace tictac {

// ---- few rows: bound by the bytes of the weights ----
// A workgroup has 16 outputs, its eight waves an eighth of k each: weights go from memory to the matrix instruction without LDS, sixteen bytes per
// lane, eight loads under way.  TB blocks of 16 rows of x.  The sums of the waves meet in LDS.
constexpr int kFewWaves = 8;

template <int TB>
__global__ __launch_bounds__(kFewWaves * 64) void linear_few_kernel(LinearArgs p, const int8_t *xq, int64_t ld_xq, const float *xs)
{
    __shared__ i32x4 sums[kFewWaves][TB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, fk = (lane >> 4) * 16;
    const int64_t o0 = (int64_t)blockIdx.x * 16;
    const int32_t units = (int32_t)((p.cols + 127) / 128);
    const int8_t *w = p.w + min(o0 + row, p.outs - 1) * p.ld_w + fk;
    const int8_t *x[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) x[b] = xq + min((int64_t)b * 16 + row, p.rows - 1) * ld_xq + fk;
    i32x4 acc[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[b] = i32x4{};
    int32_t u = wave;
    for (; u + 3 * kFewWaves < units; u += 4 * kFewWaves) {
        i32x4 fw[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) fw[k] = __builtin_nontemporal_load((const i32x4 *)(w + (int64_t)(u + (k >> 1) * kFewWaves) * 128 + (k & 1) * 64));
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int b = 0; b < TB; ++b)
                acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[k], *(const i32x4 *)(x[b] + (int64_t)(u + (k >> 1) * kFewWaves) * 128 + (k & 1) * 64), acc[b], 0, 0, 0);
    }
    for (; u < units; u += kFewWaves)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const i32x4 fw = *(const i32x4 *)(w + (int64_t)u * 128 + k * 64);
#pragma unroll
            for (int b = 0; b < TB; ++b)
                acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, *(const i32x4 *)(x[b] + (int64_t)u * 128 + k * 64), acc[b], 0, 0, 0);
        }
#pragma unroll
    for (int b = 0; b < TB; ++b) sums[wave][b][lane] = acc[b];
    __syncthreads();
    // lane l of a block holds outputs 4 (l / 16) .. + 3 of row l % 16; a thread finishes one output
    for (int i = threadIdx.x; i < TB * 256; i += kFewWaves * 64) {
        const int b = i >> 8, o = i & 15, t = (i >> 4) & 15;
        int32_t sum = 0;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) sum += sums[k][b][(o >> 2) * 16 + t][o & 3];
        const int64_t at = (int64_t)b * 16 + t;
        if (at >= p.rows || o0 + o >= p.outs) continue;
        float v = (float)sum * (xs[at] * p.ws[o0 + o]);
        if (p.bias) v += param(p.bias, p.bias_dtype, o0 + o);
        put_param(p.y, p.dtype, at * p.ld_y + o0 + o, v);
    }
}

constexpr int64_t kFewRows = 64;

size_t linear_q8_workspace(int32_t from_floats, int64_t rows, int64_t cols, int64_t outs)
{
    size_t bytes = 0;
    if (from_floats) bytes += (size_t)rows * rows8_stride(cols) + ((size_t)rows * 4 + 255) / 256 * 256;
    if (rows > kFewRows) bytes += product_parts_bytes(product_splits((int32_t)outs, (int32_t)rows, (int32_t)(rows8_stride(cols) / 128)), (int32_t)outs, (int32_t)rows);
    return bytes;
}

hipError_t launch_linear_q8(const LinearArgs &p, hipStream_t s)
{
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
    if (p.rows <= kFewRows) {
        const dim3 grid((unsigned)((p.outs + 15) / 16)), block(kFewWaves * 64);
        if (p.rows <= 16) hipLaunchKernelGGL(linear_few_kernel<1>, grid, block, 0, s, p, xq, ld_xq, xs);
        else if (p.rows <= 32) hipLaunchKernelGGL(linear_few_kernel<2>, grid, block, 0, s, p, xq, ld_xq, xs);
        else hipLaunchKernelGGL(linear_few_kernel<4>, grid, block, 0, s, p, xq, ld_xq, xs);
        return hipGetLastError();
    }
    ProductArgs a{};
    a.p = (const char *)p.w; a.ld_p = p.ld_w;
    a.q = (const char *)xq; a.ld_q = ld_xq;
    a.R = (int32_t)p.outs; a.C = (int32_t)p.rows;
    a.steps = a.p_steps = (int32_t)(rows8_stride(p.cols) / 128);
    a.splits = product_splits(a.R, a.C, a.steps);
    a.out = p.y; a.ld_out = p.ld_y; a.dtype = p.dtype;
    a.p_scale = p.ws; a.q_scale = xs; a.bias = p.bias; a.bias_dtype = p.bias_dtype;
    a.parts = room;
    return launch_product_i8(a, s);
}

// ---- backward: operands with k contiguous ----
// Columns of int8 rows as bf16 rows: out[c][r] = q[r][c], zeros for r from `rows` to `padded`.  64 x 64 through LDS.
__global__ __launch_bounds__(256) void transpose_rows8_kernel(int64_t rows, int64_t cols, const int8_t *q, int64_t ld, __bf16 *out, int64_t padded)
{
    __shared__ uint16_t tile[64][66];                           // (33 words a row: a column lies in all banks)
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    {
        const int64_t r = r0 + (threadIdx.x >> 2);
        const int c = (threadIdx.x & 3) * 16;
        i32x4 v{};
        if (r < rows) v = *(const i32x4 *)(q + r * ld + c0 + c);         // (c0 + 64 <= ld: rows are padded to 128)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float f = (float)((v[i >> 2] << (24 - 8 * (i & 3))) >> 24);
            tile[threadIdx.x >> 2][c + i] = (uint16_t)(__builtin_bit_cast(uint32_t, f) >> 16);      // (exact: eight bits)
        }
    }
    __syncthreads();
    const int64_t c = c0 + (threadIdx.x >> 2);
    const int r = (threadIdx.x & 3) * 16;
    if (c >= cols) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        i32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = tile[r + h * 8 + 2 * i][threadIdx.x >> 2] | (uint32_t)tile[r + h * 8 + 2 * i + 1][threadIdx.x >> 2] << 16;
        *(i32x4 *)(out + c * padded + r0 + r + h * 8) = w;
    }
}

// dy times a scale in PIECES bf16 values that add up to it: all but the last cut off, which leaves the rest exact, the last rounded.
template <int PIECES>
__device__ __forceinline__ void cut(float v, uint16_t *piece)
{
#pragma unroll
    for (int k = 0; k < PIECES - 1; ++k) {
        const uint32_t high = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
        piece[k] = (uint16_t)(high >> 16);
        v -= __builtin_bit_cast(float, high);
    }
    const __bf16 last = (__bf16)v;
    piece[PIECES - 1] = __builtin_bit_cast(uint16_t, last);
}

// out[t][piece][o] = pieces of dy[t][o] ws[o], zeros for o from `outs` to `padded`
template <int DT, int PIECES>
__global__ __launch_bounds__(256) void scaled_rows_kernel(int64_t rows, int64_t outs, const void *dy, int64_t ld_dy, const float *ws, uint16_t *out, int64_t padded)
{
    using E = Elem<DT>;
    const int64_t o = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (o >= padded) return;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = o + i < outs ? ws[o + i] : 0.0f;
    for (int64_t t = blockIdx.y; t < rows; t += gridDim.y) {
        const typename E::type *row = (const typename E::type *)dy + t * ld_dy;
        float v[8];
        if (o + 8 <= outs && ((uintptr_t)(row + o) & 15) == 0) {
            E::floats(E::load(row + o), v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = o + i < outs ? E::to_float(row[o + i]) : 0.0f;
        }
        uint16_t c[8][PIECES];
#pragma unroll
        for (int i = 0; i < 8; ++i) cut<PIECES>(v[i] * s[i], c[i]);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            i32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = c[2 * i][k] | (uint32_t)c[2 * i + 1][k] << 16;
            *(i32x4 *)(out + (t * PIECES + k) * padded + o) = w;
        }
    }
}

// out[o][piece][t] = pieces of dy[t][o] xs[t], zeros for t from `rows` to `padded`; sums of dy over each 64 rows.
template <int DT, int PIECES>
__global__ __launch_bounds__(256) void scaled_columns_kernel(int64_t rows, int64_t outs, const void *dy, int64_t ld_dy, const float *xs, uint16_t *out, int64_t padded, float *sums)
{
    using E = Elem<DT>;
    using T = typename E::type;
    __shared__ float tile[64][65];
    const int64_t t0 = (int64_t)blockIdx.y * 64, o0 = (int64_t)blockIdx.x * 64;
    const int o = threadIdx.x & 63, quarter = threadIdx.x >> 6;
    for (int i = quarter; i < 64; i += 4)
        tile[i][o] = t0 + i < rows && o0 + o < outs ? E::to_float(((const T *)dy)[(t0 + i) * ld_dy + o0 + o]) : 0.0f;
    __syncthreads();
    if (sums && quarter == 0 && o0 + o < outs) {
        float sum = 0.0f;
        for (int i = 0; i < 64; ++i) sum += tile[i][o];
        sums[(int64_t)blockIdx.y * outs + o0 + o] = sum;
    }
    if (!out) return;
    const int row = threadIdx.x >> 2, t = (threadIdx.x & 3) * 16;
    if (o0 + row >= outs) return;
    uint16_t c[16][PIECES];
#pragma unroll
    for (int i = 0; i < 16; ++i) cut<PIECES>(t0 + t + i < rows ? tile[t + i][row] * xs[t0 + t + i] : 0.0f, c[i]);
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = c[h * 8 + 2 * i][k] | (uint32_t)c[h * 8 + 2 * i + 1][k] << 16;
            *(i32x4 *)(out + ((o0 + row) * PIECES + k) * padded + t0 + t + h * 8) = w;
        }
}

// Adds up the sums of 64 rows each in their order.
__global__ __launch_bounds__(1024) void column_sums_kernel(int64_t parts, int64_t outs, const float *sums, void *db, int32_t dt)
{
    __shared__ float shared[16][64];
    const int64_t o = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int wave = threadIdx.x >> 6;
    const int64_t per = (parts + 15) / 16;
    float sum = 0.0f;
    if (o < outs)
        for (int64_t k = wave * per; k < min(parts, (wave + 1) * per); ++k) sum += sums[k * outs + o];
    shared[wave][threadIdx.x & 63] = sum;
    __syncthreads();
    if (wave || o >= outs) return;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += shared[k][threadIdx.x & 63];
    put_param(db, dt, o, sum);
}

static int pieces_of(int32_t dtype) { return dtype == TICTAC_F32 ? 3 : dtype == TICTAC_F16 ? 2 : 1; }

// The workspace of one backward call; the two products come one after the other and use the same room.
struct BackwardRoom {
    int64_t padded_o, padded_t;
    size_t sums, p, q, parts, bytes;            // offsets
};
static BackwardRoom backward_room(int32_t dtype, int64_t rows, int64_t cols, int64_t outs)
{
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const int pieces = pieces_of(dtype);
    BackwardRoom r{};
    r.padded_o = (outs + 63) / 64 * 64;
    r.padded_t = (rows + 63) / 64 * 64;
    r.sums = 0;
    r.p = up((size_t)(r.padded_t / 64) * outs * 4);
    const size_t p = (size_t)cols * (r.padded_o > r.padded_t ? r.padded_o : r.padded_t) * 2;
    const size_t qx = (size_t)rows * r.padded_o * pieces * 2, qw = (size_t)outs * r.padded_t * pieces * 2;
    r.q = r.p + up(p);
    r.parts = r.q + up(qx > qw ? qx : qw);
    const size_t px = product_parts_bytes(product_splits((int32_t)cols, (int32_t)rows, (int32_t)(r.padded_o / 64 * pieces)), (int32_t)cols, (int32_t)rows);
    const size_t pw = product_parts_bytes(product_splits((int32_t)cols, (int32_t)outs, (int32_t)(r.padded_t / 64 * pieces)), (int32_t)cols, (int32_t)outs);
    r.bytes = r.parts + up(px > pw ? px : pw);
    return r;
}
size_t linear_q8_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t outs) { return backward_room(dtype, rows, cols, outs).bytes; }

template <int DT, int PIECES>
static hipError_t backward(const LinearArgs &p, hipStream_t s)
{
    const BackwardRoom room = backward_room(DT, p.rows, p.cols, p.outs);
    char *at = (char *)p.workspace;
    ProductArgs a{};
    a.p = at + room.p;
    a.q = at + room.q;
    a.R = (int32_t)p.cols;
    a.dtype = DT;
    a.parts = at + room.parts;
    if (p.dx && p.rows) {
        if (p.outs) {
            hipLaunchKernelGGL(transpose_rows8_kernel, dim3((unsigned)((p.cols + 63) / 64), (unsigned)(room.padded_o / 64)), dim3(256), 0, s, p.outs, p.cols, p.w, p.ld_w,
                               (__bf16 *)a.p, room.padded_o);
            hipLaunchKernelGGL((scaled_rows_kernel<DT, PIECES>), dim3((unsigned)((room.padded_o + 2047) / 2048), (unsigned)(p.rows < 4096 ? p.rows : 4096)), dim3(256), 0, s, p.rows, p.outs,
                               p.dy, p.ld_dy, p.ws, (uint16_t *)a.q, room.padded_o);
        }
        a.ld_p = room.padded_o * 2;
        a.ld_q = room.padded_o * 2 * PIECES;
        a.C = (int32_t)p.rows;
        a.p_steps = (int32_t)(room.padded_o / 64);
        a.steps = a.p_steps * PIECES;
        a.splits = product_splits(a.R, a.C, a.steps);
        a.out = p.dx;
        a.ld_out = p.ld_dx;
        if (const hipError_t e = launch_product_bf16(a, s); e != hipSuccess) return e;
    }
    if (p.outs && (p.dw || p.db)) {
        float *sums = (float *)(at + room.sums);
        if (p.rows)
            hipLaunchKernelGGL((scaled_columns_kernel<DT, PIECES>), dim3((unsigned)((p.outs + 63) / 64), (unsigned)(room.padded_t / 64)), dim3(256), 0, s, p.rows, p.outs, p.dy, p.ld_dy,
                               p.xs, p.dw ? (uint16_t *)a.q : nullptr, room.padded_t, p.db ? sums : nullptr);
        if (p.db)
            hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((p.outs + 63) / 64)), dim3(1024), 0, s, room.padded_t / 64, p.outs, sums, p.db, p.dtype);
    }
    if (p.dw && p.outs) {
        if (p.rows)
            hipLaunchKernelGGL(transpose_rows8_kernel, dim3((unsigned)((p.cols + 63) / 64), (unsigned)(room.padded_t / 64)), dim3(256), 0, s, p.rows, p.cols, p.xq, p.ld_xq,
                               (__bf16 *)a.p, room.padded_t);
        a.ld_p = room.padded_t * 2;
        a.ld_q = room.padded_t * 2 * PIECES;
        a.C = (int32_t)p.outs;
        a.p_steps = (int32_t)(room.padded_t / 64);
        a.steps = a.p_steps * PIECES;
        a.splits = product_splits(a.R, a.C, a.steps);
        a.out = p.dw;
        a.ld_out = p.ld_dw;
        if (const hipError_t e = launch_product_bf16(a, s); e != hipSuccess) return e;
    }
    return hipGetLastError();
}

hipError_t launch_linear_q8_backward(const LinearArgs &p, hipStream_t s)
{
    if (p.dtype == TICTAC_F32) return backward<TICTAC_F32, 3>(p, s);
    return p.dtype == TICTAC_F16 ? backward<TICTAC_F16, 2>(p, s) : backward<TICTAC_BF16, 1>(p, s);
}

}  // namespace tictac
