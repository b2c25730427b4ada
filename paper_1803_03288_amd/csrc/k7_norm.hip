// Layer norm over the rows of x:
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd w + b
// and its gradients, with xh = (x - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
// Statistics and sums in float32, from a row held in registers: the variance is that of the differences from the mean, not a
// difference of large sums.  The output can be 8-bit rows with a scale per row (the operand of the product that follows), and the
// input can be kept in 8 bits from the same pass; the backward pass takes the input itself or those 8-bit rows.
// Bound by memory: a row is read once and stays in registers; the parameters stay there from row to row.  8192 x 4096 bfloat16 with its saved rows: 34 us,
// 5.0 TB/s; gradients of 16384 x 4096 from saved rows: 68 us, 5.0 TB/s, and 5 for the second kernel; one row: 3 us.
#include <algorithm>

#include "rows8.h"

// Which products and sums are one operation is written out (fmaf): the kernels for rows on and off 16-byte boundaries, for a wave and for a
// workgroup then give the same bits.
#pragma clang fp contract(off)

namespace tictac {

// Sums and maxima over the threads of a row: a wave, or a workgroup through LDS.  Two sets of cells in turn, so that one barrier a
// reduction is enough.
template <int THREADS>
struct RowReduce {
    static constexpr int kWaves = THREADS / 64;
    float (*cells)[2][kWaves];          // LDS, [2][2][kWaves]
    int turn = 0;
    __device__ __forceinline__ void sum2(float &a, float &b)
    {
        a = wave_sum_f32(a);
        b = wave_sum_f32(b);
        if (THREADS == 64) return;
        if ((threadIdx.x & 63) == 0) { cells[turn][0][threadIdx.x >> 6] = a; cells[turn][1][threadIdx.x >> 6] = b; }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) { a += cells[turn][0][i]; b += cells[turn][1][i]; }
        turn ^= 1;
    }
    __device__ __forceinline__ float sum(float a)
    {
        a = wave_sum_f32(a);
        if (THREADS == 64) return a;
        if ((threadIdx.x & 63) == 0) cells[turn][0][threadIdx.x >> 6] = a;
        __syncthreads();
        a = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) a += cells[turn][0][i];
        turn ^= 1;
        return a;
    }
    __device__ __forceinline__ uint32_t max(uint32_t m)
    {
        m = wave_max_u32(m);
        if (THREADS == 64) return m;
        if ((threadIdx.x & 63) == 0) cells[turn][0][threadIdx.x >> 6] = __builtin_bit_cast(float, m);
        __syncthreads();
        m = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) m = ::max(m, __builtin_bit_cast(uint32_t, cells[turn][0][i]));
        turn ^= 1;
        return m;
    }
};

// Threads per row and chunks of eight columns per thread: a wave holds up to 1 024 columns (forward, in whole eights,
// 1 536: 16000 x 1536 bfloat16 17.3 us, by four waves 21.8), four waves 4 096, eight 8 192 (6000 x 5368 float16 with its saved
// rows: 56 us; by four waves 65, by sixteen 74), sixteen 16 384 (the backward pass keeps dw and db of those in LDS).  Longer rows are read several times (norm_long_kernel).
constexpr int64_t kLongest = 16384;

template <int THREADS>
struct RowShape {
    static constexpr int kBlock = THREADS < 256 ? 256 : THREADS;        // threads of a workgroup
    static constexpr int kRows = kBlock / THREADS;                      // rows it has under way
};

template <int DT, bool WIDE, int THREADS, int NC>
__global__ __launch_bounds__(RowShape<THREADS>::kBlock, 4) void layer_norm_kernel(NormArgs p)
{
    using E = Elem<DT>;
    using T = typename E::type;
    constexpr int kRows = RowShape<THREADS>::kRows;
    __shared__ float cells[2][2][RowReduce<THREADS>::kWaves];
    RowReduce<THREADS> r{cells};
    const int t = threadIdx.x % THREADS;
    const int64_t cols = p.cols, padded = (cols + 127) / 128 * 128, groups = padded / 128;
    const float per = 1.0f / (float)cols;
    float w[NC][8], b[NC][8];
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) { w[j][i] = 1.0f; b[j][i] = 0.0f; }
    if (p.weight) params_at_once<THREADS, NC>(p.weight, p.param_dtype, t * 8, cols, w);
    if (p.bias) params_at_once<THREADS, NC>(p.bias, p.param_dtype, t * 8, cols, b);
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS; row < p.rows; row += (int64_t)gridDim.x * kRows) {
        float v[NC][8];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            E::floats(load8<DT, WIDE>((const T *)p.x + row * p.ld_x, (int64_t)(j * THREADS + t) * 8, cols), v[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[j][i];
        }
        if (p.xq) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t col = (int64_t)(j * THREADS + t) * 8;
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[j][i]));
                const RowScale s = row_scale(row16_max(m));
                if (col >= padded) continue;
                *(uint2 *)(p.xq + row * p.ld_xq + col) = quantized8(v[j], s);
                if ((t & 15) == 0) p.xs[row * groups + (col >> 7)] = s.scale;
            }
        }
        const float mean = r.sum(sum) * per;
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t col = (int64_t)(j * THREADS + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = col + i < cols ? v[j][i] - mean : 0.0f;
                v[j][i] = d;
                sq = fmaf(d, d, sq);
            }
        }
        const float rstd = 1.0f / sqrtf(fmaf(r.sum(sq), per, p.eps));
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t col = (int64_t)(j * THREADS + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[j][i] = col + i < cols ? fmaf(v[j][i] * rstd, w[j][i], b[j][i]) : 0.0f;
                m = max(m, magnitude(v[j][i]));
            }
            if (p.y) store8<DT, WIDE>((T *)p.y + row * p.ld_y, col, cols, v[j]);
        }
        if (p.yq) {
            const RowScale s = row_scale(r.max(m));
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t col = (int64_t)(j * THREADS + t) * 8;
                if (col < padded) *(uint2 *)(p.yq + row * p.ld_yq + col) = quantized8(v[j], s);
            }
            if (t == 0) p.ys[row] = s.scale;
        }
        if (t == 0) { p.mean[row] = mean; p.rstd[row] = rstd; }
    }
}

// ---- rows of any length: read again for every step, which the caches serve (512 x 65536 bfloat16 with its saved rows: 56 us) ----
// A thread's sum over such a row, eight columns at a time: what each addition rounds off is kept beside it (exactly: a + b = t + e), so that the sum is as
// near as one of 64 additions at any length.  Added one after the other, 2^22 values of 0.1 give a mean that is off by 4e-5 of it.
struct LongSum {
    float sum = 0.0f, low = 0.0f;
    __device__ __forceinline__ void add(float v)
    {
        const float t = sum + v, b = t - sum;
        low += (sum - (t - b)) + (v - b);
        sum = t;
    }
    __device__ __forceinline__ float value() const { return low - low == 0.0f ? sum + low : sum; }          // (an infinity leaves NaN in low)
};

template <int DT, bool WIDE>
__device__ __forceinline__ void input8(const NormArgs &p, int64_t row, int64_t col, float *v)
{
    Elem<DT>::floats(load8<DT, WIDE>((const typename Elem<DT>::type *)p.x + row * p.ld_x, col, p.cols), v);
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs p)
{
    using T = typename Elem<DT>::type;
    __shared__ float cells[2][2][16];
    RowReduce<1024> r{cells};
    const int64_t cols = p.cols, padded = (cols + 127) / 128 * 128, groups = padded / 128;
    const float per = 1.0f / (float)cols;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        LongSum sum, sq;
        for (int64_t col = threadIdx.x * 8; col < padded; col += 8192) {
            float v[8], eight = 0.0f;
            uint32_t m = 0;
            input8<DT, WIDE>(p, row, col, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) { eight += v[i]; m = max(m, magnitude(v[i])); }
            sum.add(eight);
            if (!p.xq) continue;
            const RowScale s = row_scale(row16_max(m));         // (128 columns: all 16 lanes are in the loop, or none)
            *(uint2 *)(p.xq + row * p.ld_xq + col) = quantized8(v, s);
            if ((threadIdx.x & 15) == 0) p.xs[row * groups + (col >> 7)] = s.scale;
        }
        const float mean = r.sum(sum.value()) * per;
        for (int64_t col = threadIdx.x * 8; col < cols; col += 8192) {
            float v[8], eight = 0.0f;
            input8<DT, WIDE>(p, row, col, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = col + i < cols ? v[i] - mean : 0.0f;
                eight = fmaf(d, d, eight);
            }
            sq.add(eight);
        }
        const float rstd = 1.0f / sqrtf(fmaf(r.sum(sq.value()), per, p.eps));
        uint32_t m = 0;
        RowScale s{0.0f, 0.0f};
        for (int turn = 0; turn < (p.yq ? 2 : 1); ++turn) {     // (the second time with the largest magnitude known)
            for (int64_t col = threadIdx.x * 8; col < padded; col += 8192) {
                float v[8], w[8], b[8];
                input8<DT, WIDE>(p, row, col, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) { w[i] = 1.0f; b[i] = 0.0f; }
                if (p.weight) params8(p.weight, p.param_dtype, col, cols, w);
                if (p.bias) params8(p.bias, p.param_dtype, col, cols, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = col + i < cols ? fmaf((v[i] - mean) * rstd, w[i], b[i]) : 0.0f;
                    m = max(m, magnitude(v[i]));
                }
                if (turn == 0 && p.y) store8<DT, WIDE>((T *)p.y + row * p.ld_y, col, cols, v);
                if (turn == 1) *(uint2 *)(p.yq + row * p.ld_yq + col) = quantized8(v, s);
            }
            if (turn == 0 && p.yq) s = row_scale(r.max(m));
        }
        if (threadIdx.x == 0) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
            if (p.yq) p.ys[row] = s.scale;
        }
    }
}

// ---- backward ----
// A workgroup takes every so many-th row and keeps the sums of its rows for dw and db in registers; they go to the workspace, [workgroup][2][cols],
// and a second kernel adds them up in the order of the workgroups: the same sums at every run, without atomics.
constexpr int64_t kStrips = 512;

template <int DT, bool WIDE, bool SAVED>
struct NormRow {                                    // eight columns of dy and of x as they lie in memory
    typename Elem<DT>::raw dy, x;
    uint2 q;
    float s;
    __device__ __forceinline__ void load(const NormArgs &p, int64_t row, int64_t col, int64_t groups)
    {
        using T = typename Elem<DT>::type;
        dy = load8<DT, WIDE>((const T *)p.dy + row * p.ld_dy, col, p.cols);
        if (!SAVED) {
            x = load8<DT, WIDE>((const T *)p.x + row * p.ld_x, col, p.cols);
        } else if (col < p.cols) {
            q = *(const uint2 *)(p.xq + row * p.ld_xq + col);
            s = p.xs[row * groups + (col >> 7)];
        } else {
            q = uint2{0, 0};
            s = 0.0f;
        }
    }
    // dy, and x - mean with one rounding (where x lies near the mean, that of q * scale alone would be as large as what is left)
    __device__ __forceinline__ void floats(float mean, float *g, float *d) const
    {
        Elem<DT>::floats(dy, g);
        if (!SAVED) Elem<DT>::floats(x, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = SAVED ? fmaf(whole8(q, i), s, -mean) : d[i] - mean;
    }
};

// SUMS: dw and db are asked for; in LDS where the registers do not hold them beside a row (THREADS * NC > 1024): 16 bytes of a thread's own at a time, without
// conflicts and without barriers (3887 x 9264 bfloat16: 54 us, 105 with registers that spill; 3887 x 16384 float32: 177, 294).
constexpr bool sums_in_lds(int threads, int nc) { return threads * nc > 1024; }

template <int DT, bool WIDE, bool SAVED, int THREADS, int NC, bool SUMS>
__device__ __forceinline__ void backward_rows(const NormArgs &p, int32_t blocks)          // the workgroups 0 .. blocks - 1
{
    using T = typename Elem<DT>::type;
    constexpr int kRows = RowShape<THREADS>::kRows;
    constexpr bool kRegisters = SUMS && !sums_in_lds(THREADS, NC);
    extern __shared__ f32x4 lds[];                              // [dw, db][NC][2][THREADS]
    __shared__ float cells[2][2][RowReduce<THREADS>::kWaves];
    __shared__ float join[kRows > 1 ? kRows * 2 * NC * THREADS * 8 : 1];
    RowReduce<THREADS> r{cells};
    const int t = threadIdx.x % THREADS;
    const int64_t cols = p.cols, groups = (cols + 127) / 128, step = (int64_t)blocks * kRows;
    const float per = 1.0f / (float)cols;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
    NormRow<DT, WIDE, SAVED> next[NC];
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (row < p.rows) {
#pragma unroll
        for (int j = 0; j < NC; ++j) next[j].load(p, row, (int64_t)(j * THREADS + t) * 8, groups);
        next_mean = p.mean[row];
        next_rstd = p.rstd[row];
    }
    float w[NC][8], dw[NC][8], db[NC][8];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { w[j][i] = 1.0f; dw[j][i] = db[j][i] = 0.0f; }
        if (SUMS && !kRegisters)
#pragma unroll
            for (int k = 0; k < 4; ++k) lds[((k >> 1) * NC * 2 + j * 2 + (k & 1)) * THREADS + t] = f32x4{};
        if (p.weight) params8(p.weight, p.param_dtype, (int64_t)(j * THREADS + t) * 8, cols, w[j]);
    }
    for (; row < p.rows; row += step) {
        float g[NC][8], xh[NC][8];
        float sum_g = 0.0f, sum_gx = 0.0f;
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t col = (int64_t)(j * THREADS + t) * 8;
            next[j].floats(mean, g[j], xh[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[j][i] = col + i < cols ? xh[j][i] * rstd : 0.0f;
                if (kRegisters) {
                    dw[j][i] = fmaf(g[j][i], xh[j][i], dw[j][i]);
                    db[j][i] += g[j][i];
                }
            }
            if (SUMS && !kRegisters)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    f32x4 &a = lds[(j * 2 + k) * THREADS + t], &b = lds[(NC * 2 + j * 2 + k) * THREADS + t];
                    f32x4 x = a, y = b;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[i] = fmaf(g[j][k * 4 + i], xh[j][k * 4 + i], x[i]);
                        y[i] += g[j][k * 4 + i];
                    }
                    a = x;
                    b = y;
                }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[j][i] *= w[j][i];
                sum_g += g[j][i];
                sum_gx = fmaf(g[j][i], xh[j][i], sum_gx);
            }
        }
        if (row + step < p.rows) {                              // the next row's loads are under way during the sums
#pragma unroll
            for (int j = 0; j < NC; ++j) next[j].load(p, row + step, (int64_t)(j * THREADS + t) * 8, groups);
            next_mean = p.mean[row + step];
            next_rstd = p.rstd[row + step];
        }
        r.sum2(sum_g, sum_gx);
        sum_g *= per;
        sum_gx *= per;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * fmaf(-xh[j][i], sum_gx, g[j][i] - sum_g);
            if (p.dx) store8<DT, WIDE>((T *)p.dx + row * p.ld_dx, (int64_t)(j * THREADS + t) * 8, cols, d);
        }
    }
    if (!SUMS || !p.workspace) return;
    float *part = (float *)p.workspace + (int64_t)blockIdx.x * 2 * cols;
    if (kRows > 1) {                                            // the rows of a workgroup first, in order
        constexpr int kWidth = NC * THREADS * 8;
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                join[(threadIdx.x / THREADS * 2 + 0) * kWidth + (j * THREADS + t) * 8 + i] = dw[j][i];
                join[(threadIdx.x / THREADS * 2 + 1) * kWidth + (j * THREADS + t) * 8 + i] = db[j][i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * kWidth; c += RowShape<THREADS>::kBlock) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kRows; ++k) sum += join[k * 2 * kWidth + c];
            const int col = c % kWidth;
            if (col < cols) part[c / kWidth * cols + col] = sum;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t col = (int64_t)(j * THREADS + t) * 8 + i;
            if (!kRegisters) {
                dw[j][i] = lds[(j * 2 + (i >> 2)) * THREADS + t][i & 3];
                db[j][i] = lds[(NC * 2 + j * 2 + (i >> 2)) * THREADS + t][i & 3];
            }
            if (col < cols) { part[col] = dw[j][i]; part[cols + col] = db[j][i]; }
        }
}

// dy, and x - mean from x or from the 8-bit rows (NormRow), col < cols
template <int DT, bool WIDE>
__device__ __forceinline__ void inputs8(const NormArgs &p, int64_t row, int64_t col, float mean, float *g, float *d)
{
    const int64_t groups = (p.cols + 127) / 128;
    if (p.x) {
        NormRow<DT, WIDE, false> r;
        r.load(p, row, col, groups);
        r.floats(mean, g, d);
    } else {
        NormRow<DT, WIDE, true> r;
        r.load(p, row, col, groups);
        r.floats(mean, g, d);
    }
}

template <int DT, bool WIDE, bool SAVED, int THREADS, int NC>
__global__ __launch_bounds__(RowShape<THREADS>::kBlock) void layer_norm_backward_kernel(NormArgs p)
{
    backward_rows<DT, WIDE, SAVED, THREADS, NC, true>(p, gridDim.x);
}

// Small inputs, which the caches hold: dx by a workgroup per row, and beside them workgroups of 16 to 64 columns that go over all rows again for dw and db.
// One launch and no workspace, where the other form's second launch would cost as much again (77 x 1023 float32: 6.7 us, 11.7 in two).
constexpr int64_t kSmall = 1 << 21;                 // elements
static bool is_small(int64_t rows, int64_t cols) { return rows * cols <= kSmall && rows <= 1024 && cols <= kLongest; }

// columns of such a workgroup: the other threads take every so many-th row each, eight rows at least where there are as many
__host__ __device__ inline int small_columns(int64_t rows, int threads) { return rows >= threads / 2 ? 16 : rows >= threads / 8 ? 32 : 64; }

template <int DT, bool WIDE, bool SAVED, int THREADS, int NC>
__global__ __launch_bounds__(THREADS) void layer_norm_backward_small_kernel(NormArgs p)
{
    if ((int64_t)blockIdx.x < p.rows) {
        backward_rows<DT, WIDE, SAVED, THREADS, NC, false>(p, (int32_t)p.rows);
        return;
    }
    using T = typename Elem<DT>::type;
    __shared__ float sums[2][THREADS];
    const int wide = small_columns(p.rows, THREADS), slices = THREADS / wide, c = threadIdx.x % wide, slice = threadIdx.x / wide;
    const int64_t col = ((int64_t)blockIdx.x - p.rows) * wide + c, at = min(col, p.cols - 1), groups = (p.cols + 127) / 128;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 8
    for (int64_t row = slice; row < p.rows; row += slices) {
        const float g = Elem<DT>::to_float(((const T *)p.dy)[row * p.ld_dy + at]), mean = p.mean[row];
        const float d = SAVED ? fmaf((float)p.xq[row * p.ld_xq + at], p.xs[row * groups + (at >> 7)], -mean) : Elem<DT>::to_float(((const T *)p.x)[row * p.ld_x + at]) - mean;
        dw = fmaf(g, d * p.rstd[row], dw);
        db += g;
    }
    sums[0][threadIdx.x] = dw;
    sums[1][threadIdx.x] = db;
    __syncthreads();
    if (slice || col >= p.cols) return;
    for (int k = 1; k < slices; ++k) { dw += sums[0][k * wide + c]; db += sums[1][k * wide + c]; }
    if (p.dweight) put_param(p.dweight, p.param_dtype, col, dw);
    if (p.dbias) put_param(p.dbias, p.param_dtype, col, db);
}

// dx of rows of any length, read twice (512 x 65536 bfloat16: 75 us)
template <int DT, bool WIDE>
__global__ __launch_bounds__(1024) void norm_long_dx_kernel(NormArgs p)
{
    using E = Elem<DT>;
    using T = typename E::type;
    __shared__ float cells[2][2][16];
    RowReduce<1024> r{cells};
    const int64_t cols = p.cols;
    const float per = 1.0f / (float)cols;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float mean = p.mean[row], rstd = p.rstd[row];
        LongSum of_g, of_gx;
        float sum_g = 0.0f, sum_gx = 0.0f;
        for (int turn = 0; turn < 2; ++turn) {
            for (int64_t col = threadIdx.x * 8; col < cols; col += 8192) {
                float g[8], v[8], w[8], eight_g = 0.0f, eight_gx = 0.0f;
                inputs8<DT, WIDE>(p, row, col, mean, g, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = 1.0f;
                if (p.weight) params8(p.weight, p.param_dtype, col, cols, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = col + i < cols ? v[i] * rstd : 0.0f;
                    g[i] *= w[i];
                    if (turn == 0) { eight_g += g[i]; eight_gx = fmaf(g[i], v[i], eight_gx); }
                    else v[i] = rstd * fmaf(-v[i], sum_gx, g[i] - sum_g);
                }
                if (turn == 0) { of_g.add(eight_g); of_gx.add(eight_gx); }
                else store8<DT, WIDE>((T *)p.dx + row * p.ld_dx, col, cols, v);
            }
            if (turn == 0) {
                sum_g = of_g.value();
                sum_gx = of_gx.value();
                r.sum2(sum_g, sum_gx);
                sum_g *= per;
                sum_gx *= per;
            }
        }
    }
}

// Sums for dw and db where rows are too long for a workgroup's registers: eight columns per thread, every so many-th row
// (512 x 65536 bfloat16: 40 us).
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void norm_long_params_kernel(NormArgs p)
{
    const int64_t cols = p.cols, col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= cols) return;
    float dw[8] = {}, db[8] = {};
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const float mean = p.mean[row], rstd = p.rstd[row];
        float g[8], v[8];
        inputs8<DT, WIDE>(p, row, col, mean, g, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) { dw[i] = fmaf(g[i], v[i] * rstd, dw[i]); db[i] += g[i]; }
    }
    float *part = (float *)p.workspace + (int64_t)blockIdx.y * 2 * cols;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) { part[col + i] = dw[i]; part[cols + col + i] = db[i]; }
}

// Adds up the strips, [strips][2][cols]: 64 columns per workgroup, sixteen waves take a sixteenth of the strips each.  A grid's threads are counted in 32
// bits: workgroups go over the columns in turns where there are more than kParamsBlocks of them (2^25 columns).
constexpr int64_t kParamsBlocks = 1 << 20;
__global__ __launch_bounds__(1024) void norm_params_kernel(int32_t strips, int64_t cols, const float *part, void *dweight, void *dbias, int32_t dt)
{
    __shared__ float sums[16][64];
    const int wave = threadIdx.x >> 6, per = (strips + 15) / 16;
    for (int64_t first = (int64_t)blockIdx.x * 64; first < 2 * cols; first += (int64_t)gridDim.x * 64) {
        const int64_t at = first + (threadIdx.x & 63);
        float sum = 0.0f;
        if (at < 2 * cols) {
            int k = wave * per;
            const int last = min(strips, (wave + 1) * per);
            for (; k + 8 <= last; k += 8) {                     // (eight loads under way)
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(k + i) * 2 * cols + at];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += v[i];
            }
            for (; k < last; ++k) sum += part[(int64_t)k * 2 * cols + at];
        }
        sums[wave][threadIdx.x & 63] = sum;
        __syncthreads();
        if (wave == 0 && at < 2 * cols) {
            sum = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) sum += sums[k][threadIdx.x & 63];
            if (at < cols) {
                if (dweight) put_param(dweight, dt, at, sum);
            } else if (dbias) {
                put_param(dbias, dt, at - cols, sum);
            }
        }
        __syncthreads();                                        // (read before the next turn's are written)
    }
}

// ---- launches ----
static unsigned few(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

template <int DT, bool WIDE>
static hipError_t forward(const NormArgs &p, hipStream_t s)
{
    const int64_t c = p.cols;
    // as many workgroups as the compute units hold stay for all rows (1 024 of four waves: twice as many take 3 % longer on average, half as many 15)
    if (c <= 512) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 64, 1>), dim3(few((p.rows + 3) / 4, 1024)), dim3(256), 0, s, p);
    else if (c <= 1024) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 64, 2>), dim3(few((p.rows + 3) / 4, 1024)), dim3(256), 0, s, p);
    else if (WIDE && c <= 1536) hipLaunchKernelGGL((layer_norm_kernel<DT, true, 64, 3>), dim3(few((p.rows + 3) / 4, 1024)), dim3(256), 0, s, p);
    else if (c <= 2048) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 256, 1>), dim3(few(p.rows, 1024)), dim3(256), 0, s, p);
    else if (c <= 4096) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 256, 2>), dim3(few(p.rows, 1024)), dim3(256), 0, s, p);
    else if (c <= 8192) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 512, 2>), dim3(few(p.rows, 1024)), dim3(512), 0, s, p);
    else if (c <= kLongest) hipLaunchKernelGGL((layer_norm_kernel<DT, WIDE, 1024, 2>), dim3(few(p.rows, 512)), dim3(1024), 0, s, p);
    else hipLaunchKernelGGL((norm_long_kernel<DT, WIDE>), dim3(few(p.rows, 1 << 16)), dim3(1024), 0, s, p);
    return hipGetLastError();
}

// Workgroups that sum up dw and db.  Rows of more than 4 096 columns go to workgroups of 1 024 threads, and half as many: as many waves are busy, and half of
// the sums are left to be added up (900 x 5368 float32: 21 us, 34 in workgroups of 256 with 32 columns a thread; 16000 x 8192 bfloat16: 152, 163).  Longer
// ones are summed by workgroups of 2 048 columns: 2 048 of those in all, of four rows at least (512 x 65536 bfloat16, a strip per row: 165 us, and 50 to add
// them up).
static int64_t strips_of(int64_t rows, int64_t cols)
{
    const int64_t blocks = cols <= 1024 || cols > kLongest ? (rows + 3) / 4 : rows;
    return std::min(blocks, cols <= 4096 ? kStrips : cols <= kLongest ? kStrips / 2 : std::max<int64_t>(1, 2048 / ((cols + 2047) / 2048)));
}
size_t layer_norm_backward_workspace(int64_t rows, int64_t cols) { return is_small(rows, cols) ? 0 : (size_t)strips_of(rows, cols) * 2 * cols * sizeof(float); }

template <int DT, bool WIDE, bool SAVED>
static hipError_t launch_backward_rows(const NormArgs &p, unsigned strips, hipStream_t s)
{
    const int64_t c = p.cols;
    if (c <= 512) hipLaunchKernelGGL((layer_norm_backward_kernel<DT, WIDE, SAVED, 64, 1>), dim3(strips), dim3(256), 0, s, p);
    else if (c <= 1024) hipLaunchKernelGGL((layer_norm_backward_kernel<DT, WIDE, SAVED, 64, 2>), dim3(strips), dim3(256), 0, s, p);
    else if (c <= 2048) hipLaunchKernelGGL((layer_norm_backward_kernel<DT, WIDE, SAVED, 256, 1>), dim3(strips), dim3(256), 0, s, p);
    else if (c <= 4096) hipLaunchKernelGGL((layer_norm_backward_kernel<DT, WIDE, SAVED, 256, 2>), dim3(strips), dim3(256), 0, s, p);
    else if (c <= 8192) hipLaunchKernelGGL((layer_norm_backward_kernel<DT, WIDE, SAVED, 1024, 1>), dim3(strips), dim3(1024), 0, s, p);
    else {
        const size_t lds = 2 * 2 * 2 * 1024 * sizeof(f32x4);
        const auto kernel = layer_norm_backward_kernel<DT, WIDE, SAVED, 1024, 2>;
        if (const hipError_t e = ensure_dynamic_lds((const void *)kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3(strips), dim3(1024), lds, s, p);
    }
    return hipGetLastError();
}

template <int DT, bool WIDE, bool SAVED>
static hipError_t backward_small(const NormArgs &p, hipStream_t s)
{
    // more threads for longer rows, and for the columns of many rows
    const bool many = p.cols > 2048 || p.rows > 256;
    const int wide = small_columns(p.rows, many ? 1024 : 256);
    const dim3 grid((unsigned)(p.rows + (p.dweight || p.dbias ? (p.cols + wide - 1) / wide : 0)));
    const auto kernel = !many            ? layer_norm_backward_small_kernel<DT, WIDE, SAVED, 256, 1>
                        : p.cols <= 8192 ? layer_norm_backward_small_kernel<DT, WIDE, SAVED, 1024, 1>
                                         : layer_norm_backward_small_kernel<DT, WIDE, SAVED, 1024, 2>;
    hipLaunchKernelGGL(kernel, grid, dim3(many ? 1024 : 256), 0, s, p);
    return hipGetLastError();
}

template <int DT, bool WIDE>
static hipError_t backward(const NormArgs &p, hipStream_t s)
{
    if (p.rows && is_small(p.rows, p.cols)) return p.x ? backward_small<DT, WIDE, false>(p, s) : backward_small<DT, WIDE, true>(p, s);
    const unsigned strips = (unsigned)strips_of(p.rows, p.cols);
    if (!strips) {                                              // (no rows: the sums are zero)
    } else if (p.cols > kLongest) {
        if (p.dx) hipLaunchKernelGGL((norm_long_dx_kernel<DT, WIDE>), dim3(few(p.rows, 1 << 16)), dim3(1024), 0, s, p);
        if (p.workspace) hipLaunchKernelGGL((norm_long_params_kernel<DT, WIDE>), dim3((unsigned)((p.cols + 2047) / 2048), strips), dim3(256), 0, s, p);
    } else if (p.x) {
        if (const hipError_t e = launch_backward_rows<DT, WIDE, false>(p, strips, s); e != hipSuccess) return e;
    } else {
        if (const hipError_t e = launch_backward_rows<DT, WIDE, true>(p, strips, s); e != hipSuccess) return e;
    }
    if (p.dweight || p.dbias)
        hipLaunchKernelGGL(norm_params_kernel, dim3(few((2 * p.cols + 63) / 64, kParamsBlocks)), dim3(1024), 0, s, (int32_t)strips, p.cols, (const float *)p.workspace, p.dweight, p.dbias, p.param_dtype);
    return hipGetLastError();
}

hipError_t launch_layer_norm(const NormArgs &p, hipStream_t s)
{
    const bool wide = wide_rows(p.x, p.dtype, p.ld_x, p.cols) && (!p.y || wide_rows(p.y, p.dtype, p.ld_y, p.cols));
    return BY_TYPE(p.dtype, wide, forward, p, s);
}

hipError_t launch_layer_norm_backward(const NormArgs &p, hipStream_t s)
{
    const bool wide = (!p.x || wide_rows(p.x, p.dtype, p.ld_x, p.cols)) && wide_rows(p.dy, p.dtype, p.ld_dy, p.cols) &&
                      (!p.dx || wide_rows(p.dx, p.dtype, p.ld_dx, p.cols));
    return BY_TYPE(p.dtype, wide, backward, p, s);
}

}  // namespace tictac
