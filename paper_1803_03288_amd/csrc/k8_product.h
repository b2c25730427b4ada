// The tiled product behind the layers with 8-bit weights, forward and backward:
//   out[c][r] = sum over k of P[r][k] Q[c][k]
// P and Q have k contiguous and padded with zeros to whole steps of 128 bytes: 128 int8 or 64 bf16 values.  Both types take the same path
// through LDS, sixteen bytes per lane, and differ in the matrix instruction alone.  r, along which the output is contiguous, is the row
// index of the matrix instruction, so that a lane has four consecutive outputs.
#pragma once

#include "rows8.h"

namespace tictac {

struct ProductArgs {
    const char *p, *q;
    int64_t ld_p, ld_q;         // bytes
    int32_t R, C;
    int32_t steps;              // of 128 bytes, along q
    int32_t p_steps;            // p starts again after so many: q holds `steps / p_steps` pieces side by side
    int32_t splits;             // the steps are dealt to so many workgroups per tile, which leave sums in `parts`
    void *out;
    int64_t ld_out;
    int32_t dtype;              // of out
    // int8: out = sum * (q_scale[c] * p_scale[r]) + bias[r]; bf16: out = sum, or sum + bias[r]
    const float *p_scale, *q_scale;
    const void *bias;
    int32_t bias_dtype;
    void *parts;                // [splits][C][R], int32 or float32
};

// A sum of products of int8 values, as float32.  131 072 of -128 and -128 come to 2^31, one more than int32 holds, and wrap round to -2^31, which no other
// sum of as many is: the least is 131 072 (-128) 127.  The tiles have kernels of their own for so many columns (the comparison costs 0.7 % of 8192 x 4096 -> 16384
// and of 4165 x 916 -> 5071; 8192 x 131072 -> 8192 by tiles of 128 x 128 instead of 256 x 256: 9.4 ms, 8.1).
constexpr int32_t kWidest = 131072;         // the most columns that are taken
__device__ __forceinline__ float exact_sum(int32_t sum) { return sum == INT32_MIN ? 0x1p31f : (float)sum; }

// Sums of `parts` rows of floats, [parts][n], in their order, as a vector of `dtype`: rides along with the products of a backward pass.
struct ColumnSums {
    const float *sums;
    int64_t parts, n;
    void *out;                  // NULL: none
    int32_t dtype;
};

// How the products of one launch are dealt to workgroups: the tile, and into how many parts each product's steps are cut.
struct ProductShape { int32_t R, C, steps; };
struct ProductPlan {
    int32_t tile;               // one of kCosts.tiles, or kTile256
    int32_t splits[2];
};
constexpr int32_t kTile256 = 3;

// What tiles take: see kCosts.
struct ProductTile { int32_t r, c; float fixed, step, step2; };
struct ProductCosts {
    ProductTile tiles[3];
    int32_t longest;            // steps of a part, at most
    bool beside;                // the longest workgroups go on beside the starts and ends of others, and up to two per compute unit the time rises with their number
    float joined;               // bytes of parts that are written and read again in a us
    float first256, tile256, next256, step256, half256;         // tiles of 256 x 256: what a launch, a tile and each turn but the first take beside the steps, a step, the least of a step
};
ProductPlan plan_products(const ProductShape *shapes, int n, const ProductCosts &costs);
ProductPlan plan_products(const ProductShape *shapes, int n);
inline size_t product_parts_bytes(int32_t splits, int32_t R, int32_t C) { return splits > 1 ? (size_t)splits * R * C * 4 : 0; }
hipError_t launch_product_i8(const ProductArgs &a, int32_t tile, hipStream_t s);
hipError_t launch_products_bf16(const ProductArgs *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s);     // one or two products, of one output type, in one launch
hipError_t launch_product_bf16_biased(const ProductArgs &a, int32_t tile, hipStream_t s);      // float32 outputs, bias added
hipError_t launch_product_join_i8(const ProductArgs &a, hipStream_t s);        // the sums in `parts` to the output
hipError_t launch_product_join_bf16(const ProductArgs &a, hipStream_t s);
hipError_t launch_product_join_biased(const ProductArgs &a, hipStream_t s);    // float32 sums, bias added

}  // namespace tictac
