// The tiled product of 8-bit floats in blocks: out[c][r] = sum over blocks b of 128 of k of 2^(e_p[r][b] + e_q[c][b]) sum over b of P[r][k] Q[c][k] (+ bias[r]).
// P holds e4m3, Q e4m3 or e5m2; a block is a step of the tiles of k8_tiles.h.
#pragma once

#include "f8.h"
#include "k8_product.h"

namespace tictac {

struct ProductF8Args : ProductArgs {
    const uint8_t *p_e, *q_e;           // scales as bytes, a row for each `1 << shift` rows of P or Q; readable up to the next multiple of four
    int64_t ld_pe, ld_qe;
    int32_t p_shift, q_shift;
    int32_t q_format;
};

// One product, or two of one output type and one format of Q, in one launch; outputs are float16 or bfloat16.
hipError_t launch_products_f8(const ProductF8Args *a, int n, int32_t tile, const ColumnSums &c, hipStream_t s);
ProductPlan plan_products_f8(const ProductShape *shapes, int n);

}  // namespace tictac
