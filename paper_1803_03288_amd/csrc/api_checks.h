// Checks of sizes, strides and pointers that the entry points of the layers' operators share: each returns a status and leaves a message.
#pragma once

#include "internal.h"

namespace tictac {

constexpr int64_t kMostCols = 131072;           // |q| <= 128: sums of the products of so many int8 values fit int32, but for one (exact_sum)
constexpr int64_t kMostRows = 1 << 21;          // of the products (offsets inside a tile are 32 bits)
constexpr int64_t kMostStride = 1 << 24;        // bytes between 8-bit rows of the products, for the same reason

inline int check_dtype(const char *what, int32_t dt)
{
    if (dt == TICTAC_F32 || dt == TICTAC_F16 || dt == TICTAC_BF16) return TICTAC_OK;
    set_error("%s = %d is no tictac_dtype", what, dt);
    return TICTAC_ERR_UNSUPPORTED;
}
inline int check_sizes(int64_t rows, int64_t cols)
{
    if (rows >= 0 && cols >= 1 && rows <= INT64_C(1) << 40 && cols <= INT64_C(1) << 30) return TICTAC_OK;
    set_error("%lld rows of %lld columns: expected no fewer than none of at least one (at most 2^40 of 2^30)", (long long)rows, (long long)cols);
    return TICTAC_ERR_UNSUPPORTED;
}
inline int check_group(int32_t group)
{
    if (group == 0 || group == kRows8Group) return TICTAC_OK;
    set_error("group = %d, expected 0 (a scale per row) or %d", group, kRows8Group);
    return TICTAC_ERR_UNSUPPORTED;
}
// rows that are read may lie on each other (a stride of zero: one row for all), rows that are written may not
inline int check_read(const char *what, const void *p, int32_t dt, int64_t rows, int64_t ld)
{
    if (!p) { set_error("%s is NULL", what); return TICTAC_ERR_NULL; }
    if (ld < 0 || ld > INT64_C(1) << 40) { set_error("stride of %s = %lld", what, (long long)ld); return TICTAC_ERR_UNSUPPORTED; }
    if ((uintptr_t)p % (dt == TICTAC_F32 ? 4 : 2)) { set_error("%s does not lie on a boundary of its elements", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
inline int check_write(const char *what, const void *p, int32_t dt, int64_t rows, int64_t cols, int64_t ld)
{
    if (const int rc = check_read(what, p, dt, rows, ld); rc != TICTAC_OK) return rc;
    if (rows > 1 && ld < cols) { set_error("stride of %s = %lld, rows hold %lld", what, (long long)ld, (long long)cols); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
inline int check_rows8(const char *what, const int8_t *q, const float *scale, int64_t rows, int64_t cols, int64_t ld, int64_t most = INT64_C(1) << 40)
{
    if (!q || !scale) { set_error("%s or its scales are NULL", what); return TICTAC_ERR_NULL; }
    const int64_t padded = (cols + 127) / 128 * 128;
    if (ld % 128 || ld < padded || ld > most) {
        set_error("stride of %s = %lld, expected a multiple of 128 from %lld to %lld", what, (long long)ld, (long long)padded, (long long)most);
        return TICTAC_ERR_UNSUPPORTED;
    }
    if ((uintptr_t)q & 15 || (uintptr_t)scale & 3) { set_error("%s: rows lie on 16-byte boundaries, scales on 4-byte ones", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
inline int check_floats(const char *what, const void *p, int32_t dt, bool needed)
{
    if (!p && needed) { set_error("%s is NULL", what); return TICTAC_ERR_NULL; }
    if ((uintptr_t)p % (dt == TICTAC_F32 ? 4 : 2)) { set_error("%s does not lie on a boundary of its elements", what); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
inline int check_workspace(const void *p, size_t have, size_t need)
{
    if (need && !p) { set_error("workspace is NULL, %zu bytes are needed", need); return TICTAC_ERR_NULL; }
    if (have < need) { set_error("workspace of %zu bytes, %zu are needed", have, need); return TICTAC_ERR_NO_MEM; }
    if ((uintptr_t)p & 255) { set_error("workspace does not lie on a 256-byte boundary"); return TICTAC_ERR_UNSUPPORTED; }
    return TICTAC_OK;
}
inline int check_product(int64_t rows, int64_t cols, int64_t outs)
{
    // (the last: tiles of a product, whose threads a grid counts in 32 bits)
    if (rows >= 0 && outs >= 0 && cols >= 1 && rows <= kMostRows && outs <= kMostRows && cols <= kMostCols && (rows + 255) / 256 * ((outs + 255) / 256) < 1 << 22)
        return TICTAC_OK;
    set_error("%lld rows, %lld columns, %lld outputs: the products take at most 2^21 rows and outputs of 1 to 2^17 columns", (long long)rows, (long long)cols, (long long)outs);
    return TICTAC_ERR_UNSUPPORTED;
}

#define TT_CHECK(expr)                               \
    do {                                             \
        const int rc_ = (expr);                      \
        if (rc_ != TICTAC_OK) return rc_;            \
    } while (0)

}  // namespace tictac
