// What the calls on matrices of rows share on the host: types, checks, errors.
#pragma once
#include "rows.h"

namespace {

template <class F>
inline int with_type(int dtype, F f)
{
    if (dtype == LEANN_F32) return f((float *)nullptr);
    if (dtype == LEANN_BF16) return f((bf16_t *)nullptr);
    return f((f16_t *)nullptr);
}

// Outputs that the caches would not hold until they are read go past them: dropout + LayerNorm, dropout and the gradient in a row over 131 072 x 768 bf16 take 421
// instead of 436 us, over 65 536 rows 215 and 217; over 16 384 rows it would be 64 instead of 62.
inline int streams(int64_t rows, int64_t cols, size_t size) { return (double)rows * cols * size >= 96e6; }

inline int check_matrix(const char *call, int64_t rows, int64_t cols, int dtype)
{
    if (rows < 0 || cols < 1 || (dtype != LEANN_F32 && dtype != LEANN_BF16 && dtype != LEANN_F16)) {
        leann_set_error("%s: negative row count, no columns or unknown type", call);
        return LEANN_EINVAL;
    }
    if (rows > 0x7fffffffll || cols > 0x7fffffffll - 8) {
        leann_set_error("%s: %lld x %lld elements are not covered (rows and columns below 2^31)", call, (long long)rows, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

inline int check_rows(const char *call, const char *what, const void *p, int64_t ld, int64_t cols)
{
    if (!p) {
        leann_set_error("%s: %s is null", call, what);
        return LEANN_EINVAL;
    }
    if (ld < cols) {
        leann_set_error("%s: rows of %s are %lld elements apart and %lld long", call, what, (long long)ld, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

inline int launched(const char *call)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LEANN_OK;
    leann_set_error("%s: launch failed: %s", call, hipGetErrorString(e));
    return LEANN_EDEVICE;
}

}  // namespace
