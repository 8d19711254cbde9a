// What the calls on listed rows share: the list, sums that halves of a wavefront exchange, checks of their arguments.
#pragma once
#include "row_types.h"

// rows listed
struct RowList {
    const int32_t* rows;
    const int64_t* n_rows_dev;
    int64_t max_rows, n, first;      // first: of this launch
};
__device__ __forceinline__ int64_t row_count(const RowList& L) {
    const int64_t k = L.n_rows_dev ? *L.n_rows_dev : L.max_rows;
    return k < 0 ? 0 : (k > L.max_rows ? L.max_rows : k);
}
__device__ __forceinline__ int64_t row_at(const RowList& L, int64_t k, int64_t count) {
    if (k >= count) return -1;
    const int64_t r = L.rows ? L.rows[k] : k;
    return r < 0 || r >= L.n ? -1 : r;
}

// Lanes l and l + HALF (of 64 for HALF = 32, of every 32 for 16) add up a and b between them: the first has a's sum, the other b's
template <int HALF>
__device__ __forceinline__ float half_sums(float a, float b) {
    static_assert(HALF == 32 || HALF == 16, "lanes that can be exchanged");
    const unsigned int x = __float_as_uint(a), y = __float_as_uint(b);
    const auto r = HALF == 32 ? __builtin_amdgcn_permlane32_swap(x, y, false, false) : __builtin_amdgcn_permlane16_swap(x, y, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int HALF>
__device__ __forceinline__ double half_sums(double a, double b) {
    static_assert(HALF == 32 || HALF == 16, "lanes that can be exchanged");
    const fg_u32x2 x = __builtin_bit_cast(fg_u32x2, a), y = __builtin_bit_cast(fg_u32x2, b);
    fg_u32x2 first, second;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto r = HALF == 32 ? __builtin_amdgcn_permlane32_swap(x[i], y[i], false, false) : __builtin_amdgcn_permlane16_swap(x[i], y[i], false, false);
        first[i] = r[0], second[i] = r[1];
    }
    return __builtin_bit_cast(double, first) + __builtin_bit_cast(double, second);
}

static inline fg_status_t check_rows(const char* who, const int32_t* rows_dev, const int64_t* n_rows_dev, int64_t max_rows, int64_t n, int32_t d) {
    if (max_rows < 0 || max_rows > INT32_MAX || n < 0 || n > INT32_MAX) FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (d <= 0) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d must be positive", who, d);
    if (!rows_dev && max_rows > n) FG_FAIL(FG_ERR_SHAPE, "%s: max_rows = %lld without a list, but n = %lld rows", who, (long long)max_rows, (long long)n);
    if (((uintptr_t)rows_dev & 3) || ((uintptr_t)n_rows_dev & 7)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: the list or its count is not aligned", who);
    return FG_OK;
}
// one array of n rows: type, stride and alignment
static inline fg_status_t check_array(const char* who, const char* what, const void* p, int64_t stride, int element, int32_t d) {
    if (stride < (int64_t)d * element) FG_FAIL(FG_ERR_SHAPE, "%s: the stride of %s is smaller than its row", who, what);
    if (((uintptr_t)p | (uintptr_t)stride) & (uintptr_t)(element - 1)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: %s or its stride is not aligned to its element", who, what);
    return FG_OK;
}
#define FG_TRY(expr)                   \
    do {                               \
        const fg_status_t s_ = (expr); \
        if (s_ != FG_OK) return s_;    \
    } while (0)
