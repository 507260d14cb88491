/*
 * What the operators' entry points (cfa_ops.cu, cfa_step.cu) check their arguments with.  Not part of
 * the C ABI.
 */
#ifndef CFA_CHECKS_H
#define CFA_CHECKS_H

#include <cstdarg>
#include <cstdio>

#include "cfa_ops.h"

namespace cfa_checks {

constexpr uint64_t kAlign = 256; /* of the workspace and its parts */

inline cfa_status refuse(cfa_status st, const char *fmt, ...)
{
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    cfa_internal_set_error(msg);
    return st;
}

inline cfa_status cuda_result(const char *what, cudaError_t e)
{
    if (e == cudaSuccess) return CFA_OK;
    return refuse(CFA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

/* Bytes from the first element of a matrix to its last; false if they do not fit 62 bits. */
inline bool extent(int64_t rows, int64_t cols, int64_t stride, uint64_t size, uint64_t *bytes)
{
    *bytes = 0;
    if (rows == 0 || cols == 0) return true;
    const unsigned __int128 n =
        ((unsigned __int128)(rows - 1) * (uint64_t)(rows > 1 ? stride : 0) + (uint64_t)cols) * size;
    if (n >> 62) return false;
    *bytes = (uint64_t)n;
    return true;
}

inline bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    const uint64_t p = (uint64_t)(uintptr_t)a, q = (uint64_t)(uintptr_t)b;
    return na && nb && p < q + nb && q < p + na;
}

inline bool off_grid(const void *p, uint64_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

inline uint64_t aligned(uint64_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

inline bool is_half(int32_t dtype) { return dtype == CFA_DTYPE_BF16 || dtype == CFA_DTYPE_F16; }

constexpr int64_t kMost = 1ll << 31; /* rows, columns and strides stay below this */

inline bool size_ok(int64_t n, int64_t least) { return n >= least && n < kMost; }

} // namespace cfa_checks

#endif /* CFA_CHECKS_H */
