// Checks of arguments that the entry points share.
#pragma once

#include "block_common.h"

namespace maddness {

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;

inline bool aligned(const void *p, int64_t a) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)a == 0; }

inline bool floating(int32_t dtype) { return dtype == MADDNESS_F32 || dtype == MADDNESS_F16 || dtype == MADDNESS_BF16; }

inline int64_t bytes_of(int32_t dtype) { return dtype == MADDNESS_F32 ? 4 : dtype == kE4M3 ? 1 : 2; }

inline int check_size(int64_t v, const char *name)
{
    if (v < 0) return fail(MADDNESS_E_INVAL, "%s = %lld is negative", name, (long long)v);
    if (v > kMostRows) return fail(MADDNESS_E_UNSUPPORTED, "%s = %lld, supported are up to 2^31 - 1", name, (long long)v);
    return MADDNESS_OK;
}

// A matrix of a floating type (or nullptr where it has no elements).
inline int check_floats(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const char *name)
{
    if (!floating(dtype)) return fail(MADDNESS_E_INVAL, "%s: dtype = %d is not F32, F16 or BF16", name, dtype);
    if (rows == 0 || cols == 0) return MADDNESS_OK;
    if (!x) return fail(MADDNESS_E_INVAL, "%s is NULL", name);
    if (ld < cols) return fail(MADDNESS_E_INVAL, "%s: row stride %lld is smaller than its %lld columns", name, (long long)ld, (long long)cols);
    if (!aligned(x, bytes_of(dtype))) return fail(MADDNESS_E_ALIGN, "%s not aligned to its element size", name);
    return MADDNESS_OK;
}

}  // namespace maddness
