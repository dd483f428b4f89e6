// Argument checks of the calls that work on rows (layer norm, bias + GELU, distillation).
#pragma once
#include "tmask_host.hpp"

// Returns from the calling function with the code of a check that fails.
#define TMASK_TRY(call)            \
    do {                           \
        const int rc_ = (call);    \
        if (rc_ != TMASK_OK)       \
            return rc_;            \
    } while (0)

namespace tmask {

inline bool known(tmask_dtype dt) { return dt == TMASK_F32 || dt == TMASK_BF16; }

inline size_t size_of(tmask_dtype dt) { return dt == TMASK_F32 ? 4 : 2; }

inline bool valid_sizes(int64_t rows, int64_t cols) { return rows >= 0 && cols > 0 && rows <= 0x7FFFFFFF && cols <= 0x7FFFFFFF; }

// one tensor of a call: rows x cols of `size`-byte elements
inline int check_rows(const char *name, const void *p, int64_t ld, int64_t rows, int64_t cols, size_t size, bool needed)
{
    if (!p)
        return needed ? fail(TMASK_ERR_NULL, "%s is NULL", name) : TMASK_OK;
    if (rows > 1 && (ld < cols || ld > 0x7FFFFFFF))
        return fail(TMASK_ERR_SHAPE, "leading dimension of %s: %lld (at least %lld, below 2^31)", name, (long long)ld, (long long)cols);
    if ((uintptr_t)p % size)
        return fail(TMASK_ERR_ALIGN, "%s is not aligned to its element type", name);
    return TMASK_OK;
}

inline int check_vector(const char *name, const void *p, size_t size, bool needed) { return check_rows(name, p, 0, 1, 1, size, needed); }

inline int check_workspace(const void *workspace, size_t bytes, size_t needed)
{
    if (needed && (!workspace || ((uintptr_t)workspace & 255) || bytes < needed))
        return fail(TMASK_ERR_WORKSPACE, "a workspace of %zu bytes, 256-byte aligned, is needed (got %zu)", needed, workspace ? bytes : (size_t)0);
    return TMASK_OK;
}

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TMASK_OK : hip_fail(e, what);
}

}  // namespace tmask
