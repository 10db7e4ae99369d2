// Argument checks of the C entry points.
#pragma once

#include <initializer_list>

#include "internal.hpp"

namespace dm {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline int check_ptr(const void* p, const char* name) {
    if (!p) return set_error(DM_ERR_ARG, "%s is NULL", name);
    if (!aligned16(p)) return set_error(DM_ERR_ARG, "%s is not 16-byte aligned", name);
    return DM_OK;
}

// an output that begins where an input (or another output) does
inline int check_apart(const void* out, const char* name, std::initializer_list<const void*> others) {
    for (const void* p : others)
        if (out && out == p) return set_error(DM_ERR_ARG, "%s aliases another tensor of the call", name);
    return DM_OK;
}

inline int check_dtype(int32_t dt) {
    if (dt != DM_F32 && dt != DM_F16 && dt != DM_BF16)
        return set_error(DM_ERR_UNSUPPORTED, "unsupported dtype %d", dt);
    return DM_OK;
}

inline int check_drop(const dm_dropout* d) {
    if (d && !(d->p >= 0.f && d->p < 1.f)) return set_error(DM_ERR_ARG, "dropout p=%g outside [0,1)", d->p);
    return DM_OK;
}

inline int check_rows(int64_t rows, int32_t cols, int32_t max_cols) {
    if (rows < 0 || cols <= 0) return set_error(DM_ERR_ARG, "bad shape rows=%lld cols=%d", (long long)rows, cols);
    if (cols % 8) return set_error(DM_ERR_UNSUPPORTED, "row length %d is not a multiple of 8", cols);
    if (max_cols && cols > max_cols) return set_error(DM_ERR_UNSUPPORTED, "row length %d above %d", cols, max_cols);
    if (rows > (int64_t)INT32_MAX * 8) return set_error(DM_ERR_UNSUPPORTED, "too many rows");
    return DM_OK;
}

#define DM_TRY(x)                      \
    do {                               \
        int _rc = (x);                 \
        if (_rc != DM_OK) return _rc;  \
    } while (0)

inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace dm
