// Checks of arguments that several calls share.
#pragma once

#include "st_internal.h"

namespace st {

inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// rows of `width` 16-bit numbers, moved 16 bytes at a time
inline int check_matrix(const char *name, const void *p, int64_t stride, int64_t width) {
    if (!p) return fail(ST_EINVAL, "%s is NULL", name);
    if ((uintptr_t)p & 15) return fail(ST_EINVAL, "%s is not aligned to 16 bytes", name);
    if (stride < width || stride % 8) return fail(ST_EINVAL, "%s: row stride %lld, needs a multiple of 8 from %lld on", name, (long long)stride, (long long)width);
    return ST_OK;
}
// Matrices of `rows` rows, read and written by one call, must not share memory; with one stride they may be columns side by side.
inline int check_apart(const char *in_name, const void *in, int64_t in_stride, int64_t in_width, const char *out_name, const void *out,
                       int64_t out_stride, int64_t out_width, int rows) {
    if (!rows) return ST_OK;
    const uintptr_t i0 = (uintptr_t)in, o0 = (uintptr_t)out;
    const uintptr_t i1 = i0 + 2 * (((uintptr_t)rows - 1) * in_stride + in_width), o1 = o0 + 2 * (((uintptr_t)rows - 1) * out_stride + out_width);
    if (i1 <= o0 || o1 <= i0) return ST_OK;
    if (in_stride == out_stride) {
        const int64_t d = ((int64_t)o0 - (int64_t)i0) / 2 % in_stride, at = d < 0 ? d + in_stride : d;  // column of in's rows that out starts at
        if (at >= in_width && at + out_width <= in_stride) return ST_OK;
    }
    return fail(ST_EINVAL, "%s and %s share memory", in_name, out_name);
}
inline int launched(const char *what, hipError_t e) {
    return e == hipSuccess ? ST_OK : fail(ST_EHIP, "%s: %s", what, hipGetErrorString(e));
}


}  // namespace st
