// Checks of arguments that the entry points share (internal, host only).
#pragma once

#include "common.h"

#include <algorithm>

namespace specattn {

inline bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
inline int log2i(int x) { int s = 0; while ((1 << s) < x) ++s; return s; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline specattn_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return SPECATTN_OK;
    if (!ws) { set_error("workspace is NULL, %zu bytes needed", need); return SPECATTN_EWORKSPACE; }
    if (!aligned(ws, 256)) { set_error("workspace must be 256-byte aligned"); return SPECATTN_EWORKSPACE; }
    if (have < need) { set_error("workspace has %zu bytes, %zu needed", have, need); return SPECATTN_EWORKSPACE; }
    return SPECATTN_OK;
}

inline specattn_status check_pages(const int32_t *page_table, int page_size, int max_pages, int n_max)
{
    if (!is_pow2(page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
    if (page_table && (int64_t)max_pages * page_size < n_max) { set_error("page table is shorter than n_max"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

// Whether rows of `bytes` bytes (or elements) at these strides share any: dimension by dimension from the smallest stride up, each has to lie beyond all that
// the ones before it reach.
struct Dim { int64_t size; __int128 stride; };
inline bool rows_overlap(Dim a, Dim b, Dim c, int64_t bytes)
{
    Dim dims[] = {a, b, c};
    for (Dim &d : dims) d.stride = d.stride < 0 ? -d.stride : d.stride;
    std::sort(dims, dims + 3, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    __int128 reach = bytes;
    for (const Dim &d : dims) {
        if (d.size <= 1) continue;
        if (d.stride < reach) return true;
        reach += (d.size - 1) * d.stride;
    }
    return false;
}

}  // namespace specattn
