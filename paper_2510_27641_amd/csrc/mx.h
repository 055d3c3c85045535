// Shared declarations of the kernels around the 4-bit cache and of the eviction (internal; the public ABI is
// include/specattn.h).
#pragma once

#include "common.h"

namespace specattn {

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Where the rows of a cache lie; offsets in bytes.
struct MxCache {
    uint8_t *codes, *scales;
    int64_t codes_b, codes_h, codes_n, codes_page;
    int64_t scales_b, scales_h, scales_n, scales_page;
    const int32_t *page_table;
    int page_shift, max_pages, num_pages;
    int B, H_kv, n_max, d;
};

struct MxRowsLaunch {
    MxCache c;
    void *k, *v;
    int dtype, T;
    int64_t stride_b, stride_h, stride_t;   // elements
    const int32_t *starts, *counts;
};
specattn_status launch_mx_store(const MxRowsLaunch &a, hipStream_t stream);
specattn_status launch_mx_load(const MxRowsLaunch &a, hipStream_t stream);

// `a` holds what a call over an unreduced cache has as well: queries, lists, outputs, workspace
struct MxAttnLaunch {
    AttnLaunch a;
    MxCache c;
};
size_t mx_attn_workspace_bytes(int rows, int G, int T, int d);
specattn_status launch_mx_attn(const MxAttnLaunch &l, hipStream_t stream);
specattn_status mx_attn_configure();

size_t evict_workspace_bytes(const specattn_evict_args *e);
specattn_status launch_evict_select(const specattn_evict_args *e, void *workspace, hipStream_t stream);
specattn_status launch_evict_move(const specattn_move_args *m, hipStream_t stream);

}  // namespace specattn
