// Shared declarations of the kernels of a serving loop in pages: page tables, rows into the cache, prompts, drafted trees (internal;
// the public ABI is include/specattn.h).
#pragma once

#include "common.h"

namespace specattn {

size_t pages_workspace_bytes(const specattn_pages_args *p);
specattn_status launch_pages(const specattn_pages_args *p, void *workspace, hipStream_t stream);
specattn_status launch_store(const specattn_store_args *s, hipStream_t stream);
size_t prompt_workspace_bytes(const specattn_prompt_args *p);
specattn_status launch_prompt(const specattn_prompt_args *p, hipStream_t stream);
size_t tree_workspace_bytes(const specattn_tree_args *t);
specattn_status launch_tree(const specattn_tree_args *t, hipStream_t stream);
specattn_status prompt_configure();
specattn_status tree_configure();

}  // namespace specattn
