// C ABI of the serving loop in pages: host-side argument checks and dispatch.
#include "checks.h"
#include "serve.h"

#include <initializer_list>

namespace specattn {
namespace {

specattn_status check_pages_args(const specattn_pages_args *p)
{
    if (!p) { set_error("pages args are NULL"); return SPECATTN_EINVAL; }
    if (!p->page_table || !p->free_pages || !p->free_count || !p->free_count_out || !p->seq_lens || !p->new_lens || !p->lens_out) { set_error("page_table, free_pages, the free counts and the lengths must not be NULL"); return SPECATTN_EINVAL; }
    if (p->B <= 0 || p->max_pages_per_seq <= 0 || p->num_pages <= 0) { set_error("B, max_pages_per_seq and num_pages must be positive"); return SPECATTN_EINVAL; }
    if ((p->positions || p->owners) && !p->slots) { set_error("positions and owners come with slots"); return SPECATTN_EINVAL; }
    if (p->slots && p->token_capacity <= 0) { set_error("token_capacity must be positive"); return SPECATTN_EINVAL; }
    if (!is_pow2(p->page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
    if ((int64_t)p->num_pages * p->page_size > INT32_MAX) { set_error("slots are counted in 31 bits"); return SPECATTN_ESHAPE; }
    if ((int64_t)p->max_pages_per_seq * p->page_size > INT32_MAX) { set_error("positions are counted in 31 bits"); return SPECATTN_ESHAPE; }
    if ((int64_t)p->B * p->max_pages_per_seq > INT32_MAX) { set_error("entries of the page table are counted in 31 bits"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

specattn_status check_store(const specattn_store_args *s)
{
    if (!s) { set_error("store args are NULL"); return SPECATTN_EINVAL; }
    if (!s->k || !s->v || !s->k_cache || !s->v_cache || !s->slots) { set_error("k, v, the caches and slots must not be NULL"); return SPECATTN_EINVAL; }
    if (s->B <= 0 || s->T <= 0 || s->H_kv <= 0 || s->d <= 0 || s->num_slots <= 0 || s->num_pages <= 0 || s->page_size <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    if (s->dtype != SPECATTN_F32 && s->dtype != SPECATTN_BF16 && s->dtype != SPECATTN_F16) { set_error("unknown dtype %d", (int)s->dtype); return SPECATTN_EUNSUPPORTED; }
    const int64_t es = s->dtype == SPECATTN_F32 ? 4 : 2;
    if ((int64_t)s->B * s->T > INT32_MAX) { set_error("rows are counted in 31 bits"); return SPECATTN_ESHAPE; }
    if ((int64_t)s->H_kv * s->d > (1 << 24)) { set_error("a token has more than 2^24 elements"); return SPECATTN_ESHAPE; }
    if (s->d * es % 16) { set_error("a row must be a multiple of 16 bytes"); return SPECATTN_EALIGN; }
    const int64_t strides[] = {s->stride_b, s->stride_t, s->stride_h, s->cache_stride_page, s->cache_stride_n, s->cache_stride_h};
    for (int64_t st : strides) {
        if (st < 0) { set_error("strides must not be negative"); return SPECATTN_ESHAPE; }
        if (st * es % 16) { set_error("strides must be multiples of 16 bytes"); return SPECATTN_EALIGN; }
    }
    const void *tensors[] = {s->k, s->v, s->k_cache, s->v_cache};
    for (const void *p : tensors)
        if (!aligned(p, 16)) { set_error("k, v and the caches must be 16-byte aligned"); return SPECATTN_EALIGN; }
    if (rows_overlap({s->num_pages, s->cache_stride_page}, {s->H_kv, s->cache_stride_h}, {s->page_size, s->cache_stride_n}, s->d)) { set_error("rows of the cache share bytes"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

// What both attention calls ask of their sizes, types and places in memory.
specattn_status check_heads(int H_q, int H_kv, int d, specattn_dtype dtype)
{
    if (H_q <= 0 || H_kv <= 0 || d <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    if (dtype != SPECATTN_BF16 && dtype != SPECATTN_F16) { set_error("queries, keys and values are bf16 or fp16"); return SPECATTN_EUNSUPPORTED; }
    if (H_q % H_kv) { set_error("H_q is not a multiple of H_kv"); return SPECATTN_ESHAPE; }
    if (d != 64 && d != 128) { set_error("d must be 64 or 128"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}
specattn_status check_places(std::initializer_list<const void *> pointers, std::initializer_list<int64_t> strides)
{
    for (const void *p : pointers)
        if (!aligned(p, 16)) { set_error("tensors must be 16-byte aligned"); return SPECATTN_EALIGN; }
    for (int64_t st : strides)
        if (st % 8) { set_error("strides must be multiples of 16 bytes"); return SPECATTN_EALIGN; }
    return SPECATTN_OK;
}
specattn_status check_pool(const int32_t *page_table, int page_size, int max_pages, int n_max, int num_pages, int64_t stride_page)
{
    const specattn_status st = check_pages(page_table, page_size, max_pages, n_max);
    if (st != SPECATTN_OK) return st;
    if (num_pages <= 0) { set_error("num_pages must be positive"); return SPECATTN_EINVAL; }
    if (stride_page <= 0) { set_error("kv_stride_page must be positive"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

// Row offsets go to the kernels in units of 16 bytes in 32 bits.
specattn_status check_reach(int64_t outer, int64_t outer_stride, int64_t inner, int64_t inner_stride)
{
    const __int128 reach = (__int128)(outer - 1) * outer_stride + (__int128)(inner - 1) * inner_stride;
    if (outer_stride < 0 || inner_stride < 0) { set_error("strides must not be negative"); return SPECATTN_ESHAPE; }
    if (reach * 2 >= ((__int128)1 << 36)) { set_error("the rows of a kv head must lie within 64 GiB of its first one"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

specattn_status check_prompt(const specattn_prompt_args *p)
{
    if (!p) { set_error("prompt args are NULL"); return SPECATTN_EINVAL; }
    if (!p->q || !p->k || !p->v || !p->q_starts || (!p->out && !p->out_lowp)) { set_error("q, k, v, q_starts and one of out and out_lowp must not be NULL"); return SPECATTN_EINVAL; }
    if (p->B <= 0 || p->total_q <= 0) { set_error("B and total_q must be positive"); return SPECATTN_EINVAL; }
    specattn_status st = check_heads(p->H_q, p->H_kv, p->d, p->dtype);
    if (st != SPECATTN_OK) return st;
    if ((int64_t)p->total_q * p->H_q > (1 << 30)) { set_error("more than 2^30 query rows"); return SPECATTN_ESHAPE; }
    // (a launch has fewer than 2^32 threads along an axis: 512 for every 256 query rows, and for what is left of each sequence and kv head)
    if ((int64_t)p->B * p->H_kv > (1 << 21)) { set_error("too many sequences"); return SPECATTN_ESHAPE; }
    if (p->page_table) {
        if (!p->seq_lens) { set_error("keys and values in pages need seq_lens"); return SPECATTN_EINVAL; }
        if (p->kv_starts) { set_error("kv_starts is for packed keys and values"); return SPECATTN_EINVAL; }
        st = check_pool(p->page_table, p->page_size, p->max_pages_per_seq, 1, p->num_pages, p->kv_stride_page);
        if (st != SPECATTN_OK) return st;
        if ((int64_t)p->max_pages_per_seq * p->page_size > (1 << 30)) { set_error("more than 2^30 positions per sequence"); return SPECATTN_ESHAPE; }
    } else {
        if (p->seq_lens) { set_error("seq_lens is for keys and values in pages (packed ones take kv_starts)"); return SPECATTN_EINVAL; }
        if (p->total_kv <= 0) { set_error("total_kv must be positive"); return SPECATTN_EINVAL; }
        if (p->total_kv > (1 << 30)) { set_error("more than 2^30 positions"); return SPECATTN_ESHAPE; }
    }
    if (p->kv_stride_n < p->d) { set_error("kv_stride_n is smaller than d"); return SPECATTN_ESHAPE; }
    st = p->page_table ? check_reach(p->num_pages, p->kv_stride_page, p->page_size, p->kv_stride_n) : check_reach(1, 0, p->total_kv, p->kv_stride_n);
    if (st != SPECATTN_OK) return st;
    return check_places({p->q, p->k, p->v, p->out, p->out_lowp}, {p->q_stride_t, p->q_stride_h, p->kv_stride_n, p->kv_stride_h, p->page_table ? p->kv_stride_page : 0});
}

specattn_status check_tree(const specattn_tree_args *t)
{
    if (!t) { set_error("tree args are NULL"); return SPECATTN_EINVAL; }
    if (!t->q || !t->k || !t->v || !t->k_new || !t->v_new || !t->tree_masks || (!t->out && !t->out_lowp)) { set_error("q, k, v, k_new, v_new, tree_masks and one of out and out_lowp must not be NULL"); return SPECATTN_EINVAL; }
    const bool dense = !t->indices && !t->counts;
    if (!dense && (!t->indices || !t->counts)) { set_error("indices and counts must both be given, or both be NULL (dense)"); return SPECATTN_EINVAL; }
    if (dense && t->indices_are_physical) { set_error("indices_are_physical without an index list"); return SPECATTN_EINVAL; }
    if (t->B <= 0 || t->T <= 0 || t->n_max <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    specattn_status st = check_heads(t->H_q, t->H_kv, t->d, t->dtype);
    if (st != SPECATTN_OK) return st;
    if (t->T > SPECATTN_MAX_TREE) { set_error("T exceeds %d", SPECATTN_MAX_TREE); return SPECATTN_ESHAPE; }
    if ((int64_t)t->B * t->H_q > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
    if ((int64_t)(t->H_q / t->H_kv) * t->T > 65536) { set_error("more than 65536 query rows per kv head"); return SPECATTN_ESHAPE; }
    if (!dense && t->idx_capacity < 1) { set_error("idx_capacity must be at least 1"); return SPECATTN_ESHAPE; }
    if (!dense && t->idx_stride_row < t->idx_capacity) { set_error("idx_stride_row is smaller than idx_capacity"); return SPECATTN_ESHAPE; }
    if (t->chunk_size < 0 || (t->chunk_size > 1 && (!is_pow2(t->chunk_size) || t->chunk_size > 1024))) { set_error("chunk_size must be 0, 1 or a power of two up to 1024"); return SPECATTN_ESHAPE; }
    if (t->chunk_size > 1 && (dense || t->indices_are_physical)) { set_error("chunk lists are not available with dense calls or physical indices"); return SPECATTN_EUNSUPPORTED; }
    const int64_t most = dense ? t->n_max : (int64_t)t->idx_capacity * (t->chunk_size > 1 ? t->chunk_size : 1);
    if (most > (1 << 24)) { set_error("more than 2^24 positions per row"); return SPECATTN_ESHAPE; }
    if (t->page_table || t->indices_are_physical) {
        st = check_pool(t->page_table, t->page_size, t->max_pages_per_seq, t->n_max, t->num_pages, t->kv_stride_page);
        if (st != SPECATTN_OK) return st;
    } else if (t->num_pages > 0) {
        set_error("a pool without a page table takes lists of pool slots alone (num_pages is 0 for a contiguous cache)");
        return SPECATTN_EINVAL;
    }
    if (t->kv_stride_n < t->d) { set_error("kv_stride_n is smaller than d"); return SPECATTN_ESHAPE; }
    const bool pool = t->page_table || t->indices_are_physical;
    st = pool ? check_reach(t->num_pages, t->kv_stride_page, t->page_size, t->kv_stride_n) : check_reach(1, 0, t->n_max, t->kv_stride_n);
    if (st != SPECATTN_OK) return st;
    return check_places({t->q, t->k, t->v, t->k_new, t->v_new, t->out, t->out_lowp},
                        {t->q_stride_b, t->q_stride_h, t->q_stride_t, t->kv_stride_n, t->kv_stride_h, pool ? t->kv_stride_page : t->kv_stride_b});
}

}  // namespace
}  // namespace specattn

using namespace specattn;

extern "C" {

size_t specattn_pages_workspace_size(const specattn_pages_args *args)
{
    if (check_pages_args(args) != SPECATTN_OK) { clear_error(); return 0; }
    return pages_workspace_bytes(args);
}

specattn_status specattn_pages_update(const specattn_pages_args *args, void *workspace, size_t workspace_bytes, void *stream)
{
    clear_error();
    specattn_status st = check_pages_args(args);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(args));
    if (st != SPECATTN_OK) return st;
    return launch_pages(args, workspace, static_cast<hipStream_t>(stream));
}

specattn_status specattn_cache_store(const specattn_store_args *args, void *stream)
{
    clear_error();
    const specattn_status st = check_store(args);
    if (st != SPECATTN_OK) return st;
    return launch_store(args, static_cast<hipStream_t>(stream));
}

size_t specattn_prompt_workspace_size(const specattn_prompt_args *args)
{
    if (check_prompt(args) != SPECATTN_OK) { clear_error(); return 0; }
    return prompt_workspace_bytes(args);
}

specattn_status specattn_prompt_attn(const specattn_prompt_args *args, void *stream)
{
    clear_error();
    specattn_status st = check_prompt(args);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(args->workspace, args->workspace_bytes, prompt_workspace_bytes(args));
    if (st != SPECATTN_OK) return st;
    return launch_prompt(args, static_cast<hipStream_t>(stream));
}

size_t specattn_tree_workspace_size(const specattn_tree_args *args)
{
    if (check_tree(args) != SPECATTN_OK) { clear_error(); return 0; }
    return tree_workspace_bytes(args);
}

specattn_status specattn_tree_attn(const specattn_tree_args *args, void *stream)
{
    clear_error();
    specattn_status st = check_tree(args);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(args->workspace, args->workspace_bytes, tree_workspace_bytes(args));
    if (st != SPECATTN_OK) return st;
    return launch_tree(args, static_cast<hipStream_t>(stream));
}

}  // extern "C"
