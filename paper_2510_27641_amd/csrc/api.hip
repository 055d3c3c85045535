// C ABI of the library: host-side argument checks and dispatch.  Nothing here touches device
// memory; every check runs before the first launch so that a failing call writes nothing.
#include "common.h"
#include "mx.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

// Scratch memory of specattn_sparse_decode_attn_static: the split partials and the rows' shares of one
// attention call.  Every GPU the library runs on holds its own copy of this array until the process ends.
// In host code the name is only a handle for hipGetSymbolAddress; kernels get the address it returns.
static __device__ __align__(256) unsigned char scratch[SPECATTN_STATIC_SCRATCH_BYTES];

namespace specattn {

static thread_local char g_error[512] = "";

void set_error(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof(g_error), fmt, ap);
    va_end(ap);
}

void clear_error() { g_error[0] = '\0'; }

int cu_count()
{
    static int cached = 0;
    if (cached > 0) return cached;
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && cus > 0) {
        cached = cus;
        return cus;
    }
    (void)hipGetLastError();
    return 256;
}

specattn_status check_launch(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return SPECATTN_OK;
    set_error("%s: %s", what, hipGetErrorString(e));
    return SPECATTN_EHIP;
}

namespace {

bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2i(int x) { int s = 0; while ((1 << s) < x) ++s; return s; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

specattn_status check_select(const specattn_select_args *s, bool fused)
{
    if (!s) { set_error("select args are NULL"); return SPECATTN_EINVAL; }
    if (!s->probs || !s->counts) { set_error("probs and counts must not be NULL"); return SPECATTN_EINVAL; }
    if (!fused && !s->indices && !s->block_counts && !s->kept_mask) { set_error("indices, block_counts and kept_mask must not all be NULL"); return SPECATTN_EINVAL; }
    if (s->B <= 0 || s->H_kv <= 0 || s->n_max <= 0) { set_error("B, H_kv and n_max must be positive"); return SPECATTN_EINVAL; }
    if (!(s->top_p > 0.0f && s->top_p <= 1.0f)) { set_error("top_p must lie in (0, 1]"); return SPECATTN_EINVAL; }
    if (s->n_max > SPECATTN_MAX_N) { set_error("n_max %d exceeds %d", s->n_max, SPECATTN_MAX_N); return SPECATTN_ESHAPE; }
    if ((int64_t)s->B * s->H_kv > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
    if (s->indices && !fused) {
        if (s->idx_capacity < 1) { set_error("idx_capacity must be at least 1"); return SPECATTN_ESHAPE; }
        if (s->idx_stride_row < s->idx_capacity) { set_error("idx_stride_row is smaller than idx_capacity"); return SPECATTN_ESHAPE; }
    }
    if (s->chunk_size < 0 || (s->chunk_size > 1 && (!is_pow2(s->chunk_size) || s->chunk_size > 1024))) { set_error("chunk_size must be 0, 1 or a power of two up to 1024"); return SPECATTN_ESHAPE; }
    if (s->chunk_size > 1 && (s->emit_physical || s->block_counts || s->kept_mask)) { set_error("chunk-granular selection is not available with emit_physical, block_counts or kept_mask"); return SPECATTN_EUNSUPPORTED; }
    if (s->bisect_iters < 0 || s->bisect_iters > 64) { set_error("bisect_iters must lie in 0..64"); return SPECATTN_ESHAPE; }
    if (s->bisect_iters > 0 && (fused || s->block_counts || s->kept_mask || s->chunk_size > 1 || !s->indices)) { set_error("the bisection mode needs an index list and is not available with the fused call, block_counts or chunks"); return SPECATTN_EUNSUPPORTED; }
    if (s->probs_stride_h < s->n_max || s->probs_stride_b < s->n_max) { set_error("probs strides are smaller than n_max"); return SPECATTN_ESHAPE; }
    if (s->emit_physical) {
        if (!s->page_table) { set_error("emit_physical needs a page table"); return SPECATTN_EINVAL; }
        if (!is_pow2(s->page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
        if ((int64_t)s->max_pages_per_seq * s->page_size < s->n_max) { set_error("page table is shorter than n_max"); return SPECATTN_ESHAPE; }
    }
    return SPECATTN_OK;
}

specattn_status check_attn(const specattn_attn_args *a, bool fused)
{
    if (!a) { set_error("attention args are NULL"); return SPECATTN_EINVAL; }
    if (!a->q || !a->k || !a->v || !a->out) { set_error("q, k, v and out must not be NULL"); return SPECATTN_EINVAL; }
    const bool dense = !fused && !a->indices && !a->counts;     // no list: attend to every position
    if (!fused && !dense && (!a->indices || !a->counts)) { set_error("indices and counts must both be given, or both be NULL (dense)"); return SPECATTN_EINVAL; }
    if (dense && a->indices_are_physical) { set_error("indices_are_physical without an index list"); return SPECATTN_EINVAL; }
    if (a->B <= 0 || a->H_q <= 0 || a->H_kv <= 0 || a->T <= 0 || a->d <= 0 || a->n_max <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    if (a->dtype != SPECATTN_F32 && a->dtype != SPECATTN_BF16 && a->dtype != SPECATTN_F16) { set_error("unknown dtype %d", (int)a->dtype); return SPECATTN_EUNSUPPORTED; }
    if (a->H_q % a->H_kv) { set_error("H_q is not a multiple of H_kv"); return SPECATTN_ESHAPE; }
    if (a->T > SPECATTN_MAX_T) { set_error("T exceeds %d", SPECATTN_MAX_T); return SPECATTN_ESHAPE; }
    if (a->d != 64 && a->d != 128) { set_error("d must be 64 or 128"); return SPECATTN_ESHAPE; }
    {
        // more than 64 query rows per kv head only fit the 16-bit route at d = 128 (the fp32 kernel's tables hold 64,
        // and d = 64 has to be able to run there when its workspace is small)
        AttnLaunch probe{};
        probe.dtype = (int)a->dtype; probe.d = a->d; probe.T = a->T; probe.H_kv = a->H_kv;
        if ((a->H_q / a->H_kv) * a->T > 64 && !(attn_mfma_supported(probe) && a->d == 128)) { set_error("G*T exceeds 64 query rows per kv head (only bf16 / fp16 with d = 128 and H_kv <= %d take more)", ATTN_MFMA_MAX_ROWS); return SPECATTN_ESHAPE; }
    }
    if (!fused && !dense && a->idx_capacity < 1) { set_error("idx_capacity must be at least 1"); return SPECATTN_ESHAPE; }
    if (!fused && !dense && a->idx_stride_row < a->idx_capacity) { set_error("idx_stride_row is smaller than idx_capacity"); return SPECATTN_ESHAPE; }
    const bool paged = a->page_table != nullptr || a->indices_are_physical;
    if (paged) {
        if (!is_pow2(a->page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
        if (a->page_table && (int64_t)a->max_pages_per_seq * a->page_size < a->n_max) { set_error("page table is shorter than n_max"); return SPECATTN_ESHAPE; }
        if (a->kv_stride_page <= 0) { set_error("kv_stride_page must be positive"); return SPECATTN_ESHAPE; }
    }
    if (a->chunk_size < 0 || (a->chunk_size > 1 && (!is_pow2(a->chunk_size) || a->chunk_size > 1024))) { set_error("chunk_size must be 0, 1 or a power of two up to 1024"); return SPECATTN_ESHAPE; }
    if (a->chunk_size > 1 && !fused && (dense || a->indices_are_physical)) { set_error("chunk lists are not available with dense calls or physical indices"); return SPECATTN_EUNSUPPORTED; }
    if (a->out_lowp && !aligned(a->out_lowp, 16)) { set_error("out_lowp must be 16-byte aligned"); return SPECATTN_EALIGN; }
    if ((a->k_new == nullptr) != (a->v_new == nullptr)) { set_error("k_new and v_new must both be given or both be NULL"); return SPECATTN_EINVAL; }
    if (a->k_new && (!aligned(a->k_new, 16) || !aligned(a->v_new, 16))) { set_error("k_new and v_new must be 16-byte aligned"); return SPECATTN_EALIGN; }
    if (a->kv_stride_n < a->d) { set_error("kv_stride_n is smaller than d"); return SPECATTN_ESHAPE; }
    const size_t es = a->dtype == SPECATTN_F32 ? 4 : 2;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->out, 16)) { set_error("q, k, v and out must be 16-byte aligned"); return SPECATTN_EALIGN; }
    const int64_t strides[] = {a->q_stride_b, a->q_stride_h, a->q_stride_t, a->kv_stride_b, a->kv_stride_h,
                               a->kv_stride_n, paged ? a->kv_stride_page : 0};
    for (int64_t st : strides)
        if ((st * (int64_t)es) % 16) { set_error("strides must be multiples of 16 bytes"); return SPECATTN_EALIGN; }
    return SPECATTN_OK;
}

specattn_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return SPECATTN_OK;
    if (!ws) { set_error("workspace is NULL, %zu bytes needed", need); return SPECATTN_EWORKSPACE; }
    if (!aligned(ws, 256)) { set_error("workspace must be 256-byte aligned"); return SPECATTN_EWORKSPACE; }
    if (have < need) { set_error("workspace has %zu bytes, %zu needed", have, need); return SPECATTN_EWORKSPACE; }
    return SPECATTN_OK;
}

// The fused call keeps the kept set on chip (mask source of the matrix-core kernel) for bf16 / fp16 with d = 128
// and single positions.  Everything else the two separate calls take (fp32, d = 64, chunk-granular selection)
// runs as those two calls with the list in the caller's workspace instead of caller-visible memory.
bool fused_on_chip(const specattn_select_args *s, const specattn_attn_args *a)
{
    AttnLaunch probe{};
    probe.dtype = (int)a->dtype; probe.d = a->d; probe.T = a->T; probe.H_kv = a->H_kv;
    return attn_mfma_supported(probe) && a->d == 128 && s->chunk_size <= 1;
}
// The least workspace with which a selection of few long rows is split over many workgroups: 32 KiB of counters and a bit
// per position for every row (what such a call asked for when its row histograms were added up in memory).  From it up to
// what specattn_workspace_size asks for, the slices of a row share one histogram.  With less, and for the other shapes
// that are split with less than is asked for, every row is handled by one workgroup.
size_t select_split_asked_bytes(const specattn_select_args *s)
{
    const size_t rows = (size_t)s->B * s->H_kv;
    if (s->n_max < 65536 || rows * 2048 > (size_t)s->n_max) return SIZE_MAX;
    return union_workspace_bytes(s->B, s->H_kv, 1, s->n_max) + rows * 32768 + ((rows * 88 + 255) & ~(size_t)255);
}
size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }
// Positions that the list of a fused call over rows of n positions can stand for: the row, rounded up to whole chunks.
int fused_positions(const specattn_select_args *s, int n)
{
    const int64_t chunk = s->chunk_size > 1 ? s->chunk_size : 1;
    return (int)std::min<int64_t>((n + chunk - 1) / chunk * chunk, INT32_MAX);
}

SelectLaunch make_select(const specattn_select_args *s)
{
    SelectLaunch l{};
    l.probs = s->probs;
    l.stride_b = s->probs_stride_b;
    l.stride_h = s->probs_stride_h;
    l.B = s->B; l.H_kv = s->H_kv; l.n_max = s->n_max;
    l.seq_lens = s->seq_lens;
    l.top_p = s->top_p;
    l.indices = s->indices;
    l.idx_stride = s->idx_stride_row;
    l.idx_capacity = s->indices ? s->idx_capacity : 0;
    l.counts = s->counts;
    l.thresholds = s->thresholds;
    l.row_flags = s->row_flags;
    l.page_table = s->page_table;
    l.page_shift = s->emit_physical ? log2i(s->page_size) : 0;
    l.max_pages = s->max_pages_per_seq;
    l.emit_physical = s->emit_physical;
    l.block_counts = s->block_counts;
    l.blocks_per_row = (s->n_max + SEL_BLOCK - 1) / SEL_BLOCK;
    l.n_tokens = s->n_max;
    l.chunk_shift = 0;
    l.kept_mask = s->kept_mask;
    return l;
}

AttnLaunch make_attn(const specattn_attn_args *a)
{
    AttnLaunch l{};
    l.q = a->q; l.k = a->k; l.v = a->v;
    l.dtype = (int)a->dtype;
    l.B = a->B; l.H_q = a->H_q; l.H_kv = a->H_kv; l.T = a->T; l.d = a->d; l.n_max = a->n_max;
    l.sm_scale = a->sm_scale > 0.0f ? a->sm_scale : 1.0f / std::sqrt((float)a->d);
    l.q_stride_b = a->q_stride_b; l.q_stride_h = a->q_stride_h; l.q_stride_t = a->q_stride_t;
    l.kv_stride_b = a->kv_stride_b; l.kv_stride_h = a->kv_stride_h; l.kv_stride_n = a->kv_stride_n;
    l.page_table = a->page_table;
    const bool paged = a->page_table != nullptr || a->indices_are_physical;
    l.page_shift = paged ? log2i(a->page_size) : 0;
    l.max_pages = a->max_pages_per_seq;
    l.kv_stride_page = a->kv_stride_page;
    l.indices = a->indices;
    l.idx_stride = a->idx_stride_row;
    l.counts = a->counts;
    l.idx_capacity = a->idx_capacity;
    l.indices_are_physical = a->indices_are_physical;
    l.chunk_shift = a->chunk_size > 1 ? log2i(a->chunk_size) : 0;
    l.dense = (!a->indices && !a->counts) ? 1 : 0;          // the fused call overwrites counts afterwards
    if (l.dense) l.idx_capacity = a->n_max;
    l.k_new = a->k_new;
    l.v_new = a->v_new;
    l.out = a->out;
    l.out_lowp = a->out_lowp;
    l.lse = a->lse;
    l.workspace = a->workspace;
    l.workspace_bytes = a->workspace_bytes;
    l.seq_lens = a->seq_lens;
    return l;
}

// ---- the 4-bit cache and the eviction --------------------------------------------------------
specattn_status check_pages(const int32_t *page_table, int page_size, int max_pages, int n_max)
{
    if (!is_pow2(page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
    if (page_table && (int64_t)max_pages * page_size < n_max) { set_error("page table is shorter than n_max"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

// Whether rows of `bytes` bytes (or elements) at these strides share any: dimension by dimension from the smallest stride up, each has to lie beyond all that
// the ones before it reach.
struct Dim { int64_t size; __int128 stride; };
bool rows_overlap(Dim a, Dim b, Dim c, int64_t bytes)
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

specattn_status check_mx_cache(const specattn_mx_cache *c, bool pool)
{
    if (!c->codes || !c->scales) { set_error("codes and scales must not be NULL"); return SPECATTN_EINVAL; }
    if (c->B <= 0 || c->H_kv <= 0 || c->n_max <= 0 || c->d <= 0) { set_error("the cache's sizes must be positive"); return SPECATTN_EINVAL; }
    if (c->d != 64 && c->d != 128) { set_error("d must be 64 or 128"); return SPECATTN_ESHAPE; }
    if ((int64_t)c->B * c->H_kv > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
    // (its rows do not lie at _stride_b and slot * _stride_n: they would be taken from, and put, where others are)
    if (!pool && c->num_pages > 0) { set_error("a pool without a page table takes lists of pool slots alone (num_pages is 0 for a contiguous cache)"); return SPECATTN_EINVAL; }
    if (pool) {
        const specattn_status st = check_pages(c->page_table, c->page_size, c->max_pages_per_seq, c->n_max);
        if (st != SPECATTN_OK) return st;
        if (c->num_pages <= 0) { set_error("num_pages must be positive"); return SPECATTN_EINVAL; }
        if (c->codes_stride_page <= 0 || c->scales_stride_page <= 0) { set_error("page strides must be positive"); return SPECATTN_ESHAPE; }
    }
    if (c->codes_stride_n < c->d || c->scales_stride_n < c->d / 16) { set_error("codes_stride_n and scales_stride_n must not be smaller than d and d / 16"); return SPECATTN_ESHAPE; }
    if (c->codes_stride_h < 0 || c->scales_stride_h < 0 || (!pool && (c->codes_stride_b < 0 || c->scales_stride_b < 0))) { set_error("strides must not be negative"); return SPECATTN_ESHAPE; }
    const int64_t codes[] = {c->codes_stride_h, c->codes_stride_n, pool ? c->codes_stride_page : c->codes_stride_b};
    const int64_t scales[] = {c->scales_stride_h, c->scales_stride_n, pool ? c->scales_stride_page : c->scales_stride_b};
    for (int i = 0; i < 3; ++i)
        if (codes[i] % 16 || scales[i] % 4) { set_error("strides of the codes must be multiples of 16 bytes, of the scales of 4"); return SPECATTN_EALIGN; }
    if (!aligned(c->codes, 16) || !aligned(c->scales, 4)) { set_error("codes must be 16-byte, scales 4-byte aligned"); return SPECATTN_EALIGN; }
    return SPECATTN_OK;
}

MxCache make_mx_cache(const specattn_mx_cache *c, bool pool)
{
    MxCache m{};
    m.codes = c->codes; m.scales = c->scales;
    m.codes_b = c->codes_stride_b; m.codes_h = c->codes_stride_h; m.codes_n = c->codes_stride_n; m.codes_page = c->codes_stride_page;
    m.scales_b = c->scales_stride_b; m.scales_h = c->scales_stride_h; m.scales_n = c->scales_stride_n; m.scales_page = c->scales_stride_page;
    m.page_table = c->page_table;
    m.page_shift = pool ? log2i(c->page_size) : 0;
    m.max_pages = c->max_pages_per_seq;
    m.num_pages = c->num_pages;
    m.B = c->B; m.H_kv = c->H_kv; m.n_max = c->n_max; m.d = c->d;
    return m;
}

specattn_status check_mx_rows(const specattn_mx_rows_args *r, bool store)
{
    if (!r) { set_error("rows args are NULL"); return SPECATTN_EINVAL; }
    const specattn_mx_cache *c = &r->cache;
    const bool pool = c->page_table != nullptr;
    const specattn_status st = check_mx_cache(c, pool);
    if (st != SPECATTN_OK) return st;
    // what is written must not share bytes: the rows of the cache here, those of k and v below
    const int64_t outer = pool ? c->num_pages : c->B, inner = pool ? c->page_size : c->n_max;
    if (store && (rows_overlap({outer, pool ? c->codes_stride_page : c->codes_stride_b}, {c->H_kv, c->codes_stride_h}, {inner, c->codes_stride_n}, c->d) ||
                  rows_overlap({outer, pool ? c->scales_stride_page : c->scales_stride_b}, {c->H_kv, c->scales_stride_h}, {inner, c->scales_stride_n}, c->d / 16))) {
        set_error("rows of the cache share bytes");
        return SPECATTN_ESHAPE;
    }
    if (!r->k || !r->v) { set_error("k and v must not be NULL"); return SPECATTN_EINVAL; }
    if (r->T <= 0) { set_error("T must be positive"); return SPECATTN_EINVAL; }
    // (256 threads to 32 rows or more, and a launch has fewer than 2^32 along an axis; rows are counted in 31 bits, whole workgroups of them)
    if (r->T > (1 << 28)) { set_error("more than 2^28 rows per sequence"); return SPECATTN_ESHAPE; }
    if (r->dtype != SPECATTN_F32 && r->dtype != SPECATTN_BF16 && r->dtype != SPECATTN_F16) { set_error("unknown dtype %d", (int)r->dtype); return SPECATTN_EUNSUPPORTED; }
    const int64_t es = r->dtype == SPECATTN_F32 ? 4 : 2;
    if ((r->stride_b * es) % 16 || (r->stride_h * es) % 16 || (r->stride_t * es) % 16) { set_error("strides must be multiples of 16 bytes"); return SPECATTN_EALIGN; }
    if (!store && rows_overlap({c->B, r->stride_b}, {c->H_kv, r->stride_h}, {r->T, r->stride_t}, c->d)) { set_error("rows of k and v share bytes"); return SPECATTN_ESHAPE; }
    if (!aligned(r->k, 16) || !aligned(r->v, 16)) { set_error("k and v must be 16-byte aligned"); return SPECATTN_EALIGN; }
    return SPECATTN_OK;
}

MxRowsLaunch make_mx_rows(const specattn_mx_rows_args *r)
{
    MxRowsLaunch l{};
    l.c = make_mx_cache(&r->cache, r->cache.page_table != nullptr);
    l.k = r->k; l.v = r->v;
    l.dtype = (int)r->dtype;
    l.T = r->T;
    l.stride_b = r->stride_b; l.stride_h = r->stride_h; l.stride_t = r->stride_t;
    l.starts = r->starts; l.counts = r->counts;
    return l;
}

specattn_status check_mx_attn(const specattn_mx_attn_args *a)
{
    if (!a) { set_error("attention args are NULL"); return SPECATTN_EINVAL; }
    const specattn_mx_cache *c = &a->cache;
    const bool pool = c->page_table != nullptr || a->indices_are_physical;
    const specattn_status st = check_mx_cache(c, pool);
    if (st != SPECATTN_OK) return st;
    if (!a->q || (!a->out && !a->out_lowp)) { set_error("q and one of out and out_lowp must not be NULL"); return SPECATTN_EINVAL; }
    const bool dense = !a->indices && !a->counts;
    if (!dense && (!a->indices || !a->counts)) { set_error("indices and counts must both be given, or both be NULL (dense)"); return SPECATTN_EINVAL; }
    if (dense && a->indices_are_physical) { set_error("indices_are_physical without an index list"); return SPECATTN_EINVAL; }
    if (a->H_q <= 0 || a->T <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    if (a->dtype != SPECATTN_BF16 && a->dtype != SPECATTN_F16) { set_error("queries of a 4-bit cache are bf16 or fp16"); return SPECATTN_EUNSUPPORTED; }
    if (a->H_q % c->H_kv) { set_error("H_q is not a multiple of H_kv"); return SPECATTN_ESHAPE; }
    if (a->T > SPECATTN_MAX_T) { set_error("T exceeds %d", SPECATTN_MAX_T); return SPECATTN_ESHAPE; }
    if (!dense && a->idx_capacity < 1) { set_error("idx_capacity must be at least 1"); return SPECATTN_ESHAPE; }
    if (!dense && a->idx_stride_row < a->idx_capacity) { set_error("idx_stride_row is smaller than idx_capacity"); return SPECATTN_ESHAPE; }
    if (a->chunk_size < 0 || (a->chunk_size > 1 && (!is_pow2(a->chunk_size) || a->chunk_size > 1024))) { set_error("chunk_size must be 0, 1 or a power of two up to 1024"); return SPECATTN_ESHAPE; }
    if (a->chunk_size > 1 && (dense || a->indices_are_physical)) { set_error("chunk lists are not available with dense calls or physical indices"); return SPECATTN_EUNSUPPORTED; }
    // the tiles of a launch are counted in 31 bits, and row offsets go to the kernel in units of 16 (codes) and 4 bytes (scales) in 32 bits
    const int64_t most = dense ? c->n_max : (int64_t)a->idx_capacity * (a->chunk_size > 1 ? a->chunk_size : 1);
    if (most > (1 << 24)) { set_error("more than 2^24 positions per row"); return SPECATTN_ESHAPE; }
    const __int128 reach = pool ? (__int128)(c->num_pages - 1) * c->codes_stride_page + (__int128)(c->page_size - 1) * c->codes_stride_n : (__int128)(c->n_max - 1) * c->codes_stride_n;
    const __int128 scales_reach = pool ? (__int128)(c->num_pages - 1) * c->scales_stride_page + (__int128)(c->page_size - 1) * c->scales_stride_n : (__int128)(c->n_max - 1) * c->scales_stride_n;
    if (reach >= ((__int128)1 << 36) || scales_reach >= ((__int128)1 << 34)) { set_error("the rows of a kv head must lie within 64 GiB of its first one (their scales within 16 GiB)"); return SPECATTN_ESHAPE; }
    if ((a->k_new == nullptr) != (a->v_new == nullptr)) { set_error("k_new and v_new must both be given or both be NULL"); return SPECATTN_EINVAL; }
    if (!aligned(a->q, 16) || !aligned(a->k_new, 16) || !aligned(a->v_new, 16) || !aligned(a->out, 16) || !aligned(a->out_lowp, 16)) { set_error("q, k_new, v_new, out and out_lowp must be 16-byte aligned"); return SPECATTN_EALIGN; }
    if (a->q_stride_b % 8 || a->q_stride_h % 8 || a->q_stride_t % 8) { set_error("strides must be multiples of 16 bytes"); return SPECATTN_EALIGN; }
    return SPECATTN_OK;
}

MxAttnLaunch make_mx_attn(const specattn_mx_attn_args *a)
{
    const specattn_mx_cache *c = &a->cache;
    const bool pool = c->page_table != nullptr || a->indices_are_physical;
    MxAttnLaunch m{};
    m.c = make_mx_cache(c, pool);
    if (a->indices_are_physical) m.c.page_table = nullptr;
    AttnLaunch &l = m.a;
    l.q = a->q;
    l.dtype = (int)a->dtype;
    l.B = c->B; l.H_q = a->H_q; l.H_kv = c->H_kv; l.T = a->T; l.d = c->d; l.n_max = c->n_max;
    l.sm_scale = a->sm_scale > 0.0f ? a->sm_scale : 1.0f / std::sqrt((float)c->d);
    l.q_stride_b = a->q_stride_b; l.q_stride_h = a->q_stride_h; l.q_stride_t = a->q_stride_t;
    l.page_table = m.c.page_table;
    l.page_shift = m.c.page_shift;
    l.max_pages = c->max_pages_per_seq;
    l.indices = a->indices;
    l.idx_stride = a->idx_stride_row;
    l.counts = a->counts;
    l.idx_capacity = a->idx_capacity;
    l.indices_are_physical = a->indices_are_physical;
    l.chunk_shift = a->chunk_size > 1 ? log2i(a->chunk_size) : 0;
    l.dense = (!a->indices && !a->counts) ? 1 : 0;
    l.k_new = a->k_new;
    l.v_new = a->v_new;
    l.out = a->out;
    l.out_lowp = a->out_lowp;
    l.lse = a->lse;
    l.workspace = a->workspace;
    l.workspace_bytes = a->workspace_bytes;
    l.seq_lens = a->seq_lens;
    return m;
}

constexpr int MAX_EVICT_ROWS = (1 << 22) - 1;                 // a launch has fewer than 2^32 threads along an axis, a row 1024

specattn_status check_evict(const specattn_evict_args *e)
{
    if (!e) { set_error("evict args are NULL"); return SPECATTN_EINVAL; }
    if (!e->scores || !e->positions || !e->scores_out || !e->positions_out || !e->next_positions || !e->move_src || !e->move_dst || !e->move_counts || !e->new_lens) { set_error("scores, positions, their outputs, next_positions, the moves and new_lens must not be NULL"); return SPECATTN_EINVAL; }
    if (e->B <= 0 || e->H <= 0 || e->n_max <= 0 || e->budget <= 0) { set_error("B, H, n_max and budget must be positive"); return SPECATTN_EINVAL; }
    if (!(e->decay >= 0.0 && e->decay <= 1.0)) { set_error("decay must lie in [0, 1]"); return SPECATTN_EINVAL; }
    if (e->new_lens == e->seq_lens) { set_error("new_lens must not be seq_lens"); return SPECATTN_EINVAL; }
    if (e->n_max > SPECATTN_MAX_N) { set_error("n_max %d exceeds %d", e->n_max, SPECATTN_MAX_N); return SPECATTN_ESHAPE; }
    if (e->probs) {
        if (e->H_draft <= 0 || e->S <= 0) { set_error("H_draft and S must be positive"); return SPECATTN_EINVAL; }
        if (e->H_draft % e->H) { set_error("H_draft is not a multiple of H"); return SPECATTN_ESHAPE; }
        if ((int64_t)e->B * e->H_draft * e->S > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
        if (e->probs_stride_row < e->n_max) { set_error("probs_stride_row is smaller than n_max"); return SPECATTN_ESHAPE; }
    }
    if ((int64_t)e->B * e->H > MAX_EVICT_ROWS) { set_error("too many rows"); return SPECATTN_ESHAPE; }
    if (e->row_stride_h < e->n_max || e->row_stride_b < e->n_max) { set_error("row strides are smaller than n_max"); return SPECATTN_ESHAPE; }
    if (rows_overlap({e->B, e->row_stride_b}, {e->H, e->row_stride_h}, {1, 0}, e->n_max)) { set_error("rows of the scores share entries"); return SPECATTN_ESHAPE; }
    if (e->sinks < 0 || e->recent < 0 || (int64_t)e->sinks + e->recent > e->budget) { set_error("sinks and recent must not be negative, nor exceed the budget together"); return SPECATTN_ESHAPE; }
    if (e->move_capacity < 1 || e->move_capacity < std::min(e->budget, e->n_max - e->budget)) { set_error("move_capacity must be at least 1 and hold min(budget, n_max - budget) moves"); return SPECATTN_ESHAPE; }
    if (e->move_stride_row < e->move_capacity) { set_error("move_stride_row is smaller than move_capacity"); return SPECATTN_ESHAPE; }
    return SPECATTN_OK;
}

specattn_status check_move(const specattn_move_args *m)
{
    if (!m) { set_error("move args are NULL"); return SPECATTN_EINVAL; }
    if (!m->move_src || !m->move_dst || !m->move_counts) { set_error("the moves must not be NULL"); return SPECATTN_EINVAL; }
    if (m->B <= 0 || m->H <= 0 || m->n_max <= 0) { set_error("B, H and n_max must be positive"); return SPECATTN_EINVAL; }
    if (m->n_max > SPECATTN_MAX_N) { set_error("n_max %d exceeds %d", m->n_max, SPECATTN_MAX_N); return SPECATTN_ESHAPE; }
    if (m->move_capacity < 1 || m->move_capacity > m->n_max) { set_error("move_capacity must lie in 1..n_max"); return SPECATTN_ESHAPE; }
    if (m->move_stride_row < m->move_capacity) { set_error("move_stride_row is smaller than move_capacity"); return SPECATTN_ESHAPE; }
    if (m->num_planes < 1 || m->num_planes > SPECATTN_MAX_PLANES) { set_error("num_planes must lie in 1..%d", SPECATTN_MAX_PLANES); return SPECATTN_ESHAPE; }
    if (m->page_table) {
        const specattn_status st = check_pages(m->page_table, m->page_size, m->max_pages_per_seq, m->n_max);
        if (st != SPECATTN_OK) return st;
    }
    for (int i = 0; i < m->num_planes; ++i) {
        const specattn_move_plane *p = &m->planes[i];
        if (!p->data) { set_error("plane %d has no data", i); return SPECATTN_EINVAL; }
        if (p->H_kv <= 0 || p->H_kv % m->H) { set_error("H_kv of plane %d is not a positive multiple of H", i); return SPECATTN_ESHAPE; }
        if ((int64_t)m->B * p->H_kv > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
        if (p->row_bytes < 4 || p->row_bytes > 8192 || p->row_bytes % 4) { set_error("row_bytes of plane %d must be a multiple of 4 up to 8192", i); return SPECATTN_ESHAPE; }
        if (p->stride_n < p->row_bytes) { set_error("stride_n of plane %d is smaller than row_bytes", i); return SPECATTN_ESHAPE; }
        if (m->page_table && (p->num_pages <= 0 || p->stride_page <= 0)) { set_error("plane %d needs num_pages and a page stride", i); return SPECATTN_ESHAPE; }
        const int unit = p->row_bytes % 16 == 0 ? 16 : p->row_bytes % 8 == 0 ? 8 : 4;
        const int64_t outer = m->page_table ? p->stride_page : p->stride_b;
        if (p->stride_h < 0 || outer < 0) { set_error("strides of plane %d must not be negative", i); return SPECATTN_ESHAPE; }      // (offsets below 0 mean no such slot)
        if (!aligned(p->data, unit) || p->stride_h % unit || p->stride_n % unit || outer % unit) { set_error("data and strides of plane %d must be multiples of %d bytes", i, unit); return SPECATTN_EALIGN; }
    }
    for (int i = 0; i < m->num_planes; ++i) {
        const specattn_move_plane *p = &m->planes[i];
        const Dim outer = m->page_table ? Dim{p->num_pages, p->stride_page} : Dim{m->B, p->stride_b}, inner = {m->page_table ? m->page_size : m->n_max, p->stride_n};
        if (rows_overlap(outer, {p->H_kv, p->stride_h}, inner, p->row_bytes)) { set_error("rows of plane %d share bytes", i); return SPECATTN_ESHAPE; }
    }
    return SPECATTN_OK;
}

}  // namespace
}  // namespace specattn

using namespace specattn;

extern "C" {

static size_t workspace_bytes(const specattn_select_args *sel, const specattn_attn_args *attn, bool full);

specattn_status specattn_topp_select(const specattn_select_args *sel, void *workspace, size_t workspace_bytes,
                                     void *stream)
{
    clear_error();
    specattn_status st = check_select(sel, false);
    if (st != SPECATTN_OK) return st;
    const bool plain = sel->bisect_iters == 0 && sel->chunk_size <= 1;
    const size_t need = specattn_workspace_size(sel, nullptr);
    // the plain selection works without a workspace; with one, few long rows are split over many workgroups
    const bool given = plain && need > 0 && workspace && aligned(workspace, 256);
    const bool asked = given && workspace_bytes >= select_split_asked_bytes(sel);
    const bool split = asked || (given && workspace_bytes >= need);
    if (asked && sel->kept_mask) { set_error("kept_mask is not written by the split selection of few long rows: call without a workspace"); return SPECATTN_EUNSUPPORTED; }
    if (!plain) {
        st = check_workspace(workspace, workspace_bytes, need);
        if (st != SPECATTN_OK) return st;
    }
    SelectLaunch l = make_select(sel);
    if (split && !sel->kept_mask) return launch_select_multi_wg(l, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    if (sel->bisect_iters > 0) {                    // Algorithm 2 as the paper runs it, then the mask and compaction passes
        // workspace: [tau][valid][flags][block counts][ballots], the layout of the union with one member per row
        const size_t rows = (size_t)sel->B * sel->H_kv, a256 = (rows * 4 + 255) & ~(size_t)255;
        char *ws = static_cast<char *>(workspace);
        float *tau = sel->thresholds ? sel->thresholds : reinterpret_cast<float *>(ws);
        int32_t *valid = reinterpret_cast<int32_t *>(ws + a256);
        uint32_t *mflags = reinterpret_cast<uint32_t *>(ws + 2 * a256);
        hipStream_t hs = static_cast<hipStream_t>(stream);
        st = launch_bisect_thresholds(l, sel->bisect_iters, tau, valid, mflags, hs);
        if (st != SPECATTN_OK) return st;
        return launch_threshold_union(sel->probs, sel->probs_stride_b, sel->probs_stride_h, sel->B, sel->H_kv, 1, sel->n_max,
                                      sel->seq_lens, tau, valid, mflags, ws + 3 * a256, sel->indices, sel->idx_stride_row,
                                      sel->idx_capacity, sel->counts, sel->row_flags, sel->page_table, sel->page_size,
                                      sel->max_pages_per_seq, sel->emit_physical, nullptr, hs);
    }
    if (sel->chunk_size > 1) {                      // the selection runs over chunk masses
        const int cs = log2i(sel->chunk_size);
        const int nc = (sel->n_max + sel->chunk_size - 1) >> cs;
        l.n_max = nc;
        l.chunk_shift = cs;
        l.blocks_per_row = (nc + SEL_BLOCK - 1) / SEL_BLOCK;
        if (select_takes_chunks(sel->B * sel->H_kv, sel->n_max, nc)) return launch_select_chunks(l, static_cast<hipStream_t>(stream));
        float *mass = static_cast<float *>(workspace);
        st = launch_chunk_masses(sel->probs, sel->probs_stride_b, sel->probs_stride_h, sel->B, sel->H_kv, sel->n_max,
                                 sel->seq_lens, cs, nc, mass, static_cast<hipStream_t>(stream));
        if (st != SPECATTN_OK) return st;
        l.probs = mass;
        l.stride_b = (int64_t)sel->H_kv * nc;
        l.stride_h = nc;
    }
    return launch_select(l, static_cast<hipStream_t>(stream));
}

static specattn_status check_union(const specattn_union_args *u)
{
    if (!u) { set_error("union args are NULL"); return SPECATTN_EINVAL; }
    if (!u->probs || !u->counts || !u->indices) { set_error("probs, indices and counts must not be NULL"); return SPECATTN_EINVAL; }
    if (!(u->top_p > 0.0f && u->top_p <= 1.0f)) { set_error("top_p must be in (0, 1]"); return SPECATTN_EINVAL; }
    if (u->B <= 0 || u->H_draft <= 0 || u->S <= 0 || u->H_kv <= 0 || u->n_max <= 0) { set_error("sizes must be positive"); return SPECATTN_EINVAL; }
    if (u->H_draft % u->H_kv) { set_error("H_draft is not a multiple of H_kv"); return SPECATTN_ESHAPE; }
    if (u->n_max > SPECATTN_MAX_N) { set_error("n_max exceeds %d", SPECATTN_MAX_N); return SPECATTN_ESHAPE; }
    if ((int64_t)u->B * u->H_draft * u->S > (1 << 24)) { set_error("too many rows"); return SPECATTN_ESHAPE; }
    if (u->probs_stride_row < u->n_max) { set_error("probs_stride_row is smaller than n_max"); return SPECATTN_ESHAPE; }
    if (u->idx_capacity < 1) { set_error("idx_capacity must be at least 1"); return SPECATTN_ESHAPE; }
    if (u->idx_stride_row < u->idx_capacity) { set_error("idx_stride_row is smaller than idx_capacity"); return SPECATTN_ESHAPE; }
    if (u->emit_physical && !u->page_table) { set_error("emit_physical needs a page table"); return SPECATTN_EINVAL; }
    if (u->page_table) {
        if (!is_pow2(u->page_size)) { set_error("page_size must be a power of two"); return SPECATTN_ESHAPE; }
        if ((int64_t)u->max_pages_per_seq * u->page_size < u->n_max) { set_error("page table is shorter than n_max"); return SPECATTN_ESHAPE; }
    }
    return SPECATTN_OK;
}

size_t specattn_union_workspace_size(const specattn_union_args *u)
{
    if (!u || u->B <= 0 || u->H_draft <= 0 || u->S <= 0 || u->H_kv <= 0 || u->n_max <= 0 || u->H_draft % u->H_kv) return 0;
    const int M = (u->H_draft / u->H_kv) * u->S;
    return union_workspace_bytes(u->B, u->H_kv, M, u->n_max) + union_masks_bytes(u->B, u->H_kv, M, u->n_max);
}

specattn_status specattn_topp_select_union(const specattn_union_args *u, void *workspace, size_t workspace_bytes,
                                           void *stream)
{
    clear_error();
    specattn_status st = check_union(u);
    if (st != SPECATTN_OK) return st;
    // (accepted without room for the members' kept bits: the rows are then read a second time)
    st = check_workspace(workspace, workspace_bytes, union_workspace_bytes(u->B, u->H_kv, (u->H_draft / u->H_kv) * u->S, u->n_max));
    if (st != SPECATTN_OK) return st;
    return launch_union(u, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

specattn_status specattn_sparse_decode_attn(const specattn_attn_args *attn, void *stream)
{
    clear_error();
    specattn_status st = check_attn(attn, false);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(attn->workspace, attn->workspace_bytes, workspace_bytes(nullptr, attn, false));
    if (st != SPECATTN_OK) return st;
    return launch_attn(make_attn(attn), static_cast<hipStream_t>(stream));
}

specattn_status specattn_lists_to_csr(const int32_t *indices, int64_t idx_stride_row, int32_t idx_capacity,
                                      const int32_t *counts, int32_t rows, int64_t *indptr, int32_t *packed, void *stream)
{
    clear_error();
    if (!counts || !indptr || (packed && !indices)) { set_error("counts and indptr must not be NULL, and packed needs indices"); return SPECATTN_EINVAL; }
    if (rows <= 0) { set_error("rows must be positive"); return SPECATTN_EINVAL; }
    if (idx_capacity < 1 || (packed && idx_stride_row < idx_capacity)) { set_error("idx_capacity must be at least 1 and idx_stride_row no smaller"); return SPECATTN_ESHAPE; }
    return launch_csr(indices, idx_stride_row, counts, rows, idx_capacity, indptr, packed, static_cast<hipStream_t>(stream));
}

specattn_status specattn_check_lists(const specattn_attn_args *attn, int64_t pool_slots, int32_t *n_bad, void *stream)
{
    clear_error();
    specattn_status st = check_attn(attn, false);
    if (st != SPECATTN_OK) return st;
    if (!attn->indices) { set_error("a dense call has no index list to check"); return SPECATTN_EINVAL; }
    if (!n_bad || pool_slots < 0) { set_error("n_bad must not be NULL and pool_slots must not be negative"); return SPECATTN_EINVAL; }
    return launch_check_lists(make_attn(attn), pool_slots, n_bad, static_cast<hipStream_t>(stream));
}

specattn_status specattn_fused(const specattn_select_args *sel, const specattn_attn_args *attn, void *stream)
{
    clear_error();
    specattn_status st = check_select(sel, true);
    if (st != SPECATTN_OK) return st;
    st = check_attn(attn, true);
    if (st != SPECATTN_OK) return st;
    if (sel->B != attn->B || sel->H_kv != attn->H_kv || sel->n_max != attn->n_max) {
        set_error("selection and attention arguments describe different rows");
        return SPECATTN_ESHAPE;
    }
    if (sel->reuse_selection && (!sel->kept_mask || !sel->block_counts)) {
        set_error("reuse_selection needs block_counts and kept_mask");
        return SPECATTN_EINVAL;
    }
    if (attn->indices_are_physical) {
        set_error("the fused call has no index list: indices_are_physical does not apply (pass the page table)");
        return SPECATTN_EUNSUPPORTED;
    }
    st = check_workspace(attn->workspace, attn->workspace_bytes, workspace_bytes(sel, attn, false));
    if (st != SPECATTN_OK) return st;
    const int rows = sel->B * sel->H_kv;
    const bool full = attn->workspace_bytes >= workspace_bytes(sel, attn, true);
    const size_t attn_bytes = (full ? attn_workspace_bytes : attn_workspace_accepted_bytes)(rows, attn->H_q / attn->H_kv, attn->T, attn->d, fused_positions(sel, attn->n_max));
    if (!fused_on_chip(sel, attn)) {
        // selection into the workspace, then attention over that list
        if (sel->reuse_selection || sel->block_counts || sel->kept_mask) {
            set_error("reuse_selection, block_counts and kept_mask belong to the on-chip fused path (bf16 / fp16, d = 128, single positions)");
            return SPECATTN_EUNSUPPORTED;
        }
        const int chunk = sel->chunk_size > 1 ? sel->chunk_size : 1;
        const int cap = (sel->n_max + chunk - 1) / chunk;
        char *ws = static_cast<char *>(attn->workspace);
        specattn_select_args s2 = *sel;
        s2.indices = reinterpret_cast<int32_t *>(ws + attn_bytes);
        s2.idx_stride_row = cap;
        s2.idx_capacity = cap;
        s2.emit_physical = 0;
        const size_t list_bytes = a256((size_t)rows * cap * sizeof(int32_t));
        // (a call accepted with less room than it asks for selects with one workgroup per row)
        const size_t sel_bytes = full ? specattn_workspace_size(&s2, nullptr) : attn->workspace_bytes - attn_bytes - list_bytes;
        st = specattn_topp_select(&s2, sel_bytes ? ws + attn_bytes + list_bytes : nullptr, sel_bytes, stream);
        if (st != SPECATTN_OK) return st;
        specattn_attn_args a2 = *attn;
        a2.indices = s2.indices;
        a2.idx_stride_row = cap;
        a2.idx_capacity = cap;
        a2.counts = sel->counts;
        a2.chunk_size = sel->chunk_size;
        a2.indices_are_physical = 0;
        a2.seq_lens = sel->seq_lens;
        a2.workspace_bytes = attn_bytes;
        return specattn_sparse_decode_attn(&a2, stream);
    }
    AttnLaunch al = make_attn(attn);
    const int blocks = (sel->n_max + SEL_BLOCK - 1) / SEL_BLOCK;
    // workspace: [attention partials][block counts: rows * blocks ints][kept mask: rows * blocks * 32 words]
    al.workspace_bytes = attn_bytes;
    char *extra = static_cast<char *>(attn->workspace) + attn_bytes;
    int32_t *bc = sel->block_counts ? sel->block_counts : reinterpret_cast<int32_t *>(extra);
    extra += ((size_t)rows * blocks * sizeof(int32_t) + 255) & ~(size_t)255;
    uint32_t *mask = sel->kept_mask ? sel->kept_mask : reinterpret_cast<uint32_t *>(extra);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!sel->reuse_selection) {
        SelectLaunch sl = make_select(sel);
        sl.indices = nullptr;
        sl.idx_capacity = 0;
        sl.block_counts = bc;
        sl.blocks_per_row = blocks;
        sl.kept_mask = mask;
        st = launch_select(sl, s);
        if (st != SPECATTN_OK) return st;
    }
    al.indices = nullptr;
    al.dense = 0;
    al.counts = sel->counts;
    al.idx_capacity = sel->n_max;
    al.idx_stride = 0;
    al.seq_lens = sel->seq_lens;
    al.kept_mask = mask;
    al.block_counts = bc;
    al.blocks_per_row = blocks;
    return launch_attn_mfma(al, s);
}

// What a call asks for (full), or the least it is accepted with: an attention call with less room than it asks for takes
// fewer query rows per launch, or the kernel with the smaller partials.
static size_t workspace_bytes(const specattn_select_args *sel, const specattn_attn_args *attn, bool full)
{
    if (!sel && !attn) return 0;
    if (sel && !attn) {                               // token selection keeps its state on chip;
        if (sel->bisect_iters > 0) {
            if (sel->B <= 0 || sel->H_kv <= 0 || sel->n_max <= 0) return 0;
            return union_workspace_bytes(sel->B, sel->H_kv, 1, sel->n_max);
        }
        if (sel->chunk_size <= 1) {                   // optional: lets few long rows be split over many workgroups
            if (sel->B <= 0 || sel->H_kv <= 0 || sel->n_max <= 0 || !sel->indices || sel->block_counts) return 0;
            if (!select_multi_wg_preferred(sel->B * sel->H_kv, sel->n_max, sel->top_p)) return 0;
            return select_multi_wg_bytes(sel->B * sel->H_kv, sel->n_max);
        }
        if (sel->B <= 0 || sel->H_kv <= 0 || sel->n_max <= 0 || !is_pow2(sel->chunk_size)) return 0;
        const size_t nc = ((size_t)sel->n_max + sel->chunk_size - 1) / sel->chunk_size;
        return ((size_t)sel->B * sel->H_kv * nc * sizeof(float) + 255) & ~(size_t)255;
    }
    if (attn->B <= 0 || attn->H_kv <= 0 || attn->H_q <= 0 || attn->T <= 0 || attn->d <= 0) return 0;
    if (attn->H_q % attn->H_kv) return 0;
    const int rows = attn->B * attn->H_kv;
    const bool dense = !attn->indices && !attn->counts;
    const int cap = sel ? fused_positions(sel, attn->n_max) : dense ? attn->n_max : attn->idx_capacity * (attn->chunk_size > 1 ? attn->chunk_size : 1);
    if (cap <= 0) return 0;
    size_t bytes = (full ? attn_workspace_bytes : attn_workspace_accepted_bytes)(rows, attn->H_q / attn->H_kv, attn->T, attn->d, cap);
    if (sel && !fused_on_chip(sel, attn)) {           // fused by way of a list in the workspace
        if (sel->n_max <= 0) return 0;
        const int chunk = sel->chunk_size > 1 ? sel->chunk_size : 1;
        const int lcap = (sel->n_max + chunk - 1) / chunk;
        specattn_select_args s2 = *sel;
        s2.indices = reinterpret_cast<int32_t *>(0x1000);      // (only tested for NULL by the size query)
        size_t sel_bytes = specattn_workspace_size(&s2, nullptr);
        if (!full && chunk == 1 && sel_bytes > 0) {            // the plain selection runs without a workspace as well
            const size_t asked = select_split_asked_bytes(&s2);
            sel_bytes = std::min(sel_bytes, asked == SIZE_MAX ? 0 : asked);
        }
        bytes = a256(bytes) + a256((size_t)rows * lcap * sizeof(int32_t)) + sel_bytes;
        return bytes;
    }
    if (sel) {                                        // fused: room for the block counts and the kept mask
        const size_t blocks = ((size_t)attn->n_max + SEL_BLOCK - 1) / SEL_BLOCK;
        bytes += ((size_t)rows * blocks * sizeof(int32_t) + 255) & ~(size_t)255;
        bytes += ((size_t)rows * blocks * (SEL_BLOCK / 32) * sizeof(uint32_t) + 255) & ~(size_t)255;
    }
    return bytes;
}

size_t specattn_workspace_size(const specattn_select_args *sel, const specattn_attn_args *attn)
{
    return workspace_bytes(sel, attn, true);
}

specattn_status specattn_mx_store(const specattn_mx_rows_args *args, void *stream)
{
    clear_error();
    const specattn_status st = check_mx_rows(args, true);
    if (st != SPECATTN_OK) return st;
    return launch_mx_store(make_mx_rows(args), static_cast<hipStream_t>(stream));
}

specattn_status specattn_mx_load(const specattn_mx_rows_args *args, void *stream)
{
    clear_error();
    const specattn_status st = check_mx_rows(args, false);
    if (st != SPECATTN_OK) return st;
    return launch_mx_load(make_mx_rows(args), static_cast<hipStream_t>(stream));
}

size_t specattn_mx_workspace_size(const specattn_mx_attn_args *a)
{
    if (!a || a->cache.B <= 0 || a->cache.H_kv <= 0 || a->H_q <= 0 || a->T <= 0 || a->T > SPECATTN_MAX_T || a->H_q % a->cache.H_kv) return 0;
    if ((a->cache.d != 64 && a->cache.d != 128) || (int64_t)a->cache.B * a->cache.H_kv > (1 << 24)) return 0;
    return mx_attn_workspace_bytes(a->cache.B * a->cache.H_kv, a->H_q / a->cache.H_kv, a->T, a->cache.d);
}

specattn_status specattn_mx_decode_attn(const specattn_mx_attn_args *args, void *stream)
{
    clear_error();
    specattn_status st = check_mx_attn(args);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(args->workspace, args->workspace_bytes, specattn_mx_workspace_size(args));
    if (st != SPECATTN_OK) return st;
    return launch_mx_attn(make_mx_attn(args), static_cast<hipStream_t>(stream));
}

size_t specattn_evict_workspace_size(const specattn_evict_args *e)
{
    if (!e || e->B <= 0 || e->H <= 0 || e->n_max <= 0 || e->n_max > SPECATTN_MAX_N || (int64_t)e->B * e->H > MAX_EVICT_ROWS) return 0;
    return evict_workspace_bytes(e);
}

specattn_status specattn_evict_select(const specattn_evict_args *args, void *workspace, size_t workspace_bytes, void *stream)
{
    clear_error();
    specattn_status st = check_evict(args);
    if (st != SPECATTN_OK) return st;
    st = check_workspace(workspace, workspace_bytes, evict_workspace_bytes(args));
    if (st != SPECATTN_OK) return st;
    return launch_evict_select(args, workspace, static_cast<hipStream_t>(stream));
}

specattn_status specattn_evict_move(const specattn_move_args *args, void *stream)
{
    clear_error();
    const specattn_status st = check_move(args);
    if (st != SPECATTN_OK) return st;
    return launch_evict_move(args, static_cast<hipStream_t>(stream));
}

// Device address of this GPU's copy of `scratch`, looked up once per device (any thread may call).
static specattn_status static_scratch(void **out)
{
    constexpr int MAX_DEVICES = 64;
    static std::mutex mu;
    static void *ptr[MAX_DEVICES] = {nullptr};
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) {
        (void)hipGetLastError();
        set_error("no current device, or its ordinal is beyond %d", MAX_DEVICES - 1);
        return SPECATTN_EHIP;
    }
    std::lock_guard<std::mutex> lock(mu);
    if (!ptr[dev]) {
        void *p = nullptr;
        const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p) {
            (void)hipGetLastError();
            set_error("hipGetSymbolAddress(scratch) failed on device %d: %s", dev, hipGetErrorString(e));
            return SPECATTN_EHIP;
        }
        ptr[dev] = p;
    }
    *out = ptr[dev];
    return SPECATTN_OK;
}

specattn_status specattn_sparse_decode_attn_static(const specattn_attn_args *attn, void *stream)
{
    clear_error();
    specattn_status st = check_attn(attn, false);
    if (st != SPECATTN_OK) return st;
    // the least the call runs with: batches beyond 512 rows then go out in launches of 512 rows
    const bool dense = !attn->indices && !attn->counts;
    const int cap = dense ? attn->n_max : attn->idx_capacity * (attn->chunk_size > 1 ? attn->chunk_size : 1);
    const size_t need = cap <= 0 ? 0 : attn_workspace_min_bytes(attn->B * attn->H_kv, attn->H_q / attn->H_kv, attn->T, attn->d, cap);
    if (need == 0 || need > (size_t)SPECATTN_STATIC_SCRATCH_BYTES) {
        set_error("this call needs %zu bytes of scratch memory; the built-in buffer holds %zu", need,
                  (size_t)SPECATTN_STATIC_SCRATCH_BYTES);
        return SPECATTN_EWORKSPACE;
    }
    void *ws = nullptr;
    st = static_scratch(&ws);
    if (st != SPECATTN_OK) return st;
    AttnLaunch l = make_attn(attn);
    l.workspace = ws;
    l.workspace_bytes = SPECATTN_STATIC_SCRATCH_BYTES;
    return launch_attn(l, static_cast<hipStream_t>(stream));
}

specattn_status specattn_init(void)
{
    clear_error();
    void *ws = nullptr;
    const specattn_status st = static_scratch(&ws);
    if (st != SPECATTN_OK) return st;
    const specattn_status sg = attn_generic_configure();
    if (sg != SPECATTN_OK) return sg;
    const specattn_status sm = layer_map_configure();
    if (sm != SPECATTN_OK) return sm;
    const specattn_status sx = mx_attn_configure();
    if (sx != SPECATTN_OK) return sx;
    return attn_mfma_configure();
}

const char *specattn_last_error(void) { return g_error; }

int specattn_version(void) { return 1010; }

}  // extern "C"
