// Attention of a tree of drafted tokens (Section 3.1.2, Eq. 2-3, with Algorithm 1's verification over a tree of drafts in place of a chain).
//
// A unit is a kv head of a sequence with up to 128 of its G * T query rows; its tiles are those of the kept positions and one of the tree's
// nodes behind them.  The tiles of all units form one line that is cut into equal shares, one per workgroup, whatever the counts are.  A unit
// that lies in one share is finished there; of the others every share leaves a partial result (reference, sum, unnormalised rows), and
// tree_merge_kernel joins them in the order of the shares, so that repeated calls give the same bits.
#include "attn_rows.h"
#include "checks.h"

#include <algorithm>
#include <cmath>
#include <mutex>

namespace specattn {
namespace {

constexpr int MAX_UNITS = 2048;                               // rows (b, h) per launch: their prefix of tiles lies in LDS
constexpr int MIN_TILES = 2;                                  // of a share: a partial result costs about as much as a tile

struct TreeArgs {
    const uint16_t *q;
    const char *k, *v, *k_new, *v_new;
    const uint64_t *masks;
    const int32_t *node_counts, *seq_lens, *indices, *counts, *page_table;
    float *out, *lse;
    void *out_lowp;
    float *slots;                                             // partial results: [slot][rows][d], then references and sums [slot][2][rows]
    float *slots_ml;
    int2 *parts;                                              // [unit] first and last share of the unit
    int64_t q_b, q_h, q_t;                                    // elements
    int64_t kv_b, kv_h;                                       // bytes
    uint32_t step_n, step_page;                               // between rows and pages of the cache, in units of 16 bytes
    int64_t idx_stride;
    FastDivisor per_h, per_t;
    int H_q, H_kv, T, G, n_max, slots_per_row, pages, page_shift, max_pages, chunk_shift, capacity, physical;
    int row0, rows, blocks;                                   // this launch's rows (b, h), and units per row
    float sm_scale;
};

__device__ __forceinline__ int nodes_of(const TreeArgs &a, int b)
{
    return a.node_counts ? min(max(a.node_counts[b], 0), a.T) : a.T;
}
// Positions that row r of sequence b attends to in the cache.
__device__ __forceinline__ int count_of(const TreeArgs &a, int r, int b)
{
    const bool dense = !a.indices;
    int len = a.n_max;
    if (dense || a.chunk_shift) len = a.seq_lens ? min(max(a.seq_lens[b], 0), a.n_max) : a.n_max;
    if (dense) return len;
    const int c = min(max(a.counts[r], 0), a.capacity);
    if (!a.chunk_shift || c == 0) return c;
    // the list ascends, so the last chunk alone can reach past the length
    const int64_t end = ((int64_t)a.indices[r * a.idx_stride + c - 1] + 1) << a.chunk_shift;
    const int cut = (int)min(max(end - len, (int64_t)0), (int64_t)1 << a.chunk_shift);
    return (c << a.chunk_shift) - cut;
}
__device__ __forceinline__ int tiles_of(int count, int nodes)
{
    return max((count + 63) / 64 + (nodes > 0), 1);           // (a row without any still has to be written)
}

// A row's keys and values.
template <int D> __device__ __forceinline__ CacheRows cache_rows(const TreeArgs &a, int row, int b, int h)
{
    CacheRows src;
    const int64_t head = h * a.kv_h + (a.pages ? 0 : b * a.kv_b);
    src.k = a.k + head;
    src.v = a.v + head;
    src.step_n = a.step_n; src.step_page = a.step_page;
    src.list = a.indices ? a.indices + row * a.idx_stride : nullptr;
    src.table = a.page_table && !a.physical ? a.page_table + (int64_t)b * a.max_pages : nullptr;
    src.chunk_shift = a.chunk_shift; src.page_shift = a.page_shift; src.pages = a.pages;
    src.slots = a.slots_per_row;
    src.k_new = a.k_new + (int64_t)row * a.T * D * 2;
    src.v_new = a.v_new + (int64_t)row * a.T * D * 2;
    return src;
}

// A finished row: query row qr of kv head h, elements 8 e .. 8 e + 7.
template <int D, bool F16> __device__ __forceinline__ void finish_row(const TreeArgs &a, const Joined &j, int b, int h, int qr, int nodes, int e)
{
    const bool none = qr - a.per_t.divide(qr) * a.T >= nodes || j.sum == 0.0f;
    const int64_t to = ((int64_t)b * a.H_q + h * a.G) * a.T + qr;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = none ? 0.0f : j.o[i];
    store_row<F16>(a.out, a.out_lowp, to * D + 8 * e, o, none ? 0.0f : 1.0f / j.sum);
    if (a.lse && e == 0) a.lse[to] = none ? -INFINITY : log_sum<F16>(j.ref, j.sum);
}

// The line of tiles in n shares, the first `more` of them one tile longer than `each`.
struct Shares {
    int n, each, more;
    __device__ __forceinline__ Shares(int total, int most)
    {
        n = min(most, max(total / MIN_TILES, 1));
        each = (int)((uint32_t)total / (uint32_t)n);
        more = total - each * n;
    }
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int of(int tile) const
    {
        const int longer = more * (each + 1);
        return tile < longer ? (int)((uint32_t)tile / (uint32_t)(each + 1)) : more + (int)((uint32_t)(tile - longer) / (uint32_t)max(each, 1));
    }
};

template <int D, bool F16, int NW, int WQ, int PARTS>
__global__ __launch_bounds__(NW * 64, NW / 4) void tree_kernel(TreeArgs a)
{
    typedef Geo<D, NW, WQ, 128> G;
    constexpr int THREADS = G::THREADS;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int *prefix = reinterpret_cast<int *>(smem + G::LDS_BYTES);       // [rows + 1] tiles ahead of a row
    __shared__ int wave_sums[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    {
        const int per = (a.rows + THREADS - 1) / THREADS;
        int mine = 0;
        for (int i = 0; i < per; ++i) {
            const int r = tid * per + i;
            if (r >= a.rows) break;
            const int b = a.per_h.divide(a.row0 + r);
            const int n = tiles_of(count_of(a, a.row0 + r, b), nodes_of(a, b)) * a.blocks;
            prefix[r + 1] = n;
            mine += n;
        }
        const int up = wave_inclusive_sum(mine);
        if (lane == 63) wave_sums[wave] = up;
        __syncthreads();
        int before = up - mine;
        for (int w = 0; w < wave; ++w) before += wave_sums[w];
        for (int i = 0; i < per; ++i) {
            const int r = tid * per + i;
            if (r >= a.rows) break;
            before += prefix[r + 1];
            prefix[r + 1] = before;
        }
        if (tid == 0) prefix[0] = 0;
        __syncthreads();
    }
    auto tiles_before = [&](int row) { return __builtin_amdgcn_readfirstlane(prefix[row]); };
    const Shares shares(tiles_before(a.rows), gridDim.x);
    const int share = blockIdx.x;
    if (share >= shares.n) return;
    int at = shares.begin(share);
    const int end = shares.begin(share + 1);
    int r = 0;                                                // the row that the share begins in
    for (int lo = 0, hi = a.rows; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (tiles_before(mid) <= at) lo = mid; else hi = mid;
        r = lo;
    }
    const int wq = wave % WQ, wk = wave / WQ;
    const int queries = a.G * a.T;
    while (at < end) {
        const TreeArgs &a = arguments_again<TreeArgs>();
        while (tiles_before(r + 1) <= at) ++r;
        const int row_at = tiles_before(r), n = (int)((uint32_t)(tiles_before(r + 1) - row_at) / (uint32_t)a.blocks);   // tiles of each of the row's units
        const int block = (int)((uint32_t)(at - row_at) / (uint32_t)n);
        const int unit_at = row_at + block * n;
        const int first = at - unit_at, last = min(n, end - unit_at);
        const int unit = r * a.blocks + block;
        const int row = a.row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
        const int count = count_of(a, row, b), nodes = nodes_of(a, b);
        const int cached = (count + G::TILE - 1) / G::TILE;

        RowsOfWave<G, F16, PARTS> rows;
        rows.start(wk, a.sm_scale);
        const int q0 = block * G::QROWS + wq * 32;
        auto query = [q0, queries, b, h](const TreeArgs &a, int i) -> const uint16_t * {
            const int c = min(q0 + i, queries - 1), g = a.per_t.divide(c);
            return a.q + b * a.q_b + (h * a.G + g) * a.q_h + (c - g * a.T) * a.q_t;
        };
        auto node_seen = [q0, queries, b](const TreeArgs &a, int nodes, int i) -> uint64_t {      // nodes that query row i of this wave attends to
            const int c = min(q0 + i, queries - 1), t = c - a.per_t.divide(c) * a.T;
            return t < nodes ? a.masks[(int64_t)b * a.T + t] & low_bits(nodes) : 0;
        };
        const uint16_t *mine = query(a, lane & 31);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) rows.q[c] = *reinterpret_cast<const typename Half<F16>::x8 *>(mine + (2 * c + (lane >> 5)) * 8);
        const bool live = q0 < queries;                       // (a wave without query rows only fetches)
        const uint64_t my_nodes = last > cached ? node_seen(a, nodes, lane & 31) >> (wk * G::SPAN) : 0;
        // (a row without anything has a tile in the line all the same, which holds nothing to read)
        const int stop = nodes > 0 ? last : min(last, cached);
        auto where = [&]() {
            CacheRows src = cache_rows<D>(arguments_again<TreeArgs>(), row, b, h);
            src.count = count;
            src.nodes = nodes;
            return src;
        };
        run_tiles<G, F16, PARTS, true>(rows, where, first, stop, cached, live ? stop : first, smem, [&](int t, uint64_t &word) {
            const int in = count - t * G::TILE - wk * G::SPAN;
            word = t < cached ? low_bits(in) : my_nodes;
            return t < cached && in >= G::SPAN;
        });
        const uint64_t bad = __ballot(live && rows.spoiled());
        rows.leave(smem);
        const TreeArgs &o = arguments_again<TreeArgs>();
        if (bad) {
            const CacheRows old = where();
            mend_rows<G, F16>(bad, o.sm_scale * LOG2E, old, first, last, cached, wk, smem, [&](int i) { return query(o, i); }, [&](int t, int i) {
                return t >= cached ? node_seen(o, old.nodes, i) >> (wk * G::SPAN) : low_bits(old.count - t * G::TILE - wk * G::SPAN);
            });
        }
        const bool whole = first == 0 && last == n;
        const int64_t slot = share + unit;
        if (first == 0 && tid == 0) o.parts[unit] = make_int2(share, shares.of(unit_at + n - 1));
        emit_rows<G>(smem, [&](int c, const Joined &j, int e) {
            const int qr = block * G::QROWS + c;
            if (qr >= queries) return;
            if (whole) finish_row<D, F16>(o, j, b, h, qr, nodes, e);
            else leave_slot<D>(o.slots, o.slots_ml, slot, G::QROWS, c, e, j);
        });
        __syncthreads();                                      // the tile buffers are free again
        at = unit_at + last;
    }
}

// Units that several shares worked on: their partial results joined, in the order of the shares; a wave for each query row.
template <int D, bool F16> __global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int qrows)
{
    const int unit = blockIdx.x;
    const int2 parts = a.parts[unit];
    if (parts.x == parts.y) return;
    const int r = unit / a.blocks, block = unit - r * a.blocks;
    const int row = a.row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
    const int c = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int qr = block * qrows + c;
    if (c >= qrows || qr >= a.G * a.T) return;
    const Joined j = joined_slots<D>(a.slots, a.slots_ml, parts.x + unit, parts.y - parts.x + 1, qrows, c);
    if (lane < D / 8) finish_row<D, F16>(a, j, b, h, qr, nodes_of(a, b), lane);
}

// Workgroups by query rows: 64 of them to four waves, 128 to eight (two share rows), 256 to eight.
int rows_per_unit(int queries) { return queries <= 64 ? 64 : queries <= 128 ? 128 : 256; }

typedef void (*TreeKernel)(TreeArgs);
template <int D, bool F16, int PARTS> TreeKernel by_rows(int qrows)
{
    return qrows == 64 ? tree_kernel<D, F16, 4, 2, PARTS> : qrows == 128 ? tree_kernel<D, F16, 8, 4, PARTS> : tree_kernel<D, F16, 8, 8, PARTS>;
}
template <int D, bool F16> TreeKernel by_parts(int parts, int qrows) { return parts == 1 ? by_rows<D, F16, 1>(qrows) : by_rows<D, F16, 2>(qrows); }
TreeKernel variant(int d, bool f16, int parts, int qrows)
{
    return d == 128 ? (f16 ? by_parts<128, true>(parts, qrows) : by_parts<128, false>(parts, qrows))
                    : (f16 ? by_parts<64, true>(parts, qrows) : by_parts<64, false>(parts, qrows));
}
size_t lds_size(int d, int qrows, int rows)
{
    const size_t tiles = d == 128 ? (qrows == 64 ? Geo<128, 4, 2, 128>::LDS_BYTES : Geo<128, 8, 4, 128>::LDS_BYTES) : (qrows == 64 ? Geo<64, 4, 2, 128>::LDS_BYTES : Geo<64, 8, 4, 128>::LDS_BYTES);
    return tiles + (size_t)(rows + 1) * 4;
}
size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

struct Layout { size_t parts, rows, ml; };
Layout layout(int d, int qrows, int units)
{
    const size_t slots = (size_t)cu_count() + units;
    return {a256((size_t)units * sizeof(int2)), slots * qrows * d * sizeof(float), a256(slots * 2 * qrows * sizeof(float))};
}

}  // namespace

size_t tree_workspace_bytes(const specattn_tree_args *t)
{
    const int queries = t->H_q / t->H_kv * t->T, qrows = rows_per_unit(queries), blocks = (queries + qrows - 1) / qrows;
    const Layout l = layout(t->d, qrows, (int)std::min<int64_t>((int64_t)t->B * t->H_kv, MAX_UNITS) * blocks);
    return l.parts + l.rows + l.ml;
}

specattn_status tree_configure()
{
    constexpr int MAX_DEVICES = 64;
    static std::mutex mu;
    static bool done[MAX_DEVICES] = {false};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) {
        (void)hipGetLastError();
        set_error("no current device");
        return SPECATTN_EHIP;
    }
    std::lock_guard<std::mutex> lock(mu);
    if (done[dev]) return SPECATTN_OK;
    for (int k = 0; k < 24; ++k) {
        const int d = k & 1 ? 128 : 64, qrows = 64 << (k >> 3);
        const size_t bytes = lds_size(d, qrows, MAX_UNITS);
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(variant(d, k & 2, k & 4 ? 2 : 1, qrows)), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) {
            (void)hipGetLastError();
            set_error("cannot reserve %zu bytes of LDS", bytes);
            return SPECATTN_EHIP;
        }
    }
    done[dev] = true;
    return SPECATTN_OK;
}

specattn_status launch_tree(const specattn_tree_args *t, hipStream_t stream)
{
    specattn_status st = tree_configure();
    if (st != SPECATTN_OK) return st;
    TreeArgs a{};
    a.q = static_cast<const uint16_t *>(t->q);
    a.k = static_cast<const char *>(t->k); a.v = static_cast<const char *>(t->v);
    a.k_new = static_cast<const char *>(t->k_new); a.v_new = static_cast<const char *>(t->v_new);
    a.masks = t->tree_masks; a.node_counts = t->node_counts; a.seq_lens = t->seq_lens;
    a.indices = t->indices; a.counts = t->counts; a.page_table = t->page_table;
    a.out = t->out; a.lse = t->lse; a.out_lowp = t->out_lowp;
    a.q_b = t->q_stride_b; a.q_h = t->q_stride_h; a.q_t = t->q_stride_t;
    a.kv_b = t->kv_stride_b * 2; a.kv_h = t->kv_stride_h * 2;
    a.step_n = (uint32_t)(t->kv_stride_n / 8); a.step_page = (uint32_t)(t->kv_stride_page / 8);
    a.idx_stride = t->idx_stride_row;
    a.per_h = FastDivisor(t->H_kv); a.per_t = FastDivisor(t->T);
    a.H_q = t->H_q; a.H_kv = t->H_kv; a.T = t->T; a.G = t->H_q / t->H_kv; a.n_max = t->n_max;
    const bool paged = t->page_table || t->indices_are_physical;
    a.physical = t->indices_are_physical;
    a.pages = paged ? t->num_pages : 0;
    a.page_shift = paged ? log2i(t->page_size) : 0;
    a.max_pages = t->max_pages_per_seq;
    a.slots_per_row = a.physical ? (int)std::min<int64_t>((int64_t)t->num_pages * t->page_size, INT32_MAX) : t->n_max;
    a.chunk_shift = t->chunk_size > 1 ? log2i(t->chunk_size) : 0;
    a.capacity = t->idx_capacity;
    a.sm_scale = t->sm_scale > 0.0f ? t->sm_scale : 1.0f / std::sqrt((float)t->d);
    const int queries = a.G * a.T, qrows = rows_per_unit(queries), rows = t->B * t->H_kv;
    a.blocks = (queries + qrows - 1) / qrows;
    const bool f16 = t->dtype == SPECATTN_F16;
    const Layout l = layout(t->d, qrows, std::min(rows, MAX_UNITS) * a.blocks);
    char *ws = static_cast<char *>(t->workspace);
    a.parts = reinterpret_cast<int2 *>(ws);
    a.slots = reinterpret_cast<float *>(ws + l.parts);
    a.slots_ml = reinterpret_cast<float *>(ws + l.parts + l.rows);
    const int64_t most = t->indices ? (int64_t)t->idx_capacity << a.chunk_shift : t->n_max;
    for (a.row0 = 0; a.row0 < rows; a.row0 += a.rows) {
        a.rows = (int)std::min<int64_t>({rows - a.row0, MAX_UNITS, (int64_t)(1 << 30) / (a.blocks * (most / 64 + 2))});     // tiles are counted in 31 bits
        variant(t->d, f16, t->out ? 2 : 1, qrows)<<<cu_count(), qrows == 64 ? 256 : 512, lds_size(t->d, qrows, a.rows), stream>>>(a);
        st = check_launch("tree_kernel");
        if (st != SPECATTN_OK) return st;
        const auto merge = t->d == 128 ? (f16 ? tree_merge_kernel<128, true> : tree_merge_kernel<128, false>) : (f16 ? tree_merge_kernel<64, true> : tree_merge_kernel<64, false>);
        merge<<<dim3(a.rows * a.blocks, (std::min(queries, qrows) + 3) / 4), 256, 0, stream>>>(a, qrows);
        st = check_launch("tree_merge_kernel");
        if (st != SPECATTN_OK) return st;
    }
    return SPECATTN_OK;
}

}  // namespace specattn
