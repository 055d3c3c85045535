// Attention of a tree of drafted tokens (Section 3.1.2, Eq. 2-3, with Algorithm 1's verification over a tree of drafts in place of a chain).
//
// A unit is a kv head of a sequence with up to 256 of its G * T query rows; its tiles are those of the kept positions and one of the tree's
// nodes behind them.  The tiles of all units form one line that is cut into equal shares, one per workgroup, whatever the counts are.  A unit
// that lies in one share is finished there; of the others every share leaves a partial result (reference, sum, unnormalised rows; two at most to a share), and
// tree_merge_kernel joins them in the order of the shares, so that repeated calls give the same bits.
//
// Few rows: bound by memory and by what a share spends ahead of and behind its tiles (finding its rows, the first fetches, partial results: 10 to 15 us, the joining 5 to
// 9): 8 trees of 16 nodes, 32 heads over 8, a quarter of 32768 positions 70 to 72 us, 252 MB (3.5 TB/s); one tree of 26 over a third of 8192 24 to 25 us.  Many rows: by the tile
// loop's products: 16 trees of 64 nodes, 64 heads over 8 in fp16, 40 % of 256 to 16384 positions in pages 113 to 124 us (0.47 to 0.52 PFLOP/s), 14 to 17 of them the joining.
#include "attn_rows.h"
#include "checks.h"

#include <algorithm>
#include <cmath>
#include <mutex>

namespace specattn {
namespace {

constexpr int MAX_UNITS = 2048;                               // rows (b, h) per launch: their prefix of tiles lies in LDS
constexpr int MIN_TILES = 4;                                  // of a share
constexpr int FEW = 64;                                       // rows that a wave scans by itself
constexpr int WHOLE_TILES = 8;                                // units of up to so many are not cut: joining them takes a second launch
// Tiles that a unit costs beside its own: 10 us or so for finding its rows, first fetches and putting its result down.  (us with 4 / 8 / 10 / 14: 16
// trees of 64 nodes over 256 to 16384 positions 131 / 131 / 122 / 134, 64 of 8 over 64 to 4096 72 / 66 / 65 / 65, 8 of 64 over 8192 65 / 64 / 59 / 60.)
constexpr int SETUP = 10;

struct TreeArgs {
    const uint16_t *q;
    const char *k, *v, *k_new, *v_new;
    const uint64_t *masks;
    const int32_t *node_counts, *seq_lens, *indices, *counts, *page_table;
    float *out, *lse;
    void *out_lowp;
    float *slots;                                             // partial results: [slot][rows][d], then references and sums [slot][2][rows]; two slots to a share
    float *slots_ml;
    int2 *parts;                                              // [unit] first and last share of the unit
    int64_t q_b, q_h, q_t;                                    // elements
    int64_t kv_b, kv_h;                                       // bytes
    uint32_t step_n, step_page;                               // between rows and pages of the cache, in units of 16 bytes
    int64_t idx_stride;
    FastDivisor per_h, per_t;
    int H_q, H_kv, T, G, n_max, slots_per_row, pages, page_shift, max_pages, chunk_shift, capacity, physical;
    int row0, rows, blocks;                                   // this launch's rows (b, h), and units per row
    int whole;                                                // 1: a workgroup to a unit
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

// The line of all units' tiles, cut into n shares.  Picking a unit up and putting its result down costs a share about as much as a few tiles: a
// unit takes `setup` places ahead of its tiles, and a cut that would fall there, or close to a unit's ends, is made between the units
// instead, so that no partial results are left for little.  Where there are no more units than workgroups, and the largest is not much longer than a
// share would be, every unit is a share.
struct Line {
    const int *prefix;                                        // [rows + 1] tiles of the units of the rows ahead of a row (LDS), or null:
    int ahead;                                                // of up to FEW rows, those ahead of row `lane`
    int rows, blocks, tiles, n, setup, each, more, slack;
    bool direct;
    __device__ __forceinline__ Line(const int *prefix_, int ahead_, int tiles_, int largest, int rows_, int blocks_, int most)
        : prefix(prefix_), ahead(ahead_), rows(rows_), blocks(blocks_), tiles(tiles_)
    {
        n = min(most, max(tiles / MIN_TILES, 1));
        setup = min(SETUP, (int)((uint32_t)tiles / (uint32_t)n) / 2);
        direct = rows * blocks <= most && largest <= (int)((uint32_t)tiles / (uint32_t)n) + SETUP;
        if (direct) n = rows * blocks;
        const int total = tiles + setup * rows * blocks;
        each = (int)((uint32_t)total / (uint32_t)n);
        more = total - each * n;
        slack = each / 8;
    }
    __device__ __forceinline__ int row_at(int r) const
    {
        const int before = r == rows ? tiles : prefix ? __builtin_amdgcn_readfirstlane(prefix[r]) : __builtin_amdgcn_readlane(ahead, r);
        return before + setup * r * blocks;
    }
    __device__ __forceinline__ int row_of(int place) const     // (as all below: by a whole wave)
    {
        const int lane = threadIdx.x & 63;
        if (!prefix) return __popcll(__ballot(lane < rows && ahead + setup * lane * blocks <= place)) - 1;
        // every `step`th row first, then those in between
        const int step = (rows + 63) >> 6;
        const int coarse = min(lane * step, rows - 1);
        const int from = (__popcll(__ballot(lane * step < rows && prefix[coarse] + setup * coarse * blocks <= place)) - 1) * step;
        const int fine = min(from + lane, rows - 1);
        return from + __popcll(__ballot(lane < step && from + lane < rows && prefix[fine] + setup * fine * blocks <= place)) - 1;
    }
    __device__ __forceinline__ int begin(int w) const         // where share w begins
    {
        const int place = w * each + min(w, more);
        if (w == 0 || w == n) return place;
        const int r = row_of(place), at = row_at(r), per = (int)((uint32_t)(row_at(r + 1) - at) / (uint32_t)blocks);
        const int in = (int)((uint32_t)(place - at) % (uint32_t)per);
        return in <= setup + slack ? place - in : per - in <= slack ? place + per - in : place;
    }
    __device__ __forceinline__ int of(int place) const        // the share that a place lies in
    {
        const int longer = more * (each + 1);
        int w = place < longer ? (int)((uint32_t)place / (uint32_t)(each + 1)) : more + (int)((uint32_t)(place - longer) / (uint32_t)max(each, 1));
        while (w > 0 && place < begin(w)) --w;
        while (w + 1 < n && place >= begin(w + 1)) ++w;
        return w;
    }
};

template <int D, bool F16, int NW, int WQ, int PARTS>
__global__ __launch_bounds__(NW * 64, NW / 4) void tree_kernel(TreeArgs a)
{
    typedef Geo<D, NW, WQ, 128> G;
    constexpr int THREADS = G::THREADS;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int *prefix = reinterpret_cast<int *>(smem + G::LDS_BYTES);       // [rows + 1] tiles ahead of a row
    int ahead = 0, tiles = 0, largest = 0, counts = 0;        // (counts: of up to FEW rows, that of row `lane`)
    if (!a.whole && a.rows <= FEW) {                          // every wave for itself, a lane to a row
        int n = 0;
        if (lane < a.rows) {
            const int b = a.per_h.divide(a.row0 + lane);
            counts = count_of(a, a.row0 + lane, b);
            n = tiles_of(counts, nodes_of(a, b)) * a.blocks;
        }
        const int up = wave_inclusive_sum(n);
        ahead = up - n;
        largest = wave_largest(n);
        tiles = __builtin_amdgcn_readlane(up, 63);
        prefix = nullptr;
    } else if (!a.whole) {
        __shared__ int wave_sums[NW], wave_most[NW];
        const int per = (a.rows + THREADS - 1) / THREADS;
        int mine = 0;
        for (int i = 0; i < per; ++i) {
            const int r = tid * per + i;
            if (r >= a.rows) break;
            const int b = a.per_h.divide(a.row0 + r);
            const int n = tiles_of(count_of(a, a.row0 + r, b), nodes_of(a, b)) * a.blocks;
            prefix[r + 1] = n;
            mine += n;
            largest = max(largest, n);
        }
        const int up = wave_inclusive_sum(mine);
        largest = wave_largest(largest);
        if (lane == 63) {
            wave_sums[wave] = up;
            wave_most[wave] = largest;
        }
        __syncthreads();
        for (int w = 0; w < NW; ++w) largest = max(largest, __builtin_amdgcn_readfirstlane(wave_most[w]));
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
        tiles = __builtin_amdgcn_readfirstlane(prefix[a.rows]);
    }
    const Line line(prefix, ahead, tiles, (int)((uint32_t)largest / (uint32_t)a.blocks), a.rows, a.blocks, gridDim.x);
    const bool by_unit = a.whole || line.direct;
    const int share = blockIdx.x;
    int at = 0, end = 1, r = 0;
    if (!a.whole && share >= line.n) return;
    if (!by_unit) {
        at = line.begin(share);
        end = line.begin(share + 1);
        r = line.row_of(at);
    }
    const int wq = wave % WQ, wk = wave / WQ;
    const int queries = a.G * a.T;
    while (at < end) {
        const TreeArgs &a = arguments_again<TreeArgs>();
        int block, unit_at = 0, tiles_at = 0, n = 0, first = 0, last = 0;
        if (by_unit) {
            r = (int)((uint32_t)share / (uint32_t)a.blocks);
            block = share - r * a.blocks;
            at = 1;
        } else {
            while (line.row_at(r + 1) <= at) ++r;
            const int row_at = line.row_at(r), per = (int)((uint32_t)(line.row_at(r + 1) - row_at) / (uint32_t)a.blocks);
            n = per - line.setup;
            block = (int)((uint32_t)(at - row_at) / (uint32_t)per);
            unit_at = row_at + block * per;
            tiles_at = unit_at + line.setup;
            first = max(at - tiles_at, 0);
            last = min(n, end - tiles_at);
            at = unit_at + per;
            if (last <= first) continue;
        }
        const int unit = r * a.blocks + block;
        const int row = a.row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
        const int count = !a.whole && a.rows <= FEW ? __builtin_amdgcn_readlane(counts, r) : count_of(a, row, b), nodes = nodes_of(a, b);
        const int cached = (count + G::TILE - 1) / G::TILE;
        if (by_unit) last = n = tiles_of(count, nodes);

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
            mend_rows(bad, rows, old, first, last, cached, wk, smem, [&](int t, int i) {
                return t >= cached ? node_seen(o, old.nodes, i) >> (wk * G::SPAN) : low_bits(old.count - t * G::TILE - wk * G::SPAN);
            });
        }
        const bool whole = first == 0 && last == n;
        const int64_t slot = 2 * share + (first == 0);       // (a share has two partial results at most: of its first unit's end, and of its last unit's beginning)
        if (first == 0 && wave == 0 && !o.whole) {            // (all of the wave: it looks the share up together)
            const int2 parts = make_int2(share, by_unit ? share : line.of(tiles_at + n - 1));
            if (lane == 0) o.parts[unit] = parts;
        }
        emit_rows<G>(smem, [&](int c, const Joined &j, int e) {
            const int qr = block * G::QROWS + c;
            if (qr >= queries) return;
            if (whole) finish_row<D, F16>(o, j, b, h, qr, nodes, e);
            else leave_slot<D>(o.slots, o.slots_ml, slot, G::QROWS, c, e, j);
        });
        __syncthreads();                                      // the tile buffers are free again
    }
}

// Units that several shares worked on: their partial results joined, in the order of the shares.
template <int D, bool F16, int N> __global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int qrows)
{
    const int unit = blockIdx.x;
    const int2 parts = a.parts[unit];
    if (parts.x == parts.y) return;
    const int r = unit / a.blocks, block = unit - r * a.blocks;
    const int row = a.row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
    const int lane = threadIdx.x & 63, nodes = nodes_of(a, b), queries = a.G * a.T;
    const Slots<D> slots = {a.slots, a.slots_ml, 2 * (int64_t)parts.x + 1, 2 * (int64_t)parts.x, 2, parts.y - parts.x + 1, qrows};
    slots.template join<N>((blockIdx.y * 4 + (threadIdx.x >> 6)) * N, min(qrows, queries - block * qrows), [&](int c, const Joined &j) {
        if (lane < D / 8) finish_row<D, F16>(a, j, b, h, block * qrows + c, nodes, lane);
    });
}

// Query rows of a unit: 64 for four waves or 128 for eight, two of which share rows, or 256 for eight.  (us of calls with 65 to 128 rows to a kv
// head, units of 128 / 256: 8 x 32 nodes over 7500 of 32768 positions 79 / 83, 32 x 26 over 1640 of 4096 59 / 65.)
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
typedef void (*MergeKernel)(TreeArgs, int);
template <int D, bool F16> MergeKernel merge_by_rows(int per) { return per == 1 ? tree_merge_kernel<D, F16, 1> : tree_merge_kernel<D, F16, MERGE_ROWS>; }
MergeKernel merge_variant(int d, bool f16, int per)
{
    return d == 128 ? (f16 ? merge_by_rows<128, true>(per) : merge_by_rows<128, false>(per)) : (f16 ? merge_by_rows<64, true>(per) : merge_by_rows<64, false>(per));
}
template <int D> size_t lds_of(int qrows) { return qrows == 64 ? Geo<D, 4, 2, 128>::LDS_BYTES : Geo<D, 8, 8, 128>::LDS_BYTES; }
size_t lds_size(int d, int qrows, int rows) { return (d == 128 ? lds_of<128>(qrows) : lds_of<64>(qrows)) + (size_t)(rows + 1) * 4; }
size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call is cut: query rows of a unit, units to a row (b, h), rows to a launch, tiles of a unit at most, whether each unit has a workgroup, and workgroups
// of a launch of so many rows.
struct Cut {
    int qrows, blocks, rows;
    int64_t tiles;
    bool whole;
    int grid(int rows) const { return whole ? rows * blocks : (int)std::min<int64_t>(cu_count(), (rows * blocks * tiles + MIN_TILES - 1) / MIN_TILES); }
};
Cut cut(const specattn_tree_args *t)
{
    Cut c;
    const int queries = t->H_q / t->H_kv * t->T;
    c.qrows = rows_per_unit(queries);
    c.blocks = (queries + c.qrows - 1) / c.qrows;
    const int64_t most = t->indices ? (int64_t)t->idx_capacity << (t->chunk_size > 1 ? log2i(t->chunk_size) : 0) : t->n_max;
    c.tiles = (most + 63) / 64 + 1;
    c.rows = (int)std::min<int64_t>({(int64_t)t->B * t->H_kv, MAX_UNITS, (int64_t)(1 << 30) / (c.blocks * (most / 64 + 2))});      // tiles are counted in 31 bits
    c.whole = c.tiles <= WHOLE_TILES;
    return c;
}
struct Layout { size_t parts, rows, ml; };
Layout layout(int d, const Cut &c)
{
    if (c.whole) return {0, 0, 0};                            // (every unit is finished where it is computed)
    const size_t units = (size_t)c.rows * c.blocks, slots = 2 * (size_t)c.grid(c.rows);
    return {a256(units * sizeof(int2)), slots * c.qrows * d * sizeof(float), a256(slots * 2 * c.qrows * sizeof(float))};
}

}  // namespace

size_t tree_workspace_bytes(const specattn_tree_args *t)
{
    const Layout l = layout(t->d, cut(t));
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
    const Cut c = cut(t);
    const int rows = t->B * t->H_kv;
    a.blocks = c.blocks;
    a.whole = c.whole;
    const bool f16 = t->dtype == SPECATTN_F16;
    const Layout l = layout(t->d, c);
    char *ws = static_cast<char *>(t->workspace);
    a.parts = reinterpret_cast<int2 *>(ws);
    a.slots = reinterpret_cast<float *>(ws + l.parts);
    a.slots_ml = reinterpret_cast<float *>(ws + l.parts + l.rows);
    for (a.row0 = 0; a.row0 < rows; a.row0 += a.rows) {
        a.rows = std::min(rows - a.row0, c.rows);
        const int units = a.rows * a.blocks;
        variant(t->d, f16, t->out ? 2 : 1, c.qrows)<<<c.grid(a.rows), c.qrows == 64 ? 256 : 512, lds_size(t->d, c.qrows, a.rows), stream>>>(a);
        st = check_launch("tree_kernel");
        if (st != SPECATTN_OK) return st;
        if (a.whole) continue;
        const int per = units * 4 >= cu_count() ? MERGE_ROWS : 1;
        merge_variant(t->d, f16, per)<<<dim3(units, (std::min(a.G * a.T, c.qrows) + 4 * per - 1) / (4 * per)), 256, 0, stream>>>(a, c.qrows);
        st = check_launch("tree_merge_kernel");
        if (st != SPECATTN_OK) return st;
    }
    return SPECATTN_OK;
}

}  // namespace specattn
