// Causal attention over packed prompts of different lengths (Eq. 1; the prefill whose keys and values the selection later chooses from), alone or
// behind a prefix that the cache holds.
//
// A unit is 256 query rows (128 or 64 in small calls) - tokens times query heads - of one kv head of a sequence: row i of a sequence stands for
// token i / G and head i % G, so that the heads that share keys and values meet them together, and a unit's rows end within 256 / G positions
// of each other.  Units of a kv head follow each other in steps of H_kv workgroups, which keeps a head's keys and values on few XCDs, and
// units that see the most come first.  Where there are too few units for the GPU, each one's tiles are cut into parts, and
// prompt_merge_kernel joins their partial results in order.
//
// Bound by the tile loop's products and exponentials (attn_rows.h), in short prompts by the setup and the write-out of a unit beside few tiles: 32768 tokens
// 7.9 to 8.6 ms (1.03 to 1.11 PFLOP/s, from card to card), 4 pieces of 512 tokens behind 16384 cached positions, 64 heads over 8 in fp16 676 to 728 us (0.97 to 1.04), 24 prompts of 32 to 2048 tokens
// 165 to 172 us (0.67), 37 tokens by 8 heads at d = 64 5.1 to 5.4 us (a launch).  Single tokens, 32 heads over 8 and 8192 positions in pages: 64 sequences 375 us, 16 (a workgroup to each kv head, half
// of the CUs without any) 160.
#include "attn_rows.h"
#include "checks.h"

#include <algorithm>
#include <cmath>
#include <mutex>

namespace specattn {
namespace {

struct PromptArgs {
    const uint16_t *q;
    const char *k, *v;
    const int32_t *q_starts, *kv_starts, *page_table, *seq_lens;
    float *out, *lse;
    void *out_lowp;
    float *slots, *slots_ml;                                  // partial results, as in the tree kernel; slot = unit * parts + part
    int64_t q_t, q_h;                                         // elements
    int64_t kv_n, kv_h;                                       // bytes
    uint32_t step_n, step_page;                               // between rows and pages, in units of 16 bytes
    FastDivisor per_g;
    int B, H_q, H_kv, G, total_q, total_kv, pages, page_shift, max_pages, parts;
    float sm_scale;
};

// Where a sequence's rows lie.
struct Sequence {
    int q0, q_len, kv0, kv_len;
};
__device__ __forceinline__ Sequence sequence(const PromptArgs &a, int b)
{
    Sequence s;
    s.q0 = min(max(a.q_starts[b], 0), a.total_q);
    s.q_len = max(min(a.q_starts[b + 1], a.total_q) - s.q0, 0);
    if (a.pages) {
        s.kv0 = 0;
        s.kv_len = (int)min((int64_t)max(a.seq_lens[b], 0), (int64_t)a.max_pages << a.page_shift);
    } else {
        s.kv0 = min(max(a.kv_starts[b], 0), a.total_kv);
        s.kv_len = max(min(a.kv_starts[b + 1], a.total_kv) - s.kv0, 0);
    }
    return s;
}

// Unit `index` of a kv head: its sequence, and its number within it; false behind the last unit.  Of up to 64 sequences, units that see the most come
// first, whatever sequence they belong to, so that what is left at the end is short: unit (b, i) is of rank i + (what its sequence has in
// the cache ahead of its queries, in units), ranks are taken from the highest down and within a rank sequences in order.  More sequences follow
// each other, the last unit of each first.
template <int QROWS, int THREADS> __device__ __forceinline__ bool find_unit(const PromptArgs &a, int index, int &b, int &tile, Sequence &s, int *lds)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int W = THREADS / 64;
    int *found = lds + W;                                     // [6]
    if (a.B == 1) {
        s = sequence(a, 0);
        const int n = (int)(((int64_t)s.q_len * a.G + QROWS - 1) / QROWS);
        b = 0;
        tile = n - 1 - index;
        return tile >= 0;
    }
    if (a.B <= 64) {                                          // every wave for itself, a lane to a sequence
        Sequence mine{};
        int n = 0, r = 0;
        if (lane < a.B) {
            mine = sequence(a, lane);
            n = (int)(((int64_t)mine.q_len * a.G + QROWS - 1) / QROWS);
            r = (int)min((int64_t)max(mine.kv_len - mine.q_len, 0) * a.G / QROWS, (int64_t)1 << 28);
        }
        auto units_from = [&](int rank) { return __builtin_amdgcn_readlane(wave_inclusive_sum(min(max(n + r - rank, 0), n)), 63); };
        if (index >= units_from(0)) return false;
        int lo = 0;
        for (int hi = wave_largest(n ? r + n : 0); hi - lo > 1;) {
            const int mid = lo + (hi - lo) / 2;
            if (units_from(mid) > index) lo = mid; else hi = mid;
        }
        const int nth = index - units_from(lo + 1);
        const uint64_t there = __ballot(r <= lo && lo < r + n);
        const uint64_t it = __ballot(((there >> lane) & 1) && __popcll(there & ((1ull << lane) - 1)) == nth);
        b = __builtin_ctzll(it);
        tile = lo - __builtin_amdgcn_readlane(r, b);
        s.q0 = __builtin_amdgcn_readlane(mine.q0, b); s.q_len = __builtin_amdgcn_readlane(mine.q_len, b);
        s.kv0 = __builtin_amdgcn_readlane(mine.kv0, b); s.kv_len = __builtin_amdgcn_readlane(mine.kv_len, b);
        return true;
    }
    if (tid == 0) found[0] = -1;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        Sequence mine{};
        int n = 0;
        if (b0 + tid < a.B) {
            mine = sequence(a, b0 + tid);
            n = (int)(((int64_t)mine.q_len * a.G + QROWS - 1) / QROWS);
        }
        const int up = wave_inclusive_sum(n);
        __syncthreads();
        if (lane == 63) lds[wave] = up;
        __syncthreads();
        int all = 0, ahead = before + up - n;
        for (int w = 0; w < W; ++w) {
            if (w < wave) ahead += lds[w];
            all += lds[w];
        }
        if (index >= ahead && index < ahead + n) {
            found[0] = b0 + tid;
            found[1] = n - 1 - (index - ahead);
            found[2] = mine.q0; found[3] = mine.q_len; found[4] = mine.kv0; found[5] = mine.kv_len;
        }
        before += all;
        if (index < before) break;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(found[0]);
    tile = __builtin_amdgcn_readfirstlane(found[1]);
    s.q0 = __builtin_amdgcn_readfirstlane(found[2]); s.q_len = __builtin_amdgcn_readfirstlane(found[3]);
    s.kv0 = __builtin_amdgcn_readfirstlane(found[4]); s.kv_len = __builtin_amdgcn_readfirstlane(found[5]);
    return b >= 0;
}

__device__ __forceinline__ CacheRows cache_rows(const PromptArgs &a, const Sequence &s, int b, int h)
{
    CacheRows src{};
    const int64_t from = h * a.kv_h + (a.pages ? 0 : (int64_t)s.kv0 * a.kv_n);
    src.k = a.k + from;
    src.v = a.v + from;
    src.step_n = a.step_n; src.step_page = a.step_page;
    src.table = a.pages ? a.page_table + (int64_t)b * a.max_pages : nullptr;
    src.page_shift = a.page_shift; src.pages = a.pages;
    src.slots = max(s.kv_len, 1);
    src.count = s.kv_len;
    return src;
}

// A finished row: query row qr of a sequence's kv head h, elements 8 e .. 8 e + 7.  (A row that sees nothing is zeros, whatever it holds: an infinity or NaN
// that rows beside it see has come into it as 0 * infinity.)
template <int D, bool F16> __device__ __forceinline__ void finish_row(const PromptArgs &a, const Joined &j, int q0, int h, int qr, int e)
{
    const bool none = j.sum == 0.0f;
    const int t = a.per_g.divide(qr);
    const int64_t to = (int64_t)(q0 + t) * a.H_q + h * a.G + qr - t * a.G;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = none ? 0.0f : j.o[i];
    store_row<F16>(a.out, a.out_lowp, to * D + 8 * e, o, none ? 0.0f : 1.0f / j.sum);
    if (a.lse && e == 0) a.lse[to] = none ? -INFINITY : log_sum<F16>(j.ref, j.sum);
}

template <int D, bool F16, int NW, int WQ, int PARTS, bool PAGED>
__global__ __launch_bounds__(NW * 64, WQ == 2 ? 1 : 2) void prompt_kernel(PromptArgs a)
{
    typedef Geo<D, NW, WQ, WQ == 4 ? 64 : 128> G;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ int lds[NW + 6];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int index = blockIdx.x / a.H_kv, h = blockIdx.x - index * a.H_kv;
    int b, tile;
    Sequence s;
    if (!find_unit<G::QROWS, G::THREADS>(a, index, b, tile, s, lds)) return;
    const int queries = s.q_len * a.G;                        // below 2^31: so are total_q * H_q
    const int ahead = s.kv_len - s.q_len;                     // token t sees positions up to t + ahead
    const int unit_q0 = tile * G::QROWS;
    const int last_token = a.per_g.divide(min(unit_q0 + G::QROWS, queries) - 1);
    const int n = (min(max(last_token + ahead + 1, 0), s.kv_len) + G::TILE - 1) / G::TILE;
    const int part = blockIdx.y;
    const int first = (int)((int64_t)n * part / a.parts), last = (int)((int64_t)n * (part + 1) / a.parts);

    const int wq = wave % WQ, wk = wave / WQ;
    RowsOfWave<G, F16, PARTS> rows;
    rows.start(wk, a.sm_scale);
    const int q0 = unit_q0 + wq * 32;
    auto token = [q0, queries](const PromptArgs &a, int i) { return a.per_g.divide(min(q0 + i, queries - 1)); };
    auto query = [q0, queries, s, h](const PromptArgs &a, int i) -> const uint16_t * {
        const int c = min(q0 + i, queries - 1), t = a.per_g.divide(c);
        return a.q + (int64_t)(s.q0 + t) * a.q_t + (h * a.G + c - t * a.G) * a.q_h;
    };
    const uint16_t *mine = query(a, lane & 31);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) rows.q[c] = *reinterpret_cast<const typename Half<F16>::x8 *>(mine + (2 * c + (lane >> 5)) * 8);
    // positions that this lane's row sees, and the fewest and most that a row of the wave does
    const int sees = max(token(a, lane & 31) + ahead + 1, 0);
    const bool live = q0 < queries;
    const int fewest = __builtin_amdgcn_readfirstlane(max(token(a, 0) + ahead + 1, 0)), most = __builtin_amdgcn_readfirstlane(max(token(a, 31) + ahead + 1, 0));
    const int own = live ? min(last, (max(most - wk * G::SPAN, 0) + G::TILE - 1) / G::TILE) : first;
    run_tiles<G, F16, PARTS, PAGED>(rows, [&]() { return cache_rows(arguments_again<PromptArgs>(), s, b, h); }, first, last, n, own, smem, [&](int t, uint64_t &word) {
        const int at = t * G::TILE + wk * G::SPAN;
        word = low_bits(sees - at);
        return at + G::SPAN <= fewest;
    });
    const uint64_t bad = __ballot(live && rows.spoiled());
    rows.leave(smem);
    const PromptArgs &o = arguments_again<PromptArgs>();
    if (bad) {
        const CacheRows old = cache_rows(o, s, b, h);
        mend_rows(bad, rows, old, first, last, n, wk, smem, [&](int t, int i) {
            return low_bits(max(token(o, i) + ahead + 1, 0) - t * G::TILE - wk * G::SPAN);
        });
    }
    const int64_t slot = (int64_t)blockIdx.x * o.parts + part;
    emit_rows<G>(smem, [&](int c, const Joined &j, int e) {
        const int qr = unit_q0 + c;
        if (qr >= queries) return;
        if (o.parts == 1) finish_row<D, F16>(o, j, s.q0, h, qr, e);
        else leave_slot<D>(o.slots, o.slots_ml, slot, G::QROWS, c, e, j);
    });
}

// The parts of a unit joined, in order.
template <int D, bool F16, int QROWS> __global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a)
{
    __shared__ int lds[4 + 6];
    const int index = blockIdx.x / a.H_kv, h = blockIdx.x - index * a.H_kv;
    int b, tile;
    Sequence s;
    if (!find_unit<QROWS, 256>(a, index, b, tile, s, lds)) return;
    const int lane = threadIdx.x & 63, queries = s.q_len * a.G;
    const int64_t slot = (int64_t)blockIdx.x * a.parts;
    const Slots<D> slots = {a.slots, a.slots_ml, slot, slot, 1, a.parts, QROWS};
    slots.template join<1>(blockIdx.y * 4 + (threadIdx.x >> 6), min(QROWS, queries - tile * QROWS), [&](int c, const Joined &j) {
        if (lane < D / 8) finish_row<D, F16>(a, j, s.q0, h, tile * QROWS + c, lane);
    });
}

typedef void (*PromptKernel)(PromptArgs);
// Workgroups by query rows: 64 of them to four waves, two of which share them; 128 to four waves, two workgroups to a CU; 256 to eight.
template <int D, bool F16, int PARTS> PromptKernel by_rows(int qrows, bool paged)
{
    if (paged) return qrows == 64 ? prompt_kernel<D, F16, 4, 2, PARTS, true> : qrows == 128 ? prompt_kernel<D, F16, 4, 4, PARTS, true> : prompt_kernel<D, F16, 8, 8, PARTS, true>;
    return qrows == 64 ? prompt_kernel<D, F16, 4, 2, PARTS, false> : qrows == 128 ? prompt_kernel<D, F16, 4, 4, PARTS, false> : prompt_kernel<D, F16, 8, 8, PARTS, false>;
}
template <int D, bool F16> PromptKernel by_parts(int parts, int qrows, bool paged) { return parts == 1 ? by_rows<D, F16, 1>(qrows, paged) : by_rows<D, F16, 2>(qrows, paged); }
PromptKernel variant(int d, bool f16, int parts, int qrows, bool paged)
{
    return d == 128 ? (f16 ? by_parts<128, true>(parts, qrows, paged) : by_parts<128, false>(parts, qrows, paged))
                    : (f16 ? by_parts<64, true>(parts, qrows, paged) : by_parts<64, false>(parts, qrows, paged));
}
template <int D, bool F16> PromptKernel merge_by_rows(int qrows) { return qrows == 64 ? prompt_merge_kernel<D, F16, 64> : qrows == 128 ? prompt_merge_kernel<D, F16, 128> : prompt_merge_kernel<D, F16, 256>; }
PromptKernel merge_variant(int d, bool f16, int qrows)
{
    return d == 128 ? (f16 ? merge_by_rows<128, true>(qrows) : merge_by_rows<128, false>(qrows)) : (f16 ? merge_by_rows<64, true>(qrows) : merge_by_rows<64, false>(qrows));
}
template <int D> size_t lds_of(int qrows) { return qrows == 64 ? Geo<D, 4, 2, 128>::LDS_BYTES : qrows == 128 ? Geo<D, 4, 4, 64>::LDS_BYTES : Geo<D, 8, 8, 128>::LDS_BYTES; }
size_t lds_size(int d, int qrows) { return d == 128 ? lds_of<128>(qrows) : lds_of<64>(qrows); }
size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call is cut: query rows of a unit, workgroups per kv head at most (no length is known on the host), parts of a unit.
struct Cut { int qrows, units, parts; };
Cut cut(const specattn_prompt_args *p)
{
    Cut c;
    const int64_t queries = (int64_t)p->total_q * (p->H_q / p->H_kv);
    // Few positions to a sequence: two workgroups of 128 rows to a CU, so that one computes while the other sets up or writes out; many: 256 rows that
    // share what is fetched.  us with 128 / 256 rows, 32 heads over 8: 512 tokens 17.7 / 21.5, 1024 29 / 36, 2048 60 / 65, 4096 154 / 148, 8192 568 / 565,
    // 32768 8550 / 8150; 24 sequences of 32 to 2048 189 / 202; 4 x 512 behind 4096 to 16384 (64 heads) 861 / 823.  (In pages the table says how many there can be.)
    const int64_t reach = p->page_table ? (int64_t)p->max_pages_per_seq * p->page_size : p->total_kv;
    c.qrows = queries <= (int64_t)64 * p->B ? 64 : (p->page_table ? reach : reach / p->B) < 3000 ? 128 : 256;
    c.units = (int)(queries / c.qrows + p->B);
    const int64_t all = (int64_t)c.units * p->H_kv, wanted = cu_count() * (c.qrows == 128 ? 2 : 1);
    c.parts = (int)std::min<int64_t>(std::max<int64_t>(wanted / all, 1), std::max<int64_t>(reach / 512, 1));
    return c;
}

}  // namespace

size_t prompt_workspace_bytes(const specattn_prompt_args *p)
{
    const Cut c = cut(p);
    if (c.parts == 1) return 0;
    const size_t rows = (size_t)c.units * p->H_kv * c.parts * c.qrows;
    return a256(rows * p->d * sizeof(float)) + a256(rows * 2 * sizeof(float));
}

specattn_status prompt_configure()
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
    for (int k = 0; k < 48; ++k) {
        const int d = k & 1 ? 128 : 64, qrows = 64 << (k >> 4);
        const size_t bytes = lds_size(d, qrows);
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(variant(d, k & 2, k & 4 ? 2 : 1, qrows, k & 8)), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) {
            (void)hipGetLastError();
            set_error("cannot reserve %zu bytes of LDS", bytes);
            return SPECATTN_EHIP;
        }
    }
    done[dev] = true;
    return SPECATTN_OK;
}

specattn_status launch_prompt(const specattn_prompt_args *p, hipStream_t stream)
{
    specattn_status st = prompt_configure();
    if (st != SPECATTN_OK) return st;
    PromptArgs a{};
    a.q = static_cast<const uint16_t *>(p->q);
    a.k = static_cast<const char *>(p->k); a.v = static_cast<const char *>(p->v);
    a.q_starts = p->q_starts; a.kv_starts = p->kv_starts ? p->kv_starts : p->q_starts;
    a.page_table = p->page_table; a.seq_lens = p->seq_lens;
    a.out = p->out; a.lse = p->lse; a.out_lowp = p->out_lowp;
    a.q_t = p->q_stride_t; a.q_h = p->q_stride_h;
    a.kv_n = p->kv_stride_n * 2; a.kv_h = p->kv_stride_h * 2;
    a.step_n = (uint32_t)(p->kv_stride_n / 8); a.step_page = (uint32_t)(p->kv_stride_page / 8);
    a.B = p->B; a.H_q = p->H_q; a.H_kv = p->H_kv; a.G = p->H_q / p->H_kv;
    a.per_g = FastDivisor(a.G);
    a.total_q = p->total_q; a.total_kv = p->total_kv;
    a.pages = p->page_table ? p->num_pages : 0;
    a.page_shift = p->page_table ? log2i(p->page_size) : 0;
    a.max_pages = p->max_pages_per_seq;
    a.sm_scale = p->sm_scale > 0.0f ? p->sm_scale : 1.0f / std::sqrt((float)p->d);
    const Cut c = cut(p);
    a.parts = c.parts;
    const size_t rows = (size_t)c.units * p->H_kv * c.parts * c.qrows;
    a.slots = static_cast<float *>(p->workspace);
    a.slots_ml = reinterpret_cast<float *>(static_cast<char *>(p->workspace) + a256(rows * p->d * sizeof(float)));
    const bool f16 = p->dtype == SPECATTN_F16;
    variant(p->d, f16, p->out ? 2 : 1, c.qrows, p->page_table)<<<dim3(c.units * p->H_kv, c.parts), c.qrows == 256 ? 512 : 256, lds_size(p->d, c.qrows), stream>>>(a);
    st = check_launch("prompt_kernel");
    if (st != SPECATTN_OK || c.parts == 1) return st;
    merge_variant(p->d, f16, c.qrows)<<<dim3(c.units * p->H_kv, c.qrows / 4), 256, 0, stream>>>(a);
    return check_launch("prompt_merge_kernel");
}

}  // namespace specattn
