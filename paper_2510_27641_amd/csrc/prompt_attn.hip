// Causal attention over packed prompts of different lengths (Eq. 1; the prefill whose keys and values the selection later chooses from), alone or
// behind a prefix that the cache holds.
//
// A unit is 128 query rows - tokens times query heads - of one kv head of a sequence: row i of a sequence stands for token i / G and head
// i % G, so that the heads that share keys and values meet them together, and a unit's rows end within 128 / G positions of each other.
// Units of a kv head follow each other in steps of H_kv workgroups, which keeps a head's keys and values on few XCDs, and the last tokens
// of a sequence, which see the most, come first.  Where there are too few units for the GPU, each one's tiles are cut into parts, and
// prompt_merge_kernel joins their partial results in order.
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
    int64_t kv_n, kv_h, kv_page;                              // bytes
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

// Unit `index` of a kv head: its sequence, and its number within it (the last one first); false behind the last unit.
template <int QROWS> __device__ __forceinline__ bool find_unit(const PromptArgs &a, int index, int &b, int &tile, int *wave_sums)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ int found[2];
    int before = 0;
    if (tid == 0) found[0] = -1;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        int n = 0;
        if (b0 + tid < a.B) {
            const int q0 = min(max(a.q_starts[b0 + tid], 0), a.total_q);
            n = (int)(((int64_t)max(min(a.q_starts[b0 + tid + 1], a.total_q) - q0, 0) * a.G + QROWS - 1) / QROWS);
        }
        const int up = wave_inclusive_sum(n);
        __syncthreads();
        if (lane == 63) wave_sums[wave] = up;
        __syncthreads();
        int all = 0, ahead = before + up - n;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) ahead += wave_sums[w];
            all += wave_sums[w];
        }
        if (index >= ahead && index < ahead + n) {
            found[0] = b0 + tid;
            found[1] = n - 1 - (index - ahead);
        }
        before += all;
        if (index < before) break;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(found[0]);
    tile = __builtin_amdgcn_readfirstlane(found[1]);
    return b >= 0;
}

template <int D, bool F16, int WQ, int PARTS>
__global__ __launch_bounds__(THREADS, 2) void prompt_kernel(PromptArgs a)
{
    typedef Geo<D, WQ> G;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ int wave_sums[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int index = blockIdx.x / a.H_kv, h = blockIdx.x - index * a.H_kv;
    int b, tile;
    if (!find_unit<G::QROWS>(a, index, b, tile, wave_sums)) return;
    const Sequence s = sequence(a, b);
    const int queries = s.q_len * a.G;                        // below 2^31: so are total_q * H_q
    const int ahead = s.kv_len - s.q_len;                     // token t sees positions up to t + ahead
    const int unit_q0 = tile * G::QROWS;
    const int last_token = a.per_g.divide(min(unit_q0 + G::QROWS, queries) - 1);
    const int n = (min(max(last_token + ahead + 1, 0), s.kv_len) + G::TILE - 1) / G::TILE;
    const int part = blockIdx.y;
    const int first = (int)((int64_t)n * part / a.parts), last = (int)((int64_t)n * (part + 1) / a.parts);

    CacheRows src{};
    const int64_t from = a.pages ? 0 : (int64_t)s.kv0 * a.kv_n;
    src.k = a.k + h * a.kv_h + from;
    src.v = a.v + h * a.kv_h + from;
    src.stride_n = a.kv_n; src.stride_page = a.kv_page;
    src.table = a.pages ? a.page_table + (int64_t)b * a.max_pages : nullptr;
    src.page_shift = a.page_shift; src.pages = a.pages;
    src.slots = max(s.kv_len, 1);
    src.count = s.kv_len;

    const int wq = wave % WQ, wk = wave / WQ;
    RowsOfWave<D, F16, WQ, PARTS> rows;
    rows.start(wk, a.sm_scale);
    const int q0 = unit_q0 + wq * 32;
    auto token = [&](int i) { return a.per_g.divide(min(q0 + i, queries - 1)); };
    auto query = [&](int i) -> const uint16_t * {
        const int c = min(q0 + i, queries - 1), t = a.per_g.divide(c);
        return a.q + (int64_t)(s.q0 + t) * a.q_t + (h * a.G + c - t * a.G) * a.q_h;
    };
    const uint16_t *mine = query(lane & 31);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) rows.q[c] = *reinterpret_cast<const typename Half<F16>::x8 *>(mine + (2 * c + (lane >> 5)) * 8);
    // positions that this lane's row sees, and the fewest and most that a row of the wave does
    const int sees = max(token(lane & 31) + ahead + 1, 0);
    const bool live = q0 < queries;
    const int fewest = __builtin_amdgcn_readfirstlane(max(token(0) + ahead + 1, 0)), most = __builtin_amdgcn_readfirstlane(max(token(31) + ahead + 1, 0));
    run_tiles<D, F16, WQ, PARTS, false>(rows, src, first, last, n, smem, [&](int t, uint64_t &word) {
        const int at = t * G::TILE + wk * G::SPAN;
        if (!live || at >= most) return NOTHING;
        if (at + G::SPAN <= fewest) return EVERYTHING;
        word = low_bits(sees - at);
        return SOME;
    });
    const uint64_t bad = __ballot(live && rows.spoiled());
    rows.leave(smem);
    if (bad)
        mend_rows<D, F16, WQ>(bad, rows.scale, src, first, last, n, wk, smem, query, [&](int t, uint64_t &word, int i) {
            word = low_bits(max(token(i) + ahead + 1, 0) - t * G::TILE - wk * G::SPAN);
            return SOME;
        });
    __syncthreads();
    constexpr int LANES = D / 8;
    const int e = tid % LANES;
    for (int c = tid / LANES; c < G::QROWS; c += THREADS / LANES) {
        const int qr = unit_q0 + c;
        if (qr >= queries) break;
        const Joined j = joined<D, WQ>(smem, c, e);
        if (a.parts == 1) {
            const bool none = j.sum == 0.0f;
            const int t = a.per_g.divide(qr);
            const int64_t to = (int64_t)(s.q0 + t) * a.H_q + h * a.G + qr - t * a.G;
            store_row<F16>(a.out, a.out_lowp, to * D + 8 * e, j.o, none ? 0.0f : 1.0f / j.sum);
            if (a.lse && e == 0) a.lse[to] = none ? -INFINITY : log_sum<F16>(j.ref, j.sum);
        } else {
            const int64_t slot = (int64_t)blockIdx.x * a.parts + part;
            float *o = a.slots + (slot * G::QROWS + c) * D + 8 * e;
            *reinterpret_cast<f32x4 *>(o) = f32x4{j.o[0], j.o[1], j.o[2], j.o[3]};
            *reinterpret_cast<f32x4 *>(o + 4) = f32x4{j.o[4], j.o[5], j.o[6], j.o[7]};
            if (e == 0) {
                a.slots_ml[slot * 2 * G::QROWS + c] = j.ref;
                a.slots_ml[slot * 2 * G::QROWS + G::QROWS + c] = j.sum;
            }
        }
    }
}

// The parts of a unit joined, in order.
template <int D, bool F16, int QROWS> __global__ __launch_bounds__(THREADS) void prompt_merge_kernel(PromptArgs a)
{
    __shared__ int wave_sums[WAVES];
    const int index = blockIdx.x / a.H_kv, h = blockIdx.x - index * a.H_kv;
    int b, tile;
    if (!find_unit<QROWS>(a, index, b, tile, wave_sums)) return;
    const Sequence s = sequence(a, b);
    constexpr int LANES = D / 8;
    const int c = blockIdx.y * (THREADS / LANES) + threadIdx.x / LANES, e = threadIdx.x % LANES;
    const int qr = tile * QROWS + c;
    if (c >= QROWS || qr >= s.q_len * a.G) return;
    float ref = -INFINITY;
    const int64_t slot0 = (int64_t)blockIdx.x * a.parts;
    for (int w = 0; w < a.parts; ++w) ref = fmaxf(ref, a.slots_ml[(slot0 + w) * 2 * QROWS + c]);
    float sum = 0.0f, o[8] = {};
    for (int w = 0; w < a.parts; ++w) {
        const int64_t slot = slot0 + w;
        const float m = a.slots_ml[slot * 2 * QROWS + c];
        if (m == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(m - ref);
        sum = fmaf(f, a.slots_ml[slot * 2 * QROWS + QROWS + c], sum);
        const float *p = a.slots + (slot * QROWS + c) * D + 8 * e;
        const f32x4 x = *reinterpret_cast<const f32x4 *>(p), y = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[i] = fmaf(f, x[i], o[i]);
            o[4 + i] = fmaf(f, y[i], o[4 + i]);
        }
    }
    const bool none = sum == 0.0f;
    const int t = a.per_g.divide(qr);
    const int64_t to = (int64_t)(s.q0 + t) * a.H_q + h * a.G + qr - t * a.G;
    store_row<F16>(a.out, a.out_lowp, to * D + 8 * e, o, none ? 0.0f : 1.0f / sum);
    if (a.lse && e == 0) a.lse[to] = none ? -INFINITY : log_sum<F16>(ref, sum);
}

typedef void (*PromptKernel)(PromptArgs);
template <int D, bool F16, int PARTS> PromptKernel by_waves(int wq)
{
    return wq == 1 ? prompt_kernel<D, F16, 1, PARTS> : prompt_kernel<D, F16, 4, PARTS>;
}
template <int D, bool F16> PromptKernel by_parts(int parts, int wq) { return parts == 1 ? by_waves<D, F16, 1>(wq) : by_waves<D, F16, 2>(wq); }
PromptKernel variant(int d, bool f16, int parts, int wq)
{
    return d == 128 ? (f16 ? by_parts<128, true>(parts, wq) : by_parts<128, false>(parts, wq)) : (f16 ? by_parts<64, true>(parts, wq) : by_parts<64, false>(parts, wq));
}
PromptKernel merge_variant(int d, bool f16, int wq)
{
    if (d == 128) return f16 ? (wq == 1 ? prompt_merge_kernel<128, true, 32> : prompt_merge_kernel<128, true, 128>) : (wq == 1 ? prompt_merge_kernel<128, false, 32> : prompt_merge_kernel<128, false, 128>);
    return f16 ? (wq == 1 ? prompt_merge_kernel<64, true, 32> : prompt_merge_kernel<64, true, 128>) : (wq == 1 ? prompt_merge_kernel<64, false, 32> : prompt_merge_kernel<64, false, 128>);
}
size_t lds_size(int d, int wq)
{
    if (d == 128) return wq == 1 ? Geo<128, 1>::LDS_BYTES : Geo<128, 4>::LDS_BYTES;
    return wq == 1 ? Geo<64, 1>::LDS_BYTES : Geo<64, 4>::LDS_BYTES;
}
size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call is cut: waves over query rows, workgroups per kv head at most (no length is known on the host), parts of a unit.
struct Cut { int wq, units, parts; };
Cut cut(const specattn_prompt_args *p)
{
    Cut c;
    const int64_t queries = (int64_t)p->total_q * (p->H_q / p->H_kv);
    c.wq = queries <= (int64_t)32 * p->B ? 1 : 4;
    c.units = (int)(queries / (32 * c.wq) + p->B);
    const int64_t all = (int64_t)c.units * p->H_kv, wanted = 2 * cu_count();
    // positions that a sequence has at most, in tiles
    const int64_t reach = p->page_table ? (int64_t)p->max_pages_per_seq * p->page_size : p->total_kv;
    c.parts = (int)std::min<int64_t>(std::max<int64_t>(wanted / all, 1), std::max<int64_t>(reach / 512, 1));
    return c;
}

}  // namespace

size_t prompt_workspace_bytes(const specattn_prompt_args *p)
{
    const Cut c = cut(p);
    if (c.parts == 1) return 0;
    const size_t rows = (size_t)c.units * p->H_kv * c.parts * 32 * c.wq;
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
    for (int k = 0; k < 16; ++k) {
        const int d = k & 1 ? 128 : 64, wq = k & 8 ? 4 : 1;
        const size_t bytes = lds_size(d, wq);
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(variant(d, k & 2, k & 4 ? 2 : 1, wq)), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) {
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
    a.kv_n = p->kv_stride_n * 2; a.kv_h = p->kv_stride_h * 2; a.kv_page = p->kv_stride_page * 2;
    a.B = p->B; a.H_q = p->H_q; a.H_kv = p->H_kv; a.G = p->H_q / p->H_kv;
    a.per_g = FastDivisor(a.G);
    a.total_q = p->total_q; a.total_kv = p->total_kv;
    a.pages = p->page_table ? p->num_pages : 0;
    a.page_shift = p->page_table ? log2i(p->page_size) : 0;
    a.max_pages = p->max_pages_per_seq;
    a.sm_scale = p->sm_scale > 0.0f ? p->sm_scale : 1.0f / std::sqrt((float)p->d);
    const Cut c = cut(p);
    a.parts = c.parts;
    const size_t rows = (size_t)c.units * p->H_kv * c.parts * 32 * c.wq;
    a.slots = static_cast<float *>(p->workspace);
    a.slots_ml = reinterpret_cast<float *>(static_cast<char *>(p->workspace) + a256(rows * p->d * sizeof(float)));
    const bool f16 = p->dtype == SPECATTN_F16;
    variant(p->d, f16, p->out ? 2 : 1, c.wq)<<<dim3(c.units * p->H_kv, c.parts), THREADS, lds_size(p->d, c.wq), stream>>>(a);
    st = check_launch("prompt_kernel");
    if (st != SPECATTN_OK || c.parts == 1) return st;
    const int per = THREADS / (p->d / 8);
    merge_variant(p->d, f16, c.wq)<<<dim3(c.units * p->H_kv, (32 * c.wq + per - 1) / per), THREADS, 0, stream>>>(a);
    return check_launch("prompt_merge_kernel");
}

}  // namespace specattn
