// Page tables, free pages and the slots of new tokens, from the lengths that the sequences have and are to have.
//
// Whole numbers only, and latency: a step of a serving batch moves a few hundred words.  What each sequence returns and asks for is summed up over the
// sequences by one workgroup; what follows from the sums - table entries, returned pages, slots - is then written by as many threads as there
// are entries, each finding its sequence by halving.  A new page may be one that another sequence has just returned: it is looked up where that
// sequence's table still holds it, so that no thread waits for another's store.  Small calls do both in one workgroup and one launch.
//
// 64 sequences that gain or lose up to 8 tokens: 7.2 to 8.5 us, a launch and a chain of four dependent trips to memory.  256 prompts of up to 4096 tokens,
// 12.6 MB of slots, positions and owners: 11.5 to 12 us in two launches (3.6 and 8; a copy of as many bytes would take 2.5).
#include "checks.h"
#include "serve.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int MAP_THREADS = 256;
constexpr int MAP_STARTS = 4096;
constexpr int ONE_WORKGROUP = 1024;                           // sequences that it holds in LDS

struct PagesArgs {
    int32_t *table, *free_pages;
    const int32_t *free_count, *seq_lens, *new_lens;
    int32_t *free_count_out, *lens_out, *token_starts, *slots, *positions, *owners;
    uint32_t *flags;
    int B, page_shift, max_pages, num_pages, capacity;
};

// A sequence: its lengths before and after (equal where nothing happens to it), and how many pages are returned, taken, and how many
// tokens come, ahead of its own.
struct Record {
    int now, then, given, taken;
};
struct Totals {
    int count, stack;                                         // free pages before, and with the returned ones
};
struct Plan {
    const Record *records;
    const int *starts;                                        // [B] first new token
    const Totals *totals;
};

// Sums that stop at 2^32 - 1: they stay comparable with any limit below, whatever the lengths say.
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
__device__ __forceinline__ uint32_t wave_sums(uint32_t v)
{
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
    v = add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
    return v;
}
// Sums of N values over the threads ahead of this one, and over all.
template <int N> struct Sums { uint32_t ahead[N], all[N]; };
template <int N> __device__ __forceinline__ Sums<N> block_sums(const uint32_t (&v)[N], uint32_t *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums<N> s;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t up = wave_sums(v[k]);
        if (lane == 63) lds[k * PLAN_WAVES + wave] = up;
        s.ahead[k] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)up, 0x138, 0xf, 0xf, true);       // of the lane before (0 in the first)
        s.all[k] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int w = 0; w < PLAN_WAVES; ++w) {
            const uint32_t x = lds[k * PLAN_WAVES + w];
            s.ahead[k] = w < wave ? add(s.ahead[k], x) : s.ahead[k];
            s.all[k] = add(s.all[k], x);
        }
    return s;
}

__device__ __forceinline__ int pages_of(const PagesArgs &a, int len) { return (int)(((uint32_t)len + (1u << a.page_shift) - 1) >> a.page_shift); }

__device__ void plan(const PagesArgs &a, Record *records, int *starts, Totals *totals, uint32_t *lds)
{
    const int tid = threadIdx.x;
    const int64_t reach = (int64_t)a.max_pages << a.page_shift;
    const int count = min(max(*a.free_count, 0), a.num_pages);
    auto read = [&](int b, int &now, int &then, uint32_t &flag) {
        now = a.seq_lens[b];
        then = a.new_lens[b];
        flag = now < 0 || now > reach || then < 0 ? SPECATTN_ROW_INVALID : then > reach ? SPECATTN_ROW_OVERFLOW : 0;
    };
    // what is returned in all comes first; of up to PLAN_THREADS sequences it is known when it is needed
    uint32_t given_all = 0;
    for (int b0 = 0; a.B > PLAN_THREADS && b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        int now, then;
        uint32_t flag, gives[1] = {0};
        if (b < a.B) {
            read(b, now, then, flag);
            if (!flag && then < now) gives[0] = (uint32_t)(pages_of(a, now) - pages_of(a, then));
        }
        given_all = add(given_all, block_sums(gives, lds).all[0]);
    }
    uint32_t given = 0, asked = 0, came = 0;                  // ahead of these sequences
    int taken_all = 0, tokens_all = 0, stack = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        int now = 0, then = 0;
        uint32_t flag = SPECATTN_ROW_INVALID, gives = 0, asks = 0, tokens = 0;
        if (b < a.B) read(b, now, then, flag);
        if (!flag) {
            gives = then < now ? (uint32_t)(pages_of(a, now) - pages_of(a, then)) : 0;
            asks = then > now ? (uint32_t)(pages_of(a, then) - pages_of(a, now)) : 0;
        }
        const uint32_t pages[2] = {gives, asks};
        const Sums<2> p = block_sums(pages, lds);
        if (a.B <= PLAN_THREADS) given_all = p.all[0];
        stack = (int)min((uint64_t)count + given_all, (uint64_t)a.num_pages);
        const uint32_t given_before = add(given, p.ahead[0]), asked_before = add(asked, p.ahead[1]);
        given = add(given, p.all[0]);
        asked = add(asked, p.all[1]);
        if (asks && add(asked_before, asks) > (uint32_t)stack) flag |= SPECATTN_ROW_OVERFLOW;
        if (!flag && then > now) tokens = (uint32_t)(then - now);
        const uint32_t coming[1] = {tokens};
        const Sums<1> c = block_sums(coming, lds);
        if (tokens && add(add(came, c.ahead[0]), tokens) > (uint32_t)a.capacity) flag |= SPECATTN_ROW_OVERFLOW;
        came = add(came, c.all[0]);
        // (sequences are refused from one on, as far as they ask for anything, so that what is granted lies without gaps)
        const bool grows = !flag && then > now;
        const uint32_t grants[2] = {grows ? (uint32_t)(then - now) : 0, grows ? asks : 0};
        Sums<2> g = {{c.ahead[0], 0}, {c.all[0], p.all[1]}};
        if (__syncthreads_or(flag == SPECATTN_ROW_OVERFLOW)) g = block_sums(grants, lds);
        if (b < a.B) {
            const int start = tokens_all + (int)g.ahead[0];
            records[b] = Record{now, flag ? now : then, (int)given_before, (int)asked_before};
            starts[b] = start;
            if (a.token_starts) a.token_starts[b] = start;
            a.lens_out[b] = flag ? now : then;
            if (a.flags) a.flags[b] = flag;
        }
        tokens_all += (int)g.all[0];
        taken_all += (int)g.all[1];
    }
    if (tid == 0) {
        totals->count = count;
        totals->stack = stack;
        if (a.token_starts) a.token_starts[a.B] = tokens_all;
        *a.free_count_out = stack - taken_all;
    }
}

// The last of n ascending values that is not above x.
template <typename F> __device__ __forceinline__ int last_not_above(int n, int x, F &&value)
{
    int lo = 0;
    for (int hi = n; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (value(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Entry i of the stack of free pages with the returned ones on it.
__device__ __forceinline__ int stack_entry(const PagesArgs &a, const Plan &p, int i)
{
    const int count = p.totals->count;
    if (i < count) return a.free_pages[i];
    const int rank = i - count;
    const int b = last_not_above(a.B, rank, [&](int x) { return p.records[x].given; });
    const Record r = p.records[b];
    return a.table[(int64_t)b * a.max_pages + pages_of(a, r.then) + rank - r.given];
}

// Table entries and returned pages, LANES threads to a sequence.
template <int LANES> __device__ __forceinline__ void write_pages(const PagesArgs &a, const Plan &p, int64_t thread, int64_t threads)
{
    const int lane = (int)(thread % LANES);
    for (int64_t b = thread / LANES; b < a.B; b += threads / LANES) {
        const Record r = p.records[b];
        const int have = pages_of(a, r.now), need = pages_of(a, r.then);
        int32_t *row = a.table + b * a.max_pages;
        for (int k = lane; k < need - have; k += LANES) row[have + k] = stack_entry(a, p, p.totals->stack - 1 - r.taken - k);
        for (int k = lane; k < have - need; k += LANES) {
            const int64_t to = (int64_t)p.totals->count + r.given + k;
            if (to < a.num_pages) a.free_pages[to] = row[need + k];
        }
    }
}

// Slots of new tokens; -1 behind the last one.  A thread takes four tokens at a time, so that their lookups are under way together.
__device__ __forceinline__ void write_tokens(const PagesArgs &a, const Plan &p, int64_t thread, int64_t threads)
{
    constexpr int U = 4;
    const Record last = p.records[a.B - 1];
    const int tokens = p.starts[a.B - 1] + max(last.then - last.now, 0);
    const int stack = p.totals->stack;
    for (int64_t i0 = thread; i0 < a.capacity; i0 += U * threads) {
        int b[U], place[U], page[U];
        Record r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * threads;
            b[u] = i < tokens ? last_not_above(a.B, (int)i, [&](int x) { return p.starts[x]; }) : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = p.records[max(b[u], 0)];
            place[u] = b[u] < 0 ? -1 : r[u].now + (int)(i0 + u * threads) - p.starts[b[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            page[u] = -1;
            if (b[u] < 0) continue;
            const int have = pages_of(a, r[u].now), at = place[u] >> a.page_shift;
            page[u] = at < have ? a.table[(int64_t)b[u] * a.max_pages + at] : stack_entry(a, p, stack - 1 - r[u].taken - (at - have));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * threads;
            if (i >= a.capacity) continue;
            const bool some = page[u] >= 0 && page[u] < a.num_pages;
            a.slots[i] = some ? (int)(((uint32_t)page[u] << a.page_shift) | ((uint32_t)place[u] & ((1u << a.page_shift) - 1))) : -1;
            if (a.positions) a.positions[i] = place[u];
            if (a.owners) a.owners[i] = b[u];
        }
    }
}

__global__ __launch_bounds__(PLAN_THREADS) void pages_kernel(PagesArgs a)
{
    __shared__ Record records[ONE_WORKGROUP];
    __shared__ int starts[ONE_WORKGROUP];
    __shared__ Totals totals;
    __shared__ uint32_t lds[2 * PLAN_WAVES];
    plan(a, records, starts, &totals, lds);
    __syncthreads();
    const Plan p = {records, starts, &totals};
    write_pages<16>(a, p, threadIdx.x, PLAN_THREADS);
    if (a.slots) write_tokens(a, p, threadIdx.x, PLAN_THREADS);
}

__global__ __launch_bounds__(PLAN_THREADS) void pages_plan_kernel(PagesArgs a, Record *records, int *starts, Totals *totals)
{
    __shared__ uint32_t lds[2 * PLAN_WAVES];
    plan(a, records, starts, totals, lds);
}

// (the tokens' sequences are found in LDS, as far as they fit there: every step of halving the starts in memory is a trip to L2)
__global__ __launch_bounds__(MAP_THREADS) void pages_map_kernel(PagesArgs a, Plan p)
{
    __shared__ int starts[MAP_STARTS];
    if (a.B <= MAP_STARTS) {
        for (int i = threadIdx.x; i < a.B; i += MAP_THREADS) starts[i] = p.starts[i];
        __syncthreads();
        p.starts = starts;
    }
    const int64_t thread = (int64_t)blockIdx.x * MAP_THREADS + threadIdx.x, threads = (int64_t)gridDim.x * MAP_THREADS;
    write_pages<64>(a, p, thread, threads);
    if (a.slots) write_tokens(a, p, thread, threads);
}

size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t pages_workspace_bytes(const specattn_pages_args *p)
{
    return 256 + a256((size_t)p->B * sizeof(Record)) + a256((size_t)p->B * sizeof(int));
}

specattn_status launch_pages(const specattn_pages_args *p, void *workspace, hipStream_t stream)
{
    PagesArgs a{};
    a.table = p->page_table; a.free_pages = p->free_pages;
    a.free_count = p->free_count; a.seq_lens = p->seq_lens; a.new_lens = p->new_lens;
    a.free_count_out = p->free_count_out; a.lens_out = p->lens_out;
    a.token_starts = p->token_starts; a.slots = p->slots; a.positions = p->positions; a.owners = p->owners;
    a.flags = p->row_flags;
    a.B = p->B; a.page_shift = log2i(p->page_size); a.max_pages = p->max_pages_per_seq; a.num_pages = p->num_pages;
    a.capacity = p->slots ? p->token_capacity : INT32_MAX;
    if (p->B <= ONE_WORKGROUP && (!p->slots || p->token_capacity <= 8 * PLAN_THREADS)) {
        pages_kernel<<<1, PLAN_THREADS, 0, stream>>>(a);
        return check_launch("pages_kernel");
    }
    char *ws = static_cast<char *>(workspace);
    Totals *totals = reinterpret_cast<Totals *>(ws);
    Record *records = reinterpret_cast<Record *>(ws + 256);
    int *starts = reinterpret_cast<int *>(ws + 256 + a256((size_t)p->B * sizeof(Record)));
    pages_plan_kernel<<<1, PLAN_THREADS, 0, stream>>>(a, records, starts, totals);
    const specattn_status st = check_launch("pages_plan_kernel");
    if (st != SPECATTN_OK) return st;
    const int64_t items = std::max<int64_t>(p->slots ? p->token_capacity : 0, (int64_t)p->B * 64);
    pages_map_kernel<<<(int)std::min<int64_t>((items + MAP_THREADS - 1) / MAP_THREADS, 8 * cu_count()), MAP_THREADS, 0, stream>>>(a, Plan{records, starts, totals});
    return check_launch("pages_map_kernel");
}

}  // namespace specattn
