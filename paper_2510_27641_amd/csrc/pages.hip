// Page tables, free pages and the slots of new tokens, from the lengths that the sequences have and are to have.
//
// Whole numbers only, and latency: a step of a serving batch moves a few hundred words.  What each sequence returns and asks for is summed up over the
// sequences by one workgroup; what follows from the sums - table entries, returned pages, slots - is then written by as many threads as there
// are entries, each finding its sequence by halving.  A new page may be one that another sequence has just returned: it is looked up where that
// sequence's table still holds it, so that no thread waits for another's store.  Small calls do both in one workgroup and one launch.
#include "checks.h"
#include "serve.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int MAP_THREADS = 256;
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
// Sum of v over the threads ahead of this one, and over all.
__device__ __forceinline__ uint32_t block_sums(uint32_t v, uint32_t &all, uint32_t *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t up = wave_sums(v);
    __syncthreads();
    if (lane == 63) lds[wave] = up;
    __syncthreads();
    uint32_t ahead = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)up, 0x138, 0xf, 0xf, true);   // of the lane before (0 in the first)
    all = 0;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
        const uint32_t s = lds[w];
        ahead = w < wave ? add(ahead, s) : ahead;
        all = add(all, s);
    }
    return ahead;
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
    uint32_t given_all = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        int now, then;
        uint32_t flag, all, gives = 0;
        if (b < a.B) {
            read(b, now, then, flag);
            if (!flag && then < now) gives = (uint32_t)(pages_of(a, now) - pages_of(a, then));
        }
        block_sums(gives, all, lds);
        given_all = add(given_all, all);
    }
    const int stack = (int)min((uint64_t)count + given_all, (uint64_t)a.num_pages);
    uint32_t given = 0, asked = 0, came = 0;                  // ahead of these sequences
    int taken_all = 0, tokens_all = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        int now = 0, then = 0;
        uint32_t flag = SPECATTN_ROW_INVALID, gives = 0, asks = 0, tokens = 0, all;
        if (b < a.B) read(b, now, then, flag);
        if (!flag) {
            gives = then < now ? (uint32_t)(pages_of(a, now) - pages_of(a, then)) : 0;
            asks = then > now ? (uint32_t)(pages_of(a, then) - pages_of(a, now)) : 0;
        }
        const uint32_t given_before = add(given, block_sums(gives, all, lds));
        given = add(given, all);
        const uint32_t asked_before = add(asked, block_sums(asks, all, lds));
        asked = add(asked, all);
        if (asks && add(asked_before, asks) > (uint32_t)stack) flag |= SPECATTN_ROW_OVERFLOW;
        if (!flag && then > now) tokens = (uint32_t)(then - now);
        const uint32_t came_before = add(came, block_sums(tokens, all, lds));
        came = add(came, all);
        if (tokens && add(came_before, tokens) > (uint32_t)a.capacity) flag |= SPECATTN_ROW_OVERFLOW;
        const bool grows = !flag && then > now;
        // (sequences are refused from one on, as far as they ask for anything, so that what is granted lies without gaps)
        const uint32_t granted = block_sums(grows ? (uint32_t)(then - now) : 0, all, lds) + (uint32_t)tokens_all;
        if (b < a.B) {
            records[b] = Record{now, flag ? now : then, (int)given_before, (int)asked_before};
            starts[b] = (int)granted;
            if (a.token_starts) a.token_starts[b] = (int)granted;
            a.lens_out[b] = flag ? now : then;
            if (a.flags) a.flags[b] = flag;
        }
        tokens_all += (int)all;
        block_sums(grows ? asks : 0, all, lds);
        taken_all += (int)all;
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

// Table entries and returned pages of sequences first, first + step, ...: a wave each.
__device__ __forceinline__ void write_pages(const PagesArgs &a, const Plan &p, int first, int step)
{
    const int lane = threadIdx.x & 63;
    for (int b = first; b < a.B; b += step) {
        const Record r = p.records[b];
        const int have = pages_of(a, r.now), need = pages_of(a, r.then);
        int32_t *row = a.table + (int64_t)b * a.max_pages;
        for (int k = lane; k < need - have; k += 64) row[have + k] = stack_entry(a, p, p.totals->stack - 1 - r.taken - k);
        for (int k = lane; k < have - need; k += 64) {
            const int64_t to = (int64_t)p.totals->count + r.given + k;
            if (to < a.num_pages) a.free_pages[to] = row[need + k];
        }
    }
}

// Slots of new tokens first, first + step, ...; -1 behind the last one.
__device__ __forceinline__ void write_tokens(const PagesArgs &a, const Plan &p, int64_t first, int64_t step)
{
    const Record last = p.records[a.B - 1];
    const int tokens = p.starts[a.B - 1] + max(last.then - last.now, 0);
    for (int64_t i = first; i < a.capacity; i += step) {
        int slot = -1, place = -1, b = -1;
        if (i < tokens) {
            b = last_not_above(a.B, (int)i, [&](int x) { return p.starts[x]; });
            const Record r = p.records[b];
            place = r.now + (int)i - p.starts[b];
            const int have = pages_of(a, r.now), at = place >> a.page_shift;
            const int page = at < have ? a.table[(int64_t)b * a.max_pages + at] : stack_entry(a, p, p.totals->stack - 1 - r.taken - (at - have));
            if (page >= 0 && page < a.num_pages) slot = (int)(((uint32_t)page << a.page_shift) | ((uint32_t)place & ((1u << a.page_shift) - 1)));
        }
        a.slots[i] = slot;
        if (a.positions) a.positions[i] = place;
        if (a.owners) a.owners[i] = b;
    }
}

__global__ __launch_bounds__(PLAN_THREADS) void pages_kernel(PagesArgs a)
{
    __shared__ Record records[ONE_WORKGROUP];
    __shared__ int starts[ONE_WORKGROUP];
    __shared__ Totals totals;
    __shared__ uint32_t lds[PLAN_WAVES];
    plan(a, records, starts, &totals, lds);
    __syncthreads();
    const Plan p = {records, starts, &totals};
    write_pages(a, p, threadIdx.x >> 6, PLAN_WAVES);
    if (a.slots) write_tokens(a, p, threadIdx.x, PLAN_THREADS);
}

__global__ __launch_bounds__(PLAN_THREADS) void pages_plan_kernel(PagesArgs a, Record *records, int *starts, Totals *totals)
{
    __shared__ uint32_t lds[PLAN_WAVES];
    plan(a, records, starts, totals, lds);
}

__global__ __launch_bounds__(MAP_THREADS) void pages_map_kernel(PagesArgs a, Plan p)
{
    const int64_t thread = (int64_t)blockIdx.x * MAP_THREADS + threadIdx.x, threads = (int64_t)gridDim.x * MAP_THREADS;
    write_pages(a, p, (int)(thread >> 6), (int)(threads >> 6));
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
