// Eviction from a cache by accumulated attention weight (selection of the slots that stay, moves of their rows).
//
// score' = fp32(decay * score + the rows' entries, added up in fp64 member by member), one rounding in all, so that the
// state does not depend on how the work is cut.  A slot's key is its score as an unsigned number of the same order (NaN
// lowest of all, tokens that have to stay highest of all); the K slots that stay are those above the K-th largest key, which radix
// passes over the keys find, and the lowest slots among those that equal it.  What stays beyond the new length moves into the
// holes below it: as many bytes as slots dropped there, instead of a new copy of everything behind the first hole.
//
// Bound by memory where rows are long, by the chain of launches and of radix passes where they are short.  64 rows of 32768 slots, 20
// entries each, a quarter stays, 4-bit cache: sums 38 us (0.2 GB, 5.3 TB/s), selection in slices 4.7 + 4.9 + 13.6 + 7.9, moves 29 us; 4
// sequences of up to 131072, half stays, 8 bf16 heads: moves 93 us (4.4 TB/s; a plain copy 4.8).  64 rows of 8197: 7.3 + 12.8 + 4.1 us.
#include "mx.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int ADD_THREADS = 256, ADD_SLOTS = 4;               // a thread adds up slots j, j + 256, j + 512, j + 768
constexpr int PICK_THREADS = 1024;                            // of a workgroup that holds a whole row
constexpr int SLICE_THREADS = 512, SLICE_KEYS = 8, SLICE = SLICE_THREADS * SLICE_KEYS;       // and of one that holds a slice of it: keys per thread, slots
constexpr int MAX_SLICES = SPECATTN_MAX_N / SLICE;
// A key is found 12, 10 and 10 bits at a time: with 11 in the first pass, four bins per octave, the lanes that meet in one counter, which are
// added one after the other, took most of it.
constexpr int TOP_BITS = 12, MID_BITS = 10, LOW_BITS = 10;
constexpr int TOP_BINS = 1 << TOP_BITS, MID_BINS = 1 << MID_BITS, LOW_BINS = 1 << LOW_BITS, TOP_SHIFT = 32 - TOP_BITS;
// Bytes of a row that its selecting workgroup adds up itself, a launch less.  In one launch / two, us: 64 rows of 1024 slots with one entry each,
// 12 KiB, 10.5 / 11.6; 512 rows of 2048 with one, 24 KiB, 23.1 / 26.7; with five entries 1024 slots are even, 28 KiB (64 rows 12.1 / 11.9, 512 rows
// 24.9 / 21.6), and with 16 no longer, 72 KiB (14.6 / 12.6, 33.7 / 23.8): one CU waits for one trip of entries after the other.  (Longer rows with up to
// three entries would gain beyond the line: 64 rows of 4096 with three, 80 KiB, 12.4 / 14.0.)
constexpr int64_t ADD_ITSELF = 32 << 10;
constexpr uint32_t KEY_STAYS = 0xffffffffu, KEY_NAN = 0;

struct EvictLaunch {
    specattn_evict_args e;
    uint32_t *keys;                                           // [B*H][stride]
    int stride;                                               // n_max, rounded up to whole threads of either kind of workgroup
    // rows that are cut up
    uint32_t *hist;                                           // [B*H][TOP_BINS]
    uint32_t *candidates;                                     // [B*H][stride]: of every slice, its keys in the bin of the K-th largest, in slot order
    int32_t *info;                                            // [B*H][slices][4]: keys above that bin and in it, each below and beyond the new length
    int slices;                                               // 0: rows are not cut up
    int members;                                              // rows of probs per score row
};

__device__ __forceinline__ int row_length(const specattn_evict_args &e, int b)
{
    return e.seq_lens ? min(max(e.seq_lens[b], 0), e.n_max) : e.n_max;
}

__device__ __forceinline__ uint32_t key_of(float score)
{
    if (score != score) return KEY_NAN;
    const uint32_t u = __float_as_uint(score + 0.0f);         // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// New scores and keys of slots first, first + GAP, ... of row r; WIDTH neighbouring slots at each place.
template <int PLACES, int WIDTH, int GAP> __device__ __forceinline__ void add_slots(const EvictLaunch &l, int r, int b, int h, int len, int first)
{
    typedef float Wide __attribute__((ext_vector_type(WIDTH)));
    const specattn_evict_args &e = l.e;
    if (first >= len) return;
    const int64_t row = b * e.row_stride_b + h * e.row_stride_h;
    const int next = e.next_positions[b];
    double sum[PLACES][WIDTH];
    int at[PLACES], place[PLACES][WIDTH];
    // (behind the row: its last place again, not written; with WIDTH > 1 rows are padded to whole places.  Places in the text are asked for
    // here, not where they are used: a trip to memory less, 1 us of 8.2 for 64 rows of 8197.)
#pragma unroll
    for (int k = 0; k < PLACES; ++k) {
        at[k] = min(first + k * GAP, (len - 1) / WIDTH * WIDTH);
        const Wide x = *reinterpret_cast<const Wide *>(e.scores + row + at[k]);
#pragma unroll
        for (int i = 0; i < WIDTH; ++i) {
            sum[k][i] = e.decay * (double)x[i];
            place[k][i] = e.positions[row + min(first + k * GAP + i, len - 1)];
        }
    }
    const float *probs = e.probs + b * e.probs_stride_b + (int64_t)h * l.members * e.probs_stride_row;
    constexpr int TRIP = 4;                                   // rows requested together
    for (int m0 = 0; m0 < l.members; m0 += TRIP) {
        Wide x[TRIP][PLACES];
#pragma unroll
        for (int t = 0; t < TRIP; ++t)                        // (behind the last row: that one again, not added)
#pragma unroll
            for (int k = 0; k < PLACES; ++k) x[t][k] = __builtin_nontemporal_load(reinterpret_cast<const Wide *>(probs + min(m0 + t, l.members - 1) * e.probs_stride_row + at[k]));
#pragma unroll
        for (int t = 0; t < TRIP; ++t)
#pragma unroll
            for (int k = 0; k < PLACES; ++k)
#pragma unroll
                for (int i = 0; i < WIDTH; ++i) sum[k][i] += m0 + t < l.members ? (double)x[t][k][i] : 0.0;
    }
#pragma unroll
    for (int k = 0; k < PLACES; ++k)
#pragma unroll
        for (int i = 0; i < WIDTH; ++i) {
            const int j = first + k * GAP + i;
            if (j >= len) continue;
            const float score = (float)sum[k][i];
            const bool stays = place[k][i] < e.sinks || place[k][i] >= (int64_t)next - e.recent;
            e.scores_out[row + j] = score;
            l.keys[(int64_t)r * l.stride + j] = stays ? KEY_STAYS : key_of(score);
        }
}

// WIDTH 4 where rows start and lie at whole 16 bytes.
template <int WIDTH> __global__ __launch_bounds__(ADD_THREADS) void evict_add_kernel(EvictLaunch l)
{
    const specattn_evict_args &e = l.e;
    for (int r = blockIdx.y; r < e.B * e.H; r += gridDim.y) {
        const int b = r / e.H, h = r - b * e.H, len = row_length(e, b);
        if (l.slices && blockIdx.x == 0) {                    // (the launches behind this one add to these)
            for (int i = threadIdx.x; i < TOP_BINS; i += ADD_THREADS) l.hist[(int64_t)r * TOP_BINS + i] = 0;
            if (e.row_flags && threadIdx.x == 0) e.row_flags[r] = 0;
        }
        add_slots<ADD_SLOTS / WIDTH, WIDTH, ADD_THREADS * WIDTH>(l, r, b, h, len, blockIdx.x * ADD_THREADS * ADD_SLOTS + threadIdx.x * WIDTH);
    }
}

// Shared memory of a selecting workgroup.
template <int THREADS> struct Pick {
    uint32_t bins[TOP_BINS];
    int wave_sum[THREADS / 64][2];
    int found[2];
    uint32_t kept[THREADS];                                   // a bit per key of a thread
};

__device__ __forceinline__ int wave_last(int v) { return __builtin_amdgcn_readlane(v, 63); }

// The bin that holds the K-th largest of the counted entries (there are as many at least), and how many lie above it.  Called by all threads,
// which take the bins from the highest down, BINS / THREADS each.
template <int BINS, int THREADS> __device__ __forceinline__ void locate(Pick<THREADS> &s, int K, int &bin, int &above)
{
    constexpr int PER = BINS > THREADS ? BINS / THREADS : 1;
    const int tid = threadIdx.x, wave = tid / 64;
    __syncthreads();
    const int top = BINS - 1 - tid * PER;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += top >= 0 ? s.bins[top - (i + tid) % PER] : 0;       // (each thread from a place of its own: other banks)
    int upto = wave_inclusive_sum(mine);
    if (tid % 64 == 63) s.wave_sum[wave][0] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += s.wave_sum[w][0];
    if (upto - mine < K && K <= upto) {
        int over = upto - mine, at = top;
        for (int c; over + (c = s.bins[at]) < K; --at) over += c;
        s.found[0] = at;
        s.found[1] = over;
    }
    __syncthreads();
    bin = s.found[0];
    above = s.found[1];
}
template <int BINS, int THREADS> __device__ __forceinline__ void clear(Pick<THREADS> &s)
{
    for (int i = threadIdx.x; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
}

// A row's arrays.
struct EvictRow {
    int r, b, h, len, K;
    float *scores;
    const int32_t *from;
    int32_t *to, *src, *dst;
    __device__ __forceinline__ EvictRow(const specattn_evict_args &e, int row) : r(row), b(row / e.H)
    {
        h = row - b * e.H;
        len = row_length(e, b);
        K = min(len, e.budget);
        const int64_t at = b * e.row_stride_b + h * e.row_stride_h;
        scores = e.scores_out + at;
        from = e.positions + at;
        to = e.positions_out + at;
        src = e.move_src + row * e.move_stride_row;
        dst = e.move_dst + row * e.move_stride_row;
    }
};

// A thread's keys: those of KEYS consecutive slots from `first`.
template <int KEYS> struct Held {
    uint32_t key[KEYS] __attribute__((aligned(16)));
    int first;
    __device__ __forceinline__ void load(const uint32_t *keys, int start, int len)
    {
        first = start + threadIdx.x * KEYS;
        if (first >= len) return;                             // (what lies behind the row is not looked at)
#pragma unroll
        for (int k = 0; k < KEYS; k += 4) *reinterpret_cast<uint4 *>(key + k) = *reinterpret_cast<const uint4 *>(keys + first + k);
    }
};

// Keys above `cut` and equal to it, below and beyond slot K; two counts to a word, the lower half that of the slots below K.
struct Sides { uint32_t above = 0, equal = 0; };
template <int KEYS> __device__ __forceinline__ Sides count_sides(const Held<KEYS> &x, uint32_t cut, int shift, int K, int len)
{
    Sides n;
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
        const int j = x.first + k;
        const uint32_t key = x.key[k] >> shift, one = j >= len ? 0 : j < K ? 1 : 1 << 16;
        n.above += key > cut ? one : 0;
        n.equal += key == cut ? one : 0;
    }
    return n;
}
// The same of all slots ahead of this thread's in the workgroup, and in all of it.
template <int THREADS> __device__ __forceinline__ Sides scan_sides(Pick<THREADS> &s, Sides n, Sides &all)
{
    const int wave = threadIdx.x / 64;
    Sides upto;
    upto.above = wave_inclusive_sum(n.above);
    upto.equal = wave_inclusive_sum(n.equal);
    __syncthreads();
    if (threadIdx.x % 64 == 63) { s.wave_sum[wave][0] = upto.above; s.wave_sum[wave][1] = upto.equal; }
    __syncthreads();
    all = Sides();
    upto.above -= n.above;
    upto.equal -= n.equal;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t a = s.wave_sum[w][0], e = s.wave_sum[w][1];
        if (w < wave) { upto.above += a; upto.equal += e; }
        all.above += a;
        all.equal += e;
    }
    return upto;
}

// What lies ahead of a slot in its row: keys above the cut and equal to it below K and beyond.  `need` of the equal keys stay, the lowest
// slots first.
struct Ahead {
    int above_l = 0, equal_l = 0, above_r = 0, equal_r = 0;
    __device__ __forceinline__ void add(Sides n)
    {
        above_l += n.above & 0xffff; equal_l += n.equal & 0xffff;
        above_r += n.above >> 16; equal_r += n.equal >> 16;
    }
    // holes among `slots` slots below K, movers among those beyond
    __device__ __forceinline__ int holes(int slots, int need) const { return slots - above_l - min(need, equal_l); }
    __device__ __forceinline__ int movers(int need) const { return above_r + min(max(need - equal_l, 0), equal_r); }
};

// Writes a thread's part of the lists, and which of its slots stay.
template <int KEYS, int THREADS> __device__ __forceinline__ void emit(const EvictRow &w, const Held<KEYS> &x, uint32_t cut, int need, const Ahead &ahead, Pick<THREADS> &s)
{
    int equals = ahead.equal_l + ahead.equal_r, hole = ahead.holes(min(x.first, w.K), need), mover = ahead.movers(need);
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
        const int j = x.first + k;
        const bool in = j < w.len, low = j < w.K, equal = in && x.key[k] == cut, kept = in && (x.key[k] > cut || (equal && equals < need));
        equals += equal;
        if (low && !kept) w.dst[hole++] = j;
        if (!low && kept) w.src[mover++] = j;
        bits |= (uint32_t)kept << k;
    }
    s.kept[threadIdx.x] = bits;
}

// to[j] = from[j] for begin <= j < end, eight requests of a thread at a time
template <int THREADS> __device__ __forceinline__ void copy_range(int32_t *to, const int32_t *from, int begin, int end)
{
    for (int j0 = begin + threadIdx.x; j0 < end; j0 += 8 * THREADS) {
        int32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = from[min(j0 + k * THREADS, end - 1)];
#pragma unroll
        for (int k = 0; k < 8; ++k) if (j0 + k * THREADS < end) to[j0 + k * THREADS] = v[k];
    }
}

__device__ __forceinline__ bool nan_among(const float *scores, int from, int to, int threads)
{
    int bad = 0;
    for (int j = from + threadIdx.x; j < to; j += threads) bad |= scores[j] != scores[j];
    return __syncthreads_or(bad);
}

// One workgroup per row of up to 1024 KEYS slots, which are read once; with ADD it adds them up itself.
template <int KEYS, bool ADD> __global__ __launch_bounds__(PICK_THREADS) void evict_pick_kernel(EvictLaunch l)
{
    __shared__ Pick<PICK_THREADS> s;
    const specattn_evict_args &e = l.e;
    const int tid = threadIdx.x;
    const EvictRow w(e, blockIdx.x);
    if constexpr (ADD) {
        add_slots<KEYS, 1, PICK_THREADS>(l, w.r, w.b, w.h, w.len, tid);
        __syncthreads();                                      // (the keys are read back by other threads)
    }
    Held<KEYS> x;
    if (w.len > w.K) x.load(l.keys + (int64_t)w.r * l.stride, 0, w.len);
    if (tid == 0 && w.h == 0) e.new_lens[w.b] = w.K;
    if (e.row_flags) {
        const bool bad = nan_among(w.scores, 0, w.len, PICK_THREADS);
        if (tid == 0) e.row_flags[w.r] = bad ? SPECATTN_ROW_INVALID : 0u;
    }
    if (w.from != w.to) copy_range<PICK_THREADS>(w.to, w.from, 0, w.K);
    if (w.len == w.K) {                                       // nothing leaves
        if (tid == 0) e.move_counts[w.r] = 0;
        return;
    }
    int bin, above, need = w.K;
    clear<TOP_BINS>(s);
#pragma unroll
    for (int k = 0; k < KEYS; ++k) if (x.first + k < w.len) atomicAdd(&s.bins[x.key[k] >> TOP_SHIFT], 1u);
    locate<TOP_BINS>(s, need, bin, above);
    uint32_t cut = bin;
    need -= above;
    clear<MID_BINS>(s);
#pragma unroll
    for (int k = 0; k < KEYS; ++k) if (x.first + k < w.len && x.key[k] >> TOP_SHIFT == cut) atomicAdd(&s.bins[x.key[k] >> LOW_BITS & (MID_BINS - 1)], 1u);
    locate<MID_BINS>(s, need, bin, above);
    cut = cut << MID_BITS | bin;
    need -= above;
    clear<LOW_BINS>(s);
#pragma unroll
    for (int k = 0; k < KEYS; ++k) if (x.first + k < w.len && x.key[k] >> LOW_BITS == cut) atomicAdd(&s.bins[x.key[k] & (LOW_BINS - 1)], 1u);
    locate<LOW_BINS>(s, need, bin, above);
    cut = cut << LOW_BITS | bin;                              // kept: every key above it, and the first `need` that equal it
    need -= above;

    Sides all;
    Ahead ahead, row;
    ahead.add(scan_sides(s, count_sides(x, cut, 0, w.K, w.len), all));
    row.add(all);
    emit(w, x, cut, need, ahead, s);
    const int moves = row.movers(need);
    if (tid == 0) e.move_counts[w.r] = moves;
    __syncthreads();
    for (int i = tid; i < moves; i += PICK_THREADS) {
        const int a = w.src[i], d = w.dst[i];
        w.scores[d] = w.scores[a];
        w.to[d] = w.from[a];
    }
    __syncthreads();
    for (int j = w.K + tid; j < w.len; j += PICK_THREADS) { w.scores[j] = 0.0f; w.to[j] = -1; }
}

// Rows that are cut into slices, one workgroup each, in four launches: the keys' highest bits are counted; the K-th largest key's bin
// is located and the slice's keys in it set aside; the K-th largest is found among those of all slices and the lists are written; the
// rows' own state moves.
__global__ __launch_bounds__(SLICE_THREADS) void evict_count_kernel(EvictLaunch l)
{
    __shared__ Pick<SLICE_THREADS> s;
    const EvictRow w(l.e, blockIdx.x);
    const int start = blockIdx.y * SLICE;
    if (w.len == w.K || start >= w.len) return;
    Held<SLICE_KEYS> x;
    x.load(l.keys + (int64_t)w.r * l.stride, start, w.len);
    clear<TOP_BINS>(s);
#pragma unroll
    for (int k = 0; k < SLICE_KEYS; ++k) if (x.first + k < w.len) atomicAdd(&s.bins[x.key[k] >> TOP_SHIFT], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < TOP_BINS; i += SLICE_THREADS) if (s.bins[i]) atomicAdd(&l.hist[(int64_t)w.r * TOP_BINS + i], s.bins[i]);
}

__global__ __launch_bounds__(SLICE_THREADS) void evict_collect_kernel(EvictLaunch l)
{
    __shared__ Pick<SLICE_THREADS> s;
    const specattn_evict_args &e = l.e;
    const EvictRow w(e, blockIdx.x);
    const int tid = threadIdx.x, start = blockIdx.y * SLICE;
    if (start >= w.len) return;
    if (e.row_flags && nan_among(w.scores, start, min(start + SLICE, w.len), SLICE_THREADS) && tid == 0) atomicOr(&e.row_flags[w.r], SPECATTN_ROW_INVALID);
    if (w.len == w.K) return;
    Held<SLICE_KEYS> x;
    x.load(l.keys + (int64_t)w.r * l.stride, start, w.len);
    for (int i = tid; i < TOP_BINS; i += SLICE_THREADS) s.bins[i] = l.hist[(int64_t)w.r * TOP_BINS + i];
    int bin, above;
    locate<TOP_BINS>(s, w.K, bin, above);
    Sides all;
    const Sides ahead = scan_sides(s, count_sides(x, (uint32_t)bin, TOP_SHIFT, w.K, w.len), all);
    if (tid < 4) l.info[((int64_t)w.r * l.slices + blockIdx.y) * 4 + tid] = tid == 0 ? all.above & 0xffff : tid == 1 ? all.equal & 0xffff : tid == 2 ? all.above >> 16 : all.equal >> 16;
    uint32_t *to = l.candidates + (int64_t)w.r * l.stride + start + (ahead.equal & 0xffff) + (ahead.equal >> 16);
#pragma unroll
    for (int k = 0; k < SLICE_KEYS; ++k) if (x.first + k < w.len && x.key[k] >> TOP_SHIFT == (uint32_t)bin) *to++ = x.key[k];
}

__global__ __launch_bounds__(SLICE_THREADS) void evict_emit_kernel(EvictLaunch l)
{
    constexpr int STAGED = 8192;                              // candidates of a row that are looked at in shared memory
    __shared__ Pick<SLICE_THREADS> s;
    __shared__ int first[MAX_SLICES + 1];                     // of each slice's candidates among the row's
    __shared__ int ahead[5];                                  // of this slice: above the cut and equal to it below K and beyond; candidates below K
    __shared__ uint32_t staged[STAGED];
    const specattn_evict_args &e = l.e;
    const EvictRow w(e, blockIdx.x);
    const int tid = threadIdx.x, slice = blockIdx.y, start = slice * SLICE, end = min(start + SLICE, w.len);
    if (tid == 0 && w.h == 0 && slice == 0) e.new_lens[w.b] = w.K;
    if (w.len == w.K) {
        if (w.from != w.to) copy_range<SLICE_THREADS>(w.to, w.from, start, end);
        if (tid == 0 && slice == 0) e.move_counts[w.r] = 0;
        return;
    }
    if (start >= w.len) return;
    const int slices = (w.len + SLICE - 1) / SLICE;
    const uint32_t *candidates = l.candidates + (int64_t)w.r * l.stride;
    Held<SLICE_KEYS> x;
    x.load(l.keys + (int64_t)w.r * l.stride, start, w.len);
    for (int i = tid; i < TOP_BINS; i += SLICE_THREADS) s.bins[i] = l.hist[(int64_t)w.r * TOP_BINS + i];
    if (tid < 5) ahead[tid] = 0;
    __syncthreads();
    if (tid < 64) {
        int base = 0;
        for (int v0 = 0; v0 < slices; v0 += 64) {
            const int v = v0 + tid;
            int4 n = {0, 0, 0, 0};
            if (v < slices) n = *reinterpret_cast<const int4 *>(l.info + ((int64_t)w.r * l.slices + v) * 4);
            const int upto = base + wave_inclusive_sum(n.y + n.w);
            if (v < slices) first[v + 1] = upto;
            if (v < slice) { atomicAdd(&ahead[0], n.x); atomicAdd(&ahead[2], n.z); }
            if (n.y) atomicAdd(&ahead[4], n.y);
            base = wave_last(upto);
        }
        if (tid == 0) first[0] = 0;
    }
    int bin, above, need = w.K;
    locate<TOP_BINS>(s, need, bin, above);
    uint32_t cut = bin;
    need -= above;
    const int all = first[slices], below = ahead[4], mine = first[slice];
    auto from_memory = [&](int i) {                           // candidate i of the row
        int lo = 0, hi = slices;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first[mid] <= i) lo = mid; else hi = mid;
        }
        return candidates[lo * SLICE + i - first[lo]];
    };
    const bool few = all <= STAGED;
    if (few)
#pragma unroll 4
        for (int i = tid; i < all; i += SLICE_THREADS) staged[i] = from_memory(i);
    auto each = [&](int n, auto &&f) {
        if (few) for (int i = tid; i < n; i += SLICE_THREADS) f(i, staged[i]);
        else
#pragma unroll 4
            for (int i = tid; i < n; i += SLICE_THREADS) f(i, from_memory(i));
    };
    clear<MID_BINS>(s);
    each(all, [&](int, uint32_t key) { atomicAdd(&s.bins[key >> LOW_BITS & (MID_BINS - 1)], 1u); });
    locate<MID_BINS>(s, need, bin, above);
    cut = cut << MID_BITS | bin;
    need -= above;
    clear<LOW_BINS>(s);
    each(all, [&](int, uint32_t key) { if (key >> LOW_BITS == cut) atomicAdd(&s.bins[key & (LOW_BINS - 1)], 1u); });
    locate<LOW_BINS>(s, need, bin, above);
    cut = cut << LOW_BITS | bin;
    need -= above;
    // (candidates below K come first, as slots do)
    int n[4] = {0, 0, 0, 0};
    each(mine, [&](int i, uint32_t key) {
        n[0] += i < below && key > cut; n[1] += i < below && key == cut;
        n[2] += i >= below && key > cut; n[3] += i >= below && key == cut;
    });
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int sum = wave_last(wave_inclusive_sum(n[k]));
        if (tid % 64 == 0 && sum) atomicAdd(&ahead[k], sum);
    }
    __syncthreads();
    Ahead at;
    at.above_l = ahead[0]; at.equal_l = ahead[1]; at.above_r = ahead[2]; at.equal_r = ahead[3];
    Ahead upto = at;
    Sides sides;
    at.add(scan_sides(s, count_sides(x, cut, 0, w.K, w.len), sides));
    upto.add(sides);
    emit(w, x, cut, need, at, s);
    if (slice == slices - 1 && tid == 0) e.move_counts[w.r] = upto.movers(need);
    if (w.from != w.to) copy_range<SLICE_THREADS>(w.to, w.from, start, min(end, w.K));
    __syncthreads();
    for (int j = max(start, w.K) + tid; j < end; j += SLICE_THREADS)
        if (!(s.kept[(j - start) / SLICE_KEYS] >> (j - start) % SLICE_KEYS & 1)) { w.scores[j] = 0.0f; w.to[j] = -1; }
}

__global__ __launch_bounds__(256) void evict_state_kernel(EvictLaunch l)
{
    const EvictRow w(l.e, blockIdx.x);
    const int n = l.e.move_counts[w.r];
    for (int i = blockIdx.y * 256 + threadIdx.x; i < n; i += gridDim.y * 256) {
        const int a = w.src[i], d = w.dst[i];
        w.scores[d] = w.scores[a];
        w.to[d] = w.from[a];
        w.scores[a] = 0.0f;
        w.to[a] = -1;
    }
}

struct MoveLaunch {
    specattn_move_args m;
    int page_shift;
    int unit_shift[SPECATTN_MAX_PLANES];                      // log2 of the bytes moved at a time
    FastDivisor per_row[SPECATTN_MAX_PLANES];                 // by the units of a row
};

constexpr int MOVE_THREADS = 256, MOVE_FLIGHT = 8;           // requests of a lane under way

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Byte offset of a slot in a plane; false if there is no such slot.
__device__ __forceinline__ bool move_offset(const MoveLaunch &l, const specattn_move_plane &p, int b, int kv, int slot, int64_t &at)
{
    if (slot < 0 || slot >= l.m.n_max) return false;
    if (!l.m.page_table) { at = b * p.stride_b + kv * p.stride_h + slot * p.stride_n; return true; }
    const int page = l.m.page_table[(int64_t)b * l.m.max_pages_per_seq + (slot >> l.page_shift)];
    at = page * p.stride_page + kv * p.stride_h + (int64_t)(slot & ((1 << l.page_shift) - 1)) * p.stride_n;
    return page >= 0 && page < p.num_pages;
}

// A wave takes 64 moves of one head: their slots and pages are looked up once, a lane each, then the lanes go through the rows' units together.
template <typename V> __device__ __forceinline__ void move_rows(const MoveLaunch &l, const specattn_move_plane &p, const FastDivisor &per_row, int units)
{
    const int share = p.H_kv / l.m.H, all = l.m.B * p.H_kv, lane = threadIdx.x % 64;
    const int first = __builtin_amdgcn_readfirstlane(blockIdx.x * MOVE_THREADS + threadIdx.x / 64 * 64);
    uint8_t *data = static_cast<uint8_t *>(p.data);
    for (int y = blockIdx.y; y < all; y += gridDim.y) {
        const int b = y / p.H_kv, kv = y - b * p.H_kv, r = b * l.m.H + kv / share;
        const int moves = min(min(max(l.m.move_counts[r], 0), l.m.move_capacity) - first, 64);
        if (moves <= 0) continue;
        int64_t from = -1, to = -1;
        if (lane < moves) {
            const int64_t list = r * l.m.move_stride_row + first + lane;
            const int src = l.m.move_src[list], dst = l.m.move_dst[list];
            if (!move_offset(l, p, b, kv, src, from) || !move_offset(l, p, b, kv, dst, to)) from = -1;
        }
        const int items = moves * units;
        for (int i0 = 0; i0 < items; i0 += 64 * MOVE_FLIGHT) {
            V value[MOVE_FLIGHT];
            int64_t at[MOVE_FLIGHT];
#pragma unroll
            for (int k = 0; k < MOVE_FLIGHT; ++k) {
                const int item = min(i0 + 64 * k + lane, items - 1), m = per_row.divide(item), u = (item - m * units) * (int)sizeof(V);
                const int64_t f = __shfl(from, m, 64), t = __shfl(to, m, 64);
                at[k] = i0 + 64 * k + lane < items && f >= 0 ? t + u : -1;
                if (f >= 0) value[k] = __builtin_nontemporal_load(reinterpret_cast<const V *>(data + f + u));
            }
#pragma unroll
            for (int k = 0; k < MOVE_FLIGHT; ++k) if (at[k] >= 0) *reinterpret_cast<V *>(data + at[k]) = value[k];
        }
    }
}

__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(MoveLaunch l)
{
    const int z = blockIdx.z;
    const specattn_move_plane &p = l.m.planes[z];
    const int units = p.row_bytes >> l.unit_shift[z];
    if (l.unit_shift[z] == 4) move_rows<u32x4>(l, p, l.per_row[z], units);
    else if (l.unit_shift[z] == 3) move_rows<u32x2>(l, p, l.per_row[z], units);
    else move_rows<uint32_t>(l, p, l.per_row[z], units);
}

}  // namespace

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Rows that one workgroup cannot hold are cut up, and so are longer ones that leave most of the GPU idle.  In one workgroup each / cut up, us,
// one entry to add, 8, 64, 72, 128, 512 rows: of 16384 slots 21 / 24, 28 / 32, 29 / 37, 35 / 46, 97 / 134; of 16400 slots, where a thread
// holds 32 keys in place of 16, 27 / 23, 35 / 34, 36 / 36, 42 / 45, 111 / 139; of 32768 slots 37 / 26, 50 / 48, 52 / 52, 65 / 80, 214 / 280.
static int evict_slices(const specattn_evict_args *e)
{
    const int rows = e->B * e->H;
    return e->n_max <= 16 * PICK_THREADS || (e->n_max <= 32 * PICK_THREADS && rows > 64) ? 0 : (e->n_max + SLICE - 1) / SLICE;
}

static int evict_stride(const specattn_evict_args *e) { return (e->n_max + 31) & ~31; }

size_t evict_workspace_bytes(const specattn_evict_args *e)
{
    const size_t rows = (size_t)e->B * e->H, keys = align256(rows * evict_stride(e) * sizeof(uint32_t)), slices = evict_slices(e);
    return slices ? 2 * keys + align256(rows * TOP_BINS * sizeof(uint32_t)) + align256(rows * slices * 4 * sizeof(int32_t)) : keys;
}

specattn_status launch_evict_select(const specattn_evict_args *e, void *workspace, hipStream_t stream)
{
    EvictLaunch l;
    l.e = *e;
    l.members = e->probs ? e->H_draft / e->H * e->S : 0;
    l.slices = evict_slices(e);
    const int rows = e->B * e->H;
    char *ws = static_cast<char *>(workspace);
    l.stride = evict_stride(e);
    const size_t keys = align256((size_t)rows * l.stride * sizeof(uint32_t));
    l.keys = reinterpret_cast<uint32_t *>(ws);
    l.candidates = reinterpret_cast<uint32_t *>(ws + keys);
    l.hist = reinterpret_cast<uint32_t *>(ws + 2 * keys);
    l.info = reinterpret_cast<int32_t *>(ws + 2 * keys + align256((size_t)rows * TOP_BINS * sizeof(uint32_t)));
    specattn_status st;
    // A workgroup that holds its row also adds it up where that is little to read: a launch less.
    const bool small = l.slices == 0 && (int64_t)e->n_max * (l.members + 2) * (int64_t)sizeof(float) <= ADD_ITSELF;
    if (!small) {
        const int64_t elements = (l.members ? e->probs_stride_b | e->probs_stride_row : 0) | e->row_stride_b | e->row_stride_h | e->n_max;
        const bool wide = elements % 4 == 0 && (reinterpret_cast<uintptr_t>(e->probs) | reinterpret_cast<uintptr_t>(e->scores)) % 16 == 0;
        const dim3 grid((e->n_max + ADD_THREADS * ADD_SLOTS - 1) / (ADD_THREADS * ADD_SLOTS), std::min(rows, 65535));
        if (wide) evict_add_kernel<4><<<grid, ADD_THREADS, 0, stream>>>(l);
        else evict_add_kernel<1><<<grid, ADD_THREADS, 0, stream>>>(l);
        if ((st = check_launch("evict_add_kernel")) != SPECATTN_OK) return st;
    }
    if (l.slices == 0) {
        static_assert(ADD_ITSELF / (2 * sizeof(float)) <= 8 * PICK_THREADS, "a row that its workgroup adds up itself must fit 8 keys to a thread");
        if (small) evict_pick_kernel<8, true><<<rows, PICK_THREADS, 0, stream>>>(l);
        else if (e->n_max <= 8 * PICK_THREADS) evict_pick_kernel<8, false><<<rows, PICK_THREADS, 0, stream>>>(l);
        else if (e->n_max <= 16 * PICK_THREADS) evict_pick_kernel<16, false><<<rows, PICK_THREADS, 0, stream>>>(l);
        else evict_pick_kernel<32, false><<<rows, PICK_THREADS, 0, stream>>>(l);
        return check_launch("evict_pick_kernel");
    }
    const dim3 grid(rows, l.slices);
    evict_count_kernel<<<grid, SLICE_THREADS, 0, stream>>>(l);
    if ((st = check_launch("evict_count_kernel")) != SPECATTN_OK) return st;
    evict_collect_kernel<<<grid, SLICE_THREADS, 0, stream>>>(l);
    if ((st = check_launch("evict_collect_kernel")) != SPECATTN_OK) return st;
    evict_emit_kernel<<<grid, SLICE_THREADS, 0, stream>>>(l);
    if ((st = check_launch("evict_emit_kernel")) != SPECATTN_OK) return st;
    evict_state_kernel<<<dim3(rows, std::min((e->move_capacity + 255) / 256, 1024)), 256, 0, stream>>>(l);
    return check_launch("evict_state_kernel");
}

specattn_status launch_evict_move(const specattn_move_args *m, hipStream_t stream)
{
    MoveLaunch l;
    l.m = *m;
    l.page_shift = 0;
    while (m->page_table && (1 << l.page_shift) < m->page_size) ++l.page_shift;
    int rows = 0;
    for (int z = 0; z < m->num_planes; ++z) {
        const int bytes = m->planes[z].row_bytes;
        l.unit_shift[z] = bytes % 16 == 0 ? 4 : bytes % 8 == 0 ? 3 : 2;
        l.per_row[z] = FastDivisor(bytes >> l.unit_shift[z]);
        rows = std::max(rows, m->B * m->planes[z].H_kv);
    }
    evict_move_kernel<<<dim3((m->move_capacity + MOVE_THREADS - 1) / MOVE_THREADS, std::min(rows, 65535), m->num_planes), MOVE_THREADS, 0, stream>>>(l);
    return check_launch("evict_move_kernel");
}

}  // namespace specattn
