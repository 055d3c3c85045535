// Eviction from a cache by accumulated attention weight (selection of the slots that stay, moves of their rows).
//
// score' = fp32(decay * score + the rows' entries, added up in fp64 member by member), one rounding in all, so that the
// state does not depend on how the work is cut.  A slot's key is its score as an unsigned number of the same order (NaN
// lowest of all, tokens that have to stay highest of all); the K slots that stay are those above the K-th largest key, which radix
// passes over the keys find, and the lowest slots among those that equal it.  What stays beyond the new length moves into the
// holes below it: as many bytes as slots dropped there, instead of a new copy of everything behind the first hole.
#include "mx.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int ADD_THREADS = 256, ADD_SLOTS = 4;               // a thread adds up slots j, j + 256, j + 512, j + 768
constexpr int PICK_WAVES = 16, PICK_THREADS = PICK_WAVES * 64;
constexpr uint32_t KEY_STAYS = 0xffffffffu, KEY_NAN = 0;

struct EvictLaunch {
    specattn_evict_args e;
    uint32_t *keys;                                           // [B*H][n_max]
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

__global__ __launch_bounds__(ADD_THREADS) void evict_add_kernel(EvictLaunch l)
{
    const specattn_evict_args &e = l.e;
    for (int r = blockIdx.y; r < e.B * e.H; r += gridDim.y) {
        const int b = r / e.H, h = r - b * e.H, len = row_length(e, b);
        const int first = blockIdx.x * ADD_THREADS * ADD_SLOTS + threadIdx.x;
        const int64_t row = b * e.row_stride_b + h * e.row_stride_h;
        const int next = e.next_positions[b];
        double sum[ADD_SLOTS];
        int at[ADD_SLOTS];
#pragma unroll
        for (int k = 0; k < ADD_SLOTS; ++k) {
            at[k] = min(first + k * ADD_THREADS, len - 1);    // (behind the row: its last slot again, not written)
            sum[k] = len > 0 ? e.decay * (double)e.scores[row + at[k]] : 0.0;
        }
        if (first >= len) continue;
        const float *probs = e.probs + b * e.probs_stride_b + (int64_t)h * l.members * e.probs_stride_row;
#pragma unroll 4
        for (int m = 0; m < l.members; ++m)
#pragma unroll
            for (int k = 0; k < ADD_SLOTS; ++k) sum[k] += (double)__builtin_nontemporal_load(probs + m * e.probs_stride_row + at[k]);
#pragma unroll
        for (int k = 0; k < ADD_SLOTS; ++k) {
            const int j = first + k * ADD_THREADS;
            if (j >= len) continue;
            const float score = (float)sum[k];
            const int64_t place = e.positions[row + j];
            const bool stays = place < e.sinks || place >= (int64_t)next - e.recent;
            e.scores_out[row + j] = score;
            l.keys[(int64_t)r * e.n_max + j] = stays ? KEY_STAYS : key_of(score);
        }
    }
}

struct Pick {
    uint32_t bins[2048];
    int wave_sum[PICK_WAVES][4];                              // above / equal to the K-th key, below / beyond the new length
    int found[2];
};

// The bin that holds the K-th largest of the counted entries, and how many lie above it.  Called by all threads.
__device__ __forceinline__ void locate(Pick &s, int bins, int K, int &bin, int &above)
{
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    __syncthreads();
    if (wave == 0) {                                          // lane i holds the i-th highest run of bins
        const int run = bins / 64, top = bins - 1 - lane * run;
        int mine = 0;
        for (int i = 0; i < run; ++i) mine += s.bins[top - i];
        const int upto = wave_inclusive_sum(mine);
        if (upto - mine < K && K <= upto) {
            int over = upto - mine;
            for (int i = 0; i < run; ++i) {
                const int c = s.bins[top - i];
                if (over + c >= K) { s.found[0] = top - i; s.found[1] = over; break; }
                over += c;
            }
        }
    }
    __syncthreads();
    bin = s.found[0];
    above = s.found[1];
}

// One workgroup per row.
__global__ __launch_bounds__(PICK_THREADS) void evict_pick_kernel(EvictLaunch l)
{
    __shared__ Pick s;
    const specattn_evict_args &e = l.e;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    for (int r = blockIdx.x; r < e.B * e.H; r += gridDim.x) {
        const int b = r / e.H, h = r - b * e.H, len = row_length(e, b), K = min(len, e.budget);
        const int64_t row = b * e.row_stride_b + h * e.row_stride_h;
        const uint32_t *keys = l.keys + (int64_t)r * e.n_max;
        float *scores = e.scores_out + row;
        const int32_t *from = e.positions + row;
        int32_t *to = e.positions_out + row;
        int32_t *src = e.move_src + r * e.move_stride_row, *dst = e.move_dst + r * e.move_stride_row;
        if (tid == 0 && h == 0) e.new_lens[b] = K;
        if (e.row_flags) {
            int bad = 0;
            for (int j = tid; j < len; j += PICK_THREADS) bad |= scores[j] != scores[j];
            bad = __syncthreads_or(bad);
            if (tid == 0) e.row_flags[r] = bad ? SPECATTN_ROW_INVALID : 0u;
        }
        if (len == K) {                                       // nothing leaves
            if (tid == 0) e.move_counts[r] = 0;
            if (from != to) for (int j = tid; j < len; j += PICK_THREADS) to[j] = from[j];
            continue;
        }
        // The K-th largest key: 11, 11 and 10 bits at a time.
        uint32_t prefix = 0;
        int need = K;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < bins; i += PICK_THREADS) s.bins[i] = 0;
            __syncthreads();
            for (int j = tid; j < len; j += PICK_THREADS) {
                const uint32_t key = keys[j];
                if (pass == 0 || (key >> (shift + (pass == 2 ? 10 : 11))) == prefix) atomicAdd(&s.bins[(key >> shift) & (bins - 1)], 1u);
            }
            int bin, above;
            locate(s, bins, need, bin, above);
            prefix = (prefix << (pass == 2 ? 10 : 11)) | (uint32_t)bin;
            need -= above;
        }
        const uint32_t cut = prefix;                          // kept: every key above it, and the first `need` that equal it
        // Each wave takes a run of the row.
        const int run = ((len + PICK_WAVES - 1) / PICK_WAVES + 63) & ~63, j0 = min(wave * run, len), j1 = min(j0 + run, len);
        int above_l = 0, equal_l = 0, above_r = 0, equal_r = 0;
        for (int j = j0; j < j1; j += 64) {
            const uint32_t key = j + lane < j1 ? keys[j + lane] : 0;
            const bool in = j + lane < j1;
            const uint64_t below = __ballot(j + lane < K), above = __ballot(in && key > cut), equal = __ballot(in && key == cut);
            above_l += __popcll(above & below);
            equal_l += __popcll(equal & below);
            above_r += __popcll(above & ~below);
            equal_r += __popcll(equal & ~below);
        }
        if (lane == 0) {
            s.wave_sum[wave][0] = above_l; s.wave_sum[wave][1] = equal_l;
            s.wave_sum[wave][2] = above_r; s.wave_sum[wave][3] = equal_r;
        }
        __syncthreads();
        int equals = 0, hole = 0, mover = 0, all_movers = 0;  // ahead of this wave's run; of the row
        int my_equals = 0, my_hole = 0, my_mover = 0;
        for (int w = 0; w < PICK_WAVES; ++w) {
            if (w == wave) { my_equals = equals; my_hole = hole; my_mover = all_movers; }
            const int w0 = min(w * run, len), w1 = min(w0 + run, len);
            const int ties_l = min(max(need - equals, 0), s.wave_sum[w][1]);
            const int ties_r = min(max(need - equals - s.wave_sum[w][1], 0), s.wave_sum[w][3]);
            hole += max(min(w1, K) - w0, 0) - s.wave_sum[w][0] - ties_l;
            all_movers += s.wave_sum[w][2] + ties_r;
            equals += s.wave_sum[w][1] + s.wave_sum[w][3];
        }
        equals = my_equals; hole = my_hole; mover = my_mover;
        const uint64_t before = ((uint64_t)1 << lane) - 1;
        for (int j = j0; j < j1; j += 64) {
            const bool in = j + lane < j1;
            const uint32_t key = in ? keys[j + lane] : 0;
            const uint64_t equal = __ballot(in && key == cut);
            const bool kept = in && (key > cut || (key == cut && equals + __popcll(equal & before) < need));
            const bool low = j + lane < K;
            const uint64_t holes = __ballot(in && low && !kept), movers = __ballot(in && !low && kept);
            if (in && low && !kept) dst[hole + __popcll(holes & before)] = j + lane;
            if (in && !low && kept) src[mover + __popcll(movers & before)] = j + lane;
            if (kept && low && from != to) to[j + lane] = from[j + lane];
            hole += __popcll(holes);
            mover += __popcll(movers);
            equals += __popcll(equal);
        }
        if (tid == 0) e.move_counts[r] = all_movers;
        __syncthreads();
        for (int i = tid; i < all_movers; i += PICK_THREADS) {
            const int a = src[i], d = dst[i];
            scores[d] = scores[a];
            to[d] = from[a];
        }
        __syncthreads();
        for (int j = K + tid; j < len; j += PICK_THREADS) { scores[j] = 0.0f; to[j] = -1; }
        __syncthreads();                                      // (the bins are used again)
    }
}

struct MoveLaunch {
    specattn_move_args m;
    int page_shift;
    int unit_shift[SPECATTN_MAX_PLANES];                      // log2 of the bytes moved at a time
    FastDivisor per_row[SPECATTN_MAX_PLANES];                 // by the units of a row
};

constexpr int MOVE_THREADS = 256, MOVE_ITEMS = 4;

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

template <typename V> __device__ __forceinline__ void move_rows(const MoveLaunch &l, const specattn_move_plane &p, const FastDivisor &per_row, int units)
{
    const int share = p.H_kv / l.m.H, all = l.m.B * p.H_kv;
    uint8_t *data = static_cast<uint8_t *>(p.data);
    for (int y = blockIdx.y; y < all; y += gridDim.y) {
        const int b = y / p.H_kv, kv = y - b * p.H_kv, r = b * l.m.H + kv / share;
        const int items = min(max(l.m.move_counts[r], 0), l.m.move_capacity) * units;
        const int first = blockIdx.x * MOVE_THREADS * MOVE_ITEMS + threadIdx.x;
        if (first >= items) continue;
        V value[MOVE_ITEMS];
        int64_t from, to[MOVE_ITEMS];
        bool there[MOVE_ITEMS];
#pragma unroll
        for (int k = 0; k < MOVE_ITEMS; ++k) {
            const int item = first + k * MOVE_THREADS;
            there[k] = false;
            if (item >= items) continue;
            const int i = per_row.divide(item), u = item - i * units;
            const int64_t list = r * l.m.move_stride_row + i;
            there[k] = move_offset(l, p, b, kv, l.m.move_src[list], from) && move_offset(l, p, b, kv, l.m.move_dst[list], to[k]);
            to[k] += u * (int)sizeof(V);
            if (there[k]) value[k] = __builtin_nontemporal_load(reinterpret_cast<const V *>(data + from + u * (int)sizeof(V)));
        }
#pragma unroll
        for (int k = 0; k < MOVE_ITEMS; ++k) if (there[k]) *reinterpret_cast<V *>(data + to[k]) = value[k];
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

size_t evict_workspace_bytes(const specattn_evict_args *e)
{
    return ((size_t)e->B * e->H * e->n_max * sizeof(uint32_t) + 255) & ~(size_t)255;
}

specattn_status launch_evict_select(const specattn_evict_args *e, void *workspace, hipStream_t stream)
{
    EvictLaunch l;
    l.e = *e;
    l.keys = static_cast<uint32_t *>(workspace);
    l.members = e->probs ? e->H_draft / e->H * e->S : 0;
    const int rows = e->B * e->H;
    evict_add_kernel<<<dim3((e->n_max + ADD_THREADS * ADD_SLOTS - 1) / (ADD_THREADS * ADD_SLOTS), std::min(rows, 65535)), ADD_THREADS, 0, stream>>>(l);
    const specattn_status st = check_launch("evict_add_kernel");
    if (st != SPECATTN_OK) return st;
    evict_pick_kernel<<<rows, PICK_THREADS, 0, stream>>>(l);
    return check_launch("evict_pick_kernel");
}

specattn_status launch_evict_move(const specattn_move_args *m, hipStream_t stream)
{
    MoveLaunch l;
    l.m = *m;
    l.page_shift = 0;
    while (m->page_table && (1 << l.page_shift) < m->page_size) ++l.page_shift;
    int64_t most = 0;
    int rows = 0;
    for (int z = 0; z < m->num_planes; ++z) {
        const int bytes = m->planes[z].row_bytes;
        l.unit_shift[z] = bytes % 16 == 0 ? 4 : bytes % 8 == 0 ? 3 : 2;
        l.per_row[z] = FastDivisor(bytes >> l.unit_shift[z]);
        most = std::max(most, (int64_t)m->move_capacity * (bytes >> l.unit_shift[z]));
        rows = std::max(rows, m->B * m->planes[z].H_kv);
    }
    const int per = MOVE_THREADS * MOVE_ITEMS;
    evict_move_kernel<<<dim3((int)((most + per - 1) / per), std::min(rows, 65535), m->num_planes), MOVE_THREADS, 0, stream>>>(l);
    return check_launch("evict_move_kernel");
}

}  // namespace specattn
