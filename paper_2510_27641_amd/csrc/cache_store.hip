// Rows of keys and values into the slots of a cache: the rows of prompts, and the accepted nodes of drafted trees.
//
// Bound by memory: every byte is read once and written once.  A thread moves 16 bytes of a key row and of the value row beside it, for four
// such pieces that it asks for together.
//
// 131072 rows of 8 heads by 128 in fp16 (537 MB of keys and values read and as much written): 108 us, 4.95 TB/s, where a copy of 1 GiB reaches 5.17.  The
// accepted nodes of 64 trees, 1.8 MB: 4.2 to 4.7 us, a launch and two dependent trips to memory.
#include "serve.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int THREADS = 256;
constexpr int PIECES = 4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct StoreArgs {
    const char *k, *v;
    char *k_cache, *v_cache;
    const int32_t *slots, *rows;
    int64_t b, t, h;                                          // bytes, of k and v
    int64_t page, n, head;                                    // bytes, of the caches
    FastDivisor per_row, per_head, per_t, per_page;           // by the pieces of a row of all heads and of one head, by T, by the page size
    int pieces, head_pieces, T, page_size, num_pages;
    int64_t num_rows;
    int first, items;                                         // pieces of this launch: slots from `first` on
};

__global__ __launch_bounds__(THREADS) void store_kernel(StoreArgs a)
{
    const char *from[PIECES];
    int64_t to[PIECES];
    u32x4 k[PIECES], v[PIECES];
    const int base = blockIdx.x * (THREADS * PIECES) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int item = base + i * THREADS;
        to[i] = -1;
        if (item >= a.items) continue;
        const int token = a.per_row.divide(item), piece = item - token * a.pieces;
        const int head = a.per_head.divide(piece), at = (piece - head * a.head_pieces) * 16;
        const int slot = a.slots[a.first + token], row = a.rows ? a.rows[a.first + token] : a.first + token;
        if (slot < 0 || row < 0 || row >= a.num_rows) continue;
        const int page = a.per_page.divide(slot), b = a.per_t.divide(row);
        if (page >= a.num_pages) continue;
        to[i] = page * a.page + (slot - page * a.page_size) * a.n + head * a.head + at;
        from[i] = a.k + (b * a.b + (row - b * a.T) * a.t + head * a.h + at);
        k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from[i]));
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.v + (from[i] - a.k)));
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        if (to[i] < 0) continue;
        *reinterpret_cast<u32x4 *>(a.k_cache + to[i]) = k[i];
        *reinterpret_cast<u32x4 *>(a.v_cache + to[i]) = v[i];
    }
}

}  // namespace

specattn_status launch_store(const specattn_store_args *s, hipStream_t stream)
{
    const int es = s->dtype == SPECATTN_F32 ? 4 : 2;
    StoreArgs a{};
    a.k = static_cast<const char *>(s->k); a.v = static_cast<const char *>(s->v);
    a.k_cache = static_cast<char *>(s->k_cache); a.v_cache = static_cast<char *>(s->v_cache);
    a.slots = s->slots; a.rows = s->rows;
    a.b = s->stride_b * es; a.t = s->stride_t * es; a.h = s->stride_h * es;
    a.page = s->cache_stride_page * es; a.n = s->cache_stride_n * es; a.head = s->cache_stride_h * es;
    a.head_pieces = s->d * es / 16;
    a.pieces = a.head_pieces * s->H_kv;
    a.per_row = FastDivisor(a.pieces); a.per_head = FastDivisor(a.head_pieces); a.per_t = FastDivisor(s->T); a.per_page = FastDivisor(s->page_size);
    a.T = s->T; a.page_size = s->page_size; a.num_pages = s->num_pages;
    a.num_rows = (int64_t)s->B * s->T;
    const int most = (1 << 30) / a.pieces;                    // slots of a launch: its pieces are counted in 31 bits
    for (int64_t first = 0; first < s->num_slots; first += most) {
        a.first = (int)first;
        a.items = (int)std::min<int64_t>(most, s->num_slots - first) * a.pieces;
        store_kernel<<<(a.items + THREADS * PIECES - 1) / (THREADS * PIECES), THREADS, 0, stream>>>(a);
        const specattn_status st = check_launch("store_kernel");
        if (st != SPECATTN_OK) return st;
    }
    return SPECATTN_OK;
}

}  // namespace specattn
