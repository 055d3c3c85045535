// Sparse decode attention (Section 3.1.2, Eq. 2-3; Section 3.5) over a cache in 4 bits, d = 128 or 64, up to 64 query rows
// per kv head and launch.
//
// Work split: the attended positions of all rows, in tiles of 32, form one line; the line is cut into equal shares, one per
// workgroup of eight waves (one per CU).  A share that crosses row boundaries yields one partial (m, l, o) per (row, share)
// in slot share + row; mx_merge_kernel combines a row's partials in share order.  Inside a share tile k goes to wave k mod 8,
// so every sum is taken in a fixed order.
//
// Per wave and tile, codes and scales go from memory straight into LDS (global_load_lds): d/16 lanes fetch the d bytes of a
// position as one piece, 1 KiB per instruction, and the list words and page numbers that tell where they lie come the same way, two and
// four tiles earlier.  A wave holds three tiles: one in use, two on their way, 68 KiB per CU at d = 128, and waits by the
// number of requests behind the ones it needs.  (Requests straight into registers, one tile ahead: a tile took as long as a trip
// to memory; 8 dense sequences of up to 32768 positions 45 us.)  From LDS,
//   keys     lane (p, g) = (lane % 16, lane / 16) takes a quarter of the codes of positions p and 16 + p, d/4 elements that lie
//            in one block, so one scale serves all of a lane's conversions.  The contraction runs over the elements in the order
//            the lanes hold them; the queries are laid out to match.
//   values   lane (c, g) takes d/16 consecutive elements of the eight positions 4g .. 4g+3 and 16+4g .. 16+4g+3: what a
//            column tile of the second product needs of those positions, for d/16 column tiles
//   S^T = K Q^T, O^T += V^T P^T on mfma 16x16x32 in bf16.  The codes times their scales are exact in bf16, bf16 queries are
//   exact, fp16 queries go in two exact parts.  The first product leaves the weights of a query in the lanes that hold the
//   values' positions, so weights never leave their lane.  A weight goes in three bf16 parts, 24 significant bits: two leave 2^-17 of
//   it, more than the fp32 sums do.
// (The matrix instructions that take 4-bit operands and scales directly, with the queries in two 8-bit parts, measured 2e-5 of
// the sum of magnitudes on random operands, far from fp32: their sums are aligned in few bits.)
#include "mx.h"

#include <algorithm>
#include <mutex>

namespace specattn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int NW = 8;                     // waves per workgroup
constexpr int THREADS = NW * 64;
constexpr int TILE = 32;                  // positions per tile
constexpr int MAX_ROWS = 1024;            // rows per launch: two to a thread
constexpr int SEG_COST = 6;               // cost of picking a row up, in tiles
constexpr int PARTS = 3;                  // bf16 parts of a weight
constexpr float RANGE = 8.0f;             // weights are taken in units of 2^ref; ref moves when one exceeds 2^RANGE

template <int D> struct Geo {
    static constexpr int KW = D / 32;     // words of key codes per lane and position: k-steps of the first product
    static constexpr int DT = D / 16;     // column tiles of the output, and value elements per lane and position
    static constexpr int PITCH = D + 4;   // floats of a row in the merge buffer
    static constexpr int LPR = D / 16;    // lanes that fetch the codes of one position
    static constexpr int RPI = 64 / LPR;  // positions per instruction
    static constexpr int CI = TILE / RPI; // instructions per tile: position CI * j + k is the j-th of instruction k
    static constexpr int CODES = TILE * D;
    // 16-byte piece c of the codes of position `pos` lies in place c ^ swz(pos), so that both reads spread over all banks: keys, one piece
    // of each of 16 positions, and values, 64 (32) bytes of the positions 4g + i of four g.
    static __device__ __forceinline__ int swz(int pos) { return D == 128 ? (pos & 3) | ((pos >> 3 & 1) << 2) : (pos & 1) | (pos >> 3 & 1) << 1; }
    static __device__ __forceinline__ int piece(int pos, int c) { return (pos % CI) * 1024 + (pos / CI) * D + ((c ^ swz(pos)) * 16); }
};

constexpr int DEPTH = 3;                  // tiles of a wave: in use and on their way

// A wave's part of the LDS.
template <int D> struct WaveLds {
    uint8_t codes[DEPTH][Geo<D>::CODES];
    uint32_t scales[DEPTH][64];           // d = 128: of the keys of the 32 positions, then of the values; d = 64: of both
    uint32_t words[DEPTH][64];            // list words
    int32_t pages[DEPTH][64];             // page numbers
    uint32_t codes_at[TILE];              // row offsets of the tile that is requested next
};

template <int D> struct MergeLds {
    float o[NW][16][Geo<D>::PITCH];
    float ml[NW][16][2];
};

template <int D, int NQ, int QP> struct Lds {
    static constexpr bool Q = NQ * QP > 2;                                    // queries wait in LDS, else in registers
    static constexpr int Q_BYTES = Q ? NQ * QP * Geo<D>::KW * 1024 : 16;
    union {
        WaveLds<D> wave[NW];
        MergeLds<D> merge;
    };
    uint8_t q[Q_BYTES] __attribute__((aligned(16)));
    int prefix[MAX_ROWS + 1];
    int count[MAX_ROWS];
    int red[2][NW];
};
static_assert(sizeof(Lds<128, 4, 2>) <= 160 * 1024, "a workgroup must fit a CU's LDS");

// Requests 16 or 4 bytes per lane from `src` to `to` + 16 or 4 * lane in LDS.  Counts as one request of the wave in order; nobody but
// wait_requests waits for it.
__device__ __forceinline__ void request16(const void *src, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(src), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void request4(const void *src, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(to) : "memory", "m0");
}
// Waits until at most N of the wave's requests are under way.
template <int N> __device__ __forceinline__ void wait_requests() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds_offset(const void *p) { return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p); }

__device__ __forceinline__ uint32_t bits(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ uint32_t to_bf16(float a, float b) { return bits(__builtin_convertvector(f32x2{a, b}, bf16x2)); }
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ f32x4 mfma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
{
    const u32x4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// Elements 2B and 2B + 1 of eight codes.  (The conversion takes a scale's exponent alone.)
template <int B> __device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale) { return bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B)); }
__device__ __forceinline__ float shuffle_xor(float x, int mask) { return __shfl_xor(x, mask, 64); }

// Reduction over a workgroup: sums of a and b.
__device__ __forceinline__ void sum_two(int a, int b, int (&red)[2][NW], int &ta, int &tb)
{
    const int wave = threadIdx.x / 64;
    a = __builtin_amdgcn_readlane(wave_inclusive_sum(a), 63);
    b = __builtin_amdgcn_readlane(wave_inclusive_sum(b), 63);
    if (threadIdx.x % 64 == 0) { red[0][wave] = a; red[1][wave] = b; }
    __syncthreads();
    ta = tb = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) { ta += red[0][w]; tb += red[1][w]; }
}

struct Share { int size, head; };         // units of the line per workgroup, and ahead of a row's tiles

template <int D, int NQ, int QP> __global__ __launch_bounds__(THREADS) void mx_attn_kernel(MxAttnLaunch p, int row0, int rows, int heads)
{
    typedef Geo<D> G;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds_bytes[];
    Lds<D, NQ, QP> &lds = *reinterpret_cast<Lds<D, NQ, QP> *>(lds_bytes);
    const AttnLaunch &a = p.a;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, low = lane % 16, g = lane / 16;
    const int me = blockIdx.x;

    // The line: every workgroup works it out for itself.
    int cnt[2], tiles = 0, filled = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 2 * tid + i;
        cnt[i] = r < rows ? attn_row_count(a, row0 + r, p.per_h.divide(row0 + r)) : 0;
        lds.count[r] = cnt[i];
        tiles += (cnt[i] + TILE - 1) / TILE;
        filled += cnt[i] > 0;
    }
    int all_tiles, all_rows;
    sum_two(tiles, filled, lds.red, all_tiles, all_rows);
    const int W = gridDim.x;
    // Few tiles: shares of 8, 16, 24 or 32 tiles, each of one row, so that no workgroup has to pick up a second one.
    Share share = {0, 0};
    if (all_rows < W) {
        const int least = (all_tiles + W - all_rows - 1) / (W - all_rows);
        const int size = max((least + NW - 1) / NW, 1) * NW;
        if (size <= 4 * NW) share.size = size;
    }
    const bool whole = share.size > 0;
    if (!whole) { share.head = SEG_COST; share.size = (all_tiles + SEG_COST * all_rows + W - 1) / W; }
    int cost[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = (cnt[i] + TILE - 1) / TILE;
        cost[i] = t == 0 ? 0 : whole ? (t + share.size - 1) / share.size * share.size : t + SEG_COST;
    }
    __syncthreads();                                              // (red is used again)
    const int upto = wave_inclusive_sum(cost[0] + cost[1]);
    if (lane == 63) lds.red[0][wave] = upto;
    __syncthreads();
    int before = upto - cost[0] - cost[1];
    for (int w = 0; w < wave; ++w) before += lds.red[0][w];
    lds.prefix[2 * tid] = before;
    lds.prefix[2 * tid + 1] = before + cost[0];
    if (tid == THREADS - 1) lds.prefix[MAX_ROWS] = before + cost[0] + cost[1];
    __syncthreads();

    const int total = lds.prefix[MAX_ROWS];
    int u = me * share.size;
    const int u_end = min(u + share.size, total);
    if (u >= u_end) return;
    int r = 0;                                                    // the row that holds unit u
    {
        int lo = 0, hi = MAX_ROWS;                                // prefix[lo] <= u < prefix[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (lds.prefix[mid] <= u) lo = mid; else hi = mid;
        }
        r = lo;
    }
    uint16_t *row_parts = static_cast<uint16_t *>(a.workspace);                // [rows][2]: first and last share of a row
    float *slots = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + (((size_t)rows * 4 + 255) & ~(size_t)255));
    const int queries = heads * a.T;
    const float to_log2 = a.sm_scale * 1.44269504088896340736f;

    for (; u < u_end; u = lds.prefix[r + 1], ++r) {
        const int row_start = lds.prefix[r], n = lds.count[r], row_tiles = (n + TILE - 1) / TILE;
        const int t0 = max(0, u - row_start - share.head), t1 = min(row_tiles, u_end - row_start - share.head);
        if (t1 <= t0) continue;                                   // (an empty row, or the share ends ahead of the row's first tile)
        const int row = row0 + r, b = p.per_h.divide(row), h = row - b * a.H_kv;

        // queries: element j of k-step s in lane (q, g) is element (d/4) g + 8 s + j of query 16 qt + q
        uint32_t qf[Lds<D, NQ, QP>::Q ? 1 : NQ * QP][G::KW][4];
        {
            auto fetch = [&](int qt, int s, uint32_t (&part)[QP][4]) {
                const int i = qt * 16 + low, gh = p.per_t.divide(i), t = i - gh * a.T;
                u32x4 w = {0, 0, 0, 0};
                if (i < queries)
                    w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + b * a.q_stride_b + (int64_t)(h * (a.H_q / a.H_kv) + a.g_first + gh) * a.q_stride_h
                                                        + t * a.q_stride_t + (D / 4) * g + 8 * s);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (QP == 1) part[0][k] = w[k];
                    else {
                        const float x = (float)__builtin_bit_cast(_Float16, (uint16_t)w[k]), y = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[k] >> 16));
                        part[0][k] = to_bf16(x, y);
                        part[1][k] = to_bf16(x - low_half(part[0][k]), y - high_half(part[0][k]));
                    }
                }
            };
            if constexpr (Lds<D, NQ, QP>::Q) {
                for (int k = wave; k < NQ * G::KW; k += NW) {
                    uint32_t part[QP][4];
                    fetch(k / G::KW, k % G::KW, part);
#pragma unroll
                    for (int q = 0; q < QP; ++q) *reinterpret_cast<u32x4 *>(lds.q + ((q * NQ * G::KW + k) * 64 + lane) * 16) = u32x4{part[q][0], part[q][1], part[q][2], part[q][3]};
                }
                __syncthreads();
            } else {
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
                    for (int s = 0; s < G::KW; ++s) {
                        uint32_t part[QP][4];
                        fetch(qt, s, part);
#pragma unroll
                        for (int q = 0; q < QP; ++q)
#pragma unroll
                            for (int k = 0; k < 4; ++k) qf[q * NQ + qt][s][k] = part[q][k];
                    }
            }
        }

        f32x4 acc[NQ][G::DT];
        float ref[NQ], sum[NQ];
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            ref[qt] = -INFINITY;
            sum[qt] = 0.0f;
#pragma unroll
            for (int t = 0; t < G::DT; ++t) acc[qt][t] = f32x4{0, 0, 0, 0};
        }

        const int32_t *list = a.dense ? nullptr : a.indices + (int64_t)row * a.idx_stride;
        const int32_t *pages = p.c.page_table ? p.c.page_table + (int64_t)b * p.c.max_pages : nullptr;
        const bool paged = pages || a.indices_are_physical;
        const uint8_t *codes = p.c.codes + (paged ? 0 : b * p.c.codes_b) + h * p.c.codes_h;
        const uint8_t *scales = p.c.scales + (paged ? 0 : b * p.c.scales_b) + h * p.c.scales_h;
        const uint32_t codes_n = (uint32_t)(p.c.codes_n >> 4), scales_n = (uint32_t)(p.c.scales_n >> 2);
        const uint32_t codes_page = (uint32_t)(p.c.codes_page >> 4), scales_page = (uint32_t)(p.c.scales_page >> 2);
        const int last_slot = a.indices_are_physical ? INT32_MAX : a.n_max - 1;

        // A tile goes through three steps, each two tiles ahead of the next: its list words are requested; its pages; its codes and
        // scales.  Tiles are counted per wave: the wave's tile i is tile t0 + wave + i * NW of the row.  (Tiles past the share's end are
        // requested like others, clamped to the row, and not used.)
        WaveLds<D> &mine = lds.wave[wave];
        const uint32_t codes_lds = lds_offset(mine.codes), scales_lds = lds_offset(mine.scales), words_lds = lds_offset(mine.words), pages_lds = lds_offset(mine.pages);
        const bool listed = !a.dense, looked_up = pages != nullptr;
        const int base_tile = t0 + wave;
        auto list_rank = [&](int i) { return min((base_tile + i * NW) * TILE + lane % TILE, n - 1); };
        auto list_at = [&](int i) { return list + (list_rank(i) >> a.chunk_shift); };
        auto slot_of = [&](int i, int word) -> int {
            if (!listed) return list_rank(i);                     // (below the length: inside the cache)
            if (a.chunk_shift) word = (word << a.chunk_shift) | (list_rank(i) & ((1 << a.chunk_shift) - 1));
            return min(max(word, 0), last_slot);
        };
        auto request_words = [&](int i, int at) { if (listed) request4(list_at(i), words_lds + at * 256); };
        auto request_pages = [&](int slot, int at) { if (looked_up) request4(pages + (slot >> a.page_shift), pages_lds + at * 256); };
        auto request_codes = [&](int slot, int page, int at) {
            uint32_t in = (uint32_t)slot;
            if (paged) {
                if (!looked_up) page = slot >> a.page_shift;
                page = min(max(page, 0), p.c.num_pages - 1);
                in &= (1u << a.page_shift) - 1;
            } else page = 0;
            mine.codes_at[lane % TILE] = in * codes_n + (uint32_t)page * codes_page;
            const uint8_t *from = scales + ((uint64_t)(in * scales_n + (uint32_t)page * scales_page) << 2) + (D == 128 ? lane / 32 * 4 : 0);
            uint32_t off[G::CI];
#pragma unroll
            for (int k = 0; k < G::CI; ++k) off[k] = mine.codes_at[lane / G::LPR * G::CI + k];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (what was read of the buffer that is written now has arrived)
#pragma unroll
            for (int k = 0; k < G::CI; ++k)
                request16(codes + ((uint64_t)off[k] << 4) + ((lane % G::LPR) ^ G::swz(lane / G::LPR * G::CI + k)) * 16, codes_lds + at * G::CODES + k * 1024);
            request4(from, scales_lds + at * 256);
        };
        auto use = [&](int at, int t) {
            const uint8_t *codes_in = mine.codes[at];
            const uint8_t *scales_in = reinterpret_cast<const uint8_t *>(mine.scales[at]);
            f32x4 s[NQ][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float scale = scale_of(scales_in[4 * (16 * i + low) + (D == 128 ? g : g / 2)]);
                uint32_t key_codes[G::KW];
                if constexpr (D == 128) {
                    const u32x4 w = *reinterpret_cast<const u32x4 *>(codes_in + G::piece(16 * i + low, g));
#pragma unroll
                    for (int k = 0; k < 4; ++k) key_codes[k] = w[k];
                } else {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(codes_in + G::piece(16 * i + low, g / 2) + g % 2 * 8);
                    key_codes[0] = w[0];
                    key_codes[1] = w[1];
                }
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) s[qt][i] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < G::KW; ++k) {
                    const uint32_t w = key_codes[k];
                    const uint32_t key[4] = {pair_of<0>(w, scale), pair_of<1>(w, scale), pair_of<2>(w, scale), pair_of<3>(w, scale)};
#pragma unroll
                    for (int q = 0; q < QP * NQ; ++q) {
                        if constexpr (Lds<D, NQ, QP>::Q) {
                            const u32x4 v = *reinterpret_cast<const u32x4 *>(lds.q + ((q * G::KW + k) * 64 + lane) * 16);
                            const uint32_t f[4] = {v[0], v[1], v[2], v[3]};
                            s[q % NQ][i] = mfma(key, f, s[q % NQ][i]);
                        } else s[q % NQ][i] = mfma(key, qf[q][k], s[q % NQ][i]);
                    }
                }
            }
            const int left = n - t * TILE;
            if (left < TILE) {                                    // a row's last tile: what lies behind it repeats its last position
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int qt = 0; qt < NQ; ++qt) s[qt][i][k] = 16 * i + 4 * g + k < left ? s[qt][i][k] : -INFINITY;
            }
            uint32_t w[NQ][PARTS][4];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
                __builtin_amdgcn_sched_barrier(0);
                float most = -INFINITY;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) { s[qt][i][k] *= to_log2; most = fmaxf(most, s[qt][i][k]); }
                if (__any(most > ref[qt] + RANGE)) {
                    most = fmaxf(most, shuffle_xor(most, 16));
                    most = fmaxf(most, shuffle_xor(most, 32));
                    const float now = fmaxf(ref[qt], most), shrink = __builtin_amdgcn_exp2f(ref[qt] - now);
                    const float factor = ref[qt] == -INFINITY ? 0.0f : shrink;
                    ref[qt] = now;
                    sum[qt] *= factor;
#pragma unroll
                    for (int d = 0; d < G::DT; ++d) acc[qt][d] *= factor;
                }
                float e[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    e[k] = __builtin_amdgcn_exp2f(s[qt][k / 4][k % 4] - ref[qt]);
                    sum[qt] += e[k];
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x0 = e[2 * k], x1 = e[2 * k + 1];
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        w[qt][part][k] = to_bf16(x0, x1);
                        if (part + 1 < PARTS) { x0 -= low_half(w[qt][part][k]); x1 -= high_half(w[qt][part][k]); }
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            uint32_t v[8];
            float scale[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 four = *reinterpret_cast<const u32x4 *>(scales_in + (D == 128 ? 128 : 0) + 4 * (16 * i + 4 * g));
                const int block = D == 128 ? low / 4 : 2 + low / 8;        // byte of a position's word
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int pos = 16 * i + 4 * g + j;
                    scale[4 * i + j] = __uint_as_float(__builtin_amdgcn_alignbit(four[j], four[j], 8 * block + 9));    // the byte goes to the exponent's place
                    const uint8_t *src = codes_in + G::piece(pos, D == 128 ? 4 + low / 4 : 2 + low / 8);
                    if constexpr (D == 128) v[4 * i + j] = *reinterpret_cast<const uint32_t *>(src + low % 4 * 4);
                    else v[4 * i + j] = *reinterpret_cast<const uint16_t *>(src + low % 8 * 2);
                }
            }
            auto columns = [&](auto which) {                      // elements 2B and 2B + 1 of the lane's eight (four)
                constexpr int B = decltype(which)::value;
                __builtin_amdgcn_sched_barrier(0);
                uint32_t even[4], odd[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t first = pair_of<B>(v[2 * j], scale[2 * j]), second = pair_of<B>(v[2 * j + 1], scale[2 * j + 1]);
                    even[j] = __builtin_amdgcn_perm(second, first, 0x05040100);
                    odd[j] = __builtin_amdgcn_perm(second, first, 0x07060302);
                }
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        acc[qt][2 * B] = mfma(even, w[qt][part], acc[qt][2 * B]);
                        acc[qt][2 * B + 1] = mfma(odd, w[qt][part], acc[qt][2 * B + 1]);
                    }
            };
            columns(std::integral_constant<int, 0>{});
            columns(std::integral_constant<int, 1>{});
            if constexpr (D == 128) {
                columns(std::integral_constant<int, 2>{});
                columns(std::integral_constant<int, 3>{});
            }
        };

        if (base_tile < t1) {
            int slot[2 * (DEPTH - 1)], page[DEPTH - 1] = {};
            static_assert(DEPTH == 3, "the requests below are two tiles apart");
            for (int i = 0; i < 4; ++i) slot[i] = slot_of(i, listed ? *list_at(i) : 0);
            if (looked_up) for (int i = 0; i < 2; ++i) page[i] = pages[slot[i] >> a.page_shift];
            for (int i = 0; i < 2; ++i) {
                request_codes(slot[i], page[i], i);
                request_pages(slot[2 + i], (2 + i) % DEPTH);
                request_words(4 + i, (4 + i) % DEPTH);
            }
            int ready = slot[2], next = slot[3], at = 0;          // slots of tiles i + 2 and i + 3; tile i lies in buffer `at`
            for (int i = 0, t = base_tile; t < t1; ++i, t += NW) {
                // all but what the last iteration requested
                constexpr int R = G::CI + 1;
                if (listed && looked_up) wait_requests<R + 2>();
                else if (listed || looked_up) wait_requests<R + 1>();
                else wait_requests<R>();
                const int prev = at == 0 ? DEPTH - 1 : at - 1, after = at == DEPTH - 1 ? 0 : at + 1;      // buffers of tiles i + 2, i + 1 (i + 4)
                const int word = listed ? (int)mine.words[after][lane] : 0, in_page = looked_up ? mine.pages[prev][lane] : 0;
                request_codes(ready, in_page, prev);
                ready = next;
                next = slot_of(i + 4, word);
                request_pages(next, after);
                request_words(i + 6, at);
                use(at, t);
                at = after;
            }
            wait_requests<0>();                                   // (the buffers are used for other things next)
        }
        __syncthreads();

        // The eight waves' states, one query tile at a time.
        const bool tail = a.k_new != nullptr, alone = t0 == 0 && t1 == row_tiles && !tail;
        float *slot_o = slots + (size_t)(me + r) * NQ * 16 * (D + 2), *slot_ml = slot_o + NQ * 16 * D;
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            float l = sum[qt];
            l += shuffle_xor(l, 16);
            l += shuffle_xor(l, 32);
            if (g == 0) { lds.merge.ml[wave][low][0] = ref[qt]; lds.merge.ml[wave][low][1] = l; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < G::DT; d += 4)
                    *reinterpret_cast<f32x4 *>(&lds.merge.o[wave][low][G::DT * (4 * g + i) + d]) = f32x4{acc[qt][d][i], acc[qt][d + 1][i], acc[qt][d + 2][i], acc[qt][d + 3][i]};
            __syncthreads();
            const int q = tid / (D / 4), at = tid % (D / 4) * 4;
            if (q < 16) {
                float top = -INFINITY, all = 0.0f, m[NW];
#pragma unroll
                for (int w = 0; w < NW; ++w) { m[w] = lds.merge.ml[w][q][0]; top = fmaxf(top, m[w]); }
                f32x4 o = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float f = m[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[w] - top);
                    all += f * lds.merge.ml[w][q][1];
                    o += f * *reinterpret_cast<const f32x4 *>(&lds.merge.o[w][q][at]);
                }
                const int i = qt * 16 + q;
                if (!alone) {
                    *reinterpret_cast<f32x4 *>(slot_o + i * D + at) = o;
                    if (at == 0) { slot_ml[2 * i] = top; slot_ml[2 * i + 1] = all; }
                } else if (i < queries) {
                    const int gh = p.per_t.divide(i), tq = i - gh * a.T;
                    const int64_t orow = ((int64_t)b * a.H_q + h * (a.H_q / a.H_kv) + a.g_first + gh) * a.T + tq;
                    o = o / all;
                    if (a.out) *reinterpret_cast<f32x4 *>(a.out + orow * D + at) = o;
                    if (a.out_lowp)
                        for (int k = 0; k < 4; ++k) st_lowp(a.out_lowp, orow * D + at + k, o[k], a.dtype);
                    if (a.lse && at == 0) a.lse[orow] = (top + __builtin_amdgcn_logf(all)) * 0.69314718055994530942f;
                }
            }
            __syncthreads();
        }
        if (tid == 0 && t0 == 0) row_parts[2 * r] = (uint16_t)me;
        if (tid == 0 && t1 == row_tiles) row_parts[2 * r + 1] = (uint16_t)me;
    }
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int k = 1; k < 64; k *= 2) x += shuffle_xor(x, k);
    return x;
}

// One wave per (row, query): the row's partials in share order, then the new tokens behind the cache up to the query's own.
template <int D> __global__ __launch_bounds__(256) void mx_merge_kernel(MxAttnLaunch p, int row0, int rows, int heads, int padded)
{
    constexpr int E = D / 64;                                     // elements per lane
    const AttnLaunch &a = p.a;
    const int lane = threadIdx.x % 64, queries = heads * a.T;
    const int r = blockIdx.y, i = blockIdx.x * 4 + threadIdx.x / 64;
    if (i >= queries) return;
    const int row = row0 + r, b = p.per_h.divide(row), h = row - b * a.H_kv;
    const uint16_t *row_parts = static_cast<const uint16_t *>(a.workspace);
    const float *slots = reinterpret_cast<const float *>(static_cast<const char *>(a.workspace) + (((size_t)rows * 4 + 255) & ~(size_t)255));
    const int gh = p.per_t.divide(i), t = i - gh * a.T, head = h * (a.H_q / a.H_kv) + a.g_first + gh;
    const int64_t orow = ((int64_t)b * a.H_q + head) * a.T + t;
    float m = -INFINITY, l = 0.0f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    if (attn_row_count(a, row, b) > 0) {
        const int first = row_parts[2 * r], last = row_parts[2 * r + 1];
        if (first == last && !a.k_new) return;                    // finished by its only workgroup
        for (int w = first; w <= last; ++w) {
            const float *slot = slots + (size_t)(w + r) * padded * (D + 2);
            const float mw = slot[padded * D + 2 * i], lw = slot[padded * D + 2 * i + 1];
            const float now = fmaxf(m, mw);
            const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now), fw = __builtin_amdgcn_exp2f(mw - now);
            l = l * f + lw * fw;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * f + slot[i * D + E * lane + e] * fw;
            m = now;
        }
    }
    if (a.k_new) {
        auto value = [&](const void *x, int64_t at) {
            const uint16_t w = static_cast<const uint16_t *>(x)[at];
            return a.dtype == SPECATTN_F16 ? (float)__builtin_bit_cast(_Float16, w) : __uint_as_float((uint32_t)w << 16);
        };
        float q[E];
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = value(a.q, b * a.q_stride_b + (int64_t)head * a.q_stride_h + t * a.q_stride_t + E * lane + e);
        for (int j = 0; j <= t; ++j) {
            const int64_t at = ((int64_t)row * a.T + j) * D + E * lane;
            float dot = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) dot += q[e] * value(a.k_new, at + e);
            const float s = wave_sum(dot) * (a.sm_scale * 1.44269504088896340736f), now = fmaxf(m, s);
            const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now), fw = __builtin_amdgcn_exp2f(s - now);
            l = l * f + fw;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * f + value(a.v_new, at + e) * fw;
            m = now;
        }
    }
    const bool any = l != 0.0f;                                   // (also where l is NaN)
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = any ? o[e] / l : 0.0f;
        if (a.out) a.out[orow * D + E * lane + e] = x;
        if (a.out_lowp) st_lowp(a.out_lowp, orow * D + E * lane + e, x, a.dtype);
    }
    if (a.lse && lane == 0) a.lse[orow] = any ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

template <int D, int NQ> const void *variant(bool f16)
{
    return f16 ? reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, 2>) : reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, 1>);
}
template <int D> const void *variant(int nq, bool f16)
{
    return nq == 1 ? variant<D, 1>(f16) : nq == 2 ? variant<D, 2>(f16) : nq == 3 ? variant<D, 3>(f16) : variant<D, 4>(f16);
}
const void *variant(int d, int nq, bool f16) { return d == 128 ? variant<128>(nq, f16) : variant<64>(nq, f16); }
template <int D, int NQ> size_t lds_size(bool f16) { return f16 ? sizeof(Lds<D, NQ, 2>) : sizeof(Lds<D, NQ, 1>); }
template <int D> size_t lds_size(int nq, bool f16) { return nq == 1 ? lds_size<D, 1>(f16) : nq == 2 ? lds_size<D, 2>(f16) : nq == 3 ? lds_size<D, 3>(f16) : lds_size<D, 4>(f16); }
size_t lds_size(int d, int nq, bool f16) { return d == 128 ? lds_size<128>(nq, f16) : lds_size<64>(nq, f16); }

// Query heads of a kv head per launch: groups of more than 64 query rows go out in equal parts.
int heads_per_launch(int G, int T)
{
    const int most = 64 / T, parts = (G + most - 1) / most;
    return (G + parts - 1) / parts;
}

}  // namespace

size_t mx_attn_workspace_bytes(int rows, int G, int T, int d)
{
    const int per = std::min(rows, MAX_ROWS), padded = (heads_per_launch(G, T) * T + 15) / 16 * 16;
    return (((size_t)per * 4 + 255) & ~(size_t)255) + (((size_t)(cu_count() + per) * padded * (d + 2) * sizeof(float) + 255) & ~(size_t)255);
}

specattn_status mx_attn_configure()
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
        const int d = k & 1 ? 128 : 64, nq = (k >> 1 & 3) + 1;
        const bool f16 = k & 8;
        if (hipFuncSetAttribute(variant(d, nq, f16), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_size(d, nq, f16)) != hipSuccess) {
            (void)hipGetLastError();
            set_error("cannot reserve %zu bytes of LDS", lds_size(d, nq, f16));
            return SPECATTN_EHIP;
        }
    }
    done[dev] = true;
    return SPECATTN_OK;
}

specattn_status launch_mx_attn(const MxAttnLaunch &l, hipStream_t stream)
{
    specattn_status st = mx_attn_configure();
    if (st != SPECATTN_OK) return st;
    const int rows = l.a.B * l.a.H_kv, G = l.a.H_q / l.a.H_kv, per = heads_per_launch(G, l.a.T);
    for (int first = 0; first < G; first += per) {
        const int heads = std::min(per, G - first), nq = (heads * l.a.T + 15) / 16;
        MxAttnLaunch part = l;
        part.a.g_first = first;
        part.per_h = FastDivisor(l.a.H_kv);
        part.per_t = FastDivisor(l.a.T);
        for (int row0 = 0; row0 < rows; row0 += MAX_ROWS) {
            int here = std::min(MAX_ROWS, rows - row0), at = row0, h = heads;
            void *args[] = {&part, &at, &here, &h};
            const bool f16 = l.a.dtype == SPECATTN_F16;
            if (hipLaunchKernel(variant(l.a.d, nq, f16), dim3(cu_count()), dim3(THREADS), args, lds_size(l.a.d, nq, f16), stream) != hipSuccess) return check_launch("mx_attn_kernel");
            st = check_launch("mx_attn_kernel");
            if (st != SPECATTN_OK) return st;
            const dim3 grid((heads * l.a.T + 3) / 4, here);
            if (l.a.d == 128) mx_merge_kernel<128><<<grid, 256, 0, stream>>>(part, row0, here, heads, nq * 16);
            else mx_merge_kernel<64><<<grid, 256, 0, stream>>>(part, row0, here, heads, nq * 16);
            st = check_launch("mx_merge_kernel");
            if (st != SPECATTN_OK) return st;
        }
    }
    return SPECATTN_OK;
}

}  // namespace specattn
