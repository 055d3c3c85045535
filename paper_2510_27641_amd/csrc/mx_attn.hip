// Sparse decode attention (Section 3.1.2, Eq. 2-3; Section 3.5) over a cache in 4 bits, d = 128 or 64, up to 64 query rows
// per kv head and launch.
//
// Work split: the attended positions of a row go in tiles of 32, and consecutive tiles to one share, a workgroup's work.  Inside a share
// tile k goes to wave k mod (waves), so every sum is taken in a fixed order.  A row in one share is finished there; otherwise each
// leaves a partial (m, l, o), o the average of its values, in slot share + row, and mx_merge_kernel combines a row's partials in share order.
//
// Per wave and tile, codes and scales go from memory straight into LDS (global_load_lds): d/16 lanes fetch the d bytes of a
// position as one piece, 1 KiB per instruction, and the list words and page numbers that tell where they lie come the same way, one trip
// each ahead.  A wave holds three tiles, one in use and two on their way (12 waves: two, one on its way), 68 (51) KiB under way per CU at d = 128, and
// waits by the number of requests behind the ones it needs.  (Requests straight into registers, one tile ahead: a tile took as long as a trip
// to memory; 8 dense sequences of up to 32768 positions 45 us / 39.)  From LDS,
//   keys     lane (p, g) = (lane % 16, lane / 16) takes a quarter of the codes of positions p and 16 + p, d/4 elements that lie
//            in one block, so one scale serves all of a lane's conversions.  The contraction runs over the elements in the order
//            the lanes hold them; the queries are laid out to match.
//   values   lane (c, g) takes d/16 consecutive elements of the eight positions 4g .. 4g+3 and 16+4g .. 16+4g+3: what a
//            column tile of the second product needs of those positions, for d/16 column tiles
//   S^T = K Q^T on mfma 16x16x32.  In bf16 codes times scales are exact, and so are bf16 queries.  fp16 queries are not: their keys go in
//   fp16, in units of the largest scale of a position, and scores are multiplied by it.  (Queries in two exact bf16 parts took twice the
//   matrix instructions: 64 sequences of 8 kv heads, 4 heads by 5 queries, up to 65536 positions, a third kept: 294 us / 250.)
//   O^T += V^T P^T in fp16: a weight goes in two parts, 22 significant bits (bf16 took three: a third more matrix and twice the vector
//   instructions), and the scales in units that follow the largest one of a block, since fp16 has not their range.  The first product
//   leaves the weights of a query in the lanes that hold the values' positions, so weights never leave their lane.
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
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Waves per workgroup, and tiles of a wave in use and on their way.  Up to 64 rows a workgroup has a CU to itself: 12 waves where registers
// allow it (one query tile; 8 dense sequences of up to 32768 positions 39 us / 44 with 8), else 8.  Beyond, two workgroups of 4 share it,
// so that one works while the other changes rows (64 sequences of 8 kv heads, two query tiles: 240 us / 250 with one of 8).
template <int NQ, bool FEW> struct Waves {
    static constexpr int N = !FEW ? 4 : NQ == 1 ? 12 : 8, DEPTH = N == 12 ? 2 : 3, THREADS = N * 64;
};
constexpr int TILE = 32;                  // positions per tile
constexpr int MAX_ROWS = 512;             // rows per launch: two for each thread
constexpr int SEG_COST = 10;              // cost of picking a row up, in tiles
constexpr int PARTS = 2;                  // fp16 parts of a weight
// Weights are taken in units of 2^ref.  ref puts the largest weight so far at 2^HEAD and moves when one exceeds 2^RANGE: fp16 ends at 2^16
// and, downwards, at 2^-24, so that a weight 2^-36 below the largest still counts.
constexpr float HEAD = 12.0f, RANGE = 15.0f;
// Values are taken in units of 2^(unit - 127), a byte per block that follows the largest scale of the wave's positions up.  Codes times
// scales are exact in fp16 down to 2^-FAR of that; values under smaller scales are rounded to multiples of 2^-24 of it.
constexpr int FAR = 22;

template <int D> struct Geo {
    static constexpr int KW = D / 32;     // words of key codes per lane and position: k-steps of the first product
    static constexpr int DT = D / 16;     // column tiles of the output, and value elements per lane and position
    static constexpr int PITCH = D + 4;   // floats of a row in the merge buffer
    static constexpr int LPR = D / 16;    // lanes that fetch the codes of one position
    static constexpr int RPI = 64 / LPR;  // positions per instruction
    static constexpr int CI = TILE / RPI; // instructions per tile: instruction k fetches positions RPI k, RPI k + 1, ...
    static constexpr int CODES = TILE * D;
    // 16-byte piece c of the codes of position `pos` lies in place c ^ swz(pos), so that both reads spread over all banks: keys, one piece
    // of each of 16 positions, and values, 64 (32) bytes of the positions 4g + i of four g.
    static __device__ __forceinline__ int swz(int pos) { return D == 128 ? (pos >> 1 & 3) | (pos >> 2 & 1) << 2 : pos >> 2 & 3; }
    static __device__ __forceinline__ int piece(int pos, int c) { return pos * D + ((c ^ swz(pos)) * 16); }
};

// A wave's part of the LDS.
template <int D, int DEPTH> struct WaveLds {
    uint8_t codes[DEPTH][Geo<D>::CODES];
    uint32_t scales[DEPTH][64];           // d = 128: of the keys of the 32 positions, then of the values; d = 64: of both
    uint32_t words[DEPTH][64];            // list words
    int32_t pages[DEPTH][64];             // page numbers
    uint32_t codes_at[TILE];              // row offsets of the tile that is requested next; position p in place p % RPI * CI + p / RPI
    float unit[TILE];                     // fp16 queries: largest scale of a position's keys, times what scores are scaled by
    uint32_t unit_byte[TILE];             // the same scale as a byte
};

template <int D, int NW> struct MergeLds {
    float o[NW][16][Geo<D>::PITCH];
    f32x4 ml[NW][16];                     // ref, the sum of weights over 2^e, 2^e (e: that sum's exponent; o is over 2^e as well)
};

template <int D, int NQ, bool FEW> struct Lds {
    static constexpr int NW = Waves<NQ, FEW>::N;
    static constexpr bool Q = NQ > 2;                                                   // queries wait in LDS, else in registers
    static constexpr int Q_BYTES = Q ? NQ * Geo<D>::KW * 1024 : 16;
    union {
        WaveLds<D, Waves<NQ, FEW>::DEPTH> wave[NW];
        MergeLds<D, NW> merge;
    };
    uint8_t q[Q_BYTES] __attribute__((aligned(16)));
    int prefix[MAX_ROWS + 1];
    int count[MAX_ROWS];
    int red[2][NW];
};
template <int D, int NQ> constexpr bool fits() { return sizeof(Lds<D, NQ, true>) <= 160 * 1024 && sizeof(Lds<D, NQ, false>) <= 80 * 1024; }
static_assert(fits<128, 1>() && fits<128, 2>() && fits<128, 3>() && fits<128, 4>() && fits<64, 1>() && fits<64, 2>() && fits<64, 3>() && fits<64, 4>(), "one workgroup, or two, must fit a CU's LDS");

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
__device__ __forceinline__ f32x4 mfma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
{
    const u32x4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c)
{
    const u32x4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}
// x less the low, the high half of w: exact where the half is x cut to fp16.
__device__ __forceinline__ float less_low(float x, uint32_t w)
{
    float y;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(w), "v"(x));
    return y;
}
__device__ __forceinline__ float less_high(float x, uint32_t w)
{
    float y;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(w), "v"(x));
    return y;
}
// Elements 2B and 2B + 1 of eight codes.  (The conversion takes a scale's exponent alone.)
__device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale, int B)
{
    return bits(B == 0 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0) : B == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)
              : B == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}
__device__ __forceinline__ uint32_t half_pair_of(uint32_t codes, float scale, int B)
{
    const f16x2 x = B == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0) : B == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1)
                  : B == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3);
    return __builtin_bit_cast(uint32_t, x);
}
template <typename T> __device__ __forceinline__ T lds_at(uint32_t offset) { return *(const __attribute__((address_space(3))) T *)offset; }
// The largest of three, NaNs aside.  (Written as fmaxf every operand is made quiet first: an instruction more for each.)
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
__device__ __forceinline__ float shuffle_xor(float x, int mask) { return __shfl_xor(x, mask, 64); }

// What the kernels need of a call.  Row offsets of codes in units of 16 bytes, of scales in units of 4.
struct MxArgs {
    const int32_t *indices;
    const uint8_t *codes, *scales;
    const int32_t *page_table;
    const uint16_t *q;
    float *out, *lse;
    void *out_lowp;
    uint32_t *row_parts;                  // [rows]: first and last share of a row, 16 bits each, or EMPTY
    float *slots;                         // partial (row, share) in slot share + row: [16 NQ][D] o, [16 NQ][2] m and l
    int64_t idx_stride, codes_b, codes_h, scales_b, scales_h, q_b, q_h, q_t;
    uint32_t codes_n, codes_page, scales_n, scales_page;
    FastDivisor per_h, per_t;
    int max_pages, page_shift, last_page, last_slot;
    int end_chunk;                        // the first chunk number behind the cache; larger ones have no position in 32 bits
    int H_q, H_kv, T, first_head, queries, chunk_shift;
    int paged, tail, dtype;               // paged: 1 by a page table, 2 by the list itself
    float to_log2;
    const uint16_t *k_new, *v_new;        // (the merge alone)
};

// What the line of tiles depends on: the kernels' leading arguments, which come in registers with the launch.
struct Lengths {
    const int32_t *counts, *seq_lens;
    uint32_t per_h_mul;
    int per_h_shift, rows, row0, n_max, capacity, dense, chunk_shift;
};
#define LENGTHS_PARAMS const int32_t *counts, const int32_t *seq_lens, uint32_t per_h_mul, int per_h_shift, int rows, int row0, int n_max, int capacity, int dense, int chunk_shift

// Positions that row r of the call attends to.
__device__ __forceinline__ int positions_of(const Lengths &c, const MxArgs &a, int r)
{
    int len = c.n_max;
    if (c.seq_lens && (c.dense || c.chunk_shift)) {
        FastDivisor per_h;
        per_h.mul = c.per_h_mul;
        per_h.shift = c.per_h_shift;
        len = min(max(c.seq_lens[per_h.divide(r)], 0), c.n_max);
    }
    if (c.dense) return len;
    const int n = min(max(c.counts[r], 0), c.capacity);
    if (!c.chunk_shift || n == 0) return n;
    // ascending chunks: only the last can reach past the sequence's length
    const int over = (int)min((int64_t)1 << c.chunk_shift, max((int64_t)0, (((int64_t)a.indices[r * a.idx_stride + n - 1] + 1) << c.chunk_shift) - len));
    return (n << c.chunk_shift) - over;
}

// x / y rounded up, for quotients below 2^22
__device__ __forceinline__ int divide_up(int x, int y)
{
    int q = (int)ceilf((float)x * __builtin_amdgcn_rcpf((float)y));
    q -= (int64_t)(q - 1) * y >= x;
    q += (int64_t)q * y < x;
    return q;
}
constexpr uint32_t EMPTY = 0xffffffffu;   // the parts of a row that attends to nothing

__device__ __forceinline__ int wave_last(int v) { return __builtin_amdgcn_readlane(v, 63); }

// How the work is cut.  FEW, up to 64 rows, which every wave holds one to a lane: each row goes to whole workgroups, as many as its
// tiles take at `size` tiles each, the smallest size at which the workgroups suffice (small ones in whole rounds of the waves); the
// row's tiles are dealt to them evenly.  Otherwise the tiles of all rows form one line with SEG_COST ahead of every row, and every
// workgroup takes an equal stretch of it (10 or 20 tiles: 240 us both, 64 sequences as above).  Whole workgroups need no tables and pick up
// one row: 64 rows of 7500 positions 23 us / 28 in equal stretches (one query tile), 31 / 38 (two); 8 rows of 1900 13.9 / 16.1.
template <int D, int NQ, bool F16, bool FEW> __global__ __launch_bounds__((Waves<NQ, FEW>::THREADS), 2) void mx_attn_kernel(LENGTHS_PARAMS, MxArgs a)
{
    typedef Geo<D> G;
    constexpr int NW = Waves<NQ, FEW>::N, DEPTH = Waves<NQ, FEW>::DEPTH, AHEAD = DEPTH - 1, THREADS = Waves<NQ, FEW>::THREADS;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds_bytes[];
    Lds<D, NQ, FEW> &lds = *reinterpret_cast<Lds<D, NQ, FEW> *>(lds_bytes);
    const Lengths lengths = {counts, seq_lens, per_h_mul, per_h_shift, rows, row0, n_max, capacity, dense, chunk_shift};
    const int tid = threadIdx.x, lane = tid % 64, low = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int me = blockIdx.x;
    int my_n = 0;                                                 // FEW: of row `lane`
    if constexpr (FEW) my_n = positions_of(lengths, a, row0 + min(lane, rows - 1));
    SPECATTN_PRELOAD(a.indices); SPECATTN_PRELOAD(a.codes); SPECATTN_PRELOAD(a.scales); SPECATTN_PRELOAD(a.page_table); SPECATTN_PRELOAD(a.q); SPECATTN_PRELOAD(a.row_parts);
    SPECATTN_PRELOAD(a.idx_stride); SPECATTN_PRELOAD(a.codes_h); SPECATTN_PRELOAD(a.scales_h); SPECATTN_PRELOAD(a.q_h); SPECATTN_PRELOAD(a.q_t); SPECATTN_PRELOAD(a.codes_n);
    SPECATTN_PRELOAD(a.per_h.mul); SPECATTN_PRELOAD(a.per_t.mul); SPECATTN_PRELOAD(a.max_pages); SPECATTN_PRELOAD(a.H_q); SPECATTN_PRELOAD(a.first_head); SPECATTN_PRELOAD(a.paged);

    int r, t0, t1, n, u = 0, u_end = 0, size = 0;                 // this workgroup's first row, its tiles of it, the row's positions
    if constexpr (FEW) {
        my_n = lane < rows ? my_n : 0;
        const int tiles = (my_n + TILE - 1) / TILE, all = wave_last(wave_inclusive_sum(tiles)), W = gridDim.x;
        int s = max((all + W - 1) / W, NW), groups, upto;
        if (s <= 4 * NW) s = (s + NW - 1) / NW * NW;
        while (true) {
            groups = divide_up(tiles, s);
            upto = wave_inclusive_sum(groups);
            const int need = wave_last(upto);
            if (need <= W) break;
            s += s <= 4 * NW ? NW : max(1, s * (need - W) / W);
        }
        if (me == 0 && tid < rows) a.row_parts[tid] = my_n == 0 ? EMPTY : (uint32_t)(upto - groups) | (uint32_t)(upto - 1) << 16;
        const uint64_t mine = __ballot(me >= upto - groups && me < upto);
        if (mine == 0) return;
        r = __builtin_ctzll(mine);
        n = __builtin_amdgcn_readlane(my_n, r);
        const int row_tiles = (n + TILE - 1) / TILE, parts = __builtin_amdgcn_readlane(groups, r), k = me - (__builtin_amdgcn_readlane(upto, r) - parts);
        const int even = __builtin_amdgcn_readfirstlane(divide_up(row_tiles + 1, parts)) - 1, more = row_tiles - even * parts;       // (row_tiles / parts rounded down)
        t0 = k * even + min(k, more);
        t1 = t0 + even + (k < more);
    } else {
        int c[2], tiles = 0, filled = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int x = 2 * tid + i;
            c[i] = x < rows ? positions_of(lengths, a, row0 + x) : 0;
            lds.count[x] = c[i];
            tiles += (c[i] + TILE - 1) / TILE;
            filled += c[i] > 0;
        }
        tiles = wave_last(wave_inclusive_sum(tiles));
        filled = wave_last(wave_inclusive_sum(filled));
        if (lane == 0) { lds.red[0][wave] = tiles; lds.red[1][wave] = filled; }
        __syncthreads();
        tiles = filled = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) { tiles += lds.red[0][w]; filled += lds.red[1][w]; }
        size = max(1, (int)(((int64_t)tiles + (int64_t)SEG_COST * filled + gridDim.x - 1) / gridDim.x));
        const int first = c[0] ? (c[0] + TILE - 1) / TILE + SEG_COST : 0, second = c[1] ? (c[1] + TILE - 1) / TILE + SEG_COST : 0;
        const int upto = wave_inclusive_sum(first + second);
        __syncthreads();                                          // (red is used again)
        if (lane == 63) lds.red[0][wave] = upto;
        __syncthreads();
        int before = upto - first - second, total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) before += lds.red[0][w];
            total += lds.red[0][w];
        }
        lds.prefix[2 * tid] = before;
        lds.prefix[2 * tid + 1] = before + first;
        if (tid == THREADS - 1) lds.prefix[MAX_ROWS] = total;
        if (me == 0) {                                            // first and last share of every row
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int start = (i ? before + first : before) + SEG_COST;
                if (2 * tid + i < rows)
                    a.row_parts[2 * tid + i] = c[i] == 0 ? EMPTY : (uint32_t)(start / size) | (uint32_t)((start + (c[i] + TILE - 1) / TILE - 1) / size) << 16;
            }
        }
        // the thread whose rows hold this workgroup's first unit says so
        u = me * size;
        if (u >= before && u < before + first + second) lds.red[1][0] = u < before + first ? 2 * tid : 2 * tid + 1;
        __syncthreads();
        u_end = min(u + size, total);
        if (u >= u_end) return;
        r = __builtin_amdgcn_readfirstlane(lds.red[1][0]);
    }

    for (bool more = true; more; ++r) {
        if constexpr (!FEW) {
            const int row_start = __builtin_amdgcn_readfirstlane(lds.prefix[r]);
            n = __builtin_amdgcn_readfirstlane(lds.count[r]);
            t0 = max(0, u - row_start - SEG_COST);
            t1 = min((n + TILE - 1) / TILE, u_end - row_start - SEG_COST);
            u = __builtin_amdgcn_readfirstlane(lds.prefix[r + 1]);
            more = u < u_end;
            if (t1 <= t0) continue;                               // (an empty row, or the share ends ahead of the row's first tile)
        } else more = false;
        const int row_tiles = (n + TILE - 1) / TILE, row = row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
        const int head0 = h * (a.H_q / a.H_kv) + a.first_head;

        // queries: element j of k-step s in lane (q, g) is element (d/4) g + 8 s + j of query 16 qt + q
        uint32_t qf[Lds<D, NQ, FEW>::Q ? 1 : NQ][G::KW][4];
        {
            auto query = [&](int qt) {
                const int i = min(qt * 16 + low, a.queries - 1), gh = a.per_t.divide(i), t = i - gh * a.T;      // (behind the last query: that one again)
                return a.q + b * a.q_b + (head0 + gh) * a.q_h + t * a.q_t + (D / 4) * g;
            };
            if constexpr (Lds<D, NQ, FEW>::Q) {
                for (int k = wave; k < NQ * G::KW; k += NW) *reinterpret_cast<u32x4 *>(lds.q + (k * 64 + lane) * 16) = *reinterpret_cast<const u32x4 *>(query(k / G::KW) + 8 * (k % G::KW));
                __syncthreads();
            } else {
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) {
                    const uint16_t *from = query(qt);
#pragma unroll
                    for (int s = 0; s < G::KW; ++s) {
                        const u32x4 w = *reinterpret_cast<const u32x4 *>(from + 8 * s);
#pragma unroll
                        for (int k = 0; k < 4; ++k) qf[qt][s][k] = w[k];
                    }
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

        // A tile goes through three steps, each AHEAD of the wave's tiles ahead of the next: its list words are requested; its pages; its codes and
        // scales.  Tiles are counted per wave: the wave's tile i is tile t0 + wave + i * NW of the row.  (Tiles past the share's end are
        // requested like others, clamped to the row, and not used.)
        WaveLds<D, DEPTH> &mine = lds.wave[wave];
        const uint32_t codes_lds = lds_offset(mine.codes), scales_lds = lds_offset(mine.scales), words_lds = lds_offset(mine.words), pages_lds = lds_offset(mine.pages);
        const int32_t *list = a.indices + row * a.idx_stride, *pages = a.page_table + (int64_t)b * a.max_pages;
        const uint8_t *codes = a.codes + (a.paged ? 0 : b * a.codes_b) + h * a.codes_h + ((lane % G::LPR) ^ G::swz(lane / G::LPR)) * 16;
        const uint8_t *scales = a.scales + (a.paged ? 0 : b * a.scales_b) + h * a.scales_h + (D == 128 ? lane / 32 * 4 : 0);
        const bool listed = !dense, looked_up = a.paged == 1;
        const int base_tile = t0 + wave, in_tile = lane % TILE;
        const int at_place = in_tile % G::RPI * G::CI + in_tile / G::RPI;
        // where the lane reads its keys (positions low, 16 + low), its values (4g + i, 16 + 4g + i) and their scales, in buffer 0
        const uint32_t keys_lds = codes_lds + G::piece(low, D == 128 ? g : g / 2) + (D == 128 ? 0 : g % 2 * 8);
        const uint32_t values_lds = codes_lds + G::piece(4 * g, D == 128 ? 4 + low / 4 : 2 + low / 8) + (D == 128 ? low % 4 * 4 : low % 8 * 2);
        const uint32_t values2_lds = codes_lds + G::piece(4 * g + 2, D == 128 ? 4 + low / 4 : 2 + low / 8) + (D == 128 ? low % 4 * 4 : low % 8 * 2) - 2 * D;     // (places of i = 2, 3)
        const uint32_t key_scale_lds = scales_lds + 4 * low + (F16 ? 0 : D == 128 ? g : g / 2), value_scale_lds = scales_lds + (D == 128 ? 128 : 0) + 16 * g;
        auto list_rank = [&](int i) { return min((base_tile + i * NW) * TILE + in_tile, n - 1); };
        auto list_at = [&](int i) { return list + (list_rank(i) >> a.chunk_shift); };
        auto slot_of = [&](int i, int word) -> int {
            if (!listed) return list_rank(i);                     // (below the length: inside the cache)
            if (a.chunk_shift) word = (int)((uint32_t)min(max(word, -1), a.end_chunk) << a.chunk_shift) | (list_rank(i) & ((1 << a.chunk_shift) - 1));
            return min(max(word, 0), a.last_slot);
        };
        auto request_words = [&](int i, int at) { if (listed) request4(list_at(i), words_lds + at * 256); };
        auto request_pages = [&](int slot, int at) { if (looked_up) request4(pages + (slot >> a.page_shift), pages_lds + at * 256); };
        auto request_codes = [&](int slot, int page, int at) {
            uint32_t code_at, scale_at;
            if (a.paged) {
                if (!looked_up) page = slot >> a.page_shift;
                page = min(max(page, 0), a.last_page);
                const uint32_t in = (uint32_t)slot & ((1u << a.page_shift) - 1);
                code_at = in * a.codes_n + (uint32_t)page * a.codes_page;
                scale_at = in * a.scales_n + (uint32_t)page * a.scales_page;
            } else {
                code_at = (uint32_t)slot * a.codes_n;
                scale_at = (uint32_t)slot * a.scales_n;
            }
            mine.codes_at[at_place] = code_at;
            uint32_t off[G::CI];
#pragma unroll
            for (int k = 0; k < G::CI; ++k) off[k] = mine.codes_at[lane / G::LPR * G::CI + k];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (what was read of the buffer that is written now has arrived)
            request4(scales + ((uint64_t)scale_at << 2), scales_lds + at * 256);
#pragma unroll
            for (int k = 0; k < G::CI; ++k)
                request16(codes + ((uint64_t)off[k] << 4), codes_lds + at * G::CODES + k * 1024);
        };

        uint32_t w[NQ][PARTS][4], v[8];
        int v_scale[8], unit = 0;                                 // scale bytes of the lane's block; unit: of the same block
        auto add_values = [&]() {
#pragma unroll
            for (int B = 0; B < G::DT / 2; ++B) {                 // elements 2B and 2B + 1 of the lane's
                uint32_t even[4], odd[4];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t first = half_pair_of(v[2 * j], __int_as_float(v_scale[2 * j]), B), second = half_pair_of(v[2 * j + 1], __int_as_float(v_scale[2 * j + 1]), B);
                    even[j] = __builtin_amdgcn_perm(second, first, 0x05040100);
                    odd[j] = __builtin_amdgcn_perm(second, first, 0x07060302);
                }
#pragma unroll
                for (int part = 0; part < PARTS; ++part)
#pragma unroll
                    for (int qt = 0; qt < NQ; ++qt) {
                        acc[qt][2 * B] = mfma_f16(even, w[qt][part], acc[qt][2 * B]);
                        acc[qt][2 * B + 1] = mfma_f16(odd, w[qt][part], acc[qt][2 * B + 1]);
                    }
            }
        };
        if (base_tile < t1) {
            int slot[2 * AHEAD], page[AHEAD] = {};
#pragma unroll
            for (int i = 0; i < 2 * AHEAD; ++i) slot[i] = listed ? *list_at(i) : 0;
#pragma unroll
            for (int i = 0; i < 2 * AHEAD; ++i) slot[i] = slot_of(i, slot[i]);
            if (looked_up)
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) page[i] = pages[slot[i] >> a.page_shift];
#pragma unroll 1
            for (int i = 0; i < AHEAD; ++i) {                     // (one copy of the code: a launch starts with none of it in the caches)
                request_codes(slot[0], page[0], i);
                request_pages(slot[AHEAD], i == 0 ? AHEAD % DEPTH : (AHEAD + 1) % DEPTH);
                request_words(2 * AHEAD + i, i == 0 ? 2 * AHEAD % DEPTH : (2 * AHEAD + 1) % DEPTH);
                const int first = slot[0];
#pragma unroll
                for (int k = 0; k + 1 < 2 * AHEAD; ++k) slot[k] = slot[k + 1];
                slot[2 * AHEAD - 1] = first;
                page[0] = page[AHEAD - 1];
            }
            int at = 0;                                           // tile i lies in buffer `at`; slot[]: of tiles i + AHEAD ...
            for (int i = 0, t = base_tile; t < t1; ++i, t += NW) {
                // all but what the last AHEAD - 1 iterations requested
                constexpr int R = G::CI + 1;
                if (listed && looked_up) wait_requests<(AHEAD - 1) * (R + 2)>();
                else if (listed || looked_up) wait_requests<(AHEAD - 1) * (R + 1)>();
                else wait_requests<(AHEAD - 1) * R>();
                const int prev = at == 0 ? DEPTH - 1 : at - 1, after = at == DEPTH - 1 ? 0 : at + 1;
                const int word_at = DEPTH == 2 ? at : after;      // of tile i + 2 AHEAD, like its pages
                const uint32_t codes_in = at * G::CODES, scales_in = at * 256;
                const int word = listed ? (int)mine.words[word_at][lane] : 0, in_page = looked_up ? mine.pages[prev][lane] : 0;
                uint32_t key[2][G::KW], key_scale[2];
                if constexpr (F16) {                              // keys in units of the largest scale of their position
                    const uint32_t four = lds_at<uint32_t>(scales_lds + scales_in + 4 * in_tile);
                    uint32_t top = max(four & 255, four >> 8 & 255);
                    if constexpr (D == 128) top = max(max(top, four >> 16 & 255), four >> 24);
                    mine.unit[in_tile] = top == 255 ? NAN : __uint_as_float(top << 23) * a.to_log2;
                    mine.unit_byte[in_tile] = top;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (F16) key_scale[k] = lds_at<uint32_t>(key_scale_lds + scales_in + 64 * k) >> (D == 128 ? g : g / 2) * 8 & 255;
                    else key_scale[k] = lds_at<uint8_t>(key_scale_lds + scales_in + 64 * k);
                    if constexpr (D == 128) {
                        const u32x4 x = lds_at<u32x4>(keys_lds + codes_in + 16 * D * k);
#pragma unroll
                        for (int s = 0; s < 4; ++s) key[k][s] = x[s];
                    } else {
                        const u32x2 x = lds_at<u32x2>(keys_lds + codes_in + 16 * D * k);
                        key[k][0] = x[0];
                        key[k][1] = x[1];
                    }
                }
                request_codes(slot[0], in_page, prev);
#pragma unroll
                for (int k = 0; k + 1 < AHEAD; ++k) slot[k] = slot[k + 1];
                slot[AHEAD - 1] = slot_of(i + 2 * AHEAD, word);
                request_pages(slot[AHEAD - 1], word_at);
                request_words(i + 3 * AHEAD, DEPTH == 2 ? after : at);

                f32x4 s[NQ][2], unit_of[2];
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) s[qt][0] = s[qt][1] = f32x4{0, 0, 0, 0};
                float scale_of[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (F16) {
                        scale_of[k] = __int_as_float(max((int)(key_scale[k] - mine.unit_byte[16 * k + low]) + 127, 0) << 23);
                        unit_of[k] = *reinterpret_cast<const f32x4 *>(&mine.unit[16 * k + 4 * g]);
                    } else scale_of[k] = __uint_as_float(key_scale[k] << 23);
                }
#pragma unroll
                for (int step = 0; step < G::KW; ++step)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t f[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) f[j] = F16 ? half_pair_of(key[k][step], scale_of[k], j) : pair_of(key[k][step], scale_of[k], j);
#pragma unroll
                        for (int qt = 0; qt < NQ; ++qt) {
                            uint32_t y[4];
                            if constexpr (Lds<D, NQ, FEW>::Q) {
                                const u32x4 x = *reinterpret_cast<const u32x4 *>(lds.q + ((qt * G::KW + step) * 64 + lane) * 16);
#pragma unroll
                                for (int j = 0; j < 4; ++j) y[j] = x[j];
                            } else
#pragma unroll
                                for (int j = 0; j < 4; ++j) y[j] = qf[qt][step][j];
                            s[qt][k] = F16 ? mfma_f16(f, y, s[qt][k]) : mfma(f, y, s[qt][k]);
                        }
                    }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const u32x4 four = lds_at<u32x4>(value_scale_lds + scales_in + 64 * k);
                    const int block = D == 128 ? low / 4 : 2 + low / 8;        // byte of a position's word
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v_scale[4 * k + j] = (int)__builtin_amdgcn_ubfe(four[j], 8 * block, 8);
                        const uint32_t from = (j < 2 ? values_lds : values2_lds) + codes_in + (16 * k + j) * D;
                        if constexpr (D == 128) v[4 * k + j] = lds_at<uint32_t>(from);
                        else v[4 * k + j] = lds_at<uint16_t>(from);
                    }
                }
                // The scores are read by the vector unit next, in another block of the program.  The compiler has been seen to leave the wait
                // that a matrix result needs ahead of it out there: it is written out.
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) {
                    if (qt == 0) asm volatile("s_nop 7\n\ts_nop 7" : "+v"(s[qt][0]), "+v"(s[qt][1]));
                    else asm volatile("" : "+v"(s[qt][0]), "+v"(s[qt][1]));
                }
                if constexpr (F16)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
#pragma unroll
                        for (int qt = 0; qt < NQ; ++qt) s[qt][k / 4][k % 4] *= unit_of[k / 4][k % 4];
                const int left = n - t * TILE;
                if (__builtin_expect(left < TILE, 0)) {                                // a row's last tile: what lies behind it repeats its last position
#pragma unroll
                    for (int k = 0; k < 8; ++k)
#pragma unroll
                        for (int qt = 0; qt < NQ; ++qt) s[qt][k / 4][k % 4] = 16 * (k / 4) + 4 * g + k % 4 < left ? s[qt][k / 4][k % 4] : -INFINITY;
                }
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) {
                    __builtin_amdgcn_sched_barrier(0);
                    float most = max3(max3(s[qt][0][0], s[qt][0][1], s[qt][0][2]), max3(s[qt][0][3], s[qt][1][0], s[qt][1][1]), max3(s[qt][1][2], s[qt][1][3], s[qt][1][3]));
                    if constexpr (!F16) most *= a.to_log2;
                    if (__builtin_expect(__any(most > ref[qt] + RANGE), 0)) {
                        most = fmaxf(most, shuffle_xor(most, 16));
                        most = fmaxf(most, shuffle_xor(most, 32));
                        const float now = fmaxf(ref[qt], most - HEAD), factor = ref[qt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[qt] - now);
                        ref[qt] = now;
                        sum[qt] *= factor;
#pragma unroll
                        for (int d = 0; d < G::DT; ++d) acc[qt][d] *= factor;
                    }
                    float e[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) e[k] = __builtin_amdgcn_exp2f(F16 ? s[qt][k / 4][k % 4] - ref[qt] : __builtin_fmaf(s[qt][k / 4][k % 4], a.to_log2, -ref[qt]));
                    sum[qt] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        w[qt][0][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(e[2 * k], e[2 * k + 1]));
                        w[qt][1][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(less_low(e[2 * k], w[qt][0][k]), less_high(e[2 * k + 1], w[qt][0][k])));
                    }
                }
                // scales in units of 2^(unit - 127)
                int most_v = v_scale[0], least_v = v_scale[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) { most_v = max(most_v, v_scale[j]); least_v = min(least_v, v_scale[j]); }
                if (__builtin_expect(__any(most_v > unit || least_v < unit - FAR), 0)) {
                    int top = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = max(top, v_scale[j] == 255 ? 0 : v_scale[j]);
                    top = max(top, __shfl_xor(top, 16, 64));      // (the lanes of a block hold the same positions but for g)
                    top = max(top, __shfl_xor(top, 32, 64));
                    if (__any(top > unit)) {
                        const int now = max(unit, top), down = __shfl(unit - now, D == 128 ? 4 * g : 8 * (g / 2), 64);     // (lane group g sums up columns of that lane's block)
                        unit = now;
#pragma unroll
                        for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
                            for (int d = 0; d < G::DT; ++d)
#pragma unroll
                                for (int k = 0; k < 4; ++k) acc[qt][d][k] = __builtin_ldexpf(acc[qt][d][k], down);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) v_scale[j] = v_scale[j] == 255 ? unit + 128 : max(v_scale[j], unit - 100);    // (NaN; zero)
                }
                const int unit_bits = (127 - unit) * (1 << 23);
#pragma unroll
                for (int j = 0; j < 8; ++j) v_scale[j] = (int)((uint32_t)v_scale[j] << 23) + unit_bits;
                add_values();
                at = after;
            }
            wait_requests<0>();                                   // (the buffers are used for other things next)
            // The sums leave the units of weights and values for those of the values over 2^e, e the exponent of the sum of weights: what
            // comes out lies below the largest value, however many there are (in the weights' units sums of values beyond 2^103 are infinite).
            const int up = __shfl(unit, D == 128 ? 4 * g : 8 * (g / 2), 64) - 127;
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
                sum[qt] += shuffle_xor(sum[qt], 16);
                sum[qt] += shuffle_xor(sum[qt], 32);
                const int scale = up - __builtin_amdgcn_frexp_expf(sum[qt]);
#pragma unroll
                for (int d = 0; d < G::DT; ++d)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[qt][d][k] = __builtin_ldexpf(acc[qt][d][k], scale);
            }
        }
        __syncthreads();

        // The waves' states, one query tile at a time.
        const bool alone = t0 == 0 && t1 == row_tiles && !a.tail;
        float *slot_o = a.slots + (size_t)(me + r) * NQ * 16 * (D + 2), *slot_ml = slot_o + NQ * 16 * D;
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            if (g == 0) {
                const int e = __builtin_amdgcn_frexp_expf(sum[qt]);
                lds.merge.ml[wave][low] = f32x4{ref[qt], __builtin_ldexpf(sum[qt], -e), __builtin_ldexpf(1.0f, e), 0.0f};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < G::DT; d += 4)
                    *reinterpret_cast<f32x4 *>(&lds.merge.o[wave][low][G::DT * (4 * g + i) + d]) = f32x4{acc[qt][d][i], acc[qt][d + 1][i], acc[qt][d + 2][i], acc[qt][d + 3][i]};
            __syncthreads();
            for (int x = tid; x < 16 * D / 4; x += THREADS) {
                const int q = x / (D / 4), col = x % (D / 4) * 4;
                float top = -INFINITY, all = 0.0f, f[NW];
                f32x4 ml[NW];
#pragma unroll
                for (int k = 0; k < NW; ++k) { ml[k] = lds.merge.ml[k][q]; top = fmaxf(top, ml[k][0]); }
#pragma unroll
                for (int k = 0; k < NW; ++k) {
                    f[k] = ml[k][0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[k][0] - top) * ml[k][2];
                    all += f[k] * ml[k][1];
                }
                const float inverse = 1.0f / all;
                f32x4 o = {0, 0, 0, 0};                           // the weighted average of the waves': never beyond the largest value
#pragma unroll
                for (int k = 0; k < NW; ++k) o += f[k] * inverse * *reinterpret_cast<const f32x4 *>(&lds.merge.o[k][q][col]);
                const int i = qt * 16 + q;
                if (!alone) {
                    *reinterpret_cast<f32x4 *>(slot_o + i * D + col) = o;
                    if (col == 0) { slot_ml[2 * i] = top; slot_ml[2 * i + 1] = all; }
                } else if (i < a.queries) {
                    const int gh = a.per_t.divide(i), tq = i - gh * a.T;
                    const int64_t orow = ((int64_t)b * a.H_q + head0 + gh) * a.T + tq;
                    if (a.out) *reinterpret_cast<f32x4 *>(a.out + orow * D + col) = o;
                    if (a.out_lowp)
                        for (int k = 0; k < 4; ++k) st_lowp(a.out_lowp, orow * D + col + k, o[k], a.dtype);
                    if (a.lse && col == 0) a.lse[orow] = (top + __builtin_amdgcn_logf(all)) * 0.69314718055994530942f;
                }
            }
            __syncthreads();
        }
    }
}

template <int E> struct Word { typedef uint32_t type; };
template <> struct Word<1> { typedef uint16_t type; };

// One wave per (row, query): the row's partials in share order, eight to a trip to memory, then the new tokens behind the cache up to
// the query's own.  (Their rows asked for ahead of the partials and their scores taken together; one after the other, 8 rows with 5 new tokens
// 17.8 us / 16.3 for the call.)
template <int D, bool TAIL> __global__ __launch_bounds__(256) void mx_merge_kernel(const uint32_t *row_parts, const float *slots, int row0, int padded, int queries, MxArgs a)
{
    constexpr int E = D / 64, TRIP = 8, NEW = SPECATTN_MAX_T;     // elements per lane
    const int lane = threadIdx.x % 64;
    const int r = blockIdx.y, i = blockIdx.x * 4 + threadIdx.x / 64;
    if (i >= queries) return;
    const uint32_t parts = row_parts[r];
    SPECATTN_PRELOAD(a.out); SPECATTN_PRELOAD(a.lse); SPECATTN_PRELOAD(a.out_lowp); SPECATTN_PRELOAD(a.per_h.mul); SPECATTN_PRELOAD(a.per_t.mul); SPECATTN_PRELOAD(a.H_q);
    if constexpr (TAIL) { SPECATTN_PRELOAD(a.k_new); SPECATTN_PRELOAD(a.v_new); SPECATTN_PRELOAD(a.q); SPECATTN_PRELOAD(a.q_b); SPECATTN_PRELOAD(a.q_h); SPECATTN_PRELOAD(a.q_t); }
    const int row = row0 + r, b = a.per_h.divide(row), h = row - b * a.H_kv;
    const int gh = a.per_t.divide(i), t = i - gh * a.T, head = h * (a.H_q / a.H_kv) + a.first_head + gh;
    const int64_t orow = ((int64_t)b * a.H_q + head) * a.T + t;
    // The new tokens' rows are requested ahead of everything else: E elements of a lane in a word.
    typedef typename Word<E>::type W;
    W q = {}, k_new[NEW] = {}, v_new[NEW] = {};
    auto value = [&](W x, int e) { return a.dtype == SPECATTN_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)(x >> 16 * e)) : __uint_as_float((uint32_t)(uint16_t)(x >> 16 * e) << 16); };
    if constexpr (TAIL) {
        q = *reinterpret_cast<const W *>(a.q + b * a.q_b + head * a.q_h + t * a.q_t + E * lane);
#pragma unroll
        for (int j = 0; j < NEW; ++j) {                           // (behind the query's own: that one again)
            const int64_t at = ((int64_t)row * a.T + min(j, t)) * D + E * lane;
            k_new[j] = *reinterpret_cast<const W *>(a.k_new + at);
            v_new[j] = *reinterpret_cast<const W *>(a.v_new + at);
        }
    }
    float m = -INFINITY, l = 0.0f, o[E];                          // o: the average so far, as in the partials; sums of large values have no fp32
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    if (parts != EMPTY) {
        const int first = parts & 0xffff, last = parts >> 16;
        if (first == last && !TAIL) return;                       // finished by its only workgroup
        for (int w = first; w <= last; w += TRIP) {
            float mw[TRIP], lw[TRIP], ow[TRIP][E];
#pragma unroll
            for (int k = 0; k < TRIP; ++k) {                      // (behind the last: that one again)
                const float *slot = slots + (size_t)(min(w + k, last) + r) * padded * (D + 2);
                const f32x2 ml = *reinterpret_cast<const f32x2 *>(slot + padded * D + 2 * i);
                mw[k] = ml[0];
                lw[k] = ml[1];
#pragma unroll
                for (int e = 0; e < E; ++e) ow[k][e] = slot[i * D + E * lane + e];
            }
            __builtin_amdgcn_sched_barrier(0);                    // all requested before the first is used
            float now = m;
#pragma unroll
            for (int k = 0; k < TRIP; ++k) now = fmaxf(now, w + k <= last ? mw[k] : -INFINITY);
            const float before = m == -INFINITY ? 0.0f : l * __builtin_amdgcn_exp2f(m - now);
            l = before;
#pragma unroll
            for (int k = 0; k < TRIP; ++k) {
                lw[k] = w + k <= last ? lw[k] * __builtin_amdgcn_exp2f(mw[k] - now) : 0.0f;
                l += lw[k];
            }
            const float inverse = 1.0f / l;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= before * inverse;
#pragma unroll
            for (int k = 0; k < TRIP; ++k) {
                if (w + k > last) break;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] += ow[k][e] * (lw[k] * inverse);
            }
            m = now;
        }
    }
    if constexpr (TAIL) {
        float s[NEW];
#pragma unroll
        for (int j = 0; j < NEW; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) s[j] += value(q, e) * value(k_new[j], e);
        }
#pragma unroll
        for (int k = 1; k < 64; k *= 2)
#pragma unroll
            for (int j = 0; j < NEW; ++j) s[j] += shuffle_xor(s[j], k);
        float now = m;
#pragma unroll
        for (int j = 0; j < NEW; ++j) {
            s[j] = j <= t ? s[j] * a.to_log2 : -INFINITY;
            now = fmaxf(now, s[j]);
        }
        const float before = m == -INFINITY ? 0.0f : l * __builtin_amdgcn_exp2f(m - now);
        l = before;
#pragma unroll
        for (int j = 0; j < NEW; ++j) {
            s[j] = j <= t ? __builtin_amdgcn_exp2f(s[j] - now) : 0.0f;
            l += s[j];
        }
        const float inverse = 1.0f / l;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= before * inverse;
#pragma unroll
        for (int j = 0; j < NEW; ++j) {
            if (j > t) break;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += value(v_new[j], e) * (s[j] * inverse);
        }
        m = now;
    }
    const bool any = l != 0.0f;                                   // (also where l is NaN)
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = any ? o[e] : 0.0f;
        if (a.out) a.out[orow * D + E * lane + e] = x;
        if (a.out_lowp) st_lowp(a.out_lowp, orow * D + E * lane + e, x, a.dtype);
    }
    if (a.lse && lane == 0) a.lse[orow] = any ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

template <int D, int NQ> const void *variant(bool f16, bool few)
{
    return f16 ? few ? reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, true, true>) : reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, true, false>)
               : few ? reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, false, true>) : reinterpret_cast<const void *>(mx_attn_kernel<D, NQ, false, false>);
}
template <int D> const void *variant(int nq, bool f16, bool few)
{
    return nq == 1 ? variant<D, 1>(f16, few) : nq == 2 ? variant<D, 2>(f16, few) : nq == 3 ? variant<D, 3>(f16, few) : variant<D, 4>(f16, few);
}
const void *variant(int d, int nq, bool f16, bool few) { return d == 128 ? variant<128>(nq, f16, few) : variant<64>(nq, f16, few); }
template <int D, int NQ> size_t lds_size(bool few) { return few ? sizeof(Lds<D, NQ, true>) : sizeof(Lds<D, NQ, false>); }
template <int D> size_t lds_size(int nq, bool few) { return nq == 1 ? lds_size<D, 1>(few) : nq == 2 ? lds_size<D, 2>(few) : nq == 3 ? lds_size<D, 3>(few) : lds_size<D, 4>(few); }
size_t lds_size(int d, int nq, bool few) { return d == 128 ? lds_size<128>(nq, few) : lds_size<64>(nq, few); }
int threads_of(int nq, bool few) { return !few ? Waves<1, false>::THREADS : nq == 1 ? Waves<1, true>::THREADS : Waves<2, true>::THREADS; }

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
    return (((size_t)per * 4 + 255) & ~(size_t)255) + (((size_t)(2 * cu_count() + per) * padded * (d + 2) * sizeof(float) + 255) & ~(size_t)255);
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
    for (int k = 0; k < 32; ++k) {
        const int d = k & 1 ? 128 : 64, nq = (k >> 1 & 3) + 1;
        const bool f16 = k & 8, few = k & 16;
        if (hipFuncSetAttribute(variant(d, nq, f16, few), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_size(d, nq, few)) != hipSuccess) {
            (void)hipGetLastError();
            set_error("cannot reserve %zu bytes of LDS", lds_size(d, nq, few));
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
    const AttnLaunch &c = l.a;
    const int rows = c.B * c.H_kv, G = c.H_q / c.H_kv, per = heads_per_launch(G, c.T);
    MxArgs a{};
    a.indices = c.indices;
    a.codes = l.c.codes; a.scales = l.c.scales; a.page_table = l.c.page_table;
    a.q = static_cast<const uint16_t *>(c.q);
    a.out = c.out; a.lse = c.lse; a.out_lowp = c.out_lowp;
    a.idx_stride = c.idx_stride;
    a.codes_b = l.c.codes_b; a.codes_h = l.c.codes_h; a.scales_b = l.c.scales_b; a.scales_h = l.c.scales_h;
    a.q_b = c.q_stride_b; a.q_h = c.q_stride_h; a.q_t = c.q_stride_t;
    a.codes_n = (uint32_t)(l.c.codes_n >> 4); a.codes_page = (uint32_t)(l.c.codes_page >> 4);
    a.scales_n = (uint32_t)(l.c.scales_n >> 2); a.scales_page = (uint32_t)(l.c.scales_page >> 2);
    a.per_h = FastDivisor(c.H_kv); a.per_t = FastDivisor(c.T);
    a.max_pages = l.c.max_pages; a.page_shift = l.c.page_shift; a.last_page = l.c.num_pages - 1;
    a.last_slot = c.indices_are_physical ? (int)std::min<int64_t>(((int64_t)l.c.num_pages << l.c.page_shift) - 1, INT32_MAX) : c.n_max - 1;
    a.H_q = c.H_q; a.H_kv = c.H_kv; a.T = c.T;
    a.chunk_shift = c.chunk_shift;
    a.end_chunk = std::min((a.last_slot >> a.chunk_shift) + 1, INT32_MAX >> a.chunk_shift);
    a.paged = l.c.page_table ? 1 : c.indices_are_physical ? 2 : 0; a.tail = c.k_new != nullptr; a.dtype = c.dtype;
    a.to_log2 = c.sm_scale * 1.44269504088896340736f;
    a.k_new = static_cast<const uint16_t *>(c.k_new); a.v_new = static_cast<const uint16_t *>(c.v_new);
    for (int first = 0; first < G; first += per) {
        a.first_head = first;
        a.queries = std::min(per, G - first) * c.T;
        const int nq = (a.queries + 15) / 16;
        for (int row0 = 0; row0 < rows; row0 += MAX_ROWS) {
            int here = std::min(MAX_ROWS, rows - row0), at = row0;
            a.row_parts = static_cast<uint32_t *>(c.workspace);
            a.slots = reinterpret_cast<float *>(static_cast<char *>(c.workspace) + (((size_t)here * 4 + 255) & ~(size_t)255));
            Lengths n = {c.counts, c.seq_lens, a.per_h.mul, a.per_h.shift, here, at, c.n_max, c.idx_capacity, c.dense, c.chunk_shift};
            void *args[] = {&n.counts, &n.seq_lens, &n.per_h_mul, &n.per_h_shift, &n.rows, &n.row0, &n.n_max, &n.capacity, &n.dense, &n.chunk_shift, &a};
            const bool f16 = c.dtype == SPECATTN_F16;
            const bool few = here <= std::min(64, cu_count());
            if (hipLaunchKernel(variant(c.d, nq, f16, few), dim3(few ? cu_count() : 2 * cu_count()), dim3(threads_of(nq, few)), args, lds_size(c.d, nq, few), stream) != hipSuccess) return check_launch("mx_attn_kernel");
            st = check_launch("mx_attn_kernel");
            if (st != SPECATTN_OK) return st;
            const dim3 grid((a.queries + 3) / 4, here);
            auto merge = c.d == 128 ? a.tail ? mx_merge_kernel<128, true> : mx_merge_kernel<128, false> : a.tail ? mx_merge_kernel<64, true> : mx_merge_kernel<64, false>;
            merge<<<grid, 256, 0, stream>>>(a.row_parts, a.slots, at, nq * 16, a.queries, a);
            st = check_launch("mx_merge_kernel");
            if (st != SPECATTN_OK) return st;
        }
    }
    return SPECATTN_OK;
}

}  // namespace specattn
