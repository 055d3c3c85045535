// Attention of many query rows per kv head (prompts, trees of drafted tokens; bf16 or fp16, d = 128 or 64): the tile loop that
// both kernels share.
//
// A workgroup of four or eight waves takes up to 32 * WQ query rows of one kv head - rows of all its query heads, which share keys and
// values - over tiles of 64 positions.  Tiles go from memory straight to LDS (16-byte chunks in a swizzled order), into a ring of
// buffers, three tiles (d = 64: seven) ahead of their turn.
//   S^T = K Q^T    : mfma 32x32x16, A = K fragment (ds_read_b128), B = Q fragment (registers)
//   softmax        : one pass, a running reference per query row that follows its maximum up
//   O^T += V^T P^T : A = V^T fragment (ds_read_b64_tr_b16), B = P
// A query row is a column of S^T and O^T and stays in one lane and the lane 32 beyond it: the 16 scores that a lane holds of 32
// positions are, eight by eight, the B fragment of the second product when the positions of its k-steps are numbered the same
// way (slot 8 h + j of 16 stands for position 8 (j / 4) + 4 h + j % 4), so weights never leave their lane.
// With fewer query rows than the waves have room for, two waves share rows and take one half of a tile each; their results are joined in LDS at the end.
//
// A tile costs a wave 32 matrix instructions (d = 128; 1024 cycles of its SIMD's matrix unit) and about 190 vector ones, 32 of them exponentials.
// One causal prompt of 32768 positions, 32 heads over 8, bf16: 7.9 to 8.6 ms, 1.03 to 1.11 PFLOP/s (a library product of 8192^3 reaches 1.20), the matrix units busy for 51 %
// of the cycles at 1.94 GHz.  Two groups of waves that take turns between products and softmax, and fetches spread between the products, took the same time.
#pragma once

#include "serve.h"

namespace specattn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The element types.  Weights are taken in units of 2^ref, the row's running reference: the largest lies between 2^HEAD and 2^(HEAD + SLACK)
// of them, and a tile moves the reference only when it leaves that range (that scales all accumulators).  bf16 has the exponents of
// fp32.  fp16 ends at 2^-24: with 2^12 for the largest, weights down to 2^-36 of it are still told apart.
template <bool F16> struct Half;
template <> struct Half<false> {
    static constexpr float HEAD = 0.0f, SLACK = 8.0f;
    typedef bf16x8 x8;
    typedef bf16x2 x2;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
};
template <> struct Half<true> {
    static constexpr float HEAD = 12.0f, SLACK = 3.0f;
    typedef f16x8 x8;
    typedef f16x2 x2;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float widen(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
};

// The kernel's arguments (its only ones) read once more: what follows the tile loop then does not hold registers throughout it.
template <typename ARGS> __device__ __forceinline__ const ARGS &arguments_again()
{
    auto p = (const __attribute__((address_space(4))) ARGS *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const ARGS *)p;
}

// Two values in the element type, the first in the low half (round to nearest even).
template <bool F16> __device__ __forceinline__ uint32_t pack2(float x, float y)
{
    const f32x2 pair = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, typename Half<F16>::x2));
}

// A workgroup of NW waves, WQ of them side by side over query rows, with a ring of RING KB of tiles.
template <int DIM, int NW_, int WQ_, int RING> struct Geo {
    static constexpr int D = DIM, NW = NW_, WQ = WQ_;
    static constexpr int THREADS = NW * 64;
    static constexpr int WK = NW / WQ;                        // waves that share query rows
    static constexpr int SUBS = 2 / WK;                       // pieces of 32 positions of a tile that a wave takes
    static constexpr int SPAN = 32 * SUBS;                    // its positions of a tile
    static constexpr int TILE = 64;
    static constexpr int QROWS = 32 * WQ;
    static constexpr int ROW_BYTES = D * 2;
    static constexpr int CHUNKS = ROW_BYTES / 16;             // lanes that fetch a row
    static constexpr int RPI = 64 / CHUNKS;                   // rows that a wave fetches at a time
    static constexpr int LOADS = TILE / RPI / NW;             // times it does so, of keys and of values
    static constexpr int TILE_BYTES = TILE * ROW_BYTES;
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES;        // keys, values
    static constexpr int STAGES = RING * 1024 / STAGE_BYTES;  // tiles under way or in use
    static constexpr int BATCH = RING / 2;                    // tiles whose rows are looked up at a time
    static constexpr int OFF_TABLE = STAGES * STAGE_BYTES;    // uint32[BATCH * TILE] where the rows lie, in units of 16 bytes
    static constexpr int OFF_ML = OFF_TABLE + BATCH * TILE * 4;       // float[2][NW][32]: references and sums of the waves' rows
    static constexpr int LDS_BYTES = OFF_ML + 2 * NW * 32 * 4;
    static_assert(NW * 32 * D * 4 <= STAGES * STAGE_BYTES, "the waves' results are laid out over the tile buffers");
    static_assert(WK == 1 || WK == 2, "a tile has two pieces of 32 positions");
    static_assert((STAGES & (STAGES - 1)) == 0, "tiles take the buffers in turn");
    // 16-byte chunk c of row r lies in place c ^ swz(r): both the key reads (a chunk of 32 rows) and the transposing value reads (4 rows x
    // 32 bytes to 16 lanes) then spread over all banks.
    static __device__ __forceinline__ int swz(int row)
    {
        return (D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    }
};

// 16 bytes per lane from memory to LDS, to `to` + 16 * lane.  Written out because the compiler, which cannot tell where such a load goes,
// makes every read of LDS wait for it; the loop's own wait stands ahead of its barrier.
__device__ __forceinline__ void load_to_lds(const void *src, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory", "m0");
}
// All but the last N loads of this wave have arrived, LDS is read and written, and the other waves are here.
template <int N> __device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }
// As tile_barrier with the loads of `tiles` tiles of N left under way (at most MOST).
template <int N, int MOST> __device__ __forceinline__ void tile_barrier_behind(int tiles)
{
    if constexpr (MOST == 0) tile_barrier<0>();
    else if (tiles >= MOST) tile_barrier<MOST * N>();
    else tile_barrier_behind<N, MOST - 1>(tiles);
}
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p; }

// Over the two lanes that hold a query row.
__device__ __forceinline__ float pair_max(float x)
{
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float pair_sum(float x)
{
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

// The largest of a wave's values, none of them negative (steps as in wave_inclusive_sum).
__device__ __forceinline__ int wave_largest(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}

// The low `n` bits (none below 1, all from 64 on).
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// Values near the end of fp32 (with bf16; with fp16 no sum comes close): rows whose unnormalised values times LARGE pass it are computed once more, with weights that add up to
// less than 2^-MORE, so that 2^MORE parts of a row (the GPU's workgroups are fewer) can be joined as they are.
constexpr float LARGE = 262144.0f;                            // 2^18
constexpr int MORE = 12;

// The reference of a part as it is put down: minus infinity says that nothing was attended to, which is not so where a score was NaN.
__device__ __forceinline__ float reference(float ref, float sum) { return sum == sum ? ref : sum; }

// One wave's 32 query rows.
// PARTS: parts of the element type that a weight enters the second product in.  Where the result is asked for in that type alone, one:
// its rounding (half a step, averaged over the row) is below the result's own.  Where it is asked for in fp32, two.  (One part / two: a causal prompt of 32768 tokens
// 8.0 / 11.1 ms, 4 x 512 tokens behind 4096 to 15872 in pages 667 / 910 us, 8 trees of 16 nodes over 7536 of 32768 positions 62 / 68, 16 of 64 over 3276 of 8192 138 / 180.)
template <typename G, bool F16, int PARTS> struct RowsOfWave {
    static constexpr int D = G::D;
    typedef typename Half<F16>::x8 x8;
    x8 q[D / 16];
    f32x16 o[D / 32];
    f32x16 s[G::SUBS];                                        // scores of a tile
    u32x4 p[G::SUBS][2][PARTS];                               // weights of a tile, in the element type
    float ref, sum;                                           // in powers of two; of this lane's positions alone
    float over;                                               // what rounding has put into the sum beyond its terms
    float scale;                                              // of the scores, log2(e) in it
    uint32_t key_at, value_at;                                // where this lane's first fragments lie in a tile

    __device__ __forceinline__ void start(int wk, float sm_scale)
    {
#pragma unroll
        for (int t = 0; t < D / 32; ++t) o[t] = f32x16{};
        ref = -INFINITY;
        sum = over = 0.0f;
        scale = sm_scale * LOG2E;
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const int krow = lane & 31;
        key_at = (wk * G::SPAN + krow) * G::ROW_BYTES + ((half ^ G::swz(krow)) << 4);
        const int vrow = 4 * half + ((lane & 15) >> 2);       // of eight, and the 16 bytes of a row's first 64 that hold its elements
        const int chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        value_at = G::TILE_BYTES + (wk * G::SPAN + vrow) * G::ROW_BYTES + ((chunk ^ G::swz(vrow)) << 4) + 8 * (lane & 1);
    }

    // Fragments are asked for four at a time, a step of four products ahead of their use; the compiler, left alone, asks for each where it is
    // needed and waits.
    struct Four { x8 f[4]; };
    static constexpr int ADD_STEPS = G::SUBS * 2 * (D / 32) / 4, SCORE_STEPS = G::SUBS * (D / 16) / 4;
    __device__ __forceinline__ Four values(const char *buf, int step) const
    {
        Four x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = step * 4 + i, t = n % (D / 32), b = n / (D / 32);        // 32 elements, 16 positions
            const uint32_t at = (value_at ^ (t << 6)) + b * 16 * G::ROW_BYTES;
            const uint32_t at8 = (value_at ^ (t << 6) ^ 32) + (b * 16 + 8) * G::ROW_BYTES;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(buf + at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(buf + at8));
            x.f[i] = __builtin_bit_cast(x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return x;
    }
    __device__ __forceinline__ Four keys(const char *buf, int step) const
    {
        Four x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = step * 4 + i, u = n % G::SUBS, c = n / G::SUBS;
            x.f[i] = *reinterpret_cast<const x8 *>(buf + ((key_at ^ (c << 5)) + u * 32 * G::ROW_BYTES));
        }
        return x;
    }
    __device__ __forceinline__ void add_step(const Four &x, int step)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = step * 4 + i, t = n % (D / 32), b = n / (D / 32);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) o[t] = Half<F16>::mfma(x.f[i], __builtin_bit_cast(x8, p[b / 2][b % 2][part]), o[t]);
        }
    }
    __device__ __forceinline__ void score_step(const Four &x, int step)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = step * 4 + i, u = n % G::SUBS, c = n / G::SUBS;
            s[u] = Half<F16>::mfma(x.f[i], q[c], s[u]);
        }
    }
    // Scores of the tile at buf (LDS).
    __device__ __forceinline__ void score(const char *buf)
    {
#pragma unroll
        for (int u = 0; u < G::SUBS; ++u) s[u] = f32x16{};
        Four ready = keys(buf, 0);
#pragma unroll
        for (int step = 0; step < SCORE_STEPS; ++step) {
            Four next = ready;
            if (step + 1 < SCORE_STEPS) next = keys(buf, step + 1);
            __builtin_amdgcn_sched_barrier(0);
            score_step(ready, step);
            __builtin_amdgcn_sched_barrier(0);
            ready = next;
        }
    }
    // Weighted values of the tile at buf; its first fragments are in `ready`.
    __device__ __forceinline__ void add(const char *buf, Four ready)
    {
#pragma unroll
        for (int step = 0; step < ADD_STEPS; ++step) {
            Four next = ready;
            if (step + 1 < ADD_STEPS) next = values(buf, step + 1);
            __builtin_amdgcn_sched_barrier(0);
            add_step(ready, step);
            __builtin_amdgcn_sched_barrier(0);
            ready = next;
        }
    }

    // Scores of tile t into weights.  (The total is compensated; the products add up in fp32, sixteen positions at a time.)
    template <typename SEEN> __device__ __forceinline__ void weigh(SEEN &&seen, int t)
    {
        uint64_t word = 0;
        if (!seen(t, word)) {
            const uint64_t mine = word >> (4 * ((threadIdx.x & 63) >> 5));
#pragma unroll
            for (int u = 0; u < G::SUBS; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((mine >> (32 * u + 8 * (i / 4) + i % 4)) & 1)) s[u][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < G::SUBS; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        top = pair_max(top) * scale;
        const bool far = top > ref + Half<F16>::SLACK;
        if (__any(far)) {                                     // (each row for itself: what its neighbours see has no part in its rounding)
            const float by = far ? __builtin_amdgcn_exp2f(ref - top) : 1.0f;
            ref = far ? top : ref;
            sum *= by;
            over *= by;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= by;
        }
        const float from = ref == -INFINITY ? 0.0f : Half<F16>::HEAD - ref;
        float part[4] = {};                                   // a tile's weights by themselves, in four sums
#pragma unroll
        for (int u = 0; u < G::SUBS; ++u) {
            float w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(s[u][i], scale, from));
                part[i & 3] += w[i];
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = w[8 * b + 2 * i], y = w[8 * b + 2 * i + 1];
                    p[u][b][0][i] = pack2<F16>(x, y);
                    if (PARTS == 2)
                        p[u][b][PARTS - 1][i] = pack2<F16>(x - Half<F16>::widen((uint16_t)p[u][b][0][i]), y - Half<F16>::widen((uint16_t)(p[u][b][0][i] >> 16)));
                }
        }
        // (compensated, W. Kahan 1965: equal weights added to a long sum one by one are all rounded the same way)
        const float tile = ((part[0] + part[1]) + (part[2] + part[3])) - over, next = sum + tile;
        over = (next - sum) - tile;
        sum = next;
    }

    // Whether a row with finite scores holds a value that is not finite, or so large that parts of a row could pass fp32 together: an infinity or NaN
    // came in, as 0 * infinity from behind its mask or as what the row sees, or values are near the end of fp32 (never so with sums below 2^104, always from 2^111 on).
    __device__ __forceinline__ bool spoiled() const
    {
        float x = 0.0f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) x = fmaf(o[t][i], LARGE, x);
        return !(x - x == 0.0f) && sum - sum == 0.0f && ref > -INFINITY && ref < INFINITY;
    }

    // Result of this wave into its part of the LDS: unnormalised rows (16-byte chunks in a swizzled order), references and sums.
    __device__ __forceinline__ void leave(char *smem)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 31, half = lane >> 5;
        char *mine = smem + wave * 32 * D * 4;
        sum = pair_sum(sum - over);
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 x = {o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
                *reinterpret_cast<f32x4 *>(mine + row * D * 4 + (((8 * t + 2 * j + half) ^ (row & (D / 4 - 1))) << 4)) = x;
            }
        if (half == 0) {
            float *ml = reinterpret_cast<float *>(smem + G::OFF_ML);
            ml[wave * 32 + row] = reference(ref, sum);
            ml[G::NW * 32 + wave * 32 + row] = sum;
        }
    }
};

// Four elements at 4 * chunk of query row `row` of the wave whose part begins at `part`.
template <int D> __device__ __forceinline__ f32x4 left_row(const char *part, int row, int chunk)
{
    return *reinterpret_cast<const f32x4 *>(part + row * D * 4 + ((chunk ^ (row & (D / 4 - 1))) << 4));
}

// Rows joined over the waves that share them: eight elements at 8 * `at` of query row `row` (of 32 * WQ).
struct Joined {
    float ref, sum;
    float o[8];
};
template <typename G> __device__ __forceinline__ Joined joined(const char *smem, int row, int at)
{
    constexpr int D = G::D, WQ = G::WQ;
    const float *ml = reinterpret_cast<const float *>(smem + G::OFF_ML);
    const int wq = row >> 5, in = row & 31;
    Joined j;
    if constexpr (G::WK == 1) {
        j.ref = ml[wq * 32 + in];
        j.sum = ml[G::NW * 32 + wq * 32 + in];
        const f32x4 a = left_row<D>(smem + wq * 32 * D * 4, in, 2 * at), b = left_row<D>(smem + wq * 32 * D * 4, in, 2 * at + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            j.o[i] = a[i];
            j.o[4 + i] = b[i];
        }
        return j;
    }
    j.ref = -INFINITY;
#pragma unroll
    for (int k = 0; k < G::WK; ++k) j.ref = fmaxf(j.ref, ml[(k * WQ + wq) * 32 + in]);
    j.sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) j.o[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < G::WK; ++k) {
        const int wave = k * WQ + wq;
        const float m = ml[wave * 32 + in];
        if (m == -INFINITY) continue;                         // nothing was attended to (its values are zeros)
        const float f = __builtin_amdgcn_exp2f(m - j.ref);    // (NaN where scores were)
        j.sum = fmaf(f, ml[G::NW * 32 + wave * 32 + in], j.sum);
        const f32x4 a = left_row<D>(smem + wave * 32 * D * 4, in, 2 * at), b = left_row<D>(smem + wave * 32 * D * 4, in, 2 * at + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            j.o[i] = fmaf(f, a[i], j.o[i]);
            j.o[4 + i] = fmaf(f, b[i], j.o[4 + i]);
        }
    }
    return j;
}

// Calls emit(row, Joined, eight) for all query rows of the workgroup, a lane for every eight elements.  Rows that no waves share are taken by the wave
// that left them; for the others all waves have to be here first.
template <typename G, typename EMIT> __device__ __forceinline__ void emit_rows(const char *smem, EMIT &&emit)
{
    constexpr int LANES = G::D / 8;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if constexpr (G::WK == 1) {
#pragma unroll 4
        for (int k = 0; k < 32 * LANES / 64; ++k) {
            const int row = wave * 32 + k * (64 / LANES) + lane / LANES;
            emit(row, joined<G>(smem, row, lane % LANES), lane % LANES);
        }
    } else {
        __syncthreads();
#pragma unroll 2
        for (int k = 0; k < G::QROWS * LANES / G::THREADS; ++k) {
            const int row = k * (G::THREADS / LANES) + tid / LANES;
            emit(row, joined<G>(smem, row, tid % LANES), tid % LANES);
        }
    }
}

// log-sum-exp of a row.
template <bool F16> __device__ __forceinline__ float log_sum(float ref, float sum)
{
    return sum == 0.0f ? -INFINITY : (ref - Half<F16>::HEAD + __builtin_amdgcn_logf(sum)) * LN2;
}

// Eight elements of a finished row.
template <bool F16> __device__ __forceinline__ void store_row(float *out, void *out_lowp, int64_t element, const float (&o)[8], float by)
{
    if (out) {
        const f32x4 a = {o[0] * by, o[1] * by, o[2] * by, o[3] * by}, b = {o[4] * by, o[5] * by, o[6] * by, o[7] * by};
        *reinterpret_cast<f32x4 *>(out + element) = a;
        *reinterpret_cast<f32x4 *>(out + element + 4) = b;
    }
    if (out_lowp) {
        const u32x4 x = {pack2<F16>(o[0] * by, o[1] * by), pack2<F16>(o[2] * by, o[3] * by), pack2<F16>(o[4] * by, o[5] * by), pack2<F16>(o[6] * by, o[7] * by)};
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(out_lowp) + element) = x;
    }
}

// Where the keys and values of one kv head lie: `count` ranks of the cache - the entries of a list of positions, of chunks or of pool slots,
// or positions themselves - and behind them, in a tile of their own, `nodes` rows of new tokens.  A rank beyond the last one reads the last
// one's row, an entry outside the cache the nearest row inside it: what is read always belongs to the call.
struct CacheRows {
    const char *k, *v;
    uint32_t step_n, step_page;                               // between rows and between pages, in units of 16 bytes
    const int32_t *list;                                      // null: rank = position
    const int32_t *table;                                     // the sequence's pages, or null
    int chunk_shift, page_shift, pages;                       // pages 0: contiguous
    int slots;                                                // positions (or pool slots) there are
    int count;
    const char *k_new, *v_new;
    int nodes;

    __device__ __forceinline__ int word(int rank) const { return list ? list[rank >> chunk_shift] : rank; }
    __device__ __forceinline__ int position(int rank, int w) const
    {
        if (list && chunk_shift) {
            w = min(max(w, 0), (slots - 1) >> chunk_shift);
            w = (w << chunk_shift) | (rank & ((1 << chunk_shift) - 1));
        }
        return min(max(w, 0), slots - 1);
    }
    __device__ __forceinline__ int page(int pos) const { return table ? table[pos >> page_shift] : pages ? pos >> page_shift : 0; }
    // where a row begins, in units of 16 bytes (the host sees to it that these fit in 32 bits)
    __device__ __forceinline__ uint32_t unit(int pos, int pg) const
    {
        if (!pages) return (uint32_t)pos * step_n;
        return (uint32_t)min(max(pg, 0), pages - 1) * step_page + (uint32_t)(pos & ((1 << page_shift) - 1)) * step_n;
    }
};

// Tiles [first, last) of the rows that `where()` tells (asked again for every batch of tiles, so that not all of it is held throughout) for this workgroup, of which this wave computes those below `own`; the tiles behind `cached` hold the new tokens.
// `seen(tile, word)`: whether this wave's rows see all of its part of the tile; if not, word has a bit for each position that this lane's row sees.  LOOKUP: rows are found through lists or pages, many tiles' at a time ahead of the first of them, and wait in LDS; otherwise a rank is a position
// of a contiguous cache.  On return every wave is done with the tile buffers.
template <typename G, bool F16, int PARTS, bool LOOKUP, typename WHERE, typename SEEN>
__device__ __forceinline__ void run_tiles(RowsOfWave<G, F16, PARTS> &rows, WHERE &&where, int first, int last, int cached, int own, char *smem, SEEN &&seen)
{
    constexpr int N = G::LOADS, S = G::STAGES, STEP = G::NW * G::RPI;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t to = lds_address(smem) + wave * 1024;
    const int row0 = wave * G::RPI + lane / G::CHUNKS;        // this lane's first row of a tile; the others lie STEP apart
    uint32_t *table = reinterpret_cast<uint32_t *>(smem + G::OFF_TABLE);
    int chunk[N];
#pragma unroll
    for (int i = 0; i < N; ++i) chunk[i] = ((lane & (G::CHUNKS - 1)) ^ G::swz(row0 + i * STEP)) * 16;
    for (int base = first; base < last; base += G::BATCH) {
        const int end = min(last, base + G::BATCH);
        const CacheRows src = where();
        if (LOOKUP) {
            constexpr int E = G::BATCH * G::TILE / G::THREADS;
            const int from = base * G::TILE, n = (min(end, cached) - base) * G::TILE;
            int at[E];
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i * G::THREADS < n) at[i] = src.word(min(from + i * G::THREADS + tid, src.count - 1));
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i * G::THREADS < n) at[i] = src.position(min(from + i * G::THREADS + tid, src.count - 1), at[i]);
            int page[E];
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i * G::THREADS < n) page[i] = src.page(at[i]);
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i * G::THREADS < n) table[i * G::THREADS + tid] = src.unit(at[i], page[i]);
            __syncthreads();
        }
        auto ask = [&](int t) {
            uint32_t unit[N];
            const bool old = t < cached;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int row = row0 + i * STEP;
                if (!old) unit[i] = (uint32_t)min(row, max(src.nodes, 1) - 1) * (G::ROW_BYTES / 16);
                else if (LOOKUP) unit[i] = table[(t - base) * G::TILE + row];
                else unit[i] = src.unit(min(t * G::TILE + row, src.count - 1), 0);
            }
            const char *k = old ? src.k : src.k_new, *v = old ? src.v : src.v_new;
            const uint32_t buf = to + (t & (S - 1)) * G::STAGE_BYTES;
#pragma unroll
            for (int i = 0; i < N; ++i) load_to_lds(k + ((uint64_t)unit[i] * 16 + chunk[i]), buf + i * G::NW * 1024);
#pragma unroll
            for (int i = 0; i < N; ++i) load_to_lds(v + ((uint64_t)unit[i] * 16 + chunk[i]), buf + G::TILE_BYTES + i * G::NW * 1024);
        };
        for (int t = base; t < min(end, base + S - 1); ++t) ask(t);
        // (the queries are waited for here: left to the place where they are used first, the wait would stand inside the loop)
#pragma unroll
        for (int c = 0; c < G::D / 16; ++c) {
            u32x4 x = __builtin_bit_cast(u32x4, rows.q[c]);
            asm volatile("" : "+v"(x));
            rows.q[c] = __builtin_bit_cast(typename Half<F16>::x8, x);
        }
        const int mine = min(end, own);                       // tiles that this wave has rows for
        auto top = [&](int t) {
            tile_barrier_behind<2 * N, S - 2>(min(end - 1 - t, S - 2));
            if (t + S - 1 < end) ask(t + S - 1);
        };
        int t = base;
        for (; t < mine; ++t) {
            top(t);
            const char *buf = smem + (t & (S - 1)) * G::STAGE_BYTES;
            rows.score(buf);
            const auto ready = rows.values(buf, 0);
            rows.weigh(seen, t);
            rows.add(buf, ready);
        }
        for (; t < end; ++t) top(t);
        tile_barrier<0>();
    }
}

// Rows of this wave that an infinity or NaN among the values has come into, from a place that their mask hides (0 * infinity) or one that they see, or whose
// unnormalised values came close to the end of fp32: once more, all of them together, from what they attend to alone.  Runs behind leave(), over the same tiles, for one wave by
// itself: fragments come straight from memory, 32 elements at a time.  In the product, values that are not finite count as 0; beside it, plus and minus count those that
// a row gives a weight to (a NaN as both, and so anything of weight 0 that is seen, as 0 * infinity is NaN).  bf16 weights are taken in units in which a row's add up to
// less than 2^-MORE; with fp16 no sum comes near the end of fp32.
// `seen(tile, row)`: the positions that a row of the wave sees.
// With an infinity in the first value of one causal prompt, which sends every row here: 2048 tokens, 8 heads over 2, bf16 150 us (42 without it), 32768 tokens, 32
// heads over 8 73 ms (8.2).
template <typename G, bool F16, int PARTS, typename SEEN>
__device__ __forceinline__ void mend_rows(uint64_t which, const RowsOfWave<G, F16, PARTS> &rows, const CacheRows &src, int first, int last, int cached, int wk, char *smem, SEEN seen)
{
    constexpr int D = G::D;
    constexpr uint32_t INF = F16 ? 0x7c00 : 0x7f80, ONE = F16 ? 0x3c00 : 0x3f80, SIGN = 0x8000;
    typedef typename Half<F16>::x8 x8;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                             // (what follows from it is not computed ahead, for rows that are not mended)
    const int lane = tid & 63, wave = tid >> 6, row = lane & 31, half = lane >> 5;
    float *ml = reinterpret_cast<float *>(smem + G::OFF_ML) + wave * 32;
    char *mine = smem + wave * 32 * D * 4;
    const bool bad = (((uint32_t)which | (uint32_t)(which >> 32)) >> row) & 1;
    const float ref = ml[row], sum = ml[G::NW * 32 + row];
    const int scale = F16 ? 0 : __builtin_amdgcn_frexp_expf(sum) + MORE;
    const float from = Half<F16>::HEAD - ref, by = __builtin_ldexpf(1.0f, -scale);
#pragma unroll 1
    for (int e = 0; e < D / 32; ++e) {
        f32x16 o{}, plus{}, minus{};
#pragma unroll 1
        for (int t = first; t < last; ++t) {
            const uint64_t word = bad ? seen(t, row) : 0;
            const bool old = t < cached;
#pragma unroll 1
            for (int u = 0; u < G::SUBS; ++u) {
                const uint32_t bits = (uint32_t)(word >> (32 * u));
                if (!__any(bits != 0)) continue;
                const int in = wk * G::SPAN + 32 * u + row;
                uint32_t unit;                                // where the row of position `row` of these 32 lies
                if (old) {
                    const int rank = min(t * G::TILE + in, src.count - 1);
                    const int pos = src.position(rank, src.word(rank));
                    unit = src.unit(pos, src.page(pos));
                } else unit = (uint32_t)min(in, max(src.nodes, 1) - 1) * (G::ROW_BYTES / 16);
                const char *k = (old ? src.k : src.k_new) + ((uint64_t)unit * 16 + half * 16), *v = (old ? src.v : src.v_new) + (32 * e + row) * 2;
                f32x16 s{};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) s = Half<F16>::mfma(*reinterpret_cast<const x8 *>(k + 32 * c), rows.q[c], s);
#pragma unroll
                for (int b = 0; b < 2; ++b) {                 // 16 positions
                    uint32_t x[8], odd = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const uint16_t *>(v + (uint64_t)(uint32_t)__shfl((int)unit, 16 * b + 8 * (i / 4) + 4 * half + i % 4) * 16);
                    u32x4 value, more, less, hi, lo, live, dead;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float w[2];
                        uint32_t f[2], m[2], l[2], on[2], off[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int n = 8 * b + 2 * i + j;
                            const bool sees = (bits >> (8 * (n / 4) + 4 * half + n % 4)) & 1;
                            w[j] = sees ? __builtin_amdgcn_exp2f(fmaf(s[n], rows.scale, from)) * by : 0.0f;
                            const uint32_t y = x[2 * i + j];
                            const bool wild = (y & INF) == INF;
                            odd |= wild;
                            f[j] = wild ? 0 : y;
                            m[j] = wild && y != (SIGN | INF) ? ONE : 0;
                            l[j] = wild && y != INF ? ONE : 0;
                            on[j] = w[j] > 0.0f ? ONE : 0;
                            off[j] = sees && !(w[j] > 0.0f) ? ONE : 0;
                        }
                        value[i] = f[0] | f[1] << 16;
                        more[i] = m[0] | m[1] << 16;
                        less[i] = l[0] | l[1] << 16;
                        live[i] = on[0] | on[1] << 16;
                        dead[i] = off[0] | off[1] << 16;
                        hi[i] = pack2<F16>(w[0], w[1]);
                        lo[i] = pack2<F16>(w[0] - Half<F16>::widen((uint16_t)hi[i]), w[1] - Half<F16>::widen((uint16_t)(hi[i] >> 16)));
                    }
                    o = Half<F16>::mfma(__builtin_bit_cast(x8, value), __builtin_bit_cast(x8, hi), o);
                    o = Half<F16>::mfma(__builtin_bit_cast(x8, value), __builtin_bit_cast(x8, lo), o);
                    if (__any(odd)) {
                        const x8 any = __builtin_bit_cast(x8, more | less);
                        plus = Half<F16>::mfma(__builtin_bit_cast(x8, more), __builtin_bit_cast(x8, live), plus);
                        minus = Half<F16>::mfma(__builtin_bit_cast(x8, less), __builtin_bit_cast(x8, live), minus);
                        plus = Half<F16>::mfma(any, __builtin_bit_cast(x8, dead), plus);
                        minus = Half<F16>::mfma(any, __builtin_bit_cast(x8, dead), minus);
                    }
                }
            }
        }
        if (!bad) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = 4 * j + i;
                x[i] = o[n] + (plus[n] > 0.0f ? INFINITY : 0.0f) + (minus[n] > 0.0f ? -INFINITY : 0.0f);
            }
            *reinterpret_cast<f32x4 *>(mine + row * D * 4 + (((8 * e + 2 * j + half) ^ (row & (D / 4 - 1))) << 4)) = x;
        }
    }
    if (!F16 && bad && half == 0) {
        ml[row] = ref + scale;
        ml[G::NW * 32 + row] = sum * by;
    }
}

// Eight elements of a partial result.
template <int D> __device__ __forceinline__ void leave_slot(float *rows, float *ml, int64_t slot, int qrows, int c, int e, const Joined &j)
{
    float *x = rows + (slot * qrows + c) * D + 8 * e;
    *reinterpret_cast<f32x4 *>(x) = f32x4{j.o[0], j.o[1], j.o[2], j.o[3]};
    *reinterpret_cast<f32x4 *>(x + 4) = f32x4{j.o[4], j.o[5], j.o[6], j.o[7]};
    if (e == 0) {
        ml[slot * 2 * qrows + c] = reference(j.ref, j.sum);
        ml[slot * 2 * qrows + qrows + c] = j.sum;
    }
}

// Query rows that a wave of a merge kernel joins: four, whose loads go together, where units are so many that each is in few parts; one otherwise.
constexpr int MERGE_ROWS = 4;

// Query rows of n partial results, the first in slot `head`, part i in slot base + i * step ([slot][qrows][D] unnormalised, references and sums [slot][2][qrows]), joined by one
// wave: D / 8 lanes take a slot's row, eight elements each, and 512 / D slots go side by side; the order of all sums is fixed.  Every lane gets the
// total and the elements of its place.
template <int D> struct Slots {
    static constexpr int LANES = D / 8, SIDE = 64 / LANES;
    const float *rows, *ml;
    int64_t head, base;
    int step, n, qrows;

    __device__ __forceinline__ int64_t slot(int i) const { return i == 0 ? head : base + i * step; }
    __device__ __forceinline__ void together(Joined &j) const // over the slots that lie side by side
    {
#pragma unroll
        for (int step = LANES; step < 64; step *= 2) {
            j.sum += __shfl_xor(j.sum, step);
#pragma unroll
            for (int i = 0; i < 8; ++i) j.o[i] += __shfl_xor(j.o[i], step);
        }
    }
    // Up to SIDE slots: N rows' loads under way together.
    template <int N> __device__ __forceinline__ void few(const int (&c)[N], Joined (&j)[N]) const
    {
        const int lane = threadIdx.x & 63, e = lane % LANES, side = lane / LANES;
        const int64_t at = slot(min(side, n - 1));
        f32x4 x[N], y[N];
        float m[N], l[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            m[k] = ml[at * 2 * qrows + c[k]];
            l[k] = ml[at * 2 * qrows + qrows + c[k]];
            x[k] = *reinterpret_cast<const f32x4 *>(rows + (at * qrows + c[k]) * D + 8 * e);
            y[k] = *reinterpret_cast<const f32x4 *>(rows + (at * qrows + c[k]) * D + 8 * e + 4);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float mine = side < n ? m[k] : -INFINITY;
            j[k].ref = mine;
#pragma unroll
            for (int step = LANES; step < 64; step *= 2) j[k].ref = fmaxf(j[k].ref, __shfl_xor(j[k].ref, step));
            const float f = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - j[k].ref);
            const bool some = mine != -INFINITY;              // (nothing attended to: zeros)
            j[k].sum = some ? f * l[k] : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                j[k].o[i] = some ? f * x[k][i] : 0.0f;
                j[k].o[4 + i] = some ? f * y[k][i] : 0.0f;
            }
            together(j[k]);
        }
    }
    __device__ __forceinline__ Joined many(int c) const
    {
        const int lane = threadIdx.x & 63, e = lane % LANES, side = lane / LANES;
        Joined j;
        j.ref = -INFINITY;
        for (int i = lane; i < n; i += 64) j.ref = fmaxf(j.ref, ml[slot(i) * 2 * qrows + c]);
#pragma unroll
        for (int step = 32; step; step >>= 1) j.ref = fmaxf(j.ref, __shfl_xor(j.ref, step));
        j.sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) j.o[i] = 0.0f;
        constexpr int U = 4;                                  // slots that a lane asks for together
        for (int i0 = side; i0 < n; i0 += U * SIDE) {
            f32x4 x[U], y[U];
            float m[U], l[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = slot(min(i0 + u * SIDE, n - 1));
                const float *p = rows + (at * qrows + c) * D + 8 * e;
                m[u] = ml[at * 2 * qrows + c];
                l[u] = ml[at * 2 * qrows + qrows + c];
                x[u] = *reinterpret_cast<const f32x4 *>(p);
                y[u] = *reinterpret_cast<const f32x4 *>(p + 4);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * SIDE >= n || m[u] == -INFINITY) continue;
                const float f = __builtin_amdgcn_exp2f(m[u] - j.ref);
                j.sum = fmaf(f, l[u], j.sum);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    j.o[i] = fmaf(f, x[u][i], j.o[i]);
                    j.o[4 + i] = fmaf(f, y[u][i], j.o[4 + i]);
                }
            }
        }
        together(j);
        return j;
    }
    // Rows c0 .. c0 + N - 1 of at most `all`; done(row, Joined) is called for each.
    template <int N, typename DONE> __device__ __forceinline__ void join(int c0, int all, DONE &&done) const
    {
        if (c0 >= all) return;
        if (n > SIDE) {
            for (int k = 0; k < N && c0 + k < all; ++k) done(c0 + k, many(c0 + k));
            return;
        }
        int c[N];
        Joined j[N];
#pragma unroll
        for (int k = 0; k < N; ++k) c[k] = min(c0 + k, all - 1);
        few(c, j);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (c0 + k < all) done(c0 + k, j[k]);
    }
};
}  // namespace
}  // namespace specattn
