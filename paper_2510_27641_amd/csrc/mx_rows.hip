// Rows into the 4-bit cache and back out of it.
//
// A block of 32 elements x gets the scale 2^X, X = floor(log2(max |x|)) - 2, so that the largest magnitude lies in [4, 8)
// of it, and every element the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it.  The exponent comes from the bits of the
// largest magnitude as an integer, which orders infinities and NaNs above everything else; x * 2^-X is exact, and the
// hardware's conversion rounds half to even and takes what lies beyond 6 to 6.
//
// Bound by memory: 4 bytes read and 1.06 written per element pair of bf16.  A lane takes 8 consecutive elements, so that
// four lanes share a block and its largest magnitude is two lane moves away; the lanes of a position write its d bytes of codes
// as one piece.  4 sequences x 8 heads x 32768 positions of d = 128 in bf16, 0.68 GB: into the cache 119 us (5.7 TB/s), out of it 100 us
// (6.8 TB/s; a plain read reaches 6.8, a copy 4.8).
#include "mx.h"

#include <algorithm>

namespace specattn {
namespace {

constexpr int THREADS = 256;

template <int DTYPE> struct Elem;
template <> struct Elem<SPECATTN_F32> { static constexpr int BYTES = 4; };
template <> struct Elem<SPECATTN_BF16> { static constexpr int BYTES = 2; };
template <> struct Elem<SPECATTN_F16> { static constexpr int BYTES = 2; };

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as they lie in memory, and in fp32.
template <int DTYPE> struct Eight { u32x4 w[Elem<DTYPE>::BYTES / 2]; };
template <int DTYPE> __device__ __forceinline__ Eight<DTYPE> load_eight(const void *p, int64_t element)
{
    Eight<DTYPE> e;
    const u32x4 *src = reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(p) + element * Elem<DTYPE>::BYTES);
#pragma unroll
    for (int i = 0; i < Elem<DTYPE>::BYTES / 2; ++i) e.w[i] = __builtin_nontemporal_load(src + i);
    return e;
}
template <int DTYPE> __device__ __forceinline__ void widen(const Eight<DTYPE> &e, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (DTYPE == SPECATTN_F32) x[i] = __uint_as_float(e.w[i / 4][i % 4]);
        else {
            const uint16_t half = (uint16_t)(e.w[0][i / 2] >> (16 * (i % 2)));
            x[i] = DTYPE == SPECATTN_BF16 ? __uint_as_float((uint32_t)half << 16) : (float)__builtin_bit_cast(_Float16, half);
        }
    }
}
template <int DTYPE> __device__ __forceinline__ void store_eight(void *p, int64_t element, const float (&x)[8])
{
    u32x4 *dst = reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(p) + element * Elem<DTYPE>::BYTES);
    if constexpr (DTYPE == SPECATTN_F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 w = {__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3])};
            __builtin_nontemporal_store(w, dst + i);
        }
    } else {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2_t pair = {x[2 * i], x[2 * i + 1]};
            if constexpr (DTYPE == SPECATTN_BF16) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2));
            else w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, f16x2));
        }
        __builtin_nontemporal_store(w, dst);
    }
}

// Byte offsets of slot `slot` of (b, h) in the codes and the scales; false if there is no such slot.
__device__ __forceinline__ bool slot_offsets(const MxCache &c, int b, int h, int64_t slot, int64_t &codes, int64_t &scales)
{
    if (slot < 0 || slot >= c.n_max) return false;
    if (!c.page_table) {
        codes = b * c.codes_b + h * c.codes_h + slot * c.codes_n;
        scales = b * c.scales_b + h * c.scales_h + slot * c.scales_n;
        return true;
    }
    const int64_t page = c.page_table[(int64_t)b * c.max_pages + (slot >> c.page_shift)];
    const int64_t in = slot & ((1 << c.page_shift) - 1);
    codes = page * c.codes_page + h * c.codes_h + in * c.codes_n;
    scales = page * c.scales_page + h * c.scales_h + in * c.scales_n;
    return page >= 0 && page < c.num_pages;
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v)      // over four neighbouring lanes
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true));     // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
}

// Scale byte of the block that four lanes hold, and the codes of this lane's eight elements.
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t &codes)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = quad_max(top);
    codes = 0;
    if (top >= 0x7f800000u) return 255;
    const int scale = max((int)(top >> 23) - 2, 0);               // X + 127 (largest: 252)
    const float inverse = __uint_as_float((uint32_t)(254 - scale) << 23);      // 2^-X
#define SPECATTN_PAIR(I) codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2 * I] * inverse, x[2 * I + 1] * inverse, 1.0f, I)
    SPECATTN_PAIR(0); SPECATTN_PAIR(1); SPECATTN_PAIR(2); SPECATTN_PAIR(3);
#undef SPECATTN_PAIR
    return (uint32_t)scale;
}

// 2^(byte - 127): below the normal numbers for byte 0, NaN for byte 255
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}

// A workgroup takes THREADS / LANES * U rows of one (b, h); a row takes D / 4 lanes, first those of its keys, then those
// of its values.
template <int D, int DTYPE, int U, bool LOAD> __global__ __launch_bounds__(THREADS) void mx_rows_kernel(MxRowsLaunch a)
{
    constexpr int LANES = D / 4, ROWS = THREADS / LANES;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const bool value = lane >= LANES / 2;
    const int at = lane % (LANES / 2);                            // eight elements at 8 * at of the row
    void *side = value ? a.v : a.k;
    const int rows = a.c.B * a.c.H_kv;
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        const int b = r / a.c.H_kv, h = r - b * a.c.H_kv;
        const int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
        const int64_t start = a.starts ? a.starts[b] : 0;
        const int first = blockIdx.x * ROWS * U + sub;
        const int64_t base = b * a.stride_b + h * a.stride_h + 8 * at;
        int64_t codes[U], scales[U];
        bool there[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = first + u * ROWS;
            there[u] = t < count && slot_offsets(a.c, b, h, start + t, codes[u], scales[u]);
            if (!there[u]) codes[u] = scales[u] = 0;
        }
        if constexpr (!LOAD) {
            // (rows that are left out: others instead, so that all requests go out together; behind a condition each: 154 us for 125)
            Eight<DTYPE> e[U];
#pragma unroll
            for (int u = 0; u < U; ++u) e[u] = load_eight<DTYPE>(side, base + min(first + u * ROWS, a.T - 1) * a.stride_t);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!there[u]) continue;                          // (the four lanes of a block together)
                float x[8];
                widen<DTYPE>(e[u], x);
                uint32_t word;
                const uint32_t scale = quantise(x, word);
                *reinterpret_cast<uint32_t *>(a.c.codes + codes[u] + 4 * lane) = word;
                // the four blocks of 16 lanes make a word
                uint32_t four = scale << lane / 4 % 4 * 8;
                four |= (uint32_t)__builtin_amdgcn_update_dpp(0, four, 0x124, 0xf, 0xf, true);      // four lanes on in the row of 16
                four |= (uint32_t)__builtin_amdgcn_update_dpp(0, four, 0x128, 0xf, 0xf, true);      // and eight
                if (lane % 16 == 0) *reinterpret_cast<uint32_t *>(a.c.scales + scales[u] + lane / 4) = four;
            }
        } else {
            uint32_t word[U], scale[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                word[u] = *reinterpret_cast<const uint32_t *>(a.c.codes + codes[u] + 4 * lane);
                scale[u] = a.c.scales[scales[u] + lane / 4];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!there[u]) continue;
                const float s = scale_value(scale[u]);
                float x[8];
#define SPECATTN_PAIR(I) { const f32x2_t p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[u], 1.0f, I); x[2 * I] = p[0] * s; x[2 * I + 1] = p[1] * s; }
                SPECATTN_PAIR(0) SPECATTN_PAIR(1) SPECATTN_PAIR(2) SPECATTN_PAIR(3)
#undef SPECATTN_PAIR
                store_eight<DTYPE>(side, base + (first + u * ROWS) * a.stride_t, x);
            }
        }
    }
}

template <int D, int DTYPE, bool LOAD> specattn_status launch_rows(const MxRowsLaunch &a, hipStream_t stream)
{
    constexpr int ROWS = THREADS / (D / 4);
    constexpr int U = 4;
    const int rows = std::min(a.c.B * a.c.H_kv, 65535);
    if (a.T <= ROWS) mx_rows_kernel<D, DTYPE, 1, LOAD><<<dim3(1, rows), THREADS, 0, stream>>>(a);
    else mx_rows_kernel<D, DTYPE, U, LOAD><<<dim3((a.T + ROWS * U - 1) / (ROWS * U), rows), THREADS, 0, stream>>>(a);
    return check_launch(LOAD ? "mx_rows_kernel (load)" : "mx_rows_kernel (store)");
}

template <bool LOAD> specattn_status launch_any(const MxRowsLaunch &a, hipStream_t stream)
{
    if (a.c.d == 128)
        return a.dtype == SPECATTN_F32 ? launch_rows<128, SPECATTN_F32, LOAD>(a, stream)
             : a.dtype == SPECATTN_BF16 ? launch_rows<128, SPECATTN_BF16, LOAD>(a, stream) : launch_rows<128, SPECATTN_F16, LOAD>(a, stream);
    return a.dtype == SPECATTN_F32 ? launch_rows<64, SPECATTN_F32, LOAD>(a, stream)
         : a.dtype == SPECATTN_BF16 ? launch_rows<64, SPECATTN_BF16, LOAD>(a, stream) : launch_rows<64, SPECATTN_F16, LOAD>(a, stream);
}

}  // namespace

specattn_status launch_mx_store(const MxRowsLaunch &a, hipStream_t stream) { return launch_any<false>(a, stream); }
specattn_status launch_mx_load(const MxRowsLaunch &a, hipStream_t stream) { return launch_any<true>(a, stream); }

}  // namespace specattn
