// Device helpers of the operators of a training step: octets of rows of any alignment, draws of an octet, sums over a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"
#include "layers.h"

namespace conef {

// Workgroups of a launch that may need more of them than one axis of a grid counts (fewer than 2^32 threads): rows of 2^21, of up to 1024
// threads each.  The last row may have some that are nobody's.
constexpr int kGridRow = 21;
inline dim3 grid_of(int64_t groups)
{
    const int64_t row = (int64_t)1 << kGridRow;
    return groups <= row ? dim3((unsigned)groups) : dim3((unsigned)row, (unsigned)((groups + row - 1) >> kGridRow));
}
__device__ __forceinline__ uint32_t group_index() { return blockIdx.x + (blockIdx.y << kGridRow); }

// Sixteen bytes at any address that an element may have: the hardware takes them in one access.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};          // to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint32_t, v);
}

// elements of an octet with `left` of its row from it on, 0 to 8
__device__ __forceinline__ int octet_left(int64_t left) { return left >= 8 ? 8 : left > 0 ? (int)left : 0; }

// An octet as it lies in memory.
template <bool BF16>
struct Octet {
    u32x4_any w[BF16 ? 1 : 2];
};

// `left` elements (8 or more: all) of the octet that starts at element `at`; the others are 0.  Of an octet that its row does not fill
// every element is loaded on its own, all of them at once: those beyond the end are the last one again, and not taken.
template <bool BF16>
__device__ __forceinline__ Octet<BF16> fetch_octet(const void *data, int64_t at, int left)
{
    Octet<BF16> o = {};
    if constexpr (BF16) {
        const uint16_t *p = static_cast<const uint16_t *>(data) + at;
        if (left >= 8) {
            o.w[0] = *reinterpret_cast<const u32x4_any *>(p);
        } else if (left > 0) {
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = p[i < left ? i : left - 1];
#pragma unroll
            for (int i = 0; i < 8; ++i) o.w[0][i >> 1] |= i < left ? e[i] << (16 * (i & 1)) : 0u;
        }
    } else {
        const float *p = static_cast<const float *>(data) + at;
        if (left >= 8) {
            o.w[0] = *reinterpret_cast<const u32x4_any *>(p);
            o.w[1] = *reinterpret_cast<const u32x4_any *>(p + 4);
        } else if (left > 0) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = p[i < left ? i : left - 1];
#pragma unroll
            for (int i = 0; i < 8; ++i) o.w[i >> 2][i & 3] = i < left ? __float_as_uint(e[i]) : 0u;
        }
    }
    return o;
}

// The same for rows of 8 columns at least, in two steps, so that loads can be under way while other work is done: an octet that its row does not
// fill is fetched as what lies in the row's last sixteen (thirty-two) bytes, and moved down when it is used.
template <bool BF16>
__device__ __forceinline__ void begin_octet(Octet<BF16> &o, const void *data, int64_t at, int left)
{
    if (left <= 0) return;
    at -= left < 8 ? 8 - left : 0;
    if constexpr (BF16) {
        o.w[0] = *reinterpret_cast<const u32x4_any *>(static_cast<const uint16_t *>(data) + at);
    } else {
        const float *p = static_cast<const float *>(data) + at;
        o.w[0] = *reinterpret_cast<const u32x4_any *>(p);
        o.w[1] = *reinterpret_cast<const u32x4_any *>(p + 4);
    }
}

// its elements; those beyond the row's end are 0
template <bool BF16>
__device__ __forceinline__ void finish_octet(const Octet<BF16> &o, int left, float v[8])
{
    constexpr int N = BF16 ? 4 : 8;
    uint32_t w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = o.w[i >> 2][i & 3];
    if (left < 8) {
        const int s = left > 0 ? 8 - left : 8, words = BF16 ? s >> 1 : s;
#pragma unroll
        for (int step = N; step; step /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = words & step ? (i + step < N ? w[i + step] : 0u) : w[i];
        if constexpr (BF16) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = s & 1 ? (w[i] >> 16 | (i + 1 < N ? w[i + 1] << 16 : 0u)) : w[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BF16) v[i] = __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
        else v[i] = __uint_as_float(w[i]);
    }
}

template <bool BF16>
__device__ __forceinline__ void widen(const Octet<BF16> &o, float v[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BF16) v[i] = __uint_as_float((i & 1) ? o.w[0][i >> 1] & 0xFFFF0000u : o.w[0][i >> 1] << 16);
        else v[i] = __uint_as_float(o.w[i >> 2][i & 3]);
    }
}

template <bool BF16>
__device__ __forceinline__ void load_octet(const void *data, int64_t at, int left, float v[8])
{
    widen<BF16>(fetch_octet<BF16>(data, at, left), v);
}

// sixteen bytes to any address; PAST: past the caches
template <bool PAST>
__device__ __forceinline__ void store_16(void *p, u32x4_any v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, static_cast<u32x4_any *>(p));
    else *static_cast<u32x4_any *>(p) = v;
}

// Writes the octet's first `left` elements; v becomes what has been written (rounded to bf16 where the elements are).
template <bool BF16, bool PAST = false>
__device__ __forceinline__ void store_octet(void *data, int64_t at, int left, float v[8])
{
    if constexpr (BF16) {
        uint16_t *p = static_cast<uint16_t *>(data) + at;
        u32x4_any u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
        }
        if (left >= 8) {
            store_16<PAST>(p, u);
        } else if (left > 0) {
            // four, two, one
            typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
            typedef uint32_t u32_any __attribute__((aligned(2)));
            if (left & 4) *reinterpret_cast<u32x2_any *>(p) = u32x2_any{u[0], u[1]};
            const uint32_t a = left & 4 ? u[2] : u[0], b = left & 4 ? u[3] : u[1];
            p += left & 4;
            if (left & 2) *reinterpret_cast<u32_any *>(p) = a;
            if (left & 1) p[left & 2] = (uint16_t)(left & 2 ? b : a);
        }
    } else {
        float *p = static_cast<float *>(data) + at;
        u32x4_any a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = __float_as_uint(v[i]);
            b[i] = __float_as_uint(v[4 + i]);
        }
        if (left >= 8) {
            store_16<PAST>(p, a);
            store_16<PAST>(p + 4, b);
        } else if (left > 0) {
            typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(4)));
            if (left & 4) store_16<false>(p, a);
            // (of the vectors, not of v: a choice between places of v would put v into memory)
            const uint32_t c = left & 4 ? b[0] : a[0], d = left & 4 ? b[1] : a[1], e = left & 4 ? b[2] : a[2];
            p += left & 4;
            if (left & 2) *reinterpret_cast<u32x2_any *>(p) = u32x2_any{c, d};
            if (left & 1) p[left & 2] = __uint_as_float(left & 2 ? e : c);
        }
    }
}

// the four words that hold the eight 16-bit draws of an octet
__device__ __forceinline__ void octet_draws(const Draws &d, uint32_t octet, uint32_t out[4])
{
    philox4x32_10(octet, d.word, d.step_lo, d.step_hi, d.seed_lo, d.seed_hi, out);
}

// v <- v * scale where it is kept, else 0
__device__ __forceinline__ void drop_octet(const DropArgs &d, uint32_t octet, float v[8])
{
    uint32_t u[4];
    octet_draws(d.draws, octet, u);
    const uint32_t high = d.threshold << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (u[i] << 16) >= high ? v[2 * i] * d.scale : 0.0f;
        v[2 * i + 1] = u[i] >= high ? v[2 * i + 1] * d.scale : 0.0f;
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// sum over each G lanes of a wave, in every one of them: quads, halves and wholes of a row of 16, then across the rows
template <int G>
__device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(G == 8 || G == 16 || G == 32 || G == 64, "");
    v += dpp<0xB1>(v);          // lane ^ 1
    v += dpp<0x4E>(v);          // lane ^ 2
    v += dpp<0x141>(v);         // the other quad of a half row
    if constexpr (G >= 16) v += dpp<0x140>(v);         // the other half row
    if constexpr (G >= 32) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (G == 64) {
        auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// sum over the 64 / G lanes of a wave with the same place in their G, in every one of them
template <int G>
__device__ __forceinline__ float places_sum(float v)
{
    if constexpr (G <= 8) v += dpp<0x128>(v);          // half a row on
    if constexpr (G <= 16) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (G <= 32) {
        auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

}  // namespace conef
