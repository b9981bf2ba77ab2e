// A tile in LDS that is read by columns.
#pragma once
#include <type_traits>

#include "layers_device.h"

namespace conef {

// 128 rows of 64 columns in LDS, for reading eight rows of a column.  bf16: by transposing reads, sixteen lanes 4 rows x 16 columns at a
// time; a row has half the banks, and where in it a piece of 16 columns lies goes by the row, so that the eight rows that half a
// wave reads from lie in banks of their own.  fp32: element by element.
template <bool BF16>
struct Turned {
    static constexpr int kPitch = BF16 ? 64 : 66;
    typedef std::conditional_t<BF16, uint16_t, float> Elem;
    Elem e[128 * kPitch];

    static __device__ __forceinline__ int piece(int row, int col) { return ((col >> 4) ^ (row >> 1 & 1) ^ (row >> 2 & 2)) << 4; }

    __device__ __forceinline__ void put(int row, int col, const Octet<BF16> &o)
    {
        if constexpr (BF16) {
            *reinterpret_cast<uint4 *>(e + row * kPitch + piece(row, col) + (col & 8)) = make_uint4(o.w[0][0], o.w[0][1], o.w[0][2], o.w[0][3]);
        } else {
            uint2 *p = reinterpret_cast<uint2 *>(e + row * kPitch + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = make_uint2(o.w[i >> 1][2 * (i & 1)], o.w[i >> 1][2 * (i & 1) + 1]);
        }
    }

    // rows row .. row + 7 (row: a multiple of 8, the same for 16 lanes) of column col + lane % 16
    __device__ __forceinline__ Octet<BF16> get(int row, int col, int lane) const
    {
        Octet<BF16> o;
        if constexpr (BF16) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int from = row + (lane >> 2 & 3);
            const Elem *p = e + from * kPitch + piece(from, col) + 4 * (lane & 3);          // (the row four on has the same place)
            union { s16x4 v; uint2 u; } lo, hi;
            lo.v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
            hi.v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * kPitch));
            o.w[0] = u32x4_any{lo.u.x, lo.u.y, hi.u.x, hi.u.y};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) o.w[i >> 2][i & 3] = __float_as_uint(e[(row + i) * kPitch + col + (lane & 15)]);
        }
        return o;
    }
};

}  // namespace conef
