// C = alpha A B^T + beta C of two packed operands of microscaled 4-bit floating point, on the matrix instructions that take such
// operands with their scales (v_mfma_scale_f32_16x16x128_f8f6f4).
//
// Lane l of such an instruction holds one block of an operand: row l % 16, elements 32 (l / 16) .. + 31 of 128, sixteen bytes, and in
// one byte of a register the block's scale.  A packed operand holds its codes in that order, 1024 bytes an instruction, and its
// scales four row groups to a register, so a tile goes from memory to LDS and from there to registers as it lies, without a
// bank conflict.  The instruction's first operand is B's rows: then a lane holds four consecutive columns of one row of C.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "layers_device.h"

namespace conef {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// scale of the first operand in byte OA of sa, of the second in byte OB of sb; code 4: 4-bit floating point
template <int OA, int OB>
__device__ __forceinline__ f32x4 mfma_mx(v4i a, v4i b, f32x4 c, int sa, int sb)
{
    const v8i wa = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, wb = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, OA, sa, OB, sb);
}

template <typename F, int... I>
__device__ __forceinline__ void unroll_impl(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unroll(F &&f)
{
    unroll_impl(f, std::make_integer_sequence<int, N>{});
}

// alpha v (+ beta c), to four neighbours of a row of C
template <bool BF16>
__device__ __forceinline__ void store_four(const MxProductArgs &a, int64_t row, int64_t col, f32x4 v)
{
    const int64_t at = row * a.c.pitch + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (col + i >= a.n) return;
        float x = a.alpha * v[i];
        if constexpr (BF16) {
            uint16_t *p = static_cast<uint16_t *>(a.c.data) + at + i;
            if (a.beta != 0.0f) x = __builtin_fmaf(a.beta, bf16_bits_to_f32(*p), x);
            *p = (uint16_t)pack_bf16(x, x);
        } else {
            float *p = static_cast<float *>(a.c.data) + at + i;
            if (a.beta != 0.0f) x = __builtin_fmaf(a.beta, *p, x);
            *p = x;
        }
    }
}

// WM x WN waves of TM x TN tiles of 16 x 16; 128 elements of the long axis at a time.
template <bool BF16, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void k_mx_product(MxProductArgs a, int64_t pieces, int64_t a_groups, int64_t b_groups,
                                                             int64_t tiles_m)
{
    constexpr int kM = WM * TM * 16, kN = WN * TN * 16, kWaves = WM * WN;
    __shared__ __attribute__((aligned(16))) uint8_t lds[(kM + kN) * 64 + (kM + kN) * 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int64_t m0 = (int64_t)(blockIdx.x % tiles_m) * kM, n0 = (int64_t)(blockIdx.x / tiles_m) * kN;
    f32x4 acc[TN][TM] = {};
    for (int64_t kc = 0; kc < pieces; ++kc) {
        // a row group beyond the operand's last takes the last one's place: what comes of it is not stored
        for (int g = wave; g < (kM + kN) / 16; g += kWaves) {
            const bool is_a = g < kM / 16;
            const int64_t group = is_a ? min(m0 / 16 + g, a_groups - 1) : min(n0 / 16 + g - kM / 16, b_groups - 1);
            const uint8_t *src = (is_a ? a.a.codes : a.b.codes) + (group * pieces + kc) * 1024;
            *reinterpret_cast<v4i *>(lds + g * 1024 + lane * 16) = *reinterpret_cast<const v4i *>(src + lane * 16);
        }
        for (int g = wave; g < (kM + kN) / 64; g += kWaves) {
            const bool is_a = g < kM / 64;
            const int64_t group = is_a ? min(m0 / 64 + g, a_groups / 4 - 1) : min(n0 / 64 + g - kM / 64, b_groups / 4 - 1);
            const uint8_t *src = (is_a ? a.a.scales : a.b.scales) + (group * pieces + kc) * 256;
            *reinterpret_cast<int *>(lds + (kM + kN) * 64 + g * 256 + lane * 4) = *reinterpret_cast<const int *>(src + lane * 4);
        }
        __syncthreads();
        const uint8_t *la = lds + wm * TM * 1024 + lane * 16, *lb = lds + (kM / 16 + wn * TN) * 1024 + lane * 16;
        const uint8_t *sa = lds + (kM + kN) * 64 + wm * TM * 64 + lane * 4, *sb = lds + (kM + kN) * 64 + kM * 4 + wn * TN * 64 + lane * 4;
        v4i fa[TM], fb[TN];
        int ea[TM / 4], eb[TN / 4];
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = *reinterpret_cast<const v4i *>(la + i * 1024);
#pragma unroll
        for (int i = 0; i < TN; ++i) fb[i] = *reinterpret_cast<const v4i *>(lb + i * 1024);
#pragma unroll
        for (int i = 0; i < TM / 4; ++i) ea[i] = *reinterpret_cast<const int *>(sa + i * 256);
#pragma unroll
        for (int i = 0; i < TN / 4; ++i) eb[i] = *reinterpret_cast<const int *>(sb + i * 256);
        unroll<TN>([&](auto j) {
            unroll<TM>([&](auto i) {
                constexpr int I = decltype(i)::value, J = decltype(j)::value;
                acc[J][I] = mfma_mx<J % 4, I % 4>(fb[J], fa[I], acc[J][I], eb[J / 4], ea[I / 4]);
            });
        });
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + (wm * TM + i) * 16 + (lane & 15);
        if (row >= a.m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) store_four<BF16>(a, row, n0 + (wn * TN + j) * 16 + 4 * (lane >> 4), acc[j][i]);
    }
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace

size_t mx_product_workspace(int64_t m, int64_t n, int64_t k)
{
    (void)m; (void)n; (void)k;
    return 0;
}

void launch_mx_product(const MxProductArgs &a, bool bf16, hipStream_t st)
{
    const int64_t pieces = (a.k + 127) / 128, a_groups = (a.m + 63) / 64 * 4, b_groups = (a.n + 63) / 64 * 4;
    const int64_t tiles_m = (a.m + 127) / 128, tiles_n = (a.n + 127) / 128;
    by_bool(bf16, [&](auto b) {
        hipLaunchKernelGGL((k_mx_product<decltype(b)::value, 2, 2, 4, 4>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, st, a, pieces,
                           a_groups, b_groups, tiles_m);
    });
}

}  // namespace conef
