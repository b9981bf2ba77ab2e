// Quantisation to microscaled 4-bit floating point and back.
//
// A block of 32 consecutive elements of a row shares a scale 2^s (one byte, s + 127); an element is a sign and one of 0, 0.5, 1,
// 1.5, 2, 3, 4, 6, times the scale.  With e = floor(log2(largest magnitude of the block)):
//   to nearest   s = e - 2, so that magnitudes over the scale are below 8; ties go to the even code, those above 6 to 6;
//   stochastic   s = e - 2, or e - 1 where the largest is above 6 * 2^(e - 2): nothing is cut off, and a value between two
//                neighbours goes to the upper one with the probability of its distance from the lower, to 16 bits (downwards).
// A block with an infinity or a NaN has the scale byte 255, which stands for NaN in all of it.
#include <type_traits>

#include "layers_device.h"

namespace conef {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;              // rows and columns of a workgroup
constexpr int kPitch = 130;             // of the tile in LDS: four rows 8 apart lie 8 banks apart

// The scale byte of a block and the factor that takes its elements over the scale (exact: 2^(127 - byte) is normal)
__device__ __forceinline__ uint32_t scale_byte(uint32_t most_bits, bool stochastic)
{
    const uint32_t e = most_bits >> 23;
    if (e == 255) return 255;
    uint32_t s = e > 2 ? e - 2 : 0;
    // (below 2^-125 the scale is the smallest there is, and what it divides stays below 4)
    if (stochastic && e >= 2 && (most_bits & 0x7FFFFFu) > 0x400000u) s = e - 1;
    return s;
}

// Code of a value over its scale, to nearest even
__device__ __forceinline__ uint32_t code_nearest(float v)
{
    const float a = fabsf(v);
    const uint32_t c = (uint32_t)(a > 0.25f) + (uint32_t)(a >= 0.75f) + (uint32_t)(a > 1.25f) + (uint32_t)(a >= 1.75f) +
                       (uint32_t)(a > 2.5f) + (uint32_t)(a >= 3.5f) + (uint32_t)(a > 5.0f);
    return c | (__float_as_uint(v) >> 31 << 3);
}

// The same with a 16-bit draw u: in units of 2^-17 the step below 2 is 65536, from 2 on twice, from 4 on four times that.
__device__ __forceinline__ uint32_t code_stochastic(float v, uint32_t u)
{
    const uint32_t f = (uint32_t)(fabsf(v) * 131072.0f);
    const uint32_t wide = (uint32_t)(f >= (1u << 18)) + (uint32_t)(f >= (1u << 19));
    const uint32_t c = (((f >> wide) + u) >> 16) + 2 * wide;
    return c | (__float_as_uint(v) >> 31 << 3);
}

// Quantises a block of which each of four neighbouring lanes holds an octet: returns the lane's eight codes and the block's
// scale byte.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t quantise_quad(const float v[8], const Draws &d, uint32_t octet, uint32_t &byte)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);       // (a NaN's bits are above infinity's)
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xF, 0xF, true));
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xF, 0xF, true));
    byte = scale_byte(most, STOCHASTIC);
    if (byte == 255) return 0;
    const float over = __uint_as_float((254u - byte) << 23);
    uint32_t codes = 0;
    if constexpr (STOCHASTIC) {
        uint32_t u[4];
        octet_draws(d, octet, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) codes |= code_stochastic(v[i] * over, (i & 1) ? u[i >> 1] >> 16 : u[i >> 1] & 0xFFFFu) << (4 * i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) codes |= code_nearest(v[i] * over) << (4 * i);
    }
    return codes;
}

// A workgroup takes 128 x 128 elements.  By rows: a wave takes 16 rows, of which its lanes read 32 columns at a time, four
// lanes a block, and writes the 256 bytes of that piece together.  By columns: the same on the tile in LDS, turned.
template <bool BF16, bool STOCHASTIC, bool BY_ROWS, bool BY_COLS>
__global__ __launch_bounds__(kThreads) void k_mx_quantise(MxQuantArgs a, int64_t row_pieces, int64_t col_pieces, int64_t padded_rows,
                                                          int64_t padded_cols)
{
    typedef std::conditional_t<BF16, uint16_t, float> Elem;
    __shared__ Elem tile[BY_COLS ? kTile * kPitch : 1];
    __shared__ __attribute__((aligned(4))) uint8_t scales[2][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane >> 2, q = lane & 3;
    const int64_t tc = blockIdx.x % col_pieces, tr = blockIdx.x / col_pieces, row0 = tr * kTile, col0 = tc * kTile;
    const uint32_t per_row = (uint32_t)((a.cols + 7) >> 3), per_col = (uint32_t)((a.rows + 7) >> 3);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int group = wave + 4 * h;
        const int64_t row = row0 + 16 * group + r;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int64_t col = col0 + 32 * b + 8 * q;
            float v[8];
            load_octet<BF16>(a.x.data, row * a.x.pitch + col, row < a.rows ? (int)max<int64_t>(min<int64_t>(a.cols - col, 8), 0) : 0, v);
            if constexpr (BY_COLS) {
                Elem *t = tile + (16 * group + r) * kPitch + 32 * b + 8 * q;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (BF16) t[i] = (uint16_t)(__float_as_uint(v[i]) >> 16);
                    else t[i] = v[i];
                }
            }
            if constexpr (BY_ROWS) {
                if (row0 + 16 * group < padded_rows) {
                    uint32_t byte;
                    const uint32_t c = quantise_quad<STOCHASTIC>(v, a.draws, (uint32_t)row * per_row + (uint32_t)(col >> 3), byte);
                    const int64_t piece = (row0 / 16 + group) * col_pieces + tc;
                    *reinterpret_cast<uint32_t *>(a.by_rows.codes + piece * 1024 + b * 256 + lane * 4) = c;
                    if (q == 0) scales[0][(group >> 2) * 256 + b * 64 + r * 4 + (group & 3)] = (uint8_t)byte;
                }
            }
        }
    }
    __syncthreads();
    if constexpr (BY_COLS) {
        Draws d = a.draws;
        d.word += kMxColWord - kMxRowWord;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int group = wave + 4 * h;
            const int64_t col = col0 + 16 * group + r;                       // a row of the turned matrix
            if (col0 + 16 * group >= padded_cols) continue;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int64_t row = row0 + 32 * b + 8 * q;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const Elem e = tile[(32 * b + 8 * q + i) * kPitch + 16 * group + r];
                    if constexpr (BF16) v[i] = __uint_as_float((uint32_t)e << 16);
                    else v[i] = e;
                }
                uint32_t byte;
                const uint32_t c = quantise_quad<STOCHASTIC>(v, d, (uint32_t)col * per_col + (uint32_t)(row >> 3), byte);
                const int64_t piece = (col0 / 16 + group) * row_pieces + tr;
                *reinterpret_cast<uint32_t *>(a.by_cols.codes + piece * 1024 + b * 256 + lane * 4) = c;
                if (q == 0) scales[1][(group >> 2) * 256 + b * 64 + r * 4 + (group & 3)] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    // scales: two pieces of 256 bytes each way
    const int half = (threadIdx.x >> 6) & 1, form = threadIdx.x >> 7;
    const uint32_t word = reinterpret_cast<const uint32_t *>(scales[form])[half * 64 + lane];
    if (BY_ROWS && form == 0 && row0 + 64 * half < padded_rows)
        *reinterpret_cast<uint32_t *>(a.by_rows.scales + ((row0 / 64 + half) * col_pieces + tc) * 256 + lane * 4) = word;
    if (BY_COLS && form == 1 && col0 + 64 * half < padded_cols)
        *reinterpret_cast<uint32_t *>(a.by_cols.scales + ((col0 / 64 + half) * row_pieces + tr) * 256 + lane * 4) = word;
}

// What a packed operand stands for: 16 rows a wave, 128 columns, four lanes a block.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_mx_dequantise(MxDequantArgs a, int64_t pieces, int64_t groups)
{
    const int64_t p = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (p >= groups * pieces) return;
    const int64_t group = p / pieces, tc = p - group * pieces;
    const int lane = threadIdx.x & 63, r = lane >> 2, q = lane & 3;
    const int64_t row = group * 16 + r;
    const uint8_t *scales = a.in.scales + ((group >> 2) * pieces + tc) * 256 + r * 4 + (group & 3);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const uint32_t c = *reinterpret_cast<const uint32_t *>(a.in.codes + p * 1024 + b * 256 + lane * 4);
        const uint32_t byte = scales[b * 64];
        const float step = byte == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte ? byte << 23 : 0x400000u);
        const int64_t col = tc * 128 + 32 * b + 8 * q;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = (c >> (4 * i)) & 7;
            // 0, 0.5, then (2 + (m & 1)) 2^(m / 2 - 2)
            const float x = m < 2 ? 0.5f * (float)m : __uint_as_float(((126 + (m >> 1)) << 23) | ((m & 1) << 22));
            v[i] = __uint_as_float(__float_as_uint(x) | ((c >> (4 * i + 3)) & 1) << 31) * step;
        }
        if (row < a.rows && col < a.cols)
            store_octet<BF16>(a.out.data, row * a.out.pitch + col, (int)min<int64_t>(a.cols - col, 8), v);
    }
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace

void launch_mx_quantise(const MxQuantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t row_pieces = (a.rows + 127) / 128, col_pieces = (a.cols + 127) / 128;
    const int64_t padded_rows = (a.rows + 63) / 64 * 64, padded_cols = (a.cols + 63) / 64 * 64;
    const dim3 grid((unsigned)(row_pieces * col_pieces));
    by_bool(bf16, [&](auto b) {
        by_bool(a.stochastic != 0, [&](auto s) {
            auto go = [&](auto rows, auto cols) {
                hipLaunchKernelGGL((k_mx_quantise<decltype(b)::value, decltype(s)::value, decltype(rows)::value, decltype(cols)::value>),
                                   grid, dim3(kThreads), 0, st, a, row_pieces, col_pieces, padded_rows, padded_cols);
            };
            if (!a.by_cols.codes) go(std::true_type{}, std::false_type{});
            else if (!a.by_rows.codes) go(std::false_type{}, std::true_type{});
            else go(std::true_type{}, std::true_type{});
        });
    });
}

void launch_mx_dequantise(const MxDequantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t pieces = (a.cols + 127) / 128, groups = (a.rows + 15) / 16;
    const dim3 grid((unsigned)((pieces * groups + 3) / 4));
    by_bool(bf16, [&](auto b) {
        hipLaunchKernelGGL((k_mx_dequantise<decltype(b)::value>), grid, dim3(kThreads), 0, st, a, pieces, groups);
    });
}

}  // namespace conef
