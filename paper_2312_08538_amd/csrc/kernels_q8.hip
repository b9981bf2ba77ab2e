// Quantisation to 8-bit floating point with a scale for each block of 128 elements of a row, and back.
//
// The scale is the smallest power of two 2^(b - 127) for which the block's largest magnitude over it is no larger than 448 (E4M3) or
// 57344 (E5M2): both are 1.75 2^t, so b is the exponent of that magnitude less t, and one more for a mantissa above 1.75.  A power of two as a scale costs
// an element no precision (its own exponent makes up for it, down to where the format's ends: 2^-17 and 2^-31 of the block's largest), the division is exact, so that an
// element is rounded once, and the matrix instructions take it as it is.
#include <type_traits>

#include "q8_device.h"
#include "turned_device.h"

namespace conef {

namespace {

constexpr int kThreads = 256;

// A workgroup takes 64 rows of 128 columns, or 128 rows of 128 columns if it quantises by columns too.  By rows: a wave takes 16 rows, four lanes each; a lane reads four
// octets 32 columns apart, so that four lanes read 64 bytes (bf16) together, and half a wave writes a square of 256 bytes at a time.  By columns: the same on the tile in
// LDS, turned, 16 columns a wave.
// Bound by memory: 8192 x 8192 bf16 by rows 30.2 us, by columns 30.1 (6.7 TB/s), both ways of one read 42.1 (6.4); fp32 57.6, 58.9 and 73.6 (6.0).
template <bool BF16, bool E5M2, bool BY_ROWS, bool BY_COLS>
__global__ __launch_bounds__(BY_COLS ? 512 : 256) void k_q8_quantise(Q8QuantArgs a, int64_t row_pieces, int64_t col_pieces, int64_t padded_rows,
                                                                     int64_t padded_cols)
{
    constexpr int kRows = BY_COLS ? 128 : 64;
    __shared__ __attribute__((aligned(16))) std::conditional_t<BY_COLS, Turned<BF16>, char> tile[2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane >> 2, q = lane & 3;
    const uint32_t group = group_index();
    const int64_t row0 = group / col_pieces * kRows, piece = group % col_pieces, col0 = piece * 128;
    if (row0 >= a.rows) return;
    Octet<BF16> o[4];
    const int64_t row = row0 + 16 * wave + r;
    auto fetch = [&](bool whole) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int64_t col = col0 + 32 * b + 8 * q;
            o[b] = fetch_octet<BF16>(a.x.data, row * a.x.pitch + col, whole ? 8 : row < a.rows ? octet_left(a.cols - col) : 0);
        }
    };
    if (row0 + kRows <= a.rows && col0 + 128 <= a.cols) fetch(true);
    else fetch(false);
    if constexpr (BY_COLS) {
#pragma unroll
        for (int b = 0; b < 4; ++b) tile[b >> 1].put(16 * wave + r, 32 * (b & 1) + 8 * q, o[b]);
    }
    if (BY_ROWS && row0 + 16 * wave < padded_rows) {
        float v[4][8];
        uint32_t most = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            widen<BF16>(o[b], v[b]);
            most = max(most, largest(v[b]));
        }
        const uint32_t byte = q8_scale<E5M2>(quad_largest(most));
        uint8_t *to = a.by_rows.codes + ((row0 / 16 + wave) * col_pieces + piece) * 2048 + (q >> 1) * 256 + r * 16 + (q & 1) * 8;
#pragma unroll
        for (int b = 0; b < 4; ++b) *reinterpret_cast<uint2 *>(to + b * 512) = q8_codes<E5M2>(v[b], byte);
        if (q == 0) a.by_rows.scales[piece * padded_rows + row] = (uint8_t)byte;
    }
    if constexpr (BY_COLS) {
        __syncthreads();
        const int c16 = lane & 15, q16 = lane >> 4;
        const int64_t strip = col0 + 16 * wave;                                    // rows of the turned matrix
        if (strip >= padded_cols) return;
        float v[4][8];
        uint32_t most = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            widen<BF16>(tile[wave >> 2].get(32 * b + 8 * q16, 16 * (wave & 3), lane), v[b]);
            most = max(most, largest(v[b]));
        }
        const uint32_t byte = q8_scale<E5M2>(rows_largest(most));
        uint8_t *to = a.by_cols.codes + (strip / 16 * row_pieces + row0 / 128) * 2048 + (q16 >> 1) * 256 + c16 * 16 + (q16 & 1) * 8;
#pragma unroll
        for (int b = 0; b < 4; ++b) *reinterpret_cast<uint2 *>(to + b * 512) = q8_codes<E5M2>(v[b], byte);
        if (q16 == 0) a.by_cols.scales[row0 / 128 * padded_cols + strip + c16] = (uint8_t)byte;
    }
}

// What a packed operand stands for: 16 rows a wave, 128 columns, so that a store writes 128 bytes of each of eight rows.  Bound by memory: 8192 x 8192 into bf16 30.9 us
// (6.5 TB/s), into fp32 50.3 (6.7).
template <bool BF16, bool E5M2, bool PAST>
__global__ __launch_bounds__(kThreads) void k_q8_dequantise(Q8DequantArgs a, int64_t pieces, int64_t groups, int64_t padded_rows)
{
    const int64_t p = (int64_t)group_index() * (kThreads / 64) + (threadIdx.x >> 6);
    if (p >= groups * pieces) return;
    const int64_t group = p / pieces, tc = p - group * pieces;
    constexpr int kElements = BF16 ? 8 : 4, kAcross = 8 * kElements;
    const int lane = threadIdx.x & 63, q = lane & 7;
#pragma unroll
    for (int i = 0; i < 2 * 128 / kAcross; ++i) {
        const int r = (i & 1) * 8 + (lane >> 3), in_piece = (i >> 1) * kAcross + q * kElements;
        const uint8_t *at = a.in.codes + p * 2048 + (in_piece >> 4) * 256 + r * 16 + (in_piece & 15);
        const int64_t row = group * 16 + r, col = tc * 128 + in_piece, place = row * a.out.pitch + col;
        const uint32_t byte = a.in.scales[tc * padded_rows + row];
        float v[8];
        q8_values<E5M2>(*reinterpret_cast<const uint32_t *>(at), byte, v);
        if constexpr (BF16) q8_values<E5M2>(*reinterpret_cast<const uint32_t *>(at + 4), byte, v + 4);
        if (row >= a.rows || col >= a.cols) continue;
        if constexpr (BF16) {
            store_octet<true, PAST>(a.out.data, place, octet_left(a.cols - col), v);
        } else {
            float *to = static_cast<float *>(a.out.data) + place;
            if (col + 4 <= a.cols) {
                store_16<PAST>(to, u32x4_any{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (col + e < a.cols) to[e] = v[e];
            }
        }
    }
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace

void launch_q8_quantise(const Q8QuantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t row_pieces = (a.rows + 127) / 128, col_pieces = (a.cols + 127) / 128;
    const int64_t padded_rows = (a.rows + 63) / 64 * 64, padded_cols = (a.cols + 63) / 64 * 64;
    const dim3 grid = grid_of((a.by_cols.codes ? row_pieces : padded_rows / 64) * col_pieces);
    by_bool(bf16, [&](auto b) {
        by_bool(a.e5m2 != 0, [&](auto f) {
            auto go = [&](auto rows, auto cols) {
                hipLaunchKernelGGL((k_q8_quantise<decltype(b)::value, decltype(f)::value, decltype(rows)::value, decltype(cols)::value>), grid,
                                   dim3(decltype(cols)::value ? 512 : 256), 0, st, a, row_pieces, col_pieces, padded_rows, padded_cols);
            };
            if (!a.by_cols.codes) go(std::true_type{}, std::false_type{});
            else if (a.by_rows.codes) go(std::true_type{}, std::true_type{});
            else go(std::false_type{}, std::true_type{});
        });
    });
}

void launch_q8_dequantise(const Q8DequantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t pieces = (a.cols + 127) / 128, groups = (a.rows + 15) / 16, padded_rows = (a.rows + 63) / 64 * 64;
    const dim3 grid = grid_of((pieces * groups + 3) / 4);
    // Past the caches, where these do not hold what is written anyway and no line is written in halves: 8192 x 8192 into fp32 50 us / 67, into bf16 30.9 / 30.9.
    const int64_t size = bf16 ? 2 : 4;
    const bool whole = a.out.pitch * size % 64 == 0 && reinterpret_cast<uintptr_t>(a.out.data) % 64 == 0;
    const bool past = whole && a.rows * a.cols * size > (int64_t)32 << 20;
    by_bool(bf16, [&](auto b) {
        by_bool(a.e5m2 != 0, [&](auto f) {
            by_bool(past, [&](auto p) {
                hipLaunchKernelGGL((k_q8_dequantise<decltype(b)::value, decltype(f)::value, decltype(p)::value>), grid, dim3(kThreads), 0, st, a, pieces,
                                   groups, padded_rows);
            });
        });
    });
}

}  // namespace conef
