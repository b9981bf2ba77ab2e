// Quantisation to microscaled 4-bit floating point and back.
//
// A block of 32 consecutive elements of a row shares a scale 2^s (one byte, s + 127); an element is a sign and one of 0, 0.5, 1,
// 1.5, 2, 3, 4, 6, times the scale.  With e = floor(log2(largest magnitude of the block)):
//   to nearest   s = e - 2, so that magnitudes over the scale are below 8; ties go to the even code, those above 6 to 6;
//   stochastic   s = e - 2, or e - 1 where the largest is above 6 * 2^(e - 2): nothing is cut off, and a value between two
//                neighbours goes to the upper one with the probability of its distance from the lower, to 16 bits (downwards).
// A block with an infinity or a NaN has the scale byte 255, which stands for NaN in all of it.
#include <type_traits>

#include "turned_device.h"

namespace conef {

namespace {

constexpr int kThreads = 256;

// The scale byte of a block whose largest magnitude has these bits: its exponent less 2, at least 0; stochastic: one more for a mantissa
// above 1.5, by a carry (below 2^-125 the scale is the smallest there is, and what it divides stays below 4).
__device__ __forceinline__ uint32_t scale_byte(uint32_t most, bool stochastic)
{
    const uint32_t s = ((max(most, 2u << 23) + (stochastic ? 0x3FFFFFu : 0u)) >> 23) - 2;
    return most >= 255u << 23 ? 255u : s;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The values of an octet, each in the lower of two neighbouring registers, as the conversion that rounds stochastically takes
// them.  What the upper one holds is not used: the empty asm is its definition, without an instruction.
struct Values {
    f32x2 v[8];

    __device__ __forceinline__ Values()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "=v"(v[i]));
    }
};

template <bool BF16>
__device__ __forceinline__ void widen(const Octet<BF16> &o, Values &x)
{
    float v[8];
    widen<BF16>(o, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i].x = v[i];
}

// Eight values over the scale of byte `byte` as codes, by the conversion instructions.  They take the scale from a float's exponent
// (0: 2^-127), denormal values as they are, and keep 6 for what is above it.  The one that rounds stochastically adds its
// random word to the bits it drops, aligned at the top, for the lower of its two values: with a draw in the upper half of that word, zeros
// below, it rounds up iff floor(65536 f) + draw >= 65536.  The upper value gets other bits of the word, so each value takes an
// instruction of its own, of which the lower four bits count: four codes are put together from there in five more.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t codes_over(const Values &x, uint32_t byte, const uint32_t u[4])
{
    const float scale = __uint_as_float(byte << 23);
    if constexpr (STOCHASTIC) {
        uint32_t two[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t low = u[i] << 16, high = u[i] & 0xFFFF0000u;
            const uint32_t even = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(low, x.v[2 * i], low, scale, 0);
            const uint32_t odd = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(high, x.v[2 * i + 1], high, scale, 0);
            two[i] = (even & 0xFu) | (odd << 4 & ~0xFu);
        }
        const uint32_t low = __builtin_amdgcn_perm(two[1], two[0], 0x00000400u), high = __builtin_amdgcn_perm(two[3], two[2], 0x00000400u);
        return __builtin_amdgcn_perm(high, low, 0x05040100u);
    } else {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[0].x, x.v[1].x, scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2].x, x.v[3].x, scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[4].x, x.v[5].x, scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[6].x, x.v[7].x, scale, 3);
    }
}

// bits of the largest magnitude; a NaN's if there is one (its bits are above infinity's)
__device__ __forceinline__ uint32_t largest(const Values &x)
{
    float m = fabsf(x.v[0].x);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __builtin_elementwise_maximum(m, fabsf(x.v[i].x));
    return __float_as_uint(m) & 0x7FFFFFFFu;
}

// Quantises a block of which each of four lanes holds an octet, `most` the largest magnitude of all four: returns the lane's eight codes and
// the block's scale byte.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t quantise_octet(const Values &x, uint32_t most, const Draws &d, uint32_t octet, uint32_t &byte)
{
    byte = scale_byte(most, STOCHASTIC);
    uint32_t u[4] = {};
    if constexpr (STOCHASTIC) octet_draws(d, octet, u);
    const uint32_t c = codes_over<STOCHASTIC>(x, byte, u);
    return byte == 255 ? 0 : c;
}

// the largest over the lanes l ^ 1, l ^ 2 / over l ^ 16, l ^ 32
__device__ __forceinline__ uint32_t quad_largest(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t rows_largest(uint32_t m)
{
    auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)r[0], (uint32_t)r[1]);
    r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max((uint32_t)r[0], (uint32_t)r[1]);
}

// A workgroup takes 64 rows of 128 columns, or 128 rows of 64 columns if it quantises by columns too.  By rows: a wave takes 16 rows, of which
// its lanes read 32 columns at a time, four lanes a block, and writes the 256 bytes of that piece together.  By columns: the same on
// the tile in LDS, turned, the four octets of a block 16 lanes apart.
// 8192 x 8192 in bf16 both ways: to nearest 45 us, 205 MB at 4.5 TB/s (by rows alone 32 us, 170 MB at 5.3, by columns alone 37), bound by memory;
// stochastically 60 us (35 by rows, 39 by columns), both ways bound by its vector instructions, 113 an octet and way: 40 for the Philox call, eight conversions, which take 16 cycles each, 19 around
// them.  (The same with the codes computed from integers: 100 us.)  64 columns and not 128 in the tile (of four waves): 1203 x 1000 in fp32 4.7 / 6.0 us.
template <bool BF16, bool STOCHASTIC, bool BY_ROWS, bool BY_COLS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_mx_quantise(MxQuantArgs a, int64_t row_pieces, int64_t col_pieces, int64_t col_tiles,
                                                          int64_t padded_rows, int64_t padded_cols)
{
    constexpr int kRows = BY_COLS ? 128 : 64, kCols = BY_COLS ? 64 : 128, kBlocks = kCols / 32, kTurns = kRows / 16 / WAVES;
    static_assert(kTurns * WAVES * 16 == kRows, "");
    __shared__ __attribute__((aligned(16))) std::conditional_t<BY_COLS, Turned<BF16>, char> tile;
    __shared__ __attribute__((aligned(4))) uint8_t scales[2][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane >> 2, q = lane & 3;
    const uint32_t group = group_index();
    const int64_t row0 = group / col_tiles * kRows, col0 = group % col_tiles * kCols;
    if (row0 >= a.rows) return;
    const uint32_t per_row = (uint32_t)((a.cols + 7) >> 3), per_col = (uint32_t)((a.rows + 7) >> 3);
    Octet<BF16> o[kTurns][kBlocks];
    auto fetch = [&](bool whole) {
#pragma unroll
        for (int h = 0; h < kTurns; ++h) {
            const int64_t row = row0 + 16 * (wave + WAVES * h) + r;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const int64_t col = col0 + 32 * b + 8 * q;
                o[h][b] = fetch_octet<BF16>(a.x.data, row * a.x.pitch + col, whole ? 8 : row < a.rows ? octet_left(a.cols - col) : 0);
            }
        }
    };
    if (row0 + kRows <= a.rows && col0 + kCols <= a.cols) fetch(true);
    else fetch(false);
    if constexpr (BY_COLS) {
#pragma unroll
        for (int h = 0; h < kTurns; ++h)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) tile.put(16 * (wave + WAVES * h) + r, 32 * b + 8 * q, o[h][b]);
    }
    if constexpr (BY_ROWS) {
        const int64_t piece0 = row0 / 16 * col_pieces + col0 / 128;
        const int block0 = BY_COLS ? (int)(col0 >> 5 & 3) : 0;               // of the piece
#pragma unroll
        for (int h = 0; h < kTurns; ++h) {
            const int group16 = wave + WAVES * h;
            const int64_t row = row0 + 16 * group16 + r;
            if (row0 + 16 * group16 >= padded_rows) continue;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                Values v;
                widen<BF16>(o[h][b], v);
                uint32_t byte;
                const uint32_t octet = (uint32_t)row * per_row + (uint32_t)((col0 + 32 * b + 8 * q) >> 3);
                const uint32_t c = quantise_octet<STOCHASTIC>(v, quad_largest(largest(v)), a.draws, octet, byte);
                *reinterpret_cast<uint32_t *>(a.by_rows.codes + (piece0 + group16 * col_pieces) * 1024 + (block0 + b) * 256 + lane * 4) = c;
                if (q == 0) scales[0][(group16 >> 2) * 64 * kBlocks + b * 64 + r * 4 + (group16 & 3)] = (uint8_t)byte;
            }
        }
    }
    __syncthreads();
    if constexpr (BY_COLS) {
        Draws d = a.draws;
        d.word += kMxColWord - kMxRowWord;
        const int c16 = lane & 15, q16 = lane >> 4, strip = wave & 3;
        const int64_t col = col0 + 16 * strip + c16;                          // a row of the turned matrix
        if (col0 < padded_cols) {
            uint8_t *codes = a.by_cols.codes + ((col0 / 16 + strip) * row_pieces + row0 / 128) * 1024 + c16 * 16 + q16 * 4;
#pragma unroll
            for (int i = 0; i < 16 / WAVES; ++i) {
                const int b = (wave >> 2) * (16 / WAVES) + i;
                Values v;
                widen<BF16>(tile.get(32 * b + 8 * q16, 16 * strip, lane), v);
                uint32_t byte;
                const uint32_t octet = (uint32_t)col * per_col + (uint32_t)((row0 + 32 * b + 8 * q16) >> 3);
                const uint32_t c = quantise_octet<STOCHASTIC>(v, rows_largest(largest(v)), d, octet, byte);
                *reinterpret_cast<uint32_t *>(codes + b * 256) = c;
                if (q16 == 0) scales[1][b * 64 + c16 * 4 + strip] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    // the tile's scales, 256 bytes each way: by rows 64 bytes a block, two blocks of each 64 rows where there are 128
    if (BY_ROWS && wave == 0) {
        const int half = BY_COLS ? lane >> 5 : 0;
        if (row0 + 64 * half < padded_rows)
            *reinterpret_cast<uint32_t *>(a.by_rows.scales + ((row0 / 64 + half) * col_pieces + col0 / 128) * 256 + (BY_COLS ? (col0 >> 5 & 3) * 64 : 0) +
                                          (lane - half * 32) * 4) = reinterpret_cast<const uint32_t *>(scales[0])[lane];
    }
    if (BY_COLS && wave == 1 && col0 < padded_cols)
        *reinterpret_cast<uint32_t *>(a.by_cols.scales + (col0 / 64 * row_pieces + row0 / 128) * 256 + lane * 4) =
            reinterpret_cast<const uint32_t *>(scales[1])[lane];
}

// What eight codes stand for
__device__ __forceinline__ void values(uint32_t c, uint32_t byte, float v[8])
{
    const float scale = __uint_as_float(byte << 23);
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = d[0]; v[5] = d[1]; v[6] = e[0]; v[7] = e[1];
    if (byte == 255)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7FC00000u);
}

// What a packed operand stands for: 16 rows a wave, 128 columns, so that a store writes whole lines (four lanes a block, 64 bytes of a line at a time: 29 us, in
// fp32 111).  Bound by memory: 8192 x 8192 in bf16 22 us, 170 MB at 7.8 TB/s, of which a part stays in the last cache, in fp32 48, 304 MB at 6.3.  A store's 128 bytes
// are cut where the tile is, so rows that do not begin on a line have two lines to each: 8192 x 8191 takes 55 us, in fp32 136, 16384 x 3000 in fp32 84 (bf16 23).
template <bool BF16, bool PAST>
__global__ __launch_bounds__(kThreads) void k_mx_dequantise(MxDequantArgs a, int64_t pieces, int64_t groups)
{
    const int64_t p = (int64_t)group_index() * (kThreads / 64) + (threadIdx.x >> 6);
    if (p >= groups * pieces) return;
    const int64_t group = p / pieces, tc = p - group * pieces;
    // a store: 8 rows of 128 bytes, 16 a lane
    constexpr int kElements = BF16 ? 8 : 4, kAcross = 8 * kElements;
    const int lane = threadIdx.x & 63, q = lane & 7;
#pragma unroll
    for (int i = 0; i < 2 * 128 / kAcross; ++i) {
        const int r = (i & 1) * 8 + (lane >> 3), in_piece = (i >> 1) * kAcross + q * kElements, b = in_piece >> 5;
        const uint8_t *at = a.in.codes + p * 1024 + b * 256 + r * 16 + (in_piece & 31) / 2;
        const uint32_t c = BF16 ? *reinterpret_cast<const uint32_t *>(at) : *reinterpret_cast<const uint16_t *>(at);
        const uint32_t byte = a.in.scales[((group >> 2) * pieces + tc) * 256 + b * 64 + r * 4 + (group & 3)];
        const int64_t row = group * 16 + r, col = tc * 128 + in_piece, place = row * a.out.pitch + col;
        float v[8];
        values(c, byte, v);
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

void launch_mx_quantise(const MxQuantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t row_pieces = (a.rows + 127) / 128, col_pieces = (a.cols + 127) / 128;
    const int64_t padded_rows = (a.rows + 63) / 64 * 64, padded_cols = (a.cols + 63) / 64 * 64;
    const int64_t col_tiles = a.by_cols.codes ? 2 * col_pieces : col_pieces;
    const dim3 grid = grid_of((a.by_cols.codes ? row_pieces : padded_rows / 64) * col_tiles);
    by_bool(bf16, [&](auto b) {
        by_bool(a.stochastic != 0, [&](auto s) {
            auto go = [&](auto rows, auto cols, auto waves) {
                constexpr int W = decltype(waves)::value;
                hipLaunchKernelGGL((k_mx_quantise<decltype(b)::value, decltype(s)::value, decltype(rows)::value, decltype(cols)::value, W>),
                                   grid, dim3(64 * W), 0, st, a, row_pieces, col_pieces, col_tiles, padded_rows, padded_cols);
            };
            const std::integral_constant<int, 4> four;
            auto by_cols = [&](auto waves) {
                if (a.by_rows.codes) go(std::true_type{}, std::true_type{}, waves);
                else go(std::false_type{}, std::true_type{}, waves);
            };
            // Eight waves to a tile while there are at most two tiles a CU, which is when a tile's latency counts.  us: 1000 x 515 fp32 3.1 / 3.8, stochastically
            // 4.3 / 5.0, 2048 x 2048 bf16 6.3 / 6.5; but 8192 x 8192 bf16 64.8 / 60.2.
            if (!a.by_cols.codes) go(std::true_type{}, std::false_type{}, four);
            else if (grid.x <= 512) by_cols(std::integral_constant<int, 8>{});
            else by_cols(four);
        });
    });
}

void launch_mx_dequantise(const MxDequantArgs &a, bool bf16, hipStream_t st)
{
    const int64_t pieces = (a.cols + 127) / 128, groups = (a.rows + 15) / 16;
    const dim3 grid = grid_of((pieces * groups + 3) / 4);
    // Values that the dies' caches do not hold go past them: 8192 x 8192 in bf16, another buffer each time, 26 / 36 us; but not rows that end
    // within 64 bytes, of which halves would be written twice: 16384 x 3000 in bf16 27 / 62.
    const int64_t size = bf16 ? 2 : 4;
    const bool whole = a.out.pitch * size % 64 == 0 && reinterpret_cast<uintptr_t>(a.out.data) % 64 == 0;
    const bool past = whole && a.rows * a.cols * size > (int64_t)32 << 20;
    by_bool(bf16, [&](auto b) {
        by_bool(past, [&](auto p) {
            hipLaunchKernelGGL((k_mx_dequantise<decltype(b)::value, decltype(p)::value>), grid, dim3(kThreads), 0, st, a, pieces, groups);
        });
    });
}

}  // namespace conef
