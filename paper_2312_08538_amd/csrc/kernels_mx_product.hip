// C = alpha A B^T + beta C of two packed operands of microscaled 4-bit floating point, on the matrix instructions that take such
// operands with their scales (v_mfma_scale_f32_16x16x128_f8f6f4).
//
// Lane l of such an instruction holds one block of an operand: row l % 16, elements 32 (l / 16) .. + 31 of 128, sixteen bytes, and in
// one byte of a register the block's scale.  A packed operand holds its codes in that order, 1024 bytes an instruction, and its
// scales four row groups to a register, so a tile goes from memory to LDS and from there to registers as it lies, without a
// bank conflict.  The instruction's first operand is B's rows: then a lane holds four consecutive columns of one row of C.
//
// What bounds it: the instructions alone, from registers, reach 6.8 PFLOP/s on zeros and 5.8 on random operands, where the card's power sets the
// clock (the form of 32 x 32 x 64 9.8 and 6.6, but it adds to twice as many accumulators a product, and the same kernels on it took 259 us
// for 8192 x 8192 x 8192 where this one then took 246, 251 for 4096 x 50304 x 2048 where this one took 235: both before tiles streamed).  8192 x 8192 x 8192
// reaches 4.7 PFLOP/s (231 to 240 us: the clock goes by the box), 8192 x 2048 x 8192 4.5.  Of those 240 us, without its loads to LDS it would take 208, without its
// reads from there 219, without either 189, without the products 126.  With a shorter axis C's bytes and each tile's beginning weigh more: 4096 x 50304 x 2048
// 3.9 (213 to 218 us), without stores 10 us less.  Its 3152 tiles are 12.3 for each of 256 workgroups, so a thirteenth turn, with 80 of them at work, is some 5 % of it.
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

// Sixteen bytes (or four) a lane from `src` to LDS, one lane's after the other's: `dst` is the wave's.
template <int BYTES>
__device__ __forceinline__ void to_lds(const uint8_t *src, uint8_t *dst)
{
    const auto *from = (const __attribute__((address_space(1))) void *)src;
    auto *to = (__attribute__((address_space(3))) void *)dst;
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds(from, to, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds(from, to, 4, 0, 0);
}

// all but the last N loads of this wave have arrived, and all its reads from LDS
template <int N>
__device__ __forceinline__ void wait_loads()
{
    // (the builtin, which the compiler counts with: bits 3:0 and 15:14 loads, 6:4 exports, 11:8 LDS)
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4 << 14) | 7 << 4);
    asm volatile("" ::: "memory");
}

// alpha v (+ beta c) to N neighbours of a row of C.  Old elements of C are read one at a time, behind the last product, and in large tiles what is written then
// does not go by way of LDS: with beta = 1 4096 x 50304 x 2048 takes 619 us (beta = 0: 213), 4096 x 8192 x 2048 93 (40), 8192 x 2048 x 8192 85 (61).
template <bool BF16, bool ADD, bool PAST, int N>
__device__ __forceinline__ void store_row(const MxProductArgs &a, int64_t row, int64_t col, const float *v)
{
    const int64_t at = row * a.c.pitch + col;
    const int left = (int)(a.n - col < N ? a.n - col : N);
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = a.alpha * v[i];
        if (ADD && i < left)
            x[i] = __builtin_fmaf(a.beta, BF16 ? bf16_bits_to_f32(static_cast<const uint16_t *>(a.c.data)[at + i]) : static_cast<const float *>(a.c.data)[at + i], x[i]);
    }
    if constexpr (BF16) {
        uint16_t *p = static_cast<uint16_t *>(a.c.data) + at;
        uint32_t u[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) u[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        if (left == N && N == 8) {
            store_16<PAST>(p, u32x4_any{u[0], u[1], u[2], u[3]});
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = (uint16_t)(u[i / 2] >> (16 * (i & 1)));
    } else {
        float *p = static_cast<float *>(a.c.data) + at;
        if (left == N && N == 4) {
            store_16<PAST>(p, u32x4_any{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])});
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = x[i];
    }
}

// The four columns that a lane holds of each of two neighbouring tiles of 16, to C.  bf16: two rows of 16 lanes exchange halves first, so that a
// lane has eight columns of one of the tiles and writes 16 bytes.
template <bool BF16, bool ADD, bool PAST>
__device__ __forceinline__ void store_pair(const MxProductArgs &a, int64_t row, int64_t col, int quad, f32x4 u, f32x4 v)
{
    if constexpr (BF16) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(u[i]), __float_as_uint(v[i]), false, false);
            x[i] = __uint_as_float(r[0]);
            x[4 + i] = __uint_as_float(r[1]);
        }
        col += 16 * (quad & 1) + 8 * (quad >> 1);
        if (row < a.m && col < a.n) store_row<true, ADD, PAST, 8>(a, row, col, x);
    } else if (row < a.m) {
        const float x[4] = {u[0], u[1], u[2], u[3]}, y[4] = {v[0], v[1], v[2], v[3]};
        if (col + 4 * quad < a.n) store_row<false, ADD, PAST, 4>(a, row, col + 4 * quad, x);
        if (col + 16 + 4 * quad < a.n) store_row<false, ADD, PAST, 4>(a, row, col + 16 + 4 * quad, y);
    }
}

// Fragments of one step along the long axis: a wave's TM + TN operands of 16 rows and their scales, four operands to a register.
template <int TM, int TN>
struct Step {
    v4i a[TM], b[TN];
    int ea[(TM + 3) / 4], eb[(TN + 3) / 4];
};

// A product's shape in tiles; items are tiles times parts of the long axis (`per_part` pieces, the last may have fewer), parts outermost.
struct Shape {
    int pieces, a_groups, b_groups, tiles_m, tiles_n, per_part, items;
};

// WM x WN waves of TM x TN tiles of 16 x 16; 128 elements of the long axis (one piece) a step, STAGES of them in LDS.  Step s + STAGES is
// fetched into the place of step s as soon as every wave has that in registers, and the fragments of step s + 1 are read while
// those of step s are multiplied, so there is one barrier a step and nothing is waited for that was not asked for a step before.
// WAVES: waves a SIMD, of all the workgroups that a CU is to hold.
template <bool BF16, bool ADD, bool PAST, int WM, int WN, int TM, int TN, int STAGES, int WAVES>
__global__ __launch_bounds__(64 * WM * WN, WAVES) void k_mx_product(MxProductArgs a, Shape z)
{
    constexpr int kM = WM * TM * 16, kN = WN * TN * 16, kWaves = WM * WN, kStage = (kM + kN) * 68;
    constexpr int kCodeLoads = (kM + kN) / 16 / kWaves, kScaleLoads = ((kM + kN) / 64 + kWaves - 1) / kWaves;
    constexpr int kLoads = kCodeLoads + kScaleLoads;
    static_assert((kM + kN) / 16 % kWaves == 0 && kM % 64 == 0 && kN % 64 == 0 && TM % 2 == 0 && TN % 2 == 0 && STAGES >= 2, "");
    static_assert((STAGES - 1) * kLoads < 64, "the counter of loads");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    // Workgroups go to the eight dies in turn; each die gets a run of neighbouring items, rows of tiles in eights, so that what its
    // workgroups read at one time stays in its cache.
    const int die = blockIdx.x & 7, per_die = z.items >> 3, more = z.items & 7, tiles = z.tiles_m * z.tiles_n;
    const int item = die * per_die + (die < more ? die : more) + (int)(blockIdx.x >> 3), tile = item % tiles, part = item / tiles;
    const int band = tile / (8 * z.tiles_n), in_band = tile - band * 8 * z.tiles_n, high = min(z.tiles_m - 8 * band, 8);
    const int m0 = (8 * band + in_band % high) * kM, n0 = in_band / high * kN;
    const int first = part * z.per_part, pieces = min(z.per_part, z.pieces - first);

    // what this wave fetches: 1024 bytes of codes at a time, 256 of scales; a row group beyond the operand's last takes the last
    // one's place (what comes of it is not stored)
    const uint8_t *src[kCodeLoads], *scale_src[kScaleLoads];
    int scale_dst[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kCodeLoads; ++i) {
        const int g = wave + i * kWaves;
        const bool is_a = g < kM / 16;
        const int group = is_a ? min(m0 / 16 + g, z.a_groups - 1) : min(n0 / 16 + g - kM / 16, z.b_groups - 1);
        src[i] = (is_a ? a.a.codes : a.b.codes) + ((int64_t)group * z.pieces + first) * 1024;
    }
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int g = (wave + i * kWaves) % ((kM + kN) / 64);       // (some twice, so that every wave has as many loads in flight)
        const bool is_a = g < kM / 64;
        const int group = is_a ? min(m0 / 64 + g, z.a_groups / 4 - 1) : min(n0 / 64 + g - kM / 64, z.b_groups / 4 - 1);
        scale_src[i] = (is_a ? a.a.scales : a.b.scales) + ((int64_t)group * z.pieces + first) * 256;
        scale_dst[i] = (kM + kN) * 64 + g * 256;
    }
    auto fetch = [&](int s, int slot) {
        uint8_t *to = lds + slot * kStage;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) to_lds<16>(src[i] + (int64_t)s * 1024 + lane * 16, to + (wave + i * kWaves) * 1024);
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) to_lds<4>(scale_src[i] + (int64_t)s * 256 + lane * 4, to + scale_dst[i]);
    };
    const int la = wm * TM * 1024 + lane * 16, lb = (kM / 16 + wn * TN) * 1024 + lane * 16;
    const int sa = (kM + kN) * 64 + wm * TM / 4 * 256 + lane * 4, sb = (kM + kN) * 64 + kM * 4 + wn * TN / 4 * 256 + lane * 4;
    typedef Step<TM, TN> S;
    auto read = [&](int slot, S &f) {
        const uint8_t *from = lds + slot * kStage;
        // (two tiles of 16 rows a wave: every other wave has the upper two of a register's scales)
#pragma unroll
        for (int i = 0; i < (TM + 3) / 4; ++i) f.ea[i] = *reinterpret_cast<const int *>(from + sa + i * 256) >> (TM == 2 ? wm % 2 * 16 : 0);
#pragma unroll
        for (int i = 0; i < (TN + 3) / 4; ++i) f.eb[i] = *reinterpret_cast<const int *>(from + sb + i * 256) >> (TN == 2 ? wn % 2 * 16 : 0);
#pragma unroll
        for (int i = 0; i < TN; ++i) f.b[i] = *reinterpret_cast<const v4i *>(from + lb + i * 1024);
#pragma unroll
        for (int i = 0; i < TM; ++i) f.a[i] = *reinterpret_cast<const v4i *>(from + la + i * 1024);
    };
    f32x4 acc[TN][TM] = {};
    int slot = 0;
    // Step s: its fragments are in `now`; those of the next one go to `next` (behind the last step: what is left there, for nothing), a read
    // after every few products: reads wait for LDS in the order of their issue, and products behind them would wait with them.
    auto step = [&](int s, auto steady, const S &now, S &next) {
        const int after = slot + 1 == STAGES ? 0 : slot + 1;
        wait_loads<decltype(steady)::value ? (STAGES - 2) * kLoads : 0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (decltype(steady)::value || s + STAGES < pieces) fetch(s + STAGES, slot);
        __builtin_amdgcn_sched_barrier(0);
        read(after, next);
        unroll<TM>([&](auto i) {
            unroll<TN>([&](auto j) {
                constexpr int I = decltype(i)::value, J = decltype(j)::value;
                acc[J][I] = mfma_mx<J % 4, I % 4>(now.b[J], now.a[I], acc[J][I], now.eb[J / 4], now.ea[I / 4]);
            });
        });
        unroll<TM + TN>([&](auto r) {
            constexpr int R = decltype(r)::value, kReads = TM + TN, kProducts = TM * TN;
            __builtin_amdgcn_sched_group_barrier(0x008, (R + 1) * kProducts / kReads - R * kProducts / kReads, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        });
        __builtin_amdgcn_sched_barrier(0);
        slot = after;
    };

    for (int s = 0; s < min(pieces, STAGES); ++s) fetch(s, s);
    if (pieces >= STAGES) wait_loads<(STAGES - 1) * kLoads>();
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    S even, odd;
    read(0, even);
    int s = 0;
    // (steps in twos, so that fragments need not be moved; the loop of steady steps is a block without branches: the compiler would move
    // products over a branch, away from the reads that they are to hide)
    for (; s + 1 + STAGES < pieces; s += 2) {
        step(s, std::true_type{}, even, odd);
        step(s + 1, std::true_type{}, odd, even);
    }
    for (; s < pieces; s += 2) {
        step(s, std::false_type{}, even, odd);
        if (s + 1 >= pieces) odd = S{};
        step(s + 1, std::false_type{}, odd, even);
    }
    if (a.partials) {
        a.c.data = a.partials + (int64_t)part * a.m * a.n;
        a.c.pitch = a.n;
    }
    if constexpr (ADD) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = m0 + (wm * TM + i) * 16 + (lane & 15);
#pragma unroll
            for (int j = 0; j < TN; j += 2) store_pair<BF16, ADD, PAST>(a, row, n0 + (wn * TN + j) * 16, lane >> 4, acc[j][i], acc[j + 1][i]);
        }
    } else {
        // By way of LDS, as many rows at a time as fit, so that a store writes whole rows of the tile.
        constexpr int kSize = BF16 ? 2 : 4, kPitch = kN * kSize + 16, kFit = STAGES * kStage / kPitch;
        constexpr int kTurns = kM <= kFit ? 1 : kM / 2 <= kFit ? 2 : 4, kTiles = TM / kTurns, kRows = kM / kTurns, kPieces = kN * kSize / 16;
        static_assert(kRows <= kFit && TM % kTurns == 0 && kRows * kPieces % (64 * kWaves) == 0, "");
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                uint8_t *to = lds + ((wm * kTiles + i) * 16 + (lane & 15)) * kPitch + wn * TN * 16 * kSize;
#pragma unroll
                for (int j = 0; j < TN; j += 2) {
                    const f32x4 u = acc[j][turn * kTiles + i], v = acc[j + 1][turn * kTiles + i];
                    if constexpr (BF16) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            auto x = __builtin_amdgcn_permlane16_swap(pack_bf16(a.alpha * u[2 * e], a.alpha * u[2 * e + 1]),
                                                                      pack_bf16(a.alpha * v[2 * e], a.alpha * v[2 * e + 1]), false, false);
                            w[e] = x[0];
                            w[2 + e] = x[1];
                        }
                        const int col = j * 16 + 16 * ((lane >> 4) & 1) + 8 * (lane >> 5);
                        *reinterpret_cast<uint4 *>(to + col * 2) = make_uint4(w[0], w[1], w[2], w[3]);
                    } else {
                        const int col = j * 16 + 4 * (lane >> 4);
                        *reinterpret_cast<float4 *>(to + col * 4) = make_float4(a.alpha * u[0], a.alpha * u[1], a.alpha * u[2], a.alpha * u[3]);
                        *reinterpret_cast<float4 *>(to + col * 4 + 64) = make_float4(a.alpha * v[0], a.alpha * v[1], a.alpha * v[2], a.alpha * v[3]);
                    }
                }
            }
            __syncthreads();
#pragma unroll 4
            for (int s = 0; s < kRows * kPieces / (64 * kWaves); ++s) {
                const int at = s * 64 * kWaves + threadIdx.x, r = at / kPieces, c = at % kPieces;
                const int64_t row = m0 + r / (kTiles * 16) * (TM * 16) + turn * kTiles * 16 + r % (kTiles * 16), col = n0 + c * (16 / kSize);
                if (row >= a.m || col >= a.n) continue;
                const uint4 w = *reinterpret_cast<const uint4 *>(lds + r * kPitch + c * 16);
                uint8_t *to = static_cast<uint8_t *>(a.c.data) + (row * a.c.pitch + col) * kSize;
                if (col + 16 / kSize <= a.n) {
                    store_16<PAST>(to, u32x4_any{w.x, w.y, w.z, w.w});
                } else if constexpr (BF16) {
                    const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (col + i < a.n) reinterpret_cast<uint16_t *>(to)[i] = (uint16_t)(e[i >> 1] >> (16 * (i & 1)));
                } else {
                    const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col + i < a.n) reinterpret_cast<uint32_t *>(to)[i] = e[i];
                }
            }
        }
    }
}

// Tiles one after the other by as many workgroups as there are CUs: WM x WN waves of TM x TN tiles of 16 x 16, steps and waits as above.  The last
// steps of a tile fetch the first of the next one, and a wave writes its part of C while the others go on, by way of 16 rows of 128 bytes in
// LDS that are its own, so that a store writes whole lines.
template <bool BF16, bool ADD, bool PAST, int WM, int WN, int TM, int TN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mx_stream(MxProductArgs a, Shape z)
{
    constexpr int kM = WM * TM * 16, kN = WN * TN * 16, kWaves = WM * WN, kStage = (kM + kN) * 68;
    constexpr int kCodeLoads = (kM + kN) / 16 / kWaves, kScaleLoads = ((kM + kN) / 64 + kWaves - 1) / kWaves;
    constexpr int kLoads = kCodeLoads + kScaleLoads, kSize = BF16 ? 2 : 4, kPitch = 144;
    static_assert((kM + kN) / 16 % kWaves == 0 && TM % 4 == 0 && TN == 4 && STAGES >= 2 && (STAGES - 1) * kLoads < 64, "");
    // (one array: with a second one the compiler waits for all loads before it reads either)
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * kStage + (ADD ? 0 : kWaves * 16 * kPitch)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    // (items to dies as above; a die's workgroups take its run in turn)
    const int die = blockIdx.x & 7, per_die = z.items >> 3, more = z.items & 7;
    const int end = (die + 1) * per_die + min(die + 1, more), stride = ((int)gridDim.x - die + 7) >> 3;
    int item = die * per_die + min(die, more) + (int)(blockIdx.x >> 3), m0, n0;
    struct Sources {
        const uint8_t *codes[kCodeLoads], *scales[kScaleLoads];
    } src, next_src;
    auto point = [&](int to, Sources &p) {
        const int band = to / (8 * z.tiles_n), in_band = to - band * 8 * z.tiles_n, high = min(z.tiles_m - 8 * band, 8);
        m0 = (8 * band + in_band % high) * kM;
        n0 = in_band / high * kN;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) {
            const int g = wave + i * kWaves;
            const bool is_a = g < kM / 16;
            const int group = is_a ? min(m0 / 16 + g, z.a_groups - 1) : min(n0 / 16 + g - kM / 16, z.b_groups - 1);
            p.codes[i] = (is_a ? a.a.codes : a.b.codes) + (int64_t)group * z.pieces * 1024;
        }
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const int g = (wave + i * kWaves) % ((kM + kN) / 64);
            const bool is_a = g < kM / 64;
            const int group = is_a ? min(m0 / 64 + g, z.a_groups / 4 - 1) : min(n0 / 64 + g - kM / 64, z.b_groups / 4 - 1);
            p.scales[i] = (is_a ? a.a.scales : a.b.scales) + (int64_t)group * z.pieces * 256;
        }
    };
    int left = z.pieces;                // of the tile that is being fetched
    auto fetch = [&](int slot) {
        uint8_t *to = lds + slot * kStage;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) to_lds<16>(src.codes[i] + lane * 16, to + (wave + i * kWaves) * 1024);
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) to_lds<4>(src.scales[i] + lane * 4, to + (kM + kN) * 64 + (wave + i * kWaves) % ((kM + kN) / 64) * 256);
        const bool over = --left == 0;
        left = over ? z.pieces : left;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) src.codes[i] = over ? next_src.codes[i] : src.codes[i] + 1024;
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) src.scales[i] = over ? next_src.scales[i] : src.scales[i] + 256;
    };
    const int la = wm * TM * 1024 + lane * 16, lb = (kM / 16 + wn * TN) * 1024 + lane * 16;
    const int sa = (kM + kN) * 64 + wm * TM / 4 * 256 + lane * 4, sb = (kM + kN) * 64 + kM * 4 + wn * TN / 4 * 256 + lane * 4;
    typedef Step<TM, TN> S;
    auto read = [&](int slot, S &f) {
        const uint8_t *from = lds + slot * kStage;
#pragma unroll
        for (int i = 0; i < TM / 4; ++i) f.ea[i] = *reinterpret_cast<const int *>(from + sa + i * 256);
#pragma unroll
        for (int i = 0; i < TN / 4; ++i) f.eb[i] = *reinterpret_cast<const int *>(from + sb + i * 256);
#pragma unroll
        for (int i = 0; i < TN; ++i) f.b[i] = *reinterpret_cast<const v4i *>(from + lb + i * 1024);
#pragma unroll
        for (int i = 0; i < TM; ++i) f.a[i] = *reinterpret_cast<const v4i *>(from + la + i * 1024);
    };
    f32x4 acc[TN][TM];
    int slot = 0;
    auto step = [&](const S &now, S &next) {
        const int after = slot + 1 == STAGES ? 0 : slot + 1;
        wait_loads<(STAGES - 2) * kLoads>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        fetch(slot);
        __builtin_amdgcn_sched_barrier(0);
        read(after, next);
        unroll<TM>([&](auto i) {
            unroll<TN>([&](auto j) {
                constexpr int I = decltype(i)::value, J = decltype(j)::value;
                acc[J][I] = mfma_mx<J % 4, I % 4>(now.b[J], now.a[I], acc[J][I], now.eb[J / 4], now.ea[I / 4]);
            });
        });
        unroll<TM + TN>([&](auto r) {
            constexpr int R = decltype(r)::value, kReads = TM + TN, kProducts = TM * TN;
            __builtin_amdgcn_sched_group_barrier(0x008, (R + 1) * kProducts / kReads - R * kProducts / kReads, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        });
        __builtin_amdgcn_sched_barrier(0);
        slot = after;
    };

    point(item, src);
    for (int s = 0; s < STAGES; ++s) fetch(s);          // (a tile has more pieces)
    wait_loads<(STAGES - 1) * kLoads>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    S even, odd;
    read(0, even);
    for (;;) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{};
        const int row0 = m0 + wm * TM * 16, col0 = n0 + wn * TN * 16;
        item += stride;
        const bool go_on = item < end;
        point(go_on ? item : item - stride, next_src);       // (behind the last tile: fetched for nothing)
        int s = 0;
        for (; s + 1 < z.pieces; s += 2) {
            step(even, odd);
            step(odd, even);
        }
        if (s < z.pieces) {
            step(even, odd);
            even = odd;
        }
        if constexpr (ADD) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; j += 2)
                    store_pair<BF16, ADD, PAST>(a, row0 + i * 16 + (lane & 15), col0 + j * 16, lane >> 4, acc[j][i], acc[j + 1][i]);
        } else {
            uint8_t *mine = lds + STAGES * kStage + wave * 16 * kPitch;
            constexpr int kUnit = 128 / kSize, kUnits = TN * 16 / kUnit, kPairs = kUnit / 32;
            auto write = [&](auto inside) {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int h = 0; h < kUnits; ++h) {
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) {
                            const f32x4 u = acc[2 * (h * kPairs + q)][i], v = acc[2 * (h * kPairs + q) + 1][i];
                            uint8_t *to = mine + (lane & 15) * kPitch + q * 32 * kSize;
                            if constexpr (BF16) {
                                uint32_t w[4];
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    auto x = __builtin_amdgcn_permlane16_swap(pack_bf16(a.alpha * u[2 * e], a.alpha * u[2 * e + 1]),
                                                                              pack_bf16(a.alpha * v[2 * e], a.alpha * v[2 * e + 1]), false, false);
                                    w[e] = x[0];
                                    w[2 + e] = x[1];
                                }
                                *reinterpret_cast<uint4 *>(to + 32 * ((lane >> 4) & 1) + 16 * (lane >> 5)) = make_uint4(w[0], w[1], w[2], w[3]);
                            } else {
                                *reinterpret_cast<float4 *>(to + 16 * (lane >> 4)) = make_float4(a.alpha * u[0], a.alpha * u[1], a.alpha * u[2], a.alpha * u[3]);
                                *reinterpret_cast<float4 *>(to + 64 + 16 * (lane >> 4)) = make_float4(a.alpha * v[0], a.alpha * v[1], a.alpha * v[2], a.alpha * v[3]);
                            }
                        }
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const int r = 8 * g + (lane >> 3), c = lane & 7;
                            const int64_t row = row0 + i * 16 + r, col = col0 + h * kUnit + c * (16 / kSize);
                            const uint4 w = *reinterpret_cast<const uint4 *>(mine + r * kPitch + c * 16);
                            if (!decltype(inside)::value && (row >= a.m || col >= a.n)) continue;
                            uint8_t *to = static_cast<uint8_t *>(a.c.data) + (row * a.c.pitch + col) * kSize;
                            if (decltype(inside)::value || col + 16 / kSize <= a.n) {
                                store_16<PAST>(to, u32x4_any{w.x, w.y, w.z, w.w});
                            } else {
                                const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                                for (int x = 0; x < 16 / kSize; ++x) {
                                    if (col + x >= a.n) continue;
                                    if constexpr (BF16) reinterpret_cast<uint16_t *>(to)[x] = (uint16_t)(e[x >> 1] >> (16 * (x & 1)));
                                    else reinterpret_cast<uint32_t *>(to)[x] = e[x];
                                }
                            }
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
            };
            if (row0 + TM * 16 <= a.m && col0 + TN * 16 <= a.n) write(std::true_type{});
            else write(std::false_type{});
        }
        if (!go_on) break;
    }
    wait_loads<0>();                    // what was fetched for nothing is in LDS before that is another workgroup's
}

// Few rows of A (16 MT at most): a workgroup takes 16 rows of B, read once, straight to registers; its WAVES waves take pieces of the long axis in
// turn, and their sums are added in order.  8 x 8192 x 2048, 9 MB: 2.8 us in a graph, 3.3 with the host's launch.
template <bool BF16, bool ADD, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_mx_rows(MxProductArgs a, int pieces)
{
    __shared__ f32x4 sums[WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = group_index();
    if (group * 16 >= a.n) return;
    const uint8_t *b = a.b.codes + group * pieces * 1024 + lane * 16, *eb = a.b.scales + (group >> 2) * pieces * 256 + lane * 4;
    const uint8_t *ac = a.a.codes + lane * 16, *ea = a.a.scales + lane * 4;
    const int shift = (int)(group & 3) * 8;
    f32x4 acc[MT] = {};
    constexpr int kDeep = 4;
    for (int p0 = wave; p0 < pieces; p0 += kDeep * WAVES) {
        v4i fb[kDeep], fa[kDeep][MT];
        int sb[kDeep], sa[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int p = min(p0 + d * WAVES, pieces - 1);
            fb[d] = *reinterpret_cast<const v4i *>(b + (int64_t)p * 1024);
            sb[d] = *reinterpret_cast<const int *>(eb + (int64_t)p * 256) >> shift;
            sa[d] = *reinterpret_cast<const int *>(ea + (int64_t)p * 256);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[d][i] = *reinterpret_cast<const v4i *>(ac + ((int64_t)i * pieces + p) * 1024);
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
            if (p0 + d * WAVES < pieces)
                unroll<MT>([&](auto i) {
                    constexpr int I = decltype(i)::value;
                    acc[I] = mfma_mx<0, I>(fb[d], fa[d][I], acc[I], sb[d], sa[d]);
                });
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += WAVES) {
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][i][lane];
        const int64_t row = i * 16 + (lane & 15), col = group * 16 + 4 * (lane >> 4);
        const float x[4] = {v[0], v[1], v[2], v[3]};
        if (row < a.m && col < a.n) store_row<BF16, ADD, false, 4>(a, row, col, x);
    }
}

// Adds the parts of the long axis in their order, four columns a thread.
template <bool BF16, bool ADD>
__global__ __launch_bounds__(256) void k_mx_join(MxProductArgs a, int parts, uint32_t fours_a_row)
{
    const uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = (int64_t)(t / fours_a_row), col = (int64_t)(t % fours_a_row) * 4;
    if (row >= a.m) return;
    const int left = (int)(a.n - col < 4 ? a.n - col : 4);
    float v[4] = {};
    for (int p = 0; p < parts; ++p) {
        const float *from = a.partials + ((int64_t)p * a.m + row) * a.n + col;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) v[i] += from[i];
    }
    store_row<BF16, ADD, false, 4>(a, row, col, v);
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

enum Tiles { kRows, kTiny, kSmall, kWide, kLarge, kStream };

struct Choice {
    Tiles tiles;
    int parts, per_part;                // of the long axis
};

constexpr int kCus = 256;

// Which kernel, and whether C goes past the caches.  us of a call (bf16 C, beta = 0 unless said otherwise; two kernels' times are of one session, and between
// sessions and boxes a kernel's differs by some 4 %), the one taken / the next best:
//   rows (m <= 64)   8 x 8192 x 2048 2.7 / 4.8 tiny (in graphs), 1 x 50304 x 2048 11.3 / 11.8 small, 64 x 2048 x 8192 5.4 / 9.8 tiny in 4 parts; but more
//                    than 16 rows are read once a workgroup, which with enough of these costs more than a tile's waste: 64 x 50304 x 16384 166 / 86
//                    small, 32 x 16384 x 8192 15.1 / 13.3, 64 x 50304 x 2048 21.6 / 19.4 (32 x 50304 x 2048 14.5 / 17.7)
//   stream, 256 x 256, one tile after the other, from four to a CU on:  8192 x 8192 x 8192 240 / 249 large, 4096 x 50304 x 2048 215 / 224 wide,
//                    8192 x 8192 x 1536 53 / 58 wide, 16384 x 8192 x 4096 241 / 261 large; but 6144 x 4096 x 2048 33 / 28 wide
//   large, 256 x 256, eight waves: the fewest reads, but a CU holds one workgroup, which begins and ends alone; for long sums of fewer
//                    tiles: 8192 x 2048 x 8192, one tile a CU, 60 / 66 wide, 63 stream.  No rule here looks at what is left of tiles over CUs: a little more than one
//                    a CU are two turns, and there wide ones would be better: 8448 x 2048 x 8192 99 / 88 wide, 100 stream; 9984 x 2048 x 8192 101 / 91 wide
//   wide, 256 x 128, two workgroups a CU:  4096 x 8192 x 2048 38.7 / 38.1 stream; 8192 x 32768 x 1024 184 small / 190
//   small, 128 x 128, three a CU:  2048 x 50304 x 768 65 / 69 wide, 2048 x 2048 x 16384 43 / 56 in 2 parts, 60 tiny; 512 x 8192 x 2048 9.4 / 11.8 tiny; and where half
//                    of a larger one would be beyond the rows: 128 x 50304 x 8192 37 / 50 large
//   tiny, 64 x 64, where small ones do not reach every CU:  1024 x 1024 x 1024 4.0 / 5.6, 16384 x 16 x 4096 8.4 / 11.7, 128 x 4096 x 1024 3.8 / 5.5
// The long axis in parts, added up by a launch of its own: 256 x 256 x 8192 9.4 in 4 parts / 12.6, but 200 x 1024 x 4096 8.7 in 2 / 7.6.
// Past the caches what those of the dies do not hold: 8192 x 32768 x 1024 184 / 270, 8192 x 8192 x 2048 in fp32 88 / 97, 4096 x 8192 x 2048 42 / 43;
// streams only what the card's last cache does not hold either: 4096 x 50304 x 2048 205 / 236, but 8192 x 8192 x 2048 75 / 67; large tiles nothing, as
// fewer than 1024 of them are a C of less than that cache.
// And not rows that end within 64 bytes, of which halves would be written twice (within 16 if the last cache does not hold C): 2000 x 50300 x 300
// 46 / 89, 4096 x 50303 x 2048 290 / 336, 8192 x 16001 x 700 87 / 128; but 8192 x 32760 x 1024 218 past the caches / 280.
Choice choose(int64_t m, int64_t n, int64_t k)
{
    const int64_t pieces = std::max<int64_t>((k + 127) / 128, 1);
    auto tiles = [&](int64_t tm, int64_t tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); };
    const bool deep = m > 16 && tiles(64, 64) >= kCus && (m + 15) / 16 * pieces >= 64;
    if (m <= 64 && !deep) return {kRows, 1, (int)pieces};
    if (std::min(m, n) > 128 && tiles(256, 256) >= 192 && pieces >= 12) return {tiles(256, 256) >= 4 * kCus ? kStream : pieces >= 32 ? kLarge : kWide, 1, (int)pieces};
    if (tiles(128, 128) >= 200) return {kSmall, 1, (int)pieces};
    const int64_t parts = pieces < 64 ? 1 : std::max<int64_t>(std::min<int64_t>(kCus / tiles(64, 64), pieces / 16), 1);
    const int64_t per = (pieces + parts - 1) / parts;
    return {kTiny, (int)((pieces + per - 1) / per), (int)per};
}

template <bool BF16, bool ADD, bool PAST, int WM, int WN, int TM, int TN, int STAGES, int WAVES>
void launch_tiles(const MxProductArgs &a, const Choice &c, hipStream_t st)
{
    constexpr int kM = WM * TM * 16, kN = WN * TN * 16;
    Shape z;
    z.pieces = (int)((a.k + 127) / 128);
    z.a_groups = (int)((a.m + 63) / 64 * 4);
    z.b_groups = (int)((a.n + 63) / 64 * 4);
    z.tiles_m = (int)((a.m + kM - 1) / kM);
    z.tiles_n = (int)((a.n + kN - 1) / kN);
    z.per_part = c.per_part;
    z.items = z.tiles_m * z.tiles_n * c.parts;
    hipLaunchKernelGGL((k_mx_product<BF16, ADD, PAST, WM, WN, TM, TN, STAGES, WAVES>), dim3((unsigned)z.items), dim3(64 * WM * WN), 0, st, a, z);
}

template <bool BF16, bool ADD, bool PAST>
void launch_stream(const MxProductArgs &a, hipStream_t st)
{
    Shape z;
    z.pieces = z.per_part = (int)((a.k + 127) / 128);
    z.a_groups = (int)((a.m + 63) / 64 * 4);
    z.b_groups = (int)((a.n + 63) / 64 * 4);
    z.tiles_m = (int)((a.m + 255) / 256);
    z.tiles_n = (int)((a.n + 255) / 256);
    z.items = z.tiles_m * z.tiles_n;
    hipLaunchKernelGGL((k_mx_stream<BF16, ADD, PAST, 2, 4, 8, 4, 4>), dim3((unsigned)std::min(z.items, kCus)), dim3(512), 0, st, a, z);
}

template <bool BF16, bool ADD>
void launch_rows(const MxProductArgs &a, hipStream_t st)
{
    const int64_t groups = (a.n + 15) / 16;
    const int pieces = (int)((a.k + 127) / 128);
    auto go = [&](auto mt, auto waves) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((k_mx_rows<BF16, ADD, decltype(mt)::value, W>), grid_of(groups), dim3(64 * W), 0, st, a, pieces);
    };
    auto by_waves = [&](auto mt) {
        if (pieces > 4 && (groups < 2 * kCus || pieces >= 64)) go(mt, std::integral_constant<int, 8>{});
        else go(mt, std::integral_constant<int, 4>{});
    };
    if (a.m <= 16) by_waves(std::integral_constant<int, 1>{});
    else if (a.m <= 32) by_waves(std::integral_constant<int, 2>{});
    else by_waves(std::integral_constant<int, 4>{});
}

}  // namespace

size_t mx_product_workspace(int64_t m, int64_t n, int64_t k)
{
    const Choice c = choose(m, n, k);
    return c.parts > 1 ? (size_t)c.parts * (size_t)m * (size_t)n * sizeof(float) : 0;
}

void launch_mx_product(const MxProductArgs &a, bool bf16, hipStream_t st)
{
    const Choice c = choose(a.m, a.n, a.k);
    if (c.parts > 1) {
        MxProductArgs p = a;
        p.alpha = 1.0f;                     // (beta is for the launch that adds the parts)
        launch_tiles<false, false, false, 2, 2, 2, 2, 4, 4>(p, c, st);
    }
    const int64_t size = bf16 ? 2 : 4, bytes = a.m * a.n * size, last = (int64_t)256 << 20;
    const int64_t ends = (a.c.pitch * size) | (int64_t)reinterpret_cast<uintptr_t>(a.c.data);
    const bool past = bytes > (c.tiles == kStream ? last : last / 8) && (ends % 64 == 0 || (ends % 16 == 0 && bytes > last));
    by_bool(bf16, [&](auto b) {
        by_bool(a.beta != 0.0f, [&](auto add) {
            constexpr bool B = decltype(b)::value, ADD = decltype(add)::value;
            if (c.tiles == kRows) {
                launch_rows<B, ADD>(a, st);
            } else if (c.parts > 1) {
                const uint32_t fours = (uint32_t)((a.n + 3) / 4);
                hipLaunchKernelGGL((k_mx_join<B, ADD>), dim3((unsigned)(((uint64_t)a.m * fours + 255) / 256)), dim3(256), 0, st, a, c.parts,
                                   fours);
            } else if (c.tiles == kTiny) {
                launch_tiles<B, ADD, false, 2, 2, 2, 2, 4, 4>(a, c, st);
            } else if (c.tiles == kLarge) {
                launch_tiles<B, ADD, false, 2, 4, 8, 4, 4, 2>(a, c, st);
            } else {
                by_bool(past, [&](auto p) {
                    constexpr bool PAST = decltype(p)::value;
                    if (c.tiles == kSmall) launch_tiles<B, ADD, PAST, 2, 2, 4, 4, 3, 3>(a, c, st);
                    else if (c.tiles == kStream) launch_stream<B, ADD, PAST>(a, st);
                    else launch_tiles<B, ADD, PAST, 2, 2, 8, 4, 3, 2>(a, c, st);
                });
            }
        });
    });
}

}  // namespace conef
