// Products A B^T whose operands lie in steps of 128 bytes along the long axis, whatever their elements are: 128 of 8 bits, 64 of 16, 32
// of 32.  A step of 32 rows is the same fragment in every case, 64 bytes a lane in two halves; only the instructions that
// multiply it differ.  Also what such kernels share with others: loads to LDS, waits, loops that are unrolled with constants.
#pragma once
#include <type_traits>
#include <utility>

#include "layers_device.h"

namespace conef {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// What A's elements are; B's are the same, but E4M3 beside E5M2.  The instructions that take 8 bits add sixteen products at a time to 13 bits below the
// largest of them (what is below is cut off) and that to the sum in fp32.  WIDE_*: elements are widened to bf16, times their scale, on their way to
// the instructions of 16 bits, whose products and sums have all bits of fp32; these take twice as long.  Both ways hold what elements stand for exactly (in bf16 down
// to 2^-133).
struct Kind {
    static constexpr int E4M3 = 0, E5M2 = 1, BF16 = 2, F32 = 3, WIDE_E4M3 = 4, WIDE_E5M2 = 5;
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// eight elements of 8 bits times the scale of byte `byte` (255: NaN)
template <bool E5M2>
__device__ __forceinline__ bf16x8 widen_octet(int lo, int hi, int byte)
{
    const float scale = __uint_as_float((uint32_t)byte << 23);
    bf16x2 v[4];
    if constexpr (E5M2) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    }
    return bf16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

constexpr int kCus = 256;

static __device__ const uint32_t kZeros[4] = {};

// An operand.  By rows: `rows` of them, `pitch` bytes apart, pitch (below 2^29) and address multiples of 16.  Packed: squares of 16 rows and 16 bytes,
// 256 bytes each, eight of them a step (2048 bytes), the steps of 16 rows one after the other; `rows` a multiple of 16.
// 8 bits, packed only: `scales` holds `rows` bytes a step, and rows is a multiple of 64.
struct Side {
    const uint8_t *data = nullptr, *scales = nullptr;
    int64_t pitch = 0;
    int rows = 0;
};

// A product in tiles; items are tiles times parts of the long axis (`per_part` steps, the last may have fewer), parts outermost.  `last`: bytes of the
// last step that are elements, a multiple of 16 (by rows; packed operands are filled up with zeros).
struct Shape {
    int steps = 0, last = 128, tiles_m = 0, tiles_n = 0, per_part = 0, items = 0;
};

// Workgroups go to the eight dies in turn; each die gets a run of neighbouring items, rows of tiles in eights, so that what its workgroups read
// at one time stays in its cache.
struct Place {
    int m, n, part;             // in tiles
};
__device__ __forceinline__ Place place_of(const Shape &z, int block)
{
    const int die = block & 7, per_die = z.items >> 3, more = z.items & 7, tiles = z.tiles_m * z.tiles_n;
    const int item = die * per_die + (die < more ? die : more) + (block >> 3), tile = item % tiles;
    const int band = tile / (8 * z.tiles_n), in_band = tile - band * 8 * z.tiles_n, high = min(z.tiles_m - 8 * band, 8);
    return {8 * band + in_band % high, in_band / high, item / tiles};
}

// WM x WN waves of TM x TN tiles of 32 x 32, STAGES steps in LDS.  A step is two halves of 64 bytes: while one is multiplied the next is read
// from LDS, and behind the first half's products, when a wave has all of a step in registers, the step STAGES on is fetched into its
// place.  So there is one barrier a step, and what it waits for was asked for a step before.
template <int KIND, bool BY_ROWS, int WM, int WN, int TM, int TN, int STAGES>
struct Tile {
    static constexpr bool kWide = KIND == Kind::WIDE_E4M3 || KIND == Kind::WIDE_E5M2, kScaled = KIND == Kind::E4M3 || KIND == Kind::E5M2 || kWide;
    static constexpr int kM = WM * TM * 32, kN = WN * TN * 32, kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kCodes = (kM + kN) * 128, kStage = kCodes + (kScaled ? 512 : 0), kBytes = STAGES * kStage;
    static constexpr int kUnits = (kM + kN) / 8 / kWaves, kLoads = kUnits + (kScaled ? 1 : 0);
    static_assert((kM + kN) / 8 % kWaves == 0 && kM <= 256 && kN <= 256 && STAGES >= 2, "");
    static_assert(!kScaled || (!BY_ROWS && kWaves % 2 == 0), "");
    static_assert((STAGES - 1) * kLoads < 64, "the counter of loads");
    // a wave's 32 rows of an output on their way through LDS
    static constexpr int kPitch = TN * 32 + 4;
    static_assert(kWaves * 32 * kPitch * 4 <= kBytes, "");

    struct Half {
        v8i a[TM], b[TN];
        int ea[kScaled ? TM : 1], eb[kScaled ? TN : 1];
    };

    typedef f32x16 Sums[TN][TM];

    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ int wave_m() { return wave() % WM; }
    static __device__ __forceinline__ int wave_n() { return wave() / WM; }

    // The first operand of the instructions is B's rows: then a lane holds, of one row of the product (lane % 32), columns 8 q + 4 (lane / 32) + e
    // of 32 in registers 4 q + e.
    static __device__ __forceinline__ void multiply(const v8i &b, const v8i &a, f32x16 &c, int eb, int ea)
    {
        if constexpr (kScaled) {
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, KIND == Kind::E5M2 ? 1 : 0, 0, eb, 0, ea);
        } else if constexpr (KIND == Kind::BF16) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const v4i x = {b[4 * q], b[4 * q + 1], b[4 * q + 2], b[4 * q + 3]}, y = {a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(b[q]), __int_as_float(a[q]), c, 0, 0, 0);
        }
    }
    static constexpr int kEach = kWide ? 4 : kScaled ? 1 : KIND == Kind::BF16 ? 2 : 8;          // instructions of a multiply

    // acc <- rows m0 .. of A times rows n0 .. of B, over `steps` steps from `first` on.  Rows beyond an operand's last are some other of its
    // rows (what comes of them is not used).
    static __device__ __forceinline__ void run(const Side &a, const Side &b, const Shape &z, int m0, int n0, int first, int steps, uint8_t *lds, Sums &acc)
    {
        const int lane = threadIdx.x & 63, w = wave();
        // what this wave fetches: 1024 bytes at a time, eight rows or half of sixteen; 256 of scales
        const uint8_t *src[kUnits], *scale_src = nullptr;
        uint32_t off[BY_ROWS ? kUnits : 1];
        int scale_step = 0;
        if constexpr (BY_ROWS) {
            // (a row is less than 2^29 bytes from the next: seven of these fit 32 bits)
            const int r = lane >> 3, chunk = (lane & 7) ^ r;
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int row = 8 * (w + i * kWaves);
                const bool is_a = row < kM;
                const int at = is_a ? m0 + row : n0 + row - kM, rows = is_a ? a.rows : b.rows;
                const int64_t pitch = is_a ? a.pitch : b.pitch;
                const int from = min(at, rows - 1);
                src[i] = (is_a ? a.data : b.data) + from * pitch + (int64_t)first * 128;
                off[i] = (uint32_t)((min(at + r, rows - 1) - from) * (uint32_t)pitch) + chunk * 16;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int unit = w + i * kWaves;
                const bool is_a = unit < kM / 8;
                const int group = is_a ? min(m0 / 16 + unit / 2, a.rows / 16 - 1) : min(n0 / 16 + (unit - kM / 8) / 2, b.rows / 16 - 1);
                src[i] = (is_a ? a.data : b.data) + ((int64_t)group * z.steps + first) * 2048 + (unit & 1) * 1024;
            }
            if constexpr (kScaled) {
                const Side &of = w & 1 ? b : a;
                scale_step = of.rows;
                scale_src = of.scales + (int64_t)first * of.rows + min((w & 1 ? n0 : m0) + lane * 4, of.rows - 4);
            }
        }
        auto fetch = [&](int s, int slot) {
            uint8_t *to = lds + slot * kStage;
            if constexpr (BY_ROWS) {
                if (first + s + 1 == z.steps && z.last < 128) {         // what is behind a row's end is zeros
                    const bool there = ((lane & 7) ^ (lane >> 3)) * 16 < z.last;
#pragma unroll
                    for (int i = 0; i < kUnits; ++i)
                        to_lds<16>(there ? src[i] + (int64_t)s * 128 + off[i] : reinterpret_cast<const uint8_t *>(kZeros), to + (w + i * kWaves) * 1024);
                    return;
                }
#pragma unroll
                for (int i = 0; i < kUnits; ++i) to_lds<16>(src[i] + (int64_t)s * 128 + off[i], to + (w + i * kWaves) * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < kUnits; ++i) to_lds<16>(src[i] + (int64_t)s * 2048 + lane * 16, to + (w + i * kWaves) * 1024);
                if constexpr (kScaled) to_lds<4>(scale_src + (int64_t)s * scale_step, to + kCodes + (w & 1) * 256);
            }
        };
        // Where this lane's fragments begin: row lane % 32; of a half's four pieces of 16 bytes two, by lane / 32.  By rows a row's pieces lie exchanged, by the
        // row, so that neither way of reading has a bank conflict.
        const int r = lane & 31, g = lane >> 5;
        int at[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int chunk = 4 * h + 2 * g + q;
                at[h][q] = BY_ROWS ? (r >> 3) * 1024 + (r & 7) * 128 + (chunk ^ (r & 7)) * 16 : (r >> 4) * 2048 + chunk * 256 + (r & 15) * 16;
            }
        const int la = wave_m() * TM * 4096, lb = kM * 128 + wave_n() * TN * 4096;
        auto read = [&](int slot, auto half, Half &f) {
            constexpr int H = decltype(half)::value;
            const uint8_t *from = lds + slot * kStage;
            auto one = [&](const uint8_t *p) {
                const v4i lo = *reinterpret_cast<const v4i *>(p + at[H][0]), hi = *reinterpret_cast<const v4i *>(p + at[H][1]);
                return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            };
            if constexpr (kScaled) {
#pragma unroll
                for (int i = 0; i < TM; ++i) f.ea[i] = from[kCodes + (wave_m() * TM + i) * 32 + r];
#pragma unroll
                for (int j = 0; j < TN; ++j) f.eb[j] = from[kCodes + 256 + (wave_n() * TN + j) * 32 + r];
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) f.b[j] = one(from + lb + j * 4096);
#pragma unroll
            for (int i = 0; i < TM; ++i) f.a[i] = one(from + la + i * 4096);
        };
        constexpr int kReads = (TM + TN) * (kScaled ? 3 : 2), kProducts = TM * TN * kEach;
        auto products = [&](const Half &f) {
            if constexpr (kWide) {
                unroll<4>([&](auto q) {
                    constexpr int Q = decltype(q)::value;
                    bf16x8 x[TN], y[TM];
#pragma unroll
                    for (int j = 0; j < TN; ++j) x[j] = widen_octet<false>(f.b[j][2 * Q], f.b[j][2 * Q + 1], f.eb[j]);
#pragma unroll
                    for (int i = 0; i < TM; ++i) y[i] = widen_octet<KIND == Kind::WIDE_E5M2>(f.a[i][2 * Q], f.a[i][2 * Q + 1], f.ea[i]);
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j], y[i], acc[j][i], 0, 0, 0);
                });
            } else {
                unroll<TM>([&](auto i) {
                    unroll<TN>([&](auto j) {
                        constexpr int I = decltype(i)::value, J = decltype(j)::value;
                        multiply(f.b[J], f.a[I], acc[J][I], f.eb[kScaled ? J : 0], f.ea[kScaled ? I : 0]);
                    });
                });
            }
            // a few reads behind every few products: reads wait for LDS in the order of their issue, and products behind them would wait with them
            constexpr int kTurns = kProducts < 8 ? kProducts : 8;
            unroll<kTurns>([&](auto t) {
                constexpr int T = decltype(t)::value;
                __builtin_amdgcn_sched_group_barrier(0x008, (T + 1) * kProducts / kTurns - T * kProducts / kTurns, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (T + 1) * kReads / kTurns - T * kReads / kTurns, 0);
            });
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[j][i] = f32x16{};
        const std::integral_constant<int, 0> low;
        const std::integral_constant<int, 1> high;
        int slot = 0;
        Half even, odd;
        for (int s = 0; s < min(steps, STAGES); ++s) fetch(s, s);
        if (steps >= STAGES) wait_loads<(STAGES - 1) * kLoads>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, low, even);
        __builtin_amdgcn_sched_barrier(0);
        auto step = [&](int s, auto steady) {
            const int after = slot + 1 == STAGES ? 0 : slot + 1;
            read(slot, high, odd);
            products(even);
            wait_loads<decltype(steady)::value ? (STAGES - 2) * kLoads : 0>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (decltype(steady)::value || s + STAGES < steps) fetch(s + STAGES, slot);
            __builtin_amdgcn_sched_barrier(0);
            read(after, low, even);             // (behind the last step: what is left there, for nothing)
            products(odd);
            slot = after;
        };
        int s = 0;
        for (; s + STAGES < steps; ++s) step(s, std::true_type{});
        for (; s < steps; ++s) step(s, std::false_type{});
    }

    // The product by eight neighbours of a row at a time, by way of LDS, where each wave turns 32 rows of its own: f(row, col, v) of the tile's row and
    // column and eight sums; a wave's lanes hold eight rows of TN * 32 columns (TN = 2; else sixteen of 32).
    template <typename F>
    static __device__ __forceinline__ void octets(const Sums &acc, uint8_t *lds, F &&f)
    {
        const int lane = threadIdx.x & 63;
        float *mine = reinterpret_cast<float *>(lds) + wave() * 32 * kPitch;
        wait_loads<0>();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4 *>(mine + (lane & 31) * kPitch + j * 32 + 8 * q + 4 * (lane >> 5)) =
                        f32x4{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
            __builtin_amdgcn_wave_barrier();
            constexpr int kAcross = TN * 4, kHigh = 64 / kAcross;
#pragma unroll
            for (int t = 0; t < 32 / kHigh; ++t) {
                const int r = t * kHigh + lane / kAcross, c = lane % kAcross * 8;
                const f32x4 x = *reinterpret_cast<const f32x4 *>(mine + r * kPitch + c), y = *reinterpret_cast<const f32x4 *>(mine + r * kPitch + c + 4);
                float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                f((wave_m() * TM + i) * 32 + r, wave_n() * TN * 32 + c, v);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// alpha v + beta c of eight neighbours of C's row, `left` of them there
template <bool BF16, bool ADD, bool PAST>
__device__ __forceinline__ void put_octet(const RowsOut &c, int64_t row, int64_t col, int left, float alpha, float beta, float v[8])
{
    const int64_t at = row * c.pitch + col;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = alpha * v[i];
    if constexpr (ADD) {
        float old[8];
        load_octet<BF16>(c.data, at, left, old);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(beta, old[i], v[i]);
    }
    store_octet<BF16, PAST>(c.data, at, left, v);
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace conef
