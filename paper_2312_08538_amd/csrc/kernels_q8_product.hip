// C = alpha A B^T + beta C of two packed operands of 8-bit floating point with a scale for each block of 128, on the matrix instructions that take such
// operands with powers of two as scales (v_mfma_scale_f32_16x16x128_f8f6f4): the scale costs nothing, and a sum stays in
// its register from the first step of the long axis to the last.  C in fp32 is summed by the instructions of 16 bits (Kind::WIDE_*).
//
// What bounds it: on random operands these instructions alone reach 4.1 to 4.3 PFLOP/s here (the 32 x 32 x 64 ones 3.7 to 3.8).  8192 x 8192 x 2048 into bf16 takes 121 to 125 us, 2.2 PFLOP/s, and
// 8192 x 2048 x 8192 103 us, 2.7: the matrix units are busy in 51 and 66 % of the cycles and waves wait in 32 and 26 % of theirs, whatever the clock (which falls under load, besides).  Two steps are all that LDS
// holds of the large tiles, so that a step's loads are waited for from half a step behind the asking on; and of 134 MB of C, 26 us at a copy's rate, little overlaps.
// Into fp32 240 to 262 and 196 to 204 (1.1 and 1.4 PFLOP/s; 16-bit instructions alone: 1.9 to 2.0): with eight rows of tiles a wave widens B's fragments again for each of them.
#include <algorithm>

#include "product_device.h"

namespace conef {

namespace {

template <int KIND, bool BF16, bool ADD, bool PAST, int WM, int WN, int TM, int TN, int STAGES, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void k_q8_product(Q8ProductArgs p, Side a, Side b, Shape z)
{
    typedef Tile<KIND, false, WM, WN, TM, TN, STAGES> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kBytes];
    if (group_index() >= (uint32_t)z.items) return;
    const Place at = place_of(z, (int)group_index());
    const int first = at.part * z.per_part;
    typename T::Sums acc;
    T::run(a, b, z, at.m * T::kM, at.n * T::kN, first, min(z.per_part, z.steps - first), lds, acc);
    if (p.partials) {
        p.c.data = p.partials + (int64_t)at.part * p.m * p.n;
        p.c.pitch = p.n;
    }
    if constexpr (BF16 && !ADD) {
        T::template store_bf16<PAST>(acc, lds, p.c, p.m, p.n, (int64_t)at.m * T::kM, (int64_t)at.n * T::kN, p.alpha);
        return;
    }
    T::octets(acc, lds, [&](int r, int c, float v[8]) {
        const int64_t row = (int64_t)at.m * T::kM + r, col = (int64_t)at.n * T::kN + c;
        if (row < p.m && col < p.n) put_octet<BF16, ADD, PAST>(p.c, row, col, octet_left(p.n - col), p.alpha, p.beta, v);
    });
}

// Few rows of A (16 MT at most): a workgroup takes 16 rows of B, read once, straight to registers; its WAVES waves take steps of the long axis in
// turn, and their sums are added in order.  Elements are widened for it: the products hide behind the loads.  Bound by B's bytes where B is large (1 x 50304 x 2048 17.5 us,
// 5.9 TB/s), else by the way to memory and back: 8 x 8192 x 2048 3.8 us, a launch 2.6.
template <bool E5M2, bool BF16, bool ADD, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_q8_rows(Q8ProductArgs p, int steps, int64_t a_rows, int64_t b_rows)
{
    __shared__ f32x4 sums[WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int64_t group = group_index();
    if (group * 16 >= p.n) return;
    const uint8_t *b = p.b.codes + group * steps * 2048 + g * 512 + r * 16, *eb = p.b.scales + group * 16 + r;
    const uint8_t *a = p.a.codes + g * 512 + r * 16, *ea = p.a.scales + r;
    f32x4 acc[MT] = {};
    constexpr int kDeep = MT == 4 ? 2 : 4;
    for (int s0 = wave; s0 < steps; s0 += kDeep * WAVES) {
        v4i fb[kDeep][2], fa[kDeep][MT][2];
        int sb[kDeep], sa[kDeep][MT];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int64_t s = min(s0 + d * WAVES, steps - 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) fb[d][h] = *reinterpret_cast<const v4i *>(b + s * 2048 + h * 256);
            sb[d] = eb[s * b_rows];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int h = 0; h < 2; ++h) fa[d][i][h] = *reinterpret_cast<const v4i *>(a + (i * steps + s) * 2048 + h * 256);
                sa[d][i] = ea[s * a_rows + 16 * i];
            }
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
            if (s0 + d * WAVES < steps)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bf16x8 x = widen_octet<false>(fb[d][q >> 1][2 * (q & 1)], fb[d][q >> 1][2 * (q & 1) + 1], sb[d]);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const bf16x8 y = widen_octet<E5M2>(fa[d][i][q >> 1][2 * (q & 1)], fa[d][i][q >> 1][2 * (q & 1) + 1], sa[d][i]);
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[i], 0, 0, 0);
                    }
                }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += WAVES) {
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][i][lane];
        // four columns of a row: the row's neighbour quad is 16 lanes on, so even quads write eight
        const int64_t row = i * 16 + r, col = group * 16 + 8 * (g >> 1);
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[e]), __float_as_uint(v[e]), false, false);
            x[e] = __uint_as_float(s[0]);
            x[4 + e] = __uint_as_float(s[1]);
        }
        if (!(g & 1) && row < p.m && col < p.n) put_octet<BF16, ADD, false>(p.c, row, col, octet_left(p.n - col), p.alpha, p.beta, x);
    }
}

// Adds the parts of the long axis in their order, eight columns a thread.
template <bool BF16, bool ADD>
__global__ __launch_bounds__(256) void k_q8_join(Q8ProductArgs p, int parts, uint32_t octets_a_row)
{
    const uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = (int64_t)(t / octets_a_row), col = (int64_t)(t % octets_a_row) * 8;
    if (row >= p.m) return;
    const int left = octet_left(p.n - col);
    float v[8] = {};
    for (int part = 0; part < parts; ++part) {
        float x[8];
        load_octet<false>(p.partials, ((int64_t)part * p.m + row) * p.n + col, left, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += x[i];
    }
    put_octet<BF16, ADD, false>(p.c, row, col, left, p.alpha, p.beta, v);
}

enum Tiles { kRows, kTiny, kSmall, kWide, kLarge };

struct Choice {
    Tiles tiles;
    int parts, per_part;                // of the long axis
};

// Which kernel.  us of a call in a graph, the one taken / others (C in bf16; in fp32, where the matrix instructions take twice as long and elements are widened, after a
// semicolon):
//   rows    8 x 8192 x 2048 3.9 / 6.2 tiny; 3.9 / 9.9.  More than 16 rows are read again by every workgroup: 64 x 8192 x 2048 6.2 / 6.4; 6.3 / 10.4, but 64 x 50304 x 2048 27.3 / 21.1 tiny;
//           30.1 / 25.8, and over a long axis, which tiles cut in parts, 64 x 2048 x 8192 14.4 / 10.4 in 4; 14.7 / 14.3
//   large   256 x 256, one workgroup a CU: 4096 x 4096 x 2048 32.3 / 36.6 wide, 37.2 small; 4096 x 8192 x 2048 65.0 / 68.5, 69.0; 8192 x 2048 x 8192 103 / 117; fp32: 197 / 228
//   wide    256 x 128, where large ones do not reach most CUs: 4096 x 2048 x 8192 60.1 / 71.7 small, 81.3 large; 116 / 121, 162
//   small   128 x 128: 512 x 8192 x 2048 14.3 / 17.0 wide, 17.5 tiny; 25.2 / 32.1, 27.9; 2048 x 2048 x 2048 13.4 / 16.7, 16.5; 24.4 / 31.9, 26.3.  And where a tile's end weighs as much as its
//           steps: 16384 x 4096 x 512 51.5 / 55.6 large; 90.5 / 135; into fp32 up to 32 steps: 4096 x 8192 x 2048 127 / 149
//   tiny    64 x 64: 1000 x 1203 x 515 5.5 / 7.5 small; 7.5 / 10.1; 128 x 4096 x 1024 4.8 / 7.6; 7.1 / 12.2
// The long axis in parts, added up by a launch of its own: 256 x 256 x 8192 10.3 in 8, 9.9 in 4 / 15.3; 12.1, 13.6 / 30.0; 300 x 2000 x 9000 16.5 in 3 / 17.5; 22.8 / 34.1.
Choice choose(int64_t m, int64_t n, int64_t k, bool bf16)
{
    const int64_t steps = std::max<int64_t>((k + 127) / 128, 1);
    auto tiles = [&](int64_t tm, int64_t tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); };
    // (no columns: no tiles, whose number divides below, and no launch)
    if (n == 0 || m <= 16 || (m <= 64 && steps < 32 && tiles(64, 64) < kCus)) return {kRows, 1, (int)steps};
    if (std::min(m, n) > 128 && steps >= (bf16 ? 8 : 32)) {
        if (tiles(256, 256) >= 192) return {kLarge, 1, (int)steps};
        if (tiles(256, 128) >= 192) return {kWide, 1, (int)steps};
    }
    if (m > 64 && tiles(128, 128) >= 200) return {kSmall, 1, (int)steps};
    const int64_t parts = steps < 32 ? 1 : std::max<int64_t>(std::min<int64_t>(2 * kCus / tiles(64, 64), steps / 8), 1);
    const int64_t per = (steps + parts - 1) / parts;
    return {kTiny, (int)((steps + per - 1) / per), (int)per};
}

template <int KIND, bool BF16, bool ADD, bool PAST, int WM, int WN, int TM, int TN, int STAGES, int OCC>
void launch_tiles(const Q8ProductArgs &p, const Choice &c, hipStream_t st)
{
    constexpr int kM = WM * TM * 16, kN = WN * TN * 16;
    Shape z;
    z.steps = (int)((p.k + 127) / 128);
    z.tiles_m = (int)((p.m + kM - 1) / kM);
    z.tiles_n = (int)((p.n + kN - 1) / kN);
    z.per_part = c.per_part;
    z.items = z.tiles_m * z.tiles_n * c.parts;
    Side a, b;
    a.data = p.a.codes, a.scales = p.a.scales, a.rows = (int)((p.m + 63) / 64 * 64);
    b.data = p.b.codes, b.scales = p.b.scales, b.rows = (int)((p.n + 63) / 64 * 64);
    hipLaunchKernelGGL((k_q8_product<KIND, BF16, ADD, PAST, WM, WN, TM, TN, STAGES, OCC>), grid_of(z.items), dim3(64 * WM * WN), 0, st, p, a, b, z);
}

template <bool E5M2, bool BF16, bool ADD>
void launch_rows(const Q8ProductArgs &p, hipStream_t st)
{
    const int64_t groups = (p.n + 15) / 16;
    const int steps = (int)((p.k + 127) / 128);
    auto go = [&](auto mt, auto waves) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((k_q8_rows<E5M2, BF16, ADD, decltype(mt)::value, W>), grid_of(groups), dim3(64 * W), 0, st, p, steps, (p.m + 63) / 64 * 64,
                           (p.n + 63) / 64 * 64);
    };
    // Eight waves where there are few workgroups, or a long axis keeps each busy: 8 x 2048 x 8192 5.5 us / 6.7 on four, 16 x 1024 x 16384 7.2 / 8.4, 8 x 8192 x 2048 3.8 / 3.8.
    auto by_waves = [&](auto mt) {
        if (steps > 4 && (groups < 2 * kCus || steps >= 64)) go(mt, std::integral_constant<int, 8>{});
        else go(mt, std::integral_constant<int, 4>{});
    };
    if (p.m <= 16) by_waves(std::integral_constant<int, 1>{});
    else if (p.m <= 32) by_waves(std::integral_constant<int, 2>{});
    else by_waves(std::integral_constant<int, 4>{});
}

}  // namespace

size_t q8_product_workspace(int64_t m, int64_t n, int64_t k)
{
    const Choice c = choose(m, n, k, true);             // (parts are of the smallest tiles, which either type takes for the same sizes)
    return c.parts > 1 ? (size_t)c.parts * (size_t)m * (size_t)n * sizeof(float) : 0;
}

void launch_q8_product(const Q8ProductArgs &a, bool bf16, hipStream_t st)
{
    const Choice c = choose(a.m, a.n, a.k, bf16);
    // What the dies' caches do not hold goes past them, so that operands stay there: 8192 x 8192 x 2048 bf16 122 / 134 us; but not rows that end within 64 bytes, of which
    // halves would be written twice, and not what is read first (beta).
    const int64_t size = bf16 ? 2 : 4, ends = (a.c.pitch * size) | (int64_t)reinterpret_cast<uintptr_t>(a.c.data);
    const bool past = a.m * a.n * size > (int64_t)32 << 20 && ends % 64 == 0;
    by_bool(a.a_e5m2 != 0, [&](auto e5m2) {
        by_bool(bf16, [&](auto b) {
            // C in fp32 is summed in fp32 throughout; what the instructions of 8 bits cut off is an eighth of C's rounding to bf16 and less.
            constexpr bool B = decltype(b)::value, E = decltype(e5m2)::value;
            constexpr int K = B ? (E ? Kind::E5M2 : Kind::E4M3) : (E ? Kind::WIDE_E5M2 : Kind::WIDE_E4M3);
            if (c.parts > 1) {
                Q8ProductArgs p = a;
                p.alpha = 1.0f;                 // (alpha and beta are for the launch that adds the parts)
                launch_tiles<K, false, false, false, 2, 2, 2, 2, 4, 2>(p, c, st);
            }
            by_bool(a.beta != 0.0f, [&](auto add) {
                constexpr bool ADD = decltype(add)::value;
                if (c.tiles == kRows) {
                    launch_rows<E, B, ADD>(a, st);
                } else if (c.parts > 1) {
                    const uint32_t octets = (uint32_t)((a.n + 7) / 8);
                    hipLaunchKernelGGL((k_q8_join<B, ADD>), dim3((unsigned)(((uint64_t)a.m * octets + 255) / 256)), dim3(256), 0, st, a, c.parts, octets);
                } else if (c.tiles == kTiny) {
                    launch_tiles<K, B, ADD, false, 2, 2, 2, 2, 4, 2>(a, c, st);
                } else {
                    by_bool(past, [&](auto p) {
                        constexpr bool PAST = decltype(p)::value && !ADD;
                        if (c.tiles == kSmall) launch_tiles<K, B, ADD, PAST, 2, 2, 4, 4, 2, 2>(a, c, st);
                        else if (c.tiles == kWide) launch_tiles<K, B, ADD, PAST && !B, 4, 2, 4, 4, 3, 2>(a, c, st);          // (fewer than 192 large tiles are no 32 MB in bf16)
                        else launch_tiles<K, B, ADD, PAST, 2, 4, 8, 4, 2, 2>(a, c, st);
                    });
                }
            });
        });
    });
}

}  // namespace conef
