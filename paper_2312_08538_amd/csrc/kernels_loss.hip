// Softmax cross entropy of a vocabulary's logits l = x w^T and its gradient, without the logits ever being in memory.
//
// Forward: the product's tiles end in each row's largest logit and the sum of exponentials over it, 8 bytes a row and tile; k_loss_join adds these up.
// Backward, a piece of the vocabulary at a time: the tiles of the product end in d = dloss / s (exp(l - lse) - [v = target]), rounded to the
// operands' type and packed twice, by rows for dx = s d w and by columns for dw = s d^T x.  s is the largest magnitude of dloss: then, where all tokens weigh the same, a
// target's element is next to -1 and rounding does not move it; dloss itself, 1 / 3686 say, is off by 0.3 % in bf16, and so would all targets' shares be.  Both products then read operands whose steps lie as the matrix
// instructions take them; w and x are turned for that (k_loss_turn), which is a pass over memory where a product is width (tokens) times as much work.
// A sum over the vocabulary goes from piece to piece in fp32.
//
// What bounds it: four products, the logits twice.  4096 x 50304 x 2048 bf16, 844 GFLOP each: forward 0.67 to 0.69 ms (1.2 PFLOP/s; storing the logits would add 412 MB twice), backward 2.35 to 2.4 ms, a piece of 8192
// columns 131 us of gradient, 109 of dx and 105 of dw (1.05, 1.26 and 1.31 PFLOP/s; a library's product of these sizes 1.1 to 1.25 here), 12 of turning w; the matrix units are busy in 51 to 63 % of the cycles, waves wait in 30 to 34 % of
// theirs.  1001 x 5003 x 515 fp32, 5.2 GFLOP each: 52, 57, 56, 57 us, where the instructions alone take 33 to 37.
#include <algorithm>

#include "product_device.h"
#include "turned_device.h"

namespace conef {

namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLeast = -3.402823466e38f;              // below every logit but -inf

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// fp32: with what rounding v log2(e) leaves out, |v| 2^-24 of the result otherwise
template <int KIND>
__device__ __forceinline__ float exp_of(float v)
{
    if constexpr (KIND == Kind::F32) {
        constexpr float kRest = 1.92596298e-8f, kLn2 = 0.693147181f;             // log2(e) = kLog2e + kRest
        const float t = v * kLog2e, r = __builtin_fmaf(v, kRest, __builtin_fmaf(v, kLog2e, -t)), e = __builtin_amdgcn_exp2f(t);
        return e > 0.0f && e < __builtin_inff() ? __builtin_fmaf(e * kLn2, r, e) : e;
    } else {
        return exp_of(v);
    }
}

template <int KIND>
constexpr bool is_bf16() { return KIND == Kind::BF16; }

// ---------------------------------------------------------------- operands
// Rows of any alignment as a packed operand: an octet a lane, sixteen rows of four octets a wave.
template <bool BF16>
__global__ __launch_bounds__(256) void k_loss_pack(Rows x, int64_t rows, int64_t cols, int64_t padded_rows, int steps, uint8_t *out)
{
    constexpr int kStep = BF16 ? 64 : 32;               // elements
    const int64_t fours = ((int64_t)steps * kStep + 31) / 32, id = (int64_t)group_index() * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int64_t row = id / fours * 16 + (lane & 15), col = id % fours * 32 + 8 * (lane >> 4);
    if (row >= padded_rows) return;
    const Octet<BF16> o = fetch_octet<BF16>(x.data, row * x.pitch + col, row < rows ? octet_left(cols - col) : 0);
    uint8_t *to = out + ((row >> 4) * steps + col / kStep) * 2048 + col % kStep / (BF16 ? 8 : 4) * 256 + (row & 15) * 16;
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) *reinterpret_cast<uint4 *>(to + h * 256) = make_uint4(o.w[h][0], o.w[h][1], o.w[h][2], o.w[h][3]);
}

// The transpose as a packed operand: its rows are x's columns, its long axis x's rows.  128 rows of 64 columns a workgroup, turned in LDS.
// `targets` (or null): rows without one of 0 .. vocab - 1 are zeros, since what the product multiplies them by is 0, and 0 times NaN or infinity is not.
// Bound by memory: 8192 x 2048 bf16, 67 MB, 10.9 us (6.2 TB/s).
template <bool BF16>
__global__ __launch_bounds__(256) void k_loss_turn(Rows x, int64_t rows, int64_t cols, int64_t padded_cols, int steps, uint8_t *out, const int64_t *targets,
                                                   int64_t vocab)
{
    constexpr int kStep = BF16 ? 64 : 32;
    __shared__ __attribute__((aligned(16))) Turned<BF16> tile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t strips = padded_cols / 64, group = group_index(), row0 = group / strips * 128, col0 = group % strips * 64, depth = (int64_t)steps * kStep;
    if (row0 >= depth) return;
    bool there[4];                                      // (beforehand: a target between two octets' loads would keep them apart)
#pragma unroll
    for (int i = 0; i < 4; ++i) there[i] = row0 + i * 32 + (threadIdx.x >> 3) < rows;
    if (targets) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t of = targets[min(row0 + i * 32 + (threadIdx.x >> 3), rows - 1)];
            there[i] = there[i] && of >= 0 && of < vocab;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
        const int64_t row = row0 + r;
        tile.put(r, c, fetch_octet<BF16>(x.data, row * x.pitch + col0 + c, there[i] ? octet_left(cols - col0 - c) : 0));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = (i * 4 + (lane >> 4)) * 8;
        const int64_t row = row0 + r, col = col0 + 16 * wave;
        const Octet<BF16> o = tile.get(r, 16 * wave, lane);
        if (row >= depth) continue;
        uint8_t *to = out + ((col >> 4) * steps + row / kStep) * 2048 + row % kStep / (BF16 ? 8 : 4) * 256 + (lane & 15) * 16;
#pragma unroll
        for (int h = 0; h < (BF16 ? 1 : 2); ++h) *reinterpret_cast<uint4 *>(to + h * 256) = make_uint4(o.w[h][0], o.w[h][1], o.w[h][2], o.w[h][3]);
    }
}

// ---------------------------------------------------------------- forward
struct StatArgs {
    int64_t tokens = 0, vocab = 0;          // vocab: of the piece, which begins at `first`
    int64_t first = 0;
    const int64_t *targets = nullptr;
    float2 *stats = nullptr;                // a tile's largest logit of a row, and the sum of exp(l - that)
    float *hit = nullptr;                   // the target's logit
};

template <int KIND, bool BY_ROWS, int WM, int WN, int TM, int TN, int STAGES, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void k_loss_logits(StatArgs p, Side a, Side b, Shape z)
{
    typedef Tile<KIND, BY_ROWS, WM, WN, TM, TN, STAGES> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kBytes + T::kM * 4];
    if (group_index() >= (uint32_t)z.items) return;
    const Place at = place_of(z, (int)group_index());
    int *targets = reinterpret_cast<int *>(lds + T::kBytes);         // in the piece, or -1; asked for before the product, read behind it
    for (int r = threadIdx.x; r < T::kM; r += T::kThreads) {
        const int64_t row = (int64_t)at.m * T::kM + r, of = row < p.tokens ? p.targets[row] : -1;
        targets[r] = of >= p.first && of < p.first + p.vocab ? (int)(of - p.first) : -1;
    }
    typename T::Sums acc;
    T::run(a, b, z, at.m * T::kM, at.n * T::kN, 0, z.steps, lds, acc);
    const int lane = threadIdx.x & 63, col0 = at.n * T::kN + T::wave_n() * TN * 16 + 4 * (lane >> 4);
    float2 *red = reinterpret_cast<float2 *>(lds);          // [WN][kM]
    wait_loads<0>();
    __syncthreads();
    const bool whole = (int64_t)(at.n + 1) * T::kN <= p.vocab;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = (T::wave_m() * TM + i) * 16 + (lane & 15);
        const int64_t row = (int64_t)at.m * T::kM + r;
        if (!whole) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col0 + j * 16 + e >= p.vocab) acc[j][i][e] = -__builtin_inff();
        }
        const int target = targets[r] - col0;              // (none: below 0)
        float most = kLeast;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                most = fmaxf(most, acc[j][i][e]);
                if (target == j * 16 + e) p.hit[row] = acc[j][i][e];
            }
        // (the four lanes that share a row are sixteen apart)
        auto across = [](float v, auto f) {
            auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
            r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
        };
        // (an infinite logit less the largest finite one is infinity, less itself it would be NaN)
        most = fminf(across(most, [](float x, float y) { return fmaxf(x, y); }), -kLeast);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += exp_of<KIND>(acc[j][i][e] - most);
        sum = across(sum, [](float x, float y) { return x + y; });
        if (lane < 16) red[T::wave_n() * T::kM + r] = make_float2(most, sum);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < T::kM; r += T::kThreads) {
        const int64_t row = (int64_t)at.m * T::kM + r;
        if (row >= p.tokens) continue;
        float most = kLeast, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WN; ++w) most = fmaxf(most, red[w * T::kM + r].x);
#pragma unroll
        for (int w = 0; w < WN; ++w) sum += red[w * T::kM + r].y * exp_of(red[w * T::kM + r].x - most);
        p.stats[at.n * p.tokens + row] = make_float2(most, sum);
    }
}

// lse and loss of sixteen rows a workgroup: 64 threads to a row, a share of its tiles each.  4 to 5 us from 16 x 50257 to 4096 x 50304 under a profiler, most of it the launch.
__global__ __launch_bounds__(1024) void k_loss_join(const float2 *stats, const float *hit, const int64_t *targets, int64_t tokens, int64_t vocab, int tiles,
                                                    float *loss, float *lse)
{
    __shared__ float2 red[64][16];
    const int r = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t row = (int64_t)group_index() * 16 + r;
    float most = kLeast, sum = 0.0f;
    if (row < tokens)
        for (int t = part; t < tiles; t += 64 * 8) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = t + 64 * u < tiles ? stats[(int64_t)(t + 64 * u) * tokens + row] : make_float2(kLeast, 0.0f);
            float high = most;
#pragma unroll
            for (int u = 0; u < 8; ++u) high = fmaxf(high, v[u].x);
            sum *= exp_of(most - high);
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u].y * exp_of(v[u].x - high);
            most = high;
        }
    red[part][r] = make_float2(most, sum);
    for (int step = 32; step; step /= 2) {
        __syncthreads();
        if (part >= step) continue;
        const float2 u = red[part][r], v = red[part + step][r];
        const float high = fmaxf(u.x, v.x);
        red[part][r] = make_float2(high, u.y * exp_of(u.x - high) + v.y * exp_of(v.x - high));
    }
    if (part || row >= tokens) return;
    const double total = (double)red[0][r].x + log((double)red[0][r].y);
    if (lse) lse[row] = (float)total;
    if (loss) {
        const int64_t t = targets[row];
        loss[row] = t >= 0 && t < vocab ? (float)(total - (double)hit[row]) : 0.0f;
    }
}

// ---------------------------------------------------------------- backward
// The largest finite magnitude of dloss among tokens that have a target, or 1 if that is 0.
__global__ __launch_bounds__(1024) void k_loss_scale(const float *dloss, const int64_t *targets, int64_t tokens, int64_t vocab, float *scale)
{
    __shared__ float red[16];
    float most = 0.0f;
    for (int64_t i = threadIdx.x; i < tokens; i += 8 * 1024) {
        float v[8];
        int64_t of[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t t = min(i + 1024 * u, tokens - 1);
            v[u] = fabsf(dloss[t]);
            of[u] = targets[t];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) most = v[u] < __builtin_inff() && of[u] >= 0 && of[u] < vocab ? fmaxf(most, v[u]) : most;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 16; ++w) most = fmaxf(most, red[w]);
    *scale = most > 0.0f ? most : 1.0f;
}

struct GradArgs {
    int64_t tokens = 0, vocab = 0, first = 0, all = 0;          // vocab: of the piece, which begins at `first` of `all`
    const int64_t *targets = nullptr;
    const float *lse = nullptr, *dloss = nullptr, *scale = nullptr;         // dloss null: 1 each, and so is the scale
    uint8_t *by_rows = nullptr, *by_cols = nullptr;             // either may be null
    int64_t padded_tokens = 0, padded_vocab = 0;                // to 64
};

// Eight neighbours along a packed operand's long axis, `at` its row and `along` the first of them
template <bool BF16>
__device__ __forceinline__ void put_packed(uint8_t *out, int64_t at, int64_t along, int64_t depth, const float v[8])
{
    constexpr int kStep = BF16 ? 64 : 32;
    uint8_t *to = out + ((at >> 4) * (depth / kStep) + along / kStep) * 2048 + along % kStep / (BF16 ? 8 : 4) * 256 + (at & 15) * 16;
    if constexpr (BF16) {
        *reinterpret_cast<uint4 *>(to) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
        *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(to + 256) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

template <int KIND, bool BY_ROWS, int WM, int WN, int TM, int TN, int STAGES, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void k_loss_gradient(GradArgs p, Side a, Side b, Shape z)
{
    typedef Tile<KIND, BY_ROWS, WM, WN, TM, TN, STAGES> T;
    constexpr bool BF16 = is_bf16<KIND>();
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kBytes + T::kM * sizeof(float4)];
    if (group_index() >= (uint32_t)z.items) return;
    const Place at = place_of(z, (int)group_index());
    // Of each row its share of the gradient (0: no target), lse, and the target's place in the piece: asked for before the product, read behind it.
    float4 *about = reinterpret_cast<float4 *>(lds + T::kBytes);
    for (int r = threadIdx.x; r < T::kM; r += T::kThreads) {
        const int64_t row = (int64_t)at.m * T::kM + r, of = row < p.tokens ? p.targets[row] : -1;
        const bool there = of >= 0 && of < p.all, here = of >= p.first && of < p.first + p.vocab;
        about[r] = make_float4(there ? (p.dloss ? p.dloss[row] / *p.scale : 1.0f) : 0.0f, there ? p.lse[row] : 0.0f, __int_as_float(here ? (int)(of - p.first) : -1),
                               __int_as_float(there));
    }
    typename T::Sums acc;
    T::run(a, b, z, at.m * T::kM, at.n * T::kN, 0, z.steps, lds, acc);
    const int lane = threadIdx.x & 63;
    float *mine = reinterpret_cast<float *>(lds) + T::wave() * 32 * T::kPitch;
    wait_loads<0>();
    __syncthreads();
    const int64_t col0 = (int64_t)at.n * T::kN + T::wave_n() * TN * 16;
#pragma unroll
    for (int i = 0; i < TM; i += 2) {
        const int64_t row0 = (int64_t)at.m * T::kM + (T::wave_m() * TM + i) * 16;
        T::turn(acc, i, mine);
        constexpr int kAcross = TN * 2, kHigh = 64 / kAcross;
#pragma unroll
        for (int t = 0; t < 32 / kHigh; ++t) {
            const int r = t * kHigh + lane / kAcross, c = lane % kAcross * 8;
            const int64_t row = row0 + r, col = col0 + c;
            float *from = mine + r * T::kPitch + c;
            const float4 of = about[(T::wave_m() * TM + i) * 16 + r];
            const int target = __float_as_int(of.z) - (int)col;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = exp_of<KIND>(from[e] - of.y) - (target == e ? 1.0f : 0.0f);
                v[e] = __float_as_int(of.w) && col + e < p.vocab ? of.x * d : 0.0f;         // (no target: whatever the logits are)
            }
            *reinterpret_cast<f32x4 *>(from) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4 *>(from + 4) = f32x4{v[4], v[5], v[6], v[7]};
            if (p.by_rows && row < p.padded_tokens && col < p.padded_vocab) put_packed<BF16>(p.by_rows, row, col, p.padded_vocab, v);
        }
        __builtin_amdgcn_wave_barrier();
        if (p.by_cols) {
            constexpr int kWide = TN * 16, kTall = 64 / kWide;             // columns that a wave takes at a time, and octets of rows
#pragma unroll
            for (int t = 0; t < 4 / kTall; ++t) {
                const int c = lane % kWide, r = (t * kTall + lane / kWide) * 8;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mine[(r + e) * T::kPitch + c];
                if (row0 + r < p.padded_tokens && col0 + c < p.padded_vocab) put_packed<BF16>(p.by_cols, col0 + c, row0 + r, p.padded_tokens, v);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// out <- alpha (scale sum + base) + beta out
struct SumArgs {
    int64_t m = 0, n = 0;
    float alpha = 1.0f, beta = 0.0f;
    const float *scale = nullptr;           // null: 1
    const float *base = nullptr;            // m x n, dense: what earlier pieces came to
    RowsOut out;
    float *partials = nullptr;              // of the long axis in parts: m x n each
};

template <bool BF16>
__device__ __forceinline__ void put_sum(const SumArgs &p, int64_t row, int64_t col, int left, float v[8])
{
    if (p.scale) {
        const float s = *p.scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = s * v[i];
    }
    if (p.base) {
        float b[8];
        load_octet<false>(p.base, row * p.n + col, left, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = b[i] + v[i];
    }
    if (p.beta != 0.0f) put_octet<BF16, true, false>(p.out, row, col, left, p.alpha, p.beta, v);
    else put_octet<BF16, false, false>(p.out, row, col, left, p.alpha, 0.0f, v);
}

template <int KIND, bool BF16, int WM, int WN, int TM, int TN, int STAGES, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void k_loss_product(SumArgs p, Side a, Side b, Shape z)
{
    typedef Tile<KIND, false, WM, WN, TM, TN, STAGES> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kBytes];
    if (group_index() >= (uint32_t)z.items) return;
    const Place at = place_of(z, (int)group_index());
    const int first = at.part * z.per_part;
    typename T::Sums acc;
    T::run(a, b, z, at.m * T::kM, at.n * T::kN, first, min(z.per_part, z.steps - first), lds, acc);
    T::octets(acc, lds, [&](int r, int c, float v[8]) {
        const int64_t row = (int64_t)at.m * T::kM + r, col = (int64_t)at.n * T::kN + c;
        if (row >= p.m || col >= p.n) return;
        if (p.partials) store_octet<false>(p.partials + (int64_t)at.part * p.m * p.n, row * p.n + col, octet_left(p.n - col), v);
        else put_sum<BF16>(p, row, col, octet_left(p.n - col), v);
    });
}

// Adds the parts of the long axis in their order, eight columns a thread.
template <bool BF16>
__global__ __launch_bounds__(256) void k_loss_parts(SumArgs p, int parts, uint32_t octets_a_row)
{
    const uint64_t t = (uint64_t)group_index() * 256 + threadIdx.x;
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
    put_sum<BF16>(p, row, col, left, v);
}

// ---------------------------------------------------------------- plans
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Columns of the vocabulary that are worked on at a time: d of some 2^25 elements, which with its two forms the card's last cache holds, but 4096 columns at least
// (a product's long axis, and the bytes of dx that go from piece to piece).  4096 x 50304 x 2048, both passes: 2^24 elements 3210 us, 2^25 3100, 2^26 3135, 2^27 3080 in four times the
// workspace.  Of w, which is turned (and packed, if it has to be) a piece at a time, some 2^28 elements, so that few tokens of a wide w do not need all of it once more: 16 x 256000 x 8192
// bf16 backward 5.2 ms in 0.55 GB / 4.6 in 4.3 as one piece / 5.4 in 2^27 elements / 5.7 in 2^26; 64 x 100000 x 4096 1055 us / 1020 as one.
int64_t piece_of(int64_t tokens, int64_t vocab, int64_t width)
{
    const int64_t most = std::min(((int64_t)1 << 25) / std::max<int64_t>(tokens, 1), ((int64_t)1 << 28) / width);
    const int64_t v = std::max<int64_t>(most / 256 * 256, 4096);
    return vocab <= v + v / 4 ? vocab : v;
}

constexpr std::integral_constant<int, 1> one;
constexpr std::integral_constant<int, 2> two;
constexpr std::integral_constant<int, 3> three;
constexpr std::integral_constant<int, 4> four;
constexpr std::integral_constant<int, 8> eight;

enum Tiles { kTiny, kSmall, kWide, kLarge };

Tiles tiles_for(int64_t m, int64_t n, bool bf16)
{
    auto tiles = [&](int64_t tm, int64_t tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); };
    // fp32: the matrix instructions take sixteen times as long as those of 16 bits, so that the smallest tiles' reads hide behind them, too, and many tiles make even turns:
    // us of 1024 x 5056 x 512 alone 48 (three steps in LDS, three workgroups a CU; two and four 55), of 128 x 128 69; 4096 x 4096 x 2048, 1024 of these, 511 and 466 (147 TFLOP/s;
    // the instructions alone 141 to 157, by the clock)
    if (!bf16) return tiles(128, 128) >= 4 * kCus ? kSmall : kTiny;
    // bf16, us of the forward pass, the one taken / others: large 4096 x 4096 x 2048 61.6 / 67.4 wide, 71.9 small; 4096 x 8192 x 2048 115 / 129, 134; wide 1024 x 8192 x 768 20.1 / 20.5 small,
    // 26.7 large; small 512 x 8192 x 2048 33.4 / 33.7 tiny, 32.3 wide; tiny 256 x 8192 x 2048 23.2 / 32.9 small.
    if (std::min(m, n) > 128 && tiles(256, 256) >= 192) return kLarge;
    if (std::min(m, n) > 128 && tiles(256, 128) >= 192) return kWide;
    if (m > 64 && tiles(128, 128) >= 200) return kSmall;
    return kTiny;
}

// waves, tiles of a wave, steps in LDS, waves a SIMD
template <bool BF16, typename F>
void by_tiles(Tiles t, F &&go)
{
    if (t == kSmall) {
        go(two, two, four, four, two, two);
    } else if constexpr (!BF16) {
        go(two, two, two, two, three, three);
    } else {
        if (t == kTiny) go(two, two, two, two, four, two);
        else if (t == kWide) go(four, two, four, four, three, two);
        else go(two, four, eight, four, two, two);
    }
}

struct Cut {
    Tiles tiles;
    int parts, per_part;
};

// of a product of `steps` along its long axis
Cut cut_of(int64_t m, int64_t n, int64_t steps, bool bf16)
{
    const Tiles t = tiles_for(m, n, bf16);
    if (t != kTiny) return {t, 1, (int)steps};
    const int64_t tiles = std::max<int64_t>(((m + 63) / 64) * ((n + 63) / 64), 1);
    const int64_t parts = std::max<int64_t>(std::min<int64_t>((bf16 ? 2 : 3) * kCus / tiles, steps / 8), 1), per = std::max<int64_t>((steps + parts - 1) / parts, 1);
    return {t, (int)std::max<int64_t>((steps + per - 1) / per, 1), (int)per};
}

// The workspace: both passes' packed x and a piece's packed w (where these do not lie as the kernels take them); forward: a row's statistics by tiles; backward: d by rows and by
// columns, a piece of w turned (a large one in the place of the packed one, which only the launch before it reads), x turned, dx as it grows, parts of a long axis.
struct Layout {
    int64_t piece, esz, depth_w;                            // depth_w: bytes of a row of x or w, up to 128
    size_t x, w, stats, hit, scale, rows, cols, w_t, x_t, grown, parts, end;
};

Layout layout_of(int64_t tokens, int64_t vocab, int64_t width, bool bf16)
{
    Layout l;
    l.esz = bf16 ? 2 : 4;
    l.piece = piece_of(tokens, vocab, width);
    l.depth_w = up(width * l.esz, 128);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const int64_t t64 = up(tokens, 64), v64 = up(l.piece, 64), d64 = up(width, 64);
    l.x = take((size_t)t64 * l.depth_w);
    // One place for both forms of a piece of w, but for pieces that the dies' caches hold: writing over what was read there last costs 1001 x 5003 x 515 fp32 244.2 us / 242.4 in two;
    // one place of 94 MB, 3 x 24640 x 1796 bf16 174 / 197.
    const size_t packed = (size_t)v64 * l.depth_w, turned = (size_t)v64 * d64 * l.esz;
    const bool in_one = std::max(packed, turned) > (size_t)32 << 20;
    l.w = take(in_one ? std::max(packed, turned) : packed);
    l.w_t = in_one ? l.w : take(turned);
    const size_t shared = at;
    l.stats = take((size_t)tokens * ((vocab + 63) / 64 + vocab / l.piece + 1) * sizeof(float2));
    l.hit = take((size_t)tokens * sizeof(float));
    const size_t forward = at;
    at = shared;
    l.scale = take(sizeof(float));
    l.rows = take((size_t)t64 * v64 * l.esz);
    l.cols = take((size_t)t64 * v64 * l.esz);
    l.x_t = take((size_t)d64 * t64 * l.esz);
    l.grown = take(l.piece < vocab ? (size_t)tokens * width * sizeof(float) : 0);
    size_t most = 0;
    for (const int64_t n : {std::min(l.piece, vocab), vocab % l.piece}) {
        const Cut x = cut_of(tokens, width, up(n, 64) * l.esz / 128, bf16), w = cut_of(n, width, t64 * l.esz / 128, bf16);
        most = std::max(most, x.parts > 1 ? (size_t)x.parts * tokens * width : 0);
        most = std::max(most, w.parts > 1 ? (size_t)w.parts * n * width : 0);
    }
    l.parts = take(most * sizeof(float));
    l.end = std::max(at, forward);
    return l;
}

// x and w lie as the kernels take them
bool in_place(const LossArgs &a, int64_t esz)
{
    auto fits = [&](const Rows &r) {
        return reinterpret_cast<uintptr_t>(r.data) % 16 == 0 && r.pitch * esz % 16 == 0 && r.pitch * esz < (int64_t)1 << 29;
    };
    return a.width * esz % 16 == 0 && fits(a.x) && fits(a.w);
}

Rows rows_from(const Rows &r, int64_t first, int64_t esz) { return {static_cast<const uint8_t *>(r.data) + first * r.pitch * esz, r.pitch}; }

template <bool BF16>
void pack(const Rows &x, int64_t rows, int64_t cols, int64_t depth, uint8_t *out, hipStream_t st)
{
    const int64_t padded = up(rows, 64), steps = depth / 128, fours = (steps * (BF16 ? 64 : 32) + 31) / 32;
    hipLaunchKernelGGL((k_loss_pack<BF16>), grid_of((padded / 16 * fours + 3) / 4), dim3(256), 0, st, x, rows, cols, padded, (int)steps, out);
}

template <bool BF16>
void turn(const Rows &x, int64_t rows, int64_t cols, uint8_t *out, hipStream_t st, const int64_t *targets = nullptr, int64_t vocab = 0)
{
    constexpr int kStep = BF16 ? 64 : 32;
    const int64_t padded = up(cols, 64), depth = up(rows, 64);
    hipLaunchKernelGGL((k_loss_turn<BF16>), grid_of((depth + 127) / 128 * (padded / 64)), dim3(256), 0, st, x, rows, cols, padded, (int)(depth / kStep), out,
                       targets, vocab);
}

Side packed_side(const uint8_t *data, int64_t rows)
{
    Side s;
    s.data = data;
    s.rows = (int)up(rows, 64);
    return s;
}

template <int KIND, typename F>
void with_operands(const LossArgs &a, const Layout &l, bool direct, int64_t first, int64_t n, hipStream_t st, F &&go)
{
    constexpr bool BF16 = is_bf16<KIND>();
    const Rows w = rows_from(a.w, first, l.esz);
    Side x_side, w_side;
    if (direct) {
        x_side.data = static_cast<const uint8_t *>(a.x.data), x_side.pitch = a.x.pitch * l.esz, x_side.rows = (int)a.tokens;
        w_side.data = static_cast<const uint8_t *>(w.data), w_side.pitch = a.w.pitch * l.esz, w_side.rows = (int)n;
        go(std::true_type{}, x_side, w_side);
    } else {
        pack<BF16>(w, n, a.width, l.depth_w, a.workspace + l.w, st);
        go(std::false_type{}, packed_side(a.workspace + l.x, a.tokens), packed_side(a.workspace + l.w, n));
    }
}

template <int KIND>
void forward(const LossArgs &a, hipStream_t st)
{
    constexpr bool BF16 = is_bf16<KIND>();
    const Layout l = layout_of(a.tokens, a.vocab, a.width, BF16);
    const bool direct = in_place(a, l.esz);
    if (!direct) pack<BF16>(a.x, a.tokens, a.width, l.depth_w, a.workspace + l.x, st);
    float2 *stats = reinterpret_cast<float2 *>(a.workspace + l.stats);
    int tiles = 0;
    const int64_t piece = direct ? a.vocab : l.piece;
    for (int64_t first = 0; first < a.vocab; first += piece) {
        const int64_t n = std::min(piece, a.vocab - first);
        with_operands<KIND>(a, l, direct, first, n, st, [&](auto by_rows, const Side &x, const Side &w) {
            auto go = [&](auto wm, auto wn, auto tm, auto tn, auto stages, auto occ) {
                constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value;
                Shape z;
                z.steps = z.per_part = (int)(l.depth_w / 128);
                z.last = (int)((a.width * l.esz - 1) % 128 + 1);
                z.tiles_m = (int)((a.tokens + WM * TM * 16 - 1) / (WM * TM * 16));
                z.tiles_n = (int)((n + WN * TN * 16 - 1) / (WN * TN * 16));
                z.items = z.tiles_m * z.tiles_n;
                StatArgs p;
                p.tokens = a.tokens, p.vocab = n, p.first = first, p.targets = a.targets;
                p.stats = stats + (int64_t)tiles * a.tokens;
                p.hit = reinterpret_cast<float *>(a.workspace + l.hit);
                hipLaunchKernelGGL((k_loss_logits<KIND, decltype(by_rows)::value, WM, WN, TM, TN, decltype(stages)::value, decltype(occ)::value>),
                                   grid_of(z.items), dim3(64 * WM * WN), 0, st, p, x, w, z);
                tiles += z.tiles_n;
            };
            const Tiles t = tiles_for(a.tokens, n, BF16);
            if (a.tokens <= 32) go(one, two, two, two, four, two);
            else by_tiles<BF16>(t, go);
        });
    }
    hipLaunchKernelGGL(k_loss_join, grid_of((a.tokens + 15) / 16), dim3(1024), 0, st, stats, reinterpret_cast<float *>(a.workspace + l.hit), a.targets,
                       a.tokens, a.vocab, tiles, a.loss, a.lse_out);
}

// out <- alpha (A B^T + base) + beta out of packed operands of `depth` elements
template <int KIND, bool OUT>
void product(SumArgs p, const uint8_t *a, const uint8_t *b, int64_t depth, float *partials, hipStream_t st)
{
    constexpr int kStep = is_bf16<KIND>() ? 64 : 32;
    const Cut c = cut_of(p.m, p.n, depth / kStep, is_bf16<KIND>());
    p.partials = c.parts > 1 ? partials : nullptr;
    auto go = [&](auto wm, auto wn, auto tm, auto tn, auto stages, auto occ) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value;
        Shape z;
        z.steps = (int)(depth / kStep);
        z.per_part = c.per_part;
        z.tiles_m = (int)((p.m + WM * TM * 16 - 1) / (WM * TM * 16));
        z.tiles_n = (int)((p.n + WN * TN * 16 - 1) / (WN * TN * 16));
        z.items = z.tiles_m * z.tiles_n * c.parts;
        hipLaunchKernelGGL((k_loss_product<KIND, OUT, WM, WN, TM, TN, decltype(stages)::value, decltype(occ)::value>), grid_of(z.items), dim3(64 * WM * WN), 0, st, p, packed_side(a, p.m), packed_side(b, p.n), z);
    };
    by_tiles<is_bf16<KIND>()>(c.tiles, go);
    if (c.parts > 1) {
        const uint32_t octets = (uint32_t)((p.n + 7) / 8);
        hipLaunchKernelGGL((k_loss_parts<OUT>), grid_of((p.m * octets + 255) / 256), dim3(256), 0, st, p, c.parts, octets);
    }
}

template <int KIND>
void backward(const LossArgs &a, hipStream_t st)
{
    constexpr bool BF16 = is_bf16<KIND>();
    const Layout l = layout_of(a.tokens, a.vocab, a.width, BF16);
    if (a.tokens == 0) {                        // a sum of nothing
        SumArgs p;
        p.m = a.vocab, p.n = a.width, p.alpha = 0.0f, p.beta = a.beta, p.out = a.dw;
        const uint32_t octets = (uint32_t)((p.n + 7) / 8);
        if (a.dw.data) hipLaunchKernelGGL((k_loss_parts<BF16>), grid_of((p.m * octets + 255) / 256), dim3(256), 0, st, p, 0, octets);
        return;
    }
    const bool direct = in_place(a, l.esz);
    if (!direct) pack<BF16>(a.x, a.tokens, a.width, l.depth_w, a.workspace + l.x, st);
    float *scale = a.dloss ? reinterpret_cast<float *>(a.workspace + l.scale) : nullptr;
    if (scale) hipLaunchKernelGGL(k_loss_scale, dim3(1), dim3(1024), 0, st, a.dloss, a.targets, a.tokens, a.vocab, scale);
    if (a.dw.data) turn<BF16>(a.x, a.tokens, a.width, a.workspace + l.x_t, st, a.targets, a.vocab);
    float *partials = reinterpret_cast<float *>(a.workspace + l.parts), *grown = reinterpret_cast<float *>(a.workspace + l.grown);
    for (int64_t first = 0; first < a.vocab; first += l.piece) {
        const int64_t n = std::min(l.piece, a.vocab - first);
        with_operands<KIND>(a, l, direct, first, n, st, [&](auto by_rows, const Side &x, const Side &w) {
            auto go = [&](auto wm, auto wn, auto tm, auto tn, auto stages, auto occ) {
                constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value;
                static_assert(WM * TM * 16 % 64 == 0 && WN * TN * 16 % 64 == 0, "the packed forms are whole to 64 both ways");
                Shape z;
                z.steps = z.per_part = (int)(l.depth_w / 128);
                z.last = (int)((a.width * l.esz - 1) % 128 + 1);
                z.tiles_m = (int)((a.tokens + WM * TM * 16 - 1) / (WM * TM * 16));
                z.tiles_n = (int)((n + WN * TN * 16 - 1) / (WN * TN * 16));
                z.items = z.tiles_m * z.tiles_n;
                GradArgs p;
                p.tokens = a.tokens, p.vocab = n, p.first = first, p.all = a.vocab;
                p.targets = a.targets, p.lse = a.lse, p.dloss = a.dloss, p.scale = scale;
                p.by_rows = a.dx.data ? a.workspace + l.rows : nullptr;
                p.by_cols = a.dw.data ? a.workspace + l.cols : nullptr;
                p.padded_tokens = up(a.tokens, 64), p.padded_vocab = up(n, 64);
                hipLaunchKernelGGL((k_loss_gradient<KIND, decltype(by_rows)::value, WM, WN, TM, TN, decltype(stages)::value, decltype(occ)::value>),
                                   grid_of(z.items), dim3(64 * WM * WN), 0, st, p, x, w, z);
            };
            const Tiles t = tiles_for(a.tokens, n, BF16);
            by_tiles<BF16>(t, go);
        });
        if (a.dx.data) {
            turn<BF16>(rows_from(a.w, first, l.esz), n, a.width, a.workspace + l.w_t, st);
            SumArgs p;
            p.m = a.tokens, p.n = a.width, p.scale = scale;
            p.base = first ? grown : nullptr;
            const bool done = first + n == a.vocab;
            p.out = done ? a.dx : RowsOut{grown, a.width};
            if (done) product<KIND, BF16>(p, a.workspace + l.rows, a.workspace + l.w_t, up(n, 64), partials, st);
            else product<KIND, false>(p, a.workspace + l.rows, a.workspace + l.w_t, up(n, 64), partials, st);
        }
        if (a.dw.data) {
            SumArgs p;
            p.m = n, p.n = a.width, p.scale = scale;
            p.alpha = a.alpha, p.beta = a.beta;
            p.out = {static_cast<uint8_t *>(a.dw.data) + first * a.dw.pitch * l.esz, a.dw.pitch};
            product<KIND, BF16>(p, a.workspace + l.cols, a.workspace + l.x_t, up(a.tokens, 64), partials, st);
        }
    }
}

}  // namespace

size_t loss_workspace(int64_t tokens, int64_t vocab, int64_t width, bool bf16) { return layout_of(tokens, vocab, width, bf16).end; }

void launch_loss_forward(const LossArgs &a, bool bf16, hipStream_t st)
{
    if (bf16) forward<Kind::BF16>(a, st);
    else forward<Kind::F32>(a, st);
}

void launch_loss_backward(const LossArgs &a, bool bf16, hipStream_t st)
{
    if (bf16) backward<Kind::BF16>(a, st);
    else backward<Kind::F32>(a, st);
}

}  // namespace conef
