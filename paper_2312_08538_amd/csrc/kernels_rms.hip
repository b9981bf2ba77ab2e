// Root-mean-square norm with the residual's addition in front of it and its output as a packed operand of 8 bits, and its backward pass.
//
// z = residual + x, rstd = 1 / sqrt(mean(z^2) + eps), y = z rstd gamma.  From the stored z on everything is computed in 64 bits, whose vector
// instructions take twice as long as those of 32 here and hide behind the loads: a value that lies next to a border of the 8-bit grid is rounded to the
// side that it is on, and y, the codes and rstd are each rounded once.  With a = dy gamma and hat = z rstd:
//   dz = rstd (a - hat mean(a hat)) + dz_in,   dgamma = sum over rows of dy hat,
// in fp32 (its results are not rounded to 8 bits), sums over more than 128 rows in fp64, in a fixed order; a long row's mean in fp64.
#include <algorithm>
#include <type_traits>

#include "q8_device.h"

namespace conef {

namespace {

constexpr int kThreads = 256;
constexpr int kMostCols = 8192;                 // the widest rows that a workgroup holds in registers

constexpr int threads_of(int g) { return g > kThreads ? g : kThreads; }

template <int CTRL>
__device__ __forceinline__ double dpp64(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true), hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// sum over each G lanes of a wave, in every one of them, as lanes_sum's
template <int G>
__device__ __forceinline__ double lanes_sum64(double v)
{
    static_assert(G == 16 || G == 32 || G == 64, "");
    v += dpp64<0xB1>(v);
    v += dpp64<0x4E>(v);
    v += dpp64<0x141>(v);
    v += dpp64<0x140>(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    uint32_t lo = (uint32_t)b, hi = (uint32_t)(b >> 32);
    if constexpr (G >= 32) {
        auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
        v = __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
    }
    if constexpr (G == 64) {
        const uint64_t c = __builtin_bit_cast(uint64_t, v);
        lo = (uint32_t)c, hi = (uint32_t)(c >> 32);
        auto l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
        v = __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
    }
    return v;
}

// Sum over the G lanes that share a row, in every one of them.  G > 64 (a workgroup's threads): `red` holds 2 x G / 64 values, used in turn by
// consecutive calls (`turn`), so one barrier a call is enough.
template <int G, typename T>
__device__ __forceinline__ T group_sum(T v, T *red, int &turn)
{
    constexpr int kLanes = G < 64 ? G : 64;
    if constexpr (sizeof(T) == 8) v = lanes_sum64<kLanes>(v);
    else v = lanes_sum<kLanes>(v);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        T *slot = red + turn * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        T s[W];
#pragma unroll
        for (int w = 0; w < W; ++w) s[w] = slot[w];
#pragma unroll
        for (int step = 1; step < W; step *= 2)
#pragma unroll
            for (int w = 0; w + step < W; w += 2 * step) s[w] += s[w + step];
        v = s[0];
    }
    return v;
}

// A row's octets, begun and finished.  Rows of fewer than 8 columns, which have sixteen lanes, are loaded element by element.
template <bool BF16, int G>
__device__ __forceinline__ void begin(Octet<BF16> &o, const void *data, int64_t at, int left, int cols)
{
    if (G == 16 && cols < 8) o = fetch_octet<BF16>(data, at, left);
    else begin_octet<BF16>(o, data, at, left);
}
template <bool BF16, int G>
__device__ __forceinline__ void finish(const Octet<BF16> &o, int left, int cols, float v[8])
{
    if (G == 16 && cols < 8) widen<BF16>(o, v);
    else finish_octet<BF16>(o, left, v);
}

template <int G, int V>
__device__ __forceinline__ void load_columns(const float *p, int cols, int t, float out[V][8])
{
    Octet<false> o[V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) begin<false, G>(o[v], p, 8 * (t + G * v), cols - 8 * (t + G * v), cols);
#pragma unroll
    for (int v = 0; v < V; ++v) finish<false, G>(o[v], cols - 8 * (t + G * v), cols, out[v]);
}

// 1 / sqrt(v), from the instruction's 2^-23 by a step whose error is that to the third power; 0 and infinity as they are
__device__ __forceinline__ double inverse_root(double v)
{
    const double y = __builtin_amdgcn_rsq(v), e = __builtin_fma(-v * y, y, 1.0), z = __builtin_fma(y * e, __builtin_fma(0.375, e, 0.5), y);
    return y > 0.0 && y < __builtin_inf() ? z : y;
}

// A value of 64 bits in 32, rounded to odd (the last bit set if anything is lost): what is rounded from there to fewer bits is as if rounded from the value itself.  That holds for
// magnitudes of 2^-126 and more; below, the cast rounds to nearest, to a multiple of 2^-149, and the second rounding may go the other way for a value within 2^-150 of a tie.
__device__ __forceinline__ float to_odd(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)b, kept = (lo & 0xE0000000u) | (lo & 0x1FFFFFFFu ? 0x20000000u : 0u);
    return (float)__builtin_bit_cast(double, (b >> 32) << 32 | kept);
}

// y of an octet: rounded to odd in `odd`, and, if it is wanted, stored
template <bool BF16>
__device__ __forceinline__ void norm_octet(const RmsArgs &a, const float z[8], const float gamma[8], double rstd, int64_t row, int64_t col, int left, float odd[8])
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double v = (double)z[i] * rstd * (double)gamma[i];
        odd[i] = to_odd(v);
        y[i] = BF16 ? odd[i] : (float)v;
        if (i >= left) odd[i] = 0.0f;           // (0 rstd is no 0 if rstd is infinite)
    }
    if (a.y.data) store_octet<BF16>(a.y.data, row * a.y.pitch + col, left, y);
}

// G lanes hold a row, V octets each: octet v of lane t starts at column 8 (t + G v), so that sixteen lanes hold a block.  The next row's octets are on their way while
// a row is worked on.  H > 0: a packed output.  A workgroup then takes H neighbouring rows, since a line of packed codes holds four of them (a square of 256 bytes
// sixteen): the codes wait in LDS, a square's rows turned by its index, so that the lanes of a wave write to different banks.
// Bound by memory: 16384 x 2048 bf16 with residual and codes, 235 MB, 43 us (5.4 TB/s); 777 x 5003 fp32 13.0 us (a copy's rate: 9.9); 64 x 2048 3.5 us, of
// which a launch is 2.6.
template <bool BF16, int G, int V, bool FUSED, int H>
__global__ __launch_bounds__(threads_of(G)) void k_rms_forward(RmsArgs a, int64_t padded_rows, int64_t pieces)
{
    constexpr int kRows = threads_of(G) / G, kGroup = H ? H : kRows, kPer = kGroup / kRows;
    static_assert(kPer * kRows == kGroup, "");
    __shared__ double red[G > 64 ? 2 * G / 64 : 1];
    __shared__ __attribute__((aligned(16))) uint8_t codes[H ? H * G * V * 8 : 16];
    int turn = 0;
    const int t = threadIdx.x % G, mine = threadIdx.x / G;
    const int64_t rows = H ? padded_rows : a.rows;
    const double inv = 1.0 / (double)a.cols;
    Octet<BF16> x[V] = {}, r[FUSED ? V : 1] = {};
    auto fetch = [&](int64_t from) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v), left = from < a.rows ? a.cols - col : 0;
            begin<BF16, G>(x[v], a.x.data, from * a.x.pitch + col, left, a.cols);
            if constexpr (FUSED) begin<BF16, G>(r[v], a.residual.data, from * a.residual.pitch + col, left, a.cols);
        }
    };
    fetch((int64_t)blockIdx.x * kGroup + mine);
    float gamma[V][8];
    load_columns<G, V>(a.gamma, a.cols, t, gamma);
    for (int64_t group = blockIdx.x; group * kGroup < rows; group += gridDim.x) {
#pragma unroll 1
        for (int i = 0; i < kPer; ++i) {
            if (H && group * kGroup + i * kRows >= a.rows) break;               // (of what fills the operand up there is nothing to compute)
            const int64_t row = group * kGroup + i * kRows + mine;
            const bool there = row < a.rows;
            float z[V][8];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int col = 8 * (t + G * v);
                finish<BF16, G>(x[v], a.cols - col, a.cols, z[v]);
                if constexpr (FUSED) {
                    float add[8];
                    finish<BF16, G>(r[v], a.cols - col, a.cols, add);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[v][e] = add[e] + z[v][e];
                    store_octet<BF16>(a.z.data, row * a.z.pitch + col, there ? a.cols - col : 0, z[v]);
                }
            }
            fetch(i + 1 < kPer ? row + kRows : (group + gridDim.x) * kGroup + mine);
            double sum = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)z[v][e], (double)z[v][e], sum);
            sum = group_sum<G>(sum, red, turn);
            const double rstd = inverse_root(__builtin_fma(sum, inv, (double)a.eps));
            if (there && t == 0 && a.rstd_out) a.rstd_out[row] = (float)rstd;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int octet = t + G * v, col = 8 * octet;
                float y[8];
                norm_octet<BF16>(a, z[v], gamma[v], rstd, row, col, there ? a.cols - col : 0, y);
                if constexpr (H > 0) {
                    const uint32_t byte = q8_scale<false>(neighbours_largest<16>(largest(y)));
                    const int square = octet >> 1, at = i * kRows + mine;
                    *reinterpret_cast<uint2 *>(codes + square * (16 * H) + ((at + square) % H) * 16 + (octet & 1) * 8) = q8_codes<false>(y, byte);
                    if (there && (octet & 15) == 0 && octet < 16 * pieces) a.packed.scales[(octet >> 4) * padded_rows + row] = (uint8_t)byte;
                }
            }
        }
        if constexpr (H > 0) {
            __syncthreads();
            const int64_t row0 = group * kGroup;
            uint8_t *to = a.packed.codes + row0 / 16 * pieces * 2048 + row0 % 16 * 16;
            for (int u = threadIdx.x; u < (int)pieces * 8 * H; u += threads_of(G)) {
                const int square = u / H, at = u % H;
                const bool there = row0 + at < a.rows;
                const uint4 c = *reinterpret_cast<const uint4 *>(codes + square * (16 * H) + ((at + square) % H) * 16);
                *reinterpret_cast<uint4 *>(to + (int64_t)square * 256 + at * 16) = there ? c : make_uint4(0, 0, 0, 0);
                if (!there && (square & 7) == 0) a.packed.scales[(square >> 3) * padded_rows + row0 + at] = 0;
            }
            __syncthreads();
        }
    }
}

// A row of any length, in two sweeps over it by a workgroup.
template <bool BF16, bool FUSED>
__global__ __launch_bounds__(kThreads) void k_rms_forward_long(RmsArgs a, int64_t padded_rows, int64_t pieces)
{
    __shared__ double red[8];
    int turn = 0;
    const bool packed = a.packed.codes != nullptr;
    const double inv = 1.0 / (double)a.cols;
    for (int64_t row = blockIdx.x; row < (packed ? padded_rows : a.rows); row += gridDim.x) {
        const bool there = row < a.rows;
        const void *src = FUSED ? a.z.data : a.x.data;
        const int64_t at = row * (FUSED ? a.z.pitch : a.x.pitch), end = packed ? pieces * 128 : a.cols;
        double sum = 0.0;
        for (int64_t col = 8 * threadIdx.x; there && col < a.cols; col += 8 * kThreads) {
            const int left = octet_left(a.cols - col);
            float z[8];
            load_octet<BF16>(a.x.data, row * a.x.pitch + col, left, z);
            if constexpr (FUSED) {
                float r[8];
                load_octet<BF16>(a.residual.data, row * a.residual.pitch + col, left, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = r[i] + z[i];
                store_octet<BF16>(a.z.data, at + col, left, z);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)z[i], (double)z[i], sum);
        }
        sum = group_sum<kThreads>(sum, red, turn);
        const double rstd = inverse_root(__builtin_fma(sum, inv, (double)a.eps));
        if (there && threadIdx.x == 0 && a.rstd_out) a.rstd_out[row] = (float)rstd;
        // (whole blocks: the sixteen lanes that share one go round together)
        for (int64_t col = 8 * threadIdx.x; col < end; col += 8 * kThreads) {
            const int left = there ? octet_left(a.cols - col) : 0;
            float z[8], gamma[8], y[8];
            load_octet<BF16>(src, at + col, left, z);
            load_octet<false>(a.gamma, col, left, gamma);
            norm_octet<BF16>(a, z, gamma, rstd, row, col, left, y);
            if (packed) {
                const uint32_t byte = q8_scale<false>(neighbours_largest<16>(largest(y)));
                *reinterpret_cast<uint2 *>(a.packed.codes + (row / 16 * pieces + col / 128) * 2048 + (col >> 4 & 7) * 256 + (row & 15) * 16 + (col & 8)) =
                    q8_codes<false>(y, byte);
                if (col % 128 == 0) a.packed.scales[col / 128 * padded_rows + row] = (uint8_t)byte;
            }
        }
    }
}

// Adds dz_in, writes dz.
template <bool BF16>
__device__ __forceinline__ void finish_dz(const RmsArgs &a, int64_t row, int64_t col, int left, const float dz_in[8], float v[8])
{
    if (a.dz_in.data) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += dz_in[i];
    }
    store_octet<BF16>(a.dz.data, row * a.dz.pitch + col, left, v);
}

// Bound by memory: 16384 x 2048 bf16 with dz_in, 268 MB, 47 us with the sums behind it (5.7 TB/s); 777 x 5003 fp32 18 (three rows a CU, one after the other).
// Each workgroup takes every gridDim-th row (or 256 / G of them) and keeps its share of dgamma in registers, since a lane sees the same columns
// in every row; k_rms_columns adds the shares.  The next row's octets are on their way while a row is worked on.
template <bool BF16, int G, int V>
__global__ __launch_bounds__(threads_of(G)) void k_rms_backward(RmsArgs a)
{
    constexpr int kRows = threads_of(G) / G;
    __shared__ float red[G > 64 ? 2 * G / 64 : 1];
    __shared__ float share[G > 64 ? 1 : 8 * G * V];
    int turn = 0;
    const int t = threadIdx.x % G;
    const float inv = 1.0f / (float)a.cols;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
    Octet<BF16> z_next[V] = {}, dy_next[V] = {}, in_next[V] = {};
    float rstd_next = 0.0f;
    auto fetch = [&](int64_t from) {
        if (from < a.rows) rstd_next = a.rstd[from];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v), left = from < a.rows ? a.cols - col : 0;
            begin<BF16, G>(z_next[v], a.z_in.data, from * a.z_in.pitch + col, left, a.cols);
            begin<BF16, G>(dy_next[v], a.dy.data, from * a.dy.pitch + col, left, a.cols);
            if (a.dz_in.data) begin<BF16, G>(in_next[v], a.dz_in.data, from * a.dz_in.pitch + col, left, a.cols);
        }
    };
    fetch(row);
    float gamma[V][8], dgamma[V][8] = {};
    load_columns<G, V>(a.gamma, a.cols, t, gamma);
    for (; row < a.rows; row += stride) {
        Octet<BF16> z[V], dy[V], in[V];
        const float rstd = rstd_next;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            z[v] = z_next[v];
            dy[v] = dy_next[v];
            in[v] = in_next[v];
        }
        fetch(row + stride);
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float zv[8], dv[8];
            const int left = a.cols - 8 * (t + G * v);
            finish<BF16, G>(z[v], left, a.cols, zv);
            finish<BF16, G>(dy[v], left, a.cols, dv);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hat = i < left ? zv[i] * rstd : 0.0f;          // (0 rstd is no 0 if rstd is infinite)
                sum = __builtin_fmaf(dv[i] * gamma[v][i], hat, sum);
                dgamma[v][i] = __builtin_fmaf(dv[i], hat, dgamma[v][i]);
            }
        }
        if (a.dz.data) {
            const float mean = group_sum<G>(sum, red, turn) * inv;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float zv[8], dv[8], add[8], w[8];
                const int col = 8 * (t + G * v), left = a.cols - col;
                finish<BF16, G>(z[v], left, a.cols, zv);
                finish<BF16, G>(dy[v], left, a.cols, dv);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = rstd * (dv[i] * gamma[v][i] - zv[i] * rstd * mean);
                if (a.dz_in.data) finish<BF16, G>(in[v], left, a.cols, add);
                finish_dz<BF16>(a, row, col, left, add, w);
            }
        }
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * a.cols;
    if constexpr (G > 64) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v);
            store_octet<false>(out, col, a.cols - col, dgamma[v]);
        }
    } else {
        // the rows of a wave, the workgroup's waves one after the other, then columns of the sum by all threads
        auto place = [&](int v, int i) -> float & { return share[(v * 8 + i) * G + t]; };
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) dgamma[v][i] = places_sum<G>(dgamma[v][i]);
        for (int g = 0; g < kThreads / 64; ++g) {
            if ((int)threadIdx.x / 64 == g && (threadIdx.x & 63) < G)
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) place(v, i) = g ? place(v, i) + dgamma[v][i] : dgamma[v][i];
            __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += kThreads) {
            const int octet = c >> 3;
            out[c] = share[((octet / G) * 8 + (c & 7)) * G + octet % G];
        }
    }
}

// Rows of more than 8192 columns: two sweeps by a workgroup; the sums over rows are k_rms_column_parts's, which reads dy and z once more.  The mean is
// summed in 64 bits: a lane's share of a row has no bound here, and in 32 the mean of 3000001 equal terms was off by 4.8e-6 of itself, 80 times 2^-24.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_rms_backward_long(RmsArgs a)
{
    __shared__ double red[8];
    int turn = 0;
    const double inv = 1.0 / (double)a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        double sum = 0.0;
        float z[8], dy[8], gamma[8], w[8];
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = octet_left(a.cols - col);
            load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
            load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
            load_octet<false>(a.gamma, col, left, gamma);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) sum = __builtin_fma((double)(dy[i] * gamma[i]), (double)(z[i] * rstd), sum);
        }
        const float mean = (float)(group_sum<kThreads>(sum, red, turn) * inv);
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = octet_left(a.cols - col);
            load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
            load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
            load_octet<false>(a.gamma, col, left, gamma);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = rstd * (dy[i] * gamma[i] - z[i] * rstd * mean);
            float in[8];
            if (a.dz_in.data) load_octet<BF16>(a.dz_in.data, row * a.dz_in.pitch + col, left, in);
            finish_dz<BF16>(a, row, col, left, in, w);
        }
    }
}

// Shares of dgamma for rows too long for registers: workgroup (x, y) takes 2048 columns of every gridDim.y-th row.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_rms_column_parts(RmsArgs a)
{
    const int64_t col = 8 * ((int64_t)blockIdx.x * kThreads + threadIdx.x);
    if (col >= a.cols) return;
    const int left = octet_left(a.cols - col);
    float dgamma[8] = {};
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row];
        float z[8], dy[8];
        load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
        load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
#pragma unroll
        for (int i = 0; i < 8; ++i) dgamma[i] = __builtin_fmaf(dy[i], z[i] * rstd, dgamma[i]);
    }
    store_octet<false>(a.partials + (int64_t)blockIdx.y * a.cols, col, left, dgamma);
}

// Adds the shares: 64 of the sums a workgroup, sixteen threads to a sum.
__global__ __launch_bounds__(1024) void k_rms_columns(const float *partials, int parts, int cols, float *dgamma)
{
    __shared__ double red[16][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const int64_t c = (int64_t)group_index() * 64 + lane, n = cols;
    double s = 0.0;
    if (c < n && parts > 0) {
        int p = part;
        for (; p + 112 < parts; p += 128) {                 // eight loads on their way at a time
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = partials[(p + 16 * u) * n + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += (double)v[u];
        }
        float v[8];                                         // (loaded without a branch: eight that wait for one another cost 500 x 8192 fp32 1.3 us)
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = partials[min(p + 16 * u, parts - 1) * n + c];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (p + 16 * u < parts) s += (double)v[u];
    }
    red[part][lane] = s;
    __syncthreads();
    if (part || c >= n) return;
#pragma unroll
    for (int p = 1; p < 16; ++p) s += red[p][lane];
    dgamma[c] = (float)s;
}

// Lanes to a row and octets a lane: the fewest that hold a row in 8 or 16 columns each up to 1024 columns, so that a row ends without a barrier and a
// workgroup has several (16384 x 1024 bf16 on 64 lanes 21.3 us, the three quarters as many elements of 8192 x 1536 on 256 lanes 21.8); beyond that an octet a lane, since a
// row's values of 64 bits are many registers.
template <typename F>
void by_width(int64_t cols, F &&go)
{
    using std::integral_constant;
    typedef integral_constant<int, 1> One;
    typedef integral_constant<int, 2> Two;
    if (cols <= 128) go(integral_constant<int, 16>{}, One{});
    else if (cols <= 256) go(integral_constant<int, 32>{}, One{});
    else if (cols <= 512) go(integral_constant<int, 64>{}, One{});
    else if (cols <= 1024) go(integral_constant<int, 64>{}, Two{});
    else if (cols <= 2048) go(integral_constant<int, 256>{}, One{});
    else if (cols <= 4096) go(integral_constant<int, 512>{}, One{});
    else if (cols <= 6144) go(integral_constant<int, 768>{}, One{});
    else go(integral_constant<int, 1024>{}, One{});
}

// Workgroups of the backward pass: about as many as the card holds at a time, but four rows each (two of the widest) where that leaves one a CU: their shares of dgamma are
// written and read again.  us / with as many as there are rows: 512 x 2048 bf16 7.9 / 9.3, 1024 x 2048 9.9 / 10.6, 300 x 8192 11.8 / 13.2; in between / with the whole number
// that the card holds: 1500 x 2048 11.6 / 11.9, 500 x 8192 fp32 18.7 / 19.4.
// A lane adds its rows' terms in fp32, kMostAdded of them at the most, so that its sum's error has a bound: of more rows there are whole turns of workgroups
// (in one turn the sum of 20000000 equal terms, five columns of them, was off by 1.2e-5).  us / in one turn: 131072 x 2048 bf16 321 / 305, 40000 x 4096 193 / 180, 1000000 x 700 876 / 1070.
constexpr int64_t kMostAdded = 128;
int64_t parts_of(int64_t rows, int64_t cols)
{
    int64_t most = 512, few = 256, least = 4, per = 1;
    if (cols > kMostCols) {
        few = most;
    } else {
        by_width(cols, [&](auto g, auto) {
            constexpr int G = decltype(g)::value;
            per = threads_of(G) / G;
            if (G <= 64) few = most = 1024;
            if (G >= 512) most = 256;
            if (G > 512) few = 128, least = 2;
        });
    }
    const int64_t turn = kMostAdded * per * most;                   // rows
    if (rows > turn) return (rows + turn - 1) / turn * most;
    return std::min({rows, std::max((rows + least - 1) / least, few), most});
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace

void launch_rms_forward(const RmsArgs &a, bool bf16, hipStream_t st)
{
    const bool packed = a.packed.codes != nullptr;
    const int64_t padded_rows = (a.rows + 63) / 64 * 64, pieces = ((int64_t)a.cols + 127) / 128, rows = packed ? padded_rows : a.rows;
    by_bool(bf16, [&](auto b) {
        by_bool(a.z.data != nullptr, [&](auto fused) {
            constexpr bool B = decltype(b)::value, F = decltype(fused)::value;
            if (a.cols > kMostCols) {
                hipLaunchKernelGGL((k_rms_forward_long<B, F>), dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), dim3(kThreads), 0, st, a, padded_rows, pieces);
                return;
            }
            by_width(a.cols, [&](auto g, auto v) {
                constexpr int G = decltype(g)::value, V = decltype(v)::value, kRows = threads_of(G) / G;
                constexpr int kFew = kRows, kLow = kRows > 4 ? kRows : 4, kHigh = G <= 512 ? 16 : 8, kFull = G == 256 ? 1024 : 512;
                // Rows a workgroup, us: one row, so that all CUs work, 64 x 2048 bf16 3.5, 256 x 8192 7.4 / four rows 6.6, 12.6; four 2048 x 2048 9.7, 1024 x 8192 15 / one row 10.9, 24.  Whole
                // squares of codes where 512 workgroups have them: 8192 x 4096 43.3, 16384 x 1024 21.3, 4096 x 8192 (half ones) 45.6 / four rows 44.8, eight rows 23.1, four 51.0;
                // 1024 workgroups of one row at a time in 256 threads: with the values' launch behind it 16384 x 2048 113 us a step / four rows 118, but 8192 x 2048 27.3 alone / 23.6.
                // And only where their turns are filled to three quarters (of 256 threads, three fifths): 28000 x 2048 80.9 / four rows 85.8, 32000 x 2048 91.6 / 95.4, 20000 x 1024 29.4 /
                // 30.7, but 17000 x 2048 57.7 / 53.1, 20000 x 2048 64.4 / 64.1, 9000 x 4096 66.6 / 55.7, 12000 x 4096 72.5 / 69.5, 9000 x 1024 15.7 / 14.6, 9000 x 5120 98.1 / 94.2.
                const int64_t full = kFull * kHigh, turns = (rows + full - 1) / full;
                const bool filled = rows >= full && (G == 256 ? rows * 5 >= turns * full * 3 : rows * 4 >= turns * full * 3);
                auto go = [&](auto h) {
                    constexpr int H = decltype(h)::value, kGroup = H ? H : kRows;
                    const int64_t groups = (rows + kGroup - 1) / kGroup;
                    hipLaunchKernelGGL((k_rms_forward<B, G, V, F, H>), dim3((unsigned)std::min<int64_t>(groups, 2048)), dim3(threads_of(G)), 0, st, a, padded_rows,
                                       pieces);
                };
                if (!packed) go(std::integral_constant<int, 0>{});
                else if (rows <= 512) go(std::integral_constant<int, kFew>{});
                else if (!filled) go(std::integral_constant<int, kLow>{});
                else go(std::integral_constant<int, kHigh>{});
            });
        });
    });
}

int64_t rms_partials(int64_t rows, int64_t cols)
{
    return parts_of(rows, cols);
}

void launch_rms_backward(const RmsArgs &a, bool bf16, hipStream_t st)
{
    const int64_t parts = rms_partials(a.rows, a.cols);
    int used = (int)parts;
    if (parts > 0) by_bool(bf16, [&](auto b) {
        constexpr bool B = decltype(b)::value;
        if (a.cols > kMostCols) {
            // (first: dz may take the place of dy or z)
            if (a.partials)
                hipLaunchKernelGGL((k_rms_column_parts<B>), dim3((unsigned)(((int64_t)a.cols + 2047) / 2048), (unsigned)parts), dim3(kThreads), 0, st, a);
            if (a.dz.data)
                hipLaunchKernelGGL((k_rms_backward_long<B>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(kThreads), 0, st, a);
            return;
        }
        by_width(a.cols, [&](auto g, auto v) {
            constexpr int G = decltype(g)::value;
            const int64_t per = threads_of(G) / G;
            used = (int)std::min<int64_t>((a.rows + per - 1) / per, parts);
            hipLaunchKernelGGL((k_rms_backward<B, G, decltype(v)::value>), dim3((unsigned)used), dim3(threads_of(G)), 0, st, a);
        });
    });
    if (a.dgamma)
        hipLaunchKernelGGL(k_rms_columns, grid_of(((int64_t)a.cols + 63) / 64), dim3(1024), 0, st, a.partials, used, a.cols, a.dgamma);
}

}  // namespace conef
