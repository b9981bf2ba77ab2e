// Dropout whose mask is drawn again where it is needed, and layer norm's forward and backward pass with that dropout and the
// residual in front of it.
//
// z = residual + keep(x) / (share kept), y = (z - mean) rstd gamma + beta; the statistics of a row are those of z as it is
// stored, so that the backward pass, which reads the stored z, differentiates what was computed.
// With a = dy gamma and hat = (z - mean) rstd:
//   dz = rstd (a - mean(a) - hat mean(a hat)) + dz_in,   dx = keep(dz) / (share kept),
//   dgamma = sum over rows of dy hat,   dbeta = sum over rows of dy.
// All sums are fp32 in a fixed order (no atomics), those over rows fp64 at the last level; a row's variance is that of the values less
// their mean, in a second sweep over registers.
#include <algorithm>
#include <type_traits>

#include "layers_device.h"

namespace conef {

namespace {

constexpr int kThreads = 256;
constexpr int kForwardCols = 16384, kBackwardCols = 12288;      // the widest rows that a workgroup holds in registers

inline bool in_registers(int64_t cols, int most) { return cols <= most; }

// threads of a workgroup in which G share a row
constexpr int threads_of(int g) { return g > kThreads ? g : kThreads; }

// ---------------------------------------------------------------- dropout
// An octet a thread, which takes one Philox call.  Bound by memory: 16384 x 4096 in bf16 with a residual 68 us, 403 MB at 5.9 TB/s (a copy of
// a gigabyte reaches 5.1; some of this comes from the card's last cache); the 150 vector instructions of an octet hide behind the loads.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutArgs a, uint32_t octets, uint32_t per_row)
{
    const uint32_t o = group_index() * kThreads + threadIdx.x;
    if (o >= octets) return;
    const uint32_t row = o / per_row;
    const int col = (int)(o - row * per_row) * 8, left = a.cols - col;
    float v[8];
    load_octet<BF16>(a.x.data, row * a.x.pitch + col, left, v);
    drop_octet(a.d, o, v);
    if (a.residual.data) {
        float r[8];
        load_octet<BF16>(a.residual.data, row * a.residual.pitch + col, left, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r[i] + v[i];
    }
    store_octet<BF16>(a.y.data, row * a.y.pitch + col, left, v);
}

// ---------------------------------------------------------------- layer norm
// Sums of N values over the G lanes that share a row, in every one of them.  G > 64 (a workgroup's threads): `red` holds 2 x G / 64 x N
// floats, used in turn by consecutive calls (`turn`), so one barrier a call is enough.
template <int G, int N>
__device__ __forceinline__ void group_sum(float v[N], float *red, int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<(G < 64 ? G : 64)>(v[i]);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float *slot = red + turn * W * N;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) slot[(threadIdx.x >> 6) * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s[W];
#pragma unroll
            for (int w = 0; w < W; ++w) s[w] = slot[w * N + i];
#pragma unroll
            for (int step = 1; step < W; step *= 2)
#pragma unroll
                for (int w = 0; w + step < W; w += 2 * step) s[w] += s[w + step];
            v[i] = s[0];
        }
    }
}

// A row's octets, begun and finished.  Rows of fewer than 8 columns, which have eight lanes, are loaded element by element.
template <bool BF16, int G>
__device__ __forceinline__ void begin(Octet<BF16> &o, const void *data, int64_t at, int left, int cols)
{
    if (G == 8 && cols < 8) o = fetch_octet<BF16>(data, at, left);
    else begin_octet<BF16>(o, data, at, left);
}
template <bool BF16, int G>
__device__ __forceinline__ void finish(const Octet<BF16> &o, int left, int cols, float v[8])
{
    if (G == 8 && cols < 8) widen<BF16>(o, v);
    else finish_octet<BF16>(o, left, v);
}

// a row's gamma or beta, laid out like the row
template <int G, int V>
__device__ __forceinline__ void load_columns(const float *p, int cols, int t, float out[V][8])
{
    Octet<false> o[V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) begin<false, G>(o[v], p, 8 * (t + G * v), cols - 8 * (t + G * v), cols);
#pragma unroll
    for (int v = 0; v < V; ++v) finish<false, G>(o[v], cols - 8 * (t + G * v), cols, out[v]);
}

// G lanes hold a row, V octets each: octet v of lane t starts at column 8 (t + G v).  The next row's octets are on their way while a row is
// worked on.  Bound by memory where there are rows enough for that: 16384 x 2048 in bf16 with dropout and residual 54 us, 268 MB at 5.0 TB/s,
// without them 26 us; 777 x 5003 in fp32, three rows a CU, 17 us, 62 MB at 3.7 TB/s: as many rows again as are worked on are on their way, and no more.
template <bool BF16, int G, int V, bool FUSED>
__global__ __launch_bounds__(threads_of(G)) void k_norm_forward(NormArgs a)
{
    constexpr int kRows = threads_of(G) / G;
    __shared__ float red[G > 64 ? 2 * G / 64 : 1];
    int turn = 0;
    const int t = threadIdx.x % G;
    const float inv = 1.0f / (float)a.cols;
    const uint32_t per_row = ((uint32_t)a.cols + 7) >> 3;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
    Octet<BF16> x[V] = {}, r[FUSED ? V : 1] = {};
    auto fetch = [&](int64_t from) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v), left = from < a.rows ? a.cols - col : 0;
            begin<BF16, G>(x[v], a.x.data, from * a.x.pitch + col, left, a.cols);
            if (FUSED && a.residual.data) begin<BF16, G>(r[v], a.residual.data, from * a.residual.pitch + col, left, a.cols);
        }
    };
    fetch(row);
    float gamma[V][8], beta[V][8];
    load_columns<G, V>(a.gamma, a.cols, t, gamma);
    load_columns<G, V>(a.beta, a.cols, t, beta);
    for (; row < a.rows; row += stride) {
        float z[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v);
            finish<BF16, G>(x[v], a.cols - col, a.cols, z[v]);
            if constexpr (FUSED) {
                if (a.drop) drop_octet(a.d, (uint32_t)row * per_row + (uint32_t)(t + G * v), z[v]);
                if (a.residual.data) {
                    float add[8];
                    finish<BF16, G>(r[v], a.cols - col, a.cols, add);
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[v][i] = add[i] + z[v][i];
                }
                store_octet<BF16>(a.z.data, row * a.z.pitch + col, a.cols - col, z[v]);
            }
        }
        fetch(row + stride);
        float sum[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += z[v][i];
        group_sum<G, 1>(sum, red, turn);
        const float mean = sum[0] / (float)a.cols;          // (not times inv: a constant row's mean is its value, and 1 / sqrt(eps) multiplies what it is off by)
        sum[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = 8 * (t + G * v) + i < a.cols ? z[v][i] - mean : 0.0f;
                sum[0] = __builtin_fmaf(c, c, sum[0]);
            }
        group_sum<G, 1>(sum, red, turn);
        const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps);
        if (t == 0) {
            if (a.mean_out) a.mean_out[row] = mean;
            if (a.rstd_out) a.rstd_out[row] = rstd;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = __builtin_fmaf((z[v][i] - mean) * rstd, gamma[v][i], beta[v][i]);
            store_octet<BF16>(a.y.data, row * a.y.pitch + col, a.cols - col, z[v]);
        }
    }
}

// A row of any length, in three sweeps over it by a workgroup.
template <bool BF16, bool FUSED>
__global__ __launch_bounds__(kThreads) void k_norm_forward_long(NormArgs a)
{
    __shared__ float red[8];
    int turn = 0;
    const float inv = 1.0f / (float)a.cols;
    const uint32_t per_row = ((uint32_t)a.cols + 7) >> 3;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void *src = FUSED ? a.z.data : a.x.data;
        const int64_t at = row * (FUSED ? a.z.pitch : a.x.pitch);
        float sum[1] = {0.0f};
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
            float z[8];
            load_octet<BF16>(a.x.data, row * a.x.pitch + col, left, z);
            if constexpr (FUSED) {
                if (a.drop) drop_octet(a.d, (uint32_t)row * per_row + (uint32_t)(col >> 3), z);
                if (a.residual.data) {
                    float r[8];
                    load_octet<BF16>(a.residual.data, row * a.residual.pitch + col, left, r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = r[i] + z[i];
                }
                store_octet<BF16>(a.z.data, at + col, left, z);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) sum[0] += z[i];
        }
        group_sum<kThreads, 1>(sum, red, turn);
        const float mean = sum[0] / (float)a.cols;          // (as above)
        sum[0] = 0.0f;
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
            float z[8];
            load_octet<BF16>(src, at + col, left, z);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) sum[0] = __builtin_fmaf(z[i] - mean, z[i] - mean, sum[0]);
        }
        group_sum<kThreads, 1>(sum, red, turn);
        const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean_out) a.mean_out[row] = mean;
            if (a.rstd_out) a.rstd_out[row] = rstd;
        }
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
            float z[8], gamma[8], beta[8];
            load_octet<BF16>(src, at + col, left, z);
            load_octet<false>(a.gamma, col, left, gamma);
            load_octet<false>(a.beta, col, left, beta);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = __builtin_fmaf((z[i] - mean) * rstd, gamma[i], beta[i]);
            store_octet<BF16>(a.y.data, row * a.y.pitch + col, left, z);
        }
    }
}

// hat and a = dy gamma of an octet
__device__ __forceinline__ void hat_and_a(const float z[8], const float dy[8], const float gamma[8], float mean, float rstd,
                                          float hat[8], float a[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hat[i] = (z[i] - mean) * rstd;
        a[i] = dy[i] * gamma[i];
    }
}

// Adds dz_in, writes dz and, from the unrounded values, dx.
template <bool BF16>
__device__ __forceinline__ void finish_dz(const NormArgs &a, int64_t row, int64_t col, int left, uint32_t octet, const float dz_in[8],
                                          float v[8])
{
    if (a.dz_in.data) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += dz_in[i];
    }
    if (a.dx.data) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[i];
        if (a.drop) drop_octet(a.d, octet, x);
        store_octet<BF16>(a.dx.data, row * a.dx.pitch + col, left, x);
    }
    if (a.dz.data) store_octet<BF16>(a.dz.data, row * a.dz.pitch + col, left, v);
}

// Each workgroup takes every gridDim-th row (or 256 / G of them) and keeps its share of dgamma and dbeta in registers, since a lane
// sees the same columns in every row; k_norm_columns adds the shares.  The next row's octets are on their way while a row is worked on.
// Bound by memory: 16384 x 2048 in bf16 with dropout and residual's gradient 68 us with the shares' sum, of which that is 4: 336 MB, and 8 MB of
// shares written and read, at 5.2 TB/s; 777 x 5003 in fp32 23 us with 4 of them, 88 MB and twice 10 at 4.7 TB/s.
template <bool BF16, int G, int V>
__global__ __launch_bounds__(threads_of(G)) void k_norm_backward(NormArgs a)
{
    constexpr int kRows = threads_of(G) / G;
    __shared__ float red[G > 64 ? 4 * G / 64 : 1];
    constexpr bool kInLds = G >= 768 && V == 2;         // the shares, which registers do not hold; nor,
    constexpr bool kAhead = !kInLds || (BF16 && G == 768);          // of these but some, the next row
    __shared__ float share[G > 64 && !kInLds ? 1 : 2 * 8 * G * V];
    int turn = 0;
    const int t = threadIdx.x % G;
    const float inv = 1.0f / (float)a.cols;
    const uint32_t per_row = ((uint32_t)a.cols + 7) >> 3;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
    Octet<BF16> z_next[V] = {}, dy_next[V] = {}, in_next[V] = {};
    float mean_next = 0.0f, rstd_next = 0.0f;
    auto fetch = [&](int64_t from) {
        if (from < a.rows) {
            mean_next = a.mean[from];
            rstd_next = a.rstd[from];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v), left = from < a.rows ? a.cols - col : 0;
            begin<BF16, G>(z_next[v], a.z_in.data, from * a.z_in.pitch + col, left, a.cols);
            begin<BF16, G>(dy_next[v], a.dy.data, from * a.dy.pitch + col, left, a.cols);
            if (a.dz_in.data) begin<BF16, G>(in_next[v], a.dz_in.data, from * a.dz_in.pitch + col, left, a.cols);
        }
    };
    if constexpr (kAhead) fetch(row);
    float gamma[V][8], dgamma[V][8] = {}, dbeta[V][8] = {};
    load_columns<G, V>(a.gamma, a.cols, t, gamma);
    // (element i of lane t's octet v in place (8 v + i) G + t, so that neighbours lie in neighbouring banks)
    auto place = [&](int v, int i) -> float * { return share + (v * 8 + i) * G + t; };
    if constexpr (kInLds)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) place(v, i)[0] = place(v, i)[8 * G * V] = 0.0f;
    for (; row < a.rows; row += stride) {
        if constexpr (!kAhead) fetch(row);
        Octet<BF16> z[V], dy[V], in[V];
        const float mean = mean_next, rstd = rstd_next;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            z[v] = z_next[v];
            dy[v] = dy_next[v];
            in[v] = in_next[v];
        }
        if constexpr (kAhead) fetch(row + stride);
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float zv[8], dv[8], hat[8], w[8];
            const int left = a.cols - 8 * (t + G * v);
            finish<BF16, G>(z[v], left, a.cols, zv);
            finish<BF16, G>(dy[v], left, a.cols, dv);
            hat_and_a(zv, dv, gamma[v], mean, rstd, hat, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // Columns beyond the row's end have dy = gamma = 0, but (0 - mean) rstd may be infinite there where no hat of the row is.  (An element's choice, up to
                // 4 % of the pass; behind a branch the octet's hats take eight more registers: 16384 x 3000 in bf16 79 us for 65.)
                sums[0] += w[i];
                sums[1] = __builtin_fmaf(w[i], i < left ? hat[i] : 0.0f, sums[1]);
                if constexpr (kInLds) {
                    float *p = place(v, i);
                    p[0] = __builtin_fmaf(dv[i], hat[i], p[0]);
                    p[8 * G * V] += dv[i];
                } else {
                    dgamma[v][i] = __builtin_fmaf(dv[i], hat[i], dgamma[v][i]);
                    dbeta[v][i] += dv[i];
                }
            }
        }
        if (a.dz.data || a.dx.data) {
            group_sum<G, 2>(sums, red, turn);
            const float m0 = sums[0] * inv, m1 = sums[1] * inv;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float zv[8], dv[8], hat[8], w[8], add[8];
                const int col = 8 * (t + G * v), left = a.cols - col;
                finish<BF16, G>(z[v], left, a.cols, zv);
                finish<BF16, G>(dy[v], left, a.cols, dv);
                hat_and_a(zv, dv, gamma[v], mean, rstd, hat, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = rstd * ((w[i] - m0) - hat[i] * m1);
                if (a.dz_in.data) finish<BF16, G>(in[v], left, a.cols, add);
                finish_dz<BF16>(a, row, col, left, (uint32_t)row * per_row + (uint32_t)(t + G * v), add, w);
            }
        }
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (G > 64) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = 8 * (t + G * v);
            if constexpr (kInLds)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dgamma[v][i] = place(v, i)[0];
                    dbeta[v][i] = place(v, i)[8 * G * V];
                }
            store_octet<false>(out, col, a.cols - col, dgamma[v]);
            store_octet<false>(out + a.cols, col, a.cols - col, dbeta[v]);
        }
    } else {
        // the rows of a wave, the workgroup's waves one after the other, then columns of the sum by all threads
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dgamma[v][i] = places_sum<G>(dgamma[v][i]);
                dbeta[v][i] = places_sum<G>(dbeta[v][i]);
            }
        for (int g = 0; g < kThreads / 64; ++g) {
            if ((int)threadIdx.x / 64 == g && (threadIdx.x & 63) < G)
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float *p = place(v, i), *q = p + 8 * G * V;
                        *p = g ? *p + dgamma[v][i] : dgamma[v][i];
                        *q = g ? *q + dbeta[v][i] : dbeta[v][i];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += kThreads) {
            const int octet = c >> 3, at = ((octet / G) * 8 + (c & 7)) * G + octet % G;
            out[c] = share[at];
            out[a.cols + c] = share[8 * G * V + at];
        }
    }
}

// Rows of more than 12288 columns: two sweeps by a workgroup; the sums over rows are k_norm_column_parts's, which reads dy and z once more: with it 4096 x 16384 in
// bf16 takes 233 us, where its bytes, read once, are 134 at a copy's rate.  (1024 threads have 128 registers each, too few for an fp32 row of 16384 even with the
// shares in LDS.  A bf16 row might fit; the bound is the same for both types, and a kernel for it alone was not tried.)
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_norm_backward_long(NormArgs a)
{
    __shared__ float red[16];
    int turn = 0;
    const float inv = 1.0f / (float)a.cols;
    const uint32_t per_row = ((uint32_t)a.cols + 7) >> 3;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sums[2] = {0.0f, 0.0f}, z[8], dy[8], gamma[8], hat[8], w[8];
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
            load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
            load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
            load_octet<false>(a.gamma, col, left, gamma);
            hat_and_a(z, dy, gamma, mean, rstd, hat, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sums[0] += w[i];
                if (i < left) sums[1] = __builtin_fmaf(w[i], hat[i], sums[1]);          // (as in k_norm_backward)
            }
        }
        group_sum<kThreads, 2>(sums, red, turn);
        const float m0 = sums[0] * inv, m1 = sums[1] * inv;
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kThreads) {
            const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
            load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
            load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
            load_octet<false>(a.gamma, col, left, gamma);
            hat_and_a(z, dy, gamma, mean, rstd, hat, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = rstd * ((w[i] - m0) - hat[i] * m1);
            float in[8];
            if (a.dz_in.data) load_octet<BF16>(a.dz_in.data, row * a.dz_in.pitch + col, left, in);
            finish_dz<BF16>(a, row, col, left, (uint32_t)row * per_row + (uint32_t)(col >> 3), in, w);
        }
    }
}

// Shares of dgamma and dbeta for rows too long for registers: workgroup (x, y) takes 2048 columns of every gridDim.y-th row.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_norm_column_parts(NormArgs a)
{
    const int64_t col = 8 * ((int64_t)blockIdx.x * kThreads + threadIdx.x);
    if (col >= a.cols) return;
    const int left = (int)(a.cols - col < 8 ? a.cols - col : 8);
    float dgamma[8] = {}, dbeta[8] = {};
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float z[8], dy[8];
        load_octet<BF16>(a.z_in.data, row * a.z_in.pitch + col, left, z);
        load_octet<BF16>(a.dy.data, row * a.dy.pitch + col, left, dy);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dgamma[i] = __builtin_fmaf(dy[i], (z[i] - mean) * rstd, dgamma[i]);
            dbeta[i] += dy[i];
        }
    }
    float *out = a.partials + (int64_t)blockIdx.y * 2 * a.cols;
    store_octet<false>(out, col, left, dgamma);
    store_octet<false>(out + a.cols, col, left, dbeta);
}

// Adds the shares: 64 of the 2 cols sums a workgroup, sixteen threads to a sum.
__global__ __launch_bounds__(1024) void k_norm_columns(const float *partials, int parts, int cols, float *dgamma, float *dbeta)
{
    __shared__ double red[16][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const int64_t c = (int64_t)group_index() * 64 + lane, n = 2 * (int64_t)cols;
    double s = 0.0;
    if (c < n) {
        int p = part;
        for (; p + 112 < parts; p += 128) {                 // eight loads on their way at a time
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = partials[(p + 16 * u) * n + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += (double)v[u];
        }
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p + 16 * u < parts ? partials[(p + 16 * u) * n + c] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += (double)v[u];
    }
    red[part][lane] = s;
    __syncthreads();
    if (part || c >= n) return;
#pragma unroll
    for (int p = 1; p < 16; ++p) s += red[p][lane];
    float *out = c < cols ? dgamma : dbeta;
    if (out) out[c < cols ? c : c - cols] = (float)s;
}

// Rows of 2048 columns and more on an octet a lane, as many waves (in twos) as they have octets for.
template <int G, int MOST, typename F>
void by_lanes(int64_t cols, F &&go)
{
    if (cols <= 8 * G) go(std::integral_constant<int, G>{}, std::integral_constant<int, 1>{});
    else if constexpr (8 * G < MOST) by_lanes<G + 128, MOST>(cols, go);
}

// Lanes to a row and octets a lane.  Rows of up to 256 columns share a wave, 8 to 32 lanes each: 32768 x 100 in bf16 forward 8.8 us, backward 15.3 with both
// kernels, a wave to a row 19 and 29; 32768 x 7, which eight lanes load element by element, 5.4 and 12.2, by a workgroup to a row 78 and 118 (all fused).
// Otherwise two octets a lane at most, which registers hold together with the next row on its way.  A wave to a row needs no barrier, but
// four octets a lane (2048 columns) take 256 registers: the backward pass of 16384 x 2048 in bf16 then takes 86 us, with a workgroup to
// a row 75.  Rows of 2048 columns to MOST take one octet a lane: up to 8192 in the fused forward pass, 6144 in the backward pass, whose registers hold
// no more.  us, so / 256 or 512 lanes of two: forward 777 x 5003 fp32 17.8 / 20.7, 8192 x 5120 bf16 65 / 72, 4096 x 7000 fp32 89 / 102, 8192 x 2560
// bf16 34 / 38, 4096 x 8192 bf16 52 / 50; backward 777 x 5003 fp32 23 / 26, 8192 x 5120 bf16 93 / 106, 16384 x 3000 bf16 100 / 115, 8192 x 4096
// fp32 133 / 135.  A forward pass that is not fused has little to hold: 777 x 5003 fp32 11.0 / 9.9, 8192 x 5120 bf16 39 / 37.
// Beyond 8192 768 lanes or 1024: forward 3000 x 10000 bf16 51 / 58, 2000 x 10000 fp32 70 / 69, 300 x 12000 fp32 17.6 / 20.0; backward, with shares in LDS,
// 768 or, as any other length, in two sweeps: 3000 x 10000 bf16 71 / 119, 2000 x 10000 fp32 95 / 149.
constexpr int kFusedLanes = 8192, kBackwardLanes = 6144, kPairs = 0;

template <int MOST, typename F>
void by_width(int64_t cols, F &&go)
{
    using std::integral_constant;
    typedef integral_constant<int, 1> One;
    typedef integral_constant<int, 2> Two;
    if (cols <= 64) go(integral_constant<int, 8>{}, One{});
    else if (cols <= 128) go(integral_constant<int, 16>{}, One{});
    else if (cols <= 256) go(integral_constant<int, 32>{}, One{});
    else if (cols <= 512) go(integral_constant<int, 64>{}, One{});
    else if (cols <= 1024) go(integral_constant<int, 64>{}, Two{});
    else if (cols <= 2048) go(integral_constant<int, 256>{}, One{});
    else if (cols <= MOST) {
        if constexpr (MOST > 0) by_lanes<384, MOST>(cols, go);
    } else if (cols <= 4096) {
        if constexpr (MOST < 4096) go(integral_constant<int, 256>{}, Two{});
    } else if (cols <= 8192) {
        if constexpr (MOST < 8192) go(integral_constant<int, 512>{}, Two{});
    } else if (cols <= 12288) {
        go(integral_constant<int, 768>{}, Two{});
    } else {
        if constexpr (MOST != kBackwardLanes) go(integral_constant<int, 1024>{}, Two{});      // (the backward pass has no rows as wide)
    }
}

// Workgroups of the forward pass: about as many as the card holds at a time, so that each works on several rows with the next one on its way.
// us, so many / 2048, all fused: 777 x 5003 fp32 16.7 / 18.6, 8192 x 1024 bf16 14.0 / 14.9, 4096 x 16384 bf16 100 / 117, 16384 x 2048 bf16 53 / 53.
constexpr int forward_groups(int g, int v) { return g * v > 640 ? 512 : g * v > 256 || v == 2 ? 768 : 1536; }

// Workgroups of the backward pass of rows of that width: as many as the card holds at a time (four or two of 256 threads a CU, else two or one), but
// four rows each (two of more than 512 lanes) where that leaves one for a CU (every other one): their shares of dgamma and dbeta are written and read
// again.  us with both kernels, not fused, so / with a row each: 1024 x 2048 bf16 11.3 / 18.0, 500 x 4000 bf16 12.5 / 17.6, 256 x 5003 fp32 12.8 / 15.8.  At most
// 512 of 256 threads, or 1024: 16384 x 2048 bf16 fused 65 / 73 (not fused 42 / 41), fp32 134 / 139; 256 of 512 threads, or 512: 4096 x 4096
// fp32 66 / 69, 16384 x 3500 fp32 208 / 228.
int64_t parts_of(int64_t rows, int64_t cols)
{
    int64_t most = 512, few = 256, least = 4;
    if (!in_registers(cols, kBackwardCols)) return std::min(rows, most);
    by_width<kBackwardLanes>(cols, [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, V = decltype(v)::value;
        if (G == 64) few = most = V == 1 ? 1024 : 512;
        if (G < 64) few = most;
        if (G >= 512) most = 256;
        if (G * V > 512) few = 128, least = 2;
    });
    return std::min({rows, std::max((rows + least - 1) / least, few), most});
}

template <typename F>
void by_bool(bool v, F &&go)
{
    if (v) go(std::true_type{});
    else go(std::false_type{});
}

}  // namespace

void launch_dropout(const DropoutArgs &a, bool bf16, hipStream_t st)
{
    const uint32_t per_row = ((uint32_t)a.cols + 7) / 8, octets = (uint32_t)a.rows * per_row;
    const dim3 grid = grid_of(((int64_t)octets + kThreads - 1) / kThreads);
    by_bool(bf16, [&](auto b) { hipLaunchKernelGGL((k_dropout<decltype(b)::value>), grid, dim3(kThreads), 0, st, a, octets, per_row); });
}

void launch_norm_forward(const NormArgs &a, bool bf16, hipStream_t st)
{
    by_bool(bf16, [&](auto b) {
        by_bool(a.z.data != nullptr, [&](auto fused) {
            if (!in_registers(a.cols, kForwardCols)) {
                const dim3 grid((unsigned)std::min<int64_t>(a.rows, 1 << 20));
                hipLaunchKernelGGL((k_norm_forward_long<decltype(b)::value, decltype(fused)::value>), grid, dim3(kThreads), 0, st, a);
                return;
            }
            by_width<decltype(fused)::value ? kFusedLanes : kPairs>(a.cols, [&](auto g, auto v) {
                constexpr int G = decltype(g)::value;
                const int64_t per = threads_of(G) / G, groups = (a.rows + per - 1) / per;
                hipLaunchKernelGGL((k_norm_forward<decltype(b)::value, G, decltype(v)::value, decltype(fused)::value>),
                                   dim3((unsigned)std::min<int64_t>(groups, forward_groups(G, decltype(v)::value))), dim3(threads_of(G)), 0, st, a);
            });
        });
    });
}

int64_t norm_partials(int64_t rows, int64_t cols)
{
    return parts_of(rows, cols);
}

void launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t st)
{
    const int64_t parts = norm_partials(a.rows, a.cols);
    int used = (int)parts;
    if (parts > 0) by_bool(bf16, [&](auto b) {
        if (!in_registers(a.cols, kBackwardCols)) {
            // (first: dz may take the place of dy or z)
            if (a.partials)
                hipLaunchKernelGGL((k_norm_column_parts<decltype(b)::value>), dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)parts),
                                   dim3(kThreads), 0, st, a);
            if (a.dz.data || a.dx.data)
                hipLaunchKernelGGL((k_norm_backward_long<decltype(b)::value>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)),
                                   dim3(kThreads), 0, st, a);
            return;
        }
        by_width<kBackwardLanes>(a.cols, [&](auto g, auto v) {
            constexpr int G = decltype(g)::value;
            const int64_t per = threads_of(G) / G;
            used = (int)std::min<int64_t>((a.rows + per - 1) / per, parts);
            hipLaunchKernelGGL((k_norm_backward<decltype(b)::value, G, decltype(v)::value>), dim3((unsigned)used), dim3(threads_of(G)), 0, st, a);
        });
    });
    if (a.dgamma || a.dbeta)
        hipLaunchKernelGGL(k_norm_columns, grid_of((2 * (int64_t)a.cols + 63) / 64), dim3(1024), 0, st, a.partials, used, a.cols,
                           a.dgamma, a.dbeta);
}

}  // namespace conef
