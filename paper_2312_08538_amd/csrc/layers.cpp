// C ABI of a training step's own operators (conef_dropout_*, conef_norm_*, conef_mx_*): argument checks and launches.  No call here
// has a context: sizes and pointers are all there is, and nothing is kept from one call for the next.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/conef.h"
#include "layers.h"

using namespace conef;

namespace {

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline int launched() { return hipGetLastError() == hipSuccess ? CONEF_OK : CONEF_EHIP; }

inline size_t element(int dtype) { return dtype == CONEF_F32 ? 4 : 2; }

constexpr int64_t kMostSide = (int64_t)1 << 31;

// rows of elements: a type, sides below 2^31, octets of all rows below 2^32 (they count the draws, and blocks of a grid)
bool bad_shape(int64_t rows, int64_t cols, int dtype)
{
    return (dtype != CONEF_F32 && dtype != CONEF_BF16) || rows < 0 || rows >= kMostSide || cols < 1 || cols >= kMostSide ||
           rows * ((cols + 7) / 8) >= (int64_t)1 << 32;
}

// a matrix that the call needs (or may need): there, aligned to its elements, rows not overlapping
bool bad_rows(const void *data, int64_t pitch, int64_t cols, int dtype)
{
    return !data || misaligned(data, element(dtype)) || pitch < cols || pitch >= (int64_t)1 << 40;
}

bool bad_optional(const void *data, int64_t pitch, int64_t cols, int dtype) { return data && bad_rows(data, pitch, cols, dtype); }

bool bad_floats(const float *p) { return !p || misaligned(p, 4); }

// false if the description is not valid
bool drop_args(const conef_drop *drop, DropArgs &out)
{
    if (!(drop->p >= 0.0f && drop->p < 1.0f) || drop->site >= kMaxSites) return false;
    const uint32_t t = (uint32_t)std::floor((double)drop->p * 65536.0 + 0.5);
    out.threshold = t > 65535 ? 65535 : t;
    out.scale = (float)(65536.0 / (double)(65536 - out.threshold));
    out.draws = {kDropWord + drop->site, (uint32_t)drop->step, (uint32_t)(drop->step >> 32), (uint32_t)drop->seed,
                 (uint32_t)(drop->seed >> 32)};
    return true;
}

int dropout(const conef_drop *drop, int64_t rows, int64_t cols, int dtype, const void *x, int64_t x_pitch, const void *residual,
            int64_t residual_pitch, void *y, int64_t y_pitch, void *hip_stream)
{
    DropoutArgs a;
    if (!drop || !drop_args(drop, a.d) || bad_shape(rows, cols, dtype)) return CONEF_EINVAL;
    if (rows == 0) return CONEF_OK;
    if (bad_rows(x, x_pitch, cols, dtype) || bad_optional(residual, residual_pitch, cols, dtype) || bad_rows(y, y_pitch, cols, dtype))
        return CONEF_EINVAL;
    a.rows = rows;
    a.cols = (int)cols;
    a.x = {x, x_pitch};
    a.residual = {residual, residual_pitch};
    a.y = {y, y_pitch};
    launch_dropout(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

bool bad_packed(const void *codes, const void *scales) { return !codes || !scales || misaligned(codes, 16) || misaligned(scales, 16); }

// sides of a packed operand: below 2^30, and both turns of it have to be countable
bool bad_sides(int64_t rows, int64_t cols)
{
    return rows < 0 || cols < 0 || rows >= kMostSide / 2 || cols >= kMostSide / 2 || rows * ((cols + 7) / 8) >= (int64_t)1 << 32 ||
           cols * ((rows + 7) / 8) >= (int64_t)1 << 32;
}

}  // namespace

extern "C" {

int conef_dropout_forward(const conef_drop *drop, int64_t rows, int64_t cols, int dtype, const void *x, int64_t x_pitch,
                          const void *residual, int64_t residual_pitch, void *y, int64_t y_pitch, void *hip_stream)
{
    return dropout(drop, rows, cols, dtype, x, x_pitch, residual, residual_pitch, y, y_pitch, hip_stream);
}

int conef_dropout_backward(const conef_drop *drop, int64_t rows, int64_t cols, int dtype, const void *dy, int64_t dy_pitch, void *dx,
                           int64_t dx_pitch, void *hip_stream)
{
    return dropout(drop, rows, cols, dtype, dy, dy_pitch, nullptr, 0, dx, dx_pitch, hip_stream);
}

int conef_norm_forward(const conef_drop *drop, float eps, int64_t rows, int64_t cols, int dtype, const void *x, int64_t x_pitch,
                       const void *residual, int64_t residual_pitch, const float *gamma, const float *beta, void *z_out, int64_t z_pitch,
                       void *y, int64_t y_pitch, float *mean_out, float *rstd_out, void *hip_stream)
{
    NormArgs a;
    if (bad_shape(rows, cols, dtype) || !(eps >= 0.0f) || !std::isfinite(eps)) return CONEF_EINVAL;
    if (drop && !drop_args(drop, a.d)) return CONEF_EINVAL;
    if (rows == 0) return CONEF_OK;                                 // a matrix of no rows may have no address
    if ((drop || residual) && !z_out) return CONEF_EINVAL;          // the backward pass needs what the norm was taken of
    if (!drop && !residual && z_out) return CONEF_EINVAL;
    if (bad_rows(x, x_pitch, cols, dtype) || bad_optional(residual, residual_pitch, cols, dtype) ||
        bad_optional(z_out, z_pitch, cols, dtype) || bad_rows(y, y_pitch, cols, dtype) || bad_floats(gamma) || bad_floats(beta) ||
        misaligned(mean_out, 4) || misaligned(rstd_out, 4) || y == z_out)
        return CONEF_EINVAL;
    a.rows = rows;
    a.cols = (int)cols;
    a.drop = drop != nullptr;
    a.eps = eps;
    a.x = {x, x_pitch};
    a.residual = {residual, residual_pitch};
    a.z = {z_out, z_pitch};
    a.y = {y, y_pitch};
    a.gamma = gamma;
    a.beta = beta;
    a.mean_out = mean_out;
    a.rstd_out = rstd_out;
    launch_norm_forward(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int conef_norm_workspace(int64_t rows, int64_t cols, size_t *bytes)
{
    if (!bytes || bad_shape(rows, cols, CONEF_F32)) return CONEF_EINVAL;
    *bytes = (size_t)norm_partials(rows, cols) * 2 * (size_t)cols * sizeof(float);
    return CONEF_OK;
}

int conef_norm_backward(const conef_drop *drop, int64_t rows, int64_t cols, int dtype, const void *dy, int64_t dy_pitch, const void *z,
                        int64_t z_pitch, const float *gamma, const float *mean, const float *rstd, const void *dz_in,
                        int64_t dz_in_pitch, void *dz, int64_t dz_pitch, void *dx, int64_t dx_pitch, float *dgamma, float *dbeta,
                        void *workspace, void *hip_stream)
{
    NormArgs a;
    if (bad_shape(rows, cols, dtype)) return CONEF_EINVAL;
    if (drop && !drop_args(drop, a.d)) return CONEF_EINVAL;
    if (dx && !drop) return CONEF_EINVAL;                           // without a dropout dx is dz
    if (rows > 0 && !dz && !dx && !dgamma && !dbeta) return CONEF_EINVAL;
    if (misaligned(dgamma, 4) || misaligned(dbeta, 4)) return CONEF_EINVAL;
    const bool columns = dgamma || dbeta;
    if (rows > 0) {
        if (bad_rows(dy, dy_pitch, cols, dtype) || bad_rows(z, z_pitch, cols, dtype) || bad_floats(gamma) || bad_floats(mean) ||
            bad_floats(rstd) || bad_optional(dz_in, dz_in_pitch, cols, dtype) || bad_optional(dz, dz_pitch, cols, dtype) ||
            bad_optional(dx, dx_pitch, cols, dtype) || (dz && dz == dx))
            return CONEF_EINVAL;
        if (columns && (!workspace || misaligned(workspace, 16))) return CONEF_EINVAL;
    } else if (!columns) {
        return CONEF_OK;
    }
    a.rows = rows;
    a.cols = (int)cols;
    a.drop = drop != nullptr;
    a.dy = {dy, dy_pitch};
    a.z_in = {z, z_pitch};
    a.dz_in = {dz_in, dz_in_pitch};
    a.dz = {dz, dz_pitch};
    a.dx = {dx, dx_pitch};
    a.gamma = gamma;
    a.mean = mean;
    a.rstd = rstd;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.partials = columns ? static_cast<float *>(workspace) : nullptr;
    launch_norm_backward(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int conef_mx_sizes(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (bad_sides(rows, cols)) return CONEF_EINVAL;
    const size_t elements = (size_t)round_up(rows, 64) * (size_t)round_up(cols, 128);
    if (code_bytes) *code_bytes = elements / 2;
    if (scale_bytes) *scale_bytes = elements / 32;
    return CONEF_OK;
}

int conef_mx_quantise(const void *x, int64_t x_pitch, int64_t rows, int64_t cols, int dtype, int rounding, uint64_t seed, uint32_t site,
                      uint64_t step, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, void *hip_stream)
{
    if ((dtype != CONEF_F32 && dtype != CONEF_BF16) || bad_sides(rows, cols)) return CONEF_EINVAL;
    if ((rounding != CONEF_MX_NEAREST && rounding != CONEF_MX_STOCHASTIC) || site >= kMaxSites) return CONEF_EINVAL;
    if (rows == 0 || cols == 0) return CONEF_OK;
    if (!codes && !codes_t) return CONEF_EINVAL;
    if (bad_rows(x, x_pitch, cols, dtype)) return CONEF_EINVAL;
    if ((codes || scales) && bad_packed(codes, scales)) return CONEF_EINVAL;
    if ((codes_t || scales_t) && bad_packed(codes_t, scales_t)) return CONEF_EINVAL;
    MxQuantArgs a;
    a.rows = rows;
    a.cols = cols;
    a.x = {x, x_pitch};
    a.by_rows = {codes, scales};
    a.by_cols = {codes_t, scales_t};
    a.draws = {kMxRowWord + site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32)};
    a.stochastic = rounding == CONEF_MX_STOCHASTIC;
    launch_mx_quantise(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int conef_mx_dequantise(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out, int64_t out_pitch, int dtype,
                        void *hip_stream)
{
    if ((dtype != CONEF_F32 && dtype != CONEF_BF16) || bad_sides(rows, cols)) return CONEF_EINVAL;
    if (rows == 0 || cols == 0) return CONEF_OK;
    if (bad_packed(codes, scales) || bad_rows(out, out_pitch, cols, dtype)) return CONEF_EINVAL;
    MxDequantArgs a;
    a.rows = rows;
    a.cols = cols;
    a.in = {codes, scales};
    a.out = {out, out_pitch};
    launch_mx_dequantise(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int conef_mx_product_workspace(int64_t m, int64_t n, int64_t k, size_t *bytes)
{
    if (!bytes || bad_sides(m, n) || bad_sides(m, k) || bad_sides(n, k)) return CONEF_EINVAL;
    *bytes = mx_product_workspace(m, n, k);
    return CONEF_OK;
}

int conef_mx_product(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales, int64_t m,
                     int64_t n, int64_t k, float alpha, float beta, void *c, int64_t c_pitch, int dtype, void *workspace,
                     void *hip_stream)
{
    if ((dtype != CONEF_F32 && dtype != CONEF_BF16) || bad_sides(m, n) || bad_sides(m, k) || bad_sides(n, k)) return CONEF_EINVAL;
    if (m == 0 || n == 0) return CONEF_OK;
    if (bad_rows(c, c_pitch, n, dtype)) return CONEF_EINVAL;
    if (k > 0 && (bad_packed(a_codes, a_scales) || bad_packed(b_codes, b_scales))) return CONEF_EINVAL;
    const size_t room = mx_product_workspace(m, n, k);
    if (room && (!workspace || misaligned(workspace, 256))) return CONEF_EINVAL;
    MxProductArgs a;
    a.m = m;
    a.n = n;
    a.k = k;
    a.a = {a_codes, a_scales};
    a.b = {b_codes, b_scales};
    a.alpha = alpha;
    a.beta = beta;
    a.c = {c, c_pitch};
    a.partials = room ? static_cast<float *>(workspace) : nullptr;
    launch_mx_product(a, dtype == CONEF_BF16, static_cast<hipStream_t>(hip_stream));
    return launched();
}

}  // extern "C"
