// Launch interface between the C ABI (layers.cpp) and the kernels of a training step's own operators: dropout and layer
// norm (kernels_norm.hip), quantisation to microscaled 4-bit floating point (kernels_mx.hip) and the product of two operands
// in that format (kernels_mx_product.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace conef {

// second counter word of the draws, plus the caller's site (< kMaxSites): apart from every matrix index and from each other
constexpr uint32_t kDropWord = 0xC0000000u, kMxRowWord = 0xC8000000u, kMxColWord = 0xD0000000u, kMaxSites = 1u << 27;

struct Draws {
    uint32_t word = 0, step_lo = 0, step_hi = 0, seed_lo = 0, seed_hi = 0;
};

// An element is kept iff its 16-bit draw is at least `threshold`; scale = fl32(65536 / (65536 - threshold)).
struct DropArgs {
    Draws draws;
    uint32_t threshold = 0;
    float scale = 1.0f;
};

// rows x cols elements with `pitch` elements from one row to the next
struct Rows {
    const void *data = nullptr;
    int64_t pitch = 0;
};
struct RowsOut {
    void *data = nullptr;
    int64_t pitch = 0;
};

struct NormArgs {
    int64_t rows = 0;
    int cols = 0;
    int drop = 0;               // the dropout is there
    float eps = 0.0f;
    DropArgs d;
    // forward: x (and residual) in, z (their sum) and y out; backward: dy, z (and dz_in) in, dz (and dx) out
    Rows x, residual, dy, z_in, dz_in;
    RowsOut z, y, dz, dx;
    const float *gamma = nullptr, *beta = nullptr, *mean = nullptr, *rstd = nullptr;
    float *mean_out = nullptr, *rstd_out = nullptr, *dgamma = nullptr, *dbeta = nullptr, *partials = nullptr;
};

struct DropoutArgs {
    int64_t rows = 0;
    int cols = 0;
    DropArgs d;
    Rows x, residual;
    RowsOut y;
};

void launch_dropout(const DropoutArgs &a, bool bf16, hipStream_t st);
void launch_norm_forward(const NormArgs &a, bool bf16, hipStream_t st);
void launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t st);
int64_t norm_partials(int64_t rows, int64_t cols);      // rows of partial sums of dgamma and dbeta (2 cols floats each)

// Packed operand: rows in 64s, columns in 128s (`pieces` of them).  Codes: pieces of 16 rows x 128 columns, 1024 bytes, byte
// (block % 4) * 256 + (row % 16) * 16 + (col % 32) / 2; scales: pieces of 64 rows x 4 blocks, 256 bytes, byte
// (block % 4) * 64 + (row % 16) * 4 + (row % 64) / 16; pieces of a row group one after the other.
struct MxOut {
    uint8_t *codes = nullptr, *scales = nullptr;
};
struct MxIn {
    const uint8_t *codes = nullptr, *scales = nullptr;
};

struct MxQuantArgs {
    int64_t rows = 0, cols = 0;
    Rows x;
    MxOut by_rows, by_cols;
    Draws draws;                // word: kMxRowWord + site
    int stochastic = 0;
};

struct MxDequantArgs {
    int64_t rows = 0, cols = 0;
    MxIn in;
    RowsOut out;
};

struct MxProductArgs {
    int64_t m = 0, n = 0, k = 0;
    MxIn a, b;
    float alpha = 1.0f, beta = 0.0f;
    RowsOut c;
    float *partials = nullptr;
};

void launch_mx_quantise(const MxQuantArgs &a, bool bf16, hipStream_t st);
void launch_mx_dequantise(const MxDequantArgs &a, bool bf16, hipStream_t st);
void launch_mx_product(const MxProductArgs &a, bool bf16, hipStream_t st);
size_t mx_product_workspace(int64_t m, int64_t n, int64_t k);

}  // namespace conef
