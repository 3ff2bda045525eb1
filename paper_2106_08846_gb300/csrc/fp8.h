// Operands and products in 8-bit floating point (fp8_*.cu): host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

constexpr int kFp8Block = 128;   // columns that share a scale

inline int64_t fp8_blocks(int64_t cols) { return (cols + kFp8Block - 1) / kFp8Block; }
inline int64_t fp8_scale_cols(const bsr_fp8_matrix_t &m) { return (m.rows + m.tile - 1) / m.tile; }
inline int64_t fp8_bytes(const bsr_fp8_matrix_t &m) { return m.batch * m.rows * fp8_blocks(m.cols) * kFp8Block; }
inline int64_t fp8_words(int64_t cols) { return (fp8_blocks(cols) + 3) / 4; }   // of four blocks' exponents
inline int64_t fp8_exponents(const bsr_fp8_matrix_t &m) { return m.batch * fp8_words(m.cols) * fp8_blocks(m.rows) * 512; }
inline int64_t fp8_scales(const bsr_fp8_matrix_t &m) { return m.batch * fp8_blocks(m.cols) * fp8_scale_cols(m); }

// x [batch, R, C] as `rows` [batch, R, C] and as `columns` [batch, C, R]; either may be NULL.
cudaError_t launch_fp8_quantize(const void *x, bsr_dtype_t dt, int64_t batch, int64_t R, int64_t C, int tile, bsr_fp8_t type,
                                const bsr_fp8_matrix_t *rows, const bsr_fp8_matrix_t *columns, const int32_t *used, cudaStream_t s);

struct Fp8Product {
    bsr_fp8_matrix_t a, b;
    const float *bias;
    void *Y;
    bsr_dtype_t dt;
    bsr_group_t group;
    const int32_t *offsets;
    int groups;
    float *ws;
};
int64_t fp8_product_workspace(const Fp8Product &p);
cudaError_t launch_fp8_product(const Fp8Product &p, cudaStream_t s);
// The first error that a kernel recorded on the current device since the last call; synchronises the device.
cudaError_t fp8_product_status(int *code);

}  // namespace bsr
