// The products of the gated block on the tensor cores (gated_mma.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

enum GatedMode : int {
    GM_FORWARD = 0,    // H = act(G) * U
    GM_BACKWARD = 1,   // dG, dU (and sums of them over 32 tokens) from G, U and dH
    GM_PRODUCT = 2,    // a plain product: dX; dWg and dWu
};

// A bf16 matrix of `rows` x `cols` values, `ld` apart, in `planes` parts whose
// sum it is (3 for fp32; bf16 1, or 2 for an A of 16 bits' precision).
struct Planes {
    const uint16_t *p;
    int64_t rows, cols, ld;
    int planes;
};

struct GatedMma {
    int mode;
    bsr_dtype_t dt;           // of the outputs and dH
    Planes a, b0, b1;
    bool a_side, b_side;      // the operand is stored [K, M] (or [K, N]), M (or N) contiguous; else [M, K]
    int64_t M, N, K;          // sizes of the product; gated modes: M tokens, N features
    int64_t b_seam;           // GM_PRODUCT: from this k on, the columns of A meet b1 (0: b0 only)
    // gated modes
    const float *bg, *bu;
    bsr_act_t act;
    const void *dH;
    void *H;
    int d_planes;
    uint16_t *D;              // d_planes of [M, 2 Fp]: dG, then dU from column Fp on
    int64_t Fp;
    float *sums;              // [ceil(M / 32), 2 Fp], or NULL
    // GM_PRODUCT: rows below row_seam go to out0, those from it on to out1, `out_rows` in each
    void *out0, *out1;
    int64_t row_seam, out_rows;
    float *parts;             // part_bytes
    // chosen by plan_gated_mma
    int half, steps, splits;
    int64_t tiles, tiles_n, whole, part_bytes;
};

// Chooses, from the sizes, the tile width, the steps of a tile and, for
// GM_PRODUCT, which tiles have their K split into how many parts.
void plan_gated_mma(GatedMma &g);
cudaError_t launch_gated_mma(const GatedMma &g, cudaStream_t s);

// The first error that a kernel of this file recorded on the current device
// since the last call; synchronises the device.
cudaError_t gated_mma_status(int *code);

}  // namespace bsr
