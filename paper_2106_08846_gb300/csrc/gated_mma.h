// The products of the gated block on the tensor cores (gated_mma.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

enum GatedMode : int {
    GM_FORWARD = 0,    // H = act(G) * U
    GM_BACKWARD = 1,   // dG, dU (and sums of them over runs of tokens) from G, U and dH
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
    Planes a, b0, b1;         // gated modes: Wg and Wu in b0 and b1, of whole groups of 32 rows (zeros past N)
    // GM_PRODUCT: B is stored [K, N], N contiguous; with a_side A is stored [K, M], M contiguous. Else [M, K], [N, K].
    bool a_side;
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
    float *sums;              // of sum_rows rows of dG and dU each, [.., 2 Fp] (an even count of 16s), or NULL
    // GM_PRODUCT: rows below row_seam go to out0, those from it on to out1, `out_rows` in each
    void *out0, *out1;
    int64_t row_seam, out_rows;
};

struct GatedShape {
    int steps, splits;               // of a tile: steps, and the parts of one that is not whole
    int64_t tiles_n, tiles, whole;   // tiles along N; all; the first ones, which are not split
};
// How products run: the tile width, their order, and which tiles have their K
// split into how many parts.
struct GatedPlan {
    int jobs, half;
    bool drained;                    // accumulators are added up in registers
    int order[2];                    // shape[i] is g[order[i]]'s
    GatedShape shape[2];
    int64_t units, part_bytes;
    float *parts;                    // part_bytes of workspace
};

// Rows of GatedMma::sums: one for so many rows of dG and dU.
inline int sum_rows(const GatedPlan &p) { return p.half == 128 || (p.drained && p.half == 64) ? 32 : 16; }

// The plan of g, or of two GM_PRODUCTs (as many parts each) in one launch, from
// the modes and sizes, with at most so many part_bytes.
GatedPlan plan_gated_mma(const GatedMma *g, int n, int64_t most_bytes);
// dbg and dbu from GM_BACKWARD's sums (NULL: not wanted): `rows` of them.
struct GatedBias {
    const float *sums = nullptr;
    int64_t rows = 0, F = 0, Fp = 0;
    float *dbg = nullptr, *dbu = nullptr;
};
// Runs them; GM_PRODUCTs also the biases' gradients, in their last launch.
cudaError_t launch_gated_mma(const GatedMma *g, const GatedPlan &p, cudaStream_t s, const GatedBias &b = GatedBias());
cudaError_t launch_gated_bias(const GatedBias &b, cudaStream_t s);

// The first error that a kernel of this file recorded on the current device
// since the last call; synchronises the device.
cudaError_t gated_mma_status(int *code);

}  // namespace bsr
