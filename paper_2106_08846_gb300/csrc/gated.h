// The gated feed-forward block (gated*.cu): host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

struct GatedCall {
    const void *X, *Wg, *Wu;
    const float *bg, *bu;
    int64_t N, F, K;
    bsr_dtype_t dt;
    bsr_act_t act;
    void *ws;
    void *H;                          // forward
    const void *dH;                   // backward
    void *dX, *dWg, *dWu;
    float *dbg, *dbu;
};

// Bytes of GatedCall::ws.
int64_t gated_workspace(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, bool backward);
// Forward for up to kGatedFew tokens, without a workspace (gated_few.cu).
constexpr int64_t kGatedFew = 32;
cudaError_t launch_gated_few(const GatedCall &c, cudaStream_t s);
cudaError_t launch_gated(const GatedCall &c, cudaStream_t s);
cudaError_t launch_gated_backward(const GatedCall &c, cudaStream_t s);

}  // namespace bsr
