// The residual step between two blocks (residual_norm.cu): host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

constexpr int64_t kRnMaxD = 16384;   // a row is held in the registers of at most 1024 threads

struct RnForward {
    bsr_residual_norm_t p;
    const void *y, *h, *gate;
    void *h_out, *z;
    int64_t N;
};

struct RnBackward {
    bsr_residual_norm_t p;
    const void *y, *h_out, *gate, *dh_out, *dz;
    void *dy, *dh;
    bsr_residual_norm_grads_t g;
    int64_t N;
    float *ws;
};

cudaError_t launch_residual_norm(const RnForward &a, cudaStream_t s);
cudaError_t launch_residual_norm_backward(const RnBackward &a, cudaStream_t s);
// Bytes of RnBackward::ws.
int64_t residual_norm_workspace(const bsr_residual_norm_t &p, int64_t N);

}  // namespace bsr
