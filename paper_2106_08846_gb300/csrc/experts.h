// Rows sorted by expert and added up again (experts.cu): host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsr.h"

namespace bsr {

constexpr int kMostExperts = 1024, kMostChoices = 64, kMostAlign = 1024;

cudaError_t launch_expert_order(const bsr_experts_t &p, const int32_t *experts, cudaStream_t s);
// Xs from X; and the same rows of dY as the gradient of a sum without weights.
cudaError_t launch_expert_rows(const bsr_experts_t &p, const void *X, void *Xs, int64_t D, bsr_dtype_t dt, cudaStream_t s);
cudaError_t launch_expert_sum(const bsr_experts_t &p, const void *Ys, const float *weights, void *Y, int64_t D, bsr_dtype_t dt,
                              cudaStream_t s);
cudaError_t launch_expert_sum_backward(const bsr_experts_t &p, const void *Ys, const float *weights, const void *dY, void *dYs,
                                       float *dweights, int64_t D, bsr_dtype_t dt, cudaStream_t s);

}  // namespace bsr
