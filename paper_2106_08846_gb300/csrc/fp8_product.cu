// Products of 8-bit operands: Y = a b' + bias, sums over blocks of 128 with a scale each.
#include <cuda_fp8.h>

#include <algorithm>

#include "elem.cuh"
#include "fp8.h"
#include "launch.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

__device__ __forceinline__ float value_of(uint8_t q, int type) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(q, type == BSR_E5M2 ? __NV_E5M2 : __NV_E4M3)));
}

template <typename T>
__global__ void __launch_bounds__(256) k_fp8_product(const __grid_constant__ Fp8Product p, int64_t KB) {
    const int64_t m = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31), n = (int64_t)blockIdx.y * 8 + (threadIdx.x >> 5), ld = KB * kFp8Block;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    if (m >= p.b.rows || n >= p.a.rows) return;
    int64_t b0 = 0, b1 = KB, batch = 0, out = n * p.b.rows + m;
    if (p.group == BSR_GROUP_ROWS) {
        int e = 0;
        while (e < p.groups && !(n >= p.offsets[e] && n < p.offsets[e + 1])) e++;
        if (e == p.groups) return;
        batch = e;
    } else if (p.group == BSR_GROUP_COLUMNS) {
        b0 = min(KB, (int64_t)max(0, p.offsets[blockIdx.z]) / kFp8Block), b1 = min(KB, (int64_t)max(0, p.offsets[blockIdx.z + 1]) / kFp8Block);
        out += blockIdx.z * p.a.rows * p.b.rows;
    }
    const int64_t a_cols = (p.a.rows + p.a.tile - 1) / p.a.tile, b_cols = (p.b.rows + p.b.tile - 1) / p.b.tile;
    const uint8_t *qa = static_cast<const uint8_t *>(p.a.q) + n * ld, *qb = static_cast<const uint8_t *>(p.b.q) + (batch * p.b.rows + m) * ld;
    float sum = 0.f;
    for (int64_t b = b0; b < b1; b++) {
        float t = 0.f;
        for (int k = 0; k < kFp8Block; k++)
            t = fmaf(value_of(qa[b * kFp8Block + k], p.a.type), value_of(qb[b * kFp8Block + k], p.b.type), t);
        sum = fmaf(t, p.a.scale[b * a_cols + n / p.a.tile] * p.b.scale[(batch * KB + b) * b_cols + m / p.b.tile], sum);
    }
    if (p.bias) sum += p.bias[batch * p.b.rows + m];
    static_cast<T *>(p.Y)[out] = from_f32<T>(sum);
}

}  // namespace

int64_t fp8_product_workspace(const Fp8Product &) { return 0; }

cudaError_t launch_fp8_product(const Fp8Product &p, cudaStream_t s) {
    const int64_t gx = (p.b.rows + 31) / 32, gy = (p.a.rows + 7) / 8, gz = p.group == BSR_GROUP_COLUMNS ? p.groups : 1;
    if (gx > INT32_MAX || gy > 65535 || gz > 65535) return cudaErrorInvalidConfiguration;
    auto kernel = p.dt == BSR_F32 ? k_fp8_product<float> : k_fp8_product<uint16_t>;
    return launch_kernel(kernel, dim3((unsigned)gx, (unsigned)gy, (unsigned)gz), dim3(256), 0, s, p, fp8_blocks(p.a.cols));
}

cudaError_t fp8_product_status(int *code) {
    *code = 0;
    return cudaSuccess;
}

}  // namespace bsr
