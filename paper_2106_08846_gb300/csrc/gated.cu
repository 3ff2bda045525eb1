// The gated feed-forward block
//
//   G = X Wg' + bg,  U = X Wu' + bu,  H = act(G) * U
//
// and its backward pass, which computes G and U again:
//
//   dG = dH U act'(G),  dU = dH act(G)
//   dX = dG Wg + dU Wu,  dWg = dG' X,  dWu = dU' X,  dbg = sum dG,  dbu = sum dU
//
// in fp32 multiply-adds on 64 x 64 tiles staged through shared memory.
#include <algorithm>

#include "act.cuh"
#include "bsr_internal.h"
#include "elem.cuh"
#include "gated.h"
#include "launch.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

constexpr int T = 64, KS = 16;

// One operand element (r, k) at p[r * rs + k * ks].
template <typename E>
struct Operand {
    const E *p;
    int64_t rs, ks, rows;
};

// acc (+)= A B' for a 64 x 64 tile at (m0, n0); 256 threads, 4 x 4 values each.
template <typename A, typename B>
__device__ __forceinline__ void tile_product(float (&acc)[4][4], Operand<A> a, Operand<B> b, int64_t K, int64_t m0, int64_t n0) {
    __shared__ float as[KS][T + 1], bs[KS][T + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int64_t k0 = 0; k0 < K; k0 += KS) {
        __syncthreads();
        for (int e = threadIdx.x; e < T * KS; e += 256) {
            // neighbours along the contiguous side
            const int ra = a.ks == 1 ? e / KS : e % T, ka = a.ks == 1 ? e % KS : e / T;
            as[ka][ra] = m0 + ra < a.rows && k0 + ka < K ? to_f32(a.p[(m0 + ra) * a.rs + (k0 + ka) * a.ks]) : 0.f;
            const int rb = b.ks == 1 ? e / KS : e % T, kb = b.ks == 1 ? e % KS : e / T;
            bs[kb][rb] = n0 + rb < b.rows && k0 + kb < K ? to_f32(b.p[(n0 + rb) * b.rs + (k0 + kb) * b.ks]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < KS; k++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = fmaf(as[k][ty + 16 * i], bs[k][tx + 16 * j], acc[i][j]);
    }
}

template <typename E, bool BACK>
__global__ void __launch_bounds__(256) k_gated(const __grid_constant__ GatedCall c, float *dG, float *dU) {
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t n0 = (int64_t)blockIdx.y * T, f0 = (int64_t)blockIdx.x * T;
    float g[4][4] = {}, u[4][4] = {};
    const Operand<E> x{static_cast<const E *>(c.X), c.K, 1, c.N};
    tile_product(g, x, Operand<E>{static_cast<const E *>(c.Wg), c.K, 1, c.F}, c.K, n0, f0);
    tile_product(u, x, Operand<E>{static_cast<const E *>(c.Wu), c.K, 1, c.F}, c.K, n0, f0);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const int64_t n = n0 + ty + 16 * i, f = f0 + tx + 16 * j, at = n * c.F + f;
            if (n >= c.N || f >= c.F) continue;
            const float gv = g[i][j] + (c.bg ? c.bg[f] : 0.f), uv = u[i][j] + (c.bu ? c.bu[f] : 0.f);
            if constexpr (BACK) {
                const float d = to_f32(static_cast<const E *>(c.dH)[at]);
                const float2 a = activate_slope<false>(c.act, gv);
                dG[at] = d * uv * a.y;
                dU[at] = d * a.x;
            } else {
                static_cast<E *>(c.H)[at] = from_f32<E>(activate<false>(c.act, gv) * uv);
            }
        }
}

// out[m, n] = A0 B0' + A1 B1' (K columns each; A1.p may be NULL), row-major with n_cols columns
template <typename E>
__global__ void __launch_bounds__(256) k_product(Operand<float> a0, Operand<E> b0, Operand<float> a1, Operand<E> b1, int64_t K,
                                                 E *out) {
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t m0 = (int64_t)blockIdx.y * T, n0 = (int64_t)blockIdx.x * T;
    float acc[4][4] = {};
    tile_product(acc, a0, b0, K, m0, n0);
    if (a1.p) tile_product(acc, a1, b1, K, m0, n0);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < a0.rows && n < b0.rows) out[m * b0.rows + n] = from_f32<E>(acc[i][j]);
        }
}

// out[f] = sum over n of d[n, f], a column a thread
__global__ void __launch_bounds__(256) k_column_sums(const float *d, int64_t N, int64_t F, float *out) {
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t f = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (f >= F) return;
    float s = 0.f;
    for (int64_t n = 0; n < N; n++) s += d[n * F + f];
    out[f] = s;
}

unsigned tiles(int64_t n) { return (unsigned)((n + T - 1) / T); }

template <typename E>
cudaError_t forward(const GatedCall &c, cudaStream_t s) {
    return launch_kernel(k_gated<E, false>, dim3(tiles(c.F), tiles(c.N)), dim3(256), 0, s, c, (float *)nullptr, (float *)nullptr);
}

template <typename E>
cudaError_t backward(const GatedCall &c, cudaStream_t s) {
    float *dG = static_cast<float *>(c.ws), *dU = dG + c.N * c.F;
    const E *X = static_cast<const E *>(c.X), *Wg = static_cast<const E *>(c.Wg), *Wu = static_cast<const E *>(c.Wu);
    cudaError_t e = cudaSuccess;
    if (c.N > 0) e = launch_kernel(k_gated<E, true>, dim3(tiles(c.F), tiles(c.N)), dim3(256), 0, s, c, dG, dU);
    if (e == cudaSuccess && c.dX && c.N > 0)
        e = launch_kernel(k_product<E>, dim3(tiles(c.K), tiles(c.N)), dim3(256), 0, s, Operand<float>{dG, c.F, 1, c.N},
                          Operand<E>{Wg, 1, c.K, c.K}, Operand<float>{dU, c.F, 1, c.N}, Operand<E>{Wu, 1, c.K, c.K}, c.F,
                          static_cast<E *>(c.dX));
    for (int i = 0; i < 2; i++) {
        const float *d = i ? dU : dG;
        void *dW = i ? c.dWu : c.dWg;
        float *db = i ? c.dbu : c.dbg;
        if (e == cudaSuccess && dW)
            e = launch_kernel(k_product<E>, dim3(tiles(c.K), tiles(c.F)), dim3(256), 0, s, Operand<float>{d, 1, c.F, c.F},
                              Operand<E>{X, 1, c.K, c.K}, Operand<float>{nullptr, 1, 1, 0}, Operand<E>{nullptr, 1, 1, 0}, c.N,
                              static_cast<E *>(dW));
        if (e == cudaSuccess && db)
            e = launch_kernel(k_column_sums, dim3((unsigned)((c.F + 255) / 256)), dim3(256), 0, s, d, c.N, c.F, db);
    }
    return e;
}

}  // namespace

int64_t gated_workspace(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, bool backward) {
    return backward ? 2 * N * F * 4 : 0;
}

cudaError_t launch_gated(const GatedCall &c, cudaStream_t s) {
    return c.dt == BSR_F32 ? forward<float>(c, s) : forward<uint16_t>(c, s);
}

cudaError_t launch_gated_backward(const GatedCall &c, cudaStream_t s) {
    return c.dt == BSR_F32 ? backward<float>(c, s) : backward<uint16_t>(c, s);
}

}  // namespace bsr
