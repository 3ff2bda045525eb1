// The residual step between two blocks of a transformer layer, one pass over
// the data (backward: residual_norm_backward.cu).
//
//   t  = post(y);  h' = alpha h + s * gate * t;  z = pre(h')
//
// with post and pre a LayerNorm, an RMSNorm or nothing. A row of D features is
// held in registers from its only read on; means and deviations are sums over the
// threads that hold it, the deviation from the centred row, all in fp32. z is made
// from h' before h' is rounded. Arithmetic is on pairs of features.
//
// Forward, up to 1024 features a row is one warp's: no barriers, every load of the
// row on its way at once. Wider rows are a group of threads', eight or sixteen
// features each.
//
// What bounds it: DRAM (y and h in, h' and z out): 16384 x 1024 bf16 with a gate for
// 512 tokens 25 us, 134 MB at 79% of the copy rate; 16384 x 768 fp32 41 us, 201 MB at
// 72%; 4096 x 4096 bf16 33 us. One row of 1024: 2.6 us, the launch and one read's
// latency. Rows that are no runs of eight on 16-byte boundaries pay for shifting them
// into place and for stores of single words (16384 x 1193 bf16: 21% of the copy rate).
#include <algorithm>

#include "launch.cuh"
#include "residual_norm.cuh"

namespace bsr {

namespace {

// WARP: a warp to a row. Rows `ahead` further on are asked for into L2: registers
// hold too few loads to keep DRAM busy (16384 x 1024 bf16: 25.9 us without, 25.1 with).
template <typename TB, typename TS, int V, int L, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024, WARP ? (V < 3 ? 4 : sizeof(TS) == 2 ? 3 : 2) : 1)
k_residual_norm(const __grid_constant__ RnForward a, int64_t ahead) {
    __shared__ float4 words[WARP ? 1 : kMaxGroups][64];
    const int t = threadIdx.x, NT = WARP ? 32 : blockDim.x, D = (int)a.p.D;
    const float over_d = 1.f / (float)D;
    GroupSum<WARP> sum{words[WARP ? 0 : threadIdx.y], NT, (int)threadIdx.y, 0};
    if (!WARP) sum.init();
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t n = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; n < a.N; n += (int64_t)gridDim.x * blockDim.y) {
        Run x[V];
        Raw<TS, L> h[V];
        {
            Raw<TB, L> y[V];
#pragma unroll
            for (int i = 0; i < V; i++) y[i] = load_run<TB, L, false>(static_cast<const TB *>(a.y) + n * D, D, i, t, NT);
            if (a.h) {
#pragma unroll
                for (int i = 0; i < V; i++) h[i] = load_run<TS, L, false>(static_cast<const TS *>(a.h) + n * D, D, i, t, NT);
            }
            if (n + ahead < a.N) {
                const int64_t at = (n + ahead) * D;
                for (int e = t * 128; e < D * (int)sizeof(TB); e += NT * 128) ptx::prefetch_l2(static_cast<const char *>(a.y) + at * sizeof(TB) + e);
                if (a.h)
                    for (int e = t * 128; e < D * (int)sizeof(TS); e += NT * 128) ptx::prefetch_l2(static_cast<const char *>(a.h) + at * sizeof(TS) + e);
            }
#pragma unroll
            for (int i = 0; i < V; i++) x[i] = y[i].run();
        }
        if (a.p.post != BSR_NORM_NONE) {
            normalise<V, L>(x, a.p.post, a.p.post_eps, D, over_d, t, NT, sum);
            affine<V, L>(x, a.p.post_w, a.p.post_b, D, t, NT);
        }
        if (a.gate) {
            const TB *gate = static_cast<const TB *>(a.gate) + n / a.p.gate_tokens * D;
#pragma unroll
            for (int i = 0; i < V; i++) {
                const Run p = load_const<TB, L>(gate, D, i, t, NT);
#pragma unroll
                for (int j = 0; j < 4; j++) x[i].v[j] = mul2(x[i].v[j], p.v[j]);
            }
        }
        affine<V, L>(x, a.p.scale, nullptr, D, t, NT);
        if (a.h) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const Run hr = h[i].run();
#pragma unroll
                for (int j = 0; j < 4; j++) x[i].v[j] = fma2(all2(a.p.alpha), hr.v[j], x[i].v[j]);
            }
        }
        if (a.h_out) {
#pragma unroll
            for (int i = 0; i < V; i++) store_run<TS, L>(static_cast<TS *>(a.h_out) + n * D, D, i, t, NT, x[i]);
        }
        if (a.p.pre != BSR_NORM_NONE) {
            normalise<V, L>(x, a.p.pre, a.p.pre_eps, D, over_d, t, NT, sum);
            affine<V, L>(x, a.p.pre_w, a.p.pre_b, D, t, NT);
#pragma unroll
            for (int i = 0; i < V; i++) store_run<TB, L>(static_cast<TB *>(a.z) + n * D, D, i, t, NT, x[i]);
        }
    }
}

template <typename TB, typename TS, int V>
cudaError_t forward_warps(const RnForward &a, cudaStream_t s) {
    const int sms = sm_count();
    // as many rows to a CTA as leave all SMs some
    const int R = (int)std::max<int64_t>(1, std::min<int64_t>(V == 1 ? 8 : V < 4 ? 4 : 2, a.N / (4 * sms))), L = layout_of(a.p, V, 32);
    const dim3 block(32, R), grid((unsigned)std::min<int64_t>((a.N + R - 1) / R, INT32_MAX));
    auto kernel = L == FULL   ? k_residual_norm<TB, TS, V, FULL, true>
                  : L == RUNS ? k_residual_norm<TB, TS, V, RUNS, true>
                              : k_residual_norm<TB, TS, V, ANY, true>;
    return launch_kernel(kernel, grid, block, 0, s, a, (int64_t)sms * 24);   // (about the rows that run at once)
}

template <typename TB, typename TS, int V>
cudaError_t forward_groups(const RnForward &a, cudaStream_t s) {
    const int NT = (int)((a.p.D + 8 * V - 1) / (8 * V) + 31) / 32 * 32, R = std::max(1, std::min(kMaxGroups, 256 / NT)), L = layout_of(a.p, V, NT);
    const dim3 block(NT, R), grid((unsigned)std::min<int64_t>((a.N + R - 1) / R, INT32_MAX));
    auto kernel = L == FULL   ? k_residual_norm<TB, TS, V, FULL, false>
                  : L == RUNS ? k_residual_norm<TB, TS, V, RUNS, false>
                              : k_residual_norm<TB, TS, V, ANY, false>;
    return launch_kernel(kernel, grid, block, 0, s, a, (int64_t)sm_count() * std::max(1, 1024 / NT));
}

template <typename TB, typename TS>
cudaError_t forward(const RnForward &a, cudaStream_t s) {
    const int64_t D = a.p.D;
    if (D <= 256) return forward_warps<TB, TS, 1>(a, s);
    if (D <= 512) return forward_warps<TB, TS, 2>(a, s);
    if (D <= 768) return forward_warps<TB, TS, 3>(a, s);
    if (D <= 1024) return forward_warps<TB, TS, 4>(a, s);
    return forward_groups<TB, TS, 2>(a, s);
}

}  // namespace

cudaError_t launch_residual_norm(const RnForward &a, cudaStream_t s) {
    if (a.N == 0) return cudaSuccess;
    if (a.p.block_dt == BSR_F32) return forward<float, float>(a, s);
    return a.p.stream_dt == BSR_F32 ? forward<uint16_t, float>(a, s) : forward<uint16_t, uint16_t>(a, s);
}

}  // namespace bsr
