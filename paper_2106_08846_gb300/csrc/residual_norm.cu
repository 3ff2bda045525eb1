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
// row on its way at once. Wider rows are a group of threads', sixteen features each.
//
// What bounds it: DRAM (y and h in, h' and z out) and, with more parameters, L1, from
// which they are read. 16384 x 1024 bf16: one RMSNorm 21.4 us, 134 MB at 92% of the copy
// rate; two with a gate for 512 tokens 24.8 us, 80%; two LayerNorms with biases, a scale
// and a gate 34.7 us, 57%. 16384 x 768 fp32, LayerNorms with biases 41 us, 72%; 4096 x
// 4096 bf16, RMSNorms 26 us, 75%. One row of 1024: 2.5 us, the launch and one read's
// latency. Rows that are no runs of eight on 16-byte boundaries pay for shifting them
// into place and for stores of single words (5000 x 1193 bf16: one RMSNorm 17.5 us, 40%,
// two LayerNorms with biases, scale and gate 32 us, 22%; 16384 x 1023 fp32 72% and 46%).
#include <algorithm>
#include <type_traits>

#include "launch.cuh"
#include "residual_norm.cuh"

namespace bsr {

namespace {

// ROWS: rows at a time. The parameters come from L1, for each row again, as many bytes
// as y and h and more (one of 1024 values costs 2 us in 16384 rows); for two rows at a
// time half as often, and a sum's barrier or shuffles serve both. WARP: a warp to a
// row. Rows `ahead` further on are asked for into L2: registers hold too few loads to
// keep DRAM busy (16384 x 1024 bf16: 25.9 us without, 25.1 with). THREADS: the most of
// a CTA; CTAS: so many to an SM.
template <typename TB, typename TS, int V, int L, bool WARP, int ROWS, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) k_residual_norm(const __grid_constant__ RnForward a, int64_t ahead) {
    __shared__ float4 words[WARP ? 1 : kMaxGroups][64];
    const int t = threadIdx.x, NT = WARP ? 32 : blockDim.x, D = (int)a.p.D;
    const float over_d = 1.f / (float)D;
    GroupSum<WARP> sum{words[WARP ? 0 : threadIdx.y], NT, (int)threadIdx.y, 0};
    if (!WARP) sum.init();
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t n = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * ROWS; n < a.N; n += (int64_t)gridDim.x * blockDim.y * ROWS) {
        Run x[ROWS][V];
        Raw<TS, L> h[ROWS][V];
        // (past the last row: that row once more, which nothing is stored of)
        auto row_of = [&](int k) { return ROWS == 1 ? n : min(n + k, a.N - 1); };
        {
            Raw<TB, L> y[ROWS][V];
#pragma unroll
            for (int k = 0; k < ROWS; k++)
#pragma unroll
                for (int i = 0; i < V; i++) y[k][i] = load_run<TB, L, false>(static_cast<const TB *>(a.y) + row_of(k) * D, D, i, t, NT, row_at_end<L>(a.N - 1 - row_of(k), D));
            if (a.h) {
#pragma unroll
                for (int k = 0; k < ROWS; k++)
#pragma unroll
                    for (int i = 0; i < V; i++) h[k][i] = load_run<TS, L, false>(static_cast<const TS *>(a.h) + row_of(k) * D, D, i, t, NT, row_at_end<L>(a.N - 1 - row_of(k), D));
            }
            if (n + ahead < a.N) {
                const int64_t at = (n + ahead) * D;
                const int rows = (int)min((int64_t)ROWS, a.N - n - ahead);
                for (int e = t * 128; e < rows * D * (int)sizeof(TB); e += NT * 128) ptx::prefetch_l2(static_cast<const char *>(a.y) + at * sizeof(TB) + e);
                if (a.h)
                    for (int e = t * 128; e < rows * D * (int)sizeof(TS); e += NT * 128) ptx::prefetch_l2(static_cast<const char *>(a.h) + at * sizeof(TS) + e);
            }
#pragma unroll
            for (int k = 0; k < ROWS; k++)
#pragma unroll
                for (int i = 0; i < V; i++) x[k][i] = y[k][i].run();
        }
        if (a.p.post != BSR_NORM_NONE) {
            normalise<V, L>(x, a.p.post, a.p.post_eps, D, over_d, t, NT, sum);
            affine<V, L>(x, a.p.post_w, a.p.post_b, D, t, NT);
        }
        if (a.gate) {
            const TB *gate = static_cast<const TB *>(a.gate);
            // (a division of 64 bits takes more instructions than a row's other arithmetic)
            auto gate_of = [&](int64_t row) {
                return a.N >> 32 ? row / a.p.gate_tokens : (int64_t)((uint32_t)row / (uint32_t)a.p.gate_tokens);
            };
            const int64_t gates = L == ANY ? gate_of(a.N - 1) + 1 : 0;   // the gate's rows
            const int64_t first = gate_of(row_of(0)), last = ROWS == 1 ? first : gate_of(row_of(ROWS - 1));
#pragma unroll
            for (int i = 0; i < V; i++) {
                const Run p = load_gate<TB, L>(gate + first * D, D, i, t, NT, row_at_end<L>(gates - 1 - first, D));
                times(x[0][i], p);
                if (ROWS == 2)
                    times(x[ROWS - 1][i], last == first ? p : load_gate<TB, L>(gate + last * D, D, i, t, NT, row_at_end<L>(gates - 1 - last, D)));
            }
        }
        affine<V, L>(x, a.p.scale, nullptr, D, t, NT);
        if (a.h) {
#pragma unroll
            for (int k = 0; k < ROWS; k++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const Run hr = h[k][i].run();
#pragma unroll
                    for (int j = 0; j < 4; j++) x[k][i].v[j] = fma2(all2(a.p.alpha), hr.v[j], x[k][i].v[j]);
                }
        }
        auto store = [&](auto *to) {
#pragma unroll
            for (int k = 0; k < ROWS; k++) {
                if (ROWS > 1 && n + k >= a.N) break;
#pragma unroll
                for (int i = 0; i < V; i++) store_run<std::remove_pointer_t<decltype(to)>, L, THREADS / 32>(to + (n + k) * D, D, i, t, NT, x[k][i]);
            }
        };
        if (a.h_out) store(static_cast<TS *>(a.h_out));
        if (a.p.pre != BSR_NORM_NONE) {
            normalise<V, L>(x, a.p.pre, a.p.pre_eps, D, over_d, t, NT, sum);
            affine<V, L>(x, a.p.pre_w, a.p.pre_b, D, t, NT);
            store(static_cast<TB *>(a.z));
        }
    }
}

// CTAs of R groups of NT threads.
template <typename TB, typename TS, int V, bool WARP, int ROWS, int THREADS, int CTAS>
cudaError_t launch(const RnForward &a, int NT, int R, int64_t ahead, cudaStream_t s) {
    const int L = layout_of(a.p, V, NT);
    const dim3 block(NT, R), grid((unsigned)std::min<int64_t>((a.N + R * ROWS - 1) / (R * ROWS), INT32_MAX));
    auto kernel = L == FULL   ? k_residual_norm<TB, TS, V, FULL, WARP, ROWS, THREADS, CTAS>
                  : L == RUNS ? k_residual_norm<TB, TS, V, RUNS, WARP, ROWS, THREADS, CTAS>
                              : k_residual_norm<TB, TS, V, ANY, WARP, ROWS, THREADS, CTAS>;
    return launch_kernel(kernel, grid, block, 0, s, a, ahead);
}

// Parameters' rows that are read for each row.
int params_of(const RnForward &a) {
    return (a.p.post_w != nullptr) + (a.p.post_b != nullptr) + (a.p.pre_w != nullptr) + (a.p.pre_b != nullptr) + (a.p.scale != nullptr) +
           (a.gate != nullptr);
}

// Two rows at a time pay from three parameters on (16384 x 768 bf16, RMSNorms with
// their weights: 17.6 us so and one by one; with a scale 18.7 and 19.9; LayerNorms with
// biases, scale and gate 24.9 and 27.4), if they leave all SMs work.
template <typename TB, typename TS, int V>
cudaError_t forward_warps(const RnForward &a, cudaStream_t s) {
    const int sms = sm_count();
    constexpr int most = V == 1 ? 8 : V < 4 ? 4 : 2, size = sizeof(TS);
    // as many rows to a CTA as leave all SMs some
    const int R = (int)std::max<int64_t>(1, std::min<int64_t>(most, a.N / (4 * sms)));
    const int64_t ahead = (int64_t)sms * 24;   // (about the rows that run at once)
    if constexpr (size * V <= 6) {   // (more do not fit the registers: 16384 x 1024 bf16 36.1 us, one by one 35.0)
        if (params_of(a) >= 3 && a.N >= 32 * sms) return launch<TB, TS, V, true, 2, 256, size * V <= 2 ? 4 : size * V <= 4 ? 3 : 2>(a, 32, most, ahead, s);
    }
    return launch<TB, TS, V, true, 1, 256, V < 3 ? 4 : size == 2 ? 3 : 2>(a, 32, R, ahead, s);
}

template <typename TB, typename TS>
cudaError_t forward_groups(const RnForward &a, cudaStream_t s) {
    constexpr int V = 2;
    const int sms = sm_count(), NT = (int)((a.p.D + 8 * V - 1) / (8 * V) + 31) / 32 * 32, R = std::max(1, std::min(kMaxGroups, 256 / NT));
    const int64_t ahead = (int64_t)sms * std::max(1, 1024 / NT);
    // (fp32 streams: with the registers that CTAs of 512 threads leave they also need fewer
    // spills; 6000 x 2560, RMSNorms on an fp32 stream 32.1 us, one by one 36.2)
    if (NT <= 512 && (sizeof(TS) == 4 || params_of(a) >= 3) && a.N >= 4 * R * sms) return launch<TB, TS, V, false, 2, 512, 1>(a, NT, R, ahead, s);
    return launch<TB, TS, V, false, 1, 1024, 1>(a, NT, R, ahead, s);
}

template <typename TB, typename TS>
cudaError_t forward(const RnForward &a, cudaStream_t s) {
    const int64_t D = a.p.D;
    if (D <= 256) return forward_warps<TB, TS, 1>(a, s);
    if (D <= 512) return forward_warps<TB, TS, 2>(a, s);
    if (D <= 768) return forward_warps<TB, TS, 3>(a, s);
    if (D <= 1024) return forward_warps<TB, TS, 4>(a, s);
    return forward_groups<TB, TS>(a, s);
}

}  // namespace

cudaError_t launch_residual_norm(const RnForward &a, cudaStream_t s) {
    if (a.N == 0) return cudaSuccess;
    RnForward b = a;
    b.p.gate_tokens = std::min(b.p.gate_tokens, b.N);   // (as few bits as N)
    if (b.p.block_dt == BSR_F32) return forward<float, float>(b, s);
    return b.p.stream_dt == BSR_F32 ? forward<uint16_t, float>(b, s) : forward<uint16_t, uint16_t>(b, s);
}

}  // namespace bsr
