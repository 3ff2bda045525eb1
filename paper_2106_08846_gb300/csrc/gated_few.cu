// The gated feed-forward block for a few tokens (single tokens of a served
// request): reading the weights is the work.
//
// A lane reads 16 contiguous bytes of a weight row at a time, four lanes 64 bytes,
// the eight warps of a CTA in turn along K; the weights go from memory to registers
// as they lie. The warps add their sums through shared memory, in a fixed order.
//
// bf16: a warp takes eight features, an MMA's sixteen rows being their rows of Wg
// and of Wu, so that a thread finds G and U of a feature side by side; its eight
// columns are tokens. The 16 bytes of a lane hold its part of two MMAs: which
// columns of K meet in one is free, as long as weights and activations agree.
// fp32: likewise, values split into the three bf16 parts whose sum they are, and a product
// as the six part products that are not below 2^-24 of it; one token or two by
// multiply-adds, two columns of K to an instruction and four lanes to a feature. (768 into
// 2048: one token 4.5 us, two 4.7, by parts 7.3. Three and four tokens by multiply-adds
// 6.3 there, 8.4 against 8.9 for 1024 into 4096, and 8.4 against 7.9 for 770 into 1000.)
//
// What bounds it: DRAM, and for small weights the time of a launch and of one read.
// 1024 into 4096, bf16: 1 to 8 tokens 4.5 us (16.8 MB, 2.5 us at the copy rate), 16
// tokens 6.2, 32 tokens 7.8 (the products' own kernel 9.7); fp32: 1 token 6.6 us
// (33.6 MB, 5.0 us), 3 to 8 tokens 9.0, 32 tokens 17.6 (30.6). Four CTAs to an SM, so that
// all of them run at once: three took 0.3 us more.
#include <algorithm>

#include "act.cuh"
#include "bsr_internal.h"
#include "elem.cuh"
#include "gated.h"
#include "launch.cuh"
#include "parts.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

constexpr int kWarps = 8;
constexpr int kAhead = 4;   // 16-byte reads of either weight on their way at a time

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The parts of four fp32 values, in pairs (p[k]: part k of both pairs).
__device__ __forceinline__ void split(const uint4 &v, uint32_t (&p)[3][2]) {
    uint32_t a[3], b[3];
    parts_of(__uint_as_float(v.x), __uint_as_float(v.y), a);
    parts_of(__uint_as_float(v.z), __uint_as_float(v.w), b);
#pragma unroll
    for (int k = 0; k < 3; k++) p[k][0] = a[k], p[k][1] = b[k];
}

// 16 bytes of a row from column k on; where CHECK, 0 past column K. Rows start on
// 16-byte boundaries (and K is a multiple of 16 bytes) where ALIGNED. STREAM: read once.
template <typename T, bool ALIGNED, bool CHECK, bool STREAM>
__device__ __forceinline__ uint4 load16(const T *row, int k, int K) {
    if constexpr (ALIGNED) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (!CHECK || k < K) {
            if constexpr (STREAM)
                asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                             : "l"(row + k));
            else
                v = __ldg(reinterpret_cast<const uint4 *>(row + k));
        }
        return v;
    } else {
        constexpr int per = 4 / sizeof(T);
        uint32_t w[4] = {};
#pragma unroll
        for (int j = 0; j < 4 * per; j++)
            if (!CHECK || k + j < K) {
                if constexpr (per == 2) w[j / 2] |= (uint32_t)__ldg(row + k + j) << (16 * (j & 1));
                else w[j] = __float_as_uint(__ldg(row + k + j));
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Calls body(k, checked) for this lane's columns k of each kAhead reads of a warp:
// kAhead spans of 64 bytes, kWarps spans apart; `checked` (a compile-time constant)
// where some may lie past K. LONG: calls pause() after every kPause whole ones.
template <bool B>
struct Checked {
    static constexpr bool value = B;
};
constexpr int kPause = 8;
template <typename T>
constexpr int kStride = kAhead * kWarps * 64 / (int)sizeof(T);   // columns of a call of body, of all warps
template <typename T, bool LONG, typename F, typename P>
__device__ __forceinline__ void along_k(int K, F body, P pause) {
    constexpr int span = 64 / sizeof(T), stride = kStride<T>;
    const int lane0 = (threadIdx.x >> 5) * span + (threadIdx.x & 3) * (16 / (int)sizeof(T));
    int k0 = 0, until = kPause * stride;
    for (; k0 + stride <= K; k0 += stride) {
        if (LONG && k0 == until) {
            pause();
            until += kPause * stride;
        }
        body(k0 + lane0, Checked<false>{});
    }
    if (k0 < K) body(k0 + lane0, Checked<true>{});
}

// NT eights of tokens. LONG (bf16): K of more than kPause strides. The accumulation drops
// bits (7e-9 of a sum of one sign with a column), so a long sum goes on in shared memory.
// (In short ones the test alone took 0.3 us, for 8 tokens of 1024 into 4096.)
template <typename T, int NT, bool ALIGNED, bool LONG>
__global__ void __launch_bounds__(32 * kWarps, NT == 1 ? 4 : NT == 2 ? 3 : 2) k_gated_few(const __grid_constant__ GatedCall c) {
    constexpr int step = kWarps * 64 / sizeof(T);
    __shared__ float4 sums[kWarps][NT][32];
    ptx::pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2;
    const int K = (int)c.K;
    const int64_t f = std::min<int64_t>((int64_t)blockIdx.x * 8 + g, c.F - 1);
    const T *wg = static_cast<const T *>(c.Wg) + f * c.K, *wu = static_cast<const T *>(c.Wu) + f * c.K;
    const T *x[NT];
#pragma unroll
    for (int n = 0; n < NT; n++) x[n] = static_cast<const T *>(c.X) + std::min<int64_t>(8 * n + g, c.N - 1) * c.K;
    float acc[NT][4] = {};
    bool kept = false;   // whether `sums` has what came before acc
    auto keep = [&]() {
#pragma unroll
        for (int n = 0; n < NT; n++) {
            float4 &s = sums[warp][n][lane];
            const float4 old = LONG && kept ? s : make_float4(0.f, 0.f, 0.f, 0.f);
            s = make_float4(old.x + acc[n][0], old.y + acc[n][1], old.z + acc[n][2], old.w + acc[n][3]);
#pragma unroll
            for (int j = 0; j < 4; j++) acc[n][j] = 0.f;
        }
    };
    ptx::pdl_wait();
    along_k<T, LONG>(K, [&](int k, auto checked) {
        constexpr bool CHECK = decltype(checked)::value;
        uint4 a[kAhead], b[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            a[i] = load16<T, ALIGNED, CHECK, true>(wg, k + i * step, K);
            b[i] = load16<T, ALIGNED, CHECK, true>(wu, k + i * step, K);
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            if constexpr (sizeof(T) == 2) {
                const uint32_t ga[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, ua[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    const uint4 v = load16<T, ALIGNED, CHECK, false>(x[n], k + i * step, K);
                    const uint32_t xv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; j += 2) mma(acc[n], ga[j], ua[j], ga[j + 1], ua[j + 1], xv[j], xv[j + 1]);
                }
            } else {
                uint32_t g[3][2], u[3][2];
                split(a[i], g);
                split(b[i], u);
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    uint32_t xv[3][2];
                    split(load16<T, ALIGNED, CHECK, false>(x[n], k + i * step, K), xv);
                    // the accumulation in an MMA drops bits: the small products first, and
                    // 16 columns at a time added here (in one accumulator throughout the
                    // error of 1024 columns was 2.5e-6 of H, that of plain sums 0.9e-6)
                    float sum[4] = {};
#pragma unroll
                    for (int p = 2; p >= 0; p--)
#pragma unroll
                        for (int w = p; w >= 0; w--) mma(sum, g[w][0], u[w][0], g[w][1], u[w][1], xv[p - w][0], xv[p - w][1]);
#pragma unroll
                    for (int j = 0; j < 4; j++) acc[n][j] += sum[j];
                }
            }
        }
    }, [&]() {
        keep();
        kept = true;
    });
    keep();
    __syncthreads();
    // feature lane / 4 and tokens 2 (lane % 4), + 1 of each eight: G in x, y, U in z, w
    for (int e = threadIdx.x; e < NT * 32; e += 32 * kWarps) {
        const int n = e >> 5, l = e & 31;
        const int64_t fe = (int64_t)blockIdx.x * 8 + (l >> 2), t = 8 * n + 2 * (l & 3);
        if (fe >= c.F) continue;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kWarps; k++) {
            const float4 v = sums[k][n][l];
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const float bg = c.bg ? __ldg(c.bg + fe) : 0.f, bu = c.bu ? __ldg(c.bu + fe) : 0.f;
        float2 h;
        with_act(c.act, [&](auto tag) {
            h = unpack2(mul2(activate<decltype(tag)::value, sizeof(T) == 2>(pack2(s.x + bg, s.y + bg)), pack2(s.z + bu, s.w + bu)));
        });
        T *out = static_cast<T *>(c.H) + fe;
        if (t < c.N) out[t * c.F] = from_f32<T>(h.x);
        if (t + 1 < c.N) out[(t + 1) * c.F] = from_f32<T>(h.y);
    }
}

// fp32, up to TOKENS tokens.
template <int TOKENS, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps, 4) k_gated_few_f32(const __grid_constant__ GatedCall c) {
    constexpr int step = kWarps * 16;
    __shared__ float2 sums[kWarps][8][TOKENS];
    ptx::pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int K = (int)c.K;
    const int64_t f = std::min<int64_t>((int64_t)blockIdx.x * 8 + g, c.F - 1);
    const float *wg = static_cast<const float *>(c.Wg) + f * c.K, *wu = static_cast<const float *>(c.Wu) + f * c.K;
    const int tokens = (int)c.N;
    const float *X = static_cast<const float *>(c.X);
    F2 G[TOKENS], U[TOKENS];   // of even and odd columns
#pragma unroll
    for (int n = 0; n < TOKENS; n++) G[n] = U[n] = all2(0.f);
    ptx::pdl_wait();
    along_k<float, false>(K, [&](int k, auto checked) {
        constexpr bool CHECK = decltype(checked)::value;
        uint4 a[kAhead], b[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            a[i] = load16<float, ALIGNED, CHECK, true>(wg, k + i * step, K);
            b[i] = load16<float, ALIGNED, CHECK, true>(wu, k + i * step, K);
        }
        auto two = [](uint32_t lo, uint32_t hi) { return pack2(__uint_as_float(lo), __uint_as_float(hi)); };
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const F2 a0 = two(a[i].x, a[i].y), a1 = two(a[i].z, a[i].w), b0 = two(b[i].x, b[i].y), b1 = two(b[i].z, b[i].w);
            const float *x = X;
#pragma unroll
            for (int n = 0; n < TOKENS; n++) {
                const uint4 v = load16<float, ALIGNED, CHECK, false>(x, k + i * step, K);
                const F2 x0 = two(v.x, v.y), x1 = two(v.z, v.w);
                G[n] = fma2(a1, x1, fma2(a0, x0, G[n]));
                U[n] = fma2(b1, x1, fma2(b0, x0, U[n]));
                if (n + 1 < tokens) x += K;   // (past the last token: its own row again)
            }
        }
    }, []() {});
#pragma unroll
    for (int n = 0; n < TOKENS; n++) {
        const float2 gs = unpack2(G[n]), us = unpack2(U[n]);
        float2 s = make_float2(gs.x + gs.y, us.x + us.y);
#pragma unroll
        for (int d = 1; d < 4; d *= 2) {
            s.x += __shfl_xor_sync(0xffffffffu, s.x, d);
            s.y += __shfl_xor_sync(0xffffffffu, s.y, d);
        }
        if (q == 0) sums[warp][g][n] = s;
    }
    __syncthreads();
    const int e = threadIdx.x, fl = e & 7, n = e >> 3;
    const int64_t fe = (int64_t)blockIdx.x * 8 + fl;
    if (n >= tokens || fe >= c.F) return;
    float2 s = make_float2(c.bg ? __ldg(c.bg + fe) : 0.f, c.bu ? __ldg(c.bu + fe) : 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; k++) s.x += sums[k][fl][n].x, s.y += sums[k][fl][n].y;
    with_act(c.act, [&](auto tag) {
        static_cast<float *>(c.H)[(int64_t)n * c.F + fe] = unpack2(activate<decltype(tag)::value, false>(all2(s.x))).x * s.y;
    });
}

template <typename T, int NT>
cudaError_t launch(const GatedCall &c, cudaStream_t s) {
    const bool aligned = c.K * sizeof(T) % 16 == 0;
    auto kernel = aligned ? k_gated_few<T, NT, true, false> : k_gated_few<T, NT, false, false>;
    if constexpr (sizeof(T) == 2) {
        if (c.K > kPause * kStride<T>) kernel = aligned ? k_gated_few<T, NT, true, true> : k_gated_few<T, NT, false, true>;
    }
    return launch_kernel(kernel, dim3((unsigned)((c.F + 7) / 8)), dim3(32 * kWarps), 0, s, c);
}
template <int TOKENS>
cudaError_t launch_f32(const GatedCall &c, cudaStream_t s) {
    return launch_kernel(c.K % 4 == 0 ? k_gated_few_f32<TOKENS, true> : k_gated_few_f32<TOKENS, false>,
                         dim3((unsigned)((c.F + 7) / 8)), dim3(32 * kWarps), 0, s, c);
}

}  // namespace

cudaError_t launch_gated_few(const GatedCall &c, cudaStream_t s) {
    if (c.dt == BSR_BF16) return c.N <= 8 ? launch<uint16_t, 1>(c, s) : c.N <= 16 ? launch<uint16_t, 2>(c, s) : launch<uint16_t, 4>(c, s);
    return c.N == 1    ? launch_f32<1>(c, s)
           : c.N == 2  ? launch_f32<2>(c, s)
           : c.N <= 8  ? launch<float, 1>(c, s)
           : c.N <= 16 ? launch<float, 2>(c, s)
                       : launch<float, 4>(c, s);
}

}  // namespace bsr
