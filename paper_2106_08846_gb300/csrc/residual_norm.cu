// The residual step between two blocks of a transformer layer, one pass over
// the data in each direction.
//
//   t  = post(y);  h' = alpha h + s * gate * t;  z = pre(h')
//
// with post and pre a LayerNorm, an RMSNorm or nothing. A row of D features is
// held by a group of threads, eight features a thread (or twice eight), from
// its only read on; means and deviations are sums over the group, the deviation
// from the centred row, all in fp32. z is made from h' before h' is rounded.
//
// Backward, with xh a normalised row, r its 1 / deviation and [..] for
// LayerNorm only:
//
//   a = dz w_pre;  dH = dh' + r (a - [mean a] - hh mean(a hh));  dh = alpha dH
//   c = s gate dH w_post;  dy = r (c - [mean c] - yh mean(c yh))
//
// and sums over tokens for the parameters. A group works through runs of
// consecutive tokens that share a gate row and holds its features' sums in
// registers; the groups' sums are added in a fixed order by a second kernel, so
// results do not change from run to run.
//
// What bounds it: DRAM. Forward reads y and h and writes h' and z, backward
// reads y, h', dh', dz and writes dy, dh.
#include <algorithm>

#include "bsr_internal.h"
#include "elem.cuh"
#include "launch.cuh"
#include "ptx.cuh"
#include "residual_norm.h"

namespace bsr {

namespace {

constexpr int kMaxGroups = 8;     // rows in work per CTA
constexpr int kSums = 5;          // parameter gradients: scale, post_w, post_b, pre_w, pre_b

// The features of thread t of NT: where VEC, V runs of eight; else every NT-th.
template <bool VEC>
__device__ __forceinline__ int feature(int i, int j, int t, int NT) {
    return VEC ? 8 * (t + i * NT) + j : (8 * i + j) * NT + t;
}

__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t *p, float (&x)[8]) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; k++) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; k++)
        w[k] = from_f32<uint16_t>(x[2 * k]) | (uint32_t)from_f32<uint16_t>(x[2 * k + 1]) << 16;
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// A row's features of this thread; 0 past the row's end, `absent` everywhere without a row.
template <typename T, int V, bool VEC>
__device__ __forceinline__ void load_row(const T *row, int D, int t, int NT, float (&x)[8 * V], float absent = 0.f) {
#pragma unroll
    for (int i = 0; i < V; i++) {
        if constexpr (VEC) {
            float v[8] = {};
            if (row && feature<VEC>(i, 0, t, NT) < D) load8(row + feature<VEC>(i, 0, t, NT), v);
#pragma unroll
            for (int j = 0; j < 8; j++) x[8 * i + j] = row ? v[j] : absent;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int e = feature<VEC>(i, j, t, NT);
                x[8 * i + j] = !row ? absent : e < D ? to_f32(row[e]) : 0.f;
            }
        }
    }
}
template <typename T, int V, bool VEC>
__device__ __forceinline__ void store_row(T *row, int D, int t, int NT, const float (&x)[8 * V]) {
#pragma unroll
    for (int i = 0; i < V; i++) {
        if constexpr (VEC) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = x[8 * i + j];
            if (feature<VEC>(i, 0, t, NT) < D) store8(row + feature<VEC>(i, 0, t, NT), v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int e = feature<VEC>(i, j, t, NT);
                if (e < D) row[e] = from_f32<T>(x[8 * i + j]);
            }
        }
    }
}

// Sums over the NT threads of a group, the same in each of them. The two
// halves of the group's shared words are used in turn, so one barrier does:
// a half is written again only after the other half's barrier.
struct GroupSum {
    float *words;   // [2][32][2]
    int NT, id, turn;
    __device__ __forceinline__ void operator()(float &a, float &b) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, d);
            b += __shfl_xor_sync(0xffffffffu, b, d);
        }
        if (NT == 32) return;
        float2 *w = reinterpret_cast<float2 *>(words) + 32 * turn;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = make_float2(a, b);
        ptx::named_barrier(1 + id, NT);
        a = b = 0.f;
        for (int k = 0; k < NT / 32; k++) {
            const float2 v = w[k];
            a += v.x;
            b += v.y;
        }
    }
};

// Normalises a row in place and returns 1 / deviation.
template <int V, bool VEC>
__device__ __forceinline__ float normalise(float (&x)[8 * V], int how, float eps, int D, int t, int NT, GroupSum &sum) {
    float mean = 0.f, none = 0.f;
    if (how == BSR_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < 8 * V; k++) mean += x[k];
        sum(mean, none);
        mean /= (float)D;
    }
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < 8 * V; k++) {
        x[k] = feature<VEC>(k / 8, k % 8, t, NT) < D ? x[k] - mean : 0.f;
        sq = fmaf(x[k], x[k], sq);
    }
    sum(sq, none);
    const float r = 1.f / sqrtf(sq / (float)D + eps);
#pragma unroll
    for (int k = 0; k < 8 * V; k++) x[k] *= r;
    return r;
}

template <typename TB, typename TS, int V, bool VEC>
__global__ void __launch_bounds__(1024) k_residual_norm(const __grid_constant__ RnForward a) {
    __shared__ float words[kMaxGroups][128];
    const int t = threadIdx.x, NT = blockDim.x, D = (int)a.p.D;
    GroupSum sum{words[threadIdx.y], NT, (int)threadIdx.y, 0};
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t n = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; n < a.N; n += (int64_t)gridDim.x * blockDim.y) {
        float x[8 * V], v[8 * V], w[8 * V];
        load_row<TB, V, VEC>(static_cast<const TB *>(a.y) + n * D, D, t, NT, x);
        load_row<TS, V, VEC>(a.h ? static_cast<const TS *>(a.h) + n * D : nullptr, D, t, NT, v);
        if (a.p.post != BSR_NORM_NONE) {
            normalise<V, VEC>(x, a.p.post, a.p.post_eps, D, t, NT, sum);
            load_row<float, V, VEC>(a.p.post_w, D, t, NT, w, 1.f);
#pragma unroll
            for (int k = 0; k < 8 * V; k++) x[k] *= w[k];
            load_row<float, V, VEC>(a.p.post_b, D, t, NT, w);
#pragma unroll
            for (int k = 0; k < 8 * V; k++) x[k] += w[k];
        }
        if (a.gate) {
            load_row<TB, V, VEC>(static_cast<const TB *>(a.gate) + n / a.p.gate_tokens * D, D, t, NT, w);
#pragma unroll
            for (int k = 0; k < 8 * V; k++) x[k] *= w[k];
        }
        load_row<float, V, VEC>(a.p.scale, D, t, NT, w, 1.f);
#pragma unroll
        for (int k = 0; k < 8 * V; k++) {
            x[k] *= w[k];
            if (a.h) x[k] = fmaf(a.p.alpha, v[k], x[k]);
        }
        if (a.h_out) store_row<TS, V, VEC>(static_cast<TS *>(a.h_out) + n * D, D, t, NT, x);
        if (a.p.pre != BSR_NORM_NONE) {
            normalise<V, VEC>(x, a.p.pre, a.p.pre_eps, D, t, NT, sum);
            load_row<float, V, VEC>(a.p.pre_w, D, t, NT, w, 1.f);
#pragma unroll
            for (int k = 0; k < 8 * V; k++) x[k] *= w[k];
            load_row<float, V, VEC>(a.p.pre_b, D, t, NT, w);
#pragma unroll
            for (int k = 0; k < 8 * V; k++) x[k] += w[k];
            store_row<TB, V, VEC>(static_cast<TB *>(a.z) + n * D, D, t, NT, x);
        }
    }
}

// How the backward pass shares out its tokens: `units` runs of at most `len`
// tokens, `slices` to a gate row (without a gate: to all tokens), taken in turn
// by `workers` groups.
struct RnSplit {
    int64_t units, slices, len, span, workers;
};

struct RnBackwardArgs {
    RnBackward b;
    RnSplit split;
    float *sums;        // [workers][kSums][D]
    float *gate_sums;   // [units][D], where a gate row has several slices
};

// The gradient of a norm's input, g that of the normalised row xh.
template <int V>
__device__ __forceinline__ void norm_grad(float (&g)[8 * V], const float (&xh)[8 * V], float r, int how, int D,
                                          GroupSum &sum) {
    float m = 0.f, mx = 0.f;
#pragma unroll
    for (int k = 0; k < 8 * V; k++) {
        m += g[k];
        mx = fmaf(g[k], xh[k], mx);
    }
    sum(m, mx);
    m = how == BSR_NORM_LAYER ? m / (float)D : 0.f;
    mx /= (float)D;
#pragma unroll
    for (int k = 0; k < 8 * V; k++) g[k] = r * (g[k] - m - xh[k] * mx);
}

template <typename TB, typename TS, int V, bool VEC>
__global__ void __launch_bounds__(V == 1 ? 512 : 1024) k_residual_norm_backward(const __grid_constant__ RnBackwardArgs args) {
    __shared__ float words[kMaxGroups][128];
    const RnBackward &a = args.b;
    const int t = threadIdx.x, NT = blockDim.x, D = (int)a.p.D;
    GroupSum sum{words[threadIdx.y], NT, (int)threadIdx.y, 0};
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    float acc[kSums][8 * V] = {};
    const int64_t worker = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool want_gate = a.gate && a.g.dgate;
    for (int64_t u = worker; u < args.split.units; u += args.split.workers) {
        const int64_t row = u / args.split.slices, slice = u - row * args.split.slices;
        const int64_t n0 = row * args.split.span + slice * args.split.len;
        const int64_t n1 = min(min(n0 + args.split.len, (row + 1) * args.split.span), a.N);
        float gate_acc[8 * V] = {};
        for (int64_t n = n0; n < n1; n++) {
            float y[8 * V], g[8 * V], w[8 * V];
            load_row<TB, V, VEC>(static_cast<const TB *>(a.y) + n * D, D, t, NT, y);
            load_row<TS, V, VEC>(a.dh_out ? static_cast<const TS *>(a.dh_out) + n * D : nullptr, D, t, NT, g);   // dH
            if (a.p.pre != BSR_NORM_NONE) {
                float hh[8 * V], dz[8 * V];
                load_row<TS, V, VEC>(static_cast<const TS *>(a.h_out) + n * D, D, t, NT, hh);
                load_row<TB, V, VEC>(static_cast<const TB *>(a.dz) + n * D, D, t, NT, dz);
                const float r = normalise<V, VEC>(hh, a.p.pre, a.p.pre_eps, D, t, NT, sum);
                load_row<float, V, VEC>(a.p.pre_w, D, t, NT, w, 1.f);
#pragma unroll
                for (int k = 0; k < 8 * V; k++) {
                    acc[3][k] = fmaf(dz[k], hh[k], acc[3][k]);
                    acc[4][k] += dz[k];
                    dz[k] *= w[k];
                }
                norm_grad<V>(dz, hh, r, a.p.pre, D, sum);
#pragma unroll
                for (int k = 0; k < 8 * V; k++) g[k] += dz[k];
            }
            if (a.dh) {
#pragma unroll
                for (int k = 0; k < 8 * V; k++) w[k] = a.p.alpha * g[k];
                store_row<TS, V, VEC>(static_cast<TS *>(a.dh) + n * D, D, t, NT, w);
            }
            // y becomes yh, and g the gradient of t
            float gate[8 * V], s[8 * V], r = 0.f;
            load_row<TB, V, VEC>(a.gate ? static_cast<const TB *>(a.gate) + row * D : nullptr, D, t, NT, gate, 1.f);
            load_row<float, V, VEC>(a.p.scale, D, t, NT, s, 1.f);
            float b[8 * V];
            if (a.p.post != BSR_NORM_NONE) {
                r = normalise<V, VEC>(y, a.p.post, a.p.post_eps, D, t, NT, sum);
                load_row<float, V, VEC>(a.p.post_w, D, t, NT, w, 1.f);
                load_row<float, V, VEC>(a.p.post_b, D, t, NT, b);
            }
#pragma unroll
            for (int k = 0; k < 8 * V; k++) {
                const float tv = a.p.post != BSR_NORM_NONE ? fmaf(y[k], w[k], b[k]) : y[k];
                gate_acc[k] = fmaf(tv * s[k], g[k], gate_acc[k]);
                acc[0][k] = fmaf(tv * gate[k], g[k], acc[0][k]);
                g[k] *= s[k] * gate[k];
            }
            if (a.p.post != BSR_NORM_NONE) {
#pragma unroll
                for (int k = 0; k < 8 * V; k++) {
                    acc[1][k] = fmaf(g[k], y[k], acc[1][k]);
                    acc[2][k] += g[k];
                    g[k] *= w[k];
                }
                norm_grad<V>(g, y, r, a.p.post, D, sum);
            }
            if (a.dy) store_row<TB, V, VEC>(static_cast<TB *>(a.dy) + n * D, D, t, NT, g);
        }
        if (want_gate) {
            if (args.gate_sums) store_row<float, V, VEC>(args.gate_sums + u * D, D, t, NT, gate_acc);
            else store_row<TB, V, VEC>(static_cast<TB *>(a.g.dgate) + row * D, D, t, NT, gate_acc);
        }
    }
    if (worker >= args.split.workers) return;
    float *const dst[kSums] = {a.g.dscale, a.g.dpost_w, a.g.dpost_b, a.g.dpre_w, a.g.dpre_b};
#pragma unroll
    for (int k = 0; k < kSums; k++)
        if (dst[k]) store_row<float, V, VEC>(args.sums + (worker * kSums + k) * D, D, t, NT, acc[k]);
}

// Adds the workers' sums (blockIdx.y < kSums) or a gate row's slices, 32
// features a CTA: 32 x 8 threads, each every eighth entry, then the eight.
template <typename TB>
__global__ void __launch_bounds__(256) k_residual_norm_sums(const __grid_constant__ RnBackwardArgs args) {
    __shared__ float part[8][33];
    const RnBackward &a = args.b;
    const int64_t D = a.p.D, d = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float *const dst[kSums] = {a.g.dscale, a.g.dpost_w, a.g.dpost_b, a.g.dpre_w, a.g.dpre_b};
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t job = blockIdx.y; job < kSums + (args.gate_sums ? args.split.units / args.split.slices : 0); job += gridDim.y) {
        const float *src;
        int64_t n, stride;
        if (job < kSums) {
            if (!dst[job]) continue;
            src = args.sums + job * D, n = args.split.workers, stride = kSums * D;
        } else {
            src = args.gate_sums + (job - kSums) * args.split.slices * D, n = args.split.slices, stride = D;
        }
        float s = 0.f;
        if (d < D)
            for (int64_t k = threadIdx.y; k < n; k += 8) s += src[k * stride + d];
        part[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        if (threadIdx.y == 0 && d < D) {
            s = 0.f;
            for (int k = 0; k < 8; k++) s += part[k][threadIdx.x];
            if (job < kSums) dst[job][d] = s;
            else static_cast<TB *>(a.g.dgate)[(job - kSums) * D + d] = from_f32<TB>(s);
        }
        __syncthreads();
    }
}

int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        cudaGetLastError();
    return n;
}

// Threads of a group and groups of a CTA.
struct RnShape {
    int V, NT, R;
};
RnShape shape_of(int64_t D) {
    RnShape s;
    s.V = D > 4096 ? 2 : 1;
    s.NT = (int)((D + 8 * s.V - 1) / (8 * s.V) + 31) / 32 * 32;
    s.R = std::max(1, std::min(kMaxGroups, 256 / s.NT));
    return s;
}

bool any_sum(const bsr_residual_norm_grads_t &g) { return g.dscale || g.dpost_w || g.dpost_b || g.dpre_w || g.dpre_b; }

RnSplit split_of(const bsr_residual_norm_t &p, int64_t N) {
    const RnShape sh = shape_of(p.D);
    // groups that an SM holds at once, by the backward kernel's registers
    const int64_t most = (int64_t)sm_count() * std::max(1, 512 / sh.NT);
    RnSplit s;
    s.span = p.gate_tokens > 0 ? std::min<int64_t>(p.gate_tokens, N) : N;
    const int64_t rows = (N + s.span - 1) / s.span, len = std::max<int64_t>(1, (N + most - 1) / most);
    s.slices = (s.span + len - 1) / len;
    s.len = (s.span + s.slices - 1) / s.slices;
    s.slices = (s.span + s.len - 1) / s.len;
    s.units = rows * s.slices;
    s.workers = std::min(s.units, most);
    return s;
}

bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <typename TB, typename TS>
cudaError_t forward(const RnForward &a, cudaStream_t s) {
    const RnShape sh = shape_of(a.p.D);
    const bool vec = a.p.D % 8 == 0 && aligned(a.p.scale) && aligned(a.p.post_w) && aligned(a.p.post_b) &&
                     aligned(a.p.pre_w) && aligned(a.p.pre_b);
    const dim3 block(sh.NT, sh.R), grid((unsigned)std::min<int64_t>((a.N + sh.R - 1) / sh.R, INT32_MAX));
    auto kernel = sh.V == 1 ? (vec ? k_residual_norm<TB, TS, 1, true> : k_residual_norm<TB, TS, 1, false>)
                            : (vec ? k_residual_norm<TB, TS, 2, true> : k_residual_norm<TB, TS, 2, false>);
    return launch_kernel(kernel, grid, block, 0, s, a);
}

template <typename TB, typename TS>
cudaError_t backward(const RnBackward &b, cudaStream_t s) {
    RnBackwardArgs a;
    a.b = b;
    a.split = split_of(b.p, b.N);
    a.sums = b.ws;
    a.gate_sums = b.gate && b.g.dgate && a.split.slices > 1 ? b.ws + a.split.workers * kSums * b.p.D : nullptr;
    const RnShape sh = shape_of(b.p.D);
    const bool vec = b.p.D % 8 == 0 && aligned(b.p.scale) && aligned(b.p.post_w) && aligned(b.p.post_b) &&
                     aligned(b.p.pre_w) && aligned(b.p.pre_b);
    const dim3 block(sh.NT, sh.R), grid((unsigned)((a.split.workers + sh.R - 1) / sh.R));
    auto kernel = sh.V == 1 ? (vec ? k_residual_norm_backward<TB, TS, 1, true> : k_residual_norm_backward<TB, TS, 1, false>)
                            : (vec ? k_residual_norm_backward<TB, TS, 2, true> : k_residual_norm_backward<TB, TS, 2, false>);
    cudaError_t e = launch_kernel(kernel, grid, block, 0, s, a);
    if (e != cudaSuccess || (!any_sum(b.g) && !a.gate_sums)) return e;
    const int64_t jobs = kSums + (a.gate_sums ? a.split.units / a.split.slices : 0);
    return launch_kernel(k_residual_norm_sums<TB>, dim3((unsigned)((b.p.D + 31) / 32), (unsigned)std::min<int64_t>(jobs, 65535)),
                         dim3(32, 8), 0, s, a);
}

}  // namespace

int64_t residual_norm_workspace(const bsr_residual_norm_t &p, int64_t N) {
    if (N == 0) return 0;
    const RnSplit s = split_of(p, N);
    return (s.workers * kSums + (p.gate_tokens > 0 && s.slices > 1 ? s.units : 0)) * p.D * 4;
}

cudaError_t launch_residual_norm(const RnForward &a, cudaStream_t s) {
    if (a.N == 0) return cudaSuccess;
    if (a.p.block_dt == BSR_F32) return forward<float, float>(a, s);
    return a.p.stream_dt == BSR_F32 ? forward<uint16_t, float>(a, s) : forward<uint16_t, uint16_t>(a, s);
}

cudaError_t launch_residual_norm_backward(const RnBackward &a, cudaStream_t s) {
    if (a.N == 0) {   // sums of nothing
        float *const sums[kSums] = {a.g.dscale, a.g.dpost_w, a.g.dpost_b, a.g.dpre_w, a.g.dpre_b};
        for (float *p : sums)
            if (p && cudaMemsetAsync(p, 0, (size_t)a.p.D * 4, s) != cudaSuccess) return cudaGetLastError();
        return cudaSuccess;
    }
    if (a.p.block_dt == BSR_F32) return backward<float, float>(a, s);
    return a.p.stream_dt == BSR_F32 ? backward<uint16_t, float>(a, s) : backward<uint16_t, uint16_t>(a, s);
}

}  // namespace bsr
