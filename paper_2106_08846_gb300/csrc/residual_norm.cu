// The residual step between two blocks of a transformer layer, one pass over
// the data in each direction.
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
// Backward, with xh a normalised row, r its 1 / deviation and [..] for
// LayerNorm only:
//
//   a = dz w_pre;  dH = dh' + r (a - [mean a] - hh mean(a hh));  dh = alpha dH
//   c = s gate dH w_post;  dy = r (c - [mean c] - yh mean(c yh))
//
// and sums over tokens for the parameters. A thread has the same features in every
// row that its group works on: it keeps their parameters and their sums in
// registers, and the next row is on its way while one is worked on. A group adds up
// three times to a row: the means; the squares with what the pre norm's gradient
// needs (its sums are of the centred row, the deviation put in afterwards); the
// post norm's gradient. The groups' sums are added in a fixed order by a second
// kernel, so results do not change from run to run.
//
// What bounds it: DRAM. Forward reads y and h and writes h' and z, backward
// reads y, h', dh', dz and writes dy, dh.
#include <algorithm>

#include "bsr_internal.h"
#include "elem.cuh"
#include "launch.cuh"
#include "pair.cuh"
#include "ptx.cuh"
#include "residual_norm.h"

namespace bsr {

namespace {

constexpr int kMaxGroups = 8;     // rows in work per CTA
constexpr int kSums = 5;          // parameter gradients: scale, post_w, post_b, pre_w, pre_b

// How a row lies in a group's NT threads: every NT-th feature to a thread, runs of
// eight, or runs of eight with none past the row's end.
enum Layout : int { SINGLES = 0, RUNS = 1, FULL = 2 };

// Feature j of run i of thread t, and whether it is one.
template <int L>
__device__ __forceinline__ int feature(int i, int j, int t, int NT) {
    return L != SINGLES ? 8 * (t + i * NT) + j : (8 * i + j) * NT + t;
}
template <int L>
__device__ __forceinline__ bool inside(int i, int j, int t, int NT, int D) {
    return L == FULL || feature<L>(i, j, t, NT) < D;
}

// A run of eight features, in pairs; as it lies in memory.
struct Run {
    F2 v[4];
};
template <typename T>
struct Raw {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ F2 two(int j) const {
        if constexpr (sizeof(T) == 4) return pack2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        else return pack2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
    __device__ __forceinline__ Run run() const {
        Run r;
#pragma unroll
        for (int j = 0; j < 4; j++) r.v[j] = two(j);
        return r;
    }
};
__device__ __forceinline__ Run all_run(float x) {
    Run r;
#pragma unroll
    for (int j = 0; j < 4; j++) r.v[j] = all2(x);
    return r;
}

// Run i of a row; 0 past the row's end. CONST: of an array that the kernel does not write.
template <typename T, int L, bool CONST>
__device__ __forceinline__ Raw<T> load_run(const T *row, int D, int i, int t, int NT) {
    Raw<T> r;
    if constexpr (L != SINGLES) {
        const int e = feature<L>(i, 0, t, NT);
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; h++) {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (inside<L>(i, 0, t, NT, D)) {
                const uint4 *p = reinterpret_cast<const uint4 *>(row + e) + h;
                u = CONST ? __ldg(p) : *p;
            }
            r.w[4 * h] = u.x, r.w[4 * h + 1] = u.y, r.w[4 * h + 2] = u.z, r.w[4 * h + 3] = u.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2 * (int)sizeof(T); j++) r.w[j] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int e = feature<L>(i, j, t, NT);
            if (e < D) {
                const T v = CONST ? __ldg(row + e) : row[e];
                if constexpr (sizeof(T) == 4) r.w[j] = __float_as_uint(v);
                else r.w[j / 2] |= (uint32_t)v << (16 * (j & 1));
            }
        }
    }
    return r;
}
template <typename T, int L>
__device__ __forceinline__ Run load_const(const T *row, int D, int i, int t, int NT) {
    return load_run<T, L, true>(row, D, i, t, NT).run();
}
template <typename T, int L>
__device__ __forceinline__ void store_run(T *row, int D, int i, int t, int NT, const Run &r) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float2 u = unpack2(r.v[j]);
        x[2 * j] = u.x, x[2 * j + 1] = u.y;
    }
    if constexpr (L != SINGLES) {
        const int e = feature<L>(i, 0, t, NT);
        if (!inside<L>(i, 0, t, NT, D)) return;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int h = 0; h < 2; h++) reinterpret_cast<float4 *>(row + e)[h] = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; k++) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
            *reinterpret_cast<uint4 *>(row + e) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int e = feature<L>(i, j, t, NT);
            if (e < D) row[e] = from_f32<T>(x[j]);
        }
    }
}

// x - m where there is a feature (x is 0 elsewhere, and stays so)
template <int L>
__device__ __forceinline__ void centre(Run &x, float m, int D, int i, int t, int NT) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if constexpr (L != SINGLES) x.v[j] = add2(x.v[j], all2(inside<L>(i, 0, t, NT, D) ? -m : 0.f));
        else x.v[j] = add2(x.v[j], pack2(inside<L>(i, 2 * j, t, NT, D) ? -m : 0.f, inside<L>(i, 2 * j + 1, t, NT, D) ? -m : 0.f));
    }
}
__device__ __forceinline__ float both(F2 x) {
    const float2 u = unpack2(x);
    return u.x + u.y;
}

// Sums over the NT threads of a group, the same in each of them. Lanes exchange
// halves of the values until each has one to add up; the warps' sums meet in shared
// memory, four warps to a group of words (of absent warps 0). Its two halves are used
// in turn, so one barrier does: a half is written again only after the other half's
// barrier. FOUR: at most four warps.
template <bool FOUR>
struct GroupSum {
    float4 *words;   // [2][32]
    int NT, id, turn;
    __device__ __forceinline__ void init() {   // before the group's first barrier
        for (int k = threadIdx.x; k < 64; k += NT) words[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (NT > 32) ptx::named_barrier(1 + id, NT);
    }
    template <int N>   // 1, 2 or 4
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        const int lane = threadIdx.x & 31;
        float a[N];
#pragma unroll
        for (int k = 0; k < N; k++) a[k] = v[k];
#pragma unroll
        for (int n = N, d = 16; n > 1; n /= 2, d /= 2) {
#pragma unroll
            for (int k = 0; k < n / 2; k++) {
                const float mine = lane & d ? a[k + n / 2] : a[k], other = lane & d ? a[k] : a[k + n / 2];
                a[k] = mine + __shfl_xor_sync(0xffffffffu, other, d);
            }
        }
        constexpr int last = N == 4 ? 4 : N == 2 ? 8 : 16;
#pragma unroll
        for (int d = last; d > 0; d /= 2) a[0] += __shfl_xor_sync(0xffffffffu, a[0], d);
        // value k is lane (32 / N) * (k's bits, the first exchange's the highest)
        if (NT == 32) {
#pragma unroll
            for (int k = 0; k < N; k++) v[k] = __shfl_sync(0xffffffffu, a[0], 32 / N * k);
            return;
        }
        // a warp's values side by side, but a value's four warps in one float4
        float *w = reinterpret_cast<float *>(words + 32 * turn);
        turn ^= 1;
        const int warp = threadIdx.x >> 5;
        if ((lane & (32 / N - 1)) == 0) w[16 * (warp >> 2) + 4 * (lane / (32 / N)) + (warp & 3)] = a[0];
        ptx::named_barrier(1 + id, NT);
        F2 s[N];
#pragma unroll
        for (int k = 0; k < N; k++) {
            const float4 u = reinterpret_cast<const float4 *>(w)[k];
            s[k] = add2(pack2(u.x, u.y), pack2(u.z, u.w));
        }
        if (!FOUR)
            for (int g = 1; g < (NT + 127) / 128; g++)
#pragma unroll
                for (int k = 0; k < N; k++) {
                    const float4 u = reinterpret_cast<const float4 *>(w)[4 * g + k];
                    s[k] = add2(s[k], add2(pack2(u.x, u.y), pack2(u.z, u.w)));
                }
#pragma unroll
        for (int k = 0; k < N; k++) v[k] = both(s[k]);
    }
};

// Normalises a row in place.
template <int V, int L, typename Sum>
__device__ __forceinline__ void normalise(Run (&x)[V], int how, float eps, int D, float over_d, int t, int NT, Sum &sum) {
    F2 s;
    float one[1];
    if (how == BSR_NORM_LAYER) {
        s = all2(0.f);
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) s = add2(s, x[i].v[j]);
        one[0] = both(s);
        sum(one);
#pragma unroll
        for (int i = 0; i < V; i++) centre<L>(x[i], one[0] * over_d, D, i, t, NT);
    }
    s = all2(0.f);
#pragma unroll
    for (int i = 0; i < V; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) s = fma2(x[i].v[j], x[i].v[j], s);
    one[0] = both(s);
    sum(one);
    const F2 r = all2(rsqrtf(fmaf(one[0], over_d, eps)));
#pragma unroll
    for (int i = 0; i < V; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) x[i].v[j] = mul2(x[i].v[j], r);
}
// x * w + b with a parameter's row each, where there is one
template <int V, int L>
__device__ __forceinline__ void affine(Run (&x)[V], const float *w, const float *b, int D, int t, int NT) {
    if (w) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const Run p = load_const<float, L>(w, D, i, t, NT);
#pragma unroll
            for (int j = 0; j < 4; j++) x[i].v[j] = mul2(x[i].v[j], p.v[j]);
        }
    }
    if (b) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const Run p = load_const<float, L>(b, D, i, t, NT);
#pragma unroll
            for (int j = 0; j < 4; j++) x[i].v[j] = add2(x[i].v[j], p.v[j]);
        }
    }
}

// WARP: a warp to a row. Rows `ahead` further on are asked for into L2: registers
// hold too few loads to keep DRAM busy (16384 x 1024 bf16: 29.4 us without).
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
        Raw<TS> h[V];
        {
            Raw<TB> y[V];
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
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) x[i].v[j] = fma2(all2(a.p.alpha), h[i].two(j), x[i].v[j]);
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

// The four rows of a token as they lie in memory.
template <typename TB, typename TS, int V>
struct Token {
    Raw<TB> y[V], dz[V];
    Raw<TS> h[V], dh[V];
};
template <typename TB, typename TS, int V, int L>
__device__ __forceinline__ void load_token(const RnBackward &a, int64_t n, int D, int t, int NT, Token<TB, TS, V> &k) {
    const bool pre = a.p.pre != BSR_NORM_NONE;
    const int64_t at = n * D;
#pragma unroll
    for (int i = 0; i < V; i++) {
        k.y[i] = load_run<TB, L, false>(static_cast<const TB *>(a.y) + at, D, i, t, NT);
        if (a.dh_out) k.dh[i] = load_run<TS, L, false>(static_cast<const TS *>(a.dh_out) + at, D, i, t, NT);
        if (pre) {
            k.h[i] = load_run<TS, L, true>(static_cast<const TS *>(a.h_out) + at, D, i, t, NT);
            k.dz[i] = load_run<TB, L, false>(static_cast<const TB *>(a.dz) + at, D, i, t, NT);
        }
    }
}

// What a unit of tokens of one gate row adds to the parameters' gradients follows
// from two sums for each feature, Q = sum dH yh and S = sum dH: with t = yh w + b,
// sum t dH = w Q + b S, from which the gate's gradient is scale times and the
// scale's gate times that, and post_w's and post_b's are scale gate Q and
// scale gate S. THREADS: the most of a CTA. KEEP: the next token is on its way in
// registers (rows of more than 4096 features leave none for it). GATE, BIAS:
// whether there may be a gate, and a bias; without a gate, all units are one.
template <typename TB, typename TS, int V, int L, int THREADS, bool GATE, bool BIAS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 3 : 1) k_residual_norm_backward(const __grid_constant__ RnBackwardArgs args) {
    constexpr bool KEEP = V == 1;
    __shared__ float4 words[kMaxGroups][64];
    const RnBackward &a = args.b;
    const int t = threadIdx.x, NT = blockDim.x, D = (int)a.p.D;
    const float over_d = 1.f / (float)D;
    GroupSum<THREADS == 128> sum{words[threadIdx.y], NT, (int)threadIdx.y, 0};
    sum.init();
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t worker = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool post = a.p.post != BSR_NORM_NONE, pre = a.p.pre != BSR_NORM_NONE;
    const bool post_layer = a.p.post == BSR_NORM_LAYER, pre_layer = a.p.pre == BSR_NORM_LAYER;
    const bool scaled = (GATE && a.gate) || a.p.scale;
    Run Q[V], S[V], dpre_w[V], dpre_b[V], dscale[V], dpost_w[V], dpost_b[V], post_w[V], pre_w[V], sg[V];
    auto zero = [&](Run (&r)[V]) {
#pragma unroll
        for (int i = 0; i < V; i++) r[i] = all_run(0.f);
    };
    auto param = [&](Run (&r)[V], const float *p, float absent) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            r[i] = all_run(absent);
            if (p) r[i] = load_const<float, L>(p, D, i, t, NT);
        }
    };
    zero(Q), zero(S), zero(dpre_w), zero(dpre_b), zero(dscale), zero(dpost_w), zero(dpost_b);
    if (KEEP) {
        param(post_w, a.p.post_w, 1.f);
        param(pre_w, a.p.pre_w, 1.f);
    }
    // the tokens of a unit, and of the worker's next one
    auto first_of = [&](int64_t u) {
        const int64_t row = u / args.split.slices;
        return row * args.split.span + (u - row * args.split.slices) * args.split.len;
    };
    Token<TB, TS, V> next = {};
    if (KEEP && worker < args.split.units) load_token<TB, TS, V, L>(a, first_of(worker), D, t, NT, next);
    const bool mine = worker < args.split.units;
    for (int64_t u = worker; u < args.split.units; u += args.split.workers) {
        const int64_t row = u / args.split.slices, n0 = first_of(u);
        const int64_t n1 = min(min(n0 + args.split.len, (row + 1) * args.split.span), a.N);
        const int64_t later = u + args.split.workers < args.split.units ? first_of(u + args.split.workers) : -1;
        const TB *const gate_row = GATE && a.gate ? static_cast<const TB *>(a.gate) + row * D : nullptr;
        // scale times gate
        param(sg, a.p.scale, 1.f);
        if (gate_row) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const Run g = load_const<TB, L>(gate_row, D, i, t, NT);
#pragma unroll
                for (int j = 0; j < 4; j++) sg[i].v[j] = mul2(sg[i].v[j], g.v[j]);
            }
        }
        for (int64_t n = n0; n < n1; n++) {
            Run y[V], hh[V], g[V], dz[V];
            if (!KEEP) load_token<TB, TS, V, L>(a, n, D, t, NT, next);
#pragma unroll
            for (int i = 0; i < V; i++) {
                y[i] = next.y[i].run();
                hh[i] = next.h[i].run();
                g[i] = next.dh[i].run();   // dH
                dz[i] = next.dz[i].run();
            }
            const int64_t after = n + 1 < n1 ? n + 1 : later;
            if (KEEP && after >= 0) load_token<TB, TS, V, L>(a, after, D, t, NT, next);
            if (post_layer || pre_layer) {
                F2 sh = all2(0.f), sy = all2(0.f);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        sh = add2(sh, hh[i].v[j]);
                        sy = add2(sy, y[i].v[j]);
                    }
                float m[2] = {both(sh), both(sy)};
                sum(m);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    if (pre_layer) centre<L>(hh[i], m[0] * over_d, D, i, t, NT);
                    if (post_layer) centre<L>(y[i], m[1] * over_d, D, i, t, NT);
                }
            }
            float ry = 1.f;
            if (pre) {
                if (!KEEP) param(pre_w, a.p.pre_w, 1.f);
                F2 sh = all2(0.f), sy = all2(0.f), sa = all2(0.f), sx = all2(0.f);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const F2 aw = mul2(dz[i].v[j], pre_w[i].v[j]);
                        sy = fma2(y[i].v[j], y[i].v[j], sy);
                        sh = fma2(hh[i].v[j], hh[i].v[j], sh);
                        sa = add2(sa, aw);
                        sx = fma2(aw, hh[i].v[j], sx);
                        if (BIAS) dpre_b[i].v[j] = add2(dpre_b[i].v[j], dz[i].v[j]);
                    }
                float s[4] = {both(sh), both(sy), both(sa), both(sx)};
                sum(s);
                if (post) ry = rsqrtf(fmaf(s[1], over_d, a.p.post_eps));
                // r (a - [mean a] - hh mean(a hh)), hh = r times the centred row
                const float r = rsqrtf(fmaf(s[0], over_d, a.p.pre_eps));
                const F2 r2 = all2(r), ma = all2(pre_layer ? -s[2] * over_d : 0.f), mx = all2(-s[3] * r * over_d);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const F2 xh = mul2(hh[i].v[j], r2);
                        dpre_w[i].v[j] = fma2(dz[i].v[j], xh, dpre_w[i].v[j]);
                        g[i].v[j] = fma2(r2, fma2(xh, mx, fma2(dz[i].v[j], pre_w[i].v[j], ma)), g[i].v[j]);
                    }
            } else if (post) {
                F2 sy = all2(0.f);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) sy = fma2(y[i].v[j], y[i].v[j], sy);
                float s[1] = {both(sy)};
                sum(s);
                ry = rsqrtf(fmaf(s[0], over_d, a.p.post_eps));
            }
            if (a.dh) {
                const F2 alpha = all2(a.p.alpha);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    Run out;
#pragma unroll
                    for (int j = 0; j < 4; j++) out.v[j] = mul2(alpha, g[i].v[j]);
                    store_run<TS, L>(static_cast<TS *>(a.dh) + n * D, D, i, t, NT, out);
                }
            }
            if (!KEEP && post) param(post_w, a.p.post_w, 1.f);
            F2 sc = all2(0.f), sx = all2(0.f);
            const F2 ry2 = all2(ry);
#pragma unroll
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const F2 yh = post ? mul2(y[i].v[j], ry2) : y[i].v[j];
                    Q[i].v[j] = fma2(g[i].v[j], yh, Q[i].v[j]);
                    if (BIAS) S[i].v[j] = add2(S[i].v[j], g[i].v[j]);
                    F2 c = scaled ? mul2(g[i].v[j], sg[i].v[j]) : g[i].v[j];
                    if (post) {
                        c = mul2(c, post_w[i].v[j]);
                        sc = add2(sc, c);
                        sx = fma2(c, yh, sx);
                    }
                    g[i].v[j] = c;
                    y[i].v[j] = yh;
                }
            if (post) {
                float s[2] = {both(sc), both(sx)};
                sum(s);
                const F2 mc = all2(post_layer ? -s[0] * over_d : 0.f), mx = all2(-s[1] * over_d);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) g[i].v[j] = mul2(ry2, fma2(y[i].v[j], mx, add2(g[i].v[j], mc)));
            }
            if (a.dy) {
#pragma unroll
                for (int i = 0; i < V; i++) store_run<TB, L>(static_cast<TB *>(a.dy) + n * D, D, i, t, NT, g[i]);
            }
        }
        if (GATE || later < 0) {   // what the unit (without a gate: all of the worker's) adds to the gradients
            Run P[V], b[V], scale[V], gate[V];
            param(post_w, a.p.post_w, 1.f);
            param(b, a.p.post_b, 0.f);
            param(scale, a.p.scale, 1.f);
#pragma unroll
            for (int i = 0; i < V; i++) {
                gate[i] = all_run(1.f);
                if (gate_row) gate[i] = load_const<TB, L>(gate_row, D, i, t, NT);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    P[i].v[j] = fma2(post_w[i].v[j], Q[i].v[j], mul2(b[i].v[j], S[i].v[j]));
                    dscale[i].v[j] = fma2(gate[i].v[j], P[i].v[j], dscale[i].v[j]);
                    dpost_w[i].v[j] = fma2(sg[i].v[j], Q[i].v[j], dpost_w[i].v[j]);
                    dpost_b[i].v[j] = fma2(sg[i].v[j], S[i].v[j], dpost_b[i].v[j]);
                    P[i].v[j] = mul2(P[i].v[j], scale[i].v[j]);
                }
                if (gate_row && a.g.dgate) {
                    if (args.gate_sums) store_run<float, L>(args.gate_sums + u * D, D, i, t, NT, P[i]);
                    else store_run<TB, L>(static_cast<TB *>(a.g.dgate) + row * D, D, i, t, NT, P[i]);
                }
            }
            zero(Q), zero(S);
        }
    }
    if (!mine) return;
    auto put = [&](int k, const float *wanted, const Run (&r)[V]) {
        if (!wanted) return;
#pragma unroll
        for (int i = 0; i < V; i++) store_run<float, L>(args.sums + (worker * kSums + k) * D, D, i, t, NT, r[i]);
    };
    put(0, a.g.dscale, dscale);
    put(1, a.g.dpost_w, dpost_w);
    put(2, a.g.dpost_b, dpost_b);
    put(3, a.g.dpre_w, dpre_w);
    put(4, a.g.dpre_b, dpre_b);
}

// Adds the workers' sums (blockIdx.y < kSums: one parameter's) or gate rows'
// slices (`rows` of them to a blockIdx.y), 32 features a CTA: 32 x 32 threads, each
// every so-manieth entry of a row, then those of a row.
template <typename TB>
__global__ void __launch_bounds__(1024) k_residual_norm_sums(const __grid_constant__ RnBackwardArgs args, int rows) {
    __shared__ float part[32][33];
    const RnBackward &a = args.b;
    const int64_t D = a.p.D, d = (int64_t)blockIdx.x * 32 + threadIdx.x, out = (int64_t)blockIdx.x * 32 + threadIdx.y;
    ptx::pdl_launch_dependents();
    const int y = blockIdx.y;
    if (y < kSums) {
        float *const dst = y == 0 ? a.g.dscale : y == 1 ? a.g.dpost_w : y == 2 ? a.g.dpost_b : y == 3 ? a.g.dpre_w : a.g.dpre_b;
        ptx::pdl_wait();
        if (!dst) return;
        float s = 0.f;
        if (d < D) {
#pragma unroll 8
            for (int64_t k = threadIdx.y; k < args.split.workers; k += 32) s += args.sums[(k * kSums + y) * D + d];
        }
        part[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        s = part[threadIdx.x][threadIdx.y];   // feature threadIdx.y, an entry a lane
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
        if (threadIdx.x == 0 && out < D) dst[out] = s;
        return;
    }
    ptx::pdl_wait();
    const int64_t slices = args.split.slices, gate_rows = args.split.units / slices;
    const int lanes = 32 / rows;   // of threadIdx.y to a row
    for (int64_t r0 = (int64_t)(y - kSums) * rows; r0 < gate_rows; r0 += (int64_t)(gridDim.y - kSums) * rows) {
        const int64_t r = r0 + threadIdx.y / lanes;
        float s = 0.f;
        if (d < D && r < gate_rows)
            for (int64_t k = threadIdx.y % lanes; k < slices; k += lanes) s += args.gate_sums[(r * slices + k) * D + d];
        part[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        if (threadIdx.y % lanes == 0 && d < D && r < gate_rows) {
            s = 0.f;
            for (int k = 0; k < lanes; k++) s += part[threadIdx.y + k][threadIdx.x];
            static_cast<TB *>(a.g.dgate)[r * D + d] = from_f32<TB>(s);
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

// Backward: runs of eight and threads of a group, and groups of a CTA.
struct RnShape {
    int V, NT, R;
};
RnShape shape_of(int64_t D) {
    RnShape s;
    s.V = D > 4096 ? 2 : 1;
    s.NT = (int)((D + 8 * s.V - 1) / (8 * s.V) + 31) / 32 * 32;
    s.R = std::max(1, std::min(kMaxGroups, 128 / s.NT));
    return s;
}

bool any_sum(const bsr_residual_norm_grads_t &g) { return g.dscale || g.dpost_w || g.dpost_b || g.dpre_w || g.dpre_b; }

RnSplit split_of(const bsr_residual_norm_t &p, int64_t N) {
    const RnShape sh = shape_of(p.D);
    // groups that an SM holds at once, by the backward kernel's registers
    const int64_t most = (int64_t)sm_count() * std::max(1, 384 / sh.NT);
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

// The layout of rows of D features in V runs of NT threads.
int layout_of(const bsr_residual_norm_t &p, int V, int NT) {
    const bool runs = p.D % 8 == 0 && aligned(p.scale) && aligned(p.post_w) && aligned(p.post_b) && aligned(p.pre_w) && aligned(p.pre_b);
    return !runs ? SINGLES : p.D == (int64_t)8 * V * NT ? FULL : RUNS;
}

template <typename TB, typename TS, int V>
cudaError_t forward_warps(const RnForward &a, cudaStream_t s) {
    const int sms = sm_count();
    // as many rows to a CTA as leave all SMs some
    const int R = (int)std::max<int64_t>(1, std::min<int64_t>(8, a.N / (4 * sms))), L = layout_of(a.p, V, 32);
    const dim3 block(32, R), grid((unsigned)std::min<int64_t>((a.N + R - 1) / R, INT32_MAX));
    auto kernel = L == FULL   ? k_residual_norm<TB, TS, V, FULL, true>
                  : L == RUNS ? k_residual_norm<TB, TS, V, RUNS, true>
                              : k_residual_norm<TB, TS, V, SINGLES, true>;
    return launch_kernel(kernel, grid, block, 0, s, a, (int64_t)sms * 24);   // (about the rows that run at once)
}

template <typename TB, typename TS>
cudaError_t forward(const RnForward &a, cudaStream_t s) {
    const int64_t D = a.p.D;
    if (D <= 256) return forward_warps<TB, TS, 1>(a, s);
    if (D <= 512) return forward_warps<TB, TS, 2>(a, s);
    if (D <= 768) return forward_warps<TB, TS, 3>(a, s);
    if (D <= 1024) return forward_warps<TB, TS, 4>(a, s);
    const int NT = (int)((D + 15) / 16 + 31) / 32 * 32, R = std::max(1, std::min(kMaxGroups, 256 / NT)), L = layout_of(a.p, 2, NT);
    const dim3 block(NT, R), grid((unsigned)std::min<int64_t>((a.N + R - 1) / R, INT32_MAX));
    auto kernel = L == FULL   ? k_residual_norm<TB, TS, 2, FULL, false>
                  : L == RUNS ? k_residual_norm<TB, TS, 2, RUNS, false>
                              : k_residual_norm<TB, TS, 2, SINGLES, false>;
    return launch_kernel(kernel, grid, block, 0, s, a, (int64_t)sm_count() * std::max(1, 1024 / NT));
}

template <typename TB, typename TS, int L>
auto few_threads(bool gate, bool bias) {   // 128 threads at most: what is not there costs nothing
    return gate ? (bias ? k_residual_norm_backward<TB, TS, 1, L, 128, true, true> : k_residual_norm_backward<TB, TS, 1, L, 128, true, false>)
                : (bias ? k_residual_norm_backward<TB, TS, 1, L, 128, false, true> : k_residual_norm_backward<TB, TS, 1, L, 128, false, false>);
}

template <typename TB, typename TS>
cudaError_t backward(const RnBackward &b, cudaStream_t s) {
    RnBackwardArgs a;
    a.b = b;
    a.split = split_of(b.p, b.N);
    a.sums = b.ws;
    a.gate_sums = b.gate && b.g.dgate && a.split.slices > 1 ? b.ws + a.split.workers * kSums * b.p.D : nullptr;
    const RnShape sh = shape_of(b.p.D);
    const int L = layout_of(b.p, sh.V, sh.NT), threads = sh.NT * sh.R;
    const dim3 block(sh.NT, sh.R), grid((unsigned)((a.split.workers + sh.R - 1) / sh.R));
    const bool gate = b.gate, bias = b.p.post_b || b.p.pre_b;
    auto kernel = sh.V == 1 && threads <= 128
                      ? (L == FULL   ? few_threads<TB, TS, FULL>(gate, bias)
                         : L == RUNS ? few_threads<TB, TS, RUNS>(gate, bias)
                                     : few_threads<TB, TS, SINGLES>(gate, bias))
                  : sh.V == 1
                      ? (L != SINGLES ? k_residual_norm_backward<TB, TS, 1, RUNS, 512, true, true>
                                      : k_residual_norm_backward<TB, TS, 1, SINGLES, 512, true, true>)
                  : threads <= 512
                      ? (L != SINGLES ? k_residual_norm_backward<TB, TS, 2, RUNS, 512, true, true>
                                      : k_residual_norm_backward<TB, TS, 2, SINGLES, 512, true, true>)
                      : (L != SINGLES ? k_residual_norm_backward<TB, TS, 2, RUNS, 1024, true, true>
                                      : k_residual_norm_backward<TB, TS, 2, SINGLES, 1024, true, true>);
    cudaError_t e = launch_kernel(kernel, grid, block, 0, s, a);
    if (e != cudaSuccess || (!any_sum(b.g) && !a.gate_sums)) return e;
    int rows = 1;   // gate rows to a CTA: as many as have a thread for each slice
    while (rows < 32 && 2 * rows * a.split.slices <= 32) rows *= 2;
    const int64_t gates = a.gate_sums ? (a.split.units / a.split.slices + rows - 1) / rows : 0;
    return launch_kernel(k_residual_norm_sums<TB>, dim3((unsigned)((b.p.D + 31) / 32), (unsigned)(kSums + std::min<int64_t>(gates, 1024))),
                         dim3(32, 32), 0, s, a, rows);
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
