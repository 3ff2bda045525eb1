// The gradients of the residual step, t = post(y), h' = alpha h + s * gate * t,
// z = pre(h'), in one pass over the data. With xh a normalised row, r its
// 1 / deviation and [..] for LayerNorm only:
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
// What bounds it: DRAM (y, h', dh', dz in, dy, dh out): 16384 x 1024, a bf16 block on an
// fp32 stream with a gate for 512 tokens, 61 us, 302 MB at 73% of the copy rate; 16384 x
// 768 fp32 65 us, 302 MB at 68%. Rows of more than 4096 features do not fit the
// registers that a thread has for them: 12 to 24%.
#include <algorithm>

#include "launch.cuh"
#include "residual_norm.cuh"

namespace bsr {

namespace {

constexpr int kSums = 5;   // parameter gradients: scale, post_w, post_b, pre_w, pre_b

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
template <typename TB, typename TS, int V, int L>
struct Token {
    Raw<TB, L> y[V], dz[V];
    Raw<TS, L> h[V], dh[V];
};
template <typename TB, typename TS, int V, int L>
__device__ __forceinline__ void load_token(const RnBackward &a, int64_t n, int D, int t, int NT, Token<TB, TS, V, L> &k) {
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
// registers (rows of more than 4096 features leave none for it). BIAS: whether there
// may be one. GATE: none, a row of it for runs of tokens, or one for each token.
// Without a gate all units are one. With one for each token, so they are: the gate
// goes into dH before Q and S, and its own gradient is the token's. With runs, what
// units add up to is held in shared memory (3 D values to a group), a thread's own
// features each. At 128 registers four CTAs of 128 threads share an
// SM: three, at 168, took 109 us for 16384 x 1024 of a bf16 block on an fp32 stream.
enum Gate : int { NONE = 0, OF_RUNS = 1, OF_TOKENS = 2 };

template <typename TB, typename TS, int V, int L, int THREADS, int GATE, bool BIAS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 4 : 1) k_residual_norm_backward(const __grid_constant__ RnBackwardArgs args) {
    constexpr bool KEEP = V == 1 && (L != ANY || THREADS == 128);
    extern __shared__ float4 unit_sums[];
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
    Run Q[V], S[V], dpre_w[V], dpre_b[V], pre_w[V], wc[V];   // wc: scale gate post_w
    // dscale, dpost_w, dpost_b (k) of run i
    float4 *const mine_s = unit_sums + (size_t)threadIdx.y * 3 * 2 * V * NT + t;
    auto unit_sum = [&](int k, int i, int h) -> float4 & { return mine_s[((k * V + i) * 2 + h) * NT]; };
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
    zero(Q), zero(S), zero(dpre_w), zero(dpre_b);
    if (KEEP) param(pre_w, a.p.pre_w, 1.f);
    if (GATE == OF_RUNS) {
#pragma unroll
        for (int k = 0; k < 3; k++)
#pragma unroll
            for (int i = 0; i < V; i++) unit_sum(k, i, 0) = unit_sum(k, i, 1) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // the first token of a unit (of a last gate row's units some may lie past the last
    // token: they add nothing, and nothing is read for them)
    auto first_of = [&](int64_t u) {
        const int64_t row = u / args.split.slices;
        return row * args.split.span + (u - row * args.split.slices) * args.split.len;
    };
    Token<TB, TS, V, L> next = {};
    if (KEEP && worker < args.split.units && first_of(worker) < a.N) load_token<TB, TS, V, L>(a, first_of(worker), D, t, NT, next);
    for (int64_t u = worker; u < args.split.units; u += args.split.workers) {
        const int64_t row = u / args.split.slices, n0 = first_of(u);
        const int64_t n1 = min(min(n0 + args.split.len, (row + 1) * args.split.span), a.N);
        const int64_t later = u + args.split.workers < args.split.units ? first_of(u + args.split.workers) : -1;
        const TB *const gate_row = GATE == OF_RUNS && a.gate ? static_cast<const TB *>(a.gate) + row * D : nullptr;
        auto times = [&](Run &r, const Run &s) {
#pragma unroll
            for (int j = 0; j < 4; j++) r.v[j] = mul2(r.v[j], s.v[j]);
        };
        param(wc, a.p.scale, 1.f);
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (gate_row) times(wc[i], load_const<TB, L>(gate_row, D, i, t, NT));
            if (a.p.post_w) times(wc[i], load_const<float, L>(a.p.post_w, D, i, t, NT));
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
            if (KEEP && after >= 0 && after < a.N) load_token<TB, TS, V, L>(a, after, D, t, NT, next);
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
            const F2 ry2 = all2(ry);
            if constexpr (GATE == OF_TOKENS) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const Run gate = load_const<TB, L>(static_cast<const TB *>(a.gate) + n * D, D, i, t, NT);
                    if (a.g.dgate) {   // scale t dH
                        Run d = y[i];
                        if (post) {
#pragma unroll
                            for (int j = 0; j < 4; j++) d.v[j] = mul2(d.v[j], ry2);
                        }
                        if (a.p.post_w) times(d, load_const<float, L>(a.p.post_w, D, i, t, NT));
                        if (a.p.post_b) {
                            const Run b = load_const<float, L>(a.p.post_b, D, i, t, NT);
#pragma unroll
                            for (int j = 0; j < 4; j++) d.v[j] = add2(d.v[j], b.v[j]);
                        }
                        if (a.p.scale) times(d, load_const<float, L>(a.p.scale, D, i, t, NT));
                        times(d, g[i]);
                        store_run<TB, L>(static_cast<TB *>(a.g.dgate) + n * D, D, i, t, NT, d);
                    }
                    times(g[i], gate);
                }
            }
            F2 sc = all2(0.f), sx = all2(0.f);
#pragma unroll
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const F2 yh = post ? mul2(y[i].v[j], ry2) : y[i].v[j];
                    Q[i].v[j] = fma2(g[i].v[j], yh, Q[i].v[j]);
                    if (BIAS) S[i].v[j] = add2(S[i].v[j], g[i].v[j]);
                    const F2 c = mul2(g[i].v[j], wc[i].v[j]);
                    if (post) {
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
        if (GATE == OF_RUNS || later < 0) {   // what the unit (else: all of the worker's) adds to the gradients
            float *const out = args.sums + worker * kSums * D;
#pragma unroll
            for (int i = 0; i < V; i++) {
                Run w = all_run(1.f), b = all_run(0.f), scale = all_run(1.f), gate = all_run(1.f), P, R;
                if (a.p.post_w) w = load_const<float, L>(a.p.post_w, D, i, t, NT);
                if (a.p.post_b) b = load_const<float, L>(a.p.post_b, D, i, t, NT);
                if (a.p.scale) scale = load_const<float, L>(a.p.scale, D, i, t, NT);
                if (gate_row) gate = load_const<TB, L>(gate_row, D, i, t, NT);
#pragma unroll
                for (int j = 0; j < 4; j++) P.v[j] = fma2(w.v[j], Q[i].v[j], mul2(b.v[j], S[i].v[j]));
                Run sg = scale;
                times(sg, gate);
                // dscale gate P, dpost_w scale gate Q, dpost_b scale gate S
#pragma unroll
                for (int k = 0; k < 3; k++) {
                    R = k == 0 ? P : k == 1 ? Q[i] : S[i];
                    times(R, k == 0 ? gate : sg);
                    if (GATE == OF_RUNS) {
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            float4 &s = unit_sum(k, i, h);
                            const float4 old = s;
                            R.v[2 * h] = add2(R.v[2 * h], pack2(old.x, old.y));
                            R.v[2 * h + 1] = add2(R.v[2 * h + 1], pack2(old.z, old.w));
                            const float2 lo = unpack2(R.v[2 * h]), hi = unpack2(R.v[2 * h + 1]);
                            s = make_float4(lo.x, lo.y, hi.x, hi.y);
                        }
                    }
                    if (later < 0 && (k == 0 ? a.g.dscale : k == 1 ? a.g.dpost_w : a.g.dpost_b)) store_run<float, L>(out + k * D, D, i, t, NT, R);
                }
                if (gate_row && a.g.dgate) {
                    times(P, scale);
                    if (args.gate_sums) store_run<float, L>(args.gate_sums + u * D, D, i, t, NT, P);
                    else store_run<TB, L>(static_cast<TB *>(a.g.dgate) + row * D, D, i, t, NT, P);
                }
                if (later < 0) {
                    if (a.g.dpre_w) store_run<float, L>(out + 3 * D, D, i, t, NT, dpre_w[i]);
                    if (a.g.dpre_b) store_run<float, L>(out + 4 * D, D, i, t, NT, dpre_b[i]);
                }
            }
            zero(Q), zero(S);
        }
    }
}

// Adds the workers' sums (blockIdx.y < kSums: one parameter's) or gate rows'
// slices (`rows` of them to a blockIdx.y), 32 features a CTA: 32 x 32 threads. The
// threads of a feature take its entries in turn; their sums are added in their order.
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

// Backward: runs of eight and threads of a group, and groups of a CTA.
struct RnShape {
    int V, NT, R;
};
RnShape shape_of(int64_t D) {
    RnShape s;
    s.V = D > 4096 ? 2 : 1;
    s.NT = (int)((D + 8 * s.V - 1) / (8 * s.V) + 31) / 32 * 32;
    s.R = s.NT == 32 ? 4 : s.NT == 64 ? 2 : 1;
    return s;
}

bool any_sum(const bsr_residual_norm_grads_t &g) { return g.dscale || g.dpost_w || g.dpost_b || g.dpre_w || g.dpre_b; }

// Whether the gate has a row for each token (wide rows have no kernel for it: runs of one).
bool of_tokens(const bsr_residual_norm_t &p) { return p.gate_tokens == 1 && shape_of(p.D).V == 1; }

RnSplit split_of(const bsr_residual_norm_t &p, int64_t N) {
    const RnShape sh = shape_of(p.D);
    // groups that an SM holds at once, by the backward kernel's registers
    // (128 a thread, and warps are given them four at a time)
    const int64_t most = (int64_t)sm_count() * std::max(1, 512 / ((sh.NT * sh.R + 127) / 128 * 128)) * sh.R;
    RnSplit s;
    s.span = p.gate_tokens > 0 && !of_tokens(p) ? std::min<int64_t>(p.gate_tokens, N) : N;
    const int64_t rows = (N + s.span - 1) / s.span, len = std::max<int64_t>(1, (N + most - 1) / most);
    s.slices = (s.span + len - 1) / len;
    s.len = (s.span + s.slices - 1) / s.slices;
    s.slices = (s.span + s.len - 1) / s.len;
    s.units = rows * s.slices;
    s.workers = std::min(s.units, most);
    return s;
}

template <typename TB, typename TS>
cudaError_t backward(const RnBackward &b, cudaStream_t s) {
    RnBackwardArgs a;
    a.b = b;
    const bool tokens = of_tokens(b.p);
    a.split = split_of(b.p, b.N);
    a.sums = b.ws;
    a.gate_sums = b.gate && b.g.dgate && !tokens && a.split.slices > 1 ? b.ws + a.split.workers * kSums * b.p.D : nullptr;
    const RnShape sh = shape_of(b.p.D);
    const int L = layout_of(b.p, sh.V, sh.NT), threads = sh.NT * sh.R;
    const dim3 block(sh.NT, sh.R), grid((unsigned)((a.split.workers + sh.R - 1) / sh.R));
    const bool gate = b.gate, bias = b.p.post_b || b.p.pre_b;
    // a kernel of its own for what is common: without a gate, and full rows without a bias
    using K = void (*)(RnBackwardArgs);
    K kernel;
    if (tokens && sh.V == 1) {
        kernel = threads <= 128 ? (L == FULL   ? k_residual_norm_backward<TB, TS, 1, FULL, 128, OF_TOKENS, true>
                                   : L == RUNS ? k_residual_norm_backward<TB, TS, 1, RUNS, 128, OF_TOKENS, true>
                                               : k_residual_norm_backward<TB, TS, 1, ANY, 128, OF_TOKENS, true>)
                                : (L != ANY ? k_residual_norm_backward<TB, TS, 1, RUNS, 512, OF_TOKENS, true>
                                                : k_residual_norm_backward<TB, TS, 1, ANY, 512, OF_TOKENS, true>);
    } else if (sh.V == 1 && threads <= 128) {
        if (L == FULL)
            kernel = gate ? (bias ? k_residual_norm_backward<TB, TS, 1, FULL, 128, OF_RUNS, true> : k_residual_norm_backward<TB, TS, 1, FULL, 128, OF_RUNS, false>)
                          : (bias ? k_residual_norm_backward<TB, TS, 1, FULL, 128, NONE, true> : k_residual_norm_backward<TB, TS, 1, FULL, 128, NONE, false>);
        else if (L == RUNS)
            kernel = gate ? k_residual_norm_backward<TB, TS, 1, RUNS, 128, OF_RUNS, true> : k_residual_norm_backward<TB, TS, 1, RUNS, 128, NONE, true>;
        else
            kernel = k_residual_norm_backward<TB, TS, 1, ANY, 128, OF_RUNS, true>;
    } else if (sh.V == 1) {
        kernel = L == ANY ? k_residual_norm_backward<TB, TS, 1, ANY, 512, OF_RUNS, true>
                 : gate       ? k_residual_norm_backward<TB, TS, 1, RUNS, 512, OF_RUNS, true>
                              : k_residual_norm_backward<TB, TS, 1, RUNS, 512, NONE, true>;
    } else if (threads <= 512) {
        kernel = L == ANY ? k_residual_norm_backward<TB, TS, 2, ANY, 512, OF_RUNS, true> : k_residual_norm_backward<TB, TS, 2, RUNS, 512, OF_RUNS, true>;
    } else {
        kernel = L == ANY ? k_residual_norm_backward<TB, TS, 2, ANY, 1024, OF_RUNS, true> : k_residual_norm_backward<TB, TS, 2, RUNS, 1024, OF_RUNS, true>;
    }
    const size_t smem = (size_t)threads * 3 * 2 * sh.V * 16;   // (up to 192 KB, at 16384 features)
    if (smem > 32 * 1024) {   // (beside 8 KB that every kernel has)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    cudaError_t e = launch_kernel(kernel, grid, block, smem, s, a);
    if (e != cudaSuccess || (!any_sum(b.g) && !a.gate_sums)) return e;
    int rows = 1;   // gate rows to a CTA: as many as leave a thread eight slices at most
    while (rows < 32 && 2 * rows * a.split.slices <= 256) rows *= 2;
    const int64_t gates = a.gate_sums ? (a.split.units / a.split.slices + rows - 1) / rows : 0;
    // in plain stream order: launched ahead of time, its CTAs and those of the call
    // after it took the SMs from one another (16384 x 768 fp32, calls back to back:
    // 103 us, so 72)
    k_residual_norm_sums<TB><<<dim3((unsigned)((b.p.D + 31) / 32), (unsigned)(kSums + std::min<int64_t>(gates, 1024))), dim3(32, 32), 0, s>>>(a, rows);
    return cudaGetLastError();
}

}  // namespace

int64_t residual_norm_workspace(const bsr_residual_norm_t &p, int64_t N) {
    if (N == 0) return 0;
    const RnSplit s = split_of(p, N);
    return (s.workers * kSums + (p.gate_tokens > 0 && !of_tokens(p) && s.slices > 1 ? s.units : 0)) * p.D * 4;
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
