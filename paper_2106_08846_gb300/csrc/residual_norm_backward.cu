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
// 768 fp32 65 us, 302 MB at 68%. Rows of more than 4096 features are a cluster's, whose
// CTAs exchange their sums through distributed shared memory, which they wait for three
// times a row: 27 to 30%.
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
    int ctas;           // to a row
};

// The rows of a token as they lie in memory; GATE: its own gate too.
template <typename TB, typename TS, int L>
struct Token {
    Raw<TB, L> y, dz, gate;
    Raw<TS, L> h, dh;
};
template <bool GATE, typename TB, typename TS, int L>
__device__ __forceinline__ void load_token(const RnBackward &a, int64_t n, int D, int t, Token<TB, TS, L> &k) {
    const int64_t at = n * D;
    const bool at_end = row_at_end<L>(a.N - 1 - n, D);
    k.y = load_run<TB, L, false>(static_cast<const TB *>(a.y) + at, D, 0, t, 0, at_end);
    if (a.dh_out) k.dh = load_run<TS, L, false>(static_cast<const TS *>(a.dh_out) + at, D, 0, t, 0, at_end);
    if (a.p.pre != BSR_NORM_NONE) {
        k.h = load_run<TS, L, true>(static_cast<const TS *>(a.h_out) + at, D, 0, t, 0, at_end);
        k.dz = load_run<TB, L, false>(static_cast<const TB *>(a.dz) + at, D, 0, t, 0, at_end);
    }
    if (GATE) k.gate = load_run<TB, L, true>(static_cast<const TB *>(a.gate) + at, D, 0, t, 0, at_end);
}

// What a unit of tokens of one gate row adds to the parameters' gradients follows
// from two sums for each feature, Q = sum dH yh and S = sum dH: with t = yh w + b,
// sum t dH = w Q + b S, from which the gate's gradient is scale times and the
// scale's gate times that, and post_w's and post_b's are scale gate Q and
// scale gate S. A thread has eight features. THREADS: the most of a CTA. CLUSTER: a
// row is a cluster's (more than 4096 features). KEEP: the next token is on its way in
// registers (odd rows, which take more, leave none for it in large CTAs). BIAS: whether
// there may be one. GATE: none, a row of it for runs of tokens, or one for each token.
// Without a gate all units are one. With one for each token, so they are: the gate
// goes into dH before Q and S, and its own gradient is the token's. With runs, what
// units add up to is held in shared memory (24 values to a thread). At 128 registers
// four CTAs of 128 threads share an SM: three, at 168, took 109 us for 16384 x 1024 of
// a bf16 block on an fp32 stream.
enum Gate : int { NONE = 0, OF_RUNS = 1, OF_TOKENS = 2 };

template <typename TB, typename TS, int L, int THREADS, int GATE, bool BIAS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 4 : 1) k_residual_norm_backward(const __grid_constant__ RnBackwardArgs args) {
    constexpr bool KEEP = L != ANY || THREADS == 128;
    // a token's own gate is on its way with its rows, but for fp32 streams of bf16 blocks
    // and odd rows, where it would cost more spills than it hides (16384 x 1024 bf16 67.3
    // us without, 62.8 with; 8000 x 2048 of a bf16 block on an fp32 stream 71.9 and 81.9)
    constexpr bool GATE_AHEAD = GATE == OF_TOKENS && L != ANY && sizeof(TB) == sizeof(TS);
    extern __shared__ float4 unit_sums[];
    __shared__ float4 words[CLUSTER ? 2 : kMaxGroups][64];   // (CLUSTER: one group, and the CTAs' sums)
    const RnBackward &a = args.b;
    const int NT = blockDim.x, D = (int)a.p.D;
    const int t = (CLUSTER ? (int)ptx::cluster_rank() * NT : 0) + threadIdx.x;   // features 8 t ..
    const float over_d = 1.f / (float)D;
    GroupSum<THREADS == 128, CLUSTER> sum{words[threadIdx.y], NT, (int)threadIdx.y, 0};
    sum.init();
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t worker = CLUSTER ? blockIdx.x / (unsigned)args.ctas : (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool post = a.p.post != BSR_NORM_NONE, pre = a.p.pre != BSR_NORM_NONE;
    const bool post_layer = a.p.post == BSR_NORM_LAYER, pre_layer = a.p.pre == BSR_NORM_LAYER;
    Run Q, S, dpre_w, dpre_b, pre_w, wc;   // wc: scale gate post_w
    // dscale, dpost_w, dpost_b (k)
    float4 *const mine_s = unit_sums + (size_t)threadIdx.y * 3 * 2 * NT + threadIdx.x;
    auto unit_sum = [&](int k, int h) -> float4 & { return mine_s[(k * 2 + h) * NT]; };
    // a parameter, 1 where there is none; past the row's end 0: dH is not 0 there, but
    // what the LayerNorm's gradient takes out of the row, which no sum may take in again
    auto param = [&](Run &r, const float *p) {
        r = p ? load_param<L>(p, D, 0, t, 0) : row_run<L>(1.f, D, 0, t, 0);
    };
    Q = S = dpre_w = dpre_b = all_run(0.f);
    param(pre_w, a.p.pre_w);
    if (GATE == OF_RUNS) {
#pragma unroll
        for (int k = 0; k < 3; k++) unit_sum(k, 0) = unit_sum(k, 1) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // the first token of a unit (of a last gate row's units some may lie past the last
    // token: they add nothing, and nothing is read for them)
    auto first_of = [&](int64_t u) {
        const int64_t row = u / args.split.slices;
        return row * args.split.span + (u - row * args.split.slices) * args.split.len;
    };
    Token<TB, TS, L> next = {};
    if (KEEP && worker < args.split.units && first_of(worker) < a.N) load_token<GATE_AHEAD>(a, first_of(worker), D, t, next);
    for (int64_t u = worker; u < args.split.units; u += args.split.workers) {
        const int64_t row = u / args.split.slices, n0 = first_of(u);
        const int64_t n1 = min(min(n0 + args.split.len, (row + 1) * args.split.span), a.N);
        const int64_t later = u + args.split.workers < args.split.units ? first_of(u + args.split.workers) : -1;
        const int64_t gate_rows = L == ANY ? args.split.units / args.split.slices : 0;
        const TB *const gate_row = GATE == OF_RUNS && a.gate ? static_cast<const TB *>(a.gate) + row * D : nullptr;
        param(wc, a.p.scale);
        if (gate_row) times(wc, load_gate<TB, L>(gate_row, D, 0, t, 0, row_at_end<L>(gate_rows - 1 - row, D)));
        if (a.p.post_w) times(wc, load_param<L>(a.p.post_w, D, 0, t, 0));
        for (int64_t n = n0; n < n1; n++) {
            if (!KEEP) load_token<GATE_AHEAD>(a, n, D, t, next);
            Run y = next.y.run(), hh = next.h.run(), g = next.dh.run(), dz = next.dz.run();   // g: dH
            Run gate;
            if (GATE_AHEAD) gate = next.gate.run();
            const int64_t after = n + 1 < n1 ? n + 1 : later;
            if (KEEP && after >= 0 && after < a.N) load_token<GATE_AHEAD>(a, after, D, t, next);
            if (post_layer || pre_layer) {
                F2 sh = all2(0.f), sy = all2(0.f);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    sh = add2(sh, hh.v[j]);
                    sy = add2(sy, y.v[j]);
                }
                float m[2] = {both(sh), both(sy)};
                sum(m);
                if (pre_layer) centre<L>(hh, m[0] * over_d, D, 0, t, 0);
                if (post_layer) centre<L>(y, m[1] * over_d, D, 0, t, 0);
            }
            float ry = 1.f;
            if (pre) {
                F2 sh = all2(0.f), sy = all2(0.f), sa = all2(0.f), sx = all2(0.f);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const F2 aw = mul2(dz.v[j], pre_w.v[j]);
                    sy = fma2(y.v[j], y.v[j], sy);
                    sh = fma2(hh.v[j], hh.v[j], sh);
                    sa = add2(sa, aw);
                    sx = fma2(aw, hh.v[j], sx);
                    if (BIAS) dpre_b.v[j] = add2(dpre_b.v[j], dz.v[j]);
                }
                float s[4] = {both(sh), both(sy), both(sa), both(sx)};
                sum(s);
                if (post) ry = rsqrtf(fmaf(s[1], over_d, a.p.post_eps));
                // r (a - [mean a] - hh mean(a hh)), hh = r times the centred row
                const float r = rsqrtf(fmaf(s[0], over_d, a.p.pre_eps));
                const F2 r2 = all2(r), ma = all2(pre_layer ? -s[2] * over_d : 0.f), mx = all2(-s[3] * r * over_d);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const F2 xh = mul2(hh.v[j], r2);
                    dpre_w.v[j] = fma2(dz.v[j], xh, dpre_w.v[j]);
                    g.v[j] = fma2(r2, fma2(xh, mx, fma2(dz.v[j], pre_w.v[j], ma)), g.v[j]);
                }
            } else if (post) {
                F2 sy = all2(0.f);
#pragma unroll
                for (int j = 0; j < 4; j++) sy = fma2(y.v[j], y.v[j], sy);
                float s[1] = {both(sy)};
                sum(s);
                ry = rsqrtf(fmaf(s[0], over_d, a.p.post_eps));
            }
            if (a.dh) {
                Run out = all_run(a.p.alpha);
                times(out, g);
                store_run<TS, L, THREADS / 32>(static_cast<TS *>(a.dh) + n * D, D, 0, t, 0, out);
            }
            const F2 ry2 = all2(ry);
            if constexpr (GATE == OF_TOKENS) {
                if (!GATE_AHEAD) gate = load_gate<TB, L>(static_cast<const TB *>(a.gate) + n * D, D, 0, t, 0, row_at_end<L>(a.N - 1 - n, D));
                if (a.g.dgate) {   // scale t dH
                    Run d = y;
                    if (post) {
#pragma unroll
                        for (int j = 0; j < 4; j++) d.v[j] = mul2(d.v[j], ry2);
                    }
                    if (a.p.post_w) times(d, load_param<L>(a.p.post_w, D, 0, t, 0));
                    if (a.p.post_b) {
                        const Run b = load_param<L>(a.p.post_b, D, 0, t, 0);
#pragma unroll
                        for (int j = 0; j < 4; j++) d.v[j] = add2(d.v[j], b.v[j]);
                    }
                    if (a.p.scale) times(d, load_param<L>(a.p.scale, D, 0, t, 0));
                    times(d, g);
                    store_run<TB, L, THREADS / 32>(static_cast<TB *>(a.g.dgate) + n * D, D, 0, t, 0, d);
                }
                times(g, gate);
            }
            F2 sc = all2(0.f), sx = all2(0.f);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const F2 yh = post ? mul2(y.v[j], ry2) : y.v[j];
                Q.v[j] = fma2(g.v[j], yh, Q.v[j]);
                if (BIAS) S.v[j] = add2(S.v[j], g.v[j]);
                const F2 c = mul2(g.v[j], wc.v[j]);
                if (post) {
                    sc = add2(sc, c);
                    sx = fma2(c, yh, sx);
                }
                g.v[j] = c;
                y.v[j] = yh;
            }
            if (post) {
                float s[2] = {both(sc), both(sx)};
                sum(s);
                const F2 mc = all2(post_layer ? -s[0] * over_d : 0.f), mx = all2(-s[1] * over_d);
#pragma unroll
                for (int j = 0; j < 4; j++) g.v[j] = mul2(ry2, fma2(y.v[j], mx, add2(g.v[j], mc)));
            }
            if (a.dy) store_run<TB, L, THREADS / 32>(static_cast<TB *>(a.dy) + n * D, D, 0, t, 0, g);
        }
        if (GATE == OF_RUNS || later < 0) {   // what the unit (else: all of the worker's) adds to the gradients
            float *const out = args.sums + worker * kSums * D;
            Run w = all_run(1.f), b = all_run(0.f), scale = all_run(1.f), gate = all_run(1.f), P, R;
            if (a.p.post_w) w = load_param<L>(a.p.post_w, D, 0, t, 0);
            if (a.p.post_b) b = load_param<L>(a.p.post_b, D, 0, t, 0);
            if (a.p.scale) scale = load_param<L>(a.p.scale, D, 0, t, 0);
            if (gate_row) gate = load_gate<TB, L>(gate_row, D, 0, t, 0, row_at_end<L>(gate_rows - 1 - row, D));
#pragma unroll
            for (int j = 0; j < 4; j++) P.v[j] = fma2(w.v[j], Q.v[j], mul2(b.v[j], S.v[j]));
            Run sg = scale;
            times(sg, gate);
            // dscale gate P, dpost_w scale gate Q, dpost_b scale gate S
#pragma unroll
            for (int k = 0; k < 3; k++) {
                R = k == 0 ? P : k == 1 ? Q : S;
                times(R, k == 0 ? gate : sg);
                if (GATE == OF_RUNS) {
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        float4 &s = unit_sum(k, h);
                        const float4 old = s;
                        R.v[2 * h] = add2(R.v[2 * h], pack2(old.x, old.y));
                        R.v[2 * h + 1] = add2(R.v[2 * h + 1], pack2(old.z, old.w));
                        const float2 lo = unpack2(R.v[2 * h]), hi = unpack2(R.v[2 * h + 1]);
                        s = make_float4(lo.x, lo.y, hi.x, hi.y);
                    }
                }
                if (later < 0 && (k == 0 ? a.g.dscale : k == 1 ? a.g.dpost_w : a.g.dpost_b)) store_run<float, L, THREADS / 32>(out + k * D, D, 0, t, 0, R);
            }
            if (gate_row && a.g.dgate) {
                times(P, scale);
                if (args.gate_sums) store_run<float, L, THREADS / 32>(args.gate_sums + u * D, D, 0, t, 0, P);
                else store_run<TB, L, THREADS / 32>(static_cast<TB *>(a.g.dgate) + row * D, D, 0, t, 0, P);
            }
            if (later < 0) {
                if (a.g.dpre_w) store_run<float, L, THREADS / 32>(out + 3 * D, D, 0, t, 0, dpre_w);
                if (a.g.dpre_b) store_run<float, L, THREADS / 32>(out + 4 * D, D, 0, t, 0, dpre_b);
            }
            Q = S = all_run(0.f);
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

// Backward: CTAs to a row, threads of one that work on it, and rows of a CTA. A
// thread has eight features: with sixteen, a row to a CTA, the sums did not fit its
// registers (2000 x 8192 bf16 122 us, so 109; 1000 x 16384, a bf16 block on an fp32
// stream, 349, so 143). More and smaller CTAs pay more for each other's sums (CTAs of
// 256 threads: 112 and 238).
struct RnShape {
    int C, NT, R;
};
RnShape shape_of(int64_t D) {
    RnShape s;
    s.C = D > 8192 ? 4 : D > 4096 ? 2 : 1;
    s.NT = (int)((D + 8 * s.C - 1) / (8 * s.C) + 31) / 32 * 32;
    s.R = s.NT == 32 ? 4 : s.NT == 64 ? 2 : 1;
    return s;
}

bool any_sum(const bsr_residual_norm_grads_t &g) { return g.dscale || g.dpost_w || g.dpost_b || g.dpre_w || g.dpre_b; }

// Whether the gate has a row for each token.
bool of_tokens(const bsr_residual_norm_t &p) { return p.gate_tokens == 1; }

RnSplit split_of(const bsr_residual_norm_t &p, int64_t N) {
    const RnShape sh = shape_of(p.D);
    // groups that run at once, by the backward kernel's registers (128 a thread, and
    // warps are given them four at a time); clusters of four do not fill all parts of
    // the GPU (36 of 38)
    const int64_t sms = sm_count();
    const int64_t most = sh.C == 1 ? sms * std::max(1, 512 / ((sh.NT * sh.R + 127) / 128 * 128)) * sh.R
                                   : std::max<int64_t>(1, sh.C == 2 ? sms / 2 : sms / 4 * 15 / 16);
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
    const int L = layout_of(b.p, sh.C, sh.NT), threads = sh.NT * sh.R;
    const dim3 block(sh.NT, sh.R), grid((unsigned)((a.split.workers + sh.R - 1) / sh.R * sh.C));
    a.ctas = sh.C;
    const bool gate = b.gate, bias = b.p.post_b || b.p.pre_b;
    // a kernel of its own for what is common: without a gate, and full rows without a bias
    using K = void (*)(RnBackwardArgs);
    K kernel;
    if (sh.C > 1) {
        kernel = tokens ? (L == ANY ? k_residual_norm_backward<TB, TS, ANY, 512, OF_TOKENS, true, true>
                                    : k_residual_norm_backward<TB, TS, RUNS, 512, OF_TOKENS, true, true>)
                        : (L == ANY ? k_residual_norm_backward<TB, TS, ANY, 512, OF_RUNS, true, true>
                                    : k_residual_norm_backward<TB, TS, RUNS, 512, OF_RUNS, true, true>);
    } else if (tokens) {
        kernel = threads <= 128 ? (L == FULL   ? k_residual_norm_backward<TB, TS, FULL, 128, OF_TOKENS, true, false>
                                   : L == RUNS ? k_residual_norm_backward<TB, TS, RUNS, 128, OF_TOKENS, true, false>
                                               : k_residual_norm_backward<TB, TS, ANY, 128, OF_TOKENS, true, false>)
                                : (L != ANY ? k_residual_norm_backward<TB, TS, RUNS, 512, OF_TOKENS, true, false>
                                            : k_residual_norm_backward<TB, TS, ANY, 512, OF_TOKENS, true, false>);
    } else if (threads <= 128) {
        if (L == FULL)
            kernel = gate ? (bias ? k_residual_norm_backward<TB, TS, FULL, 128, OF_RUNS, true, false> : k_residual_norm_backward<TB, TS, FULL, 128, OF_RUNS, false, false>)
                          : (bias ? k_residual_norm_backward<TB, TS, FULL, 128, NONE, true, false> : k_residual_norm_backward<TB, TS, FULL, 128, NONE, false, false>);
        else if (L == RUNS)
            kernel = gate ? k_residual_norm_backward<TB, TS, RUNS, 128, OF_RUNS, true, false> : k_residual_norm_backward<TB, TS, RUNS, 128, NONE, true, false>;
        else
            kernel = k_residual_norm_backward<TB, TS, ANY, 128, OF_RUNS, true, false>;
    } else {
        kernel = L == ANY ? k_residual_norm_backward<TB, TS, ANY, 512, OF_RUNS, true, false>
                 : gate   ? k_residual_norm_backward<TB, TS, RUNS, 512, OF_RUNS, true, false>
                          : k_residual_norm_backward<TB, TS, RUNS, 512, NONE, true, false>;
    }
    const size_t smem = (size_t)threads * 3 * 2 * 16;   // (up to 48 KB)
    if (smem > 24 * 1024) {   // (beside up to 24 KB that a kernel has)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    cudaError_t e = launch_clusters(kernel, sh.C, grid, block, smem, s, a);
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
