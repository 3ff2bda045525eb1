// The gated feed-forward block
//
//   G = X Wg' + bg,  U = X Wu' + bu,  H = act(G) * U
//
// and its backward pass, which computes G and U again:
//
//   dG = dH U act'(G),  dU = dH act(G)
//   dX = dG Wg + dU Wu,  dWg = dG' X,  dWu = dU' X,  dbg = sum dG,  dbu = sum dU
//
// The products run on the tensor cores (gated_mma.cu). dG and dU stand side by
// side in the workspace as one bf16 matrix [N, 2 Fp], so that dX is one product
// over 2 Fp columns and dWg and dWu are one product of 2 Fp rows. Operands that
// the copy engine cannot read in place are laid out first: fp32 ones as three
// bf16 parts, bf16 ones padded whose rows do not start on 16-byte boundaries or
// whose weights are not whole groups of 32 rows.
#include <algorithm>

#include "bsr_internal.h"
#include "gated.h"
#include "gated_mma.h"
#include "launch.cuh"
#include "parts.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

// One matrix to lay out: rows x K values to parts of rows x Kp.
struct Source {
    const void *src;
    uint16_t *dst;
    int64_t rows, padded;   // rows, and those of a part (zeros past the matrix)
};
struct Sources {
    Source m[3];
    int64_t K, Kp;
    int vec;   // K is a multiple of 8 (rows start on 16-byte boundaries)
};

// Eight columns a thread; fp32: their three parts.
template <typename T>
__global__ void __launch_bounds__(256) k_lay_out(const __grid_constant__ Sources a) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const Source m = a.m[blockIdx.y];
    const int64_t eights = a.Kp / 8, total = m.padded * eights;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / eights, c = (i - row * eights) * 8;
        const T *src = static_cast<const T *>(m.src) + row * a.K + c;
        const bool there = row < m.rows;
        uint32_t w[PARTS][4];
        if constexpr (PARTS == 1) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const uint32_t v = there && c + j < a.K ? src[j] : (uint16_t)0;
                w[0][j / 2] = j & 1 ? w[0][j / 2] | v << 16 : v;
            }
        } else {
            float v[8];
            if (a.vec && there) {
                const float4 p = reinterpret_cast<const float4 *>(src)[0], q = reinterpret_cast<const float4 *>(src)[1];
                v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w, v[4] = q.x, v[5] = q.y, v[6] = q.z, v[7] = q.w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = there && c + j < a.K ? src[j] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 4; j++) {
                uint32_t p[3];
                parts_of(v[2 * j], v[2 * j + 1], p);
#pragma unroll
                for (int k = 0; k < 3; k++) w[k][j] = p[k];
            }
        }
#pragma unroll
        for (int p = 0; p < PARTS; p++)
            *reinterpret_cast<uint4 *>(m.dst + ((int64_t)p * m.padded + row) * a.Kp + c) = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
    }
}

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// The workspace of a call, and its products.
struct Plan {
    int parts, d_parts;   // bf16 matrices to an operand, and to dG and dU
    bool lay_out;
    int64_t Kp, Fp, Fr;   // padded sizes; the weights' rows
    int64_t x_at, wg_at, wu_at, d_at, sums_at, parts_at, bytes;
    GatedMma main, grads[2];   // dX; dWg and dWu
    GatedPlan main_plan, grads_plan;
};

// Up to this many tokens the weights' and their gradients' bytes bound the
// products, and a second part of dG and dU, which keeps 16 of their bits, costs
// next to nothing; a gradient of few tokens is a sum of few terms, in which
// roundings to 8 bits do not average out.
constexpr int64_t kFewTokens = 128;

Plan make_plan(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, bool backward, bool dx, bool dw) {
    Plan p = {};
    p.parts = dt == BSR_F32 ? 3 : 1;
    p.d_parts = dt == BSR_F32 ? 3 : N <= kFewTokens ? 2 : 1;
    p.lay_out = dt == BSR_F32 || K % 8 != 0 || F % 32 != 0;
    p.Fr = p.lay_out ? round_up(F, backward ? 64 : 32) : F;
    p.Kp = round_up(K, 8);
    p.Fp = backward ? round_up(F, 64) : F;
    auto take = [&](int64_t bytes) {
        const int64_t at = p.bytes;
        p.bytes += round_up(bytes, 256);
        return at;
    };
    if (p.lay_out) {
        p.x_at = take(p.parts * N * p.Kp * 2);
        p.wg_at = take(p.parts * p.Fr * p.Kp * 2);
        p.wu_at = take(p.parts * p.Fr * p.Kp * 2);
    }
    GatedMma &m = p.main;
    m.mode = backward ? GM_BACKWARD : GM_FORWARD;
    m.a.planes = p.parts;
    m.M = N, m.N = F, m.K = K, m.Fp = p.Fp;
    p.main_plan = plan_gated_mma(&m, 1, 0);
    if (!backward) return p;
    p.d_at = take(p.d_parts * N * 2 * p.Fp * 2);
    p.sums_at = take((N + 31) / 32 * 2 * 2 * p.Fp * 4);
    GatedMma &x = p.grads[0], &w = p.grads[1];
    x.mode = w.mode = GM_PRODUCT;
    x.a.planes = w.a.planes = m.d_planes = p.d_parts;
    x.M = N, x.N = K, x.K = 2 * p.Fp;
    x.b_seam = p.Fp;
    x.row_seam = x.out_rows = N;
    w.M = 2 * p.Fp, w.N = K, w.K = N;
    w.a_side = true;
    w.row_seam = p.Fp, w.out_rows = F;
    p.parts_at = p.bytes;
    if (dx || dw) {
        // (where only some gradients are wanted: within the workspace of a call for all)
        const int64_t most = dx && dw ? INT64_MAX : plan_gated_mma(&x, 2, INT64_MAX).part_bytes;
        p.grads_plan = plan_gated_mma(dx ? &x : &w, dx + dw, most);
        take(p.grads_plan.part_bytes);
    }
    return p;
}

// The plan of these sizes. Choosing tiles and parts takes 5 to 15 us, and a call
// needs its plan twice (for its workspace too), so each thread keeps the last few.
const Plan &plan_of(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, bool backward, bool dx = true, bool dw = true) {
    struct Kept {
        int64_t key[4];
        Plan plan;
    };
    constexpr int kKept = 16;
    thread_local Kept kept[kKept] = {};   // (N is at least 1 in a key)
    thread_local int next = 0;
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) cudaGetLastError();
    const int64_t key[4] = {N, F, K, (int64_t)device << 8 | (int64_t)dt << 3 | backward << 2 | dx << 1 | (int)dw};
    for (const Kept &k : kept)
        if (std::equal(key, key + 4, k.key)) return k.plan;
    Kept &k = kept[next];
    next = (next + 1) % kKept;
    k.plan = make_plan(N, F, K, dt, backward, dx, dw);
    std::copy(key, key + 4, k.key);
    return k.plan;
}

// The operands X, Wg and Wu as the tensor cores read them.
cudaError_t operands(const GatedCall &c, const Plan &p, Planes (&m)[3], cudaStream_t s) {
    const void *src[3] = {c.X, c.Wg, c.Wu};
    const int64_t rows[3] = {c.N, c.F, c.F}, padded[3] = {c.N, p.Fr, p.Fr}, at[3] = {p.x_at, p.wg_at, p.wu_at};
    Sources a;
    a.K = c.K, a.Kp = p.Kp;
    a.vec = c.K % 8 == 0;
    for (int i = 0; i < 3; i++) {
        uint16_t *dst = reinterpret_cast<uint16_t *>(static_cast<unsigned char *>(c.ws) + at[i]);
        a.m[i] = Source{src[i], dst, rows[i], padded[i]};
        m[i] = Planes{p.lay_out ? dst : static_cast<const uint16_t *>(src[i]), padded[i], p.lay_out ? p.Kp : c.K, p.lay_out ? p.Kp : c.K,
                      p.parts};
    }
    if (!p.lay_out) return cudaSuccess;
    const int64_t blocks = (std::max(c.N, c.F) * (p.Kp / 8) + 255) / 256;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, 2048), 3);
    return c.dt == BSR_F32 ? launch_kernel(k_lay_out<float>, grid, dim3(256), 0, s, a)
                           : launch_kernel(k_lay_out<uint16_t>, grid, dim3(256), 0, s, a);
}

}  // namespace

int64_t gated_workspace(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, bool backward) {
    if (N == 0 || (!backward && N <= kGatedFew)) return 0;
    return plan_of(N, F, K, dt, backward).bytes;
}

cudaError_t launch_gated(const GatedCall &c, cudaStream_t s) {
    if (c.N <= kGatedFew) return launch_gated_few(c, s);
    Plan p = plan_of(c.N, c.F, c.K, c.dt, false);
    Planes m[3];
    cudaError_t e = operands(c, p, m, s);
    if (e != cudaSuccess) return e;
    GatedMma &g = p.main;
    g.dt = c.dt;
    g.a = m[0], g.b0 = m[1], g.b1 = m[2];
    g.bg = c.bg, g.bu = c.bu;
    g.act = c.act;
    g.H = c.H;
    return launch_gated_mma(&g, p.main_plan, s);
}

cudaError_t launch_gated_backward(const GatedCall &c, cudaStream_t s) {
    const bool dx = c.dX, dw = c.dWg;
    Plan p = plan_of(c.N, c.F, c.K, c.dt, true, dx, dw);
    unsigned char *ws = static_cast<unsigned char *>(c.ws);
    Planes m[3];
    cudaError_t e = operands(c, p, m, s);
    if (e != cudaSuccess) return e;
    GatedMma &g = p.main, &x = p.grads[0], &w = p.grads[1];
    g.dt = x.dt = w.dt = c.dt;
    g.a = m[0], g.b0 = m[1], g.b1 = m[2];
    g.bg = c.bg, g.bu = c.bu;
    g.act = c.act;
    g.dH = c.dH;
    g.D = reinterpret_cast<uint16_t *>(ws + p.d_at);
    g.sums = c.dbg || c.dbu ? reinterpret_cast<float *>(ws + p.sums_at) : nullptr;
    e = launch_gated_mma(&g, p.main_plan, s);
    x.a = w.a = Planes{g.D, c.N, 2 * p.Fp, 2 * p.Fp, p.d_parts};
    x.b0 = m[1], x.b1 = m[2];
    x.out0 = x.out1 = c.dX;
    w.b0 = m[0];
    w.out0 = c.dWg, w.out1 = c.dWu;
    p.grads_plan.parts = reinterpret_cast<float *>(ws + p.parts_at);
    GatedBias b;
    if (g.sums) {
        b.sums = g.sums;
        b.rows = (c.N + 31) / 32 * (32 / sum_rows(p.main_plan));
        b.F = c.F, b.Fp = p.Fp;
        b.dbg = c.dbg, b.dbu = c.dbu;
    }
    if (e != cudaSuccess) return e;
    if (dx || dw) return launch_gated_mma(dx ? &x : &w, p.grads_plan, s, b);
    return launch_gated_bias(b, s);
}

}  // namespace bsr
