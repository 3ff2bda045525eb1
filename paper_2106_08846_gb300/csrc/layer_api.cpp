// C entry points of the operators beside the product (include/bsr.h): argument
// checks and launches on the current device. They keep nothing between calls but the
// gated block's choice of tiles for the last few sizes, per thread, and the device's
// status word, until bsr_check_status.
#include <algorithm>
#include <cmath>

#include "bsr_internal.h"
#include "gated.h"
#include "gated_mma.h"
#include "host.h"
#include "residual_norm.h"

using namespace bsr;

namespace {

// The buffers of one call, checked together: alignment, where they live, and
// that no output overlaps another buffer, but for the input whose place it may
// take (`over`: the same address).
struct Buffers {
    struct One {
        const void *p;
        size_t bytes;
        const void *over[2];
        bool out;
    };
    One all[24];
    int n = 0;
    bool misaligned = false;

    void add(const void *p, size_t bytes, size_t align, bool out, const void *over0 = nullptr, const void *over1 = nullptr) {
        if (!p) return;
        misaligned |= reinterpret_cast<uintptr_t>(p) % align != 0;
        all[n++] = One{p, bytes, {over0, over1}, out};
    }
    void in(const void *p, size_t bytes, size_t align = 16) { add(p, bytes, align, false); }
    void out(const void *p, size_t bytes, size_t align = 16, const void *over0 = nullptr, const void *over1 = nullptr) {
        add(p, bytes, align, true, over0, over1);
    }
    bsr_status_t check() const {
        if (misaligned) return BSR_ERR_ALIGNMENT;
        for (int i = 0; i < n; i++) {
            if (!all[i].out) continue;
            for (int j = 0; j < n; j++) {
                if (j == i || (all[j].out && j < i)) continue;
                if (!overlaps(all[i].p, all[i].bytes, all[j].p, all[j].bytes)) continue;
                const bool same = all[i].p == all[j].p && all[i].bytes == all[j].bytes && !all[j].out;
                if (!same || (all[i].p != all[i].over[0] && all[i].p != all[i].over[1])) return BSR_ERR_INVALID_ARG;
            }
        }
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess) {
            cudaGetLastError();
            return BSR_ERR_CUDA;
        }
        for (int i = 0; i < n; i++)
            if (all[i].bytes && classify(all[i].p, device) != PK_DEVICE) return BSR_ERR_INVALID_ARG;
        return BSR_OK;
    }
};

bsr_status_t launched(cudaError_t e) {
    if (e == cudaSuccess) return BSR_OK;
    cudaGetLastError();
    return BSR_ERR_CUDA;
}

bool known(bsr_dtype_t dt) { return dt == BSR_F32 || dt == BSR_BF16; }
bool known(bsr_norm_t n) { return n == BSR_NORM_NONE || n == BSR_NORM_LAYER || n == BSR_NORM_RMS; }

// What all calls of the residual step check; with a gate, its rows too.
bsr_status_t check_residual(const bsr_residual_norm_t *p, int64_t N, bool gate) {
    if (!p || N < 0) return BSR_ERR_INVALID_ARG;
    if (!known(p->block_dt) || !known(p->stream_dt) || (p->block_dt == BSR_F32 && p->stream_dt != BSR_F32))
        return BSR_ERR_UNSUPPORTED;
    if (!known(p->post) || !known(p->pre)) return BSR_ERR_UNSUPPORTED;
    if (p->D < 1 || p->D > kRnMaxD || N > INT64_MAX / (8 * kRnMaxD)) return BSR_ERR_SHAPE;
    if (gate && p->gate_tokens < 1) return BSR_ERR_INVALID_ARG;
    // (a NaN is none of these)
    if ((p->post != BSR_NORM_NONE && !(p->post_eps >= 0.f)) || (p->pre != BSR_NORM_NONE && !(p->pre_eps >= 0.f)))
        return BSR_ERR_INVALID_ARG;
    if ((p->post == BSR_NORM_NONE && (p->post_w || p->post_b)) || (p->pre == BSR_NORM_NONE && (p->pre_w || p->pre_b)))
        return BSR_ERR_INVALID_ARG;
    return BSR_OK;
}

size_t gate_bytes(const bsr_residual_norm_t *p, int64_t N) {
    return (N == 0 ? 0 : (size_t)((N - 1) / p->gate_tokens) + 1) * p->D * dtype_size(p->block_dt);
}

void add_params(Buffers &b, const bsr_residual_norm_t *p) {
    for (const float *w : {p->scale, p->post_w, p->post_b, p->pre_w, p->pre_b}) b.in(w, (size_t)p->D * 4, 4);
}

constexpr int64_t kGatedMost = (int64_t)1 << 20;

bsr_status_t check_gated(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt) {
    if (!known(dt)) return BSR_ERR_UNSUPPORTED;
    if (N < 0) return BSR_ERR_INVALID_ARG;
    if (F < 1 || K < 1 || F > kGatedMost || K > kGatedMost || N > (int64_t)1 << 30 || N * std::max(F, K) >= (int64_t)1 << 38)
        return BSR_ERR_SHAPE;
    return BSR_OK;
}
bool known(bsr_act_t a) { return a >= BSR_ACT_SILU && a <= BSR_ACT_SIGMOID; }

}  // namespace

extern "C" {

bsr_status_t bsr_residual_norm(const bsr_residual_norm_t *p, const void *y, const void *h, const void *gate, void *h_out,
                               void *z, int64_t N, void *stream) {
    bsr_status_t st = check_residual(p, N, gate != nullptr);
    if (st != BSR_OK) return st;
    if ((p->pre == BSR_NORM_NONE) != (z == nullptr) || (!z && !h_out)) return N == 0 ? BSR_OK : BSR_ERR_INVALID_ARG;
    if (N == 0) return BSR_OK;
    if (!y) return BSR_ERR_INVALID_ARG;
    const size_t yb = (size_t)N * p->D * dtype_size(p->block_dt), hb = (size_t)N * p->D * dtype_size(p->stream_dt);
    Buffers b;
    b.in(y, yb);
    b.in(h, hb);
    if (gate) b.in(gate, gate_bytes(p, N));
    add_params(b, p);
    b.out(h_out, hb, 16, h);
    b.out(z, yb, 16, y);
    if ((st = b.check()) != BSR_OK) return st;
    return launched(launch_residual_norm(RnForward{*p, y, h, gate, h_out, z, N}, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_residual_norm_workspace(const bsr_residual_norm_t *p, int64_t N, size_t *bytes) {
    if (!bytes) return BSR_ERR_INVALID_ARG;
    *bytes = 0;
    const bsr_status_t st = check_residual(p, N, false);
    if (st == BSR_OK) *bytes = (size_t)residual_norm_workspace(*p, N);
    return st;
}

bsr_status_t bsr_residual_norm_backward(const bsr_residual_norm_t *p, const void *y, const void *h_out, const void *gate,
                                        const void *dh_out, const void *dz, void *dy, void *dh,
                                        const bsr_residual_norm_grads_t *grads, int64_t N, void *ws, size_t ws_bytes,
                                        void *stream) {
    bsr_status_t st = check_residual(p, N, gate != nullptr);
    if (st != BSR_OK) return st;
    bsr_residual_norm_grads_t g = {};
    if (grads) g = *grads;
    if ((g.dgate && !gate && N > 0) || (g.dscale && !p->scale) || (g.dpost_w && !p->post_w) || (g.dpost_b && !p->post_b) ||
        (g.dpre_w && !p->pre_w) || (g.dpre_b && !p->pre_b))
        return BSR_ERR_INVALID_ARG;
    const size_t yb = (size_t)N * p->D * dtype_size(p->block_dt), hb = (size_t)N * p->D * dtype_size(p->stream_dt);
    bsr_residual_norm_t q = *p;
    if (!gate) q.gate_tokens = 0;   // one run of all tokens
    const size_t need = (size_t)residual_norm_workspace(q, N);
    Buffers b;
    add_params(b, p);
    for (float *d : {g.dscale, g.dpost_w, g.dpost_b, g.dpre_w, g.dpre_b}) b.out(d, (size_t)p->D * 4, 4);
    if (N > 0) {
        const bool pre = p->pre != BSR_NORM_NONE;
        if (!y || pre != (dz != nullptr) || (pre && !h_out)) return BSR_ERR_INVALID_ARG;
        if (need > ws_bytes) return BSR_ERR_CAPACITY;
        if (need && !ws) return BSR_ERR_INVALID_ARG;
        b.in(y, yb);
        if (pre) b.in(h_out, hb);
        b.in(dh_out, hb);
        b.in(dz, yb);
        if (gate) b.in(gate, gate_bytes(p, N));
        b.out(dy, yb, 16, y, dz);
        b.out(dh, hb, 16, dh_out);
        if (g.dgate) b.out(g.dgate, gate_bytes(p, N));
        b.out(ws, need);
    }
    if ((st = b.check()) != BSR_OK) return st;
    const RnBackward a{q, y, h_out, gate, dh_out, dz, dy, dh, g, N, static_cast<float *>(ws)};
    return launched(launch_residual_norm_backward(a, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_gated_workspace(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, int backward, size_t *bytes) {
    if (!bytes) return BSR_ERR_INVALID_ARG;
    *bytes = 0;
    const bsr_status_t st = check_gated(N, F, K, dt);
    if (st == BSR_OK) *bytes = (size_t)gated_workspace(N, F, K, dt, backward != 0);
    return st;
}

bsr_status_t bsr_gated(const void *X, const void *Wg, const void *Wu, const float *bg, const float *bu, void *H, int64_t N,
                       int64_t F, int64_t K, bsr_dtype_t dt, bsr_act_t act, void *ws, size_t ws_bytes, void *stream) {
    bsr_status_t st = check_gated(N, F, K, dt);
    if (st != BSR_OK) return st;
    if (!known(act)) return BSR_ERR_UNSUPPORTED;
    if (N == 0) return BSR_OK;
    if (!X || !Wg || !Wu || !H) return BSR_ERR_INVALID_ARG;
    const size_t es = dtype_size(dt), need = (size_t)gated_workspace(N, F, K, dt, false);
    if (need > ws_bytes) return BSR_ERR_CAPACITY;
    if (need && !ws) return BSR_ERR_INVALID_ARG;
    Buffers b;
    b.in(X, (size_t)N * K * es);
    for (const void *w : {Wg, Wu}) b.in(w, (size_t)F * K * es);
    for (const float *v : {bg, bu}) b.in(v, (size_t)F * 4, 4);
    b.out(H, (size_t)N * F * es);
    b.out(ws, need);
    if ((st = b.check()) != BSR_OK) return st;
    GatedCall c = {X, Wg, Wu, bg, bu, N, F, K, dt, act, ws};
    c.H = H;
    return launched(launch_gated(c, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_gated_backward(const void *X, const void *Wg, const void *Wu, const float *bg, const float *bu,
                                const void *dH, void *dX, void *dWg, void *dWu, float *dbg, float *dbu, int64_t N, int64_t F,
                                int64_t K, bsr_dtype_t dt, bsr_act_t act, void *ws, size_t ws_bytes, void *stream) {
    bsr_status_t st = check_gated(N, F, K, dt);
    if (st != BSR_OK) return st;
    if (!known(act)) return BSR_ERR_UNSUPPORTED;
    if (!dWg != !dWu || (dbg && !bg) || (dbu && !bu)) return BSR_ERR_INVALID_ARG;
    const size_t es = dtype_size(dt), need = (size_t)gated_workspace(N, F, K, dt, true);
    Buffers b;
    for (void *w : {dWg, dWu}) b.out(w, (size_t)F * K * es);
    for (float *v : {dbg, dbu}) b.out(v, (size_t)F * 4, 4);
    if (N > 0) {
        if (!X || !Wg || !Wu || !dH) return BSR_ERR_INVALID_ARG;
        if (need > ws_bytes) return BSR_ERR_CAPACITY;
        if (need && !ws) return BSR_ERR_INVALID_ARG;
        b.in(X, (size_t)N * K * es);
        for (const void *w : {Wg, Wu}) b.in(w, (size_t)F * K * es);
        for (const float *v : {bg, bu}) b.in(v, (size_t)F * 4, 4);
        b.in(dH, (size_t)N * F * es);
        b.out(dX, (size_t)N * K * es);
        b.out(ws, need);
    }
    if ((st = b.check()) != BSR_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (N == 0) {   // sums of nothing
        for (void *w : {dWg, dWu})
            if (w && cudaMemsetAsync(w, 0, (size_t)F * K * es, s) != cudaSuccess) return launched(cudaErrorUnknown);
        for (float *v : {dbg, dbu})
            if (v && cudaMemsetAsync(v, 0, (size_t)F * 4, s) != cudaSuccess) return launched(cudaErrorUnknown);
        return BSR_OK;
    }
    GatedCall c = {X, Wg, Wu, bg, bu, N, F, K, dt, act, ws};
    c.dH = dH;
    c.dX = dX, c.dWg = dWg, c.dWu = dWu;
    c.dbg = dbg, c.dbu = dbu;
    return launched(launch_gated_backward(c, s));
}

bsr_status_t bsr_check_status(void) {
    int code = DEV_OK;
    const bsr_status_t st = launched(gated_mma_status(&code));
    return st == BSR_OK && code == DEV_TIMEOUT ? BSR_ERR_TIMEOUT : st;
}

}  // extern "C"
