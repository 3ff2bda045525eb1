// C entry points of expert layers and 8-bit products (include/bsr.h): argument checks
// and launches on the current device. They keep nothing between calls but the device's
// status word, until bsr_check_status.
#include <algorithm>

#include "buffers.h"
#include "experts.h"
#include "fp8.h"

using namespace bsr;

namespace {

using bsr::known;
bool known(bsr_fp8_t t) { return t == BSR_E4M3 || t == BSR_E5M2; }

constexpr int64_t kMostSide = (int64_t)1 << 20, kMostValues = (int64_t)1 << 38;

bool sizes(int64_t N, int k, int E, int align) {
    return N >= 0 && N < (int64_t)1 << 30 && k >= 1 && k <= kMostChoices && E >= 1 && E <= kMostExperts && align >= 1 && align <= kMostAlign;
}
// Rows that N tokens may take; sizes that are known to be good.
int64_t capacity(int64_t N, int k, int E, int align) {
    const int64_t pairs = N * k;
    return (pairs + std::min<int64_t>(E, pairs) * (align - 1)) / align * align;
}

bsr_status_t check_experts(const bsr_experts_t *p) {
    if (!p || p->N < 0) return BSR_ERR_INVALID_ARG;
    if (!sizes(p->N, p->k, p->E, p->align) || p->R > INT32_MAX || capacity(p->N, p->k, p->E, p->align) > INT32_MAX) return BSR_ERR_SHAPE;
    if (p->R < capacity(p->N, p->k, p->E, p->align)) return BSR_ERR_CAPACITY;
    if (p->N > 0 && (!p->offsets || !p->place || !p->source)) return BSR_ERR_INVALID_ARG;
    return BSR_OK;
}
bsr_status_t check_rows(const bsr_experts_t *p, int64_t D, bsr_dtype_t dt) {
    const bsr_status_t st = check_experts(p);
    if (st != BSR_OK) return st;
    if (!known(dt)) return BSR_ERR_UNSUPPORTED;
    if (D < 1 || D > kMostSide || D * std::max(p->R, p->N) >= kMostValues) return BSR_ERR_SHAPE;
    return BSR_OK;
}
void add_order(Buffers &b, const bsr_experts_t *p, bool out) {
    b.add(p->offsets, (size_t)(p->E + 1) * 4, 4, out);
    b.add(p->place, (size_t)(p->N * p->k) * 4, 4, out);
    b.add(p->source, (size_t)p->R * 4, 4, out);
}

bsr_status_t check_matrix(const bsr_fp8_matrix_t *m) {
    if (m->batch < 0 || m->rows < 0 || m->cols < 0) return BSR_ERR_INVALID_ARG;
    if (!known(m->type)) return BSR_ERR_UNSUPPORTED;
    if (m->tile != 1 && m->tile != kFp8Block) return BSR_ERR_UNSUPPORTED;
    if (m->batch > 65535 || m->rows >= (int64_t)1 << 31 || m->cols >= (int64_t)1 << 31) return BSR_ERR_SHAPE;
    const int64_t ld = fp8_blocks(m->cols) * kFp8Block;
    if (ld > 0 && m->rows > kMostValues / ld) return BSR_ERR_SHAPE;
    if (m->rows * ld > 0 && m->batch > kMostValues / (m->rows * ld)) return BSR_ERR_SHAPE;
    return BSR_OK;
}
void add_matrix(Buffers &b, const bsr_fp8_matrix_t *m, bool out) {
    b.add(m->q, (size_t)fp8_bytes(*m), 16, out);
    b.add(m->exponent, (size_t)fp8_exponents(*m), 16, out);
    if (out) b.add(m->scale, (size_t)fp8_scales(*m) * 4, 4, out);
}

// What both calls of the product check.
bsr_status_t check_product(const bsr_fp8_matrix_t *a, const bsr_fp8_matrix_t *b, bsr_dtype_t dt, bsr_group_t group, int64_t groups) {
    if (!a || !b) return BSR_ERR_INVALID_ARG;
    for (const bsr_fp8_matrix_t *m : {a, b}) {
        const bsr_status_t st = check_matrix(m);
        if (st != BSR_OK) return st;
    }
    if (!known(dt) || (group != BSR_GROUP_NONE && group != BSR_GROUP_ROWS && group != BSR_GROUP_COLUMNS)) return BSR_ERR_UNSUPPORTED;
    if (group != BSR_GROUP_NONE && (groups < 1 || groups > kMostExperts)) return BSR_ERR_SHAPE;
    if (a->cols != b->cols || a->batch != 1 || b->batch != (group == BSR_GROUP_ROWS ? groups : 1)) return BSR_ERR_SHAPE;
    const int64_t each = group == BSR_GROUP_COLUMNS ? groups : 1;
    if (b->rows > 0 && a->rows > kMostValues / b->rows / each) return BSR_ERR_SHAPE;
    return BSR_OK;
}

}  // namespace

extern "C" {

bsr_status_t bsr_expert_capacity(int64_t N, int k, int E, int align, int64_t *rows) {
    if (!rows || N < 0) return BSR_ERR_INVALID_ARG;
    *rows = 0;
    if (!sizes(N, k, E, align) || capacity(N, k, E, align) > INT32_MAX) return BSR_ERR_SHAPE;
    *rows = capacity(N, k, E, align);
    return BSR_OK;
}

bsr_status_t bsr_expert_order(const bsr_experts_t *p, const int32_t *experts, void *stream) {
    bsr_status_t st = check_experts(p);
    if (st != BSR_OK) return st;
    if (!p->offsets || (p->N > 0 && !experts) || (p->R > 0 && !p->source)) return BSR_ERR_INVALID_ARG;
    Buffers b;
    add_order(b, p, true);
    b.in(experts, (size_t)(p->N * p->k) * 4, 4);
    if ((st = b.check()) != BSR_OK) return st;
    return launched(launch_expert_order(*p, experts, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_expert_rows(const bsr_experts_t *p, const void *X, void *Xs, int64_t D, bsr_dtype_t dt, void *stream) {
    bsr_status_t st = check_rows(p, D, dt);
    if (st != BSR_OK) return st;
    if (p->N == 0) return BSR_OK;
    if (!X || !Xs) return BSR_ERR_INVALID_ARG;
    const size_t row = (size_t)D * dtype_size(dt);
    Buffers b;
    add_order(b, p, false);
    b.in(X, p->N * row);
    b.out(Xs, p->R * row);
    if ((st = b.check()) != BSR_OK) return st;
    return launched(launch_expert_rows(*p, X, Xs, D, dt, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_expert_sum(const bsr_experts_t *p, const void *Ys, const float *weights, void *Y, int64_t D, bsr_dtype_t dt,
                            void *stream) {
    bsr_status_t st = check_rows(p, D, dt);
    if (st != BSR_OK) return st;
    if (p->N == 0) return BSR_OK;
    if (!Ys || !Y) return BSR_ERR_INVALID_ARG;
    const size_t row = (size_t)D * dtype_size(dt);
    Buffers b;
    add_order(b, p, false);
    b.in(Ys, p->R * row);
    b.in(weights, (size_t)(p->N * p->k) * 4, 4);
    b.out(Y, p->N * row);
    if ((st = b.check()) != BSR_OK) return st;
    return launched(launch_expert_sum(*p, Ys, weights, Y, D, dt, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_expert_sum_backward(const bsr_experts_t *p, const void *Ys, const float *weights, const void *dY, void *dYs,
                                     float *dweights, int64_t D, bsr_dtype_t dt, void *stream) {
    bsr_status_t st = check_rows(p, D, dt);
    if (st != BSR_OK) return st;
    if (p->N == 0) return BSR_OK;
    if (!dY || (dweights && (!weights || !Ys))) return BSR_ERR_INVALID_ARG;
    if (!dYs && !dweights) return BSR_OK;
    const size_t row = (size_t)D * dtype_size(dt);
    Buffers b;
    add_order(b, p, false);
    if (dweights) b.in(Ys, p->R * row);
    b.in(weights, (size_t)(p->N * p->k) * 4, 4);
    b.in(dY, p->N * row);
    b.out(dYs, p->R * row);
    b.out(dweights, (size_t)(p->N * p->k) * 4, 4);
    if ((st = b.check()) != BSR_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!weights) return launched(launch_expert_rows(*p, dY, dYs, D, dt, s));   // the rows themselves
    return launched(launch_expert_sum_backward(*p, Ys, weights, dY, dYs, dweights, D, dt, s));
}

bsr_status_t bsr_fp8_quantize(const void *x, bsr_dtype_t dt, const bsr_fp8_matrix_t *rows, const bsr_fp8_matrix_t *columns,
                              const int32_t *used, void *stream) {
    const bsr_fp8_matrix_t *m = rows ? rows : columns;
    if (!m) return BSR_ERR_INVALID_ARG;
    for (const bsr_fp8_matrix_t *c : {rows, columns}) {
        const bsr_status_t st = c ? check_matrix(c) : BSR_OK;
        if (st != BSR_OK) return st;
    }
    if (!known(dt)) return BSR_ERR_UNSUPPORTED;
    const int64_t R = rows ? rows->rows : columns->cols, C = rows ? rows->cols : columns->rows;
    if (rows && columns &&
        (columns->rows != C || columns->cols != R || rows->batch != columns->batch || rows->tile != columns->tile || rows->type != columns->type))
        return BSR_ERR_SHAPE;
    if (used && m->batch != 1) return BSR_ERR_SHAPE;
    if (m->batch == 0 || R == 0 || C == 0) return BSR_OK;
    if (!x) return BSR_ERR_INVALID_ARG;
    Buffers b;
    b.in(x, (size_t)(m->batch * R * C) * dtype_size(dt));
    b.in(used, 4, 4);
    for (const bsr_fp8_matrix_t *c : {rows, columns}) {
        if (!c) continue;
        if (!c->q || !c->exponent) return BSR_ERR_INVALID_ARG;
        add_matrix(b, c, true);
    }
    const bsr_status_t st = b.check();
    if (st != BSR_OK) return st;
    return launched(launch_fp8_quantize(x, dt, m->batch, R, C, m->tile, m->type, rows, columns, used, static_cast<cudaStream_t>(stream)));
}

bsr_status_t bsr_fp8_product_workspace(const bsr_fp8_matrix_t *a, const bsr_fp8_matrix_t *b, bsr_dtype_t dt, bsr_group_t group,
                                       int64_t groups, size_t *bytes) {
    if (!bytes) return BSR_ERR_INVALID_ARG;
    *bytes = 0;
    const bsr_status_t st = check_product(a, b, dt, group, groups);
    if (st == BSR_OK) *bytes = (size_t)fp8_product_workspace(Fp8Product{*a, *b, nullptr, nullptr, dt, group, nullptr, (int)groups, nullptr});
    return st;
}

bsr_status_t bsr_fp8_product(const bsr_fp8_matrix_t *a, const bsr_fp8_matrix_t *b, const float *bias, void *Y, bsr_dtype_t dt,
                             bsr_group_t group, const int32_t *offsets, int64_t groups, void *ws, size_t ws_bytes, void *stream) {
    bsr_status_t st = check_product(a, b, dt, group, groups);
    if (st != BSR_OK) return st;
    if ((group == BSR_GROUP_NONE) != (offsets == nullptr) || (bias && group == BSR_GROUP_COLUMNS)) return BSR_ERR_INVALID_ARG;
    const int64_t each = group == BSR_GROUP_COLUMNS ? groups : 1;
    if (a->rows == 0 || b->rows == 0) return BSR_OK;
    if (!Y || (a->cols > 0 && (!a->q || !a->exponent || !b->q || !b->exponent))) return BSR_ERR_INVALID_ARG;
    Fp8Product p = {*a, *b, bias, Y, dt, group, offsets, (int)groups, static_cast<float *>(ws)};
    const size_t need = (size_t)fp8_product_workspace(p);
    if (need > ws_bytes) return BSR_ERR_CAPACITY;
    if (need && !ws) return BSR_ERR_INVALID_ARG;
    Buffers l;
    add_matrix(l, a, false);
    add_matrix(l, b, false);
    l.in(bias, (size_t)(b->batch * b->rows) * 4, 4);
    l.in(offsets, (size_t)(groups + 1) * 4, 4);
    l.out(Y, (size_t)(each * a->rows * b->rows) * dtype_size(dt));
    if (need) l.out(ws, need);
    if ((st = l.check()) != BSR_OK) return st;
    return launched(launch_fp8_product(p, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
