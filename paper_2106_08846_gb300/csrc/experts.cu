// Tokens sorted by expert and added up again with the router's weights.
//
//   c_e = #{(n, j): x_nj = e},  o_0 = 0,  o_{e+1} = o_e + align ceil(c_e / align)
//   place[n, j] = o_e + the rank of (n, j) among the choices of e = x_nj
//   Xs[place[n, j]] = X[n];   Y[n] = sum_j w_nj Ys[place[n, j]]
//
// Order: one launch. A warp takes a contiguous run of the choices twice, 32 at a
// time (eight times 32 on their way): lanes with equal experts find each other, the first adds their number to
// the warp's count of that expert (no atomics: the order is by index, the same in
// every call). Between the passes the counts of the warps, and of a cluster's CTAs
// through distributed shared memory, become first rows.
//
// Rows and sums: one pass over the data, a warp to 2 KB of a token's row (16-byte words; sums of
// one choice: 4 KB, of two: 1 KB; backward: to a choice's whole row).
//
// What bounds them: DRAM, and the order the choices' bits (16384 tokens of 4 of 64
// experts 8.8 us, a ballot a bit and choice, on 16 SMs). 16384 x 1024 bf16: rows of 4
// choices 29.3 us, 168 MB at 84% of the copy rate; their sum 30, 83%; the sum's gradients for 2 choices
// 31, 80%. 9920 x 1344 fp32, 2 choices: 29.9 us, 79%, bf16 12.0, 98%, their gradients 41.8, 94%, and 25.0, 78%. One token: order 3.6, rows 1.5,
// launches and a read's latency. Rows that are no multiples of 16 bytes go in smaller words
// (8192 x 1023 bf16, 2 choices: order and rows 16, their sum 15 us, 48%).
//
// Inputs are read by plain loads, none by the read-only path: a kernel starts while the
// one before it, whose output they may be, still runs.
#include <algorithm>
#include <atomic>

#include "elem.cuh"
#include "experts.h"
#include "launch.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

constexpr int kOrderThreads = 1024, kWarps = kOrderThreads / 32, kAtOnce = 8;

__device__ __forceinline__ int32_t load_cluster(uint32_t addr) {
    int32_t v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// The lanes with the same expert (below 2^bits) as this one; none for lanes without one
// (-1). A bit at a time: the instruction that compares values takes as long as there are
// different ones (65536 choices of 64 experts: 16.5 us for the whole kernel).
template <int BITS>
__device__ __forceinline__ uint32_t lanes_with(int32_t x) {
    uint32_t same = __ballot_sync(0xffffffffu, x >= 0);
#pragma unroll
    for (int b = 0; b < BITS; b++) {
        const int32_t mine = x << (31 - b) >> 31;   // the bit, in all bits
        same &= ~(__ballot_sync(0xffffffffu, mine < 0) ^ (uint32_t)mine);
    }
    return x >= 0 ? same : 0;
}

// Dynamic shared memory: counts[warps][E], then totals of this CTA [E], of all [E], first rows [E].
// BITS: of experts' numbers.
template <int BITS>
__global__ void __launch_bounds__(kOrderThreads, 1) k_expert_order(const __grid_constant__ bsr_experts_t p, const int32_t *experts,
                                                                   unsigned ctas) {
    extern __shared__ int32_t words[];
    __shared__ int32_t sums[kWarps];
    const int E = p.E, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t *count = words, *mine = words + kWarps * E, *all = mine + E, *first = all + E;
    const uint32_t rank = ctas > 1 ? ptx::cluster_rank() : 0;
    const int64_t pairs = p.N * p.k, warps = (int64_t)ctas * kWarps, per = ((pairs + warps - 1) / warps + 31) / 32 * 32;
    const int64_t lo = min(pairs, (rank * kWarps + warp) * per), hi = min(pairs, lo + per);
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int i = threadIdx.x; i < kWarps * E; i += kOrderThreads) count[i] = 0;
    __syncthreads();
    int32_t x[kAtOnce];   // (kept for the second pass if they are all)
    auto fetch = [&](int64_t i0) {
#pragma unroll
        for (int t = 0; t < kAtOnce; t++) {
            const int64_t i = i0 + 32 * t + lane;
            const int32_t v = i < hi ? experts[i] : -1;
            x[t] = (uint32_t)v < (uint32_t)E ? v : -1;
        }
    };
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kAtOnce) {
        fetch(i0);
#pragma unroll
        for (int t = 0; t < kAtOnce; t++) {
            if (i0 + 32 * t >= hi) break;
            const uint32_t same = lanes_with<BITS>(x[t]);
            if (x[t] >= 0 && lane == __ffs((int)same) - 1) count[warp * E + x[t]] += __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    const int e = threadIdx.x;
    if (e < E) {   // the warps' counts become what the warps before have
        int32_t run = 0;
#pragma unroll 8
        for (int w = 0; w < kWarps; w++) {
            const int32_t c = count[w * E + e];
            count[w * E + e] = run;
            run += c;
        }
        mine[e] = run;
    }
    if (ctas > 1) ptx::cluster_barrier();
    else __syncthreads();
    int32_t before = 0, total = 0;
    if (e < E) {
        for (uint32_t r = 0; r < ctas; r++) {
            const int32_t c = r == rank ? mine[e] : load_cluster(ptx::map_to_cta(mine + e, r));
            before += r < rank ? c : 0;
            total += c;
        }
    }
    const int32_t padded = (int32_t)(((uint32_t)total + (uint32_t)p.align - 1) / (uint32_t)p.align * (uint32_t)p.align);   // (below 2^31, not so the sum)
    int32_t upto = padded;   // inclusive sums: of the warp's experts, then of the warps'
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        int32_t v = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int32_t u = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += u;
        }
        sums[lane] = v;
    }
    __syncthreads();
    const int32_t used = sums[kWarps - 1];
    if (e < E) {
        const int32_t at = upto - padded + (warp ? sums[warp - 1] : 0);
        all[e] = total;
        first[e] = at;
#pragma unroll 8
        for (int w = 0; w < kWarps; w++) count[w * E + e] += at + before;
        if (rank == 0) p.offsets[e] = at;
    }
    if (rank == 0 && threadIdx.x == 0) p.offsets[E] = used;
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kAtOnce) {
        if (hi - lo > 32 * kAtOnce) fetch(i0);
#pragma unroll
        for (int t = 0; t < kAtOnce; t++) {
            if (i0 + 32 * t >= hi) break;
            const int64_t i = i0 + 32 * t + lane;
            const uint32_t same = lanes_with<BITS>(x[t]);
            const int32_t row = x[t] >= 0 ? count[warp * E + x[t]] + __popc(same & ((1u << lane) - 1)) : -1;
            __syncwarp();
            if (x[t] >= 0 && lane == __ffs((int)same) - 1) count[warp * E + x[t]] += __popc(same);
            __syncwarp();
            if (i < hi) p.place[i] = row;
            if (row >= 0) p.source[row] = (int32_t)i;
        }
    }
    // rows that nobody was sent to: behind an expert's, and behind the last one's
    for (int f = (int)rank * kWarps + warp; f < E; f += (int)ctas * kWarps) {
        const int64_t end = f + 1 < E ? first[f + 1] : used;   // (rows up to 2^31 - 1: past them 32 bits end)
        for (int64_t r = (int64_t)first[f] + all[f] + lane; r < end; r += 32) p.source[r] = -1;
    }
    for (int64_t r = used + (int64_t)rank * kOrderThreads + threadIdx.x; r < p.R; r += (int64_t)ctas * kOrderThreads) p.source[r] = -1;
    if (ctas > 1) ptx::cluster_barrier();   // nobody reads this CTA's counts any more
}

// ---- rows in words of 2 to 16 bytes, as their addresses allow

template <typename T, typename W>
struct Word {
    static constexpr int n = sizeof(W) / sizeof(T);
    union {
        W w;
        T v[n];
    };
};

// w = *p where `on` (else w has no value), without a branch: with one, the compiler puts each load where it
// is used, one behind the other (16384 x 1024 bf16, 4 choices: 42 us for 29.5).
__device__ __forceinline__ void load_if(uint4 &w, const uint4 *p, bool on) {
    asm volatile("{\n.reg .pred on;\nsetp.ne.u32 on, %5, 0;\n@on ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                 : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(p), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void load_if(uint2 &w, const uint2 *p, bool on) {
    asm volatile("{\n.reg .pred on;\nsetp.ne.u32 on, %3, 0;\n@on ld.global.v2.u32 {%0, %1}, [%2];\n}"
                 : "=r"(w.x), "=r"(w.y) : "l"(p), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void load_if(uint32_t &w, const uint32_t *p, bool on) {
    asm volatile("{\n.reg .pred on;\nsetp.ne.u32 on, %2, 0;\n@on ld.global.u32 %0, [%1];\n}" : "=r"(w) : "l"(p), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void load_if(uint16_t &w, const uint16_t *p, bool on) {
    asm volatile("{\n.reg .pred on;\nsetp.ne.u32 on, %2, 0;\n@on ld.global.u16 %0, [%1];\n}" : "=h"(w) : "l"(p), "r"((uint32_t)on) : "memory");
}

// Of a row, a lane holds at once (words of 2 bytes, 8192 x 1023 bf16 of one choice: four 17.9 us, eight 13.7).
template <typename W>
constexpr int kWords = sizeof(W) == 16 ? 4 : 8;

__device__ __forceinline__ int32_t row_of(const bsr_experts_t &p, int64_t pair) {
    const int32_t r = p.place[pair];
    return r >= 0 && r < p.R ? r : -1;   // (rows out of range: not sent)
}

// Zeros in the rows below offsets[E] that nobody was sent to: unit u is 2 KB of eight rows.
// (Whole rows, 32 to a warp, took 16 us where 17 experts' 2000 rows of 7 KB are zeros.)
constexpr int kZeroRows = 8;
template <typename W>
__device__ __forceinline__ void zero_rows(const bsr_experts_t &p, W *out, int64_t words, int64_t u, int64_t parts) {
    const int lane = threadIdx.x & 31;
    const int64_t first = u / parts * kZeroRows, at = u % parts * 32 * kWords<W> + lane;
    const int64_t used = min((int64_t)p.offsets[p.E], p.R), r = first + lane;
    uint32_t mask = __ballot_sync(0xffffffffu, lane < kZeroRows && r < used && p.source[r] < 0);
    while (mask) {
        W *row = out + (first + __ffs((int)mask) - 1) * words + at;
        mask &= mask - 1;
#pragma unroll
        for (int v = 0; v < kWords<W>; v++)
            if (at + 32 * v < words) row[32 * v] = W{};
    }
}

template <typename W>
__global__ void __launch_bounds__(256) k_expert_rows(const __grid_constant__ bsr_experts_t p, const W *X, W *Xs, int64_t words,
                                                     int64_t parts) {
    const int lane = threadIdx.x & 31;
    const int64_t copies = p.N * parts, units = copies + (p.R + kZeroRows - 1) / kZeroRows * parts;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
        if (u >= copies) {
            zero_rows(p, Xs, words, u - copies, parts);
            continue;
        }
        const int64_t n = u / parts, at = (u - n * parts) * 32 * kWords<W> + lane;
        W x[kWords<W>];
#pragma unroll
        for (int v = 0; v < kWords<W>; v++)
            if (at + 32 * v < words) x[v] = X[n * words + at + 32 * v];
        int32_t row = -1;
        for (int j = 0; j < p.k; j++) {
            if (j % 32 == 0) row = j + lane < p.k ? row_of(p, n * p.k + j + lane) : -1;
            const int64_t r = __shfl_sync(0xffffffffu, row, j % 32);
            if (r < 0) continue;
#pragma unroll
            for (int v = 0; v < kWords<W>; v++)
                if (at + 32 * v < words) Xs[r * words + at + 32 * v] = x[v];
        }
    }
}

// ROWS: choices whose rows are on their way at once; WORDS of each a lane: eight of one choice, 32 bytes of
// two, four words of four. (Four of four for all: 9920 rows of 1344 fp32 features of one choice 28 us for 20; four of
// two choices: bf16 15 for 12.4, fp32 31.6 for 29.9; four words of 2 bytes, 8192 x 1023: 19.8 for 15.4.
// Two CTAs an SM: 128 registers, or one of 140.)
template <typename T, typename W, int WORDS, int ROWS>
__global__ void __launch_bounds__(256, 2) k_expert_sum(const __grid_constant__ bsr_experts_t p, const W *Ys, const float *weights, W *Y,
                                                    int64_t words, int64_t parts) {
    constexpr int n_w = Word<T, W>::n;
    const int lane = threadIdx.x & 31;
    const int64_t units = p.N * parts;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
        const int64_t n = u / parts, at = (u - n * parts) * 32 * WORDS + lane;
        float sum[WORDS][n_w] = {};
        for (int j0 = 0; j0 < p.k; j0 += ROWS) {
            Word<T, W> y[ROWS][WORDS];
            int64_t r[ROWS];
            float w[ROWS];
#pragma unroll
            for (int j = 0; j < ROWS; j++) {
                const int64_t pair = n * p.k + min(j0 + j, p.k - 1);
                const int32_t row = row_of(p, pair);
                r[j] = j0 + j < p.k ? row : -1;
                w[j] = weights ? weights[pair] : 1.f;
            }
#pragma unroll
            for (int j = 0; j < ROWS; j++)
#pragma unroll
                for (int v = 0; v < WORDS; v++)
                    load_if(y[j][v].w, Ys + r[j] * words + at + 32 * v, r[j] >= 0 && at + 32 * v < words);
#pragma unroll
            for (int j = 0; j < ROWS; j++) {
                if (r[j] < 0) continue;
#pragma unroll
                for (int v = 0; v < WORDS; v++)
                    if (at + 32 * v < words) {
#pragma unroll
                        for (int i = 0; i < n_w; i++) sum[v][i] = fmaf(w[j], to_f32(y[j][v].v[i]), sum[v][i]);
                    }
            }
        }
#pragma unroll
        for (int v = 0; v < WORDS; v++) {
            if (at + 32 * v >= words) break;
            Word<T, W> y;
#pragma unroll
            for (int i = 0; i < n_w; i++) y.v[i] = from_f32<T>(sum[v][i]);
            Y[n * words + at + 32 * v] = y.w;
        }
    }
}

// dYs = w dY, dw = <Ys, dY>: a warp to a choice.
template <typename T, typename W>
__global__ void __launch_bounds__(256) k_expert_sum_backward(const __grid_constant__ bsr_experts_t p, const W *Ys, const float *weights,
                                                             const W *dY, W *dYs, float *dweights, int64_t words,
                                                             int64_t parts) {
    constexpr int n_w = Word<T, W>::n;
    const int lane = threadIdx.x & 31;
    const int64_t pairs = p.N * p.k, units = pairs + (dYs ? (p.R + kZeroRows - 1) / kZeroRows * parts : 0);
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
        if (u >= pairs) {
            zero_rows(p, dYs, words, u - pairs, parts);
            continue;
        }
        const int64_t n = u / p.k, r = row_of(p, u);
        if (r < 0) {
            if (dweights && lane == 0) dweights[u] = 0.f;
            continue;
        }
        const float w = weights[u];
        float dot = 0.f;
        for (int64_t at = lane; at < words; at += 32 * kWords<W>) {
            Word<T, W> d[kWords<W>], y[kWords<W>];
#pragma unroll
            for (int v = 0; v < kWords<W>; v++) {
                if (at + 32 * v >= words) break;
                d[v].w = dY[n * words + at + 32 * v];
                if (dweights) y[v].w = Ys[r * words + at + 32 * v];
            }
#pragma unroll
            for (int v = 0; v < kWords<W>; v++) {
                if (at + 32 * v >= words) break;
                Word<T, W> o;
#pragma unroll
                for (int i = 0; i < n_w; i++) {
                    const float g = to_f32(d[v].v[i]);
                    if (dweights) dot = fmaf(g, to_f32(y[v].v[i]), dot);
                    o.v[i] = from_f32<T>(w * g);
                }
                if (dYs) dYs[r * words + at + 32 * v] = o.w;
            }
        }
        if (!dweights) continue;
#pragma unroll
        for (int m = 16; m; m /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, m);
        if (lane == 0) dweights[u] = dot;
    }
}

template <int BITS>
cudaError_t order(const bsr_experts_t &p, const int32_t *experts, cudaStream_t s) {
    static std::atomic<uint64_t> attr_set{0}, wide_set{0};
    int dev = 0;
    cudaGetDevice(&dev);
    const uint64_t bit = 1ull << (dev & 63);
    cudaError_t e = allow_smem(k_expert_order<BITS>, (kWarps + 3) * (1 << BITS) * 4, attr_set);
    if (e == cudaSuccess && !(wide_set.load() & bit)) {
        e = cudaFuncSetAttribute(k_expert_order<BITS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess) wide_set.fetch_or(bit);
    }
    if (e != cudaSuccess) return e;
    const int64_t pairs = p.N * p.k;
    const unsigned ctas = pairs <= 4 * kOrderThreads ? 1 : pairs <= 16 * kOrderThreads ? 8 : 16;
    return launch_clusters(k_expert_order<BITS>, ctas, dim3(ctas), dim3(kOrderThreads), (size_t)(kWarps + 3) * p.E * 4, s, p, experts, ctas);
}

unsigned grid_of(int64_t units) { return (unsigned)std::min<int64_t>(std::max<int64_t>((units + 7) / 8, 1), 1 << 20); }

// f(T(), W()) with the element type and the widest word that rows of D are made of.
template <typename F>
cudaError_t by_word(int64_t D, bsr_dtype_t dt, F f) {
    const int64_t bytes = D * (dt == BSR_F32 ? 4 : 2);
    if (dt == BSR_F32) return bytes % 16 == 0 ? f(float(), uint4()) : bytes % 8 == 0 ? f(float(), uint2()) : f(float(), uint32_t());
    return bytes % 16 == 0  ? f(uint16_t(), uint4())
           : bytes % 8 == 0 ? f(uint16_t(), uint2())
           : bytes % 4 == 0 ? f(uint16_t(), uint32_t())
                            : f(uint16_t(), uint16_t());
}

}  // namespace

cudaError_t launch_expert_order(const bsr_experts_t &p, const int32_t *experts, cudaStream_t s) {
    return p.E <= 16 ? order<4>(p, experts, s) : p.E <= 64 ? order<6>(p, experts, s) : order<10>(p, experts, s);
}

cudaError_t launch_expert_rows(const bsr_experts_t &p, const void *X, void *Xs, int64_t D, bsr_dtype_t dt, cudaStream_t s) {
    return by_word(D, dt, [&](auto t, auto w) {
        using W = decltype(w);
        const int64_t words = D * (int64_t)sizeof(t) / (int64_t)sizeof(W), parts = (words + 32 * kWords<W> - 1) / (32 * kWords<W>);
        return launch_kernel(k_expert_rows<W>, dim3(grid_of((p.N + (p.R + kZeroRows - 1) / kZeroRows) * parts)), dim3(256), 0, s, p,
                             static_cast<const W *>(X), static_cast<W *>(Xs), words, parts);
    });
}

cudaError_t launch_expert_sum(const bsr_experts_t &p, const void *Ys, const float *weights, void *Y, int64_t D, bsr_dtype_t dt,
                              cudaStream_t s) {
    return by_word(D, dt, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        const int64_t words = D * (int64_t)sizeof(T) / (int64_t)sizeof(W);
        auto run = [&](auto kernel, int at_once) {
            const int64_t parts = (words + 32 * at_once - 1) / (32 * at_once);
            return launch_kernel(kernel, dim3(grid_of(p.N * parts)), dim3(256), 0, s, p, static_cast<const W *>(Ys), weights, static_cast<W *>(Y),
                                 words, parts);
        };
        constexpr int two = sizeof(W) >= 4 ? 32 / (int)sizeof(W) : 8;
        return p.k == 1 ? run(k_expert_sum<T, W, 8, 1>, 8) : p.k == 2 ? run(k_expert_sum<T, W, two, 2>, two) : run(k_expert_sum<T, W, 4, 4>, 4);
    });
}

cudaError_t launch_expert_sum_backward(const bsr_experts_t &p, const void *Ys, const float *weights, const void *dY, void *dYs,
                                       float *dweights, int64_t D, bsr_dtype_t dt, cudaStream_t s) {
    return by_word(D, dt, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        const int64_t words = D * (int64_t)sizeof(T) / (int64_t)sizeof(W), parts = (words + 32 * kWords<W> - 1) / (32 * kWords<W>);
        const int64_t units = p.N * p.k + (dYs ? (p.R + kZeroRows - 1) / kZeroRows * parts : 0);
        return launch_kernel(k_expert_sum_backward<T, W>, dim3(grid_of(units)), dim3(256), 0, s, p, static_cast<const W *>(Ys), weights,
                             static_cast<const W *>(dY), static_cast<W *>(dYs), dweights, words, parts);
    });
}

}  // namespace bsr
