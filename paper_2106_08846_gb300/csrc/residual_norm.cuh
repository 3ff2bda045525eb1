// What the kernels of the residual step share: how a row lies in the threads that
// hold it, and sums over them.
#pragma once

#include "bsr_internal.h"
#include "elem.cuh"
#include "pair.cuh"
#include "ptx.cuh"
#include "residual_norm.h"
#include "run_blocks.h"

namespace bsr {

namespace {

constexpr int kMaxGroups = 8;     // rows in work per CTA

// How rows lie in memory: anywhere, runs of eight on 16-byte boundaries, or such
// with none past the row's end. A thread has V runs of eight features.
enum Layout : int { ANY = 0, RUNS = 1, FULL = 2 };

// Feature j of run i of thread t, and whether it is one.
__device__ __forceinline__ int feature(int i, int j, int t, int NT) { return 8 * (t + i * NT) + j; }
template <int L>
__device__ __forceinline__ bool inside(int i, int j, int t, int NT, int D) {
    return L == FULL || feature(i, j, t, NT) < D;
}

// A run of eight features, in pairs.
struct Run {
    F2 v[4];
};
template <typename T>
__device__ __forceinline__ Run run_of(const uint32_t (&w)[2 * sizeof(T)]) {
    Run r;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if constexpr (sizeof(T) == 4) r.v[j] = pack2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        else r.v[j] = pack2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
    return r;
}

// A run as it is loaded: its words; or (ANY) the 16-byte blocks that hold it, the
// place of its first byte in them and the values that are there. The blocks' other
// bytes lie beside the run in its array.
template <typename T, int L>
struct Raw {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ Run run() const { return run_of<T>(w); }
};
template <typename T>
struct Raw<T, ANY> {
    uint32_t w[2 * sizeof(T) + 4];
    int at, n;
    __device__ __forceinline__ Run run() const {
        constexpr int words = 2 * sizeof(T);
        uint32_t a[words + 4], r[words];
#pragma unroll
        for (int k = 0; k < words + 4; k++) a[k] = w[k];
        if (at & 4) {
#pragma unroll
            for (int k = 0; k < words + 3; k++) a[k] = a[k + 1];
        }
        if (at & 8) {
#pragma unroll
            for (int k = 0; k < words + 2; k++) a[k] = a[k + 2];
        }
#pragma unroll
        for (int k = 0; k < words; k++) {
            r[k] = sizeof(T) == 2 && (at & 2) ? __funnelshift_r(a[k], a[k + 1], 16) : a[k];
            if constexpr (sizeof(T) == 4) {
                if (k >= n) r[k] = 0;
            } else {
                if (2 * k >= n) r[k] = 0;
                else if (2 * k + 1 >= n) r[k] &= 0xffffu;
            }
        }
        return run_of<T>(r);
    }
};
__device__ __forceinline__ Run all_run(float x) {
    Run r;
#pragma unroll
    for (int j = 0; j < 4; j++) r.v[j] = all2(x);
    return r;
}
// x in run i of a row, 0 past the row's end.
template <int L>
__device__ __forceinline__ Run row_run(float x, int D, int i, int t, int NT) {
    Run r = all_run(inside<L>(i, 0, t, NT, D) ? x : 0.f);
    if constexpr (L == ANY) {
#pragma unroll
        for (int j = 0; j < 4; j++)
            r.v[j] = pack2(inside<L>(i, 2 * j, t, NT, D) ? x : 0.f, inside<L>(i, 2 * j + 1, t, NT, D) ? x : 0.f);
    }
    return r;
}

// Run i of a row; 0 past the row's end. CONST: of an array that the kernel does not
// write (a row that it may write is read once: the parameters keep their place in L1). An
// earlier kernel may write it, so it is no read-only load; in order with the wait for that
// kernel, but with nothing else (plain C++ loads, 16384 tokens of 1024 backward: 62.6 us for 61.3).
template <bool CONST>
__device__ __forceinline__ uint4 load_block(const void *p) {
    uint4 u;
    if constexpr (CONST)
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                     : "l"(p)
                     : "memory");
    return u;
}
__device__ __forceinline__ uint32_t load_value(const float *p) { return *reinterpret_cast<const uint32_t *>(p); }
__device__ __forceinline__ uint32_t load_value(const uint16_t *p) { return *p; }
// ANY: at_end, where at_array_end holds for the row, whose last runs are then read value by
// value (by its blocks the call would read up to 14 bytes past y, h and the others).
template <typename T, int L, bool CONST>
__device__ __forceinline__ Raw<T, L> load_run(const T *row, int D, int i, int t, int NT, bool at_end) {
    Raw<T, L> r;
    const int e = feature(i, 0, t, NT);
    if constexpr (L != ANY) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; h++) {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (inside<L>(i, 0, t, NT, D)) u = load_block<CONST>(row + e + 8 * h / (int)(sizeof(T) / 2));
            r.w[4 * h] = u.x, r.w[4 * h + 1] = u.y, r.w[4 * h + 2] = u.z, r.w[4 * h + 3] = u.w;
        }
    } else {
        const uintptr_t first = reinterpret_cast<uintptr_t>(row + e);
        const char *const blocks = reinterpret_cast<const char *>(first & ~(uintptr_t)15);
        r.n = min(8, D - e);
        r.at = read_run<sizeof(T)>(
            r.w, (int)(first & 15), r.n, at_end && at_row_end(D - e),
            [&](int k, uint32_t *w) {
                const uint4 u = load_block<CONST>(blocks + 16 * k);
                w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
            },
            [&](int j) { return load_value(row + e + j); });
    }
    return r;
}
// A run of a parameter, which may begin on any boundary of 4 bytes (ANY).
template <int L>
__device__ __forceinline__ Run load_param(const float *p, int D, int i, int t, int NT) {
    if constexpr (L != ANY) {
        return load_run<float, L, true>(p, D, i, t, NT, false).run();
    } else {
        uint32_t w[8];
        const int e = feature(i, 0, t, NT), n = D - e;
        read_run<4>(
            w, 0, n, n < 8 || reinterpret_cast<uintptr_t>(p) % 16 != 0,
            [&](int k, uint32_t *v) {
                const uint4 u = load_block<true>(p + e + 4 * k);
                v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
            },
            [&](int j) { return load_value(p + e + j); });
        return run_of<float>(w);
    }
}
// A run of a gate's row.
template <typename T, int L>
__device__ __forceinline__ Run load_gate(const T *row, int D, int i, int t, int NT, bool at_end) {
    return load_run<T, L, true>(row, D, i, t, NT, at_end).run();
}
template <int L>
__device__ __forceinline__ bool row_at_end(int64_t rows, int D) {
    return L == ANY && at_array_end(rows, D);
}
// A warp's kilobyte of shared memory; WARPS: the most of a CTA.
template <int WARPS>
__device__ __forceinline__ float *stage() {
    __shared__ float4 words[WARPS][64];
    return reinterpret_cast<float *>(words[(threadIdx.y * blockDim.x + threadIdx.x) >> 5]);
}
// By whole warps. ANY: a warp's fp32 runs, which are contiguous, change lanes through
// shared memory, so that an instruction's stores lie side by side: a lane's eight
// values one by one cost a write of their 32-byte sector each (3000 x 771 fp32, one norm
// 21.5 us, so 15.6; 16384 x 1023 114 and 55). bf16 runs go in four stores and gain nothing
// by the detour.
template <typename T, int L, int WARPS>
__device__ __forceinline__ void store_run(T *row, int D, int i, int t, int NT, const Run &r) {
    const int lane = threadIdx.x & 31, left = D - feature(i, 0, t, NT);   // values of the row from this lane's on
    T *const p = row + feature(i, 0, t, NT);
    if constexpr (sizeof(T) == 4 && L == ANY) {
        const int all = left + 8 * lane;   // from the warp's first on
        if (all <= 0) return;
        float *const buf = stage<WARPS>();
        __syncwarp();   // (the last run has been read)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float2 u = unpack2(r.v[2 * h]), w = unpack2(r.v[2 * h + 1]);
            reinterpret_cast<float4 *>(buf)[2 * lane + h] = make_float4(u.x, u.y, w.x, w.y);
        }
        __syncwarp();
        T *const first = p - 8 * lane;
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (32 * j + lane < all) first[32 * j + lane] = buf[32 * j + lane];
    } else if constexpr (sizeof(T) == 4) {
        if (!inside<L>(i, 0, t, NT, D)) return;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float2 u = unpack2(r.v[2 * h]), w = unpack2(r.v[2 * h + 1]);
            reinterpret_cast<float4 *>(p)[h] = make_float4(u.x, u.y, w.x, w.y);
        }
    } else {
        if (!inside<L>(i, 0, t, NT, D)) return;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const float2 u = unpack2(r.v[k]);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(u.y), "f"(u.x));
        }
        if constexpr (L != ANY) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (left < 8) {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (j < left) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        } else if (reinterpret_cast<uintptr_t>(p) & 2) {
            p[0] = (uint16_t)w[0];
#pragma unroll
            for (int k = 0; k < 3; k++) *reinterpret_cast<uint32_t *>(p + 1 + 2 * k) = __funnelshift_r(w[k], w[k + 1], 16);
            p[7] = (uint16_t)(w[3] >> 16);
        } else {
#pragma unroll
            for (int k = 0; k < 4; k++) *reinterpret_cast<uint32_t *>(p + 2 * k) = w[k];
        }
    }
}

// x - m where there is a feature (x is 0 elsewhere, and stays so)
template <int L>
__device__ __forceinline__ void centre(Run &x, float m, int D, int i, int t, int NT) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if constexpr (L != ANY) x.v[j] = add2(x.v[j], all2(inside<L>(i, 0, t, NT, D) ? -m : 0.f));
        else x.v[j] = add2(x.v[j], pack2(inside<L>(i, 2 * j, t, NT, D) ? -m : 0.f, inside<L>(i, 2 * j + 1, t, NT, D) ? -m : 0.f));
    }
}
__device__ __forceinline__ float both(F2 x) {
    const float2 u = unpack2(x);
    return u.x + u.y;
}

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

// Sums over the NT threads of a group, the same in each of them. Lanes exchange
// halves of the values until each has one to add up; the warps' sums meet in shared
// memory, four warps to a group of words (of absent warps 0). Its two halves are used
// in turn, so one barrier does: a half is written again only after the other half's
// barrier. FOUR: at most four warps. CLUSTER: a CTA's threads are the group's part in
// it; the CTAs then write their sums into each other's shared memory, likewise in two
// halves, and add them up in the order of their ranks.
template <bool FOUR, bool CLUSTER = false>
struct GroupSum {
    float4 *words;   // [2][32]; CLUSTER: then [2][CTAs]
    int NT, id, turn;
    __device__ __forceinline__ void init() {   // before the group's first barrier
        for (int k = threadIdx.x; k < 64; k += NT) words[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (NT > 32) ptx::named_barrier(1 + id, NT);
        if (CLUSTER) ptx::cluster_barrier();   // the other CTAs have begun
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
        if constexpr (CLUSTER) {
            const uint32_t ctas = cluster_size();
            float *const all = reinterpret_cast<float *>(words + 64 + 4 * turn);
            if (threadIdx.x < ctas) {
#pragma unroll
                for (int k = 0; k < N; k++)
                    ptx::store_cluster(ptx::map_to_cta(all + 4 * ptx::cluster_rank() + k, threadIdx.x), __float_as_uint(v[k]));
            }
            __syncwarp();
            ptx::cluster_barrier();
#pragma unroll
            for (int k = 0; k < N; k++) {
                float c = all[k];
                for (uint32_t r = 1; r < ctas; r++) c += all[4 * r + k];
                v[k] = c;
            }
        }
    }
};

__device__ __forceinline__ void times(Run &r, const Run &s) {
#pragma unroll
    for (int j = 0; j < 4; j++) r.v[j] = mul2(r.v[j], s.v[j]);
}

// Normalises rows in place.
template <int V, int L, int ROWS, typename Sum>
__device__ __forceinline__ void normalise(Run (&x)[ROWS][V], int how, float eps, int D, float over_d, int t, int NT, Sum &sum) {
    float s[ROWS];
    if (how == BSR_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < ROWS; k++) {
            F2 c = all2(0.f);
#pragma unroll
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) c = add2(c, x[k][i].v[j]);
            s[k] = both(c);
        }
        sum(s);
#pragma unroll
        for (int k = 0; k < ROWS; k++)
#pragma unroll
            for (int i = 0; i < V; i++) centre<L>(x[k][i], s[k] * over_d, D, i, t, NT);
    }
#pragma unroll
    for (int k = 0; k < ROWS; k++) {
        F2 c = all2(0.f);
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) c = fma2(x[k][i].v[j], x[k][i].v[j], c);
        s[k] = both(c);
    }
    sum(s);
#pragma unroll
    for (int k = 0; k < ROWS; k++) {
        const F2 r = all2(rsqrtf(fmaf(s[k], over_d, eps)));
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) x[k][i].v[j] = mul2(x[k][i].v[j], r);
    }
}
// x * w + b with a parameter's row each, where there is one
template <int V, int L, int ROWS>
__device__ __forceinline__ void affine(Run (&x)[ROWS][V], const float *w, const float *b, int D, int t, int NT) {
    if (w) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const Run p = load_param<L>(w, D, i, t, NT);
#pragma unroll
            for (int k = 0; k < ROWS; k++) times(x[k][i], p);
        }
    }
    if (b) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const Run p = load_param<L>(b, D, i, t, NT);
#pragma unroll
            for (int k = 0; k < ROWS; k++)
#pragma unroll
                for (int j = 0; j < 4; j++) x[k][i].v[j] = add2(x[k][i].v[j], p.v[j]);
        }
    }
}

int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        cudaGetLastError();
    return n;
}

bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The layout of rows of D features in V runs of NT threads.
int layout_of(const bsr_residual_norm_t &p, int V, int NT) {
    const bool runs = p.D % 8 == 0 && aligned(p.scale) && aligned(p.post_w) && aligned(p.post_b) && aligned(p.pre_w) && aligned(p.pre_b);
    return !runs ? ANY : p.D == (int64_t)8 * V * NT ? FULL : RUNS;
}

}  // namespace

}  // namespace bsr
