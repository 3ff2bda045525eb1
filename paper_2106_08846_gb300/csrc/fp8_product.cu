// Products of 8-bit operands on the tensor cores.
//
//   Y[n, m] = bias[m] + sum_b sa[b, n] sb[b, m] sum_{k in block b} qa[n, k] qb[m, k]
//
// A cluster of two CTAs works on a tile of 256 rows of a by 2 `half` rows of b. A
// block of 128 columns is a step: four MMAs (M = 256, N = 2 half, K = 32) into a
// fresh accumulator buffer, which the epilogue takes out, scales and adds in
// registers while the next step's MMAs fill the other buffer.
//
//   warps 0, 1, 3  producers, a step each in turn: 128 rows of a and `half` of b a
//                  CTA, 128 bytes each, by TMA (128-byte swizzle) into a stage of the ring
//   warp 2         MMAs of the pair's first CTA
//   warps 4 .. 11  epilogue: 32 rows and half of the columns each, up to 128 sums a thread
//                  (registers handed over by the other four warps)
//
// A step of 256 columns is 512 SM cycles of MMAs; its epilogue reads 128 KB of
// tensor memory an SM and makes a multiply-add of each value (256 cycles, packed).
// Where each of b's rows has a scale of its own, one more multiplication.
//
// Persistent: one CTA per SM. Runs of rows: tiles of 256 rows from each run's first
// one on; the table of the runs' tiles is made by every CTA from the offsets on the device.
// Runs of columns: a tile's steps are the run's. Tiles of sums too few to fill the
// GPU have them split; the parts are added in their order by a second launch.
//
// Every wait is bounded by the global timer; a timeout is recorded, stops every
// role, lets the issued copies and MMAs finish, frees the tensor memory and
// returns.
#include <algorithm>
#include <atomic>
#include <cstdlib>

#include "bsr_internal.h"
#include "eight.cuh"
#include "experts.h"
#include "fp8.h"
#include "launch.cuh"
#include "ptx.cuh"
#include "status.cuh"
#include "tcgen05.cuh"

namespace bsr {

namespace {

constexpr int kEpiWarp0 = 4, kMmaWarp = 2, kEpiWarps = 8, kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kProducers = 3, kStages = 8;
constexpr uint32_t kABytes = 128 * 128;       // a CTA's rows of a, a step
constexpr uint32_t kAccCols = 256;
constexpr uint32_t kScaleBytes = kEpiWarps * 128 * 4;
constexpr uint32_t kMaxSmem = 227 * 1024 - 12 * 1024;   // (static: the runs' table, barriers)
constexpr uint64_t kDrainNs = 200000000ull;   // bound for copies and MMAs already issued
// Registers of a thread: (4 warps * 72 + 8 warps * 216) * 32 is what 384 threads are launched with (168 each).
constexpr int kFewRegs = 72, kManyRegs = 216;

__device__ int g_status;

struct Args {
    CUtensorMap a, b;
    const float *sa, *sb, *bias;
    int64_t rows, M;          // of a; of b (columns of Y)
    int64_t sa_cols, sb_cols, KB;
    int a_shift;              // rows of a that share a scale: 1 << a_shift
    int group, E;
    const int32_t *offsets;
    unsigned tiles_m, tiles_n;
    int splits;               // of a tile's steps
    int half, ns;
    uint32_t stage_bytes, idesc;
    void *Y;
    float *parts;             // [units][256][2 half] where splits > 1
    int align;                // bytes (at most 16) that rows of Y are aligned to
    uint64_t wait_ns;
    int stall_step;           // test hook: this step of each tile is never loaded (-1: none)
};

struct Unit {
    int64_t m0, m1, n0;   // first row, end of the rows, first column
    int64_t out;          // rows of Y before this unit's matrix
    int batch, part;
    int i0, i1;           // steps
};

// The runs: their ends, and the tiles of rows before each.
struct Runs {
    int32_t at[kMostExperts + 1];
    uint32_t first[kMostExperts + 1];
};

__device__ __forceinline__ Unit unit_at(const Args &a, const Runs &r, unsigned v) {
    Unit u;
    u.out = 0;
    u.batch = 0;
    u.part = -1;
    u.i0 = 0;
    u.i1 = (int)a.KB;
    if (a.group == BSR_GROUP_ROWS) {
        const unsigned t = v / a.tiles_n;
        int lo = 0, hi = a.E;   // the last run whose tiles begin at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (r.first[mid] <= t) lo = mid;
            else hi = mid;
        }
        u.batch = lo;
        u.m0 = r.at[lo] + (int64_t)(t - r.first[lo]) * 256;
        u.m1 = r.at[lo + 1];
        u.n0 = (int64_t)(v - t * a.tiles_n) * 2 * a.half;
        return u;
    }
    unsigned tile = v;
    if (a.group == BSR_GROUP_COLUMNS) {
        const unsigned tiles = a.tiles_m * a.tiles_n, e = v / tiles;
        tile = v - e * tiles;
        u.out = (int64_t)e * a.rows;
        u.i0 = r.at[e];
        u.i1 = max(r.at[e], r.at[e + 1]);
    } else if (a.splits > 1) {
        u.part = (int)v;
        tile = v / (unsigned)a.splits;
        const unsigned k = v - tile * (unsigned)a.splits;
        u.i0 = (int)(a.KB * k / a.splits);
        u.i1 = (int)(a.KB * (k + 1) / a.splits);
    }
    const unsigned tm = tile / a.tiles_n;
    u.m0 = (int64_t)tm * 256;
    u.m1 = a.rows;
    u.n0 = (int64_t)(tile - tm * a.tiles_n) * 2 * a.half;
    return u;
}

// The unit of a pair in a round of them: all rounds but the first are taken
// backwards, so that who had a long unit there is the last to have one more.
__device__ __forceinline__ unsigned unit_in(unsigned round, unsigned pair, unsigned pairs) {
    return round * pairs + (round ? pairs - 1 - pair : pair);
}

// Scales of a step as a thread loads them: of its own row of a, and of its warp's
// columns' rows of b (COL: of columns 4 lane .. 4 lane + 3).
template <bool COL>
struct Scales {
    float a, b[COL ? 4 : 1];
};

// COL: each row of b has a scale of its own, else 128 of them share one.
template <typename T, bool COL>
__global__ void __launch_bounds__(kThreads, 1) k_fp8_product(const __grid_constant__ Args a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *base = ptx::align_smem(smem_raw);
    const int ns = a.ns;
    const uint32_t stage_bytes = a.stage_bytes;
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], done;
    __shared__ int stop, loads[kProducers][2];   // loads[producer][CTA of the pair]: steps loaded
    __shared__ int freed, handed;                // commits issued to `empty` and to `acc_full`
    __shared__ uint32_t tmem_s;
    __shared__ Runs runs;

    // (a shuffle, so that the warp index and what follows from it is uniform)
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();
    const unsigned pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < ns; s++) {
            ptx::mbar_init(&full[s], 1);   // a producer's arrival, and its bytes
            ptx::mbar_init(&empty[s], 1);
        }
        for (int i = 0; i < 2; i++) {
            ptx::mbar_init(&acc_full[i], 1);
            ptx::mbar_init(&acc_empty[i], 2 * kEpiWarps);
        }
        ptx::mbar_init(&done, 1);
        stop = freed = handed = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kMmaWarp) tc5::alloc_pair(&tmem_s, 2 * kAccCols);
    if (warp == 0 && ptx::elect_one()) {
        ptx::prefetch_tensormap(&a.a);
        ptx::prefetch_tensormap(&a.b);
    }
    tc5::fence_before();
    __syncthreads();
    ptx::cluster_barrier();   // the other CTA's barriers exist
    tc5::fence_after();
    ptx::pdl_launch_dependents();   // (after the allocation: ptx.cuh)
    ptx::pdl_wait();                // operands and offsets may be an earlier kernel's, and Y may be read by one
    unsigned units = a.tiles_m * a.tiles_n * (unsigned)a.splits;
    if (a.group != BSR_GROUP_NONE) {
        // within what there is, in steps for columns
        const bool by_rows = a.group == BSR_GROUP_ROWS;
        for (int e = threadIdx.x; e <= a.E; e += kThreads) {
            const int64_t o = max(0, __ldg(a.offsets + e));
            runs.at[e] = (int32_t)(by_rows ? min(o, a.rows) : min(o / kFp8Block, a.KB));
        }
        __syncthreads();
        if (warp == 0 && by_rows) {
            uint32_t before = 0;
            for (int e0 = 0; e0 < a.E; e0 += 32) {
                const int e = e0 + lane;
                const uint32_t tiles = e < a.E ? (uint32_t)(max(0, runs.at[e + 1] - runs.at[e]) + 255) / 256 : 0;
                uint32_t upto = tiles;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += x;
                }
                if (e < a.E) runs.first[e] = before + upto - tiles;
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
            if (lane == 0) runs.first[a.E] = before;
        }
        __syncthreads();
        units = by_rows ? runs.first[a.E] * a.tiles_n : units * (unsigned)a.E;
    }
    const uint32_t tmem = tmem_s;
    const bool elected = ptx::elect_one();
    // stops every role of this pair; a timeout is recorded
    auto halt = [&]() {
        if (elected) {
            if (!aborted(&stop)) set_status(&g_status, DEV_TIMEOUT);
            atomicExch(&stop, 1);
            ptx::store_cluster(ptx::map_to_cta(&stop, rank ^ 1), 1);
        }
    };

    // ---- producers: the pair's steps prod, prod + np, ... No more producers
    // than stages: one that waits for step g - ns to be consumed has to know that
    // step g - 2 ns was, or the stage's barrier, which tells phases apart by their
    // parity, would let it pass a round early; its last wait, for step
    // g - np - ns, tells it so if np <= ns.
    const int prod = warp < kMmaWarp ? warp : kMmaWarp, np = min(kProducers, ns);
    const bool producer = warp < kEpiWarp0 && warp != kMmaWarp && prod < np;
    unsigned round = 0, v = pair;
    Unit un = {};
    int i = 0, s = prod % ns, issued = 0;
    uint32_t phase = 1 ^ ((prod / ns) & 1);   // the parity of `empty` that a first use of a stage passes at once
    uint32_t stalled = 0;                     // test hook: stages whose load was left out
    const uint32_t smem0 = ptx::smem_addr(base), bar0 = ptx::smem_addr(&full[0]);
    const uint32_t first0 = ptx::map_to_cta(&full[0], 0);   // `full` of the pair's first CTA
    // to the unit of step i, which may lie beyond this one's last; false: none left
    auto seek = [&]() {
        while (i >= un.i1) {
            const int over = i - un.i1;
            v = unit_in(++round, pair, pairs);
            if (v >= units) return false;
            un = unit_at(a, runs, v);
            i = un.i0 + over;
        }
        return true;
    };
    auto load_step = [&]() {
        if (i - un.i0 == a.stall_step) {   // never loaded: its consumer times out
            stalled |= 1u << s;
        } else if (elected) {
            const uint32_t dst = smem0 + s * stage_bytes, bar = first0 + 8 * s;
            if (rank == 0) ptx::mbar_arrive_expect_tx_at(bar0 + 8 * s, 2 * stage_bytes);
            ptx::tma_load_2d_pair_at(dst, &a.a, i * kFp8Block, (int)(un.m0 + rank * 128), bar);
            ptx::tma_load_3d_pair_at(dst + kABytes, &a.b, i * kFp8Block, (int)(un.n0 + rank * a.half), un.batch, bar);
        }
        issued++;
        for (s += np; s >= ns; s -= ns) phase ^= 1;
        i += np;
        return seek();
    };
    bool more = false;
    // (each in its role's own branch, so that the compiler knows what a role has)
    if (warp >= kEpiWarp0) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
        const int q = warp & 3, share = (warp - kEpiWarp0) >> 2;   // tensor-memory lanes 32 q .., columns from half * share on
        const int groups = a.half / 32;                            // of 32 columns
        float *col_s = reinterpret_cast<float *>(base + (size_t)ns * stage_bytes) + (warp - kEpiWarp0) * 128;
        int ab = 0;
        uint32_t fphase = 0;
        bool ok = true;
        for (; ok && v < units; v = unit_in(++round, pair, pairs)) {
            un = unit_at(a, runs, v);
            const int64_t row0 = un.m0 + rank * 128 + 32 * q, col0 = un.n0 + share * a.half;
            // where this thread's scales lie; rows and columns that are not there take another's
            const float *sa = a.sa + (min(row0 + lane, a.rows - 1) >> a.a_shift);
            const float *sb = a.sb + (int64_t)un.batch * a.KB * a.sb_cols + (COL ? 0 : min(col0 >> 7, a.sb_cols - 1));
            auto fetch = [&](int b, Scales<COL> &f) {
                if (b >= un.i1) return;
                f.a = __ldg(sa + b * a.sa_cols);
                if constexpr (COL) {
#pragma unroll
                    for (int j = 0; j < 4; j++) f.b[j] = __ldg(sb + b * a.sb_cols + min(col0 + 4 * lane + j, a.M - 1));
                } else {
                    f.b[0] = __ldg(sb + b * a.sb_cols);
                }
            };
            F2 acc[4][2][2][4];   // [group][16 rows][8 rows][pair of columns]
#pragma unroll
            for (int g = 0; g < 4; g++)
#pragma unroll
                for (int j = 0; j < 16; j++) acc[g][j >> 3][(j >> 2) & 1][j & 3] = all2(0.f);
            Scales<COL> f0, f1;   // of even and odd steps, two steps ahead
            fetch(un.i0, f0);
            fetch(un.i0 + 1, f1);
            for (int b = un.i0; b < un.i1; b++) {
                float fa;
                auto take = [&](Scales<COL> &f) {
                    fa = COL ? f.a : f.a * f.b[0];
                    if constexpr (COL) {
                        __syncwarp();
                        *reinterpret_cast<float4 *>(col_s + 4 * lane) = make_float4(f.b[0], f.b[1], f.b[2], f.b[3]);
                        __syncwarp();
                    }
                    fetch(b + 2, f);
                };
                if ((b - un.i0) & 1) take(f1);
                else take(f0);
                F2 fr[4];   // factors of rows lane / 4 + 8 h
#pragma unroll
                for (int h = 0; h < 4; h++) fr[h] = all2(__shfl_sync(0xffffffffu, fa, (lane >> 2) + 8 * h));
                ok = __all_sync(0xffffffffu, wait_or_abort(&acc_full[ab], fphase, a.wait_ns * (uint64_t)(un.i1 - un.i0 + 2), &stop));
                if (!ok) {
                    halt();
                    break;
                }
                tc5::fence_after();
                const uint32_t tm = tmem + (uint32_t)ab * kAccCols + ((uint32_t)(32 * q) << 16) + share * a.half;
                uint32_t r[2][2][16];   // a group ahead
                tc5::ld_16x32(tm, r[0][0]);
                tc5::ld_16x32(tm + (16u << 16), r[0][1]);
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    if (g >= groups) break;
                    tc5::ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; j++) {   // no use of a loaded register moves above the wait
                        asm volatile("" : "+r"(r[g & 1][0][j]));
                        asm volatile("" : "+r"(r[g & 1][1][j]));
                    }
                    if (g + 1 < groups) {
                        if (g < 3) {
                            tc5::ld_16x32(tm + 32 * (g + 1), r[(g + 1) & 1][0]);
                            tc5::ld_16x32(tm + (16u << 16) + 32 * (g + 1), r[(g + 1) & 1][1]);
                        }
                    } else {   // the last columns are in registers: the buffer is handed back
                        tc5::fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive_remote(ptx::map_to_cta(&acc_empty[ab], 0));
                    }
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        F2 fc;
                        if constexpr (COL) {
                            const float2 c = *reinterpret_cast<const float2 *>(col_s + 32 * g + 8 * j + 2 * (lane & 3));
                            fc = pack2(c.x, c.y);
                        }
#pragma unroll
                        for (int h = 0; h < 4; h++) {
                            const uint32_t *x = &r[g & 1][h >> 1][4 * j + 2 * (h & 1)];
                            F2 p = pack2(__uint_as_float(x[0]), __uint_as_float(x[1]));
                            if constexpr (COL) p = mul2(p, fc);
                            acc[g][h >> 1][h & 1][j] = fma2(p, fr[h], acc[g][h >> 1][h & 1][j]);
                        }
                    }
                }
                ab ^= 1;
                if (ab == 0) fphase ^= 1;
            }
            if (!ok) break;
            // rows lane / 4 + 8 h, columns 32 g + 8 j + 2 (lane % 4), + 1
            const int c4 = lane & 3;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                if (g >= groups) break;
                const int64_t c = col0 + 32 * g;
                if (un.part >= 0) {
#pragma unroll
                    for (int h = 0; h < 4; h++) {
                        const int64_t row = row0 - un.m0 + (lane >> 2) + 8 * h;
                        float *at = a.parts + ((int64_t)un.part * 256 + row) * 2 * a.half + (c - un.n0) + 2 * c4;
#pragma unroll
                        for (int j = 0; j < 4; j++) *reinterpret_cast<float2 *>(at + 8 * j) = unpack2(acc[g][h >> 1][h & 1][j]);
                    }
                    continue;
                }
                F2 add[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int64_t at = c + 8 * j + 2 * c4;
                    const float *bias = a.bias + (int64_t)un.batch * a.M + at;
                    add[j] = a.bias ? pack2(at < a.M ? __ldg(bias) : 0.f, at + 1 < a.M ? __ldg(bias + 1) : 0.f) : all2(0.f);
                }
#pragma unroll
                for (int h = 0; h < 4; h++) {
                    F2 x[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) x[j] = add2(acc[g][h >> 1][h & 1][j], add[j]);
                    uint32_t w[4];
                    if constexpr (sizeof(T) == 2) {
#pragma unroll
                        for (int j = 0; j < 4; j++) w[j] = pack_bf16(x[j]);
                        turn_words(w);
                    }
                    const int64_t row = row0 + (lane >> 2) + 8 * h;
                    if (row >= un.m1) continue;
                    T *out = static_cast<T *>(a.Y) + (un.out + row) * a.M;
                    if constexpr (sizeof(T) == 2) {
                        Eight<T> e;
#pragma unroll
                        for (int j = 0; j < 4; j++) e.w[j] = w[j];
                        store8(out + c + 8 * c4, a.M - (c + 8 * c4), a.align, e);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const int64_t at = c + 8 * j + 2 * c4;
                            const float2 y = unpack2(x[j]);
                            if (at + 2 <= a.M && a.align >= 8) {
                                *reinterpret_cast<float2 *>(out + at) = y;
                            } else {
                                if (at < a.M) out[at] = y.x;
                                if (at + 1 < a.M) out[at + 1] = y.y;
                            }
                        }
                    }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
        if (producer) {
            if (v < units) {
                un = unit_at(a, runs, v);
                i = un.i0 + prod;
                more = seek();
            }
            while (more) {
                const bool got = wait_or_abort(&empty[s], phase, a.wait_ns, &stop);
                if (!__all_sync(0xffffffffu, got && !aborted(&stop))) {
                    halt();
                    break;
                }
                more = load_step();
            }
            if (elected) {
                loads[prod][rank] = issued;
                ptx::store_cluster(ptx::map_to_cta(&loads[prod][rank], rank ^ 1), (uint32_t)issued);
            }
        } else if (warp == kMmaWarp) {
            if (rank == 0) {
                int ab = 0, n_steps = 0;
                uint32_t fphase = 0, aphase = 1;
                bool ok = true;
                s = 0;
                const uint64_t ad0 = tc5::desc_sw128(smem0), bd0 = tc5::desc_sw128(smem0 + kABytes);
                for (; ok && v < units; v = unit_in(++round, pair, pairs)) {
                    un = unit_at(a, runs, v);
                    for (i = un.i0; i < un.i1; i++) {
                        ok = __all_sync(0xffffffffu, wait_or_abort(&acc_empty[ab], aphase, a.wait_ns, &stop) &&
                                                         wait_or_abort(&full[s], fphase, a.wait_ns, &stop));
                        if (!ok) break;
                        tc5::fence_after();
                        if (elected) {
                            const uint64_t at = (uint64_t)((s * stage_bytes) >> 4);
    #pragma unroll
                            for (int j = 0; j < kFp8Block / 32; j++)   // (32 bytes along the rows)
                                tc5::mma_ss_pair_8bit(tmem + (uint32_t)ab * kAccCols, ad0 + at + 2 * j, bd0 + at + 2 * j, a.idesc, j > 0);
                            tc5::commit_pair(&empty[s]);
                            tc5::commit_pair(&acc_full[ab]);
                        }
                        __syncwarp();
                        n_steps++;
                        if (++s == ns) {
                            s = 0;
                            fphase ^= 1;
                        }
                        ab ^= 1;
                        if (ab == 0) aphase ^= 1;
                    }
                    if (!ok) halt();
                }
                // every MMA issued has completed before the tensor memory is freed
                if (elected) {
                    tc5::commit_pair(&done);
                    freed = handed = n_steps;
                    ptx::store_cluster(ptx::map_to_cta(&freed, 1), (uint32_t)n_steps);
                    ptx::store_cluster(ptx::map_to_cta(&handed, 1), (uint32_t)n_steps);
                }
                __syncwarp();
                ptx::mbar_wait_bounded(&done, 0, kDrainNs);
            }
        }
    }
    // every MMA completed (the issuer waited for `done`), and neither CTA reads
    // or signals the other's shared memory any more
    auto meet = [&]() {
        __syncwarp();
        ptx::cluster_barrier();
    };
    tc5::fence_before();
    meet();
    if (aborted(&stop)) {
        // (the same for both CTAs.) The loads that only one CTA's producer
        // issued are completed by the other's, so that every barrier phase can
        // finish, and the CTA whose barriers count the bytes waits for those
        // that no later load of their stage shows to be complete: no copy
        // outlives the CTAs
        if (producer) {
            int most[kProducers];
            for (int p = 0; p < np; p++) most[p] = max(loads[p][0], loads[p][1]);
            while (more && issued < most[prod]) more = load_step();
            for (int k = max(0, issued - ns); rank == 0 && k < issued; k++) {
                const int g = prod + np * k, later = g + ns;
                if (later / np >= most[later % np] && !((stalled >> (g % ns)) & 1))
                    ptx::mbar_wait_bounded(&full[g % ns], (uint32_t)(g / ns) & 1, kDrainNs);
            }
        }
        meet();
    }
    if (warp == kMmaWarp) {
        // a commit arrives by itself, at both CTAs: each waits for the last
        // arrival at every barrier of its own before it gives up its tensor
        // memory and its shared memory (a barrier a lane)
        uint64_t *bar = nullptr;
        int last = 0;   // the phase of the last arrival
        if (lane < ns && lane < freed) {
            bar = &empty[lane];
            last = (freed - 1 - lane) / ns;
        } else if (lane >= 29 && lane - 29 < min(2, handed)) {
            bar = &acc_full[lane - 29];
            last = (handed - 1 - (lane - 29)) / 2;
        } else if (lane == 31) {
            bar = &done;
        }
        if (bar) ptx::mbar_wait_bounded(bar, (uint32_t)last & 1, kDrainNs);
        __syncwarp();
        tc5::fence_after();
        tc5::dealloc_pair(tmem, 2 * kAccCols);
    }
}

// The parts of split tiles, added in their order, and the bias: four columns a thread.
template <typename T>
__global__ void __launch_bounds__(256) k_fp8_join(const __grid_constant__ Args a) {
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int fours = a.half / 2, width = 2 * a.half;
    const unsigned tile = blockIdx.x / (unsigned)fours, tm = tile / a.tiles_n, tn = tile - tm * a.tiles_n;
    const int e = (int)(blockIdx.x % (unsigned)fours) * 256 + threadIdx.x, r = e / fours, x = (e - r * fours) * 4;
    const int64_t row = (int64_t)tm * 256 + r, c = (int64_t)tn * width + x;
    if (row >= a.rows || c >= a.M) return;
    float f[4] = {};
    for (int k = 0; k < a.splits; k++) {
        const float4 p = *reinterpret_cast<const float4 *>(a.parts + (((int64_t)tile * a.splits + k) * 256 + r) * width + x);
        f[0] += p.x, f[1] += p.y, f[2] += p.z, f[3] += p.w;
    }
    T *out = static_cast<T *>(a.Y) + row * a.M + c;
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (c + j < a.M) out[j] = from_f32<T>(f[j] + (a.bias ? __ldg(a.bias + c + j) : 0.f));
}

int pairs_of_sms() {
    int dev = 0, n = 152;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        cudaGetLastError();
    return std::max(1, n / 2);
}

struct Plan {
    int half, splits;
    int64_t tiles_m, tiles_n, units;   // (by rows: at most so many)
};

// Half the columns of a tile, and the parts of its steps, by the cycles that the
// busiest pair takes: a step, a unit's start and end, and a second launch that adds parts.
Plan plan_of(const Fp8Product &p) {
    const int64_t pairs = pairs_of_sms(), KB = fp8_blocks(p.a.cols);
    Plan best = {};
    double best_t = 0;
    for (int half : {128, 64, 32}) {
        Plan q = {half, 1, (p.a.rows + 255) / 256, (p.b.rows + 2 * half - 1) / (2 * half), 0};
        const double step = half == 128 ? 560 : half == 64 ? 400 : 330, unit = 1500 + 10 * half;
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (p.group != BSR_GROUP_NONE || s > KB)) break;
            q.splits = s;
            int64_t tiles = q.tiles_m * q.tiles_n;
            double steps = (double)((KB + s - 1) / s);
            if (p.group == BSR_GROUP_ROWS) {   // (as if every run ended in the middle of a tile)
                tiles = (p.a.rows / 256 + std::min<int64_t>(p.groups, p.a.rows)) * q.tiles_n;
            } else if (p.group == BSR_GROUP_COLUMNS) {
                tiles *= p.groups;
                steps = std::max(1.0, (double)KB / p.groups);
            }
            q.units = tiles * s;
            const double rounds = (double)((q.units + pairs - 1) / pairs);
            const double join = s > 1 ? 6000 + (double)q.units * 2 * half * 256 * 4 * 2 / 4000 : 0;
            const double t = rounds * (steps * step + unit) + join;
            if (best_t == 0 || t < best_t) best_t = t, best = q;
        }
    }
    return best;
}

cudaError_t encode(const bsr_fp8_matrix_t &m, bool batch, int rows, CUtensorMap *map) {
    auto enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t ld = (cuuint64_t)fp8_blocks(m.cols) * kFp8Block;
    const cuuint64_t dims[3] = {ld, (cuuint64_t)m.rows, (cuuint64_t)m.batch};
    const cuuint64_t strides[2] = {ld, ld * (cuuint64_t)m.rows};
    const cuuint32_t box[3] = {kFp8Block, (cuuint32_t)rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, batch ? 3 : 2, m.q, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

template <typename T, bool COL>
cudaError_t launch(const Args &a, unsigned grid, cudaStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    cudaError_t e = allow_smem(k_fp8_product<T, COL>, kMaxSmem, attr_set);
    if (e != cudaSuccess) return e;
    return launch_clusters(k_fp8_product<T, COL>, 2, dim3(grid), dim3(kThreads), a.ns * a.stage_bytes + kScaleBytes + 1024, s, a);
}

}  // namespace

int64_t fp8_product_workspace(const Fp8Product &p) {
    if (p.a.rows == 0 || p.b.rows == 0) return 0;
    const Plan q = plan_of(p);
    return q.splits > 1 ? q.units * 256 * 2 * q.half * 4 : 0;
}

cudaError_t launch_fp8_product(const Fp8Product &p, cudaStream_t s) {
    const Plan q = plan_of(p);
    if (q.units > INT32_MAX) return cudaErrorInvalidConfiguration;
    Args a = {};
    a.sa = p.a.scale, a.sb = p.b.scale, a.bias = p.bias;
    a.rows = p.a.rows, a.M = p.b.rows;
    a.sa_cols = fp8_scale_cols(p.a), a.sb_cols = fp8_scale_cols(p.b);
    a.KB = fp8_blocks(p.a.cols);
    a.a_shift = p.a.tile == 1 ? 0 : 7;
    a.group = p.group, a.E = p.groups;
    a.offsets = p.offsets;
    a.tiles_m = (unsigned)q.tiles_m, a.tiles_n = (unsigned)q.tiles_n;
    a.splits = q.splits;
    a.half = q.half;
    a.stage_bytes = kABytes + (uint32_t)q.half * kFp8Block;
    a.ns = (int)std::min<uint32_t>(kStages, (kMaxSmem - 1024 - kScaleBytes) / a.stage_bytes);
    a.idesc = tc5::idesc_8bit(p.a.type, p.b.type, 256, 2 * q.half);
    a.Y = p.Y;
    a.parts = p.ws;
    const uintptr_t addresses = reinterpret_cast<uintptr_t>(p.Y) | (uintptr_t)(p.b.rows * (p.dt == BSR_F32 ? 4 : 2)) | 16;
    a.align = (int)(addresses & (~addresses + 1));
    const char *limit = std::getenv("BSR_WAIT_LIMIT_NS"), *stall = std::getenv("BSR_TEST_STALL_CHUNK");
    a.wait_ns = limit ? std::strtoull(limit, nullptr, 10) : 1000000000ull;
    a.stall_step = stall ? std::atoi(stall) : -1;
    cudaError_t e = cudaSuccess;
    if (a.KB > 0) {   // (sums of nothing load nothing)
        e = encode(p.a, false, 128, &a.a);
        if (e == cudaSuccess) e = encode(p.b, true, q.half, &a.b);
    }
    if (e != cudaSuccess) return e;
    const unsigned grid = 2 * (unsigned)std::min<int64_t>(q.units, pairs_of_sms());
    const bool f32 = p.dt == BSR_F32, col = p.b.tile == 1;
    e = f32 ? (col ? launch<float, true>(a, grid, s) : launch<float, false>(a, grid, s))
            : (col ? launch<uint16_t, true>(a, grid, s) : launch<uint16_t, false>(a, grid, s));
    if (e != cudaSuccess || q.splits == 1) return e;
    const dim3 joins((unsigned)(q.tiles_m * q.tiles_n * (q.half / 2)));
    return launch_kernel(f32 ? k_fp8_join<float> : k_fp8_join<uint16_t>, joins, dim3(256), 0, s, a);
}

cudaError_t fp8_product_status(int *code) {
    const int ok = DEV_OK;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(code, g_status, sizeof ok);
    if (e == cudaSuccess && *code != ok) e = cudaMemcpyToSymbol(g_status, &ok, sizeof ok);
    return e;
}

}  // namespace bsr
