// Products of 8-bit operands on the tensor cores.
//
//   Y[n, m] = bias[m] + sum_b sa[b, n] sb[b, m] sum_{k in block b} qa[n, k] qb[m, k]
//
// A cluster of two CTAs works on a tile of 256 rows of a by 2 `half` rows of b. A
// block of 128 columns is a step: four MMAs (M = 256, N = 2 half, K = 32), which
// multiply by the rows' scales themselves, powers of two as bytes in tensor memory.
//
//   warps 0, 1     128 rows of a a CTA, 128 bytes each, by TMA (128-byte swizzle) into a
//                  stage of the ring, a step each in turn; every fourth block the
//                  rows' exponents of four blocks with it
//   warps 3, 4     the same of `half` rows of b
//   warp 2         MMAs of the pair's first CTA, and before them the exponents' copy
//                  from shared to tensor memory
//   warps 8 .. 15  epilogue: 32 rows and half of the columns each. Where 128 of b's rows
//                  share their scales, its rows are loaded in the order that leaves a thread 16
//                  columns side by side, and four lanes store 128 bytes of a row (bf16) straight from
//                  tensor memory; else through 2 KB of shared memory a warp
//
// Measured at 16384 tokens of 1024 features into 4096: scaling outside the MMAs (a fresh
// accumulator for each step, every value of it taken out, scaled and added in registers)
// 174 us; exponents made of fp32 scales by three more warps, whose way from the other CTA's
// registers every step waited for, 102, so bsr_fp8_quantize lays them out as tensor memory
// has them; results by shuffles 60, through buffers 55, straight 54, and put out of L2
// before the operands 48 to 50.
//
// What bounds it: 48 to 50 us there (2.75 to 2.85 PFLOP/s), the tensor pipe busy 54% of the
// time: with eight steps to a tile, the hand-over of an accumulator (1300 of 6600
// cycles: the commit, the shared columns' way out, the other CTA's word) and loads that
// take up to 3200 cycles while all CTAs store, as long as the ring's six steps; shared
// memory is at 27% of its rate, L2 at 38%. Sums of 4096 and 8192 columns: 2.65 and 2.75
// PFLOP/s, 560 to 600 cycles a step and the last round in part empty. Few tokens: 6 to
// 7 us, 5000 cycles until the first load, one tile's steps, and the way out.
//
// A step is 512 SM cycles of MMAs at 256 columns. Two accumulators of 256 columns and
// the exponents do not fit 512 columns: the second begins at column 192, and the
// epilogue takes the 64 columns that they share first, before the next tile's MMAs.
//
// The accumulators lose bits with every addition of 32 products, always towards zero: at
// most 2^-23 of a sum of one sign, 4e-9 a column (measured over 1024 columns 1.7e-7 on average,
// 6.1e-7 at most; over 16384 9.7e-6 and 1.2e-5). bf16 results: up to 16384 columns (2^-14 at most, where the result
// is rounded by up to 2^-8); fp32 ones: up to 1024 (4e-6). Longer sums are drained every 1024
// columns into registers, 128 a thread (handed over by the other warps).
//
// Persistent: one CTA per SM. Runs of rows: tiles of 256 rows from a multiple of 128 on,
// as the exponents lie, the rows of other runs left out; the table of the runs' tiles is
// made by every CTA from the offsets on the device.
// Runs of columns: a tile's steps are the run's, which ends where blocks do. Tiles of sums too few to fill the
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

constexpr int kEpiWarp0 = 8, kMmaWarp = 2, kEpiWarps = 8, kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kProducers = 2, kStages = 7, kLeastStages = 6;   // producers: of a, and of b; stages that fit, of 128 columns and of 256
constexpr uint32_t kABytes = 128 * 128;       // a CTA's rows of a, a step
constexpr uint32_t kOverlap = 64;             // columns that the accumulators of 256 columns share
// Tensor memory behind them: sets of exponents, of a in the first four of 16 columns.
constexpr uint32_t kScaleCol = 512 - kOverlap, kScaleCols = 16, kAllCols = 512;
constexpr int kScaleSets = kOverlap / kScaleCols;
constexpr int kScaleSteps = 4;                // blocks whose exponents make a word
constexpr uint32_t kScaleBytes = 3 * 512;     // a stage's exponents: of 128 rows of a, 256 of b
constexpr int kDrainSteps = 8;                // steps of a drained accumulator, and of fp32 sums that are not drained
constexpr int kMostSteps = 128;               // of bf16 ones
constexpr uint32_t kTurnBytes = 2048;         // of an epilogue warp: 32 rows of 64 bytes
constexpr uint32_t kMaxSmem = 227 * 1024 - 9 * 1024;   // (static: the runs' table, barriers)
constexpr uint64_t kDrainNs = 200000000ull;   // bound for copies and MMAs already issued
// Registers of a thread: 8 warps of 56 and 8 of 200 are what 512 threads are launched with (128 each).
constexpr int kFewRegs = 56, kManyRegs = 200;

__device__ int g_status;

struct Args {
    CUtensorMap a, b, ea, eb; // values; exponents
    const float *bias;
    int64_t rows, M, KB;      // of a; of b (columns of Y); blocks
    int64_t cols;             // of a and b
    int group, E;
    const int32_t *offsets;
    unsigned tiles_m, tiles_n;
    int splits;               // of a tile's steps, each a multiple of kScaleSteps
    int half, ns;
    uint32_t stage_bytes, idesc;
    void *Y;
    float *parts;             // [units][256][2 half] where splits > 1
    int align;                // bytes (at most 16) that rows of Y are aligned to
    uint64_t wait_ns;
    int stall_step;           // test hook: this step of each tile is never loaded (-1: none)
};

struct Unit {
    int64_t m0, r0, r1, n0;   // first row; the rows that are the unit's; first column
    int64_t out;              // rows of Y before this unit's matrix
    int batch, part;
    int i0, i1;               // steps
    float fill;               // the result of no steps
};

// The runs: their ends, and the tiles of rows before each; of columns, whether the end is none.
struct Runs {
    int32_t at[kMostExperts + 1];
    uint32_t first[kMostExperts + 1];
};

// What the units follow from, in registers.
struct Sizes {
    int64_t rows;
    int KB, group, E, splits, width;   // width: columns of a tile
    unsigned tiles_m, tiles_n;
};

__device__ __forceinline__ Unit unit_of(const Sizes &a, const Runs &r, unsigned v) {
    Unit u;
    u.out = 0;
    u.batch = 0;
    u.part = -1;
    u.i0 = 0;
    u.i1 = a.KB;
    u.fill = 0.f;
    if (a.group == BSR_GROUP_ROWS) {
        const unsigned t = v / a.tiles_n;
        int lo = 0, hi = a.E;   // the last run whose tiles begin at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (r.first[mid] <= t) lo = mid;
            else hi = mid;
        }
        u.batch = lo;
        u.r0 = r.at[lo];
        u.r1 = r.at[lo + 1];
        u.m0 = u.r0 / 128 * 128 + (int64_t)(t - r.first[lo]) * 256;
        u.n0 = (int64_t)(v - t * a.tiles_n) * a.width;
        return u;
    }
    unsigned tile = v;
    if (a.group == BSR_GROUP_COLUMNS) {
        const unsigned tiles = a.tiles_m * a.tiles_n, e = v / tiles;
        tile = v - e * tiles;
        u.out = (int64_t)e * a.rows;
        u.i0 = r.at[e];
        u.i1 = max(r.at[e], r.at[e + 1]);
        if (r.first[e] | r.first[e + 1]) u.i1 = u.i0, u.fill = __uint_as_float(0x7fffffffu);   // NaN
    } else if (a.splits > 1) {
        u.part = (int)v;
        tile = v / (unsigned)a.splits;
        const unsigned k = v - tile * (unsigned)a.splits, words = (unsigned)(a.KB + kScaleSteps - 1) / kScaleSteps;
        u.i0 = (int)(words * k / (unsigned)a.splits) * kScaleSteps;
        u.i1 = min(a.KB, (int)(words * (k + 1) / (unsigned)a.splits) * kScaleSteps);
    }
    const unsigned tm = tile / a.tiles_n;
    u.m0 = (int64_t)tm * 256;
    u.r0 = 0;
    u.r1 = a.rows;
    u.n0 = (int64_t)(tile - tm * a.tiles_n) * a.width;
    return u;
}

// One copy of the code for all roles, as cold instructions are what a short call waits
// for; but for drained sums, whose registers a call would push out.
__device__ __noinline__ Unit unit_call(Sizes a, const Runs &r, unsigned v) { return unit_of(a, r, v); }
template <bool DRAIN>
__device__ __forceinline__ Unit unit_at(const Sizes &a, const Runs &r, unsigned v) {
    return DRAIN ? unit_of(a, r, v) : unit_call(a, r, v);
}

// A bounded wait that gives up when another role stopped; the timer is read every 64 tries.
__device__ __forceinline__ bool wait_long(uint64_t *bar, uint32_t parity, uint64_t limit_ns, const int *flag) {
    uint64_t t0 = 0;
    while (true) {
#pragma unroll 1
        for (int k = 0; k < 64; k++)
            if (ptx::mbar_try_wait(bar, parity)) return true;
        if (aborted(flag)) return false;
        const uint64_t t = ptx::globaltimer();
        if (t0 == 0) t0 = t;
        else if (t - t0 > limit_ns) return false;
    }
}
// (its code once for all roles, as unit_call)
__device__ __noinline__ bool wait_call(uint64_t *bar, uint32_t parity, uint64_t limit_ns, const int *flag) {
    return wait_long(bar, parity, limit_ns, flag);
}
template <bool DRAIN>
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, uint64_t limit_ns, const int *flag) {
    return ptx::mbar_try_wait(bar, parity) || (DRAIN ? wait_long(bar, parity, limit_ns, flag) : wait_call(bar, parity, limit_ns, flag));
}
// Stops every role of the pair; a timeout is recorded.
__device__ __forceinline__ void halt_pair(int *stop, uint32_t rank) {
    if (!aborted(stop)) set_status(&g_status, DEV_TIMEOUT);
    atomicExch(stop, 1);
    ptx::store_cluster(ptx::map_to_cta(stop, rank ^ 1), 1);
}

__device__ __noinline__ void halt_call(int *stop, uint32_t rank) { halt_pair(stop, rank); }

// Tiles of the rows o .. p - 1, from a multiple of 128 on.
__device__ __forceinline__ uint32_t tiles_of(int32_t o, int32_t p) {
    return p > o ? ((uint32_t)p - (uint32_t)o / 128 * 128 + 255) / 256 : 0;
}

// The unit of a pair in a round of them: all rounds but the first are taken
// backwards, so that who had a long unit there is the last to have one more.
__device__ __forceinline__ unsigned unit_in(unsigned round, unsigned pair, unsigned pairs) {
    return round * pairs + (round ? pairs - 1 - pair : pair);
}

// Where 16 bytes of the 64 of a row lie, so that eight lanes' rows, and the four runs of two rows, fall on different banks.
__device__ __forceinline__ uint4 *turned(unsigned char *buf, int row, int chunk) {
    return reinterpret_cast<uint4 *>(buf + row * 64 + 16 * (chunk ^ ((row >> 1) & 3)));
}

// 16 rows of the result from `row` on x 64 columns from c on, of b's rows in order: x as
// tc5::ld_16x64 leaves it is 16 columns from c + 16 (lane % 4) on of this thread, of rows
// lane / 4 and + 8. The stores ask to be put out of L2 before the operands, which other
// CTAs read (16384 tokens of 1024 into 4096: 54 us without, 49.5 so). The lanes, parted by
// their rows, meet at the end: the next tc5::ld_16x64 is one instruction of the warp.
template <typename T>
__device__ __forceinline__ void put_ordered(const Args &a, const Unit &un, int64_t row, int64_t c, float (&x)[32]) {
    const int lane = threadIdx.x & 31;
    c += 16 * (lane & 3);
    row += lane >> 2;
    const bool there = c < a.M;   // (64 columns are there or not)
    if (there && a.bias) {
        const float *bias = a.bias + (int64_t)un.batch * a.M + c;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float b0 = bias[2 * i], b1 = bias[2 * i + 1];
            x[4 * i] += b0, x[4 * i + 1] += b1, x[4 * i + 2] += b0, x[4 * i + 3] += b1;
        }
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        if (!there || row + 8 * h < un.r0 || row + 8 * h >= un.r1) continue;
        T *out = static_cast<T *>(a.Y) + (un.out + row + 8 * h) * a.M + c;
        uint32_t w[8];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = pack_bf16(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]);
            ptx::st_global_32_first_out(out, w);
        } else {
#pragma unroll
            for (int k = 0; k < 2; k++) {
#pragma unroll
                for (int i = 0; i < 4; i++)
                    w[2 * i] = __float_as_uint(x[16 * k + 4 * i + 2 * h]), w[2 * i + 1] = __float_as_uint(x[16 * k + 4 * i + 2 * h + 1]);
                ptx::st_global_32_first_out(out + 8 * k, w);
            }
        }
    }
    __syncwarp();
}

// 32 rows of the result from `row` on x 32 columns from c on; x: those of row + lane.
template <typename T>
__device__ __forceinline__ void put(const Args &a, const Unit &un, int64_t row, int64_t c, float (&x)[32], unsigned char *buf) {
    const int lane = threadIdx.x & 31, up = lane >> 2, chunk = lane & 3;
    const bool part = un.part >= 0;
    if (a.bias && !part) {
        const float *bias = a.bias + (int64_t)un.batch * a.M + c;
#pragma unroll
        for (int j = 0; j < 32; j++) x[j] += c + j < a.M ? bias[j] : 0.f;
    }
    if (sizeof(T) == 2 && !part) {
#pragma unroll
        for (int j = 0; j < 4; j++)
            *turned(buf, lane, j) = make_uint4(pack_bf16(x[8 * j], x[8 * j + 1]), pack_bf16(x[8 * j + 2], x[8 * j + 3]),
                                               pack_bf16(x[8 * j + 4], x[8 * j + 5]), pack_bf16(x[8 * j + 6], x[8 * j + 7]));
        __syncwarp();
        T *out = static_cast<T *>(a.Y) + (un.out + row + up) * a.M + c + 8 * chunk;
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = *turned(buf, up + 8 * i, chunk);
        const int lo = (int)max((int64_t)-1, min((int64_t)32, un.r0 - row - up)), hi = (int)max((int64_t)-1, min((int64_t)32, un.r1 - row - up));
        const int64_t n = a.M - (c + 8 * chunk);
        if (a.align == 16 && n >= 8) {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (8 * i >= lo && 8 * i < hi) *reinterpret_cast<uint4 *>(out + 8 * i * a.M) = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                Eight<uint16_t> e;
                e.w[0] = w[i].x, e.w[1] = w[i].y, e.w[2] = w[i].z, e.w[3] = w[i].w;
                if (8 * i >= lo && 8 * i < hi) store8(reinterpret_cast<uint16_t *>(out + 8 * i * a.M), n, a.align, e);
            }
        }
        __syncwarp();
    } else {
        // (fp32: 16 columns at a time)
#pragma unroll
        for (int half = 0; half < 2; half++) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float *v = x + 16 * half + 4 * j;
                *turned(buf, lane, j) = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            }
            __syncwarp();
            const int64_t at = c + 16 * half + 4 * chunk;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint4 w = *turned(buf, up + 8 * i, chunk);
                const int64_t r = row + up + 8 * i;
                if (part) {
                    *reinterpret_cast<uint4 *>(a.parts + ((int64_t)un.part * 256 + (r - un.m0)) * 2 * a.half + (at - un.n0)) = w;
                } else if (r >= un.r0 && r < un.r1) {
                    float *out = static_cast<float *>(a.Y) + (un.out + r) * a.M + at;
                    if (at + 4 <= a.M && a.align == 16) {
                        *reinterpret_cast<uint4 *>(out) = w;
                    } else {
                        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; j++)
                            if (at + j < a.M) out[j] = __uint_as_float(v[j]);
                    }
                }
            }
            __syncwarp();
        }
    }
}

template <typename T, bool DRAIN, bool ORDERED>
__global__ void __launch_bounds__(kThreads, 1) k_fp8_product(const __grid_constant__ Args a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *base = ptx::align_smem(smem_raw);
    const int ns = a.ns;
    const uint32_t stage_bytes = a.stage_bytes;
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], done;
    __shared__ int stop, loads[2][kProducers][2];   // loads[a or b][producer][CTA of the pair]: steps loaded
    __shared__ int freed, handed;                // commits issued to `empty` and to `acc_full`
    __shared__ uint32_t tmem_s;
    __shared__ Runs runs;

    // (a shuffle, so that the warp index and what follows from it is uniform)
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();
    const unsigned pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) stop = freed = handed = 0;
    if (threadIdx.x < 32) {   // a barrier a lane: two producers' arrivals with their bytes, commits, the epilogue warps of both CTAs
        if (lane < kStages) ptx::mbar_init(&full[lane], 2);
        else if (lane < 2 * kStages) ptx::mbar_init(&empty[lane - kStages], 1);
        else if (lane < 2 * kStages + 2) ptx::mbar_init(&acc_full[lane & 1], 1);
        else if (lane < 2 * kStages + 4) ptx::mbar_init(&acc_empty[lane & 1], 2 * kEpiWarps);
        else if (lane == 31) ptx::mbar_init(&done, 1);
        ptx::fence_barrier_init();
    }
    if (warp == kMmaWarp) tc5::alloc_pair(&tmem_s, kAllCols);
    if (warp == 1 && a.KB > 0 && ptx::elect_one()) {
        ptx::prefetch_tensormap(&a.a);
        ptx::prefetch_tensormap(&a.b);
        ptx::prefetch_tensormap(&a.ea);
        ptx::prefetch_tensormap(&a.eb);
    }
    tc5::fence_before();
    __syncthreads();
    ptx::cluster_barrier();   // the other CTA's barriers exist
    tc5::fence_after();
    ptx::pdl_launch_dependents();   // (after the allocation: ptx.cuh)
    ptx::pdl_wait();                // operands and offsets may be an earlier kernel's, and Y may be read by one
    unsigned units = a.tiles_m * a.tiles_n * (unsigned)a.splits;
    if (a.group != BSR_GROUP_NONE) {
        // within what there is, in steps for columns: an offset inside a block, whose columns
        // share scales and MMAs, is reported, and the runs that it ends are NaN
        const bool by_rows = a.group == BSR_GROUP_ROWS;
        for (int e = threadIdx.x; e <= a.E; e += kThreads) {
            const int64_t o = max(0, a.offsets[e]);
            if (by_rows) {
                runs.at[e] = (int32_t)min(o, a.rows);
                continue;
            }
            runs.at[e] = (int32_t)(o < a.cols ? o / kFp8Block : a.KB);
            runs.first[e] = o < a.cols && o % kFp8Block != 0;
            if (runs.first[e]) set_status(&g_status, DEV_OFFSETS);
        }
        __syncthreads();
        if (warp == 0 && by_rows) {
            uint32_t before = 0;
            for (int e0 = 0; e0 < a.E; e0 += 32) {
                const int e = e0 + lane;
                const uint32_t tiles = e < a.E ? tiles_of(runs.at[e], runs.at[e + 1]) : 0;
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
    const Sizes sizes = {a.rows, (int)a.KB, a.group, a.E, a.splits, 2 * a.half, a.tiles_m, a.tiles_n};
    const uint32_t tmem = tmem_s;
    const bool elected = ptx::elect_one();
    auto halt = [&]() {
        if (!elected) return;
        if (DRAIN) halt_pair(&stop, rank);
        else halt_call(&stop, rank);
    };

    // ---- producers: the pair's steps prod, prod + np, ... No more producers
    // than stages: one that waits for step g - ns to be consumed has to know that
    // step g - 2 ns was, or the stage's barrier, which tells phases apart by their
    // parity, would let it pass a round early; its last wait, for step
    // g - np - ns, tells it so if np <= ns.
    constexpr int np = kProducers;
    const bool producer = warp < 5 && warp != kMmaWarp, of_b = warp > kMmaWarp;
    const int prod = of_b ? warp - 3 : warp;
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
            un = unit_at<DRAIN>(sizes, runs, v);
            i = un.i0 + over;
        }
        return true;
    };
    auto load_step = [&]() {
        if (i - un.i0 == a.stall_step) {   // never loaded: its consumer times out
            stalled |= 1u << s;
        } else if (elected) {
            const uint32_t dst = smem0 + s * stage_bytes, bar = first0 + 8 * s;
            const bool scales = i == un.i0 || i % kScaleSteps == 0;
            const int m = (int)(un.m0 + rank * 128), n = (int)un.n0, nb = n + (int)rank * a.half;
            const uint32_t words = of_b ? (a.half == 128 ? 1024 : 512) : 512;
            if (rank == 0) ptx::mbar_arrive_expect_tx_at(bar0 + 8 * s, 2 * ((of_b ? stage_bytes - kABytes : kABytes) + (scales ? words : 0)));
            const uint32_t to = smem0 + ns * stage_bytes + s * kScaleBytes;
            if (!of_b) {
                ptx::tma_load_2d_pair_at(dst, &a.a, i * kFp8Block, m, bar);
                if (scales) ptx::tma_load_3d_pair_at(to, &a.ea, 0, m / 128, i / kScaleSteps, bar);
            } else {
                if constexpr (ORDERED) ptx::tma_load_5d_pair_at(dst + kABytes, &a.b, i * kFp8Block, 0, 0, 0, (int)((un.batch * a.M + nb) / 64), bar);
                else ptx::tma_load_3d_pair_at(dst + kABytes, &a.b, i * kFp8Block, nb, un.batch, bar);
                if (scales) ptx::tma_load_4d_pair_at(to + 512, &a.eb, 0, n / 128, i / kScaleSteps, un.batch, bar);
            }
        }
        issued++;
        for (s += np; s >= ns; s -= ns) phase ^= 1;
        i += np;
        return seek();
    };
    bool more = false;
    // Accumulators: of 256 columns they share kOverlap, and the epilogue hands those of
    // one tile over for the next tile's; narrower ones are handed back for the next but one.
    const bool shared_cols = a.half == 128;
    const uint32_t acc_step = shared_cols ? 256 - kOverlap : 128;
    if (warp >= kEpiWarp0) {
        if constexpr (DRAIN) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
        const int q = warp & 3, share = (warp - kEpiWarp0) >> 2;   // tensor-memory lanes 32 q .., half the columns
        const int groups = a.half / 32, first = share * groups;      // of 32 columns
        unsigned char *buf = base + (size_t)ns * (stage_bytes + kScaleBytes) + (warp - kEpiWarp0) * kTurnBytes;
        int ab = 0;
        uint32_t fphase = 0;
        bool ok = true;
        auto wait_acc = [&](const Unit &u) {
            ok = __all_sync(0xffffffffu, wait_for<DRAIN>(&acc_full[ab], fphase, a.wait_ns * (uint64_t)(u.i1 - u.i0 + 2), &stop));
            if (!ok) halt();
            tc5::fence_after();
            return tmem + (uint32_t)ab * acc_step + ((uint32_t)(32 * q) << 16) + 32 * first;
        };
        auto hand_back = [&]() {
            tc5::fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_remote(ptx::map_to_cta(&acc_empty[ab], 0));
        };
        auto next_acc = [&]() {
            ab ^= 1;
            if (ab == 0) fphase ^= 1;
        };
        auto loaded = [&](uint32_t (&r)[32]) {
#pragma unroll
            for (int j = 0; j < 32; j++) asm volatile("" : "+r"(r[j]));   // no use of a loaded register moves above the wait
        };
        for (; ok && v < units; v = unit_in(++round, pair, pairs)) {
            un = unit_at<DRAIN>(sizes, runs, v);
            const int64_t row = un.m0 + rank * 128 + 32 * q, col = un.n0 + 32 * first;
            if constexpr (!DRAIN) {
                const bool any = un.i1 > un.i0;
                uint32_t tm = 0;
                // the columns that the next tile's accumulator has too, first: two groups of one share
                const bool back = shared_cols && ab == 0, mine = !shared_cols || (ab == 0 ? share == 1 : share == 0);
                if (any) {
                    tm = wait_acc(un);
                    if (!ok) break;
                    if (!mine) hand_back();
                }
#pragma unroll 1
                for (int p = 0; p < groups; p += 2) {
                    const int g = back ? groups - 2 - p : p;
                    uint32_t r[2][32];
#pragma unroll
                    for (int j = 0; j < 32; j++) r[0][j] = r[1][j] = __float_as_uint(un.fill);
                    if (any) {
                        if constexpr (ORDERED) {
                            tc5::ld_16x64(tm + 32 * g, r[0]);
                            tc5::ld_16x64(tm + (16u << 16) + 32 * g, r[1]);
                        } else {
                            tc5::ld32(tm + 32 * g, r[0]);
                            tc5::ld32(tm + 32 * g + 32, r[1]);
                        }
                        tc5::ld_wait();
                        loaded(r[0]);
                        loaded(r[1]);
                        if (mine && p == 0) hand_back();   // (narrow tiles: all columns)
                    }
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        float x[32];
#pragma unroll
                        for (int j = 0; j < 32; j++) x[j] = __uint_as_float(r[k][j]);
                        if constexpr (ORDERED) put_ordered<T>(a, un, row + 16 * k, col + 32 * g, x);
                        else put<T>(a, un, row, col + 32 * (g + k), x, buf);
                    }
                }
                if (any) next_acc();
            } else {
                float sum[4][32];   // [32 columns, or ORDERED 16 rows of 64]
#pragma unroll
                for (int g = 0; g < 4; g++)
#pragma unroll
                    for (int j = 0; j < 32; j++) sum[g][j] = un.fill;
                for (int b = un.i0; b < un.i1; b += kDrainSteps) {
                    const uint32_t tm = wait_acc(un);
                    if (!ok) break;
                    // handed back after its shared columns, if it has them (the last group's at the end)
                    const int back = !shared_cols ? groups - 1 : share == ab ? -1 : share == 0 ? 1 : 3;
                    if (back < 0) hand_back();
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        if (g >= groups) break;
                        uint32_t r[32];
                        if constexpr (ORDERED) tc5::ld_16x64(tm + ((uint32_t)(16 * (g & 1)) << 16) + 64 * (g / 2), r);
                        else tc5::ld32(tm + 32 * g, r);
                        tc5::ld_wait();
                        loaded(r);
                        if (g == back) hand_back();
#pragma unroll
                        for (int j = 0; j < 32; j++) sum[g][j] += __uint_as_float(r[j]);
                    }
                    next_acc();
                }
                if (!ok) break;
                // one copy of the code, the sums handed on from group to group
#pragma unroll 1
                for (int g = 0; g < groups; g++) {
                    if constexpr (ORDERED) put_ordered<T>(a, un, row + 16 * (g & 1), col + 64 * (g / 2), sum[0]);
                    else put<T>(a, un, row, col + 32 * g, sum[0], buf);
#pragma unroll
                    for (int k = 0; k < 3; k++)
#pragma unroll
                        for (int j = 0; j < 32; j++) sum[k][j] = sum[k + 1][j];
                }
            }
        }
    } else {
        if constexpr (DRAIN) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
        if (producer) {
            if (v < units) {
                un = unit_at<DRAIN>(sizes, runs, v);
                i = un.i0 + prod;
                more = seek();
            }
            while (more) {
                const bool got = wait_for<DRAIN>(&empty[s], phase, a.wait_ns, &stop);
                if (!__all_sync(0xffffffffu, got && !aborted(&stop))) {
                    halt();
                    break;
                }
                more = load_step();
            }
            if (elected) {
                loads[of_b][prod][rank] = issued;
                ptx::store_cluster(ptx::map_to_cta(&loads[of_b][prod][rank], rank ^ 1), (uint32_t)issued);
            }
        } else if (warp == kMmaWarp && rank == 0) {
            if (elected) {   // (one thread throughout: what the others would cost is in the MMAs' way)
                int n_steps = 0, n_acc = 0, n_sets = 0;
                uint32_t fphase = 0;
                // the last steps of the last sets of exponents, the oldest first, with their stages and phases
                int end_step[kScaleSets], end_stage[kScaleSets];
                uint32_t end_phase[kScaleSets];
                bool ok = true;
                s = 0;
                const uint64_t ad0 = tc5::desc_sw128(smem0), bd0 = tc5::desc_sw128(smem0 + kABytes);
                const uint64_t sd0 = tc5::desc(smem0 + ns * stage_bytes, 16, 128);   // (eight rows of 16 bytes side by side)
                uint32_t set = tmem + kScaleCol - kScaleCols;
                for (; ok && v < units; v = unit_in(++round, pair, pairs)) {
                    un = unit_at<DRAIN>(sizes, runs, v);
                    for (i = un.i0; i < un.i1; i++) {
                        const int b = i - un.i0;
                        const bool fresh = DRAIN ? b % kDrainSteps == 0 : b == 0, last = i + 1 == un.i1 || (DRAIN && (b + 1) % kDrainSteps == 0);
                        const bool scales = b == 0 || i % kScaleSteps == 0;
                        if (scales) {
                            // the set's last readers are done (a copy does not wait for MMAs): so the stage's
                            // barrier says, or the stage has been filled again since
                            set = n_sets % kScaleSets == 0 ? tmem + kScaleCol : set + kScaleCols;
                            if (n_sets >= kScaleSets && n_steps - end_step[0] <= ns)
                                ok = wait_for<DRAIN>(&empty[end_stage[0]], end_phase[0], a.wait_ns, &stop);
                            n_sets++;
#pragma unroll
                            for (int k = 0; k + 1 < kScaleSets; k++)
                                end_step[k] = end_step[k + 1], end_stage[k] = end_stage[k + 1], end_phase[k] = end_phase[k + 1];
                        }
                        ok = ok && wait_for<DRAIN>(&full[s], fphase, a.wait_ns, &stop);
                        if (!ok) break;
                        tc5::fence_after();
                        if (scales) {
                            const uint64_t sd = sd0 + (uint64_t)((s * kScaleBytes) >> 4);
                            tc5::copy_pair_32x16(set, sd);
                            tc5::copy_pair_32x16(set + 4, sd + (512 >> 4));
                            if (shared_cols) tc5::copy_pair_32x16(set + 8, sd + (1024 >> 4));
                        }
                        if (fresh) {   // the accumulator before (the next but one) is taken out as far as it must be
                            const int before = n_acc - (shared_cols ? 1 : 2);
                            if (before >= 0) {
                                ok = wait_for<DRAIN>(&acc_empty[before & 1], (uint32_t)(before >> 1) & 1, a.wait_ns, &stop);
                                if (!ok) break;
                                tc5::fence_after();
                            }
                        }
                        const uint64_t stage = (uint64_t)((s * stage_bytes) >> 4);
                        const uint32_t idesc = a.idesc | tc5::idesc_byte((uint32_t)i % kScaleSteps), acc = tmem + (uint32_t)(n_acc & 1) * acc_step;
#pragma unroll
                        for (int j = 0; j < kFp8Block / 32; j++)   // (32 bytes along the rows)
                            tc5::mma_ss_pair_scaled(acc, ad0 + stage + 2 * j, bd0 + stage + 2 * j, idesc, set, set + 4, !fresh | (j > 0));
                        tc5::commit_pair(&empty[s]);
                        if (last) {
                            tc5::commit_pair(&acc_full[n_acc & 1]);
                            n_acc++;
                        }
                        end_step[kScaleSets - 1] = n_steps, end_stage[kScaleSets - 1] = s, end_phase[kScaleSets - 1] = fphase;
                        n_steps++;
                        if (++s == ns) {
                            s = 0;
                            fphase ^= 1;
                        }
                    }
                    if (!ok) halt();
                }
                // every MMA issued has completed before the tensor memory is freed
                tc5::commit_pair(&done);
                freed = n_steps, handed = n_acc;
                ptx::store_cluster(ptx::map_to_cta(&freed, 1), (uint32_t)n_steps);
                ptx::store_cluster(ptx::map_to_cta(&handed, 1), (uint32_t)n_acc);
            }
            __syncwarp();
            ptx::mbar_wait_bounded(&done, 0, kDrainNs);
        }
    }
    // every MMA completed (the issuer waited for `done`), and neither CTA reads
    // or signals the other's shared memory any more
    tc5::fence_before();
    ptx::cluster_barrier();
    if (aborted(&stop)) {
        // (the same for both CTAs.) The loads that only some of a step's producers
        // issued are completed by the others, so that every barrier phase can
        // finish, and the CTA whose barriers count the bytes waits for those
        // that no later load of their stage shows to be complete: no copy
        // outlives the CTAs
        if (producer) {
            int most[kProducers];
            for (int p = 0; p < np; p++) most[p] = max(max(loads[0][p][0], loads[0][p][1]), max(loads[1][p][0], loads[1][p][1]));
            while (more && issued < most[prod]) more = load_step();
            for (int k = max(0, issued - ns); rank == 0 && k < issued; k++) {
                const int g = prod + np * k, later = g + ns;
                if (later / np >= most[later % np] && !((stalled >> (g % ns)) & 1))
                    ptx::mbar_wait_bounded(&full[g % ns], (uint32_t)(g / ns) & 1, kDrainNs);
            }
        }
        ptx::cluster_barrier();
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
        tc5::dealloc_pair(tmem, kAllCols);
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
        if (c + j < a.M) out[j] = from_f32<T>(f[j] + (a.bias ? a.bias[c + j] : 0.f));
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
// Measured (bf16, one tile a pair): a step of 256 columns 0.26 to 0.34 us, of 128 0.19 to 0.22. What
// is chosen against the other side, us: 256 tokens of 1024 into 1024 128 columns 6.3, 256 7.5; 4096 tokens
// 256 columns 8.6, 128 9.5; 16384 of 1024 into 4096 50 and 62; 3000 of 768 into 768 128 columns 7.3, 256 7.5. Splits: 64 of 4096 into 1024
// four 9.1, none 11.2; 256 of 16384 into 1024 eight to ten 13.5, none 28.7; 1024 of 1024 into 1024 none 6.4, two 10.2.
Plan plan_of(const Fp8Product &p) {
    const int64_t pairs = pairs_of_sms(), KB = fp8_blocks(p.a.cols), words = (KB + kScaleSteps - 1) / kScaleSteps;
    Plan best = {};
    double best_t = 0;
    for (int half : {128, 64}) {
        Plan q = {half, 1, (p.a.rows + 255) / 256, (p.b.rows + 2 * half - 1) / (2 * half), 0};
        const double step = half == 128 ? 540 : 400, unit = 1000 + 10 * half;
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (p.group != BSR_GROUP_NONE || s > words)) break;
            q.splits = s;
            int64_t tiles = q.tiles_m * q.tiles_n;
            double steps = s == 1 ? (double)KB : (double)((words + s - 1) / s * kScaleSteps);
            if (p.group == BSR_GROUP_ROWS) {   // (as if every run ended in the middle of a tile)
                tiles = (p.a.rows / 256 + 2 * std::min<int64_t>(p.groups, p.a.rows)) * q.tiles_n;
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

// b's rows in groups of 64, a group's in the order that gives a thread 16 columns side by
// side (row 8 i + 2 q + e of a box: 16 q + 2 i + e of the group; i < 8, q < 4, e < 2).
cudaError_t encode_ordered(const bsr_fp8_matrix_t &m, int rows, CUtensorMap *map) {
    auto enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t ld = (cuuint64_t)fp8_blocks(m.cols) * kFp8Block;
    const cuuint64_t dims[5] = {ld, 2, 4, 8, (cuuint64_t)(m.batch * m.rows / 64)};
    const cuuint64_t strides[4] = {ld, 16 * ld, 2 * ld, 64 * ld};
    const cuuint32_t box[5] = {kFp8Block, 2, 4, 8, (cuuint32_t)(rows / 64)};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, m.q, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

cudaError_t encode_exponents(const bsr_fp8_matrix_t &m, bool batch, int rows, CUtensorMap *map) {
    auto enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t runs = (cuuint64_t)fp8_blocks(m.rows), words = (cuuint64_t)fp8_words(m.cols);
    const cuuint64_t dims[4] = {128, runs, words, (cuuint64_t)m.batch};
    const cuuint64_t strides[3] = {512, 512 * runs, 512 * runs * words};
    const cuuint32_t box[4] = {128, (cuuint32_t)(rows / 128), 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, batch ? 4 : 3, m.exponent, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

// Whether results go to memory straight from tensor memory: the order of b's rows must not
// matter to their exponents, tiles' 64 columns be all there, and rows of Y start on 32 bytes.
bool ordered(const Fp8Product &p, const Plan &q) {
    return p.b.tile == kFp8Block && p.b.rows % 64 == 0 && q.splits == 1 && reinterpret_cast<uintptr_t>(p.Y) % 32 == 0;
}

template <typename T, bool DRAIN, bool ORDERED>
cudaError_t launch(const Args &a, unsigned grid, cudaStream_t s) {
    static std::atomic<uint64_t> attr_set{0};
    cudaError_t e = allow_smem(k_fp8_product<T, DRAIN, ORDERED>, kMaxSmem, attr_set);
    if (e != cudaSuccess) return e;
    return launch_clusters(k_fp8_product<T, DRAIN, ORDERED>, 2, dim3(grid), dim3(kThreads), a.ns * (a.stage_bytes + kScaleBytes) + kEpiWarps * kTurnBytes + 1024, s, a);
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
    a.bias = p.bias;
    a.rows = p.a.rows, a.M = p.b.rows;
    a.KB = fp8_blocks(p.a.cols), a.cols = p.a.cols;
    a.group = p.group, a.E = p.groups;
    a.offsets = p.offsets;
    a.tiles_m = (unsigned)q.tiles_m, a.tiles_n = (unsigned)q.tiles_n;
    a.splits = q.splits;
    a.half = q.half;
    a.stage_bytes = kABytes + (uint32_t)q.half * kFp8Block;
    static_assert(kLeastStages * (2 * kABytes + kScaleBytes) + kEpiWarps * kTurnBytes + 1024 <= kMaxSmem, "stages");
    a.ns = (int)std::min<uint32_t>(kStages, (kMaxSmem - 1024 - kEpiWarps * kTurnBytes) / (a.stage_bytes + kScaleBytes));
    a.idesc = tc5::idesc_scaled(p.a.type, p.b.type, 256, 2 * q.half);
    a.Y = p.Y;
    a.parts = p.ws;
    const uintptr_t addresses = reinterpret_cast<uintptr_t>(p.Y) | (uintptr_t)(p.b.rows * (p.dt == BSR_F32 ? 4 : 2)) | 16;
    a.align = (int)(addresses & (~addresses + 1));
    const char *limit = std::getenv("BSR_WAIT_LIMIT_NS"), *stall = std::getenv("BSR_TEST_STALL_CHUNK");
    a.wait_ns = limit ? std::strtoull(limit, nullptr, 10) : 1000000000ull;
    a.stall_step = stall ? std::atoi(stall) : -1;
    const bool order = ordered(p, q);
    cudaError_t e = cudaSuccess;
    if (a.KB > 0) {   // (sums of nothing load nothing)
        e = encode(p.a, false, 128, &a.a);
        if (e == cudaSuccess) e = order ? encode_ordered(p.b, q.half, &a.b) : encode(p.b, true, q.half, &a.b);
        if (e == cudaSuccess) e = encode_exponents(p.a, false, 128, &a.ea);
        if (e == cudaSuccess) e = encode_exponents(p.b, true, q.half == 128 ? 256 : 128, &a.eb);
    }
    if (e != cudaSuccess) return e;
    const unsigned grid = 2 * (unsigned)std::min<int64_t>(q.units, pairs_of_sms());
    const int64_t steps = q.splits == 1 ? a.KB : (fp8_words(p.a.cols) + q.splits - 1) / q.splits * kScaleSteps;
    const bool f32 = p.dt == BSR_F32, drained = steps > (f32 ? kDrainSteps : kMostSteps);
    auto run = [&](auto t) {
        using T = decltype(t);
        if (order) return drained ? launch<T, true, true>(a, grid, s) : launch<T, false, true>(a, grid, s);
        return drained ? launch<T, true, false>(a, grid, s) : launch<T, false, false>(a, grid, s);
    };
    e = f32 ? run(float()) : run(uint16_t());
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
