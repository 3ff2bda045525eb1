// The products of the gated feed-forward block on the tensor cores.
//
// One kernel for three of them: G and U with the activation and the product (or
// its derivatives) on the way out, and the plain products of the backward pass.
// A cluster of two CTAs works on a tile of 256 rows by 2 `half` columns; in the
// gated modes one CTA loads `half` rows of Wg and the other of Wu, so that the
// same thread finds G and U of a feature in its tensor-memory lane.
//
//   warps 0, 1, 3  producers, a step each in turn: 64 columns of K, the A tile
//                  (128 rows a CTA) and the B tile (`half` rows) by TMA (128-byte
//                  swizzle) into a stage of the ring
//   warp 2         MMAs (M = 256, N = 2 half, K = 16) of the pair's first CTA
//   warps 4 ..     epilogue, 16 (drained accumulators: 8) warps: 32 rows and a share of the
//                  columns each, straight from tensor memory to global memory
//
// A step is 512 SM cycles of MMAs at 256 columns (fp32: six times that). Waiting for a
// stage, its loads and moving on take a producer about 750 cycles, so one warp
// for A and one for B were the bound (8192 tokens of 1024 features into 4096,
// bf16: 95 us, the MMAs 62). Stages of 128 columns were too few to cover the
// loads' latency (89 us).
//
// Persistent: one CTA per SM; two accumulator buffers of 256 columns let a
// tile's epilogue overlap the next tile's MMAs. The epilogue waits for its loads
// and stores more than it computes, hence the many warps. Two plain products may
// share a launch, and those tiles that would fill the last round only in part have
// their K split.
//
// What bounds it: the MMAs, at the power limit's clocks in long runs; 1024 features
// into 4096, bf16, 8192 tokens: forward 73 us (1.89 PFLOP/s) for the kernel in short
// runs, 85 in a long run of calls; the backward pass's first product with its epilogue,
// which reads dH and writes dG and dU, 94 us; its plain products, 275 GFLOP, 147 us
// (1.87 PFLOP/s, the tensor pipe busy 84% of the time). Few tokens: the weights' bytes and the latency of one tile (128
// tokens of 768 into 2048 9 us). fp32 forward, 1000 tokens of 768 into 2048: 34 us,
// 19.6 at six part products of bf16 each, the rest laying out the operands and, with
// one tile a pair, its start and epilogue.
//
// The accumulators leave tensor memory so that a thread has two runs of eight
// features, of two rows, and the four threads beside it the next ones: 64 (fp32:
// 128) contiguous bytes of a row, eight rows an instruction. A row a lane took 61
// cycles an instruction of 32 bytes a lane, in the way of the MMAs' reads of
// shared memory (backward pass, 8192 tokens of 1024 into 4096: 12900 cycles a tile
// of 8200 cycles of MMAs). To that end the weights' rows are loaded in another
// order: row 8 i + 2 q + e of 32 is feature 8 q + 2 i + e (i, q < 4, e < 2), a box
// of a five-dimensional tensor. In plain products (bf16) the four threads exchange
// their columns.
//
// Operands stored with K along rows (weights for dX; dG, dU and X for the
// weights' gradients) are read in place: TMA boxes of 64 x 64 and descriptors
// with M or N contiguous.
//
// fp32 operands come as three bf16 parts whose sum they are (8 bits of the
// significand each, rounded to nearest), and a product is the six of nine part
// products that are not below 2^-24 of it (bf16 products may have an A of two parts). The tensor cores'
// fp32 accumulation drops bits with every addition, so the small products of a
// step come first and the accumulators are added to registers after every step.
//
// Every wait is bounded by the global timer; a timeout is recorded, stops every
// role, lets the issued copies and MMAs finish, frees the tensor memory and
// returns.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdlib>

#include "act.cuh"
#include "bsr_internal.h"
#include "eight.cuh"
#include "elem.cuh"
#include "gated_mma.h"
#include "launch.cuh"
#include "parts.cuh"
#include "ptx.cuh"
#include "status.cuh"
#include "tcgen05.cuh"

namespace bsr {

namespace {

constexpr int KC = 64;                        // columns of K per chunk
constexpr uint32_t kABytes = 128 * 128;       // a CTA's A tile
constexpr int kEpiWarp0 = 4, kMmaWarp = 2;
constexpr int epi_warps(bool drained) { return drained ? 8 : 16; }
constexpr int threads_of(bool drained) { return 32 * (kEpiWarp0 + epi_warps(drained)); }
// Drained accumulators go into registers every so many steps: fp32's after each, those
// of a gated mode with bf16 sums of more than kMostSteps after 512 columns.
constexpr int drain_steps(bool f32) { return f32 ? 1 : 8; }
constexpr int kStages = 8;
constexpr uint32_t kBiasBytes = 8 * 128 * 4;  // a warp's share of bg and bu: 64 (fp32), 32 features
constexpr uint32_t kMaxSmem = 227 * 1024 - 1024;
constexpr uint32_t kAccCols = 256;
constexpr int kProducers = 3;
// Steps of a bf16 sum in the accumulators at most: the accumulators lose about 7e-9 of a sum of
// one sign with each column, always towards zero, over so many (16384 columns) 2^-13, a
// sixteenth of the most that a bf16 result is rounded by. Longer sums of plain products
// are split, their parts added in fp32; those of the gated modes are drained.
constexpr int kMostSteps = 256;
constexpr uint64_t kDrainNs = 200000000ull;   // bound for copies and MMAs already issued

__device__ int g_status;

// One product.
struct Job {
    CUtensorMap a, b0, b1;
    int64_t M, N;             // rows; columns (gated modes: features)
    unsigned tiles_n;         // tiles along N
    unsigned whole;           // tiles that are one unit (the first ones)
    unsigned split_units;     // units of the others
    int splits;               // of each of them
    int steps, seam;          // steps of a tile; the step from which b1 is read
    uint32_t idesc;
    int a_side;
    int groups;               // gated modes: groups of 32 rows of a part of B
    void *out0, *out1;        // gated forward: H in out0
    int64_t row_seam, out_rows;
    int align;                // bytes (at most 16) that output (and dH) rows are aligned to
};

struct Args {
    Job job[2];
    unsigned units;           // the jobs' whole tiles, then their split ones
    int half, ns;
    uint32_t stage_bytes;
    int a_tiles, b_tiles;     // in a stage
    const float *bg, *bu;
    int act;
    const void *dH;
    uint16_t *D;
    int d_planes;
    int64_t Fp;
    float *sums;
    float *parts;
    uint64_t wait_ns;
    int stall_step;           // test hook: this step of each tile is never loaded (-1: none)
};

struct Unit {
    int64_t m0, n0;   // first row, first column (gated modes: feature)
    int i0, i1;       // steps
    int part;         // index of the unit's part, -1 for a whole tile
    int job;
};

template <int MODE>
__device__ __forceinline__ Unit unit_at(const Args &a, unsigned v) {
    Unit u;
    u.part = -1;
    u.job = 0;
    unsigned tile = v;
    if (MODE == GM_PRODUCT) {
        const unsigned w0 = a.job[0].whole, wholes = w0 + a.job[1].whole;
        if (v < wholes) {
            u.job = v >= w0;
            if (u.job) tile -= w0;
        } else {
            u.part = (int)(v - wholes);
            u.job = (unsigned)u.part >= a.job[0].split_units;
            tile = (unsigned)u.part - (u.job ? a.job[0].split_units : 0);
        }
    }
    const Job &j = a.job[u.job];
    u.i0 = 0;
    u.i1 = j.steps;
    if (MODE == GM_PRODUCT && u.part >= 0) {
        const unsigned s = (unsigned)j.splits, k = tile % s;
        tile = j.whole + tile / s;
        u.i0 = (int)((int64_t)j.steps * k / s);
        u.i1 = (int)((int64_t)j.steps * (k + 1) / s);
    }
    const unsigned tm = tile / j.tiles_n, tn = tile - tm * j.tiles_n;
    u.m0 = (int64_t)tm * 256;
    u.n0 = (int64_t)tn * (MODE == GM_PRODUCT ? 2 * a.half : a.half);
    return u;
}

// The unit of a pair in a round of them: all rounds but the first are taken
// backwards, so that who had a short unit there is the first to have one more (the
// units come longest first).
__host__ __device__ __forceinline__ unsigned unit_in(unsigned round, unsigned pair, unsigned pairs) {
    return round * pairs + (round ? pairs - 1 - pair : pair);
}

// The products of a step, the smallest first: parts of A and B. fp32: (2,0) (1,1)
// (0,2) (1,0) (0,1) (0,0); two parts of A: (1,0) (0,0).
template <bool F32>
__device__ __forceinline__ int a_tile_of(int i, int n) {
    return F32 ? (0x001012 >> (4 * i)) & 3 : n - 1 - i;
}
template <bool F32>
__device__ __forceinline__ int b_tile_of(int i) {
    return F32 ? (0x010210 >> (4 * i)) & 3 : 0;
}

// dH of row `row` from feature c on; 0 past the matrix.
template <typename T>
__device__ __forceinline__ void fetch(const Args &a, const Job &job, int64_t row, int64_t c, Eight<T> &r) {
    load8(static_cast<const T *>(a.dH) + row * job.N + c, row < job.M ? job.N - c : 0, job.align, r);
}

// Sums of eight values, in pairs, over the lanes with the same lane % 4: lane l
// gets that of value l / 4.
__device__ __forceinline__ float row_sums(const F2 (&p)[4]) {
    const int lane = threadIdx.x & 31;
    float v[8], b[4], c[2];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float2 u = unpack2(p[j]);
        v[2 * j] = u.x, v[2 * j + 1] = u.y;
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {   // lanes with bit 4 keep the upper four
        const float mine = lane & 16 ? v[j + 4] : v[j], other = lane & 16 ? v[j] : v[j + 4];
        b[j] = mine + __shfl_xor_sync(0xffffffffu, other, 16);
    }
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const float mine = lane & 8 ? b[j + 2] : b[j], other = lane & 8 ? b[j] : b[j + 2];
        c[j] = mine + __shfl_xor_sync(0xffffffffu, other, 8);
    }
    const float mine = lane & 4 ? c[1] : c[0], other = lane & 4 ? c[0] : c[1];
    return mine + __shfl_xor_sync(0xffffffffu, other, 4);
}

// Puts out G and U (v and w: eight features from c on, in pairs, of rows `row` and
// row + 8) of a gated mode: H, or dG and dU, whose sums over the rows are added to
// sg and su.
template <int MODE, typename T>
__device__ __forceinline__ void put_gated(const Args &a, const Job &job, int64_t row, int64_t c, F2 (&v)[2][4], F2 (&w)[2][4],
                                          const float *bias_g, const float *bias_u, const Eight<T> (&dh)[2], F2 (&sg)[4],
                                          F2 (&su)[4]) {
    constexpr bool FAST = sizeof(T) == 2;
    if (a.bg || a.bu) {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const float4 g = *reinterpret_cast<const float4 *>(bias_g + 2 * j), u = *reinterpret_cast<const float4 *>(bias_u + 2 * j);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                v[h][j] = add2(v[h][j], pack2(g.x, g.y)), v[h][j + 1] = add2(v[h][j + 1], pack2(g.z, g.w));
                w[h][j] = add2(w[h][j], pack2(u.x, u.y)), w[h][j + 1] = add2(w[h][j + 1], pack2(u.z, u.w));
            }
        }
    }
    if constexpr (MODE == GM_FORWARD) {
        with_act(a.act, [&](auto tag) {
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int j = 0; j < 4; j++) v[h][j] = mul2(activate<decltype(tag)::value, FAST>(v[h][j]), w[h][j]);
        });
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if (row + 8 * h >= job.M) continue;
            store8(static_cast<T *>(job.out0) + (row + 8 * h) * job.N + c, job.N - c, job.align, eight_of<T>(v[h]));
        }
    } else {
        with_act(a.act, [&](auto tag) {
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const F2 d = two_of(dh[h], j);
                    F2 slope;
                    const F2 act = activate_slope<decltype(tag)::value, FAST>(v[h][j], slope);
                    v[h][j] = mul2(mul2(d, w[h][j]), slope);
                    w[h][j] = mul2(d, act);
                }
        });
        // (no rows past the matrix: X and dH are 0 there, but a feature's weights and
        // biases need not be finite)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if (row + 8 * h >= job.M) continue;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                sg[j] = add2(sg[j], v[h][j]);
                su[j] = add2(su[j], w[h][j]);
            }
        }
        if (c >= a.Fp) return;
        // 0 past the features, whatever a row of X with an infinity makes of weights of 0
        if (c + 8 > job.N) {
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float2 x = unpack2(v[h][j]), y = unpack2(w[h][j]);
                    const bool one = c + 2 * j < job.N, two = c + 2 * j + 1 < job.N;
                    v[h][j] = pack2(one ? x.x : 0.f, two ? x.y : 0.f);
                    w[h][j] = pack2(one ? y.x : 0.f, two ? y.y : 0.f);
                }
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if (row + 8 * h >= job.M) continue;
            uint16_t *at = a.D + (row + 8 * h) * 2 * a.Fp + c;
            if constexpr (FAST) {
                if (a.d_planes == 1) {
                    store8(at, 8, 16, eight_of<uint16_t>(v[h]));
                    store8(at + a.Fp, 8, 16, eight_of<uint16_t>(w[h]));
                } else {
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        uint32_t p[4][2];
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const float2 x = unpack2(k ? w[h][j] : v[h][j]);
                            parts_of(x.x, x.y, p[j]);
                        }
#pragma unroll
                        for (int i = 0; i < 2; i++)
                            *reinterpret_cast<uint4 *>(at + k * a.Fp + i * 2 * a.Fp * job.M) = make_uint4(p[0][i], p[1][i], p[2][i], p[3][i]);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    uint32_t p[4][3];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float2 x = unpack2(k ? w[h][j] : v[h][j]);
                        parts_of(x.x, x.y, p[j]);
                    }
#pragma unroll
                    for (int i = 0; i < 3; i++)
                        *reinterpret_cast<uint4 *>(at + k * a.Fp + i * 2 * a.Fp * job.M) = make_uint4(p[0][i], p[1][i], p[2][i], p[3][i]);
                }
            }
        }
    }
}

// Puts out 16 rows x 32 columns of a plain product, from row `row` (of this thread:
// row and row + 8) and column c on; x as tc5::ld_16x32 leaves it.
template <typename T>
__device__ __forceinline__ void put_product(const Args &a, const Job &job, const Unit &u, int64_t row, int64_t c, const float (&x)[16]) {
    const int q = threadIdx.x & 3;
    if (u.part >= 0) {   // [256][2 half] of this unit
        float *at = a.parts + ((int64_t)u.part * 256 + (row - u.m0)) * 2 * a.half + (c - u.n0) + 2 * q;
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int i = 0; i < 4; i++)
                *reinterpret_cast<float2 *>(at + 8 * h * 2 * a.half + 8 * i) = make_float2(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]);
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        uint32_t w[4];   // bf16: two columns each
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = pack_bf16(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]);
            turn_words(w);
        }
        const int64_t m = row + 8 * h;
        const bool second = m >= job.row_seam;
        const int64_t r = second ? m - job.row_seam : m;
        if (m >= job.M || r >= job.out_rows) continue;
        T *out = static_cast<T *>(second ? job.out1 : job.out0) + r * job.N;
        if constexpr (sizeof(T) == 2) {
            Eight<T> e;
#pragma unroll
            for (int i = 0; i < 4; i++) e.w[i] = w[i];
            store8(out + c + 8 * q, job.N - (c + 8 * q), job.align, e);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int64_t at = c + 8 * i + 2 * q;
                if (at + 2 <= job.N && job.align >= 8) {
                    *reinterpret_cast<float2 *>(out + at) = make_float2(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]);
                } else {
                    if (at < job.N) out[at] = x[4 * i + 2 * h];
                    if (at + 1 < job.N) out[at + 1] = x[4 * i + 2 * h + 1];
                }
            }
        }
    }
}

template <int MODE, typename T, bool DRAIN>
__global__ void __launch_bounds__(threads_of(DRAIN), 1) k_gated_mma(const __grid_constant__ Args a) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int kEpiWarps = epi_warps(DRAIN), kDrain = drain_steps(F32);
    extern __shared__ unsigned char smem_raw[];
    unsigned char *base = ptx::align_smem(smem_raw);
    const int ns = a.ns;
    const uint32_t stage_bytes = a.stage_bytes, b_at = a.a_tiles * kABytes, b_bytes = (uint32_t)a.half * 128;
    float *bias_s = reinterpret_cast<float *>(base + (size_t)ns * stage_bytes);
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], done;
    __shared__ int stop, loads[kProducers][2];   // loads[producer][CTA of the pair]: steps loaded
    __shared__ int freed, handed;                // commits issued to `empty` and to `acc_full`
    __shared__ uint32_t tmem_s;

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
    tc5::fence_before();
    __syncthreads();
    ptx::cluster_barrier();   // the other CTA's barriers exist
    tc5::fence_after();
    ptx::pdl_launch_dependents();   // (after the allocation: ptx.cuh)
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
            if (v >= a.units) return false;
            un = unit_at<MODE>(a, v);
            i = un.i0 + over;
        }
        return true;
    };
    auto load_step = [&]() {
        if (i == a.stall_step) {   // never loaded: its consumer times out
            stalled |= 1u << s;
        } else if (elected) {
            const Job &job = a.job[un.job];
            const uint32_t dst = smem0 + s * stage_bytes, bar = first0 + 8 * s;
            if (rank == 0) ptx::mbar_arrive_expect_tx_at(bar0 + 8 * s, 2 * (a.a_tiles * kABytes + a.b_tiles * b_bytes));
            const int m = (int)(un.m0 + rank * 128), n = (int)(un.n0 + (MODE == GM_PRODUCT ? rank * a.half : 0));
            const bool second = MODE == GM_PRODUCT && job.seam && i >= job.seam;
            const int k = i * KC, kb = second ? (i - job.seam) * KC : k;
            const CUtensorMap *map = (MODE == GM_PRODUCT ? second : rank) ? &job.b1 : &job.b0;
            for (int t = 0; t < a.a_tiles; t++) {
                const uint32_t to = dst + t * kABytes;
                if (MODE == GM_PRODUCT && job.a_side) {
                    ptx::tma_load_3d_pair_at(to, &job.a, m, k, t, bar);
                    ptx::tma_load_3d_pair_at(to + 8192, &job.a, m + 64, k, t, bar);
                } else {
                    ptx::tma_load_3d_pair_at(to, &job.a, k, m, t, bar);
                }
            }
            for (int t = 0; t < a.b_tiles; t++) {
                const uint32_t to = dst + b_at + t * b_bytes;
                if (MODE == GM_PRODUCT) {   // (b_side: every plain product's)
                    for (int j = 0; j < a.half; j += 64) ptx::tma_load_3d_pair_at(to + 128 * j, map, n + j, kb, t, bar);
                } else {   // (a part's rows are whole groups of 32, and the parts lie behind one another)
                    ptx::tma_load_5d_pair_at(to, map, kb, 0, 0, 0, n / 32 + t * job.groups, bar);
                }
            }
        }
        issued++;
        for (s += np; s >= ns; s -= ns) phase ^= 1;
        i += np;
        return seek();
    };
    bool more = false;
    if (producer) {
        if (elected) {
            for (int j = 0; j < (MODE == GM_PRODUCT ? 2 : 1); j++) {
                ptx::prefetch_tensormap(&a.job[j].a);
                ptx::prefetch_tensormap(&a.job[j].b0);
                ptx::prefetch_tensormap(&a.job[j].b1);
            }
        }
        un = unit_at<MODE>(a, v);
        i = un.i0 + prod;
        more = seek();
        ptx::pdl_wait();   // every operand may be an earlier kernel's output
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
            int ab = 0, n_freed = 0, n_handed = 0;
            uint32_t fphase = 0, aphase = 1;
            bool ok = true;
            s = 0;
            ptx::pdl_wait();   // the waits below are bounded from here on
            for (; ok && v < a.units; v = unit_in(++round, pair, pairs)) {
                un = unit_at<MODE>(a, v);
                const Job &job = a.job[un.job];
                const bool a_side = MODE == GM_PRODUCT && job.a_side, b_side = MODE == GM_PRODUCT;
                const uint64_t ad0 = a_side ? tc5::desc_sw128_mn(smem0, 8192) : tc5::desc_sw128(smem0);
                const uint64_t bd0 = b_side ? tc5::desc_sw128_mn(smem0 + b_at, 8192) : tc5::desc_sw128(smem0 + b_at);
                // 16 of K: two groups of eight 128-byte rows, or 32 bytes along the rows
                const uint32_t a_step = a_side ? 128 : 2, b_step = b_side ? 128 : 2, idesc = job.idesc;
                for (i = un.i0; ok && i < un.i1; i++) {
                    const uint32_t d = tmem + (uint32_t)ab * kAccCols;
                    const bool fresh = DRAIN ? (i - un.i0) % kDrain == 0 : i == un.i0;
                    if (fresh) {   // into a fresh accumulator buffer
                        ok = __all_sync(0xffffffffu, wait_or_abort(&acc_empty[ab], aphase, a.wait_ns, &stop));
                        if (!ok) break;
                    }
                    ok = __all_sync(0xffffffffu, wait_or_abort(&full[s], fphase, a.wait_ns, &stop));
                    if (!ok) break;
                    tc5::fence_after();
                    if (elected) {
                        const uint64_t at = (uint64_t)((s * stage_bytes) >> 4);
                        const int n = F32 ? 6 : a.a_tiles;
#pragma unroll
                        for (int t = 0; t < (F32 ? 6 : 2); t++) {
                            if (t >= n) break;
                            const uint64_t ad = ad0 + at + a_tile_of<F32>(t, n) * (kABytes >> 4);
                            const uint64_t bd = bd0 + at + b_tile_of<F32>(t) * (b_bytes >> 4);
#pragma unroll
                            for (int j = 0; j < KC / 16; j++)
                                tc5::mma_ss_pair(d, ad + j * a_step, bd + j * b_step, idesc,
                                                 !fresh | (t > 0) | (j > 0));
                        }
                        tc5::commit_pair(&empty[s]);
                    }
                    __syncwarp();
                    n_freed++;
                    if (++s == ns) {
                        s = 0;
                        fphase ^= 1;
                    }
                    if (i + 1 == un.i1 || (DRAIN && (i + 1 - un.i0) % kDrain == 0)) {
                        if (elected) tc5::commit_pair(&acc_full[ab]);
                        __syncwarp();
                        n_handed++;
                        ab ^= 1;
                        if (ab == 0) aphase ^= 1;
                    }
                }
                if (!ok) halt();
            }
            // every MMA issued has completed before the tensor memory is freed
            if (elected) {
                tc5::commit_pair(&done);
                freed = n_freed;
                handed = n_handed;
                ptx::store_cluster(ptx::map_to_cta(&freed, 1), (uint32_t)n_freed);
                ptx::store_cluster(ptx::map_to_cta(&handed, 1), (uint32_t)n_handed);
            }
            __syncwarp();
            ptx::mbar_wait_bounded(&done, 0, kDrainNs);
        }
    } else if (warp >= kEpiWarp0) {
        constexpr int kShares = kEpiWarps / 4, kMost = 8 / kShares;   // warps to 32 rows; most pieces of one
        const int q = warp & 3, hc = (warp - kEpiWarp0) >> 2;          // tensor-memory lanes 32 q .., share hc
        float *bs = bias_s + (warp - kEpiWarp0) * (kMost * 32);
        // this warp's pieces: gated modes, of 16 rows x 32 features (G and U), the
        // rows' halves of a group of features behind each other; products, of 32 rows
        // x 32 columns
        const int all = a.half / 16, each = (all + kShares - 1) / kShares, first = hc * each,
                  pieces = max(0, min(each, all - first));
        const bool both = each > 1;   // a warp has both halves of its groups
        ptx::pdl_wait();   // the outputs and dH may be an earlier kernel's
        int ab = 0;
        uint32_t fphase = 0;
        bool ok = true;
        // a piece's row and feature of this thread, gated modes
        auto row_of = [&](const Unit &u, int p) { return u.m0 + rank * 128 + 32 * q + 16 * ((first + p) & 1) + (lane >> 2); };
        auto col_of = [&](const Unit &u, int p) { return u.n0 + 32 * ((first + p) >> 1) + 8 * (lane & 3); };
        // waits for the next accumulator buffer; its columns of this warp's lanes
        auto wait_acc = [&](const Unit &u) {
            const uint64_t limit = a.wait_ns * (uint64_t)(u.i1 - u.i0 + 2);
            ok = __all_sync(0xffffffffu, wait_or_abort(&acc_full[ab], fphase, limit, &stop));
            if (!ok) halt();
            tc5::fence_after();
            return tmem + (uint32_t)ab * kAccCols + ((uint32_t)(32 * q) << 16);
        };
        // hands the buffer back, its last columns being in registers
        auto hand_back = [&]() {
            tc5::fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_remote(ptx::map_to_cta(&acc_empty[ab], 0));
            ab ^= 1;
            if (ab == 0) fphase ^= 1;
        };
        // a piece of the accumulators at tm
        auto load_piece = [&](uint32_t tm, int p, uint32_t (&r0)[16], uint32_t (&r1)[16]) {
            __syncwarp();   // (the piece before may have parted the lanes by their rows)
            if constexpr (MODE == GM_PRODUCT) {
                tc5::ld_16x32(tm + 32 * (first + p), r0);
                tc5::ld_16x32(tm + (16u << 16) + 32 * (first + p), r1);
            } else {
                const uint32_t at = tm + ((uint32_t)(16 * ((first + p) & 1)) << 16) + 32 * ((first + p) >> 1);
                tc5::ld_16x32(at, r0);
                tc5::ld_16x32(at + a.half, r1);
            }
            tc5::ld_wait();
#pragma unroll
            for (int j = 0; j < 16; j++) {   // no use of a loaded register moves above the wait
                asm volatile("" : "+r"(r0[j]));
                asm volatile("" : "+r"(r1[j]));
            }
        };
        // sums of dG and dU over the rows of the pieces of one group of features
        F2 sg[4], su[4];
        auto put = [&](const Job &job, int p, const float (&x)[16], const float (&y)[16], const Eight<T> (&dh)[2]) {
            if constexpr (MODE == GM_PRODUCT) {
                const int64_t row = un.m0 + rank * 128 + 32 * q + (lane >> 2), c = un.n0 + 32 * (first + p);
                put_product<T>(a, job, un, row, c, x);
                put_product<T>(a, job, un, row + 16, c, y);
            } else {
                F2 g[2][4], u[2][4];
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        g[h][j] = pack2(x[4 * j + 2 * h], x[4 * j + 2 * h + 1]);
                        u[h][j] = pack2(y[4 * j + 2 * h], y[4 * j + 2 * h + 1]);
                    }
                const int64_t row = row_of(un, p), c = col_of(un, p);
                const float *b = bs + 32 * (((first + p) >> 1) - (first >> 1)) + 8 * (lane & 3);
                if (MODE == GM_BACKWARD && (!both || !(p & 1))) {
#pragma unroll
                    for (int j = 0; j < 4; j++) sg[j] = su[j] = all2(0.f);
                }
                put_gated<MODE, T>(a, job, row, c, g, u, b, b + 16 * kMost, dh, sg, su);
                // the rows' sums: feature c + lane / 4 of this lane's eight
                if (MODE == GM_BACKWARD && a.sums && (!both || (p & 1)) && c < a.Fp) {
                    const float g1 = row_sums(sg), u1 = row_sums(su);
                    const int64_t block = (un.m0 + rank * 128 + 32 * q) / 32;
                    if (32 * block < job.M) {
                        float *at = a.sums + ((both ? block : 2 * block + ((first + p) & 1)) * 2 * a.Fp) + c + (lane >> 2);
                        at[0] = g1;
                        at[a.Fp] = u1;
                    }
                }
            }
        };
        // bf16: dH of the unit to come (it is read from DRAM, 3000 cycles when the
        // loads of the operands are in its way)
        Eight<T> ahead[DRAIN ? 1 : kMost][2];
        if constexpr (MODE == GM_BACKWARD && !DRAIN) {
            if (v < a.units) {
                un = unit_at<MODE>(a, v);
#pragma unroll
                for (int p = 0; p < kMost; p++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
                        if (p < pieces) fetch(a, a.job[0], row_of(un, p) + 8 * h, col_of(un, p), ahead[p][h]);
            }
        }
        for (; ok && v < a.units; v = unit_in(++round, pair, pairs)) {
            un = unit_at<MODE>(a, v);
            const Job &job = a.job[un.job];
            if (MODE != GM_PRODUCT && (a.bg || a.bu)) {
                __syncwarp();   // (the last unit's biases have been read)
                for (int j = lane; j < 16 * kMost; j += 32) {
                    const int64_t f = un.n0 + 32 * (first >> 1) + j;
                    bs[j] = a.bg && f < job.N ? a.bg[f] : 0.f;
                    bs[16 * kMost + j] = a.bu && f < job.N ? a.bu[f] : 0.f;
                }
                __syncwarp();
            }
            if constexpr (!DRAIN) {
                const uint32_t tm = wait_acc(un);
                if (!ok) break;
                if (pieces == 0) hand_back();
                const unsigned vn = unit_in(round + 1, pair, pairs);
                const Unit next = MODE == GM_BACKWARD && vn < a.units ? unit_at<MODE>(a, vn) : un;
#pragma unroll
                for (int p = 0; p < kMost; p++) {
                    if (p >= pieces) break;
                    uint32_t r0[16], r1[16];
                    load_piece(tm, p, r0, r1);
                    float x[16], y[16];
#pragma unroll
                    for (int j = 0; j < 16; j++) x[j] = __uint_as_float(r0[j]), y[j] = __uint_as_float(r1[j]);
                    if (p + 1 == pieces) hand_back();
                    Eight<T> dh[2];
                    if constexpr (MODE == GM_BACKWARD) {   // this unit's, on its way since the last one; the next unit's
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            dh[h] = ahead[p][h];
                            fetch(a, job, row_of(next, p) + 8 * h, col_of(next, p), ahead[p][h]);
                        }
                    }
                    put(job, p, x, y, dh);
                }
            } else {
                float g[kMost][16], w[kMost][16];   // the sums of what was drained so far
                if constexpr (MODE == GM_BACKWARD) {   // dH comes from DRAM: into L2 meanwhile
                    for (int p = 0; p < pieces; p++)
                        for (int h = 0; h < 2; h++) {
                            const int64_t row = row_of(un, p) + 8 * h, c = col_of(un, p);
                            if (row < job.M && c < job.N) ptx::prefetch_l2(static_cast<const T *>(a.dH) + row * job.N + c);
                        }
                }
#pragma unroll
                for (int p = 0; p < kMost; p++)
#pragma unroll
                    for (int j = 0; j < 16; j++) g[p][j] = w[p][j] = 0.f;
                for (int b = un.i0; b < un.i1; b += kDrain) {
                    const uint32_t tm = wait_acc(un);
                    if (!ok) break;
#pragma unroll
                    for (int p = 0; p < kMost; p++) {
                        if (p >= pieces) break;
                        uint32_t r0[16], r1[16];
                        load_piece(tm, p, r0, r1);
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            g[p][j] += __uint_as_float(r0[j]);
                            w[p][j] += __uint_as_float(r1[j]);
                        }
                    }
                    hand_back();
                }
                if (!ok) break;
                // one copy of the code for all pieces (unrolled, it came from beyond the
                // instruction caches), the sums handed on from piece to piece
#pragma unroll 1
                for (int p = 0; p < pieces; p++) {
                    Eight<T> dh[2];
                    if constexpr (MODE == GM_BACKWARD) {
#pragma unroll
                        for (int h = 0; h < 2; h++) fetch(a, job, row_of(un, p) + 8 * h, col_of(un, p), dh[h]);
                    }
                    put(job, p, g[0], w[0], dh);
#pragma unroll
                    for (int k = 0; k + 1 < kMost; k++)
#pragma unroll
                        for (int j = 0; j < 16; j++) g[k][j] = g[k + 1][j], w[k][j] = w[k + 1][j];
                }
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

// What is left after the products, in one launch: the CTAs below `joins` add up
// the parts of the split tiles, in their order, four columns a thread and half / 2
// CTAs to a tile; those above sum the 2 Fp columns of dG's and dU's sums (n rows of
// them), 32 columns a CTA, 32 x 8 threads, each every eighth row, then the eight.
template <typename T>
__global__ void __launch_bounds__(256) k_gated_finish(const __grid_constant__ Args a, unsigned joins, int64_t n, int64_t F, float *dbg,
                                                      float *dbu) {
    __shared__ float part[8][33];
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    if (blockIdx.x < joins) {
        const int fours = a.half / 2, width = 2 * a.half;
        const unsigned tile = blockIdx.x / (unsigned)fours;
        const Job &j0 = a.job[0], &j1 = a.job[1];
        const unsigned n0 = j0.split_units / (unsigned)j0.splits;
        const unsigned first = tile < n0 ? tile * (unsigned)j0.splits : j0.split_units + (tile - n0) * (unsigned)j1.splits;
        const Unit un = unit_at<GM_PRODUCT>(a, j0.whole + j1.whole + first);
        const Job &job = a.job[un.job];
        const int e = (int)(blockIdx.x % (unsigned)fours) * 256 + threadIdx.x, r = e / fours, x = (e - r * fours) * 4;
        const int64_t row = un.m0 + r, c = un.n0 + x;
        const bool second = row >= job.row_seam;
        const int64_t at = second ? row - job.row_seam : row;
        if (row >= job.M || c >= job.N || at >= job.out_rows) return;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < job.splits; k++) {
            const float4 p = *reinterpret_cast<const float4 *>(a.parts + ((int64_t)(un.part + k) * 256 + r) * width + x);
            t.x += p.x, t.y += p.y, t.z += p.z, t.w += p.w;
        }
        T *out = static_cast<T *>(second ? job.out1 : job.out0) + at * job.N + c;
        const float f[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (c + j < job.N) out[j] = from_f32<T>(f[j]);
        return;
    }
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = (int64_t)(blockIdx.x - joins) * 32 + lane;
    float s = 0.f;
#pragma unroll 16
    for (int64_t k = w; k < n; k += 8) s += a.sums[k * 2 * a.Fp + c];
    part[w][lane] = s;
    __syncthreads();
    if (w) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; k++) s += part[k][lane];
    const int64_t f = c < a.Fp ? c : c - a.Fp;
    float *out = c < a.Fp ? dbg : dbu;
    if (out && f < F) out[f] = s;
}

// `side`: boxes of 64 columns x 64 rows; else of 64 columns x `rows` rows.
cudaError_t encode(const Planes &m, bool side, int rows, CUtensorMap *map) {
    auto enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows, (cuuint64_t)m.planes};
    const cuuint64_t strides[2] = {(cuuint64_t)m.ld * 2, (cuuint64_t)m.ld * 2 * (cuuint64_t)m.rows};
    const cuuint32_t box[3] = {64, (cuuint32_t)(side ? 64 : rows), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t *>(m.p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

// The weights of a gated mode: rows in groups of 32, a group's in the order that
// the epilogue wants (row 8 i + 2 q + e of a box: 8 q + 2 i + e of the group).
cudaError_t encode_weights(const Planes &m, int rows, CUtensorMap *map) {
    auto enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t ld = (cuuint64_t)m.ld * 2;
    const cuuint64_t dims[5] = {(cuuint64_t)m.cols, 2, 4, 4, (cuuint64_t)(m.rows / 32 * m.planes)};
    const cuuint64_t strides[4] = {ld, 8 * ld, 2 * ld, 32 * ld};
    const cuuint32_t box[5] = {64, 2, 4, 4, (cuuint32_t)(rows / 32)};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<uint16_t *>(m.p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

int pairs_of_sms() {
    int dev = 0, n = 152;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        cudaGetLastError();
    return std::max(1, n / 2);
}

// One job's arguments.
template <int MODE, typename T>
cudaError_t job_of(const GatedMma &g, const GatedShape &sh, int half, Job &j) {
    j.M = g.M, j.N = g.N;
    j.tiles_n = (unsigned)sh.tiles_n;
    j.whole = (unsigned)sh.whole;
    j.splits = sh.splits;
    j.split_units = (unsigned)((sh.tiles - sh.whole) * sh.splits);
    j.steps = sh.steps;
    j.seam = (int)(g.b_seam / KC);
    j.idesc = tc5::idesc(false, 256, 2 * half) | (g.a_side ? tc5::kIdescAmn : 0) | (MODE == GM_PRODUCT ? tc5::kIdescBmn : 0);
    j.a_side = g.a_side;
    j.out0 = MODE == GM_FORWARD ? g.H : g.out0;
    j.out1 = g.out1;
    j.row_seam = g.row_seam, j.out_rows = g.out_rows;
    const uintptr_t addresses = reinterpret_cast<uintptr_t>(j.out0) | reinterpret_cast<uintptr_t>(j.out1) |
                                reinterpret_cast<uintptr_t>(g.dH) | (uintptr_t)(g.N * sizeof(T)) | 16;
    j.align = (int)(addresses & (~addresses + 1));
    cudaError_t e = encode(g.a, g.a_side, 128, &j.a);
    j.groups = (int)(g.b0.rows / 32);
    for (int i = 0; i < 2 && e == cudaSuccess; i++) {
        const Planes &b = i && g.b1.p ? g.b1 : g.b0;
        CUtensorMap *map = i ? &j.b1 : &j.b0;
        e = MODE == GM_PRODUCT ? encode(b, true, 64, map) : encode_weights(b, half, map);
    }
    return e;
}

template <typename T>
cudaError_t finish(const Args &a, int64_t joins, const GatedBias &b, cudaStream_t s) {
    const int64_t sums = b.sums ? 2 * b.Fp / 32 : 0;
    if (joins + sums == 0) return cudaSuccess;
    if (joins + sums > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_kernel(k_gated_finish<T>, dim3((unsigned)(joins + sums)), dim3(256), 0, s, a, (unsigned)joins, b.rows, b.F, b.dbg, b.dbu);
}

template <int MODE, typename T, bool DRAIN>
cudaError_t launch(const GatedMma *g, const GatedPlan &p, const GatedBias &b, cudaStream_t s) {
    Args a = {};
    if (p.units > INT32_MAX) return cudaErrorInvalidConfiguration;
    a.units = (unsigned)p.units;
    a.half = p.half;
    a.a_tiles = g->a.planes;
    a.b_tiles = g->a.planes == 3 ? 3 : 1;
    a.stage_bytes = a.a_tiles * kABytes + a.b_tiles * (uint32_t)p.half * 128;
    a.ns = (int)std::min<uint32_t>(kStages, (kMaxSmem - 1024 - kBiasBytes) / a.stage_bytes);
    a.bg = g->bg, a.bu = g->bu;
    a.act = g->act;
    a.dH = g->dH;
    a.D = g->D, a.d_planes = g->d_planes;
    a.Fp = g->Fp;
    a.sums = g->sums;
    a.parts = p.parts;
    const char *limit = std::getenv("BSR_WAIT_LIMIT_NS"), *stall = std::getenv("BSR_TEST_STALL_CHUNK");
    a.wait_ns = limit ? std::strtoull(limit, nullptr, 10) : 1000000000ull;
    a.stall_step = stall ? std::atoi(stall) : -1;
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < p.jobs && e == cudaSuccess; i++) e = job_of<MODE, T>(g[p.order[i]], p.shape[i], p.half, a.job[i]);
    if (p.jobs == 1) {   // (no units of its own)
        a.job[1] = a.job[0];
        a.job[1].whole = a.job[1].split_units = 0;
    }
    static std::atomic<uint64_t> attr_set{0};
    if (e == cudaSuccess) e = allow_smem(k_gated_mma<MODE, T, DRAIN>, kMaxSmem, attr_set);
    if (e != cudaSuccess) return e;
    const unsigned grid = 2 * (unsigned)std::min<int64_t>(p.units, pairs_of_sms());
    e = launch_clusters(k_gated_mma<MODE, T, DRAIN>, 2, dim3(grid), dim3(threads_of(DRAIN)),
                        a.ns * a.stage_bytes + kBiasBytes + 1024, s, a);
    if (MODE != GM_PRODUCT || e != cudaSuccess) return e;
    int64_t joins = 0;
    for (int i = 0; i < p.jobs; i++) joins += (p.shape[i].tiles - p.shape[i].whole) * (p.half / 2);
    a.sums = const_cast<float *>(b.sums);
    a.Fp = b.Fp;
    return finish<T>(a, joins, b, s);
}

// What a plan takes, in SM cycles: the pair that has most to do, as unit_in hands
// the units out. Gives up where that must be over `most`.
double cycles_of(const GatedPlan &p, int groups, int pairs, double most) {
    // four MMAs of 256 columns take 512; narrower tiles wait for their loads, 400 for each
    // pair of tiles of A and B. A unit's start and end: 1500; of fp32 its epilogue too,
    // whose registers the next unit's sums need
    const bool f32 = groups == 6;
    const int tiles = f32 ? 3 : groups;
    const double step = std::max(groups * 512.0 * p.half / 128, tiles * 400.0), unit = f32 ? 12000.0 * p.half / 128 : 1500;
    // the parts are written and read again, and a launch added
    const double join = p.part_bytes ? 5000 + (double)p.part_bytes * 2 / 4000 : 0;
    int64_t count[4] = {};
    double length[4] = {}, total = 0, longest = 0;
    for (int i = 0; i < p.jobs; i++) {
        const GatedShape &sh = p.shape[i];
        count[i] = sh.whole;
        length[i] = sh.steps * step + unit;
        count[2 + i] = (sh.tiles - sh.whole) * sh.splits;
        length[2 + i] = (sh.steps + sh.splits - 1) / sh.splits * step + unit;
    }
    for (int k = 0; k < 4; k++) {
        total += (double)count[k] * length[k];
        if (count[k]) longest = std::max(longest, length[k]);
    }
    const double least = std::max(total / pairs, longest) + join;
    if (least >= most) return least;
    // whole rounds of the first kind are the same for all
    double base = 0;
    int64_t taken = 0;
    if (count[0] > pairs) {
        const int64_t rounds = count[0] / pairs - 1;
        base = (double)rounds * length[0];
        taken = rounds * pairs;
    }
    constexpr int kMostPairs = 256;
    double load[kMostPairs] = {};
    pairs = std::min(pairs, kMostPairs);
    unsigned v = 0;
    for (int k = 0; k < 4; k++)
        for (int64_t n = k == 0 ? taken : 0; n < count[k]; n++, v++) {
            const unsigned round = v / pairs, at = v % pairs;
            load[round ? pairs - 1 - at : at] += length[k];
        }
    return base + *std::max_element(load, load + pairs) + join;
}

}  // namespace

GatedPlan plan_gated_mma(const GatedMma *g, int n, int64_t most_bytes) {
    const int64_t pairs = pairs_of_sms();
    const bool product = g->mode == GM_PRODUCT;
    const int groups = g->a.planes == 3 ? 6 : g->a.planes;   // of four MMAs to a step
    GatedPlan best = {};
    double best_t = 0;
    for (int half : {128, 64, 32}) {
        if (product && half < 64) break;   // (a box of 64 columns)
        GatedPlan p = {};
        p.jobs = n;
        p.half = half;
        for (int i = 0; i < n; i++) {
            GatedShape &sh = p.shape[i];
            sh.steps = (int)((g[i].K + KC - 1) / KC);
            sh.tiles_n = product ? (g[i].N + 2 * half - 1) / (2 * half) : (g[i].Fp + half - 1) / half;
            sh.tiles = (g[i].M + 255) / 256 * sh.tiles_n;
        }
        p.drained = groups == 6 || (!product && p.shape[0].steps > kMostSteps);
        // the first `whole` tiles of each job as one unit, the others split
        auto consider = [&](const int64_t (&whole)[2], const int (&splits)[2]) {
            GatedPlan q = p;
            q.units = 0;
            q.part_bytes = 0;
            // the job with the longer units first
            const int l0 = (p.shape[0].steps + splits[0] - 1) / splits[0], l1 = n > 1 ? (p.shape[1].steps + splits[1] - 1) / splits[1] : 0;
            q.order[0] = n > 1 && l1 > l0;
            q.order[1] = 1 - q.order[0];
            for (int i = 0; i < n; i++) {
                GatedShape &sh = q.shape[i];
                sh = p.shape[q.order[i]];
                sh.splits = splits[q.order[i]];
                sh.whole = sh.splits == 1 ? sh.tiles : whole[q.order[i]];
                const int64_t parts = (sh.tiles - sh.whole) * sh.splits;
                q.units += sh.whole + parts;
                q.part_bytes += parts * 256 * 2 * half * 4;
            }
            if (q.part_bytes > most_bytes) return;
            const double t = cycles_of(q, groups, (int)pairs, best_t ? best_t : 1e300);
            if (best_t == 0 || t < best_t) {
                best_t = t;
                best = q;
            }
        };
        // a sum's parts at least
        int least[2] = {1, 1};
        for (int i = 0; i < n && product && groups != 6; i++) least[i] = (p.shape[i].steps + kMostSteps - 1) / kMostSteps;
        consider({0, 0}, least);
        if (!product) continue;
        for (int s0 : {1, 2, 3, 4, 5, 6, 8, 12, 16})
            for (int s1 : {1, 2, 3, 4, 6, 8, 12, 16})
                if (s0 + s1 > 2 && s0 <= p.shape[0].steps && (n > 1 ? s1 <= p.shape[1].steps : s1 == 1))
                    consider({0, 0}, {std::max(s0, least[0]), std::max(s1, least[1])});
        if (least[0] + least[1] > 2) continue;
        // only those tiles of the shorter sums that would fill the last round in part
        const int last = n > 1 && p.shape[1].steps <= p.shape[0].steps;
        const int64_t rest = (p.shape[0].tiles + (n > 1 ? p.shape[1].tiles : 0)) % pairs;
        for (int s = 2; s <= 16 && s <= p.shape[last].steps && rest <= p.shape[last].tiles; s++) {
            int64_t whole[2] = {};
            int splits[2] = {1, 1};
            whole[last] = p.shape[last].tiles - rest;
            splits[last] = s;
            consider(whole, splits);
        }
    }
    return best;
}

cudaError_t launch_gated_mma(const GatedMma *g, const GatedPlan &p, cudaStream_t s, const GatedBias &b) {
    const bool f32 = g->dt == BSR_F32;
    switch (g->mode) {
        case GM_FORWARD:
            return f32         ? launch<GM_FORWARD, float, true>(g, p, b, s)
                   : p.drained ? launch<GM_FORWARD, uint16_t, true>(g, p, b, s)
                               : launch<GM_FORWARD, uint16_t, false>(g, p, b, s);
        case GM_BACKWARD:
            return f32         ? launch<GM_BACKWARD, float, true>(g, p, b, s)
                   : p.drained ? launch<GM_BACKWARD, uint16_t, true>(g, p, b, s)
                               : launch<GM_BACKWARD, uint16_t, false>(g, p, b, s);
        default: return f32 ? launch<GM_PRODUCT, float, true>(g, p, b, s) : launch<GM_PRODUCT, uint16_t, false>(g, p, b, s);
    }
}

cudaError_t launch_gated_bias(const GatedBias &b, cudaStream_t s) {
    Args a = {};
    a.sums = const_cast<float *>(b.sums);
    a.Fp = b.Fp;
    return finish<float>(a, 0, b, s);
}

cudaError_t gated_mma_status(int *code) {
    const int ok = DEV_OK;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(code, g_status, sizeof ok);
    if (e == cudaSuccess && *code != ok) e = cudaMemcpyToSymbol(g_status, &ok, sizeof ok);
    return e;
}

}  // namespace bsr
