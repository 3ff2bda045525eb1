// Values in 8-bit floating point with a power of two for each block of 128.
//
//   s = 2^ceil(log2(max |x| / most)) over a block (1 x 128 along the sum, or
//   128 x 128), most 448 (e4m3) or 57344 (e5m2);  q = x / s, rounded to nearest even
//
// A power of two, so that x / s is exact and each value is rounded once; a block's
// largest value lands in the upper half of the range, and with 4 (5) bits of
// exponent a finer scale would keep no more bits of the others. s = 1 for a block of zeros, at
// least 2^-126. Values that are not finite become NaN and have no part in s.
//
// One pass: a CTA holds 128 x 128 values in registers (bf16 in pairs, as they lie), takes
// the largest of each row's 128 (16 lanes) and of each column's (the lanes' eight rows, then the eight
// warps'), and writes them as they lie and transposed, through shared memory, so
// that both operands of a later product have the sum's axis contiguous. Infinities, which
// would be the largest, are made NaN first.
//
// x is read by plain loads, not by the read-only path: the kernel starts while the one
// before it, whose output x may be, still runs.
//
// What bounds it: DRAM. bf16, both ways: 16384 x 1024 10.3 us (68 MB, 97% of the copy rate,
// part of it from L2), 8192 x 4096 22.8 (88%); by rows 16384 x 1024 6.0; fp32 both ways
// 8192 x 4096 36.7 (82%). Rows that are not aligned are read value by value (8192 x 1023
// bf16 10.6, x 1024 6.5).
#include <algorithm>

#include "elem.cuh"
#include "fp8.h"
#include "launch.cuh"
#include "ptx.cuh"

namespace bsr {

namespace {

struct QArgs {
    const void *x;
    int64_t R, C, KB, RB;   // blocks of columns and of rows
    uint8_t *q, *qt;        // rows of 128 KB and of 128 RB bytes
    int64_t e_bytes, et_bytes;   // of a matrix's exponents
    float *s, *st;          // (NULL: not wanted)
    uint8_t *e, *et;        // exponents as bytes, in the tensor cores' order
    const int32_t *used;
    int align;              // bytes (at most 16) that rows of x are aligned to
};

// The exponent of a block's scale, from the bits of its largest size.
template <bool E5M2>
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    if (top == 0) return 0;
    // most is 1.75 2^8 or 1.75 2^15; 0x600000 is .75 in the significand
    const int e = (int)(top >> 23) - 127 - (E5M2 ? 15 : 8) + ((top & 0x7fffff) > 0x600000);
    return max(e, -126);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Where the exponent of block b of row r is (matrices of `runs` x 128 rows).
__device__ __forceinline__ int64_t exponent_at(int64_t r, int64_t b, int64_t runs) {
    return ((b >> 2) * runs + (r >> 7)) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4 + (b & 3);
}

// Two values in 8 bits each (the first one's low).
template <bool E5M2>
__device__ __forceinline__ uint32_t round2(float y0, float y1) {
    uint16_t r;
    if constexpr (E5M2) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y1), "f"(y0));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y1), "f"(y0));
    return r;
}
// Eight values of a row: bf16 in pairs, fp32 one by one. Sizes: of pairs or values,
// a maximum with a NaN is the other operand.
template <typename T>
struct Row;

template <>
struct Row<uint16_t> {
    static constexpr int words = 4, each = 2;
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint16_t *p, int n, int align) {
        if (n >= 8 && align == 16) {
            const uint4 u = *reinterpret_cast<const uint4 *>(p);
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else if (n >= 8 && align >= 4) {
#pragma unroll
            for (int j = 0; j < 4; j++) w[j] = reinterpret_cast<const uint32_t *>(p)[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
                w[j] = (2 * j < n ? (uint32_t)p[2 * j] : 0) | (2 * j + 1 < n ? (uint32_t)p[2 * j + 1] : 0) << 16;
        }
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ __forceinline__ uint32_t size(int j) const {
        uint32_t a;
        asm("abs.bf16x2 %0, %1;" : "=r"(a) : "r"(w[j]));
        return a;
    }
    __device__ __forceinline__ void no_infinities() {   // (they become NaN)
#pragma unroll
        for (int j = 0; j < words; j++) w[j] |= ((w[j] & 0x7fffu) == 0x7f80u ? 0x7fffu : 0) | ((w[j] & 0x7fff0000u) == 0x7f800000u ? 0x7fff0000u : 0);
    }
    // the bits, as fp32, of the larger value of a pair of sizes; a NaN is no size
    static __device__ __forceinline__ uint32_t top(uint32_t a) {
        const uint32_t t = larger(a, a >> 16 | a << 16) & 0xffffu;
        return t > 0x7f80u ? 0 : t << 16;
    }
    static __device__ __forceinline__ uint32_t low(uint32_t a) { return (a & 0xffffu) > 0x7f80u ? 0 : a << 16; }
    static __device__ __forceinline__ uint32_t high(uint32_t a) { return a >> 16 > 0x7f80u ? 0 : a & 0xffff0000u; }
    // 2^-e, and word j times it (exact, but for values that 8 bits do not have)
    static __device__ __forceinline__ uint32_t factor(int e0, int e1) { return (uint32_t)(127 - e0) << 7 | (uint32_t)(127 - e1) << 23; }
    __device__ __forceinline__ float2 scaled(int j, uint32_t f) const {
        uint32_t y;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(w[j]), "r"(f));
        return make_float2(__uint_as_float(y << 16), __uint_as_float(y & 0xffff0000u));
    }
};

template <>
struct Row<float> {
    static constexpr int words = 8, each = 1;
    float w[8];
    __device__ __forceinline__ void load(const float *p, int n, int align) {
        if (n >= 8 && align == 16) {
            const float4 u = *reinterpret_cast<const float4 *>(p), v = reinterpret_cast<const float4 *>(p)[1];
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w, w[4] = v.x, w[5] = v.y, w[6] = v.z, w[7] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) w[j] = j < n ? p[j] : 0.f;
        }
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    __device__ __forceinline__ uint32_t size(int j) const { return __float_as_uint(w[j]) & 0x7fffffffu; }
    __device__ __forceinline__ void no_infinities() {
#pragma unroll
        for (int j = 0; j < words; j++)
            if (size(j) == 0x7f800000u) w[j] = __uint_as_float(0x7fffffffu);
    }
    static __device__ __forceinline__ uint32_t top(uint32_t a) { return a > 0x7f800000u ? 0 : a; }
    static __device__ __forceinline__ uint32_t low(uint32_t a) { return top(a); }
    static __device__ __forceinline__ float factor(int e0, int) { return power_of_two(-e0); }
    __device__ __forceinline__ float scaled(int j, float f) const { return w[j] * f; }
};

struct Place {
    int64_t kb, rb, batch, row0, R;   // row0: this thread's first row; R: rows in use
};

// The largest sizes of a thread's eight rows, as words of two columns' or one's.
template <typename T>
__device__ __forceinline__ void row_tops(const Row<T> (&x)[8], uint32_t (&t)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        t[i] = x[i].size(0);
#pragma unroll
        for (int j = 1; j < Row<T>::words; j++) t[i] = Row<T>::larger(t[i], x[i].size(j));
    }
}

// Half of n words of each lane (those that differ from it in bit `m` of the lane have the
// others): the maxima of both lanes' words.
template <typename X, int n>
__device__ __forceinline__ void halve(uint32_t (&w)[n], int m, int lane) {
    const bool up = lane & m;
#pragma unroll
    for (int j = 0; j < n / 2; j++) {
        const uint32_t mine = up ? w[j + n / 2] : w[j], other = up ? w[j] : w[j + n / 2];
        w[j] = X::larger(mine, __shfl_xor_sync(0xffffffffu, other, m));
    }
}

// What is left when the values and the rows' largest sizes are in registers: 256 threads,
// warp w, half h of it, lane l of the half: rows 16 w + 8 h + i, columns 8 l + j.
template <typename T, bool E5M2, bool TILE, bool ROWS, bool COLUMNS>
__device__ __forceinline__ void quantize(const QArgs &a, const Place &at, const Row<T> (&x)[8], uint32_t (&t)[8],
                                         uint32_t (&tops)[8][kFp8Block], unsigned char *turned) {
    using X = Row<T>;
    constexpr int words = X::words, each = X::each;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = lane >> 4, l = lane & 15;
    int tile_e = 0;
    if constexpr (TILE) {
        uint32_t top = t[0];
#pragma unroll
        for (int i = 1; i < 8; i++) top = X::larger(top, t[i]);
        top = __reduce_max_sync(0xffffffffu, X::top(top));
        if (lane == 0) tops[warp][0] = top;
        __syncthreads();
        top = tops[0][0];
#pragma unroll
        for (int w = 1; w < 8; w++) top = max(top, tops[w][0]);
        tile_e = scale_exponent<E5M2>(top);
        if (threadIdx.x == 0) {
            if (ROWS && a.s) a.s[(at.batch * a.KB + at.kb) * a.RB + at.rb] = power_of_two(tile_e);
            if (COLUMNS && a.st) a.st[(at.batch * a.RB + at.rb) * a.KB + at.kb] = power_of_two(tile_e);
        }
        const int r = threadIdx.x;   // of the block
        if (r < kFp8Block) {
            if (ROWS) a.e[at.batch * a.e_bytes + exponent_at(at.rb * kFp8Block + r, at.kb, a.RB)] = (uint8_t)(tile_e + 127);
            if (COLUMNS) a.et[at.batch * a.et_bytes + exponent_at(at.kb * kFp8Block + r, at.rb, a.KB)] = (uint8_t)(tile_e + 127);
        }
    }
    if constexpr (ROWS) {
        // Of the half warp's lanes, each comes to have one row (bf16: two), whose scale it
        // works out and the others ask it for.
        auto f = X::factor(tile_e, tile_e);
        if constexpr (!TILE) {
            int e[each], row;
            if constexpr (each == 2) {
                uint32_t w[4];   // rows 2 p and 2 p + 1
#pragma unroll
                for (int p = 0; p < 4; p++)
                    w[p] = X::larger(__byte_perm(t[2 * p], t[2 * p + 1], 0x5410), __byte_perm(t[2 * p], t[2 * p + 1], 0x7632));
                halve<X>(w, 8, lane);
                uint32_t v[2] = {w[0], w[1]};
                halve<X>(v, 4, lane);
#pragma unroll
                for (int m = 2; m; m /= 2) v[0] = X::larger(v[0], __shfl_xor_sync(0xffffffffu, v[0], m));
                e[0] = scale_exponent<E5M2>(X::low(v[0])), e[1] = scale_exponent<E5M2>(X::high(v[0]));
                row = 2 * (l >> 2) + (l & 1);
            } else {
                halve<X>(t, 8, lane);
                uint32_t v[4] = {t[0], t[1], t[2], t[3]};
                halve<X>(v, 4, lane);
                uint32_t u[2] = {v[0], v[1]};
                halve<X>(u, 2, lane);
                u[0] = X::larger(u[0], __shfl_xor_sync(0xffffffffu, u[0], 1));
                e[0] = scale_exponent<E5M2>(X::top(u[0]));
                row = l >> 1;
            }
            f = X::factor(e[0], e[each - 1]);
            if ((each == 2 ? (l & 2) : (l & 1)) == 0 && at.row0 + row < at.R) {
                const int mine = each == 2 && (l & 1) ? e[each - 1] : e[0];
                if (a.s) a.s[(at.batch * a.KB + at.kb) * a.R + at.row0 + row] = power_of_two(mine);
                a.e[at.batch * a.e_bytes + exponent_at(at.row0 + row, at.kb, a.RB)] = (uint8_t)(mine + 127);
            }
        }
        uint8_t *q = a.q + ((at.batch * a.R + at.row0) * a.KB + at.kb) * kFp8Block + 8 * l;
        const int64_t step = a.KB * kFp8Block;
        const int rows = (int)min((int64_t)8, at.R - at.row0);
        auto two = f;   // (bf16: of two rows)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            auto g = f;
            if constexpr (!TILE) {
                if constexpr (each == 2) {
                    if (i % 2 == 0) two = __shfl_sync(0xffffffffu, f, (lane & 16) + 2 * i);
                    g = __byte_perm(two, two, i % 2 ? 0x3232 : 0x1010);
                } else {
                    g = __shfl_sync(0xffffffffu, f, (lane & 16) + 2 * i);
                }
            }
            uint32_t b[4];   // two bytes each
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if constexpr (each == 2) {
                    const float2 y = x[i].scaled(j, g);
                    b[j] = round2<E5M2>(y.x, y.y);
                } else {
                    b[j] = round2<E5M2>(x[i].scaled(2 * j, g), x[i].scaled(2 * j + 1, g));
                }
            }
            if (i < rows) *reinterpret_cast<uint2 *>(q) = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
            q += step;
        }
    }
    if constexpr (COLUMNS) {
        if constexpr (!TILE) {
#pragma unroll
            for (int j = 0; j < words; j++) {
                uint32_t top = x[0].size(j);
#pragma unroll
                for (int i = 1; i < 8; i++) top = X::larger(top, x[i].size(j));
                top = X::larger(top, __shfl_xor_sync(0xffffffffu, top, 16));
                if (h == 0) tops[warp][words * l + j] = top;
            }
            __syncthreads();
            if (threadIdx.x < words * 16) {   // a word's columns
                uint32_t top = tops[0][threadIdx.x];
#pragma unroll
                for (int w = 1; w < 8; w++) top = X::larger(top, tops[w][threadIdx.x]);
                int e[each];
                e[0] = scale_exponent<E5M2>(X::low(top));
                if constexpr (each == 2) e[1] = scale_exponent<E5M2>(X::high(top));
#pragma unroll
                for (int k = 0; k < each; k++) {
                    const int64_t c = at.kb * kFp8Block + each * threadIdx.x + k;
                    if (c >= a.C) break;
                    if (a.st) a.st[(at.batch * a.RB + at.rb) * a.C + c] = power_of_two(e[k]);
                    a.et[at.batch * a.et_bytes + exponent_at(c, at.rb, a.KB)] = (uint8_t)(e[k] + 127);
                }
                const auto f = X::factor(e[0], e[each - 1]);
                tops[0][threadIdx.x] = *reinterpret_cast<const uint32_t *>(&f);
            }
            __syncthreads();
        }
        // eight rows of a column are eight bytes of the transposed block, whose 16 runs of
        // eight are turned by the column's group: 16 lanes write to 16 different banks' pairs
        const int run = 2 * warp + h;
#pragma unroll
        for (int j = 0; j < words; j++) {
            auto f = X::factor(tile_e, tile_e);
            if constexpr (!TILE) f = *reinterpret_cast<const decltype(f) *>(&tops[0][words * l + j]);
            uint32_t b[each][4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                if constexpr (each == 2) {
                    const float2 y = x[i].scaled(j, f), z = x[i + 1].scaled(j, f);
                    b[0][i / 2] = round2<E5M2>(y.x, z.x);
                    b[each - 1][i / 2] = round2<E5M2>(y.y, z.y);
                } else {
                    b[0][i / 2] = round2<E5M2>(x[i].scaled(j, f), x[i + 1].scaled(j, f));
                }
            }
#pragma unroll
            for (int k = 0; k < each; k++)
                *reinterpret_cast<uint2 *>(turned + (8 * l + each * j + k) * kFp8Block + 8 * (run ^ l)) =
                    make_uint2(b[k][0] | b[k][1] << 16, b[k][2] | b[k][3] << 16);
        }
        __syncthreads();
        uint8_t *qt = a.qt + ((at.batch * a.C + at.kb * kFp8Block) * a.RB + at.rb) * kFp8Block + 8 * l;
        const int left = (int)min((int64_t)kFp8Block, a.C - at.kb * kFp8Block);
        const int64_t step = a.RB * kFp8Block;
        qt += (2 * warp + h) * step;
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const int c = 2 * warp + h + 16 * k;
            if (c < left) *reinterpret_cast<uint2 *>(qt) = *reinterpret_cast<const uint2 *>(turned + c * kFp8Block + 8 * (l ^ (c >> 3)));
            qt += 16 * step;
        }
    }
}

// (CTAs an SM, registers a thread: bf16 both ways 8192 x 4096 four, 64: 22.8 us, three 24.8, two 29; fp32 two, 128: 36.7,
// three 40.4)
template <typename T, bool E5M2, bool TILE, bool ROWS, bool COLUMNS>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) k_fp8_quantize(const __grid_constant__ QArgs a) {
    using X = Row<T>;
    __shared__ uint32_t tops[8][kFp8Block];
    __shared__ __align__(16) unsigned char turned[COLUMNS ? kFp8Block * kFp8Block : 16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = lane >> 4, l = lane & 15;
    Place at;
    const unsigned rb = blockIdx.x / (unsigned)a.KB;
    at.rb = rb, at.kb = blockIdx.x - rb * (unsigned)a.KB, at.batch = blockIdx.y;
    at.row0 = at.rb * kFp8Block + 16 * warp + 8 * h;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    at.R = a.used ? min(a.R, (int64_t)max(0, *a.used)) : a.R;
    if (at.rb * kFp8Block >= at.R) return;
    X x[8];
    const int64_t col0 = at.kb * kFp8Block + 8 * l;
    const T *from = static_cast<const T *>(a.x) + (at.batch * a.R + at.row0) * a.C + col0;
    if (a.align == 16 && (at.rb + 1) * kFp8Block <= at.R && (at.kb + 1) * kFp8Block <= a.C) {   // (no test between the loads)
#pragma unroll
        for (int i = 0; i < 8; i++) x[i].load(from + i * a.C, 8, 16);
    } else {
        const int n = (int)max((int64_t)0, min((int64_t)8, a.C - col0));
#pragma unroll
        for (int i = 0; i < 8; i++) x[i].load(from + i * a.C, at.row0 + i < at.R ? n : 0, a.align);
    }
    uint32_t t[8];
    row_tops(x, t);
    uint32_t top = t[0];
#pragma unroll
    for (int i = 1; i < 8; i++) top = X::larger(top, t[i]);
    if (__syncthreads_or(X::top(top) == 0x7f800000u)) {   // (an infinity would be the largest)
#pragma unroll
        for (int i = 0; i < 8; i++) x[i].no_infinities();
        row_tops(x, t);
    }
    quantize<T, E5M2, TILE, ROWS, COLUMNS>(a, at, x, t, tops, turned);
}

template <typename T, bool E5M2, bool TILE>
cudaError_t launch(const QArgs &a, int64_t batch, cudaStream_t s) {
    if (a.KB * a.RB > INT32_MAX || batch > 65535) return cudaErrorInvalidConfiguration;
    auto kernel = a.q && a.qt ? k_fp8_quantize<T, E5M2, TILE, true, true>
                  : a.q       ? k_fp8_quantize<T, E5M2, TILE, true, false>
                              : k_fp8_quantize<T, E5M2, TILE, false, true>;
    return launch_kernel(kernel, dim3((unsigned)(a.KB * a.RB), (unsigned)batch), dim3(256), 0, s, a);
}

template <typename T>
cudaError_t launch(const QArgs &a, int64_t batch, int tile, bsr_fp8_t type, cudaStream_t s) {
    if (type == BSR_E5M2) return tile == 1 ? launch<T, true, false>(a, batch, s) : launch<T, true, true>(a, batch, s);
    return tile == 1 ? launch<T, false, false>(a, batch, s) : launch<T, false, true>(a, batch, s);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void *x, bsr_dtype_t dt, int64_t batch, int64_t R, int64_t C, int tile, bsr_fp8_t type,
                                const bsr_fp8_matrix_t *rows, const bsr_fp8_matrix_t *columns, const int32_t *used, cudaStream_t s) {
    QArgs a = {};
    a.x = x;
    a.R = R, a.C = C;
    a.KB = fp8_blocks(C), a.RB = fp8_blocks(R);
    if (rows) a.q = static_cast<uint8_t *>(rows->q), a.s = rows->scale, a.e = rows->exponent;
    if (columns) a.qt = static_cast<uint8_t *>(columns->q), a.st = columns->scale, a.et = columns->exponent;
    a.e_bytes = fp8_words(C) * a.RB * 512, a.et_bytes = fp8_words(R) * a.KB * 512;
    a.used = used;
    const int64_t bytes = C * (dt == BSR_F32 ? 4 : 2) | 16;
    a.align = (int)(bytes & -bytes);
    return dt == BSR_F32 ? launch<float>(a, batch, tile, type, s) : launch<uint16_t>(a, batch, tile, type, s);
}

}  // namespace bsr
