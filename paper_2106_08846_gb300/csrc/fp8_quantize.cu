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
// One pass: a CTA holds 128 x 128 values in registers, takes the largest of each
// row's 128 (16 lanes) and of each column's (the lanes' eight rows, then the eight
// warps'), and writes them as they lie and transposed, through shared memory, so
// that both operands of a later product have the sum's axis contiguous.
//
// What bounds it: DRAM.
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

// |x| as bits, 0 where it is not finite
__device__ __forceinline__ uint32_t size_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0;
}

// Two values times a power of two, in 8 bits each (the first one's low).
template <bool E5M2>
__device__ __forceinline__ uint32_t round2(float x0, float x1, float inv) {
    float y0 = x0 * inv, y1 = x1 * inv;
    y0 = fmaf(y0, 0.f, y0), y1 = fmaf(y1, 0.f, y1);   // infinities become NaN
    uint16_t r;
    if constexpr (E5M2) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y1), "f"(y0));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y1), "f"(y0));
    return r;
}

// Eight values of a row from p on, n of which are there (the others 0).
template <typename T>
__device__ __forceinline__ void load_eight(const T *p, int64_t n, int align, float (&x)[8]) {
    if (n >= 8 && align == 16) {
        if constexpr (sizeof(T) == 2) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; j++) x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        } else {
            const float4 u = __ldg(reinterpret_cast<const float4 *>(p)), v = __ldg(reinterpret_cast<const float4 *>(p) + 1);
            x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
        }
    } else if (sizeof(T) == 2 && n >= 8 && align >= 4) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t w = __ldg(reinterpret_cast<const uint32_t *>(p) + j);
            x[2 * j] = __uint_as_float(w << 16), x[2 * j + 1] = __uint_as_float(w & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = j < n ? to_f32(__ldg(p + j)) : 0.f;
    }
}

// 256 threads: warp w, half h of it, lane l of the half: rows 16 w + 8 h + i, columns 8 l + j.
template <typename T, bool E5M2, bool TILE, bool ROWS, bool COLUMNS>
__global__ void __launch_bounds__(256) k_fp8_quantize(const __grid_constant__ QArgs a) {
    __shared__ uint32_t tops[8][kFp8Block];
    __shared__ __align__(16) unsigned char turned[COLUMNS ? kFp8Block * kFp8Block : 16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = lane >> 4, l = lane & 15;
    const int64_t kb = blockIdx.x % a.KB, rb = blockIdx.x / a.KB, batch = blockIdx.y;
    const int64_t row0 = rb * kFp8Block + 16 * warp + 8 * h, col0 = kb * kFp8Block + 8 * l;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t R = a.used ? min(a.R, (int64_t)max(0, __ldg(a.used))) : a.R;
    if (rb * kFp8Block >= R) return;
    float x[8][8];
    const T *from = static_cast<const T *>(a.x) + (batch * a.R + row0) * a.C + col0;
#pragma unroll
    for (int i = 0; i < 8; i++) load_eight(from + i * a.C, row0 + i < R ? a.C - col0 : 0, a.align, x[i]);
    uint32_t row_top[8], col_top[8] = {};
#pragma unroll
    for (int i = 0; i < 8; i++) {
        row_top[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const uint32_t b = size_bits(x[i][j]);
            row_top[i] = max(row_top[i], b);
            if (COLUMNS && !TILE) col_top[j] = max(col_top[j], b);
        }
    }
    int tile_e = 0;
    if constexpr (TILE) {
        uint32_t t = row_top[0];
#pragma unroll
        for (int i = 1; i < 8; i++) t = max(t, row_top[i]);
        t = __reduce_max_sync(0xffffffffu, t);
        if (lane == 0) tops[warp][0] = t;
        __syncthreads();
        t = tops[0][0];
#pragma unroll
        for (int w = 1; w < 8; w++) t = max(t, tops[w][0]);
        tile_e = scale_exponent<E5M2>(t);
        if (threadIdx.x == 0) {
            if (ROWS && a.s) a.s[(batch * a.KB + kb) * a.RB + rb] = power_of_two(tile_e);
            if (COLUMNS && a.st) a.st[(batch * a.RB + rb) * a.KB + kb] = power_of_two(tile_e);
        }
        const int r = threadIdx.x;   // of the block
        if (r < kFp8Block) {
            if (ROWS) a.e[batch * a.e_bytes + exponent_at(rb * kFp8Block + r, kb, a.RB)] = (uint8_t)(tile_e + 127);
            if (COLUMNS) a.et[batch * a.et_bytes + exponent_at(kb * kFp8Block + r, rb, a.KB)] = (uint8_t)(tile_e + 127);
        }
    }
    if constexpr (ROWS) {
        int mine = 0;   // of row l, for lanes l < 8
#pragma unroll
        for (int i = 0; i < 8; i++) {
            int e = tile_e;
            if constexpr (!TILE) {
#pragma unroll
                for (int m = 8; m; m /= 2) row_top[i] = max(row_top[i], __shfl_xor_sync(0xffffffffu, row_top[i], m));
                e = scale_exponent<E5M2>(row_top[i]);
                if (l == i) mine = e;
            }
            const float inv = power_of_two(-e);
            const uint32_t w0 = round2<E5M2>(x[i][0], x[i][1], inv) | round2<E5M2>(x[i][2], x[i][3], inv) << 16,
                           w1 = round2<E5M2>(x[i][4], x[i][5], inv) | round2<E5M2>(x[i][6], x[i][7], inv) << 16;
            if (row0 + i < R) *reinterpret_cast<uint2 *>(a.q + ((batch * a.R + row0 + i) * a.KB + kb) * kFp8Block + 8 * l) = make_uint2(w0, w1);
        }
        if (!TILE && l < 8 && row0 + l < R) {
            if (a.s) a.s[(batch * a.KB + kb) * a.R + row0 + l] = power_of_two(mine);
            a.e[batch * a.e_bytes + exponent_at(row0 + l, kb, a.RB)] = (uint8_t)(mine + 127);
        }
    }
    if constexpr (COLUMNS) {
        if constexpr (!TILE) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                col_top[j] = max(col_top[j], __shfl_xor_sync(0xffffffffu, col_top[j], 16));
                if (h == 0) tops[warp][8 * l + j] = col_top[j];
            }
            __syncthreads();
            if (threadIdx.x < kFp8Block) {
                uint32_t t = tops[0][threadIdx.x];
#pragma unroll
                for (int w = 1; w < 8; w++) t = max(t, tops[w][threadIdx.x]);
                const int e = scale_exponent<E5M2>(t);
                const int64_t c = kb * kFp8Block + threadIdx.x;
                if (c < a.C) {
                    if (a.st) a.st[(batch * a.RB + rb) * a.C + c] = power_of_two(e);
                    a.et[batch * a.et_bytes + exponent_at(c, rb, a.KB)] = (uint8_t)(e + 127);
                }
                tops[0][threadIdx.x] = __float_as_uint(power_of_two(-e));
            }
            __syncthreads();
        }
        // eight rows of a column are eight bytes of the transposed block, whose 16 runs of
        // eight are turned by the column's group: 16 lanes write to 16 different banks' pairs
        const int run = 2 * warp + h;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float inv = TILE ? power_of_two(-tile_e) : __uint_as_float(tops[0][8 * l + j]);
            const uint32_t w0 = round2<E5M2>(x[0][j], x[1][j], inv) | round2<E5M2>(x[2][j], x[3][j], inv) << 16,
                           w1 = round2<E5M2>(x[4][j], x[5][j], inv) | round2<E5M2>(x[6][j], x[7][j], inv) << 16;
            *reinterpret_cast<uint2 *>(turned + (8 * l + j) * kFp8Block + 8 * (run ^ l)) = make_uint2(w0, w1);
        }
        __syncthreads();
        for (int c = 2 * warp + h; c < kFp8Block; c += 16) {
            const int64_t col = kb * kFp8Block + c;
            if (col >= a.C) break;
            const uint2 w = *reinterpret_cast<const uint2 *>(turned + c * kFp8Block + 8 * (l ^ (c >> 3)));
            *reinterpret_cast<uint2 *>(a.qt + ((batch * a.C + col) * a.RB + rb) * kFp8Block + 8 * l) = w;
        }
    }
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
