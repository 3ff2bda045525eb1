// Eight values of a row, as results leave the tensor cores' accumulators: packed,
// exchanged between lanes, loaded and stored in words as wide as rows are aligned.
#pragma once

#include <cstdint>

#include "elem.cuh"
#include "pair.cuh"

namespace bsr {

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Eight values of a row as they lie in memory: 16 bytes of bf16, 32 of fp32.
template <typename T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
};
__device__ __forceinline__ F2 two_of(const Eight<uint16_t> &r, int j) {
    return pack2(__uint_as_float(r.w[j] << 16), __uint_as_float(r.w[j] & 0xffff0000u));
}
__device__ __forceinline__ F2 two_of(const Eight<float> &r, int j) {
    return pack2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1]));
}
__device__ __forceinline__ uint32_t pack_bf16(F2 x) {
    const float2 u = unpack2(x);
    return pack_bf16(u.x, u.y);
}
template <typename T>
__device__ __forceinline__ Eight<T> eight_of(const F2 (&v)[4]) {
    Eight<T> r;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if constexpr (sizeof(T) == 2) {
            r.w[j] = pack_bf16(v[j]);
        } else {
            const float2 u = unpack2(v[j]);
            r.w[2 * j] = __float_as_uint(u.x), r.w[2 * j + 1] = __float_as_uint(u.y);
        }
    }
    return r;
}
// Eight values to p, n of which are there (the rest is past the row's end), in
// stores as wide as the rows are aligned; and from p, 0 past the end.
template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t n, int align, const Eight<T> &r) {
    constexpr int words = 2 * sizeof(T);
    if (n >= 8 && align == 16) {
#pragma unroll
        for (int h = 0; h < words / 4; h++)
            reinterpret_cast<uint4 *>(p)[h] = make_uint4(r.w[4 * h], r.w[4 * h + 1], r.w[4 * h + 2], r.w[4 * h + 3]);
    } else if (n >= 8 && align >= 8) {
#pragma unroll
        for (int h = 0; h < words / 2; h++) reinterpret_cast<uint2 *>(p)[h] = make_uint2(r.w[2 * h], r.w[2 * h + 1]);
    } else if (n >= 8 && align >= 4) {
#pragma unroll
        for (int h = 0; h < words; h++) reinterpret_cast<uint32_t *>(p)[h] = r.w[h];
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            if (j >= n) break;
            if constexpr (sizeof(T) == 2) p[j] = (uint16_t)(r.w[j / 2] >> (16 * (j & 1)));
            else p[j] = __uint_as_float(r.w[j]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t n, int align, Eight<T> &r) {
    constexpr int words = 2 * sizeof(T);
    if (n >= 8 && align == 16) {
#pragma unroll
        for (int h = 0; h < words / 4; h++) {
            const uint4 u = reinterpret_cast<const uint4 *>(p)[h];
            r.w[4 * h] = u.x, r.w[4 * h + 1] = u.y, r.w[4 * h + 2] = u.z, r.w[4 * h + 3] = u.w;
        }
    } else if (n >= 8 && align >= 8) {
#pragma unroll
        for (int h = 0; h < words / 2; h++) {
            const uint2 u = reinterpret_cast<const uint2 *>(p)[h];
            r.w[2 * h] = u.x, r.w[2 * h + 1] = u.y;
        }
    } else if (n >= 8 && align >= 4) {
#pragma unroll
        for (int h = 0; h < words; h++) r.w[h] = reinterpret_cast<const uint32_t *>(p)[h];
    } else {
#pragma unroll
        for (int j = 0; j < words; j++) r.w[j] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            if (j >= n) break;
            if constexpr (sizeof(T) == 2) r.w[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
            else r.w[j] = __float_as_uint(p[j]);
        }
    }
}

// Words of two columns each: word i of lane j of four has columns 8 i + 2 j, + 1; word j
// of lane i will, so that a lane has eight columns: for each bit of i and j, the lanes
// that differ in it exchange the words that differ from the lane in it.
__device__ __forceinline__ void turn_words(uint32_t (&w)[4]) {
    const int q = threadIdx.x & 3;
#pragma unroll
    for (int bit = 1; bit < 4; bit *= 2)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (i & bit) continue;
            const uint32_t got = __shfl_xor_sync(0xffffffffu, q & bit ? w[i] : w[i | bit], bit);
            if (q & bit) w[i] = got;
            else w[i | bit] = got;
        }
}

}  // namespace bsr
