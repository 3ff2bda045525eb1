// fp32 values as bf16 parts.
#pragma once

#include <cstdint>

namespace bsr {

// The parts of x and y, pairs of the same part in a word, x in its lower half: each the
// rounding of what the parts before it left, at most 2^-8 of them. The sum of three is
// the value. None overflows (a value that would goes to the largest); of an infinity the
// last part is one, and the others have its sign.
template <int N>
__device__ __forceinline__ void parts_of(float x, float y, uint32_t (&p)[N]) {
#pragma unroll
    for (int k = 0; k + 1 < N; k++) {
        asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(p[k]) : "f"(y), "f"(x));
        x -= __uint_as_float(p[k] << 16);
        y -= __uint_as_float(p[k] & 0xffff0000u);
    }
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[N - 1]) : "f"(y), "f"(x));
}

}  // namespace bsr
