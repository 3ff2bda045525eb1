// Reads of a run of up to eight values that starts anywhere: by the 16-byte blocks of
// memory that hold it, or where one of them may reach out of its array, one by one.
// Host code too, so that what is read can be checked there.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define BSR_HOST_DEVICE __host__ __device__ __forceinline__
#define BSR_UNROLL _Pragma("unroll")
#else
#define BSR_HOST_DEVICE inline
#define BSR_UNROLL
#endif

namespace bsr {

// Whether a run's blocks may reach out of its array, which begins on a 16-byte boundary:
// whether fewer than eight values of it lie past the run, which has the row's next `left`
// values, at most eight, of D; `rows` rows follow. The first test is a row's.
BSR_HOST_DEVICE bool at_array_end(int64_t rows, int D) { return rows * D < 8; }
BSR_HOST_DEVICE bool at_row_end(int left) { return left < 16; }

// A run of n values (none: <= 0), SIZE bytes each, whose first byte is byte `at` of a
// block, to w, 0 past its end, if `singly`; else the blocks that hold it, and what lies
// beside it in them. block(k, u) reads the k-th block, value(j) the run's j-th value.
// Returns the place of the run's first byte in w.
template <int SIZE, int WORDS, typename Block, typename Value>
BSR_HOST_DEVICE int read_run(uint32_t (&w)[WORDS], int at, int n, bool singly, Block block, Value value) {
    BSR_UNROLL
    for (int k = 0; k < WORDS; k++) w[k] = 0;
    if (singly) {
        BSR_UNROLL
        for (int j = 0; j < 8; j++)
            if (j < n) w[j * SIZE / 4] |= (uint32_t)value(j) << (j * SIZE % 4 * 8);
        return 0;
    }
    BSR_UNROLL
    for (int k = 0; k < WORDS / 4; k++)
        if (n > 0 && 16 * k < at + n * SIZE) block(k, w + 4 * k);
    return at;
}

}  // namespace bsr
