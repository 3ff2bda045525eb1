// What the residual step reads of rows that start anywhere, checked on the host:
// every byte of a run, and no byte outside its array.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "run_blocks.h"

namespace {

struct Array {
    int base, bytes;   // address (of a 16-byte block's byte 0 on), and size
    std::vector<unsigned char> seen, values;   // (values: from address 0 on, with room beside the array)
    const char *what;
    Array(int base, int bytes, const char *what) : base(base), bytes(bytes), seen(bytes), values(base + bytes + 32), what(what) {
        for (size_t i = 0; i < values.size(); i++) values[i] = (unsigned char)(i * 151 + 7);
    }
    void touch(int at, int n) {
        if (at % n) fail("unaligned", at, n);
        if (at < base || at + n > base + bytes) fail("outside the array", at, n);
        for (int i = 0; i < n; i++) seen[at - base + i] = 1;
    }
    void fail(const char *why, int at, int n) {
        std::printf("%s: %d bytes at %d, %s (array of %d bytes at %d)\n", what, n, at, why, bytes, base);
        std::exit(1);
    }
};

// As the kernels read run `e` .. e + 7 of a row at `row`.
template <int SIZE, int WORDS>
void read(Array &a, int row, int D, int e, bool singly) {
    const int first = row + e * SIZE, left = D - e, n = left < 8 ? left : 8;
    uint32_t w[WORDS];
    std::memset(a.seen.data(), 0, a.seen.size());
    const int at = bsr::read_run<SIZE>(
        w, first & 15, n, singly,
        [&](int k, uint32_t *u) {
            const int from = (first & ~15) + 16 * k;
            a.touch(from, 16);
            std::memcpy(u, a.values.data() + from, 16);
        },
        [&](int j) {
            a.touch(first + j * SIZE, SIZE);
            uint32_t v = 0;
            std::memcpy(&v, a.values.data() + first + j * SIZE, SIZE);
            return v;
        });
    for (int i = 0; i < n * SIZE; i++)
        if (!a.seen[first - a.base + i] || reinterpret_cast<unsigned char *>(w)[at + i] != a.values[first + i])
            a.fail("not read", first + i, 1);
}

template <int SIZE>
void rows_of(int N, int D) {
    Array a(0, N * D * SIZE, "rows");
    for (int n = 0; n < N; n++) {
        const bool at_end = bsr::at_array_end(N - 1 - n, D);
        for (int e = 0; e < D + 16; e += 8) read<SIZE, 2 * SIZE + 4>(a, n * D * SIZE, D, e, at_end && bsr::at_row_end(D - e));
    }
}

}  // namespace

int main() {
    for (int D = 1; D <= 70; D++) {
        for (int N = 1; N <= 20; N++) {
            rows_of<2>(N, D);
            rows_of<4>(N, D);
        }
        for (int base = 64; base < 80; base += 4) {   // a parameter
            Array a(base, D * 4, "parameter");
            for (int e = 0; e < D + 16; e += 8) read<4, 8>(a, base, D, e, D - e < 8 || base % 16 != 0);
        }
    }
    std::puts("all runs inside");
    return 0;
}
