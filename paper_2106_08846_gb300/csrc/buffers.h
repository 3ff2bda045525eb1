// The buffers of one call of an operator without a handle, checked together.
#pragma once

#include "bsr_internal.h"
#include "host.h"

namespace bsr {

// Alignment, where they live, and that no output overlaps another buffer, but for
// the input whose place it may take (`over`: the same address).
struct Buffers {
    struct One {
        const void *p;
        size_t bytes;
        const void *over[2];
        bool out;
    };
    One all[24];
    int n = 0;
    bool misaligned = false;

    void add(const void *p, size_t bytes, size_t align, bool out, const void *over0 = nullptr, const void *over1 = nullptr) {
        if (!p) return;
        misaligned |= reinterpret_cast<uintptr_t>(p) % align != 0;
        all[n++] = One{p, bytes, {over0, over1}, out};
    }
    void in(const void *p, size_t bytes, size_t align = 16) { add(p, bytes, align, false); }
    void out(const void *p, size_t bytes, size_t align = 16, const void *over0 = nullptr, const void *over1 = nullptr) {
        add(p, bytes, align, true, over0, over1);
    }
    bsr_status_t check() const {
        if (misaligned) return BSR_ERR_ALIGNMENT;
        for (int i = 0; i < n; i++) {
            if (!all[i].out) continue;
            for (int j = 0; j < n; j++) {
                if (j == i || (all[j].out && j < i)) continue;
                if (!overlaps(all[i].p, all[i].bytes, all[j].p, all[j].bytes)) continue;
                const bool same = all[i].p == all[j].p && all[i].bytes == all[j].bytes && !all[j].out;
                if (!same || (all[i].p != all[i].over[0] && all[i].p != all[i].over[1])) return BSR_ERR_INVALID_ARG;
            }
        }
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess) {
            cudaGetLastError();
            return BSR_ERR_CUDA;
        }
        for (int i = 0; i < n; i++)
            if (all[i].bytes && classify(all[i].p, device) != PK_DEVICE) return BSR_ERR_INVALID_ARG;
        return BSR_OK;
    }
};

inline bsr_status_t launched(cudaError_t e) {
    if (e == cudaSuccess) return BSR_OK;
    cudaGetLastError();
    return BSR_ERR_CUDA;
}

inline bool known(bsr_dtype_t dt) { return dt == BSR_F32 || dt == BSR_BF16; }

}  // namespace bsr
