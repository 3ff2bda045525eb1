// Host-side helpers of the C entry points: the device of a call, where its
// pointers live, and whether its buffers overlap.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace bsr {

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

enum PtrKind { PK_DEVICE, PK_HOST, PK_BAD };

// Where a pointer lives, relative to the handle's device.
inline PtrKind classify(const void *p, int device) {
    cudaPointerAttributes at;
    cudaError_t e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) { cudaGetLastError(); return PK_BAD; }
    switch (at.type) {
        case cudaMemoryTypeDevice: return at.device == device ? PK_DEVICE : PK_BAD;
        case cudaMemoryTypeManaged: return PK_DEVICE;
        case cudaMemoryTypeHost:
        case cudaMemoryTypeUnregistered: return PK_HOST;
        default: return PK_BAD;
    }
}

inline bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na && nb && x < y + nb && y < x + na;
}

}  // namespace bsr
