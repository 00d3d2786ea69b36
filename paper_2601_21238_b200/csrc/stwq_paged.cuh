// Shared by the translation units of the paged cache and of the sampler.
#pragma once

#include "stwq_internal.cuh"

static inline bool stwq_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether a [T, H, d] output with these token and head strides puts no two elements in one place (token-major,
// head-major, or a view of a wider row).
static inline bool stwq_disjoint(int64_t T, int H, int d, int64_t ts, int64_t hs)
{
    if (T == 1 && H == 1) return true;
    if (T == 1) return hs >= d;
    if (H == 1) return ts >= d;
    return (hs >= d && ts >= hs * (H - 1) + d) || (ts >= d && hs >= ts * (T - 1) + d);
}

// Make the context's device current for the duration of a call.
struct StwqDevGuard {
    int prev = -1;
    bool switched = false;
    explicit StwqDevGuard(int dev)
    {
        if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) {
            cudaSetDevice(dev);
            switched = true;
        }
    }
    ~StwqDevGuard()
    {
        if (switched) cudaSetDevice(prev);
    }
};
