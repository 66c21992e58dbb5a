// Rows that a few warps of a CTA share: sums and maxima of a row, and one outcome of the
// wait for it.
#pragma once

#include "crc_device.cuh"

namespace crc {

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The warps that share a row: `warps` of them, `id` the row's number in the CTA.
struct RowTeam {
    int warps, id, thread, threads;
    __device__ __forceinline__ explicit RowTeam(int w)
        : warps(w), id((threadIdx.x >> 5) / w), thread(threadIdx.x - id * 32 * w), threads(32 * w) {}
    // the whole CTA
    __device__ __forceinline__ RowTeam()
        : warps(blockDim.x >> 5), id(0), thread(threadIdx.x), threads(blockDim.x) {}
};

// Sum (or NaN-keeping maximum) of v over a row's warps, in one fixed order; every
// thread gets it.  `buf`: a float a warp of the CTA, not in use by an earlier
// reduction that a thread may still be reading.
template <bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* buf, const RowTeam& t) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    if (t.warps == 1) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) buf[threadIdx.x >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + t.id), "r"(t.threads) : "memory");
    v = lane < t.warps ? buf[t.id * t.warps + lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    return v;
}

// A row's wait has one outcome for its team.  Every thread waits with a limit of its own,
// and a phase that completes near that limit is seen by some and not by others; one that
// left alone would leave the rest at the team's barrier, which has no limit.  So nobody
// leaves before the row's reduction: tell() before it (`ok`: this thread's wait; returns
// the warp's), all() after it, the same answer for every thread.  `lost`: a word of the
// team, zero at first, not that of the row before (a thread may still be reading it).
__device__ __forceinline__ bool row_tell(bool ok, uint32_t* lost) {
    ok = __all_sync(kFull, ok);
    if (!ok && (threadIdx.x & 31) == 0) *lost = 1u;
    return ok;
}
__device__ __forceinline__ bool row_all(bool warp_ok, const uint32_t* lost, const RowTeam& t) {
    return t.warps == 1 ? warp_ok : *const_cast<const volatile uint32_t*>(lost) == 0u;
}

}  // namespace crc
