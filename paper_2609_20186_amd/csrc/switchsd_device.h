// switchsd_device.h -- device helpers shared by the kernels around the step
// (switchsd_logits.hip, switchsd_pages.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "switchsd_internal.h"

namespace switchsd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int clampi(int v, int lo, int hi) {
    return v < lo ? lo : (v > hi ? hi : v);
}

// Inclusive sum over the wave's lanes: row shifts, then two row broadcasts.
__device__ __forceinline__ int wave_scan(int v) {
#define SWITCHSD_STEP(ctrl, mask) \
    v += __builtin_amdgcn_update_dpp(0, v, ctrl, mask, 0xf, false);
    SWITCHSD_STEP(0x111, 0xf)
    SWITCHSD_STEP(0x112, 0xf)
    SWITCHSD_STEP(0x114, 0xf)
    SWITCHSD_STEP(0x118, 0xf)
    SWITCHSD_STEP(0x142, 0xa)
    SWITCHSD_STEP(0x143, 0xc)
#undef SWITCHSD_STEP
    return v;
}

// Values that one work-group hands to another travel through agent-scope
// atomics, which are coherent across the XCDs without any L2 write-back.
__device__ __forceinline__ unsigned long long ld_u64(const unsigned long long *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void st_u64(unsigned long long *p, unsigned long long v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void st_u32(uint32_t *p, uint32_t v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Wave 0 arrives at a ticket, after all of its outstanding memory operations;
// true (wave-uniform) for the last of `expected` arrivals.
__device__ __forceinline__ bool arrive(uint32_t *ticket, uint32_t expected) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
    uint32_t old = 0;
    if (threadIdx.x == 0)
        old = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    old = __shfl(old, 0);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    return old + 1u == expected;
}

// Pointer jumping over a draft's nodes.  State of node i: bit 31 = every edge
// from i up to `anc` holds, bits 16..30 = how many those are, bits 0..15 =
// anc.  A round replaces a state by its composition with that of anc, which
// doubles the covered path; the anchor's state (holds, 0 edges, itself) is the
// identity.
constexpr uint32_t kHolds = 0x80000000u;
__device__ __forceinline__ uint32_t jump_compose(uint32_t s1, uint32_t s2) {
    return (s1 & s2 & kHolds) | ((s1 & 0x7FFF0000u) + (s2 & 0x7FFF0000u)) | (s2 & 0xFFFFu);
}

}  // namespace switchsd
