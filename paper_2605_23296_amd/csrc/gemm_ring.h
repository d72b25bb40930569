// What the GEMM kernels with a ring of LDS stages share: barriers that do not drain the loads in flight, and the order of tiles.
#pragma once
#include "common.h"

// Waits until at most N_IN_FLIGHT of this wave's global loads are outstanding (the older ones have landed in
// LDS) and all of its LDS reads have returned, then joins the workgroup barrier.  Unlike __syncthreads() it
// does not drain the newer loads.
template <int N_IN_FLIGHT>
__device__ __forceinline__ void ring_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
    static_assert(N_IN_FLIGHT >= 0 && N_IN_FLIGHT < 64, "vector-memory counter is 6 bits");
    __builtin_amdgcn_sched_barrier(0);
    // simm16: vmcnt[3:0] | expcnt (7 = no wait) << 4 | lgkmcnt (0) << 8 | vmcnt[5:4] << 14
    __builtin_amdgcn_s_waitcnt((N_IN_FLIGHT & 15) | (7 << 4) | (0 << 8) | ((N_IN_FLIGHT >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#endif
}
__device__ __forceinline__ void plain_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#endif
}
__device__ __forceinline__ void wave_priority_high() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_setprio(1);
#endif
}
__device__ __forceinline__ void wave_priority_normal() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_setprio(0);
#endif
}

// workgroup i of n that are dealt round robin -> its place in the order of tiles
__device__ __forceinline__ int xcd_order(int i, int n) {
    const int per = n / 8, rem = n % 8, xcd = i % 8;
    return xcd * per + min(xcd, rem) + i / 8;
}
// place in the order -> row tile, column tile (n_mtiles row tiles)
template <int GM>
__device__ __forceinline__ void tile_at(int pid, int n_mtiles, int n_ntiles, int& tm, int& tn) {
    const int per_group = GM * n_ntiles;
    const int first_m = (pid / per_group) * GM;
    const int gsize = min(GM, n_mtiles - first_m);
    tm = first_m + (pid % per_group) % gsize;
    tn = (pid % per_group) / gsize;
}
