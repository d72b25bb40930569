// What the GEMM kernels with a ring of LDS stages share: barriers that do not drain the loads in flight, and the order of tiles.
#pragma once
#include <algorithm>

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

// How the 256 x 256 kernel cuts M rows: slots of 256 x 256 (a last row tile of more than 128 rows is one), and 128 x 256
// tiles of a bottom row tile of at most 128 rows.
struct LargeTiles {
    int64_t slots;
    int64_t bottom;
};
static inline LargeTiles large_tiles(int64_t M, int n_ntiles) {
    const int64_t rest = M % 256;
    return {(M / 256 + (rest > 128 ? 1 : 0)) * n_ntiles, rest > 0 && rest <= 128 ? n_ntiles : 0};
}

// The tile forms, by time: which one for C[M, N] over K elements of 2 bytes (gemm_bf16.hip); n_full: slots that TILE_256 takes as whole tiles.
enum { TILE_256 = 0, TILE_128, TILE_128_128, TILE_128_64, TILE_64_128, TILE_64_64, TILE_FORMS };
int pick_tile(int64_t M, int N, int K, int epilogue, int n_cus, int64_t* n_full);
