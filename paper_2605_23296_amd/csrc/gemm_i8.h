// What the kernels for products of codes share: the call, and an output from its sums.
#pragma once
#include <atomic>

#include "common.h"

typedef int intx4 __attribute__((ext_vector_type(4)));

#define I8_BK 128   // k-tile: a row of it is one 128-byte line

struct GemmI8Params {
    const int8_t* X;
    const float* xs;
    const int8_t* W;
    const float* ws;
    const void* R;
    void* C;
    int64_t M;
    int N;    // output columns (F for SwiGLU, whose W has 2N rows)
    int K;
    int n_mtiles, n_ntiles;
    int n_full;  // 256 x 256 kernel, plain product: workgroups that take a whole tile (the others take halves)
    int* sums;   // of k-slices
    int f32;  // C and R are fp32 rather than bf16
    GroupedArgs g;
};

// what chunks of 16 codes beyond K are read from, on the activations' side
static __device__ const int8_t zero_codes[16] __attribute__((aligned(16))) = {};

// gemv_i8.hip : at most this many rows, of a tile of the experts' map or of the call; of the call up to MOST where that pays
#define I8_STREAM_ROWS 16
#define I8_STREAM_ROWS_MOST 48
int launch_stream_i8(compact_ctx* ctx, GemmI8Params& p, bool glu, hipStream_t s);

// the kernel may use that much LDS, on every device that it runs on (a set bit is a device that knows)
static inline int allow_lds(compact_ctx* ctx, const void* kernel, size_t bytes, std::atomic<uint64_t>& known) {
    int dev = 0;
    HIP_TRY(ctx, hipGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (known.load(std::memory_order_relaxed) & bit) return COMPACT_OK;
    HIP_TRY(ctx, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    known.fetch_or(bit, std::memory_order_relaxed);
    return COMPACT_OK;
}

// One output from its sums; the same roundings wherever it is computed.
#pragma clang fp contract(off)
__device__ __forceinline__ float i8_value(int sum, float xs, float ws) { return (float)sum * xs * ws; }
__device__ __forceinline__ float i8_glu(float g, float u, bool f32) {
    if (f32) return g / (1.0f + expf(-g)) * u;
    // what a bf16 result does not see: exp2(-g log2 e), off by up to 3.4e-6 of the value at g = -80, and the reciprocal to one unit in the last
    // place (a division to half a unit is ten instructions, 64 times a lane, while the matrix pipe waits)
    return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
}

__device__ __forceinline__ void i8_put(const GemmI8Params& p, int64_t o, float v) {
    if (p.f32)
        ((float*)p.C)[o] = v + (p.R ? ((const float*)p.R)[o] : 0.f);
    else
        ((bf16*)p.C)[o] = (bf16)(v + (p.R ? (float)((const bf16*)p.R)[o] : 0.f));
}
