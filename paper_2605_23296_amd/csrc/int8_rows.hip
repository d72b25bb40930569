// Rows as 8-bit codes, and the norms around a block whose rows leave as codes.
#include "common.h"
#include "int8_codes.h"
#include "vecio.h"

#define NT 256

// largest |x| of the workgroup, as bits: they are ordered as the values are, infinities and NaN above all of them
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// A workgroup per row: the largest value, then the codes.
template <typename T>
__global__ __launch_bounds__(NT) void quant_i8_kernel(const T* __restrict__ x, int64_t x_stride, int cols, int8_t* __restrict__ q,
                                                      float* __restrict__ scale) {
    __shared__ uint32_t red[NT / 64];
    const int64_t row = blockIdx.x;
    const T* xr = x + row * x_stride;
    uint32_t m = 0;
    for (int c = threadIdx.x; c < cols; c += NT) m = max(m, abs_bits(to_f32(xr[c])));
    const RowCodes rc = row_codes(block_max(m, red));
    for (int c = threadIdx.x; c < cols; c += NT) q[row * cols + c] = (int8_t)code_of<T>(to_f32(xr[c]), rc);
    if (threadIdx.x == 0) scale[row] = rc.scale;
}

int launch_quant_i8(compact_ctx* ctx, const void* x, int64_t x_stride, int64_t rows, int cols, int8_t* q, float* scale, hipStream_t s) {
    if (rows == 0) return COMPACT_OK;
    if (ctx->cfg.dtype == COMPACT_BF16)
        quant_i8_kernel<bf16><<<(unsigned)rows, NT, 0, s>>>((const bf16*)x, x_stride, cols, q, scale);
    else
        quant_i8_kernel<float><<<(unsigned)rows, NT, 0, s>>>((const float*)x, x_stride, cols, q, scale);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

// A workgroup per row, the row in registers: a thread holds the 8-element pieces threadIdx + 256 i.  (h, n may be x or b: nothing is
// written before the whole row has been read, and no pointer promises to be alone.)
template <typename T, int P>
__global__ __launch_bounds__(NT) void block_norm_kernel(const BlockNormArgs a, int d, float eps) {
    __shared__ float red[NT / 64];
    __shared__ uint32_t redm[NT / 64];
    const int64_t row = blockIdx.x;
    float v[P][8], b[P][8];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (threadIdx.x + i * NT) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = b[i][j] = 0.f;
        if (c < d) {
            load8((const T*)a.x + row * d + c, v[i]);
            if (a.b) load8((const T*)a.b + row * d + c, b[i]);
        }
    }
    if (a.b) {
        float inv = 1.f;
        if (a.g_post) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += b[i][j] * b[i][j];
            inv = 1.0f / sqrtf(block_sum(ss, red) / (float)d + eps);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (threadIdx.x + i * NT) * 8;
            if (c >= d) continue;
            float g[8];
            if (a.g_post) {
                load8((const T*)a.g_post + c, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) b[i][j] = b[i][j] * inv * g[j];
            }
            if (a.gate) {
                load8((const T*)a.gate + row * a.gate_stride + c, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) b[i][j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = to_f32(from_f32<T>(v[i][j] + a.alpha * b[i][j]));
        }
    }
    float inv = 0.f;
    if (a.g_pre) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
        inv = 1.0f / sqrtf(block_sum(ss, red) / (float)d + eps);
    }
    __syncthreads();
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (threadIdx.x + i * NT) * 8;
        if (c >= d) continue;
        if (a.h) store8((T*)a.h + row * d + c, v[i]);
        if (a.g_pre) {
            float g[8];
            load8((const T*)a.g_pre + c, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] = to_f32(from_f32<T>(v[i][j] * inv * g[j]));
                m = max(m, abs_bits(v[i][j]));
            }
            if (a.n) store8((T*)a.n + row * d + c, v[i]);
        }
    }
    if (!a.q) return;
    const RowCodes rc = row_codes(block_max(m, redm));
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (threadIdx.x + i * NT) * 8;
        if (c < d) *reinterpret_cast<uint2*>(a.q + row * d + c) = codes8<T>(v[i], rc);
    }
    if (threadIdx.x == 0) a.q_scale[row] = rc.scale;
}

template <typename T>
static void run_block_norm(const BlockNormArgs& a, int d, float eps, hipStream_t s) {
    const unsigned rows = (unsigned)a.rows;
    switch ((d + NT * 8 - 1) / (NT * 8)) {   // (d_model is at most 8192)
        case 1: block_norm_kernel<T, 1><<<rows, NT, 0, s>>>(a, d, eps); break;
        case 2: block_norm_kernel<T, 2><<<rows, NT, 0, s>>>(a, d, eps); break;
        case 3: block_norm_kernel<T, 3><<<rows, NT, 0, s>>>(a, d, eps); break;
        default: block_norm_kernel<T, 4><<<rows, NT, 0, s>>>(a, d, eps); break;
    }
}
int launch_block_norm(compact_ctx* ctx, const BlockNormArgs& a, hipStream_t s) {
    if (a.rows == 0) return COMPACT_OK;
    if (ctx->cfg.dtype == COMPACT_BF16)
        run_block_norm<bf16>(a, ctx->cfg.d_model, ctx->cfg.rms_eps, s);
    else
        run_block_norm<float>(a, ctx->cfg.d_model, ctx->cfg.rms_eps, s);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}
