// Rows as 8-bit codes, and the norms around a block whose rows leave as codes.  Both are bound by HBM and read a row once: it waits in
// registers for its largest value or its sum of squares.  Codes of 1652 x 14336 13.2 us (5.4 TB/s; an element at a time and twice 99), of 65536 x 2880 89 (6.4);
// norm with a block's output of 32768 x 4096 rows 181 us (5.9 TB/s, what a copy of that size reaches), of 8 rows 5.0.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "int8_codes.h"
#include "vecio.h"

#define NT 256

// largest |x| of the wavefront, of the workgroup, as bits: they are ordered as the values are, infinities and NaN above all of them
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
    v = wave_max_bits(v);
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

// 8 elements as they lie in memory
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
    bf16x8 v;
    __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const bf16x8*>(p); }
    __device__ __forceinline__ void zero() { v = bf16x8{}; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float)v[j];
    }
};
template <>
struct Piece<float> {
    floatx4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const floatx4*>(p);
        b = *reinterpret_cast<const floatx4*>(p + 4);
    }
    __device__ __forceinline__ void zero() { a = b = floatx4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[j] = a[j];
            f[4 + j] = b[j];
        }
    }
};

// TPR threads per row (64: a wavefront, four rows a workgroup; else a workgroup), a thread holds the pieces thread + TPR i: the row is read once.
template <typename T, int TPR, int P>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void quant_i8_kernel(const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols,
                                                                         int8_t* __restrict__ q, float* __restrict__ scale) {
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1;
    __shared__ uint32_t red[TPR / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (row >= rows) return;   // (a whole wavefront; only where rows need no barrier)
    const T* xr = x + row * x_stride;
    Piece<T> v[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c < cols)
            v[i].load(xr + c);
        else
            v[i].zero();
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float f[8];
        v[i].get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(f[j]));
    }
    m = wave_max_bits(m);
    if (TPR > 64) {
        if ((t & 63) == 0) red[t / 64] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) m = max(m, red[w]);
    }
    const RowCodes rc = row_codes(m);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (t + i * TPR) * 8;
        float f[8];
        v[i].get(f);
        if (c < cols) *reinterpret_cast<uint2*>(q + row * cols + c) = codes8<T>(f, rc);
    }
    if (t == 0) scale[row] = rc.scale;
}

// Rows that are too long for that, or whose pieces of 8 are not aligned: the largest value, then the codes, an element at a time.
// (The column is unsigned: with up to 2^31 - 1 of them, the step past the last one does not fit an int.)
template <typename T>
__global__ __launch_bounds__(1024) void quant_i8_any_kernel(const T* __restrict__ x, int64_t x_stride, int cols, int8_t* __restrict__ q,
                                                            float* __restrict__ scale) {
    __shared__ uint32_t red[16];
    const int64_t row = blockIdx.x;
    const T* xr = x + row * x_stride;
    uint32_t m = 0;
    for (uint32_t c = threadIdx.x; c < (uint32_t)cols; c += 1024) m = max(m, abs_bits(to_f32(xr[c])));
    m = wave_max_bits(m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) m = max(m, red[w]);
    const RowCodes rc = row_codes(m);
    for (uint32_t c = threadIdx.x; c < (uint32_t)cols; c += 1024) q[row * cols + c] = (int8_t)code_of<T>(to_f32(xr[c]), rc);
    if (threadIdx.x == 0) scale[row] = rc.scale;
}

template <typename T, int TPR, int P>
static void run_quant(const T* x, int64_t x_stride, int64_t rows, int cols, int8_t* q, float* scale, hipStream_t s) {
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1;
    quant_i8_kernel<T, TPR, P><<<(unsigned)((rows + RPW - 1) / RPW), TPR < 256 ? 256 : TPR, 0, s>>>(x, x_stride, rows, cols, q, scale);
}
template <typename T>
static void quant_rows(const T* x, int64_t x_stride, int64_t rows, int cols, int8_t* q, float* scale, hipStream_t s) {
    // A wavefront per row up to 4 pieces a lane, and up to 6 where rows fill the chip anyway (no barrier, all lanes at work: 65536 x 2880 in workgroups of
    // 256 leaves 30 % of the lanes idle); beyond, as many threads as hold the row in 4 or 8 pieces each.
    const bool wide = cols % 8 == 0 && x_stride % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & 7) == 0;
    const int pieces = cols / 8;
    if (!wide || pieces > 8192)
        quant_i8_any_kernel<T><<<(unsigned)rows, 1024, 0, s>>>(x, x_stride, cols, q, scale);
    else if (pieces <= 64)
        run_quant<T, 64, 1>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 128)
        run_quant<T, 64, 2>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 256)
        run_quant<T, 64, 4>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 384 && rows >= 1024)
        run_quant<T, 64, 6>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 512)
        run_quant<T, 256, 2>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 1024)
        run_quant<T, 256, 4>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 2048)
        run_quant<T, 512, 4>(x, x_stride, rows, cols, q, scale, s);
    else if (pieces <= 4096)
        run_quant<T, 1024, 4>(x, x_stride, rows, cols, q, scale, s);
    else
        run_quant<T, 1024, 8>(x, x_stride, rows, cols, q, scale, s);
}

// rows of a launch at most (of up to 1024 threads each)
#define ROWS_PER_LAUNCH (1ll << 21)
static_assert(ROWS_PER_LAUNCH * 1024 <= MAX_GRID_THREADS, "one launch");

int launch_quant_i8(compact_ctx* ctx, const void* x, int64_t x_stride, int64_t rows, int cols, int8_t* q, float* scale, hipStream_t s) {
    for (int64_t r = 0; r < rows; r += ROWS_PER_LAUNCH) {
        const int64_t n = std::min<int64_t>(rows - r, ROWS_PER_LAUNCH);
        if (ctx->cfg.dtype == COMPACT_BF16)
            quant_rows((const bf16*)x + r * x_stride, x_stride, n, cols, q + r * cols, scale + r, s);
        else
            quant_rows((const float*)x + r * x_stride, x_stride, n, cols, q + r * cols, scale + r, s);
        LAUNCH_CHECK(ctx);
    }
    return COMPACT_OK;
}

// TPR threads per row (64: a wavefront, four rows a workgroup, no barrier; 256: a workgroup), the row in registers: a thread holds the 8-element pieces t + TPR i.  (h, n may be x or b: nothing is
// written before the whole row has been read, and no pointer promises to be alone.)
template <typename T, int TPR, int P>
__global__ __launch_bounds__(NT) void block_norm_kernel(const BlockNormArgs a, int d, float eps) {
    __shared__ float red[NT / 64];
    __shared__ uint32_t redm[NT / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (TPR < NT && row >= a.rows) return;
    auto sum = [&](float x) __attribute__((always_inline)) { return TPR == 64 ? wave_sum(x) : block_sum(x, red); };
    float v[P][8], b[P][8];
    // everything that the row needs is requested before anything is used: few rows would wait for each of it
    Piece<T> xv[P], bv[P], g_post[P], gate[P], g_pre[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (t + i * TPR) * 8;
        xv[i].zero();
        bv[i].zero();
        if (c < d) {
            xv[i].load((const T*)a.x + row * d + c);
            if (a.b) bv[i].load((const T*)a.b + row * d + c);
            if (a.g_post) g_post[i].load((const T*)a.g_post + c);
            if (a.gate) gate[i].load((const T*)a.gate + row * a.gate_stride + c);
            if (a.g_pre) g_pre[i].load((const T*)a.g_pre + c);
        }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        xv[i].get(v[i]);
        bv[i].get(b[i]);
    }
    if (a.b) {
        float inv = 1.f;
        if (a.g_post) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += b[i][j] * b[i][j];
            inv = 1.0f / sqrtf(sum(ss) / (float)d + eps);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c >= d) continue;
            float g[8];
            if (a.g_post) {
                g_post[i].get(g);
#pragma unroll
                for (int j = 0; j < 8; ++j) b[i][j] = b[i][j] * inv * g[j];
            }
            if (a.gate) {
                gate[i].get(g);
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
        inv = 1.0f / sqrtf(sum(ss) / (float)d + eps);
    }
    if (TPR > 64) __syncthreads();
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c >= d) continue;
        if (a.h) store8((T*)a.h + row * d + c, v[i]);
        if (a.g_pre) {
            float g[8];
            g_pre[i].get(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] = to_f32(from_f32<T>(v[i][j] * inv * g[j]));
                m = max(m, abs_bits(v[i][j]));
            }
            if (a.n) store8((T*)a.n + row * d + c, v[i]);
        }
    }
    if (!a.q) return;
    const RowCodes rc = row_codes(TPR == 64 ? wave_max_bits(m) : block_max(m, redm));
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c < d) *reinterpret_cast<uint2*>(a.q + row * d + c) = codes8<T>(v[i], rc);
    }
    if (t == 0) a.q_scale[row] = rc.scale;
}

template <typename T>
static void run_block_norm(const BlockNormArgs& a, int d, float eps, hipStream_t s) {
    const unsigned rows = (unsigned)a.rows, fours = (rows + 3) / 4;
    // (d_model is at most 8192; the choice goes by it alone: a row's bits do not depend on the others.)  A wavefront per row while it holds the row in 3
    // pieces a lane: no barrier and no idle lanes; against a workgroup per row, bf16, n and post norm and gate: 65536 x 64 29 us for 76, 65536 x 512 50 for 86,
    // 60000 x 1088 97 for 114, 60000 x 1536 126 for 135, 8 rows alike; 4 pieces a lane 30000 x 2048 87 for 90, 6 pieces 30000 x 2880 137 for 127.
    const int pieces = d / 8;
    if (pieces <= 64)
        block_norm_kernel<T, 64, 1><<<fours, NT, 0, s>>>(a, d, eps);
    else if (pieces <= 128)
        block_norm_kernel<T, 64, 2><<<fours, NT, 0, s>>>(a, d, eps);
    else if (pieces <= 192)
        block_norm_kernel<T, 64, 3><<<fours, NT, 0, s>>>(a, d, eps);
    else if (pieces <= 256)
        block_norm_kernel<T, 256, 1><<<rows, NT, 0, s>>>(a, d, eps);
    else if (pieces <= 512)
        block_norm_kernel<T, 256, 2><<<rows, NT, 0, s>>>(a, d, eps);
    else if (pieces <= 768)
        block_norm_kernel<T, 256, 3><<<rows, NT, 0, s>>>(a, d, eps);
    else
        block_norm_kernel<T, 256, 4><<<rows, NT, 0, s>>>(a, d, eps);
}
int launch_block_norm(compact_ctx* ctx, const BlockNormArgs& all, hipStream_t s) {
    const int d = ctx->cfg.d_model;
    const size_t es = dtype_size(ctx->cfg.dtype);
    for (int64_t r = 0; r < all.rows; r += ROWS_PER_LAUNCH) {
        BlockNormArgs a = all;
        a.rows = std::min<int64_t>(all.rows - r, ROWS_PER_LAUNCH);
        auto from = [&](auto*& p, int64_t stride, size_t size) {
            if (p) p = reinterpret_cast<std::decay_t<decltype(p)>>((char*)p + r * stride * size);
        };
        from(a.x, d, es), from(a.b, d, es), from(a.gate, a.gate_stride, es), from(a.h, d, es), from(a.n, d, es), from(a.q, d, 1), from(a.q_scale, 1, 4);
        if (ctx->cfg.dtype == COMPACT_BF16)
            run_block_norm<bf16>(a, d, ctx->cfg.rms_eps, s);
        else
            run_block_norm<float>(a, d, ctx->cfg.rms_eps, s);
        LAUNCH_CHECK(ctx);
    }
    return COMPACT_OK;
}
