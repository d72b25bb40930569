// Products of 8-bit codes:  C[m, n] = a_scale[m] b_scale[n] sum_k A[m, k] B[n, k], the sum in 32-bit integers.  Integer sums are the
// same in any order, so every tile form and every split of K gives the same bits.
#include <algorithm>

#include "common.h"
#include "gemm_ring.h"
#include "vecio.h"

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
    int f32;  // C and R are fp32 rather than bf16
    GroupedArgs g;
};

// what chunks of 16 codes beyond K are read from, on the activations' side
static __device__ const int8_t zero_codes[16] __attribute__((aligned(16))) = {};

struct I8Tile {
    int64_t m0;
    int rows_valid;   // 0: nothing to do
    int n0;
    const int8_t* W;
    const float* ws;
};
template <bool GROUPED, bool GLU, int BM, int OUTN, int GM>
__device__ __forceinline__ I8Tile i8_tile(const GemmI8Params& p) {
    int tm, tn;
    tile_at<GM>(xcd_order(blockIdx.x, gridDim.x), p.n_mtiles, p.n_ntiles, tm, tn);
    I8Tile t;
    t.n0 = tn * OUTN;
    t.W = p.W;
    t.ws = p.ws;
    if (GROUPED) {
        const int e = p.g.tile_expert[tm];
        t.m0 = e < 0 ? 0 : p.g.tile_row0[tm];
        t.rows_valid = e < 0 ? 0 : p.g.tile_rows[tm];
        t.W += (int64_t)max(e, 0) * p.g.b_expert_stride;
        t.ws += (int64_t)max(e, 0) * p.N * (GLU ? 2 : 1);
    } else {
        t.m0 = (int64_t)tm * BM;
        t.rows_valid = (int)min((int64_t)BM, p.M - t.m0);
    }
    return t;
}

// One output from its sums; the same roundings wherever it is computed.
#pragma clang fp contract(off)
__device__ __forceinline__ float i8_value(int sum, float xs, float ws) { return (float)sum * xs * ws; }
__device__ __forceinline__ float i8_glu(float g, float u, bool f32) {
    const float e = f32 ? expf(-g) : __expf(-g);   // (__expf: off by up to 3.4e-6 of the value at g = -80)
    return g / (1.0f + e) * u;
}

// Epilogue of one wavefront: TM x TN MFMA tiles, 16 output rows per pass through a slab of its own [16][WOUT + 4].  acc[i][j][e]: output
// row wrow + i*16 + r of the tile, column n_first + j*16 + c4*4 + e (SwiGLU: the first TN / 2 tiles are the gate, the others
// the up values of the same columns).
template <bool GLU, bool GROUPED, int TM, int TN>
__device__ __forceinline__ void i8_store(const GemmI8Params& p, const I8Tile& tp, const intx4 (&acc)[TM][TN], float* slab, int lane,
                                         int wrow, int n_first) {
    constexpr int TJ = GLU ? TN / 2 : TN, WOUT = TJ * 16, SLD = WOUT + 4;
    constexpr int NCH = WOUT / 8, NU = 16 * NCH / 64 > 0 ? 16 * NCH / 64 : 1;
    const int r = lane & 15, c4 = lane >> 4;
    float ws[TN][4];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = min(n_first + (j % TJ) * 16 + c4 * 4 + e, p.N - 1);
            ws[j][e] = tp.ws[j < TJ ? n : p.N + n];
        }
    const bool wide = p.N % 8 == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (wrow + i * 16 >= tp.rows_valid) break;   // (uniform in the wavefront)
        const int64_t xr = tp.m0 + min(wrow + i * 16 + r, tp.rows_valid - 1);
        const float xs = p.xs[GROUPED && p.g.a_gather ? (int64_t)p.g.a_gather[xr] : xr];
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            floatx4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = i8_value(acc[i][j][e], xs, ws[j][e]);
                if (GLU) v[e] = i8_glu(v[e], i8_value(acc[i][j + TJ][e], xs, ws[j + TJ][e]), p.f32);
            }
            *reinterpret_cast<floatx4*>(slab + r * SLD + j * 16 + c4 * 4) = v;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int row = (lane + 64 * u) / NCH, c = (lane + 64 * u) % NCH;
            const int lm = wrow + i * 16 + row, n = n_first + c * 8;
            if (row >= 16 || lm >= tp.rows_valid || n >= p.N) continue;
            const int64_t o = (tp.m0 + lm) * p.N + n;
            float v[8];
            const floatx4 a = *reinterpret_cast<const floatx4*>(slab + row * SLD + c * 8);
            const floatx4 b = *reinterpret_cast<const floatx4*>(slab + row * SLD + c * 8 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = a[e];
                v[4 + e] = b[e];
            }
            if (GROUPED && p.g.row_scale) {
                const float sc = p.g.row_scale[tp.m0 + lm];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= sc;
            }
            if (wide) {
                if (p.f32) {
                    if (p.R) {
                        float rv[8];
                        load8((const float*)p.R + o, rv);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += rv[e];
                    }
                    store8((float*)p.C + o, v);
                } else {
                    if (p.R) {
                        float rv[8];
                        load8((const bf16*)p.R + o, rv);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += rv[e];
                    }
                    store8((bf16*)p.C + o, v);
                }
            } else {
                for (int e = 0; e < 8 && n + e < p.N; ++e) {
                    if (p.f32)
                        ((float*)p.C)[o + e] = v[e] + (p.R ? ((const float*)p.R)[o + e] : 0.f);
                    else
                        ((bf16*)p.C)[o + e] = (bf16)(v[e] + (p.R ? (float)((const bf16*)p.R)[o + e] : 0.f));
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// BM x BN outputs per workgroup of WM x WN wavefronts, k-tiles of 128 codes in a ring of S LDS stages, one barrier per k-tile, S - 1
// k-tiles of loads in flight.  16-byte direct-to-LDS loads; chunk index XOR-ed with (row / 2) % 8, so that 16 lanes reading a chunk
// of 16 rows touch 16 different groups of banks.  The weight rows are the MFMA rows, the activation rows its columns: a
// lane ends up with 4 consecutive output columns of one row.
template <int BM, int BN, int WM, int WN, int S, bool GLU, bool GROUPED>
__global__ __launch_bounds__(WM* WN * 64) void gemm_i8_tile_kernel(const GemmI8Params p) {
    constexpr int NW = WM * WN, BK = I8_BK;
    constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
    constexpr int STAGE = (BM + BN) * BK;
    constexpr int OUTN = GLU ? BN / 2 : BN, WOUT = GLU ? WTN / 2 : WTN;
    constexpr int XU = BM / 8 / NW, WU = BN / 8 / NW;   // 8-row load units per wavefront
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && (!GLU || TN % 2 == 0), "tile rows must split over the wavefronts");
    static_assert((size_t)NW * 16 * (WOUT + 4) * 4 <= (size_t)S * STAGE, "the epilogue's slabs fit the ring");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const I8Tile tp = i8_tile<GROUPED, GLU, BM, OUTN, 8>(p);
    if (tp.rows_valid <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int r = lane & 15, c4 = lane >> 4;

    const int8_t *xsrc[XU], *wsrc[WU];
    int xc[XU], wc[WU];   // the chunk of a k-tile that the lane loads
#pragma unroll
    for (int u = 0; u < XU; ++u) {
        const int row = (wave * XU + u) * 8 + (lane >> 3);
        int64_t sr = tp.m0 + min(row, tp.rows_valid - 1);
        if (GROUPED && p.g.a_gather) sr = p.g.a_gather[sr];
        xc[u] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        xsrc[u] = p.X + sr * p.K + xc[u];
    }
#pragma unroll
    for (int u = 0; u < WU; ++u) {
        const int row = (wave * WU + u) * 8 + (lane >> 3);
        int n;
        if (GLU)
            n = row < BN / 2 ? min(tp.n0 + row, p.N - 1) : p.N + min(tp.n0 + row - BN / 2, p.N - 1);
        else
            n = min(tp.n0 + row, p.N - 1);
        wc[u] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        wsrc[u] = tp.W + (int64_t)n * p.K + wc[u];
    }
    const int nk = (p.K + BK - 1) / BK;
    auto gload = [&](int kt, int stage) {
        const int k0 = min(kt, nk - 1) * BK;   // past the end: the last k-tile again, into a stage nobody reads
        char* dst = smem + stage * STAGE;
        if (k0 + BK <= p.K) {
#pragma unroll
            for (int u = 0; u < XU; ++u) load16_to_lds(xsrc[u] + k0, dst + (wave * XU + u) * 8 * BK);
#pragma unroll
            for (int u = 0; u < WU; ++u) load16_to_lds(wsrc[u] + k0, dst + BM * BK + (wave * WU + u) * 8 * BK);
        } else {   // chunks beyond K: zeros for the activations, the row's first chunk for the weights
#pragma unroll
            for (int u = 0; u < XU; ++u)
                load16_to_lds(k0 + xc[u] < p.K ? xsrc[u] + k0 : zero_codes, dst + (wave * XU + u) * 8 * BK);
#pragma unroll
            for (int u = 0; u < WU; ++u)
                load16_to_lds(k0 + wc[u] < p.K ? wsrc[u] + k0 : wsrc[u] - wc[u], dst + BM * BK + (wave * WU + u) * 8 * BK);
        }
    };
    intx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    int foff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) foff[kk] = r * BK + (((4 * kk + c4) ^ ((r >> 1) & 7)) << 4);

    for (int i = 0; i < S - 1; ++i) gload(i, i);
    int stage = 0, fill = S - 1;
    for (int kt = 0; kt < nk; ++kt) {
        ring_barrier<(S - 2) * (XU + WU)>();   // k-tile kt has landed; everybody is done with the stage to be refilled
        gload(kt + S - 1, fill);
        const char* xl = smem + stage * STAGE + wm * WTM * BK;
        const char* wl = smem + stage * STAGE + BM * BK;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            intx4 xf[TM], wf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int row = !GLU ? wn * WTN + j * 16
                                : j < TN / 2 ? wn * (WTN / 2) + j * 16
                                             : BN / 2 + wn * (WTN / 2) + (j - TN / 2) * 16;
                wf[j] = *reinterpret_cast<const intx4*>(wl + row * BK + foff[kk]);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = *reinterpret_cast<const intx4*>(xl + i * 16 * BK + foff[kk]);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i], acc[i][j], 0, 0, 0);
        }
        stage = stage + 1 == S ? 0 : stage + 1;
        fill = fill + 1 == S ? 0 : fill + 1;
    }
    ring_barrier<0>();   // the repeated loads must not land in the slabs
    i8_store<GLU, GROUPED, TM, TN>(p, tp, acc, reinterpret_cast<float*>(smem) + wave * 16 * (WOUT + 4), lane, wm * WTM, tp.n0 + wn * WOUT);
}

template <int BM, int BN, int WM, int WN, int S, bool GLU, bool GROUPED>
static int launch_tile(compact_ctx* ctx, GemmI8Params& p, hipStream_t s) {
    constexpr int OUTN = GLU ? BN / 2 : BN;
    if (!GROUPED) p.n_mtiles = (int)((p.M + BM - 1) / BM);
    p.n_ntiles = (p.N + OUTN - 1) / OUTN;
    constexpr size_t smem = (size_t)S * (BM + BN) * I8_BK;
    static_assert(smem <= 64 * 1024, "no attribute needed");
    const int64_t tiles = (int64_t)p.n_mtiles * p.n_ntiles;
    if (tiles == 0) return COMPACT_OK;
    if (tiles > 0x7fffffff) return set_err(ctx, COMPACT_ESHAPE, "too many output tiles");
    gemm_i8_tile_kernel<BM, BN, WM, WN, S, GLU, GROUPED><<<(unsigned)tiles, WM * WN * 64, smem, s>>>(p);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

size_t gemm_i8_workspace(int64_t M, int N, int K, int epilogue) {
    (void)M, (void)N, (void)K, (void)epilogue;
    return 0;
}
int gemm_i8_group_mtile(int64_t rows, int n_experts) {
    (void)rows, (void)n_experts;
    return 64;
}

int launch_gemm_i8(compact_ctx* ctx, const GemmI8Args& a, void* ws, size_t ws_bytes, hipStream_t s) {
    (void)ws, (void)ws_bytes;
    if (a.M == 0) return COMPACT_OK;
    GemmI8Params p{};
    p.X = a.a;
    p.xs = a.a_scale;
    p.W = a.b;
    p.ws = a.b_scale;
    p.R = a.r;
    p.C = a.c;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.f32 = ctx->cfg.dtype == COMPACT_FP32;
    if (a.grouped) {
        p.g = *a.grouped;
        p.n_mtiles = a.grouped->n_mtiles;
        return a.epilogue ? launch_tile<64, 64, 2, 2, 4, true, true>(ctx, p, s) : launch_tile<64, 64, 2, 2, 4, false, true>(ctx, p, s);
    }
    return a.epilogue ? launch_tile<64, 64, 2, 2, 4, true, false>(ctx, p, s) : launch_tile<64, 64, 2, 2, 4, false, false>(ctx, p, s);
}
