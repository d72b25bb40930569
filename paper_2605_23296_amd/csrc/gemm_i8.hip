// Products of 8-bit codes:  C[m, n] = a_scale[m] b_scale[n] sum_k A[m, k] B[n, k], the sum in 32-bit integers.  Integer sums are the
// same in any order, so every tile form and every split of K gives the same bits, and the choice may look at the number of rows.
//
//  * v_mfma_i32_16x16x64_i8 takes the 16 clocks and the 16 bytes a lane of its bf16 sibling of half the depth: a k-tile is 128 codes, a
//    128-byte line of either operand, and the tiles, rings and phases are those of the bf16 products, k-tile for k-tile.  So is the rule that
//    picks a form: it is asked for K / 2 elements of 2 bytes (it was within 3 % of the best of the seven forms at 22 of 23 sizes looked at, N 4096 .. 14336, K 2880 ..
//    14336, 17 .. 32768 rows, and 8 % off at 2 * 14336 x 4096 with 17 rows: 29.8 us, 27.5 in 64 x 64 tiles);
//  * at most 16 rows, and up to 48 of few columns: gemv_i8.hip; 64 x 64 tiles that leave half of the chip idle, and a long K: slices of K, added up by a second launch;
//  * chunks beyond K (K % 128 != 0) are zeros on the activations' side; N and the rows are clamped in the loads and checked at the stores;
//  * per-row and per-column scales reach LDS with the first loads of a tile.  Read where they are used they cost two trips to memory, one
//    after the other, for every 16 rows: 2 * 14336 x 4096 at 32768 rows 3079 -> 2820 us, experts of 16384 rows 2755 -> 2508.
// Bound: large products run at the chip's power limit (1.85 GHz of 2.4; codes that are all zero: 2393 us instead of 2850), matrix pipes 70 % busy; 2.7 POP/s for
// 2 * 14336 x 4096 at 32768 rows (64 x 64 tiles alone 5881 us), 2.9 for N 4096 K 14336 at 16384 rows, 22 us for N 5120 K 2880 at 1001 rows.  A tile has
// 8 to 10 us beside its k-tiles (1.3 us each): starting the next tile's loads before this one's outputs are written hides 4 of them, but
// takes the registers and the free order of workgroups: 1.006 of the time for the first, 0.987 for experts of 16384 rows, 1.03 .. 1.06 for fewer, so it is not done.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "gemm_i8.h"
#include "gemm_ring.h"
#include "vecio.h"

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
    I8Tile t;
    t.rows_valid = 0;
    // the map's tiles with work alone are dealt out: the others are the last ones, and would be one XCD's whole share
    const int n_mtiles = GROUPED ? *p.g.n_live : p.n_mtiles, n = GROUPED ? n_mtiles * p.n_ntiles : gridDim.x;
    if (GROUPED && (int)blockIdx.x >= n) return t;
    tile_at<GM>(xcd_order(blockIdx.x, n), n_mtiles, p.n_ntiles, tm, tn);
    t.n0 = tn * OUTN;
    t.W = p.W;
    t.ws = p.ws;
    if (GROUPED) {
        const int e = p.g.tile_expert[tm];
        t.m0 = p.g.tile_row0[tm];
        t.rows_valid = p.g.tile_rows[tm];
        t.W += (int64_t)e * p.g.b_expert_stride;
        t.ws += (int64_t)e * p.N * (GLU ? 2 : 1);
    } else {
        t.m0 = (int64_t)tm * BM;
        t.rows_valid = (int)min((int64_t)BM, p.M - t.m0);
    }
    return t;
}

// The scales of a workgroup's rows and columns (and the factors of the rows) on their way to LDS, at the start: [BM] rows, [BN] weight rows of
// the tile, [BM] factors.  They are older than the ring's loads and so have landed by its first barrier; read at the end, each
// would be two trips to memory, one after the other, for every 16 rows.
template <int BM, int BN, bool GLU, bool GROUPED>
__device__ __forceinline__ void i8_load_scales(const GemmI8Params& p, const I8Tile& tp, char* sc, int wave, int lane) {
    constexpr int UX = BM / 64, UW = BN / 64;
    auto unit = [&](int u) __attribute__((always_inline)) {
        char* dst = sc + u * 256;
        if (u < UX || u >= UX + UW) {
            const int64_t row = tp.m0 + min((u < UX ? u : u - UX - UW) * 64 + lane, tp.rows_valid - 1);
            if (u < UX)
                load4_to_lds(p.xs + (GROUPED && p.g.a_gather ? (int64_t)p.g.a_gather[row] : row), dst);
            else
                load4_to_lds(p.g.row_scale + row, dst);
        } else {
            const int c = (u - UX) * 64 + lane;
            const int n = !GLU ? min(tp.n0 + c, p.N - 1) : c < BN / 2 ? min(tp.n0 + c, p.N - 1) : p.N + min(tp.n0 + c - BN / 2, p.N - 1);
            load4_to_lds(tp.ws + n, dst);
        }
    };
    const int units = UX + UW + (GROUPED && p.g.row_scale ? UX : 0);
    for (int u = wave; u < units; u += blockDim.x / 64) unit(u);
}

// Epilogue of one wavefront: TM x TN MFMA tiles, 16 output rows per pass through a slab of its own [16][WOUT + 4].  acc[i][j][e]: output
// row wrow + i*16 + r of the tile, column wcol + j*16 + c4*4 + e of it (SwiGLU: the first TN / 2 tiles are the gate, the others
// the up values of the same columns).  sc: the scales in LDS.
template <int BM, int BN, bool GLU, bool GROUPED, int TM, int TN>
__device__ __forceinline__ void i8_store(const GemmI8Params& p, const I8Tile& tp, const intx4 (&acc)[TM][TN], float* slab, const float* sc,
                                         int lane, int wrow, int wcol) {
    constexpr int TJ = GLU ? TN / 2 : TN, WOUT = TJ * 16, SLD = WOUT + 4;
    constexpr int NCH = WOUT / 8, NU = 16 * NCH / 64 > 0 ? 16 * NCH / 64 : 1;
    const int r = lane & 15, c4 = lane >> 4, n_first = tp.n0 + wcol;
    const float* gates = sc + BM + BN;
    floatx4 ws[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j)
        ws[j] = *reinterpret_cast<const floatx4*>(sc + BM + (j < TJ ? 0 : BN / 2) + wcol + (j % TJ) * 16 + c4 * 4);
    const bool wide = p.N % 8 == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (wrow + i * 16 >= tp.rows_valid) break;   // (uniform in the wavefront)
        const float xs = sc[wrow + i * 16 + r];
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
        // (rows that are not aligned: an element a lane, neighbours side by side, B of them at a time; with 8 neighbours a lane 8192 x 4100 K 4096 took
        // 175 us for 150, 221 for 178 with a residual, fp32 201 for 150, 255 for 181)
        constexpr int B = WOUT / 4 < 8 ? WOUT / 4 : 8;
        const int64_t own = (tp.m0 + wrow + i * 16) * p.N + n_first;
        for (int u0 = 0; u0 < (wide || n_first >= p.N ? 0 : WOUT / 4); u0 += B) {
            float v[B];
            int64_t o[B];
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const int row = (lane + 64 * (u0 + u)) / WOUT, c = (lane + 64 * (u0 + u)) % WOUT;
                const int lm = wrow + i * 16 + row, n = n_first + c;
                o[u] = lm < tp.rows_valid && n < p.N ? (tp.m0 + lm) * p.N + n : -1;
                v[u] = slab[row * SLD + c];
                if (GROUPED && p.g.row_scale) v[u] *= gates[lm];
            }
            if (p.R) {   // (all requested before the first is used; where there is nothing to add, the slab's first element)
                float rv[B];
                if (p.f32) {
#pragma unroll
                    for (int u = 0; u < B; ++u) rv[u] = ((const float*)p.R)[o[u] < 0 ? own : o[u]];
                } else {
#pragma unroll
                    for (int u = 0; u < B; ++u) rv[u] = (float)((const bf16*)p.R)[o[u] < 0 ? own : o[u]];
                }
#pragma unroll
                for (int u = 0; u < B; ++u) v[u] += rv[u];
            }
#pragma unroll
            for (int u = 0; u < B; ++u) {
                if (o[u] < 0) continue;
                if (p.f32)
                    ((float*)p.C)[o[u]] = v[u];
                else
                    ((bf16*)p.C)[o[u]] = (bf16)v[u];
            }
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int row = (lane + 64 * u) / NCH, c = (lane + 64 * u) % NCH;
            const int lm = wrow + i * 16 + row, n = n_first + c * 8;
            if (!wide || row >= 16 || lm >= tp.rows_valid || n >= p.N) continue;
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
                const float f = gates[lm];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= f;
            }
            float rv[8];
            if (p.R) {
                if (p.f32)
                    load8((const float*)p.R + o, rv);
                else
                    load8((const bf16*)p.R + o, rv);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += rv[e];
            }
            if (p.f32)
                store8((float*)p.C + o, v);
            else
                store8((bf16*)p.C + o, v);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Sums of a k-slice as they are: [slice][row][N, SwiGLU: 2N].
template <bool GLU, int TM, int TN>
__device__ __forceinline__ void i8_store_sums(const GemmI8Params& p, const I8Tile& tp, const intx4 (&acc)[TM][TN], int lane, int wrow,
                                              int n_first) {
    constexpr int TJ = GLU ? TN / 2 : TN;
    const int r = lane & 15, c4 = lane >> 4, cols = GLU ? 2 * p.N : p.N;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int lm = wrow + i * 16 + r;
        if (lm >= tp.rows_valid) continue;
        int* row = p.sums + ((int64_t)blockIdx.y * p.M + tp.m0 + lm) * cols;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int n = n_first + (j % TJ) * 16 + c4 * 4, at = j < TJ ? n : p.N + n;
            if (n + 4 <= p.N && p.N % 4 == 0) {
                *reinterpret_cast<intx4*>(row + at) = acc[i][j];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < p.N) row[at + e] = acc[i][j][e];
            }
        }
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
    char* const sc = smem + S * STAGE;
    i8_load_scales<BM, BN, GLU, GROUPED>(p, tp, sc, wave, lane);
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
    // gridDim.y slices of K (partial sums): this workgroup's k-tiles
    const int n_k = (p.K + BK - 1) / BK, k_lo = n_k * blockIdx.y / gridDim.y, nk = n_k * (blockIdx.y + 1) / gridDim.y - k_lo;
    auto gload = [&](int kt, int stage) {
        const int k0 = (k_lo + min(kt, nk - 1)) * BK;   // past the end: the last k-tile again, into a stage nobody reads
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
    if (gridDim.y > 1) {
        i8_store_sums<GLU, TM, TN>(p, tp, acc, lane, wm * WTM, tp.n0 + wn * WOUT);
        wait_all_memory();   // nor must they land in LDS that is another workgroup's by then
        return;
    }
    ring_barrier<0>();   // the repeated loads must not land in the slabs
    i8_store<BM, BN, GLU, GROUPED, TM, TN>(p, tp, acc, reinterpret_cast<float*>(smem) + wave * 16 * (WOUT + 4), reinterpret_cast<const float*>(sc), lane,
                                           wm * WTM, wn * WOUT);
}

// Sums of k-slices -> outputs, 4 columns a thread; the slices' sums (8 at most) are all requested before the first is used.
template <bool GLU>
__global__ __launch_bounds__(256) void gemm_i8_finish_kernel(const GemmI8Params p, int slices) {
    const int cols = GLU ? 2 * p.N : p.N;
    const int n = (blockIdx.x * 256 + threadIdx.x) * 4;
    const int64_t m = blockIdx.y;
    if (n >= p.N) return;
    const float xs = p.xs[m];
    intx4 g = intx4{0, 0, 0, 0}, u = g;
    const int* first = p.sums + m * cols + n;
    if (p.N % 4 == 0) {
        intx4 gv[8], uv[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int* row = first + (int64_t)min(s, slices - 1) * p.M * cols;
            gv[s] = *reinterpret_cast<const intx4*>(row);
            if (GLU) uv[s] = *reinterpret_cast<const intx4*>(row + p.N);
        }
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s < slices) {
                g += gv[s];
                if (GLU) u += uv[s];
            }
    } else {
        for (int s = 0; s < slices; ++s) {
            const int* row = first + (int64_t)s * p.M * cols;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < p.N) {
                    g[e] += row[e];
                    if (GLU) u[e] += row[p.N + e];
                }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) {
            float v = i8_value(g[e], xs, p.ws[n + e]);
            if (GLU) v = i8_glu(v, i8_value(u[e], xs, p.ws[p.N + n + e]), p.f32);
            i8_put(p, m * p.N + n + e, v);
        }
}

template <int BM, int BN, int WM, int WN, int S, bool GLU, bool GROUPED>
static int launch_tile(compact_ctx* ctx, GemmI8Params& p, hipStream_t s, int slices = 1) {
    constexpr int OUTN = GLU ? BN / 2 : BN;
    if (!GROUPED) p.n_mtiles = (int)((p.M + BM - 1) / BM);
    p.n_ntiles = (p.N + OUTN - 1) / OUTN;
    constexpr size_t smem = (size_t)S * (BM + BN) * I8_BK + (2 * BM + BN) * 4;
    static std::atomic<uint64_t> lds_set{0};
    TRY(allow_lds(ctx, (const void*)gemm_i8_tile_kernel<BM, BN, WM, WN, S, GLU, GROUPED>, smem, lds_set));
    const int64_t tiles = (int64_t)p.n_mtiles * p.n_ntiles;
    if (tiles == 0) return COMPACT_OK;
    if (tiles * WM * WN * 64 > MAX_GRID_THREADS) return set_err(ctx, COMPACT_ESHAPE, "too many output tiles");
    gemm_i8_tile_kernel<BM, BN, WM, WN, S, GLU, GROUPED><<<dim3((unsigned)tiles, (unsigned)slices), WM * WN * 64, smem, s>>>(p);
    LAUNCH_CHECK(ctx);
    if (slices > 1) {
        gemm_i8_finish_kernel<GLU><<<dim3((unsigned)((p.N + 1023) / 1024), (unsigned)p.M), 256, 0, s>>>(p, slices);
        LAUNCH_CHECK(ctx);
    }
    return COMPACT_OK;
}

// ---------------------------------------------------------------------------
// 256 x 256 outputs per workgroup, 8 wavefronts of 128 x 64.  The k-tiles pass through LDS as half tiles of 128 rows (16 KB), a ring of
// eight; a k-tile is four phases, one per quarter of the wavefront's output: read the half tile that the quarter needs newly (X0, W1,
// X1, then W0 of the next k-tile; the other operand is still in registers), request one half tile seven phases ahead, join a
// barrier, run 16 MFMAs, join a barrier.  The two wavefronts of a SIMD belong to groups that run half a phase apart, so that
// one's MFMAs cover the other's reads and requests; barriers wait for LDS reads and for all but the newest 12 loads.
// ---------------------------------------------------------------------------
#define LARGE_RING (9 * 128 * I8_BK)   // bytes: the ring of either kind of tile, the scales behind it
typedef std::integral_constant<int, 0> I0;
typedef std::integral_constant<int, 1> I1;
typedef std::integral_constant<int, 2> I2;
typedef std::integral_constant<int, 3> I3;

// 16 MFMAs of 64 x 32 outputs over 128 codes
template <int I, int J, int TM, int TN>
__device__ __forceinline__ void i8_mfmas(intx4 (&acc)[TM][TN], const intx4 (&xf)[4][2], const intx4 (&wf)[2][2]) {
    wave_priority_high();
#pragma unroll
    for (int n = 0; n < 16; ++n) {
        const int kk = n >> 3, mt = (n >> 1) & 3, nt = (n & 1) ^ (mt & 1);
        acc[4 * I + mt][2 * J + nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[nt][kk], xf[mt][kk], acc[4 * I + mt][2 * J + nt], 0, 0, 0);
    }
    wave_priority_normal();
    plain_barrier();
}

// CUT: K is no multiple of 128.  Where a lane reads its 16 codes of the last k-tile then: chunks beyond K are zeros on the activations' side, the row's first
// chunk on the weights'.  Called once, before the first load of that k-tile: no load is of another one after it.
__device__ __forceinline__ void i8_cut(const int8_t*& src, int chunk, int k_last, int K, bool is_x) {
    if (k_last + chunk >= K) src = (is_x ? zero_codes : src - chunk) - k_last;
}

template <bool GLU, bool GROUPED, bool CUT>
__device__ __forceinline__ void i8_tile_256(const GemmI8Params& p, const I8Tile& tp, char* smem) {
    constexpr int WN = 4, BK = I8_BK, WTM = 128, WTN = 64, TM = WTM / 16, TN = WTN / 16, HT = 128 * BK;
    constexpr int WOUT = GLU ? WTN / 2 : WTN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int r = lane & 15, c4 = lane >> 4;
    char* const sc = smem + LARGE_RING;
    i8_load_scales<256, 256, GLU, GROUPED>(p, tp, sc, wave, lane);

    // Half tiles q = 0: W0, 1: X0, 2: W1, 3: X1 (the order they are read in).  Half i of X holds tile rows wm * 128 + i * 64 + .., half j of W
    // the columns wn * 64 + j * 32 + .. of every wavefront (SwiGLU: half 0 the gate rows, half 1 the up rows of the same columns).  One
    // instruction of a wavefront fills 1 KB = 8 rows of 8 chunks, lane l at (row l / 8, position l % 8).
    const int8_t* src[4][2];
    int chunk[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int row = (wave * 2 + u) * 8 + (lane >> 3);   // row of the half tile
        chunk[u] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int64_t sr = tp.m0 + min((row >> 6) * 128 + i * 64 + (row & 63), tp.rows_valid - 1);
            if (GROUPED && p.g.a_gather) sr = p.g.a_gather[sr];
            src[1 + 2 * i][u] = p.X + sr * p.K + chunk[u];
            const int n = GLU ? min(tp.n0 + row, p.N - 1) + i * p.N : min(tp.n0 + (row >> 5) * 64 + i * 32 + (row & 31), p.N - 1);
            src[2 * i][u] = tp.W + (int64_t)n * p.K + chunk[u];
        }
    }
    intx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    const int nk = (p.K + BK - 1) / BK;
    int foff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) foff[kk] = r * BK + (((4 * kk + c4) ^ ((r >> 1) & 7)) << 4);
    const char* xs = smem + wm * 64 * BK;
    const char* ws = smem + wn * 32 * BK;

    auto gload = [&](auto qtag, int kt, int buf) __attribute__((always_inline)) {
        constexpr int q = decltype(qtag)::value;
        char* dst = smem + (buf * 4 + q) * HT + wave * 2 * 8 * BK;
        load16_to_lds(src[q][0] + kt * BK, dst);
        load16_to_lds(src[q][1] + kt * BK, dst + 8 * BK);
    };
    auto cut = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int u = 0; u < 2; ++u) i8_cut(src[q][u], chunk[u], (nk - 1) * BK, p.K, q % 2 == 1);
    };
    intx4 xf[4][2];
    auto read_w = [&](auto jtag, int buf, intx4 (&f)[2][2]) __attribute__((always_inline)) {
        constexpr int q = 2 * decltype(jtag)::value;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) f[nt][kk] = *reinterpret_cast<const intx4*>(ws + (buf * 4 + q) * HT + nt * 16 * BK + foff[kk]);
    };
    auto read_x = [&](auto itag, int buf) __attribute__((always_inline)) {
        constexpr int q = 1 + 2 * decltype(itag)::value;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) xf[mt][kk] = *reinterpret_cast<const intx4*>(xs + (buf * 4 + q) * HT + mt * 16 * BK + foff[kk]);
    };
    // One k-tile = four phases (X0 W0, X0 W1, X1 W1, X1 W0); wa holds W0 of this tile, wb receives W1 and then W0 of the next.  Past the end of
    // K the last k-tile is loaded again, into slots nobody reads.
    auto k_tile = [&](int kt, int buf, intx4 (&wa)[2][2], intx4 (&wb)[2][2]) __attribute__((always_inline)) {
        const int kn = min(kt + 2, nk - 1);
        if (CUT && kt + 2 == nk - 1) cut();
        read_x(I0{}, buf);
        gload(I0{}, kn, buf);
        ring_barrier<12>();
        i8_mfmas<0, 0>(acc, xf, wa);
        read_w(I1{}, buf, wb);
        gload(I1{}, kn, buf);
        ring_barrier<12>();
        i8_mfmas<0, 1>(acc, xf, wb);
        read_x(I1{}, buf);
        gload(I2{}, kn, buf);
        ring_barrier<12>();
        i8_mfmas<1, 1>(acc, xf, wb);
        read_w(I0{}, buf ^ 1, wb);
        gload(I3{}, kn, buf);
        ring_barrier<12>();
        i8_mfmas<1, 0>(acc, xf, wa);
    };
    // all half tiles of k-tiles 0 and 1; W0 and X0 of k-tile 0 have landed when all but 12 loads have
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (CUT && i == nk - 1) cut();
        gload(I0{}, min(i, nk - 1), i);
        gload(I1{}, min(i, nk - 1), i);
        gload(I2{}, min(i, nk - 1), i);
        gload(I3{}, min(i, nk - 1), i);
    }
    intx4 wA[2][2], wB[2][2];
    ring_barrier<12>();
    read_w(I0{}, 0, wA);
    ring_barrier<12>();
    if (wm) plain_barrier();   // the second group of wavefronts runs half a phase behind the first
    int kt = 0;
    for (; kt + 1 < nk; kt += 2) {
        k_tile(kt, 0, wA, wB);
        k_tile(kt + 1, 1, wB, wA);
    }
    if (kt < nk) k_tile(kt, 0, wA, wB);
    if (!wm) plain_barrier();
    ring_barrier<0>();   // the repeated loads of the last k-tile must not land in the slabs
    i8_store<256, 256, GLU, GROUPED, TM, TN>(p, tp, acc, reinterpret_cast<float*>(smem) + wave * 16 * (WOUT + 4), reinterpret_cast<const float*>(sc), lane,
                                             wm * WTM, wn * WOUT);
}

// The same schedule over 128 x 256 tiles (wavefronts of 64 x 64, two phases per k-tile: X0 W0, X0 W1).  A k-tile is three half tiles (W0,
// X0, W1); the ring holds three k-tiles (nine slots, 144 KB).  A phase requests three of the six 8-row pieces that a wavefront owns of
// a k-tile; 11 or 12 of them may still fly when the next phase's operands must be there.
template <bool GLU, bool GROUPED, bool CUT>
__device__ __forceinline__ void i8_tile_128(const GemmI8Params& p, const I8Tile& tp, char* smem) {
    constexpr int WN = 4, BK = I8_BK, WTM = 64, WTN = 64, TM = WTM / 16, TN = WTN / 16, HT = 128 * BK;
    constexpr int WOUT = GLU ? WTN / 2 : WTN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int r = lane & 15, c4 = lane >> 4;
    char* const sc = smem + LARGE_RING;
    i8_load_scales<128, 256, GLU, GROUPED>(p, tp, sc, wave, lane);
    const int8_t* src[3][2];   // half tiles q = 0: W0, 1: X0, 2: W1
    int chunk[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int row = (wave * 2 + u) * 8 + (lane >> 3);
        chunk[u] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        int64_t sr = tp.m0 + min(row, tp.rows_valid - 1);
        if (GROUPED && p.g.a_gather) sr = p.g.a_gather[sr];
        src[1][u] = p.X + sr * p.K + chunk[u];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = GLU ? min(tp.n0 + row, p.N - 1) + j * p.N : min(tp.n0 + (row >> 5) * 64 + j * 32 + (row & 31), p.N - 1);
            src[2 * j][u] = tp.W + (int64_t)n * p.K + chunk[u];
        }
    }
    intx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    const int nk = (p.K + BK - 1) / BK;
    int foff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) foff[kk] = r * BK + (((4 * kk + c4) ^ ((r >> 1) & 7)) << 4);
    const char* xs = smem + wm * 64 * BK;
    const char* ws = smem + wn * 32 * BK;
    // piece u of half tile q of k-tile kt (past the end: the last one again), into k-tile buffer buf
    auto gload = [&](int q, int u, int kt, int buf) __attribute__((always_inline)) {
        load16_to_lds(src[q][u] + min(kt, nk - 1) * BK, smem + (buf * 3 + q) * HT + (wave * 2 + u) * 8 * BK);
    };
    auto cut = [&](int q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) i8_cut(src[q][u], chunk[u], (nk - 1) * BK, p.K, q == 1);
    };
    auto read_w = [&](int j, int buf, intx4 (&f)[2][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) f[nt][kk] = *reinterpret_cast<const intx4*>(ws + (buf * 3 + 2 * j) * HT + nt * 16 * BK + foff[kk]);
    };
    intx4 xf[4][2], w0[2][2], w1[2][2];
    // k-tile kt in buffer b0, kt + 1 in b1, kt + 2 in b2
    auto k_tile = [&](int kt, int b0, int b1, int b2) __attribute__((always_inline)) {
        if (CUT && kt + 2 == nk - 1) cut(2);
        if (CUT && kt + 3 == nk - 1) {
            cut(0);
            cut(1);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) xf[mt][kk] = *reinterpret_cast<const intx4*>(xs + (b0 * 3 + 1) * HT + mt * 16 * BK + foff[kk]);
        gload(2, 0, kt + 2, b2);
        gload(2, 1, kt + 2, b2);
        gload(0, 0, kt + 3, b0);
        ring_barrier<11>();
        i8_mfmas<0, 0>(acc, xf, w0);
        read_w(1, b0, w1);
        read_w(0, b1, w0);
        gload(0, 1, kt + 3, b0);
        gload(1, 0, kt + 3, b0);
        gload(1, 1, kt + 3, b0);
        ring_barrier<12>();
        i8_mfmas<0, 1>(acc, xf, w1);
    };
    // k-tiles 0 and 1, and W0, X0 of k-tile 2; the first two half tiles have landed when all but 12 pieces have
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int q = 0; q < (i == 2 ? 2 : 3); ++q) {
            if (CUT && i == nk - 1) cut(q);
            gload(q, 0, i, i);
            gload(q, 1, i, i);
        }
    ring_barrier<12>();
    read_w(0, 0, w0);
    ring_barrier<12>();
    if (wm) plain_barrier();   // the second group of wavefronts runs half a phase behind the first
    int kt = 0;
    for (; kt + 2 < nk; kt += 3) {
        k_tile(kt, 0, 1, 2);
        k_tile(kt + 1, 1, 2, 0);
        k_tile(kt + 2, 2, 0, 1);
    }
    if (kt < nk) k_tile(kt, 0, 1, 2);
    if (kt + 1 < nk) k_tile(kt + 1, 1, 2, 0);
    if (!wm) plain_barrier();
    ring_barrier<0>();   // the repeated loads must not land in the slabs
    i8_store<128, 256, GLU, GROUPED, TM, TN>(p, tp, acc, reinterpret_cast<float*>(smem) + wave * 16 * (WOUT + 4), reinterpret_cast<const float*>(sc), lane,
                                             wm * WTM, wn * WOUT);
}

// Plain products: the output is cut into slots of 256 x 256, in groups of 4 row tiles per column tile (6 and 8: 0.98 .. 1.03 of the time, the most for
// K 14336); the first n_full of them are a
// workgroup each, the others two workgroups of 128 x 256, and last come the halves of a bottom row tile of at most 128 rows.  Routed
// products: a workgroup per tile of the map, in the form that its rows need.
template <bool GLU, bool GROUPED, bool CUT>
__global__ __launch_bounds__(512) void gemm_i8_kernel(const GemmI8Params p) {
    constexpr int OUTN = GLU ? 128 : 256;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    if constexpr (GROUPED) {
        // groups of 2 row tiles per column tile: a third one is another expert's as often as not (groups of 4 / 6 / 8: experts of 16384
        // rows 2265 / 2238 / 2233 us, 2207 so; of 512 rows, in tiles of 128, 8: 695, 672 so)
        const I8Tile tp = i8_tile<true, GLU, 256, OUTN, 2>(p);
        if (tp.rows_valid <= 0) return;
        if (tp.rows_valid > 128)
            i8_tile_256<GLU, true, CUT>(p, tp, smem);
        else
            i8_tile_128<GLU, true, CUT>(p, tp, smem);
    } else {
        const int i = blockIdx.x;
        int tm, tn;
        I8Tile tp;
        tp.W = p.W;
        tp.ws = p.ws;
        if (i < p.n_full) {
            tile_at<4>(xcd_order(i, p.n_full), p.n_mtiles, p.n_ntiles, tm, tn);
            tp.m0 = (int64_t)tm * 256;
            tp.n0 = tn * OUTN;
            tp.rows_valid = (int)min((int64_t)256, p.M - tp.m0);
            i8_tile_256<GLU, false, CUT>(p, tp, smem);
        } else {
            const int h = xcd_order(i - p.n_full, gridDim.x - p.n_full);
            const int slot = p.n_full + h / 2, slots = p.n_mtiles * p.n_ntiles;
            if (slot < slots) {
                tile_at<4>(slot, p.n_mtiles, p.n_ntiles, tm, tn);
                tp.m0 = (int64_t)tm * 256 + (h & 1) * 128;
            } else {
                tn = h - 2 * (slots - p.n_full);
                tp.m0 = (int64_t)p.n_mtiles * 256;
            }
            tp.n0 = tn * OUTN;
            tp.rows_valid = (int)min((int64_t)128, p.M - tp.m0);
            i8_tile_128<GLU, false, CUT>(p, tp, smem);
        }
    }
}

template <bool GLU, bool GROUPED, bool CUT>
static int launch_large_k(compact_ctx* ctx, GemmI8Params& p, int64_t n_full, hipStream_t s) {
    constexpr int OUTN = GLU ? 128 : 256;
    constexpr size_t smem = LARGE_RING + 3 * 256 * 4;   // the epilogue's slabs fit in
    static_assert((size_t)8 * 16 * (OUTN / 4 + 4) * sizeof(float) <= smem, "the epilogue's slabs fit the ring");
    static std::atomic<uint64_t> lds_set{0};
    TRY(allow_lds(ctx, (const void*)gemm_i8_kernel<GLU, GROUPED, CUT>, smem, lds_set));
    p.n_ntiles = (p.N + OUTN - 1) / OUTN;
    int64_t wgs;
    if (GROUPED) {
        wgs = (int64_t)p.n_mtiles * p.n_ntiles;
    } else {
        const LargeTiles lt = large_tiles(p.M, p.n_ntiles);
        p.n_mtiles = (int)(lt.slots / p.n_ntiles);
        p.n_full = (int)std::min(n_full, lt.slots);
        wgs = p.n_full + 2 * (lt.slots - p.n_full) + lt.bottom;
    }
    if (wgs == 0) return COMPACT_OK;
    if (wgs * 512 > MAX_GRID_THREADS) return set_err(ctx, COMPACT_ESHAPE, "too many output tiles");
    gemm_i8_kernel<GLU, GROUPED, CUT><<<dim3((unsigned)wgs), 512, smem, s>>>(p);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}
// (a branch for the cut k-tile costs products without one 3 %)
template <bool GLU, bool GROUPED>
static int launch_large(compact_ctx* ctx, GemmI8Params& p, int64_t n_full, hipStream_t s) {
    return p.K % I8_BK ? launch_large_k<GLU, GROUPED, true>(ctx, p, n_full, s) : launch_large_k<GLU, GROUPED, false>(ctx, p, n_full, s);
}

template <bool GLU, bool GROUPED>
static int launch_form(compact_ctx* ctx, int form, int64_t n_full, GemmI8Params& p, hipStream_t s, int slices = 1) {
    switch (form) {
        case TILE_256: return launch_large<GLU, GROUPED>(ctx, p, n_full, s);
        case TILE_128: return launch_large<GLU, GROUPED>(ctx, p, 0, s);
        case TILE_64_128: return launch_tile<64, 128, 2, 4, 6, GLU, GROUPED>(ctx, p, s, slices);
        default: break;
    }
    if constexpr (!GROUPED) {
        switch (form) {
            case TILE_128_128: return launch_tile<128, 128, 2, 4, 4, GLU, false>(ctx, p, s, slices);
            case TILE_128_64: return launch_tile<128, 64, 4, 2, 6, GLU, false>(ctx, p, s, slices);
            case TILE_64_64: return launch_tile<64, 64, 2, 2, 4, GLU, false>(ctx, p, s, slices);
            default: break;
        }
    }
    return set_err(ctx, COMPACT_EINVAL, "unknown GEMM tile");
}

// (Both rules count in the 256 compute units of the whole chip, not in those of the device at hand: the workspace's size goes by them, and is asked for where there may be none.)
// Slices of K for products whose 64 x 64 tiles leave half of the chip idle and more: as many as fill it, of 8 k-tiles at least, and
// from K 5120 on (the second launch, which adds the slices up, costs 3 us, and the caller's thread 1 more).  Whole and in 2, 3, 4, 5 slices, us:
//  * 64 rows: N 4096 K 4096 12.0, 11.9, 11.8, 11.1, 13.7 (N 2048 at 128 rows 10.1, 11.1, 10.6, 10.8); K 5120 15.6, 13.8, 12.6, 12.1; K 8192 20.7, 16.4, 14.4, 13.1,
//    16.7; K 14336 36 whole, 19.2 in 4, 24 in 6;
//  * N 2048 at 64 rows: K 4096 9.9, 10.6, 9.6, 9.2, 9.5, K 6144 16.2, 13.4, 11.3, 10.7, 10.3; N 1024 K 14336 32.6 whole, 16.0 in 4, 14.6 in 8;
//  * 128 tiles: N 4096 at 128 rows, K 4096 12.1, 13.0, K 5120 15.4, 15.1, K 6144 16.6, 15.1.
static int64_t gemm_i8_small_tiles(int64_t M, int N, int epilogue) { return (M + 63) / 64 * ((N + (epilogue ? 31 : 63)) / (epilogue ? 32 : 64)); }
static int gemm_i8_slices(int64_t M, int N, int K, int epilogue) {
    const int64_t tiles = gemm_i8_small_tiles(M, N, epilogue);
    const int k_tiles = (K + I8_BK - 1) / I8_BK;
    if (tiles > 128 || k_tiles < 40) return 1;
    return (int)std::min<int64_t>({256 / tiles, k_tiles / 8, 8});
}
// Whether 17 to 48 rows are a weight stream (gemv_i8.hip; M at most 16 always is), rather than 64 x 64 tiles, in slices of K if it is long.  Every workgroup of
// the stream reads all activations, at its compute unit's pace; slices are a second launch.  The stream's time, the other's = 1, at 17 / 32 / 33 / 48 rows:
//  * short K: N 2880 K 2880 0.88 / 0.88 / 0.88 / 0.90, 5120 x 2880 0.89 / 0.88 / 0.98 / 1.03, SwiGLU 4096 x 2048 0.98 / 0.97 / 1.05 / 1.06;
//  * longer ones: 512 x 4096 0.7, 6144 x 4096 0.81 / 0.83 / 0.90 / 0.90, 8192 x 4096 0.83 / 0.84 / 0.91 / 0.91, 1024 x 8192 0.70 / 0.75 / 0.84 / 0.89, 4096 x 8192
//    0.87 / 0.91 / 0.97 / 1.04, 8192 x 14336 0.92 / 0.97 / 1.01 / 1.03, 4096 x 14336 0.93 / 1.06 / 1.0 / 1.0, 2048 x 28672 1.3 and more;
//  * 64 rows: 0.80 (512 x 4096) .. 1.18 (5120 x 2880).
static bool gemm_i8_streams(int64_t M, int N, int K, int epilogue) {
    if (M <= I8_STREAM_ROWS) return true;
    const int64_t tiles = gemm_i8_small_tiles(M, N, epilogue);
    if (M > I8_STREAM_ROWS_MOST || tiles > 128) return false;
    if (K < 4096) return M <= 32 || tiles <= 64;
    // bytes that a workgroup reads for a column tile, its weight rows and the activations that are staged: the other way's second launch pays from some 400 KB on
    return (int64_t)(16 + (M <= 32 ? 32 : 48)) * K <= 400000;
}
size_t gemm_i8_workspace(int64_t M, int N, int K, int epilogue) {
    const int slices = gemm_i8_streams(M, N, K, epilogue) ? 1 : gemm_i8_slices(M, N, K, epilogue);
    return slices < 2 ? 0 : (size_t)slices * M * N * (epilogue ? 2 : 1) * sizeof(int);
}
int gemm_i8_group_mtile(int64_t rows, int n_experts, int F, int d, int n_cus) {
    // up to 9 rows an expert on average the weight stream, whose tiles of 16 rows read the weights again beyond that: 128 experts of 2880 x 2880 with 8 / 9 / 10 / 12 rows
    // each 578 / 602 / 635 / 686 us, in tiles 600 / 605 / 617 / 633; 64 of 1024 x 1408 with 7.5 / 9 / 12 rows 77 / 79 / 88, 72 / 73 / 79
    if (rows <= 9 * n_experts) return I8_STREAM_ROWS;
    const int mtile = gemm_bf16_group_mtile(rows, n_experts, F, d / 2, n_cus);
    // tiles of 256 rows that hold 128 at most are done as those; with many rounds of workgroups the others' larger steps count more than an even last round:
    // 128 experts, 4096 rows 987 for 1090 us, 512 .. 2048 rows 0.99; 64 of 1024 x 1408 (3 rounds), 2048 rows 156 for 146; 8 of 4096 x 1408, 400 rows 81 for 59
    return mtile == 128 && n_experts * (int64_t)((F + 127) / 128) >= 8 * n_cus ? 256 : mtile;
}

static GemmI8Params i8_params(compact_ctx* ctx, const GemmI8Args& a) {
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
    return p;
}

int launch_gemm_i8(compact_ctx* ctx, const GemmI8Args& a, void* ws, size_t ws_bytes, hipStream_t s) {
    if (a.M == 0) return COMPACT_OK;
    GemmI8Params p = i8_params(ctx, a);
    int n_cus = 0;
    TRY(device_cu_count(ctx, &n_cus));
    // more rows than the smallest row tiles (128 x 64: 512 threads) have workgroups for in one launch: several
    const int64_t most = 128 * (MAX_GRID_THREADS / (512 * (((int64_t)a.N + (a.epilogue ? 31 : 63)) / (a.epilogue ? 32 : 64))));
    if (!a.grouped && a.M > most) {
        const int64_t step = most < 256 ? most : most / 256 * 256, es = dtype_size(ctx->cfg.dtype);
        for (int64_t r = 0; r < a.M; r += step) {
            GemmI8Args part = a;
            part.M = std::min(a.M - r, step);
            part.a += r * a.K;
            part.a_scale += r;
            if (a.r) part.r = (const char*)a.r + r * a.N * es;
            part.c = (char*)a.c + r * a.N * es;
            TRY(launch_gemm_i8(ctx, part, ws, ws_bytes, s));
        }
        return COMPACT_OK;
    }
    if (a.grouped) {
        p.g = *a.grouped;
        p.n_mtiles = a.grouped->n_mtiles;
        const int form = p.g.mtile == 256 ? TILE_256 : p.g.mtile == 128 ? TILE_128 : TILE_64_128;
        if (p.g.mtile == I8_STREAM_ROWS) return launch_stream_i8(ctx, p, a.epilogue != 0, s);
        return a.epilogue ? launch_form<true, true>(ctx, form, 0, p, s) : launch_form<false, true>(ctx, form, 0, p, s);
    }
    const int slices = gemm_i8_slices(a.M, a.N, a.K, a.epilogue);
    const bool room = ws && ((uintptr_t)ws & 15) == 0 && ws_bytes >= gemm_i8_workspace(a.M, a.N, a.K, a.epilogue);
    // (without room for the slices' sums the stream is better than whole tiles)
    if (gemm_i8_streams(a.M, a.N, a.K, a.epilogue) || (a.M <= I8_STREAM_ROWS_MOST && slices > 1 && !room)) return launch_stream_i8(ctx, p, a.epilogue != 0, s);
    if (slices > 1 && room) {
        p.sums = (int*)ws;
        return a.epilogue ? launch_form<true, false>(ctx, TILE_64_64, 0, p, s, slices) : launch_form<false, false>(ctx, TILE_64_64, 0, p, s, slices);
    }
    int64_t n_full = 0;
    const int form = pick_tile(a.M, a.N, (a.K + 127) / 128 * 64, a.epilogue, n_cus, &n_full);
    return a.epilogue ? launch_form<true, false>(ctx, form, n_full, p, s) : launch_form<false, false>(ctx, form, n_full, p, s);
}

// For the tests, not part of compact.h: the product in tile form `form` (TILE_FORMS: whole tiles and halves mixed, as many slots
// in either), the small ones in `slices` of K with room for their sums.
extern "C" int compact_test_gemm_i8_form(compact_ctx* ctx, int32_t form, int32_t slices, void* sums, const void* a, const float* a_scale, const void* b,
                                         const float* b_scale, const void* r, void* c, int64_t M, int32_t N, int32_t K, int32_t epilogue,
                                         void* hip_stream) {
    if (!ctx || !a || !a_scale || !b || !b_scale || !c || M < 1 || N < 1 || K < 16 || K % 16 || form < 0 || form > TILE_FORMS || (epilogue != 0 && epilogue != 1) ||
        slices < 1 || slices > 8 || slices > (K + I8_BK - 1) / I8_BK || (slices > 1 && (!sums || form <= TILE_128 || form == TILE_FORMS)))
        return COMPACT_EINVAL;
    const GemmI8Args g{(const int8_t*)a, a_scale, (const int8_t*)b, b_scale, r, c, M, N, K, epilogue, nullptr};
    GemmI8Params p = i8_params(ctx, g);
    p.sums = (int*)sums;
    int64_t n_full = large_tiles(M, (N + (epilogue ? 127 : 255)) / (epilogue ? 128 : 256)).slots;
    if (form == TILE_FORMS) {
        form = TILE_256;
        n_full /= 2;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    return epilogue ? launch_form<true, false>(ctx, form, n_full, p, s, slices) : launch_form<false, false>(ctx, form, n_full, p, s, slices);
}
