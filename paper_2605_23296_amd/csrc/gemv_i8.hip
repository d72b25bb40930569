// Products of codes for at most 16 rows, and for up to 48 where that pays: a stream of the weights.  A workgroup of W wavefronts owns T tiles of 16 weight rows and
// finishes their sums over K, so there is no second launch.
//  * every load is 8 rows x 128 bytes (whole lines) and lands in LDS directly; wavefront kw takes the 128-wide pieces ("units") kw, kw + W, ...
//    of K for all T tiles and keeps a ring of its own of D tile pieces (2 KB each) and the activation codes of as many
//    units: no barrier, no wait but its own;
//  * chunks of 16 bytes sit at chunk ^ ((row / 2) % 8) of their row: 16 lanes that read one chunk of 16 rows touch 16 different bank groups;
//  * the W partial tiles meet in LDS; they are integers, so their order is of no account.
// 16 wavefronts for a plain product, with T as small as one workgroup per compute unit allows; 8 for experts, two workgroups per compute unit, so that one streams while
// the other finishes (8 for plain products: 0.97 .. 1.19 of the time); 8, and rings as deep as LDS holds, with more than 16 rows, whose activations take most of it.
// Bound: HBM.  2 * 14336 x 4096 at 8 rows 20.2 us of kernel (5.8 TB/s; in 64 x 64 tiles the call took 27.6 us, so 25.1), N 4096 K 14336 at 8 rows 13.3 a call, experts (128 of
// 2880 x 2880, top-4) of 16 rows 119 + 64 us (5.8 TB/s; in 64 x 64 tiles the whole call took 461, so 202).  Tiles of 32 rows for experts, two columns of MFMAs:
// 1.01 .. 1.09 of the time up to 8 rows an expert, at 12 0.95, where 256-row tiles take 0.92.
#include <algorithm>
#include <utility>

#include "common.h"
#include "gemm_i8.h"
#include "stream_lds.h"
#include "vecio.h"

#define GS_MAX_TILES 8
#define GS_MAX_TILES_MANY 2   // with more than 16 rows

template <class F, int... I>
__device__ __forceinline__ void for_each(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>{}), ...);
}

// XI: 8-row pieces of activations per unit (1: at most 8 rows, 2: at most 16).  D: tile pieces in a wavefront's ring.
template <int W, int T, int XI>
struct StreamShape {
    static constexpr int NX = (XI + 1) / 2;                  // MFMA columns of 16 rows
    static constexpr int depth(int d) { return XI > 2 && W * (2048 * (d + 1) + 1024 * XI * ((T + d) / T)) <= 159 * 1024 ? depth(d + 1) : d; }
    static constexpr int D = XI > 2 ? depth(2) : W > 8 && T <= 2 && XI == 2 ? 2 : 3;
    static constexpr int XD = (T - 1 + D) / T;               // units whose activations are in the ring
    static constexpr int XSLOT = XI * 1024, WSLOT = 2048;    // bytes
    static constexpr int WAVE_BYTES = D * WSLOT + XD * XSLOT;
    static constexpr int RED_BYTES = W * T * NX * 64 * 16;
    // (every load is issued, rows beyond the last one as the last one: waits count them.  Counting the activations' loads: 9 .. 16 rows 0.97 of the time)
    // loads younger than those of a unit's tile t: D - 1 tile pieces, and the activations that are requested with a unit's first
    static constexpr int younger(int t) {
        int n = 2 * (D - 1);
        for (int j = 1; j < D; ++j) n += (t + j) % T == 0 ? XI : 0;
        return n;
    }
    static constexpr int SMEM = W * WAVE_BYTES > RED_BYTES ? W * WAVE_BYTES : RED_BYTES;
    static_assert(SMEM <= 159 * 1024 / (W > 8 || XI > 2 ? 1 : 2), "16 wavefronts per compute unit, 8 with more than 16 rows");
};

template <int W, int T, int XI, bool GLU, bool GROUPED>
__global__ __launch_bounds__(W * 64) void stream_i8_kernel(const GemmI8Params p) {
    typedef StreamShape<W, T, XI> Shape;
    constexpr int D = Shape::D, XD = Shape::XD, NX = Shape::NX;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63;
    const int kw = wave_index();
    const int r = lane & 15, c = lane >> 4;
    const int n_tiles = GLU ? (p.N + 7) / 8 : (p.N + 15) / 16;
    int64_t m0 = 0;
    int rows = (int)p.M, tile0 = blockIdx.x * T;
    const int8_t* Wm = p.W;
    const float* wsc = p.ws;
    if (GROUPED) {
        const int groups = (n_tiles + T - 1) / T, tm = blockIdx.x / groups, e = p.g.tile_expert[tm];
        if (e < 0) return;
        tile0 = (blockIdx.x % groups) * T;
        m0 = p.g.tile_row0[tm];
        rows = p.g.tile_rows[tm];
        Wm += (int64_t)e * p.g.b_expert_stride;
        wsc += (int64_t)e * p.N * (GLU ? 2 : 1);
    }

    // lane l of a load: row l / 8 of 8, LDS position l % 8, hence chunk (l % 8) ^ ((row / 2) % 8) of the row's 128 bytes
    const int lrow = lane >> 3;
    const int8_t* wsrc[T][2];
    int chunk[2];   // of the even and the odd 8-row pieces
#pragma unroll
    for (int i = 0; i < 2; ++i) chunk[i] = ((lane & 7) ^ (((i * 8 + lrow) >> 1) & 7)) * 16;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int tile = min(tile0 + t, n_tiles - 1);
            const int n = GLU ? i * p.N + min(tile * 8 + lrow, p.N - 1) : min(tile * 16 + i * 8 + lrow, p.N - 1);
            wsrc[t][i] = Wm + (int64_t)n * p.K + chunk[i];
        }
    const int8_t* xsrc[XI];
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        int64_t row = m0 + min(i * 8 + lrow, rows - 1);
        if (GROUPED && p.g.a_gather) row = p.g.a_gather[row];
        xsrc[i] = p.X + row * p.K + chunk[i & 1];
    }
    char* const wring = smem + kw * Shape::WAVE_BYTES;
    char* const xring = wring + D * Shape::WSLOT;
    const int n_units = (p.K + 127) / 128;
    const int units = (n_units - kw + W - 1) / W;   // of this wavefront (may be 0)

    // chunks beyond K: zeros for the activations, the row's first chunk for the weights
    auto issue_x = [&](int u, int slot) __attribute__((always_inline)) {
        const int k = (u * W + kw) * 128;
#pragma unroll
        for (int i = 0; i < XI; ++i)
            load16_to_lds(k + chunk[i & 1] < p.K ? xsrc[i] + k : zero_codes, xring + slot * Shape::XSLOT + i * 1024);
    };
    auto issue_w = [&](const int8_t* const (&src)[2], int u, int slot) __attribute__((always_inline)) {
        const int k = (u * W + kw) * 128;
#pragma unroll
        for (int i = 0; i < 2; ++i) load16_to_lds(src[i] + (k + chunk[i] < p.K ? k : -chunk[i]), wring + slot * Shape::WSLOT + i * 1024);
    };
    intx4 acc[T][NX];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int x = 0; x < NX; ++x) acc[t][x] = intx4{0, 0, 0, 0};
    // tile pieces 0 .. D - 1 (piece q: tile q % T of unit q / T) and the activations of their units
#pragma unroll
    for (int q = 0; q < D; ++q)
        if (q / T < units) {
            if (q % T == 0) issue_x(q / T, q / T);
            issue_w(wsrc[q % T], q / T, q);
        }
    int foff[2], xoff[2];   // LDS offsets of the operand fragments of k-step h: row r, chunk 4 h + c
    const int xr = min(r, XI * 8 - 1);   // (columns beyond the rows staged are not read by anybody)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        foff[h] = r * 128 + (((4 * h + c) ^ ((r >> 1) & 7)) << 4);
        xoff[h] = xr * 128 + (((4 * h + c) ^ ((xr >> 1) & 7)) << 4);
    }
    int wslot = 0, xslot = 0;   // of the piece and of the unit that come next
    for (int u = 0; u < units; ++u) {
        intx4 xf[NX][2];
        for_each(std::make_integer_sequence<int, T>{}, [&](auto tt) __attribute__((always_inline)) {
            constexpr int t = decltype(tt)::value;
            // what is younger may still fly (near the end that is less: wait for all)
            if ((units - u) * T - t >= D)
                gs_wait<Shape::younger(t)>();
            else
                gs_wait<0>();
            if (t == 0) {
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int h = 0; h < 2; ++h) xf[x][h] = *reinterpret_cast<const intx4*>(xring + xslot * Shape::XSLOT + x * 2048 + xoff[h]);
                xslot = xslot + 1 == XD ? 0 : xslot + 1;
            }
            intx4 wf[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) wf[h] = *reinterpret_cast<const intx4*>(wring + wslot * Shape::WSLOT + foff[h]);
            gs_lds_done();   // the slots may be filled again
            const int nu = u + (t + D) / T;
            if (nu < units) {
                if ((t + D) % T == 0) {
                    // slot of unit nu: XD units after the one whose slot was read last
                    int xs = xslot + ((t + D) / T - 1) % XD;
                    issue_x(nu, xs >= XD ? xs - XD : xs);
                }
                issue_w(wsrc[(t + D) % T], nu, wslot);
            }
            wslot = wslot + 1 == D ? 0 : wslot + 1;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int x = 0; x < NX; ++x) acc[t][x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[h], xf[x][h], acc[t][x], 0, 0, 0);
        });
    }
    gs_wait<0>();
    __syncthreads();   // the rings are dead: the partial tiles take their place
    intx4* red = reinterpret_cast<intx4*>(smem);   // [W][T][NX][64]
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int x = 0; x < NX; ++x) red[((kw * T + t) * NX + x) * 64 + lane] = acc[t][x];
    __syncthreads();
    const int tile = tile0 + kw;   // wavefront kw finishes tile kw
    if (kw >= T || tile >= n_tiles) return;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
        intx4 v = red[(kw * NX + x) * 64 + lane];
#pragma unroll
        for (int w = 1; w < W; ++w) v += red[((w * T + kw) * NX + x) * 64 + lane];
        // v[e]: activation row 16 x + r, tile row 4 c + e (SwiGLU: c < 2 gate of column 4 c + e, c >= 2 up of column 4 (c - 2) + e)
        const int xr = 16 * x + r;
        const int64_t row = m0 + min(xr, rows - 1);
        const float xs = p.xs[GROUPED && p.g.a_gather ? (int64_t)p.g.a_gather[row] : row];
        const float gate = GROUPED && p.g.row_scale ? p.g.row_scale[row] : 1.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = GLU ? tile * 8 + 4 * (c & 1) + e : tile * 16 + 4 * c + e, nc = min(n, p.N - 1);
            float out;
            if (GLU) {
                const int up = __shfl_xor(v[e], 32, 64);
                out = i8_glu(i8_value(v[e], xs, wsc[nc]), i8_value(up, xs, wsc[p.N + nc]), p.f32);
            } else {
                out = i8_value(v[e], xs, wsc[nc]);
            }
            if (GROUPED) out *= gate;
            if (xr < rows && n < p.N && (!GLU || c < 2)) i8_put(p, row * p.N + n, out);
        }
    }
}

template <int W, int T, int XI, bool GLU, bool GROUPED>
static int launch_stream_form(compact_ctx* ctx, const GemmI8Params& p, hipStream_t s) {
    constexpr size_t smem = StreamShape<W, T, XI>::SMEM;
    const int n_tiles = GLU ? (p.N + 7) / 8 : (p.N + 15) / 16;
    static std::atomic<uint64_t> lds_set{0};
    TRY(allow_lds(ctx, (const void*)stream_i8_kernel<W, T, XI, GLU, GROUPED>, smem, lds_set));
    const int64_t wgs = (int64_t)((n_tiles + T - 1) / T) * (GROUPED ? p.n_mtiles : 1);
    if (wgs == 0) return COMPACT_OK;
    if (wgs * W * 64 > MAX_GRID_THREADS) return set_err(ctx, COMPACT_ESHAPE, "too many output tiles");
    stream_i8_kernel<W, T, XI, GLU, GROUPED><<<(unsigned)wgs, W * 64, smem, s>>>(p);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}
template <int T, bool GLU>
static int launch_stream_tiles(compact_ctx* ctx, const GemmI8Params& p, hipStream_t s) {
    if constexpr (T <= GS_MAX_TILES_MANY) {
        if (p.M > 32) return launch_stream_form<8, T, 6, GLU, false>(ctx, p, s);
        if (p.M > 16) return launch_stream_form<8, T, 4, GLU, false>(ctx, p, s);
    }
    return p.M <= 8 ? launch_stream_form<16, T, 1, GLU, false>(ctx, p, s) : launch_stream_form<16, T, 2, GLU, false>(ctx, p, s);
}
template <bool GLU>
static int launch_stream(compact_ctx* ctx, const GemmI8Params& p, hipStream_t s) {
    int n_cus = 0;
    TRY(device_cu_count(ctx, &n_cus));
    // as few rounds of a workgroup per compute unit as cover the matrix, evenly filled
    const int64_t n_tiles = GLU ? (p.N + 7) / 8 : (p.N + 15) / 16;
    const int most = p.M > 16 ? GS_MAX_TILES_MANY : GS_MAX_TILES;
    const int64_t rounds = (n_tiles + most * n_cus - 1) / (most * n_cus);
    switch ((n_tiles + rounds * n_cus - 1) / (rounds * n_cus)) {
        case 1: return launch_stream_tiles<1, GLU>(ctx, p, s);
        case 2: return launch_stream_tiles<2, GLU>(ctx, p, s);
        case 3: return launch_stream_tiles<3, GLU>(ctx, p, s);
        case 4: return launch_stream_tiles<4, GLU>(ctx, p, s);
        case 5: return launch_stream_tiles<5, GLU>(ctx, p, s);
        case 6: return launch_stream_tiles<6, GLU>(ctx, p, s);
        case 7: return launch_stream_tiles<7, GLU>(ctx, p, s);
        default: return launch_stream_tiles<8, GLU>(ctx, p, s);
    }
}

int launch_stream_i8(compact_ctx* ctx, GemmI8Params& p, bool glu, hipStream_t s) {
    if (p.g.tile_expert)
        return glu ? launch_stream_form<8, 8, 2, true, true>(ctx, p, s) : launch_stream_form<8, 8, 2, false, true>(ctx, p, s);
    return glu ? launch_stream<true>(ctx, p, s) : launch_stream<false>(ctx, p, s);
}
