// Attention over the paged cache in 8 bits for prompts and chunks of prompts: tiles of 128 query columns.
#include <algorithm>
#include <numeric>

#include "attn_paged.h"
#include "vecio.h"

// Chunk swizzles of the LDS tiles (16-byte chunks; the LDS has 64 banks of 4 bytes and serves a 16-byte read 16 lanes at a
// time): rows of 16 chunks by row % 16, rows of 8 chunks by (row / 2) % 8.
template <int CHUNKS>
__device__ __forceinline__ int swz(int row) { return CHUNKS == 16 ? (row & 15) : ((row >> 1) & 7); }

// Which XCD goes through which units of which KV heads: XCD x takes the heads x % xcd_heads + k * xcd_heads, shared with the
// other XCDs of the same heads unit by unit.
__device__ __forceinline__ int units_of_xcd(int x, int units, int Hkv, int xcd_heads) {
    const int share = 8 / xcd_heads, s = x / xcd_heads, all = units * (Hkv / xcd_heads);
    return (all - s + share - 1) / share;
}

// ---------------------------------------------------------------------------
// A unit is (request, tile of 128 query columns, piece of its keys, KV head): the columns of a KV head are its request's
// rows times the query heads of the group, so that a tile's heads share the keys.  A workgroup of four wavefronts takes units
// until there are none; a wavefront owns 32 columns and keeps Q^T in registers.  Steps of 64 keys: the codes of the
// next step are in flight in registers while this one is computed, are expanded to bf16 (exact) once per workgroup and
// go to LDS; S^T = K Q^T and O^T += V^T P^T by v_mfma_f32_32x32x16_bf16, softmax with a running maximum.
// ---------------------------------------------------------------------------
template <int HD, int NP, typename T>
__global__ __launch_bounds__(256, 1) void attn_paged_tile_kernel(const PagedAttnArgs a, int xcd_heads) {
    constexpr int KK = HD / 16, DT = HD / 32, KCH = HD / 8;
    constexpr int KTILE = TILE_KEYS * HD;
    constexpr int NLD = KTILE / 16 / 256;   // 16-byte pieces of codes per thread and tile
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16* lds = reinterpret_cast<bf16*>(smem);   // [2 K tiles | 2 V^T tiles]
    __shared__ int s_unit;
    const int G = a.Hq / a.Hkv, Hkv = a.Hkv, N = a.kv.n_requests;
    const int t = threadIdx.x, lane = t & 63, wave = wave_index();
    const int r = lane & 31, h = lane >> 5;
    const int shift = a.kv.page_shift, P = 1 << shift;
    const int32_t* before = a.sched + 8;
    const int units = before[N];
    const int pi_r = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);

    for (int turn = 0; turn < 8; ++turn) {
        const int x = (blockIdx.x + turn) & 7;   // its own XCD's units first, then those that others have left
        const int n_mine = units_of_xcd(x, units, Hkv, xcd_heads);
        for (;;) {
            __syncthreads();
            if (t == 0) s_unit = atomicAdd(&a.sched[x], 1);
            __syncthreads();
            const int mine = __builtin_amdgcn_readfirstlane(s_unit);
            if (mine >= n_mine) break;
            const int at = mine * (8 / xcd_heads) + x / xcd_heads;
            const int unit = at % units, kvh = at / units * xcd_heads + x % xcd_heads;
            int req = 0;
            for (int hi = N; hi - req > 1;) {   // the last request with units up to this one before it
                const int mid = (req + hi) >> 1;
                if (before[mid] <= unit)
                    req = mid;
                else
                    hi = mid;
            }
            const PagedReq rq = paged_req(a, req);
            const int tiles = n_tiles(rq.n, G), pieces = tile_pieces(tiles, rq.kv);
            const int in_req = unit - before[req], tile = tiles - 1 - in_req / pieces, piece = in_req % pieces;   // most keys first
            const int cols = min(rq.n * G - tile * TILE_COLS, TILE_COLS);
            const int span = tile_piece_rows(pieces, rq.kv);
            const int col = min(wave * 32 + r, cols - 1) + tile * TILE_COLS;
            const int row = col / G, head = kvh * G + col % G;
            const int sees = max(rq.kv - rq.n + row + 1, 0);                                        // keys this lane's column sees
            const int sees_wg = max(rq.kv - rq.n + (tile * TILE_COLS + cols - 1) / G + 1, 0);      // and the workgroup's last one
            const int sees_lo = max(rq.kv - rq.n + (tile * TILE_COLS + min(wave * 32, cols - 1)) / G + 1, 0);
            const int k_lo = piece * span, k_hi = min(min(k_lo + span, sees_wg), rq.kv);
            const int n_steps = max((k_hi - k_lo + TILE_KEYS - 1) / TILE_KEYS, 0);

            // Q^T operand: lane (column r, h) holds elements kk * 16 + h * 8 .. + 7
            bf16x8 qf[NP][KK];
            {
                const T* qp = (const T*)a.q + (size_t)(rq.row0 + row) * a.q_stride + head * HD + h * 8;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    float v[8];
                    load8(qp + kk * 16, v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        bf16 p[NP];
                        split_bf16<NP>(v[j], p);
#pragma unroll
                        for (int u = 0; u < NP; ++u) qf[u][kk][j] = p[u];
                    }
                }
            }
            floatx16 oacc[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[d][e] = 0.f;
            float m = -3e38f, l = 0.f;

            // ---- staging: thread t takes pieces i * 256 + t of a tile's codes: K piece p is row p / (HD / 16), elements
            // p % (HD / 16) * 16 .., V piece p is element p / 4, rows p % 4 * 16 ..
            uintx4 kreg[NLD], vreg[NLD];
            float ksc[NLD], vsc;
            auto fetch = [&](int step) {
                const int k0 = k_lo + step * TILE_KEYS;
                auto place = [&](int g) {   // page of granule g of the tile
                    const int tok = min(k0 + g * PAGED_GRAN, rq.kv - 1);
                    return min(max(a.kv.table[(size_t)req * a.kv.max_pages + (tok >> shift)], 0), a.kv.n_pages - 1);
                };
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const int p = i * 256 + t, krow = p / (HD / 16);
                    const size_t ph = (size_t)place(krow / PAGED_GRAN) * Hkv + kvh;
                    ksc[i] = e8m0(a.kv.ks[ph]);
                    kreg[i] = *reinterpret_cast<const uintx4*>(a.kv.k + ((ph << shift) + ((k0 + krow) & (P - 1))) * HD + p % (HD / 16) * 16);
                }
                const size_t ph = (size_t)place(t & 3) * Hkv + kvh;
                vsc = e8m0(a.kv.vs[ph]);
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const int p = i * 256 + t;
                    vreg[i] = *reinterpret_cast<const uintx4*>(a.kv.v + ((ph * HD + p / 4) << shift) + ((k0 + (t & 3) * PAGED_GRAN) & (P - 1)));
                }
            };
            auto stage = [&](int step) {
                const int live = rq.kv - (k_lo + step * TILE_KEYS) - (t & 3) * PAGED_GRAN;   // cached rows of this thread's V pieces
                bf16* ks = lds + (step & 1) * KTILE;
                bf16* vs = lds + (2 + (step & 1)) * KTILE;
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const int p = i * 256 + t, krow = p / (HD / 16), kc = p % (HD / 16) * 2, vrow = p / 4, vc = (t & 3) * 2;
                    if (live < PAGED_GRAN) {
#pragma unroll
                        for (int wd = 0; wd < 4; ++wd) vreg[i][wd] &= low_bytes(live - 4 * wd);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        *reinterpret_cast<bf16x8*>(ks + krow * HD + ((kc + j) ^ swz<KCH>(krow)) * 8) = codes8_to_bf16(kreg[i][2 * j], kreg[i][2 * j + 1], ksc[i]);
                        *reinterpret_cast<bf16x8*>(vs + vrow * TILE_KEYS + ((vc + j) ^ swz<8>(vrow)) * 8) = codes8_to_bf16(vreg[i][2 * j], vreg[i][2 * j + 1], vsc);
                    }
                }
            };
            if (n_steps > 0) {
                fetch(0);
                stage(0);
                if (n_steps > 1) fetch(1);
            }
            __syncthreads();
            for (int step = 0; step < n_steps; ++step) {
                const bf16* ks = lds + (step & 1) * KTILE;
                const bf16* vs = lds + (2 + (step & 1)) * KTILE;
                const int k0 = k_lo + step * TILE_KEYS;
                // S^T of half tt: column r, key k0 + 32 tt + (e / 8) * 16 + h * 8 + e % 8
                floatx16 sc[2];
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[tt][e] = 0.f;
                    const int krow = tt * 32 + pi_r;
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        const bf16x8 kb = *reinterpret_cast<const bf16x8*>(ks + krow * HD + ((kk * 2 + h) ^ swz<KCH>(krow)) * 8);
#pragma unroll
                        for (int u = 0; u < NP; ++u) sc[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb, qf[u][kk], sc[tt], 0, 0, 0);
                    }
                }
                if (k0 + TILE_KEYS > min(sees_lo, k_hi)) {
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (k0 + 32 * tt + (e >> 3) * 16 + h * 8 + (e & 7) >= min(sees, k_hi)) sc[tt][e] = -INFINITY;
                }
                float mx = -INFINITY;
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[tt][e]);
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * a.scale_log2;
                const float m_new = fmaxf(m, mx), corr = exp2_fast(m - m_new);
                m = m_new;
                l *= corr;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[d][e] *= corr;
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int u2 = 0; u2 < 2; ++u2) {
                        bf16x8 pf[NP];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float p = exp2_fast(__builtin_fmaf(sc[tt][u2 * 8 + e], a.scale_log2, -m));
                            l += p;
                            bf16 part[NP];
                            split_bf16<NP>(p, part);
#pragma unroll
                            for (int u = 0; u < NP; ++u) pf[u][e] = part[u];
                        }
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const int vrow = d * 32 + r;
                            const bf16x8 vb = *reinterpret_cast<const bf16x8*>(vs + vrow * TILE_KEYS + (((2 * tt + u2) * 2 + h) ^ swz<8>(vrow)) * 8);
#pragma unroll
                            for (int u = 0; u < NP; ++u) oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb, pf[u], oacc[d], 0, 0, 0);
                        }
                    }
                if (step + 1 < n_steps) {
                    stage(step + 1);
                    if (step + 2 < n_steps) fetch(step + 2);
                }
                __syncthreads();
            }
            // ---- lane (column r): elements d * 32 + (e / 4) * 8 + h * 4 + e % 4 ----
            l += __shfl_xor(l, 32, 64);
            if (wave * 32 + r < cols) {
                if (pieces == 1) {
                    const float inv = l == 0.f ? 0.f : 1.0f / l;
                    T* op = (T*)a.o + ((size_t)(rq.row0 + row) * a.Hq + head) * HD + h * 4;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) op[d * 32 + (e >> 2) * 8 + (e & 3)] = from_f32<T>(oacc[d][e] * inv);
                } else {
                    const int64_t rec = ((int64_t)req * a.rec_stride + (int64_t)row * pieces) * a.Hq + (int64_t)head * pieces + piece;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            *reinterpret_cast<floatx4*>(a.rec + rec * HD + d * 32 + g * 8 + h * 4) =
                                floatx4{oacc[d][4 * g], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]};
                    if (h == 0) *reinterpret_cast<float2*>(a.rec + a.n_rec * HD + rec * 2) = make_float2(m, l);
                }
            }
        }
    }
}

template <int HD, int NP, typename T>
static int launch_tiles(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s) {
    auto kern = attn_paged_tile_kernel<HD, NP, T>;
    const size_t smem = (size_t)4 * TILE_KEYS * HD * sizeof(bf16);
    HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    int n_cus = 0;
    if (int rc = device_cu_count(ctx, &n_cus)) return rc;
    ProfileScope ps(ctx, COMPACT_K_ATTN_PREFILL, s);
    kern<<<2 * n_cus, 256, smem, s>>>(a, std::gcd(8, a.Hkv));
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

int launch_attn_paged_tiles(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s) {
    const bool b = ctx->cfg.dtype == COMPACT_BF16;
    auto launch = ctx->cfg.head_dim == 128 ? (b ? launch_tiles<128, 1, bf16> : launch_tiles<128, 3, float>)
                                           : (b ? launch_tiles<64, 1, bf16> : launch_tiles<64, 3, float>);
    return launch(ctx, a, s);
}
