// Attention over the paged cache in 8 bits: the streaming kernel for requests of few query columns (decode steps, a few rows to
// verify), the merge of split keys, and the entry point.
#include <algorithm>

#include "attn_paged.h"
#include "vecio.h"

#define FEW_WAVES 4
#define FEW_PLD (FEW_CHUNK + 8)   // bf16 per column of the probability tile (padded against bank conflicts)

// sum over the workgroup's threads, the same for all; `red`: one int per wavefront
__device__ __forceinline__ int block_total(int v, int* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) t += red[i];
    return t;
}

// inclusive sum over the workgroup's threads
__device__ __forceinline__ int block_prefix(int v, int* red, int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int ofs = 1; ofs < 64; ofs <<= 1) {
        const int u = __shfl_up(v, ofs, 64);
        if (lane >= ofs) v += u;
    }
    __syncthreads();
    if (lane == 63) red[w] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) {
        if (i < w) v += red[i];
        total += red[i];
    }
    return v;
}

// ---------------------------------------------------------------------------
// Requests of at most 16 query columns: memory-bound, every cached byte is read once.  A work item is (request, KV head, 256
// cached rows); a persistent workgroup of four wavefronts takes a contiguous share of them.  Scores S^T = K Q^T by
// v_mfma_f32_16x16x32_bf16, 64 cached rows per wavefront; the codes go straight from memory into MFMA operands (exact in
// bf16); probabilities through LDS; output O^T = V^T P^T, HD / 4 elements per wavefront.
// NP: bf16 parts of a query and of a probability (3 for fp32 storage: all 24 bits).
// ---------------------------------------------------------------------------
template <int HD, int NP, typename T, bool TILES>
__global__ __launch_bounds__(FEW_WAVES * 64) void attn_paged_few_kernel(const PagedAttnArgs a) {
    constexpr int KH = HD / 64;                // 16-byte pieces of a K row per lane
    constexpr int RT = HD / 16 / FEW_WAVES;    // 16-element tiles of O^T per wavefront
    constexpr int VS = FEW_CHUNK / 64;         // 16-byte pieces of a V row per lane
    __shared__ __attribute__((aligned(16))) bf16 qs[NP][FEW_COLS * HD];
    __shared__ __attribute__((aligned(16))) bf16 ps[NP][FEW_COLS * FEW_PLD];
    __shared__ float s_max[FEW_WAVES][16], s_sum[FEW_WAVES][16];
    __shared__ int red[FEW_WAVES], s_first[2];
    const int N = a.kv.n_requests, G = a.Hq / a.Hkv, Hkv = a.Hkv;
    const int t = threadIdx.x, lane = t & 63, wave = wave_index();
    const int r = lane & 15, c = lane >> 4;
    const int shift = a.kv.page_shift, P = 1 << shift;

    // ---- the other kernel's schedule: units (tile, piece) before every request, nothing taken yet ----
    if (TILES && blockIdx.x == 0) {
        int before = 0;
        for (int i0 = 0; i0 < N; i0 += FEW_WAVES * 64) {
            const int i = i0 + t;
            int units = 0;
            if (i < N) {
                const PagedReq rq = paged_req(a, i);
                if (rq.n > 0 && !is_few(rq.n, G)) {
                    const int tiles = n_tiles(rq.n, G);
                    units = tiles * tile_pieces(tiles, rq.kv);
                }
            }
            int all;
            const int upto = block_prefix(units, red, all);
            if (i < N) a.sched[SCHED_UNITS + i + 1] = before + upto;
            before += all;
        }
        if (t == 0) a.sched[SCHED_UNITS] = 0;
        if (t < 8) a.sched[t * SCHED_PITCH] = 0;
        __syncthreads();
    }

    // ---- this workgroup's share: items are numbered by request, KV head, chunk ----------------------
    auto items_of = [&](int i) {
        const PagedReq rq = paged_req(a, i);
        return rq.n > 0 && is_few(rq.n, G) ? few_pieces(rq.kv) * Hkv : 0;
    };
    int mine = 0;
    for (int i = t; i < N; i += FEW_WAVES * 64) mine += items_of(i);
    const int total = block_total(mine, red);
    int w = (int)((int64_t)blockIdx.x * total / gridDim.x);
    const int w_end = (int)((int64_t)(blockIdx.x + 1) * total / gridDim.x);
    if (w >= w_end) return;
    {   // the request that item w belongs to: wavefront 0 walks over the requests, 64 at a time
        if (wave == 0) {
            int before = 0;
            for (int i0 = 0; i0 < N; i0 += 64) {
                const int n = i0 + lane < N ? items_of(i0 + lane) : 0;
                int upto = n;
#pragma unroll
                for (int ofs = 1; ofs < 64; ofs <<= 1) {
                    const int u = __shfl_up(upto, ofs, 64);
                    if (lane >= ofs) upto += u;
                }
                const uint64_t past = __ballot(before + upto > w);
                if (past) {
                    if (lane == __builtin_ctzll(past)) {
                        s_first[0] = i0 + lane;
                        s_first[1] = w - (before + upto - n);
                    }
                    break;
                }
                before += __shfl(upto, 63, 64);
            }
        }
        __syncthreads();
    }
    int req = __builtin_amdgcn_readfirstlane(s_first[0]), in_req = __builtin_amdgcn_readfirstlane(s_first[1]);
    PagedReq rq = paged_req(a, req);
    int pieces = few_pieces(rq.kv);
    int q_req = -1, q_head = -1;

    for (; w < w_end; ++w, ++in_req) {
        while (in_req >= pieces * Hkv) {   // (w < w_end: there is a request with items left)
            do {
                ++req;
                rq = paged_req(a, req);
            } while (rq.n <= 0 || !is_few(rq.n, G));
            pieces = few_pieces(rq.kv);
            in_req = 0;
        }
        const int kvh = in_req / pieces, ch = in_req - kvh * pieces;
        const int base = ch * FEW_CHUNK, n_keys = min(rq.kv - base, FEW_CHUNK), cols = rq.n * G;

        // lane l < 16 (and l + 16 ..) holds the page and the scales of granule l of the chunk
        const int gtok = max(min(base + r * PAGED_GRAN, rq.kv - 1), 0);
        const int pid = min(max(a.kv.table[(size_t)req * a.kv.max_pages + (gtok >> shift)], 0), a.kv.n_pages - 1);
        const size_t ph = (size_t)pid * Hkv + kvh;
        const float ksc = e8m0(a.kv.ks[ph]), vsc = e8m0(a.kv.vs[ph]);

        uintx4 kf[4][KH], vf[RT][VS];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            const int g = wave * 4 + tt, page = __builtin_amdgcn_readlane(pid, g);
            const uint8_t* kp = a.kv.k + ((((size_t)page * Hkv + kvh) << shift) + ((base + g * PAGED_GRAN) & (P - 1)) + r) * HD + c * 16;
#pragma unroll
            for (int s = 0; s < KH; ++s) kf[tt][s] = *reinterpret_cast<const uintx4*>(kp + s * 64);
        }
#pragma unroll
        for (int j = 0; j < VS; ++j) {
            const int g = 4 * j + c, page = __shfl(pid, g, 64);
            const uint8_t* vp = a.kv.v + ((((size_t)page * Hkv + kvh) * HD) << shift) + ((base + g * PAGED_GRAN) & (P - 1));
#pragma unroll
            for (int i = 0; i < RT; ++i)
                vf[i][j] = *reinterpret_cast<const uintx4*>(vp + ((size_t)((wave * RT + i) * 16 + r) << shift));
        }
        if (req != q_req || kvh != q_head) {   // the group's query rows, column = row * G + head of the group
            q_req = req;
            q_head = kvh;
            __syncthreads();
            for (int i = t; i < FEW_COLS * HD / 8; i += FEW_WAVES * 64) {
                const int col = i / (HD / 8), e = i % (HD / 8) * 8;
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (col < cols) load8((const T*)a.q + (size_t)(rq.row0 + col / G) * a.q_stride + (kvh * G + col % G) * HD + e, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bf16 p[NP];
                    split_bf16<NP>(x[j], p);
#pragma unroll
                    for (int u = 0; u < NP; ++u) qs[u][col * HD + e + j] = p[u];
                }
            }
            __syncthreads();
        }

        // ---- S^T = K Q^T: lane (r, c) of tile tt gets column r, rows wave * 64 + tt * 16 + 4c .. + 3 ----
        float sv[4][4];
        float mx = -INFINITY;
        const int sees = min(rq.kv - rq.n + (r < cols ? r / G : 0) + 1 - base, n_keys);   // rows of the chunk that column r sees
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KH; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bf16x8 kb = codes8_to_bf16(kf[tt][s][2 * i], kf[tt][s][2 * i + 1], 1.0f);
#pragma unroll
                    for (int u = 0; u < NP; ++u) {
                        const bf16x8 qf = *reinterpret_cast<const bf16x8*>(&qs[u][r * HD + s * 64 + c * 16 + i * 8]);
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf, acc, 0, 0, 0);
                    }
                }
            const int g = wave * 4 + tt;
            const float f = a.scale_log2 * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ksc), g));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sv[tt][e] = g * PAGED_GRAN + 4 * c + e < sees ? acc[e] * f : -INFINITY;
                mx = fmaxf(mx, sv[tt][e]);
            }
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (c == 0) s_max[wave][r] = mx;
        __syncthreads();
        float m = -3e38f;   // (finite where a column sees nothing: its probabilities are exp2(-inf) = 0)
#pragma unroll
        for (int i = 0; i < FEW_WAVES; ++i) m = fmaxf(m, s_max[i][r]);
        float l = 0.f;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            bf16x4 pv[NP];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = exp2_fast(sv[tt][e] - m);
                l += p;
                bf16 part[NP];
                split_bf16<NP>(p, part);
#pragma unroll
                for (int u = 0; u < NP; ++u) pv[u][e] = part[u];
            }
#pragma unroll
            for (int u = 0; u < NP; ++u) *reinterpret_cast<bf16x4*>(&ps[u][r * FEW_PLD + wave * 64 + tt * 16 + 4 * c]) = pv[u];
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (c == 0) s_sum[wave][r] = l;
        __syncthreads();

        // ---- O^T = V^T P^T: HD / 4 elements per wavefront over all rows of the chunk -----------------
        floatx4 oacc[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) oacc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < VS; ++j) {
            const float sc = __shfl(vsc, 4 * j + c, 64);
            if (n_keys < FEW_CHUNK) {   // whatever lies behind the cached rows must not reach the MFMA
                const int live = n_keys - (64 * j + 16 * c);
#pragma unroll
                for (int wd = 0; wd < 4; ++wd) {
                    const unsigned keep = low_bytes(live - 4 * wd);
#pragma unroll
                    for (int i = 0; i < RT; ++i) vf[i][j][wd] &= keep;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < NP; ++u) {
                    const bf16x8 pb = *reinterpret_cast<const bf16x8*>(&ps[u][r * FEW_PLD + 64 * j + 16 * c + 8 * h]);
#pragma unroll
                    for (int i = 0; i < RT; ++i)
                        oacc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8_to_bf16(vf[i][j][2 * h], vf[i][j][2 * h + 1], sc), pb, oacc[i], 0, 0, 0);
                }
        }
        float lt = s_sum[0][r];
#pragma unroll
        for (int i = 1; i < FEW_WAVES; ++i) lt += s_sum[i][r];
        // lane (r, c): column r, elements (wave * RT + i) * 16 + 4c .. + 3
        if (r < cols) {
            const int row = r / G, head = kvh * G + r % G;
            if (pieces == 1) {
                const float inv = lt == 0.f ? 0.f : 1.0f / lt;
                T* op = (T*)a.o + ((size_t)(rq.row0 + row) * a.Hq + head) * HD + 4 * c;
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) op[(wave * RT + i) * 16 + e] = from_f32<T>(oacc[i][e] * inv);
            } else {
                const int64_t rec = ((int64_t)req * a.rec_stride + (int64_t)row * pieces) * a.Hq + (int64_t)head * pieces + ch;
#pragma unroll
                for (int i = 0; i < RT; ++i) *reinterpret_cast<floatx4*>(a.rec + rec * HD + (wave * RT + i) * 16 + 4 * c) = oacc[i];
                if (wave == 0 && c == 0) *reinterpret_cast<float2*>(a.rec + a.n_rec * HD + rec * 2) = make_float2(m, lt);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Joins the pieces of the (row, query head) pairs of split requests: WAVES wavefronts each, HD / 4 lanes span a record, and a
// lane sends for MERGE_FLIGHT records before it uses one.  Four wavefronts where a request can have more than MERGE_SHORT pieces,
// one up to there.
// ---------------------------------------------------------------------------
#define MERGE_FLIGHT 8
#define MERGE_SHORT 16
template <int HD, int WAVES, typename T>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(const PagedAttnArgs a, int rows_per_req, int heads_per_wg) {
    constexpr int TPR = HD / 4, NS = 64 / TPR, STEP = NS * WAVES;   // lanes per record, records side by side
    constexpr int PAIRS = 4 / WAVES;                                  // pairs that a workgroup has in hand at a time
    __shared__ floatx4 part[WAVES == 1 ? 1 : WAVES * TPR];
    const int lane = threadIdx.x & 63, wave = wave_index(), G = a.Hq / a.Hkv;
    const int per_row = (a.Hq + heads_per_wg - 1) / heads_per_wg;
    const int id = blockIdx.x / per_row, h_lo = blockIdx.x % per_row * heads_per_wg;
    const int row = id % rows_per_req, req = id / rows_per_req;
    const PagedReq rq = paged_req(a, req);
    if (row >= rq.n) return;
    const int pieces = is_few(rq.n, G) ? few_pieces(rq.kv) : tile_pieces(n_tiles(rq.n, G), rq.kv);
    if (pieces == 1) return;   // written by the kernel before
    const int sub = WAVES == 1 ? lane / TPR : wave * NS + lane / TPR, e4 = lane % TPR;
    for (int head = h_lo + wave / WAVES; head < min(h_lo + heads_per_wg, a.Hq); head += PAIRS) {
        const int64_t rec = ((int64_t)req * a.rec_stride + (int64_t)row * pieces) * a.Hq + (int64_t)head * pieces;
        const floatx4* val = reinterpret_cast<const floatx4*>(a.rec + rec * HD) + e4;
        const float2* ml = reinterpret_cast<const float2*>(a.rec + a.n_rec * HD) + rec;
        floatx4 v[MERGE_FLIGHT];
        float2 w[MERGE_FLIGHT];
        auto load = [&](int i0) {
#pragma unroll
            for (int u = 0; u < MERGE_FLIGHT; ++u) {
                const int i = min(i0 + u * STEP + sub, pieces - 1);
                v[u] = val[(size_t)i * TPR];
                w[u] = ml[i];
            }
        };
        load(0);
        float m = -3e38f, l = 0.f;
        for (int i = lane; i < pieces; i += 64) m = fmaxf(m, ml[i].x);
        m = wave_max(m);
        for (int i = lane; i < pieces; i += 64) l += exp2_fast(ml[i].x - m) * ml[i].y;
        l = wave_sum(l);
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0;;) {
#pragma unroll
            for (int u = 0; u < MERGE_FLIGHT; ++u) {
                const float f = i0 + u * STEP + sub < pieces ? exp2_fast(w[u].x - m) : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += f != 0.f ? f * v[u][e] : 0.f;
            }
            i0 += MERGE_FLIGHT * STEP;
            if (i0 >= pieces) break;
            load(i0);
        }
#pragma unroll
        for (int ofs = TPR; ofs < 64; ofs <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], ofs, 64);
        if (WAVES > 1) {
            __syncthreads();
            if (lane < TPR) part[wave * TPR + lane] = acc;
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int i = 1; i < WAVES; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += part[i * TPR + e4][e];
        }
        if (lane < TPR) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            put4((T*)a.o + ((size_t)(rq.row0 + row) * a.Hq + head) * HD + lane * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
        }
    }
}

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------
#define TRY_RC(expr)                       \
    do {                                   \
        const int _rc = (expr);            \
        if (_rc != COMPACT_OK) return _rc; \
    } while (0)

static bool has_tiles(const compact_layer_cfg& c, int max_new) { return (int64_t)max_new * (c.n_q_heads / c.n_kv_heads) > FEW_COLS; }

// row-pieces of a request that records are kept for; 0: no request of the call is split
static int64_t record_stride(const compact_layer_cfg& c, int max_new, int max_kv) {
    const int G = c.n_q_heads / c.n_kv_heads;
    int64_t few = 0, tiles = 0;
    const int chunks = (max_kv - 1) / FEW_CHUNK + 1;
    if (chunks > 1) few = (int64_t)std::min(max_new, FEW_COLS / G) * chunks;
    // n rows in t = ceil(n G / 128) tiles, p = floor(kv / 512 t) >= 2 pieces: n p <= (128 t / G) (kv / 512 t)
    if (has_tiles(c, max_new) && max_kv >= 2 * TILE_SPLIT) tiles = (int64_t)TILE_COLS * (max_kv / TILE_SPLIT + 1) / G + 1;
    return std::max(few, tiles);
}

static size_t paged_workspace(const compact_layer_cfg& c, int n_requests, int max_new, int max_kv) {
    const size_t rec = (size_t)n_requests * record_stride(c, max_new, max_kv) * c.n_q_heads;
    return align_up(SCHED_BYTES, 256) + rec * (c.head_dim + 2) * 4;
}

static int check_bounds(compact_ctx* ctx, int n_requests, int n_rows, int max_new, int max_kv_len) {
    if (n_requests < 1 || n_rows < 0 || max_new < 1 || max_kv_len < 1)
        return set_err(ctx, COMPACT_EINVAL, "n_requests >= 1, n_rows >= 0, max_new >= 1, max_kv_len >= 1 required");
    if (n_requests > PAGED_MAX_REQUESTS) return set_err(ctx, COMPACT_ESHAPE, "more than 4096 requests");
    if (n_rows > 1 << 26) return set_err(ctx, COMPACT_ESHAPE, "n_rows must be at most 2^26");
    return COMPACT_OK;
}

extern "C" int compact_paged_workspace_bytes(const compact_ctx* ctx, int32_t n_requests, int32_t n_rows, int32_t max_new,
                                             int32_t max_kv_len, size_t* bytes) {
    if (!ctx || !bytes) return COMPACT_EINVAL;
    TRY_RC(check_bounds(const_cast<compact_ctx*>(ctx), n_requests, n_rows, max_new, max_kv_len));
    *bytes = paged_workspace(ctx->cfg, n_requests, std::max(std::min(max_new, n_rows), 1), max_kv_len);
    return COMPACT_OK;
}

template <int HD, int NP, typename T>
static int launch_attn_paged(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s) {
    const compact_layer_cfg& c = ctx->cfg;
    int n_cus = 0;
    TRY_RC(device_cu_count(ctx, &n_cus));
    const bool tiles = has_tiles(c, a.max_new);
    const int64_t most = (int64_t)((a.max_kv - 1) / FEW_CHUNK + 1) * c.n_kv_heads * a.kv.n_requests;   // work items
    if (most > INT32_MAX) return set_err(ctx, COMPACT_ESHAPE, "n_requests * max_kv_len beyond what one call indexes");
    {
        ProfileScope ps(ctx, COMPACT_K_ATTN_DECODE, s);
        auto few = tiles ? attn_paged_few_kernel<HD, NP, T, true> : attn_paged_few_kernel<HD, NP, T, false>;
        few<<<(unsigned)std::min<int64_t>(most, 3 * n_cus), FEW_WAVES * 64, 0, s>>>(a);
    }
    LAUNCH_CHECK(ctx);
    if (tiles) TRY_RC(launch_attn_paged_tiles(ctx, a, s));
    if (a.rec_stride == 0) return COMPACT_OK;
    // rows of a request whose keys may be split: 512 t * 2 <= max_kv for its t tiles
    const int G = c.n_q_heads / c.n_kv_heads;
    const int64_t few_rows = std::min(a.max_new, FEW_COLS / G), tile_rows = (int64_t)TILE_COLS * (a.max_kv / TILE_SPLIT / 2) / G + 1;
    const int64_t rows = tiles ? std::min<int64_t>(a.max_new, std::max(few_rows, tile_rows)) : few_rows;
    const int most_pieces = std::max((a.max_kv - 1) / FEW_CHUNK + 1, tiles ? a.max_kv / TILE_SPLIT : 0);
    const int pairs = most_pieces > MERGE_SHORT ? 1 : 4;   // side by side in a workgroup
    // (workgroups of rows that are not split leave at once: no more than some thousand of them)
    int heads = pairs;
    while (heads < c.n_q_heads && rows * a.kv.n_requests * ((c.n_q_heads + heads - 1) / heads) > 4096) heads *= 2;
    const int64_t wgs = rows * a.kv.n_requests * ((c.n_q_heads + heads - 1) / heads);
    if (wgs >= INT32_MAX / 256) return set_err(ctx, COMPACT_ESHAPE, "too many rows of split requests for one call");
    auto merge = pairs == 1 ? attn_paged_merge_kernel<HD, 4, T> : attn_paged_merge_kernel<HD, 1, T>;
    merge<<<(unsigned)wgs, 256, 0, s>>>(a, (int)rows, heads);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

extern "C" int compact_attn_paged(compact_ctx* ctx, const compact_paged_kv* kv, int32_t n_rows, const int32_t* d_cu,
                                  const int32_t* d_kv_len, int32_t max_new, int32_t max_kv_len, const void* d_q, int64_t q_stride,
                                  void* d_o, void* d_workspace, size_t ws_bytes, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    PagedAttnArgs a{};
    TRY_RC(paged_view(ctx, kv, true, &a.kv));
    TRY_RC(check_bounds(ctx, kv->n_requests, n_rows, max_new, max_kv_len));
    if (!d_cu || !d_kv_len || !d_q || !d_o) return set_err(ctx, COMPACT_EINVAL, "null cu, kv_len, q or o");
    const compact_layer_cfg& c = ctx->cfg;
    if (q_stride < (int64_t)c.n_q_heads * c.head_dim || q_stride % 8 != 0)
        return set_err(ctx, COMPACT_EINVAL, "q_stride must be at least n_q_heads * head_dim and a multiple of 8");
    if (((uintptr_t)d_q | (uintptr_t)d_o) & 15) return set_err(ctx, COMPACT_EINVAL, "q and o must be 16-byte aligned");
    if (n_rows == 0) return COMPACT_OK;
    max_new = std::min(max_new, n_rows);
    if (!d_workspace || ((uintptr_t)d_workspace & 15) || ws_bytes < paged_workspace(c, kv->n_requests, max_new, max_kv_len))
        return set_err(ctx, COMPACT_EWORKSPACE, "workspace missing, not 16-byte aligned or too small for the paged attention");
    a.cu = d_cu;
    a.kv_len = d_kv_len;
    a.n_rows = n_rows;
    a.max_new = max_new;
    a.max_kv = (int)std::min<int64_t>(max_kv_len, (int64_t)kv->max_pages * kv->page_rows);
    a.q = d_q;
    a.o = d_o;
    a.q_stride = q_stride;
    a.Hq = c.n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.scale_log2 = LOG2E / sqrtf((float)c.head_dim);
    a.rec_stride = record_stride(c, max_new, a.max_kv);
    a.n_rec = (int64_t)kv->n_requests * a.rec_stride * c.n_q_heads;
    a.sched = (int32_t*)d_workspace;
    a.rec = (float*)((char*)d_workspace + align_up(SCHED_BYTES, 256));
    const bool b = c.dtype == COMPACT_BF16;
    auto launch = c.head_dim == 128 ? (b ? launch_attn_paged<128, 1, bf16> : launch_attn_paged<128, 3, float>)
                                    : (b ? launch_attn_paged<64, 1, bf16> : launch_attn_paged<64, 3, float>);
    return launch(ctx, a, (hipStream_t)hip_stream);
}
