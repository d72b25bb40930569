// Attention over the paged cache in 8 bits: the streaming kernel for requests of few query columns (decode steps, a few rows to
// verify), the merge of split keys, and the entry point.
#include <algorithm>

#include "attn_paged.h"
#include "vecio.h"

#define FEW_WAVES 4
#define FEW_PLD (FEW_CHUNK + 8)   // bf16 per column of the probability tile (padded against bank conflicts)

// inclusive sum over the wavefront's lanes: inside rows of 16 lanes, then across them
__device__ __forceinline__ int wave_prefix(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31 to rows 2 and 3
#endif
    return v;
}
// inclusive sum over the workgroup's threads; `red`: one int per wavefront
__device__ __forceinline__ int block_prefix(int v, int* red, int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    v = wave_prefix(v);
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
// Requests of at most 32 query columns: memory-bound, every cached byte is read once.  A work item is (request, KV head, 256
// cached rows); a persistent workgroup of four wavefronts takes a contiguous share of them.  Scores S^T = K Q^T by
// v_mfma_f32_16x16x32_bf16, 64 cached rows per wavefront; the codes go straight from memory into MFMA operands (exact in
// bf16); probabilities through LDS; output O^T = V^T P^T, HD / 4 elements per wavefront.
// The loads run ahead of the items: the next item's K codes are sent for as soon as the scores of this one have used its own, its V
// codes behind the output, its pages' numbers and scales an item earlier still.  For the compiler to wait for no more
// than it needs (it counts outstanding loads), every load of the loop is issued unconditionally, with an address that is
// read anyway where there is no next item, and the stores stand right before the V loads.  Records are held back in LDS until the
// buffer is full or the share is done: a store in the load stream stalls it out of proportion.
// Bound: the codes' way from HBM (64 caches of 2048 rows, 8 KV heads of 128: 268 MB in 57 us, 4.7 TB/s of the 6.2 that a sum reaches;
// one cache of 32768 rows, 67 MB, 16.5 us: three loads one behind the other (lengths, page number, codes) before the first
// item, and the last workgroups' items).  256 rows per item: 512 leave no registers for the next item's loads.  Requests of
// 17 to 32 columns pay records of a quarter of the codes' bytes, written and read again (8 x 8 rows behind 16384: 268 MB of codes, 72 of
// records, 94 us with the merge; as tiles of 128 columns 106); with four column tiles, for up to 64, those and the registers cost more than they save (16 rows behind 32768: 55 us, as tiles 36).
// NP: bf16 parts of a query and of a probability (3 for fp32 storage: all 24 bits).  bf16 storage rounds a probability to bf16 for the
// second product, as the slab kernels do: one matrix instruction in place of two or three, for a relative error of 0.0016 to 0.0018 against
// 64 bits where rounding the output alone has 0.0015 to 0.0017 (prompts 0.002); their sum is of the values before the rounding.  CT: tiles of 16 columns, two where a call may
// have requests of more than 16; a column's sums are the same either way.
// ---------------------------------------------------------------------------
#define FEW_REC_SLOTS 8
// workgroups per CU (head_dim 64 has registers for four: 16 caches of 512 to 8192 rows 21.2 us instead of 18.8; two column tiles of
// head_dim 128 spill with three: 8 x 8 rows behind 16384 103 us instead of 95)
__host__ __device__ constexpr int few_resident(int hd, int np, int ct) { return (np > 1 ? 2 : 3) - (ct > 1 && hd > 64); }

// barrier that waits for this wavefront's LDS operations only: loads from memory stay in flight
__device__ __forceinline__ void lds_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));   // lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#endif
}

template <int HD, int NP, typename T, bool TILES, int CT>
__global__ __launch_bounds__(FEW_WAVES * 64, few_resident(HD, NP, CT)) void attn_paged_few_kernel(const PagedAttnArgs a, int slot_cols, int rec_slots) {
    constexpr int COLS = 16 * CT;              // query columns
    constexpr int KH = HD / 64;                // 16-byte pieces of a K row per lane
    constexpr int RT = HD / 16 / FEW_WAVES;    // 16-element tiles of O^T per wavefront
    constexpr int VS = FEW_CHUNK / 64;         // 16-byte pieces of a V row per lane
    constexpr int RLD = HD + 4;                // floats of a held record: values, maximum, sum
    __shared__ __attribute__((aligned(16))) bf16 qs[NP][COLS * HD];
    __shared__ __attribute__((aligned(16))) bf16 ps[NP][COLS * FEW_PLD];
    __shared__ float s_max[FEW_WAVES][COLS], s_sum[FEW_WAVES][COLS];
    __shared__ int red[FEW_WAVES];
    extern __shared__ __attribute__((aligned(16))) float recbuf[];   // [slot][column][RLD]
    __shared__ int64_t held_rec[FEW_REC_SLOTS];
    __shared__ int held_pieces[FEW_REC_SLOTS], held_cols[FEW_REC_SLOTS];
    const int N = a.kv.n_requests, G = a.Hq / a.Hkv, Hkv = a.Hkv;
    const int t = threadIdx.x, lane = t & 63, wave = wave_index();
    const int r = lane & 15, c = lane >> 4;
    int r_row[CT], r_head[CT];   // of column u * 16 + r
#pragma unroll
    for (int u = 0; u < CT; ++u) r_row[u] = (u * 16 + r) / G, r_head[u] = (u * 16 + r) % G;
    const int shift = a.kv.page_shift, P = 1 << shift;

    // ---- the other kernel's schedule: the requests with the longest units first (by the first two bits of their keys' number:
    // what comes last is short), units before every one of them, nothing taken yet ----
    if constexpr (TILES) {
        __shared__ int bucket[128];
        __shared__ uint16_t order[PAGED_MAX_REQUESTS];
        if (blockIdx.x == 0) {
            auto units_of = [&](const PagedReq& rq, int& length) {
                if (rq.n <= 0 || is_few(rq.n, G)) return 0;
                const int tiles = n_tiles(rq.n, G), pieces = tile_pieces(tiles, rq.kv);
                length = rq.kv / pieces;
                return tiles * pieces;
            };
            auto bucket_of = [](int length) { return 127 - (int)min(__builtin_bit_cast(unsigned, (float)length) >> 21, 639u) + 508; };   // 1 .. 2^31
            if (t < 128) bucket[t] = 0;
            __syncthreads();
            for (int i = t; i < N; i += FEW_WAVES * 64) {
                int length = 0;
                if (units_of(paged_req(a, i), length)) atomicAdd(&bucket[bucket_of(max(length, 1))], 1);
            }
            __syncthreads();
            int n_listed;
            {
                const int n = t < 128 ? bucket[t] : 0, upto = block_prefix(n, red, n_listed);
                __syncthreads();
                if (t < 128) bucket[t] = upto - n;
            }
            __syncthreads();
            for (int i = t; i < N; i += FEW_WAVES * 64) {
                int length = 0;
                if (units_of(paged_req(a, i), length)) order[atomicAdd(&bucket[bucket_of(max(length, 1))], 1)] = (uint16_t)i;
            }
            __syncthreads();
            int before = 0;
            for (int k0 = 0; k0 < n_listed; k0 += FEW_WAVES * 64) {
                const int k = k0 + t, req = k < n_listed ? order[k] : 0;
                int length, all;
                const int upto = block_prefix(k < n_listed ? units_of(paged_req(a, req), length) : 0, red, all);
                if (k < n_listed) {
                    a.sched[SCHED_UNITS + k + 1] = before + upto;
                    a.sched[SCHED_ORDER + k] = req;
                }
                before += all;
            }
            if (t == 0) {
                a.sched[SCHED_UNITS] = 0;
                a.sched[SCHED_LISTED] = n_listed;
            }
            if (t < 8) a.sched[t * SCHED_PITCH] = 0;
            __syncthreads();
        }
    }

    // ---- this workgroup's share: items are numbered by request, KV head, chunk.  Every wavefront goes over the requests by
    // itself, 64 at a time: once for their number, again for the request of the first item (which stays in the registers of
    // its lane's scan where there are no more than 64) ----------------------
    auto items_of = [&](const PagedReq& rq) { return rq.n > 0 && is_few(rq.n, G) ? few_pieces(rq.kv) * Hkv : 0; };
    PagedReq rq;
    int n_items = 0, upto = 0;   // of the lane's request, and of all up to it
    auto scan = [&](int i0) {
        rq = paged_req(a, min(i0 + lane, N - 1));
        n_items = i0 + lane < N ? items_of(rq) : 0;
        upto = wave_prefix(n_items);
    };
    int total = 0;
    for (int i0 = 0; i0 < N; i0 += 64) {
        scan(i0);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    const int w = (int)((int64_t)blockIdx.x * total / gridDim.x);
    int left = (int)((int64_t)(blockIdx.x + 1) * total / gridDim.x) - w;
    if (left <= 0) return;
    int first = 0, before = 0;   // the request of item w, 64 i0 + its lane
    uint64_t past = 0;
    for (;; first += 64) {
        if (N > 64) scan(first);
        past = __ballot(before + upto > w);
        if (past) break;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    const int at = __builtin_ctzll(past);

    // ---- items: a request's lengths come through the scalar cache, outside the counter of vector loads ----
    typedef const __attribute__((address_space(4))) int32_t* IntPtr;
    const IntPtr cu = (IntPtr)a.cu, kv_len = (IntPtr)a.kv_len;
    struct Item {
        int req, row0, n, kv, pieces, kvh, ch;
    };
    auto enter = [&](Item& it, int req) {
        it.req = req;
        it.row0 = min(max(cu[req], 0), a.n_rows);
        it.n = min(min(max(cu[req + 1], it.row0), a.n_rows) - it.row0, a.max_new);
        it.kv = min(max(kv_len[req], 0), a.max_kv);
        it.pieces = few_pieces(it.kv);
    };
    auto next_item = [&](Item& it) {   // (only called while there is one)
        if (++it.ch < it.pieces) return;
        it.ch = 0;
        if (++it.kvh < Hkv) return;
        it.kvh = 0;
        int req = it.req;
        do {
            enter(it, ++req);
        } while (it.n <= 0 || !is_few(it.n, G));
    };
    Item cur, nxt;
    cur.req = first + at;
    cur.row0 = __builtin_amdgcn_readlane(rq.row0, at);
    cur.n = __builtin_amdgcn_readlane(rq.n, at);
    cur.kv = __builtin_amdgcn_readlane(rq.kv, at);
    cur.pieces = few_pieces(cur.kv);
    {
        const int in_req = w - before - __builtin_amdgcn_readlane(upto - n_items, at);
        cur.kvh = in_req / cur.pieces;
        cur.ch = in_req - cur.kvh * cur.pieces;
    }

    // lane l holds the page of granule l % 16 of a chunk (granules past the cached rows: the last one's)
    auto load_pid = [&](const Item& it) {
        const int row = max(min(it.ch * FEW_CHUNK + r * PAGED_GRAN, it.kv - 1), 0);
        return a.kv.table[(size_t)it.req * a.kv.max_pages + (row >> shift)];
    };
    auto in_range = [&](int pid) { return min(max(pid, 0), a.kv.n_pages - 1); };
    uintx4 kf[4][KH], vf[RT][VS];
    // keep = 0 (otherwise all ones): nothing to fetch; the same instructions go out, all lanes for the same few bytes (masks, no
    // branch: both cases have to be one stream of instructions for the compiler's count of the loads)
    auto load_k = [&](const Item& it, int pid, int keep) {
        const int off = (r * HD + c * 16) & keep;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            const int g = wave * 4 + tt;
            const unsigned page = __builtin_amdgcn_readlane(pid, g);
            const uint8_t* kp = a.kv.k + ((((size_t)page * Hkv + it.kvh) << shift) + ((it.ch * FEW_CHUNK + g * PAGED_GRAN) & (P - 1))) * HD;
#pragma unroll
            for (int s = 0; s < KH; ++s) kf[tt][s] = *reinterpret_cast<const uintx4*>(kp + (off + s * 64));
        }
    };
    auto load_v = [&](const Item& it, int pid, int keep) {
        const int row = (wave * RT * 16 + r) & keep, next = (16 << shift) & keep;
#pragma unroll
        for (int j = 0; j < VS; ++j) {
            const int g = (4 * j + c) & keep;
            const unsigned page = __shfl(pid, g, 64);
            const uint8_t* vp = a.kv.v + ((((size_t)page * Hkv + it.kvh) * HD + row) << shift) + ((it.ch * FEW_CHUNK + g * PAGED_GRAN) & (P - 1));
#pragma unroll
            for (int i = 0; i < RT; ++i) vf[i][j] = *reinterpret_cast<const uintx4*>(vp + i * next);
        }
    };
    // the item's query rows: columns row * G + head of the group, 8 elements per thread
    struct alignas(16) Eight { T x[8]; };
    constexpr int QP = (COLS * HD / 8 + FEW_WAVES * 64 - 1) / (FEW_WAVES * 64);   // pieces per thread
    Eight qreg[QP];
    int q_row[QP], q_head[QP];
    const int q_e = t % (HD / 8) * 8;
    auto q_col = [&](int j) { return min((j * FEW_WAVES * 64 + t) / (HD / 8), COLS - 1); };
#pragma unroll
    for (int j = 0; j < QP; ++j) q_row[j] = q_col(j) / G, q_head[j] = q_col(j) % G;
    auto load_q = [&](const Item& it) {
#pragma unroll
        for (int j = 0; j < QP; ++j) {
            const int row = it.row0 + min(q_row[j], it.n - 1);
            qreg[j] = *reinterpret_cast<const Eight*>((const T*)a.q + (size_t)row * a.q_stride + (it.kvh * G + q_head[j]) * HD + q_e);
        }
    };

    // (sent in the order that the loop sends them: the compiler waits for a load by the least number of later ones)
    int pid = load_pid(cur);
    nxt = cur;
    if (left > 1) next_item(nxt);
    int pid_n = load_pid(nxt);
    pid = in_range(pid);
    size_t ph = (size_t)pid * Hkv + cur.kvh;
    unsigned ksb = a.kv.ks[ph], vsb = a.kv.vs[ph];
    __builtin_amdgcn_sched_barrier(0);
    load_k(cur, pid, -1);
    load_q(cur);
    __builtin_amdgcn_sched_barrier(0);
    load_v(cur, pid, -1);
    __builtin_amdgcn_sched_barrier(0);
    int q_req = -1, q_kvh = -1, n_held = 0;

    for (;;) {
        const bool has_next = left > 1;
        const int keep = here(has_next ? -1 : 0);
        const int base = cur.ch * FEW_CHUNK, n_keys = min(cur.kv - base, FEW_CHUNK), cols = cur.n * G;
        const bool wide = CT > 1 && (!TILES || cols > 16);   // (beside prompts most requests have one row: 64 of them 4 us in 100)
        // pages and scales of the next item; the page numbers of the one after it
        pid = in_range(pid_n);
        Item nn = nxt;
        if (left > 2) next_item(nn);
        pid_n = load_pid(nn);
        ph = (size_t)pid * Hkv + nxt.kvh;
        const unsigned ksb_n = a.kv.ks[ph], vsb_n = a.kv.vs[ph];

        if (cur.req != q_req || cur.kvh != q_kvh) {
            q_req = cur.req;
            q_kvh = cur.kvh;
            lds_barrier();   // (the rows before have been read)
#pragma unroll
            for (int jj = 0; jj < QP; ++jj)
                if (t + jj * FEW_WAVES * 64 < COLS * HD / 8) {
                    bf16x8 part[NP];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        bf16 p[NP];
                        split_bf16<NP>(q_col(jj) < cols ? to_f32(qreg[jj].x[j]) : 0.f, p);
#pragma unroll
                        for (int u = 0; u < NP; ++u) part[u][j] = p[u];
                    }
#pragma unroll
                    for (int u = 0; u < NP; ++u) *reinterpret_cast<bf16x8*>(&qs[u][q_col(jj) * HD + q_e]) = part[u];
                }
            lds_barrier();
        }

        // ---- S^T = K Q^T: lane (r, c) of tile tt gets columns u * 16 + r, rows wave * 64 + tt * 16 + 4c .. + 3 ----
        float sv[CT][4][4], mx[CT];
        int sees[CT];   // rows of the chunk that the column sees
#pragma unroll
        for (int u = 0; u < CT; ++u) {
            mx[u] = -INFINITY;
            sees[u] = min(cur.kv - cur.n + (u * 16 + r < cols ? r_row[u] : 0) + 1 - base, n_keys);
        }
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            floatx4 acc[CT];
#pragma unroll
            for (int w = 0; w < CT; ++w) acc[w] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KH; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bf16x8 kb = codes8_to_bf16(kf[tt][s][2 * i], kf[tt][s][2 * i + 1], 1.0f);
#pragma unroll
                    for (int w = 0; w < CT; ++w) {
                        if (w > 0 && !wide) continue;
#pragma unroll
                        for (int u = 0; u < NP; ++u) {
                            const bf16x8 qf = *reinterpret_cast<const bf16x8*>(&qs[u][(w * 16 + r) * HD + s * 64 + c * 16 + i * 8]);
                            acc[w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf, acc[w], 0, 0, 0);
                        }
                    }
                }
            const int g = wave * 4 + tt;
            const float f = a.scale_log2 * e8m0(__builtin_amdgcn_readlane(ksb, g));
#pragma unroll
            for (int w = 0; w < CT; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sv[w][tt][e] = g * PAGED_GRAN + 4 * c + e < sees[w] ? acc[w][e] * f : -INFINITY;
                    mx[w] = fmaxf(mx[w], sv[w][tt][e]);
                }
        }
        // the K registers are free
        load_k(nxt, pid, keep);
        load_q(nxt);
#pragma unroll
        for (int w = 0; w < CT; ++w) {
            mx[w] = fmaxf(mx[w], __shfl_xor(mx[w], 16, 64));
            mx[w] = fmaxf(mx[w], __shfl_xor(mx[w], 32, 64));
            if (c == 0) s_max[wave][w * 16 + r] = mx[w];
        }
        lds_barrier();
        float m[CT];   // (finite where a column sees nothing: its probabilities are exp2(-inf) = 0)
#pragma unroll
        for (int w = 0; w < CT; ++w) {
            if (w > 0 && !wide) continue;
            m[w] = -3e38f;
#pragma unroll
            for (int i = 0; i < FEW_WAVES; ++i) m[w] = fmaxf(m[w], s_max[i][w * 16 + r]);
            float l = 0.f;
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                bf16x4 pv[NP];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = exp2_fast(sv[w][tt][e] - m[w]);
                    l += p;
                    bf16 part[NP];
                    split_bf16<NP>(p, part);
#pragma unroll
                    for (int u = 0; u < NP; ++u) pv[u][e] = part[u];
                }
#pragma unroll
                for (int u = 0; u < NP; ++u) *reinterpret_cast<bf16x4*>(&ps[u][(w * 16 + r) * FEW_PLD + wave * 64 + tt * 16 + 4 * c]) = pv[u];
            }
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            if (c == 0) s_sum[wave][w * 16 + r] = l;
        }
        lds_barrier();

        // ---- O^T = V^T P^T: HD / 4 elements per wavefront over all rows of the chunk -----------------
        floatx4 oacc[CT][RT];
#pragma unroll
        for (int w = 0; w < CT; ++w)
#pragma unroll
            for (int i = 0; i < RT; ++i) oacc[w][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (n_keys < FEW_CHUNK) {   // whatever lies behind the cached rows must not reach the MFMA, scales of pages that are nobody's included
            if (r * PAGED_GRAN >= n_keys) vsb = 127;
#pragma unroll
            for (int j = 0; j < VS; ++j)
#pragma unroll
                for (int wd = 0; wd < 4; ++wd) {
                    const unsigned keep = low_bytes(n_keys - (64 * j + 16 * c) - 4 * wd);
#pragma unroll
                    for (int i = 0; i < RT; ++i) vf[i][j][wd] &= keep;
                }
        }
#pragma unroll
        for (int j = 0; j < VS; ++j) {
            const float sc = e8m0(__shfl(vsb, 4 * j + c, 64));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 vb[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) vb[i] = codes8_to_bf16(vf[i][j][2 * h], vf[i][j][2 * h + 1], sc);
#pragma unroll
                for (int w = 0; w < CT; ++w) {
                    if (w > 0 && !wide) continue;
#pragma unroll
                    for (int u = 0; u < NP; ++u) {
                        const bf16x8 pb = *reinterpret_cast<const bf16x8*>(&ps[u][(w * 16 + r) * FEW_PLD + 64 * j + 16 * c + 8 * h]);
#pragma unroll
                        for (int i = 0; i < RT; ++i) oacc[w][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb[i], pb, oacc[w][i], 0, 0, 0);
                    }
                }
            }
        }
        // lane (r, c): columns w * 16 + r, elements (wave * RT + i) * 16 + 4c .. + 3
#pragma unroll
        for (int w = 0; w < CT; ++w) {
            const int col = w * 16 + r;
            float lt = s_sum[0][col];
#pragma unroll
            for (int i = 1; i < FEW_WAVES; ++i) lt += s_sum[i][col];
            if (cur.pieces == 1) {
                if (col < cols) {
                    const float inv = lt == 0.f ? 0.f : 1.0f / lt;
                    T* op = (T*)a.o + ((size_t)(cur.row0 + r_row[w]) * a.Hq + cur.kvh * G + r_head[w]) * HD + 4 * c;
#pragma unroll
                    for (int i = 0; i < RT; ++i) put4(op + (wave * RT + i) * 16, oacc[w][i][0] * inv, oacc[w][i][1] * inv, oacc[w][i][2] * inv, oacc[w][i][3] * inv);
                }
            } else if (col < cols) {
                float* slot = recbuf + (size_t)n_held * slot_cols * RLD + col * RLD;
#pragma unroll
                for (int i = 0; i < RT; ++i) *reinterpret_cast<floatx4*>(slot + (wave * RT + i) * 16 + 4 * c) = oacc[w][i];
                if (wave == 0 && c == 0) *reinterpret_cast<float2*>(slot + HD) = make_float2(m[w], lt);
            }
        }
        if (cur.pieces > 1) {
            if (t == 0) {
                held_rec[n_held] = first_record(a, cur.req, cur.row0, 0, cur.kvh * G, cur.pieces) + cur.ch;
                held_pieces[n_held] = cur.pieces;
                held_cols[n_held] = cols;
            }
            ++n_held;
        }
        if (n_held == rec_slots || (!has_next && n_held > 0)) {
            lds_barrier();
            for (int k = 0; k < n_held; ++k) {
                const float* slot = recbuf + (size_t)k * slot_cols * RLD;
                const int pieces = held_pieces[k], n = held_cols[k];
                for (int i = t; i < n * (HD / 4); i += FEW_WAVES * 64) {
                    const int col = i / (HD / 4), e = i % (HD / 4) * 4;
                    const int64_t rec = held_rec[k] + (int64_t)(col / G) * pieces * a.Hq + (int64_t)(col % G) * pieces;
                    *reinterpret_cast<floatx4*>(a.rec + rec * HD + e) = *reinterpret_cast<const floatx4*>(slot + col * RLD + e);
                    if (e == 0) *reinterpret_cast<float2*>(a.rec + a.n_rec * HD + rec * 2) = *reinterpret_cast<const float2*>(slot + col * RLD + HD);
                }
            }
            n_held = 0;
            lds_barrier();
        }
        // the V registers are free
        load_v(nxt, pid, keep);
        asm volatile("" ::: "memory");   // (the loads stay on this side of the branch, see above)
        if (!has_next) break;
        cur = nxt;
        nxt = nn;
        ksb = ksb_n;
        vsb = vsb_n;
        --left;
    }
}

// ---------------------------------------------------------------------------
// Joins the pieces of the (row, query head) pairs of split requests.  HD / 4 lanes span a record; a lane sends for up to
// MERGE_FLIGHT records before it uses one.  With m = max m_i: o = sum 2^(m_i - m) o_i / sum 2^(m_i - m) l_i.  Bound by the launch
// and two loads one behind the other (5.2 us for 64 x 8 and for 128 pieces, traced; a call that merges nothing 4.5).  A request whose records one wavefront can send for at once has a wavefront per pair
// (32 pieces of head_dim 64: 4.0 us instead of 7.2), one with more of them all four wavefronts of the workgroup.
// ---------------------------------------------------------------------------
#define MERGE_FLIGHT 8

// WAVES wavefronts join one pair
template <int HD, int WAVES, typename T>
__device__ __forceinline__ void merge_pair(const PagedAttnArgs& a, const PagedReq& rq, int req, int row, int head, int pieces, floatx4* part) {
    constexpr int TPR = HD / 4, NS = 64 / TPR, STEP = NS * WAVES;   // lanes per record, records side by side
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int sub = WAVES == 1 ? lane / TPR : wave * NS + lane / TPR, e4 = lane % TPR;
    const int64_t rec = first_record(a, req, rq.row0, row, head, pieces);
    const floatx4* val = reinterpret_cast<const floatx4*>(a.rec + rec * HD) + e4;
    const float2* ml = reinterpret_cast<const float2*>(a.rec + a.n_rec * HD) + rec;
    floatx4 v[MERGE_FLIGHT];
    float2 w[MERGE_FLIGHT];
    auto load = [&](int i0) {
#pragma unroll
        for (int u = 0; u < MERGE_FLIGHT; ++u)
            if (i0 + u * STEP < pieces) {
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
        for (int u = 0; u < MERGE_FLIGHT; ++u)
            if (i0 + u * STEP < pieces) {
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
        if (wave > 0) return;
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

// pieces of a request's keys
__device__ __forceinline__ int pieces_of(const PagedReq& rq, int G) {
    return is_few(rq.n, G) ? few_pieces(rq.kv) : tile_pieces(n_tiles(rq.n, G), rq.kv);
}
template <int HD>
__host__ __device__ __forceinline__ bool wave_each(int pieces) { return pieces <= MERGE_FLIGHT * (256 / HD); }

// A workgroup per row and heads_per_wg query heads.
template <int HD, typename T>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(const PagedAttnArgs a, int rows_per_req, int heads_per_wg) {
    __shared__ floatx4 part[HD];
    const int G = a.Hq / a.Hkv;
    const int per_row = (a.Hq + heads_per_wg - 1) / heads_per_wg;
    const int id = blockIdx.x / per_row, h_lo = blockIdx.x % per_row * heads_per_wg, h_end = min(h_lo + heads_per_wg, a.Hq);
    const int row = id % rows_per_req, req = id / rows_per_req;
    const PagedReq rq = paged_req(a, req);
    if (row >= rq.n) return;
    const int pieces = pieces_of(rq, G);
    if (pieces == 1) return;   // written by the kernel before
    if (wave_each<HD>(pieces)) {
        for (int head = h_lo + wave_index(); head < h_end; head += 4) merge_pair<HD, 1, T>(a, rq, req, row, head, pieces, part);
    } else {
        for (int head = h_lo; head < h_end; ++head) merge_pair<HD, 4, T>(a, rq, req, row, head, pieces, part);
    }
}

// The same where a call has prompts, hardly any of whose rows are split: a fixed number of workgroups shares out the pairs
// (four at a time where a wavefront joins one) that the requests' lengths give (64 single rows behind 2048 in a call for up to
// 64 rows each: 75 us in all, 98 with a workgroup per row that there may be).
template <int HD, typename T>
__global__ __launch_bounds__(256) void attn_paged_merge_share_kernel(const PagedAttnArgs a) {
    __shared__ floatx4 part[HD];
    const int N = a.kv.n_requests, G = a.Hq / a.Hkv, lane = threadIdx.x & 63, fours = (a.Hq + 3) / 4;
    auto items_of = [&](const PagedReq& rq, int& pieces) {
        pieces = rq.n > 0 ? pieces_of(rq, G) : 1;
        return pieces == 1 ? 0 : rq.n * (wave_each<HD>(pieces) ? fours : a.Hq);
    };
    int upto = 0, n_items = 0, pieces;
    auto scan = [&](int i0) {
        n_items = items_of(paged_req(a, min(i0 + lane, N - 1)), pieces);
        if (i0 + lane >= N) n_items = 0;
        upto = wave_prefix(n_items);
    };
    int total = 0;
    for (int i0 = 0; i0 < N; i0 += 64) {
        scan(i0);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    const int w = (int)((int64_t)blockIdx.x * total / gridDim.x);
    int left = (int)((int64_t)(blockIdx.x + 1) * total / gridDim.x) - w;
    if (left <= 0) return;
    int first = 0, before = 0;
    uint64_t past = 0;
    for (;; first += 64) {
        if (N > 64) scan(first);
        past = __ballot(before + upto > w);
        if (past) break;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    const int at = __builtin_ctzll(past);
    int req = first + at, item = w - before - __builtin_amdgcn_readlane(upto - n_items, at);
    for (;; ++req, item = 0) {   // (ends: the requests' items add up to the share)
        const PagedReq rq = paged_req(a, req);
        const int end = min(items_of(rq, pieces), item + left);
        left -= max(end - item, 0);
        for (; item < end; ++item) {
            if (wave_each<HD>(pieces)) {
                const int head = item % fours * 4 + wave_index();
                if (head < a.Hq) merge_pair<HD, 1, T>(a, rq, req, item / fours, head, pieces, part);
            } else {
                merge_pair<HD, 4, T>(a, rq, req, item / a.Hq, item % a.Hq, pieces, part);
            }
        }
        if (left <= 0) return;
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

// t tiles in p >= 2 pieces: t p is at most this
static int most_split(int max_kv) { return std::max(max_kv / TILE_SPLIT, max_kv >= 2 * TILE_LONG ? TILE_FILL : 0); }

// Where the records lie: a request's row-pieces begin at req * per_req + row0 * per_row.  Three ways to hold all of them, each
// with room for the most that a request's n rows in p >= 2 pieces can be; the smallest is taken.
struct RecordLayout {
    int64_t per_req, per_row, total;   // in row-pieces; total 0: no request of the call is split
};
static RecordLayout record_layout(const compact_layer_cfg& c, int n_requests, int n_rows, int max_new, int max_kv) {
    const int G = c.n_q_heads / c.n_kv_heads, chunks = (max_kv - 1) / FEW_CHUNK + 1;
    if (chunks == 1) return {0, 0, 0};
    const int64_t few = (int64_t)std::min(max_new, FEW_COLS / G) * chunks;
    const bool tiles = has_tiles(c, max_new) && max_kv >= 2 * TILE_SPLIT;
    // by request: n rows in t = ceil(n G / 128) tiles: n p <= (128 / G) t p
    RecordLayout best = {tiles ? std::max(few, (int64_t)TILE_COLS * (most_split(max_kv) + 1) / G + 1) : few, 0, 0};
    best.total = best.per_req * n_requests;
    auto consider = [&](int64_t per_req, int64_t per_row) {
        const int64_t total = per_req * n_requests + per_row * n_rows;
        if (total < best.total) best = {per_req, per_row, total};
    };
    consider(0, chunks);   // by row: p <= chunks
    // by both: a few rows as above, t p <= kv / 512 whatever the rows, or p <= kv / 2048
    if (tiles) consider(std::max(few, (int64_t)TILE_COLS * (max_kv / TILE_SPLIT) / G), max_kv >= 2 * TILE_LONG ? max_kv / TILE_LONG : 0);
    return best;
}

static size_t paged_workspace(const compact_layer_cfg& c, int n_requests, int n_rows, int max_new, int max_kv) {
    const size_t rec = (size_t)record_layout(c, n_requests, n_rows, max_new, max_kv).total * c.n_q_heads;
    return align_up(SCHED_BYTES, 256) + rec * (c.head_dim + 2) * 4;
}

static int check_bounds(compact_ctx* ctx, int n_requests, int n_rows, int max_new, int max_kv_len) {
    if (n_requests < 1 || n_rows < 0 || max_new < 1 || max_kv_len < 1)
        return set_err(ctx, COMPACT_EINVAL, "n_requests >= 1, n_rows >= 0, max_new >= 1, max_kv_len >= 1 required");
    if (n_requests > PAGED_MAX_REQUESTS) return set_err(ctx, COMPACT_ESHAPE, "more than 4096 requests");
    if (n_rows > PAGED_MAX_ROWS) return set_err(ctx, COMPACT_ESHAPE, "n_rows must be at most 2^26");
    return COMPACT_OK;
}

extern "C" int compact_paged_workspace_bytes(const compact_ctx* ctx, int32_t n_requests, int32_t n_rows, int32_t max_new,
                                             int32_t max_kv_len, size_t* bytes) {
    if (!ctx || !bytes) return COMPACT_EINVAL;
    TRY_RC(check_bounds(const_cast<compact_ctx*>(ctx), n_requests, n_rows, max_new, max_kv_len));
    n_rows = std::max(n_rows, 1);
    *bytes = paged_workspace(ctx->cfg, n_requests, n_rows, std::min(max_new, n_rows), max_kv_len);
    return COMPACT_OK;
}

template <int HD, int NP, typename T>
static int launch_attn_paged(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s) {
    const compact_layer_cfg& c = ctx->cfg;
    int n_cus = 0;
    TRY_RC(device_cu_count(ctx, &n_cus));
    const bool tiles = has_tiles(c, a.max_new);
    const int G = c.n_q_heads / c.n_kv_heads;
    const int64_t most = (int64_t)((a.max_kv - 1) / FEW_CHUNK + 1) * c.n_kv_heads * a.kv.n_requests;   // work items
    if (most > INT32_MAX) return set_err(ctx, COMPACT_ESHAPE, "n_requests * max_kv_len beyond what one call indexes");
    {
        ProfileScope ps(ctx, COMPACT_K_ATTN_DECODE, s);
        const int ct = (int64_t)a.max_new * G > 16 ? 2 : 1;
        auto few = tiles ? attn_paged_few_kernel<HD, NP, T, true, 2> : ct == 2 ? attn_paged_few_kernel<HD, NP, T, false, 2> : attn_paged_few_kernel<HD, NP, T, false, 1>;
        const int slot_cols = std::min(a.max_new, FEW_COLS / G) * G, slot_bytes = slot_cols * (HD + 4) * (int)sizeof(float);
        const int slots = std::max(1, std::min(FEW_REC_SLOTS, (16 << 10) / slot_bytes));
        few<<<(unsigned)std::min<int64_t>(most, few_resident(HD, NP, ct) * n_cus), FEW_WAVES * 64, slots * slot_bytes, s>>>(a, slot_cols, slots);
    }
    LAUNCH_CHECK(ctx);
    if (tiles) TRY_RC(launch_attn_paged_tiles(ctx, a, s));
    if (a.n_rec == 0) return COMPACT_OK;
    // rows of a request whose keys may be split: 2 t <= t p for its t tiles
    const int64_t few_rows = std::min(a.max_new, FEW_COLS / G), tile_rows = (int64_t)TILE_COLS * most_split(a.max_kv) / 2 / G + 1;
    const int64_t rows = tiles ? std::min<int64_t>(a.max_new, std::max(few_rows, tile_rows)) : few_rows;
    if (tiles) {
        const int64_t pairs = rows * a.kv.n_requests * c.n_q_heads;
        if (pairs > INT32_MAX) return set_err(ctx, COMPACT_ESHAPE, "too many rows of split requests for one call");
        attn_paged_merge_share_kernel<HD, T><<<(unsigned)std::min<int64_t>(pairs, 4 * n_cus), 256, 0, s>>>(a);
    } else {
        // query heads per workgroup: one while that gives no more workgroups than run at once (64 rows of 32 heads by fours 5.2 us
        // instead of 5.8, one row 0.5 more), or some thousand where all four wavefronts join a pair; else four and more
        const int limit = wave_each<HD>((a.max_kv - 1) / FEW_CHUNK + 1) ? 1024 : 4096;
        int heads = 1;
        while (heads < c.n_q_heads && rows * a.kv.n_requests * ((c.n_q_heads + heads - 1) / heads) > limit) heads = std::max(4, 2 * heads);
        const int64_t wgs = rows * a.kv.n_requests * ((c.n_q_heads + heads - 1) / heads);   // (at most 32 rows of 4096 requests)
        attn_paged_merge_kernel<HD, T><<<(unsigned)wgs, 256, 0, s>>>(a, (int)rows, heads);
    }
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
    if (n_rows == 0) return COMPACT_OK;
    if (!d_cu || !d_kv_len || !d_q || !d_o) return set_err(ctx, COMPACT_EINVAL, "null cu, kv_len, q or o");
    const compact_layer_cfg& c = ctx->cfg;
    if (q_stride < (int64_t)c.n_q_heads * c.head_dim || q_stride % 8 != 0)
        return set_err(ctx, COMPACT_EINVAL, "q_stride must be at least n_q_heads * head_dim and a multiple of 8");
    if (((uintptr_t)d_q | (uintptr_t)d_o) & 15) return set_err(ctx, COMPACT_EINVAL, "q and o must be 16-byte aligned");
    max_new = std::min(max_new, n_rows);
    if (!d_workspace || ((uintptr_t)d_workspace & 15) || ws_bytes < paged_workspace(c, kv->n_requests, n_rows, max_new, max_kv_len))
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
    const RecordLayout records = record_layout(c, kv->n_requests, n_rows, max_new, a.max_kv);
    a.rec_req = (int)records.per_req;   // (at most 128 * (2^22 + 1))
    a.rec_row = (int)records.per_row;
    a.n_rec = records.total * c.n_q_heads;
    a.sched = (int32_t*)d_workspace;
    a.rec = (float*)((char*)d_workspace + align_up(SCHED_BYTES, 256));
    const bool b = c.dtype == COMPACT_BF16;
    auto launch = c.head_dim == 128 ? (b ? launch_attn_paged<128, 1, bf16> : launch_attn_paged<128, 3, float>)
                                    : (b ? launch_attn_paged<64, 1, bf16> : launch_attn_paged<64, 3, float>);
    return launch(ctx, a, (hipStream_t)hip_stream);
}
