// Attention over the paged cache in 8 bits for prompts and chunks of prompts: tiles of 128 query columns.
#include <algorithm>
#include <numeric>
#include <type_traits>

#include "attn_paged.h"
#include "vecio.h"

// Chunk swizzles of the LDS tiles (16-byte chunks; the LDS has 64 banks of 4 bytes and serves a 16-byte read 16 lanes at a
// time): rows of 16 chunks by row % 16, rows of 8 chunks by (row / 2) % 8.
template <int CHUNKS>
__device__ __forceinline__ int swz(int row) { return CHUNKS == 16 ? (row & 15) : ((row >> 1) & 7); }

// Which 16 codes of a tile a thread stages (rows of 4 pieces or of 8): a permutation within 16 lanes.  A 16-byte LDS write
// takes 8 lanes at a time on 32 banks, and a lane writes every other chunk, so that lanes 4 to 7 stand on a row whose swizzle
// is odd where that of lanes 0 to 3 is even (in order, every write took twice its time, a quarter of the LDS's; 8 prompts of
// 4096 rows 1090 us instead of 1074).
struct Piece {
    int row, part;
};
template <int PARTS>
__device__ __forceinline__ Piece staged_piece(int t) {
    if (PARTS == 8) return {(t >> 4) * 2 + (t >> 2 & 1), (t & 3) + (t >> 1 & 4)};
    return {(t >> 4) * 4 + (t >> 1 & 2) + (t >> 3 & 1), t & 3};
}

// Which XCD goes through which units of which KV heads: XCD x takes the heads x % xcd_heads + k * xcd_heads, shared with the
// other XCDs of the same heads unit by unit.
__device__ __forceinline__ int units_of_xcd(int x, int units, int Hkv, int xcd_heads) {
    const int share = 8 / xcd_heads, s = x / xcd_heads, all = units * (Hkv / xcd_heads);
    return (all - s + share - 1) / share;
}

// ---------------------------------------------------------------------------
// A unit is (request, tile of 128 query columns, piece of its keys, KV head): the columns of a KV head are its request's
// rows times the query heads of the group, so that a tile's heads share the keys.  A workgroup of four wavefronts takes units
// until there are none; a wavefront owns 32 columns and keeps Q^T in registers.  S^T = K Q^T and O^T += V^T P^T by
// v_mfma_f32_32x32x16_bf16: one query column in one lane column, so that the maxima and sums of the softmax stay in the lane
// but for one shuffle, and P^T feeds the second product from the accumulator registers (the MFMA rows of S^T are
// assigned to keys such that a lane's 8 values of a k-step are 8 consecutive keys).
// ---------------------------------------------------------------------------
struct Unit {
    PagedReq rq;
    int req, kvh, piece, pieces, cols;
    int row, head;            // of this lane's column (columns past the last one stand for it)
    int sees, sees_lo;        // keys that this lane's column sees, and the wavefront's first one
    int k_lo, k_hi, n_steps;  // keys of the piece that the workgroup's columns see, in steps of 64
    bool live;                // whether the column is there
};
// Which unit a workgroup takes next: its place in its XCD's list, -1 at the end.  The first one follows from its number, the others
// from a counter that the XCD's workgroups share, so that units of different lengths even out (the lists of the XCDs are as
// long as each other by themselves: every KV head has the same units).  One counter per 128-byte line: with all in one
// line and for the first unit too the 512 workgroups stood 54 us in line, whatever the call.
__device__ __forceinline__ int next_place(const PagedAttnArgs& a, int mine, int n, int* s_place) {
    const int wgs = gridDim.x >> 3;
    if (mine < 0) return (int)(blockIdx.x >> 3) < n ? (int)(blockIdx.x >> 3) : -1;
    if (n <= wgs) return -1;
    __syncthreads();
    if (threadIdx.x == 0) *s_place = atomicAdd(&a.sched[(blockIdx.x & 7) * SCHED_PITCH], 1) + wgs;
    __syncthreads();
    mine = __builtin_amdgcn_readfirstlane(*s_place);
    return mine < n ? mine : -1;
}
// `wave`: which 32 columns of the tile the wavefront owns
__device__ __forceinline__ Unit unit_at(const PagedAttnArgs& a, int mine, int units, int xcd_heads, int wave) {
    Unit un;
    const int r = threadIdx.x & 31, lane = threadIdx.x & 63, x = blockIdx.x & 7;
    const int G = a.Hq / a.Hkv, N = a.sched[SCHED_LISTED];
    const int32_t* before = a.sched + SCHED_UNITS;
    const int at = mine * (8 / xcd_heads) + x / xcd_heads;
    const int unit = at % units;
    un.kvh = at / units * xcd_heads + x % xcd_heads;
    int k = 0;   // the last request in the schedule with no more than `unit` units before it
    for (int i0 = 0; i0 < N; i0 += 64) {
        const uint64_t upto = __ballot(i0 + lane < N && before[min(i0 + lane, N)] <= unit);
        if (upto == 0) break;
        k = i0 + 63 - __builtin_clzll(upto);
    }
    const int req = a.sched[SCHED_ORDER + k];
    un.req = req;
    const PagedReq rq = un.rq = paged_req(a, req);
    const int tiles = n_tiles(rq.n, G), in_req = unit - before[k];
    un.pieces = tile_pieces(tiles, rq.kv);
    const int tile = tiles - 1 - in_req / un.pieces, c0 = tile * TILE_COLS;   // most keys first
    un.piece = in_req % un.pieces;
    un.cols = min(rq.n * G - c0, TILE_COLS);
    const int span = tile_piece_rows(un.pieces, rq.kv);
    const int col = min(wave * 32 + r, un.cols - 1) + c0;
    un.live = wave * 32 + r < un.cols;
    un.row = col / G;
    un.head = un.kvh * G + col % G;
    const int first = rq.kv - rq.n + 1;   // keys that row 0 sees (or none)
    un.sees = max(first + un.row, 0);
    un.sees_lo = max(first + (c0 + min(wave * 32, un.cols - 1)) / G, 0);
    un.k_lo = un.piece * span;
    un.k_hi = min(min(un.k_lo + span, max(first + (c0 + un.cols - 1) / G, 0)), rq.kv);
    un.n_steps = max((un.k_hi - un.k_lo + TILE_KEYS - 1) / TILE_KEYS, 0);
    return un;
}

// Normalised rows, or the piece's record.  Lane (column r): elements d * 32 + (e / 4) * 8 + h * 4 + e % 4; m, l: reference and
// sum of the column (l = 0: it saw nothing).
template <int HD, typename T>
__device__ __forceinline__ void put_unit(const PagedAttnArgs& a, const Unit& un, const floatx16 (&oacc)[HD / 32], float m, float l) {
    const int h = (threadIdx.x & 63) >> 5;
    if (!un.live) return;
    if (un.pieces == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        T* op = (T*)a.o + ((size_t)(un.rq.row0 + un.row) * a.Hq + un.head) * HD + h * 4;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) put4(op + d * 32 + g * 8, oacc[d][4 * g] * inv, oacc[d][4 * g + 1] * inv, oacc[d][4 * g + 2] * inv, oacc[d][4 * g + 3] * inv);
    } else {
        const int64_t rec = first_record(a, un.req, un.rq.row0, un.row, un.head, un.pieces) + un.piece;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) put4(a.rec + rec * HD + d * 32 + g * 8 + h * 4, oacc[d][4 * g], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]);
        if (h == 0) *reinterpret_cast<float2*>(a.rec + a.n_rec * HD + rec * 2) = make_float2(l == 0.f ? -3e38f : m, l);
    }
}

// fp32 storage: queries and probabilities as three bf16 parts each (all 24 bits), the codes exact in bf16.  Steps of 64 keys: the
// codes of the next one are in flight in registers while this one is computed, are expanded once per workgroup and go to LDS.
// Bound by its own order (scores, softmax, output one behind the other in a wavefront, one wavefront per SIMD): 8 prompts of
// 1024 rows, 4 + 2 heads of 64, 47 us, 0.27 PFLOP/s of bf16 products.  This storage is for checking.
template <int HD>
__global__ __launch_bounds__(256, 1) void attn_paged_tile_f32_kernel(const PagedAttnArgs a, int xcd_heads) {
    constexpr int NP = 3;
    constexpr int KK = HD / 16, DT = HD / 32, KCH = HD / 8;
    constexpr int KTILE = TILE_KEYS * HD;
    constexpr int NLD = KTILE / 16 / 256;   // 16-byte pieces of codes per thread and tile
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16* lds = reinterpret_cast<bf16*>(smem);   // [2 K tiles | 2 V^T tiles]
    __shared__ int s_place;
    const int Hkv = a.Hkv;
    const int t = threadIdx.x, lane = t & 63;
    const int r = lane & 31, h = lane >> 5;
    const int shift = a.kv.page_shift, P = 1 << shift;
    const int units = a.sched[SCHED_UNITS + a.sched[SCHED_LISTED]];
    const int pi_r = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);

    const int n_mine = units_of_xcd(blockIdx.x & 7, units, Hkv, xcd_heads);
    for (int mine = -1; (mine = next_place(a, mine, n_mine, &s_place)) >= 0;) {
        const Unit un = unit_at(a, mine, units, xcd_heads, wave_index());
        __syncthreads();   // (the tiles of the unit before have been read)
        const PagedReq& rq = un.rq;
        const int req = un.req, kvh = un.kvh, k_lo = un.k_lo, n_steps = un.n_steps;

        // Q^T operand: lane (column r, h) holds elements kk * 16 + h * 8 .. + 7
        bf16x8 qf[NP][KK];
        {
            const float* qp = (const float*)a.q + (size_t)(rq.row0 + un.row) * a.q_stride + un.head * HD + h * 8;
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
        float m = -3e38f, l = 0.f;   // (finite where a column sees nothing: its probabilities are exp2(-inf) = 0)

        // ---- staging: piece i is K row i * 4096 / HD + kp.row, elements kp.part * 16 .., and V element i * 64 + vp.row, rows
        // vp.part * 16 ..
        const Piece kp = staged_piece<HD / 16>(t), vp = staged_piece<4>(t);
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
                const int krow = i * (4096 / HD) + kp.row;
                const size_t ph = (size_t)place(krow / PAGED_GRAN) * Hkv + kvh;
                ksc[i] = e8m0(a.kv.ks[ph]);
                kreg[i] = *reinterpret_cast<const uintx4*>(a.kv.k + ((ph << shift) + ((k0 + krow) & (P - 1))) * HD + kp.part * 16);
            }
            const size_t ph = (size_t)place(vp.part) * Hkv + kvh;
            vsc = e8m0(a.kv.vs[ph]);
#pragma unroll
            for (int i = 0; i < NLD; ++i)
                vreg[i] = *reinterpret_cast<const uintx4*>(a.kv.v + ((ph * HD + i * 64 + vp.row) << shift) + ((k0 + vp.part * PAGED_GRAN) & (P - 1)));
        };
        auto stage = [&](int step) {
            const int live = rq.kv - (k_lo + step * TILE_KEYS) - vp.part * PAGED_GRAN;   // cached rows of this thread's V pieces
            bf16* ks = lds + (step & 1) * KTILE;
            bf16* vs = lds + (2 + (step & 1)) * KTILE;
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                const int krow = i * (4096 / HD) + kp.row, kc = kp.part * 2, vrow = i * 64 + vp.row, vc = vp.part * 2;
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
            if (k0 + TILE_KEYS > min(un.sees_lo, un.k_hi)) {
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (k0 + 32 * tt + (e >> 3) * 16 + h * 8 + (e & 7) >= min(un.sees, un.k_hi)) sc[tt][e] = -INFINITY;
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
        l += __shfl_xor(l, 32, 64);
        put_unit<HD, float>(a, un, oacc, m, l);
    }
}

// Waits for this wavefront's LDS operations, then for the other wavefronts; loads from memory stay in flight.
__device__ __forceinline__ void tile_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));   // lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#endif
}
__device__ __forceinline__ unsigned pack_bf16x2(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector(floatx2{a, b}, bf16x2));
}

// bf16 storage.  The three parts of the work on 32 keys (scores, softmax, output) run one behind the other inside a wavefront:
// while the matrix pipe forms the scores of half step n + 1 and the output of n - 1, the vector ALU does the softmax of n, in
// an order that is written out, as the slab path's prefill attention does it.  What the pages add: the codes of a K tile are
// requested two steps before their use and those of a V tile as well, into registers; a step later they are expanded to bf16 (exact), once
// per workgroup, and go to LDS between the matrix instructions, a piece of 16 codes every four of them.
// A probability is rounded to bf16 for the second product (a part more would cost half of the matrix time again: the error against 64 bits
// is 0.002, of the output's rounding alone 0.0017); the sums are of the values before the rounding.
// Bound (8 prompts of 4096 rows, 32 + 8 heads of 128: 1.10 TFLOP in 1076 us, 1.02 PFLOP/s where a large product reaches 1.27): no pipe
// alone.  The matrix pipes are busy 54 % of the cycles, the vector ALU issues in 55 %, the LDS works in 41 %, at 1.9 GHz of 2.4; without
// the exponentials 1044 us, with half of the fragments' reads 1056, without the staging 982.  64 columns per wavefront would halve
// the reads, but the scores then go through the accumulator registers: 1309.
template <int HD>
__global__ __launch_bounds__(256, 2) void attn_paged_tile_kernel(const PagedAttnArgs a, int xcd_heads) {
    constexpr int KK = HD / 16, DT = HD / 32, KCH = HD / 8, LHD = HD == 128 ? 7 : 6;
    constexpr int KTILE = TILE_KEYS * HD;
    constexpr int NLD = KTILE / 16 / 256;   // 16-byte pieces of codes per thread and tile
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16* lds = reinterpret_cast<bf16*>(smem);   // [2 K tiles | 2 V^T tiles]
    __shared__ int s_place;
    const int Hkv = a.Hkv;
    const int t = threadIdx.x, lane = t & 63, wave = wave_index();
    const int r = lane & 31, h = lane >> 5;
    const int shift = a.kv.page_shift, P = 1 << shift;
    const int units = a.sched[SCHED_UNITS + a.sched[SCHED_LISTED]];
    const int pi_r = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);
    const float scale_log2 = a.scale_log2;
    // (the other way round in the CU's second workgroup: tiles of up to 64 columns then load all four SIMDs)
    const int columns = blockIdx.x < gridDim.x / 2 ? wave : 3 - wave;

    // LDS byte offsets of the fragments of a tile: K row pi_r (the second half 32 rows on, same swizzle), V^T row r
    int kfo[KK], vfo[4];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kfo[kk] = 2 * (pi_r * HD + (((kk * 2 + h) ^ swz<KCH>(pi_r)) << 3));
#pragma unroll
    for (int u = 0; u < 4; ++u) vfo[u] = 2 * (r * TILE_KEYS + (((u * 2 + h) ^ swz<8>(r)) << 3));
    auto k_frag = [&](int stage, int tt, int kk) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>(smem + kfo[kk] + 2 * (stage * KTILE + tt * 32 * HD));
    };
    auto v_frag = [&](int stage, int d, int u) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>(smem + vfo[u] + 2 * ((2 + stage) * KTILE + d * 32 * TILE_KEYS));
    };
    auto zeros = []() __attribute__((always_inline)) {
        floatx16 z;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.f;
        return z;
    };
    // ---- staging: K row k_row, elements k_part * 16 .., in the wavefront's granule; V element v_row, granule v_gran = lane % 4
    const Piece kp = staged_piece<HD / 16>(t), vp = staged_piece<4>(t);
    const int k_part = kp.part, k_row = kp.row;                               // (piece i: 4096 / HD rows further on)
    const int k_off = (k_row & 15) * HD + k_part * 16;                        // byte offset in its granule
    const int v_gran = vp.part, v_row = vp.row;                               // (piece i: 64 elements further on)
    auto k_gran = [&](int i) __attribute__((always_inline)) { return (i * (4096 / HD) + wave * (1024 / HD)) >> 4; };

    const int n_mine = units_of_xcd(blockIdx.x & 7, units, Hkv, xcd_heads);
    for (int mine = -1; (mine = next_place(a, mine, n_mine, &s_place)) >= 0;) {
        const Unit un = unit_at(a, mine, units, xcd_heads, columns);
        __syncthreads();   // (the tiles of the unit before have been read)
        const int kv = un.rq.kv, k_lo = un.k_lo, n_tiles = un.n_steps;
        floatx16 oacc[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) oacc[d] = zeros();
        float l_run = 0.f, l_even = 0.f;   // sums of the probabilities: of whole tiles, and of a tile's first half
        float neg_m = 0.f;                 // the scaling reference, negated
        if (n_tiles > 0) {
            // Q^T operand: lane (column r, h) holds elements kk * 16 + h * 8 .. + 7
            bf16x8 qf[KK];
            const bf16* qp = (const bf16*)a.q + (size_t)(un.rq.row0 + un.row) * a.q_stride + un.head * HD + h * 8;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);

            // page of this lane's granule (lane % 4) of a tile; tiles past the last one and rows past the cached ones
            // stand for the last cached row
            const int32_t* table = a.kv.table + (size_t)un.req * a.kv.max_pages;
            auto load_pid = [&](int tile) __attribute__((always_inline)) {
                return table[min(k_lo + tile * TILE_KEYS + v_gran * PAGED_GRAN, kv - 1) >> shift];
            };
            auto in_range = [&](int pid) __attribute__((always_inline)) { return min(max(pid, 0), a.kv.n_pages - 1); };
            uintx4 kreg[NLD], vreg[NLD];
            unsigned ksb, vsb;   // scale bytes of the lane's granule
            const uint8_t* kpage[NLD];
            const uint8_t* vpage;
            // requests for K tile `tile` (in pages pid) are made ready, and sent piece by piece
            auto k_ready = [&](int tile, int pid) __attribute__((always_inline)) {
                const unsigned ph = (unsigned)pid * Hkv + un.kvh;
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    const unsigned p = __builtin_amdgcn_readlane(ph, k_gran(i));
                    kpage[i] = a.kv.k + (((size_t)p << shift) + ((k_lo + tile * TILE_KEYS + k_gran(i) * PAGED_GRAN) & (P - 1))) * HD;
                }
                return a.kv.ks[ph];
            };
            auto v_ready = [&](int tile, int pid) __attribute__((always_inline)) {
                const unsigned ph = (unsigned)pid * Hkv + un.kvh;
                vpage = a.kv.v + ((((size_t)ph << LHD) + v_row) << shift) + ((k_lo + tile * TILE_KEYS + v_gran * PAGED_GRAN) & (P - 1));
                return a.kv.vs[ph];
            };
            auto k_load = [&](int i) __attribute__((always_inline)) { kreg[i] = *reinterpret_cast<const uintx4*>(kpage[i] + k_off); };
            auto v_load = [&](int i) __attribute__((always_inline)) { vreg[i] = *reinterpret_cast<const uintx4*>(vpage + (i * 64 << shift)); };
            // pieces that have arrived go to LDS
            auto k_put = [&](int stage, int i) __attribute__((always_inline)) {
                const float sc = e8m0(__builtin_amdgcn_readlane(ksb, k_gran(i)));
                const int row = i * (4096 / HD) + k_row;
                bf16* dst = lds + stage * KTILE + row * HD;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<bf16x8*>(dst + ((k_part * 2 + j) ^ swz<KCH>(row)) * 8) = codes8_to_bf16(kreg[i][2 * j], kreg[i][2 * j + 1], sc);
            };
            auto v_put = [&](int stage, int i) __attribute__((always_inline)) {
                const float sc = e8m0(vsb);
                const int row = i * 64 + v_row;
                bf16* dst = lds + (2 + stage) * KTILE + row * TILE_KEYS;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<bf16x8*>(dst + ((v_gran * 2 + j) ^ swz<8>(row)) * 8) = codes8_to_bf16(vreg[i][2 * j], vreg[i][2 * j + 1], sc);
            };
            // whatever lies behind the cached rows must not reach the MFMA
            auto v_trim = [&](int tile) __attribute__((always_inline)) {
                const int live = kv - (k_lo + tile * TILE_KEYS);
                if (__builtin_expect(live >= TILE_KEYS, 1)) return;
#pragma unroll
                for (int i = 0; i < NLD; ++i)
#pragma unroll
                    for (int wd = 0; wd < 4; ++wd) vreg[i][wd] &= low_bytes(live - v_gran * PAGED_GRAN - 4 * wd);
            };

            // a wavefront without columns only stages (80 requests of up to 60 rows behind up to 3000: 158 -> 149 us)
            if (columns * 32 >= un.cols) {
                int pid_k = in_range(load_pid(0)), pid_v = pid_k, pid_n = load_pid(1);
                auto request = [&](int J) __attribute__((always_inline)) {   // K of tile J, V^T of tile J - 1
                    ksb = k_ready(J, pid_k);
                    vsb = v_ready(J - 1, pid_v);
#pragma unroll
                    for (int i = 0; i < NLD; ++i) {
                        k_load(i);
                        v_load(i);
                    }
                    pid_v = pid_k;
                    pid_k = in_range(pid_n);
                    pid_n = load_pid(J + 2);
                };
                ksb = k_ready(0, pid_k);
#pragma unroll
                for (int i = 0; i < NLD; ++i) k_load(i);
                pid_k = in_range(pid_n);
                pid_n = load_pid(2);
#pragma unroll
                for (int i = 0; i < NLD; ++i) k_put(0, i);
                request(1);
                tile_barrier();
                for (int J = 1; J <= n_tiles; ++J) {
                    v_trim(J - 1);
#pragma unroll
                    for (int i = 0; i < NLD; ++i) {
                        k_put(J & 1, i);
                        v_put((J - 1) & 1, i);
                    }
                    request(J + 1);
                    tile_barrier();
                }
                continue;
            }

            floatx16 se, so;      // S^T of two halves of 32 keys: column r, key 32 n + (e / 8) * 16 + h * 8 + e % 8
            uintx4 pe[2], po[2];  // their P^T
            const int lim = min(un.sees, un.k_hi) - k_lo, lim_lo = min(un.sees_lo, un.k_hi) - k_lo;
            auto prob = [&](float v) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(__builtin_fmaf(v, scale_log2, neg_m)); };
            auto probs = [&](float ps, const floatx16& s, uintx4 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float u = prob(s[e]), v = prob(s[e + 1]);
                    ps += u;
                    ps += v;
                    p[e >> 3][(e >> 1) & 3] = pack_bf16x2(u, v);
                }
                return ps;
            };
            auto mask = [&](int n, floatx16& s) __attribute__((always_inline)) {
                if (__builtin_expect(n * 32 + 32 <= lim_lo, 1)) return;   // every column of the wavefront sees all of it
                const int q = here(lim) - n * 32 - h * 8;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((e >> 3) * 16 + (e & 7) >= q) s[e] = -INFINITY;
            };
            // The running maximum is only a scaling reference: the first tile takes its own, and while every lane's sum
            // of a tile's 32 values stays below 2^12 against the reference as it stands, it stays (fp32 sums and bf16
            // probabilities carry them without loss).  Otherwise the exact maximum is taken, the accumulators are rescaled and
            // the probabilities formed again.  A first half takes the maximum of its whole tile.  (A column that
            // sees nothing of the first tile sees nothing of the others.)
            auto settle = [&](int n, float ps, bool odd, bool first, const floatx16& s, floatx16& other, uintx4 (&p)[2])
                              __attribute__((always_inline)) {
                if (__builtin_expect(first || __any(!(ps < 4096.0f)), 0)) {
                    float mx = -INFINITY;
                    if (!odd) mask(n + 1, other);
#pragma unroll
                    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, odd ? s[e] : fmaxf(s[e], other[e]));
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    mx = mx == -INFINITY ? 0.f : __builtin_fmaf(mx, scale_log2, neg_m);
                    const float up = first ? mx : fmaxf(mx, 0.f);
                    const float corr = first ? 1.f : __builtin_amdgcn_exp2f(-up);
                    l_run *= corr;
                    neg_m -= up;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) oacc[d][e] *= corr;
                    ps = probs(odd ? l_even * corr : 0.f, s, p);
                }
                if (odd)
                    l_run += ps;
                else
                    l_even = ps;
            };

            // Step J, with K of tile J and V^T of tile J - 1 in LDS, is twice (n = 2J - 1, then n = 2J) QK^T of half
            // n + 1, softmax of half n and PV of half n - 1.  Its first half also puts K of tile J + 1 and V^T of tile J
            // into LDS and sends for those after them.
            constexpr int NM = 2 * KK, AHEAD = 4, PER = 16 / NM, PRE = 2 / PER;
            static_assert(KK == 2 * DT && NM / 4 == 2 * NLD, "as many MFMAs in either product, four to a piece");
            bf16x8 fr[2 * NM];
            int pid_v, pid_k, pid_n;   // pages of tiles J + 1, J + 2, and J + 3 (as loaded)
            unsigned ks_n = 0, vs_n = 0;
            auto half_step = [&](auto ptag, auto stag, int J, floatx16& sc, floatx16& sn, const uintx4 (&pp)[2], uintx4 (&pn)[2])
                                 __attribute__((always_inline)) {
                constexpr int part = decltype(ptag)::value, stage = decltype(stag)::value;   // stage of K; V^T lies in the other one
                auto read = [&](int g) __attribute__((always_inline)) {
                    const int i = g % NM, tt = g / NM, m = i / 2;
                    fr[g] = i & 1 ? v_frag(1 - stage, m % DT, 2 * tt + m / DT) : k_frag(stage, tt, m);
                };
                float ps = part == 0 ? l_even : 0.f, pv[16];   // part 0 is an odd half
                auto add = [&](int e) __attribute__((always_inline)) {
                    ps += pv[e];
                    if (e & 1) pn[e >> 3][(e >> 1) & 3] = here((int)pack_bf16x2(pv[e - 1], pv[e]));   // not sunk below the branch
                };
                if (part == 0) {
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) read(i);
                    v_trim(J);
                }
                mask(2 * J - 1 + part, sc);
#pragma unroll
                for (int e = 0; e < PRE * PER; ++e) pv[e] = prob(sc[e]);
#pragma unroll
                for (int i = 0; i < NM; ++i) {
                    const int g = part * NM + i, m = i / 2;
                    __builtin_amdgcn_sched_barrier(0);
                    if (g + AHEAD < 2 * NM) read(g + AHEAD);
                    if (i & 1)
                        oacc[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[g], __builtin_bit_cast(bf16x8, pp[m / DT]), oacc[m % DT], 0, 0, 0);
                    else
                        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[g], qf[m], m ? sn : zeros(), 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = (i + PRE) * PER; e < (i + PRE + 1) * PER && e < 16; ++e) pv[e] = prob(sc[e]);
#pragma unroll
                    for (int e = i ? (i + PRE - 1) * PER : 0; e < (i + PRE) * PER && e < 16; ++e) add(e);
                    if (part == 0) {
                        const int piece = i >> 2;
                        if (i == 0) {   // where the next requests go; tile J + 3's pages
                            pid_v = pid_k;
                            pid_k = in_range(pid_n);
                            ks_n = k_ready(J + 2, pid_k);
                            vs_n = v_ready(J + 1, pid_v);
                            pid_n = load_pid(J + 3);
                        }
                        if ((i & 3) == 2) {
                            if (piece < NLD) {
                                k_put(1 - stage, piece);
                                k_load(piece);
                            } else {
                                v_put(stage, piece - NLD);
                                v_load(piece - NLD);
                            }
                        }
                        if (i == NM - 1) {
                            ksb = ks_n;
                            vsb = vs_n;
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                settle(2 * J - 1 + part, ps, part == 0, false, sc, sn, pn);
            };
            auto step = [&](auto stag, int J) __attribute__((always_inline)) {
                half_step(std::integral_constant<int, 0>{}, stag, J, so, se, pe, po);
                half_step(std::integral_constant<int, 1>{}, stag, J, se, so, po, pe);
                tile_barrier();
            };
            // K of tile 0 to LDS; K of tile 1 and V^T of tile 0 requested, then their successors
            const int pid0 = in_range(load_pid(0)), pid1 = in_range(load_pid(1));
            pid_k = in_range(load_pid(2));
            pid_n = load_pid(3);
            ksb = k_ready(0, pid0);
#pragma unroll
            for (int i = 0; i < NLD; ++i) k_load(i);
#pragma unroll
            for (int i = 0; i < NLD; ++i) k_put(0, i);
            ksb = k_ready(1, pid1);
            vsb = v_ready(0, pid0);
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                k_load(i);
                v_load(i);
            }
            tile_barrier();
#pragma unroll
            for (int m = 0; m < KK; ++m) {
                se = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(0, 0, m), qf[m], m ? se : zeros(), 0, 0, 0);
                so = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(0, 1, m), qf[m], m ? so : zeros(), 0, 0, 0);
            }
            mask(0, se);
            settle(0, 0.f, false, true, se, so, pe);
            v_trim(0);
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                k_put(1, i);
                v_put(0, i);
            }
            ksb = k_ready(2, pid_k);
            vsb = v_ready(1, pid1);
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                k_load(i);
                v_load(i);
            }
            tile_barrier();
            int J = 1;
#pragma unroll 1
            for (; J + 1 < n_tiles; J += 2) {
                step(std::integral_constant<int, 1>{}, J);
                step(std::integral_constant<int, 0>{}, J + 1);
            }
            if (J < n_tiles) step(std::integral_constant<int, 1>{}, J++);
            // the last tile's second half: no scores to form
            {
                const int stage = (J - 1) & 1, n = 2 * J - 1;
                mask(n, so);
                const float ps = probs(l_even, so, po);
#pragma unroll
                for (int m = 0; m < KK; ++m)
                    oacc[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(stage, m % DT, m / DT), __builtin_bit_cast(bf16x8, pe[m / DT]),
                                                                           oacc[m % DT], 0, 0, 0);
                settle(n, ps, true, false, so, se, po);
#pragma unroll
                for (int m = 0; m < KK; ++m)
                    oacc[m % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(stage, m % DT, 2 + m / DT), __builtin_bit_cast(bf16x8, po[m / DT]),
                                                                           oacc[m % DT], 0, 0, 0);
            }
        }
        l_run += __shfl_xor(l_run, 32, 64);
        put_unit<HD, bf16>(a, un, oacc, -neg_m, l_run);
    }
}

template <int HD>
static int launch_tiles(compact_ctx* ctx, const PagedAttnArgs& a, bool b, hipStream_t s) {
    auto kern = b ? attn_paged_tile_kernel<HD> : attn_paged_tile_f32_kernel<HD>;
    const size_t smem = (size_t)4 * TILE_KEYS * HD * sizeof(bf16);
    if (!ctx->paged_lds_set) {   // (a context has one storage type and head_dim: one of the kernels)
        HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        ctx->paged_lds_set = true;
    }
    int n_cus = 0;
    if (int rc = device_cu_count(ctx, &n_cus)) return rc;
    ProfileScope ps(ctx, COMPACT_K_ATTN_PREFILL, s);
    const int grid = std::max(2 * n_cus / 8, 1) * 8;   // as many workgroups as stay resident; as many on every XCD
    kern<<<grid, 256, smem, s>>>(a, std::gcd(8, a.Hkv));
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

int launch_attn_paged_tiles(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s) {
    const bool b = ctx->cfg.dtype == COMPACT_BF16;
    return ctx->cfg.head_dim == 128 ? launch_tiles<128>(ctx, a, b, s) : launch_tiles<64>(ctx, a, b, s);
}
