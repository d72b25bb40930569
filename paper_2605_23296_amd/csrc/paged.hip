// Paged cache in 8 bits: the plan of a step (block table, slot map, rotary table from the requests' lengths, all on the GPU) and
// the write of new rows into the pages (rotation, scale by page and head, E4M3 codes).
#include <algorithm>
#include <cmath>

#include "paged.h"
#include "vecio.h"

#define TRY_RC(expr)                       \
    do {                                   \
        const int _rc = (expr);            \
        if (_rc != COMPACT_OK) return _rc; \
    } while (0)

int paged_view(compact_ctx* ctx, const compact_paged_kv* kv, bool with_pages, PagedView* out) {
    if (!kv) return set_err(ctx, COMPACT_EINVAL, "null paged kv");
    if (!kv->d_table) return set_err(ctx, COMPACT_EINVAL, "null block table");
    if (kv->n_pages < 1 || kv->max_pages < 1 || kv->n_requests < 1)
        return set_err(ctx, COMPACT_EINVAL, "n_pages, max_pages and n_requests must be >= 1");
    if (kv->n_requests > PAGED_MAX_REQUESTS) return set_err(ctx, COMPACT_ESHAPE, "more than 4096 requests");
    int shift = 0;
    while (shift < 7 && (1 << shift) < kv->page_rows) ++shift;
    if (kv->page_rows < PAGED_GRAN || (1 << shift) != kv->page_rows)
        return set_err(ctx, COMPACT_ESHAPE, "page_rows must be 16, 32, 64 or 128");
    if ((int64_t)kv->max_pages * kv->page_rows > INT32_MAX)
        return set_err(ctx, COMPACT_ESHAPE, "max_pages * page_rows must stay below 2^31");
    if (with_pages) {
        if (!kv->d_k || !kv->d_v || !kv->d_k_scale || !kv->d_v_scale) return set_err(ctx, COMPACT_EINVAL, "null pages or scales");
        if (((uintptr_t)kv->d_k | (uintptr_t)kv->d_v) & 15) return set_err(ctx, COMPACT_EINVAL, "d_k and d_v must be 16-byte aligned");
    }
    *out = PagedView{(uint8_t*)kv->d_k, (uint8_t*)kv->d_v, (uint8_t*)kv->d_k_scale, (uint8_t*)kv->d_v_scale, kv->d_table,
                     kv->n_pages, shift, kv->max_pages, kv->n_requests};
    return COMPACT_OK;
}

// ---------------------------------------------------------------------------
// Plan.  Three running sums over the requests decide everything: rows (cu), pages wanted (upto) and pages given back.  A request
// is granted iff it fits and the pages wanted up to and including it are there; since that sum only grows, those granted any
// pages are the first ones that want some, and the first page request i takes is number upto[i] - need[i] from the top of
// the stack.  Sums saturate at 2^31 - 1 (saturating addition of numbers that are not negative is associative).
//
// One launch: every workgroup forms the sums over all requests itself (a request's three numbers stay in LDS) and then
// handles PLAN_ROWS rows of the slot map and its share of the table and of the stack.  No workgroup reads what another one writes:
// table columns that are read lie below a request's length, those written above it; stack entries that are read lie below
// n_free, those written above; lengths and counters come in pairs.  Page numbers are copied, never followed, so whatever the
// device arrays hold, nothing outside them is touched.
// ---------------------------------------------------------------------------
#define PLAN_NT 256
#define PLAN_ROWS 64

struct PlanArgs {
    compact_paged_step st;
    PagedView kv;
    int half;             // head_dim / 2
    double log2_theta;
};

__device__ __forceinline__ int sat_add(int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7FFFFFFFu); }

// inclusive saturating sum over the workgroup's threads; `red`: one int per wavefront
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int ofs = 1; ofs < 64; ofs <<= 1) {
        const int u = __shfl_up(v, ofs, 64);
        if (lane >= ofs) v = sat_add(v, u);
    }
    __syncthreads();
    if (lane == 63) red[w] = v;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < PLAN_NT / 64; ++i) {
        if (i < w) before = sat_add(before, red[i]);
        total = sat_add(total, red[i]);
    }
    return sat_add(v, before);
}

// the last i in 0 .. n - 1 with a[i] <= x (a[0] = 0 <= x, a does not decrease)
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(PLAN_NT) void paged_plan_kernel(const PlanArgs a) {
    extern __shared__ int lds[];
    __shared__ int red[PLAN_NT / 64], s_pos[PLAN_ROWS], s_taken, s_refused;
    const compact_paged_step& st = a.st;
    const int N = a.kv.n_requests, shift = a.kv.page_shift, P = 1 << shift, width = a.kv.max_pages;
    int* cu = lds;                 // [N + 1] rows before request i
    int* back = cu + N + 1;        // [N + 1] pages given back by the requests before i
    int* want = back + N + 1;      // [N + 1] pages wanted by the requests before i
    const int t = threadIdx.x;
    const int n_free = min(max(st.d_n_free[0], 0), a.kv.n_pages);
    const int cap = width << shift;
    auto len_of = [&](int i) { return min(max(st.d_len[i], 0), cap); };
    auto pages = [&](int rows) { return (int)(((unsigned)rows + P - 1) >> shift); };
    // pages request i wants, its rows ending at packed row `end`; -1: it does not fit
    auto need_of = [&](int n, int len, int end) {
        if (n > cap - len || end > st.max_rows) return -1;
        return pages(len + n) - pages(len);
    };

    int c_cu = 0, c_back = 0, c_want = 0;
    for (int i0 = 0; i0 < N; i0 += PLAN_NT) {
        const int i = i0 + t;
        const int n_new = i < N ? st.d_n_new[i] : 0, len = i < N ? len_of(i) : 0;
        const int n = max(n_new, 0);
        int tot;
        const int end = sat_add(c_cu, block_scan(n, red, tot));
        c_cu = sat_add(c_cu, tot);
        const int gave = sat_add(c_back, block_scan(n_new < 0 ? pages(len) : 0, red, tot));
        c_back = sat_add(c_back, tot);
        const int need = n > 0 ? max(need_of(n, len, end), 0) : 0;
        const int upto = sat_add(c_want, block_scan(need, red, tot));
        c_want = sat_add(c_want, tot);
        if (i < N) {
            cu[i + 1] = end;
            back[i + 1] = gave;
            want[i + 1] = upto;
        }
    }
    if (t == 0) cu[0] = back[0] = want[0] = s_taken = s_refused = 0;
    __syncthreads();
    const int total = min(sat_add(n_free, back[N]), a.kv.n_pages);   // pages there are
    auto granted = [&](int i, int n, int len) {
        if (n <= 0) return false;
        const int need = need_of(n, len, cu[i + 1]);
        return need == 0 || (need > 0 && want[i + 1] <= total);
    };
    // the page at position v of the stack once the pages given back lie on it
    auto stack = [&](int v) {
        if (v < n_free) return st.d_free[v];
        const int i = last_at_most(back, N + 1, v - n_free);
        return a.kv.table[(size_t)i * width + (v - n_free - back[i])];
    };
    // per request: length, pages taken in all
    {
        int taken = 0, refused = 0;
        for (int i = t; i < N; i += PLAN_NT) {
            const int n_new = st.d_n_new[i], len = len_of(i);
            const bool ok = granted(i, n_new, len);
            if (ok && want[i + 1] > want[i]) taken = want[i + 1];   // (they do not decrease)
            refused += n_new > 0 && !ok;
            if (blockIdx.x == 0) {
                st.d_len_out[i] = n_new < 0 ? 0 : ok ? len + n_new : len;
                st.d_kv_len[i] = ok ? len + n_new : 0;
                st.d_cu[i + 1] = cu[i + 1];
                if (i == 0) st.d_cu[0] = 0;
            }
        }
        if (taken) atomicMax(&s_taken, taken);
        if (refused) atomicAdd(&s_refused, refused);
    }
    __syncthreads();
    const int taken = s_taken, left = total - taken;
    if (blockIdx.x == 0 && t == 0) {
        st.d_n_free_out[0] = left;
        st.d_n_refused[0] = s_refused;
    }
    const int gt = blockIdx.x * PLAN_NT + t, all = gridDim.x * PLAN_NT;
    for (int v = n_free + gt; v < left; v += all) st.d_free[v] = stack(v);
    for (int k = gt; k < taken; k += all) {   // the k-th page from the top of the stack
        const int i = last_at_most(want, N + 1, k);
        a.kv.table[(size_t)i * width + pages(len_of(i)) + (k - want[i])] = stack(total - 1 - k);
    }

    // ---- slot and position of this workgroup's rows, then their rotary angles --------------------
    const int r0 = blockIdx.x * PLAN_ROWS, rows = min(PLAN_ROWS, st.max_rows - r0);
    if (t < rows) {
        const int r = r0 + t;
        int pos = 0;
        int64_t slot = -1;
        if (r < cu[N]) {
            const int i = last_at_most(cu, N + 1, r), n = cu[i + 1] - cu[i], len = len_of(i);
            pos = len + (r - cu[i]);
            if (granted(i, n, len)) {
                const int p = pos >> shift, held = pages(len);
                const int page = p < held ? a.kv.table[(size_t)i * width + p] : stack(total - 1 - (want[i] + p - held));
                slot = (int64_t)page * P + (pos & (P - 1));
            }
        }
        st.d_slot[r] = slot;
        s_pos[t] = pos;
    }
    __syncthreads();
    // the angle in fp64, as the framework's other rotations form it; PLAN_NT is a multiple of half: a thread's frequency is fixed
    const int i = t % a.half;
    const double inv_freq = exp2(-2.0 * (double)i / (double)(2 * a.half) * a.log2_theta);
    for (int idx = t; idx < rows * a.half; idx += PLAN_NT) {
        double sn, cn;
        sincos((double)s_pos[idx / a.half] * inv_freq, &sn, &cn);
        reinterpret_cast<float2*>(st.d_rot)[(size_t)r0 * a.half + idx] = make_float2((float)cn, (float)sn);
    }
}

extern "C" int compact_paged_plan(compact_ctx* ctx, const compact_paged_kv* kv, const compact_paged_step* step, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    PlanArgs a;
    TRY_RC(paged_view(ctx, kv, false, &a.kv));
    if (!step) return set_err(ctx, COMPACT_EINVAL, "null step");
    if (!step->d_n_new || !step->d_len || !step->d_n_free || !step->d_free || !step->d_n_free_out || !step->d_n_refused ||
        !step->d_len_out || !step->d_kv_len || !step->d_cu || !step->d_slot || !step->d_rot)
        return set_err(ctx, COMPACT_EINVAL, "null array in the step");
    if (step->max_rows < 1) return set_err(ctx, COMPACT_EINVAL, "max_rows must be >= 1");
    if (step->max_rows > 1 << 30) return set_err(ctx, COMPACT_ESHAPE, "max_rows must be at most 2^30");
    if (step->d_len == step->d_len_out || step->d_len == step->d_kv_len || step->d_n_new == step->d_len_out || step->d_n_new == step->d_kv_len ||
        step->d_n_free == step->d_n_free_out || step->d_n_free == step->d_n_refused || step->d_len_out == step->d_kv_len ||
        step->d_n_free_out == step->d_n_refused)
        return set_err(ctx, COMPACT_EINVAL, "an output of the step is one of its inputs or another output");
    if (((uintptr_t)step->d_rot | (uintptr_t)step->d_slot) & 7)
        return set_err(ctx, COMPACT_EINVAL, "d_rot and d_slot must be 8-byte aligned");
    a.st = *step;
    a.half = ctx->cfg.head_dim / 2;
    a.log2_theta = log2((double)ctx->cfg.rope_theta);
    const size_t smem = (size_t)3 * (kv->n_requests + 1) * sizeof(int);
    paged_plan_kernel<<<(step->max_rows + PLAN_ROWS - 1) / PLAN_ROWS, PLAN_NT, smem, (hipStream_t)hip_stream>>>(a);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

// ---------------------------------------------------------------------------
// Write.  A segment is what a call writes to one page: rows with consecutive slots.  A workgroup of two wavefronts takes a
// segment and KV head: the first its K rows (rotated on the way), the second its V rows (transposed in
// registers: a lane holds 16 rows of 8 elements and stores 16 bytes per element).  Both read their rows twice, first for the
// largest value, then (from the L2) for the codes.  Further workgroups rotate q.
// ---------------------------------------------------------------------------
#define WR_NT 128
#define WR_QHEADS 8   // most query heads per wavefront of the q part

template <typename T>
struct WriteArgs {
    const T* qkv;
    T* q;
    const int64_t* slot;
    const float2* rot;
    PagedView kv;
    int n_rows, Hq, Hkv;
    int chunk;            // rows whose segments one workgroup goes through
    int n_kv_wgs;         // workgroups of the K / V part
    int q_heads;          // query heads per wavefront of the q part
};

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

template <int HD, typename T>
__global__ __launch_bounds__(WR_NT) void paged_write_kernel(const WriteArgs<T> a) {
    constexpr int HALF = HD / 2, LPT = HALF / 8, TPW = 64 / LPT;   // K and q: lanes per row (either half), rows side by side
    constexpr int VL = HD / 8, VG = 64 / VL;                         // V: lanes across a row, granules side by side
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int Hkv = a.Hkv, ld = (a.Hq + 2 * Hkv) * HD;

    if ((int)blockIdx.x >= a.n_kv_wgs) {   // ---- q: TPW rows of q_heads heads per wavefront
        const int task = ((int)blockIdx.x - a.n_kv_wgs) * (WR_NT / 64) + wave;
        const int per_row = (a.Hq + a.q_heads - 1) / a.q_heads;
        const int row = task / per_row * TPW + lane / LPT, h0 = task % per_row * a.q_heads, d = lane % LPT * 8;
        if (row >= a.n_rows) return;
        float2 cs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = a.rot[(size_t)row * HALF + d + j];
        const T* src = a.qkv + (size_t)row * ld + d;
        T* dst = a.q + (size_t)row * a.Hq * HD + d;
        for (int h = h0; h < min(h0 + a.q_heads, a.Hq); ++h) {
            float lo[8], hi[8], olo[8], ohi[8];
            load8(src + h * HD, lo);
            load8(src + h * HD + HALF, hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) rotate(lo[j], hi[j], cs[j].x, cs[j].y, olo[j], ohi[j]);
            store8(dst + h * HD, olo);
            store8(dst + h * HD + HALF, ohi);
        }
        return;
    }

    // ---- K and V: the segments that begin in this workgroup's rows
    __shared__ unsigned bad_rows[2][4];   // rows of the segment with a value that is not finite, by wavefront
    const int kvh = blockIdx.x % Hkv, shift = a.kv.page_shift, P = 1 << shift;
    const int row_lo = (int)(blockIdx.x / Hkv) * a.chunk;
    const int64_t n_slots = (int64_t)a.kv.n_pages << shift;
    auto slot_of = [&](int row) { return row >= 0 && row < a.n_rows ? a.slot[row] : (int64_t)-1; };
    uint64_t begins;
    {
        const int row = row_lo + lane;
        const int64_t s = lane < a.chunk ? slot_of(row) : -1;
        begins = __ballot(s >= 0 && s < n_slots && ((s & (P - 1)) == 0 || slot_of(row - 1) != s - 1));
    }
    for (; begins; begins &= begins - 1) {
        const int row0 = row_lo + __builtin_ctzll(begins);
        const int64_t s0 = slot_of(row0);
        const int o = (int)(s0 & (P - 1));
        const int64_t page = s0 >> shift;
        int n = 1;   // rows of the segment: up to the page's end, as long as the slots are consecutive
        for (int j0 = 1; j0 < P - o; j0 += 64) {
            const int j = j0 + lane;
            const uint64_t ends = __ballot(j >= P - o || slot_of(row0 + j) != s0 + j);
            n = ends ? j0 + __builtin_ctzll(ends) : j0 + 64;
            if (ends) break;
        }
        n = min(n, P - o);
        const size_t ph = (size_t)page * Hkv + kvh;
        __syncthreads();   // (the rows marked for the segment before have been read)
        if (threadIdx.x < 8) bad_rows[threadIdx.x >> 2][threadIdx.x & 3] = 0;
        __syncthreads();
        if (wave == 0) {
            const int d = lane % LPT * 8, sub = lane / LPT;
            const T* src = a.qkv + (size_t)row0 * ld + (a.Hq + kvh) * HD + d;
            auto rotated = [&](int j, float (&lo)[8], float (&hi)[8]) {
                float x[8], y[8];
                load8(src + (size_t)j * ld, x);
                load8(src + (size_t)j * ld + HALF, y);
                const float2* cs = a.rot + (size_t)(row0 + j) * HALF + d;
#pragma unroll
                for (int e = 0; e < 8; ++e) rotate(x[e], y[e], cs[e].x, cs[e].y, lo[e], hi[e]);
            };
            float amax = 0.f;
            for (int j = sub; j < n; j += TPW) {
                float lo[8], hi[8];
                rotated(j, lo, hi);
                bool fine = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    fine = fine && finite(lo[e]) && finite(hi[e]);
                    amax = fmaxf(amax, fmaxf(finite(lo[e]) ? fabsf(lo[e]) : 0.f, finite(hi[e]) ? fabsf(hi[e]) : 0.f));
                }
                if (!fine) atomicOr(&bad_rows[0][j >> 5], 1u << (j & 31));
            }
            amax = wave_max(amax);
            __syncthreads();
            const int before = o > 0 ? min(max((int)a.kv.ks[ph], 1), 253) : 1, byte = max(before, scale_byte(amax));
            uint8_t* kp = a.kv.k + (ph << shift) * HD;
            if (byte > before && o > 0) {
                const float down = e8m0(max(127 + before - byte, 0));
                for (int i = lane; i < o * (HD / 16); i += 64) {
                    uintx4 w = reinterpret_cast<uintx4*>(kp)[i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = recode4(w[e], down);
                    reinterpret_cast<uintx4*>(kp)[i] = w;
                }
            }
            const float up = e8m0(254 - byte);
            for (int j = sub; j < n; j += TPW) {
                float lo[8], hi[8];
                rotated(j, lo, hi);
                uintx2 wl = {to_codes4(lo[0] * up, lo[1] * up, lo[2] * up, lo[3] * up), to_codes4(lo[4] * up, lo[5] * up, lo[6] * up, lo[7] * up)};
                uintx2 wh = {to_codes4(hi[0] * up, hi[1] * up, hi[2] * up, hi[3] * up), to_codes4(hi[4] * up, hi[5] * up, hi[6] * up, hi[7] * up)};
                if ((bad_rows[0][j >> 5] | bad_rows[1][j >> 5]) >> (j & 31) & 1) wl = wh = uintx2{0x7F7F7F7Fu, 0x7F7F7F7Fu};
                uint8_t* dst = kp + (size_t)(o + j) * HD + d;
                *reinterpret_cast<uintx2*>(dst) = wl;
                *reinterpret_cast<uintx2*>(dst + HALF) = wh;
            }
            if (lane == 0) a.kv.ks[ph] = (uint8_t)byte;
        } else {
            const int d = lane % VL * 8, sub = lane / VL;
            const T* src = a.qkv + (size_t)row0 * ld + (a.Hq + Hkv + kvh) * HD + d;
            float amax = 0.f;
            for (int j = sub; j < n; j += VG) {
                float x[8];
                load8(src + (size_t)j * ld, x);
                bool fine = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    fine = fine && finite(x[e]);
                    amax = fmaxf(amax, finite(x[e]) ? fabsf(x[e]) : 0.f);
                }
                if (!fine) atomicOr(&bad_rows[1][j >> 5], 1u << (j & 31));
            }
            amax = wave_max(amax);
            __syncthreads();
            const int before = o > 0 ? min(max((int)a.kv.vs[ph], 1), 253) : 1, byte = max(before, scale_byte(amax));
            uint8_t* vp = a.kv.v + (ph << shift) * HD;
            if (byte > before && o > 0) {
                const float down = e8m0(max(127 + before - byte, 0));
                const int per = (o + PAGED_GRAN - 1) / PAGED_GRAN;   // granules that hold rows of before
                for (int i = lane; i < per * HD; i += 64) {
                    uintx4* p = reinterpret_cast<uintx4*>(vp + (size_t)(i / per) * P + i % per * PAGED_GRAN);
                    uintx4 w = *p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned rows = low_bytes(o - i % per * PAGED_GRAN - 4 * e);   // (those behind stay as they are)
                        w[e] = (recode4(w[e], down) & rows) | (w[e] & ~rows);
                    }
                    *p = w;
                }
                wait_all_memory();   // the granule in which the new rows begin is there before single bytes of it are
            }
            const float up = e8m0(254 - byte);
            for (int g = o / PAGED_GRAN + sub; g * PAGED_GRAN < o + n; g += VG) {
                const int j0 = g * PAGED_GRAN - o;   // the granule's first row in the segment
                unsigned w[8][4];                    // [element][row / 4]
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    float x[4][8];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int j = min(max(j0 + q4 * 4 + u, 0), n - 1);
                        load8(src + (size_t)j * ld, x[u]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[u][e] = finite(x[u][e]) ? x[u][e] * up : 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e][q4] = to_codes4(x[0][e], x[1][e], x[2][e], x[3][e]);
                }
                uint8_t* dst = vp + (size_t)d * P + g * PAGED_GRAN;
                if (j0 >= 0 && j0 + PAGED_GRAN <= n) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) *reinterpret_cast<uintx4*>(dst + e * P) = uintx4{w[e][0], w[e][1], w[e][2], w[e][3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int u = 0; u < PAGED_GRAN; ++u)
                            if (j0 + u >= 0 && j0 + u < n) dst[e * P + u] = (uint8_t)(w[e][u >> 2] >> (u & 3) * 8);
                }
            }
            if (lane == 0) a.kv.vs[ph] = (uint8_t)byte;
        }
    }
}

template <int HD, typename T>
static int launch_write(compact_ctx* ctx, int n_rows, const void* qkv, const PagedView& kv, const int64_t* slot, const float* rot, void* q,
                        hipStream_t s) {
    const int Hq = ctx->cfg.n_q_heads, Hkv = ctx->cfg.n_kv_heads;
    constexpr int TPW = 64 / (HD / 16);
    WriteArgs<T> a{(const T*)qkv, (T*)q, slot, (const float2*)rot, kv, n_rows, Hq, Hkv, 1, 0, 1};
    a.chunk = n_rows <= 1024 ? 1 : n_rows <= 8192 ? 8 : 32;
    const int64_t chunks = (n_rows + a.chunk - 1) / a.chunk, groups = (n_rows + TPW - 1) / TPW;
    a.q_heads = (int)std::min<int64_t>(WR_QHEADS, std::max<int64_t>(1, groups * Hq / 4096));
    const int64_t tasks = groups * ((Hq + a.q_heads - 1) / a.q_heads);
    const int64_t kv_wgs = chunks * Hkv, wgs = kv_wgs + (tasks + WR_NT / 64 - 1) / (WR_NT / 64);
    if (wgs >= INT32_MAX / WR_NT) return set_err(ctx, COMPACT_ESHAPE, "too many rows for one call");
    a.n_kv_wgs = (int)kv_wgs;
    paged_write_kernel<HD, T><<<(unsigned)wgs, WR_NT, 0, s>>>(a);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

extern "C" int compact_rope_paged_write(compact_ctx* ctx, int32_t n_rows, const void* d_qkv, const compact_paged_kv* kv,
                                        const int64_t* d_slot, const float* d_rot, void* d_q, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    if (n_rows < 0) return set_err(ctx, COMPACT_EINVAL, "n_rows must be >= 0");
    PagedView v;
    TRY_RC(paged_view(ctx, kv, true, &v));
    if (!d_qkv || !d_slot || !d_rot || !d_q) return set_err(ctx, COMPACT_EINVAL, "null qkv, slots, rotations or q");
    if (((uintptr_t)d_qkv | (uintptr_t)d_q) & 15) return set_err(ctx, COMPACT_EINVAL, "qkv and q must be 16-byte aligned");
    if (((uintptr_t)d_slot | (uintptr_t)d_rot) & 7) return set_err(ctx, COMPACT_EINVAL, "slots and rotations must be 8-byte aligned");
    if (n_rows == 0) return COMPACT_OK;
    const bool b = ctx->cfg.dtype == COMPACT_BF16;
    auto launch = ctx->cfg.head_dim == 128 ? (b ? launch_write<128, bf16> : launch_write<128, float>)
                                           : (b ? launch_write<64, bf16> : launch_write<64, float>);
    return launch(ctx, n_rows, d_qkv, v, d_slot, d_rot, d_q, (hipStream_t)hip_stream);
}
