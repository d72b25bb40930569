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
// One launch: every workgroup forms the sums over all requests itself (a request's numbers stay in LDS) and then handles its
// rows of the slot map and its share of the table and of the stack.  No workgroup reads what another one writes: table
// columns that are read lie below a request's length, those written above it; stack entries that are read lie below
// n_free, those written above; lengths and counters come in pairs.  Page numbers are copied, never followed, so whatever the
// device arrays hold, nothing outside them is touched.
// Bound: up to some thousand rows by the launch and the chain of loads and scans (64 decode steps 5.2 us, 1024 of them 7.8, traced); beyond
// that by the angles, which are formed in 64 bits, a row's from the row before by a turn, and by the writes of 8 + 4 hd bytes
// a row (8 x 4096 rows, 17 MB: 9.5 us; 512 requests with 37000 rows 13.6).
// ---------------------------------------------------------------------------
#define PLAN_NT 256

struct PlanArgs {
    compact_paged_step st;
    PagedView kv;
    int half;             // head_dim / 2
    int rows;             // rows per workgroup, a multiple of PLAN_NT / half
    double log2_theta;
};

__device__ __forceinline__ int sat_add(int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7FFFFFFFu); }

// inclusive saturating sum over the lanes of a wavefront: inside rows of 16 lanes, then across them
__device__ __forceinline__ int wave_scan(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));   // row_shr:1
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));   // row_bcast:15 to rows 1 and 3
    v = sat_add(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));   // row_bcast:31 to rows 2 and 3
#endif
    return v;
}

// the value of the lane before, 0 in lane 0
__device__ __forceinline__ int lane_before(int v) {
    const int u = __shfl_up(v, 1, 64);
    return (threadIdx.x & 63) ? u : 0;
}

// the last i in 0 .. n - 1 with a[i] <= x (a[0] = 0 <= x, a does not decrease), three places looked at side by side
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int q = (hi - lo + 3) >> 2, m1 = lo + q, m2 = min(m1 + q, hi - 1), m3 = min(m2 + q, hi - 1);
        const bool b1 = a[m1] <= x, b2 = a[m2] <= x, b3 = a[m3] <= x;
        if (b3) {
            lo = m3;
        } else {
            hi = b2 ? m3 : b1 ? m2 : m1;
            lo = b2 ? m2 : b1 ? m1 : lo;
        }
    }
    return lo;
}

__global__ __launch_bounds__(PLAN_NT) void paged_plan_kernel(const PlanArgs a) {
    extern __shared__ int lds[];
    __shared__ int red[2][3][PLAN_NT / 64], s_refused;
    const compact_paged_step& st = a.st;
    const int N = a.kv.n_requests, shift = a.kv.page_shift, P = 1 << shift, width = a.kv.max_pages;
    int* cu = lds;                 // [N + 1] rows before request i
    int* back = cu + N + 1;        // [N + 1] pages given back by the requests before i
    int* want = back + N + 1;      // [N + 1] pages wanted by the requests before i
    int* len = want + N + 1;       // [N] rows cached, inside the table
    const int t = threadIdx.x, lane = t & 63, wave = wave_index();
    const int n_free = min(max(st.d_n_free[0], 0), a.kv.n_pages);
    const int cap = width << shift;
    auto pages = [&](int rows) { return (int)(((unsigned)rows + P - 1) >> shift); };
    // pages a request wants for n > 0 more rows, the last one at packed row `end` - 1; -1: it does not fit
    auto need_of = [&](int n, int held, int end) {
        if (n > cap - held || end > st.max_rows) return -1;
        return pages(held + n) - pages(held);
    };

    // a thread takes one frequency of the rotary angles; formed while the lengths are on their way
    const int run = a.rows * a.half / PLAN_NT, my_run = t / a.half * run, my_freq = t % a.half;

    // ---- the running sums, two requests per thread at a time: `c_` = of the requests before those
    int c_cu = 0, c_back = 0, c_want = 0;
    double freq = 0.0;   // in half turns a row: the reduction of the angle is exact then, and short (512 requests with 37000 rows 14.1 -> 12.9 us)
    for (int i0 = 0, turn = 0; i0 < N; i0 += 2 * PLAN_NT, turn ^= 1) {
        int n_new[2], held[2], end[2], gave[2], upto[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = i0 + 2 * t + u;
            n_new[u] = i < N ? st.d_n_new[i] : 0;
            held[u] = i < N ? st.d_len[i] : 0;
        }
        if (i0 == 0) freq = M_1_PI * exp2(-2.0 * (double)my_freq / (double)(2 * a.half) * a.log2_theta);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            held[u] = min(max(held[u], 0), cap);
            end[u] = max(n_new[u], 0);
            gave[u] = n_new[u] < 0 ? pages(held[u]) : 0;
        }
        int s_end = wave_scan(sat_add(end[0], end[1])), s_gave = wave_scan(sat_add(gave[0], gave[1]));
        if (lane == 63) {
            red[turn][0][wave] = s_end;
            red[turn][1][wave] = s_gave;
        }
        // sums before the thread's two requests: of the lanes before it, and of the wavefronts before its own
        s_end = lane_before(s_end);
        s_gave = lane_before(s_gave);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PLAN_NT / 64; ++k) {
            if (k == wave) {
                s_end = sat_add(s_end, c_cu);
                s_gave = sat_add(s_gave, c_back);
            }
            c_cu = sat_add(c_cu, red[turn][0][k]);
            c_back = sat_add(c_back, red[turn][1][k]);
        }
        end[0] = sat_add(s_end, end[0]);
        end[1] = sat_add(end[0], end[1]);
        gave[0] = sat_add(s_gave, gave[0]);
        gave[1] = sat_add(gave[0], gave[1]);
#pragma unroll
        for (int u = 0; u < 2; ++u) upto[u] = n_new[u] > 0 ? max(need_of(n_new[u], held[u], end[u]), 0) : 0;
        int s_upto = wave_scan(sat_add(upto[0], upto[1]));
        if (lane == 63) red[turn][2][wave] = s_upto;
        s_upto = lane_before(s_upto);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PLAN_NT / 64; ++k) {
            if (k == wave) s_upto = sat_add(s_upto, c_want);
            c_want = sat_add(c_want, red[turn][2][k]);
        }
        upto[0] = sat_add(s_upto, upto[0]);
        upto[1] = sat_add(upto[0], upto[1]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = i0 + 2 * t + u;
            if (i < N) {
                cu[i + 1] = end[u];
                back[i + 1] = gave[u];
                want[i + 1] = upto[u];
                len[i] = held[u];
            }
        }
    }
    if (t == 0) cu[0] = back[0] = want[0] = s_refused = 0;
    __syncthreads();
    const int total = min(sat_add(n_free, c_back), a.kv.n_pages);   // pages there are
    auto granted = [&](int i) {
        const int n = cu[i + 1] - cu[i];
        if (n <= 0) return false;
        const int need = need_of(n, len[i], cu[i + 1]);
        return need == 0 || (need > 0 && want[i + 1] <= total);
    };
    // the page at position v of the stack once the pages given back lie on it
    auto stack = [&](int v) {
        if (v < n_free) return st.d_free[v];
        const int i = last_at_most(back, N + 1, v - n_free);
        return a.kv.table[(size_t)i * width + (v - n_free - back[i])];
    };
    // those granted pages are the first ones that want some: they take as many as the largest of the sums that is there
    const int taken = want[last_at_most(want, N + 1, total)], left = total - taken;
    if (blockIdx.x == 0) {
        int refused = 0;
        for (int i = t; i < N; i += PLAN_NT) {
            const bool ok = granted(i);
            const int n = cu[i + 1] - cu[i], held = len[i];
            refused += !ok && st.d_n_new[i] > 0;   // (where the sum of the rows is at its limit, cu does not show them)
            st.d_len_out[i] = back[i + 1] > back[i] ? 0 : ok ? held + n : held;   // (finished without a page: held = 0)
            st.d_kv_len[i] = ok ? held + n : 0;
            st.d_cu[i + 1] = cu[i + 1];
        }
        if (refused) atomicAdd(&s_refused, refused);
        __syncthreads();
        if (t == 0) {
            st.d_cu[0] = 0;
            st.d_n_free_out[0] = left;
            st.d_n_refused[0] = s_refused;
        }
    }
    const unsigned gt = blockIdx.x * PLAN_NT + t, all = gridDim.x * PLAN_NT;   // (at most 2^28: the sums below stay inside 32 bits)
    for (unsigned v = n_free + gt; v < (unsigned)left; v += all) st.d_free[v] = stack(v);
    for (unsigned k = gt; k < (unsigned)taken; k += all) {   // the k-th page from the top of the stack
        const int i = last_at_most(want, N + 1, k);
        a.kv.table[(size_t)i * width + pages(len[i]) + (k - want[i])] = stack(total - 1 - k);
    }

    // ---- slots of this workgroup's rows (their pages' numbers are on their way during the angles)
    const int r0 = blockIdx.x * a.rows, rows = min(a.rows, st.max_rows - r0);
    int page = -1, in_page = 0;
    if (t < rows && r0 + t < c_cu) {
        const int i = last_at_most(cu, N + 1, r0 + t);
        if (granted(i)) {
            const int pos = len[i] + (r0 + t - cu[i]), p = pos >> shift, held = pages(len[i]);
            page = p < held ? a.kv.table[(size_t)i * width + p] : stack(total - 1 - (want[i] + p - held));
            in_page = pos & (P - 1);
        }
    }
    // ---- rotary angles, in fp64 as the framework's other rotations have them, for a run of rows.  A row that follows the one
    // before it in its request is that row turned by the frequency once more (four multiplications in place of a sine and a
    // cosine; 16 turns lose no more than 2^-48)
    double c1 = 0.0, s1 = 0.0, cn = 0.0, sn = 0.0;
    bool turns = false;
    int i = r0 + my_run < c_cu ? last_at_most(cu, N + 1, r0 + my_run) : N;
    int ends = i < N ? cu[i + 1] : 0x7FFFFFFF, pos = i < N ? len[i] + (r0 + my_run - cu[i]) : 0;
    for (int r = r0 + my_run; r < min(r0 + my_run + run, r0 + rows); ++r) {
        bool follows = r > r0 + my_run && i < N;
        if (r >= ends) {   // the next request that has rows
            do {
                ++i;
            } while (i < N && cu[i + 1] <= r);
            ends = i < N ? cu[i + 1] : 0x7FFFFFFF;
            pos = i < N ? len[i] : 0;
            follows = false;
        }
        if (follows) {
            if (!turns) sincospi(freq, &s1, &c1);
            turns = true;
            const double c = cn * c1 - sn * s1;
            sn = sn * c1 + cn * s1;
            cn = c;
        } else {
            sincospi((double)pos * freq, &sn, &cn);
        }
        reinterpret_cast<float2*>(st.d_rot)[(size_t)r * a.half + my_freq] = make_float2((float)cn, (float)sn);
        pos += i < N;
    }
    if (t < rows) st.d_slot[r0 + t] = page < 0 ? -1 : (int64_t)page * P + in_page;
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
    if (step->max_rows > PAGED_MAX_ROWS) return set_err(ctx, COMPACT_ESHAPE, "max_rows must be at most 2^26");
    if (step->d_len == step->d_len_out || step->d_len == step->d_kv_len || step->d_n_new == step->d_len_out || step->d_n_new == step->d_kv_len ||
        step->d_n_free == step->d_n_free_out || step->d_n_free == step->d_n_refused || step->d_len_out == step->d_kv_len ||
        step->d_n_free_out == step->d_n_refused)
        return set_err(ctx, COMPACT_EINVAL, "an output of the step is one of its inputs or another output");
    if (((uintptr_t)step->d_rot | (uintptr_t)step->d_slot) & 7)
        return set_err(ctx, COMPACT_EINVAL, "d_rot and d_slot must be 8-byte aligned");
    a.st = *step;
    a.half = ctx->cfg.head_dim / 2;
    a.log2_theta = log2((double)ctx->cfg.rope_theta);
    // rows per workgroup: one run of a row per thread as long as that gives no more than 256 workgroups, up to 16 beyond, where
    // consecutive rows are cheap
    const int at_once = PLAN_NT / a.half;
    a.rows = at_once;
    while (a.rows < 16 * at_once && step->max_rows > 256 * a.rows) a.rows *= 2;
    const size_t smem = (size_t)(4 * kv->n_requests + 3) * sizeof(int);
    if (smem > (60 << 10))
        HIP_TRY(ctx, hipFuncSetAttribute(reinterpret_cast<const void*>(paged_plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    paged_plan_kernel<<<(step->max_rows + a.rows - 1) / a.rows, PLAN_NT, smem, (hipStream_t)hip_stream>>>(a);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}

// ---------------------------------------------------------------------------
// Write.  A segment is what a call writes to one page: rows with consecutive slots.  A workgroup of four wavefronts takes a
// segment and KV head: two of them its K rows (rotated on the way), two its V rows (transposed in registers: a lane holds
// 16 rows of 4 elements, a granule, and stores 16 bytes per element).  Up to 64 rows (fp32 storage: 32 K rows) are read once and kept
// in registers until the scale is known; of a longer segment all but the last rows are read a second time.  Segments of one row
// (decode steps) go four and more side by side in a wavefront, without a barrier (200 of them: 13.7 -> 8.3 us).
// Further workgroups rotate q.
// Bound by HBM from some thousand rows on: every row is read once, q and the codes are written once (8 x 4096 rows of 32 + 16
// heads of 128: 755 MB in 145 us, 5.2 TB/s, where a copy reaches 4.9 and a sum 6.2); by the launch and one chain of
// dependent loads (slot, scale, row) below: 24 decode rows 4.2 us (traced).  A single row's V touches hd lines for a
// byte each, which 1000 such rows feel (23 us, 43 MB written for 8 MB of q and 2 MB of codes).
// ---------------------------------------------------------------------------
#define WR_NT 256
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
    int unit;             // rows of a unit, one or more chunks (all of a call's, or 16 and more)
    int kv_wgs, q_wgs;    // workgroups of a unit
    int q_heads;          // query heads per wavefront of the q part
};

// A segment as its workgroup sees it.
struct Segment {
    int row0, n;      // packed rows
    int o;            // first row in the page; rows below it were written before
    size_t ph;        // page * Hkv + KV head
    int before;       // scale byte so far (1 where nothing was written before)
};

// Values that wait in registers as they came, as words (of an array of bf16 values the compiler gives every one a register of its
// own).  Without as_they_are() between their two uses it keeps what the first one made of them instead.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Raw {
    unsigned w[sizeof(T) * N / 4];
    __device__ __forceinline__ float at(int i) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        return __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void clear(int i) {
        if constexpr (sizeof(T) == 4)
            w[i] = 0;
        else
            w[i >> 1] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
    }
    // the same sign, the size of the given bits (which the type has)
    __device__ __forceinline__ void set_size(int i, unsigned size) {
        if constexpr (sizeof(T) == 4)
            w[i] = (w[i] & 0x80000000u) | size;
        else
            w[i >> 1] = i & 1 ? (w[i >> 1] & 0x8000FFFFu) | size : (w[i >> 1] & 0xFFFF8000u) | size >> 16;
    }
    __device__ __forceinline__ void as_they_are() {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) * N / 4; ++i) w[i] = (unsigned)here((int)w[i]);
    }
};

// The rotation of a pair, with what the rounded product leaves behind added again: within one rounding of the exact values, so that
// hardly a code is another one than theirs.
__device__ __forceinline__ void rotate_closely(float lo, float hi, float c, float s, float& olo, float& ohi) {
    const float p = hi * s, q = lo * s;
    olo = fmaf(lo, c, -p) - fmaf(hi, s, -p);
    ohi = fmaf(hi, c, q) + fmaf(lo, s, -q);
}

// Sizes as the bits of a float without its sign: they order like the values, and what is not finite lies at INF_BITS and above.
#define INF_BITS 0x7F800000u
__device__ __forceinline__ unsigned size_bits(float x) { return __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu; }
// a finite value within the sizes that are cached
__device__ __forceinline__ float below_top(float x) {
    const float top = __builtin_bit_cast(float, TOP_BITS);
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_fmed3f(x, -top, top);
#else
    return x;
#endif
}
__device__ __forceinline__ unsigned wave_max_bits(unsigned v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, o, 64));
    return v;
}

// What the four wavefronts tell each other: their largest finite sizes (K, K, V, V), and the rows with a value that is not
// finite, by bit.
struct WriteShared {
    unsigned top[4];
    unsigned bad[4];
};
__device__ __forceinline__ bool is_bad(const WriteShared& sh, int j) { return sh.bad[j >> 5] >> (j & 31) & 1; }
// scale byte of the segment's K (wave 0, 1) or V (2, 3); top: the wavefront's largest finite size
__device__ __forceinline__ int new_byte(WriteShared& sh, unsigned top, int before) {
    const int wave = wave_index();
    if ((threadIdx.x & 63) == 0) sh.top[wave] = top;
    __syncthreads();
    return max(before, scale_byte(__builtin_bit_cast(float, max(sh.top[wave & 2], sh.top[wave | 1]))));
}

// K rows of the segment; wavefront `half` of the two takes rows half * HOLD .. of every 2 HOLD.
template <int HD, typename T>
__device__ __forceinline__ void write_k(const WriteArgs<T>& a, const Segment& sg, int kvh, int half, WriteShared& sh) {
    constexpr int HALF = HD / 2, LPT = HALF / 8, TPW = 64 / LPT;   // lanes per row (8 elements of either half), rows side by side
    constexpr int HOLD = sizeof(T) == 2 ? 32 : 16, NG = HOLD / TPW;
    using Eight = Raw<T, 8>;
    const int lane = threadIdx.x & 63, d = lane % LPT * 8, sub = lane / LPT + half * HOLD;
    const int ld = (a.Hq + 2 * a.Hkv) * HD;
    const T* src = a.qkv + (size_t)sg.row0 * ld + (a.Hq + kvh) * HD;
    const float2* rot = a.rot + (size_t)sg.row0 * HALF;
    Eight x[NG], y[NG];   // either half of the rows, as they came (in place of rows past the segment: its last one)
    auto load = [&](int j0) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
            if (j0 + half * HOLD + g * TPW < sg.n) {
                const unsigned at = (unsigned)min(j0 + g * TPW + sub, sg.n - 1) * ld + d;
                x[g] = *reinterpret_cast<const Eight*>(src + at);
                y[g] = *reinterpret_cast<const Eight*>(src + at + HALF);
            }
    };
    auto rotated = [&](int g, int j, float (&lo)[8], float (&hi)[8]) {
        const Raw<float, 16> cs = *reinterpret_cast<const Raw<float, 16>*>(rot + ((unsigned)min(j, sg.n - 1) * HALF + d));
#pragma unroll
        for (int e = 0; e < 8; ++e) rotate_closely(x[g].at(e), y[g].at(e), cs.at(2 * e), cs.at(2 * e + 1), lo[e], hi[e]);
    };
    unsigned top = 0;
    int j0 = 0;
    for (;; j0 += 2 * HOLD) {
        load(j0);
#pragma unroll
        for (int g = 0; g < NG; ++g)
            if (j0 + half * HOLD + g * TPW < sg.n) {
                const int j = j0 + g * TPW + sub;
                float lo[8], hi[8];
                rotated(g, j, lo, hi);
                unsigned mine = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) mine = max(mine, max(size_bits(lo[e]), size_bits(hi[e])));
                if (__any(mine >= INF_BITS)) {
                    if (mine >= INF_BITS) {
                        if (j < sg.n) atomicOr(&sh.bad[j >> 5], 1u << (j & 31));
                        mine = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (size_bits(lo[e]) < INF_BITS) mine = max(mine, size_bits(lo[e]));
                            if (size_bits(hi[e]) < INF_BITS) mine = max(mine, size_bits(hi[e]));
                        }
                    }
                }
                top = max(top, mine);
                __builtin_amdgcn_sched_barrier(0);   // (one group's rotations in registers at a time)
            }
        if (j0 + 2 * HOLD >= sg.n) break;
    }
    const int byte = new_byte(sh, wave_max_bits(top), sg.before);
    uint8_t* kp = a.kv.k + (sg.ph << a.kv.page_shift) * HD;
    if (byte > sg.before && sg.o > 0) {
        const float down = e8m0(max(127 + sg.before - byte, 0));
        for (int i = lane + 64 * half; i < sg.o * (HD / 16); i += 128) {
            uintx4 w = reinterpret_cast<uintx4*>(kp)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = recode4(w[e], down);
            reinterpret_cast<uintx4*>(kp)[i] = w;
        }
    }
    const float up = e8m0(254 - byte);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        x[g].as_they_are();
        y[g].as_they_are();
    }
    for (;;) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int j = j0 + g * TPW + sub;
            if (j < sg.n) {
                float lo[8], hi[8];
                rotated(g, j, lo, hi);
                if (__builtin_amdgcn_readfirstlane(byte) >= TOP_BYTE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) lo[e] = below_top(lo[e]), hi[e] = below_top(hi[e]);
                }
                uintx2 wl = {to_codes4(lo[0] * up, lo[1] * up, lo[2] * up, lo[3] * up), to_codes4(lo[4] * up, lo[5] * up, lo[6] * up, lo[7] * up)};
                uintx2 wh = {to_codes4(hi[0] * up, hi[1] * up, hi[2] * up, hi[3] * up), to_codes4(hi[4] * up, hi[5] * up, hi[6] * up, hi[7] * up)};
                if (is_bad(sh, j)) wl = wh = uintx2{0x7F7F7F7Fu, 0x7F7F7F7Fu};
                uint8_t* dst = kp + ((unsigned)(sg.o + j) * HD + d);
                *reinterpret_cast<uintx2*>(dst) = wl;
                *reinterpret_cast<uintx2*>(dst + HALF) = wh;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (j0 == 0) break;
        j0 -= 2 * HOLD;
        load(j0);
    }
    if (lane + 64 * half == 0) a.kv.ks[sg.ph] = (uint8_t)byte;
}

// V rows of the segment, transposed; lanes of both wavefronts take granules side by side.
template <int HD, typename T>
__device__ __forceinline__ void write_v(const WriteArgs<T>& a, const Segment& sg, int kvh, int half, WriteShared& sh) {
    constexpr int VL = HD / 4, VG = 128 / VL;   // lanes across a row, granules side by side in the two wavefronts
    using Four = Raw<T, 4>;
    const int lane = threadIdx.x & 63, d = lane % VL * 4, sub = lane / VL + half * (VG / 2);
    const int ld = (a.Hq + 2 * a.Hkv) * HD, shift = a.kv.page_shift;
    const T* src = a.qkv + (size_t)sg.row0 * ld + (a.Hq + a.Hkv + kvh) * HD;
    uint8_t* vp = a.kv.v + (sg.ph << shift) * HD;
    const int g_lo = sg.o / PAGED_GRAN, g_end = (sg.o + sg.n + PAGED_GRAN - 1) / PAGED_GRAN;
    auto place = [&](int g, int e) { return reinterpret_cast<uintx4*>(vp + (((unsigned)(d + e) << shift) + g * PAGED_GRAN)); };
    Four x[PAGED_GRAN];   // the rows of a granule (in place of those that are not in the segment: the nearest one); 0 for what is not finite, no more than the top
    // returns the lane's largest finite size
    auto load = [&](int g) {
        unsigned mine = 0;
        if (g < g_end) {
#pragma unroll
            for (int u = 0; u < PAGED_GRAN; ++u) x[u] = *reinterpret_cast<const Four*>(src + ((unsigned)min(max(g * PAGED_GRAN + u - sg.o, 0), sg.n - 1) * ld + d));
#pragma unroll
            for (int u = 0; u < PAGED_GRAN; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) mine = max(mine, size_bits(x[u].at(e)));
        }
        if (__any(mine > TOP_BITS)) {
            if (mine > TOP_BITS) {
                mine = 0;
#pragma unroll
                for (int u = 0; u < PAGED_GRAN; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned size = size_bits(x[u].at(e));
                        const int j = min(max(g * PAGED_GRAN + u - sg.o, 0), sg.n - 1);
                        if (size >= INF_BITS) {
                            atomicOr(&sh.bad[j >> 5], 1u << (j & 31));
                            x[u].clear(e);
                        } else {
                            if (size > TOP_BITS) x[u].set_size(e, TOP_BITS);
                            mine = max(mine, size);
                        }
                    }
            }
        }
        return mine;
    };
    unsigned top = 0;
    int g = g_lo + sub;
    for (;; g += VG) {
        top = max(top, load(g));
        if (g - sub + VG >= g_end) break;
    }
    const int byte = new_byte(sh, wave_max_bits(top), sg.before);
    const float up = e8m0(254 - byte), down = e8m0(max(127 + sg.before - byte, 0));
    const bool grown = byte > sg.before;
#pragma unroll
    for (int u = 0; u < PAGED_GRAN; ++u) x[u].as_they_are();
    if (grown && g_lo > 0) {   // granules of earlier rows alone
        for (int i = lane + 64 * half; i < g_lo * HD; i += 128) {
            uintx4* p = reinterpret_cast<uintx4*>(vp + (((unsigned)(i / g_lo) << shift) + i % g_lo * PAGED_GRAN));
            uintx4 w = *p;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = recode4(w[e], down);
            *p = w;
        }
    }
    for (;;) {
        if (g < g_end) {
            const int old = sg.o - g * PAGED_GRAN, end = sg.o + sg.n - g * PAGED_GRAN;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uintx4 w;   // 16 rows of one element
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    w[q4] = to_codes4(x[q4 * 4].at(e) * up, x[q4 * 4 + 1].at(e) * up, x[q4 * 4 + 2].at(e) * up, x[q4 * 4 + 3].at(e) * up);
                if (old > 0 || end < PAGED_GRAN) {   // rows below o: what is there, at the new scale; behind the segment: what is there
                    const uintx4 there = *place(g, e);
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        const unsigned below = low_bytes(old - 4 * q4), upto = low_bytes(end - 4 * q4);
                        w[q4] = ((grown ? recode4(there[q4], down) : there[q4]) & below) | (w[q4] & upto & ~below) | (there[q4] & ~upto);
                    }
                }
                *place(g, e) = w;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (g - sub == g_lo) break;
        g -= VG;
        load(g);
    }
    if (lane + 64 * half == 0) a.kv.vs[sg.ph] = (uint8_t)byte;
}

// workgroups per CU
template <typename T>
__host__ __device__ constexpr int write_resident() { return sizeof(T) == 2 ? 4 : 3; }

// One row that is a segment by itself (a decode step), K and V, by HD / 8 lanes.  Nothing is read that the row does not need: its V
// codes are stored byte by byte, and earlier rows are touched only where a scale grows.
template <int HD, typename T>
__device__ __forceinline__ void write_single(const WriteArgs<T>& a, int row, int64_t slot, int kvh) {
    constexpr int HALF = HD / 2, LANES = HD / 8;
    const int l = threadIdx.x % LANES, shift = a.kv.page_shift, o = (int)(slot & ((1 << shift) - 1));
    const size_t ph = (size_t)(slot >> shift) * a.Hkv + kvh;
    const T* src = a.qkv + (size_t)row * ((a.Hq + 2 * a.Hkv) * HD) + (a.Hq + kvh) * HD;
    const Raw<T, 4> x = *reinterpret_cast<const Raw<T, 4>*>(src + l * 4), y = *reinterpret_cast<const Raw<T, 4>*>(src + HALF + l * 4);
    const Raw<T, 8> v = *reinterpret_cast<const Raw<T, 8>*>(src + a.Hkv * HD + l * 8);
    const Raw<float, 8> cs = *reinterpret_cast<const Raw<float, 8>*>(a.rot + (size_t)row * HALF + l * 4);
    const int k_before = o > 0 ? min(max((int)a.kv.ks[ph], 1), 253) : 1, v_before = o > 0 ? min(max((int)a.kv.vs[ph], 1), 253) : 1;
    float k[8], val[8];
    unsigned k_top = 0, v_top = 0;
    int bad = 0;
    auto see = [&](float f, unsigned& top) {
        const unsigned size = size_bits(f);
        bad |= size >= INF_BITS;
        top = max(top, size < INF_BITS ? size : 0u);
        return size < INF_BITS ? below_top(f) : 0.f;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) rotate_closely(x.at(e), y.at(e), cs.at(2 * e), cs.at(2 * e + 1), k[e], k[4 + e]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        k[e] = see(k[e], k_top);
        val[e] = see(v.at(e), v_top);
    }
#pragma unroll
    for (int ofs = LANES / 2; ofs > 0; ofs >>= 1) {
        k_top = max(k_top, (unsigned)__shfl_xor((int)k_top, ofs, 64));
        v_top = max(v_top, (unsigned)__shfl_xor((int)v_top, ofs, 64));
        bad |= __shfl_xor(bad, ofs, 64);
    }
    const int k_byte = max(k_before, scale_byte(__builtin_bit_cast(float, k_top))), v_byte = max(v_before, scale_byte(__builtin_bit_cast(float, v_top)));
    const float k_up = e8m0(254 - k_byte), v_up = e8m0(254 - v_byte);
    uint8_t* kp = a.kv.k + (ph << shift) * HD;
    uint8_t* vp = a.kv.v + (ph << shift) * HD + ((size_t)(l * 8) << shift);
    if (k_byte > k_before && o > 0) {
        const float down = e8m0(max(127 + k_before - k_byte, 0));
        for (int i = l; i < o * (HD / 16); i += LANES) {
            uintx4 w = reinterpret_cast<uintx4*>(kp)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = recode4(w[e], down);
            reinterpret_cast<uintx4*>(kp)[i] = w;
        }
    }
    unsigned wl = to_codes4(k[0] * k_up, k[1] * k_up, k[2] * k_up, k[3] * k_up), wh = to_codes4(k[4] * k_up, k[5] * k_up, k[6] * k_up, k[7] * k_up);
    if (bad) wl = wh = 0x7F7F7F7Fu;
    *reinterpret_cast<unsigned*>(kp + o * HD + l * 4) = wl;
    *reinterpret_cast<unsigned*>(kp + o * HD + HALF + l * 4) = wh;
    unsigned code[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) code[u] = to_codes4(val[4 * u] * v_up, val[4 * u + 1] * v_up, val[4 * u + 2] * v_up, val[4 * u + 3] * v_up);
    if (v_byte > v_before && o > 0) {   // the lane's elements of the earlier rows, granule by granule
        const float down = e8m0(max(127 + v_before - v_byte, 0));
        for (int g = 0; g * PAGED_GRAN < o; ++g) {
            uintx4 w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uintx4*>(vp + (e << shift) + g * PAGED_GRAN);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const unsigned below = low_bytes(o - g * PAGED_GRAN - 4 * q4);
                    w[e][q4] = (recode4(w[e][q4], down) & below) | (w[e][q4] & ~below);
                }
                *reinterpret_cast<uintx4*>(vp + (e << shift) + g * PAGED_GRAN) = w[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) vp[(e << shift) + o] = (uint8_t)(code[e >> 2] >> 8 * (e & 3));
    if (l == 0) {
        a.kv.ks[ph] = (uint8_t)k_byte;
        a.kv.vs[ph] = (uint8_t)v_byte;
    }
}

template <int HD, typename T>
__global__ __launch_bounds__(WR_NT, write_resident<T>()) void paged_write_kernel(const WriteArgs<T> a) {
    constexpr int HALF = HD / 2, LPT = HALF / 8, TPW = 64 / LPT;
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int Hkv = a.Hkv;

    using Eight = Raw<T, 8>;
    // A unit's workgroups are on one XCD, whose L2 they share the rotations through (workgroups go to the XCDs in turn, the
    // units of a round one place further on each time: a page's segments begin every so many units).  Those of K and V,
    // which wait more than they move (and of which those in the middle of a segment leave at once), lie evenly among the unit's others.
    // A call whose workgroups all run at once is one unit over all XCDs, K and V first.
    int at = blockIdx.x, kv_at = at < a.kv_wgs ? at : -1, unit_row = 0;   // kv_at: which of the unit's workgroups for K and V
    if (a.n_rows > a.unit) {
        const int per_unit = a.kv_wgs + a.q_wgs, round = (at >> 3) / per_unit;
        unit_row = (round * 8 + ((at + round) & 7)) * a.unit;
        at = (at >> 3) % per_unit;
        const int before = at * a.kv_wgs / per_unit;
        kv_at = (at + 1) * a.kv_wgs / per_unit > before ? before : -1;
        at -= before;
    } else {
        at -= a.kv_wgs;
    }
    if (kv_at < 0) {   // ---- q: TPW rows of q_heads heads per wavefront, four heads at a time
        const int task = at * (WR_NT / 64) + wave;
        const int per_row = (a.Hq + a.q_heads - 1) / a.q_heads;
        const int in_rows = task / per_row * TPW + lane / LPT, row = unit_row + in_rows, h0 = task % per_row * a.q_heads, d = lane % LPT * 8;
        if (in_rows >= a.unit || row >= a.n_rows) return;
        float2 cs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = a.rot[(size_t)row * HALF + d + j];
        const T* src = a.qkv + (size_t)row * ((a.Hq + 2 * Hkv) * HD) + d;
        T* dst = a.q + (size_t)row * a.Hq * HD + d;
        const int h_end = min(h0 + a.q_heads, a.Hq);
        for (int h = h0; h < h_end; h += 4) {
            Eight x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (h + u < h_end) {
                    x[u] = *reinterpret_cast<const Eight*>(src + (h + u) * HD);
                    y[u] = *reinterpret_cast<const Eight*>(src + (h + u) * HD + HALF);
                }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (h + u < h_end) {
                    float lo[8], hi[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) rotate(x[u].at(j), y[u].at(j), cs[j].x, cs[j].y, lo[j], hi[j]);
                    store8(dst + (h + u) * HD, lo);
                    store8(dst + (h + u) * HD + HALF, hi);
                }
        }
        return;
    }

    // ---- K and V: the segments that begin in this workgroup's rows
    __shared__ WriteShared sh;
    const int kvh = kv_at % Hkv, shift = a.kv.page_shift, P = 1 << shift;
    const int row_lo = unit_row + kv_at / Hkv * a.chunk;
    const int64_t n_slots = (int64_t)a.kv.n_pages << shift;
    auto slot_of = [&](int row) { return row >= 0 && row < a.n_rows ? a.slot[row] : (int64_t)-1; };
    // the slots of 64 rows from row_lo on: `cuts` marks those that do not continue the row before them in its page
    const int64_t s = slot_of(row_lo + lane), next = slot_of(row_lo + lane + 1);
    const bool cut = s < 0 || s >= n_slots || (s & (P - 1)) == 0 || slot_of(row_lo + lane - 1) != s - 1;
    const uint64_t cuts = __ballot(cut);
    uint64_t begins = __ballot(cut && s >= 0 && s < n_slots && lane < a.chunk);
    // rows that are segments by themselves: 64 / (HD / 8) of them side by side in a wavefront
    const uint64_t singles = begins & __ballot(next != s + 1 || (next & (P - 1)) == 0);
    if (singles) {
        constexpr int SIDE = 64 / (HD / 8);
        const int n = __builtin_popcountll(singles), lower = __builtin_popcountll(singles & ((1ull << lane) - 1));
        // lane k of `place` holds the k-th of them
        const int place = __builtin_amdgcn_ds_permute((singles >> lane & 1 ? lower : n + lane - lower) * 4, lane);
        for (int k0 = wave * SIDE; k0 < n; k0 += WR_NT / 64 * SIDE) {
            const int k = k0 + lane / (HD / 8), at = __shfl(place, min(k, n - 1), 64);
            const int64_t slot = ((int64_t)__shfl((int)(s >> 32), at, 64) << 32) | (unsigned)__shfl((int)s, at, 64);
            if (k < n) write_single<HD>(a, row_lo + at, slot, kvh);
        }
        begins &= ~singles;
    }
    for (; begins; begins &= begins - 1) {
        const int at = __builtin_ctzll(begins);
        Segment sg;
        sg.row0 = row_lo + at;
        const int64_t s0 = ((int64_t)__builtin_amdgcn_readlane((int)(s >> 32), at) << 32) | (unsigned)__builtin_amdgcn_readlane((int)s, at);
        sg.o = (int)(s0 & (P - 1));
        sg.ph = (size_t)(s0 >> shift) * Hkv + kvh;
        sg.before = sg.o > 0 ? min(max((int)(wave < 2 ? a.kv.ks : a.kv.vs)[sg.ph], 1), 253) : 1;
        const uint64_t later = at < 63 ? cuts >> (at + 1) : 0;
        if (later) {
            sg.n = __builtin_ctzll(later) + 1;
        } else {   // (segments of pages of 128 rows, or that begin late in the 64)
            sg.n = min(64 - at, P - sg.o);
            while (sg.n < P - sg.o) {
                const int j = sg.n + lane;
                const uint64_t ends = __ballot(j >= P - sg.o || slot_of(sg.row0 + j) != s0 + j);
                sg.n += ends ? __builtin_ctzll(ends) : 64;
                if (ends) break;
            }
        }
        __syncthreads();   // (the rows marked for the segment before have been read)
        if (threadIdx.x < 4) sh.bad[threadIdx.x] = 0;
        __syncthreads();
        if (wave < 2)
            write_k<HD>(a, sg, kvh, wave, sh);
        else
            write_v<HD>(a, sg, kvh, wave - 2, sh);
    }
}

template <int HD, typename T>
static int launch_write(compact_ctx* ctx, int n_rows, const void* qkv, const PagedView& kv, const int64_t* slot, const float* rot, void* q,
                        hipStream_t s) {
    const int Hq = ctx->cfg.n_q_heads, Hkv = ctx->cfg.n_kv_heads;
    constexpr int TPW = 64 / (HD / 16);
    WriteArgs<T> a{(const T*)qkv, (T*)q, slot, (const float2*)rot, kv, n_rows, Hq, Hkv, 1, 1, 1, 1, 1};
    // rows per workgroup of the K / V part: its segments of several rows follow each other, those of one row go side by side, and
    // a prompt leaves all but the first workgroup of a segment idle.  us, 32 + 8 heads of 128, pages of 64: 64 x 4 rows 11.2 by 4, 14.4 by 8,
    // 61.5 by 64; 1024 rows of a prompt 14.3, 11.8, 11.5; 2 x 4096 52.5, 45.8, 41.3; 4 x 4096 97, 83, 78 (pages of 16: 84 by 16,
    // 100 by 64), all before the units of XCDs below
    a.chunk = n_rows <= 512 ? 4 : n_rows <= 8192 ? 8 : std::min(1 << kv.page_shift, 64);
    const int64_t groups = (n_rows + TPW - 1) / TPW;
    a.q_heads = (int)std::min<int64_t>(WR_QHEADS, std::max<int64_t>(1, groups * Hq / 4096));
    auto workgroups = [&](int64_t unit) {   // with units of so many rows
        const int64_t kv_wgs = (unit + a.chunk - 1) / a.chunk * Hkv, tasks = (unit + TPW - 1) / TPW * ((Hq + a.q_heads - 1) / a.q_heads);
        const int64_t q_wgs = (tasks + WR_NT / 64 - 1) / (WR_NT / 64);
        a.unit = (int)unit;
        a.kv_wgs = (int)kv_wgs;
        a.q_wgs = (int)q_wgs;
        return (kv_wgs + q_wgs) * (unit < n_rows ? ((n_rows + unit - 1) / unit + 7) / 8 * 8 : 1);
    };
    // one unit where all run at once (1950 rows of fp32 storage, 4 + 2 heads of 64: 6.9 us instead of 7.5)
    int n_cus = 0;
    TRY_RC(device_cu_count(ctx, &n_cus));
    int64_t wgs = workgroups(n_rows);
    if (wgs > write_resident<T>() * n_cus) wgs = workgroups(std::max(a.chunk, 16));
    if (wgs >= INT32_MAX / WR_NT) return set_err(ctx, COMPACT_ESHAPE, "too many rows for one call");
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
    if (n_rows == 0) return COMPACT_OK;
    if (!d_qkv || !d_slot || !d_rot || !d_q) return set_err(ctx, COMPACT_EINVAL, "null qkv, slots, rotations or q");
    if (((uintptr_t)d_qkv | (uintptr_t)d_q | (uintptr_t)d_rot) & 15) return set_err(ctx, COMPACT_EINVAL, "qkv, q and the rotations must be 16-byte aligned");
    if ((uintptr_t)d_slot & 7) return set_err(ctx, COMPACT_EINVAL, "slots must be 8-byte aligned");
    const bool b = ctx->cfg.dtype == COMPACT_BF16;
    auto launch = ctx->cfg.head_dim == 128 ? (b ? launch_write<128, bf16> : launch_write<128, float>)
                                           : (b ? launch_write<64, bf16> : launch_write<64, float>);
    return launch(ctx, n_rows, d_qkv, v, d_slot, d_rot, d_q, (hipStream_t)hip_stream);
}
