// Choice of the experts of a row: scores, a bias, groups, top-k, weights.
//
// Which expert is chosen, and in which order, is a matter of single comparisons: of 131072 rows of 256 sigmoid scores with a bias some ten have two that 32 bits do not
// tell apart.  So the order is made of 64-bit values, but only of the few experts that 32 bits leave in question (a whole row in 64 bits: 527 us
// for those rows).  Bound: the vector ALU, busy without a pause in the 63 us that 8 groups and top-8 of these rows take (2.3 TB/s of logits, indices and weights); 64 rows of 128 3.5 us.
// What made it so: four rows a wavefront and candidates 527 -> 93, groups by whole lanes and candidates from a bit mask -> 80, straight loads of
// full rows and maxima of whole numbers -> 60.
#include "common.h"
#include "vecio.h"

// Monotone map of a number to 64 bits whose low 8 are its place: the larger key is the larger value to 44 bits, among equal ones the
// lower place.  No key of a number is 0.
__device__ __forceinline__ uint64_t key_of(double v, int place) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // (-0 is 0)
    const uint64_t u = b >> 63 ? ~b : b | 0x8000000000000000ull;
    return (u & ~255ull) | (uint64_t)(255 - place);
}
__device__ __forceinline__ int place_of(uint64_t key) { return 255 - (int)(key & 255); }
__device__ __forceinline__ uint64_t wave_max_key(uint64_t k) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)k, o, 64);
        k = k > other ? k : other;
    }
    return k;
}

// What the experts are ordered by: their c, or without a bias, and where no sums of scores rank the groups, the logits themselves, of which the scores
// are increasing functions.
struct RouteArgs {
    compact_route_rule rule;
    const float* logits;
    const float* bias;
    int64_t rows;
    int E, k;
    int by_logit;
    int inv_size;   // 65536 / experts of a group, rounded up: e / size = e * inv_size >> 16 for e < 256
    int lanes;      // of the 16, that share a group in the quick way to rank groups; 0: the general one
    int32_t* idx;
    float* weight;
};

// Every row that the kernel below passes on: one wavefront, lane l owns experts l, l + 64, l + 128, l + 192, all in 64 bits.
__device__ __forceinline__ void route_row(const RouteArgs& a, int64_t row) {
    const compact_route_rule& rule = a.rule;
    const int lane = threadIdx.x & 63, E = a.E, k = a.k;
    float l[4];
    double s[4], c[4];
    uint64_t key[4];
    bool live[4];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = lane + 64 * i;
        l[i] = e < E ? a.logits[row * E + e] : -INFINITY;
        if (!(l[i] == l[i])) l[i] = -INFINITY;
        live[i] = l[i] > -INFINITY;
        top = fmaxf(top, l[i]);
    }
    if (rule.score == COMPACT_SCORE_SIGMOID) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = live[i] ? 1.0 / (1.0 + exp(-(double)l[i])) : 0.0;
    } else {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] = !live[i] ? 0.0 : l[i] == top ? 1.0 : exp((double)l[i] - (double)top);
            sum += s[i];
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = lane + 64 * i;
        c[i] = a.by_logit ? (double)l[i] : s[i] + (a.bias && e < E ? (double)a.bias[e] : 0.0);
        live[i] = live[i] && c[i] > -INFINITY;   // (no NaN is)
        key[i] = e < E ? key_of(live[i] ? c[i] : -INFINITY, e) : 0;
    }
    if (rule.topk_groups < rule.n_groups) {
        const int S = E / rule.n_groups;
        uint64_t mine = 0;      // lane g: key of group g
        for (int g = 0; g < rule.n_groups; ++g) {
            double total = 0.0;
            bool any = false;
            uint64_t below = ~0ull;
            for (int j = 0; j < rule.group_top; ++j) {
                uint64_t best = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = lane + 64 * i;
                    if (e >= g * S && e < g * S + S && live[i] && key[i] < below && key[i] > best) best = key[i];
                }
                best = wave_max_key(best);
                below = best;
                if (!best) break;
                const int e = place_of(best);
                double v = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e == lane + 64 * i) v = c[i];
                total += __shfl(v, e & 63, 64);
                any = true;
            }
            if (lane == g) mine = key_of(any ? total : -INFINITY, g);
        }
        uint64_t chosen = 0;    // bit g: group g is eligible
        for (int j = 0; j < rule.topk_groups; ++j) {
            const int g = place_of(wave_max_key(mine));
            chosen |= 1ull << g;
            if (lane == g) mine = 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 64 * i;
            if (e < E && !(chosen >> (e / S) & 1)) key[i] = 0;
        }
    }
    int my_e = 0;
    double my_s = 0.0, sum = 0.0;
    for (int j = 0; j < k; ++j) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) best = best > key[i] ? best : key[i];
        const int e = place_of(wave_max_key(best));
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e == lane + 64 * i) {
                v = s[i];
                key[i] = 0;
            }
        v = __shfl(v, e & 63, 64);
        sum += v;
        if (lane == j) {
            my_e = e;
            my_s = v;
        }
    }
    if (lane < k) {
        a.idx[row * k + lane] = my_e;
        const double w = rule.renorm ? (sum > 0.0 ? my_s / sum : 0.0) : my_s;
        a.weight[row * k + lane] = (float)(w * (double)rule.factor);
    }
}

// ---- 16 lanes that have a row together: a DPP row -----------------------------------------------------------------------
template <int N>
__device__ __forceinline__ uint32_t ror16(uint32_t x) {   // from the lane N below, around
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false);
}
template <int N>
__device__ __forceinline__ float ror16(float x) {
    return __uint_as_float(ror16<N>(__float_as_uint(x)));
}
template <int N>
__device__ __forceinline__ uint32_t up16(uint32_t x) {    // from the lane N below, 0 beyond the first
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x110 + N, 0xf, 0xf, true);
}
__device__ __forceinline__ float max16(float x) {
    x = fmaxf(x, ror16<8>(x));
    x = fmaxf(x, ror16<4>(x));
    x = fmaxf(x, ror16<2>(x));
    return fmaxf(x, ror16<1>(x));
}
__device__ __forceinline__ int max16(int x) {
    x = max(x, (int)ror16<8>((uint32_t)x));
    x = max(x, (int)ror16<4>((uint32_t)x));
    x = max(x, (int)ror16<2>((uint32_t)x));
    return max(x, (int)ror16<1>((uint32_t)x));
}
// a whole number that is the larger the larger x is (and x again from it)
__device__ __forceinline__ int ordered(float x) {
    const int i = __float_as_int(x);
    return i ^ (i >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float sum16(float x) {
    x += ror16<8>(x);
    x += ror16<4>(x);
    x += ror16<2>(x);
    return x + ror16<1>(x);
}
template <int N>
__device__ __forceinline__ double ror16(double x) {
    const uint64_t b = (uint64_t)__double_as_longlong(x);
    return __longlong_as_double((long long)((uint64_t)ror16<N>((uint32_t)(b >> 32)) << 32 | ror16<N>((uint32_t)b)));
}
__device__ __forceinline__ double sum16(double x) {
    x += ror16<8>(x);
    x += ror16<4>(x);
    x += ror16<2>(x);
    return x + ror16<1>(x);
}
// how many of the 16 are larger
template <int N = 1>
__device__ __forceinline__ int larger16(float x) {
    if constexpr (N == 16)
        return 0;
    else
        return (ror16<N>(x) > x ? 1 : 0) + larger16<N + 1>(x);
}
template <int N = 1>
__device__ __forceinline__ int larger16(uint32_t hi, uint32_t lo) {
    if constexpr (N == 16) {
        return 0;
    } else {
        const uint64_t other = (uint64_t)ror16<N>(hi) << 32 | ror16<N>(lo);
        return (other > ((uint64_t)hi << 32 | lo) ? 1 : 0) + larger16<N + 1>(hi, lo);
    }
}

// the two largest of a lane's two and those of the lane that CTRL names
template <int CTRL>
__device__ __forceinline__ void join_two(float& m1, float& m2) {
    const float o1 = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m1), CTRL, 0xf, 0xf, false));
    const float o2 = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m2), CTRL, 0xf, 0xf, false));
    m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
    m1 = fmaxf(m1, o1);
}

// 16 lanes per row, four rows per wavefront; lane t of a row has experts t + 16 j.  In 32 bits the row's values tell which experts may be among the top_k:
// those that reach T less twice the error of a value, T being the top_k-th largest of the lanes' two largest each.  They are
// 8 or 9 of 256 as a rule; each goes to a lane of its own, is evaluated in 64 bits, and its place is the number of larger
// ones.  A row goes to route_row() instead if it holds an infinity or NaN where that matters, if fewer than top_k experts are live, if more
// than 16 pass, or if 32 bits do not tell the last chosen group from the first that is not.
template <int V>
__global__ __launch_bounds__(256) void route_kernel(const RouteArgs a) {
    extern __shared__ __attribute__((aligned(16))) float smem[];   // per row of the workgroup: 16 V values (with groups), 16 candidates
    const compact_route_rule& rule = a.rule;
    const int t = threadIdx.x & 15, at = threadIdx.x >> 4, E = a.E, k = a.k;
    const bool grouped = rule.topk_groups < rule.n_groups;
    uint8_t* list = reinterpret_cast<uint8_t*>(smem + (grouped ? (blockDim.x >> 4) * 16 * V : 0)) + at * 16;
    float* vals = smem + at * 16 * V;
    const int64_t row0 = ((int64_t)blockIdx.x * blockDim.x + (threadIdx.x & ~63)) >> 4;   // of the wavefront
    if (row0 >= a.rows) return;
    const int64_t mine = row0 + (at & 3), row = min(mine, a.rows - 1);
    const float* lr = a.logits + row * E;
    float v[V];
    bool slow = false;
    // (a lane's place in a row is one address for all of its experts)
    const bool full = E == 16 * V;
    auto load = [&](const float* p, float (&x)[V], float none) __attribute__((always_inline)) {
        if (full) {
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = p[t + 16 * j];
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float y = p[min(t + 16 * j, E - 1)];
                x[j] = t + 16 * j < E ? y : none;
            }
        }
    };
    load(lr, v, -INFINITY);
    // (NaN and +inf, and NaN out of the bias, are route_row()'s)
    float top = -INFINITY, all_v = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        all_v += v[j];
        top = fmaxf(top, v[j]);
    }
    slow |= !(all_v < INFINITY);   // (a sum that overflows goes there too)
    double sum = 0.0;    // of the softmax, where values are scores
    float sum32 = 0.f;   // where they are logits
    if (rule.score == COMPACT_SCORE_SOFTMAX) {
        top = max16(top);
        if (!a.by_logit) {
#pragma unroll
            for (int j = 0; j < V; ++j) sum += v[j] > -INFINITY ? exp((double)v[j] - (double)top) : 0.0;
            sum = sum16(sum);
        } else if (!rule.renorm) {
#pragma unroll
            for (int j = 0; j < V; ++j) sum32 += v[j] > -INFINITY ? __expf(v[j] - top) : 0.f;
            sum32 = sum16(sum32);
        }
    }
    if (!a.by_logit) {
        const float scale = (float)(1.0 / sum);
        float b[V];
        if (a.bias) load(a.bias, b, 0.f);
        all_v = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float sc = rule.score == COMPACT_SCORE_SIGMOID ? __builtin_amdgcn_rcpf(1.0f + __expf(-v[j])) : __expf(v[j] - top) * scale;
            if (a.bias) sc += b[j];
            v[j] = v[j] > -INFINITY ? sc : -INFINITY;
            all_v += v[j];
        }
        slow |= !(all_v < INFINITY);
    }
    if (grouped) {
#pragma unroll
        for (int j = 0; j < V; ++j) vals[t + 16 * j] = v[j];
        __builtin_amdgcn_wave_barrier();
        float m1 = -INFINITY, m2 = -INFINITY;   // the two largest
        const int share = a.lanes ? a.lanes : 1;
        if (a.lanes) {   // V neighbours a lane, then the lanes of a group
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float x = vals[t * V + j];
                m2 = fmaxf(m2, fminf(m1, x));
                m1 = fmaxf(m1, x);
            }
            if (a.lanes > 1) join_two<0xb1>(m1, m2);    // lane ^ 1
            if (a.lanes > 2) join_two<0x4e>(m1, m2);    // lane ^ 2
            if (a.lanes > 4) join_two<0x141>(m1, m2);   // 7 - lane of 8
        } else {         // lane g: group g
            const int S = E / rule.n_groups;
            if (t < rule.n_groups)
                for (int i = 0, o = t % S; i < S; ++i, o = o + 1 == S ? 0 : o + 1) {   // (each lane begins elsewhere: other banks)
                    const float x = vals[t * S + o];
                    m2 = fmaxf(m2, fminf(m1, x));
                    m1 = fmaxf(m1, x);
                }
        }
        float g = m1, size = fabsf(m1);
        if (rule.group_top == 2) {
            g = m2 > -INFINITY ? m1 + m2 : -INFINITY;
            size += fabsf(m2);
            slow |= m1 > -INFINITY && !(m2 > -INFINITY);   // (its only live expert counts alone)
        }
        // Error of g, twice: a value has 2^-21 (a score) and 2^-24 of itself, the sum 2^-24 of what is added, which may be much more than g.
        const float off = !a.by_logit && g > -INFINITY ? 0x1p-19f + size * 0x1p-22f : 0.f;
        const int above = larger16(g);   // (of all lanes: none of them may sleep)
        const bool here_is_one = t < rule.n_groups * share, chosen = here_is_one && above < rule.topk_groups * share;
        const uint32_t groups = (uint32_t)(__ballot(chosen) >> (at % 4 * 16)) & 0xffff;
        const float least = -max16(chosen ? off - g : -INFINITY), first_out = max16(here_is_one && !chosen ? g + off : -INFINITY);
        // (equal ones at the border are all chosen, or none)
        slow |= __popc(groups) != rule.topk_groups * share || !(least > -INFINITY) ||
                (!a.by_logit && !(least > first_out));
        if (a.lanes) {   // expert t + 16 j was lane (t + 16 j) / V's
            const uint32_t mine_first = groups >> (t / V);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!(mine_first >> (j * (16 / V)) & 1)) v[j] = -INFINITY;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!(groups >> ((t + 16 * j) * a.inv_size >> 16) & 1)) v[j] = -INFINITY;
        }
    }
    // T
    float m1 = -INFINITY, m2 = -INFINITY, T = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        m2 = fmaxf(m2, fminf(m1, v[j]));
        m1 = fmaxf(m1, v[j]);
    }
    {   // (as whole numbers in the same order: their maximum takes its other operand from another lane by itself)
        int i1 = ordered(m1), i2 = ordered(m2), top_i = 0;
        for (int i = 0; i < k; ++i) {
            top_i = max16(i1);
            const bool it = i1 == top_i;   // (equal ones go together: T ends lower, never too high)
            i1 = it ? i2 : i1;
            i2 = it ? ordered(-INFINITY) : i2;
        }
        T = __int_as_float(top_i ^ (top_i >> 31 & 0x7fffffff));
    }
    slow |= !(T > -INFINITY);
    // Twice the error of a value: a score has 2^-21, its sum with the bias 2^-24 of it.
    if (!a.by_logit) T -= 0x1p-19f + fabsf(T) * 0x1p-21f;
    uint32_t found = 0;   // bit j: expert t + 16 j is a candidate
#pragma unroll
    for (int j = 0; j < V; ++j) found |= v[j] >= T ? 1u << j : 0;
    const uint32_t n = __popc(found);
    uint32_t before = n;
    before += up16<1>(before);
    before += up16<2>(before);
    before += up16<4>(before);
    before += up16<8>(before);
    uint32_t total = n;
    total += ror16<8>(total);
    total += ror16<4>(total);
    total += ror16<2>(total);
    total += ror16<1>(total);
    slow |= total > 16;
    for (uint32_t pos = before - n; found && pos < 16; ++pos, found &= found - 1) list[pos] = (uint8_t)(t + 16 * (__ffs(found) - 1));
    __builtin_amdgcn_wave_barrier();
    // a candidate per lane
    const bool have = (uint32_t)t < total;
    const int e = have ? list[t] : 0;
    const double l = lr[e];
    double s, c = l;
    if (rule.score == COMPACT_SCORE_SIGMOID)
        s = 1.0 / (1.0 + exp(-l));
    else
        s = exp(l - (double)top) / (!a.by_logit ? sum : rule.renorm ? 1.0 : (double)sum32);
    if (!a.by_logit) c = s + (a.bias ? (double)a.bias[e] : 0.0);
    const uint64_t key = have ? key_of(c, e) : 0;
    const int rank = larger16((uint32_t)(key >> 32), (uint32_t)key);
    const bool chosen = have && rank < k;
    const double all = sum16(chosen ? s : 0.0);
    const uint64_t passed = __ballot(slow);
    const bool row_slow = (passed >> (at % 4 * 16) & 0xffff) != 0;
    if (chosen && mine < a.rows && !row_slow) {
        a.idx[row * k + rank] = e;
        a.weight[row * k + rank] = (float)((rule.renorm ? (all > 0.0 ? s / all : 0.0) : s) * (double)rule.factor);
    }
    if (passed)
        for (int i = 0; i < 4; ++i)
            if ((passed >> (16 * i) & 0xffff) && row0 + i < a.rows) route_row(a, row0 + i);
}

// more than 16 groups
__global__ __launch_bounds__(256) void route_rows_kernel(const RouteArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row < a.rows) route_row(a, row);
}

template <int V>
static void run_route(const RouteArgs& a, hipStream_t s) {
    // few rows: a wavefront per workgroup, over as many compute units
    const int threads = a.rows <= 4096 ? 64 : 256, per = threads / 16;
    const size_t smem = (size_t)per * ((a.rule.topk_groups < a.rule.n_groups ? 16 * V * 4 : 0) + 16);
    route_kernel<V><<<(unsigned)((a.rows + per - 1) / per), threads, smem, s>>>(a);
}

int launch_route(compact_ctx* ctx, const compact_route_rule& rule, const float* logits, const float* bias, int64_t rows, int32_t* idx,
                 float* weight, hipStream_t s) {
    constexpr int64_t most = 1ll << 25;   // rows of a launch, of up to 64 threads each
    static_assert(most * 64 <= MAX_GRID_THREADS, "one launch");
    if (rows > most) {
        for (int64_t r = 0; r < rows; r += most)
            TRY(launch_route(ctx, rule, logits + r * ctx->cfg.n_experts, bias, rows - r < most ? rows - r : most, idx + r * ctx->cfg.top_k,
                             weight + r * ctx->cfg.top_k, s));
        return COMPACT_OK;
    }
    if (rows == 0) return COMPACT_OK;
    const int E = ctx->cfg.n_experts, size = E / rule.n_groups;
    // the quick way: the experts fill the 16 lanes, and a group is 1, 2, 4 or 8 whole lanes
    const int values = E <= 16 ? 1 : E <= 32 ? 2 : E <= 64 ? 4 : E <= 128 ? 8 : 16;
    const int lanes = E == 16 * values && size % values == 0 && rule.n_groups > 1 && 16 % rule.n_groups == 0 ? 16 / rule.n_groups : 0;
    const RouteArgs a{rule, logits, bias, rows, E, ctx->cfg.top_k, !bias && (rule.topk_groups == rule.n_groups || rule.group_top == 1), (65536 + size - 1) / size, lanes, idx, weight};
    if (rule.n_groups > 16 && rule.topk_groups < rule.n_groups)
        route_rows_kernel<<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(a);
    else if (E <= 16)
        run_route<1>(a, s);
    else if (E <= 32)
        run_route<2>(a, s);
    else if (E <= 64)
        run_route<4>(a, s);
    else if (E <= 128)
        run_route<8>(a, s);
    else
        run_route<16>(a, s);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}
