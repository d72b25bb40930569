// Choice of the experts of a row: scores, a bias, groups, top-k, weights.
#include "common.h"
#include "vecio.h"

// Monotone map of a number to 64 bits whose low 8 are its place: the larger key is the larger value to 44 bits, among equal ones the
// lower place.  No key of a number is 0.
__device__ __forceinline__ uint64_t key_of(double v, int place) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
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

// One wavefront per row, lane l owns experts l, l + 64, l + 128, l + 192.
__global__ __launch_bounds__(256) void route_kernel(const compact_route_rule rule, const float* __restrict__ logits,
                                                    const float* __restrict__ bias, int64_t rows, int E, int k,
                                                    int32_t* __restrict__ idx, float* __restrict__ weight) {
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= rows) return;
    const int lane = threadIdx.x & 63;
    float l[4];
    double s[4];
    uint64_t key[4];
    bool live[4];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = lane + 64 * i;
        l[i] = e < E ? logits[row * E + e] : -INFINITY;
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
        double c = s[i] + (bias && e < E ? (double)bias[e] : 0.0);
        if (!(c == c)) c = -INFINITY;
        live[i] = live[i] && c > -INFINITY;
        key[i] = e < E ? key_of(live[i] ? c : -INFINITY, e) : 0;
        // (the values of the groups come from the keys' own numbers: kept beside them)
        l[i] = 0.f;
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
                double c = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e == lane + 64 * i) c = s[i] + (bias ? (double)bias[e] : 0.0);
                total += __shfl(c, e & 63, 64);
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
        idx[row * k + lane] = my_e;
        const double w = rule.renorm ? (sum > 0.0 ? my_s / sum : 0.0) : my_s;
        weight[row * k + lane] = (float)(w * (double)rule.factor);
    }
}

int launch_route(compact_ctx* ctx, const compact_route_rule& rule, const float* logits, const float* bias, int64_t rows, int32_t* idx,
                 float* weight, hipStream_t s) {
    if (rows == 0) return COMPACT_OK;
    route_kernel<<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(rule, logits, bias, rows, ctx->cfg.n_experts, ctx->cfg.top_k, idx, weight);
    LAUNCH_CHECK(ctx);
    return COMPACT_OK;
}
