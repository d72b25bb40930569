// C ABI of the calls around 8-bit integer weights: argument checks, workspaces, launch sequences.
#include <algorithm>

#include "common.h"

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
#define MAX_ROWS 0x7fffffffll

extern "C" int compact_quant_i8(compact_ctx* ctx, const void* d_x, int64_t x_stride, int64_t rows, int32_t cols, void* d_q,
                                float* d_scale, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    if (rows < 0 || cols < 1 || x_stride < cols) return set_err(ctx, COMPACT_EINVAL, "negative rows, no columns or rows that overlap");
    if (rows > 0 && (!d_x || !d_q || !d_scale)) return set_err(ctx, COMPACT_EINVAL, "null pointer");
    if (rows > MAX_ROWS) return set_err(ctx, COMPACT_ESHAPE, "at most 2^31 - 1 rows");
    if (!aligned(d_x, dtype_size(ctx->cfg.dtype))) return set_err(ctx, COMPACT_EINVAL, "rows are not aligned to their elements");
    return launch_quant_i8(ctx, d_x, x_stride, rows, cols, (int8_t*)d_q, d_scale, (hipStream_t)hip_stream);
}

static int check_gemm_i8(int64_t M, int32_t N, int32_t K, int32_t epilogue, const char** why) {
    *why = "bad GEMM shape";
    if (M < 0 || N < 1 || K < 1) return COMPACT_EINVAL;
    *why = "epilogue must be 0 or 1";
    if (epilogue != 0 && epilogue != 1) return COMPACT_EINVAL;
    *why = "products of codes need K % 16 == 0 and K <= 131056 (sums of 32 bits)";
    if (K % 16 != 0 || K > 131056) return COMPACT_ESHAPE;
    // (what one launch of the weight stream covers, 128 or 64 columns in 1024 threads; rows go in as many launches as they need)
    *why = "at most 2^31 - 1 rows, 2^29 - 128 columns (SwiGLU: 2^28 - 64)";
    if (M > MAX_ROWS || N > (epilogue ? (1 << 28) - 64 : (1 << 29) - 128)) return COMPACT_ESHAPE;
    return COMPACT_OK;
}

extern "C" int compact_gemm_i8_workspace_bytes(const compact_ctx* ctx, int64_t M, int32_t N, int32_t K, int32_t epilogue, size_t* bytes) {
    if (!ctx || !bytes) return COMPACT_EINVAL;
    const char* why;
    if (const int rc = check_gemm_i8(M, N, K, epilogue, &why)) return set_err(const_cast<compact_ctx*>(ctx), rc, why);
    *bytes = gemm_i8_workspace(M, N, K, epilogue);
    return COMPACT_OK;
}

extern "C" int compact_gemm_i8(compact_ctx* ctx, const void* d_a, const float* d_a_scale, const void* d_b, const float* d_b_scale,
                               const void* d_r, void* d_c, int64_t M, int32_t N, int32_t K, int32_t epilogue, void* d_workspace,
                               size_t ws_bytes, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    const char* why;
    if (const int rc = check_gemm_i8(M, N, K, epilogue, &why)) return set_err(ctx, rc, why);
    if (M == 0) return COMPACT_OK;
    if (!d_a || !d_a_scale || !d_b || !d_b_scale || !d_c) return set_err(ctx, COMPACT_EINVAL, "null operand");
    if (epilogue == 1 && d_r) return set_err(ctx, COMPACT_EINVAL, "no residual with epilogue 1");
    if (!aligned(d_a, 16) || !aligned(d_b, 16)) return set_err(ctx, COMPACT_EINVAL, "codes must be 16-byte aligned");
    const size_t es = dtype_size(ctx->cfg.dtype), need = N % 8 == 0 ? 16 : es;
    if (!aligned(d_c, need) || !aligned(d_r, need)) return set_err(ctx, COMPACT_EINVAL, "output and residual must be 16-byte aligned where N % 8 == 0");
    GemmI8Args g{};
    g.a = (const int8_t*)d_a;
    g.a_scale = d_a_scale;
    g.b = (const int8_t*)d_b;
    g.b_scale = d_b_scale;
    g.r = d_r;
    g.c = d_c;
    g.M = M;
    g.N = N;
    g.K = K;
    g.epilogue = epilogue;
    return launch_gemm_i8(ctx, g, d_workspace, ws_bytes, (hipStream_t)hip_stream);
}

extern "C" int compact_block_norm(compact_ctx* ctx, const void* d_x, const void* d_b, const void* d_g_post, const void* d_gate,
                                  int64_t gate_stride, float alpha, void* d_h, const void* d_g_pre, void* d_n, void* d_q, float* d_q_scale,
                                  int64_t rows, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    if (rows < 0) return set_err(ctx, COMPACT_EINVAL, "negative rows");
    if (rows == 0) return COMPACT_OK;   // (arrays without rows may be null)
    if (!d_h && !d_n && !d_q) return set_err(ctx, COMPACT_EINVAL, "no output is wanted");
    if ((d_q == nullptr) != (d_q_scale == nullptr)) return set_err(ctx, COMPACT_EINVAL, "codes and their scales belong together");
    if ((d_n || d_q) && !d_g_pre) return set_err(ctx, COMPACT_EINVAL, "normalised rows need the gain g_pre");
    if (!d_b && (d_h || d_g_post || d_gate)) return set_err(ctx, COMPACT_EINVAL, "h, g_post and gate need the block's output b");
    if (d_h && d_h == d_n) return set_err(ctx, COMPACT_EINVAL, "h and n are one array");
    if (!d_x) return set_err(ctx, COMPACT_EINVAL, "null rows");
    if (d_gate && gate_stride != 0 && (gate_stride < ctx->cfg.d_model || gate_stride % 8 != 0))
        return set_err(ctx, COMPACT_EINVAL, "gate_stride must be 0, or a multiple of 8 that is d_model at least");
    if (rows > MAX_ROWS) return set_err(ctx, COMPACT_ESHAPE, "at most 2^31 - 1 rows");
    for (const void* p : {d_x, d_b, d_g_post, d_gate, (const void*)d_h, d_g_pre, (const void*)d_n})
        if (!aligned(p, 16)) return set_err(ctx, COMPACT_EINVAL, "rows and gains must be 16-byte aligned");
    if (!aligned(d_q, 8)) return set_err(ctx, COMPACT_EINVAL, "codes must be 8-byte aligned");
    BlockNormArgs a{d_x, d_b, d_g_post, d_gate, gate_stride, alpha, d_h, d_n || d_q ? d_g_pre : nullptr, d_n, (int8_t*)d_q, d_q_scale, rows};
    return launch_block_norm(ctx, a, (hipStream_t)hip_stream);
}

extern "C" int compact_route(compact_ctx* ctx, const compact_route_rule* rule, const void* d_m, const void* d_w_router, float* d_logits,
                             const float* d_bias, int64_t rows, int32_t* d_expert_idx, float* d_weight, void* hip_stream) {
    if (!ctx) return COMPACT_EINVAL;
    const compact_layer_cfg& c = ctx->cfg;
    if (c.n_experts == 0) return set_err(ctx, COMPACT_EINVAL, "layer has no experts");
    if (!rule || rows < 0) return set_err(ctx, COMPACT_EINVAL, "null rule or negative rows");
    if (rule->score != COMPACT_SCORE_SOFTMAX && rule->score != COMPACT_SCORE_SIGMOID)
        return set_err(ctx, COMPACT_EINVAL, "score must be COMPACT_SCORE_SOFTMAX or COMPACT_SCORE_SIGMOID");
    if (rule->n_groups < 1 || rule->n_groups > 64 || c.n_experts % rule->n_groups != 0)
        return set_err(ctx, COMPACT_ESHAPE, "n_groups must divide n_experts and be at most 64");
    if (rule->topk_groups < 1 || rule->topk_groups > rule->n_groups || c.n_experts / rule->n_groups * rule->topk_groups < c.top_k)
        return set_err(ctx, COMPACT_ESHAPE, "topk_groups must be in 1 .. n_groups, with top_k experts at least in them");
    if (rule->group_top != 1 && rule->group_top != 2) return set_err(ctx, COMPACT_EINVAL, "group_top must be 1 or 2");
    if (rows == 0) return COMPACT_OK;   // (arrays without rows may be null)
    if ((d_m == nullptr) != (d_w_router == nullptr)) return set_err(ctx, COMPACT_EINVAL, "rows and router weights belong together");
    if (rows > MAX_ROWS) return set_err(ctx, COMPACT_ESHAPE, "at most 2^31 - 1 rows");
    if (!d_logits || !d_expert_idx || !d_weight) return set_err(ctx, COMPACT_EINVAL, "null pointer");
    hipStream_t s = (hipStream_t)hip_stream;
    if (d_m) {
        for (const void* p : {d_m, d_w_router, (const void*)d_logits})
            if (!aligned(p, 16)) return set_err(ctx, COMPACT_EINVAL, "rows, router weights and the logits that they give must be 16-byte aligned");
        TRY(launch_router_logits(ctx, d_m, d_w_router, rows, d_logits, s));
    }
    return launch_route(ctx, *rule, d_logits, d_bias, rows, d_expert_idx, d_weight, s);
}

// ---- the routed experts -----------------------------------------------------------------------------------------------
struct MoeI8Bufs {
    MoePlan plan;
    // out: an expert's rows wait in bf16 for their sum, as in compact_moe_ffn.  In fp32 16384 rows of 128 experts of 2880 x 2880, top-4, take 2362 us for 2218 (twice the bytes of
    // what is written and read again; 16 rows 193.8 for 192.8); the error against 64 bits is 0.0020 of the output, 0.0017 with fp32: the output's own
    // rounding and the codes of act make the most of it.  The choice may not go by the rows, or a row's bits would depend on the others.
    bf16 *act, *out;
    int8_t* act_q;
    float* act_scale;
};
#define MOE_I8_MIN_MTILE 16
// Rows whose products one launch covers, at any row-tile height (most tiles of 512 threads: 64 x 128): more go in pieces, whose rows have the same bits.
static int64_t moe_i8_most_rows(const compact_layer_cfg& c) {
    const int64_t n_tiles = std::max((c.ffn_dim + 63) / 64, (c.d_model + 127) / 128);
    return std::max<int64_t>(1, 64 * (MAX_GRID_THREADS / (512 * n_tiles) - c.n_experts) / c.top_k);
}
static void carve_moe_i8(Carver& cv, const compact_layer_cfg& c, int64_t rows, MoeI8Bufs& b) {
    rows = std::min(rows, moe_i8_most_rows(c));
    const int64_t rk = rows * c.top_k;
    carve_moe_plan(cv, c, rows, b.plan, MOE_I8_MIN_MTILE);
    b.act_q = (int8_t*)cv.take((size_t)rk * c.ffn_dim);
    b.act_scale = (float*)cv.take((size_t)rk * 4);
    // the experts' outputs take the place of the rows between the products, which are gone by then
    b.act = b.out = (bf16*)cv.take((size_t)rk * std::max(c.ffn_dim, c.d_model) * sizeof(bf16));
}
static int check_moe_i8(compact_ctx* ctx, int64_t rows) {
    const compact_layer_cfg& c = ctx->cfg;
    if (c.n_experts == 0) return set_err(ctx, COMPACT_EINVAL, "layer has no experts");
    if (c.dtype != COMPACT_BF16) return set_err(ctx, COMPACT_EUNSUPPORTED, "experts as codes need bf16 storage");
    if (rows < 0) return set_err(ctx, COMPACT_EINVAL, "negative rows");
    if (rows > (1ll << 26) / c.top_k) return set_err(ctx, COMPACT_ESHAPE, "at most 2^26 routed rows");
    if (c.ffn_dim > 131056) return set_err(ctx, COMPACT_ESHAPE, "products of codes need K <= 131056 (sums of 32 bits)");
    return COMPACT_OK;
}

extern "C" int compact_moe_ffn_i8_workspace_bytes(const compact_ctx* ctx, int64_t rows, size_t* bytes) {
    if (!ctx || !bytes) return COMPACT_EINVAL;
    TRY(check_moe_i8(const_cast<compact_ctx*>(ctx), rows));
    Carver cv(nullptr);
    MoeI8Bufs b;
    carve_moe_i8(cv, ctx->cfg, rows, b);
    *bytes = cv.off;
    return COMPACT_OK;
}

// mtile: rows per tile of the experts' map (0: by the rule)
static int moe_ffn_i8(compact_ctx* ctx, const compact_experts_i8* experts, const void* d_m, const float* d_m_scale, const void* d_h,
                      const int32_t* d_expert_idx, const float* d_weight, int64_t rows, void* d_y, void* d_workspace, size_t ws_bytes,
                      void* hip_stream, int mtile) {
    if (!ctx) return COMPACT_EINVAL;
    TRY(check_moe_i8(ctx, rows));
    if (!experts || !experts->d_gate_up || !experts->d_gate_up_scale || !experts->d_down || !experts->d_down_scale)
        return set_err(ctx, COMPACT_EINVAL, "missing expert weights");
    if (rows == 0) return COMPACT_OK;
    if (!d_m || !d_m_scale || !d_h || !d_expert_idx || !d_weight || !d_y) return set_err(ctx, COMPACT_EINVAL, "null pointer");
    for (const void* p : {experts->d_gate_up, experts->d_down, d_m, d_h, (const void*)d_y})
        if (!aligned(p, 16)) return set_err(ctx, COMPACT_EINVAL, "codes and rows must be 16-byte aligned");
    const compact_layer_cfg& c = ctx->cfg;
    Carver cv(d_workspace);
    MoeI8Bufs b;
    carve_moe_i8(cv, c, rows, b);
    if (!d_workspace || !aligned(d_workspace, 16) || cv.off > ws_bytes)
        return set_err(ctx, COMPACT_EWORKSPACE, "workspace too small for the expert feed-forward");
    if (const int64_t most = moe_i8_most_rows(c); rows > most) {
        for (int64_t r = 0; r < rows; r += most) {
            const int64_t o = r * c.d_model, k = r * c.top_k;
            TRY(moe_ffn_i8(ctx, experts, (const int8_t*)d_m + o, d_m_scale + r, (const bf16*)d_h + o, d_expert_idx + k, d_weight + k,
                           std::min(rows - r, most), (bf16*)d_y + o, d_workspace, ws_bytes, hip_stream, mtile));
        }
        return COMPACT_OK;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    const int64_t rk = rows * c.top_k;
    int n_cus = 0;
    TRY(device_cu_count(ctx, &n_cus));
    if (mtile == 0) mtile = gemm_i8_group_mtile(rk, c.n_experts, c.ffn_dim, c.d_model, n_cus);
    TRY(launch_moe_plan(ctx, d_expert_idx, d_weight, rows, mtile, b.plan, s));
    GroupedArgs g{};
    g.mtile = mtile;
    g.tile_expert = b.plan.tile_expert;
    g.tile_row0 = b.plan.tile_row0;
    g.tile_rows = b.plan.tile_rows;
    g.n_mtiles = (int32_t)std::min<int64_t>(rk / mtile + c.n_experts, b.plan.max_mtiles);   // the map's upper bound
    g.n_live = b.plan.offsets + c.n_experts + 1;
    g.a_gather = b.plan.sorted_token;
    g.b_expert_stride = (int64_t)2 * c.ffn_dim * c.d_model;
    GemmI8Args a{(const int8_t*)d_m, d_m_scale, (const int8_t*)experts->d_gate_up, experts->d_gate_up_scale, nullptr, b.act, rk, c.ffn_dim, c.d_model, 1, &g};
    TRY(launch_gemm_i8(ctx, a, nullptr, 0, s));
    TRY(launch_quant_i8(ctx, b.act, c.ffn_dim, rk, c.ffn_dim, b.act_q, b.act_scale, s));
    g.a_gather = nullptr;
    g.row_scale = b.plan.sorted_gate;
    g.b_expert_stride = (int64_t)c.d_model * c.ffn_dim;
    a = GemmI8Args{b.act_q, b.act_scale, (const int8_t*)experts->d_down, experts->d_down_scale, nullptr, b.out, rk, c.d_model, c.ffn_dim, 0, &g};
    TRY(launch_gemm_i8(ctx, a, nullptr, 0, s));
    return launch_moe_combine(ctx, b.out, d_h, false, b.plan.slot_of, rows, d_y, s);
}

extern "C" int compact_moe_ffn_i8(compact_ctx* ctx, const compact_experts_i8* experts, const void* d_m, const float* d_m_scale,
                                  const void* d_h, const int32_t* d_expert_idx, const float* d_weight, int64_t rows, void* d_y,
                                  void* d_workspace, size_t ws_bytes, void* hip_stream) {
    return moe_ffn_i8(ctx, experts, d_m, d_m_scale, d_h, d_expert_idx, d_weight, rows, d_y, d_workspace, ws_bytes, hip_stream, 0);
}

// For the tests, not part of compact.h: the same with row tiles of a given height.
extern "C" int compact_test_moe_ffn_i8(compact_ctx* ctx, int32_t mtile, const compact_experts_i8* experts, const void* d_m,
                                       const float* d_m_scale, const void* d_h, const int32_t* d_expert_idx, const float* d_weight,
                                       int64_t rows, void* d_y, void* d_workspace, size_t ws_bytes, void* hip_stream) {
    if (mtile != 16 && mtile != 64 && mtile != 128 && mtile != 256) return COMPACT_EINVAL;
    return moe_ffn_i8(ctx, experts, d_m, d_m_scale, d_h, d_expert_idx, d_weight, rows, d_y, d_workspace, ws_bytes, hip_stream, mtile);
}
