// Attention over the paged cache: what its kernels share.
#pragma once
#include "paged.h"

#define LOG2E 1.4426950408889634f

#define FEW_COLS 32      // query columns (rows x heads of a KV group) of a request that the streaming kernel takes: two MFMA tiles
#define FEW_CHUNK 256    // cached rows of one of its work items
#define TILE_COLS 128    // query columns of a tile of the other kernel
#define TILE_KEYS 64     // cached rows of a step of it
#define SCHED_PITCH 32   // ints between the XCDs' counters: a 128-byte line each
#define SCHED_LISTED 1   // (in the first counter's line) requests in the schedule
#define SCHED_ORDER (8 * SCHED_PITCH)                      // [listed] those requests
#define SCHED_UNITS (SCHED_ORDER + PAGED_MAX_REQUESTS)     // [listed + 1] units before each of them
#define SCHED_BYTES (sizeof(int32_t) * (SCHED_UNITS + PAGED_MAX_REQUESTS + 1))
// A request of t tiles has its keys cut into pieces of 512 t to 1024 t rows, and of 2048 to 4096 as long as that gives no more than
// 64 units per KV head, which fill the card: a chunk of a prompt behind a long cache mostly comes alone or with single rows (256 rows behind
// 8192, 32 + 8 heads of 128: 86 -> 62 us; 7 requests of up to 118 behind up to 12149 124 -> 99).  Where many come at once, the records of what
// need not have been cut cost up to an eighth (32 x 250 rows behind 4000 to 8000: 843 -> 952), which a request may not know; with 1024 to 2048
// rows it is a quarter, and with as many pieces as give 512 units in any case twice the time of 32 mixed requests.
#define TILE_SPLIT 512
#define TILE_LONG 2048
#define TILE_FILL 64

struct PagedAttnArgs {
    PagedView kv;
    const int32_t *cu, *kv_len;
    int n_rows, max_new, max_kv;   // the call's bounds (max_kv: no more than the table holds)
    const void* q;
    void* o;
    int64_t q_stride;
    int Hq, Hkv;
    float scale_log2;
    // records of requests whose keys are split: [row][query head][piece] of a request, HD values each, and behind all of them (max, sum)
    float* rec;
    int rec_req, rec_row;     // a request's place among them, in row-pieces: so many per request and packed row before it
    int64_t n_rec;            // records in all
    int32_t* sched;           // the tile kernel's schedule: units taken per XCD (SCHED_PITCH apart), requests, units before them
};

struct PagedReq {
    int row0, n, kv;   // first packed row, rows, cached rows (whatever the arrays hold: inside the buffers)
};
__device__ __forceinline__ PagedReq paged_req(const PagedAttnArgs& a, int i) {
    PagedReq r;
    r.row0 = min(max(a.cu[i], 0), a.n_rows);
    r.n = min(min(max(a.cu[i + 1], r.row0), a.n_rows) - r.row0, a.max_new);
    r.kv = min(max(a.kv_len[i], 0), a.max_kv);
    return r;
}
__device__ __forceinline__ bool is_few(int n, int group) { return n <= FEW_COLS && n * group <= FEW_COLS; }
// pieces of a request's keys (at least one, so that a request without keys has somebody to write its zeros)
__device__ __forceinline__ int few_pieces(int kv) { return max((kv + FEW_CHUNK - 1) / FEW_CHUNK, 1); }
__device__ __forceinline__ int n_tiles(int n, int group) { return (int)(((int64_t)n * group + TILE_COLS - 1) / TILE_COLS); }
__device__ __forceinline__ int tile_pieces(int tiles, int kv) { return max(max(kv / TILE_SPLIT / tiles, min(kv / TILE_LONG, TILE_FILL / tiles)), 1); }
// rows of a piece: the last piece may hold fewer
__device__ __forceinline__ int tile_piece_rows(int pieces, int kv) {
    return ((kv + pieces - 1) / pieces + TILE_KEYS - 1) / TILE_KEYS * TILE_KEYS;
}

// the first record of a request's row and query head
__device__ __forceinline__ int64_t first_record(const PagedAttnArgs& a, int req, int row0, int row, int head, int pieces) {
    return ((int64_t)req * a.rec_req + (int64_t)row0 * a.rec_row + (int64_t)row * pieces) * a.Hq + (int64_t)head * pieces;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x as the sum of NP bf16 values: rounded once (NP = 1), or all 24 bits of it (NP = 3)
template <int NP>
__device__ __forceinline__ void split_bf16(float x, bf16 (&p)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        p[i] = (bf16)x;
        x -= (float)p[i];
    }
}

__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d) { *reinterpret_cast<floatx4*>(p) = floatx4{a, b, c, d}; }
__device__ __forceinline__ void put4(bf16* p, float a, float b, float c, float d) {
    *reinterpret_cast<bf16x4*>(p) = bf16x4{(bf16)a, (bf16)b, (bf16)c, (bf16)d};
}

// attn_paged_tiles.hip
int launch_attn_paged_tiles(compact_ctx* ctx, const PagedAttnArgs& a, hipStream_t s);
