// Attention of new tokens over a paged cache (s3_paged_attention), and over listed blocks of it (s3_block_attention).
#include "attn_launch.h"

namespace {

// 0: to be launched; 1: nothing to do; negative: an error.
int check(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs, float scale,
          const void* out) {
    if (int rc = s3_kv_check(fn, c, b)) return rc;
    if (n_q < 1 || n_q % c->n_kv_heads || n_q / c->n_kv_heads > 32) return s3_fail(S3_EINVAL, "%s: %d query heads over %d", fn, n_q, c->n_kv_heads);
    if (!(scale > 0.0f) || isinf(scale)) return s3_fail(S3_EINVAL, "%s: scale %g", fn, (double)scale);
    if (b->n_tokens == 0 || b->n_seq == 0) return 1;
    if (int rc = s3_kv_check_rows(fn, "q", c, q, q_ts, q_hs, n_q)) return rc;
    if (!out || (uintptr_t)out & 15) return s3_fail(S3_EINVAL, "%s: out is null or not 16-byte aligned", fn);
    return 0;
}
int check_ws(const char* fn, const void* ws, size_t ws_bytes, size_t need) {
    if (need && (!ws || (uintptr_t)ws & 255)) return s3_fail(S3_EINVAL, "%s: workspace is null or not 256-byte aligned", fn);
    if (ws_bytes < need) return s3_fail(S3_ECAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    return S3_OK;
}

// How a call is shared out.
struct Plan {
    int G, R, qb, per_q, n_split, limit;
    bool few, many;
    int64_t few_tiles, many_tiles;
    size_t few_ws, many_ws;
    size_t bytes() const { return few_ws + many_ws; }
    Plan(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b, int window) {
        G = n_q / c->n_kv_heads;
        limit = s3_few_rows(c->dtype == S3_BF16, c->d_head, q_block != 0);
        qb = min(q_block, max(b->n_tokens, 1));
        const int most_new = min(max(b->max_new, 1), max(b->n_tokens, 1));
        const int64_t most = (int64_t)(q_block ? min(qb, most_new) : most_new) * G;
        many = most > limit;
        // Beside chunks up to 32 rows: more of them fill what the chunk leaves idle or not, by lengths that the host does not know.  us with 32 / with
        // s3_few_rows, 8 sequences of 16 tokens beside 512 at 2048: at 1000 tokens with d_head 256 139 / 200, in fp32 with 128 296 / 358, with 256 726 / 872; at 8000
        // 577 / 357, 537 / 544, 1419 / 1021.
        if (many && !q_block) limit = 32;
        // no sequence is a short one if even the others at their longest leave more rows for it
        const bool all_long = b->n_tokens > (int64_t)(b->n_seq - 1) * b->max_new + limit / G;
        few = !many || (!q_block && !all_long);
        R = (int)min(most, (int64_t)limit);                    // a sequence's, or a tile of listed blocks', are one row tile
        few_ws = few ? s3_attn_stream_workspace(c->d_head, R) : 0;
        const int rows = s3_attn_tile_rows(c);
        per_q = (int)((most + rows - 1) / rows);
        few_tiles = q_block ? s3_block_tiles(b, q_block) : min(b->n_seq, b->n_tokens);
        // row tiles that there can be: beside the streaming kernel only sequences of more than `limit` rows have any, and each ends in one
        // that is not full; none has more than max_new tokens
        const int64_t all = (int64_t)b->n_tokens * G, longs = min((int64_t)min(b->n_seq, b->n_tokens), few ? all / (limit + 1) : all);
        many_tiles = !many ? 0 : q_block ? s3_block_tiles(b, q_block) * per_q : min((all + longs * (rows - 1)) / rows, longs * ((most + rows - 1) / rows));
        const int64_t units = many_tiles * c->n_kv_heads, tokens = q_block ? (int64_t)top_b * c->page_size : b->max_kv;
        const bool ragged = !q_block && b->n_seq > 1;
        n_split = many ? s3_attn_tile_split(c, units, tokens, ragged) : 1;
        many_ws = s3_attn_tile_workspace(c, units, n_split);              // for any window
        if (many && window) n_split = min(n_split, s3_attn_tile_split(c, units, min(tokens, (int64_t)window + rows / G), ragged));
    }
};

int run(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b, AttnArgs p, const Plan& plan, void* ws, hipStream_t st) {
    p.few = plan.few ? plan.limit : 0;
    p.qb = plan.qb;
    p.per_q = plan.per_q;
    // the joins' grids; looked at before the first launch, so that a refused call has written nothing
    if (max(plan.few ? plan.few_tiles : 0, plan.many_tiles) * c->n_kv_heads >= (int64_t)1 << 22)
        return s3_fail(S3_EINVAL, "%s: %lld row tiles and %d heads are too many for one call", fn, (long long)max(plan.few_tiles, plan.many_tiles), c->n_kv_heads);
    if (plan.few)
        if (int rc = s3_attn_stream(c, p, plan.few_tiles, plan.R, ws, st)) return rc;
    return plan.many ? s3_attn_tile(c, p, plan.many_tiles, plan.n_split, (char*)ws + plan.few_ws, st) : S3_OK;
}

bool shapes_ok(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return !s3_kv_check("workspace", c, b) && n_q >= 1 && n_q % c->n_kv_heads == 0 && n_q / c->n_kv_heads <= 32;
}

}  // namespace

extern "C" size_t s3_paged_attention_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return shapes_ok(c, b, n_q) ? Plan(c, b, n_q, 0, 0, 0).bytes() : 0;
}

extern "C" int s3_paged_attention(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                  float scale, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_paged_attention";
    if (window < 0) return s3_fail(S3_EINVAL, "%s: window %d", fn, window);
    if (int rc = check(fn, c, b, q, n_q, q_ts, q_hs, scale, out)) return rc < 0 ? rc : S3_OK;
    if (window >= 1 << 30) window = 0;                        // no position is that far back: all of them, and none of the kernels' differences overflows
    const Plan plan(c, b, n_q, 0, 0, window);
    if (int rc = check_ws(fn, ws, ws_bytes, plan.bytes())) return rc;
    const int es = c->dtype == S3_BF16 ? 2 : 4;
    AttnArgs p{s3_kv_batch_args(c, b), (const char*)q, (char*)out, lse, (const char*)c->k, (const char*)c->v, nullptr, q_ts * es,
               q_hs * es, c->n_kv_heads, plan.G, n_q, window, 0, 0, 1, 0, scale * 1.4426950408889634f, 0};
    return run(fn, c, b, p, plan, ws, (hipStream_t)stream);
}

extern "C" int64_t s3_block_tiles(const s3_kv_batch* b, int q_block) {
    return b && q_block >= 1 ? ((int64_t)b->n_tokens + (int64_t)b->n_seq * (q_block - 1)) / q_block : 0;
}

extern "C" size_t s3_block_attention_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b) {
    return shapes_ok(c, b, n_q) && q_block >= 1 && top_b >= 1 ? Plan(c, b, n_q, q_block, top_b, 0).bytes() : 0;
}

extern "C" int s3_block_attention(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                  const int32_t* sel, int q_block, int top_b, float scale, void* out, float* lse, void* ws,
                                  size_t ws_bytes, void* stream) {
    const char* fn = "s3_block_attention";
    if (q_block < 1 || top_b < 1 || q_block > 1 << 20 || top_b > 4096) return s3_fail(S3_EINVAL, "%s: q_block %d, top_b %d", fn, q_block, top_b);
    if (int rc = check(fn, c, b, q, n_q, q_ts, q_hs, scale, out)) return rc < 0 ? rc : S3_OK;
    if (!sel) return s3_fail(S3_EINVAL, "%s: null sel", fn);
    const Plan plan(c, b, n_q, q_block, top_b, 0);
    if (int rc = check_ws(fn, ws, ws_bytes, plan.bytes())) return rc;
    const int es = c->dtype == S3_BF16 ? 2 : 4;
    AttnArgs p{s3_kv_batch_args(c, b), (const char*)q, (char*)out, lse, (const char*)c->k, (const char*)c->v, sel, q_ts * es,
               q_hs * es, c->n_kv_heads, plan.G, n_q, 0, 0, top_b, 1, (int)s3_block_tiles(b, q_block), scale * 1.4426950408889634f, 0};
    return run(fn, c, b, p, plan, ws, (hipStream_t)stream);
}
