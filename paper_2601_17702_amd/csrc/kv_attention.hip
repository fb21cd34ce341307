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
    int64_t few_tiles, many_tiles, few_tokens, most, all, longs, q_tiles;
    size_t few_ws, many_ws;
    size_t bytes() const { return few_ws + many_ws; }
    Plan(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b, int window) {
        G = n_q / c->n_kv_heads;
        limit = s3_few_rows(c->dtype != S3_FP32, c->d_head, q_block != 0, c->dtype == kS3E4m3);
        // Over 8 bits rows 33 to 64 are the streaming kernel's where there is much to stream, whose bytes then bound it.  us there / in the tiled kernel, 12 tokens of 32 heads
        // over 8: d_head 128, 4 sequences of 8000 37 / 33, of 16000 49 / 53, 16 of 8000 88 / 92, of 32000 273 / 355; 64, 4 of 4000 23 / 17, of 8000 29 / 29, 16 of 16000
        // 105 / 165; 256, 16 of 4000 120 / 102, of 8000 188 / 186, of 32000 513 / 719.
        if (c->dtype == kS3E4m3 && !q_block) limit = (double)min(b->n_seq, b->n_tokens) * c->n_kv_heads * b->max_kv >= 4096.0 * c->d_head ? 64 : 32;
        qb = min(q_block, max(b->n_tokens, 1));
        const int most_new = min(max(b->max_new, 1), max(b->n_tokens, 1));
        most = (int64_t)(q_block ? min(qb, most_new) : most_new) * G;
        many = most > limit;
        // Beside chunks up to 32 rows: more of them fill what the chunk leaves idle or not, by lengths that the host does not know.  us with 32 / with
        // s3_few_rows, 8 sequences of 16 tokens beside 512 at 2048: at 1000 tokens with d_head 256 139 / 200, in fp32 with 128 296 / 358, with 256 726 / 872; at 8000
        // 577 / 357, 537 / 544, 1419 / 1021.
        if (many && !q_block) limit = 32;
        // no sequence is a short one if even the others at their longest leave more rows for it
        const bool all_long = b->n_tokens > (int64_t)(b->n_seq - 1) * b->max_new + limit / G;
        few = !many || (!q_block && !all_long);
        R = (int)min(most, (int64_t)limit);                    // a sequence's, or a tile of listed blocks', are one row tile
        const int rows = s3_attn_tile_rows(c);
        q_tiles = q_block ? s3_block_tiles(b, q_block) : 0;
        few_tiles = q_block ? q_tiles : min(b->n_seq, b->n_tokens);
        all = (int64_t)b->n_tokens * G;
        longs = min((int64_t)min(b->n_seq, b->n_tokens), few ? all / (limit + 1) : all);
        cut(rows);
        const int64_t units = many_tiles * c->n_kv_heads;
        const int64_t tokens = few_tokens = q_block ? (int64_t)top_b * c->page_size : b->max_kv;
        const bool ragged = !q_block && b->n_seq > 1;
        n_split = many ? s3_attn_tile_split(c, units, tokens, ragged) : 1;
        many_ws = s3_attn_tile_workspace(c, units, n_split);              // for any window
        few_ws = few ? s3_attn_stream_workspace(c, q_block != 0, R, few_tiles * c->n_kv_heads, tokens) : 0;      // for any window
        if (window && !q_block) few_tokens = min(tokens, (int64_t)window + R / G + 32);
        if (many && window) n_split = min(n_split, s3_attn_tile_split(c, units, min(tokens, (int64_t)window + rows / G), ragged));
    }
    // Row tiles that there can be: beside the streaming kernel only sequences of more than `limit` rows have any, and each ends in one
    // that is not full; none has more than max_new tokens.
    void cut(int rows) {
        per_q = (int)((most + rows - 1) / rows);
        many_tiles = !many ? 0 : q_tiles ? q_tiles * per_q : min((all + longs * (rows - 1)) / rows, longs * ((most + rows - 1) / rows));
    }
};

int run(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b, AttnMore p, Plan plan, void* ws, hipStream_t st) {
    const bool small = plan.many && s3_small_tiles(c->dtype == kS3E4m3, c->dtype != S3_FP32, c->d_head, p.cap != 0.0f, plan.many_tiles * c->n_kv_heads, plan.n_split);
    if (small) plan.cut(128);
    p.few = plan.few ? plan.limit : 0;
    p.qb = plan.qb;
    p.per_q = plan.per_q;
    // the joins' grids; looked at before the first launch, so that a refused call has written nothing
    if (max(plan.few ? plan.few_tiles : 0, plan.many_tiles) * c->n_kv_heads >= (int64_t)1 << 22)
        return s3_fail(S3_EINVAL, "%s: %lld row tiles and %d heads are too many for one call", fn, (long long)max(plan.few_tiles, plan.many_tiles), c->n_kv_heads);
    if (plan.few)
        if (int rc = s3_attn_stream(c, p, plan.few_tiles, plan.R, plan.few_tokens, ws, st)) return rc;
    return plan.many ? s3_attn_tile(c, p, plan.many_tiles, plan.n_split, small, (char*)ws + plan.few_ws, st) : S3_OK;
}

bool shapes_ok(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return !s3_kv_check("workspace", c, b) && n_q >= 1 && n_q % c->n_kv_heads == 0 && n_q / c->n_kv_heads <= 32;
}

// An entry point's call.  c: the cache, or an 8-bit one (its scale) as one of bf16; softcap: 0 for none; sel: listed blocks, or null.
struct Call {
    const char* fn;
    const s3_kv_cache* c;
    const uint8_t* scale8;
    const s3_kv_batch* b;
    const void* q;
    int n_q;
    int64_t q_ts, q_hs;
    float scale, softcap;
    void* out;
    float* lse;
    void* ws;
    size_t ws_bytes;
    void* stream;
};
int attend(const Call& x, int window, const int32_t* sel, int q_block, int top_b) {
    if (!(x.softcap >= 0.0f && x.softcap <= 1e30f)) return s3_fail(S3_EINVAL, "%s: softcap %g", x.fn, (double)x.softcap);
    if (x.softcap > 0.0f && x.scale > 0.0f && !(x.scale / x.softcap >= 1e-30f && x.scale / x.softcap <= 1e30f))
        return s3_fail(S3_EINVAL, "%s: scale %g over softcap %g", x.fn, (double)x.scale, (double)x.softcap);
    if (int rc = check(x.fn, x.c, x.b, x.q, x.n_q, x.q_ts, x.q_hs, x.scale, x.out)) return rc < 0 ? rc : S3_OK;
    if (q_block && !sel) return s3_fail(S3_EINVAL, "%s: null sel", x.fn);
    if (window >= 1 << 30) window = 0;                        // no position is that far back: all of them, and none of the kernels' differences overflows
    s3_kv_cache c = *x.c;
    const int es = c.dtype == S3_BF16 ? 2 : 4;
    if (x.scale8) c.dtype = kS3E4m3;
    const Plan plan(&c, x.b, x.n_q, q_block, top_b, window);
    if (int rc = check_ws(x.fn, x.ws, x.ws_bytes, plan.bytes())) return rc;
    const float log2e = 1.4426950408889634f;
    const bool cap = x.softcap > 0.0f, near = cap && c.dtype != S3_FP32 && x.softcap <= kS3NearCap;
    const AttnMore p{{s3_kv_batch_args(&c, x.b), (const char*)x.q, (char*)x.out, x.lse, (const char*)c.k, (const char*)c.v, sel, x.q_ts * es, x.q_hs * es,
                      c.n_kv_heads, plan.G, x.n_q, window, 0, top_b, 1, q_block ? (int)s3_block_tiles(x.b, q_block) : 0,
                      near ? 2.0f * x.softcap * log2e : cap ? 1.0f : x.scale * log2e, 0},
                     x.scale8, cap ? x.softcap * log2e : 0.0f, cap ? x.scale / x.softcap : 0.0f, near ? x.softcap * log2e : 0.0f};
    return run(x.fn, &c, x.b, p, plan, x.ws, (hipStream_t)x.stream);
}
int check_window(const char* fn, int window) { return window < 0 ? s3_fail(S3_EINVAL, "%s: window %d", fn, window) : S3_OK; }
int check_lists(const char* fn, int q_block, int top_b) {
    return q_block < 1 || top_b < 1 || q_block > 1 << 20 || top_b > 4096 ? s3_fail(S3_EINVAL, "%s: q_block %d, top_b %d", fn, q_block, top_b) : S3_OK;
}
int check_cap(const char* fn, float softcap) { return softcap == 0.0f ? s3_fail(S3_EINVAL, "%s: softcap 0", fn) : S3_OK; }

}  // namespace

extern "C" size_t s3_paged_attention_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return shapes_ok(c, b, n_q) ? Plan(c, b, n_q, 0, 0, 0).bytes() : 0;
}

extern "C" int s3_paged_attention(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                  float scale, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_paged_attention";
    if (int rc = check_window(fn, window)) return rc;
    return attend({fn, c, nullptr, b, q, n_q, q_ts, q_hs, scale, 0.0f, out, lse, ws, ws_bytes, stream}, window, nullptr, 0, 0);
}

extern "C" int s3_paged_attention_capped(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                         float scale, float softcap, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_paged_attention_capped";
    if (int rc = check_window(fn, window)) return rc;
    if (int rc = check_cap(fn, softcap)) return rc;
    return attend({fn, c, nullptr, b, q, n_q, q_ts, q_hs, scale, softcap, out, lse, ws, ws_bytes, stream}, window, nullptr, 0, 0);
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
    if (int rc = check_lists(fn, q_block, top_b)) return rc;
    return attend({fn, c, nullptr, b, q, n_q, q_ts, q_hs, scale, 0.0f, out, lse, ws, ws_bytes, stream}, 0, sel, q_block, top_b);
}

extern "C" int s3_block_attention_capped(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                         const int32_t* sel, int q_block, int top_b, float scale, float softcap, void* out, float* lse, void* ws,
                                         size_t ws_bytes, void* stream) {
    const char* fn = "s3_block_attention_capped";
    if (int rc = check_lists(fn, q_block, top_b)) return rc;
    if (int rc = check_cap(fn, softcap)) return rc;
    return attend({fn, c, nullptr, b, q, n_q, q_ts, q_hs, scale, softcap, out, lse, ws, ws_bytes, stream}, 0, sel, q_block, top_b);
}

extern "C" size_t s3_kv8_attention_workspace(const s3_kv8_cache* c, const s3_kv_batch* b, int n_q) {
    s3_kv_cache view;
    if (s3_kv8_check("workspace", c, b, view) || !shapes_ok(&view, b, n_q)) return 0;
    view.dtype = kS3E4m3;
    return Plan(&view, b, n_q, 0, 0, 0).bytes();
}

extern "C" int s3_kv8_attention(const s3_kv8_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                float scale, float softcap, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_kv8_attention";
    s3_kv_cache view;
    if (int rc = s3_kv8_check(fn, c, b, view)) return rc;
    if (int rc = check_window(fn, window)) return rc;
    return attend({fn, &view, (const uint8_t*)c->scale, b, q, n_q, q_ts, q_hs, scale, softcap, out, lse, ws, ws_bytes, stream}, window, nullptr, 0, 0);
}

extern "C" size_t s3_kv8_block_attention_workspace(const s3_kv8_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b) {
    s3_kv_cache view;
    if (s3_kv8_check("workspace", c, b, view) || !shapes_ok(&view, b, n_q) || q_block < 1 || top_b < 1) return 0;
    view.dtype = kS3E4m3;
    return Plan(&view, b, n_q, q_block, top_b, 0).bytes();
}

extern "C" int s3_kv8_block_attention(const s3_kv8_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                      const int32_t* sel, int q_block, int top_b, float scale, float softcap, void* out, float* lse, void* ws,
                                      size_t ws_bytes, void* stream) {
    const char* fn = "s3_kv8_block_attention";
    s3_kv_cache view;
    if (int rc = s3_kv8_check(fn, c, b, view)) return rc;
    if (int rc = check_lists(fn, q_block, top_b)) return rc;
    return attend({fn, &view, (const uint8_t*)c->scale, b, q, n_q, q_ts, q_hs, scale, softcap, out, lse, ws, ws_bytes, stream}, 0, sel, q_block, top_b);
}
