// Attention of few rows over bf16 and fp32 caches, with capped scores.
#include "attn_stream_impl.inc"

int s3_attn_stream_cap(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st) {
    return c->dtype == S3_BF16 ? launch_stream<__bf16, true>(c->d_head, p, tiles, R, most_tokens, ws, st) : launch_stream<float, true>(c->d_head, p, tiles, R, most_tokens, ws, st);
}
