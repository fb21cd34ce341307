// Attention of few rows over an 8-bit cache, with capped scores.
#include "attn_stream_impl.inc"

int s3_attn_stream_8_cap(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st) {
    return launch_stream<kv_e4m3, true>(c->d_head, p, tiles, R, most_tokens, ws, st);
}
