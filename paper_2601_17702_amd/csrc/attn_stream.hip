// Attention of few rows over bf16 and fp32 caches; which of its builds a call takes.
#include "attn_stream_impl.inc"

size_t s3_attn_stream_workspace(const s3_kv_cache* c, bool list, int R, int64_t units, int64_t most_tokens) {
    return c->dtype == kS3E4m3 && s3_whole_tiles(R, list, units, most_tokens) ? 0 : s3_align((size_t)kRunGroups * 2 * slot_floats(R, c->d_head) * 4);
}

int s3_attn_stream(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st) {
    if (c->dtype == kS3E4m3) return p.cap != 0.0f ? s3_attn_stream_8_cap(c, p, tiles, R, most_tokens, ws, st) : s3_attn_stream_8(c, p, tiles, R, most_tokens, ws, st);
    if (p.cap != 0.0f) return s3_attn_stream_cap(c, p, tiles, R, most_tokens, ws, st);
    return c->dtype == S3_BF16 ? launch_stream<__bf16, false>(c->d_head, p, tiles, R, most_tokens, ws, st) : launch_stream<float, false>(c->d_head, p, tiles, R, most_tokens, ws, st);
}
