// Attention of many rows over bf16 and fp32 caches, with capped scores.
#include "attn_tile_impl.inc"

int s3_attn_tile_cap(const s3_kv_cache* c, const AttnMore& p, const TileArgs& ta, bool small, hipStream_t st) {
    return c->dtype == S3_BF16 ? launch_tile<__bf16, true>(c->d_head, p, ta, small, st) : launch_tile<float, true>(c->d_head, p, ta, small, st);
}
