// Attention of many rows over an 8-bit cache, with capped scores.
#include "attn_tile_impl.inc"

int s3_attn_tile_8_cap(const s3_kv_cache* c, const AttnMore& p, const TileArgs& ta, bool small, hipStream_t st) {
    return launch_tile<kv_e4m3, true>(c->d_head, p, ta, small, st);
}
