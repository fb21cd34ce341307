// What the attention's entry points call (host), with fewer than 2^22 tiles times heads.
#pragma once
#include "attn.h"

// The most rows of one sequence (or tile of listed blocks) that the streaming kernel takes; the tiled kernel has more, whose 256 rows a
// workgroup would stand mostly empty below.  us in the tiled / in the streaming kernel, 32 query heads over 8: 16 tokens of one sequence at
// 32768 with d_head 64: 42 / 27, of eight at 8000 with 256: 258 / 208, in fp32: 355 / 217 (32 tokens: 579 / 375); tiles of 16
// queries over 64 listed blocks of 512: 343 / 240, d_head 64: 276 / 154.  But bf16 with d_head 128, eight sequences: 66 / 73, where the tiled
// kernel's rate is best.
constexpr int s3_few_rows(bool bf16, int d_head, bool list) {
    return !bf16 ? (d_head == 128 ? 128 : 64) : list || d_head != 128 ? 64 : 32;
}

// Sequences, or tiles of listed blocks, of few rows (R: the most that one has, 128 at most); tiles: how many there can be;
// most_tokens: a bound of what one sees.
size_t s3_attn_stream_workspace(int d_head, int R);
int s3_attn_stream(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
// Its builds for capped scores, for 8-bit caches (dtype kS3E4m3), and for both.
int s3_attn_stream_cap(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
int s3_attn_stream_8(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
int s3_attn_stream_8_cap(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);

// Chunks, or tiles of listed blocks, of more rows: row tiles of s3_attn_tile_rows rows, the tokens of each in n_split parts.
int s3_attn_tile_rows(const s3_kv_cache* c);
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens, bool ragged);
size_t s3_attn_tile_workspace(const s3_kv_cache* c, int64_t units, int n_split);
struct TileArgs {
    float* slots;             // partial sums where n_split > 1
    int n_split, tiles;       // row tiles that there can be
};
int s3_attn_tile(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int n_split, void* ws, hipStream_t st);
int s3_attn_tile_cap(const s3_kv_cache* c, const AttnArgs& p, const TileArgs& ta, hipStream_t st);
int s3_attn_tile_8(const s3_kv_cache* c, const AttnArgs& p, const TileArgs& ta, hipStream_t st);
int s3_attn_tile_8_cap(const s3_kv_cache* c, const AttnArgs& p, const TileArgs& ta, hipStream_t st);
