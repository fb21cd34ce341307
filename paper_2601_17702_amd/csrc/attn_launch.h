// What the attention's entry points call (host), with fewer than 2^22 tiles times heads.
#pragma once
#include "attn.h"

// The most rows of one sequence (or tile of listed blocks) that the streaming kernel takes; the tiled kernel has more, whose 256 rows a
// workgroup would stand mostly empty below.  us in the tiled / in the streaming kernel, 32 query heads over 8: 16 tokens of one sequence at
// 32768 with d_head 64: 42 / 27, of eight at 8000 with 256: 258 / 208, in fp32: 355 / 217 (32 tokens: 579 / 375); tiles of 16
// queries over 64 listed blocks of 512: 343 / 240, d_head 64: 276 / 154.  But bf16 with d_head 128, eight sequences: 66 / 73, where the tiled
// kernel's rate is best.
constexpr int s3_few_rows(bool bf16, int d_head, bool list, bool eight) {
    return !bf16 ? (d_head == 128 ? 128 : 64) : list || eight || d_head != 128 ? 64 : 32;
}

// Over an 8-bit cache, and with capped scores over one of bf16, 16 rows are a tile of their own, and whether one workgroup takes all tokens of such a tile and head, which saves the joining launch, or the
// line is cut in equal runs, goes by the bound that the host knows: the longest tile alone takes 4 us and 1 us for every 256 tokens.  us whole / cut, 8 heads of 128: one
// sequence of 512 7.0 / 11.1, of 1024 9.1 / 11.2, of 2048 13.3 / 11.3; 8 of 1024 9.4 / 11.5, of 2048 15.9 / 14.3; 64 of 512 15.3 / 21.9, of 2048 43 / 50; 256 of 2048
// 186 / 213.  Lists are about as long as one another, so for those more; lengths beyond 2048 may lie far apart, and one of 8192 among short ones would take 39 alone.
// The other builds, on another card, with 64 / 256 channels over 8 bits, then 64, 128 and 256 over bf16 with a cap: one of 512 6.1 / 9.8, 9.8 / 12.0; 6.8 / 9.5, 7.6 / 10.0, 9.7 / 11.4; 64 of 512
// 8.6 / 12.6, 30.1 / 38.3; 14.9 / 18.4, 23.2 / 28.7, 45.5 / 54.0; 64 of 2048 24.8 / 28.8, 99.8 / 108; 42.6 / 46.4, 94.0 / 99.4, 183 / 192; 64 lists of 8192 98.8 / 102, 362 / 369; 184 / 188, 359 / 363,
// 701 / 710.  The rule does not look at the width: one of 1024 is 7.7 / 10.0 with 64 channels and 10.3 / 10.2 with 128 in bf16, but with 256 13.9 / 12.2 over 8 bits and 13.3 / 11.5 over bf16, and eight of
// 1024 15.8 / 14.9 there over 8 bits (18.6 / 25.8 over bf16): up to 2 us are lost with that width and few tiles.
constexpr bool s3_has_tiles16(bool eight, bool bf16, bool cap) { return eight || (bf16 && cap); }
constexpr bool s3_whole_tiles(int R, bool list, int64_t units, int64_t tokens) {
    return R <= 16 && (tokens <= 1024 || (units >= 256 && tokens <= (list ? 8192 : 2048)));
}

// Sequences, or tiles of listed blocks, of few rows (R: the most that one has, 128 at most); tiles: how many there can be;
// most_tokens: a bound of what one sees.
size_t s3_attn_stream_workspace(const s3_kv_cache* c, bool list, int R, int64_t units, int64_t most_tokens);
int s3_attn_stream(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
// Its builds for capped scores, for 8-bit caches (dtype kS3E4m3), and for both.
int s3_attn_stream_cap(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
int s3_attn_stream_8(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);
int s3_attn_stream_8_cap(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int R, int64_t most_tokens, void* ws, hipStream_t st);

// Chunks, or tiles of listed blocks, of more rows: row tiles of s3_attn_tile_rows rows, the tokens of each in n_split parts.
int s3_attn_tile_rows(const s3_kv_cache* c);
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens, bool ragged);
size_t s3_attn_tile_workspace(const s3_kv_cache* c, int64_t units, int n_split);
struct TileArgs {
    float* slots;             // partial sums where n_split > 1
    int n_split, tiles;       // row tiles that there can be
};
static_assert(sizeof(AttnArgs) + sizeof(TileArgs) <= 176, "arguments of the builds without caps over bf16 and fp32: see AttnMore");
int s3_attn_tile(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int n_split, bool small, void* ws, hipStream_t st);      // small: of 128 rows, where a call's other tiles would have 256
// Whether an uncut call of the builds for 8 bits and for caps takes tiles of 128 rows: where those of 256 would leave half of the 256 compute
// units idle. Dim 128, 8 heads with 4 query heads each, one sequence, tiles of 256 rows against tiles of 128, in us: 64 tokens of e4m3 11
// against 9, 256 17 against 15, 512 24 against 22, 1024 (128 units) 39 against 38; with bf16 and a cap 12 against 9, 19 against 16, 28
// against 24, 47 against 41. At 160 units and more it turns: four sequences of 300 tokens 18 against 23, of 2048 (256 units) 71 against 79.
// Dim 64, the same calls: e4m3 8.1 against 6.9, 12.4 against 10.9, 18.1 against 16.2, 29.6 against 26.5; bf16 and a cap 8.3 against 6.9, 14.2 against
// 11.7, 21.9 against 18.3, 37.4 against 31.2.
constexpr bool s3_has_small_tiles(bool eight, bool bf16, int d_head, bool cap) { return (eight || (bf16 && cap)) && d_head <= 128; }
constexpr bool s3_small_tiles(bool eight, bool bf16, int d_head, bool cap, int64_t units, int n_split) {
    return s3_has_small_tiles(eight, bf16, d_head, cap) && n_split == 1 && units <= 128;
}
int s3_attn_tile_cap(const s3_kv_cache* c, const AttnMore& p, const TileArgs& ta, bool small, hipStream_t st);
int s3_attn_tile_8(const s3_kv_cache* c, const AttnMore& p, const TileArgs& ta, bool small, hipStream_t st);
int s3_attn_tile_8_cap(const s3_kv_cache* c, const AttnMore& p, const TileArgs& ta, bool small, hipStream_t st);
