// What the attention's entry points call (host), with fewer than 2^22 tiles times heads.
#pragma once
#include "attn.h"

// Sequences, or tiles of listed blocks, of few rows (R: the most that one has, 128 at most); tiles: how many there can be.
size_t s3_attn_stream_workspace(int d_head, int R);
int s3_attn_stream(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, void* ws, hipStream_t st);

// Chunks, or tiles of listed blocks, of more rows: row tiles of s3_attn_tile_rows rows, the tokens of each in n_split parts.
int s3_attn_tile_rows(const s3_kv_cache* c);
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens, bool ragged);
size_t s3_attn_tile_workspace(const s3_kv_cache* c, int64_t units, int n_split);
int s3_attn_tile(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int n_split, void* ws, hipStream_t st);
