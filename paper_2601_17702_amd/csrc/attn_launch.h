// What the attention's entry points call (host).
#pragma once
#include "attn.h"

// Sequences, or tiles of listed blocks, of at most 32 rows (R: the most that one has); tiles: how many there can be.
size_t s3_attn_stream_workspace(int d_head, int R);
int s3_attn_stream(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, void* ws, hipStream_t st);
