// Attention of many rows over bf16 and fp32 caches; which of its builds a call takes, and into how many parts it is cut.
#include "attn_tile_impl.inc"

namespace {
int rows_of(const s3_kv_cache* c) { return c->d_head * (c->dtype == S3_FP32 ? 4 : 2) > 256 ? 128 : 256; }
}  // namespace

int s3_attn_tile_rows(const s3_kv_cache* c) { return rows_of(c); }

// Into how many parts the tokens of a row tile are cut.  One workgroup fills a compute unit, so units tiles * heads take
// ceil(units / 256) turns of all their steps; parts make the last turn fuller, at the price of writing fp32 sums and joining them.
// In us, with the rates that the kernel reaches on a compute unit: 3.8 TFLOP/s in bf16 and 0.45 in fp32, 6 us for the joining
// kernel, a part's sums written and read at 20 GB/s, and 4 us for its beginning.
// Ragged: the tiles are of several sequences whose lengths the host does not know, and those that see little count for nothing.  The cost is then
// summed over five guesses: all tiles see the most, 7/8, 3/4, 5/8 or half of them do.  us with the parts for equal lengths / with these: 217 tokens at 3519 and
// 102066, 28 heads over 4: 565 / 464; three times 300 at 2000, 20000 and 50000 with d_head 256: 1387 / 935; 500 at 3000 and 30000 in fp32: 1018 / 723; 2048 at
// 2048 beside eight times 30 at 131072: 1288 / 1018; but four times 1024 at 16384, which are equal: 939 / 1030.
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens, bool ragged) {
    const bool bf = c->dtype != S3_FP32;
    const int kt = c->d_head * (bf ? 2 : 4) > 512 ? 32 : 64;
    const int64_t steps = (tokens + kt - 1) / kt;
    const double step = 4.0 * rows_of(c) * kt * c->d_head / (bf ? 3.8e6 : 0.45e6), sums = rows_of(c) * (c->d_head + 2) * 4 / 10e3 + 4.0;
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= 64 && n <= steps; ++n) {
        int64_t turns = 0;
        for (int eighths = ragged ? 4 : 8; eighths <= 8; ++eighths) turns += (units * eighths / 8 * n + 255) / 256;
        const double cost = (double)turns * ((double)((steps + n - 1) / n) * step + (n > 1 ? sums : 0.0)) + (n > 1 ? 6.0 : 0.0) * (ragged ? 5 : 1);
        if (cost < least * 0.97) {
            least = cost;
            best = n;
        }
        if (units * n >= 2048) break;
    }
    return best;
}

size_t s3_attn_tile_workspace(const s3_kv_cache* c, int64_t units, int n_split) {
    return n_split > 1 ? s3_align((size_t)units * n_split * rows_of(c) * (c->d_head + 2) * 4) : 0;
}

int s3_attn_tile(const s3_kv_cache* c, const AttnMore& p, int64_t tiles, int n_split, bool small, void* ws, hipStream_t st) {
    const TileArgs ta{(float*)ws, n_split, (int)tiles};
    if (c->dtype == kS3E4m3) return p.cap != 0.0f ? s3_attn_tile_8_cap(c, p, ta, small, st) : s3_attn_tile_8(c, p, ta, small, st);
    if (p.cap != 0.0f) return s3_attn_tile_cap(c, p, ta, small, st);
    return c->dtype == S3_BF16 ? launch_tile<__bf16, false>(c->d_head, p, ta, small, st) : launch_tile<float, false>(c->d_head, p, ta, small, st);
}
