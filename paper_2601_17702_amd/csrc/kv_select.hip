// The blocks that each tile of queries will read (s3_block_select): scores of all candidates by matrix instructions, then the
// top_b largest of each list by a radix search on the scores' ordered keys.
#include "attn.h"

namespace {

constexpr int kThreads = 256;
constexpr int kScoreBlocks = 512;      // blocks of one scoring workgroup

struct SelectArgs {
    KvBatch b;
    const char* q;
    int64_t q_ts, q_hs;                // bytes
    const __bf16* sig;
    unsigned* keys;                    // [tiles][n_kv][nb] ordered scores, 0: no candidate
    int32_t* sel;
    int n_kv, G, qb, top, lead, tail, nb;
};

__device__ __forceinline__ unsigned order_key(float f) {         // larger float, larger key; never 0 or all ones for finite f
    const unsigned u = __float_as_uint(f + 0.0f);                // -0 counts as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A tile's place in its sequence: its rows, and the blocks it may choose from.
struct Tile {
    int s, first, n, len, t0, t1, nb;      // tokens t0 .. t1 - 1 of the sequence's n; candidates 0 .. nb - 1
    __device__ __forceinline__ bool find(const SelectArgs& p, int tile) {
        int j;
        auto count = [&](int q) {
            int f, m, l;
            kv_seq(p.b, q, f, m, l);
            return (m + p.qb - 1) / p.qb;
        };
        if (!kv_find(p.b.n_seq, tile, count, s, j)) return false;
        kv_seq(p.b, s, first, n, len);
        t0 = j * p.qb;
        t1 = min(n, t0 + p.qb);
        const int last = len - n + t1 - 1;
        nb = last < 0 ? 0 : min(min((last >> p.b.log_page) + 1, p.b.max_pages), p.nb);
        return true;
    }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void sel_score_kernel(SelectArgs p) {
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, wave = threadIdx.x >> 6;
    const int head = blockIdx.x % p.n_kv, tile = blockIdx.x / p.n_kv;
    Tile t;
    if (!t.find(p, tile)) return;
    const int b0 = blockIdx.y * kScoreBlocks;
    if (b0 >= t.nb) return;
    const int b1 = min(t.nb, b0 + kScoreBlocks);
    unsigned* keys = p.keys + ((int64_t)tile * p.n_kv + head) * p.nb;
    const int p0 = max(0, t.len - t.n + t.t0);
    const int own = p.tail > 0 ? (p0 >> p.b.log_page) - p.tail + 1 : 1 << 30;      // blocks from here on are always taken
    for (int r0 = t.t0 * p.G; r0 < t.t1 * p.G; r0 += 32) {
        // 32 rows on their grids, as operand A: channel 16 s + 8 half + e of row col
        kv_bf16x8 a[D / 16];
        const int r = r0 + col;
        float x[D / 16][8];
        unsigned big = 0;
        if (r < t.t1 * p.G) {
            const int tk = r / p.G, g = r - tk * p.G;
            const char* src = p.q + (int64_t)(t.first + tk) * p.q_ts + (int64_t)(head * p.G + g) * p.q_hs + half * (8 * (int)sizeof(T));
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int e = 0; e < 8; e += KvElem<T>::E) {
                    const auto v = *(const typename KvElem<T>::vec*)(src + (s * 16 + e) * (int)sizeof(T));
#pragma unroll
                    for (int i = 0; i < KvElem<T>::E; ++i) x[s][e + i] = (float)v[i];
                }
        } else {
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[s][e] = -INFINITY;        // a row that does not exist: zero, see below
        }
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[s][e]) & 0x7fffffffu);
        big = max(big, (unsigned)__shfl_xor((int)big, 32));
        bool ok;
        const int ex = kv_grid_exp(big, ok);
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) a[s][e] = (__bf16)(ok ? kv_grid(x[s][e], ex) : 0.0f);
        const int rows = min(32, t.t1 * p.G - r0);
        for (int b = b0 + wave * 32; b < b1; b += kThreads / 2) {
            const int blk = b + col;
            const int page = blk < b1 ? kv_page(p.b, t.s, blk) : -1;
            const __bf16* sg = p.sig + ((int64_t)max(page, 0) * p.n_kv + head) * D + half * 8;
            kv_f32x16 c;
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = 0.0f;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) c = kv_mma(a[s], *(const kv_bf16x8*)(sg + s * 16), c);
            float best = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i / 4) + 4 * half + i % 4 < rows) best = fmaxf(best, c[i]);
            best = kv_pair_max(best);
            if (half == 0 && blk < b1) {
                unsigned key = page < 0 ? 0u : blk < p.lead || blk >= own ? 0xffffffffu : order_key(best);
                if (r0 > t.t0 * p.G) key = max(key, keys[blk]);
                keys[blk] = key;
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void sel_pick_kernel(SelectArgs p) {
    __shared__ int hist[256];
    __shared__ int wsum[2 * (kThreads / 64)];
    __shared__ unsigned found[2];
    const int tid = threadIdx.x;
    const int head = blockIdx.x % p.n_kv, tile = blockIdx.x / p.n_kv;
    int32_t* out = p.sel + ((int64_t)tile * p.n_kv + head) * p.top;
    Tile t;
    const bool there = t.find(p, tile);
    const int nb = there ? t.nb : 0;
    const unsigned* keys = p.keys + ((int64_t)tile * p.n_kv + head) * p.nb;
    // the top_b-th largest key, eight bits at a time; `left`: how many of the keys equal to it are taken
    unsigned thr = 0, mask = 0;
    int left = p.top;
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < nb; i += kThreads) {
            const unsigned k = keys[i];
            if ((k & mask) == thr && k) atomicAdd(&hist[k >> shift & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int bin = 255;
            for (; bin > 0 && hist[bin] < left; --bin) left -= hist[bin];
            found[0] = (unsigned)bin;
            found[1] = (unsigned)left;
        }
        __syncthreads();
        thr |= found[0] << shift;
        left = (int)found[1];
        mask |= 255u << shift;
        __syncthreads();
    }
    // ascending blocks: larger keys, and the first `left` of the equal ones (thr 0: there are fewer candidates than asked for)
    int n = 0, eq = 0;
    for (int base = 0; base < nb; base += kThreads) {
        const int i = base + tid;
        const unsigned k = i < nb ? keys[i] : 0u;
        int total;
        const int same = k == thr && k ? 1 : 0;
        const int before = eq + s3_block_excl_scan<kThreads>(same, wsum, total);
        eq += total;
        __syncthreads();
        const int take = k > thr || (same && before < left) ? 1 : 0;
        const int at = n + s3_block_excl_scan<kThreads>(take, wsum, total);
        n += total;
        __syncthreads();
        if (take && at < p.top) out[at] = i;
    }
    for (int i = n + tid; i < p.top; i += kThreads) out[i] = -1;
}

int select_blocks(const s3_kv_cache* c, const s3_kv_batch* b) {
    return (int)max((int64_t)1, min((int64_t)b->max_pages, ((int64_t)b->max_kv + c->page_size - 1) / c->page_size));
}

}  // namespace

extern "C" size_t s3_block_select_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b) {
    if (s3_kv_check("s3_block_select_workspace", c, b) || q_block < 1) return 0;
    return s3_align((size_t)s3_block_tiles(b, q_block) * c->n_kv_heads * select_blocks(c, b) * 4);
}

extern "C" int s3_block_select(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs, int q_block,
                               int top_b, int lead, int tail, int32_t* sel, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_block_select";
    if (int rc = s3_kv_check(fn, c, b)) return rc;
    if (!c->sig) return s3_fail(S3_EINVAL, "%s: the cache has no signatures", fn);
    if (n_q < 1 || n_q % c->n_kv_heads || n_q / c->n_kv_heads > 32) return s3_fail(S3_EINVAL, "%s: %d query heads over %d", fn, n_q, c->n_kv_heads);
    if (q_block < 1 || q_block > 1 << 20 || top_b < 1 || top_b > 4096 || lead < 0 || tail < 0)
        return s3_fail(S3_EINVAL, "%s: q_block %d, top_b %d, lead %d, tail %d", fn, q_block, top_b, lead, tail);
    if ((int64_t)lead + tail + (q_block + c->page_size - 2) / c->page_size > top_b && tail > 0)
        return s3_fail(S3_EINVAL, "%s: top_b %d does not hold the blocks that are always taken", fn, top_b);
    if (lead > top_b) return s3_fail(S3_EINVAL, "%s: top_b %d, lead %d", fn, top_b, lead);
    const int64_t tiles = s3_block_tiles(b, q_block);
    if (tiles == 0) return S3_OK;
    if (b->n_tokens)
        if (int rc = s3_kv_check_rows(fn, "q", c, q, q_ts, q_hs, n_q)) return rc;
    if (!sel) return s3_fail(S3_EINVAL, "%s: null sel", fn);
    const size_t need = s3_block_select_workspace(c, b, n_q, q_block, top_b);
    if (!ws || (uintptr_t)ws & 255) return s3_fail(S3_EINVAL, "%s: workspace is null or not 256-byte aligned", fn);
    if (ws_bytes < need) return s3_fail(S3_ECAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    if (tiles * c->n_kv_heads >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "%s: too many tiles in one call", fn);
    const int es = c->dtype == S3_BF16 ? 2 : 4, nb = select_blocks(c, b);
    SelectArgs p{s3_kv_batch_args(c, b), (const char*)q, q_ts * es, q_hs * es, (const __bf16*)c->sig, (unsigned*)ws, sel,
                 c->n_kv_heads, n_q / c->n_kv_heads, q_block, top_b, lead, tail, nb};
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)(tiles * c->n_kv_heads), (unsigned)((nb + kScoreBlocks - 1) / kScoreBlocks));
    if ((int64_t)grid.x * grid.y >= (int64_t)1 << 24 || grid.y > 65535) return s3_fail(S3_EINVAL, "%s: too many tiles in one call", fn);
#define S3_SCORE(T, D) hipLaunchKernelGGL((sel_score_kernel<T, D>), grid, dim3(kThreads), 0, st, p)
    if (c->dtype == S3_BF16) {
        if (c->d_head == 64) S3_SCORE(__bf16, 64);
        else if (c->d_head == 128) S3_SCORE(__bf16, 128);
        else S3_SCORE(__bf16, 256);
    } else {
        if (c->d_head == 64) S3_SCORE(float, 64);
        else if (c->d_head == 128) S3_SCORE(float, 128);
        else S3_SCORE(float, 256);
    }
#undef S3_SCORE
    S3_HIP(hipGetLastError());
    hipLaunchKernelGGL(sel_pick_kernel, dim3(grid.x), dim3(kThreads), 0, st, p);
    S3_HIP(hipGetLastError());
    return S3_OK;
}
