// Attention of new tokens over a paged cache (s3_paged_attention), and over listed blocks of it (s3_block_attention).
#include "attn_launch.h"

namespace {

template <typename T, int D, bool LIST>
__global__ __launch_bounds__(64) void attn_rows_kernel(AttnArgs p) {
    constexpr int E = KvElem<T>::E, NW = 16 / E;
    typedef typename KvElem<T>::vec vec;
    const int lane = threadIdx.x, half = lane >> 5, col = lane & 31;
    const int head = blockIdx.x % p.n_kv;
    const int logp = p.b.log_page, P = 1 << logp;
    auto count = [&](int q) {
        int first, n, len;
        kv_seq(p.b, q, first, n, len);
        return LIST ? (n + p.qb - 1) / p.qb * p.per_q : p.few && n * p.G <= 32 ? 0 : (n * p.G + 31) / 32;
    };
    int s, j;
    const int tile = blockIdx.x / p.n_kv;
    if (!kv_find(p.b.n_seq, tile, count, s, j)) return;
    int first, n, len;
    kv_seq(p.b, s, first, n, len);
    int r0 = j * 32, r_end = n * p.G;
    if (LIST) {
        const int qt = j / p.per_q;
        r0 = qt * p.qb * p.G + (j - qt * p.per_q) * 32;
        r_end = min(n, (qt + 1) * p.qb) * p.G;
        if (r0 >= r_end) return;
    }
    AttnRows<T, D> rows;
    rows.load(p, head, first, n, len, r0 + col, r_end);
    AttnState<T, D> st;
    st.clear();
    const int last = len - n + (min(r0 + 32, r_end) - 1) / p.G;             // position of the tile's last row
    const int top_pos = min(last + 1, kv_blocks(p.b, len) << logp);         // tokens that some row may see
    const int first_pos = p.window ? max(0, len - n + r0 / p.G - p.window + 1) : 0;
    const AttnSight sight(rows.pos, top_pos, p.window);
    const int32_t* list = LIST ? p.sel + ((int64_t)(tile / p.per_q) * p.n_kv + head) * p.top : nullptr;
    const int n_sub = LIST ? p.top * (P / 16) : (top_pos - (first_pos & ~15) + 15) / 16;    // runs of 16 tokens: they lie in one page
    const int64_t page_bytes = (int64_t)P * D * (int)sizeof(T);
    for (int u = 0; u < n_sub; u += 2) {
        int base[2];
        const char *kp[2], *vp[2];
        bool on[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            int pos = -1;
            if (u + x < n_sub) {
                if (LIST) {
                    const int blk = list[(u + x) >> (logp - 4)];
                    pos = blk < 0 || blk >= p.b.max_pages ? -1 : (blk << logp) + ((u + x) & (P / 16 - 1)) * 16;
                } else {
                    pos = (first_pos & ~15) + (u + x) * 16;
                }
            }
            const int page = pos >= 0 && pos < top_pos ? kv_page(p.b, s, pos >> logp) : -1;
            on[x] = page >= 0;
            base[x] = pos;
            const int64_t at = ((int64_t)max(page, 0) * p.n_kv + head) * page_bytes;
            kp[x] = p.k + at + (pos & (P - 1)) * 16 * (on[x] ? 1 : 0);
            vp[x] = p.v + at + (on[x] ? (pos & (P - 1)) / E : 0) * (D * 16);
        }
        if (!on[0] && !on[1]) continue;
        kv_f32x16 sc[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[0][i] = 0.0f;
        const int tk = kv_token<T>(col);
        const char* ka = kp[tk >> 4] + (tk & 15) * 16 + half * (P * 16);
#pragma unroll
        for (int q = 0; q < kQSteps<D, T>; ++q) sc[0] = kv_mma(*(const vec*)(ka + (int64_t)q * 2 * P * 16), rows.q[q], sc[0]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int t = 2 * E * (i / E) + E * half + i % E, x = t >> 4, pos = base[x] + (t & 15);
            sc[0][i] = on[x] && sight.sees(pos) ? sc[0][i] : -INFINITY;
        }
        vec w[NW], vf[D / 32 * NW];
        st.softmax(sc, p.sl, w);
        unsigned big = 0;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int y = 0; y < NW; ++y) {
                const int t = E * (2 * y + half);
                vec& v = vf[dt * NW + y];
                v = kv_first(*(const vec*)(vp[t >> 4] + (t & 15) / E * (D * 16) + (dt * 32 + col) * 16), on[t >> 4] ? top_pos - base[t >> 4] - (t & 15) : 0);
                big = kv_magnitude(v, big);
            }
        const bool odd = __ballot(big >= 0x7f800000u);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int y = 0; y < NW; ++y) st.o[dt] = kv_mma(odd ? kv_finite(vf[dt * NW + y]) : vf[dt * NW + y], w[y], st.o[dt]);
        if (odd)
#pragma unroll 1
            for (int j = 0; j < 32; ++j) {
                const int x = j >> 4;
                if (!on[x] || base[x] + (j & 15) >= top_pos) continue;
                const char* v = vp[x] + (j & 15) / E * (D * 16) + j % E * (int)sizeof(T);
                st.add_nonfinite(sight.sees(base[x] + (j & 15)), [&](int c) { return (float)*(const T*)(v + c * 16); });
            }
    }
    const float l = kv_pair_sum(st.l);
    const float inv = kv_inverse(l);
    if (rows.row < 0) return;
    char* out = p.out + rows.row * (D * (int)sizeof(T));
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            typedef __attribute__((ext_vector_type(4))) T four;
            four x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (T)(st.o[dt][a * 4 + e] * inv);
            *(four*)(out + (dt * 32 + a * 8 + half * 4) * (int)sizeof(T)) = x;
        }
    if (p.lse && half == 0) p.lse[rows.row] = kv_lse(st.m, l);
}

int64_t row_tiles(const s3_kv_batch* b, int G, int rows) { return ((int64_t)b->n_tokens * G + (int64_t)b->n_seq * (rows - 1)) / rows; }

template <typename T, int D, bool LIST>
int launch(const AttnArgs& p, int64_t tiles, hipStream_t st) {
    const int64_t grid = tiles * p.n_kv;
    if (grid >= (int64_t)1 << 26) return s3_fail(S3_EINVAL, "attention: too many tokens in one call");
    hipLaunchKernelGGL((attn_rows_kernel<T, D, LIST>), dim3((unsigned)grid), dim3(64), 0, st, p);
    S3_HIP(hipGetLastError());
    return S3_OK;
}
template <bool LIST>
int launch_any(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, hipStream_t st) {
    if (c->dtype == S3_BF16) {
        if (c->d_head == 64) return launch<__bf16, 64, LIST>(p, tiles, st);
        if (c->d_head == 128) return launch<__bf16, 128, LIST>(p, tiles, st);
        return launch<__bf16, 256, LIST>(p, tiles, st);
    }
    if (c->d_head == 64) return launch<float, 64, LIST>(p, tiles, st);
    if (c->d_head == 128) return launch<float, 128, LIST>(p, tiles, st);
    return launch<float, 256, LIST>(p, tiles, st);
}

// 0: to be launched; 1: nothing to do; negative: an error.
int check(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs, float scale,
          const void* out) {
    if (int rc = s3_kv_check(fn, c, b)) return rc;
    if (n_q < 1 || n_q % c->n_kv_heads || n_q / c->n_kv_heads > 32) return s3_fail(S3_EINVAL, "%s: %d query heads over %d", fn, n_q, c->n_kv_heads);
    if (!(scale > 0.0f) || isinf(scale)) return s3_fail(S3_EINVAL, "%s: scale %g", fn, (double)scale);
    if (b->n_tokens == 0 || b->n_seq == 0) return 1;
    if (int rc = s3_kv_check_rows(fn, "q", c, q, q_ts, q_hs, n_q)) return rc;
    if (!out || (uintptr_t)out & 15) return s3_fail(S3_EINVAL, "%s: out is null or not 16-byte aligned", fn);
    return 0;
}
int check_ws(const char* fn, const void* ws, size_t ws_bytes, size_t need) {
    if (need && (!ws || (uintptr_t)ws & 255)) return s3_fail(S3_EINVAL, "%s: workspace is null or not 256-byte aligned", fn);
    if (ws_bytes < need) return s3_fail(S3_ECAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    return S3_OK;
}

// Rows of one sequence, or of one tile of listed blocks, and how the call is shared out: the streaming kernel has those of at most 32
// rows, the tiled one the others.
struct Plan {
    int G, R;
    bool few, many;
    size_t need;
    int64_t few_tiles;
    Plan(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block) {
        G = n_q / c->n_kv_heads;
        const int64_t most = (int64_t)min(q_block ? q_block : max(b->max_new, 1), max(b->n_tokens, 1)) * G;
        few = most <= 32 || (!q_block && b->n_seq > 1);
        many = most > 32;
        R = (int)min(most, (int64_t)32);
        few_tiles = q_block ? s3_block_tiles(b, q_block) : b->n_seq;
        need = few ? s3_attn_stream_workspace(c->d_head, R) : 0;
    }
};

int run(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b, AttnArgs p, const Plan& plan, int64_t tiles, void* ws, hipStream_t st) {
    p.few = plan.few && plan.many;
    if (plan.few)
        if (int rc = s3_attn_stream(c, p, plan.few_tiles, plan.R, ws, st)) return rc;
    if (plan.many) return p.sel ? launch_any<true>(c, p, tiles, st) : launch_any<false>(c, p, tiles, st);
    return S3_OK;
}

bool shapes_ok(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return !s3_kv_check("workspace", c, b) && n_q >= 1 && n_q % c->n_kv_heads == 0 && n_q / c->n_kv_heads <= 32;
}

}  // namespace

extern "C" size_t s3_paged_attention_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q) {
    return shapes_ok(c, b, n_q) ? Plan(c, b, n_q, 0).need : 0;
}

extern "C" int s3_paged_attention(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                  float scale, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "s3_paged_attention";
    if (window < 0) return s3_fail(S3_EINVAL, "%s: window %d", fn, window);
    if (int rc = check(fn, c, b, q, n_q, q_ts, q_hs, scale, out)) return rc < 0 ? rc : S3_OK;
    const Plan plan(c, b, n_q, 0);
    if (int rc = check_ws(fn, ws, ws_bytes, plan.need)) return rc;
    const int es = c->dtype == S3_BF16 ? 2 : 4;
    AttnArgs p{s3_kv_batch_args(c, b), (const char*)q, (char*)out, lse, (const char*)c->k, (const char*)c->v, nullptr, q_ts * es,
               q_hs * es, c->n_kv_heads, plan.G, n_q, window, 0, 0, 1, scale * 1.4426950408889634f, 0};
    return run(fn, c, b, p, plan, row_tiles(b, plan.G, 32), ws, (hipStream_t)stream);
}

extern "C" int64_t s3_block_tiles(const s3_kv_batch* b, int q_block) {
    return b && q_block >= 1 ? ((int64_t)b->n_tokens + (int64_t)b->n_seq * (q_block - 1)) / q_block : 0;
}

extern "C" size_t s3_block_attention_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b) {
    return shapes_ok(c, b, n_q) && q_block >= 1 && top_b >= 1 ? Plan(c, b, n_q, q_block).need : 0;
}

extern "C" int s3_block_attention(const s3_kv_cache* c, const s3_kv_batch* b, const void* q, int n_q, int64_t q_ts, int64_t q_hs,
                                  const int32_t* sel, int q_block, int top_b, float scale, void* out, float* lse, void* ws,
                                  size_t ws_bytes, void* stream) {
    const char* fn = "s3_block_attention";
    if (q_block < 1 || top_b < 1 || q_block > 1 << 20 || top_b > 4096) return s3_fail(S3_EINVAL, "%s: q_block %d, top_b %d", fn, q_block, top_b);
    if (int rc = check(fn, c, b, q, n_q, q_ts, q_hs, scale, out)) return rc < 0 ? rc : S3_OK;
    if (!sel) return s3_fail(S3_EINVAL, "%s: null sel", fn);
    const Plan plan(c, b, n_q, q_block);
    if (int rc = check_ws(fn, ws, ws_bytes, plan.need)) return rc;
    const int es = c->dtype == S3_BF16 ? 2 : 4, qb = min(q_block, b->n_tokens);
    const int per_q = (int)(((int64_t)qb * plan.G + 31) / 32);
    AttnArgs p{s3_kv_batch_args(c, b), (const char*)q, (char*)out, lse, (const char*)c->k, (const char*)c->v, sel, q_ts * es,
               q_hs * es, c->n_kv_heads, plan.G, n_q, 0, qb, top_b, per_q, scale * 1.4426950408889634f, 0};
    return run(fn, c, b, p, plan, s3_block_tiles(b, q_block) * per_q, ws, (hipStream_t)stream);
}
