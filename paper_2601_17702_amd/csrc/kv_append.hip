// Appending to a paged cache: rotation, the two layouts, the signatures (s3_kv_append), and the rotation's table.
#include "kv_cache.h"

namespace {

constexpr int kThreads = 256;

struct AppendArgs {
    KvBatch b;
    char* kc;
    char* vc;
    __bf16* sig;
    const char *k, *v, *q;
    char* q_out;
    int64_t k_ts, k_hs, v_ts, v_hs, q_ts, q_hs;      // bytes
    const float* rope;
    const int32_t* positions;
    int64_t n_pos;
    int rot, inter, n_kv, n_q;
    unsigned page_items;                             // workgroups of pages; the rest rotate queries
};

// E channels of one row and, for pairs (i, i + rot / 2), their E partners.  c, s: E (interleaved: E / 2) values each.
template <typename T>
__device__ __forceinline__ void rotate_halves(typename KvElem<T>::vec& a, typename KvElem<T>::vec& b, const float* c, const float* s) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < KvElem<T>::E; ++i) {
        const float x = (float)a[i], y = (float)b[i];
        a[i] = (T)(x * c[i] - y * s[i]);
        b[i] = (T)(y * c[i] + x * s[i]);
    }
}
template <typename T>
__device__ __forceinline__ void rotate_pairs(typename KvElem<T>::vec& a, const float* c, const float* s) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < KvElem<T>::E / 2; ++i) {
        const float x = (float)a[2 * i], y = (float)a[2 * i + 1];
        a[2 * i] = (T)(x * c[i] - y * s[i]);
        a[2 * i + 1] = (T)(y * c[i] + x * s[i]);
    }
}

// Item i of a row: one group of E channels, or a group and its partner.  How many there are, and which groups.
template <typename T, int D>
__device__ __forceinline__ int row_items(const AppendArgs& p) {
    constexpr int E = KvElem<T>::E;
    return p.rope && !p.inter ? D / E - p.rot / (2 * E) : D / E;
}
template <typename T, int D, typename Put>
__device__ __forceinline__ void row_item(const AppendArgs& p, const char* row, int item, int token, int pos, Put put) {
    constexpr int E = KvElem<T>::E;
    typedef typename KvElem<T>::vec vec;
    const int halves = p.rope && !p.inter ? p.rot / (2 * E) : 0;
    int g = item < halves ? item : item + halves;
    vec a = *(const vec*)(row + g * 16);
    if (p.rope && (item < halves || (p.inter && g * E < p.rot))) {
        int64_t r = p.positions ? p.positions[token] : pos;
        r = max((int64_t)0, min(r, p.n_pos - 1));
        const float* c = p.rope + r * p.rot;
        if (p.inter) {
            rotate_pairs<T>(a, c + g * (E / 2), c + p.rot / 2 + g * (E / 2));
        } else {
            vec b = *(const vec*)(row + (g + halves) * 16);
            rotate_halves<T>(a, b, c + g * E, c + p.rot / 2 + g * E);
            put(g + halves, b);
        }
    }
    put(g, a);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs p) {
    constexpr int E = KvElem<T>::E, NG = D / E;
    typedef typename KvElem<T>::vec vec;
    const int tid = threadIdx.x;
    const int items = row_items<T, D>(p);

    if (blockIdx.x >= p.page_items) {                // queries: one item of a row per thread
        int64_t i = (int64_t)(blockIdx.x - p.page_items) * kThreads + tid;
        const int item = (int)(i % items);
        i /= items;
        const int head = (int)(i % p.n_q);
        const int64_t token = i / p.n_q;
        if (token >= p.b.n_tokens) return;
        int s = (int)token;
        if (p.b.q_start) {                           // the last sequence that starts at or before the token
            int lo = 0, hi = p.b.n_seq;
            while (hi - lo > 1) {
                const int m = (lo + hi) / 2;
                if (p.b.q_start[m] <= token) lo = m;
                else hi = m;
            }
            s = lo;
        }
        int first, n, len;
        kv_seq(p.b, s, first, n, len);
        if (token < first || token >= first + n) return;
        char* out = p.q_out + (token * p.n_q + head) * (D * (int)sizeof(T));
        row_item<T, D>(p, p.q + token * p.q_ts + head * p.q_hs, item, (int)token, len - n + (int)(token - first),
                       [&](int g, vec x) { *(vec*)(out + g * 16) = x; });
        return;
    }

    // one page of one head
    const int h = blockIdx.x % p.n_kv;
    const int logp = p.b.log_page, P = 1 << logp;
    int s, j;
    auto count = [&](int q) {
        int first, n, len;
        kv_seq(p.b, q, first, n, len);
        const int p0 = max(0, len - n);
        return n > 0 && len > 0 ? ((len - 1) >> logp) - (p0 >> logp) + 1 : 0;
    };
    if (!kv_find(p.b.n_seq, blockIdx.x / p.n_kv, count, s, j)) return;
    int first, n, len;
    kv_seq(p.b, s, first, n, len);
    const int p0 = len - n;                          // position of the first new token (negative: tokens before the sequence)
    const int blk = (max(0, p0) >> logp) + j;
    const int page = kv_page(p.b, s, blk);
    if (page < 0) return;
    const int base = blk << logp, lo = max(p0, base) - base, hi = min(len - base, P);      // new slots lo .. hi - 1
    const int64_t at = ((int64_t)page * p.n_kv + h) * ((int64_t)P * D * (int)sizeof(T));
    char* kp = p.kc + at;
    char* vp = p.vc + at;
    for (int i = tid; i < (hi - lo) * items; i += kThreads) {
        const int slot = lo + i / items, token = first + (base + slot - p0);
        row_item<T, D>(p, p.k + token * p.k_ts + h * p.k_hs, i % items, token, base + slot,
                       [&](int g, vec x) { *(vec*)(kp + ((int64_t)g * P + slot) * 16) = x; });
    }
    for (int i = tid; i < ((hi + E - 1) / E - lo / E) * D; i += kThreads) {      // E slots of one channel
        const int c = i % D, g = lo / E + i / D;
        const char* src = p.v + h * p.v_hs + c * (int)sizeof(T);
        vec x;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int slot = g * E + e;
            if (slot >= lo && slot < hi) x[e] = *(const T*)(src + (int64_t)(first + (base + slot - p0)) * p.v_ts);
        }
        vec* dst = (vec*)(vp + ((int64_t)g * D + c) * 16);
        if (g * E >= lo && g * E + E <= hi) {
            *dst = x;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (g * E + e >= lo && g * E + e < hi) ((T*)dst)[e] = x[e];
        }
    }
    if (!p.sig) return;
    __shared__ float part[8][D];
    __shared__ unsigned biggest;
    if (tid == 0) biggest = 0;
    __threadfence_block();
    __syncthreads();
    for (int i = tid; i < NG * 8; i += kThreads) {
        const int g = i >> 3, r = i & 7;
        float sum[E] = {};
        for (int slot = r; slot < hi; slot += 8) {
            const vec x = *(const vec*)(kp + ((int64_t)g * P + slot) * 16);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += (float)x[e];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) part[r][g * E + e] = sum[e];
    }
    __syncthreads();
    float m = 0.0f;
    if (tid < D) {
        m = (((part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid])) +
             ((part[4][tid] + part[5][tid]) + (part[6][tid] + part[7][tid]))) / (float)hi;
        atomicMax(&biggest, __float_as_uint(m) & 0x7fffffffu);
    }
    __syncthreads();
    if (tid < D) {
        bool ok;
        const int e = kv_grid_exp(biggest, ok);
        p.sig[((int64_t)page * p.n_kv + h) * D + tid] = (__bf16)(ok ? kv_grid(m, e) : 0.0f);
    }
}

__global__ void kv_rope_kernel(float* table, int64_t n_pos, int half, double log_theta) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= n_pos * half) return;
    const int64_t pos = i / half;
    const int c = (int)(i % half);
    double sn, cs;
    sincos((double)pos * exp(-log_theta * (double)c / (double)half), &sn, &cs);
    table[pos * 2 * half + c] = (float)cs;
    table[pos * 2 * half + half + c] = (float)sn;
}

template <typename T, int D>
int launch_append(const AppendArgs& p, hipStream_t st) {
    AppendArgs a = p;
    const int E = KvElem<T>::E;
    const int64_t items = a.rope && !a.inter ? D / E - a.rot / (2 * E) : D / E;
    const int64_t qb = a.q ? ((int64_t)a.b.n_tokens * a.n_q * items + kThreads - 1) / kThreads : 0;
    const int64_t grid = (int64_t)a.page_items + qb;
    if (grid >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "s3_kv_append: too many tokens in one call");
    hipLaunchKernelGGL((kv_append_kernel<T, D>), dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    S3_HIP(hipGetLastError());
    return S3_OK;
}

}  // namespace

int s3_kv_check(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b) {
    if (!c || !b) return s3_fail(S3_EINVAL, "%s: null cache or batch", fn);
    if (c->dtype != S3_BF16 && c->dtype != S3_FP32) return s3_fail(S3_EINVAL, "%s: dtype %d", fn, c->dtype);
    if (c->d_head != 64 && c->d_head != 128 && c->d_head != 256) return s3_fail(S3_EINVAL, "%s: d_head %d not in {64, 128, 256}", fn, c->d_head);
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        return s3_fail(S3_EINVAL, "%s: page_size %d is no power of two from 16 to 256", fn, c->page_size);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 4096) return s3_fail(S3_EINVAL, "%s: %d pages, %d heads", fn, c->n_pages, c->n_kv_heads);
    if (!c->k || !c->v || ((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->sig) & 255)
        return s3_fail(S3_EINVAL, "%s: cache arrays must be given and 256-byte aligned", fn);
    if (b->n_seq < 0 || b->n_tokens < 0 || b->max_pages < 0 || b->max_new < 0 || b->max_kv < 0 || b->table_stride < b->max_pages)
        return s3_fail(S3_EINVAL, "%s: n_seq %d, n_tokens %d, max_pages %d, table_stride %lld, max_new %d, max_kv %d", fn, b->n_seq, b->n_tokens,
                       b->max_pages, (long long)b->table_stride, b->max_new, b->max_kv);
    if (b->n_seq > 1 << 20 || b->n_tokens > 1 << 24 || (int64_t)b->max_pages * c->page_size > 1 << 30)
        return s3_fail(S3_EINVAL, "%s: n_seq %d, n_tokens %d or max_pages %d too large", fn, b->n_seq, b->n_tokens, b->max_pages);
    if (!b->q_start && b->n_tokens != b->n_seq) return s3_fail(S3_EINVAL, "%s: without q_start there is one token per sequence", fn);
    if (b->n_seq && (!b->kv_len || !b->block_table)) return s3_fail(S3_EINVAL, "%s: null kv_len or block_table", fn);
    return S3_OK;
}

int s3_kv_check_rows(const char* fn, const char* what, const s3_kv_cache* c, const void* p, int64_t tok_stride, int64_t head_stride, int heads) {
    const int E = c->dtype == S3_BF16 ? 8 : 4;
    if (!p || (uintptr_t)p & 15) return s3_fail(S3_EINVAL, "%s: %s is null or not 16-byte aligned", fn, what);
    if (tok_stride % E || head_stride % E || tok_stride < 0 || head_stride < 0)
        return s3_fail(S3_EINVAL, "%s: strides %lld, %lld of %s are no multiples of 16 bytes", fn, (long long)tok_stride, (long long)head_stride, what);
    if (heads > 1 && head_stride < c->d_head && head_stride) return s3_fail(S3_EINVAL, "%s: heads of %s overlap", fn, what);
    return S3_OK;
}

extern "C" int s3_rope_table(float* table, int64_t n_pos, int rot_dim, double theta, void* stream) {
    if (!table || (uintptr_t)table & 15 || n_pos < 0 || n_pos > (int64_t)1 << 30 || rot_dim < 16 || rot_dim > 256 || rot_dim % 16 || !(theta > 0.0) || isinf(theta))
        return s3_fail(S3_EINVAL, "s3_rope_table: n_pos %lld, rot_dim %d, theta %g or the table's alignment", (long long)n_pos, rot_dim, theta);
    const int64_t n = n_pos * (rot_dim / 2);
    if (!n) return S3_OK;
    if ((n + 255) / 256 >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "s3_rope_table: %lld positions are too many", (long long)n_pos);
    hipLaunchKernelGGL(kv_rope_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, (hipStream_t)stream, table, n_pos, rot_dim / 2, log(theta));
    S3_HIP(hipGetLastError());
    return S3_OK;
}

extern "C" int s3_kv_append(const s3_kv_cache* c, const s3_kv_batch* b, const void* k, int64_t k_ts, int64_t k_hs, const void* v,
                            int64_t v_ts, int64_t v_hs, const float* rope, int64_t n_pos, int rot_dim, int interleaved,
                            const int32_t* positions, const void* q, int n_q, int64_t q_ts, int64_t q_hs, void* q_out, void* stream) {
    const char* fn = "s3_kv_append";
    if (int rc = s3_kv_check(fn, c, b)) return rc;
    if (b->n_tokens == 0 || b->n_seq == 0) return S3_OK;
    if (int rc = s3_kv_check_rows(fn, "k", c, k, k_ts, k_hs, c->n_kv_heads)) return rc;
    if (int rc = s3_kv_check_rows(fn, "v", c, v, v_ts, v_hs, c->n_kv_heads)) return rc;
    if (q) {
        if (n_q < 1 || n_q % c->n_kv_heads || n_q / c->n_kv_heads > 32) return s3_fail(S3_EINVAL, "%s: %d query heads over %d", fn, n_q, c->n_kv_heads);
        if (int rc = s3_kv_check_rows(fn, "q", c, q, q_ts, q_hs, n_q)) return rc;
        if (!q_out || (uintptr_t)q_out & 15) return s3_fail(S3_EINVAL, "%s: q_out is null or not 16-byte aligned", fn);
    }
    if (rope && (rot_dim < 16 || rot_dim % 16 || rot_dim > c->d_head || n_pos < 1 || (uintptr_t)rope & 15))
        return s3_fail(S3_EINVAL, "%s: rot_dim %d (a multiple of 16, d_head at most), n_pos %lld or the table's alignment", fn, rot_dim, (long long)n_pos);
    const int es = c->dtype == S3_BF16 ? 2 : 4, P = c->page_size;
    // pages that can get tokens: n tokens touch (n + P - 2) / P + 1 at most
    int64_t pages = b->n_seq + ((int64_t)b->n_tokens + (int64_t)b->n_seq * (P - 2)) / P;
    if (!b->q_start) pages = b->n_seq;
    if (pages * c->n_kv_heads >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "%s: too many tokens in one call", fn);
    AppendArgs p{s3_kv_batch_args(c, b), (char*)c->k, (char*)c->v, (__bf16*)c->sig, (const char*)k, (const char*)v, (const char*)q,
                 (char*)q_out, k_ts * es, k_hs * es, v_ts * es, v_hs * es, q_ts * es, q_hs * es, rope, positions, n_pos, rot_dim,
                 interleaved != 0, c->n_kv_heads, n_q, (unsigned)(pages * c->n_kv_heads)};
    hipStream_t st = (hipStream_t)stream;
    if (c->dtype == S3_BF16) {
        if (c->d_head == 64) return launch_append<__bf16, 64>(p, st);
        if (c->d_head == 128) return launch_append<__bf16, 128>(p, st);
        return launch_append<__bf16, 256>(p, st);
    }
    if (c->d_head == 64) return launch_append<float, 64>(p, st);
    if (c->d_head == 128) return launch_append<float, 128>(p, st);
    return launch_append<float, 256>(p, st);
}
