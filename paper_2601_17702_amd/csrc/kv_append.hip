// Appending to a paged cache: rotation, the two layouts, the signatures (s3_kv_append), and the rotation's table.
#include "kv_cache.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 4;            // whose queries one workgroup rotates, all their loads ahead, where there are many

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
    int group;                                       // tokens of such a one
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

// Slots that pass through LDS at a time: 16 KB of keys and of values, a row of 16 bytes more each (a column's reads then meet no bank twice).
template <typename T, int D> constexpr int kSlab = D * (int)sizeof(T) >= 1024 ? 16 : D * (int)sizeof(T) >= 512 ? 32 : 64;

// What bounds it: memory.  8 chunks of 2048 tokens, 32 query heads over 8 of 128 in bf16 (412 MB read and written) take 85 us, 4.8 TB/s: what a copy moves.
// Rows are read whole and pages written whole lines at a time, so both layouts' transpositions go through LDS; the signature's
// sums read the new keys there, too, and only a page's older keys come back from memory.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs p) {
    constexpr int E = KvElem<T>::E, NG = D / E, SLAB = kSlab<T, D>, ROW = D * (int)sizeof(T) + 16;
    typedef typename KvElem<T>::vec vec;
    const int tid = threadIdx.x;
    const int items = row_items<T, D>(p);

    if (blockIdx.x >= p.page_items) {                // queries: `group` tokens; a thread has the same item of a head in several of them
        const int per = p.n_q * items, side = max(1, kThreads / per);      // items of a token; tokens side by side
        const int t0 = (int)(blockIdx.x - p.page_items) * p.group, t1 = min(t0 + p.group, p.b.n_tokens);
        int s = t0;
        if (p.b.q_start) {                           // the first sequence that ends behind the first token
            s = -1;
            for (int base = 0; base < p.b.n_seq && s < 0; base += 64) {
                int f = 0, m = -1, l;
                if (base + (tid & 63) < p.b.n_seq) kv_seq(p.b, base + (tid & 63), f, m, l);
                const uint64_t behind = __ballot(f + m > t0);
                if (behind) s = base + __builtin_ctzll(behind);
            }
            if (s < 0) return;
        }
        for (int i = tid; i < per * side; i += kThreads) {
            const int x = i / per, y = i - x * per, head = y / items, item = y - head * items;
            int q = s, first, n, len;
            kv_seq(p.b, q, first, n, len);
            if (p.rope && !p.inter && side == 1 && p.group == kTokens && t0 >= first && t0 + kTokens <= first + n && item < p.rot / (2 * E)) {
                // all of one sequence: every load before the first store
                const char* src = p.q + (int64_t)t0 * p.q_ts + head * p.q_hs + item * 16;
                const int far = p.rot / 2 * (int)sizeof(T);
                vec lo2[kTokens], hi2[kTokens];
#pragma unroll
                for (int t = 0; t < kTokens; ++t) {
                    lo2[t] = *(const vec*)(src + t * p.q_ts);
                    hi2[t] = *(const vec*)(src + t * p.q_ts + far);
                }
                char* out = p.q_out + ((int64_t)t0 * p.n_q + head) * (D * (int)sizeof(T)) + item * 16;
#pragma unroll
                for (int t = 0; t < kTokens; ++t) {
                    int64_t r = p.positions ? p.positions[t0 + t] : len - n + (t0 + t - first);
                    r = max((int64_t)0, min(r, p.n_pos - 1));
                    const float* c = p.rope + r * p.rot + item * E;
                    rotate_halves<T>(lo2[t], hi2[t], c, c + p.rot / 2);
                    *(vec*)(out + (int64_t)t * p.n_q * (D * (int)sizeof(T))) = lo2[t];
                    *(vec*)(out + (int64_t)t * p.n_q * (D * (int)sizeof(T)) + far) = hi2[t];
                }
                continue;
            }
            for (int token = t0 + x; token < t1; token += side) {
                if (p.b.q_start)
                    while (q + 1 < p.b.n_seq && p.b.q_start[q + 1] <= token) kv_seq(p.b, ++q, first, n, len);
                else if (q != token)
                    kv_seq(p.b, q = token, first, n, len);
                if (token < first || token >= first + n) continue;
                char* out = p.q_out + ((int64_t)token * p.n_q + head) * (D * (int)sizeof(T));
                row_item<T, D>(p, p.q + token * p.q_ts + head * p.q_hs, item, token, len - n + (token - first),
                               [&](int g, vec z) { *(vec*)(out + g * 16) = z; });
            }
        }
        return;
    }

    // one page of one head
    __shared__ __align__(16) char lk[SLAB * ROW], lv[SLAB * ROW];
    const int h = blockIdx.x % p.n_kv;
    const int logp = p.b.log_page, P = 1 << logp;
    int s, j, first, n, len;
    auto count = [&](int n, int len) { return n > 0 && len > 0 ? ((len - 1) >> logp) - (max(0, len - n) >> logp) + 1 : 0; };
    if (!kv_find(p.b, blockIdx.x / p.n_kv, count, s, j, first, n, len)) return;
    const int p0 = len - n;                          // position of the first new token (negative: tokens before the sequence)
    const int blk = (max(0, p0) >> logp) + j;
    const int page = kv_page(p.b, s, blk);
    if (page < 0) return;
    const int base = blk << logp, lo = max(p0, base) - base, hi = min(len - base, P);      // new slots lo .. hi - 1
    const int64_t at = ((int64_t)page * p.n_kv + h) * ((int64_t)P * D * (int)sizeof(T));
    char* kp = p.kc + at;
    char* vp = p.vc + at;
    // this thread's channels and remainder of the slots in the signature's sums
    constexpr int PAIR = E == 8 ? 2 : 1, SUMS = D / PAIR * 8 / kThreads;
    float sum[SUMS][PAIR] = {};
    for (int s0 = p.sig ? 0 : lo & ~(SLAB - 1); s0 < hi; s0 += SLAB) {
        const int a = max(lo - s0, 0), b = min(hi - s0, SLAB);       // new ones of the slab: a .. b - 1; before them older ones
        if (p.sig)
            for (int i = tid; i < min(a, b) * NG; i += kThreads) {
                const int g = i / min(a, b), slot = i % min(a, b);
                *(vec*)(lk + slot * ROW + g * 16) = *(const vec*)(kp + ((int64_t)g * P + s0 + slot) * 16);
            }
        const char* vrow = p.v + h * p.v_hs;
        const char* krow = p.k + h * p.k_hs;
        const int t0 = first + (base + s0 - p0);                     // the slab's first slot, were it new
        if (b - a == SLAB && !p.inter) {
            // a whole slab: a thread has one group of channels in every IT-th slot, and takes its partners' channels from the same rows
            constexpr int STEP = kThreads / NG, IT = SLAB / STEP;
            const int g = tid % NG, slot = tid / NG, halves = p.rope ? p.rot / (2 * E) : 0;
            const bool up = g < halves, turned = g < 2 * halves;
            const int mate = up ? g + halves : turned ? g - halves : g;
            vec v[IT];
#pragma unroll
            for (int x = 0; x < IT; ++x) v[x] = *(const vec*)(vrow + (int64_t)(t0 + slot + x * STEP) * p.v_ts + g * 16);
#pragma unroll 2
            for (int x = 0; x < IT; ++x) {
                const int token = t0 + slot + x * STEP;
                const char* row = krow + (int64_t)token * p.k_ts;
                vec own = *(const vec*)(row + g * 16);
                if (turned) {
                    const vec other = *(const vec*)(row + mate * 16);
                    int64_t r = p.positions ? p.positions[token] : base + s0 + slot + x * STEP;
                    r = max((int64_t)0, min(r, p.n_pos - 1));
                    const float* c = p.rope + r * p.rot + min(g, mate) * E;
                    vec lo2 = up ? own : other, hi2 = up ? other : own;
                    rotate_halves<T>(lo2, hi2, c, c + p.rot / 2);
                    own = up ? lo2 : hi2;
                }
                *(vec*)(lk + (slot + x * STEP) * ROW + g * 16) = own;
            }
#pragma unroll
            for (int x = 0; x < IT; ++x) *(vec*)(lv + (slot + x * STEP) * ROW + g * 16) = v[x];
        } else {
            for (int i = tid; i < (b - a) * NG; i += kThreads) {
                const int slot = a + i / NG, g = i % NG;
                *(vec*)(lv + slot * ROW + g * 16) = *(const vec*)(vrow + (int64_t)(t0 + slot) * p.v_ts + g * 16);
            }
            for (int i = tid; i < (b - a) * items; i += kThreads) {
                const int slot = a + i / items;
                row_item<T, D>(p, krow + (int64_t)(t0 + slot) * p.k_ts, i % items, t0 + slot, base + s0 + slot,
                               [&](int g, vec x) { *(vec*)(lk + slot * ROW + g * 16) = x; });
            }
        }
        __syncthreads();
        if (b - a == SLAB) {
            for (int i = tid; i < SLAB * NG; i += kThreads) {
                const int g = i / SLAB, slot = i % SLAB;
                *(vec*)(kp + ((int64_t)g * P + s0 + slot) * 16) = *(const vec*)(lk + slot * ROW + g * 16);
            }
        } else {
            for (int i = tid; i < (b - a) * NG; i += kThreads) {
                const int g = i / (b - a), slot = a + i % (b - a);
                *(vec*)(kp + ((int64_t)g * P + s0 + slot) * 16) = *(const vec*)(lk + slot * ROW + g * 16);
            }
        }
        for (int i = tid; b > a && i < ((b + E - 1) / E - a / E) * D; i += kThreads) {      // E slots of one channel
            const int c = i % D, g = a / E + i / D;
            vec x;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = *(const T*)(lv + (g * E + e) * ROW + c * (int)sizeof(T));      // of other slots: not stored
            vec* dst = (vec*)(vp + ((int64_t)(s0 / E + g) * D + c) * 16);
            if (g * E >= a && g * E + E <= b) {
                *dst = x;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (g * E + e >= a && g * E + e < b) ((T*)dst)[e] = x[e];
            }
        }
        if (p.sig) {
#pragma unroll
            for (int y = 0; y < SUMS; ++y) {
                const int i = tid + y * kThreads, r = i / (D / PAIR), c = i % (D / PAIR) * PAIR;
                for (int slot = r; slot < b; slot += 8) {
#pragma unroll
                    for (int e = 0; e < PAIR; ++e) sum[y][e] += (float)*(const T*)(lk + slot * ROW + (c + e) * (int)sizeof(T));
                }
            }
        }
        __syncthreads();
    }
    if (!p.sig) return;
    __shared__ unsigned biggest[kThreads / 64];
    float* part = (float*)lk;                        // [8][D]
    static_assert(sizeof(lk) >= 8 * D * sizeof(float), "sums fit the slab");
#pragma unroll
    for (int y = 0; y < SUMS; ++y)
#pragma unroll
        for (int e = 0; e < PAIR; ++e) part[(tid + y * kThreads) * PAIR + e] = sum[y][e];
    __syncthreads();
    float m = 0.0f;
    if (tid < D)
        m = (((part[tid] + part[D + tid]) + (part[2 * D + tid] + part[3 * D + tid])) +
             ((part[4 * D + tid] + part[5 * D + tid]) + (part[6 * D + tid] + part[7 * D + tid]))) / (float)hi;
    const unsigned big = s3_wave_max_u32(__float_as_uint(m) & 0x7fffffffu);
    if ((tid & 63) == 0) biggest[tid >> 6] = big;
    __syncthreads();
    if (tid < D) {
        unsigned most = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) most = max(most, biggest[w]);
        bool ok;
        const int e = kv_grid_exp(most, ok);
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
    const int64_t qb = a.q ? (a.b.n_tokens + a.group - 1) / a.group : 0;
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
    if (b->n_seq && (!b->kv_len || (!b->block_table && b->max_pages))) return s3_fail(S3_EINVAL, "%s: null kv_len or block_table", fn);
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
                 interleaved != 0, c->n_kv_heads, n_q, (unsigned)(pages * c->n_kv_heads), b->n_tokens >= 512 ? kTokens : 1};
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
