// Tokens of a paged cache back as rows (s3_kv_read, s3_kv8_read).
//
// What bounds it: memory.  A workgroup has 32 rows of one head.  Of the keys a lane takes a row's 16-byte piece and eight rows' lie in one line; the
// values' pieces hold E tokens of a channel, so the rows' groups of E tokens are turned over through LDS, each group once
// for all consecutive rows that lie in it (rows in ascending order, as evidence spans are, read every line once).  61000 tokens of 8 heads of 128 from 8 bits
// to bf16 (378 MB): 80 us, 4.7 TB/s; 85 with 64 rows a workgroup.
#include "kv_cache.h"

namespace {

constexpr int kThreads = 256, kRows = 32;

struct ReadArgs {
    KvBatch b;
    const char* kc;
    const char* vc;
    const uint8_t* scale;
    const int32_t* positions;
    char *k, *v;
    int n_kv;
};

template <typename S, int D>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(ReadArgs p) {
    typedef typename KvStore<S>::row T;
    constexpr int E = KvStore<S>::E, ES = KvStore<S>::BYTES, NG = D / E, ROW = D * ES + 16;
    constexpr bool EIGHT = KvStore<S>::EIGHT;
    constexpr int GROUPS = kRows / E + 1;               // of E tokens: what consecutive rows lie in
    __shared__ __align__(16) char turned[GROUPS * E * ROW];
    __shared__ int pages[kRows], slots[kRows], group_of[kRows], groups[kRows], n_groups;
    const int tid = threadIdx.x, h = blockIdx.x % p.n_kv, t0 = (int)(blockIdx.x / p.n_kv) * kRows;
    const int logp = p.b.log_page, P = 1 << logp;
    const int n_rows = min(kRows, p.b.n_tokens - t0);

    if (tid < 64) {                                     // where the rows lie: a page, -1 (zeros) or -2 (of no sequence)
        const int token = t0 + tid;
        int s = t0;
        if (p.b.q_start) {                              // the first sequence that ends behind the first row
            s = -1;
            for (int base = 0; base < p.b.n_seq && s < 0; base += 64) {
                int f = 0, m = -1, l;
                if (base + tid < p.b.n_seq) kv_seq(p.b, base + tid, f, m, l);
                const uint64_t behind = __ballot(f + m > t0);
                if (behind) s = base + __builtin_ctzll(behind);
            }
        }
        int page = -2, slot = 0;
        if (tid < n_rows && s >= 0) {
            int q = p.b.q_start ? s : token, first, n, len;
            kv_seq(p.b, q, first, n, len);
            if (p.b.q_start)
                while (q + 1 < p.b.n_seq && p.b.q_start[q + 1] <= token) kv_seq(p.b, ++q, first, n, len);
            if (token >= first && token < first + n) {
                const int pos = p.positions ? p.positions[token] : len - n + (token - first);
                page = pos >= 0 && pos < len ? kv_page(p.b, q, pos >> logp) : -1;
                slot = pos & (P - 1);
            }
        }
        const int group = page >= 0 ? slot / E : -1;
        const int before_page = __shfl_up(page, 1), before_group = __shfl_up(group, 1);
        const bool begins = page >= 0 && (tid == 0 || page != before_page || group != before_group);
        const uint64_t all = __ballot(begins);
        const int mine = __popcll(all & (~(uint64_t)0 >> (63 - tid))) - 1;
        if (tid < kRows) {
            pages[tid] = page;
            slots[tid] = slot;
            group_of[tid] = page >= 0 ? mine : -1;
        }
        if (begins) groups[mine] = tid;                 // a row of it
        if (tid == 0) n_groups = __popcll(all);
    }
    __syncthreads();
    const int64_t page_bytes = (int64_t)P * D * ES;

    // A thread's pieces of the groups: of one channel, or of 8 bits of four, whose 4 x 4 squares of bytes are turned.  They are on
    // their way while the keys are read.
    constexpr int CH = EIGHT ? 4 : 1, ITEMS = (GROUPS * (D / CH) + kThreads - 1) / kThreads;
    kv_u32x4 x[ITEMS][CH];
    auto load = [&](int g0, int ng) {
#pragma unroll
        for (int y = 0; y < ITEMS; ++y) {
            const int i = tid + y * kThreads;
            if (i >= ng * (D / CH)) break;
            const int g = i / (D / CH), c = i % (D / CH) * CH, r = groups[g0 + g];
            const char* src = p.vc + ((int64_t)pages[r] * p.n_kv + h) * page_bytes + ((int64_t)(slots[r] / E) * D + c) * 16;
#pragma unroll
            for (int z = 0; z < CH; ++z) x[y][z] = *(const kv_u32x4*)(src + z * 16);
        }
    };
    auto turn = [&](int ng) {
#pragma unroll
        for (int y = 0; y < ITEMS; ++y) {
            const int i = tid + y * kThreads;
            if (i >= ng * (D / CH)) break;
            const int g = i / (D / CH), c = i % (D / CH) * CH;
            if constexpr (EIGHT) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned a0 = __builtin_amdgcn_perm(x[y][1][e], x[y][0][e], 0x05010400u), a1 = __builtin_amdgcn_perm(x[y][1][e], x[y][0][e], 0x07030602u);
                    const unsigned b0 = __builtin_amdgcn_perm(x[y][3][e], x[y][2][e], 0x05010400u), b1 = __builtin_amdgcn_perm(x[y][3][e], x[y][2][e], 0x07030602u);
                    char* dst = turned + (g * E + e * 4) * ROW + c;
                    *(unsigned*)dst = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                    *(unsigned*)(dst + ROW) = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
                    *(unsigned*)(dst + 2 * ROW) = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
                    *(unsigned*)(dst + 3 * ROW) = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
                }
            } else {
                const typename KvElem<T>::vec v = __builtin_bit_cast(typename KvElem<T>::vec, x[y][0]);
#pragma unroll
                for (int e = 0; e < E; ++e) *(T*)(turned + (g * E + e) * ROW + c * ES) = v[e];
            }
        }
    };
    // Groups go through LDS some at a time, up to four times; rows in more than that come element by element.  us so / all through LDS, 4096 tokens of 131072, 8 heads of
    // 128, 8 bits: single ones 18.0 / 23.3, by fours 13.9 / 12.4, by sixteens 12.8 / 8.9; 64 single ones 7.0 / 13.4.
    const bool scattered = n_groups > 4 * GROUPS;
    if (p.v && !scattered) load(0, min(n_groups, GROUPS));
    if (p.k)
        for (int i = tid; i < n_rows * NG; i += kThreads) {
            const int r = i / NG, g = i % NG, page = pages[r];
            if (page == -2) continue;
            const int64_t unit = (int64_t)page * p.n_kv + h;
            kv_u32x4 x = {0u, 0u, 0u, 0u};
            if (page >= 0) x = *(const kv_u32x4*)(p.kc + unit * page_bytes + ((int64_t)g * P + slots[r]) * 16);
            char* dst = p.k + (((int64_t)(t0 + r) * p.n_kv + h) * D + g * E) * (int)sizeof(T);
            if constexpr (EIGHT) {
                const float f = page >= 0 ? kv_scale(p.scale[unit * (2 * P) + slots[r]]) : 0.0f;
                kv_bf16x8 y[2];                         // k_out is aligned to 16 bytes, no more
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const kv_f32x2 a = kv_of8<false>(x[w]), b = kv_of8<true>(x[w]);
                    y[w / 2][w % 2 * 4] = (__bf16)(a[0] * f);
                    y[w / 2][w % 2 * 4 + 1] = (__bf16)(a[1] * f);
                    y[w / 2][w % 2 * 4 + 2] = (__bf16)(b[0] * f);
                    y[w / 2][w % 2 * 4 + 3] = (__bf16)(b[1] * f);
                }
                *(kv_bf16x8*)dst = y[0];
                *(kv_bf16x8*)(dst + 16) = y[1];
            } else {
                *(kv_u32x4*)dst = x;
            }
        }
    if (!p.v) return;

    if (scattered) {                                    // neighbouring lanes have neighbouring channels
        constexpr int DEEP = 4;
        for (int i0 = tid; i0 < n_rows * D; i0 += kThreads * DEEP) {
            S got[DEEP];
            unsigned code[DEEP];
#pragma unroll
            for (int y = 0; y < DEEP; ++y) {
                const int i = min(i0 + y * kThreads, n_rows * D - 1), r = i / D, c = i % D, page = max(pages[r], 0), slot = slots[r];
                const int64_t unit = (int64_t)page * p.n_kv + h;
                got[y] = *(const S*)(p.vc + unit * page_bytes + ((int64_t)(slot / E) * D + c) * 16 + slot % E * ES);
                if constexpr (EIGHT) code[y] = p.scale[unit * (2 * P) + P + slot];
            }
#pragma unroll
            for (int y = 0; y < DEEP; ++y) {
                const int i = i0 + y * kThreads, r = i / D, c = i % D;
                if (i >= n_rows * D) break;
                const int page = pages[r];
                if (page == -2) continue;
                T v;
                if constexpr (EIGHT) v = (T)(kv_of8<false>(got[y].bits)[0] * kv_scale(code[y]));
                else v = got[y];
                *(T*)(p.v + (((int64_t)(t0 + r) * p.n_kv + h) * D + c) * (int)sizeof(T)) = page >= 0 ? v : (T)0.0f;
            }
        }
        return;
    }

    constexpr int OUT = 16 / (int)sizeof(T);            // channels of a store
    for (int g0 = 0; g0 == 0 || g0 < n_groups; g0 += GROUPS) {
        const int ng = min(GROUPS, n_groups - g0);
        if (g0) load(g0, ng);
        turn(ng);
        __syncthreads();
        for (int i = tid; i < n_rows * (D / OUT); i += kThreads) {
            const int r = i / (D / OUT), c = i % (D / OUT) * OUT, page = pages[r], g = group_of[r] - g0;
            if (page == -2 || (page >= 0 ? g < 0 || g >= ng : g0 != 0)) continue;
            kv_u32x4 y = {0u, 0u, 0u, 0u};
            if (page >= 0) {
                const char* src = turned + (g * E + slots[r] % E) * ROW + c * ES;
                if constexpr (EIGHT) {
                    const float f = kv_scale(p.scale[((int64_t)page * p.n_kv + h) * (2 * P) + P + slots[r]]);
                    const uint2 x = *(const uint2*)src;
                    const kv_f32x2 a = kv_of8<false>(x.x), b = kv_of8<true>(x.x), e = kv_of8<false>(x.y), d = kv_of8<true>(x.y);
                    y = __builtin_bit_cast(kv_u32x4, kv_bf16x8{(__bf16)(a[0] * f), (__bf16)(a[1] * f), (__bf16)(b[0] * f), (__bf16)(b[1] * f),
                                                               (__bf16)(e[0] * f), (__bf16)(e[1] * f), (__bf16)(d[0] * f), (__bf16)(d[1] * f)});
                } else {
                    y = *(const kv_u32x4*)src;
                }
            }
            *(kv_u32x4*)(p.v + (((int64_t)(t0 + r) * p.n_kv + h) * D + c) * (int)sizeof(T)) = y;
        }
        __syncthreads();
    }
}

int read(const char* fn, const s3_kv_cache* c, const uint8_t* scale, const s3_kv_batch* b, const int32_t* positions, void* k, void* v, hipStream_t st) {
    if (b->n_tokens == 0 || b->n_seq == 0 || (!k && !v)) return S3_OK;
    if (((uintptr_t)k | (uintptr_t)v) & 15) return s3_fail(S3_EINVAL, "%s: k_out or v_out is not 16-byte aligned", fn);
    const int64_t grid = ((int64_t)b->n_tokens + kRows - 1) / kRows * c->n_kv_heads;
    if (grid >= (int64_t)1 << 24 || (int64_t)b->n_tokens * c->n_kv_heads * c->d_head >= (int64_t)1 << 37) return s3_fail(S3_EINVAL, "%s: too many tokens in one call", fn);
    const ReadArgs p{s3_kv_batch_args(c, b), (const char*)c->k, (const char*)c->v, scale, positions, (char*)k, (char*)v, c->n_kv_heads};
#define S3_READ(S, D) hipLaunchKernelGGL((kv_read_kernel<S, D>), dim3((unsigned)grid), dim3(kThreads), 0, st, p)
    if (scale) {
        if (c->d_head == 64) S3_READ(kv_e4m3, 64);
        else if (c->d_head == 128) S3_READ(kv_e4m3, 128);
        else S3_READ(kv_e4m3, 256);
    } else if (c->dtype == S3_BF16) {
        if (c->d_head == 64) S3_READ(__bf16, 64);
        else if (c->d_head == 128) S3_READ(__bf16, 128);
        else S3_READ(__bf16, 256);
    } else {
        if (c->d_head == 64) S3_READ(float, 64);
        else if (c->d_head == 128) S3_READ(float, 128);
        else S3_READ(float, 256);
    }
#undef S3_READ
    S3_HIP(hipGetLastError());
    return S3_OK;
}

}  // namespace

extern "C" int s3_kv_read(const s3_kv_cache* c, const s3_kv_batch* b, const int32_t* positions, void* k, void* v, void* stream) {
    if (int rc = s3_kv_check("s3_kv_read", c, b)) return rc;
    return read("s3_kv_read", c, nullptr, b, positions, k, v, (hipStream_t)stream);
}

extern "C" int s3_kv8_read(const s3_kv8_cache* c, const s3_kv_batch* b, const int32_t* positions, void* k, void* v, void* stream) {
    s3_kv_cache view;
    if (int rc = s3_kv8_check("s3_kv8_read", c, b, view)) return rc;
    return read("s3_kv8_read", &view, (const uint8_t*)c->scale, b, positions, k, v, (hipStream_t)stream);
}
