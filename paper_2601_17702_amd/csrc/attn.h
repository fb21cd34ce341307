// Pieces of the attention kernels: a wavefront's 32 rows against 32 tokens at a time.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T on 32x32 tiles, with a row of the problem in a COLUMN of the
// matrix instruction: a lane holds 16 scores of one row (the other 16 are in the lane 32 away), so maximum, sum and rescaling
// are per lane, and its 16 weights are, as they lie, the second product's operand.  For that the tokens are dealt to the first product's
// rows in an order of their own (kv_token): register i of half h is token 2 E (i / E) + E h + i % E of the 32.
#pragma once
#include <type_traits>

#include "kv_cache.h"

template <int D, typename T> constexpr int kQSteps = D * (int)sizeof(T) / 32;       // 16-byte pieces of a row per lane

// Token of the 32 in row m of the first product's tile.
template <typename S>
__device__ __forceinline__ int kv_token(int m) {
    if constexpr (KvStore<S>::E == 16) return (m & 4) << 2 | (m & 0x18) >> 1 | (m & 3);
    else if constexpr (KvStore<S>::E == 8) return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1);
    else return m;
}

__device__ __forceinline__ kv_f32x16 kv_mma(kv_bf16x8 a, kv_bf16x8 b, kv_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ kv_f32x16 kv_mma(kv_f32x4 a, kv_f32x4 b, kv_f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

struct AttnArgs {
    KvBatch b;
    const char* q;
    char* out;
    float* lse;
    const char* k;
    const char* v;
    const int32_t* sel;       // block lists, or null: all blocks
    int64_t q_ts, q_hs;       // bytes
    int n_kv, G, n_q, window;
    int qb, top, per_q, lists;// lists: tokens a tile, entries, row tiles a tile of queries (tiled kernel), how many lists there are
    float sl;                 // scale * log2(e), or what capped scores are to be multiplied by
    int few;                  // sequences of at most this many rows are the streaming kernel's
};
// What 8-bit caches and caps need beside.  The other builds are launched without it: every argument is read from memory when a workgroup begins, and with these 0.1 to 0.8 us
// of a tiled call's two launches were lost (16 tokens at 20000, 28 heads over 4: 28.1 -> 28.8; 333 at 333 in fp32 with 256 channels: 37.6 -> 38.3).
struct AttnMore : AttnArgs {
    const uint8_t* scale;     // an 8-bit cache's
    float cap, to_cap, cap_lse;      // with a cap (0: none): cap * log2(e), scale / cap, and how far up the capped scores come shifted (log2 units)
};
template <typename S, bool CAP> using kAttnArgs = std::conditional_t<KvStore<S>::EIGHT || CAP, AttnMore, AttnArgs>;
template <bool CAP> using kJoinArgs = std::conditional_t<CAP, AttnMore, AttnArgs>;

// Largest over the two lanes that share a row; their sum.  The swap hands every lane both halves' values.
__device__ __forceinline__ float kv_pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float kv_pair_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a wavefront knows of its 32 rows: row r0 + (lane & 31) of the sequence's n * G, head and token of it.
// An 8-bit cache's pieces hold 16 channels, which two instructions take: this lane's 8 of either lie side by side.
template <typename T, int D, bool SIDE_BY_SIDE = false>
struct AttnRows {
    typename KvElem<T>::vec q[kQSteps<D, T>];
    int64_t row;              // token * n_q + head, or -1
    int pos;                  // its position (-1: sees nothing)
    __device__ __forceinline__ void load(const AttnArgs& p, int head, int first, int n, int len, int r, int r_end) {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        row = -1;
        pos = -1;
        typename KvElem<T>::vec zero = {};
        if (r < r_end) {
            const int t = r / p.G, g = r - t * p.G;
            row = (int64_t)(first + t) * p.n_q + head * p.G + g;
            pos = max(len - n + t, -1);
            const char* src = p.q + (int64_t)(first + t) * p.q_ts + (int64_t)(head * p.G + g) * p.q_hs + half * (SIDE_BY_SIDE ? 32 : 16);
#pragma unroll
            for (int s = 0; s < kQSteps<D, T>; ++s) q[s] = *(const typename KvElem<T>::vec*)(src + (SIDE_BY_SIDE ? s / 2 * 64 + s % 2 * 16 : s * 32));
        } else {
#pragma unroll
            for (int s = 0; s < kQSteps<D, T>; ++s) q[s] = zero;
        }
    }
};

// Largest magnitude of a piece's elements as the bits of a float, and at least 0x7f800000 exactly where one is infinite or NaN.
__device__ __forceinline__ unsigned kv_magnitude(kv_bf16x8 v, unsigned x) {
    const kv_u32x4 u = __builtin_bit_cast(kv_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) x = max(max(x, u[i] & 0x7fffffffu), u[i] << 16 & 0x7fffffffu);
    return x;
}
__device__ __forceinline__ unsigned kv_magnitude(kv_f32x4 v, unsigned x) {
    const kv_u32x4 u = __builtin_bit_cast(kv_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) x = max(x, u[i] & 0x7fffffffu);
    return x;
}
__device__ __forceinline__ unsigned kv_magnitude(kv_u32x4 u, unsigned x) {       // e4m3: a NaN is the only such
#pragma unroll
    for (int i = 0; i < 4; ++i) x |= (((u[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) ? 0x7f800000u : 0u;
    return x;
}
// Zero in place of infinities and NaN.
__device__ __forceinline__ kv_u32x4 kv_finite(kv_u32x4 u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] &= ~(((((u[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u);
    return u;
}
__device__ __forceinline__ kv_bf16x8 kv_finite(kv_bf16x8 v) {
    kv_u32x4 u = __builtin_bit_cast(kv_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] &= (u[i] & 0x7f800000u) == 0x7f800000u ? 0xffffu : ~0u;
        u[i] &= (u[i] & 0x7f80u) == 0x7f80u ? 0xffff0000u : ~0u;
    }
    return __builtin_bit_cast(kv_bf16x8, u);
}
__device__ __forceinline__ kv_f32x4 kv_finite(kv_f32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fabsf(v[i]) < INFINITY ? v[i] : 0.0f;
    return v;
}
// The first n elements of a piece, zeros behind them (n may be negative or more than there are).
__device__ __forceinline__ kv_bf16x8 kv_first(kv_bf16x8 v, int n) {
    kv_u32x4 u = __builtin_bit_cast(kv_u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] &= n > 2 * i + 1 ? 0xffffffffu : n > 2 * i ? 0xffffu : 0u;
    return __builtin_bit_cast(kv_bf16x8, u);
}
__device__ __forceinline__ kv_f32x4 kv_first(kv_f32x4 v, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n > i ? v[i] : 0.0f;
    return v;
}

__device__ __forceinline__ kv_u32x4 kv_first(kv_u32x4 u, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] &= n >= 4 * i + 4 ? ~0u : n > 4 * i ? (1u << (n - 4 * i) * 8) - 1u : 0u;
    return u;
}

// The tokens a row sees, as low <= position <= low + span; position 2^30 is beyond all rows.
struct AttnSight {
    int low;
    unsigned span;
    __device__ __forceinline__ AttnSight(int pos, int hi, int window) {
        const int up = min(pos, hi - 1);
        low = window ? max(0, pos - window + 1) : 0;
        span = (unsigned)(up - low);
        if (up < low) {                  // none: no position is -1
            low = -1;
            span = 0;
        }
    }
    __device__ __forceinline__ bool sees(int pos) const { return (unsigned)(pos - low) <= span; }
};

// Running softmax of a row: m the scaled score (log2 units) that its weights are taken against, at most kSlack below the largest so
// far, -inf before there is one; l this lane's part of the weights' sum, o the products so far: o[dt][i] is channel 32 dt + 8 (i / 4) + 4 half + i % 4.
// Rescaling o takes D / 2 instructions per 32 tokens, more than the exponentials: it is done only where a row's largest score has
// grown by more than kSlack (weights of up to 2^kSlack are as exact as those below 1).
// SCALED: weights are multiplied by their tokens' scales, at most 2^120, before bf16 holds them: 2^127 at most so.
constexpr float kLowest = -3.402823466e38f;
// PARTS: l takes E weights' sum at a time, as many additions, but an eighth of them to the long sum: 131072 tokens leave lse 1.2e-6 of itself off with one
// at a time, 3e-7 so.
template <typename T, int D, bool SCALED = false, bool PARTS = false>
struct AttnState {
    typedef typename KvElem<T>::vec vec;
    static constexpr int E = KvElem<T>::E, NW = 16 / E;
    static constexpr float kSlack = SCALED ? 7.0f : 8.0f;
    float m, l;
    kv_f32x16 o[D / 32];
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    }
    // The largest of a lane's raw scores -> what the scaled scores of both lanes' row are taken against.
    __device__ __forceinline__ float advance(float x, float sl) {
        const float top = kv_pair_max(x) * sl;
        if (__ballot(top > m + kSlack)) {
            const float m2 = fmaxf(m, top);
            const float keep = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - m2);
            m = m2;
            l *= keep;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= keep;
        }
        return m == -INFINITY ? 0.0f : m;                       // nothing seen yet: every weight is exp2(-inf)
    }
    // Behind the last scores: a row that saw tokens, but scores of -inf only, has no weights and is NaN; m tells it from one that saw
    // nothing and is 0.  seen: the lane had a token that the row sees.
    __device__ __forceinline__ void settle(bool seen) {
        const unsigned any = seen ? 1u : 0u;
        const auto r = __builtin_amdgcn_permlane32_swap(any, any, false, false);
        if ((r[0] | r[1]) != 0 && m == -INFINITY) m = kLowest;
    }
    // Weights of E of the lane's 16 tokens: registers E y .. of raw scores, -inf where masked.  With bf16 they are rounded to bf16, the type in which the
    // matrix units take them beside bf16 values (fp32 products run at an eighth of the rate); their sum is of the unrounded ones.  Against 64 bits
    // outputs are then off by 2.0e-3 to 2.3e-3 of their norm, by 1.7e-3 with weights in fp32 (their own last rounding).
    __device__ __forceinline__ vec weights(const kv_f32x16& s, int y, float sl, float sub) {
        vec w;
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = __builtin_amdgcn_exp2f(s[y * E + e] * sl - sub);
            if (PARTS) part = e ? part + x : x;
            else l += x;
            w[e] = (T)x;
        }
        if (PARTS) l += part;
        asm volatile("" : "+v"(l));      // summed here, not behind the products: nothing else would run beside it there
        return w;
    }
    // The same of an 8-bit cache's 8 tokens, times what their values are to be scaled by (f: of four tokens each): a power of two, so that nothing
    // more is rounded, and one multiplication a weight in place of one for each of a token's values.
    __device__ __forceinline__ vec weights(const kv_f32x16& s, int y, float sl, float sub, kv_f32x4 f0, kv_f32x4 f1) {
        vec w;
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = __builtin_amdgcn_exp2f(s[y * E + e] * sl - sub);
            part = e ? part + x : x;
            w[e] = (T)(x * (e < 4 ? f0[e % 4] : f1[e % 4]));
        }
        l += part;
        asm volatile("" : "+v"(l));
        return w;
    }
    // A token whose values are not all finite, in a tile where some rows do not see it: zero took the place of its infinities and NaNs
    // in the product (0 * inf is NaN), and the rows that do see it get them here.  value(c): the token's channel c.
    template <typename V>
    __device__ __forceinline__ void add_nonfinite(bool sees, V value) {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = value(dt * 32 + i / 4 * 8 + half * 4 + i % 4);
                o[dt][i] += sees && !(fabsf(x) < INFINITY) ? x : 0.0f;
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // rare: few registers matter, not speed
            }
    }
};

// Capped scores of this lane's raw ones x: c tanh(z), z = x u, in log2 units.
//
// NEAR: c tanh(z) = 2 c r - c with r = 1 / (1 + exp(-2 z)); r takes the score's place, 2 c that of the scale, and softmax does not see the shift: a multiplication,
// an addition and two quarter-rate instructions a score more than without a cap.  lse takes it off the maximum, an exact difference from r = 1/4 on, before the sum's logarithm is
// added: behind that it is rounded to the cap's places, 2e-4 off for 5e-5 at a cap of 2048.  r is off by 2^-23 or so, the score by 2^-22 c: for
// rows of bf16, whose weights are rounded to 2^-8 of themselves, up to caps of 2048 (5e-4 there).
// Otherwise, for scores as exact as fp32 ones whatever the cap: below |z| = 0.35 by tanh's series (its next term, 1382 z^11 / 155925, is 2^-22 of z there), above as
// 1 - 2 / (1 + exp(2 z)).  Where all of a wavefront's are small, as a cap well above the scores leaves them, only the series runs.
// us with the second / with the first, chunks of 333, 826 and 2048 tokens that see 4096 each, 32 heads over 8, bf16: 484 / 342.
constexpr float kS3NearCap = 2048.0f;
template <typename V, int N>
__device__ __forceinline__ void kv_cap_near(V (&s)[N], const AttnMore& p) {
    const float k = -2.8853900817779268f * p.to_cap;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < (int)(sizeof(V) / 4); ++i) s[x][i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[x][i] * k));
}
__device__ __forceinline__ bool kv_near(const AttnMore& p) { return p.cap_lse != 0.0f; }
template <bool CAP, typename A>
__device__ __forceinline__ float kv_shift(const A& p) {
    if constexpr (CAP) return p.cap_lse;
    else return 0.0f;
}
template <typename V, int N>
__device__ __forceinline__ void kv_cap_far(V (&s)[N], const AttnMore& p) {
    const float u = p.to_cap, c = p.cap;
    float most = 0.0f;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < (int)(sizeof(V) / 4); ++i) most = fmaxf(most, fabsf(s[x][i]));
    const bool some = __ballot(!(most * u < 0.35f)) != 0;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
            const float z = s[x][i] * u, w = z * z;
            const float small = z * c * fmaf(w, fmaf(w, fmaf(w, fmaf(w, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
            if (some) {
                const float t = __builtin_amdgcn_exp2f(z * 2.8853900817779268f);
                const float large = fmaf(__builtin_amdgcn_rcpf(t + 1.0f), -2.0f * c, c);
                s[x][i] = fabsf(z) < 0.35f ? small : large;
            } else {
                s[x][i] = small;
            }
        }
}

template <bool BF16, typename V, int N>
__device__ __forceinline__ void kv_cap(V (&s)[N], const AttnMore& p) {
    if (BF16 && kv_near(p)) kv_cap_near(s, p);
    else kv_cap_far(s, p);
}

// 1 / l, or what makes a row that saw nothing 0 (infinity makes NaN of one that saw only scores of -inf); its lse.
__device__ __forceinline__ float kv_inverse(float m, float l) { return m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float kv_lse(float m, float l) { return l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f; }
// What brings sums against m (l the weights' sum) to sums against the larger m2; sums of nothing count as zero.
__device__ __forceinline__ float kv_factor(float m, float l, float m2) {
    return m == -INFINITY && l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m == m2 ? 0.0f : m - m2);
}

// Lists: the runs of 16 tokens that are there move together (their order stays), -1 entries and blocks past the end take no work.
// keep: does this thread's run stay; returns its place, and how many stay of all threads.  sums: one int per wavefront.
template <int WAVES>
__device__ __forceinline__ int kv_compact(bool keep, int* sums, int& total) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t b = __ballot(keep);
    if (lane == 0) sums[wave] = __popcll(b);
    __syncthreads();
    int at = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        at += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    __syncthreads();
    return at + __popcll(b & (((uint64_t)1 << lane) - 1));
}
