// Pieces of the attention kernels: a wavefront's 32 rows against 32 tokens at a time.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T on 32x32 tiles, with a row of the problem in a COLUMN of the
// matrix instruction: a lane holds 16 scores of one row (the other 16 are in the lane 32 away), so maximum, sum and rescaling
// are per lane, and its 16 weights are, as they lie, the second product's operand.  For that the tokens are dealt to the first product's
// rows in an order of their own (kv_token): register i of half h is token 2 E (i / E) + E h + i % E of the 32.
#pragma once
#include "kv_cache.h"

template <int D, typename T> constexpr int kQSteps = D * (int)sizeof(T) / 32;       // 16-byte pieces of a row per lane

// Token of the 32 in row m of the first product's tile.
template <typename T>
__device__ __forceinline__ int kv_token(int m) {
    if constexpr (KvElem<T>::E == 8) return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1);
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
    int qb, top, per_q;       // lists: tokens a tile, entries, tiles of 32 rows a tile of queries
    float sl;                 // scale * log2(e)
};

// Largest over the two lanes that share a row; their sum.
__device__ __forceinline__ float kv_pair_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float kv_pair_sum(float x) { return x + __shfl_xor(x, 32); }

// What a wavefront knows of its 32 rows: row r0 + (lane & 31) of the sequence's n * G, head and token of it.
template <typename T, int D>
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
            const char* src = p.q + (int64_t)(first + t) * p.q_ts + (int64_t)(head * p.G + g) * p.q_hs + half * 16;
#pragma unroll
            for (int s = 0; s < kQSteps<D, T>; ++s) q[s] = *(const typename KvElem<T>::vec*)(src + s * 32);
        } else {
#pragma unroll
            for (int s = 0; s < kQSteps<D, T>; ++s) q[s] = zero;
        }
    }
};

// Running softmax of a row: m the largest scaled score (log2 units), l this lane's part of the sum, o the products so far:
// o[dt][i] is channel 32 dt + 8 (i / 4) + 4 half + i % 4.
template <typename T, int D>
struct AttnState {
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
    // s: raw scores of 32 tokens, -inf where masked.  Leaves the weights in w.
    __device__ __forceinline__ void softmax(const kv_f32x16& s, float sl, typename KvElem<T>::vec (&w)[16 / KvElem<T>::E]) {
        constexpr int E = KvElem<T>::E;
        float x = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) x = fmaxf(x, s[i]);
        const float m2 = fmaxf(m, kv_pair_max(x) * sl);
        const float sub = m2 == -INFINITY ? 0.0f : m2;          // nothing seen yet: every weight is exp2(-inf)
        const float keep = __builtin_amdgcn_exp2f(m - sub);
        m = m2;
        l *= keep;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= keep;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(s[i] * sl - sub);
            l += e;
            w[i / E][i % E] = (T)e;
        }
    }
};
