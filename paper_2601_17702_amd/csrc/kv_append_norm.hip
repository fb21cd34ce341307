// Appending with head norms, and appending to an 8-bit cache (s3_kv_append_norm, s3_kv8_append).
//
//   y = w x / sqrt(sum x^2 / d + eps)      the mean square in 64 bits, its root's inverse r rounded to fp32 once, (x r) and (x r) w to fp32
//   rotation as in kv_append.hip, in fp32; then one rounding to the cache's type, or with 8 bits
//   code c = the smallest that leaves max|x| 2^(127 - c) <= 448, element = e4m3(x 2^(127 - c)), to nearest even
// A power of two makes both scalings exact.  e4m3 values have 4 bits in 15 octaves and 3, 2 and 1 in the three below: elements down to 1/14336 of the row's largest keep all 4, where
// max/448 as a scale would take up to an octave more.
//
// What bounds it: memory.  A row of d channels lies in d / 16 lanes, 16 channels each: where pairs are (i, i + rot / 2) eight of one half and
// their eight partners, so a rotation needs no other lane's channels, and a norm's sum is exchanged between neighbours of a row of 16 lanes only.  Two rows' loads are under way
// in a thread before the first is worked on.  Eight chunks of 2048 tokens into 8 bits, 32 query heads over 8 of 128 (379 MB): 83 to 85 us, 4.5 TB/s; 116 with 8 channels a
// lane and no loads ahead, 134 with 16 and none, 86 with four rows'.  64 single tokens: 7.1 us, a chain of loads.
#include "kv_cache.h"

namespace {

constexpr int kThreads = 256;
constexpr int kDeep = 2;               // rows of a thread whose loads are under way at a time
constexpr int kSlots = 64;             // slots of a page that pass through LDS at a time

struct NormArgs {
    KvBatch b;
    char* kc;
    char* vc;
    uint8_t* scale;
    __bf16* sig;
    const char *k, *v, *q;
    char* q_out;
    int64_t k_ts, k_hs, v_ts, v_hs, q_ts, q_hs;      // bytes
    const float* rope;
    const int32_t* positions;
    int64_t n_pos;
    int rot, inter, n_kv, n_q;
    const float *q_norm, *k_norm;                    // or null
    int64_t q_nhs, k_nhs;                            // from head to head of them
    double eps;
    unsigned page_items;                             // workgroups of pages; the rest have queries
    int group;                                       // tokens of such a one
};

constexpr int kChannels = 16;          // of a row in one lane

// This lane's channels of a row: c0 .. c0 + 7 and c1 .. c1 + 7.  Two halves of the row's, so that neighbouring lanes have neighbouring pieces, but where
// the rotation's halves are shorter than those.
template <int D>
struct Place {
    int lane, c0, c1;
    bool turn0, turn1;                               // they are in the rotation
    __device__ __forceinline__ Place(const NormArgs& p) {
        lane = threadIdx.x & (D / kChannels - 1);
        const bool apart = p.rope && !p.inter, in = apart && lane * 16 < p.rot;
        c0 = apart && !in ? lane * 16 : lane * 8;
        c1 = in ? p.rot / 2 + lane * 8 : apart ? lane * 16 + 8 : D / 2 + lane * 8;
        turn0 = in || (p.rope && p.inter && c0 < p.rot);
        turn1 = in || (p.rope && p.inter && c1 < p.rot);
    }
};

// Those of a row as they are loaded, and as numbers.
template <typename T>
struct Raw {
    typedef typename KvElem<T>::vec vec;
    static constexpr int E = KvElem<T>::E, N = 8 / E;
    vec a[2 * N];
    __device__ __forceinline__ void load(const char* row, int c0, int c1) {
#pragma unroll
        for (int y = 0; y < 2 * N; ++y) a[y] = *(const vec*)(row + ((y < N ? c0 : c1) + y % N * E) * (int)sizeof(T));
    }
    __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (float)a[i / E][i % E];
    }
};

// x of the lane that a step of a reduction over 2, 4, 8 or 16 neighbours adds: the other of a pair, of a four's halves, the mirrored one of eight and of sixteen.
template <int STEP>
__device__ __forceinline__ unsigned neighbour(unsigned x) {
    constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true);
}
// Sum, and largest, over the LANES lanes of a row, in every one of them.
template <int LANES, int STEP = 1>
__device__ __forceinline__ double row_sum(double x) {
    if constexpr (STEP < LANES) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const uint64_t o = (uint64_t)neighbour<STEP>((unsigned)(u >> 32)) << 32 | neighbour<STEP>((unsigned)u);
        return row_sum<LANES, STEP * 2>(x + __builtin_bit_cast(double, o));
    } else {
        return x;
    }
}
template <int LANES, int STEP = 1>
__device__ __forceinline__ unsigned row_max(unsigned x) {
    if constexpr (STEP < LANES) return row_max<LANES, STEP * 2>(max(x, neighbour<STEP>(x)));
    else return x;
}

// 1 / sqrt(t) to the last bit or so of 64: the unit's estimate is good to 2^-24, each step squares its error.
__device__ __forceinline__ double inverse_root(double t) {
    double r = __builtin_amdgcn_rsq(t);
    if (t < (double)INFINITY)                        // of an infinite sum it is zero, of NaN NaN
#pragma unroll
        for (int i = 0; i < 2; ++i) r = fma(0.5 * r, fma(-t * r, r, 1.0), r);
    return r;
}

// Norm (w: the head's weights, or null) and rotation (turn: the position's cosines and sines) of this lane's channels.
template <int D>
__device__ __forceinline__ void norm_turn(const NormArgs& p, const Place<D>& at, const float* w, const float* turn, float (&x)[16]) {
#pragma clang fp contract(off)
    kv_f32x4 c[2], s[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
        if (y ? at.turn1 : at.turn0) {
            const float* from = turn + (p.inter ? (y ? at.c1 : at.c0) / 2 : at.lane * 8 + y * 4);
            c[y] = *(const kv_f32x4*)from;
            s[y] = *(const kv_f32x4*)(from + p.rot / 2);
        }
    if (w) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fma((double)x[i], (double)x[i], sum);
        const float r = (float)inverse_root(row_sum<D / kChannels>(sum) * (1.0 / D) + p.eps);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const kv_f32x4 f = *(const kv_f32x4*)(w + (y < 2 ? at.c0 : at.c1) + y % 2 * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[y * 4 + i] = x[y * 4 + i] * r * f[i];
        }
    }
    if (p.inter) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
            if (y ? at.turn1 : at.turn0)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = x[y * 8 + 2 * i], v = x[y * 8 + 2 * i + 1];
                    x[y * 8 + 2 * i] = u * c[y][i] - v * s[y][i];
                    x[y * 8 + 2 * i + 1] = v * c[y][i] + u * s[y][i];
                }
    } else if (at.turn0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = x[i], v = x[8 + i];
            x[i] = u * c[i / 4][i % 4] - v * s[i / 4][i % 4];
            x[8 + i] = v * c[i / 4][i % 4] + u * s[i / 4][i % 4];
        }
    }
}

// This lane's channels in 8 bits, and the row's code.  What is not finite becomes NaN, and counts for nothing in the scale.
template <int D>
__device__ __forceinline__ kv_u32x4 to8(const float (&x)[16], unsigned& code) {
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const unsigned a = __float_as_uint(x[i]) & 0x7fffffffu;
        most = max(most, a < 0x7f800000u ? a : 0u);
    }
    code = kv_scale_code(row_max<D / kChannels>(most));
    const float by = __uint_as_float((254u - code) << 23);
    kv_u32x4 u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fabsf(x[4 * k + i]) < INFINITY ? x[4 * k + i] * by : __uint_as_float(0x7fc00000u);
        u[k] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
    }
    return u;
}

template <typename T>
__device__ __forceinline__ void store_row(char* row, int c0, int c1, const float (&x)[16]) {
    typedef typename KvElem<T>::vec vec;
    constexpr int E = KvElem<T>::E;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int y = 0; y < 8 / E; ++y) {
            vec a;
#pragma unroll
            for (int i = 0; i < E; ++i) a[i] = (T)x[h * 8 + y * E + i];
            *(vec*)(row + ((h ? c1 : c0) + y * E) * (int)sizeof(T)) = a;
        }
}

__device__ __forceinline__ const float* turn_of(const NormArgs& p, int token, int pos) {
    int64_t r = p.positions ? p.positions[token] : pos;
    r = max((int64_t)0, min(r, p.n_pos - 1));
    return p.rope + r * p.rot;
}

template <typename S, int D>
__global__ __launch_bounds__(kThreads) void kv_append_norm_kernel(NormArgs p) {
    typedef typename KvStore<S>::row T;
    constexpr int E = KvStore<S>::E, ES = KvStore<S>::BYTES, NG = D / E, L = D / kChannels, SIDE = kThreads / L, ROW = D * ES + 16;
    constexpr bool EIGHT = KvStore<S>::EIGHT;
    constexpr int SLAB = D * ES >= 1024 ? 16 : D * ES >= 512 ? 32 : kSlots;
    const int tid = threadIdx.x;
    const Place<D> at(p);
    __shared__ __align__(16) char lk[SLAB * ROW], lv[SLAB * ROW];
    __shared__ int place[kThreads];

    if (blockIdx.x >= p.page_items) {                // queries
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
        if (tid < t1 - t0) {                         // positions of the tokens; of none of a sequence: 2^30
            const int token = t0 + tid;
            int q = p.b.q_start ? s : token, first, n, len;
            kv_seq(p.b, q, first, n, len);
            if (p.b.q_start)
                while (q + 1 < p.b.n_seq && p.b.q_start[q + 1] <= token) kv_seq(p.b, ++q, first, n, len);
            place[tid] = token >= first && token < first + n ? len - n + (token - first) : 1 << 30;
        }
        __syncthreads();
        const int rows = (t1 - t0) * p.n_q;
        for (int r0 = tid / L; r0 < rows; r0 += SIDE * kDeep) {      // kDeep rows' loads before the first store
            Raw<T> raw[kDeep];
#pragma unroll
            for (int y = 0; y < kDeep; ++y) {
                const int r = min(r0 + y * SIDE, rows - 1), t = r / p.n_q;
                raw[y].load(p.q + (int64_t)(t0 + t) * p.q_ts + (r - t * p.n_q) * p.q_hs, at.c0, at.c1);
            }
#pragma unroll
            for (int y = 0; y < kDeep; ++y) {
                const int r = r0 + y * SIDE, t = r / p.n_q, head = r - t * p.n_q, token = t0 + t;
                if (r >= rows) break;                // the same for all lanes of a row
                const int pos = place[t];
                if (pos == 1 << 30) continue;
                float x[16];
                raw[y].get(x);
                norm_turn<D>(p, at, p.q_norm ? p.q_norm + head * p.q_nhs : nullptr, p.rope ? turn_of(p, token, pos) : nullptr, x);
                store_row<T>(p.q_out + ((int64_t)token * p.n_q + head) * (D * (int)sizeof(T)), at.c0, at.c1, x);
            }
        }
        return;
    }

    // one page of one head
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
    const int64_t unit = (int64_t)page * p.n_kv + h;
    char* kp = p.kc + unit * ((int64_t)P * D * ES);
    char* vp = p.vc + unit * ((int64_t)P * D * ES);
    uint8_t* codes = EIGHT ? p.scale + unit * (2 * P) : nullptr;
    uint8_t* lc = (uint8_t*)place;                   // [2][SLAB]: the slab's codes
    const float* w = p.k_norm ? p.k_norm + h * p.k_nhs : nullptr;
    // this thread's channels and remainder of the slots in the signature's sums
    constexpr int PER = D * 8 >= kThreads * 4 ? 4 : 2, SUMS = D / PER * 8 / kThreads;
    float sum[SUMS][PER] = {};
    for (int s0 = p.sig ? 0 : lo & ~(SLAB - 1); s0 < hi; s0 += SLAB) {
        const int a = max(lo - s0, 0), b = min(hi - s0, SLAB);       // new ones of the slab: a .. b - 1; before them older ones
        if (p.sig) {
            const int old = min(a, b);
            for (int i = tid; i < old * NG; i += kThreads) {
                const int g = i / old, slot = i - g * old;
                *(kv_u32x4*)(lk + slot * ROW + g * 16) = *(const kv_u32x4*)(kp + ((int64_t)g * P + s0 + slot) * 16);
            }
            if (EIGHT && tid < old) lc[tid] = codes[s0 + tid];
        }
        const int t0 = first + (base + s0 - p0);                     // the slab's first slot, were it new
        const int v0 = at.lane * 8, v1 = D / 2 + at.lane * 8;
        for (int i0 = a + tid / L; i0 < b; i0 += SIDE * kDeep) {
            Raw<T> kr[kDeep], vr[kDeep];
#pragma unroll
            for (int y = 0; y < kDeep; ++y) {
                const int64_t token = t0 + min(i0 + y * SIDE, b - 1);
                kr[y].load(p.k + h * p.k_hs + token * p.k_ts, at.c0, at.c1);
                vr[y].load(p.v + h * p.v_hs + token * p.v_ts, v0, v1);
            }
#pragma unroll
            for (int y = 0; y < kDeep; ++y) {
                const int i = i0 + y * SIDE;
                if (i >= b) break;
                float x[16];
                kr[y].get(x);
                norm_turn<D>(p, at, w, p.rope ? turn_of(p, t0 + i, base + s0 + i) : nullptr, x);
                if constexpr (EIGHT) {
                    unsigned kcode, vcode;
                    kv_u32x4 u = to8<D>(x, kcode);
                    *(uint2*)(lk + i * ROW + at.c0) = uint2{u[0], u[1]};
                    *(uint2*)(lk + i * ROW + at.c1) = uint2{u[2], u[3]};
                    vr[y].get(x);
                    u = to8<D>(x, vcode);
                    *(uint2*)(lv + i * ROW + v0) = uint2{u[0], u[1]};
                    *(uint2*)(lv + i * ROW + v1) = uint2{u[2], u[3]};
                    if (at.lane == 0) {
                        lc[i] = (uint8_t)kcode;
                        lc[SLAB + i] = (uint8_t)vcode;
                    }
                } else {
                    store_row<T>(lk + i * ROW, at.c0, at.c1, x);
                    vr[y].get(x);
                    store_row<T>(lv + i * ROW, v0, v1, x);
                }
            }
        }
        __syncthreads();
        if (b > a) {
            const int fresh = b - a;
            for (int i = tid; i < fresh * NG; i += kThreads) {
                const int g = i / fresh, slot = a + (i - g * fresh);
                *(kv_u32x4*)(kp + ((int64_t)g * P + s0 + slot) * 16) = *(const kv_u32x4*)(lk + slot * ROW + g * 16);
            }
            if (EIGHT && tid < 2 * SLAB) {
                const int slot = tid & (SLAB - 1), which = tid / SLAB;
                if (slot >= a && slot < b) codes[which * P + s0 + slot] = lc[which * SLAB + slot];
            }
            // whole groups of E slots: of one channel (8 bits: of four, whose 4 x 4 squares of bytes are turned); then the slots of groups that are partly new
            constexpr int CH = EIGHT ? 4 : 1;
            const int ga = (a + E - 1) / E, gb = b / E;
            for (int i = tid; i < (gb - ga) * (D / CH); i += kThreads) {
                const int c = i % (D / CH) * CH, g = ga + i / (D / CH);
                char* dst = vp + ((int64_t)(s0 / E + g) * D + c) * 16;
                if constexpr (EIGHT) {
                    kv_u32x4 x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        unsigned u[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) u[r] = *(const unsigned*)(lv + (g * E + e * 4 + r) * ROW + c);
                        const unsigned a0 = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), a1 = __builtin_amdgcn_perm(u[1], u[0], 0x07030602u);
                        const unsigned b0 = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u), b1 = __builtin_amdgcn_perm(u[3], u[2], 0x07030602u);
                        x[0][e] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                        x[1][e] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
                        x[2][e] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
                        x[3][e] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y) *(kv_u32x4*)(dst + y * 16) = x[y];
                } else {
                    typename KvElem<T>::vec x;
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = *(const T*)(lv + (g * E + e) * ROW + c * ES);
                    *(typename KvElem<T>::vec*)dst = x;
                }
            }
            const int before = ga <= gb ? ga * E - a : fresh, part = before + (ga <= gb ? b - gb * E : 0);
            for (int i = tid; i < part * D; i += kThreads) {
                const int k = i / D, c = i % D, slot = k < before ? a + k : gb * E + (k - before);
                *(S*)(vp + ((int64_t)(s0 + slot) / E * D + c) * 16 + slot % E * ES) = *(const S*)(lv + slot * ROW + c * ES);
            }
        }
        if (p.sig) {
#pragma unroll
            for (int y = 0; y < SUMS; ++y) {
                const int i = tid + y * kThreads, r = i / (D / PER), c = i % (D / PER) * PER;
                for (int slot = r; slot < b; slot += 8) {
                    const char* src = lk + slot * ROW + c * ES;
                    if constexpr (EIGHT) {
                        const unsigned u = PER == 4 ? *(const unsigned*)src : *(const uint16_t*)src;
                        const float f = kv_scale(lc[slot]);
                        const kv_f32x2 p0 = kv_of8<false>(u);
                        sum[y][0] += p0[0] * f;
                        sum[y][1] += p0[1] * f;
                        if constexpr (PER == 4) {
                            const kv_f32x2 p1 = kv_of8<true>(u);
                            sum[y][2] += p1[0] * f;
                            sum[y][3] += p1[1] * f;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < PER; ++e) sum[y][e] += (float)((const S*)src)[e];
                    }
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
        for (int e = 0; e < PER; ++e) part[(tid + y * kThreads) * PER + e] = sum[y][e];
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
        for (int x = 0; x < kThreads / 64; ++x) most = max(most, biggest[x]);
        bool ok;
        const int e = kv_grid_exp(most, ok);
        p.sig[unit * D + tid] = (__bf16)(ok ? kv_grid(m, e) : 0.0f);
    }
}

template <typename S, int D>
int launch(const NormArgs& p, hipStream_t st) {
    const int64_t grid = (int64_t)p.page_items + (p.q ? (p.b.n_tokens + p.group - 1) / p.group : 0);
    if (grid >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "s3_kv_append: too many tokens in one call");
    hipLaunchKernelGGL((kv_append_norm_kernel<S, D>), dim3((unsigned)grid), dim3(kThreads), 0, st, p);
    S3_HIP(hipGetLastError());
    return S3_OK;
}

int check_norm(const char* fn, const char* what, const float* w, int64_t stride, int d) {
    if (w && ((uintptr_t)w & 15 || stride % 4 || (stride && stride < d)))
        return s3_fail(S3_EINVAL, "%s: weights of %s are not 16-byte aligned, or %lld is no stride of them", fn, what, (long long)stride);
    return S3_OK;
}

// c: the cache, or an 8-bit cache (scale) as one of bf16.
int append(const char* fn, const s3_kv_cache* c, uint8_t* scale, const s3_kv_batch* b, const void* k, int64_t k_ts, int64_t k_hs, const void* v,
           int64_t v_ts, int64_t v_hs, const float* rope, int64_t n_pos, int rot_dim, int interleaved, const int32_t* positions, const void* q,
           int n_q, int64_t q_ts, int64_t q_hs, void* q_out, const s3_kv_norm* norm, hipStream_t st) {
    if (norm) {
        if (!(norm->eps > 0.0f) || isinf(norm->eps)) return s3_fail(S3_EINVAL, "%s: eps %g", fn, (double)norm->eps);
        if (int rc = check_norm(fn, "q", norm->q, norm->q_head_stride, c->d_head)) return rc;
        if (int rc = check_norm(fn, "k", norm->k, norm->k_head_stride, c->d_head)) return rc;
    }
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
    int64_t pages = b->n_seq + ((int64_t)b->n_tokens + (int64_t)b->n_seq * (P - 2)) / P;      // n tokens touch (n + P - 2) / P + 1 at most
    if (!b->q_start) pages = b->n_seq;
    if (pages * c->n_kv_heads >= (int64_t)1 << 24) return s3_fail(S3_EINVAL, "%s: too many tokens in one call", fn);
    const NormArgs p{s3_kv_batch_args(c, b), (char*)c->k, (char*)c->v, scale, (__bf16*)c->sig, (const char*)k, (const char*)v, (const char*)q,
                     (char*)q_out, k_ts * es, k_hs * es, v_ts * es, v_hs * es, q_ts * es, q_hs * es, rope, positions, n_pos, rot_dim,
                     interleaved != 0, c->n_kv_heads, n_q, norm ? norm->q : nullptr, norm ? norm->k : nullptr, norm ? norm->q_head_stride : 0,
                     norm ? norm->k_head_stride : 0, norm ? (double)norm->eps : 1.0, (unsigned)(pages * c->n_kv_heads), b->n_tokens >= 512 ? 4 : 1};
    const int d = c->d_head;
#define S3_NORM(S) (d == 64 ? launch<S, 64>(p, st) : d == 128 ? launch<S, 128>(p, st) : launch<S, 256>(p, st))
    if (scale) return S3_NORM(kv_e4m3);
    return c->dtype == S3_BF16 ? S3_NORM(__bf16) : S3_NORM(float);
#undef S3_NORM
}

}  // namespace

int s3_kv8_check(const char* fn, const s3_kv8_cache* c, const s3_kv_batch* b, s3_kv_cache& view) {
    if (!c) return s3_fail(S3_EINVAL, "%s: null cache", fn);
    view = s3_kv_cache{c->k, c->v, c->sig, S3_BF16, c->n_pages, c->page_size, c->n_kv_heads, c->d_head};
    if (int rc = s3_kv_check(fn, &view, b)) return rc;
    if (!c->scale || (uintptr_t)c->scale & 255) return s3_fail(S3_EINVAL, "%s: cache arrays must be given and 256-byte aligned", fn);
    return S3_OK;
}

extern "C" int s3_kv_append_norm(const s3_kv_cache* c, const s3_kv_batch* b, const void* k, int64_t k_ts, int64_t k_hs, const void* v,
                                 int64_t v_ts, int64_t v_hs, const float* rope, int64_t n_pos, int rot_dim, int interleaved,
                                 const int32_t* positions, const void* q, int n_q, int64_t q_ts, int64_t q_hs, void* q_out,
                                 const s3_kv_norm* norm, void* stream) {
    const char* fn = "s3_kv_append_norm";
    if (int rc = s3_kv_check(fn, c, b)) return rc;
    if (!norm) return s3_fail(S3_EINVAL, "%s: null norm (s3_kv_append has none)", fn);
    return append(fn, c, nullptr, b, k, k_ts, k_hs, v, v_ts, v_hs, rope, n_pos, rot_dim, interleaved, positions, q, n_q, q_ts, q_hs, q_out, norm,
                  (hipStream_t)stream);
}

extern "C" int s3_kv8_append(const s3_kv8_cache* c, const s3_kv_batch* b, const void* k, int64_t k_ts, int64_t k_hs, const void* v,
                             int64_t v_ts, int64_t v_hs, const float* rope, int64_t n_pos, int rot_dim, int interleaved,
                             const int32_t* positions, const void* q, int n_q, int64_t q_ts, int64_t q_hs, void* q_out,
                             const s3_kv_norm* norm, void* stream) {
    const char* fn = "s3_kv8_append";
    s3_kv_cache view;
    if (int rc = s3_kv8_check(fn, c, b, view)) return rc;
    return append(fn, &view, (uint8_t*)c->scale, b, k, k_ts, k_hs, v, v_ts, v_hs, rope, n_pos, rot_dim, interleaved, positions, q, n_q, q_ts, q_hs, q_out,
                  norm, (hipStream_t)stream);
}
