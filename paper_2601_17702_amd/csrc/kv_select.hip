// The blocks that each tile of queries will read (s3_block_select): scores of all candidates by matrix instructions, then the
// top_b largest of each list by a search for their threshold among the scores' ordered keys.
//
// Two forms.  sel_fused_kernel keeps a tile's keys in LDS: a workgroup takes some tiles of one sequence and head, all their rows in
// registers, its wavefronts walk over different signatures, and a wavefront each then picks for a tile.  Where that would leave the
// chip idle (few tiles), is not worth its longer beginning (few candidates) or does not fit LDS, sel_score_kernel spreads the scores of a tile over many
// workgroups and leaves the keys in scratch for sel_pick_kernel or, from 4097 candidates on, sel_pick_long_kernel.
//
// Measured, 32 query heads over 8, d_head 128: 32 of up to 512 blocks for 64 decoding steps 19 us (37 MB of signatures would be 8; lengths,
// table, signatures, scores and choice wait for each other); 64 of 2048 blocks for each 16 of 2048 queries 56 us, of which the scores are 44:
// every workgroup reads all signatures of a head through L2, 268 MB in all; 64 of 2048 for one query 18 us.
#include "attn.h"

namespace {

constexpr int kThreads = 256;
constexpr int kScoreBlocks = 128;      // blocks of one scoring workgroup: 32 a wavefront (512: 17.5 us a call where 128 take 14)

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

__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Where an interval of keys [lo, hi) is cut, hi - lo > 1: in the middle of the scores' values in even rounds (scores lie close
// together there, so few rounds lead to the threshold), in the middle of the keys in odd ones (no more than 64 rounds, whatever the scores).
__device__ __forceinline__ unsigned cut(unsigned lo, unsigned hi, int round) {
    if (round & 1) return lo + (hi - lo) / 2;
    const unsigned k = order_key(0.5f * key_value(lo) + 0.5f * key_value(hi));
    return min(max(k, lo + 1), hi - 1);
}

// A tile's place in its sequence: its rows, and the blocks it may choose from.
struct Tile {
    int s, first, n, len, t0, t1, nb;      // tokens t0 .. t1 - 1 of the sequence's n; candidates 0 .. nb - 1
    __device__ __forceinline__ bool find(const SelectArgs& p, int tile) {
        int j;
        if (!kv_find(p.b, tile, [&](int m, int) { return (m + p.qb - 1) / p.qb; }, s, j, first, n, len)) return false;
        t0 = j * p.qb;
        t1 = min(n, t0 + p.qb);
        const int last = len - n + t1 - 1;
        nb = last < 0 ? 0 : min(min((last >> p.b.log_page) + 1, p.b.max_pages), p.nb);
        return true;
    }
};

// 32 rows on their 8 bit grids as a matrix instruction's first operand: channel 16 s + 8 half + e of this lane's row at src (null: zeros).
template <typename T, int D>
__device__ __forceinline__ void grid_rows(const char* src, kv_bf16x8 (&a)[D / 16]) {
    const int half = (threadIdx.x & 63) >> 5;
    typename KvElem<T>::vec v[D / 16][8 / KvElem<T>::E];
    typename KvElem<T>::vec zero = {};
    unsigned big = 0;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int e = 0; e < 8 / KvElem<T>::E; ++e) {
            v[s][e] = src ? *(const typename KvElem<T>::vec*)(src + half * (8 * (int)sizeof(T)) + s * 16 * (int)sizeof(T) + e * 16) : zero;
            big = kv_magnitude(v[s][e], big);
        }
    big = max(big, (unsigned)__shfl_xor((int)big, 32));
    bool ok;
    const int ex = kv_grid_exp(big, ok);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) a[s][e] = (__bf16)(ok ? kv_grid((float)v[s][e / KvElem<T>::E][e % KvElem<T>::E], ex) : 0.0f);
}

__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(s3_wave_incl_scan(x), 63); }

// The top largest of keys[0 .. n - 1] (LDS, room for a multiple of 512; 0: no candidate; those below lead or from own on are always
// taken), by one wavefront.  An interval of keys that holds the threshold is halved, a pass over LDS each time, until at most 64 keys
// lie in it; those are ranked against each other, one a lane.  (Halving down to the threshold itself takes the key's bits in
// rounds wherever two scores tie; a radix search's counters share their leading bits, and with them the counter: both took
// three times as long.)  Ascending blocks, -1 behind them.  mid_keys: 64 words of this wavefront's own.
__device__ __forceinline__ void pick_by_wave(unsigned* keys, int n, int lead, int own, int top, unsigned* mid_keys, int32_t* out) {
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    auto read8 = [&](int base, unsigned (&k)[8]) {        // eight keys a lane at a time, whatever n is: their reads overlap
#pragma unroll
        for (int x = 0; x < 8; ++x) k[x] = keys[base + x * 64];
    };
    unsigned least = 0xffffffffu, most = 0;
    int cand = 0, always = 0;
    for (int base = lane; base < n + lane; base += 512) {
        unsigned k[8];
        read8(base, k);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int i = base + x * 64;
            const bool in = k[x] && i < n, must = in && (i < lead || i >= own);
            cand += in;
            always += must;
            least = min(least, in && !must ? k[x] : 0xffffffffu);
            most = max(most, in && !must ? k[x] : 0u);
            keys[i] = must ? 0xffffffffu : in ? k[x] : 0u;
        }
    }
    s3_wave_fence();
    cand = wave_sum(cand);
    always = wave_sum(always);
    unsigned thr = 1;                            // taken: keys above thr, and the first `equal` of those at it
    int equal = n;
    if (cand > top) {
        if (always >= top) {
            thr = 0xffffffffu;
            equal = top;
        } else {
            unsigned lo = ~s3_wave_max_u32(~least), hi = s3_wave_max_u32(most) + 1;      // more than `top` from lo on, at most that from hi on
            int from_lo = cand, from_hi = always;
            for (int round = 0; hi - lo > 1 && from_lo - from_hi > 64; ++round) {
                const unsigned mid = cut(lo, hi, round);
                int c = 0;
                for (int base = 0; base < n; base += 512) {
                    unsigned k[8];
                    read8(base + lane, k);
#pragma unroll
                    for (int x = 0; x < 8; ++x) c += __popcll(__ballot(k[x] >= mid));
                }
                if (c > top) {
                    lo = mid;
                    from_lo = c;
                } else {
                    hi = mid;
                    from_hi = c;
                }
            }
            const int need = top - from_hi;              // of those in the interval
            thr = lo;
            equal = need;
            if (from_lo - from_hi <= 64) {
                int m = 0;
                for (int base = 0; base < n; base += 512) {
                    unsigned k[8];
                    read8(base + lane, k);
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const bool in = k[x] >= lo && k[x] < hi;
                        const uint64_t b = __ballot(in);
                        if (in) mid_keys[m + __popcll(b & below)] = k[x];
                        m += __popcll(b);
                    }
                }
                s3_wave_fence();
                const unsigned mine = lane < m ? mid_keys[lane] : 0u;
                int rank = 0, greater = 0;               // keys before this one: greater, or equal and of a lower block
                for (int i = 0; i < m; ++i) {
                    const unsigned k = (unsigned)__builtin_amdgcn_readlane((int)mine, i);
                    greater += k > mine;
                    rank += k > mine || (k == mine && i < lane);
                }
                if (need > 0) {
                    const int l = __builtin_ctzll(__ballot(lane < m && rank == need - 1));
                    thr = (unsigned)__builtin_amdgcn_readlane((int)mine, l);
                    equal = need - __builtin_amdgcn_readlane(greater, l);
                } else {                                 // nothing of it
                    thr = hi - 1;
                    equal = 0;
                }
            }
        }
    }
    int at = 0, eq = 0;
    for (int base = lane; base < n + lane; base += 512) {
        unsigned k[8];
        read8(base, k);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const uint64_t bs = __ballot(k[x] == thr);
            const bool take = k[x] > thr || (k[x] == thr && eq + __popcll(bs & below) < equal);
            const uint64_t bt = __ballot(take);
            const int to = at + __popcll(bt & below);
            if (take && to < top) out[to] = base + x * 64;
            at += __popcll(bt);
            eq += __popcll(bs);
        }
    }
    for (int i = at + lane; i < top; i += 64) out[i] = -1;
}

// The choice for one tile by a workgroup of 16 wavefronts, where the candidates are many: key(i) for i < n (0: no candidate, all ones: always taken), kept in registers as
// far as they go.  Keys are counted by ballots and added up over the wavefronts, one barrier a round.
constexpr int kMine = 16;                        // keys of a thread
template <int WAVES> struct PickScratch {
    int sums[2][WAVES], cand[WAVES], always[WAVES], place[kMine * WAVES];
    unsigned least[WAVES], most[WAVES], mid_key[64], thr;
    int mid_at[64], lim;
};
template <int WAVES, typename K>
__device__ __forceinline__ void pick_by_block(K key, int n, int top, PickScratch<WAVES>& sh, int32_t* out) {
    constexpr int ALL = WAVES * 64, CHUNK = kMine * ALL;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    unsigned k[kMine];
    auto read = [&](int base) {
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int i = base + x * ALL + tid;
            k[x] = i < n ? key(i) : 0u;
        }
    };
    int round = 0;
    // how many keys satisfy f(key, i), over the workgroup
    auto count = [&](auto f) {
        int c = 0;
        for (int base = 0; base < n; base += CHUNK) {
            if (n > CHUNK) read(base);
#pragma unroll
            for (int x = 0; x < kMine; ++x)
                if (base + x * ALL < n) c += __popcll(__ballot(f(k[x], base + x * ALL + tid)));
        }
        int* sums = sh.sums[round++ & 1];
        if (lane == 0) sums[wave] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c += sums[w];
        return c;
    };
    read(0);
    unsigned least = 0xffffffffu, most = 0;
    int cand = 0, always = 0;
    for (int base = 0; base < n; base += CHUNK) {
        if (n > CHUNK) read(base);
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const bool in = k[x] != 0, must = k[x] == 0xffffffffu;
            cand += __popcll(__ballot(in));
            always += __popcll(__ballot(must));
            least = min(least, in && !must ? k[x] : 0xffffffffu);
            most = max(most, in && !must ? k[x] : 0u);
        }
    }
    least = ~s3_wave_max_u32(~least);
    most = s3_wave_max_u32(most);
    if (lane == 0) {
        sh.cand[wave] = cand;
        sh.always[wave] = always;
        sh.least[wave] = least;
        sh.most[wave] = most;
    }
    __syncthreads();
    cand = always = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        cand += sh.cand[w];
        always += sh.always[w];
        least = min(least, sh.least[w]);
        most = max(most, sh.most[w]);
    }
    // taken: keys above thr, and those at it up to block lim
    unsigned thr = 1;
    int lim = -1;
    if (cand > top) {
        unsigned lo = least, hi = most + 1;
        int from_lo = cand, from_hi = always;
        if (always >= top) {
            lo = 0xffffffffu;
            from_hi = 0;
        }
        while (hi - lo > 1 && from_lo - from_hi > 64 && always < top) {
            const unsigned mid = cut(lo, hi, round);
            const int c = count([&](unsigned x, int) { return x >= mid; });
            if (c > top) {
                lo = mid;
                from_lo = c;
            } else {
                hi = mid;
                from_hi = c;
            }
        }
        const int need = top - from_hi;              // of those in the interval
        if (need == 0) {
            thr = hi - 1;
        } else if (always < top && from_lo - from_hi <= 64) {
            const auto in = [&](unsigned x) { return x >= lo && x < hi; };
            int c = 0;
            for (int base = 0; base < n; base += CHUNK) {
                if (n > CHUNK) read(base);
#pragma unroll
                for (int x = 0; x < kMine; ++x) c += __popcll(__ballot(in(k[x])));
            }
            int* sums = sh.sums[round++ & 1];
            if (lane == 0) sums[wave] = c;
            __syncthreads();
            int m = 0, at = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                at += w < wave ? sums[w] : 0;
                m += sums[w];
            }
            for (int base = 0; base < n; base += CHUNK) {
                if (n > CHUNK) read(base);
#pragma unroll
                for (int x = 0; x < kMine; ++x) {
                    const uint64_t b = __ballot(in(k[x]));
                    if (in(k[x])) {
                        sh.mid_key[at + __popcll(b & below)] = k[x];
                        sh.mid_at[at + __popcll(b & below)] = base + x * ALL + tid;
                    }
                    at += __popcll(b);
                }
            }
            __syncthreads();
            if (wave == 0) {
                const unsigned mine = lane < m ? sh.mid_key[lane] : 0u;
                const int mine_at = lane < m ? sh.mid_at[lane] : 0;
                int rank = 0;                        // keys before this one: greater, or equal and of a lower block
                for (int i = 0; i < m; ++i) {
                    const unsigned x = (unsigned)__builtin_amdgcn_readlane((int)mine, i);
                    rank += x > mine || (x == mine && __builtin_amdgcn_readlane(mine_at, i) < mine_at);
                }
                if (lane < m && rank == need - 1) {
                    sh.thr = mine;
                    sh.lim = mine_at;
                }
            }
            __syncthreads();
            thr = sh.thr;
            lim = sh.lim;
        } else {                                     // many equal keys: the first `need` of them, found in the blocks' numbers
            thr = lo;
            int a = -1, b = n - 1;                   // up to a fewer than needed, up to b enough
            while (b - a > 1) {
                const int mid = a + (b - a) / 2;
                if (count([&](unsigned x, int i) { return x == thr && i <= mid; }) >= need) b = mid;
                else a = mid;
            }
            lim = b;
        }
    }
    int done = 0;
    for (int base = 0; base < n; base += CHUNK) {
        if (n > CHUNK) read(base);
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const bool take = k[x] > thr || (k[x] == thr && base + x * ALL + tid <= lim);
            const uint64_t b = __ballot(take);
            if (lane == 0) sh.place[x * WAVES + wave] = __popcll(b);
        }
        __syncthreads();
        // places before this wavefront's of every 64 * WAVES blocks
        int run = done, before[kMine];
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            int all = 0, mine = 0;
            if (base + x * ALL < n)
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const int c = sh.place[x * WAVES + w];
                    mine += w < wave ? c : 0;
                    all += c;
                }
            before[x] = run + mine;
            run += all;
        }
        done = run;
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int i = base + x * ALL + tid;
            const bool take = k[x] > thr || (k[x] == thr && i <= lim);
            const int to = before[x] + __popcll(__ballot(take) & below);
            if (take && to < top) out[to] = i;
        }
        __syncthreads();
    }
    for (int i = done + tid; i < top; i += ALL) out[i] = -1;
}

// tiles_wg tiles of one sequence and head.  Rows are dealt in fours, each four of one tile (a tile's last row repeated to fill them:
// the largest score does not change), and lie in NSETS sets of 32 in registers; more than that are taken in further walks.
// WHOLE: a tile is whole sets.
template <typename T, int D, int NSETS, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64, D == 256 || WAVES == 4 ? 2 : 4) void sel_fused_kernel(SelectArgs p, int tiles_wg, int tiles) {
    extern __shared__ unsigned lds_keys[];                       // [tiles_wg][stride] | [WAVES][64] | rows (NSETS > 1)
    const int stride = (p.nb + 511) & ~511;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % p.n_kv;
    const int group = blockIdx.x / p.n_kv;
    // the group's sequence, and the tiles before it and of all: every workgroup reads the sequences' lengths once
    int s = -1, j = 0, first = 0, n = 0, len = 0, tile0 = 0, tiles_all = 0, groups = 0;
    for (int base = 0; base < p.b.n_seq && (s < 0 || group == 0); base += 64) {
        int f = 0, m = 0, l = 0;
        if (base + lane < p.b.n_seq) kv_seq(p.b, base + lane, f, m, l);
        const int c = (m + p.qb - 1) / p.qb, g = (c + tiles_wg - 1) / tiles_wg;
        const int ci = s3_wave_incl_scan(c), gi = s3_wave_incl_scan(g);
        const int g_sum = __builtin_amdgcn_readlane(gi, 63);
        if (s < 0 && group < groups + g_sum) {
            const int x = __builtin_ctzll(__ballot(groups + gi > group));
            s = base + x;
            j = group - groups - (__builtin_amdgcn_readlane(gi, x) - __builtin_amdgcn_readlane(g, x));
            first = __builtin_amdgcn_readlane(f, x);
            n = __builtin_amdgcn_readlane(m, x);
            len = __builtin_amdgcn_readlane(l, x);
            tile0 = tiles_all + __builtin_amdgcn_readlane(ci, x) - __builtin_amdgcn_readlane(c, x) + j * tiles_wg;
        }
        tiles_all = kv_add_lists(tiles_all, __builtin_amdgcn_readlane(ci, 63));
        groups += g_sum;
    }
    if (group == 0)                                              // lists past the last tile
        for (int t = tiles_all + wave; t < tiles; t += WAVES)
            for (int i = lane; i < p.top; i += 64) p.sel[((int64_t)t * p.n_kv + head) * p.top + i] = -1;
    if (s < 0) return;
    const int t_first = j * tiles_wg, t_here = min(tiles_wg, (n + p.qb - 1) / p.qb - t_first);
    const int end = min(n, (t_first + t_here) * p.qb);                                    // tokens of the group end here
    const int last = len - n + end - 1;
    const int nb = last < 0 ? 0 : min(min((last >> p.b.log_page) + 1, p.b.max_pages), p.nb);
    for (int i = threadIdx.x; i < t_here * stride; i += WAVES * 64) lds_keys[i] = 0;
    __syncthreads();
    const int fours = WHOLE ? p.qb * p.G / 4 : (min(p.qb, n) * p.G + 3) / 4;               // of a tile
    for (int f0 = 0; f0 < t_here * fours; f0 += NSETS * 8) {
        // signatures are on their way before the rows are, and the next ones from the moment that a walk step's are used up
        constexpr int K = D / 16;
        auto lookup = [&](int blk) { return blk < nb ? kv_page(p.b, s, blk) : -1; };
        auto sig_of = [&](int page) { return p.sig + ((int64_t)max(page, 0) * p.n_kv + head) * D + half * 8; };
        kv_bf16x8 g[K];
        int page = lookup(wave * 32 + col), next = lookup((wave + WAVES) * 32 + col);
#pragma unroll
        for (int k = 0; k < K; ++k) g[k] = *(const kv_bf16x8*)(sig_of(page) + k * 16);
        kv_bf16x8 a[NSETS][D / 16];
        auto rows_of = [&](int x) {
            const int f = f0 + x * 8 + (col >> 2), t = f / fours;
            const int tok0 = (t_first + t) * p.qb, rows = (min(n, tok0 + p.qb) - tok0) * p.G;
            const char* src = nullptr;
            if (t < t_here) {
                const int r = tok0 * p.G + min((f - t * fours) * 4 + (col & 3), rows - 1), tk = r / p.G;
                src = p.q + (int64_t)(first + tk) * p.q_ts + (int64_t)(head * p.G + r - tk * p.G) * p.q_hs;
            }
            grid_rows<T, D>(src, a[x]);
        };
        int to[NSETS][WHOLE ? 1 : 4];                            // where the scores of this lane's fours go, or -1
        if constexpr (NSETS == 1) {
            rows_of(0);
        } else {
            // a set is put on its grid by one wavefront and handed to the others
            kv_bf16x8* rows = (kv_bf16x8*)(lds_keys + tiles_wg * stride + WAVES * 64);
            __syncthreads();
#pragma unroll
            for (int x = 0; x < NSETS; ++x)
                if (x % WAVES == wave) {
                    rows_of(x);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) rows[(x * (D / 16) + k) * 64 + lane] = a[x][k];
                }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < NSETS; ++x)
#pragma unroll
                for (int k = 0; k < D / 16; ++k) a[x][k] = rows[(x * (D / 16) + k) * 64 + lane];
        }
#pragma unroll
        for (int x = 0; x < NSETS; ++x) {
#pragma unroll
            for (int i = 0; i < (WHOLE ? 1 : 4); ++i) {
                const int tq = (f0 + x * 8 + (WHOLE ? 0 : 2 * i + half)) / fours;
                to[x][i] = tq < t_here ? tq * stride : -1;
            }
        }
        for (int b = wave * 32; b < nb; b += WAVES * 32) {
            const int blk = b + col;
            const __bf16* sg = sig_of(next);
            const int after = lookup(blk + 2 * WAVES * 32);
            kv_f32x16 c[NSETS];
#pragma unroll
            for (int x = 0; x < NSETS; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) c[x][i] = 0.0f;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int k = y * K / 2; k < (y + 1) * K / 2; ++k)
#pragma unroll
                    for (int x = 0; x < NSETS; ++x) c[x] = kv_mma(a[x][k], g[k], c[x]);
#pragma unroll
                for (int k = y * K / 2; k < (y + 1) * K / 2; ++k) g[k] = *(const kv_bf16x8*)(sg + k * 16);
            }
#pragma unroll
            for (int x = 0; x < NSETS; ++x) {
                float m[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) m[i] = fmaxf(fmaxf(c[x][4 * i], c[x][4 * i + 1]), fmaxf(c[x][4 * i + 2], c[x][4 * i + 3]));
                if constexpr (WHOLE) {
                    const float best = kv_pair_max(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
                    if (half == 0 && page >= 0 && to[x][0] >= 0) atomicMax(&lds_keys[to[x][0] + blk], order_key(best));
                } else if (page >= 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (to[x][i] >= 0) atomicMax(&lds_keys[to[x][i] + blk], order_key(m[i]));
                }
            }
            page = next;
            next = after;
        }
    }
    __syncthreads();
    for (int t = wave; t < min(t_here, tiles - tile0); t += WAVES) {        // lists past the last: q_start is not ascending
        const int tok0 = (t_first + t) * p.qb, pos0 = max(0, len - n + tok0), pos1 = len - n + min(n, tok0 + p.qb) - 1;
        const int own = p.tail > 0 ? (pos0 >> p.b.log_page) - p.tail + 1 : 1 << 30;         // blocks from here on are always taken
        const int nt = pos1 < 0 ? 0 : min((pos1 >> p.b.log_page) + 1, nb);
        pick_by_wave(lds_keys + t * stride, nt, p.lead, own, p.top, lds_keys + tiles_wg * stride + wave * 64,
                     p.sel + ((int64_t)(tile0 + t) * p.n_kv + head) * p.top);
    }
}

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
        kv_bf16x8 a[D / 16];
        const int r = r0 + col, tk = r / p.G;
        grid_rows<T, D>(r < t.t1 * p.G ? p.q + (int64_t)(t.first + tk) * p.q_ts + (int64_t)(head * p.G + r - tk * p.G) * p.q_hs : nullptr, a);
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
        int total;
        const int c = hist[255 - tid], before = s3_block_excl_scan<kThreads>(c, wsum, total);      // this bin, and those above it
        if ((before < left && left <= before + c) || (tid == 255 && total < left)) {
            found[0] = (unsigned)(255 - tid);
            found[1] = (unsigned)(left - before);
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

constexpr int kPickWaves = 16;
__global__ __launch_bounds__(kPickWaves * 64) void sel_pick_long_kernel(SelectArgs p) {
    __shared__ PickScratch<kPickWaves> scratch;
    const int head = blockIdx.x % p.n_kv, tile = blockIdx.x / p.n_kv;
    Tile t;
    const int nb = t.find(p, tile) ? t.nb : 0;
    const unsigned* keys = p.keys + ((int64_t)tile * p.n_kv + head) * p.nb;
    pick_by_block<kPickWaves>([&](int i) { return keys[i]; }, nb, p.top, scratch, p.sel + ((int64_t)tile * p.n_kv + head) * p.top);
}

int select_blocks(const s3_kv_cache* c, const s3_kv_batch* b) {
    return (int)max((int64_t)1, min((int64_t)b->max_pages, ((int64_t)b->max_kv + c->page_size - 1) / c->page_size));
}

// How a call is shared out.
struct SelectPlan {
    bool fused, whole;
    int tiles_wg, sets, nb;
    int64_t tiles, groups;
    SelectPlan(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block) {
        nb = select_blocks(c, b);
        tiles = s3_block_tiles(b, q_block);
        const int G = n_q / c->n_kv_heads, most = max(1, min(b->n_tokens, b->max_new));      // new tokens of a sequence
        const int64_t fours = ((int64_t)min(q_block, most) * G + 3) / 4;
        const int max_sets = c->d_head == 256 ? 2 : 4;
        // as many tiles as fill the registers: every signature is read once per workgroup; not more than a sequence has, nor than
        // 48 KB of keys (two workgroups a compute unit), and fewer where the chip would not be full
        int64_t t = min(max(max_sets * 8 / fours, (int64_t)1), (int64_t)(most + q_block - 1) / q_block);
        t = max((int64_t)1, min(t, (int64_t)12288 / ((nb + 511) & ~511)));
        while (t > 1 && tiles / t * c->n_kv_heads < 512) t /= 2;
        tiles_wg = (int)t;
        sets = t * fours <= 8 ? 1 : t * fours <= 16 || max_sets == 2 ? 2 : 4;
        groups = (tiles + (int64_t)b->n_seq * (t - 1)) / t;
        whole = q_block <= most && (int64_t)q_block * G % 32 == 0;
        // One kernel or scratch between two, us a call.  One tile of few rows a workgroup: the first wants a workgroup for every compute unit, and lists that are
        // worth its longer beginning (lists x candidates, one kernel / scratch: 64 x 2000 33 / 22, 64 x 8000 98 / 48, 128 x 500 18 / 13, 128 x 3000 44 / 37,
        // 256 x 300 14.7 / 13.8, 256 x 500 15.7 / 15.8, 256 x 2000 33 / 39, 512 x 200 17 / 15, 512 x 400 19 / 21, 512 x 2000 47 / 65, 1024 x 300 30 / 30,
        // 4096 x 100 92 / 48, 4096 x 500 123 / 138).  More rows, which scratch reads from every workgroup of a list: 64 rows, 8 x 200 13 / 15,
        // 8 x 500 16 / 16, 8 x 2000 36 / 22, 64 x 2000 36 / 32, 128 x 2000 37 / 47; 256 rows, 8 x 500 25 / 32, 8 x 2000 63 / 38, 64 x 2000 63 / 75.
        const int64_t lists = groups * c->n_kv_heads;
        fused = nb <= 30720 && (sets == 1 && tiles_wg == 1 ? lists >= 256 && nb >= 400 : lists >= 64 || nb <= 256);
    }
    size_t workspace(int n_kv) const { return fused ? 0 : s3_align((size_t)tiles * n_kv * nb * 4); }
};

template <typename T, int D, int NSETS, int WAVES, bool WHOLE>
int launch_fused(const SelectArgs& p, const SelectPlan& plan, hipStream_t st) {
    constexpr int extra = WAVES * 256 + (NSETS > 1 ? NSETS * 32 * D * 2 : 0);
    static S3LdsOnce once;
    if (int rc = s3_allow_lds(once, (const void*)sel_fused_kernel<T, D, NSETS, WAVES, WHOLE>, 30720 * 4 + extra)) return rc;
    hipLaunchKernelGGL((sel_fused_kernel<T, D, NSETS, WAVES, WHOLE>), dim3((unsigned)(plan.groups * p.n_kv)), dim3(WAVES * 64),
                       plan.tiles_wg * ((plan.nb + 511) & ~511) * 4 + extra, st, p, plan.tiles_wg, (int)plan.tiles);
    S3_HIP(hipGetLastError());
    return S3_OK;
}
template <typename T, int D>
int launch_select(const SelectArgs& p, const SelectPlan& plan, hipStream_t st) {
    if (plan.fused) {
        if constexpr (D < 256) {
            if (plan.sets == 4) return plan.whole ? launch_fused<T, D, 4, 4, true>(p, plan, st) : launch_fused<T, D, 4, 4, false>(p, plan, st);
        }
        if (plan.sets == 1) return launch_fused<T, D, 1, 8, false>(p, plan, st);
        return plan.whole ? launch_fused<T, D, 2, 4, true>(p, plan, st) : launch_fused<T, D, 2, 4, false>(p, plan, st);
    }
    const dim3 grid((unsigned)(plan.tiles * p.n_kv), (unsigned)((p.nb + kScoreBlocks - 1) / kScoreBlocks));
    hipLaunchKernelGGL((sel_score_kernel<T, D>), grid, dim3(kThreads), 0, st, p);
    S3_HIP(hipGetLastError());
    // us a call with the first / the second: 8 lists of 3000 candidates 22 / 24, 4096 25 / 25, 8000 45 / 25; 64 of 3000 29 / 32, 4096 35 / 35, 8000 66 / 48
    if (p.nb <= 4096) hipLaunchKernelGGL(sel_pick_kernel, dim3(grid.x), dim3(kThreads), 0, st, p);
    else hipLaunchKernelGGL(sel_pick_long_kernel, dim3(grid.x), dim3(kPickWaves * 64), 0, st, p);
    S3_HIP(hipGetLastError());
    return S3_OK;
}

}  // namespace

extern "C" size_t s3_block_select_workspace(const s3_kv_cache* c, const s3_kv_batch* b, int n_q, int q_block, int top_b) {
    (void)top_b;
    if (s3_kv_check("s3_block_select_workspace", c, b) || q_block < 1 || n_q < 1 || n_q % c->n_kv_heads) return 0;
    return SelectPlan(c, b, n_q, q_block).workspace(c->n_kv_heads);
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
    const SelectPlan plan(c, b, n_q, q_block);
    const size_t need = plan.workspace(c->n_kv_heads);
    if (need && (!ws || (uintptr_t)ws & 255)) return s3_fail(S3_EINVAL, "%s: workspace is null or not 256-byte aligned", fn);
    if (ws_bytes < need) return s3_fail(S3_ECAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    // a launch has fewer than 2^32 threads: 512 a list, or 256 for every 128 candidates of one
    const int64_t lists = tiles * c->n_kv_heads, parts = (plan.nb + kScoreBlocks - 1) / kScoreBlocks;
    if (lists >= (int64_t)1 << 23 || (!plan.fused && (lists * parts >= (int64_t)1 << 24 || parts > 65535)))
        return s3_fail(S3_EINVAL, "%s: %lld lists over %d blocks are too many for one call", fn, (long long)lists, plan.nb);
    const int es = c->dtype == S3_BF16 ? 2 : 4;
    SelectArgs p{s3_kv_batch_args(c, b), (const char*)q, q_ts * es, q_hs * es, (const __bf16*)c->sig, (unsigned*)ws, sel,
                 c->n_kv_heads, n_q / c->n_kv_heads, q_block, top_b, lead, tail, plan.nb};
    hipStream_t st = (hipStream_t)stream;
    if (c->dtype == S3_BF16)
        return c->d_head == 64 ? launch_select<__bf16, 64>(p, plan, st) : c->d_head == 128 ? launch_select<__bf16, 128>(p, plan, st) : launch_select<__bf16, 256>(p, plan, st);
    return c->d_head == 64 ? launch_select<float, 64>(p, plan, st) : c->d_head == 128 ? launch_select<float, 128>(p, plan, st) : launch_select<float, 256>(p, plan, st);
}
