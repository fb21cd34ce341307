// Attention of few rows: sequences (or tiles of listed blocks) whose new tokens times query heads per key/value head are 128 at most.
//
// The work is one pass over the keys and values, so memory bounds it: 64 decoding steps of 300 to 32768 tokens (1.86 GB)
// take 348 us with the join, 5.3 TB/s (a copy moves 4.8).  All of it, over all sequences and heads, is one line of pieces of 128 tokens, and every
// workgroup takes an equal run of that line whatever the lengths are: a long sequence is shared by many workgroups, short ones lie
// whole in one.  A workgroup's four wavefronts take 32 tokens of a piece each, keys and values straight from memory into the
// matrix instructions' operands, the next 32 tokens' keys on their way while the weights are made and the next values
// during the next scores.  Where a run ends inside a row tile, its sums go to scratch, and a second kernel joins them.
// Of 64 or 128 rows, RT sets of 32, the wavefronts have a set each and a piece has as many fewer tokens: those with the same tokens find them
// in the compute unit's cache (4300 MB of listed blocks of a long cache: 758 us where each set read its own, 419 so).
#include "attn_launch.h"

namespace {

constexpr int kThreads = 256, kWaves = 4;
template <int RT> constexpr int kPiece = 32 * kWaves / RT;      // tokens of a piece: 32 for every wavefront of a row set
constexpr int kRunGroups = 512;        // workgroups that share the line: two per compute unit
constexpr int kBatchRuns = 1024;       // runs of 16 tokens whose pages are looked up at a time

__device__ __forceinline__ int64_t wave_incl_scan64(int64_t x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t y = __shfl_up(x, d);
        if ((int)(threadIdx.x & 63) >= d) x += y;
    }
    return x;
}

// fp32 of a scratch slot: R rows' sums, their maxima and the weights' sums; whole 16-byte pieces, for R may be odd.
__host__ __device__ __forceinline__ int64_t slot_floats(int R, int D) { return ((int64_t)R * (D + 2) + 3) & ~(int64_t)3; }

// A sequence's part of the line: row tiles (one, or one a tile of listed blocks), each with n_kv heads of `pieces` pieces that begin at token lo.
struct Part {
    int first, n, len, lo, tiles, pieces;
};
template <bool LIST, int RT>
__device__ __forceinline__ Part part_of(const AttnArgs& p, int s) {
    Part r;
    kv_seq(p.b, s, r.first, r.n, r.len);
    r.lo = 0;
    if (LIST) {
        r.tiles = (r.n + p.qb - 1) / p.qb;
        r.pieces = ((p.top << p.b.log_page) + kPiece<RT> - 1) / kPiece<RT>;
    } else {
        r.tiles = r.n > 0 && r.n * p.G <= p.few ? 1 : 0;
        if (p.window) r.lo = max(0, r.len - r.n - p.window + 1) & ~31;
        const int hi = min(r.len, kv_blocks(p.b, r.len) << p.b.log_page);
        r.pieces = (max(hi - r.lo, 1) + kPiece<RT> - 1) / kPiece<RT>;         // one at least: rows that see nothing are written, too
    }
    return r;
}

// Rows of a tile: the first, and the end (32 RT of them at most, as the host saw to it).
template <bool LIST, int RT>
__device__ __forceinline__ void rows_of(const AttnArgs& p, const Part& part, int tile, int& r0, int& r_end) {
    r0 = __builtin_amdgcn_readfirstlane(LIST ? tile * p.qb * p.G : 0);
    r_end = __builtin_amdgcn_readfirstlane(min((LIST ? min(part.n, (tile + 1) * p.qb) : part.n) * p.G, r0 + 32 * RT));
}

// The line's length and equal runs of it.
template <bool LIST, int RT>
__device__ __forceinline__ int64_t line_length(const AttnArgs& p) {
    int64_t total = 0;
    for (int base = 0; base < p.b.n_seq; base += 64) {
        const int s = base + (threadIdx.x & 63);
        int64_t c = 0;
        if (s < p.b.n_seq) {
            const Part r = part_of<LIST, RT>(p, s);
            c = (int64_t)r.tiles * r.pieces * p.n_kv;
        }
        total += __shfl(wave_incl_scan64(c), 63);
    }
    return total;
}

template <typename T, int D, bool LIST, int RT>
__global__ __launch_bounds__(kThreads, D * sizeof(T) > 256 ? 1 : 2) void attn_stream_kernel(AttnArgs p, float* slots, int R) {
    constexpr int E = KvElem<T>::E, NW = 16 / E, QS = kQSteps<D, T>, ES = (int)sizeof(T), LD = D + 4, PIECE = kPiece<RT>, RUNS = PIECE / 16;
    typedef typename KvElem<T>::vec vec;
    extern __shared__ char lds[];
    __shared__ int wave_sum[kWaves];
    float* sum_m = (float*)lds;                       // [kWaves][32]
    float* sum_l = sum_m + kWaves * 32;               // [kWaves][32]
    int2* runs = (int2*)(sum_l + kWaves * 32);        // [kBatchRuns + 16]: position of 16 tokens (or beyond all), page
    float* sum_o = (float*)(runs + kBatchRuns + 16);   // [kWaves][R][LD]
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int set = wave % RT, sub_of = wave / RT, RR = min(R, 32);       // the wavefront's row set, and which 32 tokens of a piece it has
    const int logp = p.b.log_page, P = 1 << logp;
    const int64_t page_bytes = (int64_t)P * D * ES;

    const int64_t total = line_length<LIST, RT>(p);
    const int64_t per = (total + gridDim.x - 1) / gridDim.x;
    int64_t at = per * blockIdx.x;
    const int64_t end = min(total, at + per);
    if (at >= end) return;
    // sequence and place in it of the first piece; `tile0`: tiles of the sequences before it (lists)
    int s = 0, tile0 = 0;
    int64_t rem = 0;
    {
        int64_t run = 0;
        for (int base = 0; base < p.b.n_seq; base += 64) {
            const int q = base + lane;
            int64_t c = 0;
            int tiles = 0;
            if (q < p.b.n_seq) {
                const Part r = part_of<LIST, RT>(p, q);
                tiles = r.tiles;
                c = (int64_t)r.tiles * r.pieces * p.n_kv;
            }
            const int64_t incl = wave_incl_scan64(c);
            const int64_t sum = __shfl(incl, 63);
            const int t_incl = LIST ? s3_wave_incl_scan(tiles) : 0;
            if (at < run + sum) {
                const int l = __builtin_ctzll(__ballot(run + incl > at));
                s = base + l;
                rem = at - (run + __shfl(incl, l) - __shfl(c, l));
                if (LIST) tile0 = kv_add_lists(tile0, __builtin_amdgcn_readlane(t_incl, l) - __builtin_amdgcn_readlane(tiles, l));
                break;
            }
            run += sum;
            if (LIST) tile0 = kv_add_lists(tile0, __builtin_amdgcn_readlane(t_incl, 63));
        }
        s = __builtin_amdgcn_readfirstlane(s);
    }

    while (at < end) {
        const Part part = part_of<LIST, RT>(p, s);
        const int64_t size = (int64_t)part.tiles * part.pieces * p.n_kv;
        if (rem >= size) {
            ++s;
            rem = 0;
            tile0 = kv_add_lists(tile0, part.tiles);
            continue;
        }
        // all lanes' values: in scalar registers, for the vector ones are all in use
        const int c0 = __builtin_amdgcn_readfirstlane((int)(rem % part.pieces));
        const int64_t u = rem / part.pieces;
        const int tile = LIST ? __builtin_amdgcn_readfirstlane((int)(u / p.n_kv)) : 0;
        const int head = __builtin_amdgcn_readfirstlane(LIST ? (int)(u % p.n_kv) : (int)u);
        const int c1 = __builtin_amdgcn_readfirstlane((int)min((int64_t)part.pieces, c0 + (end - at)));

        int r0, r_end;
        rows_of<LIST, RT>(p, part, tile, r0, r_end);
        AttnRows<T, D> rows;
        rows.load(p, head, part.first, part.n, part.len, r0 + set * 32 + col, r_end);
        AttnState<T, D> st;
        st.clear();
        bool seen = false;
        const int pos0 = part.len - part.n + (r0 + set * 32) / p.G;               // the set's first row's position
        const int last = part.len - part.n + (r_end - 1) / p.G;                   // the last row's; its tokens end at hi
        const int hi = min(last + 1, kv_blocks(p.b, part.len) << logp);
        const AttnSight sight(rows.pos, hi, p.window);
        const int32_t* list = LIST ? p.sel + ((int64_t)(tile0 + tile) * p.n_kv + head) * p.top : nullptr;
        const int n_list = LIST && tile0 + tile < p.lists ? p.top << (logp - 4) : 0;
        for (int cb = c0; cb < c1; cb += kBatchRuns / RUNS) {
            int n = min(c1 - cb, kBatchRuns / RUNS) * RUNS;
            __syncthreads();                                                       // the last batch, the last tile's sums are read
            if (LIST) {
                int there = 0;
                for (int i0 = 0; i0 < n; i0 += kThreads) {
                    const int j = cb * RUNS + i0 + tid;
                    const int blk = i0 + tid < n && j < n_list ? list[j >> (logp - 4)] : -1;
                    const int pos = blk >= 0 && blk < p.b.max_pages ? (blk << logp) + (j & (P / 16 - 1)) * 16 : 1 << 30;
                    const int page = pos < hi ? kv_page(p.b, s, blk) : -1;
                    int total;
                    const int at = kv_compact<kWaves>(page >= 0, wave_sum, total);
                    if (page >= 0) runs[there + at] = int2{pos, page};
                    there += total;
                }
                n = (there + RUNS - 1) / RUNS * RUNS;
                if (tid < n + 8 - there) runs[there + tid] = int2{1 << 30, -1};
            } else {
                for (int i = tid; i < n + 8; i += kThreads) {
                    int pos = i < n ? part.lo + cb * PIECE + i * 16 : 1 << 30;
                    const int page = pos < hi ? kv_page(p.b, s, pos >> logp) : -1;
                    runs[i] = int2{page < 0 ? 1 << 30 : pos, page};
                }
            }
            __syncthreads();
            if (n == 0) continue;
            const int n_sub = n / RUNS;
            // keys and values in VC parts of the channels: all of them ahead, or (fp32, 256 channels) only the first, as far as registers go
            constexpr int VC = D * ES > 512 ? 2 : 1, DC = D / 32 / VC, QC = QS / VC;
            vec kf[QC], vf[DC * NW];
            int2 ra = runs[2 * sub_of], rb = runs[2 * sub_of + 1];
            auto load_k = [&](int2 a, int2 b, int part) {
                const int tk = kv_token<T>(col);
                const int2 r = tk < 16 ? a : b;
                const char* k = p.k + ((int64_t)max(r.y, 0) * p.n_kv + head) * page_bytes + ((r.y < 0 ? 0 : r.x & (P - 1)) + (tk & 15) + half * P) * 16 + part * (QC * 32) * P;
#pragma unroll
                for (int q = 0; q < QC; ++q) kf[q] = *(const vec*)(k + q * 32 * P);
            };
            auto load_v = [&](int2 a, int2 b, int part) {
#pragma unroll
                for (int y = 0; y < NW; ++y) {
                    const int t = E * (2 * y + half);                              // first of this lane's E tokens: in one run for all lanes
                    const int2 r = 2 * E * y < 16 ? a : b;
                    const char* v = p.v + ((int64_t)max(r.y, 0) * p.n_kv + head) * page_bytes + ((r.y < 0 ? 0 : r.x & (P - 1)) + (t & 15)) / E * (D * 16) + col * 16 + part * (DC * 512);
#pragma unroll
                    for (int dt = 0; dt < DC; ++dt) vf[dt * NW + y] = *(const vec*)(v + dt * 512);
                }
            };
            // some row does not see some token of the 32
            auto is_masked = [&](int2 a, int2 b) {
                const int far = max(a.x, b.x) + 15;
                return far > pos0 || far >= hi || (p.window && min(a.x, b.x) <= last - p.window);
            };
            bool odd = false;
            load_k(ra, rb, 0);
            load_v(ra, rb, 0);
            for (int i = 0; i < n_sub; ++i) {
                const int2 a = ra, b = rb;
                kv_f32x16 sc;
#pragma unroll
                for (int x = 0; x < 16; ++x) sc[x] = 0.0f;
#pragma unroll
                for (int part = 0; part < VC; ++part) {
                    if (part) {
                        load_k(a, b, part);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int q = 0; q < QC; ++q) sc = kv_mma(kf[q], rows.q[part * QC + q], sc);
                    if (VC > 1) __builtin_amdgcn_sched_barrier(0);
                }
                const bool more = i + 1 < n_sub;
                if (more) {
                    ra = runs[(i + 1) * RUNS + 2 * sub_of];
                    rb = runs[(i + 1) * RUNS + 2 * sub_of + 1];
                    load_k(ra, rb, 0);
                }
                const bool masked = is_masked(a, b);
                if (masked) {
                    asm volatile("");                                              // stays a branch: most pieces skip it
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const int t = 2 * E * (x / E) + E * half + x % E;
                        const bool sees = sight.sees((2 * E * (x / E) < 16 ? a.x : b.x) + (t & 15));
                        seen |= sees;
                        sc[x] = sees ? sc[x] : -INFINITY;
                    }
                } else {
                    seen = true;
                }
                float x = sc[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) x = fmaxf(x, sc[e]);
                const float sub = st.advance(x, p.sl);
                vec w[NW];
#pragma unroll
                for (int y = 0; y < NW; ++y) w[y] = st.weights(sc, y, p.sl, sub);
#pragma unroll
                for (int part = 0; part < VC; ++part) {
                    if (part) {
                        __builtin_amdgcn_sched_barrier(0);
                        load_v(a, b, part);
                    }
                    if (masked) {
                        unsigned big = 0;
#pragma unroll
                        for (int y = 0; y < NW; ++y) {
                            const int n = hi - (2 * E * y < 16 ? a.x : b.x) - (E * (2 * y + half) & 15);
#pragma unroll
                            for (int dt = 0; dt < DC; ++dt) {
                                vf[dt * NW + y] = kv_first(vf[dt * NW + y], n);
                                big = kv_magnitude(vf[dt * NW + y], big);
                            }
                        }
                        if (__ballot(big >= 0x7f800000u)) {
                            odd = true;
#pragma unroll
                            for (int y = 0; y < DC * NW; ++y) vf[y] = kv_finite(vf[y]);
                        }
                    }
#pragma unroll
                    for (int dt = 0; dt < DC; ++dt)
#pragma unroll
                        for (int y = 0; y < NW; ++y) st.o[part * DC + dt] = kv_mma(vf[dt * NW + y], w[y], st.o[part * DC + dt]);
                }
                if (more) load_v(ra, rb, 0);
            }
            if (odd)
                for (int i = 0; i < n_sub; ++i) {
                    const int2 a = runs[i * RUNS + 2 * sub_of], b = runs[i * RUNS + 2 * sub_of + 1];
                    if (!is_masked(a, b)) continue;
#pragma unroll 1
                    for (int j = 0; j < 32; ++j) {
                        const int2 r = j < 16 ? a : b;
                        if (r.x + (j & 15) >= hi) continue;
                        const int slot = (r.x & (P - 1)) + (j & 15);
                        const char* v = p.v + ((int64_t)r.y * p.n_kv + head) * page_bytes + slot / E * (D * 16) + slot % E * ES;
                        st.add_nonfinite(sight.sees(r.x + (j & 15)), [&](int c) { return (float)*(const T*)(v + c * 16); });
                    }
                }
        }

        // the sums of a row set's wavefronts
        st.settle(seen);
        const float l = kv_pair_sum(st.l);
        if (half == 0) {
            sum_m[wave * 32 + col] = st.m;
            sum_l[wave * 32 + col] = l;
        }
        __syncthreads();
        if (col < RR) {
            float m = sum_m[set * 32 + col];
#pragma unroll
            for (int w = RT; w < kWaves; w += RT) m = fmaxf(m, sum_m[(set + w) * 32 + col]);
            const float f = st.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st.m - m);
            float* dst = sum_o + (wave * RR + col) * LD + half * 4;
            // a wavefront that saw nothing has sums of zero; one whose sums hold a NaN keeps it through a factor of zero
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    *(kv_f32x4*)(dst + dt * 32 + x * 8) =
                        kv_f32x4{st.o[dt][4 * x] * f, st.o[dt][4 * x + 1] * f, st.o[dt][4 * x + 2] * f, st.o[dt][4 * x + 3] * f};
        }
        __syncthreads();
        const bool whole = c0 == 0 && c1 == part.pieces;
        float* slot = slots + ((int64_t)blockIdx.x * 2 + (c0 == 0)) * slot_floats(R, D);
        const int n_rows = min(R, r_end - r0);
        for (int i = tid; i < n_rows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4, first = r / 32, rr = r & 31;
            float m = sum_m[first * 32 + rr], lsum = 0.0f;
#pragma unroll
            for (int w = RT; w < kWaves; w += RT) m = fmaxf(m, sum_m[(first + w) * 32 + rr]);
            kv_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kWaves; w += RT) {
                const int x = (first + w) * 32 + rr;
                lsum += sum_l[x] * kv_factor(sum_m[x], sum_l[x], m);
                o += *(const kv_f32x4*)(sum_o + ((first + w) * RR + rr) * LD + c);
            }
            if (whole) {
                const int t = (r0 + r) / p.G;
                const int64_t row = (int64_t)(part.first + t) * p.n_q + head * p.G + (r0 + r - t * p.G);
                const float inv = kv_inverse(m, lsum);
                typedef __attribute__((ext_vector_type(4))) T four;
                *(four*)(p.out + (row * D + c) * ES) = four{(T)(o[0] * inv), (T)(o[1] * inv), (T)(o[2] * inv), (T)(o[3] * inv)};
                if (p.lse && c == 0) p.lse[row] = kv_lse(m, lsum);
            } else {
                *(kv_f32x4*)(slot + r * D + c) = o;
                if (c == 0) {
                    slot[R * D + r] = m;
                    slot[R * D + R + r] = lsum;
                }
            }
        }
        at += c1 - c0;
        rem += c1 - c0;
    }
}

// Joins the runs of the row tiles that more than one workgroup had: workgroups per tile and head that take
// 32 channels of 4 rows at a time; eight threads have a row's channels, and eight such share its runs.
template <typename T, int D, bool LIST, int RT>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs p, const float* slots, int R, int groups) {
    __shared__ float part_o[kThreads][4], part_m[kThreads], part_l[kThreads];
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t total = line_length<LIST, RT>(p);
    const int64_t per = (total + groups - 1) / groups;
    // the tile's place on the line
    const int head = blockIdx.x % p.n_kv;
    int64_t want = blockIdx.x / p.n_kv, run = 0;
    int s = -1;
    for (int base = 0; base < p.b.n_seq; base += 64) {
        const int q = base + lane;
        int64_t c = 0;
        int tiles = 0;
        if (q < p.b.n_seq) {
            const Part r = part_of<LIST, RT>(p, q);
            tiles = r.tiles;
            c = (int64_t)r.tiles * r.pieces * p.n_kv;
        }
        const int64_t incl = wave_incl_scan64(c);
        const int t_incl = s3_wave_incl_scan(tiles);
        const int t_sum = __builtin_amdgcn_readlane(t_incl, 63);
        if (want < t_sum) {
            const int l = __builtin_ctzll(__ballot(t_incl > want));
            s = base + l;
            want -= __builtin_amdgcn_readlane(t_incl, l) - __builtin_amdgcn_readlane(tiles, l);
            run += __shfl(incl, l) - __shfl(c, l);
            break;
        }
        want -= t_sum;
        run += __shfl(incl, 63);
    }
    if (s < 0) return;
    const Part part = part_of<LIST, RT>(p, s);
    const int64_t a = run + (want * p.n_kv + head) * part.pieces, b = a + part.pieces;
    const int w0 = (int)(a / per), w1 = (int)((b - 1) / per);
    if (w0 == w1) return;
    int r0, r_end;
    rows_of<LIST, RT>(p, part, (int)want, r0, r_end);
    const int n_rows = min(R, r_end - r0);
    const int64_t stride = slot_floats(R, D);
    const int k = tid >> 5;
    constexpr int kShare = kThreads / 32;
    for (int x = blockIdx.y; x < (n_rows + 3) / 4 * (D / 32); x += gridDim.y) {
        const int c = x % (D / 32) * 32 + (tid & 7) * 4, r = x / (D / 32) * 4 + (tid >> 3 & 3);
        float m = -INFINITY, l = 0.0f;
        kv_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        // sums against m and one more's against mw, both against the larger
        auto add = [&](float mw, float lw, kv_f32x4 ow) {
            const float m2 = fmaxf(m, mw), a = kv_factor(m, l, m2), b = kv_factor(mw, lw, m2);
            m = m2;
            l = l * a + lw * b;
            o = o * a + ow * b;
        };
        if (r < n_rows) {
#pragma unroll 4
            for (int w = w0 + k; w <= w1; w += kShare) {
                const float* slot = slots + (w * 2 + (w == w0)) * stride;
                add(slot[R * D + r], slot[R * D + R + r], *(const kv_f32x4*)(slot + r * D + c));
            }
        }
        part_m[tid] = m;
        part_l[tid] = l;
#pragma unroll
        for (int e = 0; e < 4; ++e) part_o[tid][e] = o[e];
        __syncthreads();
        if (k == 0 && r < n_rows) {
#pragma unroll
            for (int w = 1; w < kShare; ++w) {
                const int y = tid + w * 32;
                add(part_m[y], part_l[y], kv_f32x4{part_o[y][0], part_o[y][1], part_o[y][2], part_o[y][3]});
            }
            const int t = (r0 + r) / p.G;
            const int64_t row = (int64_t)(part.first + t) * p.n_q + head * p.G + (r0 + r - t * p.G);
            const float inv = kv_inverse(m, l);
            typedef __attribute__((ext_vector_type(4))) T four;
            *(four*)(p.out + (row * D + c) * (int)sizeof(T)) = four{(T)(o[0] * inv), (T)(o[1] * inv), (T)(o[2] * inv), (T)(o[3] * inv)};
            if (p.lse && c == 0) p.lse[row] = kv_lse(m, l);
        }
        __syncthreads();
    }
}

template <typename T, int D, bool LIST, int RT>
int launch(const AttnArgs& p, int64_t tiles, int R, float* ws, hipStream_t st) {
    static S3LdsOnce once;
    const int bytes = kWaves * 32 * 8 + (kBatchRuns + 16) * 8 + kWaves * min(R, 32) * (D + 4) * 4;
    if (int rc = s3_allow_lds(once, (const void*)attn_stream_kernel<T, D, LIST, RT>, kWaves * 32 * 8 + (kBatchRuns + 16) * 8 + kWaves * 32 * (D + 4) * 4)) return rc;
    const int64_t join = tiles * p.n_kv;
    hipLaunchKernelGGL((attn_stream_kernel<T, D, LIST, RT>), dim3(kRunGroups), dim3(kThreads), bytes, st, p, ws, R);
    S3_HIP(hipGetLastError());
    hipLaunchKernelGGL((attn_join_kernel<T, D, LIST, RT>), dim3((unsigned)join, (unsigned)max((int64_t)1, min(4096 / join, (int64_t)(D / 32 * ((R + 3) / 4))))), dim3(kThreads), 0, st, p, ws, R, kRunGroups);
    S3_HIP(hipGetLastError());
    return S3_OK;
}

// Row sets of 32 as R needs them, as many as s3_few_rows lets through.
template <typename T, int D, bool LIST>
int launch_rows(const AttnArgs& p, int64_t tiles, int R, float* ws, hipStream_t st) {
    constexpr int most = s3_few_rows(sizeof(T) == 2, D, LIST);
    if constexpr (most > 64)
        if (R > 64) return launch<T, D, LIST, 4>(p, tiles, R, ws, st);
    if constexpr (most > 32)
        if (R > 32) return launch<T, D, LIST, 2>(p, tiles, R, ws, st);
    return launch<T, D, LIST, 1>(p, tiles, R, ws, st);
}

}  // namespace

size_t s3_attn_stream_workspace(int d_head, int R) { return s3_align((size_t)kRunGroups * 2 * slot_floats(R, d_head) * 4); }

int s3_attn_stream(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int R, void* ws, hipStream_t st) {
#define S3_STREAM(T, D) (p.sel ? launch_rows<T, D, true>(p, tiles, R, (float*)ws, st) : launch_rows<T, D, false>(p, tiles, R, (float*)ws, st))
    if (c->dtype == S3_BF16) return c->d_head == 64 ? S3_STREAM(__bf16, 64) : c->d_head == 128 ? S3_STREAM(__bf16, 128) : S3_STREAM(__bf16, 256);
    return c->d_head == 64 ? S3_STREAM(float, 64) : c->d_head == 128 ? S3_STREAM(float, 128) : S3_STREAM(float, 256);
#undef S3_STREAM
}
