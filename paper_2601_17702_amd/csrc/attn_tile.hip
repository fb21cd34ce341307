// Attention of many rows: chunks of new tokens (and tiles of listed blocks) with more rows per key/value head than attn_stream.hip takes.
//
// The two products bound it.  A workgroup has WAVES wavefronts of 32 rows each, the rows of a head's G query heads token by
// token, and walks over the tokens that some row sees, KT at a time: keys and values come through registers into one of two LDS
// buffers while the other is worked on, in the layout that they have in the cache, which is the one in which every operand read
// is 16 bytes a lane from neighbouring places (no bank conflicts, no transposition).  LDS feeds 128 bytes a clock: with 32 rows a wavefront
// all of it at the matrix units' full rate, which the card's clock does not let them reach (below).
//
// Measured: 2048 tokens at 131072, 32 query heads over 8, d_head 128, bf16 (4.4 TFLOP): 4.1 ms, 1050 TFLOP/s, where a large library product
// reaches 1159 on the card.  MFMAs are busy 48 % of the cycles at 1.9 GHz; a variant half as fast ran at 2.33 GHz, so the clock gives
// way before the units are full.  d_head 256 has one wavefront a SIMD (512 registers) and 43 % of that product's rate, fp32 70 % of fp32's.
#include "attn_launch.h"

namespace {

constexpr int kBatchRuns = 1024;       // runs of 16 tokens whose pages are looked up at a time

template <typename T, int D> constexpr int kTokens = D * (int)sizeof(T) > 512 ? 32 : 64;     // tokens of a buffer

struct TileArgs {
    float* slots;             // partial sums where n_split > 1
    int n_split, tiles;       // row tiles that there can be
};

template <typename T, int D, bool LIST, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 4) void attn_tile_kernel(AttnArgs p, TileArgs ta) {
    constexpr int E = KvElem<T>::E, NW = 16 / E, QS = kQSteps<D, T>, ES = (int)sizeof(T), KT = kTokens<T, D>, NS = KT / 32;
    constexpr int THREADS = WAVES * 64, ROWS = WAVES * 32;
    constexpr int PIECES = KT * D / E, LOADS = PIECES / THREADS;       // 16-byte pieces of a buffer's keys (and of its values)
    static_assert(PIECES % THREADS == 0, "every thread has as many pieces");
    typedef typename KvElem<T>::vec vec;
    extern __shared__ char lds[];
    __shared__ int wave_sum[WAVES];
    char* buf = lds;                                                  // [2][keys | values][PIECES * 16]
    int4* runs = (int4*)(lds + 4 * PIECES * 16);                      // [kBatchRuns]: bytes to 16 tokens' page and head, slot, position (2^30: none)
    int2* spans = (int2*)(runs + kBatchRuns);                         // [kBatchRuns * 16 / KT]: a step's least and largest position
    int* odd_step = (int*)(spans + kBatchRuns * 16 / KT);             // [2]: the step whose values in that buffer were not all finite
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int logp = p.b.log_page, P = 1 << logp;
    const int64_t page_bytes = (int64_t)P * D * ES;

    // longest first: later row tiles see more
    const int head = blockIdx.x % p.n_kv;
    const int tile = ta.tiles - 1 - blockIdx.x / p.n_kv;
    auto count = [&](int n, int) { return LIST ? (n + p.qb - 1) / p.qb * p.per_q : n * p.G <= p.few ? 0 : (n * p.G + ROWS - 1) / ROWS; };
    int s, j, first, n, len;
    if (!kv_find(p.b, tile, count, s, j, first, n, len)) return;
    int r0 = j * ROWS, r_end = n * p.G;
    if (LIST) {
        const int qt = j / p.per_q;
        r0 = qt * p.qb * p.G + (j - qt * p.per_q) * ROWS;
        r_end = min(n, (qt + 1) * p.qb) * p.G;
        if (r0 >= r_end) return;
    }
    r_end = min(r_end, r0 + ROWS);
    const int hi = min(len - n + (r_end - 1) / p.G + 1, kv_blocks(p.b, len) << logp);     // tokens that some row may see
    const int lo = p.window ? max(0, len - n + r0 / p.G - p.window + 1) & ~(KT - 1) : 0;
    const int32_t* list = LIST ? p.sel + ((int64_t)(tile / p.per_q) * p.n_kv + head) * p.top : nullptr;
    const int n_list = LIST ? p.top << (logp - 4) : 0;
    const int steps = LIST ? (n_list * 16 + KT - 1) / KT : (max(hi - lo, 0) + KT - 1) / KT;
    const int split = blockIdx.y;
    const int t0 = (int)((int64_t)steps * split / ta.n_split), t1 = (int)((int64_t)steps * (split + 1) / ta.n_split);

    const int rw = r0 + wave * 32;                             // this wavefront's first row
    const int pos0 = len - n + rw / p.G;                              // its position, and the last row's
    const int pos1 = rw < r_end ? len - n + (min(rw + 32, r_end) - 1) / p.G : -1;
    AttnRows<T, D> rows;
    AttnState<T, D> st;
    rows.load(p, head, first, n, len, rw + col, r_end);
    st.clear();
    bool seen = false;
    const AttnSight sight(rows.pos, hi, p.window);

    // what some row of the workgroup does not see: such steps are masked, and their values looked at
    const int wg0 = len - n + r0 / p.G, wg1 = len - n + (r_end - 1) / p.G;
    auto partly = [&](int2 span, int first_pos, int last_pos) {
        return span.y > first_pos || span.y >= hi || (p.window && span.x <= last_pos - p.window);
    };
    auto span_of = [&](int t) {
        const int2 x = spans[t];
        return int2{__builtin_amdgcn_readfirstlane(x.x), __builtin_amdgcn_readfirstlane(x.y)};
    };
    // this thread's pieces: where they lie within their 16 tokens (the rest is the same for all of those)
    vec stage[2 * LOADS];
    const char *kp[LOADS], *vp[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int x = tid + i * THREADS;
        kp[i] = p.k + (x / KT * P + x % 16) * 16;
        vp[i] = p.v + (x / D * E % 16 / E * D + x % D) * 16;
    }
    auto fetch = [&](int t) {                                         // step t of the batch: into registers
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int4 r = runs[t * (KT / 16) + (tid + i * THREADS) % KT / 16];
            stage[i] = *(const vec*)(kp[i] + ((int64_t)(((uint64_t)(unsigned)r.y << 32) | (unsigned)r.x) + r.z * 16));
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int4 r = runs[t * (KT / 16) + (tid + i * THREADS) / D * E / 16];
            stage[LOADS + i] = *(const vec*)(vp[i] + ((int64_t)(((uint64_t)(unsigned)r.y << 32) | (unsigned)r.x) + r.z * (D * 16 / E)));
        }
    };
    // Where some row does not see some token of the step, values that are not finite leave the buffer: their products with a weight of zero
    // would be NaN.  The rows that do see them get them from memory, one token at a time (rare); what lies past the end is zero.
    auto store = [&](int t) {
        if (partly(span_of(t), wg0, wg1)) {
            unsigned big = 0;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int g = (tid + i * THREADS) / D * E;
                stage[LOADS + i] = kv_first(stage[LOADS + i], hi - runs[t * (KT / 16) + g / 16].w - g % 16);
                big = kv_magnitude(stage[LOADS + i], big);
            }
            if (big >= 0x7f800000u) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) stage[LOADS + i] = kv_finite(stage[LOADS + i]);
                odd_step[t & 1] = t;
            }
        }
        char* dst = buf + (t & 1) * (2 * PIECES * 16) + tid * 16;
#pragma unroll
        for (int i = 0; i < 2 * LOADS; ++i) *(vec*)(dst + i * THREADS * 16) = stage[i];
    };

    constexpr int kBatch = kBatchRuns / (KT / 16);                    // steps whose pages are known at a time
    for (int tb = t0; tb < t1; tb += kBatch) {
        int nb = min(kBatch, t1 - tb);
        __syncthreads();
        if (tid < 2) odd_step[tid] = -1;
        auto put = [&](int i, int pos, int page) {
            const int64_t at = ((int64_t)max(page, 0) * p.n_kv + head) * page_bytes;      // no page: any memory of the cache
            runs[i] = int4{(int)at, (int)(at >> 32), page < 0 ? 0 : pos & (P - 1), page < 0 ? 1 << 30 : pos};
        };
        if (LIST) {
            int there = 0;
            for (int i0 = 0; i0 < nb * (KT / 16); i0 += THREADS) {
                const int x = tb * (KT / 16) + i0 + tid;
                const int blk = i0 + tid < nb * (KT / 16) && x < n_list ? list[x >> (logp - 4)] : -1;
                const int pos = blk >= 0 && blk < p.b.max_pages ? (blk << logp) + (x & (P / 16 - 1)) * 16 : 1 << 30;
                const int page = pos < hi ? kv_page(p.b, s, blk) : -1;
                int total;
                const int at = kv_compact<WAVES>(page >= 0, wave_sum, total);
                if (page >= 0) put(there + at, pos, page);
                there += total;
            }
            nb = (there + KT / 16 - 1) / (KT / 16);
            if (tid < nb * (KT / 16) - there) put(there + tid, 1 << 30, -1);
            if (nb == 0) continue;
        } else {
            for (int i = tid; i < nb * (KT / 16); i += THREADS) {
                const int pos = lo + tb * KT + i * 16;
                put(i, pos, pos < hi ? kv_page(p.b, s, pos >> logp) : -1);
            }
        }
        __syncthreads();
        for (int i = tid; i < nb; i += THREADS) {
            int2 span = {1 << 30, 0};
#pragma unroll
            for (int x = 0; x < KT / 16; ++x) {
                const int pos = runs[i * (KT / 16) + x].w;
                span.x = min(span.x, pos);
                span.y = max(span.y, pos + 15);
            }
            spans[i] = span;
        }
        __syncthreads();
        fetch(0);
        store(0);
        __syncthreads();
        for (int t = 0; t < nb; ++t) {
            const bool more = t + 1 < nb;
            if (more) fetch(t + 1);
            const char* kb = buf + (t & 1) * (2 * PIECES * 16);
            const char* vb = kb + PIECES * 16;
            const int2 span = span_of(t);
            if (span.x <= pos1) {                                     // some row of the wavefront sees some token
                // kAhead operands are read ahead of the products that take them (the compiler's own order waits for each)
                constexpr int kAhead = 6, kProducts = E == 8 ? 1 : 4, DT = D / 32;
                kv_f32x16 sc[NS];
#pragma unroll
                for (int x = 0; x < NS; ++x) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[x][i] = 0.0f;
#pragma unroll
                    for (int q = 0; q < QS; ++q)
                        sc[x] = kv_mma(*(const vec*)(kb + ((2 * q + half) * KT + x * 32 + kv_token<T>(col)) * 16), rows.q[q], sc[x]);
                }
                auto values = [&](int y, vec (&v)[DT]) {              // operands of E tokens a lane
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) v[dt] = *(const vec*)(vb + ((2 * y + half) * D + dt * 32 + col) * 16);
                };
                vec v[2][DT], w[2];
                values(0, v[0]);
                __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
                for (int i = 0; i < NS * QS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, kProducts, 0);
                    if (i + kAhead < NS * QS + DT) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                const bool masked = partly(span, pos0, pos1);
                if (masked) {
                    asm volatile("");                                 // stays a branch: most steps skip it
#pragma unroll
                    for (int x = 0; x < NS; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int tk = x * 32 + 2 * E * (i / E) + E * half + i % E;
                            const bool sees = sight.sees(runs[t * (KT / 16) + (x * 32 + 2 * E * (i / E)) / 16].w + (tk & 15));
                            seen |= sees;
                            sc[x][i] = sees ? sc[x][i] : -INFINITY;
                        }
                } else {
                    seen = true;
                }
                float top = sc[0][0];
#pragma unroll
                for (int y = 0; y < NS; ++y)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[y][i]);
                const float sub = st.advance(top, p.sl);
                // the weights and operands of the next tokens are made while these tokens' products run
                w[0] = st.weights(sc[0], 0, p.sl, sub);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int y = 0; y < NS * NW; ++y) {
                    if (y + 1 < NS * NW) {
                        values(y + 1, v[(y + 1) & 1]);
                        w[(y + 1) & 1] = st.weights(sc[(y + 1) / NW], (y + 1) % NW, p.sl, sub);
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) st.o[dt] = kv_mma(v[y & 1][dt], w[y & 1], st.o[dt]);
                    if (y + 1 < NS * NW) {
                        __builtin_amdgcn_sched_group_barrier(0x100, DT, 0);
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            __builtin_amdgcn_sched_group_barrier(0x8, kProducts, 0);
                            __builtin_amdgcn_sched_group_barrier(0x402, (E * 7 / 2 + DT - 1) / DT, 0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (partly(span, wg0, wg1) && odd_step[t & 1] == t)
#pragma unroll 1
                    for (int tk = 0; tk < KT; ++tk) {
                        const int4 r = runs[t * (KT / 16) + tk / 16];
                        const int slot = r.z + (tk & 15);
                        if (r.w + (tk & 15) >= hi) continue;
                        const char* src = p.v + ((int64_t)(((uint64_t)(unsigned)r.y << 32) | (unsigned)r.x)) + slot / E * (D * 16) + slot % E * ES;
                        st.add_nonfinite(sight.sees(r.w + (tk & 15)), [&](int c) { return (float)*(const T*)(src + c * 16); });
                    }
            }
            if (more) store(t + 1);
            __syncthreads();
        }
    }

    st.settle(seen);
    const float l = kv_pair_sum(st.l);
    if (ta.n_split > 1) {
        const int row = wave * 32 + col;
        float* slot = ta.slots + ((int64_t)(tile * p.n_kv + head) * ta.n_split + split) * ((int64_t)ROWS * (D + 2));
        if (r0 + row < r_end) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    *(kv_f32x4*)(slot + row * D + dt * 32 + a * 8 + half * 4) =
                        kv_f32x4{st.o[dt][4 * a], st.o[dt][4 * a + 1], st.o[dt][4 * a + 2], st.o[dt][4 * a + 3]};
            if (half == 0) {
                slot[ROWS * D + row] = st.m;
                slot[ROWS * D + ROWS + row] = l;
            }
        }
    } else if (rows.row >= 0) {
        const float inv = kv_inverse(st.m, l);
        char* out = p.out + rows.row * (D * ES);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                typedef __attribute__((ext_vector_type(4))) T four;
                four x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (T)(st.o[dt][a * 4 + e] * inv);
                *(four*)(out + (dt * 32 + a * 8 + half * 4) * ES) = x;
            }
        if (p.lse && half == 0) p.lse[rows.row] = kv_lse(st.m, l);
    }
}

// Joins the parts of a row tile: a thread per row and 4 channels at a time.
template <typename T, int D, bool LIST, int ROWS>
__global__ __launch_bounds__(256) void attn_tile_join_kernel(AttnArgs p, TileArgs ta) {
    const int head = blockIdx.x % p.n_kv, tile = blockIdx.x / p.n_kv;
    auto count = [&](int n, int) { return LIST ? (n + p.qb - 1) / p.qb * p.per_q : n * p.G <= p.few ? 0 : (n * p.G + ROWS - 1) / ROWS; };
    int s, j, first, n, len;
    if (!kv_find(p.b, tile, count, s, j, first, n, len)) return;
    int r0 = j * ROWS, r_end = n * p.G;
    if (LIST) {
        const int qt = j / p.per_q;
        r0 = qt * p.qb * p.G + (j - qt * p.per_q) * ROWS;
        r_end = min(n, (qt + 1) * p.qb) * p.G;
    }
    const int64_t stride = (int64_t)ROWS * (D + 2);
    const float* slots = ta.slots + (int64_t)(tile * p.n_kv + head) * ta.n_split * stride;
    const int rows = min(ROWS, r_end - r0);
    for (int x = blockIdx.y * 256 + threadIdx.x; x < rows * (D / 4); x += gridDim.y * 256) {
        const int row = x / (D / 4), c = x % (D / 4) * 4;
        float m = -INFINITY, l = 0.0f;
        kv_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int w = 0; w < ta.n_split; ++w) {
            const float* slot = slots + w * stride;
            const float mw = slot[ROWS * D + row], lw = slot[ROWS * D + ROWS + row];
            const kv_f32x4 ow = *(const kv_f32x4*)(slot + row * D + c);
            const float m2 = fmaxf(m, mw), fa = kv_factor(m, l, m2), fb = kv_factor(mw, lw, m2);
            m = m2;
            l = l * fa + lw * fb;
            o = o * fa + ow * fb;
        }
        const int t = (r0 + row) / p.G;
        const int64_t at = (int64_t)(first + t) * p.n_q + head * p.G + (r0 + row - t * p.G);
        const float inv = kv_inverse(m, l);
        typedef __attribute__((ext_vector_type(4))) T four;
        *(four*)(p.out + (at * D + c) * (int)sizeof(T)) = four{(T)(o[0] * inv), (T)(o[1] * inv), (T)(o[2] * inv), (T)(o[3] * inv)};
        if (p.lse && c == 0) p.lse[at] = kv_lse(m, l);
    }
}

// Wavefronts of the builds: 256 rows a workgroup; 128 where two wavefronts of a SIMD have too few registers.
template <typename T, int D> constexpr int kWaves = D * (int)sizeof(T) > 256 ? 4 : 8;
template <typename T, int D> constexpr int kRows = kWaves<T, D> * 32;

int rows_of(const s3_kv_cache* c) { return c->d_head * (c->dtype == S3_BF16 ? 2 : 4) > 256 ? 128 : 256; }

template <typename T, int D, bool LIST>
int launch(const AttnArgs& p, const TileArgs& ta, hipStream_t st) {
    constexpr int W = kWaves<T, D>, ROWS = kRows<T, D>;
    constexpr int bytes = 4 * kTokens<T, D> * D * (int)sizeof(T) + kBatchRuns * 16 + kBatchRuns * 16 / kTokens<T, D> * 8 + 8;
    static S3LdsOnce once;
    if (int rc = s3_allow_lds(once, (const void*)attn_tile_kernel<T, D, LIST, W>, bytes)) return rc;
    const int64_t units = (int64_t)ta.tiles * p.n_kv;
    hipLaunchKernelGGL((attn_tile_kernel<T, D, LIST, W>), dim3((unsigned)units, ta.n_split), dim3(W * 64), bytes, st, p, ta);
    S3_HIP(hipGetLastError());
    if (ta.n_split > 1) {
        hipLaunchKernelGGL((attn_tile_join_kernel<T, D, LIST, ROWS>), dim3((unsigned)units, units < 64 ? 32 : 8), dim3(256), 0, st, p, ta);
        S3_HIP(hipGetLastError());
    }
    return S3_OK;
}

}  // namespace

int s3_attn_tile_rows(const s3_kv_cache* c) { return rows_of(c); }

// Into how many parts the tokens of a row tile are cut.  One workgroup fills a compute unit, so units tiles * heads take
// ceil(units / 256) turns of all their steps; parts make the last turn fuller, at the price of writing fp32 sums and joining them.
// In us, with the rates that the kernel reaches on a compute unit: 3.8 TFLOP/s in bf16 and 0.45 in fp32, 6 us for the joining
// kernel, a part's sums written and read at 20 GB/s, and 4 us for its beginning.
// Ragged: the tiles are of several sequences whose lengths the host does not know, and those that see little count for nothing.  The cost is then
// summed over five guesses: all tiles see the most, 7/8, 3/4, 5/8 or half of them do.  us with the parts for equal lengths / with these: 217 tokens at 3519 and
// 102066, 28 heads over 4: 565 / 464; three times 300 at 2000, 20000 and 50000 with d_head 256: 1387 / 935; 500 at 3000 and 30000 in fp32: 1018 / 723; 2048 at
// 2048 beside eight times 30 at 131072: 1288 / 1018; but four times 1024 at 16384, which are equal: 939 / 1030.
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens, bool ragged) {
    const bool bf = c->dtype == S3_BF16;
    const int kt = c->d_head * (bf ? 2 : 4) > 512 ? 32 : 64;
    const int64_t steps = (tokens + kt - 1) / kt;
    const double step = 4.0 * rows_of(c) * kt * c->d_head / (bf ? 3.8e6 : 0.45e6), sums = rows_of(c) * (c->d_head + 2) * 4 / 10e3 + 4.0;
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= 64 && n <= steps; ++n) {
        int64_t turns = 0;
        for (int eighths = ragged ? 4 : 8; eighths <= 8; ++eighths) turns += (units * eighths / 8 * n + 255) / 256;
        const double cost = (double)turns * ((double)((steps + n - 1) / n) * step + (n > 1 ? sums : 0.0)) + (n > 1 ? 6.0 : 0.0) * (ragged ? 5 : 1);
        if (cost < least * 0.97) {
            least = cost;
            best = n;
        }
        if (units * n >= 2048) break;
    }
    return best;
}

size_t s3_attn_tile_workspace(const s3_kv_cache* c, int64_t units, int n_split) {
    return n_split > 1 ? s3_align((size_t)units * n_split * rows_of(c) * (c->d_head + 2) * 4) : 0;
}

int s3_attn_tile(const s3_kv_cache* c, const AttnArgs& p, int64_t tiles, int n_split, void* ws, hipStream_t st) {
    const TileArgs ta{(float*)ws, n_split, (int)tiles};
#define S3_TILE(T, D) (p.sel ? launch<T, D, true>(p, ta, st) : launch<T, D, false>(p, ta, st))
    if (c->dtype == S3_BF16) return c->d_head == 64 ? S3_TILE(__bf16, 64) : c->d_head == 128 ? S3_TILE(__bf16, 128) : S3_TILE(__bf16, 256);
    return c->d_head == 64 ? S3_TILE(float, 64) : c->d_head == 128 ? S3_TILE(float, 128) : S3_TILE(float, 256);
#undef S3_TILE
}
