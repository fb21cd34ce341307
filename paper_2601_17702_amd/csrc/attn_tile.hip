// Attention of many rows: chunks of new tokens (and tiles of listed blocks) with more than 32 rows per key/value head.
//
// The two products bound it.  A workgroup has kWaves wavefronts of RS * 32 rows each, the rows of a head's G query heads token by
// token, and walks over the tokens that some row sees, KT at a time: keys and values come through registers into one of two LDS
// buffers while the other is worked on, in the layout that they have in the cache, which is the one in which every operand read
// is 16 bytes a lane from neighbouring places (no bank conflicts, no transposition).
#include "attn_launch.h"

namespace {

constexpr int kBatchRuns = 1024;       // runs of 16 tokens whose pages are looked up at a time

template <typename T, int D> constexpr int kTokens = D * (int)sizeof(T) > 512 ? 32 : 64;     // tokens of a buffer

struct TileArgs {
    float* slots;             // partial sums where n_split > 1
    int n_split, tiles;       // row tiles that there can be
};

template <typename T, int D, bool LIST, int RS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 4) void attn_tile_kernel(AttnArgs p, TileArgs ta) {
    constexpr int E = KvElem<T>::E, NW = 16 / E, QS = kQSteps<D, T>, ES = (int)sizeof(T), KT = kTokens<T, D>, NS = KT / 32;
    constexpr int THREADS = WAVES * 64, ROWS = WAVES * RS * 32;
    constexpr int PIECES = KT * D / E, LOADS = PIECES / THREADS;       // 16-byte pieces of a buffer's keys (and of its values)
    static_assert(PIECES % THREADS == 0, "every thread has as many pieces");
    typedef typename KvElem<T>::vec vec;
    extern __shared__ char lds[];
    char* buf = lds;                                                  // [2][keys | values][PIECES * 16]
    int2* runs = (int2*)(lds + 4 * PIECES * 16);                      // [kBatchRuns]: position of 16 tokens (2^30: none), page
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int logp = p.b.log_page, P = 1 << logp;
    const int64_t page_bytes = (int64_t)P * D * ES;

    // longest first: later row tiles see more
    const int head = blockIdx.x % p.n_kv;
    const int tile = ta.tiles - 1 - blockIdx.x / p.n_kv;
    auto count = [&](int q) {
        int first, n, len;
        kv_seq(p.b, q, first, n, len);
        return LIST ? (n + p.qb - 1) / p.qb * p.per_q : p.few && n * p.G <= 32 ? 0 : (n * p.G + ROWS - 1) / ROWS;
    };
    int s, j;
    if (!kv_find(p.b.n_seq, tile, count, s, j)) return;
    int first, n, len;
    kv_seq(p.b, s, first, n, len);
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

    const int rw = r0 + wave * (RS * 32);                             // this wavefront's first row
    const int pos0 = len - n + rw / p.G;                              // its position, and the last row's
    const int pos1 = rw < r_end ? len - n + (min(rw + RS * 32, r_end) - 1) / p.G : -1;
    AttnRows<T, D> rows[RS];
    AttnState<T, D> st[RS];
#pragma unroll
    for (int r = 0; r < RS; ++r) {
        rows[r].load(p, head, first, n, len, rw + r * 32 + col, r_end);
        st[r].clear();
    }

    vec stage[2 * LOADS];
    auto fetch = [&](int t) {                                         // step t of the batch: into registers
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int x = tid + i * THREADS, g = x / KT, tok = x % KT;
            const int2 r = runs[t * (KT / 16) + tok / 16];
            const char* src = p.k + ((int64_t)max(r.y, 0) * p.n_kv + head) * page_bytes + (g * P + (r.x & (P - 1)) + (tok & 15)) * 16;
            stage[i] = *(const vec*)src;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int x = tid + i * THREADS, g = x / D, c = x % D;
            const int2 r = runs[t * (KT / 16) + g * E / 16];
            const char* src = p.v + ((int64_t)max(r.y, 0) * p.n_kv + head) * page_bytes + (((r.x & (P - 1)) + g * E % 16) / E * D + c) * 16;
            // values past the end are anything: they must not meet a weight of zero as infinities
            stage[LOADS + i] = *(const vec*)src;
            if (r.x + 16 > hi) stage[LOADS + i] = kv_first(stage[LOADS + i], hi - r.x - g * E % 16);
        }
    };
    auto store = [&](int b) {
        char* dst = buf + b * (2 * PIECES * 16) + tid * 16;
#pragma unroll
        for (int i = 0; i < 2 * LOADS; ++i) *(vec*)(dst + i * THREADS * 16) = stage[i];
    };

    constexpr int kBatch = kBatchRuns / (KT / 16);                    // steps whose pages are known at a time
    for (int tb = t0; tb < t1; tb += kBatch) {
        const int nb = min(kBatch, t1 - tb);
        __syncthreads();
        for (int i = tid; i < nb * (KT / 16); i += THREADS) {
            int pos = 1 << 30, page = -1;
            if (LIST) {
                const int x = tb * (KT / 16) + i;
                const int blk = x < n_list ? list[x >> (logp - 4)] : -1;
                if (blk >= 0 && blk < p.b.max_pages) pos = (blk << logp) + (x & (P / 16 - 1)) * 16;
            } else {
                pos = lo + tb * KT + i * 16;
            }
            if (pos < hi) page = kv_page(p.b, s, pos >> logp);
            if (page < 0) pos = 1 << 30;
            runs[i] = int2{pos, page};
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
            // the tokens' positions, 16 at a time: the same in every lane
            int pos[KT / 16], least = 1 << 30, most = 0;
#pragma unroll
            for (int x = 0; x < KT / 16; ++x) {
                pos[x] = __builtin_amdgcn_readfirstlane(runs[t * (KT / 16) + x].x);
                least = min(least, pos[x]);
                most = max(most, pos[x] + 15);
            }
            if (least <= pos1) {                                      // some row of the wavefront sees some token
                const bool masked = most > pos0 || most >= hi || (p.window && least <= pos1 - p.window);
                kv_f32x16 sc[RS][NS];
#pragma unroll
                for (int x = 0; x < NS; ++x) {
#pragma unroll
                    for (int r = 0; r < RS; ++r)
#pragma unroll
                        for (int i = 0; i < 16; ++i) sc[r][x][i] = 0.0f;
#pragma unroll
                    for (int q = 0; q < QS; ++q) {
                        const vec kf = *(const vec*)(kb + ((2 * q + half) * KT + x * 32 + kv_token<T>(col)) * 16);
#pragma unroll
                        for (int r = 0; r < RS; ++r) sc[r][x] = kv_mma(kf, rows[r].q[q], sc[r][x]);
                    }
                }
                bool odd = false;
                if (masked) {
#pragma unroll
                    for (int r = 0; r < RS; ++r) {
                        const AttnSight sight(rows[r].pos, hi, p.window);
#pragma unroll
                        for (int x = 0; x < NS; ++x)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int tk = x * 32 + 2 * E * (i / E) + E * half + i % E;
                                sc[r][x][i] = sight.sees(pos[(x * 32 + 2 * E * (i / E)) / 16] + (tk & 15)) ? sc[r][x][i] : -INFINITY;
                            }
                    }
                    unsigned big = 0;
                    for (int i = lane; i < PIECES; i += 64) big = kv_magnitude(*(const vec*)(vb + i * 16), big);
                    odd = __ballot(big >= 0x7f800000u) != 0;
                }
                vec w[RS][NS * NW];
#pragma unroll
                for (int r = 0; r < RS; ++r) st[r].softmax(sc[r], p.sl, w[r]);
#pragma unroll
                for (int x = 0; x < NS; ++x)
#pragma unroll
                    for (int y = 0; y < NW; ++y)
#pragma unroll
                        for (int dt = 0; dt < D / 32; ++dt) {
                            vec vf = *(const vec*)(vb + ((x * (32 / E) + 2 * y + half) * D + dt * 32 + col) * 16);
                            if (odd) vf = kv_finite(vf);
#pragma unroll
                            for (int r = 0; r < RS; ++r) st[r].o[dt] = kv_mma(vf, w[r][x * NW + y], st[r].o[dt]);
                        }
                if (odd)
#pragma unroll 1
                    for (int tk = 0; tk < KT; ++tk) {
                        const int at = runs[t * (KT / 16) + tk / 16].x + (tk & 15);
                        const char* v = vb + tk / E * (D * 16) + tk % E * ES;
#pragma unroll
                        for (int r = 0; r < RS; ++r)
                            st[r].add_nonfinite(AttnSight(rows[r].pos, hi, p.window).sees(at), [&](int c) { return (float)*(const T*)(v + c * 16); });
                    }
            }
            if (more) store((t + 1) & 1);
            __syncthreads();
        }
    }

#pragma unroll
    for (int r = 0; r < RS; ++r) {
        const float l = kv_pair_sum(st[r].l);
        const int row = wave * (RS * 32) + r * 32 + col;
        if (ta.n_split > 1) {
            float* slot = ta.slots + ((int64_t)(tile * p.n_kv + head) * ta.n_split + split) * ((int64_t)ROWS * (D + 2));
            if (r0 + row < r_end) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int a = 0; a < 4; ++a)
                        *(kv_f32x4*)(slot + row * D + dt * 32 + a * 8 + half * 4) =
                            kv_f32x4{st[r].o[dt][4 * a], st[r].o[dt][4 * a + 1], st[r].o[dt][4 * a + 2], st[r].o[dt][4 * a + 3]};
                if (half == 0) {
                    slot[ROWS * D + row] = st[r].m;
                    slot[ROWS * D + ROWS + row] = l;
                }
            }
        } else if (rows[r].row >= 0) {
            const float inv = kv_inverse(l);
            char* out = p.out + rows[r].row * (D * ES);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    typedef __attribute__((ext_vector_type(4))) T four;
                    four x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = (T)(st[r].o[dt][a * 4 + e] * inv);
                    *(four*)(out + (dt * 32 + a * 8 + half * 4) * ES) = x;
                }
            if (p.lse && half == 0) p.lse[rows[r].row] = kv_lse(st[r].m, l);
        }
    }
}

// Joins the splits of a row tile: a thread per row and 4 channels.
template <typename T, int D, bool LIST, int ROWS>
__global__ __launch_bounds__(256) void attn_tile_join_kernel(AttnArgs p, TileArgs ta) {
    const int head = blockIdx.x % p.n_kv, tile = blockIdx.x / p.n_kv;
    auto count = [&](int q) {
        int first, n, len;
        kv_seq(p.b, q, first, n, len);
        return LIST ? (n + p.qb - 1) / p.qb * p.per_q : p.few && n * p.G <= 32 ? 0 : (n * p.G + ROWS - 1) / ROWS;
    };
    int s, j;
    if (!kv_find(p.b.n_seq, tile, count, s, j)) return;
    int first, n, len;
    kv_seq(p.b, s, first, n, len);
    int r0 = j * ROWS, r_end = n * p.G;
    if (LIST) {
        const int qt = j / p.per_q;
        r0 = qt * p.qb * p.G + (j - qt * p.per_q) * ROWS;
        r_end = min(n, (qt + 1) * p.qb) * p.G;
    }
    const int64_t stride = (int64_t)ROWS * (D + 2);
    const float* slots = ta.slots + (int64_t)(tile * p.n_kv + head) * ta.n_split * stride;
    const int x = blockIdx.y * 256 + threadIdx.x, row = x / (D / 4), c = x % (D / 4) * 4;
    if (row >= ROWS || r0 + row >= r_end) return;
    float m = -INFINITY, l = 0.0f;
    kv_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int w = 0; w < ta.n_split; ++w) m = fmaxf(m, slots[w * stride + ROWS * D + row]);
    for (int w = 0; w < ta.n_split; ++w) {
        const float mw = slots[w * stride + ROWS * D + row], lw = slots[w * stride + ROWS * D + ROWS + row];
        const float f = mw == -INFINITY && lw == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(mw == m ? 0.0f : mw - m);
        l += lw * f;
        o += *(const kv_f32x4*)(slots + w * stride + row * D + c) * f;
    }
    const int t = (r0 + row) / p.G;
    const int64_t at = (int64_t)(first + t) * p.n_q + head * p.G + (r0 + row - t * p.G);
    const float inv = kv_inverse(l);
    typedef __attribute__((ext_vector_type(4))) T four;
    *(four*)(p.out + (at * D + c) * (int)sizeof(T)) = four{(T)(o[0] * inv), (T)(o[1] * inv), (T)(o[2] * inv), (T)(o[3] * inv)};
    if (p.lse && c == 0) p.lse[at] = kv_lse(m, l);
}

// Wavefronts and row sets of the builds: 256 rows a workgroup; 128 where the operands of 256 do not fit the registers.
template <typename T, int D> constexpr int kSets = 1;
template <typename T, int D> constexpr int kWaves = D * (int)sizeof(T) > 256 ? 4 : 8;
template <typename T, int D> constexpr int kRows = kSets<T, D> * kWaves<T, D> * 32;

int rows_of(const s3_kv_cache* c) { return c->d_head * (c->dtype == S3_BF16 ? 2 : 4) > 256 ? 128 : 256; }

template <typename T, int D, bool LIST>
int launch(const AttnArgs& p, const TileArgs& ta, hipStream_t st) {
    constexpr int RS = kSets<T, D>, W = kWaves<T, D>, ROWS = kRows<T, D>;
    constexpr int bytes = 4 * kTokens<T, D> * D * (int)sizeof(T) + kBatchRuns * 8;
    static S3LdsOnce once;
    if (int rc = s3_allow_lds(once, (const void*)attn_tile_kernel<T, D, LIST, RS, W>, bytes)) return rc;
    const int64_t units = (int64_t)ta.tiles * p.n_kv;
    if (units >= (int64_t)1 << 22) return s3_fail(S3_EINVAL, "attention: too many tokens in one call");
    hipLaunchKernelGGL((attn_tile_kernel<T, D, LIST, RS, W>), dim3((unsigned)units, ta.n_split), dim3(W * 64), bytes, st, p, ta);
    S3_HIP(hipGetLastError());
    if (ta.n_split > 1) {
        hipLaunchKernelGGL((attn_tile_join_kernel<T, D, LIST, ROWS>), dim3((unsigned)units, ROWS * (D / 4) / 256), dim3(256), 0, st, p, ta);
        S3_HIP(hipGetLastError());
    }
    return S3_OK;
}

}  // namespace

int s3_attn_tile_rows(const s3_kv_cache* c) { return rows_of(c); }

// Into how many parts the tokens of a row tile are cut.  One workgroup fills a compute unit, so units tiles * heads take
// ceil(units / 256) turns of all their steps; parts make the last turn fuller, at the price of writing fp32 sums and joining them.
// In us, with the rates that the kernel reaches on a compute unit: 3.8 TFLOP/s in bf16 and 0.45 in fp32, 6 us for the joining
// kernel and a tile's sums at 20 GB/s.
int s3_attn_tile_split(const s3_kv_cache* c, int64_t units, int64_t tokens) {
    const bool bf = c->dtype == S3_BF16;
    const int kt = c->d_head * (bf ? 2 : 4) > 512 ? 32 : 64;
    const int64_t steps = (tokens + kt - 1) / kt;
    const double step = 4.0 * rows_of(c) * kt * c->d_head / (bf ? 3.8e6 : 0.45e6), sums = rows_of(c) * (c->d_head + 2) * 4 / 20e3;
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= 64 && n <= steps; ++n) {
        const double turns = (double)((units * n + 255) / 256);
        const double cost = turns * ((double)((steps + n - 1) / n) * step + (n > 1 ? sums : 0.0)) + (n > 1 ? 6.0 : 0.0);
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
    if (tiles * p.n_kv >= (int64_t)1 << 22) return s3_fail(S3_EINVAL, "attention: too many tokens in one call");
    const TileArgs ta{(float*)ws, n_split, (int)tiles};
#define S3_TILE(T, D) (p.sel ? launch<T, D, true>(p, ta, st) : launch<T, D, false>(p, ta, st))
    if (c->dtype == S3_BF16) return c->d_head == 64 ? S3_TILE(__bf16, 64) : c->d_head == 128 ? S3_TILE(__bf16, 128) : S3_TILE(__bf16, 256);
    return c->d_head == 64 ? S3_TILE(float, 64) : c->d_head == 128 ? S3_TILE(float, 128) : S3_TILE(float, 256);
#undef S3_TILE
}
