// Shared by the kernels around the paged key/value cache: layout, ragged batches, the 8 bit grid of the signatures.
#pragma once
#include "s3_common.h"

typedef __attribute__((ext_vector_type(8))) __bf16 kv_bf16x8;
typedef __attribute__((ext_vector_type(4))) float kv_f32x4;
typedef __attribute__((ext_vector_type(16))) float kv_f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned kv_u32x4;

// 16 bytes of a row: E elements.  Keys lie [page][head][d / E][slot][E], values [page][head][slot / E][d][E], so that 16 bytes
// are what a lane of a matrix instruction takes of its operand and neighbouring lanes take neighbouring pieces, in either product.
template <typename T> struct KvElem;
template <> struct KvElem<__bf16> {
    static constexpr int E = 8;
    typedef kv_bf16x8 vec;
};
template <> struct KvElem<float> {
    static constexpr int E = 4;
    typedef kv_f32x4 vec;
};

// The sequences of a call, as the kernels read them.  Lengths and page numbers come from device memory, so every use is held
// inside the arrays here: blocks to the table's width, tokens to n_tokens, pages to n_pages.
struct KvBatch {
    const int32_t* q_start;      // [n_seq + 1], or null: token s is sequence s's only one
    const int32_t* kv_len;
    const int32_t* table;        // [n_seq][table_stride]
    int n_seq, n_tokens, max_pages, n_pages, log_page;
    int64_t table_stride;
};

// Rows first .. first + n - 1 of the call are the new tokens of sequence s, whose length is len with them.
__device__ __forceinline__ void kv_seq(const KvBatch& b, int s, int& first, int& n, int& len) {
    first = s;
    n = 1;
    if (b.q_start) {
        first = b.q_start[s];
        n = b.q_start[s + 1] - first;
        if (first < 0 || first > b.n_tokens) n = 0;
        n = max(0, min(n, b.n_tokens - first));
    }
    len = max(0, min(b.kv_len[s], 1 << 30));
}
// Counts of lists summed over sequences: where starts descend the sum may be any number, and an index made of it must not wrap to below the
// array.  64 sequences have 2^30 lists at most.
__device__ __forceinline__ int kv_add_lists(int all, int more) { return min(all + more, 1 << 29); }
// Blocks that hold len tokens, as far as the table goes.
__device__ __forceinline__ int kv_blocks(const KvBatch& b, int len) {
    return min((len + (1 << b.log_page) - 1) >> b.log_page, b.max_pages);
}

// The page that holds block blk of sequence s, or -1.
__device__ __forceinline__ int kv_page(const KvBatch& b, int s, int blk) {
    if (blk < 0 || blk >= b.max_pages) return -1;
    const int p = b.table[s * b.table_stride + blk];
    return p >= 0 && p < b.n_pages ? p : -1;
}

// Item `item` of a list in which a sequence has count(n, len) entries: which sequence (and kv_seq's values of it), and which of its
// entries.  Run by a whole wavefront, 64 sequences at a time; false where the list is shorter.
template <typename F>
__device__ __forceinline__ bool kv_find(const KvBatch& b, int64_t item, F count, int& seq, int& local, int& first, int& n, int& len) {
    const int lane = threadIdx.x & 63;
    int64_t run = 0;
    for (int base = 0; base < b.n_seq; base += 64) {
        int f = 0, m = 0, l = 0, c = 0;
        if (base + lane < b.n_seq) {
            kv_seq(b, base + lane, f, m, l);
            c = count(m, l);
        }
        const int incl = s3_wave_incl_scan(c);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        if (item < run + total) {
            const int want = (int)(item - run);
            const int x = __builtin_ctzll(__ballot(incl > want));
            seq = base + x;
            local = want - (__builtin_amdgcn_readlane(incl, x) - __builtin_amdgcn_readlane(c, x));
            first = __builtin_amdgcn_readlane(f, x);
            n = __builtin_amdgcn_readlane(m, x);
            len = __builtin_amdgcn_readlane(l, x);
            return true;
        }
        run += total;
    }
    return false;
}

// 8 bit grid: a vector whose largest absolute value is m is rounded to whole multiples of 2^(floor(log2 m) - 6), at most 128 of
// them.  Returns that exponent; ok is false where the vector counts as zero (m outside [2^-40, 2^50), NaN and infinities too).
__device__ __forceinline__ int kv_grid_exp(unsigned max_abs_bits, bool& ok) {
    const int e = (int)(max_abs_bits >> 23) - 127;
    ok = e >= -40 && e < 50;
    return e - 6;
}
__device__ __forceinline__ float kv_grid(float x, int e) {      // multiples of 2^e: both scalings are exact
    return rintf(x * __uint_as_float((unsigned)(127 - e) << 23)) * __uint_as_float((unsigned)(127 + e) << 23);
}

// Checks shared by the entry points (host).
int s3_kv_check(const char* fn, const s3_kv_cache* c, const s3_kv_batch* b);
int s3_kv_check_rows(const char* fn, const char* what, const s3_kv_cache* c, const void* p, int64_t tok_stride, int64_t head_stride,
                     int heads);
static inline KvBatch s3_kv_batch_args(const s3_kv_cache* c, const s3_kv_batch* b) {
    return {b->q_start, b->kv_len, b->block_table, b->n_seq, b->n_tokens, b->max_pages, c->n_pages,
            s3_ceil_log2((unsigned)c->page_size), b->table_stride};
}
