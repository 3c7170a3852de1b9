// The 16-bit key/value cache on a caller's tensors: layout, where a row's tokens live.  Shared by the kernels that write it, move its tokens and attend to it.
//
// Inside a block of 16 tokens of a head a lane's 16 bytes are what an MFMA over 32 features, or over four tokens of two groups, takes from it:
//   K  [hd/8][token][8 features]                          lane (token, piece % 4)
//   V  [hd/32][token/4][feature%16][feature/16%2][token%4]      lane (feature % 16, token / 4) of two tiles of 16 features
#pragma once
#include "pv_matrix_common.h"

struct kv16_pool {
    char *pages;                            // 16-bit numbers
    int n_pages, n_heads, page_shift;       // page_shift: log2 of the tokens a page
};
struct kv16_seqs {                          // a call's sequences: tables on the device
    const int32_t *row_start, *prefix_len, *page_table;
    int n_seq, n_rows, table_pages;
};
struct kv16_seq {                           // one of them
    const int32_t *table;
    int table_pages, len, row0, rows;       // rows: 0 if there is none such
};

// Bytes from the pool's beginning to a head's keys (which = 0) or values (1) of a block of 16 tokens
template <int HD> __device__ inline size_t kv16_block(const kv16_pool &p, int page, int head, int which, int sub)
{
    return ((((size_t)page * p.n_heads + head) * 2 + which) * ((size_t)HD << p.page_shift) + (size_t)sub * (16 * HD)) * 2;
}
// ... and from there to feature e of token t
__device__ inline int kv16_k_at(int t, int e) { return ((e >> 3) * 128 + t * 8 + (e & 7)) * 2; }
__device__ inline int kv16_v_at(int t, int e) { return ((e >> 5) * 512 + (t >> 2) * 128 + (e & 15) * 8 + ((e >> 4) & 1) * 4 + (t & 3)) * 2; }

__device__ inline kv16_seq kv16_seq_at(const kv16_seqs &q, int s)
{
    kv16_seq r;
    r.table = q.page_table + (size_t)s * q.table_pages; r.table_pages = q.table_pages;
    r.row0 = q.row_start[s];
    r.rows = min(max(q.row_start[s + 1], 0), q.n_rows) - max(r.row0, 0);      // (no difference that wraps, whatever the table holds)
    r.len = q.prefix_len[s];
    if (r.row0 < 0 || r.rows < 0 || r.len < 0) r.rows = 0;
    return r;
}

// The sequences that N rows belong to, n_seq: none (the row lies behind the last one).  Whole waves call.
template <int N> __device__ inline void kv16_seqs_of_rows(const int32_t *row_start, int n_seq, const int (&row)[N], int (&s)[N])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0;
    for (int k = 0; k < n_seq; k += 64) {
        const int end = k + lane < n_seq ? row_start[k + lane + 1] : 0x7fffffff;
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __popcll(__ballot(end <= row[i]));
    }
}

// The physical page of a sequence's logical one; -1: behind the table, or not a page of the pool
__device__ inline int kv16_page(const kv16_seq &s, int n_pages, int logical)
{
    if (logical < 0 || logical >= s.table_pages) return -1;
    const int p = s.table[logical];
    return p >= 0 && p < n_pages ? p : -1;
}

// Two numbers of a 16-bit type
typedef __attribute__((ext_vector_type(2))) _Float16 kv16_h2;
template <typename S> __device__ inline uint32_t kv16_two(float a, float b);
template <> __device__ inline uint32_t kv16_two<__bf16>(float a, float b) { return pack_bf16(a, b); }
template <> __device__ inline uint32_t kv16_two<_Float16>(float a, float b) { const kv16_h2 h = {(_Float16)a, (_Float16)b}; return __builtin_bit_cast(uint32_t, h); }

// ---- host side ----
int pv_kv16_check_pool(const pv_kv16_pool *p);
kv16_pool pv_kv16_pool_args(const pv_kv16_pool *p);
kv16_seqs pv_kv16_seqs_args(const pv_kv8_seqs *q);
int pv_kv8_check_seqs(const pv_kv8_seqs *q);
int pv_kv8_check_rows(const char *what, const void *p, int64_t row_stride, int64_t head_stride, int dtype);   // rows of heads in memory: addresses that 16-byte accesses take
