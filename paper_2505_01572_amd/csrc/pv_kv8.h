// The 8-bit key/value cache: layout, where a row's tokens live, conversions.  Shared by the kernels that write it, read it back and attend to it.
//
// Codes are e4m3 (four significant bits, steps of 2^-9 below 2^-6, largest 448, 0x7F and 0xFF: NaN, no infinity); a block of 16 tokens of a
// head has one power-of-two scale for its keys and one for its values: a byte b stands for 2^(b - 127), from 1 to 253
// (in a block that nobody wrote, 0 is taken for 1 and 254 and 255 for 253, so that a scale and its inverse are numbers).  A power of two, because a floating code then
// stands for the same number under any scale that does not push it below 2^-6 of it: a block can be filled token by token, its scale raised when a larger token comes, and
// holds (but for its smallest numbers, under 1/14336 of its largest) what it would if all its tokens had come at once.
// Inside a block of 16 tokens (the pages are multiples of it) a lane's 16 bytes are an MFMA operand's codes:
//   K  [hd/16][token][16 features]                   lane (token, piece % 4) of two products over 32 features
//   V  [hd/64][token/4][feature%16][feature/16%4][token%4]    lane (feature % 16, token / 4) of four tiles of 16 features
#pragma once
#include "pv_matrix_common.h"

#define KV8_MIN_BYTE 27                     // smallest scale 2^-100: every code times its scale is a normal bf16

struct kv8_pool {
    uint8_t *codes, *scales;
    int n_pages, n_heads, page_shift;       // page_shift: log2 of the tokens a page
};

// The sequences of a call: tables on the device (a caller's batch), or a cache's own state (a step of the model).
struct kv8_seqs {
    const int32_t *row_start, *prefix_len, *page_table;
    int n_seq, n_rows, table_pages;
    const pv_dev_state *st;                 // a step: its sequences' states, pools and page tables; n_rows = its rows, table_pages the cache's own
    int batched, layer;                     // several sequences in it
    int first;                              // position of row 0 (-1: the sequence's length)
    size_t scales_off;                      // where a cache's scales lie behind its codes (all caches of a batch have as many pages)
};

// One sequence of it
struct kv8_seq {
    kv8_pool pool;
    const int32_t *table;
    int table_pages, len, row0, rows;       // rows: 0 if there is none such
};

// A pointer that came out of memory is one to global memory: loads through it are then no flat ones, for which every wait for LDS and for scalar loads would wait too
// (two prompts of 2048 rows 540 -> 509 us)
template <typename T> __device__ inline T *kv8_global(T *p) { return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p; }

template <int HD> __device__ inline size_t kv8_block(const kv8_pool &p, int page, int head, int which, int sub)
{
    return (((size_t)page * p.n_heads + head) * 2 + which) * ((size_t)HD << p.page_shift) + (size_t)sub * (16 * HD);
}
__device__ inline size_t kv8_scale(const kv8_pool &p, int page, int head, int which, int sub)
{
    return (((((size_t)page * p.n_heads + head) << (p.page_shift - 4)) + sub) << 1) + which;
}

// Sequence s of the call (in another layer than the call's)
template <int HD> __device__ inline kv8_seq kv8_seq_in(const kv8_seqs &q, const kv8_pool &own, int s, int layer)
{
    kv8_seq r;
    r.pool = own;
    if (q.st != nullptr) {
        r.table = q.page_table; r.table_pages = q.table_pages; r.row0 = 0; r.rows = q.n_rows;
        const pv_dev_state *st = q.st;
        char *base = (char *)own.codes;
        if (q.batched) {
            const pv_seq_ref &sq = q.st->blk.seq[s];
            st = kv8_global(sq.st); r.table = kv8_global(sq.page_table); r.table_pages = sq.n_pages; r.row0 = sq.row0; r.rows = sq.gamma; base = kv8_global((char *)sq.pool);
        }
        r.len = q.first >= 0 ? q.first : st->len;
        const size_t page_codes = ((size_t)(2 * HD) << own.page_shift) * own.n_heads, page_scales = ((size_t)2 << (own.page_shift - 4)) * own.n_heads;
        r.pool.codes = (uint8_t *)base + (size_t)layer * own.n_pages * page_codes;
        r.pool.scales = (uint8_t *)base + q.scales_off + (size_t)layer * own.n_pages * page_scales;
        return r;
    }
    r.table = q.page_table + (size_t)s * q.table_pages; r.table_pages = q.table_pages;
    r.row0 = q.row_start[s];
    r.rows = min(max(q.row_start[s + 1], 0), q.n_rows) - max(r.row0, 0);      // (no difference that wraps, whatever the table holds)
    r.len = q.prefix_len[s];
    if (r.row0 < 0 || r.rows < 0 || r.len < 0) r.rows = 0;
    return r;
}

template <int HD> __device__ inline kv8_seq kv8_seq_at(const kv8_seqs &q, const kv8_pool &own, int s) { return kv8_seq_in<HD>(q, own, s, q.layer); }

// The sequence that a row belongs to, -1: none (the row lies behind the last one).  Whole waves call.
__device__ inline int kv8_seq_of_row(const kv8_seqs &q, int row)
{
    if (q.st != nullptr) {
        if (!q.batched) return row < q.n_rows ? 0 : -1;
        int s = 0;
        for (int k = 1; k < q.st->blk.n_seq; ++k) if (row >= q.st->blk.seq[k].row0) s = k;
        return s;
    }
    const int lane = threadIdx.x & 63;
    int s = 0;
    for (int k = 0; k < q.n_seq; k += 64) {
        const int end = k + lane < q.n_seq ? q.row_start[k + lane + 1] : 0x7fffffff;
        s += __popcll(__ballot(end <= row));
    }
    return s < q.n_seq ? s : -1;
}

// The physical page of a sequence's logical one; -1: behind the table, or not a page of the pool
__device__ inline int kv8_page(const kv8_seq &s, int logical)
{
    if (logical < 0 || logical >= s.table_pages) return -1;
    const int p = s.table[logical];
    return p >= 0 && p < s.pool.n_pages ? p : -1;
}

// The same for a whole wave in two parts, so that the load is on its way long before its use: an entry of a table of at least one page, by a scalar load (which does not wait for the vector loads
// before it; behind the table's end: the last one), and whether it is a page
__device__ inline int kv8_entry(const kv8_seq &s, int logical)
{
    typedef const __attribute__((address_space(4))) int32_t *table;
    const uint32_t l = __builtin_amdgcn_readfirstlane(min((uint32_t)logical, (uint32_t)s.table_pages - 1));
    return ((table)(uintptr_t)uniform_ptr(s.table))[l];
}
__device__ inline bool kv8_is_page(const kv8_seq &s, int entry) { return (uint32_t)entry < (uint32_t)s.pool.n_pages; }

__device__ inline float kv8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // -127 < e < 128

__device__ inline int kv8_byte(int b) { return min(max(b, 1), 253); }

// The scale's byte for numbers of at most this magnitude: the smallest power of two that leaves no code above 448 = 1.75 * 2^8
__device__ inline int kv8_need(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(b, KV8_MIN_BYTE);
}

// Four numbers as codes (to nearest, ties to the even code), each times f.  |x * f| <= 448, or the number is not finite: those have no code but NaN.
__device__ inline uint32_t kv8_code4(float a, float b, float c, float d, float f)
{
    uint32_t v = 0;
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a * f, b * f, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c * f, d * f, v, true);
    return v;
}

typedef __attribute__((ext_vector_type(2))) float kv8_f2;
__device__ inline void kv8_value4(uint32_t c, float f, float v[4])
{
    const kv8_f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    v[0] = a.x * f; v[1] = a.y * f; v[2] = b.x * f; v[3] = b.y * f;
}

// Codes under another scale: f = old scale / new scale
__device__ inline uint32_t kv8_recode(uint32_t c, float f)
{
    float v[4];
    kv8_value4(c, f, v);
    return kv8_code4(v[0], v[1], v[2], v[3], 1.f);
}

// 16 consecutive numbers of a row in 32 bits, and back
template <typename T> struct kv8_el;
template <> struct kv8_el<float> {
    static __device__ inline void load(const void *p, float v[16])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float4 a = ((const float4 *)p)[i]; v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w; }
    }
    static __device__ inline void store(void *p, const float v[16])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) ((float4 *)p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
};
template <> struct kv8_el<__bf16> {
    static __device__ inline void load(const void *p, float v[16])
    {
        const uint4 a = ((const uint4 *)p)[0], b = ((const uint4 *)p)[1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ inline void store(void *p, const float v[16])
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        ((uint4 *)p)[0] = make_uint4(w[0], w[1], w[2], w[3]); ((uint4 *)p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
template <> struct kv8_el<_Float16> {
    static __device__ inline void load(const void *p, float v[16])
    {
        const uint4 a = ((const uint4 *)p)[0], b = ((const uint4 *)p)[1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { const f16x2 h = __builtin_bit_cast(f16x2, w[i]); v[2 * i] = (float)h.x; v[2 * i + 1] = (float)h.y; }
    }
    static __device__ inline void store(void *p, const float v[16])
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { const f16x2 h = {(_Float16)v[2 * i], (_Float16)v[2 * i + 1]}; w[i] = __builtin_bit_cast(uint32_t, h); }
        ((uint4 *)p)[0] = make_uint4(w[0], w[1], w[2], w[3]); ((uint4 *)p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};

// ---- host side ----
int pv_kv8_check_pool(const pv_kv8_pool *p);
int pv_kv8_check_seqs(const pv_kv8_seqs *q);
int pv_kv8_check_rows(const char *what, const void *p, int64_t row_stride, int64_t head_stride, int dtype);   // rows of heads in memory: addresses that 16-byte accesses take
kv8_pool pv_kv8_pool_args(const pv_kv8_pool *p);
kv8_seqs pv_kv8_seqs_args(const pv_kv8_seqs *q);
kv8_seqs pv_kv8_step_seqs(const pv_cache *c, int layer, int rows, int first, kv8_pool *pool);      // of a cache's own step: rows from position `first` on, -1: behind the committed tokens
