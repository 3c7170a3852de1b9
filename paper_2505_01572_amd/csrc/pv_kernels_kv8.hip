// Writing the 8-bit key/value cache (quantising new tokens) and reading it back.
#include "pv_kv8.h"

struct kv8_append_args {
    kv8_pool pool;
    kv8_seqs seqs;
    const char *src[2];                     // keys, values
    int64_t row_bytes[2], head_bytes[2];    // from one row, from one head to the next
    int chunk;                              // rows a wave looks through
};

// Blocks of 16 tokens that rows [first, first + chunk) open: for each the first row in it, the sequence, how many tokens it holds already and how many
// come.  Rows in the middle of a block are left to the wave that has its first one.
template <int HD, typename F>
__device__ inline void kv8_each_block(const kv8_seqs &seqs, const kv8_pool &pool, int first, int chunk, F work)
{
    int i = first;
    const int end = min(first + chunk, seqs.n_rows);
    while (i < end) {
        const int s = __builtin_amdgcn_readfirstlane(kv8_seq_of_row(seqs, i));
        if (s < 0) return;
        const kv8_seq q = kv8_seq_at<HD>(seqs, pool, s);
        const int local = i - q.row0;
        if (local < 0 || local >= q.rows) { ++i; continue; }
        const int stop = min(end, q.row0 + q.rows);
        for (; i < stop;) {
            const int pos = (int)((uint32_t)q.len + (uint32_t)(i - q.row0)), off = pos & 15;       // (past 2^31: negative, of no page)
            if (off != 0 && i != q.row0) { i += 16 - off; continue; }
            const int n = min(16 - off, q.row0 + q.rows - i);
            work(q, i, pos, off, n);
            i += n;
        }
        i = min(i, max(stop, q.row0 + q.rows));
    }
}

// A wave writes n new tokens behind the `off` that a block of 16 holds; load(t, p, x): 16 numbers, piece p of the t-th new token.  Each new number is read once, its code written; of earlier tokens' codes
// it touches those of a block that needs a larger scale, and of V those that share a lane's 16 bytes with the new ones.  tile: LDS, a byte a number of the block.
template <int HD, typename LOAD>
__device__ inline void kv8_write_block(uint8_t *codes, uint8_t *scale, int which, int off, int n, uint32_t *tile, LOAD load)
{
    constexpr int NP = HD / 64, PR = HD / 16;                 // pieces of 16 numbers a lane; pieces a row
    const int lane = threadIdx.x & 63;
    const int old = off > 0 ? kv8_byte(*scale) : 0;
    float x[NP][16];
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const int piece = k * 64 + lane, t = piece / PR, p = piece % PR;
        if (t >= off && t < off + n) load(t - off, p, x[k]);
        else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[k][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) { const float m = fabsf(x[k][e]); if (m < INFINITY) amax = fmaxf(amax, m); }
    }
    amax = over_wave(amax, op_max);
    const int b = max(old, kv8_need(amax));
    const float f = kv8_pow2(127 - b);
    const bool raise = off > 0 && b != old;
    const float down = raise ? (old - b > -126 ? kv8_pow2(old - b) : 0.f) : 1.f;
    uint32_t c[NP][4];
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[k][i] = kv8_code4(x[k][4 * i], x[k][4 * i + 1], x[k][4 * i + 2], x[k][4 * i + 3], f);
    if (which == 0) {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int piece = k * 64 + lane, t = piece / PR, p = piece % PR;
            uint4 *at = (uint4 *)(codes + (p * 16 + t) * 16);
            if (t >= off && t < off + n) *at = make_uint4(c[k][0], c[k][1], c[k][2], c[k][3]);
            else if (t < off && raise) { const uint4 v = *at; *at = make_uint4(kv8_recode(v.x, down), kv8_recode(v.y, down), kv8_recode(v.z, down), kv8_recode(v.w, down)); }
        }
    } else {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int piece = k * 64 + lane, t = piece / PR, p = piece % PR;
#pragma unroll
            for (int i = 0; i < 4; ++i) tile[t * (HD / 4) + p * 4 + i] = c[k][i];
        }
        __syncthreads();
        const int g = lane >> 4, jl = lane & 15;
        uint32_t keep = 0, mine = 0;                           // bytes of a dword: earlier tokens', the new ones' (the rest is left as it was)
#pragma unroll
        for (int r = 0; r < 4; ++r) { const int t = 4 * g + r; if (t < off) keep |= 0xffu << (8 * r); else if (t < off + n) mine |= 0xffu << (8 * r); }
        const bool touch = mine != 0 || (raise && keep != 0);
#pragma unroll
        for (int h = 0; h < NP; ++h) {
            uint4 *at = (uint4 *)codes + h * 64 + lane;
            uint32_t v[4], o[4] = {0, 0, 0, 0};
            if (touch && mine != 0xffffffffu) { const uint4 w = *at; o[0] = w.x; o[1] = w.y; o[2] = w.z; o[3] = w.w; }
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                uint32_t w = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) w |= (uint32_t)((const uint8_t *)tile)[(4 * g + r) * HD + (4 * h + q4) * 16 + jl] << (8 * r);
                const uint32_t e = raise ? kv8_recode(o[q4], down) : o[q4];
                v[q4] = (w & mine) | (e & keep) | (o[q4] & ~(mine | keep));
            }
            if (touch) *at = make_uint4(v[0], v[1], v[2], v[3]);
        }
        __syncthreads();
    }
    if (lane == 0 && b != old) *scale = (uint8_t)b;
}

// One wave a block, head and kind (K or V); V's bytes change places through LDS.  Bound by the read of the new rows where they are many: four sequences of up to 4096 rows, eight heads of 128, bf16
// 20.7 us (82 MB at 4.0 TB/s; a copy moves 5.2), 21.0 with keys and values in one wave; else by the trips to the tables, the scale and the rows, one after the other: 4.0 us one row, 6.2 64 sequences
// of five.
template <int HD, typename T>
__global__ void __launch_bounds__(64)
k_kv8_append(const kv8_append_args a)
{
    __shared__ uint32_t tile[16 * HD / 4];                    // codes [token][feature]
    const int which = blockIdx.x & 1, head = blockIdx.x >> 1;
    const char *src = a.src[which] + (int64_t)head * a.head_bytes[which];
    kv8_each_block<HD>(a.seqs, a.pool, blockIdx.y * a.chunk, a.chunk, [&](const kv8_seq &q, int row, int pos, int off, int n) {
        const int page = kv8_page(q, pos >> q.pool.page_shift), sub = (pos & ((1 << q.pool.page_shift) - 1)) >> 4;
        if (page < 0) return;
        kv8_write_block<HD>(q.pool.codes + kv8_block<HD>(q.pool, page, head, which, sub), q.pool.scales + kv8_scale(q.pool, page, head, which, sub), which, off, n, tile,
                            [&](int t, int p, float *x) { kv8_el<T>::load(src + (int64_t)(row + t) * a.row_bytes[which] + p * 16 * sizeof(T), x); });
    });
}

// After a draft-tree step: the accepted path's tokens, in the slots of their row numbers, are read (values of at most four significant bits: exact in bf16) and written behind the prefix, as
// appending them would have.  A wave a layer, head and kind.
template <int HD>
__global__ void __launch_bounds__(64)
k_kv8_tree(const kv8_pool pool, const kv8_seqs seqs)
{
    __shared__ uint32_t tile[16 * HD / 4];
    __shared__ __align__(16) uint16_t rows[PV_MAX_ROWS][HD];
    const int lane = threadIdx.x, which = blockIdx.x & 1, head = blockIdx.x >> 1;
    const kv8_seq q = kv8_seq_in<HD>(seqs, pool, 0, blockIdx.y);
    const int n = min(seqs.st->accepted, PV_MAX_ROWS), len0 = q.len - n, shift = q.pool.page_shift;      // (the finishing kernel has added n already)
    bool moved = false;
    for (int d = 0; d < n; ++d) {
        const int from = seqs.st->path[d], pos = len0 + from, page = kv8_page(q, pos >> shift), sub = (pos & ((1 << shift) - 1)) >> 4, t = pos & 15;
        moved = moved || from != d;
        if (page < 0) return;
        const uint8_t *codes = q.pool.codes + kv8_block<HD>(q.pool, page, head, which, sub);
        const float f = kv8_pow2(kv8_byte(q.pool.scales[kv8_scale(q.pool, page, head, which, sub)]) - 127);
        for (int e = lane; e < HD; e += 64) {
            const int at = which ? (e / 64) * 1024 + (t / 4) * 256 + (e % 16) * 16 + (e / 16 % 4) * 4 + t % 4 : (e / 16) * 256 + t * 16 + e % 16;
            rows[d][e] = pv_f32_to_bf16(__builtin_amdgcn_cvt_f32_fp8((int)codes[at], 0) * f);
        }
    }
    if (!moved) return;
    __syncthreads();
    for (int d = 0; d < n;) {
        const int pos = len0 + d, off = pos & 15, m = min(16 - off, n - d), page = kv8_page(q, pos >> shift), sub = (pos & ((1 << shift) - 1)) >> 4;
        if (page >= 0)
            kv8_write_block<HD>(q.pool.codes + kv8_block<HD>(q.pool, page, head, which, sub), q.pool.scales + kv8_scale(q.pool, page, head, which, sub), which, off, m, tile,
                                [&](int t, int p, float *x) { kv8_el<__bf16>::load(&rows[d + t][p * 16], x); });
        d += m;
    }
}

struct kv8_read_args {
    kv8_pool pool;
    kv8_seqs seqs;
    char *dst[2];
    int64_t row_bytes[2], head_bytes[2];
    int chunk;
};

// The same walk the other way, a wave a block and head, keys and values asked for together: a token whose page is not one of the pool reads as zeros.  V's bytes change places through LDS.
// Eight sequences of up to 8192 tokens, eight heads of 128, bf16: 64.6 us with a wave each for keys and values and loads through the caches, 55.9 so (277 MB, 53.7 at a copy's rate)
template <int HD, typename T>
__global__ void __launch_bounds__(64)
k_kv8_read(const kv8_read_args a)
{
    constexpr int NP = HD / 64, PR = HD / 16;
    __shared__ uint32_t tile[16 * HD / 4];
    const int lane = threadIdx.x, head = blockIdx.x;
    kv8_each_block<HD>(a.seqs, a.pool, blockIdx.y * a.chunk, a.chunk, [&](const kv8_seq &q, int row, int pos, int off, int n) {
        const int page = kv8_page(q, pos >> q.pool.page_shift), sub = (pos & ((1 << q.pool.page_shift) - 1)) >> 4;
        uint4 c[2][NP];
        float f[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NP; ++k) c[0][k] = c[1][k] = make_uint4(0u, 0u, 0u, 0u);
        if (page >= 0) {
            const uint8_t *keys = q.pool.codes + kv8_block<HD>(q.pool, page, head, 0, sub), *values = q.pool.codes + kv8_block<HD>(q.pool, page, head, 1, sub);
            const uint32_t bytes = *(const uint16_t *)(q.pool.scales + kv8_scale(q.pool, page, head, 0, sub));
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const int piece = k * 64 + lane, t = piece / PR, p = piece % PR;
                c[0][k] = load_once((const uint4 *)(keys + (p * 16 + t) * 16)); c[1][k] = load_once((const uint4 *)values + k * 64 + lane);
            }
            f[0] = kv8_pow2(kv8_byte(bytes & 0xffu) - 127); f[1] = kv8_pow2(kv8_byte(bytes >> 8) - 127);
        }
        const int g = lane >> 4, jl = lane & 15;
#pragma unroll
        for (int h = 0; h < NP; ++h) {
            const uint32_t w[4] = {c[1][h].x, c[1][h].y, c[1][h].z, c[1][h].w};
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
                for (int r = 0; r < 4; ++r) ((uint8_t *)tile)[(4 * g + r) * HD + (4 * h + q4) * 16 + jl] = (uint8_t)(w[q4] >> (8 * r));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int piece = k * 64 + lane, t = piece / PR, p = piece % PR;
            c[1][k] = *(const uint4 *)&tile[t * (HD / 4) + p * 4];
            if (t < off || t >= off + n) continue;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float v[16];
                kv8_value4(c[w][k].x, f[w], v); kv8_value4(c[w][k].y, f[w], v + 4); kv8_value4(c[w][k].z, f[w], v + 8); kv8_value4(c[w][k].w, f[w], v + 12);
                kv8_el<T>::store(a.dst[w] + (int64_t)head * a.head_bytes[w] + (int64_t)(row + t - off) * a.row_bytes[w] + p * 16 * sizeof(T), v);
            }
        }
        __syncthreads();
    });
}

// ------------------------------- host side ----------------------------------------

static size_t dtype_size(int dtype) { return dtype == PV_F32 ? 4 : 2; }

int pv_kv8_check_pool(const pv_kv8_pool *p)
{
    if (!p || !p->codes || !p->scales) { pv_set_error("null pool"); return PV_EINVAL; }
    if (p->head_dim != 64 && p->head_dim != 128) { pv_set_error("8-bit cache: head_dim must be 64 or 128, got %d", p->head_dim); return PV_EINVAL; }
    if (p->n_pages < 1 || p->n_pages >= (1 << 26)) { pv_set_error("8-bit cache: n_pages %d outside [1, 2^26)", p->n_pages); return PV_ERANGE; }
    if (p->n_kv_heads < 1 || p->n_kv_heads > 16384) { pv_set_error("8-bit cache: n_kv_heads %d outside [1, 16384]", p->n_kv_heads); return PV_ERANGE; }
    if (p->page_tokens < 16 || p->page_tokens > 65536 || (p->page_tokens & (p->page_tokens - 1))) { pv_set_error("8-bit cache: page_tokens must be a power of two from 16 to 65536, got %d", p->page_tokens); return PV_EINVAL; }
    if ((int64_t)p->n_kv_heads * p->page_tokens * p->head_dim >= 1ll << 31) { pv_set_error("8-bit cache: a page of %d heads x %d tokens: 2^32 bytes of codes or more", p->n_kv_heads, p->page_tokens); return PV_ERANGE; }
    if (((uintptr_t)p->codes & 15) || ((uintptr_t)p->scales & 1)) { pv_set_error("8-bit cache: codes must be 16-byte and scales 2-byte aligned"); return PV_EINVAL; }
    return PV_OK;
}

int pv_kv8_check_seqs(const pv_kv8_seqs *q)
{
    if (!q) { pv_set_error("null sequences"); return PV_EINVAL; }
    if (q->n_seq < 0 || q->n_rows < 0 || q->table_pages < 0) { pv_set_error("negative n_seq, n_rows or table_pages"); return PV_ERANGE; }
    if (q->n_seq > (1 << 20) || q->n_rows > (1 << 24)) { pv_set_error("n_seq %d > 2^20 or n_rows %d > 2^24", q->n_seq, q->n_rows); return PV_ERANGE; }
    if (q->n_seq > 0 && (!q->row_start || !q->prefix_len || (!q->page_table && q->table_pages > 0))) { pv_set_error("null sequence table"); return PV_EINVAL; }
    return PV_OK;
}

// rows of heads in memory: addresses that 16-byte accesses take
int pv_kv8_check_rows(const char *what, const void *p, int64_t row_stride, int64_t head_stride, int dtype)
{
    if (!p) { pv_set_error("null %s", what); return PV_EINVAL; }
    if (dtype != PV_F32 && dtype != PV_BF16 && dtype != PV_F16) { pv_set_error("bad dtype %d", dtype); return PV_EINVAL; }
    const int64_t n = 16 / (int64_t)dtype_size(dtype);
    if (((uintptr_t)p & 15) || row_stride % n || head_stride % n) { pv_set_error("%s: address and strides must be multiples of 16 bytes", what); return PV_EINVAL; }
    if (row_stride < 0 || head_stride < 0) { pv_set_error("%s: negative stride", what); return PV_EINVAL; }
    return PV_OK;
}

kv8_pool pv_kv8_pool_args(const pv_kv8_pool *p)
{
    kv8_pool r = {(uint8_t *)p->codes, (uint8_t *)p->scales, p->n_pages, p->n_kv_heads, 0};
    while ((1 << r.page_shift) < p->page_tokens) ++r.page_shift;
    return r;
}

kv8_seqs pv_kv8_seqs_args(const pv_kv8_seqs *q)
{
    kv8_seqs r = {};
    r.row_start = q->row_start; r.prefix_len = q->prefix_len; r.page_table = q->page_table;
    r.n_seq = q->n_seq; r.n_rows = q->n_rows; r.table_pages = q->table_pages;
    return r;
}

// Rows a wave looks through: 16, which open one block of a long sequence; one where sequences have fewer rows and not too many waves come out (64 sequences of up to five rows 16.2 -> 6.3 us, in
// fours 8.8; a prompt of 16384 rows 20.8 us with 16, 75.8 with one)
static int walk(int n_seq, int rows, int heads, int *chunk, unsigned *grid_y)
{
    *chunk = rows < 16 * (int64_t)n_seq && (int64_t)rows * heads * 2 <= 65536 ? 1 : 16;
    *grid_y = (unsigned)((rows + *chunk - 1) / *chunk);
    while (*grid_y > 65535) { *chunk *= 2; *grid_y = (unsigned)((rows + *chunk - 1) / *chunk); }
    return PV_OK;
}

template <int HD>
static int launch_append(const kv8_append_args &a, int dtype, unsigned gy, hipStream_t s)
{
    const dim3 grid(2 * a.pool.n_heads, gy);
    if (dtype == PV_F32) k_kv8_append<HD, float><<<grid, 64, 0, s>>>(a);
    else if (dtype == PV_BF16) k_kv8_append<HD, __bf16><<<grid, 64, 0, s>>>(a);
    else k_kv8_append<HD, _Float16><<<grid, 64, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

extern "C" int pv_kv8_append(const pv_kv8_pool *pool, const pv_kv8_seqs *seqs, const void *k, int64_t k_row_stride, int64_t k_head_stride,
                             const void *v, int64_t v_row_stride, int64_t v_head_stride, int32_t dtype, void *hip_stream)
{
    int rc;
    if ((rc = pv_kv8_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (seqs->n_rows == 0 || seqs->n_seq == 0) return PV_OK;
    if ((rc = pv_kv8_check_rows("k", k, k_row_stride, k_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("v", v, v_row_stride, v_head_stride, dtype)) != PV_OK) return rc;
    kv8_append_args a = {};
    a.pool = pv_kv8_pool_args(pool); a.seqs = pv_kv8_seqs_args(seqs);
    const int64_t e = (int64_t)dtype_size(dtype);
    a.src[0] = (const char *)k; a.row_bytes[0] = k_row_stride * e; a.head_bytes[0] = k_head_stride * e;
    a.src[1] = (const char *)v; a.row_bytes[1] = v_row_stride * e; a.head_bytes[1] = v_head_stride * e;
    unsigned gy;
    walk(seqs->n_seq, seqs->n_rows, pool->n_kv_heads, &a.chunk, &gy);
    return pool->head_dim == 128 ? launch_append<128>(a, dtype, gy, (hipStream_t)hip_stream) : launch_append<64>(a, dtype, gy, (hipStream_t)hip_stream);
}

template <int HD>
static int launch_read(const kv8_read_args &a, int dtype, unsigned gy, hipStream_t s)
{
    const dim3 grid(a.pool.n_heads, gy);
    if (dtype == PV_F32) k_kv8_read<HD, float><<<grid, 64, 0, s>>>(a);
    else if (dtype == PV_BF16) k_kv8_read<HD, __bf16><<<grid, 64, 0, s>>>(a);
    else k_kv8_read<HD, _Float16><<<grid, 64, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

extern "C" int pv_kv8_read(const pv_kv8_pool *pool, const pv_kv8_seqs *seqs, void *k, int64_t k_row_stride, int64_t k_head_stride,
                           void *v, int64_t v_row_stride, int64_t v_head_stride, int32_t dtype, void *hip_stream)
{
    int rc;
    if ((rc = pv_kv8_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (seqs->n_rows == 0 || seqs->n_seq == 0) return PV_OK;
    if ((rc = pv_kv8_check_rows("k", k, k_row_stride, k_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("v", v, v_row_stride, v_head_stride, dtype)) != PV_OK) return rc;
    kv8_read_args a = {};
    a.pool = pv_kv8_pool_args(pool); a.seqs = pv_kv8_seqs_args(seqs);
    const int64_t e = (int64_t)dtype_size(dtype);
    a.dst[0] = (char *)k; a.row_bytes[0] = k_row_stride * e; a.head_bytes[0] = k_head_stride * e;
    a.dst[1] = (char *)v; a.row_bytes[1] = v_row_stride * e; a.head_bytes[1] = v_head_stride * e;
    unsigned gy;
    walk(seqs->n_seq, seqs->n_rows, pool->n_kv_heads, &a.chunk, &gy);
    return pool->head_dim == 128 ? launch_read<128>(a, dtype, gy, (hipStream_t)hip_stream) : launch_read<64>(a, dtype, gy, (hipStream_t)hip_stream);
}

extern "C" int pv_kv8_bytes(const pv_kv8_pool *pool, size_t *codes_bytes, size_t *scales_bytes)
{
    if (!pool || !codes_bytes || !scales_bytes) { pv_set_error("null pointer"); return PV_EINVAL; }
    pv_kv8_pool p = *pool;
    if (!p.codes) p.codes = (void *)16;          // (sizes may be asked before there is memory)
    if (!p.scales) p.scales = (void *)16;
    const int rc = pv_kv8_check_pool(&p);
    if (rc != PV_OK) return rc;
    const size_t blocks = (size_t)p.n_pages * p.n_kv_heads * (p.page_tokens / 16) * 2;
    *codes_bytes = blocks * 16 * p.head_dim; *scales_bytes = blocks;
    return PV_OK;
}

// ---- a model's step ----

kv8_seqs pv_kv8_step_seqs(const pv_cache *c, int layer, int rows, int first, kv8_pool *pool)
{
    const pv_model_config &f = c->m->cfg;
    *pool = {(uint8_t *)c->d_pool, nullptr, c->n_pages, f.n_kv_heads, 0};
    while ((1 << pool->page_shift) < f.page_tokens) ++pool->page_shift;
    kv8_seqs q = {};
    q.st = c->ws.state; q.page_table = c->ws.page_table; q.table_pages = c->n_pages; q.n_rows = rows; q.layer = layer; q.first = first; q.scales_off = c->kv8_scales;
    q.batched = c->blk_units != 0 && first < 0; q.n_seq = q.batched ? c->io->batch.n_seq : 1;
    return q;
}

int pv_kv8_step_append(pv_cache *c, int layer, int rows, hipStream_t s)
{
    const pv_model_config &f = c->m->cfg;
    const int64_t kvd = (int64_t)f.n_kv_heads * f.head_dim;
    kv8_append_args a = {};
    a.seqs = pv_kv8_step_seqs(c, layer, rows, -1, &a.pool);
    for (int w = 0; w < 2; ++w) { a.src[w] = (const char *)(c->ws.kv_stage + w * kvd); a.row_bytes[w] = 4 * kvd; a.head_bytes[w] = 2 * f.head_dim; }
    unsigned gy;
    walk(a.seqs.n_seq, rows, f.n_kv_heads, &a.chunk, &gy);
    return f.head_dim == 128 ? launch_append<128>(a, PV_BF16, gy, s) : launch_append<64>(a, PV_BF16, gy, s);
}

// tokens [first, first + n) of one layer, bf16 [n][n_kv_heads * head_dim] each
int pv_kv8_export(pv_cache *c, int layer, int first, int n, uint16_t *k, uint16_t *v, hipStream_t s)
{
    const pv_model_config &f = c->m->cfg;
    kv8_read_args a = {};
    a.seqs = pv_kv8_step_seqs(c, layer, n, first, &a.pool);
    a.dst[0] = (char *)k; a.dst[1] = (char *)v;
    for (int w = 0; w < 2; ++w) { a.row_bytes[w] = (int64_t)2 * f.n_kv_heads * f.head_dim; a.head_bytes[w] = 2 * f.head_dim; }
    unsigned gy;
    walk(1, n, f.n_kv_heads, &a.chunk, &gy);
    return f.head_dim == 128 ? launch_read<128>(a, PV_BF16, gy, s) : launch_read<64>(a, PV_BF16, gy, s);
}

int pv_kv8_tree_compact(pv_cache *c, hipStream_t s)
{
    const pv_model_config &f = c->m->cfg;
    kv8_pool pool;
    const kv8_seqs q = pv_kv8_step_seqs(c, 0, PV_MAX_ROWS, -1, &pool);
    const dim3 grid(2 * f.n_kv_heads, f.n_layers);
    if (f.head_dim == 128) k_kv8_tree<128><<<grid, 64, 0, s>>>(pool, q);
    else k_kv8_tree<64><<<grid, 64, 0, s>>>(pool, q);
    PV_HIP(hipGetLastError());
    return PV_OK;
}
