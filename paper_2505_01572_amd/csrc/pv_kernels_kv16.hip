// Rotary positions; writing the 16-bit key/value cache, keys rotated on the way; moving the accepted path of a draft tree behind the prefix.
//
// A pair of features (a, b) at position p turns by p * turns[i] of a full circle:  a' = A (a cos - b sin),  b' = A (a sin + b cos),  A the amplitude.  The product is made in 64 bits and
// brought to an eighth of a turn about 0 there (at position 10^6 a product in 32 bits has lost all but two digits); what is left is small enough for 32 bits and a Taylor series.
#include "pv_kv16.h"

struct rot_args {
    const double *turns;                    // of a pair, per position
    int units, rest, interleaved;           // units of two pieces of 16 bytes that are rotated, and those that are not
    float amplitude;
    const int32_t *positions;               // of the rows; NULL: the tokens' own
};

struct rot_rows { const char *src; char *dst; int64_t src_row, src_head, dst_row, dst_head; int heads; };      // rows of heads and where they go, strides in bytes

// cos and sin of a position's angle, times the amplitude: |r| <= 1/8 turn, series up to x^9 and x^10 (what is left out is below 2^-29)
__device__ inline void rot_angle(int pos, double turns, float amplitude, float &c, float &s)
{
    const double t = (double)pos * turns, k = rint(4.0 * t);
    const float x = 6.28318530717958647692f * (float)(t - 0.25 * k), y = x * x;
    const int quarter = (int)(k - 4.0 * floor(0.25 * k));
    const float sn = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float cs = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
    s = amplitude * (quarter & 2 ? -a : a);
    c = amplitude * (((quarter + 1) & 2) ? -b : b);
}

// A thread's unit u of a row's heads: two pieces of 16 bytes, of PE numbers each, as far apart as the members of a pair are, so that neighbours read what lies side by side.  (Pairs of neighbours lie in one piece.)
template <typename T> constexpr int rot_pe() { return 16 / (int)sizeof(T); }
__device__ inline void rot_pieces(const rot_args &r, int u, int &p0, int &p1)
{
    p0 = u < r.units ? u : u + r.units;
    p1 = p0 + (u < r.units ? r.units : r.rest);
}
template <int PE> __device__ inline void rot_turn(const rot_args &r, int u, const float (&c)[PE], const float (&s)[PE], float (&a)[PE], float (&b)[PE])
{
    if (u >= r.units) return;
    if (r.interleaved) {
#pragma unroll
        for (int i = 0; i < PE / 2; ++i) {
            const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
            a[2 * i] = x * c[i] - y * s[i]; a[2 * i + 1] = fmaf(x, s[i], y * c[i]);
            b[2 * i] = z * c[PE / 2 + i] - w * s[PE / 2 + i]; b[2 * i + 1] = fmaf(z, s[PE / 2 + i], w * c[PE / 2 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PE; ++i) { const float x = a[i], y = b[i]; a[i] = x * c[i] - y * s[i]; b[i] = fmaf(x, s[i], y * c[i]); }
    }
}
template <int PE> __device__ inline void rot_angles(const rot_args &r, int u, int pos, float (&c)[PE], float (&s)[PE])
{
    if (u >= r.units) return;
    const int first = r.interleaved ? u * (PE / 2) : u * PE, second = r.interleaved ? (u + r.units) * (PE / 2) : first + PE / 2;
#pragma unroll
    for (int i = 0; i < PE; ++i) rot_angle(pos, r.turns[i < PE / 2 ? first + i : second + i - PE / 2], r.amplitude, c[i], s[i]);
}

// A piece's numbers in 32 bits, and back to memory
template <typename T> __device__ inline void rot_numbers(u32x4 w, float (&v)[rot_pe<T>()])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t d = w[i];
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(d);
        else if constexpr (__is_same(T, __bf16)) { v[2 * i] = __uint_as_float(d << 16); v[2 * i + 1] = __uint_as_float(d & 0xffff0000u); }
        else { const kv16_h2 h = __builtin_bit_cast(kv16_h2, d); v[2 * i] = (float)h.x; v[2 * i + 1] = (float)h.y; }
    }
}
template <typename S, int PE> __device__ inline void rot_store(char *p, const float (&v)[PE])
{
    if constexpr (sizeof(S) == 4) *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (PE == 4) *(uint2 *)p = make_uint2(kv16_two<S>(v[0], v[1]), kv16_two<S>(v[2], v[3]));
    else *(uint4 *)p = make_uint4(kv16_two<S>(v[0], v[1]), kv16_two<S>(v[2], v[3]), kv16_two<S>(v[4], v[5]), kv16_two<S>(v[6], v[7]));
}

// Rows of heads: a thread has a row and a unit of its features, and takes the heads first, first + step, ..., four of them on their way at once (13312 rows of 64 heads of bf16, their keys and values: 143 us one at a time, 121
// so).  8191 rows of 40 heads of f32 in pieces of 32 bytes, between which neighbours' accesses leave gaps, 87 us, so 65 (a copy of as many bytes: 65)
template <typename T>
__device__ inline void rot_heads(const rot_args &r, const rot_rows &x, int64_t row, int u, const float (&c)[rot_pe<T>()], const float (&s)[rot_pe<T>()], int first, int step)
{
    constexpr int HB = 4;
    int p0, p1;
    rot_pieces(r, u, p0, p1);
    const char *src = x.src + row * x.src_row;
    char *dst = x.dst + row * x.dst_row;
    for (int h0 = first; h0 < x.heads; h0 += HB * step) {
        u32x4 a[HB], b[HB];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const u32x4 *at = (const u32x4 *)(src + min(h0 + i * step, x.heads - 1) * x.src_head);
            if (i == 0 || h0 + i * step < x.heads) { a[i] = at[p0]; b[i] = at[p1]; }
        }
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            if (h0 + i * step >= x.heads) break;
            float v[rot_pe<T>()], w[rot_pe<T>()];
            rot_numbers<T>(a[i], v); rot_numbers<T>(b[i], w);
            rot_turn(r, u, c, s, v, w);
            char *to = dst + (h0 + i * step) * x.dst_head;
            rot_store<T>(to + p0 * 16, v); rot_store<T>(to + p1 * 16, w);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
k_rotate(const rot_args r, const rot_rows x, int n_rows, int head_units, int slots)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int u = (int)(id % head_units), slot = (int)(id / head_units % slots);
    const int64_t row = id / head_units / slots;
    if (row >= n_rows) return;
    float c[rot_pe<T>()], s[rot_pe<T>()];
    rot_angles(r, u, r.positions[row], c, s);
    rot_heads<T>(r, x, row, u, c, s, slot, slots);
}

struct kv16_append_args {
    kv16_pool pool;
    kv16_seqs seqs;
    rot_args rot;
    rot_rows k, v, q;                       // (k, v: read only; q.heads 0: none)
    int slots;                              // workgroups that share the heads of the same rows
};

// 16 rows of the call: their tokens' places, the rows' angles, then the heads.  Bound by the copy where there are many (13312 rows of 64 query and 8 kv heads of 128: 110.6 us, 4.9 TB/s; a copy of as much memory 105), by trips to memory,
// one behind the other, where there are few (64 rows: 6.5 us)
#define KV16_ROWS 16
struct kv16_place { int pos, turn, page, left; };     // token (-1: no such row), rotary position, page (-1: none), rows of the sequence from this one on (its first row: 1 << 30 more)

template <int HD, typename T, typename S>
__global__ void __launch_bounds__(256)
k_kv16_append(const kv16_append_args a)
{
    constexpr int PE = rot_pe<T>(), U = HD / (2 * PE), E = sizeof(T), NS = 256 / (KV16_ROWS * U);
    __shared__ kv16_place place[KV16_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, first = blockIdx.y * KV16_ROWS;
    {
        int row[4], s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) row[i] = first + wave * 4 + i;
        kv16_seqs_of_rows(a.seqs.row_start, a.seqs.n_seq, row, s);
        if (lane < 4) {
            const int mine = lane == 0 ? s[0] : lane == 1 ? s[1] : lane == 2 ? s[2] : s[3], at = first + wave * 4 + lane;
            kv16_place p = {-1, 0, -1, 0};
            if (mine < a.seqs.n_seq && at < a.seqs.n_rows) {
                const kv16_seq q = kv16_seq_at(a.seqs, mine);
                const int local = at - q.row0;
                const int64_t pos = (int64_t)q.len + local;
                if (local >= 0 && local < q.rows && pos <= 0x7fffffff) {
                    p.pos = (int)pos;
                    p.turn = a.rot.positions != nullptr ? a.rot.positions[at] : p.pos;
                    p.page = kv16_page(q, a.pool.n_pages, p.pos >> a.pool.page_shift);
                    p.left = q.rows - local + (local == 0 ? 1 << 30 : 0);
                }
            }
            place[wave * 4 + lane] = p;
        }
    }
    __syncthreads();
    const int u = tid % U, r = tid / U % KV16_ROWS, slot = blockIdx.x * NS + tid / (U * KV16_ROWS), slots = a.slots * NS;
    const kv16_place p = place[r];
    if (p.pos < 0) return;
    const int64_t row = first + r;
    const int in_page = p.pos & ((1 << a.pool.page_shift) - 1), sub = in_page >> 4, t = in_page & 15;
    // queries' heads, keys', values', dealt out one after the other
    auto begin = [&](int before) { const int b = (slot - before) % slots; return b < 0 ? b + slots : b; };
    float c[PE], s[PE];
    rot_angles(a.rot, u, p.turn, c, s);
    rot_heads<T>(a.rot, a.q, row, u, c, s, slot, slots);
    if (p.page < 0) return;
    int p0, p1;
    rot_pieces(a.rot, u, p0, p1);
    for (int h = begin(a.q.heads); h < a.k.heads; h += slots) {
        const u32x4 *src = (const u32x4 *)(a.k.src + row * a.k.src_row + h * a.k.src_head);
        char *dst = a.pool.pages + kv16_block<HD>(a.pool, p.page, h, 0, sub);
        float x[PE], y[PE];
        rot_numbers<T>(src[p0], x); rot_numbers<T>(src[p1], y);
        rot_turn(a.rot, u, c, s, x, y);
        rot_store<S>(dst + kv16_k_at(t, PE * p0), x); rot_store<S>(dst + kv16_k_at(t, PE * p1), y);
    }
    // values: four tokens lie side by side, and go together if they come together: with the first of them
    if ((t & 3) != 0 && !(p.left >> 30)) return;
    const int n = min(4 - (t & 3), p.left & ((1 << 30) - 1)), f0 = 32 * (u / (16 / PE)) + PE * (u % (16 / PE));
    for (int h = begin(a.q.heads + a.k.heads); h < a.v.heads; h += slots) {
        const char *src = a.v.src + row * a.v.src_row + h * a.v.src_head;
        char *dst = a.pool.pages + kv16_block<HD>(a.pool, p.page, h, 1, sub);
        auto of = [&](int i, int f) { return *(const u32x4 *)(src + i * a.v.src_row + f * E); };
        if (n == 4) {
            u32x4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = of(i, f0); y[i] = of(i, f0 + 16); }
            auto two = [&](u32x4 l, u32x4 m, int e) {
                if constexpr (__is_same(T, S)) return e & 1 ? l[e / 2] >> 16 | (m[e / 2] & 0xffff0000u) : (l[e / 2] & 0xffffu) | m[e / 2] << 16;
                else { float v[PE], w[PE]; rot_numbers<T>(l, v); rot_numbers<T>(m, w); return kv16_two<S>(v[e], w[e]); }
            };
#pragma unroll
            for (int e = 0; e < PE; ++e) *(uint4 *)(dst + kv16_v_at(t, f0 + e)) = make_uint4(two(x[0], x[1], e), two(x[2], x[3], e), two(y[0], y[1], e), two(y[2], y[3], e));
        } else {
            for (int i = 0; i < n; ++i) {
                float x[PE], y[PE];
                rot_numbers<T>(of(i, f0), x); rot_numbers<T>(of(i, f0 + 16), y);
#pragma unroll
                for (int e = 0; e < PE; ++e) { *(S *)(dst + kv16_v_at(t + i, f0 + e)) = (S)x[e]; *(S *)(dst + kv16_v_at(t + i, f0 + 16 + e)) = (S)y[e]; }
            }
        }
    }
}

struct kv16_keep_args {
    kv16_pool pool;
    kv16_seqs seqs;
    const int32_t *path, *accepted;
};

// A wave a sequence, head and kind: 16 tokens of the path at a time are read, then written (32 paths of 8 heads of 128: 4.2 us).  A path's numbers rise and none is less than its place, so what a later token comes from has not been
// written to by then.  Bound by the trips to the tables, the path and the tokens, one behind the other.
// (What a thread holds of them must not end up in LDS, where the compiler puts arrays that it cannot keep in registers: for its place there a kernel asks the launch's packet, in host memory, 17 us where 5 do.)
template <int HD>
__global__ void __launch_bounds__(64)
k_kv16_keep(const kv16_keep_args a)
{
    constexpr int B = 16, KL = HD / 8, VL = HD / 2;           // tokens at a time; lanes a token: 16 bytes of keys each; two values (features 16 apart, 8 bytes apart) each
    __shared__ int64_t sh_from[64], sh_to[64];
    const int lane = threadIdx.x, which = blockIdx.x & 1, head = blockIdx.x >> 1, shift = a.pool.page_shift;
    const int accepted = a.accepted[blockIdx.y];
    const kv16_seq q = kv16_seq_at(a.seqs, blockIdx.y);
    const int n = (int)min((int64_t)accepted + 1, (int64_t)q.rows);
    auto place = [&](int local) -> int64_t {                  // of the token's first key; of values: of its group of four's first 16 bytes, times 4, and its number in the group
        const int64_t pos = (int64_t)q.len + local;
        const int page = pos <= 0x7fffffff ? kv16_page(q, a.pool.n_pages, (int)pos >> shift) : -1, in_page = (int)pos & ((1 << shift) - 1), t = in_page & 15;
        if (page < 0) return -1;
        const int64_t block = (int64_t)kv16_block<HD>(a.pool, page, head, which, in_page >> 4);
        return which ? (block + kv16_v_at(t & ~3, 0)) * 4 + (t & 3) : block + kv16_k_at(t, 0);
    };
    char *pages = a.pool.pages;
    for (int d0 = 0; d0 < n; d0 += 64) {
        int64_t from = -1, to = -1;
        if (d0 + lane < n) {
            const int l = a.path[q.row0 + d0 + lane];
            if (l > d0 + lane && l < q.rows) { from = place(l); to = place(d0 + lane); }
        }
        if (to < 0) from = -1;
        const uint64_t moves = __ballot(from >= 0);
        sh_from[lane] = from; sh_to[lane] = to;
        __syncthreads();
        for (int b = 0; b < 64; b += B) {
            if (((moves >> b) & ((1 << B) - 1)) == 0) continue;
            if (which == 0) {
                constexpr int N = B * KL / 64;
                u32x4 x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = *(const u32x4 *)(pages + max(sh_from[b + (i * 64 + lane) / KL], (int64_t)0) + lane % KL * 256);      // (of a token that does not move: some of the pool)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = b + (i * 64 + lane) / KL;
                    if (sh_from[t] >= 0) *(u32x4 *)(pages + sh_to[t] + lane % KL * 256) = x[i];
                }
            } else {
                constexpr int N = B * VL / 64;
                const int at = lane % VL / 16 * 1024 + lane % 16 * 16;
                uint32_t x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int64_t f = max(sh_from[b + (i * 64 + lane) / VL], (int64_t)0);
                    const u32x4 v = *(const u32x4 *)(pages + f / 4 + at);      // values of features f and f + 16 of four tokens
                    const int r = (int)(f & 3) * 16;
                    x[i] = ((uint32_t)(((uint64_t)v.y << 32 | v.x) >> r) & 0xffffu) | (uint32_t)(((uint64_t)v.w << 32 | v.z) >> r) << 16;
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = b + (i * 64 + lane) / VL;
                    if (sh_from[t] >= 0) {
                        const int64_t o = sh_to[t];
                        uint16_t *to2 = (uint16_t *)(pages + o / 4 + at) + (o & 3);
                        to2[0] = (uint16_t)x[i]; to2[4] = (uint16_t)(x[i] >> 16);
                    }
                }
            }
        }
        __syncthreads();
    }
}

// ------------------------------- host side ----------------------------------------

int pv_kv16_check_pool(const pv_kv16_pool *p)
{
    if (!p || !p->pages) { pv_set_error("null pool"); return PV_EINVAL; }
    if (p->head_dim != 64 && p->head_dim != 128) { pv_set_error("16-bit cache: head_dim must be 64 or 128, got %d", p->head_dim); return PV_EINVAL; }
    if (p->dtype != PV_BF16 && p->dtype != PV_F16) { pv_set_error("16-bit cache: keys and values in bf16 or f16, got dtype %d", p->dtype); return PV_EINVAL; }
    if (p->n_pages < 1 || p->n_pages >= (1 << 26)) { pv_set_error("16-bit cache: n_pages %d outside [1, 2^26)", p->n_pages); return PV_ERANGE; }
    if (p->n_kv_heads < 1 || p->n_kv_heads > 16384) { pv_set_error("16-bit cache: n_kv_heads %d outside [1, 16384]", p->n_kv_heads); return PV_ERANGE; }
    if (p->page_tokens < 16 || p->page_tokens > 65536 || (p->page_tokens & (p->page_tokens - 1))) { pv_set_error("16-bit cache: page_tokens must be a power of two from 16 to 65536, got %d", p->page_tokens); return PV_EINVAL; }
    if ((int64_t)p->n_kv_heads * p->page_tokens * p->head_dim >= 1ll << 30) { pv_set_error("16-bit cache: a page of %d heads x %d tokens: 2^32 bytes or more", p->n_kv_heads, p->page_tokens); return PV_ERANGE; }
    if ((uintptr_t)p->pages & 15) { pv_set_error("16-bit cache: pages must be 16-byte aligned"); return PV_EINVAL; }
    return PV_OK;
}

kv16_pool pv_kv16_pool_args(const pv_kv16_pool *p)
{
    kv16_pool r = {(char *)p->pages, p->n_pages, p->n_kv_heads, 0};
    while ((1 << r.page_shift) < p->page_tokens) ++r.page_shift;
    return r;
}

kv16_seqs pv_kv16_seqs_args(const pv_kv8_seqs *q) { return {q->row_start, q->prefix_len, q->page_table, q->n_seq, q->n_rows, q->table_pages}; }

extern "C" int pv_kv16_bytes(const pv_kv16_pool *pool, size_t *bytes)
{
    if (!pool || !bytes) { pv_set_error("null pointer"); return PV_EINVAL; }
    pv_kv16_pool p = *pool;
    if (!p.pages) p.pages = (void *)16;          // (sizes may be asked before there is memory)
    const int rc = pv_kv16_check_pool(&p);
    if (rc != PV_OK) return rc;
    *bytes = (size_t)p.n_pages * p.n_kv_heads * p.page_tokens * p.head_dim * 4;
    return PV_OK;
}

static int check_rotary(const pv_rotary *r, int head_dim)
{
    if (!r || !r->turns) { pv_set_error("null rotary"); return PV_EINVAL; }
    if ((uintptr_t)r->turns & 7) { pv_set_error("rotary: turns must be 8-byte aligned"); return PV_EINVAL; }
    if (r->rotary_dim < 16 || r->rotary_dim % 16 || r->rotary_dim > head_dim) { pv_set_error("rotary_dim %d is not a multiple of 16 from 16 to head_dim %d", r->rotary_dim, head_dim); return PV_EINVAL; }
    if (!(r->amplitude - r->amplitude == 0.f)) { pv_set_error("rotary: the amplitude is not finite"); return PV_EINVAL; }
    return PV_OK;
}
static int unit_of(int dtype) { return dtype == PV_F32 ? 8 : 16; }       // numbers a thread's unit has
static rot_args rotary_of(const pv_rotary *r, const int32_t *positions, int head_dim, int dtype)
{
    const int n = unit_of(dtype);
    if (r == nullptr) return {nullptr, 0, head_dim / n, 0, 1.f, nullptr};
    return {r->turns, r->rotary_dim / n, (head_dim - r->rotary_dim) / n, r->interleaved != 0, r->amplitude, positions};
}
static rot_rows rows_of(const void *src, int64_t row, int64_t head, void *dst, int64_t dst_row, int64_t dst_head, int heads, int dtype)
{
    const int64_t e = dtype == PV_F32 ? 4 : 2;
    return {(const char *)src, (char *)dst, row * e, head * e, dst_row * e, dst_head * e, heads};
}

extern "C" int pv_rotate(const pv_rotary *rotary, const int32_t *positions, const void *x, int64_t x_row_stride, int64_t x_head_stride, void *out, int64_t out_row_stride, int64_t out_head_stride,
                         int32_t n_rows, int32_t n_heads, int32_t head_dim, int32_t dtype, void *hip_stream)
{
    if (head_dim < 16 || head_dim > 1024 || head_dim % 16) { pv_set_error("head_dim %d is not a multiple of 16 from 16 to 1024", head_dim); return PV_EINVAL; }
    int rc = check_rotary(rotary, head_dim);
    if (rc != PV_OK) return rc;
    if (n_rows < 0 || n_rows > (1 << 24)) { pv_set_error("n_rows %d outside [0, 2^24]", n_rows); return PV_ERANGE; }
    if (n_heads < 0 || n_heads > 16384) { pv_set_error("n_heads %d outside [0, 16384]", n_heads); return PV_ERANGE; }
    if (n_rows == 0 || n_heads == 0) return PV_OK;
    if (!positions || ((uintptr_t)positions & 3)) { pv_set_error("positions: null or not aligned"); return PV_EINVAL; }
    if ((rc = pv_kv8_check_rows("x", x, x_row_stride, x_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("out", out, out_row_stride, out_head_stride, dtype)) != PV_OK) return rc;
    const rot_args r = rotary_of(rotary, positions, head_dim, dtype);
    const rot_rows rows = rows_of(x, x_row_stride, x_head_stride, out, out_row_stride, out_head_stride, n_heads, dtype);
    const int units = head_dim / unit_of(dtype);
    // heads are shared by as many threads as fill the chip
    const int64_t base = (int64_t)n_rows * units;
    int64_t slots = (524288 + base - 1) / base;
    slots = slots < n_heads ? slots : n_heads;
    const unsigned grid = (unsigned)((base * slots + 255) / 256);
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == PV_F32) k_rotate<float><<<grid, 256, 0, s>>>(r, rows, n_rows, units, (int)slots);
    else if (dtype == PV_BF16) k_rotate<__bf16><<<grid, 256, 0, s>>>(r, rows, n_rows, units, (int)slots);
    else k_rotate<_Float16><<<grid, 256, 0, s>>>(r, rows, n_rows, units, (int)slots);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

template <int HD, typename S>
static int launch_append(const kv16_append_args &a, int dtype, hipStream_t s)
{
    const dim3 grid(a.slots, (a.seqs.n_rows + KV16_ROWS - 1) / KV16_ROWS);
    if (dtype == PV_F32) k_kv16_append<HD, float, S><<<grid, 256, 0, s>>>(a);
    else if (dtype == PV_BF16) k_kv16_append<HD, __bf16, S><<<grid, 256, 0, s>>>(a);
    else k_kv16_append<HD, _Float16, S><<<grid, 256, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

extern "C" int pv_kv16_append(const pv_kv16_pool *pool, const pv_kv8_seqs *seqs, const void *k, int64_t k_row_stride, int64_t k_head_stride, const void *v, int64_t v_row_stride, int64_t v_head_stride,
                              const pv_rotary *rotary, const int32_t *positions, const void *q, int64_t q_row_stride, int64_t q_head_stride, int32_t n_q_heads,
                              void *q_out, int64_t q_out_row_stride, int64_t q_out_head_stride, int32_t dtype, void *hip_stream)
{
    int rc;
    if ((rc = pv_kv16_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (seqs->n_rows > 16 * 65535) { pv_set_error("n_rows %d: more than %d", seqs->n_rows, 16 * 65535); return PV_ERANGE; }
    if (rotary && (rc = check_rotary(rotary, pool->head_dim)) != PV_OK) return rc;
    if (!rotary && (q || positions)) { pv_set_error("queries and positions go with a rotary"); return PV_EINVAL; }
    if (n_q_heads < 0 || n_q_heads > 16384) { pv_set_error("n_q_heads %d outside [0, 16384]", n_q_heads); return PV_ERANGE; }
    if ((uintptr_t)positions & 3) { pv_set_error("positions are not aligned"); return PV_EINVAL; }
    if (seqs->n_rows == 0 || seqs->n_seq == 0) return PV_OK;
    if ((rc = pv_kv8_check_rows("k", k, k_row_stride, k_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("v", v, v_row_stride, v_head_stride, dtype)) != PV_OK) return rc;
    if (q && ((rc = pv_kv8_check_rows("q", q, q_row_stride, q_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("q_out", q_out, q_out_row_stride, q_out_head_stride, dtype)) != PV_OK)) return rc;
    kv16_append_args a = {};
    a.pool = pv_kv16_pool_args(pool); a.seqs = pv_kv16_seqs_args(seqs);
    a.rot = rotary_of(rotary, positions, pool->head_dim, dtype);
    a.k = rows_of(k, k_row_stride, k_head_stride, nullptr, 0, 0, pool->n_kv_heads, dtype);
    a.v = rows_of(v, v_row_stride, v_head_stride, nullptr, 0, 0, pool->n_kv_heads, dtype);
    a.q = rows_of(q, q_row_stride, q_head_stride, q_out, q_out_row_stride, q_out_head_stride, q ? n_q_heads : 0, dtype);
    // the heads of 16 rows are shared by as many workgroups as fill the chip several times over (13312 rows of 64 heads, their keys and values: 1024 workgroups 123 us, 2048 117, 4096 111)
    const int blocks = (seqs->n_rows + KV16_ROWS - 1) / KV16_ROWS, per = 256 / (KV16_ROWS * pool->head_dim / unit_of(dtype)), heads = a.q.heads + 2 * pool->n_kv_heads;
    int slots = (4096 + blocks - 1) / blocks;
    slots = slots < (heads + per - 1) / per ? slots : (heads + per - 1) / per;
    a.slots = slots > 1 ? slots : 1;
    hipStream_t s = (hipStream_t)hip_stream;
    if (pool->head_dim == 128) return pool->dtype == PV_BF16 ? launch_append<128, __bf16>(a, dtype, s) : launch_append<128, _Float16>(a, dtype, s);
    return pool->dtype == PV_BF16 ? launch_append<64, __bf16>(a, dtype, s) : launch_append<64, _Float16>(a, dtype, s);
}

extern "C" int pv_kv16_keep(const pv_kv16_pool *pool, const pv_kv8_seqs *seqs, const int32_t *path, const int32_t *accepted, void *hip_stream)
{
    int rc;
    if ((rc = pv_kv16_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (seqs->n_seq > 65535) { pv_set_error("n_seq %d: more than 65535", seqs->n_seq); return PV_ERANGE; }
    if (seqs->n_rows == 0 || seqs->n_seq == 0) return PV_OK;
    if (!path || !accepted || ((uintptr_t)path & 3) || ((uintptr_t)accepted & 3)) { pv_set_error("path or accepted: null or not aligned"); return PV_EINVAL; }
    kv16_keep_args a = {pv_kv16_pool_args(pool), pv_kv16_seqs_args(seqs), path, accepted};
    const dim3 grid(2 * pool->n_kv_heads, seqs->n_seq);
    if (pool->head_dim == 128) k_kv16_keep<128><<<grid, 64, 0, (hipStream_t)hip_stream>>>(a);
    else k_kv16_keep<64><<<grid, 64, 0, (hipStream_t)hip_stream>>>(a);
    PV_HIP(hipGetLastError());
    return PV_OK;
}
