// Attention over the 16-bit key/value cache (pv_kv16.h) on the matrix cores: blocks of rows (decoded tokens, prompts: causal; draft trees of any number of nodes: a mask of bits).
//
// The query rows of a kv head are packed token by token: row m of a sequence is query head m % group of its token m / group.  Everything is computed transposed: S^T (keys x rows) = K Q^T,
// O^T (features x rows) = V^T P^T; the accumulators of S^T are, two groups of 16 keys side by side, the second operand of the other product.  Softmax with the running maximum and sum, all in 32 bits,
// in powers of two.  f16 weights are kept times 2^15, so that many small ones beside a large one count fully.
#include <atomic>
#include "pv_kv16.h"

struct kv16_attn_args {
    kv16_pool pool;
    kv16_seqs seqs;
    const char *q; int64_t q_row_bytes, q_head_bytes;
    char *out; int64_t out_row_bytes, out_head_bytes;
    float *lse;
    const uint64_t *mask; int words;        // [row][words]
    float *part_o, *part_ml;                // [row][query head][split][HD], [2] (maximum, sum)
    int group, n_q_heads, nsplit, chunk;    // chunk: keys a split, a multiple of 64
    float scale2;                           // |scale| log2(e), more than 0 (a scale of 0: 1, and q is 0)
    uint32_t q_and, q_xor;                  // what q passes through: its sign is the scale's
};

// A lane's value added to those of the lanes before it
__device__ inline int kv16_sums(int v)
{
#define KV16_STEP(C, M) v += __builtin_amdgcn_update_dpp(0, v, C, M, 0xF, false)
    KV16_STEP(0x111, 0xF); KV16_STEP(0x112, 0xF); KV16_STEP(0x114, 0xF); KV16_STEP(0x118, 0xF);      // within 16 lanes
    KV16_STEP(0x142, 0xA); KV16_STEP(0x143, 0xC);                                                    // lane 15 to the next 16, lane 31 to the upper half
#undef KV16_STEP
    return v;
}

// Tile `unit` of the sequences' rows, TR packed rows a tile, counted through all sequences: its sequence and its number in it (false: there are not so many).  A sequence's tables are asked for
// at once, 64 sequences at a time: one trip to memory in most calls.
template <int TR> __device__ inline bool kv16_unit(const kv16_seqs &q, int unit, int group, kv16_seq &s, int &tile)
{
    const int lane = threadIdx.x & 63;
    for (int k = 0; k < q.n_seq; k += 64) {
        const int i = min(k + lane, q.n_seq - 1), r0 = q.row_start[i], r1 = q.row_start[i + 1], len = q.prefix_len[i], r = min(max(r1, 0), q.n_rows) - max(r0, 0);
        const int rows = k + lane >= q.n_seq || r0 < 0 || r < 0 || len < 0 ? 0 : r;
        const int mine = (rows * group + TR - 1) / TR, upto = kv16_sums(mine);
        const uint64_t past = __ballot(upto > unit);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            tile = unit - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
            s.table = q.page_table + (size_t)(k + l) * q.table_pages; s.table_pages = q.table_pages;
            s.row0 = __builtin_amdgcn_readlane(r0, l); s.rows = __builtin_amdgcn_readlane(rows, l); s.len = __builtin_amdgcn_readlane(len, l);
            return true;
        }
        unit -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Keys that exist for a sequence and that some row of the tile that ends with token `last` may see
__device__ inline int kv16_keys(const kv16_seq &s, int page_shift, int last, bool masked)
{
    const int64_t want = (int64_t)s.len + (masked ? s.rows : last + 1), there = (int64_t)s.table_pages << page_shift;
    return (int)min(want, there);
}

// An entry of a table of at least one page for the whole wave, by a scalar load (behind the table's end: the last one)
__device__ inline int kv16_entry(const kv16_seq &s, int logical)
{
    typedef const __attribute__((address_space(4))) int32_t *table;
    const uint32_t l = __builtin_amdgcn_readfirstlane(min((uint32_t)logical, (uint32_t)s.table_pages - 1));
    return ((table)(uintptr_t)uniform_ptr(s.table))[l];
}

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
template <typename S> __device__ inline f32x4 kv16_mfma(uint4 a, uint4 b, f32x4 c)
{
    if constexpr (__is_same(S, __bf16)) return mfma16(a, b, c);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A query row's place: token of the block, query head, whether there is such a row (else the last one's place)
struct kv16_row { int j, head, row; bool live; };
__device__ inline kv16_row kv16_row_at(const kv16_attn_args &a, const kv16_seq &s, int kvh, int m)
{
    kv16_row r;
    const int n = s.rows * a.group;
    r.live = m < n;
    m = min(m, n - 1);
    r.j = m / a.group; r.head = kvh * a.group + (m - r.j * a.group); r.row = s.row0 + r.j;
    return r;
}

template <int HD>
__device__ inline void kv16_load_q(const kv16_attn_args &a, const kv16_row &r, int g, uint4 (&q)[HD / 32])
{
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks) {
        const uint4 v = *(const uint4 *)(a.q + r.row * a.q_row_bytes + r.head * a.q_head_bytes + (ks * 32 + g * 8) * 2);
        q[ks] = make_uint4((v.x & a.q_and) ^ a.q_xor, (v.y & a.q_and) ^ a.q_xor, (v.z & a.q_and) ^ a.q_xor, (v.w & a.q_and) ^ a.q_xor);
    }
}

template <typename S>
__device__ inline void kv16_store4(const kv16_attn_args &a, int row, int head, int e, const float y[4])
{
    *(uint2 *)(a.out + row * a.out_row_bytes + head * a.out_head_bytes + e * 2) = make_uint2(kv16_two<S>(y[0], y[1]), kv16_two<S>(y[2], y[3]));
}

// Running result for RT tiles of 16 rows: lane (g, jl) has row jl's maximum (of scores times scale2) and its part of the sum, and features 16 e + 4 g .. + 3 of the output; sum and output times 2^B
template <int HD, int RT> struct kv16_acc { f32x4 O[RT][HD / 16]; float m[RT], l[RT]; };
template <typename S> constexpr int kv16_bias() { return __is_same(S, __bf16) ? 0 : 15; }

template <int HD, int RT> __device__ inline void kv16_begin(kv16_acc<HD, RT> &A)
{
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        A.m[t] = -INFINITY; A.l[t] = 0.f;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) A.O[t][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
}

// Which of 64 keys from p on a row sees: without a mask those before `end`; with one those before len, and the slots from there on that its bits name, of the first `slots`; all before nk.  Bit i: key p + i.
__device__ inline uint64_t kv16_first(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
template <typename WORD> __device__ inline uint64_t kv16_sees(bool masked, WORD word, int words, int p, int len, int end, int slots, int nk)       // word(i): word i of the row's mask
{
    uint64_t w = kv16_first(min(end, nk) - p);
    if (masked) {
        const int s = p - len, i = max(s, 0) >> 6, sh = s & 63;          // slot of the first key
        const uint64_t lo = word(min(i, words - 1)), hi = word(min(i + 1, words - 1));       // (loads without branches)
        const uint64_t l = i < words ? lo : 0ull, h = s >= 0 && sh != 0 && i + 1 < words ? hi << (64 - sh) : 0ull;
        w = s <= -64 ? ~0ull : s < 0 ? kv16_first(-s) | l << -s : l >> sh | h;
        w &= kv16_first(slots - s);
        w &= kv16_first(nk - p);
    }
    return w;
}

// The larger of two, as one instruction: fmaxf first makes quiet NaN of NaN of numbers that come out of a product, one more instruction for each.
// (NaN and a number: the number; two NaN: infinity, with which the row's weights are NaN too)
__device__ inline float kv16_max(float a, float b)
{
    float top = INFINITY;
    asm("" : "+s"(top));                     // (or the compiler sees fmaxf in it)
    return __builtin_amdgcn_fmed3f(a, b, top);
}

// Four weights as numbers of the cache's type, and what the type leaves of them
template <typename S> __device__ inline void kv16_pairs(const float (&p)[4], uint2 &w, uint2 &low)
{
    if constexpr (__is_same(S, __bf16)) {
        split2(p[0], p[1], w.x, low.x); split2(p[2], p[3], w.y, low.y);
    } else {
        const kv16_h2 a = {(_Float16)p[0], (_Float16)p[1]}, b = {(_Float16)p[2], (_Float16)p[3]};
        w = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
        low = make_uint2(kv16_two<_Float16>(p[0] - (float)a.x, p[1] - (float)a.y), kv16_two<_Float16>(p[2] - (float)b.x, p[3] - (float)b.y));
    }
}

// Scores of NG groups of 16 keys -> weights under the new maximum (P[tile][group]: keys 4 g .. + 3; PL: what the type leaves of them); what was there is scaled to it.  see(t): which
// of the keys from 4 g on the lane's row of tile t may attend to, a bit each.
template <typename S, int HD, int RT, int NG, typename SEE>
__device__ inline void kv16_softmax(kv16_acc<HD, RT> &A, f32x4 (&X)[RT][NG], float scale2, bool edge, SEE see, uint2 (&P)[RT][NG], uint2 (&PL)[RT][NG])
{
    float keep[RT];
    bool same = true;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float mx = -INFINITY;
        if (edge) {
            const uint64_t w = see(t);
#pragma unroll
            for (int q = 0; q < NG; ++q)
#pragma unroll
                for (int r = 0; r < 4; ++r) X[t][q][r] = ((w >> (16 * q + r)) & 1) ? X[t][q][r] : -INFINITY;
        }
#pragma unroll
        for (int q = 0; q < NG; ++q) mx = kv16_max(kv16_max(mx, kv16_max(X[t][q][0], X[t][q][1])), kv16_max(X[t][q][2], X[t][q][3]));
        mx = with_lane32(with_lane16(mx, kv16_max), kv16_max);
        mx = fmaxf(mx * scale2, A.m[t]);
        const float ref = mx == -INFINITY ? 0.f : mx, c = (float)kv16_bias<S>() - ref;              // (nothing seen so far: 0)
        keep[t] = __builtin_amdgcn_exp2f(A.m[t] - ref);
        same = same && keep[t] == 1.f;
        float ps = 0.f;
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(X[t][q][r], scale2, c));
            ps += (p[0] + p[1]) + (p[2] + p[3]);
            kv16_pairs<S>(p, P[t][q], PL[t][q]);
        }
        A.l[t] = fmaf(A.l[t], keep[t], ps);
        A.m[t] = mx;
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!__all(same)) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < HD / 16; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) A.O[t][e][r] *= keep[t];
    }
}

// O += V^T P^T of NG groups of 16 keys; v(i, b): a lane's 16 bytes of group i, features 32 b ...
template <typename S, int HD, int RT, int NG, typename V>
__device__ inline void kv16_output(kv16_acc<HD, RT> &A, const uint2 (&P)[RT][NG], const uint2 (&PL)[RT][NG], V v)
{
#pragma unroll
    for (int u = 0; u < NG / 2; ++u)
#pragma unroll
        for (int b = 0; b < HD / 32; ++b) {
            const uint4 x = v(2 * u, b), y = v(2 * u + 1, b);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 va = h == 0 ? make_uint4(x.x, x.y, y.x, y.y) : make_uint4(x.z, x.w, y.z, y.w);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    f32x4 &o = A.O[t][2 * b + h];
                    o = kv16_mfma<S>(va, make_uint4(P[t][2 * u].x, P[t][2 * u].y, P[t][2 * u + 1].x, P[t][2 * u + 1].y), o);
                    o = kv16_mfma<S>(va, make_uint4(PL[t][2 * u].x, PL[t][2 * u].y, PL[t][2 * u + 1].x, PL[t][2 * u + 1].y), o);
                }
            }
            __builtin_amdgcn_sched_barrier(0);               // (or the values of all tiles are asked for first, and no registers are left)
        }
}

// Values that are not finite are kept from the rows that do not see them (0 times infinity is NaN): the products of keys that not every row sees are made with 0 in their place, and in the end infinity, of its sign, or NaN is
// added to the outputs of the rows that see one.
template <typename S> __device__ inline uint32_t kv16_strange(uint32_t w)      // 0x8000 in each half whose exponent is all ones
{
    constexpr uint32_t e = __is_same(S, __bf16) ? 0x7f807f80u : 0x7c007c00u, one = __is_same(S, __bf16) ? 0x00800080u : 0x04000400u;
    return ((w & e) + one) & 0x80008000u;
}
template <typename S> __device__ inline uint32_t kv16_plain(uint32_t w) { return w & ~((kv16_strange<S>(w) >> 15) * 0xffffu); }

// Pairs of groups of 16 keys from p0 on, step apart, up to p1: skip(p): nothing to look at there; see(t, p): which keys from p + 4 g on the lane's row of tile t may attend to; v(p, i, b): group i's values as they are, 0 where there
// are none.  (Features in the outer loop, and nothing unrolled but that: few registers beside the results.)
template <typename S, int HD, int RT, typename SKIP, typename SEE, typename V>
__device__ inline void kv16_put_strange(kv16_acc<HD, RT> &A, int p0, int p1, int step, SKIP skip, SEE see, V v)
{
    constexpr uint32_t frac = __is_same(S, __bf16) ? 0x007fu : 0x03ffu, one = __is_same(S, __bf16) ? 0x3f80u : 0x3c00u;
#pragma unroll
    for (int b = 0; b < HD / 32; ++b) {
#pragma unroll 1
        for (int p = p0; p < p1; p += step) {
            if (skip(p)) continue;
            const uint4 x = v(p, 0, b), y = v(p, 1, b);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const uint64_t w = see(t, p);
                auto two = [&](int i) { const int o = 16 * (i / 2) + 2 * (i & 1); return (uint32_t)((w >> o) & 1) * one | (uint32_t)((w >> (o + 1)) & 1) * (one << 16); };
                const uint4 seen = make_uint4(two(0), two(1), two(2), two(3));
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int sign = 0; sign < 2; ++sign) {               // infinity of this sign, or NaN
                        const uint32_t n4[4] = {h == 0 ? x.x : x.z, h == 0 ? x.y : x.w, h == 0 ? y.x : y.z, h == 0 ? y.y : y.w};
                        uint32_t c[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t st = kv16_strange<S>(n4[i]);
                            auto is = [&](int o) { const uint32_t n = (n4[i] >> o) & 0xffffu; return ((st >> (o + 15)) & 1u) && ((n & frac) != 0 || (n >> 15) == (uint32_t)sign); };
                            c[i] = (is(0) ? one : 0u) | (is(16) ? one << 16 : 0u);
                        }
                        const f32x4 n = kv16_mfma<S>(make_uint4(c[0], c[1], c[2], c[3]), seen, (f32x4){0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r) if (n[r] > 0.f) A.O[t][2 * b + h][r] += sign ? -INFINITY : INFINITY;
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
    }
}

// a row's output and lse, or its chunk's part of them
template <typename S, int HD>
__device__ inline void kv16_finish4(const kv16_attn_args &a, const kv16_row &w, int e, const float o[4], float M, float L, bool whole, int split)
{
    const size_t at = (size_t)w.row * a.n_q_heads + w.head;
    if (whole) {
        const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        kv16_store4<S>(a, w.row, w.head, e, y);
        if (a.lse != nullptr && e == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
    } else {
        *(float4 *)(a.part_o + (at * a.nsplit + split) * HD + e) = make_float4(o[0], o[1], o[2], o[3]);
        if (e == 0) *(float2 *)(a.part_ml + (at * a.nsplit + split) * 2) = make_float2(M, L);
    }
}

// Few rows: one workgroup is a kv head, a tile of 16 packed rows of a sequence, a chunk of its keys; the waves take 32 keys in turn, straight from memory to registers, and are joined
// through LDS at the end.  A weight is a pair of numbers of the cache's type (16 significant bits in bf16, 22 in f16): the matrix cores have the time.  Bound by the read of the cache: the next 32 keys' K is asked for when this one's scores are there, V when its products are.
// 32 sequences of one row and some 4000 keys of 8 heads of 128, 531 MB: 82.6 us, 6.4 TB/s (a read stream reaches 6.43); 4.6 more for the launch that joins the chunks.
template <int HD, typename S>
__global__ void __launch_bounds__(256)
k_kv16_attn(const kv16_attn_args a)
{
    constexpr int KS = HD / 32, TR = 16, OS = 68, NG = 2, STEP = 16 * NG;
    __shared__ float2 sh_ml[4][TR];
    __shared__ float sh_o[4][TR][OS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jl = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.x % a.pool.n_heads, split = blockIdx.y;       // (the tiles and chunks of a head: on one XCD where the heads are a multiple of eight)
    int tile = 0;
    kv16_seq sq;
    if (!kv16_unit<TR>(a.seqs, blockIdx.x / a.pool.n_heads, a.group, sq, tile)) return;
    const int m0 = tile * TR, nrows = sq.rows * a.group, shift = a.pool.page_shift;
    const int last = (min(m0 + TR, nrows) - 1) / a.group;
    const int nk = __builtin_amdgcn_readfirstlane(kv16_keys(sq, shift, last, a.mask != nullptr)), len = __builtin_amdgcn_readfirstlane(min(sq.len, 1 << 30));     // (no table goes further)
    const int k0 = split * a.chunk, k1 = min(k0 + a.chunk, nk);
    if (k0 >= nk && split > 0) return;      // (a sequence without keys: split 0 writes its rows)
    const bool whole = nk <= a.chunk;
    const int sure = min(nk, a.mask != nullptr ? len : len + m0 / a.group + 1);     // keys before this one are seen by every row

    const uint32_t block = (uint32_t)(2 * HD) << shift, in_page = (1u << shift) - 1;      // bytes of a head's keys in a page
    const uint64_t page_bytes = (uint64_t)2 * block * a.pool.n_heads;
    const char *base = a.pool.pages + (size_t)kvh * 2 * block;
    int page[NG], ahead[NG];
    auto pages = [&](int p0, int (&to)[NG]) {
#pragma unroll
        for (int i = 0; i < NG; ++i) to[i] = kv16_entry(sq, (p0 + 16 * i) >> shift);
    };
    auto exists = [&](int p0, int i) { return (int)(p0 + 16 * i < k1) & (int)((uint32_t)page[i] < (uint32_t)a.pool.n_pages); };       // (k1 does not lie behind the table's end)
    // Every load is made, without a branch, through a descriptor of no bytes where there is no such group: it reads nothing then and gives zeros.
    uint4 kt[NG][KS], vt[NG][KS];
    __amdgpu_buffer_rsrc_t from[NG];
    int bad = 0;
    auto load_16 = [&](int i, uint32_t off, int b) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from[i], off + lane * 16 + b * 1024, 0, 2);      // (2: each number is read once, and past the caches)
        return make_uint4(v.x, v.y, v.z, v.w);
    };
    auto load_k = [&](int p0) {
        bad = 0;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int ok = exists(p0, i), at = ok ? page[i] : 0;
            bad |= (ok ^ 1) << i;
            const char *p = uniform_ptr(base + ((uint64_t)(uint32_t)at * page_bytes + ((p0 + 16 * i) & in_page) * (2 * HD)));
            from[i] = __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, ok ? (int)(block + 32 * HD) : 0, 0x00027000);
#pragma unroll
            for (int b = 0; b < KS; ++b) kt[i][b] = load_16(i, 0, b);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int b = 0; b < KS; ++b) vt[i][b] = load_16(i, block, b);
    };

    int p0 = k0 + STEP * wave;
#pragma unroll
    for (int i = 0; i < NG; ++i) page[i] = ahead[i] = -1;
    if (p0 < k1) pages(p0, page);
    const kv16_row row = kv16_row_at(a, sq, kvh, m0 + jl);
    uint4 q[KS];
    kv16_load_q<HD>(a, row, g, q);
    const uint64_t *mrow = a.mask == nullptr ? nullptr : a.mask + (size_t)row.row * a.words;
    kv16_acc<HD, 1> A;
    kv16_begin(A);
    asm volatile("" ::: "memory");
    load_k(p0);
    load_v();
    auto sees = [&](int p) { return kv16_sees(mrow != nullptr, [&](int i) { return mrow[i]; }, a.words, p + 4 * g, len, len + row.j + 1, sq.rows, nk); };
    bool spoilt = false;                    // numbers that are not finite among values that not every row sees
    if (p0 < k1) pages(p0 + 4 * STEP, ahead);
    while (p0 < k1) {
        const int miss = bad;
        f32x4 X[1][NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            X[0][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < KS; ++b) X[0][i] = kv16_mfma<S>(kt[i][b], q[b], X[0][i]);
        }
        __builtin_amdgcn_sched_barrier(0);
        const bool edge = p0 + STEP > sure || miss != 0;
        uint64_t there = ~0ull;
#pragma unroll
        for (int i = 0; i < NG; ++i) if ((miss >> i) & 1) there &= ~(0xffffull << (16 * i));
        const int p1 = p0 + 4 * STEP;
#pragma unroll
        for (int i = 0; i < NG; ++i) page[i] = ahead[i];
        load_k(p1);
        pages(p1 + 4 * STEP, ahead);
        uint2 P[1][NG], PL[1][NG];
        kv16_softmax<S>(A, X, a.scale2, edge, [&](int) { return sees(p0) & there; }, P, PL);
        if (edge) {
            uint32_t strange = 0;
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int b = 0; b < KS; ++b) strange |= kv16_strange<S>(vt[i][b].x) | kv16_strange<S>(vt[i][b].y) | kv16_strange<S>(vt[i][b].z) | kv16_strange<S>(vt[i][b].w);
            if (__any(strange != 0)) {
                spoilt = true;
#pragma unroll
                for (int i = 0; i < NG; ++i)
#pragma unroll
                    for (int b = 0; b < KS; ++b) vt[i][b] = make_uint4(kv16_plain<S>(vt[i][b].x), kv16_plain<S>(vt[i][b].y), kv16_plain<S>(vt[i][b].z), kv16_plain<S>(vt[i][b].w));
            }
        }
        kv16_output<S>(A, P, PL, [&](int i, int b) { return vt[i][b]; });
        p0 = p1;
        load_v();
    }
    if (spoilt)
        kv16_put_strange<S, HD, 1>(A, k0 + STEP * wave, k1, 4 * STEP,
            [&](int p) { pages(p, page); return p + STEP <= sure && (exists(p, 0) & exists(p, 1)); },      // (theirs went through the products)
            [&](int, int p) { return sees(p); },
            [&](int p, int i, int b) {
                if (!exists(p, i)) return make_uint4(0u, 0u, 0u, 0u);
                return ((const uint4 *)(base + ((uint64_t)(uint32_t)page[i] * page_bytes + block + ((p + 16 * i) & in_page) * (2 * HD))))[b * 64 + lane];
            });

    // join the waves: each parks its maximum and sum and, 64 features at a time, its output
    const float unit = __builtin_bit_cast(float, (127 - kv16_bias<S>()) << 23);
    A.l[0] = with_lane32(with_lane16(A.l[0], op_add), op_add);
    if (g == 0) sh_ml[wave][jl] = make_float2(A.m[0], A.l[0] * unit);
#pragma unroll
    for (int part = 0; part < HD / 64; ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x4 o = A.O[0][4 * part + e];
            *(float4 *)&sh_o[wave][jl][e * 16 + 4 * g] = make_float4(o[0] * unit, o[1] * unit, o[2] * unit, o[3] * unit);
        }
        __syncthreads();
        const int r = threadIdx.x >> 4, c4 = threadIdx.x & 15;
        const kv16_row w = kv16_row_at(a, sq, kvh, m0 + r);
        if (!w.live) continue;
        float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) M = fmaxf(M, sh_ml[k][r].x);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = __builtin_amdgcn_exp2f(sh_ml[k][r].x - ref);
            const float4 v = *(const float4 *)&sh_o[k][r][4 * c4];
            o[0] = fmaf(f, v.x, o[0]); o[1] = fmaf(f, v.y, o[1]); o[2] = fmaf(f, v.z, o[2]); o[3] = fmaf(f, v.w, o[3]);
            L = fmaf(f, sh_ml[k][r].y, L);
        }
        kv16_finish4<S, HD>(a, w, part * 64 + 4 * c4, o, M, L, whole, split);
    }
}

// Many rows: a workgroup is a kv head, 64 RT packed rows of a sequence (16 RT a wave), a chunk of its keys.  64 keys at a time go through LDS, copied straight from memory, each wave a group of 16: values a step ahead,
// keys two, because the products with the next step's keys are made while this one's scores become weights: those keep the vector ALU busy (an exponential takes four turns, what makes a weight a pair two and a half), the products the
// matrix cores.  A weight is a pair of numbers of the cache's type, as with few rows: so a row's result has the same bits behind it whatever tile it comes to lie in.  One number a weight, 8 significant bits in bf16, adds as
// much to an output's error as its own rounding does (relative to 64 bits 2.3e-3 for 1.7e-3, in f16 2.9e-4 for 2.1e-4) and takes three quarters of the time (341 us for the 445 below).
// Two prompts of up to 2048 rows of 32 heads of 128 over up to 6100 keys and themselves, bf16: 445 us, 335 GFLOP asked for, 502 on the matrix cores, whose 1128 TFLOP/s are 91 % of what a library product of 8192^3 reaches (1242);
// they are busy 49 % of the cycles, the vector ALU 52 %.
// Values as whole 16 bytes, sorted into operands by moves or by exchanges of registers: some 3 % more.
template <int HD>
struct kv16_wide {
    static constexpr int KS = HD / 32;
    static constexpr int buffer = 4 * KS * 64;                           // uint4 of 64 keys' K or V: [group][b][lane]
    static constexpr int masks = 1024;                                   // words of masks that there is room for
    static constexpr int lds = 4 * buffer * 16 + 16 + masks * 8;         // two of K, two of V, whether numbers that are not finite were among values that not every row sees, masks of the tile's tokens
};

__device__ inline float kv16_maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }      // (NaN if either is)

// A row tile's place in the softmax: the score that weights are relative to, what to add to a score for its exponent, what the results so far are worth under it, sum of weights.  The score is the largest so far or up to 8 less
// (in powers of two): results are scaled to another only where a score goes further, which is hardly ever.  A weight is then up to 2^8, so f16 weights are kept times 2^7.
#define KV16_SLACK 8.f
template <typename S> constexpr int kv16_wide_bias() { return __is_same(S, __bf16) ? 0 : 7; }
struct kv16_tile { float m, c, keep, l; };
template <typename S> __device__ inline void kv16_under(kv16_tile &T, float mx, float scale2)      // mx: of the lane's 16 scores of the next 64 keys
{
    mx = with_lane32(with_lane16(mx, kv16_maximum), kv16_maximum) * scale2;
    const float m = mx > T.m + KV16_SLACK ? mx : T.m, ref = m == -INFINITY ? 0.f : m;      // (nothing seen so far: 0; a score that is NaN: its weight is)
    T.keep = __builtin_amdgcn_exp2f(T.m - ref); T.c = (float)kv16_wide_bias<S>() - ref; T.m = m;
}
__device__ inline float kv16_maximum4(float m, f32x4 x) { return kv16_maximum(kv16_maximum(kv16_maximum(kv16_maximum(m, x[0]), x[1]), x[2]), x[3]); }
template <typename S> __device__ inline void kv16_weights4(f32x4 x, float scale2, float c, float &sum, uint2 &w, uint2 &low)
{
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(x[r], scale2, c));
    sum += (p[0] + p[1]) + (p[2] + p[3]);
    kv16_pairs<S>(p, w, low);
    asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(low.x), "+v"(low.y), "+v"(sum));     // (made here, not where they are used: the sum put off would keep every weight)
}

template <int HD, int RT, typename S>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_kv16_attn_wide(const kv16_attn_args a)
{
    using W = kv16_wide<HD>;
    constexpr int KS = W::KS, TR = 64 * RT;
    extern __shared__ uint4 wide_lds[];
    int *spoilt = (int *)(wide_lds + 4 * W::buffer);
    uint64_t *masks = (uint64_t *)(wide_lds + 4 * W::buffer + 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jl = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.x % a.pool.n_heads, split = blockIdx.y, units = gridDim.x / a.pool.n_heads;
    int tile = 0;
    // (the last tiles of a prompt have the most keys: they begin first)
    kv16_seq sq;
    if (!kv16_unit<TR>(a.seqs, units - 1 - blockIdx.x / a.pool.n_heads, a.group, sq, tile)) return;
    const int m0 = tile * TR, nrows = sq.rows * a.group, shift = a.pool.page_shift;
    const int last = (min(m0 + TR, nrows) - 1) / a.group;
    const int nk = __builtin_amdgcn_readfirstlane(kv16_keys(sq, shift, last, a.mask != nullptr)), len = __builtin_amdgcn_readfirstlane(min(sq.len, 1 << 30));     // (no table goes further)
    const int k0 = split * a.chunk, k1 = min(k0 + a.chunk, nk);
    if (k0 >= nk && split > 0) return;
    const bool whole = nk <= a.chunk;
    const int sure = min(nk, a.mask != nullptr ? len : len + m0 / a.group + 1);     // keys before this one are seen by every row
    const int steps = (k1 - k0 + 63) >> 6, j0 = m0 / a.group;
    const bool near = a.mask != nullptr && k1 > sure && (int64_t)(last - j0 + 1) * a.words <= W::masks;

    const uint32_t block = (uint32_t)(2 * HD) << shift, in_page = (1u << shift) - 1;
    const uint64_t page_bytes = (uint64_t)2 * block * a.pool.n_heads;
    const char *base = a.pool.pages + (size_t)kvh * 2 * block;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(wide_lds)) + wave * KS * 1024;
    // this wave's group of 16 keys of step s (one that does not exist: some keys of the pool, that no row sees)
    auto page_of = [&](int s) { return kv16_entry(sq, (k0 + 64 * s + 16 * wave) >> shift); };
    auto place = [&](int s, int page) {
        const int p = k0 + 64 * s + 16 * wave, at = p < k1 && (uint32_t)page < (uint32_t)a.pool.n_pages ? page : 0;
        return uniform_ptr(base + ((uint64_t)(uint32_t)at * page_bytes + (p & in_page) * (2 * HD)));
    };
    auto copy_k = [&](int s, int page) { dma_tiles<KS>(lds0 + (uint32_t)(s & 1) * (W::buffer * 16), place(s, page), lane * 16); };
    auto copy_v = [&](int s, int page) { dma_tiles<KS>(lds0 + (uint32_t)(2 + (s & 1)) * (W::buffer * 16), place(s, page) + block, lane * 16); };
    if (threadIdx.x == 0) *spoilt = 0;      // (the first step's barrier lies before its first use)
    int page1 = 0, page2 = 0;                // of the steps one and two ahead
    bool holes = false;                      // some page of the chunk does not exist
    if (steps > 0) {
        const int page0 = page_of(0);
        page1 = page_of(1); page2 = page_of(2);
        copy_k(0, page0); copy_v(0, page0); copy_k(1, page1);
        int bad = 0;
        for (int i = (k0 >> shift) + (int)threadIdx.x; i <= (k1 - 1) >> shift; i += 256) bad |= (uint32_t)sq.table[i] >= (uint32_t)a.pool.n_pages;
        // masks that steps of this chunk will ask for (read from memory there, they held up a step by some 2 us)
        if (near) for (int i = threadIdx.x; i < (last - j0 + 1) * a.words; i += 256) masks[i] = a.mask[(size_t)(sq.row0 + j0) * a.words + i];
        holes = __syncthreads_or(bad);
    }
    uint4 q[RT][KS];
    kv16_acc<HD, RT> A;
    kv16_begin(A);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        kv16_load_q<HD>(a, kv16_row_at(a, sq, kvh, m0 + (wave * RT + t) * 16 + jl), g, q[t]);
    }
    auto sees = [&](int t, int p) {
        int l = lane;
        asm volatile("" : "+v"(l));          // (what follows is made where it is needed: kept over the loop it would take the registers of the results)
        const int at = kv16_row_at(a, sq, kvh, m0 + (wave * RT + t) * 16 + (l & 15)).j;
        if (near) return kv16_sees(true, [&](int i) { return masks[(at - j0) * a.words + i]; }, a.words, p + 4 * (l >> 4), len, 0, sq.rows, nk);
        return kv16_sees(a.mask != nullptr, [&](int i) { return a.mask[(size_t)(sq.row0 + at) * a.words + i]; }, a.words, p + 4 * (l >> 4), len, len + at + 1, sq.rows, nk);
    };
    auto missing = [&](int p0) {             // which of the step's groups do not exist
        int miss = 0;
        for (int i = 0; i < 4; ++i) miss |= (int)(p0 + 16 * i >= k1) << i;
        if (holes) for (int i = 0; i < 4; ++i) miss |= (int)((uint32_t)kv16_entry(sq, (p0 + 16 * i) >> shift) >= (uint32_t)a.pool.n_pages) << i;
        return miss;
    };
    auto wait = [&]() {                      // this wave's copies have landed, its LDS reads are done, and so it is for every wave
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto keys = [&](int s, int i, uint4 (&k)[KS]) {      // group i of step s
        const uint4 *K = wide_lds + (s & 1) * W::buffer + lane;
#pragma unroll
        for (int b = 0; b < KS; ++b) k[b] = K[(i * KS + b) * 64];
    };
    auto scores = [&](const uint4 (&k)[KS], int i, f32x4 (&X)[RT][4]) {
#pragma unroll
        for (int t = 0; t < RT; ++t) X[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < KS; ++b)
#pragma unroll
            for (int t = 0; t < RT; ++t) X[t][i] = kv16_mfma<S>(k[b], q[t][b], X[t][i]);
    };
    auto is_edge = [&](int s) { return k0 + 64 * s + 64 > sure || holes; };
    auto hide = [&](int s, f32x4 (&X)[RT][4]) {          // what rows do not see of step s
        const int p0 = k0 + 64 * s, miss = missing(p0);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const uint64_t w = sees(t, p0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) X[t][i][r] = ((w >> (16 * i + r)) & 1) && !((miss >> i) & 1) ? X[t][i][r] : -INFINITY;
        }
    };
    kv16_tile T[RT];
    auto step = [&](int s, f32x4 (&X)[RT][4], f32x4 (&next)[RT][4]) {
        wait();                              // keys of step s + 1 and values of step s are there, and no wave reads the buffers that are filled next
        if (s + 2 < steps) copy_k(s + 2, page2);
        if (s + 1 < steps) copy_v(s + 1, page1);
        page1 = page2; page2 = page_of(s + 3);
        if (is_edge(s)) {                    // each wave looks through its group's values
            uint4 *V = wide_lds + (2 + (s & 1)) * W::buffer + wave * KS * 64 + lane;
            uint32_t strange = 0;
#pragma unroll
            for (int b = 0; b < KS; ++b) {
                const uint4 v = V[b * 64];
                const uint32_t any = kv16_strange<S>(v.x) | kv16_strange<S>(v.y) | kv16_strange<S>(v.z) | kv16_strange<S>(v.w);
                if (any) V[b * 64] = make_uint4(kv16_plain<S>(v.x), kv16_plain<S>(v.y), kv16_plain<S>(v.z), kv16_plain<S>(v.w));
                strange |= any;
            }
            if (strange) *spoilt = 1;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
        // A step's work in twelve parts, in each of which the matrix cores and the vector ALU have about as much to do, LDS asked a part ahead: the scores of the next step beside the first half of the weights, the products with the
        // first half of the values beside the second half of the weights, those with the second half beside the next maximum
        uint2 P[RT][4], PL[RT][4];
        float ps[RT], mx[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) { ps[t] = 0.f; mx[t] = -INFINITY; }
        uint4 k[2][KS], va[2][2];
        // (8 bytes at a time, as an operand's registers lie: both halves in one load would have to be moved)
        uint32_t half[2] = {lane * 2u, lane * 2u + 1};
        asm volatile("" : "+v"(half[1]));
        const uint2 *V = (const uint2 *)(wide_lds + (2 + (s & 1)) * W::buffer);
        auto values = [&](int n, uint4 (&v)[2]) {            // features 32 (n % KS) ... of groups 2 (n / KS) and the next
            const int u = n / KS, b = n % KS;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint2 x = V[(2 * u * KS + b) * 128 + half[h]], y = V[((2 * u + 1) * KS + b) * 128 + half[h]];
                v[h] = make_uint4(x.x, x.y, y.x, y.y);
            }
        };
        auto products = [&](int n, const uint4 (&v)[2], const uint2 (&w)[RT][4]) {
            const int u = n / KS, b = n % KS;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < RT; ++t) A.O[t][2 * b + h] = kv16_mfma<S>(v[h], make_uint4(w[t][2 * u].x, w[t][2 * u].y, w[t][2 * u + 1].x, w[t][2 * u + 1].y), A.O[t][2 * b + h]);
        };
        auto weights = [&](int n, int half_of) {             // n of 2 RT: two groups of a tile
            const int t = n >> 1, i = 2 * half_of + (n & 1);
            kv16_weights4<S>(X[t][i], a.scale2, T[t].c, ps[t], P[t][i], PL[t][i]);
        };
        keys(s + 1, 0, k[0]);                // (behind the last step: of what the buffer holds, not used)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < 3) keys(s + 1, i + 1, k[(i + 1) & 1]); else values(0, va[0]);
            __builtin_amdgcn_sched_barrier(0);
            scores(k[i & 1], i, next);
            if (i < 2 * RT) weights(i, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (s + 1 < steps && is_edge(s + 1)) hide(s + 1, next);
        bool same = true;
#pragma unroll
        for (int t = 0; t < RT; ++t) same = same && T[t].keep == 1.f;
        if (!__all(same)) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < HD / 16; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) A.O[t][e][r] *= T[t].keep;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
            if (n + 1 < 2 * KS) values(n + 1, va[(n + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
            if (n < KS) {                    // (2 RT weights in KS parts)
#pragma unroll
                for (int w = n; w < 2 * RT; w += KS) weights(w, 1);
            } else {
#pragma unroll
                for (int w = n - KS; w < 2 * RT; w += KS) mx[w >> 1] = kv16_maximum4(kv16_maximum4(mx[w >> 1], next[w >> 1][2 * (w & 1)]), next[w >> 1][2 * (w & 1) + 1]);
            }
            products(n, va[n & 1], P);
            products(n, va[n & 1], PL);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            T[t].l = fmaf(T[t].l, T[t].keep, ps[t]);
            if (s + 1 < steps) kv16_under<S>(T[t], mx[t], a.scale2);
        }
    };
    f32x4 X0[RT][4], X1[RT][4];
    if (steps > 0) {
        wait();
#pragma unroll
        for (int i = 0; i < 4; ++i) { uint4 k[KS]; keys(0, i, k); scores(k, i, X0); }
        if (is_edge(0)) hide(0, X0);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        T[t] = {-INFINITY, 0.f, 0.f, 0.f};
        if (steps > 0) {
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = kv16_maximum4(mx, X0[t][i]);
            kv16_under<S>(T[t], mx, a.scale2);
        }
    }
    for (int s = 0; s < steps; s += 2) {
        step(s, X0, X1);
        if (s + 1 < steps) step(s + 1, X1, X0);
    }
    if (steps > 0 && *spoilt != 0)           // (written ahead of a step's last barrier)
        kv16_put_strange<S, HD, RT>(A, k0, k1, 32,
            [&](int p) { const int of = k0 + (p - k0) / 64 * 64; return of + 64 <= sure && !holes; },      // (theirs went through the products)
            [&](int t, int p) { return sees(t, p); },
            [&](int p, int i, int b) {
                const int q = p + 16 * i, page = q < k1 ? kv16_entry(sq, q >> shift) : -1;
                if ((uint32_t)page >= (uint32_t)a.pool.n_pages) return make_uint4(0u, 0u, 0u, 0u);
                return ((const uint4 *)(base + ((uint64_t)(uint32_t)page * page_bytes + block + (q & in_page) * (2 * HD))))[b * 64 + lane];
            });
    const float unit = __builtin_bit_cast(float, (127 - kv16_wide_bias<S>()) << 23);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float Z = with_lane32(with_lane16(T[t].l, op_add), op_add) * unit;
        int l = lane;
        asm volatile("" : "+v"(l));          // (the row is found anew, not kept over the loop)
        const kv16_row row = kv16_row_at(a, sq, kvh, m0 + (wave * RT + t) * 16 + (l & 15));
        if (!row.live) continue;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) {
            const float o[4] = {A.O[t][e][0] * unit, A.O[t][e][1] * unit, A.O[t][e][2] * unit, A.O[t][e][3] * unit};
            kv16_finish4<S, HD>(a, row, e * 16 + 4 * g, o, T[t].m, Z, whole, split);
        }
    }
}

// Chunks that a row, the whole wave's, and a lane's head have (0: written already, or no such row)
__device__ inline int kv16_chunks(const kv16_attn_args &a, int row, int head, int TR)
{
    const int rows[1] = {row};
    int s[1];
    kv16_seqs_of_rows(a.seqs.row_start, a.seqs.n_seq, rows, s);
    const int si = __builtin_amdgcn_readfirstlane(s[0]);
    if (si >= a.seqs.n_seq) return 0;
    const kv16_seq sq = kv16_seq_at(a.seqs, si);
    const int j = row - sq.row0;
    if (j < 0 || j >= sq.rows) return 0;
    const int tile = (j * a.group + head % a.group) / TR, last = (min((tile + 1) * TR, sq.rows * a.group) - 1) / a.group;
    const int nk = kv16_keys(sq, a.pool.page_shift, last, a.mask != nullptr);
    return nk <= a.chunk ? 0 : (nk + a.chunk - 1) / a.chunk;
}

// The chunks of a row's keys joined, up to 16 of them (a trip to the tables beside one to the chunks: 4.6 us for 32 rows of 32 heads, 6.9 for 200 of 64): HD / 4 lanes a row and head, all of its chunks on their way at once.  A wave's heads are of one row: asked for beside the sequence's tables, whatever these turn out to say
template <int HD, typename S>
__global__ void __launch_bounds__(256)
k_kv16_attn_join(const kv16_attn_args a, int TR)
{
    constexpr int TPC = HD / 4, HW = 64 / TPC, FL = 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane % TPC;
    const int per = (a.n_q_heads + HW - 1) / HW, id = blockIdx.x * 4 + wave, row = __builtin_amdgcn_readfirstlane(id / per), head0 = (id - row * per) * HW + lane / TPC;
    if (row >= a.seqs.n_rows) return;
    const int head = min(head0, a.n_q_heads - 1);
    const size_t at = (size_t)row * a.n_q_heads + head;
    const float *po = a.part_o + at * a.nsplit * HD + 4 * t;
    float2 one = ((const float2 *)(a.part_ml + at * a.nsplit * 2))[min(lane % 16, a.nsplit - 1)];
    float4 v[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) if (i < a.nsplit) v[i] = *(const float4 *)(po + (size_t)i * HD);
    const int n = kv16_chunks(a, row, head, TR);              // (a wave's heads may lie in two tiles, of different numbers of chunks)
    if (lane % 16 >= n) one = make_float2(-INFINITY, 0.f);
    const float M = with_rotated<8>(with_rotated<4>(with_rotated<2>(with_rotated<1>(one.x, op_max), op_max), op_max), op_max), ref = M == -INFINITY ? 0.f : M;
    const float w = __builtin_amdgcn_exp2f(one.x - ref);
    const float L = with_rotated<8>(with_rotated<4>(with_rotated<2>(with_rotated<1>(w * one.y, op_add), op_add), op_add), op_add);
    float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c0 = 0; c0 < 16; c0 += FL) {
        if (c0 >= a.nsplit) break;
        if (c0 > 0) {
#pragma unroll
            for (int i = 0; i < FL; ++i) if (c0 + i < a.nsplit) v[i] = *(const float4 *)(po + (size_t)(c0 + i) * HD);
        }
#pragma unroll
        for (int i = 0; i < FL; ++i) {
            const float wc = __shfl(w, (lane & ~15) + c0 + i, 64);
            if (c0 + i < n) { o[0] = fmaf(wc, v[i].x, o[0]); o[1] = fmaf(wc, v[i].y, o[1]); o[2] = fmaf(wc, v[i].z, o[2]); o[3] = fmaf(wc, v[i].w, o[3]); }      // (others: anything)
        }
    }
    if (n == 0 || head0 >= a.n_q_heads) return;
    const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    kv16_store4<S>(a, row, head, 4 * t, y);
    if (a.lse != nullptr && t == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
}

// More than 16: four waves a row and head, four chunks of each 4 HD bytes on their way a thread
template <int HD, typename S>
__global__ void __launch_bounds__(256)
k_kv16_attn_merge(const kv16_attn_args a, int TR)
{
    constexpr int TPC = HD / 4, NG = 4 * (64 / TPC), FL = 4;
    __shared__ float4 sh[4][TPC];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)(blockIdx.x / a.n_q_heads), head = (int)(blockIdx.x % a.n_q_heads);
    const size_t at = (size_t)row * a.n_q_heads + head;
    const float2 *ml = (const float2 *)(a.part_ml + at * a.nsplit * 2);
    const int t = lane % TPC, cg = wave * (64 / TPC) + lane / TPC;
    const float *po = a.part_o + at * a.nsplit * HD + 4 * t;
    // asked for beside the sequence's tables: the statistics of up to 64 chunks, and the first outputs
    float2 one = ml[min(lane, a.nsplit - 1)];
    float4 v[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) v[i] = *(const float4 *)(po + (size_t)min(cg + i * NG, a.nsplit - 1) * HD);
    const int n = kv16_chunks(a, row, head, TR);
    if (n == 0) return;
    if (lane >= n) one = make_float2(-INFINITY, 0.f);
    float M = one.x, L = 0.f;
    for (int c = 64 + lane; c < n; c += 64) M = fmaxf(M, ml[c].x);
    M = over_wave(M, op_max);
    const float ref = M == -INFINITY ? 0.f : M;
    L = one.y * __builtin_amdgcn_exp2f(one.x - ref);
    for (int c = 64 + lane; c < n; c += 64) L = fmaf(ml[c].y, __builtin_amdgcn_exp2f(ml[c].x - ref), L);
    L = over_wave(L, op_add);
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = cg; c0 < n; c0 += FL * NG) {
        if (c0 != cg) {
#pragma unroll
            for (int i = 0; i < FL; ++i) v[i] = *(const float4 *)(po + (size_t)min(c0 + i * NG, n - 1) * HD);
        }
#pragma unroll
        for (int i = 0; i < FL; ++i) {
            const int c = c0 + i * NG;
            if (c < n) {                    // (others: anything)
                const float w = __builtin_amdgcn_exp2f(ml[c].x - ref);
                o[0] = fmaf(w, v[i].x, o[0]); o[1] = fmaf(w, v[i].y, o[1]); o[2] = fmaf(w, v[i].z, o[2]); o[3] = fmaf(w, v[i].w, o[3]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { o[i] = with_lane32(o[i], op_add); if (TPC <= 16) o[i] = with_lane16(o[i], op_add); }
    if (lane < TPC) sh[wave][lane] = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (wave != 0 || lane >= TPC) return;
    const float4 x = sh[0][t], y = sh[1][t], z = sh[2][t], w = sh[3][t];
    const float inv = L == 0.f ? 0.f : 1.f / L, r[4] = {((x.x + y.x) + (z.x + w.x)) * inv, ((x.y + y.y) + (z.y + w.y)) * inv, ((x.z + y.z) + (z.z + w.z)) * inv, ((x.w + y.w) + (z.w + w.w)) * inv};
    kv16_store4<S>(a, row, head, 4 * t, r);
    if (a.lse != nullptr && lane == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
}

// ------------------------------- host side ----------------------------------------

// How a call's work is cut, from what the host knows: its rows (sequences are taken to have as many each), and how far the tables reach.
// Rows a tile: 16, straight from memory, where sequences have no more, and where the whole work is small, so that what the other kernel pays for going through LDS weighs more than keys read again for every 16 rows.  Else 64, or
// 128 where a sequence has much to do.  Eight kv heads of 128, one sequence, packed rows x keys, us from a graph with 16, 64, 128: 64 x 4000 14.0, 15.5, 18.4; 256 x 1000 13.4, 16.5, 20.8; 256 x 4000 22.2, 22.5, 26.5; 32 x 60000 60.8,
// 47.6, 62.7; 64 x 16000 28.6, 22.2, 27.0; 512 x 4000 32.9, 30.7, 32.6; 256 x 16000 67.7, 41.8, 41.4; 1024 x 4000 47.5, 44.4, 43.9; 256 x 60000 283, 115, 110.  16 sequences of up to 4000 keys, 16, 32, 128 rows each 33.9, 36.2, 51.0;
// 46.4, 37.3, 51.6; 86.1, 63.2, 92.8.
// Chunks of keys, 16 rows a tile: until there are two workgroups a CU, or four where sequences of different lengths come out at different times; few keys are one workgroup's, which saves the launch that joins.  More rows: as
// many as would take least by a count of steps (of 64 keys; three more for a workgroup's begin and end; two workgroups of a CU share it, one alone takes 0.65 as long) and of what the join has to move (one sequence of 1600 rows over
// 4301 keys, f16: 73 us with six chunks, in two rounds of workgroups, 69 with four, in one).
struct kv16_plan { int tr, units, nsplit, chunk; };

static kv16_plan plan(int n_seq, int n_rows, int group, int kv_heads, int hd, int64_t keys)
{
    kv16_plan p;
    const int64_t packed = (int64_t)n_rows * group;
    const bool little = packed * kv_heads <= (7 << 20) / (keys > 0 ? keys : 1);
    p.tr = packed <= (int64_t)16 * n_seq || little ? 16 : packed <= (int64_t)64 * n_seq || packed / n_seq <= (2 << 20) / (keys > 0 ? keys : 1) ? 64 : 128;
    p.units = (int)((packed + (int64_t)n_seq * (p.tr - 1)) / p.tr);
    const int64_t tiles = packed / p.tr > n_seq ? packed / p.tr : n_seq, base = tiles * kv_heads, most = (keys + 255) / 256;
    int64_t n, unit;
    if (p.tr == 16) {
        const int64_t want = n_seq > 1 ? 1024 : 512;
        n = (want + base - 1) / base; unit = 256;
        n = n < most ? n : most;
        n = n < 256 ? n : 256;
        if (most <= (base >= 256 ? 8 : packed <= (int64_t)16 * n_seq ? 4 : 3)) n = 1;
    } else {
        // by what each number of chunks would take, in steps of a workgroup that shares its CU with another (alone: 0.65)
        const int64_t all = ((packed + n_seq - 1) / n_seq + p.tr - 1) / p.tr * n_seq * kv_heads, steps = (keys + 63) / 64;
        double best = 0;
        n = 1; unit = 64;
        for (int64_t c = 1; c <= most && c <= 64; ++c) {
            const int64_t w = all * c;
            const double rounds = w <= 1024 ? (double)((w + 511) / 512) : w / 512.0 + 0.5, t = rounds * ((steps + c - 1) / c + 3) * (w <= 256 ? 0.65 : 1.0) + (c > 1 ? 2.0 + (double)packed * kv_heads * c * hd * 1e-6 : 0.0);
            if (c == 1 || t < best) { best = t; n = c; }
        }
    }
    n = n > 1 ? n : 1;
    p.chunk = (int)(((keys + n - 1) / n + unit - 1) / unit * unit);
    p.chunk = p.chunk > 256 ? p.chunk : 256;
    p.nsplit = (int)((keys + p.chunk - 1) / p.chunk);
    p.nsplit = p.nsplit > 1 ? p.nsplit : 1;
    return p;
}

static size_t part_bytes(const kv16_plan &p, int n_rows, int n_q_heads, int hd)
{
    return p.nsplit > 1 ? (size_t)n_rows * n_q_heads * p.nsplit * (hd + 2) * sizeof(float) : 0;
}

static int check_attention(const pv_kv16_pool *pool, const pv_kv8_seqs *seqs, int n_q_heads)
{
    int rc;
    if ((rc = pv_kv16_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (n_q_heads < 1 || n_q_heads % pool->n_kv_heads) { pv_set_error("n_q_heads %d is not a multiple of n_kv_heads %d", n_q_heads, pool->n_kv_heads); return PV_EINVAL; }
    if (((int64_t)seqs->n_rows + seqs->n_seq) * n_q_heads > (1 << 24)) { pv_set_error("(n_rows %d + n_seq %d) x n_q_heads %d: more than 2^24", seqs->n_rows, seqs->n_seq, n_q_heads); return PV_ERANGE; }
    if ((int64_t)seqs->table_pages * pool->page_tokens > (1 << 30)) { pv_set_error("table of %d pages of %d tokens: more than 2^30 tokens", seqs->table_pages, pool->page_tokens); return PV_ERANGE; }
    return PV_OK;
}

extern "C" int pv_kv16_attention_bytes(const pv_kv16_pool *pool, const pv_kv8_seqs *seqs, int32_t n_q_heads, size_t *bytes)
{
    const int rc = check_attention(pool, seqs, n_q_heads);
    if (rc != PV_OK) return rc;
    if (!bytes) { pv_set_error("null output pointer"); return PV_EINVAL; }
    const int group = n_q_heads / pool->n_kv_heads;
    *bytes = seqs->n_seq && seqs->n_rows ? part_bytes(plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, pool->head_dim, (int64_t)seqs->table_pages * pool->page_tokens), seqs->n_rows, n_q_heads, pool->head_dim) : 0;
    return PV_OK;
}

// more dynamic LDS than the default limit: allowed once on each device
template <int HD, typename S>
static int allow_lds()
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    PV_HIP(hipGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return PV_OK;
    PV_HIP(hipFuncSetAttribute((const void *)k_kv16_attn_wide<HD, 1, S>, hipFuncAttributeMaxDynamicSharedMemorySize, kv16_wide<HD>::lds));
    PV_HIP(hipFuncSetAttribute((const void *)k_kv16_attn_wide<HD, 2, S>, hipFuncAttributeMaxDynamicSharedMemorySize, kv16_wide<HD>::lds));
    if (dev < 64) done.fetch_or(bit, std::memory_order_release);
    return PV_OK;
}

template <int HD, typename S>
static int launch(const kv16_attn_args &a, const kv16_plan &p, hipStream_t s)
{
    const dim3 grid(p.units * a.pool.n_heads, p.nsplit);
    if (p.tr == 16) k_kv16_attn<HD, S><<<grid, 256, 0, s>>>(a);
    else {
        if (kv16_wide<HD>::lds > 65536) { const int rc = allow_lds<HD, S>(); if (rc != PV_OK) return rc; }
        if (p.tr == 64) k_kv16_attn_wide<HD, 1, S><<<grid, 256, kv16_wide<HD>::lds, s>>>(a);
        else k_kv16_attn_wide<HD, 2, S><<<grid, 256, kv16_wide<HD>::lds, s>>>(a);
    }
    PV_HIP(hipGetLastError());
    if (p.nsplit == 1) return PV_OK;
    if (p.nsplit > 16) k_kv16_attn_merge<HD, S><<<(unsigned)(a.seqs.n_rows * a.n_q_heads), 256, 0, s>>>(a, p.tr);
    else {
        const int per = (a.n_q_heads + 256 / HD - 1) / (256 / HD);
        k_kv16_attn_join<HD, S><<<(unsigned)(((int64_t)a.seqs.n_rows * per + 3) / 4), 256, 0, s>>>(a, p.tr);
    }
    PV_HIP(hipGetLastError());
    return PV_OK;
}

extern "C" int pv_kv16_attention(const pv_kv16_pool *pool, const pv_kv8_seqs *seqs, const void *q, int64_t q_row_stride, int64_t q_head_stride, int32_t n_q_heads,
                                 const uint64_t *mask, int32_t mask_words, float scale, void *out, int64_t out_row_stride, int64_t out_head_stride, float *lse,
                                 void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_attention(pool, seqs, n_q_heads);
    if (rc != PV_OK) return rc;
    if (mask && (mask_words < 1 || mask_words > (1 << 18))) { pv_set_error("mask_words %d outside [1, 2^18]", mask_words); return PV_ERANGE; }
    if (!(scale - scale == 0.f)) { pv_set_error("scale is not finite"); return PV_EINVAL; }
    if (seqs->n_seq == 0 || seqs->n_rows == 0) return PV_OK;
    if ((rc = pv_kv8_check_rows("q", q, q_row_stride, q_head_stride, pool->dtype)) != PV_OK || (rc = pv_kv8_check_rows("out", out, out_row_stride, out_head_stride, pool->dtype)) != PV_OK) return rc;
    if (((uintptr_t)mask & 7) || ((uintptr_t)lse & 3)) { pv_set_error("mask or lse is not aligned"); return PV_EINVAL; }
    const int group = n_q_heads / pool->n_kv_heads;
    const kv16_plan p = plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, pool->head_dim, (int64_t)seqs->table_pages * pool->page_tokens);
    const size_t need = part_bytes(p, seqs->n_rows, n_q_heads, pool->head_dim);
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    kv16_attn_args a = {};
    a.pool = pv_kv16_pool_args(pool); a.seqs = pv_kv16_seqs_args(seqs);
    a.q = (const char *)q; a.q_row_bytes = q_row_stride * 2; a.q_head_bytes = q_head_stride * 2;
    a.out = (char *)out; a.out_row_bytes = out_row_stride * 2; a.out_head_bytes = out_head_stride * 2;
    a.lse = lse; a.mask = mask; a.words = mask_words; a.group = group; a.n_q_heads = n_q_heads; a.nsplit = p.nsplit; a.chunk = p.chunk;
    a.part_o = (float *)workspace; a.part_ml = a.part_o + (size_t)seqs->n_rows * n_q_heads * p.nsplit * pool->head_dim;
    a.scale2 = scale == 0.f ? 1.f : fabsf(scale) * 1.44269504088896340736f;
    a.q_and = scale == 0.f ? 0u : ~0u; a.q_xor = scale < 0.f ? 0x80008000u : 0u;
    hipStream_t s = (hipStream_t)hip_stream;
    if (pool->head_dim == 128) return pool->dtype == PV_BF16 ? launch<128, __bf16>(a, p, s) : launch<128, _Float16>(a, p, s);
    return pool->dtype == PV_BF16 ? launch<64, __bf16>(a, p, s) : launch<64, _Float16>(a, p, s);
}
