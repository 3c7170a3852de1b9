// Attention over the 8-bit key/value cache (pv_kv8.h) on the matrix cores.
//
// The query rows of a kv head are packed token by token: row m of a sequence is query head m % group of its token m / group.  Everything is computed transposed, as in the
// attention over 16-bit pages: S^T (keys x rows) = K Q^T, O^T (features x rows) = V^T P^T; the accumulators of S^T are, two groups of 16 keys side by side, the second
// operand of the other product.  Codes become bf16 in registers, scale included (v_cvt_scalef32_pk_bf16_fp8: two codes an instruction, exact), so that any
// magnitude of keys and values is what it stands for.  Softmax with the running maximum and sum, all in 32 bits, in powers of two.
// P is carried as bf16 hi + lo: rounded to one bf16 it would add as much error as the rounding of a bf16 output and eight times that of an f16 one; one f16 has no room
// for the weights of many keys beside one that takes nearly all.  q is exact: bf16 as it is, f16 as bf16 hi + lo.
#include <stddef.h>
#include "pv_kv8.h"

enum { KV8_BF16 = 0, KV8_F16 = 1, KV8_STEP1 = 2, KV8_STEP2 = 3 };       // queries and outputs: a caller's, or a model's step (operand layouts of 1 .. 8 rows and of more)

struct kv8_attn_args {
    kv8_pool pool;
    kv8_seqs seqs;
    const char *q; int64_t q_row_bytes, q_head_bytes;
    char *out; int64_t out_row_bytes, out_head_bytes;
    float *lse;
    const uint64_t *mask;
    const uint16_t *q_hi, *q_lo; int q_rows; uint16_t *xop_o;              // a step's
    float *part_o, *part_ml;                // [row][query head][split][HD], [2] (maximum, sum)
    int group, n_q_heads, nsplit, chunk;    // chunk: keys a split, a multiple of 256
    float scale2;                           // scale * log2(e)
};

// Rows of sequence s of the call, cheaply (kv8_seq_at has the rest)
__device__ inline int kv8_rows_of(const kv8_seqs &q, int s)
{
    if (q.st != nullptr) return q.batched ? q.st->blk.seq[s].gamma : q.n_rows;
    const int r0 = q.row_start[s], r = min(q.row_start[s + 1], q.n_rows) - r0;
    return r0 < 0 || r < 0 || q.prefix_len[s] < 0 ? 0 : r;
}

// Tile `unit` of the sequences' rows, TR packed rows a tile, counted through all sequences: its sequence (-1: there are not so many) and its number in it
__device__ inline int kv8_unit(const kv8_seqs &q, int unit, int group, int TR, int &tile)
{
    const int n = q.st != nullptr ? (q.batched ? q.st->blk.n_seq : 1) : q.n_seq, lane = threadIdx.x & 63;
    for (int k = 0; k < n; k += 64) {
        const int mine = k + lane < n ? (kv8_rows_of(q, k + lane) * group + TR - 1) / TR : 0;
        int upto = mine;                    // tiles up to this sequence
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(upto, d, 64); if (lane >= d) upto += o; }
        const uint64_t past = __ballot(upto > unit);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            tile = unit - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
            return k + l;
        }
        unit -= __builtin_amdgcn_readlane(upto, 63);
    }
    return -1;
}

// Keys that exist for a sequence, and those that some row of the tile that ends with token `last` may see
__device__ inline int kv8_keys(const kv8_seq &s, int page_shift, int last, bool masked)
{
    const int64_t want = (int64_t)s.len + (masked ? s.rows : last + 1), there = (int64_t)s.table_pages << page_shift;
    return (int)min(want, there);
}

// Eight codes, two dwords of them with a scale each, as the bf16 operand of a product
typedef __attribute__((ext_vector_type(2))) short kv8_s2;
__device__ inline uint4 kv8_operand(uint32_t a, uint32_t b, float fa, float fb)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, fa, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, fa, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, fb, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, fb, true)));
}

// 0x80 in each byte of a dword of codes that is NaN
__device__ inline uint32_t kv8_nans(uint32_t c)
{
    const uint32_t y = (c & 0x7f7f7f7fu) ^ 0x7f7f7f7fu;
    return ~(((y & 0x7f7f7f7fu) + 0x7f7f7f7fu) | y) & 0x80808080u;
}

// A query row's place: token of the block, query head, whether there is such a row (else the last one's place)
struct kv8_row { int j, head, row; bool live; };
__device__ inline kv8_row kv8_row_at(const kv8_attn_args &a, const kv8_seq &s, int kvh, int m)
{
    kv8_row r;
    const int n = s.rows * a.group;
    r.live = m < n;
    m = min(m, n - 1);
    r.j = m / a.group; r.head = kvh * a.group + (m - r.j * a.group); r.row = s.row0 + r.j;
    return r;
}

// q of features 64 (ks / 2) + 16 g + 8 (ks % 2) ... + 7, the order in which a block's codes lie
template <int HD, int IO, int NQ>
__device__ inline void kv8_load_q(const kv8_attn_args &a, const kv8_row &r, int g, uint4 (&q)[NQ][HD / 32])
{
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks) {
        const int e = 64 * (ks >> 1) + 16 * g + 8 * (ks & 1);
        if constexpr (IO == KV8_BF16) q[0][ks] = *(const uint4 *)(a.q + r.row * a.q_row_bytes + r.head * a.q_head_bytes + e * 2);
        else if constexpr (IO == KV8_F16) {
            const uint4 v = *(const uint4 *)(a.q + r.row * a.q_row_bytes + r.head * a.q_head_bytes + e * 2);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t h[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const f16x2 x = __builtin_bit_cast(f16x2, w[i]); split2((float)x.x, (float)x.y, h[i], l[i]); }
            q[0][ks] = make_uint4(h[0], h[1], h[2], h[3]); q[1][ks] = make_uint4(l[0], l[1], l[2], l[3]);
        } else {
            const size_t at = q_at(r.head, r.row, e, HD, a.q_rows);
            q[0][ks] = *(const uint4 *)(a.q_hi + at); q[1][ks] = *(const uint4 *)(a.q_lo + at);
        }
    }
}

template <int HD, int IO>
__device__ inline void kv8_store4(const kv8_attn_args &a, int row, int head, int e, const float y[4])
{
    if constexpr (IO == KV8_BF16) *(uint2 *)(a.out + row * a.out_row_bytes + head * a.out_head_bytes + e * 2) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
    else if constexpr (IO == KV8_F16) {
        const f16x2 u = {(_Float16)y[0], (_Float16)y[1]}, v = {(_Float16)y[2], (_Float16)y[3]};
        *(uint2 *)(a.out + row * a.out_row_bytes + head * a.out_head_bytes + e * 2) = make_uint2(__builtin_bit_cast(uint32_t, u), __builtin_bit_cast(uint32_t, v));
    } else store_operand4<(IO == KV8_STEP1 ? 1 : 2)>(a.xop_o, a.n_q_heads * HD, row, head * HD + e, y, a.q_rows);
}

// Four groups of 16 keys on their way through a wave
struct kv8_groups {
    int page;                               // lane: physical page of group lane / 16, -1: none
    int sub;                                // and the block in it
    float fk, fv;                           // and its scales
};

// Running result for RT tiles of 16 rows: lane (g, jl) has row jl's maximum and its part of the sum, and features 16 e + 4 g .. + 3
template <int HD, int RT> struct kv8_acc { f32x4 O[RT][HD / 16]; float m[RT], l[RT]; };

// Scores of 64 keys -> weights (bf16 hi, lo) under the new maximum; what was there is scaled to it.  see(t, p): whether the lane's row of tile t may attend to key p.
template <int HD, int RT, typename SEE>
__device__ inline void kv8_softmax(kv8_acc<HD, RT> &A, f32x4 (&S)[RT][4], float scale2, bool edge, SEE see, uint32_t (&P)[RT][4][4])
{
    const int g = (threadIdx.x & 63) >> 4;
    float keep[RT];
    bool same = true;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float mx = A.m[t];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                S[t][q][r] *= scale2;
                if (edge && !see(t, 16 * q + 4 * g + r)) S[t][q][r] = -INFINITY;
                mx = fmaxf(mx, S[t][q][r]);
            }
        mx = with_lane32(with_lane16(mx, op_max), op_max);
        const float ref = mx == -INFINITY ? 0.f : mx;                  // (nothing seen so far)
        keep[t] = __builtin_amdgcn_exp2f(A.m[t] - ref);
        same = same && keep[t] == 1.f;
        float ps = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) { p[r] = __builtin_amdgcn_exp2f(S[t][q][r] - ref); ps += p[r]; }
            split2(p[0], p[1], P[t][q][0], P[t][q][2]);
            split2(p[2], p[3], P[t][q][1], P[t][q][3]);
        }
        A.l[t] = fmaf(A.l[t], keep[t], ps);
        A.m[t] = mx;
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

// One workgroup: a kv head, a tile of 16 RT packed rows of a sequence, a chunk of its keys; the waves take 64 keys in turn and are joined through LDS at the end.
template <int HD, int RT, int IO>
__global__ void __launch_bounds__(256)
k_kv8_attn(const kv8_attn_args a)
{
    constexpr int KB = HD / 64, KS = HD / 32, ET = HD / 16, NQ = IO == KV8_BF16 ? 1 : 2, TR = 16 * RT, OS = 68;
    __shared__ float2 sh_ml[4][TR];
    __shared__ float sh_o[4][TR][OS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jl = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.x % a.pool.n_heads, split = blockIdx.y;       // (the tiles and chunks of a head: on one XCD where the heads are a multiple of eight)
    int tile = 0;
    const int si = __builtin_amdgcn_readfirstlane(kv8_unit(a.seqs, blockIdx.x / a.pool.n_heads, a.group, TR, tile));
    if (si < 0) return;
    const kv8_seq sq = kv8_seq_at<HD>(a.seqs, a.pool, si);
    const int m0 = tile * TR, nrows = sq.rows * a.group, shift = sq.pool.page_shift;
    const int last = (min(m0 + TR, nrows) - 1) / a.group;
    const int nk = __builtin_amdgcn_readfirstlane(kv8_keys(sq, shift, last, a.mask != nullptr)), len = __builtin_amdgcn_readfirstlane(sq.len);
    const int k0 = split * a.chunk, k1 = min(k0 + a.chunk, nk);
    if (k0 >= nk && split > 0) return;      // (a sequence without keys: split 0 writes its rows)
    const bool whole = nk <= a.chunk;

    kv8_row row[RT];
    uint4 q[RT][NQ][KS];
    uint64_t vm[RT];
    kv8_acc<HD, RT> A;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        row[t] = kv8_row_at(a, sq, kvh, m0 + t * 16 + jl);
        kv8_load_q<HD, IO, NQ>(a, row[t], g, q[t]);
        vm[t] = a.mask != nullptr ? a.mask[row[t].row] : 0;
        A.m[t] = -INFINITY; A.l[t] = 0.f;
#pragma unroll
        for (int e = 0; e < ET; ++e) A.O[t][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const uint64_t block = (uint64_t)HD << shift;                        // bytes of a head's keys in a page
    auto groups = [&](int p0) {
        kv8_groups r;
        const int p = p0 + 16 * g;
        r.page = p < nk ? kv8_page(sq, p >> shift) : -1;
        r.sub = (p & ((1 << shift) - 1)) >> 4;
        return r;
    };
    auto scales = [&](kv8_groups &r) {
        const uint32_t b = r.page < 0 ? 0x7f7fu : *(const uint16_t *)(sq.pool.scales + kv8_scale(sq.pool, r.page, kvh, 0, r.sub));
        r.fk = kv8_pow2(kv8_byte(b & 0xffu) - 127); r.fv = kv8_pow2(kv8_byte(b >> 8) - 127);
    };
    for (int p0 = k0 + 64 * wave; p0 < k1; p0 += 256) {
        kv8_groups G = groups(p0);
        scales(G);
        uint4 kt[4][KB], vt[4][KB];
        int bad = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = __builtin_amdgcn_readlane(G.page, 16 * i), sub = __builtin_amdgcn_readlane(G.sub, 16 * i);
            if (page < 0) bad |= 1 << i;
            const uint8_t *kb = sq.pool.codes + ((uint64_t)(uint32_t)max(page, 0) * sq.pool.n_heads + kvh) * 2 * block + sub * (16 * HD);
#pragma unroll
            for (int b = 0; b < KB; ++b) { kt[i][b] = ((const uint4 *)kb)[b * 64 + lane]; vt[i][b] = ((const uint4 *)(kb + block))[b * 64 + lane]; }
        }
        f32x4 S[RT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(G.fk), 16 * i));
#pragma unroll
            for (int t = 0; t < RT; ++t) S[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const uint4 ka = kv8_operand(kt[i][b].x, kt[i][b].y, f, f), kc = kv8_operand(kt[i][b].z, kt[i][b].w, f, f);
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) { S[t][i] = mfma16(ka, q[t][n][2 * b], S[t][i]); S[t][i] = mfma16(kc, q[t][n][2 * b + 1], S[t][i]); }
            }
        }
        const bool edge = p0 + 64 > len || p0 + 64 > nk || bad != 0;
        auto see = [&](int t, int o) {
            const int p = p0 + o, slot = p - len;
            const bool in = a.mask != nullptr ? slot < 0 || (slot < 64 && ((vm[t] >> slot) & 1)) : slot <= row[t].j;
            return in && p < nk && !((bad >> (o >> 4)) & 1);
        };
        uint32_t P[RT][4][4];
        kv8_softmax<HD, RT>(A, S, a.scale2, edge, see, P);
        // values that do not exist are zeros; NaN among those that do is kept from the rows that do not see it: zero in the product, and added where a row does
        bool nans = false;
        if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = ((bad >> i) & 1) ? 0 : min(max(nk - (p0 + 16 * i + 4 * g), 0), 4);
                const uint32_t there = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
                uint32_t any = 0;
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    vt[i][b].x &= there; vt[i][b].y &= there; vt[i][b].z &= there; vt[i][b].w &= there;
                    any |= kv8_nans(vt[i][b].x) | kv8_nans(vt[i][b].y) | kv8_nans(vt[i][b].z) | kv8_nans(vt[i][b].w);
                }
                nans = nans || any != 0;
            }
            nans = __any(nans);
        }
        if (nans) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t seen[RT][4];
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int o = 16 * (2 * u + i / 2) + 4 * g + 2 * (i & 1);
                        seen[t][i] = (see(t, o) ? 0x3f80u : 0u) | (see(t, o + 1) ? 0x3f800000u : 0u);
                    }
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    uint32_t *v0 = &vt[2 * u][b].x, *v1 = &vt[2 * u + 1][b].x;
#pragma unroll
                    for (int f4 = 0; f4 < 4; ++f4) {
                        const uint32_t n0 = kv8_nans(v0[f4]) >> 7, n1 = kv8_nans(v1[f4]) >> 7;          // 1 in each NaN byte
                        v0[f4] &= ~(n0 * 0xffu); v1[f4] &= ~(n1 * 0xffu);
                        auto ones = [](uint32_t n, int at) { return ((n >> at) & 1u) * 0x3f80u | ((n >> (at + 8)) & 1u) * 0x3f800000u; };
                        const uint4 va = make_uint4(ones(n0, 0), ones(n0, 16), ones(n1, 0), ones(n1, 16));
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const f32x4 c = mfma16(va, make_uint4(seen[t][0], seen[t][1], seen[t][2], seen[t][3]), (f32x4){0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int r = 0; r < 4; ++r) if (c[r] > 0.f) A.O[t][4 * b + f4][r] = __uint_as_float(0x7fc00000u);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float f0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(G.fv), 32 * u)), f1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(G.fv), 32 * u + 16));
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const uint32_t v0[4] = {vt[2 * u][b].x, vt[2 * u][b].y, vt[2 * u][b].z, vt[2 * u][b].w}, v1[4] = {vt[2 * u + 1][b].x, vt[2 * u + 1][b].y, vt[2 * u + 1][b].z, vt[2 * u + 1][b].w};
#pragma unroll
                for (int f4 = 0; f4 < 4; ++f4) {
                    const uint4 va = kv8_operand(v0[f4], v1[f4], f0, f1);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        f32x4 &o = A.O[t][4 * b + f4];
                        o = mfma16(va, make_uint4(P[t][2 * u][0], P[t][2 * u][1], P[t][2 * u + 1][0], P[t][2 * u + 1][1]), o);
                        o = mfma16(va, make_uint4(P[t][2 * u][2], P[t][2 * u][3], P[t][2 * u + 1][2], P[t][2 * u + 1][3]), o);
                    }
                }
            }
        }
    }

    // join the waves: each parks its maximum and sum and, 64 features at a time, its output
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        A.l[t] = with_lane32(with_lane16(A.l[t], op_add), op_add);
        if (g == 0) sh_ml[wave][t * 16 + jl] = make_float2(A.m[t], A.l[t]);
    }
#pragma unroll
    for (int part = 0; part < KB; ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) *(f32x4 *)&sh_o[wave][t * 16 + jl][e * 16 + 4 * g] = A.O[t][4 * part + e];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = i * 16 + (threadIdx.x >> 4), c4 = threadIdx.x & 15;
            const kv8_row w = kv8_row_at(a, sq, kvh, m0 + r);
            if (!w.live) continue;
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) M = fmaxf(M, sh_ml[k][r].x);
            const float ref = M == -INFINITY ? 0.f : M;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = __builtin_amdgcn_exp2f(sh_ml[k][r].x - ref);
                const f32x4 v = *(const f32x4 *)&sh_o[k][r][4 * c4];
#pragma unroll
                for (int x = 0; x < 4; ++x) o[x] = fmaf(f, v[x], o[x]);
                L = fmaf(f, sh_ml[k][r].y, L);
            }
            const size_t at = (size_t)w.row * a.n_q_heads + w.head;
            if (whole) {
                const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
                kv8_store4<HD, IO>(a, w.row, w.head, part * 64 + 4 * c4, y);
                if (a.lse != nullptr && part == 0 && c4 == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
            } else {
                *(f32x4 *)(a.part_o + (at * a.nsplit + split) * HD + part * 64 + 4 * c4) = o;
                if (part == 0 && c4 == 0) *(float2 *)(a.part_ml + (at * a.nsplit + split) * 2) = make_float2(M, L);
            }
        }
    }
}

// The chunks of a row's keys joined: a wave a row and query head
template <int HD, int TR, int IO>
__global__ void __launch_bounds__(256)
k_kv8_attn_merge(const kv8_attn_args a)
{
    constexpr int TPC = HD / 4, NG = 64 / TPC;
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int row = __builtin_amdgcn_readfirstlane((int)(id / a.n_q_heads)), head = __builtin_amdgcn_readfirstlane((int)(id % a.n_q_heads));
    if (row >= a.seqs.n_rows) return;
    const int si = __builtin_amdgcn_readfirstlane(kv8_seq_of_row(a.seqs, row));
    if (si < 0) return;
    const kv8_seq sq = kv8_seq_at<HD>(a.seqs, a.pool, si);
    const int j = row - sq.row0;
    if (j < 0 || j >= sq.rows) return;
    const int tile = (j * a.group + head % a.group) / TR, last = (min((tile + 1) * TR, sq.rows * a.group) - 1) / a.group;
    const int nk = kv8_keys(sq, sq.pool.page_shift, last, a.mask != nullptr);
    if (nk <= a.chunk) return;              // (written already)
    const int n = (nk + a.chunk - 1) / a.chunk;
    const size_t at = (size_t)row * a.n_q_heads + head;
    const float2 *ml = (const float2 *)(a.part_ml + at * a.nsplit * 2);
    const float *po = a.part_o + at * a.nsplit * HD;
    float M = -INFINITY, L = 0.f;
    for (int c = lane; c < n; c += 64) M = fmaxf(M, ml[c].x);
    M = over_wave(M, op_max);
    const float ref = M == -INFINITY ? 0.f : M;
    for (int c = lane; c < n; c += 64) L = fmaf(ml[c].y, __builtin_amdgcn_exp2f(ml[c].x - ref), L);
    L = over_wave(L, op_add);
    const int t = lane % TPC, cg = lane / TPC;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c = cg; c < n; c += NG) {
        const float w = __builtin_amdgcn_exp2f(ml[c].x - ref);
        const float4 v = *(const float4 *)(po + (size_t)c * HD + 4 * t);
        o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]); o[2] = fmaf(w, v.z, o[2]); o[3] = fmaf(w, v.w, o[3]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { o[i] = with_lane32(o[i], op_add); if (TPC <= 16) o[i] = with_lane16(o[i], op_add); }
    if (lane >= TPC) return;
    const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    kv8_store4<HD, IO>(a, row, head, 4 * t, y);
    if (a.lse != nullptr && lane == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
}

// ------------------------------- host side ----------------------------------------

// How a call's work is cut
struct kv8_plan { int rt, units, nsplit, chunk; };

static kv8_plan plan(int n_seq, int n_rows, int group, int kv_heads, int64_t keys)
{
    kv8_plan p;
    p.rt = (int64_t)n_rows * group > (int64_t)16 * n_seq ? 2 : 1;
    p.units = (int)(((int64_t)n_rows * group) / (16 * p.rt)) + n_seq;
    const int64_t base = (int64_t)p.units * kv_heads, most = (keys + 255) / 256;
    int64_t n = (2048 + base - 1) / base;
    n = n < most ? n : most;
    n = n < 256 ? n : 256;
    n = n > 1 ? n : 1;
    p.chunk = (int)(((keys + n - 1) / n + 255) / 256 * 256);
    p.chunk = p.chunk > 256 ? p.chunk : 256;
    p.nsplit = (int)((keys + p.chunk - 1) / p.chunk);
    p.nsplit = p.nsplit > 1 ? p.nsplit : 1;
    return p;
}

static size_t part_bytes(const kv8_plan &p, int n_rows, int n_q_heads, int hd)
{
    return p.nsplit > 1 ? (size_t)n_rows * n_q_heads * p.nsplit * (hd + 2) * sizeof(float) : 0;
}

static int check_attention(const pv_kv8_pool *pool, const pv_kv8_seqs *seqs, int n_q_heads)
{
    int rc;
    if ((rc = pv_kv8_check_pool(pool)) != PV_OK || (rc = pv_kv8_check_seqs(seqs)) != PV_OK) return rc;
    if (n_q_heads < 1 || n_q_heads % pool->n_kv_heads) { pv_set_error("n_q_heads %d is not a multiple of n_kv_heads %d", n_q_heads, pool->n_kv_heads); return PV_EINVAL; }
    if (((int64_t)seqs->n_rows + seqs->n_seq) * n_q_heads > (1 << 24)) { pv_set_error("(n_rows %d + n_seq %d) x n_q_heads %d: more than 2^24", seqs->n_rows, seqs->n_seq, n_q_heads); return PV_ERANGE; }
    if ((int64_t)seqs->table_pages * pool->page_tokens > (1 << 30)) { pv_set_error("table of %d pages of %d tokens: more than 2^30 tokens", seqs->table_pages, pool->page_tokens); return PV_ERANGE; }
    return PV_OK;
}

extern "C" int pv_kv8_attention_bytes(const pv_kv8_pool *pool, const pv_kv8_seqs *seqs, int32_t n_q_heads, size_t *bytes)
{
    const int rc = check_attention(pool, seqs, n_q_heads);
    if (rc != PV_OK) return rc;
    if (!bytes) { pv_set_error("null output pointer"); return PV_EINVAL; }
    const int group = n_q_heads / pool->n_kv_heads;
    *bytes = seqs->n_seq && seqs->n_rows ? part_bytes(plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, (int64_t)seqs->table_pages * pool->page_tokens), seqs->n_rows, n_q_heads, pool->head_dim) : 0;
    return PV_OK;
}

template <int HD, int RT, int IO>
static int launch2(const kv8_attn_args &a, const kv8_plan &p, hipStream_t s)
{
    k_kv8_attn<HD, RT, IO><<<dim3(p.units * a.pool.n_heads, p.nsplit), 256, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    if (p.nsplit > 1) {
        const int64_t waves = (int64_t)a.seqs.n_rows * a.n_q_heads;
        k_kv8_attn_merge<HD, 16 * RT, IO><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(a);
        PV_HIP(hipGetLastError());
    }
    return PV_OK;
}

template <int HD, int IO>
static int launch(const kv8_attn_args &a, const kv8_plan &p, hipStream_t s) { return p.rt == 1 ? launch2<HD, 1, IO>(a, p, s) : launch2<HD, 2, IO>(a, p, s); }

extern "C" int pv_kv8_attention(const pv_kv8_pool *pool, const pv_kv8_seqs *seqs, const void *q, int64_t q_row_stride, int64_t q_head_stride, int32_t n_q_heads,
                                const uint64_t *mask, float scale, void *out, int64_t out_row_stride, int64_t out_head_stride, float *lse, int32_t dtype,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_attention(pool, seqs, n_q_heads);
    if (rc != PV_OK) return rc;
    if (seqs->n_seq == 0 || seqs->n_rows == 0) return PV_OK;
    if (dtype != PV_BF16 && dtype != PV_F16) { pv_set_error("attention over an 8-bit cache: queries in bf16 or f16"); return PV_EINVAL; }
    if ((rc = pv_kv8_check_rows("q", q, q_row_stride, q_head_stride, dtype)) != PV_OK || (rc = pv_kv8_check_rows("out", out, out_row_stride, out_head_stride, dtype)) != PV_OK) return rc;
    if (!(scale - scale == 0.f)) { pv_set_error("scale is not finite"); return PV_EINVAL; }
    if (((uintptr_t)mask & 7) || ((uintptr_t)lse & 3)) { pv_set_error("mask or lse is not aligned"); return PV_EINVAL; }
    const int group = n_q_heads / pool->n_kv_heads;
    const kv8_plan p = plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, (int64_t)seqs->table_pages * pool->page_tokens);
    const size_t need = part_bytes(p, seqs->n_rows, n_q_heads, pool->head_dim);
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    kv8_attn_args a = {};
    a.pool = pv_kv8_pool_args(pool); a.seqs = pv_kv8_seqs_args(seqs);
    a.q = (const char *)q; a.q_row_bytes = q_row_stride * 2; a.q_head_bytes = q_head_stride * 2;
    a.out = (char *)out; a.out_row_bytes = out_row_stride * 2; a.out_head_bytes = out_head_stride * 2;
    a.lse = lse; a.mask = mask; a.group = group; a.n_q_heads = n_q_heads; a.nsplit = p.nsplit; a.chunk = p.chunk;
    a.part_o = (float *)workspace; a.part_ml = a.part_o + (size_t)seqs->n_rows * n_q_heads * p.nsplit * pool->head_dim;
    a.scale2 = scale * 1.44269504088896340736f;
    hipStream_t s = (hipStream_t)hip_stream;
    if (pool->head_dim == 128) return dtype == PV_BF16 ? launch<128, KV8_BF16>(a, p, s) : launch<128, KV8_F16>(a, p, s);
    return dtype == PV_BF16 ? launch<64, KV8_BF16>(a, p, s) : launch<64, KV8_F16>(a, p, s);
}

// ---- a model's step ----
int pv_kv8_step_attention(pv_cache *c, const pv_kv8_step &st, hipStream_t s)
{
    const pv_model_config &f = c->m->cfg;
    kv8_attn_args a = {};
    a.seqs = pv_kv8_step_seqs(c, st.layer, st.rows, -1, &a.pool);
    a.group = f.n_q_heads / f.n_kv_heads; a.n_q_heads = f.n_q_heads;
    const int64_t room = (int64_t)c->n_pages * f.page_tokens, keys = st.prompt ? c->len + st.rows : c->attn_keys > 0 && c->attn_keys < room ? c->attn_keys : room;
    kv8_plan p = plan(a.seqs.n_seq, st.rows, a.group, f.n_kv_heads, keys);
    while (p.nsplit > 1 && part_bytes(p, st.rows, f.n_q_heads, f.head_dim) > st.n_part * sizeof(float)) { p.chunk *= 2; p.nsplit = (int)((keys + p.chunk - 1) / p.chunk); }
    // a recorded step serves all lengths up to its bound
    a.nsplit = p.nsplit; a.chunk = p.chunk;
    a.part_o = st.part; a.part_ml = st.part + (size_t)st.rows * f.n_q_heads * p.nsplit * f.head_dim;
    a.q_hi = st.q_hi; a.q_lo = st.q_lo; a.q_rows = st.q_rows; a.xop_o = st.xop_o;
    a.mask = st.prompt ? nullptr : (const uint64_t *)((const char *)c->ws.state + offsetof(pv_dev_state, rowmask));
    a.scale2 = 1.44269504088896340736f / sqrtf((float)f.head_dim);
    const bool packed = !st.prompt && pv_packs_rows(c->m, st.rows);
    if (f.head_dim == 128) return packed ? launch<128, KV8_STEP1>(a, p, s) : launch<128, KV8_STEP2>(a, p, s);
    return packed ? launch<64, KV8_STEP1>(a, p, s) : launch<64, KV8_STEP2>(a, p, s);
}
