// Attention over the 8-bit key/value cache (pv_kv8.h) on the matrix cores.
//
// The query rows of a kv head are packed token by token: row m of a sequence is query head m % group of its token m / group.  Everything is computed transposed, as in the
// attention over 16-bit pages: S^T (keys x rows) = K Q^T, O^T (features x rows) = V^T P^T; the accumulators of S^T are, two groups of 16 keys side by side, the second
// operand of the other product.  Softmax with the running maximum and sum, all in 32 bits, in powers of two.
//
// Types of the products (codes become 16-bit numbers two an instruction, exactly):
//   K   bf16 with its scale (a bf16 q has bf16's range), or f16 without, the scale then multiplying the scores (f16 q).  A step's q is a bf16 pair, two products.
//   V   f16 without its scale.  P = 2^15 times the weight, f16: 11 significant bits for weights from 2^-29 on, so that many small ones beside one that takes nearly all count fully; one bf16
//       would add as much error as the rounding of a bf16 output.  For f16 outputs P is a pair of f16, or its rounding would be as large as theirs (in a step, whose keys and values have four bits, one is enough).
//       V's scales 2^ev go into the weights' exponents, relative to the unit of the accumulators, 2^E, the largest so far; where one is below 2^-14 of that, the
//       groups of 16 keys are gone through one after the other, each in its own unit, down to 2^-64 of the largest so far (pv_kv8_units.h: what is further below adds nothing).
#include <atomic>
#include <stddef.h>
#include "pv_kv8.h"
#include "pv_kv8_units.h"

enum { KV8_BF16 = 0, KV8_F16 = 1, KV8_STEP1 = 2, KV8_STEP2 = 3 };       // queries and outputs: a caller's, or a model's step (operand layouts of 1 .. 8 rows and of more)
template <int IO> struct kv8_types {
    static constexpr bool half = IO == KV8_F16;                            // K and q in f16
    static constexpr int NQ = IO >= KV8_STEP1 ? 2 : 1, NP = IO == KV8_F16 ? 2 : 1;
};

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
    float scale2;                           // |scale| log2(e), more than 0 (a scale of 0: 1, and q is 0)
    uint32_t q_and, q_xor;                  // what q passes through: its sign is the scale's
};

// A lane's value added to those of the lanes before it
__device__ inline int kv8_sums(int v)
{
#define KV8_STEP(C, M) v += __builtin_amdgcn_update_dpp(0, v, C, M, 0xF, false)
    KV8_STEP(0x111, 0xF); KV8_STEP(0x112, 0xF); KV8_STEP(0x114, 0xF); KV8_STEP(0x118, 0xF);      // within 16 lanes
    KV8_STEP(0x142, 0xA); KV8_STEP(0x143, 0xC);                                                  // lane 15 to the next 16, lane 31 to the upper half
#undef KV8_STEP
    return v;
}

// Tile `unit` of the sequences' rows, TR packed rows a tile, counted through all sequences: its sequence and its number in it (false: there are not so many).  A sequence's tables are asked for
// at once, 64 sequences at a time: one trip to memory in most calls.
template <int HD, int TR> __device__ inline bool kv8_unit(const kv8_seqs &q, const kv8_pool &own, int unit, int group, kv8_seq &s, int &tile)
{
    const int lane = threadIdx.x & 63;
    if (q.st != nullptr) {
        if (!q.batched) { s = kv8_seq_at<HD>(q, own, 0); tile = unit; return tile * TR < s.rows * group; }
        const int mine = lane < q.n_seq ? (q.st->blk.seq[lane].gamma * group + TR - 1) / TR : 0, upto = kv8_sums(mine);
        const uint64_t past = __ballot(upto > unit);
        if (!past) return false;
        const int l = __ffsll((unsigned long long)past) - 1;
        tile = unit - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
        s = kv8_seq_at<HD>(q, own, l);
        return true;
    }
    for (int k = 0; k < q.n_seq; k += 64) {
        const int i = min(k + lane, q.n_seq - 1), r0 = q.row_start[i], r1 = q.row_start[i + 1], len = q.prefix_len[i], r = min(r1, q.n_rows) - r0;
        const int rows = k + lane >= q.n_seq || r0 < 0 || r < 0 || len < 0 ? 0 : r;
        const int mine = (rows * group + TR - 1) / TR, upto = kv8_sums(mine);
        const uint64_t past = __ballot(upto > unit);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            tile = unit - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
            s.pool = own; s.table = q.page_table + (size_t)(k + l) * q.table_pages; s.table_pages = q.table_pages;
            s.row0 = __builtin_amdgcn_readlane(r0, l); s.rows = __builtin_amdgcn_readlane(rows, l); s.len = __builtin_amdgcn_readlane(len, l);
            return true;
        }
        unit -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Keys that exist for a sequence, and those that some row of the tile that ends with token `last` may see
__device__ inline int kv8_keys(const kv8_seq &s, int page_shift, int last, bool masked)
{
    const int64_t want = (int64_t)s.len + (masked ? s.rows : last + 1), there = (int64_t)s.table_pages << page_shift;
    return (int)min(want, there);
}

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
__device__ inline f32x4 mfma16h(uint4 a, uint4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0); }

// Codes as 16-bit numbers, four of a dword at a time: f16, and bf16 times a power of two
__device__ inline uint2 kv8_f16(uint32_t c)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.f, true)));
}
__device__ inline uint2 kv8_bf16(uint32_t c, float f)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, f, true)));
}
template <bool HALF> __device__ inline uint4 kv8_key(uint32_t a, uint32_t b, float f)
{
    const uint2 u = HALF ? kv8_f16(a) : kv8_bf16(a, f), v = HALF ? kv8_f16(b) : kv8_bf16(b, f);
    return make_uint4(u.x, u.y, v.x, v.y);
}
template <bool HALF> __device__ inline f32x4 kv8_score(uint4 k, uint4 q, f32x4 s) { return HALF ? mfma16h(k, q, s) : mfma16(k, q, s); }

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
        if constexpr (NQ == 1) {
            const uint4 v = *(const uint4 *)(a.q + r.row * a.q_row_bytes + r.head * a.q_head_bytes + e * 2);
            q[0][ks] = make_uint4((v.x & a.q_and) ^ a.q_xor, (v.y & a.q_and) ^ a.q_xor, (v.z & a.q_and) ^ a.q_xor, (v.w & a.q_and) ^ a.q_xor);
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

// Running result for RT tiles of 16 rows: lane (g, jl) has row jl's maximum and its part of 2^15 times the sum, and features 16 e + 4 g .. + 3 of the output times 2^(15 - E)
template <int HD, int RT> struct kv8_acc { f32x4 O[RT][HD / 16]; float m[RT], l[RT]; int E, top; };       // E, top: kv8_next_unit

template <int HD, int RT> __device__ inline void kv8_begin(kv8_acc<HD, RT> &A)
{
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        A.m[t] = -INFINITY; A.l[t] = 0.f;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) A.O[t][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    A.E = A.top = KV8_NO_SCALE;
}

// The accumulators in another unit
template <int HD, int RT> __device__ inline void kv8_unit_is(kv8_acc<HD, RT> &A, int E)
{
    if (A.E != KV8_NO_SCALE) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < HD / 16; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) A.O[t][e][r] = ldexpf(A.O[t][e][r], A.E - E);
    }
    A.E = E;
}

// The unit for four groups of V's exponents (kv8_next_unit)
template <int HD, int RT> __device__ inline void kv8_units(kv8_acc<HD, RT> &A, const int (&ev)[4], int (&dv)[4], int &only)
{
    int E = A.E;
    kv8_next_unit(ev, E, A.top, dv, only);
    if (E != A.E) kv8_unit_is(A, E);
}

// Which of 64 keys a row sees: those before `end`, without a mask; with one, those before len, and from there on those that the mask names, before nk.  Bit i: key p + i.
__device__ inline uint64_t kv8_first(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ inline uint64_t kv8_sees(bool masked, uint64_t mask, int p, int len, int end, int nk)
{
    uint64_t w = kv8_first(min(end, nk) - p);
    if (masked) {
        const int s = len - p;
        const uint64_t m = s >= 64 ? 0ull : s >= 0 ? mask << s : s > -64 ? mask >> -s : 0ull;
        w = (kv8_first(s) | m) & kv8_first(nk - p);
    }
    return w;
}

// The larger of two, as one instruction: fmaxf first makes quiet NaN of NaN of numbers that come out of a product, one more instruction for each (two prompts of 2048 rows 440 -> 429 us).
// (NaN and a number: the number; two NaN: infinity, with which the row's weights are NaN too)
__device__ inline float kv8_max(float a, float b)
{
    float top = INFINITY;
    asm("" : "+s"(top));                     // (or the compiler sees fmaxf in it)
    return __builtin_amdgcn_fmed3f(a, b, top);
}

// Scores of 64 keys -> weights under the new maximum (P[tile][group]: keys 4 g .. + 3; PL: what f16 leaves of them, where that counts); what was there is scaled to it.  fk: K's scales where the scores lack them; see(t): which
// of the keys from 4 g on the lane's row of tile t may attend to, a bit each.
template <int HD, int RT, int IO, typename SEE>
__device__ inline void kv8_softmax(kv8_acc<HD, RT> &A, f32x4 (&S)[RT][4], float scale2, const float (&fk)[4], bool edge, SEE see, const int (&dv)[4], uint2 (&P)[RT][4], uint2 (&PL)[RT][4])
{
    constexpr bool HALF = kv8_types<IO>::half;
    float keep[RT], add[4], back[4];
    bool same = true;
#pragma unroll
    for (int q = 0; q < 4; ++q) { add[q] = (float)dv[q]; back[q] = kv8_pow2(-dv[q]); }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float mx = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float f = scale2 * fk[q];
#pragma unroll
            for (int r = 0; r < 4; ++r) if (HALF) S[t][q][r] *= f;
        }
        if (edge) {
            const uint64_t w = see(t);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][q][r] = ((w >> (16 * q + r)) & 1) ? S[t][q][r] : -INFINITY;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            mx = kv8_max(kv8_max(mx, kv8_max(S[t][q][0], S[t][q][1])), kv8_max(S[t][q][2], S[t][q][3]));
        }
        mx = with_lane32(with_lane16(mx, kv8_max), kv8_max);
        if (!HALF) mx *= scale2;
        mx = fmaxf(mx, A.m[t]);
        const float ref = mx == -INFINITY ? 0.f : mx;                  // (nothing seen so far)
        keep[t] = __builtin_amdgcn_exp2f(A.m[t] - ref);
        same = same && keep[t] == 1.f;
        float ps = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float c = (15.f - ref) + add[q];
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(HALF ? S[t][q][r] + c : fmaf(S[t][q][r], scale2, c));
            ps = fmaf((p[0] + p[1]) + (p[2] + p[3]), back[q], ps);
            const f16x2 a = {(_Float16)p[0], (_Float16)p[1]}, b = {(_Float16)p[2], (_Float16)p[3]};
            P[t][q] = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
            if constexpr (kv8_types<IO>::NP == 2) {
                const f16x2 al = {(_Float16)(p[0] - (float)a.x), (_Float16)(p[1] - (float)a.y)}, bl = {(_Float16)(p[2] - (float)b.x), (_Float16)(p[3] - (float)b.y)};
                PL[t][q] = make_uint2(__builtin_bit_cast(uint32_t, al), __builtin_bit_cast(uint32_t, bl));
            }
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

// O += V^T P^T of 64 keys; v(u, e): tile e of groups 2 u and 2 u + 1, f16
template <int HD, int RT, int IO, typename V>
__device__ inline void kv8_output(kv8_acc<HD, RT> &A, const uint2 (&P)[RT][4], const uint2 (&PL)[RT][4], V v)
{
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) {
            const uint4 va = v(u, e);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                A.O[t][e] = mfma16h(va, make_uint4(P[t][2 * u].x, P[t][2 * u].y, P[t][2 * u + 1].x, P[t][2 * u + 1].y), A.O[t][e]);
                if constexpr (kv8_types<IO>::NP == 2) A.O[t][e] = mfma16h(va, make_uint4(PL[t][2 * u].x, PL[t][2 * u].y, PL[t][2 * u + 1].x, PL[t][2 * u + 1].y), A.O[t][e]);
            }
            if (e & 1) __builtin_amdgcn_sched_barrier(0);                // (or the codes of all tiles are converted first, and no registers are left)
        }
}

// Values that are NaN are kept from the rows that do not see them: the products are made without (kv8_without_nans), and in the end the outputs of rows that see one become NaN.  64 keys; v(q, b): a
// lane's 16 codes of group q.
template <int HD, int RT, typename SEE, typename V>
__device__ inline void kv8_put_nans(kv8_acc<HD, RT> &A, SEE see, V v)
{
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint4 seen[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const uint64_t w = see(t);
            auto two = [&](int i) { const int o = 16 * (2 * u + i / 2) + 2 * (i & 1); return (uint32_t)((w >> o) & 1) * 0x3f80u | (uint32_t)((w >> (o + 1)) & 1) * 0x3f800000u; };
            seen[t] = make_uint4(two(0), two(1), two(2), two(3));
        }
#pragma unroll
        for (int b = 0; b < HD / 64; ++b) {
            const uint4 c0 = v(2 * u, b), c1 = v(2 * u + 1, b);
            const uint32_t v0[4] = {c0.x, c0.y, c0.z, c0.w}, v1[4] = {c1.x, c1.y, c1.z, c1.w};
#pragma unroll
            for (int f4 = 0; f4 < 4; ++f4) {
                const uint32_t n0 = kv8_nans(v0[f4]) >> 7, n1 = kv8_nans(v1[f4]) >> 7;          // 1 in each NaN byte
                auto ones = [](uint32_t n, int at) { return ((n >> at) & 1u) * 0x3f80u | ((n >> (at + 8)) & 1u) * 0x3f800000u; };
                const uint4 va = make_uint4(ones(n0, 0), ones(n0, 16), ones(n1, 0), ones(n1, 16));
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const f32x4 c = mfma16(va, seen[t], (f32x4){0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; ++r) if (c[r] > 0.f) A.O[t][4 * b + f4][r] = __uint_as_float(0x7fc00000u);
                }
            }
        }
    }
}
__device__ inline uint32_t kv8_without_nans(uint32_t c) { return c & ~((kv8_nans(c) >> 7) * 0xffu); }
// what of a dword of V's codes (tokens 4 g ...) lies before the end: n tokens of the group exist
__device__ inline uint32_t kv8_there(int n, int g) { const int k = min(max(n - 4 * g, 0), 4); return k == 4 ? 0xffffffffu : (1u << (8 * k)) - 1; }

// a row's output and lse, or its chunk's part of them
template <int HD, int IO>
__device__ inline void kv8_finish4(const kv8_attn_args &a, const kv8_row &w, int e, const float o[4], float M, float L, bool whole, int split)
{
    const size_t at = (size_t)w.row * a.n_q_heads + w.head;
    if (whole) {
        const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        kv8_store4<HD, IO>(a, w.row, w.head, e, y);
        if (a.lse != nullptr && e == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
    } else {
        *(float4 *)(a.part_o + (at * a.nsplit + split) * HD + e) = make_float4(o[0], o[1], o[2], o[3]);
        if (e == 0) *(float2 *)(a.part_ml + (at * a.nsplit + split) * 2) = make_float2(M, L);
    }
}

// Few rows: one workgroup is a kv head, a tile of 16 packed rows of a sequence, a chunk of its keys; the waves take 64 keys in turn, straight from memory to registers, and are joined
// through LDS at the end.  Bound by the read of the codes: the next 64 keys' K is asked for when this one's scores are there, V when its products are.  32 sequences of up to 8192 keys, one row of 32
// heads each: 44.7 us and 4.6 for the chunks' join, 266 MB at 5.9 TB/s (a read stream: 6.55); one sequence of four rows over 65000 keys 25.7 and 4.6, 133 MB at 5.2.
template <int HD, int IO>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_kv8_attn(const kv8_attn_args a)
{
    constexpr int KB = HD / 64, KS = HD / 32, NQ = kv8_types<IO>::NQ, RT = 1, TR = 16, OS = 68;
    constexpr bool HALF = kv8_types<IO>::half;
    __shared__ float2 sh_ml[4][TR];
    __shared__ float sh_o[4][TR][OS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jl = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.x % a.pool.n_heads, split = blockIdx.y;       // (the tiles and chunks of a head: on one XCD where the heads are a multiple of eight)
    int tile = 0;
    kv8_seq sq;
    if (!kv8_unit<HD, TR>(a.seqs, a.pool, blockIdx.x / a.pool.n_heads, a.group, sq, tile)) return;
    const int m0 = tile * TR, nrows = sq.rows * a.group, shift = sq.pool.page_shift;
    const int last = (min(m0 + TR, nrows) - 1) / a.group;
    const int nk = __builtin_amdgcn_readfirstlane(kv8_keys(sq, shift, last, a.mask != nullptr)), len = __builtin_amdgcn_readfirstlane(min(sq.len, 1 << 30));     // (no table goes further)
    const int k0 = split * a.chunk, k1 = min(k0 + a.chunk, nk);
    if (k0 >= nk && split > 0) return;      // (a sequence without keys: split 0 writes its rows)
    const bool whole = nk <= a.chunk;
    const int sure = min(nk, a.mask != nullptr ? len : len + m0 / a.group + 1);     // keys before this one are seen by every row

    // the four groups of 16 keys from p0 on: their table entries, known two turns ahead, and, in lanes 16 i .., group i's scales' bytes
    const uint32_t block = (uint32_t)HD << shift, page_codes = 2 * block * sq.pool.n_heads, page_scales = sq.pool.n_heads << (shift - 3), in_page = (1u << shift) - 1;    // bytes of a head's keys in a page, ...
    const uint8_t *codes = sq.pool.codes + (size_t)kvh * 2 * block, *scales = sq.pool.scales + (kvh << (shift - 3));
    int page[4] = {-1, -1, -1, -1}, ahead[4];
    uint32_t bytes = 0;
    auto pages = [&](int p0, int (&to)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = kv8_entry(sq, (p0 + 16 * i) >> shift);
    };
    auto exists = [&](int p0, int i) { return (int)(p0 + 16 * i < k1) & (int)kv8_is_page(sq, page[i]); };       // (k1 does not lie behind the table's end)
    // Every load is made, without a branch, through a descriptor of no bytes where there is no such group: it reads nothing then and gives zeros.  (The compiler counts the loads behind the one that it
    // waits for and takes the least of all ways to a place: with loads that may not be there it waited for V before the scores: 32 sequences of 1..8192 keys 52.7 -> 50.5 us)
    uint4 kt[4][KB], vt[4][KB];
    __amdgpu_buffer_rsrc_t from[4];
    int bad = 0;
    auto load_16 = [&](int i, uint32_t off, int b) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from[i], off + lane * 16 + b * 1024, 0, 2);      // (2: each code is read once, and past the caches)
        return make_uint4(v.x, v.y, v.z, v.w);
    };
    auto load_k = [&](int p0) {
        bad = 0;
        int at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const int ok = exists(p0, i); bad |= (ok ^ 1) << i; at[i] = ok ? page[i] : 0; }
        const int mine = g == 0 ? at[0] : g == 1 ? at[1] : g == 2 ? at[2] : at[3];
        bytes = *(const uint16_t *)(scales + ((uint64_t)(uint32_t)mine * page_scales + (((p0 + 16 * g) & in_page) >> 3)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t *base = uniform_ptr(codes + ((uint64_t)(uint32_t)at[i] * page_codes + ((p0 + 16 * i) & in_page) * HD));
            from[i] = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (bad >> i) & 1 ? 0 : (int)(block + 16 * HD), 0x00027000);
#pragma unroll
            for (int b = 0; b < KB; ++b) kt[i][b] = load_16(i, 0, b);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < KB; ++b) vt[i][b] = load_16(i, block, b);
    };

    int p0 = k0 + 64 * wave;
    if (p0 < k1) pages(p0, page);
    kv8_row row[RT];
    uint4 q[RT][NQ][KS];
    uint64_t vm[RT];
    kv8_acc<HD, RT> A;
    kv8_begin(A);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        row[t] = kv8_row_at(a, sq, kvh, m0 + t * 16 + jl);
        kv8_load_q<HD, IO, NQ>(a, row[t], g, q[t]);
        vm[t] = a.mask != nullptr ? a.mask[row[t].row] : 0;
    }
    asm volatile("" ::: "memory");
    load_k(p0);
    load_v();
    auto sees = [&](int t, int p) { return kv8_sees(a.mask != nullptr, vm[t], p + 4 * g, len, len + row[t].j + 1, nk); };
    bool spoilt = false;                    // NaN among values that not every row sees, or beside a page that does not exist
    int only = -1;
    ahead[0] = ahead[1] = ahead[2] = ahead[3] = -1;
    if (p0 < k1) pages(p0 + 256, ahead);
    while (p0 < k1) {
        const int miss = bad;
        float fk[4];
        int ev[4], dv[4];
        const int fk_bits = kv8_byte(bytes & 0xffu) << 23, e_v = (miss >> g) & 1 ? KV8_NO_SCALE : kv8_byte(bytes >> 8) - 127;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fk[i] = __uint_as_float(__builtin_amdgcn_readlane(fk_bits, 16 * i));
            ev[i] = __builtin_amdgcn_readlane(e_v, 16 * i);
        }
        f32x4 S[RT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int t = 0; t < RT; ++t) S[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const uint4 ka = kv8_key<HALF>(kt[i][b].x, kt[i][b].y, fk[i]), kc = kv8_key<HALF>(kt[i][b].z, kt[i][b].w, fk[i]);
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) { S[t][i] = kv8_score<HALF>(ka, q[t][n][2 * b], S[t][i]); S[t][i] = kv8_score<HALF>(kc, q[t][n][2 * b + 1], S[t][i]); }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        kv8_units(A, ev, dv, only);
        const int without = miss | (only < 0 ? 0 : 15 & ~(1 << only));    // groups that are not looked at
        const bool last_keys = p0 + 64 > sure || miss != 0, edge = last_keys || without != 0;
        uint64_t there = ~0ull;
        if (without) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if ((without >> i) & 1) there &= ~(0xffffull << (16 * i));
        }
        auto see = [&](int t) { return sees(t, p0) & there; };
        uint2 P[RT][4], PL[RT][4];
        // the next 64 keys, or these again
        const bool through = only < 0 || only == 3;
        const int p1 = through ? p0 + 256 : p0;
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = through ? ahead[i] : page[i];
        load_k(p1);
        pages(p1 + 256, ahead);
        kv8_softmax<HD, RT, IO>(A, S, a.scale2, fk, edge, see, dv, P, PL);
        if (last_keys) {
            bool nans = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t there = ((miss >> i) & 1) ? 0u : kv8_there(nk - (p0 + 16 * i), g);
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    vt[i][b].x &= there; vt[i][b].y &= there; vt[i][b].z &= there; vt[i][b].w &= there;
                    nans = nans || (kv8_nans(vt[i][b].x) | kv8_nans(vt[i][b].y) | kv8_nans(vt[i][b].z) | kv8_nans(vt[i][b].w)) != 0;
                }
            }
            if (__any(nans)) {
                spoilt = true;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < KB; ++b)
                        vt[i][b] = make_uint4(kv8_without_nans(vt[i][b].x), kv8_without_nans(vt[i][b].y), kv8_without_nans(vt[i][b].z), kv8_without_nans(vt[i][b].w));
            }
        }
        kv8_output<HD, RT, IO>(A, P, PL, [&](int u, int e) {
            auto part = [&](int i) { const uint4 c = vt[i][e / 4]; return kv8_f16(e % 4 == 0 ? c.x : e % 4 == 1 ? c.y : e % 4 == 2 ? c.z : c.w); };
            const uint2 x = part(2 * u), y = part(2 * u + 1);
            return make_uint4(x.x, x.y, y.x, y.y);
        });
        only = through ? -1 : only + 1;
        p0 = p1;
        load_v();
    }
    if (spoilt) {
        for (p0 = k0 + 64 * wave; p0 < k1; p0 += 256) {
            pages(p0, page);
            if (p0 + 64 <= sure && exists(p0, 0) & exists(p0, 1) & exists(p0, 2) & exists(p0, 3)) continue;      // (their NaN went through the products)
            kv8_put_nans<HD, RT>(A, [&](int t) { return sees(t, p0); }, [&](int i, int b) {
                if (!exists(p0, i)) return make_uint4(0u, 0u, 0u, 0u);
                const uint4 c = ((const uint4 *)(codes + ((uint64_t)(uint32_t)page[i] * page_codes + block + ((p0 + 16 * i) & in_page) * HD)))[b * 64 + lane];
                const uint32_t there = kv8_there(nk - (p0 + 16 * i), g);
                return make_uint4(c.x & there, c.y & there, c.z & there, c.w & there);
            });
        }
    }

    // join the waves: each parks its maximum and sum and, 64 features at a time, its output
    const int E = A.E == KV8_NO_SCALE ? 0 : A.E;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        A.l[t] = with_lane32(with_lane16(A.l[t], op_add), op_add);
        if (g == 0) sh_ml[wave][t * 16 + jl] = make_float2(A.m[t], A.l[t] * 0x1p-15f);
    }
#pragma unroll
    for (int part = 0; part < KB; ++part) {
        if (part) __syncthreads();
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 o = A.O[t][4 * part + e];
                *(float4 *)&sh_o[wave][t * 16 + jl][e * 16 + 4 * g] = make_float4(ldexpf(o[0], E - 15), ldexpf(o[1], E - 15), ldexpf(o[2], E - 15), ldexpf(o[3], E - 15));
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = i * 16 + (threadIdx.x >> 4), c4 = threadIdx.x & 15;
            const kv8_row w = kv8_row_at(a, sq, kvh, m0 + r);
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
            kv8_finish4<HD, IO>(a, w, part * 64 + 4 * c4, o, M, L, whole, split);
        }
    }
}

// Many rows: a workgroup is a kv head, 64 RT packed rows of a sequence (16 RT a wave), a chunk of its keys.  64 keys at a time go through LDS as 16-bit numbers: each wave asks for a
// group of 16 two steps ahead and converts it one step ahead, once for all rows, while the products of this step run in the other wave of its SIMD.  Bound by a wave's instructions: of 64 keys 64 products
// of 16 turns, and beside them some 340 vector and 150 scalar instructions (exponentials, maxima, the rounding of the weights, the codes' conversion) that overlap with the other wave's products only in part.  Two
// prompts of 2048 rows on 6100 tokens, 32 heads of 128: 419 us, 800 TFLOP/s (a library's product of 8192^3: 1254).
template <int HD, int RT>
struct kv8_wide {
    static constexpr int KS = HD / 32, ET = HD / 16;
    static constexpr int buffer = 4 * KS * 64 + 2 * ET * 64;             // uint4 of 64 keys: K [group][ks][lane], V [pair][e][lane]
    static constexpr int lds = 2 * buffer * 16 + 64;                     // and of each group its scales' bytes, and what is the matter with it
};
template <int HD, int RT, int IO>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
k_kv8_attn_wide(const kv8_attn_args a)
{
    using W = kv8_wide<HD, RT>;
    constexpr int KB = HD / 64, KS = W::KS, ET = W::ET, NQ = kv8_types<IO>::NQ, TR = 64 * RT;
    constexpr bool HALF = kv8_types<IO>::half;
    extern __shared__ uint4 wide_lds[];
    int4 *about = (int4 *)(wide_lds + 2 * W::buffer);                    // [buffer]: a dword a group: scales' bytes, bit 16: does not exist, bit 17: NaN among its values
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, jl = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.x % a.pool.n_heads, split = blockIdx.y, units = gridDim.x / a.pool.n_heads;
    int tile = 0;
    // (the last tiles of a prompt have the most keys: they begin first)
    kv8_seq sq;
    if (!kv8_unit<HD, TR>(a.seqs, a.pool, units - 1 - blockIdx.x / a.pool.n_heads, a.group, sq, tile)) return;
    const int m0 = tile * TR, nrows = sq.rows * a.group, shift = sq.pool.page_shift;
    const int last = (min(m0 + TR, nrows) - 1) / a.group;
    const int nk = __builtin_amdgcn_readfirstlane(kv8_keys(sq, shift, last, a.mask != nullptr)), len = __builtin_amdgcn_readfirstlane(min(sq.len, 1 << 30));     // (no table goes further)
    const int k0 = split * a.chunk, k1 = min(k0 + a.chunk, nk);
    if (k0 >= nk && split > 0) return;
    const bool whole = nk <= a.chunk;
    const int sure = min(nk, a.mask != nullptr ? len : len + m0 / a.group + 1);     // keys before this one are seen by every row
    const int steps = (k1 - k0 + 63) >> 6;

    // this wave's group of 16 keys of step s
    const uint32_t block = (uint32_t)HD << shift, page_codes = 2 * block * sq.pool.n_heads, page_scales = sq.pool.n_heads << (shift - 3), in_page = (1u << shift) - 1;
    const uint8_t *codes = sq.pool.codes + (size_t)kvh * 2 * block, *scales = sq.pool.scales + (kvh << (shift - 3));
    auto page_of = [&](int s) { const int p = k0 + 64 * s + 16 * wave; return kv8_entry(sq, p >> shift); };
    auto codes_of = [&](int page, int p) { return codes + ((uint64_t)(uint32_t)page * page_codes + (p & in_page) * HD); };
    u32x4 kt[KB], vt[KB];
    uint32_t bytes = 0;
    int page = -1;                           // of the group that the registers hold
    // (no branch around the loads, and their registers stay whole: the compiler waits for a load where it moves a part of it)
    auto load = [&](int s, int pg) {
        const int p = k0 + 64 * s + 16 * wave;
        page = p < k1 && kv8_is_page(sq, pg) ? pg : -1;
        const int there = max(page, 0);
        const uint8_t *at = kv8_global(uniform_ptr(codes_of(there, p)));
        bytes = *(const uint16_t *)(scales + ((uint64_t)(uint32_t)there * page_scales + ((p & in_page) >> 3)));
#pragma unroll
        for (int b = 0; b < KB; ++b) { kt[b] = ((const u32x4 *)at)[b * 64 + lane]; vt[b] = ((const u32x4 *)(at + block))[b * 64 + lane]; }
    };
    auto convert = [&](int s, int buf) {
        uint4 *L = wide_lds + buf * W::buffer;
        uint4 *Lk = L + wave * KS * 64 + lane;
        uint2 *Lv = (uint2 *)(L + 4 * KS * 64 + (wave >> 1) * ET * 64 + lane) + (wave & 1);
        const int p = k0 + 64 * s + 16 * wave;
        const uint32_t byte_k = kv8_byte(bytes & 0xffu), byte_v = kv8_byte(bytes >> 8);
        uint32_t what = page < 0 ? 1u << 16 : byte_k | byte_v << 8;
        const float f = __uint_as_float(byte_k << 23);
        const bool whole_group = page >= 0 && p + 16 <= sure;
        if (!whole_group) {
            // codes of pages that do not exist, and values behind the end, count as zero, and values that are NaN are put in at the end
            const uint32_t k_there = page < 0 ? 0u : ~0u, there = page < 0 ? 0u : kv8_there(nk - p, g);
            bool nans = false;
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                kt[b] &= k_there; vt[b] &= there;
                nans = nans || (kv8_nans(vt[b].x) | kv8_nans(vt[b].y) | kv8_nans(vt[b].z) | kv8_nans(vt[b].w)) != 0;
            }
            if (__any(nans)) {
                what |= 1u << 17;
#pragma unroll
                for (int b = 0; b < KB; ++b) vt[b] = (u32x4){kv8_without_nans(vt[b].x), kv8_without_nans(vt[b].y), kv8_without_nans(vt[b].z), kv8_without_nans(vt[b].w)};
            }
        }
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            Lk[(2 * b) * 64] = kv8_key<HALF>(kt[b].x, kt[b].y, f);
            Lk[(2 * b + 1) * 64] = kv8_key<HALF>(kt[b].z, kt[b].w, f);
            Lv[(4 * b) * 128] = kv8_f16(vt[b].x); Lv[(4 * b + 1) * 128] = kv8_f16(vt[b].y); Lv[(4 * b + 2) * 128] = kv8_f16(vt[b].z); Lv[(4 * b + 3) * 128] = kv8_f16(vt[b].w);
        }
        if (lane == 0) ((uint32_t *)(about + buf))[wave] = what;
    };
    auto sync = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // (not for the loads on their way)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    if (steps > 0) load(0, page_of(0));
    kv8_row row[RT];
    uint4 q[RT][NQ][KS];
    uint64_t vm[RT];
    kv8_acc<HD, RT> A;
    kv8_begin(A);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        row[t] = kv8_row_at(a, sq, kvh, m0 + (wave * RT + t) * 16 + jl);
        kv8_load_q<HD, IO, NQ>(a, row[t], g, q[t]);
        vm[t] = a.mask != nullptr ? a.mask[row[t].row] : 0;
    }
    auto sees = [&](int t, int p) { return kv8_sees(a.mask != nullptr, vm[t], p + 4 * g, len, len + row[t].j + 1, nk); };
    uint32_t matter = 0;
    int only = -1;
    int next = 0;
    if (steps > 0) {
        next = page_of(1);
        convert(0, 0);
        if (steps > 1) { load(1, next); next = page_of(2); }
        sync();
    }
    for (int s = 0; s < steps;) {
        const int buf = s & 1, p0 = k0 + 64 * s;
        const uint4 *Lk = wide_lds + buf * W::buffer + lane, *Lv = Lk + 4 * KS * 64;
        // LDS is asked one group of products ahead (two prompts of 2048 rows 509 -> 485 us); the page three steps ahead is asked for before all else (a wait for LDS waits for scalar loads too)
        const int after = page_of(s + 3);
        const int4 ab = about[buf];
        uint4 k[2][KS], v[2][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) k[0][ks] = Lk[ks * 64];
        __builtin_amdgcn_sched_barrier(0);
        if (only < 0 && s + 1 < steps) {
            convert(s + 1, buf ^ 1);
            if (s + 2 < steps) load(s + 2, next);
        }
        next = after;                                                    // (a group looked at again asks for the same one)
        const uint32_t what[4] = {(uint32_t)__builtin_amdgcn_readfirstlane(ab.x), (uint32_t)__builtin_amdgcn_readfirstlane(ab.y), (uint32_t)__builtin_amdgcn_readfirstlane(ab.z), (uint32_t)__builtin_amdgcn_readfirstlane(ab.w)};
        const uint32_t any = what[0] | what[1] | what[2] | what[3];
        matter |= any;
        int miss = 0, ev[4], dv[4];
        float fk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { fk[i] = __uint_as_float((what[i] & 0xffu) << 23); ev[i] = (int)((what[i] >> 8) & 0xffu) - 127; }
        if (any & 0x10000u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (what[i] & 0x10000u) { miss |= 1 << i; ev[i] = KV8_NO_SCALE; }
        }
        f32x4 S[RT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < 3) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) k[(i + 1) & 1][ks] = Lk[((i + 1) * KS + ks) * 64];
            } else { v[0][0] = Lv[0]; v[0][1] = Lv[64]; }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < RT; ++t) S[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) S[t][i] = kv8_score<HALF>(k[i & 1][ks], q[t][n][ks], S[t][i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        kv8_units(A, ev, dv, only);
        const int without = miss | (only < 0 ? 0 : 15 & ~(1 << only));    // groups that are not looked at
        const bool last_keys = p0 + 64 > sure || miss != 0, edge = last_keys || without != 0;
        uint64_t there = ~0ull;
        if (without) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if ((without >> i) & 1) there &= ~(0xffffull << (16 * i));
        }
        auto see = [&](int t) { return sees(t, p0) & there; };
        uint2 P[RT][4], PL[RT][4];
        kv8_softmax<HD, RT, IO>(A, S, a.scale2, fk, edge, see, dv, P, PL);
        kv8_output<HD, RT, IO>(A, P, PL, [&](int u, int e) {
            const int n = u * ET + e, i = n >> 1;
            if (!(n & 1) && i + 1 < ET) {
                v[(i + 1) & 1][0] = Lv[(n + 2) * 64]; v[(i + 1) & 1][1] = Lv[(n + 3) * 64];
                __builtin_amdgcn_sched_barrier(0);
            }
            return v[i & 1][n & 1];
        });
        if (only >= 0 && only < 3) { ++only; continue; }                 // (all waves alike: the exponents are the same for them)
        only = -1;
        ++s;
        sync();
    }
    if (matter & 0x20000u) {
        for (int p0 = k0; p0 < k1; p0 += 64) {
            if (p0 + 64 <= sure) continue;
            kv8_put_nans<HD, RT>(A, [&](int t) { return sees(t, p0); }, [&](int i, int b) {
                const int p = p0 + 16 * i, pg = p < k1 ? kv8_page(sq, p >> shift) : -1;
                if (pg < 0) return make_uint4(0u, 0u, 0u, 0u);
                const uint4 c = ((const uint4 *)(codes_of(pg, p) + block))[b * 64 + lane];
                const uint32_t there = kv8_there(nk - p, g);
                return make_uint4(c.x & there, c.y & there, c.z & there, c.w & there);
            });
        }
    }
    const int E = A.E == KV8_NO_SCALE ? 0 : A.E;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float L = with_lane32(with_lane16(A.l[t], op_add), op_add) * 0x1p-15f;
        if (!row[t].live) continue;
#pragma unroll
        for (int e = 0; e < ET; ++e) {
            const float o[4] = {ldexpf(A.O[t][e][0], E - 15), ldexpf(A.O[t][e][1], E - 15), ldexpf(A.O[t][e][2], E - 15), ldexpf(A.O[t][e][3], E - 15)};
            kv8_finish4<HD, IO>(a, row[t], e * 16 + 4 * g, o, A.m[t], L, whole, split);
        }
    }
}

// The chunks of a row's keys joined: WR waves a row and query head, four chunks of each 4 HD bytes on their way a thread.  Four waves where chunks are more than 16 (attention and join with one wave and with four: one row
// over 8000 keys, 32 chunks, 11.6 and 10.7 us, over 65000, 64 chunks, 30.4 and 28.7; 16 sequences of up to 8000 keys, eight chunks, 33.3 and 34.1).  4.3 - 4.8 us: a launch, and two trips to memory
template <int HD, int IO, int WR>
__global__ void __launch_bounds__(256)
k_kv8_attn_merge(const kv8_attn_args a, int TR)
{
    constexpr int TPC = HD / 4, NG = WR * (64 / TPC), FL = 4;
    __shared__ float4 sh[4][TPC];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t id = WR == 4 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    const int row = __builtin_amdgcn_readfirstlane((int)(id / a.n_q_heads)), head = __builtin_amdgcn_readfirstlane((int)(id % a.n_q_heads));
    if (row >= a.seqs.n_rows) return;
    const size_t at = (size_t)row * a.n_q_heads + head;
    const float2 *ml = (const float2 *)(a.part_ml + at * a.nsplit * 2);
    const int t = lane % TPC, cg = (WR == 4 ? wave * (64 / TPC) : 0) + lane / TPC;
    const float *po = a.part_o + at * a.nsplit * HD + 4 * t;
    // asked for beside the sequence's tables, whatever these turn out to say: the statistics of up to 64 chunks, and the first outputs
    float2 one = ml[min(lane, a.nsplit - 1)];
    float4 v[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) v[i] = *(const float4 *)(po + (size_t)min(cg + i * NG, a.nsplit - 1) * HD);
    const int si = __builtin_amdgcn_readfirstlane(kv8_seq_of_row(a.seqs, row));
    if (si < 0) return;
    const kv8_seq sq = kv8_seq_at<HD>(a.seqs, a.pool, si);
    const int j = row - sq.row0;
    if (j < 0 || j >= sq.rows) return;
    const int tile = (j * a.group + head % a.group) / TR, last = (min((tile + 1) * TR, sq.rows * a.group) - 1) / a.group;
    const int nk = kv8_keys(sq, sq.pool.page_shift, last, a.mask != nullptr);
    if (nk <= a.chunk) return;              // (written already)
    const int n = (nk + a.chunk - 1) / a.chunk;
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
    if (WR == 4) {
        if (lane < TPC) sh[wave][lane] = make_float4(o[0], o[1], o[2], o[3]);
        __syncthreads();
        if (wave != 0) return;
        const float4 x = sh[0][t], y = sh[1][t], z = sh[2][t], w = sh[3][t];
        o[0] = (x.x + y.x) + (z.x + w.x); o[1] = (x.y + y.y) + (z.y + w.y); o[2] = (x.z + y.z) + (z.z + w.z); o[3] = (x.w + y.w) + (z.w + w.w);
    }
    if (lane >= TPC) return;
    const float inv = L == 0.f ? 0.f : 1.f / L, y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    kv8_store4<HD, IO>(a, row, head, 4 * t, y);
    if (a.lse != nullptr && lane == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
}

// ------------------------------- host side ----------------------------------------

// How a call's work is cut.  Rows a tile: 16, straight from memory, where sequences have no more (in the mean: what each has is on the device), and where the whole work is small, so that what the other kernel
// pays for going through LDS weighs more than codes converted again for every 16 rows, unless more than two tiles read codes that an XCD's L2 does not hold; else 64 or 128.  Eight kv heads of 128, four query heads
// each, us with 16 and the better of 64 and 128: one sequence of 4000 keys, 8, 64, 256, 512 rows 11.0 and 13.5, 19.4 and 21.6, 42.2 and 49.8, 76.5 and 74.9; of 60000 keys, 8, 16, 64 rows
// 38.3 and 42.5, 55.8 and 45.9, 150.6 and 105.4; 16 of up to 4000, 8, 32, 256 rows each 31.0 and 38.5, 55.6 and 57.0, 257.9 and 220.6.
// Chunks of keys until there are two workgroups a CU, all begun at once, or twice as many where sequences of different lengths come out at different times: 4 rows over 65000 keys 29.9, 31.4, 39.0, 50.7 us with 256,
// 512, 1024, 2048 workgroups, 32 sequences of 256 .. 8192 keys 59.0, 63.0, 50.7, 54.5, two prompts 426, 427, 470, 464.
// Few keys are one workgroup's, which saves the launch that joins: up to 1024, 768 with more than 16 rows a sequence, 2048 where there is a workgroup a CU (in chunks and whole, from a graph, 8 kv heads: one row over 500 keys 9.2
// and 7.6 us, 760 9.3 and 8.9, 1020 9.1 and 10.1, 1500 9.5 and 12.6, called one by one 13.5 and 9.5, 13.3 and 10.0, 13.3 and 12.6; 16 rows over 760 9.5 and 10.4, 13.2 and 10.3; 32 sequences of up to 1020 17.1 and 11.9, 2040 21.8 and 18.2).
struct kv8_plan { int tr, units, nsplit, chunk; };

static kv8_plan plan(int n_seq, int n_rows, int group, int kv_heads, int hd, int64_t keys)
{
    kv8_plan p;
    const int64_t packed = (int64_t)n_rows * group;
    const bool little = packed * kv_heads <= (1 << 26) / (keys > 0 ? keys : 1) && (packed <= (int64_t)32 * n_seq || keys * 2 * hd <= 2 << 20);
    p.tr = packed <= (int64_t)16 * n_seq || little ? 16 : packed <= (int64_t)64 * n_seq ? 64 : 128;
    p.units = (int)((packed + (int64_t)n_seq * (p.tr - 1)) / p.tr);
    const int64_t tiles = packed / p.tr > n_seq ? packed / p.tr : n_seq, base = tiles * kv_heads, most = (keys + 255) / 256, want = p.tr == 16 && n_seq > 1 ? 1024 : 512;
    int64_t n = (want + base - 1) / base;
    n = n < most ? n : most;
    n = n < 256 ? n : 256;
    if (p.tr == 16 && most <= (base >= 256 ? 8 : packed <= (int64_t)16 * n_seq ? 4 : 3)) n = 1;
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
    *bytes = seqs->n_seq && seqs->n_rows ? part_bytes(plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, pool->head_dim, (int64_t)seqs->table_pages * pool->page_tokens), seqs->n_rows, n_q_heads, pool->head_dim) : 0;
    return PV_OK;
}

// more dynamic LDS than the default limit: allowed once on each device
template <int HD, int IO>
static int allow_lds()
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    PV_HIP(hipGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return PV_OK;
    PV_HIP(hipFuncSetAttribute((const void *)k_kv8_attn_wide<HD, 1, IO>, hipFuncAttributeMaxDynamicSharedMemorySize, kv8_wide<HD, 1>::lds));
    PV_HIP(hipFuncSetAttribute((const void *)k_kv8_attn_wide<HD, 2, IO>, hipFuncAttributeMaxDynamicSharedMemorySize, kv8_wide<HD, 2>::lds));
    if (dev < 64) done.fetch_or(bit, std::memory_order_release);
    return PV_OK;
}

template <int HD, int IO>
static int launch(const kv8_attn_args &a, const kv8_plan &p, hipStream_t s)
{
    const dim3 grid(p.units * a.pool.n_heads, p.nsplit);
    if (p.tr == 16) k_kv8_attn<HD, IO><<<grid, 256, 0, s>>>(a);
    else {
        if (kv8_wide<HD, 1>::lds > 65536) { const int rc = allow_lds<HD, IO>(); if (rc != PV_OK) return rc; }
        if (p.tr == 64) k_kv8_attn_wide<HD, 1, IO><<<grid, 256, kv8_wide<HD, 1>::lds, s>>>(a);
        else k_kv8_attn_wide<HD, 2, IO><<<grid, 256, kv8_wide<HD, 2>::lds, s>>>(a);
    }
    PV_HIP(hipGetLastError());
    if (p.nsplit == 1) return PV_OK;
    const int64_t waves = (int64_t)a.seqs.n_rows * a.n_q_heads;
    if (p.nsplit > 16) k_kv8_attn_merge<HD, IO, 4><<<(unsigned)waves, 256, 0, s>>>(a, p.tr);
    else k_kv8_attn_merge<HD, IO, 1><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(a, p.tr);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

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
    const kv8_plan p = plan(seqs->n_seq, seqs->n_rows, group, pool->n_kv_heads, pool->head_dim, (int64_t)seqs->table_pages * pool->page_tokens);
    const size_t need = part_bytes(p, seqs->n_rows, n_q_heads, pool->head_dim);
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    kv8_attn_args a = {};
    a.pool = pv_kv8_pool_args(pool); a.seqs = pv_kv8_seqs_args(seqs);
    a.q = (const char *)q; a.q_row_bytes = q_row_stride * 2; a.q_head_bytes = q_head_stride * 2;
    a.out = (char *)out; a.out_row_bytes = out_row_stride * 2; a.out_head_bytes = out_head_stride * 2;
    a.lse = lse; a.mask = mask; a.group = group; a.n_q_heads = n_q_heads; a.nsplit = p.nsplit; a.chunk = p.chunk;
    a.part_o = (float *)workspace; a.part_ml = a.part_o + (size_t)seqs->n_rows * n_q_heads * p.nsplit * pool->head_dim;
    a.scale2 = scale == 0.f ? 1.f : fabsf(scale) * 1.44269504088896340736f;
    a.q_and = scale == 0.f ? 0u : ~0u; a.q_xor = scale < 0.f ? 0x80008000u : 0u;
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
    kv8_plan p = plan(a.seqs.n_seq, st.rows, a.group, f.n_kv_heads, f.head_dim, keys);
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
