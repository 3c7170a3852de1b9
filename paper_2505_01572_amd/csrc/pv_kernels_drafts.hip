// Drafted tokens verified against the target's probabilities, from given random numbers (speculative sampling).
//
//   p_j = softmax(logits_j / T) of row j;  the draft in row c, behind row j, with its random number u and the drafter's probability q of it, is taken if  u q < p_j(draft).  If not, what follows row j is drawn
//   from max(p_j - q, 0), or, where no drafter's probabilities are given (q is one at the draft), from p_j without the draft; behind the last draft from p.  A node of a tree has its children tried in order,
//   each under what the refused ones before it left: taken if u (1 - sum of their p) < p_j(draft).
//   The draw: the lowest token at which the sum of probabilities, in the order of ids, passes u' times their whole.
//
// The result is whole numbers.  What a draw turns on is computed in 64 bits: with exponentials of 32 bits a sum over a vocabulary of 10^5 lands on the wrong side of one of its 10^5 borders once in some 10^5 draws (once in 10^2
// under p - q, where p's own sum moves all of them).  Whether a draft is taken turns on one border: without a drafter's probabilities rows are summed with exponentials of 32 bits, off by some 10^-7, which
// decides one draft of a chain in 10^7 otherwise and takes a third of the time.  (What remains of a row behind refused children of a tree may be less than that: there the walk looks twice.)
//   rows   a workgroup takes a segment of a row: its maximum and the sum of its exponentials.  Only of rows that a draft is behind: p of a tree's leaves, half of its nodes, and of a chain's last row is asked for only if
//          the draw is there (16 trees of up to 48 nodes, 128256 logits of bf16, all four launches: 36.9 us; with all rows 16 more)
//   walk   a tree: a workgroup a sequence joins the segments of the nodes' rows and walks along
//   rest   a workgroup a segment of the row that the draw is behind (a chain: found anew by each): what is left to draw from, summed
//   pick   a workgroup a sequence finds the segment that the draw falls in, and in that the token
// In a trace, each by itself, the rows take 17.4 us (44 MB of the 143 that the logits have; most workgroups find that they have nothing to do, which with all tables asked for at once took no less), walk 7.0, rest 7.4, pick 7.0: trips
// to memory, one behind the other (in a graph a launch's beginning lies beside the end of the one before it).  The draw by the last workgroup of the launch before it, which saves a launch, was slower: 25 -> 31 us (64 chains), 50 -> 58 (16 trees).
#include "pv_matrix_common.h"

struct __align__(16) dv_part { double sum; float top; int first; };       // of a segment: sum of e^((x - top) / T), largest logit, its lowest id (T = 0: no sum)

struct dv_args {
    const char *logits; int64_t row_bytes;
    int rows, vocab, segs, n_seq;
    const int32_t *row_start, *tokens, *parent;
    const void *u; int u64;                 // [row][2]: for taking the row's token, for the draw behind the row
    const float *probs; int64_t probs_row;
    const float *temperature; float hot;    // of a sequence, or of all
    int32_t *accepted, *next, *path;
    float *out_probs;
    dv_part *part;                          // [row][seg]
    int left;                               // segments of DV_SIZE tokens of the row that the draw is behind
    double2 *rest;                          // [seq][left]: what is left to draw from p - q, summed, and from p; or (dv_drawn: no) a dv_part of a segment, the sum without refused tokens
    int2 *walk;                             // [seq]: row that the draw is behind, whether a draft was refused there
};

#define DV_SIZE 4096
#define DV_MAX_SEGS 512

struct dv_seq { int row0, rows; };
__device__ inline dv_seq dv_seq_at(const dv_args &a, int s)
{
    dv_seq q;
    q.row0 = a.row_start[s];
    q.rows = min(max(a.row_start[s + 1], 0), a.rows) - max(q.row0, 0);        // (no difference that wraps, whatever the table holds)
    if (q.row0 < 0 || q.rows < 0) q.rows = 0;
    return q;
}
// log2(e) / T (of an infinite T: next to nothing); 0: the most probable token alone
__device__ inline double dv_cold(const dv_args &a, int s)
{
    const float t = a.temperature != nullptr ? a.temperature[s] : a.hot;
    return t > 0.f ? fmax(1.4426950408889634074 / (double)t, 1e-300) : 0.0;
}
__device__ inline double dv_u(const dv_args &a, int row, int which)
{
    const int64_t i = 2 * (int64_t)row + which;
    return a.u64 ? ((const double *)a.u)[i] : (double)((const float *)a.u)[i];
}

// 2^((x - top) cold), for a result of at most 1: a whole power of two, put into the exponent, times 2^r, |r| <= 1/2, by the polynomial of degree 8 that meets it at the nine Chebyshev points (off by 1.1 10^-12 of it at most; a sum
// of rounded probabilities turns on 10^-11 of them, so a ninth degree would buy nothing).  What is below 2^-1000, -infinity and NaN: 2^-1000.
__device__ inline double dv_power(float x, double cold, double top)
{
    const double t = fmax(((double)x - top) * cold, -1000.0), m = t + 6755399441055744.0, r = t - (m - 6755399441055744.0);      // (1.5 2^52: what is added to it is rounded to a whole number, in its low bits)
    double e = 1.3255224878668817e-06;
    e = fma(e, r, 1.5310079402249296e-05); e = fma(e, r, 0.00015403455852453838); e = fma(e, r, 0.0013333450568000645); e = fma(e, r, 0.009618129159402558);
    e = fma(e, r, 0.05550410941205933); e = fma(e, r, 0.2402265069581299); e = fma(e, r, 0.6931471805459335); e = fma(e, r, 1.0);
    const uint64_t b = __double_as_longlong(e);
    return __longlong_as_double((int64_t)((uint64_t)((uint32_t)(b >> 32) + ((uint32_t)__double_as_longlong(m) << 20)) << 32 | (uint32_t)b));
}
__device__ inline double dv_weight(float x, double cold, double top) { return x > -INFINITY ? dv_power(x, cold, top) : 0.0; }      // (NaN: 0)

template <typename T> __device__ inline float dv_one(const char *p, int64_t i);
template <> __device__ inline float dv_one<float>(const char *p, int64_t i) { return ((const float *)p)[i]; }
template <> __device__ inline float dv_one<__bf16>(const char *p, int64_t i) { return pv_bf16_to_f32(((const uint16_t *)p)[i]); }
template <> __device__ inline float dv_one<_Float16>(const char *p, int64_t i) { return (float)((const _Float16 *)p)[i]; }
// Numbers as they lie in memory, dwords w of them: number i
typedef __attribute__((ext_vector_type(2))) _Float16 dv_h2;
template <typename T> __device__ inline float dv_get(const uint32_t *w, int i);
template <> __device__ inline float dv_get<float>(const uint32_t *w, int i) { return __uint_as_float(w[i]); }
template <> __device__ inline float dv_get<__bf16>(const uint32_t *w, int i) { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
template <> __device__ inline float dv_get<_Float16>(const uint32_t *w, int i) { const dv_h2 h = __builtin_bit_cast(dv_h2, w[i >> 1]); return (float)(i & 1 ? h.y : h.x); }

// 16 bytes (8) from an address that is a multiple of 4
typedef __attribute__((ext_vector_type(2), aligned(4))) unsigned int dv_u32x2;
typedef __attribute__((ext_vector_type(4), aligned(4))) unsigned int dv_u32x4;
__device__ inline u32x4 dv_load16(const char *p) { const dv_u32x4 v = *(const dv_u32x4 *)p; return (u32x4){v.x, v.y, v.z, v.w}; }
__device__ inline u32x4 dv_load16_once(const char *p) { const dv_u32x4 v = __builtin_nontemporal_load((const dv_u32x4 *)p); return (u32x4){v.x, v.y, v.z, v.w}; }
template <typename T> __device__ constexpr uint32_t dv_none() { return sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u; }      // -infinity

// N tokens' logits and, where there are any, the drafter's probabilities from token i on; behind `end`: -infinity and 0
template <typename T, int N> __device__ inline void dv_tokens(const char *src, const float *drafter, int i, int end, float (&x)[N], float (&d)[N])
{
    constexpr int W = N * (int)sizeof(T) / 4;
    static_assert(N % 4 == 0 && (W == 2 || W % 4 == 0), "");
    const bool whole = i + N <= end;
    uint32_t w[W];
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = dv_none<T>();
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] = 0.f;
    const char *at = src + (int64_t)i * sizeof(T);
    if (whole) {
        if constexpr (W == 2) { const dv_u32x2 v = *(const dv_u32x2 *)at; w[0] = v.x; w[1] = v.y; }
        else {
#pragma unroll
            for (int k = 0; k < W / 4; ++k) { const u32x4 v = dv_load16(at + 16 * k); w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w; }
        }
    }
    if (whole && drafter != nullptr) {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            const u32x4 v = dv_load16((const char *)(drafter + i + 4 * k));
            d[4 * k] = __uint_as_float(v.x); d[4 * k + 1] = __uint_as_float(v.y); d[4 * k + 2] = __uint_as_float(v.z); d[4 * k + 3] = __uint_as_float(v.w);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = dv_get<T>(w, k);
    if (!whole && i < end) {
#pragma unroll
        for (int k = 0; k < N; ++k) if (i + k < end) { x[k] = dv_one<T>(src, i + k); if (drafter != nullptr) d[k] = drafter[i + k]; }
    }
}

// Sums over lanes N apart within 16 lanes by rotations, over the others by exchanges: vector instructions
template <int N> __device__ inline double dv_rotated(double v)
{
    const uint64_t b = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)b, 0x120 + N, 0xF, 0xF, true), hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(b >> 32), 0x120 + N, 0xF, 0xF, true);
    return v + __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
__device__ inline double dv_over_16(double v) { return dv_rotated<8>(dv_rotated<4>(dv_rotated<2>(dv_rotated<1>(v)))); }
__device__ inline double dv_over_wave(double v)
{
    v = dv_over_16(v);
    uint64_t b = __double_as_longlong(v);
    auto l = __builtin_amdgcn_permlane16_swap((uint32_t)b, (uint32_t)b, false, false), h = __builtin_amdgcn_permlane16_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    v = __longlong_as_double((int64_t)((uint64_t)h[0] << 32 | l[0])) + __longlong_as_double((int64_t)((uint64_t)h[1] << 32 | l[1]));
    b = __double_as_longlong(v);
    l = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false); h = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    return __longlong_as_double((int64_t)((uint64_t)h[0] << 32 | l[0])) + __longlong_as_double((int64_t)((uint64_t)h[1] << 32 | l[1]));
}
__device__ inline int dv_min_over_wave(int v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d, 64));
    return v;
}
// ... up to and with the own lane
__device__ inline double dv_up_to(double v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const double o = __shfl_up(v, d, 64); if (lane >= d) v += o; }
    return v;
}

// Segment seg of a row: tokens begin(seg) .. begin(seg + 1) - 1.  16 bytes of a thread begin at a multiple of four: a row of 16-bit numbers that does not has one token more in its first segment.
template <typename T> __device__ inline int dv_head(const char *src) { return sizeof(T) == 2 && ((uintptr_t)src & 2) ? 1 : 0; }
__device__ inline int dv_begin(int seg, int head, int size) { return seg == 0 ? 0 : head + seg * size; }

// Whether a draft is behind a row of a sequence: only then its probabilities are asked for here (if the draw is behind it, it is summed there).  Whole workgroups call.
__device__ inline bool dv_needed(const dv_args &a, const dv_seq &q, int row)
{
    constexpr int N = 4;
    const int local = row - q.row0;
    if (a.parent == nullptr) return local < q.rows - 1;
    if (q.rows - local - 1 > N * 256) return true;           // (more than a thread looks at)
    bool any = false;
#pragma unroll
    for (int i = 0; i < N; ++i) { const int j = local + 1 + (int)threadIdx.x + 256 * i; if (j < q.rows) any = any || a.parent[q.row0 + j] == local; }
    return __syncthreads_or(any);
}

// The rows' sums, WIDE: in 64 bits.  Those are bound by the exponentials: some 22 instruction slots a logit, 16 of them in 64 bits; the others by the read of the logits.
template <typename T, int E, bool WIDE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WIDE ? 4 : E > 32 ? 7 : 8)))
k_draft_rows(const dv_args a)
{
    constexpr int NT = 256, V = 16 / (int)sizeof(T), U = E / V, D = E * (int)sizeof(T) / 4, SIZE = NT * E;
    __shared__ float sh_top[4];
    __shared__ double sh_sum[4];
    __shared__ int sh_first[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / a.segs, seg = blockIdx.x - row * a.segs;
    const char *src = a.logits + (int64_t)row * a.row_bytes;
    const int head = dv_head<T>(src), base = head + seg * SIZE;
    int s = 0;
    for (int k = 0; k < a.n_seq; k += 64) {
        const int end = k + lane < a.n_seq ? a.row_start[k + lane + 1] : 0x7fffffff;
        s += __popcll(__ballot(end <= row));
    }
    if (tid == 0 && seg == 0) {
        if (a.path != nullptr) a.path[row] = -1;
        a.out_probs[row] = 0.f;              // (rows of a sequence: later)
    }
    if (s >= a.n_seq || !dv_needed(a, dv_seq_at(a, s), row)) return;
    uint32_t x[D];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i0 = base + (u * NT + tid) * V;
        u32x4 v = {dv_none<T>(), dv_none<T>(), dv_none<T>(), dv_none<T>()};
        if (i0 + V <= a.vocab) v = dv_load16_once(src + (int64_t)i0 * sizeof(T));
        x[4 * u] = v.x; x[4 * u + 1] = v.y; x[4 * u + 2] = v.z; x[4 * u + 3] = v.w;
    }
    // those that no 16 bytes hold: ahead of the first, behind the last
    const int behind = (a.vocab - head) % V;
    auto alone_of = [&](int t) { return t == 0 ? (seg == 0 && head ? 0 : -1) : t <= behind && seg == (a.vocab - behind - head) / SIZE ? a.vocab - behind + t - 1 : -1; };
    float x0 = -INFINITY;
    if (const int alone = alone_of(tid); alone >= 0) x0 = dv_one<T>(src, alone);
    const double cold = dv_cold(a, s);
    float top = fmaxf(x0, -INFINITY);        // (of a number and NaN the number)
#pragma unroll
    for (int i = 0; i < E; ++i) top = fmaxf(top, dv_get<T>(x, i));
    top = over_wave(top, op_max);
    if (lane == 0) sh_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sh_top[0], sh_top[1]), fmaxf(sh_top[2], sh_top[3]));
    double sum = 0.0;
    int first = 0x7fffffff;
    if (cold > 0.0) {
#pragma unroll
        for (int d = 0; d < D; ++d) if (sizeof(T) == 2) asm volatile("" : "+v"(x[d]));     // (taken apart anew: 32 bits of each number would be twice the registers)
        if constexpr (WIDE) {
            const double most = top;
            double odd = 0.0;
#pragma unroll
            for (int i = 0; i < E; ++i) { const double w = dv_power(dv_get<T>(x, i), cold, most); if (i & 1) odd += w; else sum += w; }
            sum = dv_over_wave((sum + odd) + dv_power(x0, cold, most));
        } else {
            // (x - top as it is, then the factor: a factor's product with top would be off by as much for all, and so would its own rounding be: it is a number of 32 bits just below it, and what is left of it, above 0 as well so
            // that -infinity stays what it is.)
            const double most = fmin(cold, 1e30);
            const float c = fmaxf((float)(most * (1.0 - 0x1p-23)), 0x1p-149f), c2 = fmaxf((float)(most - (double)c), 0x1p-149f);
            auto exponent = [&](float v) { const float d = v - top; return fmaf(d, c, d * c2); };
            float even = 0.f, odd = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) { const float w = __builtin_amdgcn_exp2f(exponent(dv_get<T>(x, i))); if (i & 1) odd += w; else even += w; }
            if (__any(!(even + odd < INFINITY))) {            // NaN among them: once more, with care
                even = odd = 0.f;
#pragma unroll
                for (int d = 0; d < D; ++d) if (sizeof(T) == 2) asm volatile("" : "+v"(x[d]));
#pragma unroll
                for (int i = 0; i < E; ++i) { even += __builtin_amdgcn_exp2f(fmaxf(exponent(dv_get<T>(x, i)), -256.f)); asm volatile("" : "+v"(even)); }      // (2^-256 is 0; of NaN and a number the number; one after the other: no registers for more)
            }
            even += __builtin_amdgcn_exp2f(fmaxf(exponent(x0), -256.f));
            sum = dv_over_wave((double)even + (double)odd);
        }
        if (top == -INFINITY) sum = 0.0;
    } else {
        int me = tid;
        asm volatile("" : "+v"(me));           // (found anew: kept, it would take a register that the logits need)
        const int alone = alone_of(me);
        if (alone >= 0 && x0 == top) first = alone;
#pragma unroll
        for (int i = 0; i < E; ++i) if (dv_get<T>(x, i) == top) first = min(first, base + ((i / V) * NT + tid) * V + i % V);      // (what fills a row up: only if the segment has nothing but -infinity)
        first = dv_min_over_wave(first);
    }
    if (lane == 0) { sh_sum[wave] = sum; sh_first[wave] = first; }
    __syncthreads();
    if (tid == 0) {
        dv_part p;
        p.sum = (sh_sum[0] + sh_sum[1]) + (sh_sum[2] + sh_sum[3]);
        p.top = top;
        p.first = min(min(sh_first[0], sh_first[1]), min(sh_first[2], sh_first[3]));
        a.part[(int64_t)row * a.segs + seg] = p;
    }
}

// A row's segments joined, by each GL lanes side by side: largest logit, sum of exponentials, the lowest id of the largest.  Four segments a lane stay in registers between the two passes.
struct dv_row { double sum; float top; int first; bool any; };      // any: it has probabilities (its largest logit is a number)
struct dv_parts { dv_part q[4]; };
template <int GL> __device__ inline dv_parts dv_parts_of(const dv_args &a, int row)
{
    const int l = threadIdx.x % GL;
    const dv_part *p = a.part + (int64_t)row * a.segs;
    dv_parts r;
#pragma unroll
    for (int k = 0; k < 4; ++k) { r.q[k] = {0.0, -INFINITY, 0x7fffffff}; if (l + k * GL < a.segs) r.q[k] = p[l + k * GL]; }
    return r;
}
template <int GL> __device__ inline dv_row dv_row_of(const dv_args &a, int row, double cold, const dv_parts &parts)
{
    constexpr int K = 4;
    const int l = threadIdx.x % GL;
    const dv_part *p = a.part + (int64_t)row * a.segs;
    dv_row r = {0.0, -INFINITY, 0x7fffffff, false};
#pragma unroll
    for (int k = 0; k < K; ++k) r.top = fmaxf(r.top, parts.q[k].top);
    for (int i = l + K * GL; i < a.segs; i += GL) r.top = fmaxf(r.top, p[i].top);
    r.top = with_rotated<8>(with_rotated<4>(with_rotated<2>(with_rotated<1>(r.top, op_max), op_max), op_max), op_max);
    if (GL == 64) r.top = with_lane32(with_lane16(r.top, op_max), op_max);
    r.any = r.top > -INFINITY && r.top < INFINITY;
    auto add = [&](const dv_part &v) {
        if (cold > 0.0) r.sum += v.sum * dv_weight(v.top, cold, r.top);
        else if (v.top == r.top) r.first = min(r.first, v.first);
    };
#pragma unroll
    for (int k = 0; k < K; ++k) if (k * GL < a.segs) add(parts.q[k]);
    for (int i = l + K * GL; i < a.segs; i += GL) add(p[i]);
    if (cold > 0.0) r.sum = GL == 64 ? dv_over_wave(r.sum) : dv_over_16(r.sum);
    else {
#pragma unroll
        for (int d = 1; d < GL; d <<= 1) r.first = min(r.first, __shfl_xor(r.first, d, 64));
    }
    return r;
}
// p of a token, from its logit
__device__ inline double dv_prob(const dv_args &a, const dv_row &r, float x, int token, double cold)
{
    if (!r.any || token < 0 || token >= a.vocab) return 0.0;
    if (cold == 0.0) return token == r.first ? 1.0 : 0.0;
    return dv_weight(x, cold, r.top) / r.sum;
}

// A chain: which drafts are taken, all looked at side by side, 16 lanes each.  The row behind which the draw is, and whether a draft was refused there; that row's sums in *sh_row where one was.  all: go on behind the first
// refused one, for every draft's p, and write it.
struct dv_chain_lds { dv_row row; int refused; };
template <typename T> __device__ inline int2 dv_chain(const dv_args &a, const dv_seq &q, double cold, bool all, dv_chain_lds *sh)
{
    constexpr int GL = 16;
    if (threadIdx.x == 0) sh->refused = q.rows;
    __syncthreads();
    const int n = blockDim.x / GL;
    for (int j0 = 1; j0 < q.rows; j0 += n) {             // (uniform: lanes without a draft look at the last one)
        const int j = min(j0 + (int)threadIdx.x / GL, q.rows - 1), row = q.row0 + j, token = a.tokens[row];
        const double u = dv_u(a, row, 0);
        const dv_parts parts = dv_parts_of<GL>(a, row - 1);          // (on their way while the token comes, and what depends on it)
        const int safe = min(max(token, 0), a.vocab - 1);
        const float x = dv_one<T>(a.logits + (int64_t)(row - 1) * a.row_bytes, safe);
        const double d = a.probs == nullptr ? 1.0 : safe == token ? (double)a.probs[(int64_t)row * a.probs_row + safe] : 0.0;
        const dv_row r = dv_row_of<GL>(a, row - 1, cold, parts);
        const double p = dv_prob(a, r, x, token, cold);
        if (threadIdx.x % GL == 0) {
            if (!(u * d < p)) atomicMin(&sh->refused, j);
            if (all) a.out_probs[row] = (float)p;
        }
        const int before = j0;
        __syncthreads();
        const int refused = sh->refused;
        if (refused >= before && refused < min(before + n, q.rows) && refused == j && threadIdx.x % GL == 0) sh->row = r;
        __syncthreads();
        if (!all && refused < q.rows) break;
    }
    const int refused = sh->refused;
    return make_int2(q.row0 + min(refused, q.rows) - 1, refused < q.rows);
}

// The walk along a sequence's tree: node by node what each child's p is, then one wave.  Some five trips to memory, one behind the other, for each 64 nodes.
//
// What is left behind refused children is 1 less their p, and every p of a row is off by the same small part of itself, that of the row's sum (2^-17 at most): a child whose u times what is left comes so near to its p that this decides
// is judged by what the tokens that are left weigh themselves, in 64 bits, the refused ones not among them, and what is left behind it is known from there to 2^-35 of that.  So the last child that a row allows is always taken,
// and there is a token left to draw behind refused children.  Of random numbers some 10^-5 come so near.
#define DV_NODES 1024                       // nodes at a time
#define DV_NEAR 0x1p-17
#define DV_NEAR_JUDGED 0x1p-35
struct dv_judge_lds { double sum[16], mine; uint32_t out[DV_SIZE / 32]; };
struct dv_judged { bool taken; double left, near; };       // left: behind the child, should it be refused; near: as far as that may be off
// ... for child k of node `at`.  Whole workgroups call.  (Sums of numbers that are not negative are no less than any of them, however they are rounded: of a token alone they are its weight.)
template <typename T> __device__ inline dv_judged dv_judge(const dv_args &a, const dv_seq &q, int at, int k, double cold, dv_judge_lds *sh)
{
    constexpr int NT = 1024;
    const int tid = threadIdx.x, row = q.row0 + at, token = a.tokens[q.row0 + k];
    const char *src = a.logits + (int64_t)row * a.row_bytes;
    const dv_row r = dv_row_of<64>(a, row, cold, dv_parts_of<64>(a, row));
    const double top = r.top;
    double sum = 0.0;
    for (int begin = 0; begin < a.vocab; begin += DV_SIZE) {
        for (int i = tid; i < DV_SIZE / 32; i += NT) sh->out[i] = 0u;
        __syncthreads();
        for (int i = at + 1 + tid; i < k; i += NT) {          // (child k has a token that none before it had)
            const int t = a.tokens[q.row0 + i];
            if (a.parent[q.row0 + i] == at && t >= begin && t < begin + DV_SIZE) atomicOr(&sh->out[(t - begin) >> 5], 1u << ((t - begin) & 31));
        }
        __syncthreads();
        for (int i = tid; i < DV_SIZE && begin + i < a.vocab; i += NT) {
            if ((sh->out[i >> 5] >> (i & 31)) & 1u) continue;
            const double w = dv_weight(dv_one<T>(src, begin + i), cold, top);
            if (begin + i == token) sh->mine = w;
            sum += w;
        }
        __syncthreads();
    }
    sum = dv_over_wave(sum);
    if ((tid & 63) == 0) sh->sum[tid >> 6] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) sum += sh->sum[i];
    const double mine = sh->mine;
    __syncthreads();
    return {dv_u(a, q.row0 + k, 0) * sum < mine, (sum - mine) / r.sum, DV_NEAR_JUDGED * (sum / r.sum)};
}

template <typename T>
__global__ void __launch_bounds__(1024)
k_draft_walk(const dv_args a)
{
    constexpr int NT = 1024, GL = 16;
    __shared__ double sh_p[DV_NODES], sh_u[DV_NODES], sh_left[2];
    __shared__ int sh_parent[DV_NODES], sh_token[DV_NODES], sh_walk[3];
    __shared__ dv_judge_lds sh_judge;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = blockIdx.x;
    const dv_seq q = dv_seq_at(a, s);
    if (q.rows == 0) return;
    const double cold = dv_cold(a, s);
    if (tid == 0) { a.path[q.row0] = 0; a.out_probs[q.row0] = 1.f; }
    int at = 0, depth = 0;
    const double off = cold > 0.0 ? DV_NEAR : 0.0;           // (the most probable token alone: p is 1 or 0)
    double left = 1.0, near = off;           // of p behind the refused children of `at`; as far as that, and p, may be off
    for (int n0 = 1; n0 < q.rows; n0 += DV_NODES) {
        const int n = min(DV_NODES, q.rows - n0);
        for (int i0 = 0; i0 < n; i0 += NT / GL) {
            const int i = min(i0 + tid / GL, n - 1), row = q.row0 + n0 + i, up = a.parent[row], token = a.tokens[row], safe = min(max(token, 0), a.vocab - 1);
            const double u = dv_u(a, row, 0);
            const bool good = up >= 0 && up < n0 + i;
            const int over = q.row0 + (good ? up : 0);
            const float x = dv_one<T>(a.logits + (int64_t)over * a.row_bytes, safe);
            const dv_row r = dv_row_of<GL>(a, over, cold, dv_parts_of<GL>(a, over));
            const double p = good ? dv_prob(a, r, x, token, cold) : 0.0;
            if (tid % GL == 0) { sh_p[i] = p; sh_u[i] = u; sh_parent[i] = good ? up : -1; sh_token[i] = token; a.out_probs[row] = (float)p; }
        }
        __syncthreads();
        int from = 0;                        // the first node to look at; from the second turn on it has been judged
        bool judged = false;
        dv_judged verdict = {};
        for (;;) {
            if (wave == 0) {
                int ask = -1;
                for (int b = from & ~63; b < n && ask < 0; b += 64) {
                    const int i = b + lane;
                    const int up = i < n ? sh_parent[i] : -2;
                    uint64_t todo = __ballot(up == at) & (b < from ? ~0ull << (from - b) : ~0ull);
                    while (todo) {
                        const int k = b + __ffsll((unsigned long long)todo) - 1, token = sh_token[k];
                        // a token that an earlier child has had
                        bool had = false;
                        for (int j = at + 1 - n0; j < k; j += 64) {
                            const int c = j + lane;
                            bool same = false;
                            if (c < k) same = c >= 0 ? sh_parent[c] == at && sh_token[c] == token : a.parent[q.row0 + n0 + c] == at && a.tokens[q.row0 + n0 + c] == token;
                            had = had || __any(same);
                        }
                        const double p = had ? 0.0 : sh_p[k], u = sh_u[k];
                        bool taken = u * (left + near) < p;
                        const bool known = judged && k == from;
                        if (known) taken = verdict.taken;
                        else if (u * (left - near) < p && !taken && p > 0.0) { ask = k; break; }
                        todo &= todo - 1;
                        if (taken) {
                            at = n0 + k; ++depth; left = 1.0; near = off;
                            if (lane == 0) a.path[q.row0 + depth] = at;
                            const uint64_t past = k - b == 63 ? 0ull : ~0ull << (k - b + 1);
                            todo = __ballot(up == at) & past;
                        } else if (known) { left = verdict.left; near = verdict.near; }
                        else left -= p;
                    }
                }
                if (lane == 0) { sh_walk[0] = at; sh_walk[1] = depth; sh_walk[2] = ask; sh_left[0] = left; sh_left[1] = near; }
            }
            __syncthreads();
            at = sh_walk[0]; depth = sh_walk[1]; left = sh_left[0]; near = sh_left[1]; from = sh_walk[2];
            __syncthreads();
            if (from < 0) break;
            verdict = dv_judge<T>(a, q, at, n0 + from, cold, &sh_judge);
            judged = true;
        }
    }
    if (tid == 0) { a.walk[s] = make_int2(q.row0 + at, 0); a.accepted[s] = depth; }
}

// What may not be drawn, of a chain or tree without a drafter's probabilities: the tokens refused behind the row, a bit each for a segment's tokens; false: there is none anywhere
__device__ inline bool dv_refused(const dv_args &a, const dv_seq &q, int2 w, int begin, int end, uint32_t *out)
{
    const int tid = threadIdx.x, nt = blockDim.x, from = w.x - q.row0 + 1, last = a.probs != nullptr ? 0 : a.parent != nullptr ? q.rows : w.y ? from + 1 : 0;
    if (last <= from) return false;
    for (int i = tid; i < (DV_SIZE + 32) / 32; i += nt) out[i] = 0u;
    __syncthreads();
    for (int i = from + tid; i < last; i += nt) {
        const int token = a.tokens[q.row0 + i];
        const bool mine = a.parent == nullptr || a.parent[q.row0 + i] == w.x - q.row0;
        if (mine && token >= begin && token < end) atomicOr(&out[(token - begin) >> 5], 1u << ((token - begin) & 31));
    }
    __syncthreads();
    return true;
}

// N tokens from i0 on (and, the first thread's, the one ahead of a row's first 16 bytes): what each weighs
template <typename T, int N> struct dv_left { double v[N], v0; };
template <typename T, int N>
__device__ inline void dv_weigh(const dv_args &a, const dv_row &r, const char *src, const float *drafter, int i0, int base, int begin, int end, double cold, double inv, bool some, const uint32_t *out, dv_left<T, N> &w, double &plain)
{
    float x[N], d[N], x0 = -INFINITY, d0 = 0.f;
    dv_tokens<T, N>(src, drafter, i0, end, x, d);
    if (i0 == base && begin < base) { x0 = dv_one<T>(src, 0); if (drafter != nullptr) d0 = drafter[0]; }
    if (some) {
        auto is = [&](int i) { return (out[(i - begin) >> 5] >> ((i - begin) & 31)) & 1u; };
#pragma unroll
        for (int k = 0; k < N; ++k) if (i0 + k < end && is(i0 + k)) x[k] = -INFINITY;
        if (begin < base && is(0)) x0 = -INFINITY;
    }
    plain = dv_weight(x0, cold, r.top) * inv;
    w.v0 = fmax(plain - (double)d0, 0.0);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const double p = dv_weight(x[k], cold, r.top) * inv;
        plain += p;
        w.v[k] = fmax(p - (double)d[k], 0.0);
    }
}

// Whether the draw behind row w.x is from max(p - q, 0)
__device__ inline bool dv_drawn(const dv_args &a, int2 w) { return w.y && a.probs != nullptr; }

// What is left to draw from in a segment: relative to its own largest logit, of refused tokens too, so that the row need not have been summed before; under a drafter's probabilities to the row's sum.  A chain's walk is made anew by every workgroup: it is three trips to memory, a launch for it costs more.
template <typename T>
__global__ void __launch_bounds__(256)
k_draft_rest(const dv_args a)
{
    constexpr int NT = 256, N = DV_SIZE / NT / 2;
    __shared__ dv_chain_lds sh_chain;
    __shared__ double2 sh_sum[4];
    __shared__ float sh_top[4];
    __shared__ int sh_first[4];
    __shared__ uint32_t sh_out[(DV_SIZE + 32) / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = blockIdx.x / a.left, seg = blockIdx.x - s * a.left;
    const dv_seq q = dv_seq_at(a, s);
    const double cold = dv_cold(a, s);
    if (q.rows == 0) return;
    const int2 w = a.parent != nullptr ? a.walk[s] : dv_chain<T>(a, q, cold, seg == 0, &sh_chain);
    if (a.parent == nullptr && seg == 0) {
        if (tid == 0) { a.walk[s] = w; a.accepted[s] = w.x - q.row0; a.out_probs[q.row0] = 1.f; }
        if (a.path != nullptr) for (int i = tid; i <= w.x - q.row0; i += NT) a.path[q.row0 + i] = i;
    }
    const char *src = a.logits + (int64_t)w.x * a.row_bytes;
    const int head = dv_head<T>(src), base = head + seg * DV_SIZE, begin = dv_begin(seg, head, DV_SIZE), end = min(base + DV_SIZE, a.vocab);
    const bool some = dv_refused(a, q, w, begin, end, sh_out);
    if (cold == 0.0 || !dv_drawn(a, w)) {
        float x[2][N], d[N], x0 = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k) dv_tokens<T, N>(src, nullptr, base + (k * NT + tid) * N, end, x[k], d);
        if (tid == 0 && begin < base) x0 = dv_one<T>(src, 0);
        float top = fmaxf(x0, -INFINITY);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, x[k][i]);
        top = over_wave(top, op_max);
        if (lane == 0) sh_top[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(sh_top[0], sh_top[1]), fmaxf(sh_top[2], sh_top[3]));
        double sum = 0.0;
        int id = 0x7fffffff;
        auto is = [&](int i) { return some && ((sh_out[(i - begin) >> 5] >> ((i - begin) & 31)) & 1u); };
        if (cold > 0.0) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) { const int t = base + (k * NT + tid) * N + i; const double v = dv_weight(x[k][i], cold, top); sum += t < end && is(t) ? 0.0 : v; }
            if (tid == 0 && begin < base && !is(0)) sum += dv_weight(x0, cold, top);
            sum = dv_over_wave(sum);
        } else {
            if (tid == 0 && begin < base && x0 == top) id = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) if (x[k][i] == top) id = min(id, base + (k * NT + tid) * N + i);      // (behind the row's end: only if the segment has nothing but -infinity)
            id = dv_min_over_wave(id);
        }
        if (lane == 0) { sh_sum[wave].x = sum; sh_first[wave] = id; }
        __syncthreads();
        if (tid == 0) {
            dv_part p;
            p.sum = (sh_sum[0].x + sh_sum[1].x) + (sh_sum[2].x + sh_sum[3].x); p.top = top; p.first = min(min(sh_first[0], sh_first[1]), min(sh_first[2], sh_first[3]));
            ((dv_part *)a.rest)[(int64_t)s * a.left + seg] = p;
        }
        return;
    }
    const dv_row r = sh_chain.row;
    const float *drafter = a.probs + (int64_t)(w.x + 1) * a.probs_row;
    const double inv = 1.0 / r.sum;
    double sum = 0.0, all = 0.0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        dv_left<T, N> v;
        double plain;
        dv_weigh<T, N>(a, r, src, drafter, base + (k * NT + tid) * N, base, begin, end, cold, inv, some, sh_out, v, plain);
        sum += v.v0; all += plain;
#pragma unroll
        for (int i = 0; i < N; ++i) sum += v.v[i];
    }
    sum = dv_over_wave(sum); all = dv_over_wave(all);
    if (lane == 0) sh_sum[wave] = make_double2(sum, all);
    __syncthreads();
    if (tid == 0) a.rest[(int64_t)s * a.left + seg] = make_double2((sh_sum[0].x + sh_sum[1].x) + (sh_sum[2].x + sh_sum[3].x), (sh_sum[0].y + sh_sum[1].y) + (sh_sum[2].y + sh_sum[3].y));
}

// The draw of a sequence.  Four trips to memory, one behind the other.
template <typename T>
__global__ void __launch_bounds__(512)
k_draft_pick(const dv_args a)
{
    constexpr int NT = 512, NW = NT / 64, N = DV_SIZE / NT, SC = DV_MAX_SEGS / 64;
    __shared__ double sh_wave[NW];
    __shared__ int sh_pick, sh_id;
    __shared__ uint32_t sh_out[(DV_SIZE + 32) / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = blockIdx.x;
    const dv_seq q = dv_seq_at(a, s);
    const int2 w = a.walk[s];                // (of a sequence without rows: anything)
    const double2 *rest = a.rest + (int64_t)s * a.left;
    double2 first[1];
    first[0] = lane < a.left ? rest[lane] : make_double2(0.0, 0.0);
    const double cold = dv_cold(a, s);
    if (q.rows == 0) { if (tid == 0) { a.accepted[s] = 0; a.next[s] = -1; } return; }
    const double u = dv_u(a, w.x, 1);
    const char *src = a.logits + (int64_t)w.x * a.row_bytes;
    const int head = dv_head<T>(src);
    bool drawn = dv_drawn(a, w);
    dv_row r = {1.0, -INFINITY, 0x7fffffff, false};          // (nothing but its ratios counts of a row that p alone is drawn from)
    if (drawn && cold > 0.0) r = dv_row_of<64>(a, w.x, cold, dv_parts_of<64>(a, w.x));
    else {
        const dv_part *p = (const dv_part *)rest;
        const dv_part mine = __builtin_bit_cast(dv_part, first[0]);
        if (lane < a.left) r.top = mine.top;
        for (int i = 64 + lane; i < a.left; i += 64) r.top = fmaxf(r.top, p[i].top);
        r.top = over_wave(r.top, op_max);
        r.any = r.top > -INFINITY && r.top < INFINITY;
        if (cold == 0.0) {
            if (lane < a.left && mine.top == r.top) r.first = mine.first;
            for (int i = 64 + lane; i < a.left; i += 64) if (p[i].top == r.top) r.first = min(r.first, p[i].first);
            r.first = dv_min_over_wave(r.first);
        }
    }
    if (tid == 0) sh_id = -1;
    if (!r.any) { if (tid == 0) a.next[s] = -1; return; }
    if (cold == 0.0) { if (tid == 0) a.next[s] = r.first; return; }      // (with a refused draft too: it was another token)
    const double inv = 1.0 / r.sum;
    // what the segments weigh, a lane a segment, in every wave alike
    double sums[SC], total = 0.0;            // (up to and with each)
    const bool whole = !drawn;
    for (int pass = 0; pass < 2; ++pass) {   // (nothing left of p - q, which rounding can bring about: p)
        total = 0.0;
#pragma unroll
        for (int c = 0; c < SC; ++c) {
            sums[c] = 0.0;
            if (c * 64 >= a.left) continue;
            const double2 v = c == 0 ? first[0] : c * 64 + lane < a.left ? rest[c * 64 + lane] : make_double2(0.0, 0.0);
            double some = drawn ? v.x : v.y;
            if (whole) {
                const dv_part part = __builtin_bit_cast(dv_part, v);
                some = c * 64 + lane < a.left && part.sum > 0.0 ? part.sum * dv_weight(part.top, cold, r.top) : 0.0;
            }
            sums[c] = total + dv_up_to(some);
            total = __shfl(sums[c], 63, 64);
        }
        if (total > 0.0 || !drawn) break;
        drawn = false;
    }
    const double target = u * total;
    // the first segment whose sum passes the target, or the last that weighs anything, and the sum before it
    int picked = -1;
    double before_it = 0.0;
    {
        double before = 0.0;
        bool found = false;
#pragma unroll
        for (int c = 0; c < SC; ++c) {
            if (c * 64 >= a.left || found) continue;
            double b = __shfl_up(sums[c], 1, 64);
            if (lane == 0) b = before;
            const uint64_t some = __ballot(sums[c] > b), past = __ballot(sums[c] > b && sums[c] > target);
            const int l = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : 0;
            if (some) { picked = c * 64 + l; before_it = __shfl(b, l, 64); }
            found = past != 0;
            before = __shfl(sums[c], 63, 64);
        }
    }
    const float *drafter = drawn ? a.probs + (int64_t)(w.x + 1) * a.probs_row : nullptr;
    __syncthreads();
    // the segment, and, should rounding have left nothing in it, the others in turn
    for (int turn = picked < 0 ? 0 : -1; turn < a.left; ++turn) {
        const int seg = turn < 0 ? picked : turn, base = head + seg * DV_SIZE, begin = dv_begin(seg, head, DV_SIZE), end = min(base + DV_SIZE, a.vocab), i0 = base + tid * N;
        const bool some_out = dv_refused(a, q, w, begin, end, sh_out);
        dv_left<T, N> v;                     // a thread's tokens lie side by side
        double plain;
        dv_weigh<T, N>(a, r, src, drafter, i0, base, begin, end, cold, inv, some_out, sh_out, v, plain);
        double mine = v.v0;
#pragma unroll
        for (int k = 0; k < N; ++k) mine += v.v[k];
        const double upto = dv_up_to(mine);
        if (lane == 63) sh_wave[wave] = upto;
        if (tid == 0) sh_pick = 0x7fffffff;
        __syncthreads();
        double b = turn < 0 ? before_it : 0.0;
        for (int k = 0; k < wave; ++k) b += sh_wave[k];
        b += upto - mine;
        const double bound = turn < 0 ? target : -1.0;
        const uint64_t some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && b + mine > bound);
        if (lane == 0) {
            if (past) atomicMin(&sh_pick, wave * 64 + __ffsll((unsigned long long)past) - 1);
            if (some) atomicMax(&sh_id, wave * 64 + 63 - __clzll((long long)some));      // (the last thread that has any)
        }
        __syncthreads();
        const int who = sh_pick != 0x7fffffff ? sh_pick : sh_id;
        __syncthreads();
        if (who < 0) continue;               // (the same for all)
        if (tid == who) {
            double sum = b + v.v0;
            int id = v.v0 > 0.0 ? 0 : -1;
            bool stop = v.v0 > 0.0 && sum > bound;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                sum += v.v[k];
                if (!stop && v.v[k] > 0.0) { id = i0 + k; stop = sum > bound; }
            }
            a.next[s] = id;
        }
        return;
    }
    if (tid == 0) a.next[s] = -1;            // nothing has any probability left
}

// ------------------------------- host side ----------------------------------------

// Tokens a segment of a row: 4096, or, where there are rows enough for the chip, 8192 (64-bit sums), 14336 (what registers hold at seven waves a SIMD; of 16 trees' 35 us 12288 at eight took 0.6 more, 16384 at six 0.2) or (f32) 8192.  Whether there is a drafter is not known where the workspace is measured: its size is that of 4096.
struct dv_plan { int e, segs, left; };
static dv_plan plan(int64_t rows, int vocab, bool wide, int dtype)
{
    dv_plan p;
    p.left = (vocab + DV_SIZE - 1) / DV_SIZE;
    p.e = rows * p.left <= 4096 ? 16 : wide || dtype == PV_F32 ? 32 : 56;
    p.segs = (vocab + 256 * p.e - 1) / (256 * p.e);
    return p;
}

static int check(int64_t rows, int n_seq, int vocab)
{
    if (rows < 0 || rows > (1 << 20)) { pv_set_error("rows %lld outside [0, 2^20]", (long long)rows); return PV_ERANGE; }
    if (n_seq < 0 || n_seq > (1 << 20)) { pv_set_error("n_seq %d outside [0, 2^20]", n_seq); return PV_ERANGE; }
    if (vocab < 1 || vocab > DV_SIZE * DV_MAX_SEGS) { pv_set_error("vocab %d outside [1, %d]", vocab, DV_SIZE * DV_MAX_SEGS); return PV_ERANGE; }
    // a launch has less than 2^32 threads
    const int64_t segs = (vocab + DV_SIZE - 1) / DV_SIZE;
    if (rows * segs >= (1 << 24) || n_seq * segs >= (1 << 24)) { pv_set_error("%lld rows, %d sequences of %d tokens: more than a launch takes", (long long)rows, n_seq, vocab); return PV_ERANGE; }
    return PV_OK;
}

static size_t bytes_of(int64_t rows, int n_seq, int vocab)
{
    const size_t segs = (vocab + DV_SIZE - 1) / DV_SIZE;
    return rows && n_seq ? (size_t)rows * segs * sizeof(dv_part) + (size_t)n_seq * segs * sizeof(double2) + (size_t)n_seq * sizeof(int2) : 0;
}

extern "C" int pv_verify_drafts_bytes(int64_t rows, int32_t n_seq, int32_t vocab, size_t *bytes)
{
    const int rc = check(rows, n_seq, vocab);
    if (rc != PV_OK) return rc;
    if (!bytes) { pv_set_error("null output pointer"); return PV_EINVAL; }
    *bytes = bytes_of(rows, n_seq, vocab);
    return PV_OK;
}

// a call without rows, or without sequences: every sequence is empty, every row of none
__global__ void __launch_bounds__(256) k_draft_none(int n_seq, int32_t *accepted, int32_t *next, int rows, int32_t *path, float *probs)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n_seq) { accepted[i] = 0; next[i] = -1; }
    if (i < rows) { if (path != nullptr) path[i] = -1; probs[i] = 0.f; }
}

template <typename T>
static int launch(const dv_args &a, int e, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.rows * a.segs);
    if (a.probs != nullptr) {
        if (e == 16) k_draft_rows<T, 16, true><<<grid, 256, 0, s>>>(a);
        else k_draft_rows<T, 32, true><<<grid, 256, 0, s>>>(a);
    } else {
        constexpr int most = sizeof(T) == 4 ? 32 : 56;
        if (e == 16) k_draft_rows<T, 16, false><<<grid, 256, 0, s>>>(a);
        else k_draft_rows<T, most, false><<<grid, 256, 0, s>>>(a);
    }
    PV_HIP(hipGetLastError());
    if (a.parent != nullptr) { k_draft_walk<T><<<(unsigned)a.n_seq, 1024, 0, s>>>(a); PV_HIP(hipGetLastError()); }
    k_draft_rest<T><<<(unsigned)(a.n_seq * a.left), 256, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    k_draft_pick<T><<<(unsigned)a.n_seq, 512, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    return PV_OK;
}

extern "C" int pv_verify_drafts(const int32_t *row_start, int32_t n_seq, const void *logits, int64_t row_stride, int32_t dtype, int64_t rows, int32_t vocab, const int32_t *tokens,
                                const void *u, int32_t u_is_double, const float *draft_probs, int64_t draft_row_stride, const int32_t *parent, const float *temperatures, float temperature,
                                int32_t *accepted, int32_t *next_token, int32_t *path, float *probs, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = check(rows, n_seq, vocab);
    if (rc != PV_OK) return rc;
    if (dtype != PV_F32 && dtype != PV_BF16 && dtype != PV_F16) { pv_set_error("bad dtype %d", dtype); return PV_EINVAL; }
    if (parent && draft_probs) { pv_set_error("a tree's drafts go without a drafter's probabilities"); return PV_EINVAL; }
    if (n_seq == 0 && rows == 0) return PV_OK;
    if (!row_start || (n_seq && (!accepted || !next_token)) || (rows && (!logits || !tokens || !u || !probs)) || (rows && parent && !path)) { pv_set_error("null pointer"); return PV_EINVAL; }
    if (row_stride < 0 || draft_row_stride < 0) { pv_set_error("negative row stride"); return PV_EINVAL; }
    if (!temperatures && !(temperature >= 0.f)) { pv_set_error("temperature %g is not 0 or more", (double)temperature); return PV_EINVAL; }
    const int64_t size = dtype == PV_F32 ? 4 : 2;
    if ((uintptr_t)logits % size || ((uintptr_t)row_start | (uintptr_t)tokens | (uintptr_t)draft_probs | (uintptr_t)parent | (uintptr_t)temperatures | (uintptr_t)accepted | (uintptr_t)next_token | (uintptr_t)path | (uintptr_t)probs) & 3
        || (uintptr_t)u & (u_is_double ? 7 : 3)) { pv_set_error("an array is not aligned to its type"); return PV_EINVAL; }
    const dv_plan p = plan(rows, vocab, draft_probs != nullptr, dtype);
    const size_t need = bytes_of(rows, n_seq, vocab);
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    dv_args a = {};
    a.logits = (const char *)logits; a.row_bytes = row_stride * size; a.rows = (int)rows; a.vocab = vocab; a.segs = p.segs; a.left = p.left; a.n_seq = n_seq;
    a.row_start = row_start; a.tokens = tokens; a.parent = parent; a.u = u; a.u64 = u_is_double != 0; a.probs = draft_probs; a.probs_row = draft_row_stride;
    a.temperature = temperatures; a.hot = temperature; a.accepted = accepted; a.next = next_token; a.path = path; a.out_probs = probs;
    hipStream_t s = (hipStream_t)hip_stream;
    if (rows == 0 || n_seq == 0) {
        k_draft_none<<<(unsigned)(((rows > n_seq ? (int)rows : n_seq) + 255) / 256), 256, 0, s>>>(n_seq, accepted, next_token, (int)rows, path, probs);
        const hipError_t err = hipGetLastError();
        if (n_seq == 0 && err == hipErrorNoDevice) return PV_OK;         // (a call without sequences has nothing to verify: where there is no device there is nothing to write to either)
        PV_HIP(err);
        return PV_OK;
    }
    a.part = (dv_part *)workspace; a.rest = (double2 *)(a.part + (size_t)rows * p.left); a.walk = (int2 *)(a.rest + (size_t)n_seq * p.left);
    return dtype == PV_F32 ? launch<float>(a, p.e, s) : dtype == PV_BF16 ? launch<__bf16>(a, p.e, s) : launch<_Float16>(a, p.e, s);
}
