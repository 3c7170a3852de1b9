// Drafted tokens verified against the target's probabilities, from given random numbers (speculative sampling).
//
//   p_j = softmax(logits_j / T) of row j;  the draft in row c, behind row j, with its random number u and the drafter's probability q of it, is taken if  u q < p_j(draft).  If not, what follows row j is drawn
//   from max(p_j - q, 0), or, where no drafter's probabilities are given (q is one at the draft), from p_j without the draft; behind the last draft from p.  A node of a tree has its children tried in order,
//   each under what the refused ones before it left: taken if u (1 - sum of their p) < p_j(draft).
//   The draw: the lowest token at which the sum of probabilities, in the order of ids, passes u' times their whole.
//
// The result is whole numbers, so what they turn on is computed in 64 bits: with exponentials of 32 bits a sum over a vocabulary of 10^5 lands on the wrong side of u' once in some 10^5 draws.  A
// workgroup takes a segment of a row: its maximum and the sum of its exponentials.  One workgroup a sequence joins the segments of the rows that it walks along, and reads again the one segment in which the draw falls; where a
// refused draft has a drafter's probabilities, every segment of that row is summed anew first, under max(p - q, 0).
#include "pv_matrix_common.h"

struct dv_part { double sum; float top; int first; };       // of a segment: sum of e^((x - top) / T), largest logit, its lowest id (T = 0: no sum)

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
    double *rest;                           // [seq][seg]
    int2 *walk;                             // [seq]: row that the draw is behind, whether a draft was refused there
};

struct dv_seq { int row0, rows; };
__device__ inline dv_seq dv_seq_at(const dv_args &a, int s)
{
    dv_seq q;
    q.row0 = a.row_start[s];
    q.rows = min(a.row_start[s + 1], a.rows) - q.row0;
    if (q.row0 < 0 || q.rows < 0) q.rows = 0;
    return q;
}
// 1 / T (of infinity: next to nothing); 0: the most probable token alone
__device__ inline double dv_cold(const dv_args &a, int s)
{
    const float t = a.temperature != nullptr ? a.temperature[s] : a.hot;
    return t > 0.f ? fmax(1.0 / (double)t, 1e-300) : 0.0;
}
__device__ inline double dv_u(const dv_args &a, int row, int which)
{
    const int64_t i = 2 * (int64_t)row + which;
    return a.u64 ? ((const double *)a.u)[i] : (double)((const float *)a.u)[i];
}

// e^y, y <= 0 or NaN: 2^n times the series of e^z, |z| <= ln(2) / 2, up to z^11 (what is left out is below 10^-14)
__device__ inline double dv_exp(double y)
{
    const double t = fmax(y * 1.4426950408889634074, -1100.0), n = rint(t), z = (t - n) * 0.69314718055994530942;
    double e = 1.0 / 39916800.0;
    e = fma(e, z, 1.0 / 3628800.0); e = fma(e, z, 1.0 / 362880.0); e = fma(e, z, 1.0 / 40320.0); e = fma(e, z, 1.0 / 5040.0); e = fma(e, z, 1.0 / 720.0);
    e = fma(e, z, 1.0 / 120.0); e = fma(e, z, 1.0 / 24.0); e = fma(e, z, 1.0 / 6.0); e = fma(e, z, 0.5); e = fma(e, z, 1.0); e = fma(e, z, 1.0);
    return ldexp(e, (int)n);
}
__device__ inline double dv_weight(float x, float top, double cold) { return x > -INFINITY ? dv_exp(((double)x - (double)top) * cold) : 0.0; }      // (NaN: 0)

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

// 16 bytes from an address that is a multiple of 4
typedef __attribute__((ext_vector_type(4), aligned(4))) unsigned int dv_u32x4;
__device__ inline u32x4 dv_load16(const char *p) { const dv_u32x4 v = *(const dv_u32x4 *)p; return (u32x4){v.x, v.y, v.z, v.w}; }

__device__ inline double dv_over_wave(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ inline int dv_min_over_wave(int v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d, 64));
    return v;
}

// Segment seg of a row: tokens begin(seg) .. begin(seg + 1) - 1.  Its 16 bytes of a thread begin at a multiple of four bytes: a row of 16-bit numbers that does not has one token more in its first segment.
template <typename T> __device__ inline int dv_head(const char *src) { return sizeof(T) == 2 && ((uintptr_t)src & 2) ? 1 : 0; }
__device__ inline int dv_begin(int seg, int head, int size) { return seg == 0 ? 0 : head + seg * size; }

template <typename T, int E>
__global__ void __launch_bounds__(256)
k_draft_rows(const dv_args a)
{
    constexpr int NT = 256, V = 16 / (int)sizeof(T), U = E / V, D = E * (int)sizeof(T) / 4, SIZE = NT * E;
    __shared__ float sh_top[4];
    __shared__ double sh_sum[4];
    __shared__ int sh_first[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / a.segs, seg = blockIdx.x - row * a.segs;
    const char *src = a.logits + (int64_t)row * a.row_bytes;
    const int head = dv_head<T>(src), base = head + seg * SIZE;
    uint32_t x[D];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i0 = base + (u * NT + tid) * V;
        constexpr uint32_t inf = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u;      // -infinity
        u32x4 v = {inf, inf, inf, inf};
        if (i0 + V <= a.vocab) v = dv_load16(src + (int64_t)i0 * sizeof(T));
        x[4 * u] = v.x; x[4 * u + 1] = v.y; x[4 * u + 2] = v.z; x[4 * u + 3] = v.w;
    }
    // those that no 16 bytes hold: ahead of the first, behind the last
    const int behind = (a.vocab - head) % V;
    const int alone = tid == 0 ? (seg == 0 && head ? 0 : -1) : tid <= behind && seg == (a.vocab - behind - head) / SIZE ? a.vocab - behind + tid - 1 : -1;
    const float x0 = alone >= 0 ? dv_one<T>(src, alone) : -INFINITY;
    int s = 0;
    for (int k = 0; k < a.n_seq; k += 64) {
        const int end = k + lane < a.n_seq ? a.row_start[k + lane + 1] : 0x7fffffff;
        s += __popcll(__ballot(end <= row));
    }
    if (tid == 0 && seg == 0) {
        if (a.path != nullptr) a.path[row] = -1;
        a.out_probs[row] = 0.f;              // (rows of a sequence: below)
    }
    if (s >= a.n_seq) return;
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
        sum = dv_weight(x0, top, cold);
#pragma unroll
        for (int i = 0; i < E; ++i) sum += dv_weight(dv_get<T>(x, i), top, cold);
        sum = dv_over_wave(sum);
    } else {
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

// A row's segments joined, by each GL lanes side by side: largest logit, sum of exponentials, the lowest id of the largest
struct dv_row { float top; double sum; int first; bool any; };      // any: it has probabilities (its largest logit is a number)
template <int GL> __device__ inline dv_row dv_row_of(const dv_args &a, int row, double cold)
{
    const int l = threadIdx.x % GL;
    const dv_part *p = a.part + (int64_t)row * a.segs;
    dv_row r = {-INFINITY, 0.0, 0x7fffffff, false};
    for (int i = l; i < a.segs; i += GL) r.top = fmaxf(r.top, p[i].top);
#pragma unroll
    for (int d = 1; d < GL; d <<= 1) r.top = fmaxf(r.top, __shfl_xor(r.top, d, 64));
    r.any = r.top > -INFINITY && r.top < INFINITY;
    for (int i = l; i < a.segs; i += GL) {
        const dv_part q = p[i];
        if (cold > 0.0) r.sum += q.sum * dv_weight(q.top, r.top, cold);
        else if (q.top == r.top) r.first = min(r.first, q.first);
    }
#pragma unroll
    for (int d = 1; d < GL; d <<= 1) { r.sum += __shfl_xor(r.sum, d, 64); r.first = min(r.first, __shfl_xor(r.first, d, 64)); }
    return r;
}
template <typename T> __device__ inline double dv_prob(const dv_args &a, const dv_row &r, int row, int token, double cold)
{
    if (!r.any || token < 0 || token >= a.vocab) return 0.0;
    if (cold == 0.0) return token == r.first ? 1.0 : 0.0;
    return dv_weight(dv_one<T>(a.logits + (int64_t)row * a.row_bytes, token), r.top, cold) / r.sum;
}

// A chain: which drafts are taken, all looked at side by side, 16 lanes each.  The row behind which the draw is, and whether a draft was refused there.
template <typename T> __device__ inline int2 dv_chain(const dv_args &a, const dv_seq &q, double cold, bool write, int *sh_refused)
{
    constexpr int GL = 16;
    if (threadIdx.x == 0) *sh_refused = q.rows;
    __syncthreads();
    const int n = blockDim.x / GL;
    for (int j0 = 1; j0 < q.rows; j0 += n) {             // (uniform: lanes without a draft look at the last one)
        const int j = min(j0 + (int)threadIdx.x / GL, q.rows - 1), row = q.row0 + j, token = a.tokens[row];
        const dv_row r = dv_row_of<GL>(a, row - 1, cold);
        const double p = dv_prob<T>(a, r, row - 1, token, cold);
        const double d = a.probs == nullptr ? 1.0 : token >= 0 && token < a.vocab ? (double)a.probs[(int64_t)row * a.probs_row + token] : 0.0;
        if (threadIdx.x % GL == 0) {
            if (!(dv_u(a, row, 0) * d < p)) atomicMin(sh_refused, j);
            if (write) a.out_probs[row] = (float)p;
        }
    }
    __syncthreads();
    const int refused = *sh_refused;
    return make_int2(q.row0 + min(refused, q.rows) - 1, refused < q.rows);
}

// max(p - q, 0) of a segment's tokens, summed, where a draft with a drafter's probabilities was refused
template <typename T, int E>
__global__ void __launch_bounds__(256)
k_draft_rest(const dv_args a)
{
    constexpr int NT = 256, SIZE = NT * E;
    __shared__ int sh_refused;
    __shared__ double sh_sum[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = blockIdx.x / a.segs, seg = blockIdx.x - s * a.segs;
    const dv_seq q = dv_seq_at(a, s);
    if (q.rows == 0) return;
    const double cold = dv_cold(a, s);
    const int2 w = dv_chain<T>(a, q, cold, seg == 0, &sh_refused);
    if (seg == 0 && tid == 0) a.walk[s] = w;
    if (!w.y || cold == 0.0) return;
    const dv_row r = dv_row_of<64>(a, w.x, cold);
    const char *src = a.logits + (int64_t)w.x * a.row_bytes;
    const float *drafter = a.probs + (int64_t)(w.x + 1) * a.probs_row;
    const int head = dv_head<T>(src), begin = dv_begin(seg, head, SIZE), end = min(dv_begin(seg + 1, head, SIZE), a.vocab);
    const double inv = 1.0 / r.sum;
    double sum = 0.0;
    for (int i = begin + tid; i < end; i += NT) sum += fmax(dv_weight(dv_one<T>(src, i), r.top, cold) * inv - (double)drafter[i], 0.0);
    sum = dv_over_wave(sum);
    if (lane == 0) sh_sum[wave] = sum;
    __syncthreads();
    if (tid == 0) a.rest[(int64_t)s * a.segs + seg] = (sh_sum[0] + sh_sum[1]) + (sh_sum[2] + sh_sum[3]);
}

// The draw of a sequence, and before it the walk along its tree.
#define DV_NODES 1024                       // nodes at a time
#define DV_MAX_SEGS 512
template <typename T, int E>
__global__ void __launch_bounds__(512)
k_draft_pick(const dv_args a)
{
    constexpr int NT = 512, NW = NT / 64, SIZE = 256 * E, GL = 16;
    __shared__ double sh_p[DV_NODES], sh_seg[DV_MAX_SEGS], sh_wave[NW];
    __shared__ int sh_parent[DV_NODES], sh_token[DV_NODES], sh_refused, sh_pick, sh_id;
    __shared__ uint32_t sh_out[(SIZE + 32) / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = blockIdx.x;
    const dv_seq q = dv_seq_at(a, s);
    if (q.rows == 0) { if (tid == 0) { a.accepted[s] = 0; a.next[s] = -1; } return; }
    const double cold = dv_cold(a, s);
    int node = q.row0, depth = 0;           // the row that the draw is behind
    bool refused = false;                   // ... under a drafter's probabilities
    for (int i = tid; i < a.segs; i += NT) sh_seg[i] = 0.0;
    if (a.parent == nullptr) {
        int2 w;
        if (a.probs != nullptr) w = a.walk[s];
        else w = dv_chain<T>(a, q, cold, true, &sh_refused);
        node = w.x; refused = w.y != 0; depth = node - q.row0;
        if (a.path != nullptr) for (int i = tid; i <= depth; i += NT) a.path[q.row0 + i] = i;
        if (tid == 0) a.out_probs[q.row0] = 1.f;
    } else {
        if (tid == 0) { a.path[q.row0] = 0; a.out_probs[q.row0] = 1.f; }
        int at = 0;
        double left = 1.0;
        for (int n0 = 1; n0 < q.rows; n0 += DV_NODES) {
            const int n = min(DV_NODES, q.rows - n0);
            for (int i0 = 0; i0 < n; i0 += NT / GL) {
                const int i = min(i0 + tid / GL, n - 1), local = n0 + i, up = a.parent[q.row0 + local], token = a.tokens[q.row0 + local];
                const bool good = up >= 0 && up < local;
                const int over = q.row0 + (good ? up : 0);
                const dv_row r = dv_row_of<GL>(a, over, cold);
                const double p = good ? dv_prob<T>(a, r, over, token, cold) : 0.0;
                if (tid % GL == 0) { sh_p[i] = p; sh_parent[i] = good ? up : -1; sh_token[i] = token; a.out_probs[q.row0 + local] = (float)p; }
            }
            __syncthreads();
            if (wave == 0) {
                for (int b = 0; b < n; b += 64) {
                    const int i = b + lane;
                    const int up = i < n ? sh_parent[i] : -2;
                    uint64_t todo = __ballot(up == at);
                    while (todo) {
                        const int k = b + __ffsll((unsigned long long)todo) - 1, token = sh_token[k], row = q.row0 + n0 + k;
                        // a token that an earlier child has had
                        bool had = false;
                        for (int j = max(at + 1, 1) - n0; j < k; j += 64) {
                            const int c = j + lane;
                            bool same = false;
                            if (c < k) same = c >= 0 ? sh_parent[c] == at && sh_token[c] == token : a.parent[q.row0 + n0 + c] == at && a.tokens[q.row0 + n0 + c] == token;
                            had = had || __any(same);
                        }
                        const double p = had ? 0.0 : sh_p[k];
                        todo &= todo - 1;
                        if (dv_u(a, row, 0) * left < p) {
                            at = n0 + k; ++depth; left = 1.0;
                            if (lane == 0) a.path[q.row0 + depth] = at;
                            for (int j = lane; j < a.segs; j += 64) sh_seg[j] = 0.0;
                            const uint64_t past = k - b == 63 ? 0ull : ~0ull << (k - b + 1);
                            todo = __ballot(up == at) & past;
                        } else {
                            left -= p;
                            if (p > 0.0 && lane == 0) {
                                const int head = dv_head<T>(a.logits + (int64_t)(q.row0 + at) * a.row_bytes);
                                sh_seg[max(token - head, 0) / SIZE] += p;
                            }
                        }
                    }
                }
                if (lane == 0) { sh_refused = at; sh_pick = depth; sh_wave[0] = left; }
            }
            __syncthreads();
            at = sh_refused; depth = sh_pick; left = sh_wave[0];
            __syncthreads();
        }
        node = q.row0 + at;
    }
    if (tid == 0) { a.accepted[s] = depth; sh_id = -1; }
    __syncthreads();
    const dv_row r = dv_row_of<64>(a, node, cold);
    if (!r.any) { if (tid == 0) a.next[s] = -1; return; }
    if (cold == 0.0) { if (tid == 0) a.next[s] = r.first; return; }      // (with a refused draft too: it was another token)
    const char *src = a.logits + (int64_t)node * a.row_bytes;
    const int head = dv_head<T>(src);
    // without a drafter's probabilities: the refused tokens
    const int last = a.probs != nullptr ? 0 : a.parent != nullptr ? q.rows : refused ? node - q.row0 + 2 : 0;
    const int from = node - q.row0 + 1;
    if (a.probs == nullptr && a.parent == nullptr && refused && tid == 0) {
        const int token = a.tokens[node + 1];
        if (token >= 0 && token < a.vocab) sh_seg[max(token - head, 0) / SIZE] = dv_prob<T>(a, r, node, token, cold);
    }
    __syncthreads();
    // what the segments weigh
    const double inv = 1.0 / r.sum;
    double total = 0.0;
    for (int pass = 0; pass < 2 && !(total > 0.0); ++pass) {      // (nothing left of p - q, which rounding can bring about: p)
        if (pass == 1) refused = false;
        for (int i = tid; i < a.segs; i += NT) {
            double w;
            if (refused && a.probs != nullptr) w = a.rest[(int64_t)s * a.segs + i];
            else { const dv_part p = a.part[(int64_t)node * a.segs + i]; w = p.sum * dv_weight(p.top, r.top, cold) * inv - (a.probs != nullptr ? 0.0 : sh_seg[i]); }
            sh_seg[i] = fmax(w, 0.0);
        }
        __syncthreads();
        if (wave == 0) {
            // sums up to each segment, 64 at a time
            double before = 0.0;
            for (int k = 0; k < a.segs; k += 64) {
                double v = k + lane < a.segs ? sh_seg[k + lane] : 0.0;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) { const double o = __shfl_up(v, d, 64); if (lane >= d) v += o; }
                v += before;
                before = __shfl(v, 63, 64);
                if (k + lane < a.segs) sh_seg[k + lane] = v;      // (from here on: the sum up to and with it)
            }
            if (lane == 0) sh_wave[0] = before;
        }
        __syncthreads();
        total = sh_wave[0];
        __syncthreads();
        if (a.probs == nullptr) break;
    }
    const double target = dv_u(a, node, 1) * total;
    if (wave == 0) {
        int pick = 0x7fffffff, some = -1;     // the first segment whose sum passes the target; the last that weighs anything
        for (int k = lane; k < a.segs; k += 64) {
            const double v = sh_seg[k], b = k > 0 ? sh_seg[k - 1] : 0.0;
            if (v > b) { some = max(some, k); if (v > target) pick = min(pick, k); }
        }
        pick = dv_min_over_wave(pick);
        some = -dv_min_over_wave(-some);
        if (lane == 0) sh_pick = pick != 0x7fffffff ? pick : max(some, 0);
    }
    __syncthreads();
    const int picked = sh_pick;
    const float *drafter = refused && a.probs != nullptr ? a.probs + (int64_t)(node + 1) * a.probs_row : nullptr;
    // the segment, and, should rounding have left nothing in it, the others in turn
    for (int turn = -1; turn < a.segs; ++turn) {
        const int seg = turn < 0 ? picked : turn;
        const int begin = dv_begin(seg, head, SIZE), end = min(dv_begin(seg + 1, head, SIZE), a.vocab);
        for (int i = tid; i < (SIZE + 32) / 32; i += NT) sh_out[i] = 0u;
        __syncthreads();
        for (int i = from + tid; i < last; i += NT) {
            const int token = a.tokens[q.row0 + i];
            const bool out = a.parent == nullptr || a.parent[q.row0 + i] == node - q.row0;
            if (out && token >= begin && token < end) atomicOr(&sh_out[(token - begin) >> 5], 1u << ((token - begin) & 31));
        }
        __syncthreads();
        // a thread's tokens lie side by side
        const int per = (end - begin + NT - 1) / NT, i0 = begin + tid * per, i1 = min(i0 + per, end);
        auto weight = [&](int i) {
            if ((sh_out[(i - begin) >> 5] >> ((i - begin) & 31)) & 1) return 0.0;
            const double p = dv_weight(dv_one<T>(src, i), r.top, cold) * inv;
            return drafter != nullptr ? fmax(p - (double)drafter[i], 0.0) : p;
        };
        double mine = 0.0;
        for (int i = i0; i < i1; ++i) mine += weight(i);
        double upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) { const double o = __shfl_up(upto, d, 64); if (lane >= d) upto += o; }
        if (lane == 63) sh_wave[wave] = upto;
        if (tid == 0) sh_pick = 0x7fffffff;
        __syncthreads();
        double before = turn < 0 && seg > 0 ? sh_seg[seg - 1] : 0.0;
        for (int k = 0; k < wave; ++k) before += sh_wave[k];
        const double bound = turn < 0 ? target : -1.0, b = before + (upto - mine);
        if (mine > 0.0) {
            if (b + mine > bound) atomicMin(&sh_pick, tid);
            atomicMax(&sh_id, tid);           // the last thread that has any
        }
        __syncthreads();
        const int who = sh_pick != 0x7fffffff ? sh_pick : sh_id;
        __syncthreads();
        if (who < 0) continue;               // (the same for all)
        if (tid == who) {
            double sum = b;
            int id = -1;
            for (int i = i0; i < i1; ++i) {
                const double w = weight(i);
                sum += w;
                if (w > 0.0) { id = i; if (sum > bound) break; }
            }
            a.next[s] = id;
        }
        return;
    }
    if (tid == 0) a.next[s] = -1;            // nothing has any probability left
}

// ------------------------------- host side ----------------------------------------

struct dv_plan { int e, segs; };
static dv_plan plan(int64_t rows, int vocab)
{
    dv_plan p;
    p.e = 16;
    p.segs = (vocab + 256 * p.e - 1) / (256 * p.e);
    return p;
}

static int check(int64_t rows, int n_seq, int vocab)
{
    if (rows < 0 || rows > (1 << 20)) { pv_set_error("rows %lld outside [0, 2^20]", (long long)rows); return PV_ERANGE; }
    if (n_seq < 0 || n_seq > (1 << 20)) { pv_set_error("n_seq %d outside [0, 2^20]", n_seq); return PV_ERANGE; }
    if (vocab < 1 || vocab > 4096 * DV_MAX_SEGS) { pv_set_error("vocab %d outside [1, %d]", vocab, 4096 * DV_MAX_SEGS); return PV_ERANGE; }
    // a launch has less than 2^32 threads
    const dv_plan p = plan(rows, vocab);
    if (rows * p.segs >= (1 << 24) || (int64_t)n_seq * p.segs >= (1 << 24) || (int64_t)n_seq * 512 >= (1ll << 32)) { pv_set_error("%lld rows, %d sequences of %d tokens: more than a launch takes", (long long)rows, n_seq, vocab); return PV_ERANGE; }
    return PV_OK;
}

static size_t bytes_of(int64_t rows, int n_seq, const dv_plan &p)
{
    return (size_t)rows * p.segs * sizeof(dv_part) + (size_t)n_seq * p.segs * sizeof(double) + (size_t)n_seq * sizeof(int2);
}

extern "C" int pv_verify_drafts_bytes(int64_t rows, int32_t n_seq, int32_t vocab, size_t *bytes)
{
    const int rc = check(rows, n_seq, vocab);
    if (rc != PV_OK) return rc;
    if (!bytes) { pv_set_error("null output pointer"); return PV_EINVAL; }
    *bytes = rows && n_seq ? bytes_of(rows, n_seq, plan(rows, vocab)) : 0;
    return PV_OK;
}

template <typename T, int E>
static int launch(const dv_args &a, hipStream_t s)
{
    if (a.rows > 0) { k_draft_rows<T, E><<<(unsigned)(a.rows * a.segs), 256, 0, s>>>(a); PV_HIP(hipGetLastError()); }
    if (a.probs != nullptr && a.rows > 0) { k_draft_rest<T, E><<<(unsigned)(a.n_seq * a.segs), 256, 0, s>>>(a); PV_HIP(hipGetLastError()); }
    k_draft_pick<T, E><<<(unsigned)a.n_seq, 512, 0, s>>>(a);
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
    if (n_seq == 0) return PV_OK;
    if (!row_start || !accepted || !next_token || (rows && (!logits || !tokens || !u || !probs)) || (rows && parent && !path)) { pv_set_error("null pointer"); return PV_EINVAL; }
    if (row_stride < 0 || draft_row_stride < 0) { pv_set_error("negative row stride"); return PV_EINVAL; }
    if (!temperatures && !(temperature >= 0.f)) { pv_set_error("temperature %g is not 0 or more", (double)temperature); return PV_EINVAL; }
    const int64_t size = dtype == PV_F32 ? 4 : 2;
    if ((uintptr_t)logits % size || ((uintptr_t)row_start | (uintptr_t)tokens | (uintptr_t)draft_probs | (uintptr_t)parent | (uintptr_t)temperatures | (uintptr_t)accepted | (uintptr_t)next_token | (uintptr_t)path | (uintptr_t)probs) & 3
        || (uintptr_t)u & (u_is_double ? 7 : 3)) { pv_set_error("an array is not aligned to its type"); return PV_EINVAL; }
    const dv_plan p = plan(rows, vocab);
    const size_t need = rows ? bytes_of(rows, n_seq, p) : 0;
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    dv_args a = {};
    a.logits = (const char *)logits; a.row_bytes = row_stride * size; a.rows = (int)rows; a.vocab = vocab; a.segs = p.segs; a.n_seq = n_seq;
    a.row_start = row_start; a.tokens = tokens; a.parent = parent; a.u = u; a.u64 = u_is_double != 0; a.probs = draft_probs; a.probs_row = draft_row_stride;
    a.temperature = temperatures; a.hot = temperature; a.accepted = accepted; a.next = next_token; a.path = path; a.out_probs = probs;
    a.part = (dv_part *)workspace; a.rest = (double *)(a.part + (size_t)rows * p.segs); a.walk = (int2 *)(a.rest + (size_t)n_seq * p.segs);
    hipStream_t s = (hipStream_t)hip_stream;
    return dtype == PV_F32 ? launch<float, 16>(a, s) : dtype == PV_BF16 ? launch<__bf16, 16>(a, s) : launch<_Float16, 16>(a, s);
}
