// Log probabilities of given tokens under rows of logits, with each row's entropy and most probable tokens.
//
//   lse = M + ln Z, Z = sum e^(x - M), M = max x;  log p(t) = x_t - lse;  H = -sum p ln p = ln Z - sum e^(x - M) (x - M) / Z   (two terms that are not negative: nothing cancels)
//
// A workgroup reads a segment of a row once and keeps it in registers as it comes: every thread takes its own maximum, then sums, and the threads are joined by their maxima.  The
// most probable tokens from the same registers: the threads' maxima, joined to 64 of them, are 64 different tokens, so that the k-th largest of these is a bound that k tokens reach and few others
// do (k = 20: 24 are expected); the threads that have them hand them over in LDS and each is compared with all.  What keys are compared by: the value, then the lower index first; all different, so the result is
// the same whatever order they come in.  Where the bound lets too many through (rows with many equal values, masked rows), k rounds of a plain arg-max.
// Segments of a row are joined by a second kernel.  Bound by the read of the logits, and nearly as much by the exponentials: some nine instruction slots a number, so nothing else is done to
// each; where sums come out as no numbers (masked logits, NaN), they are made again with care.
#include "pv_matrix_common.h"

#define LP_MAX_TOP 32
#define LP_ROOM 512                         // tokens above the bound that LDS has room for
#define LP_MAX_SEGS 64
#define LP_FEW 64                           // threads with such tokens that LDS has room for

struct lp_args {
    const char *logits; int64_t row_bytes;
    int64_t rows; int vocab, segs;
    const int32_t *tokens; int n_tokens, top;
    float *logprobs, *entropy, *lse;
    int32_t *top_ids; float *top_logprobs;
    float *part;                            // [row][seg][4]: maximum, sum, sum of e y
    uint64_t *keys;                         // [row][seg][top], best first
};

// Order of numbers as unsigned integers (-0 and 0 are one number); a token's key: the larger is the better one.  NaN counts as -infinity.
__device__ inline uint32_t lp_order(float x) { const uint32_t u = __float_as_uint(x); return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u); }
__device__ inline float lp_value(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ inline uint64_t lp_key(float x, int i) { return (uint64_t)lp_order(x) << 32 | (uint32_t)~i; }
__device__ inline int lp_index(uint64_t k) { return (int)~(uint32_t)k; }
__device__ inline float lp_clean(float x) { return x == x ? x + 0.f : -INFINITY; }

template <typename T> __device__ inline float lp_one(const char *p, int64_t i);
template <> __device__ inline float lp_one<float>(const char *p, int64_t i) { return ((const float *)p)[i]; }
template <> __device__ inline float lp_one<__bf16>(const char *p, int64_t i) { return pv_bf16_to_f32(((const uint16_t *)p)[i]); }
template <> __device__ inline float lp_one<_Float16>(const char *p, int64_t i) { return (float)((const _Float16 *)p)[i]; }

// Numbers as they lie in memory, dwords w of them: number i
typedef __attribute__((ext_vector_type(2))) _Float16 lp_h2;
template <typename T> __device__ inline float lp_get(const uint32_t *w, int i);
template <> __device__ inline float lp_get<float>(const uint32_t *w, int i) { return __uint_as_float(w[i]); }
template <> __device__ inline float lp_get<__bf16>(const uint32_t *w, int i) { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
template <> __device__ inline float lp_get<_Float16>(const uint32_t *w, int i) { const lp_h2 h = __builtin_bit_cast(lp_h2, w[i >> 1]); return (float)(i & 1 ? h.y : h.x); }

// Maximum, sum of 2^y, sum of 2^y y, y = (x - maximum) log2(e), of two sets
struct lp_sums { float m, s, w; };
__device__ inline void lp_under(lp_sums &a, float M)         // a set's sums under a maximum that is not less
{
    const float d = fmaxf((a.m - M) * 1.44269504088896340736f, -256.f);      // (2^-256 is 0; the product may be -infinity)
    const bool none = a.m == -INFINITY;                       // (nothing but -infinity in it)
    const float f = none ? 0.f : __builtin_amdgcn_exp2f(d);
    a.w = none ? 0.f : f * fmaf(a.s, d, a.w);
    a.s = none ? 0.f : f * a.s;
    a.m = M;
}
__device__ inline void lp_over_wave(lp_sums &a)
{
    lp_under(a, over_wave(a.m, op_max));
    a.s = over_wave(a.s, op_add); a.w = over_wave(a.w, op_add);
}

// A token's logit (no token: NaN)
template <typename T> __device__ inline float lp_logit(const lp_args &a, int64_t row, int i)
{
    const int tok = a.tokens[row * a.n_tokens + i];
    return tok >= 0 && tok < a.vocab ? lp_clean(lp_one<T>(a.logits + row * a.row_bytes, tok)) : __uint_as_float(0x7fc00000u);
}

// What a row's sums say: written by all threads of the workgroup.  x0: the logit of token tid, asked for early.
template <typename T>
__device__ inline void lp_finish(const lp_args &a, int64_t row, const lp_sums &t, int tid, int nt, const uint64_t *best, float x0)
{
    const float lz = __log2f(t.s) * 0.69314718055994530942f, lse = t.s == 0.f ? -INFINITY : t.m + lz;
    // under -infinity alone no token has a probability
    auto logp = [&](float x) { return t.s == 0.f ? -INFINITY : (x - t.m) - lz; };
    if (tid == 0) {
        if (a.lse != nullptr) a.lse[row] = lse;
        if (a.entropy != nullptr) a.entropy[row] = t.s == 0.f ? 0.f : lz - 0.69314718055994530942f * t.w / t.s;
    }
    for (int i = tid; i < a.n_tokens; i += nt) {
        const float x = i == tid ? x0 : lp_logit<T>(a, row, i);
        a.logprobs[row * a.n_tokens + i] = x == x ? logp(x) : x;
    }
    for (int i = tid; i < a.top; i += nt) {
        const uint64_t k = best[i];
        a.top_ids[row * a.top + i] = lp_index(k);
        a.top_logprobs[row * a.top + i] = logp(lp_value((uint32_t)(k >> 32)));
    }
}

// The best key of the wave, in every lane
__device__ inline uint64_t lp_wave_best(uint64_t k)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)k, d, 64); k = o > k ? o : k; }
    return k;
}

// The best `top` of n <= 64 keys in LDS, in order: the waves take keys in turn, their lanes compare them with all
__device__ inline void lp_rank(const uint64_t *keys, int n, int top, uint64_t *best, int wave, int waves)
{
    const int lane = threadIdx.x & 63;
    const uint64_t other = lane < n ? keys[lane] : 0;
    for (int i = wave; i < n; i += waves) {
        const uint64_t k = keys[i];
        const int better = __popcll(__ballot(other > k));
        if (better < top && lane == 0) best[better] = k;
    }
}

// NT threads, E numbers of a row each, from the row's first address that is a multiple of 16 bytes on; the few numbers ahead of that and behind the last 16 bytes
// go to single threads of the first and the last segment.
template <typename T, int NT, int E>
__global__ void __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(E == 64 ? 6 : sizeof(T) == 4 ? 4 : 8)))
k_logprobs(const lp_args a)
{
    constexpr int V = 16 / (int)sizeof(T), U = E / V, NW = NT / 64, D = E * (int)sizeof(T) / 4;
    __shared__ lp_sums sh_s[NW];
    __shared__ uint32_t sh_max[NT], sh_bound;
    __shared__ uint64_t sh_key[LP_ROOM], sh_best[LP_MAX_TOP];
    __shared__ int sh_n, sh_few, sh_who[LP_FEW];
    __shared__ __align__(16) uint32_t sh_x[LP_FEW][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t x[D];
    // a segment's numbers on their way into the registers
    auto place = [&](int64_t item, int64_t &row, int &seg, const char *&src, int &head) {
        row = item / a.segs; seg = (int)(item - row * a.segs);
        src = a.logits + row * a.row_bytes;
        head = min((int)(((16u - ((uint32_t)(uintptr_t)src & 15u)) & 15u) / (uint32_t)sizeof(T)), a.vocab);
    };
    auto load = [&](int64_t item) {
        int64_t row; int seg, head; const char *src;
        place(item, row, seg, src, head);
        const int base = head + seg * (NT * E);
        constexpr uint32_t inf = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u;      // -infinity
        const u32x4 none = {inf, inf, inf, inf};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i0 = base + (u * NT + tid) * V;
            u32x4 v = none;
            if (i0 + V <= a.vocab) v = __builtin_nontemporal_load((const u32x4 *)(src + (int64_t)i0 * sizeof(T)));
            x[4 * u] = v.x; x[4 * u + 1] = v.y; x[4 * u + 2] = v.z; x[4 * u + 3] = v.w;
        }
    };
    const int64_t item = blockIdx.x;
    load(item);
    int64_t row; int seg, head; const char *src;
    place(item, row, seg, src, head);
    const int base = head + seg * (NT * E);
    auto index = [&](int i) { return base + ((i / V) * NT + tid) * V + i % V; };
    float asked = 0.f;
    if (a.segs == 1 && tid < a.n_tokens) asked = lp_logit<T>(a, row, tid);
    // those that no 16 bytes hold: ahead of the row's first, behind its last
    const int behind = (a.vocab - head) % V, alone = tid < 8 ? (seg == 0 && tid < head ? tid : -1) : tid < 8 + behind && seg == (a.vocab - behind - head) / (NT * E) ? a.vocab - behind + tid - 8 : -1;
    const bool first = alone >= 0;
    const float x0 = first ? lp_clean(lp_one<T>(src, alone)) : -INFINITY;
    lp_sums t = {x0, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) t.m = fmaxf(t.m, lp_get<T>(x, i));          // (of a number and NaN the number)
#pragma unroll
    for (int d = 0; d < D; ++d) if (sizeof(T) == 2) asm volatile("" : "+v"(x[d]));     // (taken apart anew each time: 32 bits of each number would be twice the registers)
    const float ref = t.m == -INFINITY ? 0.f : t.m, c = -ref * 1.44269504088896340736f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const float y = fmaf(lp_get<T>(x, i), 1.44269504088896340736f, c), e = __builtin_amdgcn_exp2f(y);
        t.s += e;
        t.w = fmaf(e, y, t.w);
    }
    {   // What rounding left of c is in every y of the thread, and comes out of its sums
        const float off = fmaf(ref, 1.44269504088896340736f, c), f = fabsf(off) < 0.5f ? __builtin_amdgcn_exp2f(-off) : INFINITY;
        t.w = f * fmaf(-off, t.s, t.w); t.s *= f;
    }
    if (__any(!(t.s < INFINITY && t.w == t.w))) {             // -infinity (its exponential, 0, times it is no number), NaN, +infinity, products over the largest number, a maximum from some 2^23 on
        t.s = t.m == INFINITY ? __uint_as_float(0x7fc00000u) : 0.f; t.w = t.s;
#pragma unroll
        for (int d = 0; d < D; ++d) if (sizeof(T) == 2) asm volatile("" : "+v"(x[d]));     // (as above: the loop before would keep all numbers for this one)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float y = fmaxf((lp_clean(lp_get<T>(x, i)) - ref) * 1.44269504088896340736f, -256.f), e = __builtin_amdgcn_exp2f(y);      // (2^-256 is 0)
            t.s += e;
            t.w = fmaf(e, y, t.w);
            asm volatile("" : "+v"(t.s), "+v"(t.w));          // (one after the other: no registers for more)
        }
    }
    {
        const float y = fmaxf((x0 - ref) * 1.44269504088896340736f, -256.f), e = __builtin_amdgcn_exp2f(y);
        t.s += e; t.w = fmaf(e, y, t.w);
    }
    const float mine = t.m;
    lp_over_wave(t);
    if (lane == 0) sh_s[wave] = t;
    if (a.top > 0) {
        sh_max[tid] = first || index(V - 1) < a.vocab ? lp_order(mine + 0.f) : 0u;      // (a thread behind the row's end has no token)
        if (tid == 0) { sh_n = 0; sh_few = 0; }
        if (tid < LP_MAX_TOP) sh_best[tid] = 0;
    }
    __syncthreads();
    if (a.top > 0) {
        if (wave == 0) {
            uint32_t g = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) { const uint32_t o = sh_max[w * 64 + lane]; g = o > g ? o : g; }
            uint32_t bound = 0;                               // a number that `top` of the 64 maxima reach: the largest to 20 bits, or one that no more reach
            for (int b = 31; b >= 12; --b) {
                const uint32_t n = bound | 1u << b;
                const int reach = __popcll(__ballot(g >= n));
                if (reach >= a.top) bound = n;
                if (reach == a.top) break;
            }
            if (lane == 0) sh_bound = bound;
        }
        __syncthreads();
        const uint32_t bound = sh_bound;
        auto keep = [&](uint64_t k) { const int at = atomicAdd(&sh_n, 1); if (at < LP_ROOM) sh_key[at] = k; };
        const int begin = seg == 0 ? 0 : base, end = min(base + NT * E, a.vocab);
        if (bound <= 0x007fffffu) {                           // every token: to be kept, or too many
            if (end - begin > LP_ROOM) sh_n = LP_ROOM + 1;
            else for (int i = begin + tid; i < end; i += NT) keep(lp_key(lp_clean(lp_one<T>(src, i)), i));
        } else if (lp_order(mine + 0.f) >= bound) {           // few threads have any: those hand their numbers to the first wave
            if (first && lp_order(x0) >= bound) keep(lp_key(x0, alone));
            const int at = atomicAdd(&sh_few, 1);
            if (at < LP_FEW) {
                sh_who[at] = tid;
#pragma unroll
                for (int d = 0; d < D; d += 4) *(uint4 *)&sh_x[at][d] = make_uint4(x[d], x[d + 1], x[d + 2], x[d + 3]);
            } else sh_n = LP_ROOM + 1;
        }
        __syncthreads();
        const int few = sh_few <= LP_FEW ? sh_few : 0;        // (else too many)
        const float least = lp_value(bound);                  // (neither NaN reaches it nor what fills up a row)
        for (int i = tid; i < few * E; i += NT) {
            const int who = i / E, e = i - who * E, at = base + ((e / V) * NT + sh_who[who]) * V + e % V;
            const float v = lp_get<T>(sh_x[who], e);
            if (v >= least) keep(lp_key(v + 0.f, at));
        }
        __syncthreads();
        const int n = sh_n;
        if (n <= 64) lp_rank(sh_key, n, a.top, sh_best, wave, NW);
        else if (n <= LP_ROOM) {
            for (int i = tid; i < n; i += NT) {
                const uint64_t k = sh_key[i];
                int better = 0;
#pragma unroll 4
                for (int j = 0; j < n; ++j) better += sh_key[j] > k;
                if (better < a.top) sh_best[better] = k;
            }
        } else {
            uint64_t last = ~0ull;
            for (int r = 0; r < a.top; ++r) {
                uint64_t k = 0;
                // (read again: in a loop over registers the keys would have to be kept as well)
                for (int i = begin + tid; i < end; i += NT) { const uint64_t o = lp_key(lp_clean(lp_one<T>(src, i)), i); if (o < last && o > k) k = o; }
                k = lp_wave_best(k);
                if (lane == 0) sh_key[wave] = k;
                __syncthreads();
                for (int w = 0; w < NW; ++w) k = sh_key[w] > k ? sh_key[w] : k;
                if (tid == 0) sh_best[r] = k;
                last = k;
                __syncthreads();
            }
        }
        __syncthreads();
    }
    t = sh_s[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) t.m = fmaxf(t.m, sh_s[w].m);
    {
        const float M = t.m;
        t = {M, 0.f, 0.f};
        for (int w = 0; w < NW; ++w) { lp_sums o = sh_s[w]; lp_under(o, M); t.s += o.s; t.w += o.w; }
    }
    if (a.segs == 1) lp_finish<T>(a, row, t, tid, NT, sh_best, asked);
    else {
        if (tid == 0) *(float4 *)(a.part + (row * a.segs + seg) * 4) = make_float4(t.m, t.s, t.w, 0.f);
        for (int i = tid; i < a.top; i += NT) a.keys[(row * a.segs + seg) * a.top + i] = sh_best[i];
    }
}

// The segments of a row joined: a workgroup a row, a lane a segment for its sums and the bound that its best tokens give
template <typename T>
__global__ void __launch_bounds__(256)
k_logprobs_join(const lp_args a)
{
    constexpr int MOST = LP_MAX_SEGS * LP_MAX_TOP, FL = MOST / 256;
    __shared__ uint64_t sh_few[MOST], sh_best[LP_MAX_TOP];
    __shared__ int sh_n;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, total = a.segs * a.top;
    const int64_t row = blockIdx.x;
    const uint64_t *keys = a.keys + row * total;
    lp_sums t = {-INFINITY, 0.f, 0.f};
    uint64_t k[FL], g = 0;
    // the d-th best of each segment: as many of them as reach a bound bring d tokens each
    const int d = a.top > 0 ? (a.top + a.segs - 1) / a.segs : 1, want = (a.top + d - 1) / d;
    if (lane < a.segs) { const float4 p = *(const float4 *)(a.part + (row * a.segs + lane) * 4); t = {p.x, p.y, p.z}; }
    if (a.top > 0 && lane < a.segs) g = keys[lane * a.top + d - 1];
#pragma unroll
    for (int i = 0; i < FL; ++i) { k[i] = 0; if (i * 256 < total && i * 256 + tid < total) k[i] = keys[i * 256 + tid]; }
    const float asked = tid < a.n_tokens ? lp_logit<T>(a, row, tid) : 0.f;
    if (tid == 0) sh_n = 0;
    if (tid < LP_MAX_TOP) sh_best[tid] = 0;
    __syncthreads();
    if (a.top > 0) {
        uint32_t bound = 0;
        for (int b = 31; b >= 0; --b) {
            const uint32_t n = bound | 1u << b;
            const int reach = __popcll(__ballot((uint32_t)(g >> 32) >= n));
            if (reach >= want) bound = n;
            if (reach == want) break;
        }
#pragma unroll
        for (int i = 0; i < FL; ++i) if (k[i] != 0 && (uint32_t)(k[i] >> 32) >= bound) sh_few[atomicAdd(&sh_n, 1)] = k[i];
        __syncthreads();
        const int n = sh_n;
        if (n <= 64) lp_rank(sh_few, n, a.top, sh_best, wave, 4);
        else for (int i = tid; i < n; i += 256) {
            const uint64_t mine = sh_few[i];
            int better = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) better += sh_few[j] > mine;
            if (better < a.top) sh_best[better] = mine;
        }
    }
    lp_over_wave(t);
    __syncthreads();
    lp_finish<T>(a, row, t, tid, 256, sh_best, asked);
}

// ------------------------------- host side ----------------------------------------

// Segments of 4096 numbers, or of 32768: the larger where that is a row, which saves the launch that joins (8 f32 rows of 16384, five alternatives, called one by one 17.7 and 13.9 us, from a graph 8.3 and 8.9; of
// 32000 17.7 and 13.6, 8.5 and 9.1; 200 rows of 32000 17.9 and 13.8, 12.5 and 10.6), where there are rows enough for the chip, or where more than 64 segments would come out
struct lp_plan { bool large; int segs; };
static lp_plan plan(int64_t rows, int vocab)
{
    lp_plan p;
    p.large = vocab > 4096 && (vocab <= 32768 || rows >= 256 || vocab > 4096 * LP_MAX_SEGS);
    const int n = p.large ? 32768 : 4096;
    p.segs = (vocab + n - 1) / n;
    return p;
}

static int check(int64_t rows, int vocab, int top)
{
    if (rows < 0 || rows > (1 << 24)) { pv_set_error("rows %lld outside [0, 2^24)", (long long)rows); return PV_ERANGE; }
    if (vocab < 1 || vocab > 32768 * LP_MAX_SEGS) { pv_set_error("vocab %d outside [1, %d]", vocab, 32768 * LP_MAX_SEGS); return PV_ERANGE; }
    if (top < 0 || top > LP_MAX_TOP || top > vocab) { pv_set_error("top %d outside [0, min(%d, vocab)]", top, LP_MAX_TOP); return PV_ERANGE; }
    // a launch has less than 2^32 threads
    const lp_plan p = plan(rows, vocab);
    if (rows * p.segs >= (1 << 22) * (p.large ? 1ll : 4ll)) { pv_set_error("%lld rows of %d: more than a launch takes", (long long)rows, vocab); return PV_ERANGE; }
    return PV_OK;
}

extern "C" int pv_token_logprobs_bytes(int64_t rows, int32_t vocab, int32_t top, size_t *bytes)
{
    const int rc = check(rows, vocab, top);
    if (rc != PV_OK) return rc;
    if (!bytes) { pv_set_error("null output pointer"); return PV_EINVAL; }
    const lp_plan p = plan(rows, vocab);
    *bytes = p.segs > 1 ? (size_t)rows * p.segs * (16 + 8 * (size_t)top) : 0;
    return PV_OK;
}

template <typename T>
static int launch(const lp_args &a, const lp_plan &p, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.rows * a.segs);
    // 512 threads: three workgroups or more a CU, of which some load while others compute (4096 bf16 rows of 32000, 20 alternatives: 256 threads 66 us, 512 57, 1024 75, to be read in 40; 2048 f32 rows
    // 50, 45, 50)
    if (p.large) k_logprobs<T, 512, 64><<<grid, 512, 0, s>>>(a);
    else k_logprobs<T, 256, 16><<<grid, 256, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    if (a.segs > 1) { k_logprobs_join<T><<<(unsigned)a.rows, 256, 0, s>>>(a); PV_HIP(hipGetLastError()); }
    return PV_OK;
}

extern "C" int pv_token_logprobs(const void *logits, int64_t row_stride, int32_t dtype, int64_t rows, int32_t vocab, const int32_t *tokens, int32_t n_tokens, float *logprobs,
                                 float *entropy, float *lse, int32_t top, int32_t *top_ids, float *top_logprobs, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check(rows, vocab, top);
    if (rc != PV_OK) return rc;
    if (dtype != PV_F32 && dtype != PV_BF16 && dtype != PV_F16) { pv_set_error("bad dtype %d", dtype); return PV_EINVAL; }
    if (n_tokens < 0 || n_tokens > 65536) { pv_set_error("n_tokens %d outside [0, 65536]", n_tokens); return PV_ERANGE; }
    if (rows == 0) return PV_OK;
    if (!logits || (n_tokens && (!tokens || !logprobs)) || (top && (!top_ids || !top_logprobs))) { pv_set_error("null pointer"); return PV_EINVAL; }
    if (row_stride < 0) { pv_set_error("negative row stride"); return PV_EINVAL; }
    const int64_t size = dtype == PV_F32 ? 4 : 2;
    if ((uintptr_t)logits % size) { pv_set_error("logits are not aligned to their type"); return PV_EINVAL; }
    const lp_plan p = plan(rows, vocab);
    size_t need = 0;
    pv_token_logprobs_bytes(rows, vocab, top, &need);
    if (need > workspace_bytes || (need && !workspace)) { pv_set_error("workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need); return PV_ENOMEM; }
    if ((uintptr_t)workspace & 15) { pv_set_error("workspace must be 16-byte aligned"); return PV_EINVAL; }
    lp_args a = {};
    a.logits = (const char *)logits; a.row_bytes = row_stride * size; a.rows = rows; a.vocab = vocab; a.segs = p.segs;
    a.tokens = tokens; a.n_tokens = n_tokens; a.top = top; a.logprobs = logprobs; a.entropy = entropy; a.lse = lse; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.part = (float *)workspace; a.keys = (uint64_t *)((char *)workspace + (size_t)rows * p.segs * 16);
    hipStream_t s = (hipStream_t)hip_stream;
    return dtype == PV_F32 ? launch<float>(a, p, s) : dtype == PV_BF16 ? launch<__bf16>(a, p, s) : launch<_Float16>(a, p, s);
}
