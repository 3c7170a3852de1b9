// Log probabilities of given tokens under rows of logits, with each row's entropy and most probable tokens.
//
//   lse = M + ln Z, Z = sum e^(x - M), M = max x;  log p(t) = x_t - lse;  H = -sum p ln p = ln Z - sum e^(x - M) (x - M) / Z   (two terms that are not negative: nothing cancels)
//
// A workgroup reads a segment of a row once and keeps it in registers as it comes: every thread takes its own maximum, then sums, and the threads are joined by their maxima.  The
// most probable tokens from the same registers: the threads' maxima, joined to 64 of them, are 64 different tokens, so that the k-th largest of these is a bound that k tokens reach and few others
// do (k = 20: 24 are expected); those are written to LDS and each counts the better ones.  What keys are compared by: the value, then the lower index first; all different, so the result is
// the same whatever order they come in.  Where the bound lets too many through (rows with many equal values, masked rows), k rounds of a plain arg-max.
// Segments of a row are joined by a second kernel.  Bound by the read of the logits, and nearly as much by the exponentials: some nine instruction slots a number, so nothing else is done to
// each; where sums come out as no numbers (masked logits, NaN), they are made again with care.
#include "pv_matrix_common.h"

#define LP_MAX_TOP 32
#define LP_ROOM 512                         // tokens above the bound that LDS has room for
#define LP_MAX_SEGS 64

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

// What a row's sums say: written by all threads of the workgroup
template <typename T>
__device__ inline void lp_finish(const lp_args &a, int64_t row, const lp_sums &t, int tid, int nt, const uint64_t *best)
{
    const float lz = __log2f(t.s) * 0.69314718055994530942f, lse = t.s == 0.f ? -INFINITY : t.m + lz;
    // under -infinity alone no token has a probability
    auto logp = [&](float x) { return t.s == 0.f ? -INFINITY : (x - t.m) - lz; };
    if (tid == 0) {
        if (a.lse != nullptr) a.lse[row] = lse;
        if (a.entropy != nullptr) a.entropy[row] = t.s == 0.f ? 0.f : lz - 0.69314718055994530942f * t.w / t.s;
    }
    for (int i = tid; i < a.n_tokens; i += nt) {
        const int tok = a.tokens[row * a.n_tokens + i];
        a.logprobs[row * a.n_tokens + i] = tok >= 0 && tok < a.vocab ? logp(lp_clean(lp_one<T>(a.logits + row * a.row_bytes, tok))) : __uint_as_float(0x7fc00000u);
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

// The best `top` of n <= 64 keys in LDS, in order: a lane a key, counting the better ones
__device__ inline void lp_rank(const uint64_t *keys, int n, int top, uint64_t *best)
{
    const int lane = threadIdx.x & 63;
    const uint64_t k = lane < n ? keys[lane] : 0;
    const uint32_t lo = (uint32_t)k, hi = (uint32_t)(k >> 32);
    int better = 0;
    for (int j = 0; j < n; ++j) {
        const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, j);
        better += o > k;
    }
    if (lane < n && better < top) best[better] = k;
}

// NT threads, E numbers of a row each, from the row's first address that is a multiple of 16 bytes on; the few numbers ahead of that belong to the first segment's first threads.
template <typename T, int NT, int E>
__global__ void __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(8, 8)))
k_logprobs(const lp_args a)
{
    constexpr int V = 16 / (int)sizeof(T), U = E / V, NW = NT / 64, D = E * (int)sizeof(T) / 4;
    __shared__ lp_sums sh_s[NW];
    __shared__ uint32_t sh_max[NT], sh_bound;
    __shared__ uint64_t sh_key[LP_ROOM], sh_best[LP_MAX_TOP];
    __shared__ int sh_n;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.segs;
    const int seg = (int)(blockIdx.x - row * a.segs);
    const char *src = a.logits + row * a.row_bytes;
    const int head = min((int)(((16u - ((uint32_t)(uintptr_t)src & 15u)) & 15u) / (uint32_t)sizeof(T)), a.vocab), base = head + seg * (NT * E);
    uint32_t x[D];
    auto index = [&](int i) { return base + ((i / V) * NT + tid) * V + i % V; };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i0 = base + (u * NT + tid) * V;
        if (i0 + V <= a.vocab) {
            const u32x4 v = __builtin_nontemporal_load((const u32x4 *)(src + (int64_t)i0 * sizeof(T)));
            x[4 * u] = v.x; x[4 * u + 1] = v.y; x[4 * u + 2] = v.z; x[4 * u + 3] = v.w;
        } else {
            const uint32_t none = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u;      // -infinity
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                x[4 * u + d] = none;
                if constexpr (sizeof(T) == 4) { if (i0 + d < a.vocab) x[4 * u + d] = ((const uint32_t *)src)[i0 + d]; }
                else {
                    if (i0 + 2 * d < a.vocab) x[4 * u + d] = (none & 0xffff0000u) | ((const uint16_t *)src)[i0 + 2 * d];
                    if (i0 + 2 * d + 1 < a.vocab) x[4 * u + d] = (x[4 * u + d] & 0xffffu) | (uint32_t)((const uint16_t *)src)[i0 + 2 * d + 1] << 16;
                }
            }
        }
    }
    const bool first = seg == 0 && tid < head;
    const float x0 = first ? lp_clean(lp_one<T>(src, tid)) : -INFINITY;
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
    if (__any(!(t.s < INFINITY && t.w == t.w))) {             // -infinity (its exponential, 0, times it is no number), NaN, +infinity, products over the largest number
        t.s = t.m == INFINITY ? __uint_as_float(0x7fc00000u) : 0.f; t.w = t.s;
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
        sh_max[tid] = first || index(0) < a.vocab ? lp_order(mine + 0.f) : 0u;      // (a thread behind the row's end has no token)
        if (tid == 0) sh_n = 0;
        if (tid < LP_MAX_TOP) sh_best[tid] = 0;
    }
    __syncthreads();
    if (a.top > 0) {
        if (wave == 0) {
            uint32_t g = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) { const uint32_t o = sh_max[w * 64 + lane]; g = o > g ? o : g; }
            uint32_t bound = 0;                               // the largest number, to 20 bits, that `top` of the 64 maxima reach
#pragma unroll 4
            for (int b = 31; b >= 12; --b) { const uint32_t n = bound | 1u << b; if (__popcll(__ballot(g >= n)) >= a.top) bound = n; }
            if (lane == 0) sh_bound = bound;
        }
        __syncthreads();
        const uint32_t bound = sh_bound;
        auto keep = [&](uint64_t k) { const int at = atomicAdd(&sh_n, 1); if (at < LP_ROOM) sh_key[at] = k; };
        if (lp_order(mine + 0.f) >= bound) {
            if (first && lp_order(x0) >= bound) keep(lp_key(x0, tid));
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float v = lp_clean(lp_get<T>(x, i));
                if (lp_order(v) >= bound && index(i) < a.vocab) keep(lp_key(v, index(i)));
            }
        }
        __syncthreads();
        const int n = sh_n;
        if (n <= 64) { if (wave == 0) lp_rank(sh_key, n, a.top, sh_best); }
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
                for (int i = (seg == 0 ? 0 : base) + tid; i < min(base + NT * E, a.vocab); i += NT) { const uint64_t o = lp_key(lp_clean(lp_one<T>(src, i)), i); if (o < last && o > k) k = o; }
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
    if (a.segs == 1) { lp_finish<T>(a, row, t, tid, NT, sh_best); return; }
    if (tid == 0) *(float4 *)(a.part + (row * a.segs + seg) * 4) = make_float4(t.m, t.s, t.w, 0.f);
    for (int i = tid; i < a.top; i += NT) a.keys[(row * a.segs + seg) * a.top + i] = sh_best[i];
}

// The segments of a row joined: a wave a row, a lane a segment (its best tokens come in order)
template <typename T>
__global__ void __launch_bounds__(64)
k_logprobs_join(const lp_args a)
{
    __shared__ uint64_t sh_key[LP_MAX_SEGS * LP_MAX_TOP], sh_best[LP_MAX_TOP];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    lp_sums t = {-INFINITY, 0.f, 0.f};
    if (lane < a.segs) { const float4 p = *(const float4 *)(a.part + (row * a.segs + lane) * 4); t = {p.x, p.y, p.z}; }
    for (int i = lane; i < a.segs * a.top; i += 64) sh_key[i] = a.keys[row * a.segs * a.top + i];
    lp_over_wave(t);
    __syncthreads();
    int at = 0;
    for (int r = 0; r < a.top; ++r) {
        const uint64_t head = lane < a.segs && at < a.top ? sh_key[lane * a.top + at] : 0, best = lp_wave_best(head);
        if (head == best && best != 0) ++at;                  // (keys are all different)
        if (lane == 0) sh_best[r] = best;
    }
    __syncthreads();
    lp_finish<T>(a, row, t, lane, 64, sh_best);
}

// ------------------------------- host side ----------------------------------------

// Segments of 4096 numbers, or of 32768: the larger where there are rows enough for the chip and numbers enough in a row, or where more than 64 segments would come out
struct lp_plan { bool large; int segs; };
static lp_plan plan(int64_t rows, int vocab)
{
    lp_plan p;
    p.large = (rows >= 256 && vocab > 4096) || vocab > 4096 * LP_MAX_SEGS;
    const int n = p.large ? 32768 : 4096;
    p.segs = (vocab + n - 1) / n;
    return p;
}

static int check(int64_t rows, int vocab, int top)
{
    if (rows < 0 || rows > (1 << 24)) { pv_set_error("rows %lld outside [0, 2^24]", (long long)rows); return PV_ERANGE; }
    if (vocab < 1 || vocab > 32768 * LP_MAX_SEGS) { pv_set_error("vocab %d outside [1, %d]", vocab, 32768 * LP_MAX_SEGS); return PV_ERANGE; }
    if (top < 0 || top > LP_MAX_TOP || top > vocab) { pv_set_error("top %d outside [0, min(%d, vocab)]", top, LP_MAX_TOP); return PV_ERANGE; }
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
    if (p.large) k_logprobs<T, 1024, 32><<<grid, 1024, 0, s>>>(a);
    else k_logprobs<T, 256, 16><<<grid, 256, 0, s>>>(a);
    PV_HIP(hipGetLastError());
    if (a.segs > 1) { k_logprobs_join<T><<<(unsigned)a.rows, 64, 0, s>>>(a); PV_HIP(hipGetLastError()); }
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
    if (rows * p.segs >= (1 << 22) * (p.large ? 1ll : 4ll)) { pv_set_error("%lld rows of %d: more than a launch takes", (long long)rows, vocab); return PV_ERANGE; }
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
