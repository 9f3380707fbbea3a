// q8_sample.hip -- one token drawn per row of logits, from given random numbers, under temperature, top-k, top-p and min-p.
//
// With m the largest logit of a row, word i has the weight w_i = exp(-(m - l_i) / T).  The words are ordered by (logit
// descending, index ascending); each filter keeps a prefix of that order: the first k words; the shortest prefix with at
// least p of the mass of those; the words with w_i >= min_p.  With Z the mass of the shortest of these prefixes the drawn
// token is the first word of the order whose cumulative mass exceeds u Z.
//
// Weights are whole numbers, rint(w_i 2^S): their sums are exact whatever their order, so a token does not depend on which
// thread adds what, and the borders between tokens lie where sums in 64-bit floating point put them to about 1e-12.
#include "q8_internal.h"

#include <math.h>

struct SampleArgs {
    const float *logits;
    size_t ldl;
    int V;
    const float *u, *T, *top_p, *min_p;     // [n]; all but u may be NULL
    const int *top_k;
    int *tokens;
    float *logp;                            // may be NULL
    const float *E_tgt;                     // may be NULL
    float *y_emb;
    int E;
    int shift;                              // S
};

typedef unsigned long long u64;

__device__ __forceinline__ bool smp_dead(float v) { return !(v > -INFINITY); }       // -inf or NaN: cannot be drawn

// The distance below the largest logit, in double: two floats' difference can exceed the range of a float.
__device__ __forceinline__ double smp_gap(float m, float v) { return v == m ? 0.0 : (double)m - (double)v; }

// exp(-x), x >= 0; 0 past every weight that counts (and for the NaN of inf * 0, a word infinitely far below at T = inf)
__device__ __forceinline__ double smp_exp(double x) { return x <= 700.0 ? q8_exp_d(-x) : 0.0; }

struct SampleHit { u64 key, mass; };

// The first word of the order at which the cumulative (count, mass) satisfies `cond` (monotone along the order), by its key's
// bytes from the top: a histogram of one byte of the words that agree with what is known so far.
template <class Weight, class Cond>
__device__ SampleHit smp_select(const float *l, int V, Weight weight, Cond cond)
{
    __shared__ unsigned s_cnt[256];
    __shared__ u64 s_mass[256];
    __shared__ u64 s_key, s_m;
    __shared__ unsigned s_c;
    const int tid = threadIdx.x;
    if (tid == 0) { s_key = 0; s_m = 0; s_c = 0; }
    for (int level = 7; level >= 0; --level) {
        if (tid < 256) { s_cnt[tid] = 0; s_mass[tid] = 0; }
        __syncthreads();
        const u64 known = s_key;
        for (int i = tid; i < V; i += blockDim.x) {
            const float v = l[i];
            if (smp_dead(v)) continue;
            const u64 key = topk_key(v, i);
            if (level < 7 && (key >> (8 * (level + 1))) != (known >> (8 * (level + 1)))) continue;
            const int d = (int)(key >> (8 * level)) & 255;
            atomicAdd(&s_cnt[d], 1u);
            atomicAdd(&s_mass[d], weight(v));
        }
        __syncthreads();
        if (tid == 0) {
            int last = 0;
            u64 m = s_m, mlast = m;
            unsigned c = s_c, clast = c;
            bool found = false;
            for (int d = 255; d >= 0 && !found; --d)
                if (s_cnt[d]) {
                    last = d; mlast = m; clast = c;
                    m += s_mass[d]; c += s_cnt[d];
                    found = cond(c, m);
                }
            s_key = known | ((u64)last << (8 * level));
            s_m = level ? mlast : m;
            s_c = level ? clast : c;
        }
        __syncthreads();
    }
    const SampleHit r = {s_key, s_m};
    __syncthreads();
    return r;
}

__device__ __forceinline__ u64 smp_block_max(u64 v, u64 *s)
{
    v = wave_max_u64(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 r = s[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) r = s[w] > r ? s[w] : r;
    __syncthreads();
    return r;
}

// One block per row.
__global__ __launch_bounds__(1024) void sample_kernel(SampleArgs a)
{
    __shared__ u64 s_u[16], s_sum[2];
    __shared__ double s_d[16];
    const int j = blockIdx.x, tid = threadIdx.x, V = a.V;
    const float *l = a.logits + (size_t)j * a.ldl;
    u64 best = 0;
    for (int i = tid; i < V; i += 1024) {
        const float v = l[i];
        if (!smp_dead(v)) { const u64 k = topk_key(v, i); best = k > best ? k : best; }
    }
    best = smp_block_max(best, s_u);
    int token = best ? topk_key_idx(best) : -1;
    float logp = -INFINITY;
    if (best) {
        const float m = topk_key_val(best);
        const float T = a.T ? a.T[j] : 1.0f;
        const float tp = a.top_p ? a.top_p[j] : 1.0f, mp = a.min_p ? a.min_p[j] : 0.0f;
        const int k = a.top_k ? a.top_k[j] : 0;
        const bool drawn = T > 0.0f;
        const double inv = drawn ? 1.0 / (double)T : 0.0;
        const double one = (double)(1ull << a.shift);
        auto relative = [&](float v) { const double g = smp_gap(m, v); return g == 0.0 ? 1.0 : smp_exp(g * inv); };
        auto weight = [&](float v) { return (u64)rint(relative(v) * one); };
        if (tid < 2) s_sum[tid] = 0;
        __syncthreads();
        double e = 0.0;
        u64 all = 0, above = 0;
        for (int i = tid; i < V; i += 1024) {
            const float v = l[i];
            if (smp_dead(v)) continue;
            e += smp_exp(smp_gap(m, v));
            if (drawn) {
                const double r = relative(v);
                const u64 w = (u64)rint(r * one);
                all += w;
                if (r >= (double)mp) above += w;
            }
        }
        atomicAdd(&s_sum[0], all);
        atomicAdd(&s_sum[1], above);
        e = wave_sum_d(e);
        if ((tid & 63) == 0) s_d[tid >> 6] = e;
        __syncthreads();
        e = 0.0;
        for (int w = 0; w < 16; ++w) e += s_d[w];
        float picked = m;
        if (drawn) {
            u64 Z = s_sum[0];
            const u64 Zmin = mp > 0.0f ? s_sum[1] : Z;
            if (k > 0 && k < V) Z = smp_select(l, V, weight, [&](unsigned c, u64) { return c >= (unsigned)k; }).mass;
            if (tp < 1.0f) {
                const double need = (double)tp * (double)Z;
                Z = smp_select(l, V, weight, [&](unsigned, u64 s) { return (double)s >= need; }).mass;
            }
            if (Zmin < Z) Z = Zmin;
            const u64 w0 = 1ull << a.shift;
            if (Z < w0) Z = w0;
            float uu = a.u[j];
            uu = uu >= 0.0f ? fminf(uu, 0x1.fffffep-1f) : 0.0f;
            const double need = (double)uu * (double)Z;
            const u64 key = smp_select(l, V, weight, [&](unsigned, u64 s) { return (double)s > need; }).key;
            token = topk_key_idx(key);
            picked = topk_key_val(key);
        }
        logp = (float)(-smp_gap(m, picked) - log(e));
    }
    if (tid == 0) {
        a.tokens[j] = token;
        if (a.logp) a.logp[j] = logp;
    }
    if (a.E_tgt)
        for (int i = tid; i < a.E; i += 1024) a.y_emb[(size_t)j * a.E + i] = token >= 0 ? a.E_tgt[(size_t)token * a.E + i] : 0.0f;
}

q8_status q8i_sample(q8_ctx *ctx, const float *logits, int n, int V, int ldl, const q8_sampling *s, const float *u, int32_t *tokens, float *logp,
                     const float *E_tgt, int E, float *y_emb)
{
    SampleArgs a = {logits, (size_t)ldl, V, u, nullptr, nullptr, nullptr, nullptr, tokens, logp, E_tgt, y_emb, E, 0};
    if (s) { a.T = s->temperature; a.top_k = s->top_k; a.top_p = s->top_p; a.min_p = s->min_p; }
    int bits = 0;
    while (((size_t)1 << bits) < (size_t)V) ++bits;
    a.shift = 62 - bits < 46 ? 62 - bits : 46;                // the sum of V weights stays below 2^63
    hipLaunchKernelGGL(sample_kernel, dim3(n), dim3(1024), 0, ctx->stream, a);
    return q8i_launch_check(ctx, "sample");
}
