// q8_sample.hip -- one token drawn per row of logits, from given random numbers, under temperature, top-k, top-p and min-p.
//
// With m the largest logit of a row, word i has the weight w_i = exp(-(m - l_i) / T).  The words are ordered by (logit
// descending, index ascending); each filter keeps a prefix of that order: the first k words; the shortest prefix with at
// least p of the mass of those; the words with w_i >= min_p.  With Z the mass of the shortest of these prefixes the drawn
// token is the first word of the order whose cumulative mass exceeds u Z.  All three borders are found alike: "the first word
// at which (count, mass) up to it satisfies a condition that stays true further down".
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

#define SMP_BINS 2048                        // of 1/32 octave of weight each; beyond the last one every weight rounds to zero
#define SMP_LIST 1024                        // words of one bin that are ranked in LDS
#define SMP_LOG2E32 46.166241308446828384    // 32 log2(e)

// The distance below the largest logit, in double: two floats' difference can exceed the range of a float.
__device__ __forceinline__ double smp_gap(float m, float v) { return (double)m - (double)v; }

// A word's place in units of 1/32 octave of weight, x = gap c with c = 32 log2(e) / T, in fixed point: the sum with 2^20
// keeps the whole part in the high word and 32 bits of fraction in the low word.  Monotone in the logit.
struct SmpPlace {
    unsigned bin, frac;
};
__device__ __forceinline__ SmpPlace smp_place(double gap, double c)
{
    const double t = fmin(fma(gap, c, 0x1p20), 0x1p20 + SMP_BINS);
    return {(unsigned)__double2hiint(t) - 0x41300000u, (unsigned)__double2loint(t)};
}

// 2^(S - x / 32): a table over x mod 32 and a polynomial over the fraction, exp(-f 2^-32 ln 2 / 32), which interpolates at the
// Chebyshev points with the constant term held at 1 (within 2.9e-16; the fraction's 2^-33 is 2^-38.5 of the weight).
__device__ __forceinline__ double smp_weight(SmpPlace p, const double *s_pow)
{
    const double f = (double)p.frac;
    double e = -0x1.5a647398608b2p-195;
    e = fma(e, f, 0x1.3b27f902762c7p-155);
    e = fma(e, f, -0x1.c6b08b7b3d711p-116);
    e = fma(e, f, 0x1.ebfbdff7af203p-77);
    e = fma(e, f, -0x1.62e42fefa399fp-38);
    e = fma(e, f, 1.0);
    return ldexp(e * s_pow[p.bin & 31u], -(int)(p.bin >> 5));
}
// ... to the nearest whole number (below 2^47).
__device__ __forceinline__ u64 smp_whole(double w) { return (u64)__double_as_longlong(w + 0x1p52) & 0xfffffffffffffull; }

// A row of logits as a block goes through it: thread t has the pieces of four words t, t + BLOCK, ... counted from the 16-byte
// boundary at or below the row's begin.  Words outside the row and words that cannot be drawn (NaN) appear as -inf.
// NE > 0: NE words a thread, read once and kept in registers; NE == 0: read again on every pass.
template <int NE, int BLOCK> struct SmpRow {
    const float *l;
    int V, lead;                            // words before the row in its first piece
    bool top_inf;                           // the largest logit is +inf: words of +inf count as 0, others as -inf
    float v[NE ? NE : 1];

    __device__ __forceinline__ float4 piece(int c) const
    {
        const int i = 4 * c - lead;
        float4 r;
        if (i >= 0 && i + 3 < V) {
            r = *(const float4 *)(l + i);
        } else {
            r.x = i >= 0 && i < V ? l[i] : -INFINITY;
            r.y = i >= -1 && i + 1 < V ? l[i + 1] : -INFINITY;
            r.z = i >= -2 && i + 2 < V ? l[i + 2] : -INFINITY;
            r.w = i >= -3 && i + 3 < V ? l[i + 3] : -INFINITY;
        }
        r.x = fmaxf(r.x, -INFINITY); r.y = fmaxf(r.y, -INFINITY); r.z = fmaxf(r.z, -INFINITY); r.w = fmaxf(r.w, -INFINITY);
        if (top_inf) {
            r.x = r.x == INFINITY ? 0.0f : -INFINITY; r.y = r.y == INFINITY ? 0.0f : -INFINITY;
            r.z = r.z == INFINITY ? 0.0f : -INFINITY; r.w = r.w == INFINITY ? 0.0f : -INFINITY;
        }
        return r;
    }
    __device__ __forceinline__ void open(const float *row, int V_)
    {
        l = row;
        V = V_;
        lead = (int)(((uintptr_t)row & 15) >> 2);
        top_inf = false;
        if constexpr (NE > 0) {
#pragma unroll
            for (int j = 0; j < NE / 4; ++j) {
                const float4 r = piece(j * BLOCK + (int)threadIdx.x);
                v[4 * j] = r.x; v[4 * j + 1] = r.y; v[4 * j + 2] = r.z; v[4 * j + 3] = r.w;
            }
        }
    }
    __device__ __forceinline__ void share_inf()
    {
        top_inf = true;
        if constexpr (NE > 0) {
#pragma unroll
            for (int e = 0; e < NE; ++e) v[e] = v[e] == INFINITY ? 0.0f : -INFINITY;
        }
    }
    // f(four logits, index of the first), for every piece.  The logits are passed through an empty statement: what a pass computes
    // from them is not kept for the next one, for which there are no registers.
    template <class F> __device__ __forceinline__ void pieces(F f) const
    {
        if constexpr (NE > 0) {
            int first = 4 * (int)threadIdx.x - lead;
            asm volatile("" : "+v"(first));
#pragma unroll
            for (int j = 0; j < NE / 4; ++j) {
                float r[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
                asm volatile("" : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]));
                f(r, first + 4 * j * BLOCK);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const int total = (V + lead + 3) / 4;
            for (int c = threadIdx.x; c < total; c += BLOCK) {
                const float4 q = piece(c);
                const float r[4] = {q.x, q.y, q.z, q.w};
                f(r, 4 * c - lead);
            }
        }
    }
    template <class F> __device__ __forceinline__ void each(F f) const
    {
        pieces([&](const float (&r)[4], int i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f(r[e], i + e);
        });
    }
};

struct SmpShared {
    u64 mass[SMP_BINS];                     // per bin, then up to and including it
    unsigned count[SMP_BINS];
    struct { u64 key, mass; } list[SMP_LIST];
    double pow[32];                         // 2^(S - j / 32)
    u64 red_u[16];
    double red_d[16];
    unsigned red_c[16];
    u64 above, hit_key, hit_mass;
    unsigned listed, bin;
};

// One block per row.  Passes over the row: the largest logit; weights, summed into bins of 1/32 octave (LDS); for each border
// the words of the one bin that it falls into, ranked among themselves (by a histogram of their keys' bytes where there are
// more than SMP_LIST of them).
template <int NE, int BLOCK>
__global__ __launch_bounds__(BLOCK) void sample_row_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char smem[];
    SmpShared &s = *(SmpShared *)smem;
    const int j = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int WAVES = BLOCK / 64, PER = SMP_BINS / BLOCK;
    SmpRow<NE, BLOCK> row;
    row.open(a.logits + (size_t)j * a.ldl, a.V);
    const float T = a.T ? a.T[j] : 1.0f, tp = a.top_p ? a.top_p[j] : 1.0f, mp = a.min_p ? a.min_p[j] : 0.0f;
    const int k = a.top_k ? a.top_k[j] : 0;
    float u = a.u[j];
    u = u >= 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
#pragma unroll
    for (int t = 0; t < PER; ++t) { s.mass[t * BLOCK + tid] = 0; s.count[t * BLOCK + tid] = 0; }
    if (tid < 32) s.pow[tid] = ldexp(exp2(-(double)tid / 32.0), a.shift);
    if (tid == 0) { s.above = 0; s.hit_key = ~0ull; }

    float m = -INFINITY;
    row.each([&](float v, int) { m = fmaxf(m, v); });
    m = wave_max_f(m);
    if (lane == 0) s.red_d[wave] = (double)m;
    __syncthreads();
    m = (float)s.red_d[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, (float)s.red_d[w]);
    __syncthreads();

    int token = -1;
    float logp = -INFINITY;
    if (m > -INFINITY) {                                        // else: no word can be drawn
        if (m == INFINITY) { row.share_inf(); m = 0.0f; }
        const bool drawn = T > 0.0f;
        const double one = (double)(1ull << a.shift);
        // (T = inf: every finite distance counts as none, an infinite one still as infinite)
        const double c = fmax(SMP_LOG2E32 / (drawn ? (double)T : 1.0), 1e-300);
        const bool own_sum = a.logp && (T != 1.0f), some_min = drawn && mp > 0.0f;
        const double floor_w = (double)mp * one;
        double e = 0.0;
        u64 above = 0;
        row.pieces([&](const float (&v)[4], int) {
            double gap[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) gap[t] = smp_gap(m, v[t]);
            if (drawn) {
                SmpPlace p[4];
                double w[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) p[t] = smp_place(gap[t], c);
#pragma unroll
                for (int t = 0; t < 4; ++t) w[t] = smp_weight(p[t], s.pow);
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (p[t].bin < SMP_BINS) {
                        const u64 q = smp_whole(w[t]);
                        atomicAdd(&s.mass[p[t].bin], q);
                        atomicAdd(&s.count[p[t].bin], 1u);
                        if (some_min && w[t] >= floor_w) above += q;
                    }
            }
            if (own_sum) {                                      // sum of exp at T = 1: hardware exponential of the fraction of an octave
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const double x = fmin(fma(gap[t], SMP_LOG2E32 / 32.0, 0x1p20), 0x1p20 + 1024.0);
                    const float f = (float)(unsigned)__double2loint(x) * -0x1p-32f;
                    e += (double)ldexpf(__builtin_amdgcn_exp2f(f), -(int)((unsigned)__double2hiint(x) - 0x41300000u));
                }
            }
        });
        if (own_sum) e = wave_sum_d(e);
        if (lane == 0) s.red_d[wave] = e;
        if (some_min && above) atomicAdd(&s.above, above);
        __syncthreads();

        u64 Z = 0;
        if (drawn) {
            // ---- counts and masses up to and including each bin
            u64 mm[PER], sm = 0;
            unsigned cc[PER], sc = 0;
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                sm += s.mass[PER * tid + t]; mm[t] = sm;
                sc += s.count[PER * tid + t]; cc[t] = sc;
            }
            u64 im = sm;
            unsigned ic = sc;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const u64 om = __shfl_up(im, d);
                const unsigned oc = __shfl_up(ic, d);
                if (lane >= d) { im += om; ic += oc; }
            }
            if (lane == 63) { s.red_u[wave] = im; s.red_c[wave] = ic; }
            __syncthreads();
            im -= sm;
            ic -= sc;
            for (int w = 0; w < wave; ++w) { im += s.red_u[w]; ic += s.red_c[w]; }
#pragma unroll
            for (int t = 0; t < PER; ++t) { s.mass[PER * tid + t] = mm[t] + im; s.count[PER * tid + t] = cc[t] + ic; }
            __syncthreads();
            Z = s.mass[SMP_BINS - 1];
        }
        if (a.logp) {
            if (own_sum) {
                e = 0.0;
                for (int w = 0; w < WAVES; ++w) e += s.red_d[w];
            } else {
                e = (double)Z / one;
            }
        }

        // ---- the borders: 0 of the k best, 1 of top-p among them, 2 the drawn word (for T <= 0: the first word)
        for (int stage = 0; stage < 3; ++stage) {
            double need = 0.0;
            if (!drawn) {
                if (stage < 2) continue;
            } else if (stage == 0) {
                if (k <= 0 || (unsigned)k >= s.count[SMP_BINS - 1]) continue;
            } else if (stage == 1) {
                if (!(tp < 1.0f)) continue;
                need = fmax((double)tp * (double)Z, 0.5);       // (the first word is kept at top_p <= 0, too)
            } else {
                if (some_min && s.above < Z) Z = s.above;
                if (Z < (1ull << a.shift)) Z = 1ull << a.shift;
                need = (double)u * (double)Z;
            }
            auto cond = [&](unsigned cnt, u64 mass) { return stage == 0 ? cnt >= (unsigned)k : stage == 1 ? (double)mass >= need : (double)mass > need; };
            if (!drawn) {
                u64 best = 0;
                row.each([&](float v, int i) { if (v == m) { const u64 key = topk_key(v, i); best = key > best ? key : best; } });
                best = wave_max_u64(best);
                if (lane == 0) s.red_u[wave] = best;
                __syncthreads();
                for (int w = 0; w < WAVES; ++w) best = s.red_u[w] > best ? s.red_u[w] : best;
                token = topk_key_idx(best);
                logp = (float)-log(e);
                break;
            }
            // the bin
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                const int b = PER * tid + t;
                if (cond(s.count[b], s.mass[b]) && (b == 0 || !cond(s.count[b - 1], s.mass[b - 1]))) s.bin = (unsigned)b;
            }
            if (tid == 0) s.listed = 0;
            __syncthreads();
            const unsigned bin = s.bin;
            const u64 before_m = bin ? s.mass[bin - 1] : 0;
            const unsigned before_c = bin ? s.count[bin - 1] : 0, members = s.count[bin] - before_c;
            if (members <= SMP_LIST) {
                row.each([&](float v, int i) {
                    const SmpPlace p = smp_place(smp_gap(m, v), c);
                    if (p.bin == bin) {
                        const unsigned at = atomicAdd(&s.listed, 1u);
                        s.list[at].key = topk_key(v, i);
                        s.list[at].mass = smp_whole(smp_weight(p, s.pow));
                    }
                });
                __syncthreads();
                // each word against all of the list, by `parts` threads
                int lg = 0;
                while (lg < 6 && (members << (lg + 1)) <= (unsigned)BLOCK) ++lg;
                const int parts = 1 << lg, part = tid & (parts - 1);
                for (unsigned e0 = 0; e0 < members; e0 += BLOCK >> lg) {
                    const unsigned x = e0 + ((unsigned)tid >> lg);
                    const u64 key = x < members ? s.list[x].key : ~0ull;
                    u64 ms = 0;
                    unsigned cs = 0;
                    if (x < members)
                        for (unsigned o = part; o < members; o += parts)
                            if (s.list[o].key >= key) { ms += s.list[o].mass; ++cs; }
                    for (int d = 1; d < parts; d <<= 1) { ms += __shfl_xor(ms, d); cs += __shfl_xor(cs, d); }
                    if (x < members && part == 0) {
                        ms += before_m;
                        cs += before_c;
                        if (cond(cs, ms) && !cond(cs - 1, ms - s.list[x].mass)) { s.hit_key = key; s.hit_mass = ms; }
                    }
                }
                __syncthreads();
            } else {
                // the key's bytes from the top: a histogram of one byte of the bin's words that agree with what is known
                u64 known = 0, bm = before_m;
                unsigned bc = before_c;
                u64 *h_m = (u64 *)s.list;                       // [256]
                unsigned *h_c = (unsigned *)(h_m + 256);        // [256]
                for (int level = 7; level >= 0; --level) {
                    __syncthreads();
                    for (int d = tid; d < 256; d += BLOCK) { h_m[d] = 0; h_c[d] = 0; }
                    __syncthreads();
                    row.each([&](float v, int i) {
                        const SmpPlace p = smp_place(smp_gap(m, v), c);
                        if (p.bin != bin) return;
                        const u64 key = topk_key(v, i);
                        if (level < 7 && (key >> (8 * level + 8)) != (known >> (8 * level + 8))) return;
                        const int d = (int)(key >> (8 * level)) & 255;
                        atomicAdd(&h_m[d], smp_whole(smp_weight(p, s.pow)));
                        atomicAdd(&h_c[d], 1u);
                    });
                    __syncthreads();
                    if (tid == 0) {
                        u64 cm = bm;
                        unsigned ccnt = bc;
                        for (int d = 255; d >= 0; --d)
                            if (h_c[d]) {
                                if (cond(ccnt + h_c[d], cm + h_m[d])) {
                                    s.hit_key = known | ((u64)d << (8 * level));
                                    s.hit_mass = level ? cm : cm + h_m[d];
                                    s.listed = ccnt;
                                    break;
                                }
                                cm += h_m[d];
                                ccnt += h_c[d];
                            }
                    }
                    __syncthreads();
                    known = s.hit_key;
                    bm = s.hit_mass;
                    bc = s.listed;
                }
            }
            if (stage < 2) {
                Z = s.hit_mass;
            } else {
                token = topk_key_idx(s.hit_key);
                logp = (float)(-smp_gap(m, topk_key_val(s.hit_key)) - log(e));
            }
            __syncthreads();
        }
    }
    if (tid == 0) {
        a.tokens[j] = token;
        if (a.logp) a.logp[j] = logp;
    }
    if (a.E_tgt)
        for (int i = tid; i < a.E; i += BLOCK) a.y_emb[(size_t)j * a.E + i] = token >= 0 ? a.E_tgt[(size_t)token * a.E + i] : 0.0f;
}

q8_status q8i_sample(q8_ctx *ctx, const float *logits, int n, int V, int ldl, const q8_sampling *s, const float *u, int32_t *tokens, float *logp,
                     const float *E_tgt, int E, float *y_emb)
{
    SampleArgs a = {logits, (size_t)ldl, V, u, nullptr, nullptr, nullptr, nullptr, tokens, logp, E_tgt, y_emb, E, 0};
    if (s) { a.T = s->temperature; a.top_k = s->top_k; a.top_p = s->top_p; a.min_p = s->min_p; }
    int bits = 0;
    while (((size_t)1 << bits) < (size_t)V) ++bits;
    a.shift = 62 - bits < 46 ? 62 - bits : 46;                // the sum of V weights stays below 2^63
    const size_t smem = sizeof(SmpShared);
    // registers for the whole row (up to three words before it in its first piece) where a block has enough
#define SMP_GO(NE, BLOCK) hipLaunchKernelGGL((sample_row_kernel<NE, BLOCK>), dim3(n), dim3(BLOCK), smem, ctx->stream, a)
    const int words = V + 3;
    if (words <= 256 * 8) SMP_GO(8, 256);
    else if (words <= 1024 * 8) SMP_GO(8, 1024);
    else if (words <= 1024 * 24) SMP_GO(24, 1024);
    else if (words <= 1024 * 52) SMP_GO(52, 1024);
    else if (words <= 1024 * 64) SMP_GO(64, 1024);
    else SMP_GO(0, 1024);
#undef SMP_GO
    return q8i_launch_check(ctx, "sample");
}
