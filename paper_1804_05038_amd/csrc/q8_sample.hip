// q8_sample.hip -- one token drawn per row of logits, from given random numbers, under temperature, top-k, top-p and min-p.
//
// With m the largest logit of a row, word i has the weight w_i = exp(-(m - l_i) / T).  The words are ordered by (logit
// descending, index ascending); each filter keeps a prefix of that order: the first k words; the shortest prefix with at
// least p of the mass of those; the words with w_i >= min_p.  With Z the mass of the shortest of these prefixes the drawn
// token is the first word of the order whose cumulative mass exceeds u Z.  All borders are found alike: "the first word at
// which (count, mass) up to it satisfies a condition that stays true further down".
//
// Weights are whole numbers, rint(w_i 2^S): their sums are exact whatever their order, so a token does not depend on which
// thread adds what, and the borders between tokens lie where sums in 64-bit floating point put them to about 1e-12.
//
// Long rows take three launches over parts of the rows (largest logit; bins; borders and words), and every one reads the row.  Few
// rows are a chain of latencies: one of 50000 words 17 us (kernels 2 + 4 + 10 at the least), 64 of them 35.5; many are bound by memory and
// 64-bit arithmetic: 1000 of 63644 words 203 us (reading the 255 MB three times 127, the sums' LDS additions 24, the weights' 64-bit
// operations some 50).  Bins are as wide as the row's spread asks for: of 1/32 octave alone, flat rows (deviation 0.1 nat) went
// through the row again and again in one block: 64 rows of 50000 words with top-p 345 us, now 40, 12 of 250001 1328, now 55 (ordinary rows 3 %
// more).  Rows with more words in the borders' bins than their list holds, 1/32 of them, still do, for a time that grows with their length:
// one logit alone 295 us for one row of 50000 words, 1320 for 250001, 5400 for 2^20; deviation 0.1 nat and five words 8 nat above that 67 (with
// top-p 185), with top-p 764, 4900 (a sort of all words: 370 to 430, 390 to 425, 470 to 510).
#include "q8_internal.h"

#include <algorithm>
#include <math.h>

typedef unsigned long long u64;

#define SMP_BINS 2048                        // of 1/32 octave of weight each, or finer; 2048/32 octaves below the largest every weight rounds to zero
#define SMP_LOG2E32 46.166241308446828384    // 32 log2(e)
#define SMP_SMALL 2048                       // vocabularies of at most so many words: a block per row
#define SMP_MIDDLE 8192                      // ... where few rows have top-k or min_p
#define SMP_PARTS 128                        // blocks of a row
#define SMP_BLOCK 256                        // threads of these
#define SMP_ROWS 1024                        // rows of a launch
#define SMP_REACH 64.0f                      // nat below the largest logit that count in what a row spreads over
#define SMP_LIST 1536                        // words in LDS of those that lie where a row's borders do

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
    bool mass_sums;                         // at T = 1 the mass of a row stands for its sum of exponentials
    // rows over several blocks
    struct SmpRowState *state;              // [rows of the launch]
    u64 *lists;                             // [rows of the launch x list_words]: a row's words that lie where its borders do
    int list_words;
    int parts, part_pieces, row0;           // blocks of a row, 16-byte pieces of each, first row of the launch
};

// ------------------------------------------------------------------------------- weights ----

// The distance below the largest logit, in double: two floats' difference can exceed the range of a float.
__device__ __forceinline__ double smp_gap(float m, float v) { return (double)m - (double)v; }

// A word's place in units of 1/32 octave of weight, x = gap c with c = 32 log2(e) / T, in fixed point: the sum with 2^20
// keeps the whole part in the high word and 32 bits of fraction in the low word.  Monotone in the logit.  LIMIT: to SMP_BINS, where
// weights round to zero; else a place past the bins is some number that is not below SMP_BINS.
struct SmpPlace {
    unsigned bin, frac;
};
template <bool LIMIT = true> __device__ __forceinline__ SmpPlace smp_place(double gap, double c)
{
    double t = fma(gap, c, 0x1p20);
    if (LIMIT) t = fmin(t, 0x1p20 + SMP_BINS);
    return {(unsigned)__double2hiint(t) - 0x41300000u, (unsigned)__double2loint(t)};
}

__device__ const double smp_pow[32] = {         // 2^(-j / 32)
    0x1.0000000000000p+0, 0x1.f50765b6e4540p-1, 0x1.ea4afa2a490dap-1, 0x1.dfc97337b9b5fp-1,
    0x1.d5818dcfba487p-1, 0x1.cb720dcef9069p-1, 0x1.c199bdd85529cp-1, 0x1.b7f76f2fb5e47p-1,
    0x1.ae89f995ad3adp-1, 0x1.a5503b23e255dp-1, 0x1.9c49182a3f090p-1, 0x1.93737b0cdc5e5p-1,
    0x1.8ace5422aa0dbp-1, 0x1.82589994cce13p-1, 0x1.7a11473eb0187p-1, 0x1.71f75e8ec5f74p-1,
    0x1.6a09e667f3bcdp-1, 0x1.6247eb03a5585p-1, 0x1.5ab07dd485429p-1, 0x1.5342b569d4f82p-1,
    0x1.4bfdad5362a27p-1, 0x1.44e086061892dp-1, 0x1.3dea64c123422p-1, 0x1.371a7373aa9cbp-1,
    0x1.306fe0a31b715p-1, 0x1.29e9df51fdee1p-1, 0x1.2387a6e756238p-1, 0x1.1d4873168b9aap-1,
    0x1.172b83c7d517bp-1, 0x1.11301d0125b51p-1, 0x1.0b5586cf9890fp-1, 0x1.059b0d3158574p-1};

// 2^(S - x / 32): a table over x mod 32 times a polynomial over the fraction, exp(-f 2^-32 ln 2 / 32), which interpolates at the
// Chebyshev points with the constant term held at 1 (within 3.2e-13; rounding the fraction to 2^-33 is 1.7e-12).  The whole
// octaves leave the exponent.
__device__ __forceinline__ double smp_weight(SmpPlace p, const double *s_pow)
{
    const double f = (double)p.frac;
    double e = 0x1.38731c1a7139ap-155;
    e = fma(e, f, -0x1.c6ad294417fcap-116);
    e = fma(e, f, 0x1.ebfbde9d1da6cp-77);
    e = fma(e, f, -0x1.62e42fef8deebp-38);
    e = fma(e, f, 1.0);
    e *= s_pow[p.bin & 31u];
    return __hiloint2double(__double2hiint(e) - (int)((p.bin >> 5) << 20), __double2loint(e));
}
// ... to the nearest whole number (below 2^47).
__device__ __forceinline__ u64 smp_whole(double w) { return (u64)__double_as_longlong(w + 0x1p52) & 0xfffffffffffffull; }

// ---------------------------------------------------------------------------------- rows ----

// A row of logits, or a part of one, as a block goes through it: thread t has the pieces of four words t, t + BLOCK, ... of the
// part.  Words past the row and words that cannot be drawn (NaN) appear as -inf.  NE > 0: NE words a thread, read once and kept in
// registers; NE == 0: read again on every pass.
template <int NE, int BLOCK> struct SmpRow {
    __amdgpu_buffer_rsrc_t rows;
    int V, first, end;                      // pieces of the part
    bool top_inf;                           // the largest logit is +inf: words of +inf count as 0, others as -inf
    float v[NE ? NE : 1];

    __device__ __forceinline__ v4u load(int c) const { return __builtin_amdgcn_raw_buffer_load_b128(rows, c * 16, 0, 0); }
    template <bool CHECK = true> __device__ __forceinline__ void clean(v4u q, int c, float (&r)[4]) const
    {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            r[t] = fmaxf(__uint_as_float(q[t]), -INFINITY);
            if (CHECK) r[t] = 4 * c + t < V && c < end ? r[t] : -INFINITY;
            if (CHECK && top_inf) r[t] = r[t] == INFINITY ? 0.0f : -INFINITY;
        }
    }
    __device__ __forceinline__ void open(const float *row, int V_, int first_, int pieces_)
    {
        rows = q8_rsrc(row, (size_t)V_ * 4);
        V = V_;
        top_inf = false;
        first = first_;
        end = min(first_ + pieces_, (V_ + 3) / 4);
        if constexpr (NE > 0) {
            v4u q[NE / 4];
#pragma unroll
            for (int j = 0; j < NE / 4; ++j) q[j] = load(first + j * BLOCK + (int)threadIdx.x);      // (past the row: zeros, no access)
#pragma unroll
            for (int j = 0; j < NE / 4; ++j) {
                float r[4];
                clean(q[j], first + j * BLOCK + (int)threadIdx.x, r);
#pragma unroll
                for (int t = 0; t < 4; ++t) v[4 * j + t] = r[t];
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
    // f(four logits, index of the first), for every piece.  In registers, the logits and indexes pass through empty statements: what
    // a pass computes from them is not kept for the next one, for which there are no registers.
    template <class F> __device__ __forceinline__ void pieces(F f) const
    {
        if constexpr (NE > 0) {
            int at = 4 * (first + (int)threadIdx.x);
            asm volatile("" : "+v"(at));
            const int mine = (end - first + BLOCK - 1) / BLOCK;
#pragma unroll
            for (int j = 0; j < NE / 4; ++j) {
                if (j < mine) {
                    float r[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
                    asm volatile("" : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]));
                    f(r, at + 4 * j * BLOCK);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            int c = first + (int)threadIdx.x;
            if (!top_inf) {                             // as long as every thread has four whole pieces
                const int whole = min(end, V / 4);
                v4u q[4];
                int at = first;
                if (at + 4 * BLOCK <= whole) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) q[t] = load(c + t * BLOCK);
                }
                for (; at + 4 * BLOCK <= whole; at += 4 * BLOCK, c += 4 * BLOCK) {
                    v4u now[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) now[t] = q[t];
#pragma unroll
                    for (int t = 0; t < 4; ++t) q[t] = load(c + (4 + t) * BLOCK);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        float r[4];
                        clean<false>(now[t], c + t * BLOCK, r);
                        f(r, 4 * (c + t * BLOCK));
                    }
                }
            }
            for (; c < end; c += 4 * BLOCK) {
                v4u q[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) q[t] = load(c + t * BLOCK);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float r[4];
                    clean(q[t], c + t * BLOCK, r);
                    f(r, 4 * (c + t * BLOCK));
                }
            }
        }
    }
    __device__ __forceinline__ float largest() const           // of the thread's words
    {
        float m = -INFINITY;
        if constexpr (NE > 0) {
#pragma unroll
            for (int e = 0; e < NE; ++e) m = fmaxf(m, v[e]);
        } else {
            pieces([&](const float (&r)[4], int) { m = fmaxf(fmaxf(fmaxf(m, r[0]), fmaxf(r[1], r[2])), r[3]); });
        }
        return m;
    }
    // The same words, read from memory: for passes that few rows take, so that their code is not there once per piece.
    __device__ __forceinline__ SmpRow<0, BLOCK> stored() const
    {
        SmpRow<0, BLOCK> r;
        r.rows = rows; r.V = V; r.first = first; r.end = end; r.top_inf = top_inf;
        return r;
    }
    // f(key) for the words with near(logit) (cheap) and take(logit).
    template <class N, class T, class F> __device__ __forceinline__ void some(N near, T take, F f) const
    {
        pieces([&](const float (&v)[4], int i) {
            unsigned hit = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) hit |= near(v[t]) ? 1u << t : 0u;
            while (hit) {
                const int t = __ffs(hit) - 1;
                hit &= hit - 1;
                const float x = t == 0 ? v[0] : t == 1 ? v[1] : t == 2 ? v[2] : v[3];
                if (take(x)) f(topk_key(x, i + t));
            }
        });
    }
};

// Where a bin is in LDS: exchanged so that 32 threads that own eight bins each, or two, find theirs on different banks.
__device__ __forceinline__ unsigned smp_at(unsigned b) { return b ^ ((b >> 3) & 31u); }

template <int BLOCK> struct SmpShared {
    u64 mass[SMP_BINS];      // per bin (smp_at), then up to and including it
    unsigned count[SMP_BINS];
    u64 list[BLOCK];                        // keys of words that are ranked
    double pow[32];                         // 2^(S - j / 32)
    u64 red_u[16], red_v[16];
    double red_d[16];
    float red_f[16], red_g[16];
    unsigned red_c[16];
    u64 sum, above, hit_key, hit_mass, k_mass;
    unsigned listed, below, known_c, bytes[256];
};

// What a row asks for.
struct SmpAsk {
    float T, tp, mp, u;
    int k;
    bool drawn, some_min;
    double c, inv, one, floor_w;            // 32 log2(e) / T; 1 / c; 2^S; min_p 2^S
    int fine;                               // a bin is 1/32 octave over 2^fine

    // Bins for logits that spread over so much (an estimate: what lies below its end is in the last bin), as fine as 2^(most + 1) of them
    // hold it.
    __device__ __forceinline__ void spread(float d, int most = 10)
    {
        const float x = d * (float)c;
        fine = __builtin_amdgcn_readfirstlane(x < 0x1p-14f ? 24 : x < 1024.0f ? most + 127 - (int)(__float_as_uint(x) >> 23) : 0);
    }
    __device__ __forceinline__ unsigned bin(SmpPlace p) const
    {
        if (fine == 0) return min(p.bin, SMP_BINS - 1u);
        const unsigned b = __builtin_amdgcn_alignbit(p.bin, p.frac, (unsigned)(32 - fine));
        return p.bin < max((unsigned)SMP_BINS >> fine, 1u) ? min(b, SMP_BINS - 1u) : SMP_BINS - 1u;
    }

    __device__ __forceinline__ void open(const SampleArgs &a, int j)
    {
        T = a.T ? a.T[j] : 1.0f;
        tp = a.top_p ? a.top_p[j] : 1.0f;
        mp = a.min_p ? a.min_p[j] : 0.0f;
        k = a.top_k ? max(a.top_k[j], 0) : 0;
        u = a.u[j];
        u = u >= 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
        drawn = T > 0.0f;
        some_min = drawn && mp > 0.0f;
        one = (double)(1ull << a.shift);
        // (T = inf: every finite distance counts as none, an infinite one still as infinite)
        c = fmax(SMP_LOG2E32 / (drawn ? (double)T : 1.0), 1e-300);
        inv = 1.0 / c;
        fine = 0;
        floor_w = (double)mp * one;
    }
};

template <int BLOCK> __device__ __forceinline__ float smp_block_max(float v, float *red)
{
    v = wave_max_f(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < BLOCK / 64; ++w) v = fmaxf(v, red[w]);
    return v;
}

template <int CTRL, int ROWS> __device__ __forceinline__ u64 smp_from_below(u64 v)           // zero where there is no such lane
{
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xf, false);
    return ((u64)hi << 32) | lo;
}
__device__ __forceinline__ u64 smp_wave_scan(u64 v)             // up to and including each lane: within rows of 16, then over the rows
{
    v += smp_from_below<0x111, 0xf>(v);
    v += smp_from_below<0x112, 0xf>(v);
    v += smp_from_below<0x114, 0xf>(v);
    v += smp_from_below<0x118, 0xf>(v);
    v += smp_from_below<0x142, 0xa>(v);
    v += smp_from_below<0x143, 0xc>(v);
    return v;
}

// Masses and counts of the bins that each thread has, SMP_BINS / BLOCK in a row, -> s.mass, s.count: up to and including each bin.
template <int BLOCK> __device__ __forceinline__ void smp_scan(SmpShared<BLOCK> &s, u64 (&mm)[SMP_BINS / BLOCK], unsigned (&cc)[SMP_BINS / BLOCK], bool counts)
{
    constexpr int PER = SMP_BINS / BLOCK;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 sm = 0;
    unsigned sc = 0;
#pragma unroll
    for (int t = 0; t < PER; ++t) {
        sm += mm[t]; mm[t] = sm;
        sc += cc[t]; cc[t] = sc;
    }
    u64 im = smp_wave_scan(sm);
    unsigned ic = sc;
    if (counts) ic = (unsigned)smp_wave_scan(sc);
    if (lane == 63) { s.red_u[wave] = im; s.red_c[wave] = ic; }
    __syncthreads();
    im -= sm;
    ic -= sc;
    for (int w = 0; w < wave; ++w) { im += s.red_u[w]; ic += s.red_c[w]; }
#pragma unroll
    for (int t = 0; t < PER; ++t) {
        s.mass[smp_at(PER * tid + t)] = mm[t] + im;
        if (counts) s.count[smp_at(PER * tid + t)] = cc[t] + ic;
    }
    __syncthreads();
}

// ---- the words of s.list in their order ----

template <int J> __device__ __forceinline__ u64 smp_trade(u64 key, int lane, bool keep_larger)
{
    const unsigned lo = (unsigned)lane_xor_i<J>((int)(unsigned)key, lane), hi = (unsigned)lane_xor_i<J>((int)(unsigned)(key >> 32), lane);
    const u64 o = ((u64)hi << 32) | lo;
    return (key > o) == keep_larger ? key : o;
}
template <int J> __device__ __forceinline__ u64 smp_merge(u64 key, int tid, bool down)        // distances J, J / 2, ... 1
{
    key = smp_trade<J>(key, tid & 63, ((tid & J) == 0) == down);
    if constexpr (J > 1) key = smp_merge<J / 2>(key, tid, down);
    return key;
}

// The keys of s.list (s.listed of them, at most BLOCK) in descending order, one per thread (0 past the last), by a bitonic
// network: lanes trade by register moves, waves through LDS.
template <int BLOCK> __device__ __forceinline__ u64 smp_sorted(SmpShared<BLOCK> &s)
{
    const int tid = threadIdx.x;
    const unsigned members = s.listed;
    u64 key = (unsigned)tid < members ? s.list[tid] : 0;
    unsigned n = 64;
    while (n < members) n *= 2;
    if ((unsigned)(tid & ~63) < n) {
        key = smp_merge<1>(key, tid, (tid & 2) == 0);
        key = smp_merge<2>(key, tid, (tid & 4) == 0);
        key = smp_merge<4>(key, tid, (tid & 8) == 0);
        key = smp_merge<8>(key, tid, (tid & 16) == 0);
        key = smp_merge<16>(key, tid, (tid & 32) == 0);
        key = smp_merge<32>(key, tid, (tid & 64) == 0);
    }
    for (unsigned k = 128; k <= n; k *= 2) {
        const bool down = ((unsigned)tid & k) == 0;
        for (unsigned j = k / 2; j >= 64; j /= 2) {
            __syncthreads();
            s.list[tid] = key;
            __syncthreads();
            const u64 o = s.list[(unsigned)tid ^ j];
            key = (key > o) == ((((unsigned)tid & j) == 0) == down) ? key : o;
        }
        if ((unsigned)(tid & ~63) < n) key = smp_merge<32>(key, tid, down);
    }
    return key;
}

// Masses up to and including each thread's.
template <int BLOCK> __device__ __forceinline__ u64 smp_prefix(SmpShared<BLOCK> &s, u64 own)
{
    const int wave = threadIdx.x >> 6;
    u64 m = smp_wave_scan(own);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s.red_u[wave] = m;
    __syncthreads();
    for (int w = 0; w < wave; ++w) m += s.red_u[w];
    return m;
}

// ---------------------------------------------------------------------- borders by bins ----

__device__ __forceinline__ unsigned smp_rank(u64 mask) { return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0)); }

// Histogram of the weights of (a part of) a row, and per thread the mass of its words at or above the border of min_p.
// With SUM, e: the sum of the exponentials at T = 1 as well.
template <bool SUM, int BLOCK, class Row>
__device__ __forceinline__ u64 smp_histogram(const Row &row, SmpShared<BLOCK> &s, const SmpAsk &q, float m, double &e)
{
    u64 above = 0;
    row.pieces([&](const float (&v)[4], int) {
        if (SUM) {
#pragma unroll
            for (int t = 0; t < 4; t += 2) e += (double)(exp_le0(v[t] - m) + exp_le0(v[t + 1] - m));      // as the vocabulary layer's selection
        }
        SmpPlace p[4];
        double w[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) p[t] = smp_place<false>(smp_gap(m, v[t]), q.c);
#pragma unroll
        for (int t = 0; t < 4; ++t) w[t] = smp_weight(p[t], s.pow);
        unsigned bin[4];
        if (q.fine) {
#pragma unroll
            for (int t = 0; t < 4; ++t) bin[t] = q.bin(p[t]);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) bin[t] = p[t].bin;                                // (used below SMP_BINS only)
        }
        const float one = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v[0])));
        if (!__ballot(v[0] != one || v[1] != one || v[2] != one || v[3] != one)) {       // one logit: one addition, where 256 would meet
            const u64 lanes = __ballot(true);
            const unsigned words = 4u * (unsigned)__popcll(lanes);
            if (p[0].bin >= SMP_BINS) return;
            const u64 x = smp_whole(w[0]);
            if (q.some_min && w[0] >= q.floor_w) above += 4 * x;
            if (smp_rank(lanes) == 0) {
                atomicAdd(&s.mass[smp_at(bin[0])], x * words);
                if (q.k > 0) atomicAdd(&s.count[smp_at(bin[0])], words);
            }
            return;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (p[t].bin < SMP_BINS) {
                const u64 x = smp_whole(w[t]);
                const unsigned at = smp_at(bin[t]);
                atomicAdd(&s.mass[at], x);
                if (q.k > 0) atomicAdd(&s.count[at], 1u);
            }
        if (q.some_min) {
#pragma unroll
            for (int t = 0; t < 4; ++t) above += p[t].bin < SMP_BINS && w[t] >= q.floor_w ? smp_whole(w[t]) : 0;
        }
    });
    return above;
}

__device__ __forceinline__ u64 smp_mass_of(u64 key, float m, double c, const double *s_pow)
{
    const SmpPlace p = smp_place(smp_gap(m, topk_key_val(key)), c);
    return p.bin < SMP_BINS ? smp_whole(smp_weight(p, s_pow)) : 0;
}

__device__ __forceinline__ u64 smp_lane(u64 v, unsigned lane)
{
    return ((u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), (int)lane) << 32) | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, (int)lane);
}

__device__ __forceinline__ u64 smp_first(u64 v)                 // the first active lane's
{
    return ((u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(v >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)v);
}

// The first bin at which cond(count, mass up to and including it) is true; SMP_BINS - 1 if none.  By every wave for itself.
template <int BLOCK, class Cond> __device__ __forceinline__ unsigned smp_find(const SmpShared<BLOCK> &s, bool counts, Cond cond)
{
    const int lane = threadIdx.x & 63;
    constexpr int STEP = SMP_BINS / 64;
    const unsigned a = smp_at(STEP * lane + STEP - 1);
    const u64 far = __ballot(cond(counts ? s.count[a] : 0u, s.mass[a]));
    const int group = far ? __ffsll((long long)far) - 1 : 63;
    const unsigned b = smp_at(STEP * group + min(lane, STEP - 1));
    const u64 close = __ballot(cond(counts ? s.count[b] : 0u, s.mass[b]));
    return (unsigned)(STEP * group + (close ? min(__ffsll((long long)close) - 1, STEP - 1) : STEP - 1));
}

// The logits of the bins from b0 to b1, a little wider: a place is rounded to 2^-33 of 1/32 octave, which may carry a word over a border
// (bins are 2^-24 wide at the finest), and what is rounded here to below 2^-23 of the largest logit and the distance.
struct SmpWindow {
    unsigned b0, b1;
    float low, high;
    __device__ __forceinline__ void open(unsigned first, unsigned last, float m, const SmpAsk &q)
    {
        b0 = first;
        b1 = last;
        const double wide = __hiloint2double(__double2hiint(q.inv) - (q.fine << 20), __double2loint(q.inv)), am = fabs((double)m);
        const double gap0 = (double)first * wide, gap1 = last == SMP_BINS - 1 ? SMP_BINS * q.inv : ((double)last + 1.0) * wide;
        high = (float)((double)m - gap0 + 2.5e-7 * (am + gap0) + 0x1p-31 * q.inv);
        low = (float)((double)m - gap1 - 2.5e-7 * (am + gap1) - 0x1p-31 * q.inv);
    }
    __device__ __forceinline__ bool near(float v) const { return v >= low && v <= high; }
    __device__ __forceinline__ bool has(unsigned bin) const { return bin >= b0 && bin <= b1; }
};

// The drawn word of a row whose bins are in s.mass / s.count (up to and including each; counts only if top-k is in force) and
// whose mass of words at or above the min_p border is s.above: for each border the one bin that it falls into, then the
// words of that bin in their order.  words(window, f) calls f(key) for every word of a bin.  While there are more than 64, a
// histogram over 256 even parts of the range of their keys says in which of them the border lies.
template <int BLOCK, class Words>
__device__ __forceinline__ u64 smp_borders(Words words, SmpShared<BLOCK> &s, const SmpAsk &q, float m, int shift)
{
    const int tid = threadIdx.x;
    u64 Z = s.mass[smp_at(SMP_BINS - 1)], found = 0, found_m = 0;
#pragma unroll 1
    for (int stage = 0; stage < 3; ++stage) {                  // 0: of the k best, 1: of top-p among them, 2: the drawn word
        double need = 0.0;
        if (stage == 0) {
            if (q.k <= 0 || (unsigned)q.k >= s.count[smp_at(SMP_BINS - 1)]) continue;
        } else if (stage == 1) {
            if (!(q.tp < 1.0f)) continue;
            need = fmax((double)q.tp * (double)Z, 0.5);         // (the first word is kept at top_p <= 0, too)
        } else {
            if (q.some_min && s.above < Z) Z = s.above;
            if (Z < (1ull << shift)) Z = 1ull << shift;
            need = (double)q.u * (double)Z;
        }
        auto cond = [&](unsigned cnt, u64 mass) { return stage == 0 ? cnt >= (unsigned)q.k : stage == 1 ? (double)mass >= need : (double)mass > need; };
        const unsigned bin = smp_find<BLOCK>(s, stage == 0, cond);
        u64 before_m = bin ? s.mass[smp_at(bin - 1)] : 0;
        unsigned before_c = stage == 0 && bin ? s.count[smp_at(bin - 1)] : 0;
        SmpWindow win;
        win.open(bin, bin, m, q);
        u64 lowest = topk_key(win.low, 0x7fffffff), highest = topk_key(win.high, 0);
        bool again = false;
        for (int turn = 0; turn < 12; ++turn) {                 // (each at most a 256th of the keys before: nine suffice)
            if (tid == 0) s.listed = 0;
            __syncthreads();
            u64 first = 0, last = ~0ull;
            words(win, [&](u64 key) {
                if (key < lowest || key > highest) return;
                first = max(first, key);
                last = min(last, key);
                const unsigned at = atomicAdd(&s.listed, 1u);
                if (at < 64) s.list[at] = key;
            });
            __syncthreads();
            const unsigned members = s.listed;
            if (members <= 64) {                                // few: every wave for itself, each lane's word against all others
                const int lane = tid & 63;
                const u64 key = (unsigned)lane < members ? s.list[lane] : 0;
                const u64 own = key ? smp_mass_of(key, m, q.c, s.pow) : 0;
                u64 ms = before_m;
                unsigned cs = before_c;
                for (unsigned o = 0; o < members; ++o) {
                    const u64 ko = smp_lane(key, o), mo = smp_lane(own, o);
                    if (ko >= key) { ms += mo; ++cs; }
                }
                const u64 hit = __ballot(key && cond(cs, ms) && !cond(cs - 1, ms - own));
                const int at = hit ? __ffsll((long long)hit) - 1 : 0;
                found = smp_lane(key, at);
                found_m = smp_lane(ms, at);
                break;
            }
            if (again || members > BLOCK) {                     // the range that their keys have (of fewer at first, the bin's will do)
                first = wave_max_u64(first);
                last = ~wave_max_u64(~last);
                if ((tid & 63) == 0) { s.red_u[tid >> 6] = first; s.red_v[tid >> 6] = last; }
                __syncthreads();
                highest = s.red_u[0];
                lowest = s.red_v[0];
                for (int o = 1; o < BLOCK / 64; ++o) { highest = max(highest, s.red_u[o]); lowest = min(lowest, s.red_v[o]); }
                found = highest;
            }
            again = true;
            u64 *h_m = s.list;                                  // [256], the block has at least as many threads
            const int sh = max(0, 64 - 8 - __clzll((long long)(highest - lowest)));
            if (tid < 256) { h_m[tid] = 0; s.bytes[tid] = 0; }
            __syncthreads();
            words(win, [&](u64 key) {
                if (key < lowest || key > highest) return;
                const unsigned d = (unsigned)((key - lowest) >> sh), d0 = __builtin_amdgcn_readfirstlane(d);
                const u64 own = smp_mass_of(key, m, q.c, s.pow), own0 = smp_first(own);
                if (!__ballot(d != d0 || own != own0)) {        // one addition, where all would meet
                    const u64 lanes = __ballot(true);
                    if (smp_rank(lanes) == 0) {
                        atomicAdd(&h_m[d], own * (unsigned)__popcll(lanes));
                        atomicAdd(&s.bytes[d], (unsigned)__popcll(lanes));
                    }
                    return;
                }
                atomicAdd(&h_m[d], own);
                atomicAdd(&s.bytes[d], 1u);
            });
            __syncthreads();
            const unsigned d = 255u - (unsigned)tid;            // from the top
            const u64 own = tid < 256 ? h_m[d] : 0;
            const unsigned own_c = tid < 256 ? s.bytes[d] : 0;
            const u64 ms = before_m + smp_prefix<BLOCK>(s, own);
            const unsigned cs = stage == 0 ? before_c + (unsigned)smp_prefix<BLOCK>(s, own_c) : own_c;
            if (own_c && cond(cs, ms) && !cond(cs - own_c, ms - own)) { s.hit_key = lowest + ((u64)d << sh); s.hit_mass = ms - own; s.known_c = cs - own_c; }
            __syncthreads();
            lowest = s.hit_key;
            highest = lowest + ((1ull << sh) - 1);
            before_m = s.hit_mass;
            before_c = s.known_c;
            __syncthreads();
        }
        if (stage < 2) Z = found_m;
        __syncthreads();
    }
    return found;
}

// ---------------------------------------------------------------------- borders by a list ----

// The words of s.list (s.listed of them, at most BLOCK): a prefix of the row's order, all of the row's words if `whole`.
// total: the mass of the row, 0 where it was not summed (then top-k makes it unnecessary, or no other filter and a list of all
// words at or above the min_p border).  Returns the drawn word's key; 0 if a border lies below the list.
template <int BLOCK>
__device__ __forceinline__ u64 smp_borders_of_list(SmpShared<BLOCK> &s, const SmpAsk &q, float m, u64 total, bool whole, int shift)
{
    const int tid = threadIdx.x;
    const unsigned members = s.listed;
    if (members == 0) return 0;
    if (tid == 0) { s.k_mass = 0; s.hit_key = 0; s.above = 0; s.below = 0; }
    const u64 key = smp_sorted<BLOCK>(s);
    const bool mine = (unsigned)tid < members;
    const SmpPlace p = smp_place(smp_gap(m, topk_key_val(key)), q.c);
    const double w = mine && p.bin < SMP_BINS ? smp_weight(p, s.pow) : 0.0;
    const u64 own = smp_whole(w), ms = smp_prefix<BLOCK>(s, own);
    if ((unsigned)tid == members - 1) s.sum = ms;
    if (q.k > 0 && mine && tid == q.k - 1) s.k_mass = ms;
    if (q.some_min && mine) {                            // what min_p keeps ends at the last word at or above its border
        if (w >= q.floor_w) atomicMax(&s.above, ms);
        else s.below = 1;
    }
    __syncthreads();
    const u64 have = s.sum;
    u64 Z = total;
    if (q.k > 0) Z = s.k_mass ? s.k_mass : whole ? have : 0;
    else if (!total) Z = max(s.above, 1ull << shift);
    const bool min_known = q.some_min && (s.below || whole || (!q.k && !total));
    if (Z == 0) return 0;                                // the k-th word lies below the list
    if (q.tp < 1.0f) {
        const double need = fmax((double)q.tp * (double)Z, 0.5);
        if ((double)have < need) return 0;
        if (mine && (double)ms >= need && !((double)(ms - own) >= need)) s.hit_mass = ms;
        __syncthreads();
        Z = s.hit_mass;
    }
    if (q.some_min) {
        if (min_known) Z = s.above < Z ? s.above : Z;
        else if (Z > have) return 0;
    }
    if (Z < (1ull << shift)) Z = 1ull << shift;
    const double need = (double)q.u * (double)Z;
    if (!((double)have > need)) return 0;
    if (mine && (double)ms > need && !((double)(ms - own) > need)) s.hit_key = key;
    __syncthreads();
    return s.hit_key;
}

__device__ __forceinline__ void smp_write(const SampleArgs &a, int j, int token, float logp, int block)
{
    if ((unsigned)token >= (unsigned)a.V) token = -1;
    if (threadIdx.x == 0) {
        a.tokens[j] = token;
        if (a.logp) a.logp[j] = logp;
    }
    if (a.E_tgt)
        for (int i = threadIdx.x; i < a.E; i += block) a.y_emb[(size_t)j * a.E + i] = token >= 0 ? a.E_tgt[(size_t)token * a.E + i] : 0.0f;
}

// ------------------------------------------------------------------------- a block per row ----

// The row in registers.  Most rows are settled by the words at their top: with the s-th largest of each wave's 64 thread maxima,
// the least of these over the waves has at least s words of every wave at or above it; these words are collected and sorted.
// Only where a border lies below them (flat rows), the weights go into bins.
template <int NE, int BLOCK>
__global__ __launch_bounds__(BLOCK) void sample_row_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char smem[];
    SmpShared<BLOCK> &s = *(SmpShared<BLOCK> *)smem;
    const int j = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int WAVES = BLOCK / 64, PER = SMP_BINS / BLOCK;
    SmpRow<NE, BLOCK> row;
    row.open(a.logits + (size_t)j * a.ldl, a.V, 0, 0x7fffffff / 4);
    SmpAsk q;
    q.open(a, j);
    if (tid < 32) s.pow[tid] = smp_pow[tid] * q.one;
    if (tid == 0) { s.sum = 0; s.listed = 0; }

    float tm = row.largest();
    float m = smp_block_max<BLOCK>(tm, s.red_f);
    if (m == -INFINITY) { smp_write(a, j, -1, -INFINITY, BLOCK); return; }              // no word can be drawn
    if (m == INFINITY) {
        row.share_inf();
        m = 0.0f;
        tm = row.largest();
    }
    // ---- how far down the words are collected
    const int full = min(max((a.V + 3) / 256, 1), WAVES);                                // waves whose threads all have words
    const bool short_list = q.k > 0 && q.k <= 16 * full;                                 // top-k from the list alone
    const int rank = min(short_list ? (q.k + full - 1) / full : 64 / full, 64);
    const float sorted = wave_sort_desc_f(tm, lane);
    if (lane == rank - 1) s.red_g[wave] = sorted;
    __syncthreads();
    float thr = s.red_g[0];
    for (int w = 1; w < full; ++w) thr = fminf(thr, s.red_g[w]);
    const bool min_only = q.some_min && !q.k && !(q.tp < 1.0f);
    if (min_only)                                                                        // a little below the border of min_p
        thr = (float)((double)m + fmin(log((double)q.mp), 0.0) * (double)q.T * 1.000001 - 1e-6 - 1e-6 * fabs((double)m));
    if (!q.drawn) thr = m;
    const bool need_total = q.drawn && !short_list && !min_only, own_sum = a.logp && !(need_total && q.T == 1.0f);

    row.some([&](float v) { return v >= thr; }, [&](float v) { return v > -INFINITY; }, [&](u64 key) {
        const unsigned at = atomicAdd(&s.listed, 1u);
        if (at < BLOCK) s.list[at] = key;
    });
    double e = 0.0;
    if (need_total) {
        u64 sum = 0;
        row.pieces([&](const float (&v)[4], int) {
            SmpPlace p[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) p[t] = smp_place(smp_gap(m, v[t]), q.c);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum += smp_whole(smp_weight(p[t], s.pow));       // (zero past the bins)
        });
        if (sum) atomicAdd(&s.sum, sum);
    }
    if (own_sum) {
        row.pieces([&](const float (&v)[4], int) {
#pragma unroll
            for (int t = 0; t < 4; t += 2) e += (double)(exp_le0(v[t] - m) + exp_le0(v[t + 1] - m));      // as the vocabulary layer's selection
        });
        e = wave_sum_d(e);
        if (lane == 0) s.red_d[wave] = e;
    }
    __syncthreads();
    const u64 total = need_total ? s.sum : 0;
    const unsigned listed = s.listed;
    if (own_sum) {
        e = 0.0;
        for (int w = 0; w < WAVES; ++w) e += s.red_d[w];
    } else {
        e = (double)total / q.one;
    }
    __syncthreads();

    u64 key = 0;
    if (listed <= BLOCK) {
        if (q.drawn) {
            key = smp_borders_of_list<BLOCK>(s, q, m, total, thr == -INFINITY, a.shift);
        } else {                                        // the list: the words with the largest logit
            key = smp_sorted<BLOCK>(s);
            if (tid == 0) s.hit_key = key;
            __syncthreads();
            key = s.hit_key;
        }
    } else if (!q.drawn) {
        u64 best = 0;
        row.stored().pieces([&](const float (&v)[4], int i) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (v[t] == m) best = max(best, topk_key(v[t], i + t));
        });
        best = wave_max_u64(best);
        if (lane == 0) s.red_u[wave] = best;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) key = max(key, s.red_u[w]);
    }
    if (key == 0) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < PER; ++t) { s.mass[smp_at(t * BLOCK + tid)] = 0; s.count[smp_at(t * BLOCK + tid)] = 0; }
        if (tid == 0) s.above = 0;
        float far = 0.0f;
        row.pieces([&](const float (&v)[4], int) {
#pragma unroll
            for (int t = 0; t < 4; ++t) far = fmaxf(far, m - v[t] <= SMP_REACH ? m - v[t] : 0.0f);
        });
        q.spread(smp_block_max<BLOCK>(far, s.red_f));
        const u64 above = smp_histogram<false, BLOCK>(row, s, q, m, e);
        if (q.some_min && above) atomicAdd(&s.above, above);
        __syncthreads();
        u64 mm[PER];
        unsigned cc[PER];
#pragma unroll
        for (int t = 0; t < PER; ++t) { mm[t] = s.mass[smp_at(PER * tid + t)]; cc[t] = s.count[smp_at(PER * tid + t)]; }
        __syncthreads();
        smp_scan<BLOCK>(s, mm, cc, q.k > 0);
        const auto stored = row.stored();
        key = smp_borders<BLOCK>([&](const SmpWindow &win, auto f) {
            stored.some([&](float v) { return win.near(v); }, [&](float v) { const SmpPlace p = smp_place(smp_gap(m, v), q.c); return p.bin < SMP_BINS && q.bin(p) == win.b0; }, f);
        }, s, q, m, a.shift);
    }
    smp_write(a, j, topk_key_idx(key), (float)(-smp_gap(m, topk_key_val(key)) - log(e)), BLOCK);
}

// ---------------------------------------------------------------------- rows over several blocks ----

// What the launches leave for each other.
struct SmpRowState {
    u64 mass[SMP_BINS];
    unsigned count[SMP_BINS];
    double e[SMP_PARTS];                    // sum of exp at T = 1 of a part
    float top[SMP_PARTS], low[SMP_PARTS];   // its largest logit, and the lowest seen of those in reach of it
    float all_top;                          // the row's
    int fine;
    u64 above;
    unsigned listed, arrived;
};

// 1. The largest logit of each part, and how far the others lie below it (every fourth, as far as they are within SMP_REACH nat, which
// a mask's values are not); the row's sums are set to zero.
__global__ __launch_bounds__(SMP_BLOCK) void sample_top_kernel(SampleArgs a)
{
    __shared__ float red[SMP_BLOCK / 64], red_low[SMP_BLOCK / 64];
    const int j = a.row0 + blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
    SmpRowState &st = a.state[blockIdx.y];
    SmpRow<0, SMP_BLOCK> row;
    row.open(a.logits + (size_t)j * a.ldl, a.V, part * a.part_pieces, a.part_pieces);
    for (int b = part * SMP_BLOCK + tid; b < SMP_BINS; b += SMP_BLOCK * a.parts) { st.mass[b] = 0; st.count[b] = 0; }
    if (part == 0 && tid == 0) { st.above = 0; st.listed = 0; st.arrived = 0; }
    float m = -INFINITY, low = INFINITY;
    row.pieces([&](const float (&v)[4], int) {
        const float next = fmaxf(fmaxf(fmaxf(m, v[0]), fmaxf(v[1], v[2])), v[3]), cut = next - SMP_REACH;
        if (m < cut) low = next;
        low = fminf(low, v[0] >= cut ? v[0] : next);
        m = next;
    });
    const float top = smp_block_max<SMP_BLOCK>(m, red);
    low = -smp_block_max<SMP_BLOCK>(m >= top - SMP_REACH ? -low : -top, red_low);
    if (tid == 0) { st.top[part] = top; st.low[part] = low; }
}

// The row's largest logit, and its bins, by every wave for itself.
__device__ __forceinline__ float smp_row_top(const SampleArgs &a, const SmpRowState &st, SmpAsk &q)
{
    const int p0 = threadIdx.x & 63, p1 = p0 + 64;
    const float t0 = p0 < a.parts ? st.top[p0] : -INFINITY, t1 = p1 < a.parts ? st.top[p1] : -INFINITY;
    const float l0 = p0 < a.parts ? st.low[p0] : INFINITY, l1 = p1 < a.parts ? st.low[p1] : INFINITY;
    const float m = wave_max_f(fmaxf(t0, t1));
    const float d0 = t0 >= m - SMP_REACH ? m - l0 : 0.0f, d1 = t1 >= m - SMP_REACH ? m - l1 : 0.0f;
    q.spread(fminf(wave_max_f(fmaxf(d0, d1)), SMP_REACH), a.parts > 2 ? 9 : 10);
    return m;
}
static_assert(SMP_PARTS <= 128, "two parts a lane");

// The sum of the parts' sums, in one order, by every wave for itself.
__device__ __forceinline__ double smp_row_e(const SampleArgs &a, const SmpRowState &st)
{
    double e = 0.0;
    for (int p = threadIdx.x & 63; p < a.parts; p += 64) e += st.e[p];
    return wave_sum_d(e);
}

// 2. The weights of each part into bins, and the bins into the row's.
template <int NE>
__global__ __launch_bounds__(SMP_BLOCK) void sample_bins_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char smem[];
    SmpShared<SMP_BLOCK> &s = *(SmpShared<SMP_BLOCK> *)smem;
    const int j = a.row0 + blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    SmpRowState &st = a.state[blockIdx.y];
    SmpRow<NE, SMP_BLOCK> row;
    row.open(a.logits + (size_t)j * a.ldl, a.V, part * a.part_pieces, a.part_pieces);
    SmpAsk q;
    q.open(a, j);
    float m = smp_row_top(a, st, q);
    if (part == 0 && tid == 0) { st.all_top = m; st.fine = q.fine; }
    if (tid < 32) s.pow[tid] = smp_pow[tid] * q.one;
    if (m == -INFINITY) return;
    if (m == INFINITY) { row.share_inf(); m = 0.0f; }
    if (q.drawn) {
#pragma unroll
        for (int t = 0; t < SMP_BINS / SMP_BLOCK; ++t) { s.mass[smp_at(t * SMP_BLOCK + tid)] = 0; s.count[smp_at(t * SMP_BLOCK + tid)] = 0; }
    }
    __syncthreads();
    const bool own_sum = a.logp && !(a.mass_sums && q.T == 1.0f);
    double e = 0.0;
    u64 above = 0;
    if (own_sum) {
        if (q.drawn) {
            above = smp_histogram<true, SMP_BLOCK>(row, s, q, m, e);
        } else {
            row.pieces([&](const float (&v)[4], int) {
#pragma unroll
                for (int t = 0; t < 4; t += 2) e += (double)(exp_le0(v[t] - m) + exp_le0(v[t + 1] - m));
            });
        }
        e = wave_sum_d(e);
        if (lane == 0) s.red_d[wave] = e;
    } else if (q.drawn) {
        above = smp_histogram<false, SMP_BLOCK>(row, s, q, m, e);
    }
    __syncthreads();
    if (tid == 0 && own_sum) {
        e = s.red_d[0];
        for (int w = 1; w < SMP_BLOCK / 64; ++w) e += s.red_d[w];
        st.e[part] = e;
    }
    if (!q.drawn) return;
    if (q.some_min && above) atomicAdd(&st.above, above);
#pragma unroll
    for (int t = 0; t < SMP_BINS / SMP_BLOCK; ++t) {
        const int b = t * SMP_BLOCK + tid;
        const u64 x = s.mass[smp_at(b)];
        if (x) atomicAdd(&st.mass[b], x);
        const unsigned c = q.k > 0 ? s.count[smp_at(b)] : 0;
        if (c) atomicAdd(&st.count[b], c);
    }
}

// 3. The bins that the borders fall into, as far as the bins alone tell (a border's mass is known to one bin, and what depends on
// it to the bins that both ends give); the words of these bins, from every part; and the last part to be done finds the
// borders among them.
template <int NE>
__global__ __launch_bounds__(SMP_BLOCK) void sample_draw_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char smem[];
    SmpShared<SMP_BLOCK> &s = *(SmpShared<SMP_BLOCK> *)smem;
    __shared__ u64 s_found[SMP_LIST];
    __shared__ unsigned s_at, s_last;
    const int j = a.row0 + blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
    SmpRowState &st = a.state[blockIdx.y];
    SmpRow<NE, SMP_BLOCK> row;
    SmpAsk q;
    q.open(a, j);
    // (requested before anything is waited for)
    u64 mass[SMP_BINS / SMP_BLOCK];
    unsigned count[SMP_BINS / SMP_BLOCK];
#pragma unroll
    for (int t = 0; t < SMP_BINS / SMP_BLOCK; ++t) { mass[t] = st.mass[SMP_BINS / SMP_BLOCK * tid + t]; count[t] = st.count[SMP_BINS / SMP_BLOCK * tid + t]; }
    const u64 above = st.above;
    const double e_parts = smp_row_e(a, st);
    row.open(a.logits + (size_t)j * a.ldl, a.V, part * a.part_pieces, a.part_pieces);
    float m = st.all_top;
    q.fine = __builtin_amdgcn_readfirstlane(st.fine);
    if (m == -INFINITY) {                               // no word can be drawn
        if (part == 0) smp_write(a, j, -1, -INFINITY, SMP_BLOCK);
        return;
    }
    if (m == INFINITY) { row.share_inf(); m = 0.0f; }
    if (tid < 32) s.pow[tid] = smp_pow[tid] * q.one;
    if (tid == 0) s.above = above;
    SmpWindow w[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) { w[i].b0 = 1; w[i].b1 = 0; w[i].low = INFINITY; w[i].high = -INFINITY; }
    if (q.drawn) {
        smp_scan<SMP_BLOCK>(s, mass, count, q.k > 0);
        u64 low = s.mass[smp_at(SMP_BINS - 1)], high = low;
        if (q.k > 0 && (unsigned)q.k < s.count[smp_at(SMP_BINS - 1)]) {
            const unsigned b = smp_find<SMP_BLOCK>(s, true, [&](unsigned c, u64) { return c >= (unsigned)q.k; });
            w[0].open(b, b, m, q);
            low = b ? s.mass[smp_at(b - 1)] : 0;
            high = s.mass[smp_at(b)];
        }
        if (q.tp < 1.0f) {
            const double n0 = fmax((double)q.tp * (double)low, 0.5), n1 = fmax((double)q.tp * (double)high, 0.5);
            const unsigned b0 = smp_find<SMP_BLOCK>(s, false, [&](unsigned, u64 x) { return (double)x >= n0; }), b1 = smp_find<SMP_BLOCK>(s, false, [&](unsigned, u64 x) { return (double)x >= n1; });
            w[1].open(b0, b1, m, q);
            low = b0 ? s.mass[smp_at(b0 - 1)] : 0;
            high = s.mass[smp_at(b1)];
        }
        if (q.some_min) { low = min(low, above); high = min(high, above); }
        const u64 first = 1ull << a.shift;
        const double n0 = (double)q.u * (double)max(low, first), n1 = (double)q.u * (double)max(high, first);
        w[2].open(smp_find<SMP_BLOCK>(s, false, [&](unsigned, u64 x) { return (double)x > n0; }), smp_find<SMP_BLOCK>(s, false, [&](unsigned, u64 x) { return (double)x > n1; }), m, q);
    } else {
        w[2].low = w[2].high = m;
        w[2].b0 = 0; w[2].b1 = SMP_BINS;
        __syncthreads();
    }
    // ---- the words of those bins (and few beside them, which the borders pass over): every wave has a list of its own, and puts it
    // into the row's when it is full
    const bool use0 = w[0].b0 <= w[0].b1, use1 = w[1].b0 <= w[1].b1;
    const int wave = tid >> 6;
    constexpr unsigned LIST = SMP_LIST / (SMP_BLOCK / 64);
    u64 *list = a.lists + (size_t)blockIdx.y * a.list_words;
    const unsigned room = (unsigned)a.list_words;
    unsigned mine = 0;                                  // (the same in all lanes that are at work; lane 0 is to the end)
    row.pieces([&](const float (&v)[4], int i) {
        bool n[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) n[t] = w[2].near(v[t]);
        if (use0) {
#pragma unroll
            for (int t = 0; t < 4; ++t) n[t] = n[t] | w[0].near(v[t]);
        }
        if (use1) {
#pragma unroll
            for (int t = 0; t < 4; ++t) n[t] = n[t] | w[1].near(v[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u64 mask = __ballot(n[t]);
            if (mask) {
                const unsigned more = (unsigned)__popcll(mask);
                if (mine + more > LIST) {
                    const u64 active = __ballot(true);
                    const unsigned me = smp_rank(active);
                    unsigned at = 0;
                    if (me == 0) at = atomicAdd(&st.listed, mine);
                    at = __builtin_amdgcn_readfirstlane(at);
                    __builtin_amdgcn_wave_barrier();
                    for (unsigned x = me; x < mine; x += (unsigned)__popcll(active))
                        if (at + x < room) __hip_atomic_store(&list[at + x], s_found[wave * LIST + x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __builtin_amdgcn_wave_barrier();
                    mine = 0;
                }
                if (n[t]) s_found[wave * LIST + mine + smp_rank(mask)] = topk_key(v[t], i + t);
                mine += more;
            }
        }
    });
    mine = __builtin_amdgcn_readfirstlane(mine);
    if ((tid & 63) == 0) s.red_c[wave] = mine;
    __syncthreads();
    unsigned found = 0, before = 0;
#pragma unroll
    for (int o = 0; o < SMP_BLOCK / 64; ++o) {
        const unsigned c = s.red_c[o];
        if (o < wave) before += c;
        found += c;
    }
    if (tid == 0) s_at = found ? atomicAdd(&st.listed, found) : 0u;
    __syncthreads();
    for (unsigned x = tid & 63; x < mine; x += 64)
        if (s_at + before + x < room) __hip_atomic_store(&list[s_at + before + x], s_found[wave * LIST + x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    q8_stores_performed();
    __syncthreads();
    if (tid == 0) s_last = __hip_atomic_fetch_add(&st.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)a.parts - 1 ? 1u : 0u;
    __syncthreads();
    if (!s_last) return;

    // ---- the last part: the borders
    const unsigned listed = __hip_atomic_load(&st.listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    SmpRow<0, SMP_BLOCK> whole;
    whole.open(a.logits + (size_t)j * a.ldl, a.V, 0, 0x7fffffff / 4);
    whole.top_inf = row.top_inf;
    if (listed <= SMP_LIST) {                           // from here on in LDS
        for (unsigned x = tid; x < listed; x += SMP_BLOCK) s_found[x] = __hip_atomic_load(&list[x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
    }
    u64 key;
    if (q.drawn) {
        key = smp_borders<SMP_BLOCK>([&](const SmpWindow &win, auto f) {
            auto in = [&](float v) { const SmpPlace p = smp_place(smp_gap(m, v), q.c); return p.bin < SMP_BINS && q.bin(p) == win.b0; };
            if (listed > room) {
                whole.some([&](float v) { return win.near(v); }, in, f);
                return;
            }
            if (listed > SMP_LIST) {
                for (unsigned x0 = tid; x0 < listed; x0 += 4 * SMP_BLOCK) {
                    u64 k[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) k[t] = x0 + t * SMP_BLOCK < listed ? __hip_atomic_load(&list[x0 + t * SMP_BLOCK], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (k[t] && win.near(topk_key_val(k[t])) && in(topk_key_val(k[t]))) f(k[t]);
                }
                return;
            }
            for (unsigned x = tid; x < listed; x += SMP_BLOCK)
                if (in(topk_key_val(s_found[x]))) f(s_found[x]);
        }, s, q, m, a.shift);
    } else {
        u64 best = 0;
        if (listed > SMP_LIST) {
            whole.pieces([&](const float (&v)[4], int i) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (v[t] == m) best = max(best, topk_key(v[t], i + t));
            });
        } else {
            for (unsigned x = tid; x < listed; x += SMP_BLOCK) best = max(best, s_found[x]);
        }
        best = wave_max_u64(best);
        if ((tid & 63) == 0) s.red_u[tid >> 6] = best;
        __syncthreads();
        key = s.red_u[0];
        for (int w = 1; w < SMP_BLOCK / 64; ++w) key = max(key, s.red_u[w]);
    }
    const double e = a.mass_sums && q.T == 1.0f ? (double)s.mass[smp_at(SMP_BINS - 1)] / q.one : e_parts;
    smp_write(a, j, topk_key_idx(key), (float)(-smp_gap(m, topk_key_val(key)) - log(e)), SMP_BLOCK);
}

static int sample_rows(int n) { return n < SMP_ROWS ? n : SMP_ROWS; }

// Words that a row's list holds, 1/32 of the row: of Gaussian logits 0.6 % lie in the fullest bin (row of 1.4 nat deviation), and there are
// three.  Where there are more, one block goes through the row again for every border (12 rows of 250001 words 108 us instead of 26; a list of
// 16384 words at most: one row of 2^24 words 20.8 ms instead of 0.42, with top-p 33 instead of 0.82).
static int sample_list_words(int V) { return std::max(SMP_LIST, (V / 32 + 63) & ~63); }

size_t q8i_sample_bytes(int n, int V) { return V <= SMP_SMALL ? 0 : (size_t)sample_rows(n) * (sizeof(SmpRowState) + sizeof(u64) * sample_list_words(V)); }

q8_status q8i_sample(q8_ctx *ctx, const float *logits, int n, int V, int ldl, const q8_sampling *s, const float *u, int32_t *tokens, float *logp,
                     const float *E_tgt, int E, float *y_emb, void *state)
{
    SampleArgs a;
    memset(&a, 0, sizeof(a));
    a.logits = logits; a.ldl = (size_t)ldl; a.V = V; a.u = u; a.tokens = tokens; a.logp = logp; a.E_tgt = E_tgt; a.E = E; a.y_emb = y_emb;
    if (s) { a.T = s->temperature; a.top_k = s->top_k; a.top_p = s->top_p; a.min_p = s->min_p; }
    int bits = 0;
    while (((size_t)1 << bits) < (size_t)V) ++bits;
    a.shift = 62 - bits < 46 ? 62 - bits : 46;                // the sum of V weights stays below 2^63
    // words below half a unit are missing from the mass, V 2^-(S + 1) in all: up to 2^19 words 2^-25 of the largest, less than the logarithm's
    // rounding to fp32 (at 2^24 it would be 2^-15)
    a.mass_sums = V <= 1 << 19;
    const size_t smem = sizeof(SmpShared<256>);
    // A block per row while its threads hold eight words each at most and mostly find the borders among the words at the top, which
    // top-k and min_p see to (us; a block per row, several blocks): 5 rows of 2000 words 9.8, 14.8 without filters, 10.0, 17.1 with top-k, 1000
    // rows 20.4, 25.7 and 18.3, 30.8; 64 rows of 5003 words 24.0, 17.3 without filters, 12.7, 19.6 with top-k, 11.9, 17.7 with min_p,
    // 32.7, 21.2 with top-p, 1000 rows 73.9, 36.7, 40.7, 39.6, 40.6, 39.8, 98.1, 43.0.  Of 50000 words 25 to 29 against 16 to 17 (one row).
    if (V <= SMP_SMALL) {
        hipLaunchKernelGGL((sample_row_kernel<8, 256>), dim3(n), dim3(256), smem, ctx->stream, a);
        return q8i_launch_check(ctx, "sample");
    }
    if (V <= SMP_MIDDLE && n <= 256 && (a.top_k || a.min_p)) {
        hipLaunchKernelGGL((sample_row_kernel<8, 1024>), dim3(n), dim3(1024), sizeof(SmpShared<1024>), ctx->stream, a);
        return q8i_launch_check(ctx, "sample");
    }
    a.state = (SmpRowState *)state;
    a.list_words = sample_list_words(V);
    a.lists = (u64 *)(a.state + sample_rows(n));
    const int pieces = (V + 3) / 4;
    for (a.row0 = 0; a.row0 < n; a.row0 += SMP_ROWS) {
        const int rows = n - a.row0 < SMP_ROWS ? n - a.row0 : SMP_ROWS;
        // three blocks a compute unit, none of less than 2048 words: 64 rows of 50000 words 36.5 / 37.2 / 47 us with 768 / 1024 / 1536
        // blocks, 12 of 250001 26.4 / 31.6 / 40, 200 of 33658 53.9 / 58.4 / 67 (all of these before bins of a row's own width)
        int parts = (768 + rows - 1) / rows;
        if (parts > (pieces + 511) / 512) parts = (pieces + 511) / 512;
        if (parts > SMP_PARTS) parts = SMP_PARTS;
        a.part_pieces = (pieces + parts - 1) / parts;
        a.parts = (pieces + a.part_pieces - 1) / a.part_pieces;
        const dim3 grid(a.parts, rows), block(SMP_BLOCK);
        hipLaunchKernelGGL(sample_top_kernel, grid, block, 0, ctx->stream, a);
        if (a.part_pieces <= 4 * SMP_BLOCK) {
            hipLaunchKernelGGL(sample_bins_kernel<16>, grid, block, smem, ctx->stream, a);
            hipLaunchKernelGGL(sample_draw_kernel<16>, grid, block, smem, ctx->stream, a);
        } else {
            hipLaunchKernelGGL(sample_bins_kernel<0>, grid, block, smem, ctx->stream, a);
            hipLaunchKernelGGL(sample_draw_kernel<0>, grid, block, smem, ctx->stream, a);
        }
        const q8_status st = q8i_launch_check(ctx, "sample");
        if (st) return st;
    }
    return Q8_OK;
}
