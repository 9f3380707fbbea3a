// q8_delta.hip -- the gated delta rule: per token and head S = a S, u = b (v - S^T k), S = S + k u^T, o = S^T q with a state S of
// dk x dv numbers; one token for n slots, and whole sequences laid end to end.
#include "q8_internal.h"
#include "q8_parts.h"
#include "q8_route.h"

#include <algorithm>
#include <math.h>

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));

#define DELTA_EPS 1e-6f              // of the unit length of queries and keys
#define DELTA_LEAST (-200.0)         // decays below exp(-200) are zeros, and sums of these stay exact enough in 64 bits

// Up to four floats from p on (`left` of them), zeros for the others.
__device__ __forceinline__ v4f load4(const float *p, int left, int vec)
{
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (vec) {
        if (left > 0) v = *(const v4f *)p;
    } else {
        if (left > 0) v[0] = p[0];
        if (left > 1) v[1] = p[1];
        if (left > 2) v[2] = p[2];
        if (left > 3) v[3] = p[3];
    }
    return v;
}

__device__ __forceinline__ void store4(float *p, int left, int vec, v4f v)
{
    if (vec) {
        if (left > 0) *(v4f *)p = v;
    } else {
        if (left > 0) p[0] = v[0];
        if (left > 1) p[1] = v[1];
        if (left > 2) p[2] = v[2];
        if (left > 3) p[3] = v[3];
    }
}

__device__ __forceinline__ float wave_sum_f(float v)
{
    v += __int_as_float(dpp_mov_i<DPP_XOR1>(__float_as_int(v)));
    v += __int_as_float(dpp_mov_i<DPP_XOR2>(__float_as_int(v)));
    v += __int_as_float(dpp_mov_i<DPP_HALF_MIRROR>(__float_as_int(v)));
    v += __int_as_float(dpp_mov_i<DPP_MIRROR>(__float_as_int(v)));
    v += __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), SWZ_XOR16));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32));
}

__device__ __forceinline__ float unit_of(float squares) { return 1.0f / sqrtf(squares + DELTA_EPS); }

// ------------------------------------------------------------------------------- one token ----

struct DeltaStepArgs {
    q8_delta_inputs in;
    const float *state;
    const int *parent;
    float *state_out, *out;
    int slots, ldo, vec, vec_qk;     // vec: states, values and results in whole 16-byte pieces; vec_qk: queries and keys
};

// A block per slot, head and up to 4 LPR columns of the state.  Thread (r, c): columns 4 c .. 4 c + 3 of the R rows r R .. r R + R - 1, read
// once and written once.  What a token reads is a q^T S + (q k) u, so that k^T S and q^T S come from the old state in one pass and
// meet in LDS once.  Bound by memory: 64 slots of 16 heads of 128 x 128 in 28.7 us, 4.7 TB/s read and written (a copy of 4 GiB: 4.8); 1000 slots of 6
// heads of 100 x 72 in 75.8, 4.6; 5 slots of 4 heads of 64 x 64 in 4.0, a launch.
template <int LPR, int R>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaStepArgs a)
{
    constexpr int GROUPS = 256 / LPR;
    __shared__ __align__(16) float s_k[GROUPS * R], s_q[GROUPS * R];
    __shared__ v4f s_part[4][2][LPR];
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = tid % LPR, rg = tid / LPR;
    const int head = blockIdx.x % p.hv, j = blockIdx.x / p.hv, kh = head / (p.hv / p.hk), col = blockIdx.y * 4 * LPR + 4 * c, left = p.dv - col;
    const int from = a.parent ? a.parent[j] : j;
    const bool fresh = !a.state || from < 0 || from >= a.slots;
    const size_t size = (size_t)p.dk * p.dv;
    const float *S = a.state + ((size_t)(fresh ? 0 : from) * p.hv + head) * size + col;
    v4f s[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int row = rg * R + t;
        s[t] = load4(S + (size_t)row * p.dv, fresh || row >= p.dk ? 0 : left, a.vec);
    }
    const float *k = p.k + (size_t)j * p.ldk + (size_t)kh * p.dk, *q = p.q + (size_t)j * p.ldq + (size_t)kh * p.dk;
    const float g = p.g[(size_t)j * p.ldg + head], beta = p.beta[(size_t)j * p.ldb + head];
    const v4f v = load4(p.v + (size_t)j * p.ldv + (size_t)head * p.dv + col, left, a.vec);
    // every wave forms the sums over q and k for itself: dk <= 256 is four elements a lane
    const v4f kl = load4(k + 4 * lane, p.dk - 4 * lane, a.vec_qk), ql = load4(q + 4 * lane, p.dk - 4 * lane, a.vec_qk);
    if (wave == 0 && 4 * lane < GROUPS * R) {
        *(v4f *)(s_k + 4 * lane) = kl;
        *(v4f *)(s_q + 4 * lane) = ql;
    }
    float kk = 0.0f, qq = 0.0f, qk = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        kk = fmaf(kl[e], kl[e], kk);
        qq = fmaf(ql[e], ql[e], qq);
        qk = fmaf(ql[e], kl[e], qk);
    }
    kk = wave_sum_f(kk);
    qq = wave_sum_f(qq);
    qk = wave_sum_f(qk);
    const float rk = p.normalize ? unit_of(kk) : 1.0f, rq = (p.normalize ? unit_of(qq) : 1.0f) * p.scale, decay = expf(g);
    __syncthreads();
    v4f ks = {0.0f, 0.0f, 0.0f, 0.0f}, qs = ks;
    float kr[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        kr[t] = s_k[rg * R + t];
        const float qr = s_q[rg * R + t];
        s[t] *= decay;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ks[e] = fmaf(kr[t], s[t][e], ks[e]);
            qs[e] = fmaf(qr, s[t][e], qs[e]);
        }
    }
#pragma unroll
    for (int x = LPR; x < 64; x *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ks[e] += __shfl_xor(ks[e], x);
            qs[e] += __shfl_xor(qs[e], x);
        }
    if (lane < LPR) {
        s_part[wave][0][c] = ks;
        s_part[wave][1][c] = qs;
    }
    __syncthreads();
    ks = s_part[0][0][c] + s_part[1][0][c] + s_part[2][0][c] + s_part[3][0][c];
    v4f u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = beta * (v[e] - rk * ks[e]) * rk;
    float *So = a.state_out + ((size_t)j * p.hv + head) * size + col;
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int row = rg * R + t;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = fmaf(kr[t], u[e], s[t][e]);
        store4(So + (size_t)row * p.dv, row >= p.dk ? 0 : left, a.vec, s[t]);
    }
    if (tid < LPR) {
        qs = s_part[0][1][c] + s_part[1][1][c] + s_part[2][1][c] + s_part[3][1][c];
        v4f o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = rq * fmaf(qk, u[e], qs[e]);
        store4(a.out + (size_t)j * a.ldo + (size_t)head * p.dv + col, left, a.vec, o);
    }
}

static bool whole16(const void *p, int ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; }

template <int LPR> static void launch_step(q8_ctx *ctx, const DeltaStepArgs &a, int n)
{
    const dim3 grid((unsigned)((size_t)n * a.in.hv), (a.in.dv + 4 * LPR - 1) / (4 * LPR));
    const int rows = (a.in.dk * LPR + 255) / 256;                           // of a thread
    void (*const kernel)(DeltaStepArgs) = rows <= 4 ? delta_step_kernel<LPR, 4> : rows <= 8 ? delta_step_kernel<LPR, 8>
                                          : rows <= 16 ? delta_step_kernel<LPR, 16> : delta_step_kernel<LPR, 32>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, ctx->stream, a);
}

q8_status q8i_delta_step(q8_ctx *ctx, const q8_delta_inputs *in, int n, const float *state, int slots, const int *parent, float *state_out, float *out, int ldo)
{
    DeltaStepArgs a = {*in, state, parent, state_out, out, slots, ldo, 0, 0};
    a.vec = in->dv % 4 == 0 && whole16(state, 0) && whole16(state_out, 0) && whole16(in->v, in->ldv) && whole16(out, ldo);
    a.vec_qk = in->dk % 4 == 0 && whole16(in->q, in->ldq) && whole16(in->k, in->ldk);
    if (in->dv <= 32) launch_step<8>(ctx, a, n);
    else if (in->dv <= 64) launch_step<16>(ctx, a, n);
    else launch_step<32>(ctx, a, n);
    return q8i_launch_check(ctx, "delta step");
}

// -------------------------------------------------------------------------------- sequences ----

// In chunks of C = 32 tokens.  With c_i = g_1 + .. + g_i inside a chunk, D_ij = exp(c_i - c_j), A_ij = b_i D_ij (k_i k_j) for j < i and
// T = (I + A)^-1 diag(b):  U = T (V - exp(c) K S),  O = exp(c) Q S + (D_ij q_i k_j, j <= i) U,  S' = exp(c_C) S + (exp(c_C - c_j) k_j)^T U.
// A first launch forms T and the masked products of queries and keys of all chunks side by side, a second one carries the states
// from chunk to chunk, a block per sequence, head and 32 columns of the state.
#define DELTA_C Q8_DELTA_C
#define DELTA_MATRIX (DELTA_C * DELTA_C)
// What the first launch leaves of a chunk and head, in floats: T, M, then per token (6 x 32) exp(c) / |k|, exp(c) scale / |q| and exp(c_C - c) / |k|, each
// times the power of two of its row, the inverses of those powers of the key's and the query's row, and exp(c_C)
#define DELTA_ROOM (2 * DELTA_MATRIX + 6 * DELTA_C)

struct DeltaSeqArgs {
    q8_delta_inputs in;
    const int *off;
    int S, L, slots;                 // chunk c of sequence s has place off[s] / 32 + s + c: no two the same, all below L / 32 + S
    float *room;
    const float *state;
    float *state_out, *out;
    int ldo, vec_qk, vec;            // vec_qk: rows of queries and keys in whole 16-byte pieces, vec: those of values and results too
    int seg, segs;                   // 0: a block carries a whole sequence; else segments of `seg` chunks, places of segments (as those of chunks)
    float *ends, *moves;             // per place and head: the state that a segment ends with [dk x dv], and what it makes of a state [dk x dk]
};

__device__ __forceinline__ int delta_first(const DeltaSeqArgs &a, int s) { return min(max(a.off[s], 0), a.L); }

// tokens of a sequence: offsets that are out of order or out of range give none or fewer
__device__ __forceinline__ int delta_length(const DeltaSeqArgs &a, int s, int first) { return max(min(max(a.off[s + 1], 0), a.L) - first, 0); }

// Four numbers at `at`, or zeros past the end.  Loads under no condition: the compiler waits for everything in flight where a load stands in a branch.
// In single words the row's end is looked at for each (`left` numbers are the row's).
template <bool VEC>
__device__ __forceinline__ v4f fetch4(__amdgpu_buffer_rsrc_t rsrc, unsigned at, int left)
{
    v4f v;
    if constexpr (VEC) {
        v = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)at, 0, 0));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)(left > e && at < Q8_OOB ? at + 4 * e : Q8_OOB), 0, 0));
    }
    return v;
}

// A block per chunk and head.  The waves form tiles of 16 x 16 of both products (the upper right ones are zero) from rows that they load as the
// matrix operation takes them, the last the sums of the decays too; then (I + A)^-1 by substitution in blocks of 8, joined as
// -T22 A21 T11 twice.  (Powers of A instead of substitution would cancel: 32 keys alike give binomials up to 3e8.)  A row takes nothing from later tokens' rows,
// not even times the zeros above the diagonal: these may be infinite or no numbers.
// 8 x 1024 tokens of 16 heads of 128 x 128 in 51 us (median of 20 launches; the least 48): 134 MB of keys and queries read, 37 left, 3.3 TB/s; by waiting (half of the
// waves' time) for loads that all blocks of a round ask for at once.  Least times: from rows staged in LDS, with the substitution in blocks of 16, 73; the products in
// three waves 51.
template <int DKT, bool VEC>         // dk in units of 32, rounded up; VEC: rows of queries and keys in whole 16-byte pieces
__global__ __launch_bounds__(256) void delta_chunk_kernel(DeltaSeqArgs a)
{
    constexpr int PT = DELTA_C + 4, PX = 20, STEPS = 2 * DKT < 8 ? 2 * DKT : 8;
    __shared__ __align__(16) float sA[DELTA_C * PT], sT[DELTA_C * PT], sX[16 * PX], s_rk[DELTA_C], s_rq[DELTA_C], s_mk[DELTA_C], s_mq[DELTA_C], s_b[DELTA_C];
    __shared__ double s_c[DELTA_C];
    __shared__ int s_at[2];
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, gq = lane >> 4;
    const int head = blockIdx.x % p.hv, slot = blockIdx.x / p.hv, kh = head / (p.hv / p.hk);
    if (tid == 0) s_at[1] = 0;
    for (int x = tid; x < DELTA_C * PT; x += 256) sT[x] = 0.0f;
    __syncthreads();
    for (int s = tid; s < a.S; s += 256) {                                  // the sequence that has this place, if any
        const int first = delta_first(a, s), t0 = (slot - (first / DELTA_C + s)) * DELTA_C, left = delta_length(a, s, first) - t0;
        if (t0 >= 0 && left > 0) {
            s_at[0] = first + t0;
            s_at[1] = min(DELTA_C, left);
        }
    }
    __syncthreads();
    const size_t tok = (size_t)s_at[0];
    const int m = s_at[1] > 0 ? min(s_at[1], a.L - s_at[0]) : 0;
    if (m <= 0) return;                                                     // (a place that no chunk has)

    // wave 0: keys x keys and queries x keys of the first 16 tokens, 1: of the last, 2: keys of the last x keys of the first, 3: queries of the last x those
    v4f akk = {0.0f, 0.0f, 0.0f, 0.0f}, azk = akk;
    const int mt = wave > 0, nt = wave == 1, r = 16 * nt + i, rz = 16 * mt + i;
    {
        // (rows past the chunk's end lie past the end of what is described; its rows are below 2^31 bytes: pitches are at most 2^22)
        const bool keys = wave == 2;
        const int ldz = keys ? p.ldk : p.ldq;
        const __amdgpu_buffer_rsrc_t rk = q8_rsrc(p.k + tok * p.ldk + (size_t)kh * p.dk, 4 * ((size_t)(m - 1) * p.ldk + p.dk));
        const __amdgpu_buffer_rsrc_t rs = q8_rsrc((keys ? p.k : p.q) + tok * ldz + (size_t)kh * p.dk, 4 * ((size_t)(m - 1) * ldz + p.dk));
        const unsigned k = r < m ? 4u * ((unsigned)r * (unsigned)p.ldk + 4 * gq) : Q8_OOB, z0 = rz < m ? 4u * ((unsigned)rz * (unsigned)ldz + 4 * gq) : Q8_OOB;
        float kk = 0.0f, qq = 0.0f, mk = 0.0f, mq = 0.0f;
        for (int t0 = 0; t0 < 2 * DKT; t0 += STEPS) {
            v4f x[STEPS], z[STEPS];
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                const int left = p.dk - 16 * (t0 + t) - 4 * gq;
                const unsigned at = left > 0 ? 64u * (t0 + t) : Q8_OOB;
                x[t] = fetch4<VEC>(rk, max(k, at) < Q8_OOB ? k + at : Q8_OOB, left);
                z[t] = fetch4<VEC>(rs, max(z0, at) < Q8_OOB ? z0 + at : Q8_OOB, left);
            }
#pragma unroll
            for (int t = 0; t < STEPS; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) azk = __builtin_amdgcn_mfma_f32_16x16x4f32(z[t][e], x[t][e], azk, 0, 0, 0);
            if (wave < 2) {
#pragma unroll
                for (int t = 0; t < STEPS; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        akk = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t][e], x[t][e], akk, 0, 0, 0);
                        kk = fmaf(x[t][e], x[t][e], kk);
                        qq = fmaf(z[t][e], z[t][e], qq);
                        mk = fmaxf(mk, fabsf(x[t][e]));
                        mq = fmaxf(mq, fabsf(z[t][e]));
                    }
            }
        }
        if (wave < 2) {                                                     // each row once
#pragma unroll
            for (int x = 16; x < 64; x *= 2) {
                kk += __shfl_xor(kk, x);
                qq += __shfl_xor(qq, x);
                mk = fmaxf(mk, __shfl_xor(mk, x));
                mq = fmaxf(mq, __shfl_xor(mq, x));
            }
            if (gq == 0) {
                s_rk[r] = p.normalize ? unit_of(kk) : 1.0f;
                s_rq[r] = (p.normalize ? unit_of(qq) : 1.0f) * p.scale;
                s_mk[r] = mk;
                s_mq[r] = mq;
            }
        }
    }
    if (wave == 3) {
        const int t = lane & 31;
        const float g = t < m ? p.g[(tok + t) * p.ldg + head] : 0.0f;
        double c = g < (float)DELTA_LEAST ? DELTA_LEAST : (double)g;
        for (int x = 1; x < 32; x *= 2) {
            const double d = __shfl_up(c, x, 32);
            if (t >= x) c += d;
        }
        if (lane < DELTA_C) {
            s_c[t] = c;
            s_b[t] = t < m ? p.beta[(tok + t) * p.ldb + head] : 0.0f;
        }
    }
    __syncthreads();
    float *room = a.room + ((size_t)slot * p.hv + head) * DELTA_ROOM;
    {                                                                       // lane (i, gq): column i, rows 4 gq + e of a tile
        const int col = 16 * nt + i;
        if (wave == 2) akk = azk;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = 16 * mt + 4 * gq + e;
            const float d = row >= col ? expf((float)(s_c[row] - s_c[col])) * s_rk[col] : 0.0f;
            if (wave < 3) sA[row * PT + col] = row > col ? s_b[row] * s_rk[row] * d * akk[e] : 0.0f;
            if (wave != 2) room[DELTA_MATRIX + row * DELTA_C + col] = row >= col ? s_rq[row] * d * azk[e] : 0.0f;
        }
    }
    if (wave == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) room[DELTA_MATRIX + (4 * gq + e) * DELTA_C + 16 + i] = 0.0f;
        if (lane < DELTA_C) {
            float *v = room + 2 * DELTA_MATRIX, ik, iq;
            const float ek = parts_scale(s_mk[lane], ik), eq = parts_scale(s_mq[lane], iq), e = expf((float)s_c[lane]);
            v[lane] = e * s_rk[lane] * ek;
            v[DELTA_C + lane] = e * s_rq[lane] * eq;
            // (a key of zeros: no power of two of its own, so its update, which counts for nothing, must not be what a column's scale goes by)
            v[2 * DELTA_C + lane] = ik > 0.0f ? expf((float)(s_c[DELTA_C - 1] - s_c[lane])) * s_rk[lane] * ek : 0.0f;
            v[3 * DELTA_C + lane] = ik;
            v[4 * DELTA_C + lane] = iq;
            v[5 * DELTA_C + lane] = expf((float)s_c[DELTA_C - 1]);
        }
    }
    __syncthreads();
    if (tid < DELTA_C) {                                                    // the diagonal blocks of 8, a lane per column
        const int base = tid & 24, jc = tid & 7;
        v4f w[8][2];
#pragma unroll
        for (int r = 1; r < 8; ++r) {
            w[r][0] = *(const v4f *)(sA + (base + r) * PT + base);
            w[r][1] = *(const v4f *)(sA + (base + r) * PT + base + 4);
        }
        float x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float v = r == jc ? 1.0f : 0.0f;
#pragma unroll
            for (int l = 0; l < r; ++l) v = fmaf(-w[r][l >> 2][l & 3], x[l], v);
            x[r] = v;
            sT[(base + r) * PT + base + jc] = v;
        }
    }
    __syncthreads();
    {
        const int b = 16 * (tid >> 6), r = (tid >> 3) & 7, c = tid & 7;     // two blocks of 16
        float v = 0.0f;
        if (tid < 128) {
#pragma unroll
            for (int l = 0; l < 8; ++l) v = fmaf(sA[(b + 8 + r) * PT + b + l], sT[(b + l) * PT + b + c], v);
            sX[(b / 2 + r) * PX + c] = v;
        }
        __syncthreads();
        if (tid < 128) {
            v = 0.0f;
#pragma unroll
            for (int l = 0; l < 8; ++l) v = fmaf(sT[(b + 8 + r) * PT + b + 8 + l], sX[(b / 2 + min(l, r)) * PX + c], v);
            sT[(b + 8 + r) * PT + b + c] = -v;
        }
    }
    __syncthreads();
    {
        const int r = tid >> 4, c = tid & 15;
        float v = 0.0f;
#pragma unroll
        for (int l = 0; l < 16; ++l) v = fmaf(sA[(16 + r) * PT + l], sT[l * PT + c], v);
        sX[r * PX + c] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int l = 0; l < 16; ++l) v = fmaf(sT[(16 + r) * PT + 16 + l], sX[min(l, r) * PX + c], v);
        sT[(16 + r) * PT + c] = -v;
    }
    __syncthreads();
    {
        const int r = tid >> 3, c = 4 * (tid & 7);
        v4f t = *(const v4f *)(sT + r * PT + c) * *(const v4f *)(s_b + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = c + e <= r ? t[e] : 0.0f;
        *(v4f *)(room + r * DELTA_C + c) = t;
    }
}

// Sixteen lanes that point at four numbers each, sixteen of four rows (row l / 4 in lane l), transposed: a lane's number of the four rows.
__device__ __forceinline__ v4h read_transposed(const _Float16 *at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __fp16 v4fp __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(v4h, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) v4fp *)at));
#else
    return v4h();
#endif
}

__device__ __forceinline__ v8h both(v4h a, v4h b) { return (v8h){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// Where number k of a row of fp16 parts lies: a row's pieces of 16 bytes are exchanged by its number, so that sixteen rows' same piece, and four rows' same
// two pieces, lie on different banks.
template <int DKT>
__device__ __forceinline__ int delta_place(int row, int k)
{
    return row * 32 * DKT + 8 * ((k >> 3) ^ (DKT >= 4 ? row & 15 : (row >> 1) & 7)) + (k & 7);
}

// Bytes of LDS for the state's parts, and for the updates later.
template <bool MOVES> constexpr size_t delta_state_bytes(int dkt)
{
    const size_t parts = (size_t)2 * (MOVES ? 64 : 32) * 32 * dkt * 2, updates = (size_t)2 * 32 * (DELTA_C + 4) * 4;
    return parts > updates ? parts : updates;
}

// A block per sequence, head and 32 columns of the state, which stays in registers as fp32.  Its products run on the fp16 matrix cores with both sides in two
// parts (hi hi + hi lo + lo hi, within 2^-21): rows of keys and queries with a power of two each, columns of the state and of the updates too, so
// that what a column loses goes by its own size.  The two small products, of 32 x 32 with T and M, are fp32 ones.  Four waves multiply the
// keys and make the updates, four multiply the queries and make the results; all convert, and all keep an eighth of the state.  The next chunk's rows are on
// their way while one is worked on, each number in one thread's load and from there in LDS: loads of what several lanes need each cost the most here.
// 2.5 us a chunk of 32 tokens for a block alone, 4.2 for the two of a compute unit (8 x 1024 tokens of 16 heads of 128 x 128 in 133 us, median of 20 launches; the least
// 129): no unit is at its limit (vector instructions 45 %, LDS 51 %, of which a sixth conflicts, matrix cores 26 %), a chunk is a chain of four barriers.  Least times: fp32 matrix operations in four waves 197 us, parts in eight waves 157, 22 loads a wave
// turned into 8 140, rows' pieces exchanged in LDS in place of padded 127.  (Registers are bounded to 128, so that two blocks are resident.)
// SEGMENTS: in place of a sequence a block carries a part of it (below).  MOVES: no queries and no results; 64 columns, so that all eight waves multiply the keys
// (16384 tokens 248 us; 32 columns in four of the waves 320).
template <int DKT, bool VEC, bool SEGMENTS, bool MOVES>      // VEC: rows of queries, keys, values and results in whole 16-byte pieces
__global__ __launch_bounds__(512, DKT <= 4 ? 4 : 2) void delta_carry_kernel(DeltaSeqArgs a)
{
    constexpr int DKP = 32 * DKT, PART = DELTA_C * DKP, PT = DELTA_C + 4, OWN = DKT / 2;      // of a thread: pieces of four numbers of the keys and of the queries
    // columns; row tiles of the state between two of a wave, a wave's row tiles; the state's parts; the pitch of values
    constexpr int COLS = MOVES ? 64 : 32, STRIDE = MOVES ? 2 : 4, TILES = 2 * DKT / STRIDE, STATE = COLS * DKP, PV = COLS + 4;
    static_assert(DKT % 2 == 0, "eight waves share the state's tiles");
    extern __shared__ __align__(16) uint8_t s_all[];
    _Float16 *sK = (_Float16 *)s_all, *sQ = sK + 2 * PART, *sS = MOVES ? sQ : sQ + 2 * PART;      // [hi, lo][token or column][row of the state]
    float *sR = (float *)((uint8_t *)sS + delta_state_bytes<MOVES>(DKT)), *sM = sR + COLS * PT, *sV = sM + (MOVES ? 1 : 2) * 32 * PT, *s_vec = sV + 32 * PV, *s_top = s_vec + 6 * DELTA_C, *s_wtop = s_top + 128;
    float *sU = (float *)sS, *sW = MOVES ? sU : sU + 32 * PT;               // (the state's parts have been read by then) sR, sU, sW [column][token], sM [T, M][token][token], sV values and results [token][column]
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, gq = lane >> 4, mt = wave & 1, half = wave >> 2, nt = ((wave >> 1) & 1) + (MOVES ? 2 * half : 0), queries = MOVES ? 0 : half;
    const int head = blockIdx.x % p.hv, place = blockIdx.x / p.hv, kh = head / (p.hv / p.hk), lc = 16 * nt + i;
    int s = place, segment = 0, final = 0, first, length;
    bool last = true;
    if constexpr (SEGMENTS) {
        int *s_at = (int *)s_all;
        if (tid == 0) s_at[0] = -1;
        __syncthreads();
        for (int x = tid; x < a.S; x += 512) {                              // the sequence that has this place, if any (one without tokens has one)
            const int f = delta_first(a, x), g = place - (f / (DELTA_C * a.seg) + x);
            if (g >= 0 && g <= max(delta_length(a, x, f) - 1, 0) / (DELTA_C * a.seg)) s_at[0] = x;
        }
        __syncthreads();
        s = __builtin_amdgcn_readfirstlane(s_at[0]);
        if (s < 0) return;
        __syncthreads();
        first = __builtin_amdgcn_readfirstlane(delta_first(a, s));
        length = __builtin_amdgcn_readfirstlane(delta_length(a, s, first));
        segment = place - (first / (DELTA_C * a.seg) + s);
        final = max(length - 1, 0) / (DELTA_C * a.seg);
        last = segment >= final;
        first += segment * DELTA_C * a.seg;
        length = min(length - segment * DELTA_C * a.seg, DELTA_C * a.seg);
    } else {
        first = __builtin_amdgcn_readfirstlane(delta_first(a, s));
        length = __builtin_amdgcn_readfirstlane(delta_length(a, s, first));
    }
    // MOVES: columns of the state from zeros (a sequence's first segment: from its state), then those of what the segment makes of any state, from the
    // unit vectors and without values; neither is asked of a sequence's last segment, which puts the state where its end would be: the first segment starts
    // from there later, as the last one may leave the new state over the old one before the first has read it
    const int slices = (p.dv + COLS - 1) / COLS;
    const bool unit = MOVES && (int)blockIdx.y >= slices;
    if (MOVES && (segment == 0 ? last || unit : last && unit)) return;
    if (MOVES && last) length = 0;
    const int v0 = COLS * ((int)blockIdx.y - (unit ? slices : 0)), col = v0 + lc, dv = unit ? p.dk : p.dv;
    const bool live = col < dv;
    const int tile0 = MOVES ? mt : 2 * half + mt, r0 = 16 * mt + 4 * gq;
    // rows 16 (STRIDE t + tile0) + 4 gq + e of column `col` of the state
    v4f st[TILES];
    const size_t bytes = 4 * (size_t)p.dk * dv, mine = ((size_t)s * p.hv + head) * p.dk * p.dv, there = ((size_t)place * p.hv + head) * p.dk * dv;
    auto state_at = [&](int t, int e) {
        const int row = 16 * (STRIDE * t + tile0) + 4 * gq + e;
        return (int)(live && row < p.dk ? 4u * ((unsigned)row * (unsigned)dv + col) : Q8_OOB);
    };
    if (unit) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) st[t][e] = 16 * (STRIDE * t + tile0) + 4 * gq + e == col ? 1.0f : 0.0f;
    } else {                                                                // (a later segment's state is where the one before ends; none: zeros)
        const ptrdiff_t one = (ptrdiff_t)p.hv * p.dk * p.dv;
        const bool given = MOVES ? segment == 0 || last : segment == 0 && last;
        const float *from = given ? a.state + mine : a.ends + there + (segment == 0 ? final * one : -one);
        const __amdgpu_buffer_rsrc_t rs = q8_rsrc(from, (given ? a.state != nullptr : !MOVES) ? bytes : 0);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) st[t][e] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, state_at(t, e), 0, 0));
    }
    // a thread's pieces: of keys and queries, of T and M, of values and results (half of the threads), of the tokens' numbers (48 threads); offsets
    // inside a chunk: rows past its end lie past the end of what is described
    unsigned ok[OWN], oq[OWN];
#pragma unroll
    for (int x = 0; x < OWN; ++x) {
        const int y = tid + 512 * x, r = y / (DKP / 4), k = 4 * (y % (DKP / 4));
        ok[x] = k < p.dk ? 4u * ((unsigned)r * (unsigned)p.ldk + k) : Q8_OOB;
        oq[x] = k < p.dk ? 4u * ((unsigned)r * (unsigned)p.ldq + k) : Q8_OOB;
    }
    const bool values = MOVES || tid < 256;
    const int vr = MOVES ? tid >> 4 : (tid & 255) >> 3, vc = 4 * (tid & (COLS / 4 - 1)), vleft = values && !unit ? p.dv - v0 - vc : 0;
    const unsigned ov = vleft > 0 ? 4u * ((unsigned)vr * (unsigned)p.ldv + v0 + vc) : Q8_OOB, oo = vleft > 0 ? 4u * ((unsigned)vr * (unsigned)a.ldo + v0 + vc) : Q8_OOB;
    const unsigned oe = tid < 48 ? 4u * (2 * DELTA_MATRIX + 4 * tid) : Q8_OOB;
    v4f pk[OWN], pq[OWN], pm, pv, pe;
    auto fetch = [&](int t0) {
        const int m = min(DELTA_C, length - t0);
        const size_t tok = (size_t)first + t0;
        // (a chunk's rows are below 2^31 bytes: pitches are at most 2^22)
        const __amdgpu_buffer_rsrc_t rr = q8_rsrc(a.room + ((size_t)(first / DELTA_C + s + t0 / DELTA_C) * p.hv + head) * DELTA_ROOM, 4 * DELTA_ROOM);
        const __amdgpu_buffer_rsrc_t rk = q8_rsrc(p.k + tok * p.ldk + (size_t)kh * p.dk, 4 * ((size_t)(m - 1) * p.ldk + p.dk));
        const __amdgpu_buffer_rsrc_t rq = q8_rsrc(p.q + tok * p.ldq + (size_t)kh * p.dk, 4 * ((size_t)(m - 1) * p.ldq + p.dk));
        const __amdgpu_buffer_rsrc_t rv = q8_rsrc(p.v + tok * p.ldv + (size_t)head * p.dv, 4 * ((size_t)(m - 1) * p.ldv + p.dv));
        pe = fetch4<true>(rr, oe, 4);
#pragma unroll
        for (int x = 0; x < OWN; ++x) {
            const int left = p.dk - 4 * ((tid + 512 * x) % (DKP / 4));
            pk[x] = fetch4<VEC>(rk, ok[x], left);
            if constexpr (!MOVES) pq[x] = fetch4<VEC>(rq, oq[x], left);
        }
        pm = fetch4<true>(rr, !MOVES || tid < 256 ? 16u * tid : Q8_OOB, 4);
        pv = fetch4<VEC>(rv, ov, vleft);
    };
    // the largest of a column's numbers that this wave has
    auto leave_top = [&](float top, float *to) {
        top = fmaxf(top, __int_as_float(lane_xor_i<16>(__float_as_int(top), lane)));
        top = fmaxf(top, __int_as_float(lane_xor_i<32>(__float_as_int(top), lane)));
        if (gq == 0) to[lc] = top;
    };
    auto leave_state = [&] {                                                // ... and the next chunk's numbers of the tokens
        float top = 0.0f;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(st[t][e]));
        leave_top(top, s_top + COLS * tile0);
        if (tid < 48) *(v4f *)(s_vec + 4 * tid) = pe;
    };
    auto results = [&](int t0) {                                            // of the chunk at t0, from LDS
        const __amdgpu_buffer_rsrc_t ro = q8_rsrc(a.out + ((size_t)first + t0) * a.ldo + (size_t)head * p.dv, 4 * ((size_t)(min(DELTA_C, length - t0) - 1) * a.ldo + p.dv));
        const v4f o = *(const v4f *)(sV + vr * PV + vc);
        if constexpr (VEC) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, o), ro, (int)oo, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(o[e]), ro, (int)(vleft > e ? oo + 4 * e : Q8_OOB), 0, 0);
        }
    };
    if (length > 0) {
        fetch(0);
        leave_state();
        __syncthreads();
    }
    for (int t0 = 0; t0 < length; t0 += DELTA_C) {
        float inv;
        float top = fmaxf(s_top[lc], s_top[COLS + lc]);
        if constexpr (!MOVES) top = fmaxf(top, fmaxf(s_top[64 + lc], s_top[96 + lc]));
        const float cs = parts_scale(top, inv);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            uint2 hi, lo;
            parts4(st[t][0], st[t][1], st[t][2], st[t][3], inv, hi, lo);
            _Float16 *to = sS + delta_place<DKT>(lc, 16 * (STRIDE * t + tile0) + 4 * gq);
            *(uint2 *)to = hi;
            *(uint2 *)(to + STATE) = lo;
        }
#pragma unroll
        for (int x = 0; x < OWN; ++x) {
            const int y = tid + 512 * x, r = y / (DKP / 4), to = delta_place<DKT>(r, 4 * (y % (DKP / 4)));
            uint2 hi, lo;
            parts4(pk[x][0], pk[x][1], pk[x][2], pk[x][3], s_vec[3 * DELTA_C + r], hi, lo);
            *(uint2 *)(sK + to) = hi;
            *(uint2 *)(sK + PART + to) = lo;
            if constexpr (!MOVES) {
                parts4(pq[x][0], pq[x][1], pq[x][2], pq[x][3], s_vec[4 * DELTA_C + r], hi, lo);
                *(uint2 *)(sQ + to) = hi;
                *(uint2 *)(sQ + PART + to) = lo;
            }
        }
        if (!MOVES || tid < 256) *(v4f *)(sM + (tid >> 3) * PT + 4 * (tid & 7)) = pm;
        if (!MOVES && t0 > 0 && tid < 256) results(t0 - DELTA_C);                     // (a thread's piece of the results, then of the values, in one place)
        if (values) *(v4f *)(sV + vr * PV + vc) = pv;
        __syncthreads();
        if (t0 + DELTA_C < length) fetch(t0 + DELTA_C);
        const v4f eb = *(const v4f *)(s_vec + queries * DELTA_C + r0), el = *(const v4f *)(s_vec + 2 * DELTA_C + r0);
        const float keep = s_vec[5 * DELTA_C];
        v4f x0 = {0.0f, 0.0f, 0.0f, 0.0f}, x1 = x0, x2 = x0;                // keys or queries times the state
        const _Float16 *rows = queries ? sQ : sK;
#pragma unroll
        for (int t = 0; t < DKT; ++t) {
            const _Float16 *x = rows + delta_place<DKT>(16 * mt + i, 32 * t + 8 * gq), *y = sS + delta_place<DKT>(lc, 32 * t + 8 * gq);
            const v8h xh = *(const v8h *)x, xl = *(const v8h *)(x + PART), sh = *(const v8h *)y, sl = *(const v8h *)(y + STATE);
            x0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(xh, sh, x0, 0, 0, 0);
            x1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(xh, sl, x1, 0, 0, 0);
            x2 = __builtin_amdgcn_mfma_f32_16x16x32_f16(xl, sh, x2, 0, 0, 0);
        }
        // (times the power of two of the column before the rows' factors where it is below one, after them where it is above: nothing but the result passes fp32's range)
        const v4f xs = (x0 + (x1 + x2)) * fminf(cs, 1.0f) * eb * fmaxf(cs, 1.0f);
        // lane (i, gq): column i, tokens r0 + (0 .. 3)
        if (!queries) {
            v4f v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = sV[(r0 + e) * PV + lc];
            *(v4f *)(sR + lc * PT + r0) = v - xs;
        }
        __syncthreads();
        auto small = [&](const float *from, v4f o) {                        // T or M times a column, in two chains
            const float *m = sM + (32 * queries + 16 * mt + i) * PT + 4 * gq;
            const v4f m0 = *(const v4f *)m, m1 = *(const v4f *)(m + 16), y = *(const v4f *)(from + lc * PT + 4 * gq), z = *(const v4f *)(from + lc * PT + 16 + 4 * gq);
            v4f o2 = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o = __builtin_amdgcn_mfma_f32_16x16x4f32(m0[e], y[e], o, 0, 0, 0);
                o2 = __builtin_amdgcn_mfma_f32_16x16x4f32(m1[e], z[e], o2, 0, 0, 0);
            }
            return o + o2;
        };
        if (!queries) {
            const v4f u = small(sR, (v4f){0.0f, 0.0f, 0.0f, 0.0f});
            // the results take the updates, the state takes them times exp(c_C - c_j) / |k_j|
            const v4f w = u * el;
            if constexpr (!MOVES) *(v4f *)(sU + lc * PT + r0) = u;
            *(v4f *)(sW + lc * PT + r0) = w;
            leave_top(fmaxf(fmaxf(fabsf(w[0]), fabsf(w[1])), fmaxf(fabsf(w[2]), fabsf(w[3]))), s_wtop + COLS * mt);
        }
        __syncthreads();
        // tokens 8 gq + (0, 2, 4, 6, 1, 3, 5, 7) of column i: four rows of the keys that are read together lie two apart, on different banks
        const float cw = parts_scale(fmaxf(s_wtop[lc], s_wtop[COLS + lc]), inv);
        const v4f z0 = *(const v4f *)(sW + lc * PT + 8 * gq), z1 = *(const v4f *)(sW + lc * PT + 8 * gq + 4);
        union { uint2 u[2]; v8h h; } wh, wl;
        parts4(z0[0], z0[2], z1[0], z1[2], inv, wh.u[0], wl.u[0]);
        parts4(z0[1], z0[3], z1[1], z1[3], inv, wh.u[1], wl.u[1]);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int row = 8 * gq + 2 * (i >> 2), c = 16 * (STRIDE * t + tile0) + 4 * (i & 3);
            const _Float16 *k0 = sK + delta_place<DKT>(row, c), *k1 = sK + delta_place<DKT>(row + 1, c);
            const v8h kh_ = both(read_transposed(k0), read_transposed(k1));
            const v8h kl = both(read_transposed(k0 + PART), read_transposed(k1 + PART));
            v4f d = {0.0f, 0.0f, 0.0f, 0.0f};
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, wh.h, d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh_, wl.h, d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh_, wh.h, d, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) st[t][e] = fmaf(cw, d[e], keep * st[t][e]);
        }
        leave_state();
        if (!MOVES && queries) {
            v4f o = small(sU, xs);
            // A number of a column of R that is not finite is in all of the column's updates and results, and one of the updates in all results: in earlier rows
            // times the zeros above the diagonal.  The column's new state is not finite in truth either; the earlier results are formed again here, without what
            // comes after them.  (Looked at here alone, behind the chain from state to state: looked at in both products it cost 3 % of 16384 tokens.)
            if (__builtin_expect(!(fabsf(o[0]) < INFINITY), 0)) {
                int l = lane;                                               // (addresses formed here: kept from chunk to chunk they would cost registers)
                asm volatile("" : "+v"(l));
                const int r = 16 * mt + 4 * (l >> 4), at = (16 * nt + (l & 15)) * PT;
                const float *y = sR + at;
                int bad = 0;
                while (bad < DELTA_C && fabsf(y[bad]) < INFINITY) ++bad;
                if (bad == DELTA_C)
                    for (bad = 0; bad < DELTA_C && fabsf(sU[at + bad]) < INFINITY;) ++bad;
                if (bad > r && bad < DELTA_C) {                             // (of rows r .. r + 3 those from a bad one on are so again)
                    o = xs;
#pragma unroll 1
                    for (int j = 0; j < r + 4; ++j) {
                        float u = 0.0f;
#pragma unroll 1
                        for (int k = 0; k <= j; ++k) u = fmaf(sM[j * PT + k], y[k], u);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j <= r + e) o[e] = fmaf(sM[(32 + r + e) * PT + j], u, o[e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sV[(r0 + e) * PV + lc] = o[e];
        }
        __syncthreads();
    }
    if (!MOVES && length > 0 && tid < 256) results((length - 1) / DELTA_C * DELTA_C);
    float *to = MOVES ? (unit ? a.moves : a.ends) + there : a.state_out + mine;
    const __amdgpu_buffer_rsrc_t rs = q8_rsrc(to, MOVES || (last && a.state_out) ? bytes : 0);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(st[t][e]), rs, state_at(t, e), 0, 0);
}

// Few long sequences leave most of the device idle: a sequence's chunks come one after the other.  A segment of them makes F S + B of a state S, as the
// rule is linear in it: B is what it makes of zeros, F what it makes of the unit vectors without values.  These come from all segments side by side
// (MOVES), this kernel goes from segment to segment, ends[g] = F[g] ends[g - 1] + ends[g], and the results from all segments side by side again, each from
// the state that the one before ends with.  About 2.7 times the work: 16384 tokens of 16 heads of
// 128 x 128 in 580 us a call among others against 1373 in one go (one after the other under a profiler, medians: chunks 92, moves 248, this 30, results 261).  A block per sequence, head and 32 columns; products in fp32.
template <int DKT, bool VEC>         // VEC: dk in whole 16-byte pieces
__global__ __launch_bounds__(512) void delta_join_kernel(DeltaSeqArgs a)
{
    constexpr int DKP = 32 * DKT, P = DKP + 4, OWN = DKT / 2;
    __shared__ __align__(16) float sS[32 * P];                              // [column][row of the state]
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, gq = lane >> 4, nt = wave & 1, tile0 = wave >> 1;
    const int head = blockIdx.x % p.hv, s = blockIdx.x / p.hv, lc = 16 * nt + i, col = blockIdx.y * 32 + lc;
    const int first = __builtin_amdgcn_readfirstlane(delta_first(a, s)), length = __builtin_amdgcn_readfirstlane(delta_length(a, s, first));
    const int n = (length + DELTA_C * a.seg - 1) / (DELTA_C * a.seg), place = first / (DELTA_C * a.seg) + s;
    if (n < 3) return;
    const size_t size = (size_t)p.dk * p.dv, square = (size_t)p.dk * p.dk;
    auto at = [&](int t, int e) {
        const int row = 16 * (4 * t + tile0) + 4 * gq + e;
        return (int)(col < p.dv && row < p.dk ? 4u * ((unsigned)row * (unsigned)p.dv + col) : Q8_OOB);
    };
    v4f st[OWN], b[OWN], f[OWN][2 * DKT];
    auto fetch = [&](int g) {
        const __amdgpu_buffer_rsrc_t rb = q8_rsrc(a.ends + ((size_t)(place + g) * p.hv + head) * size, 4 * size);
        const __amdgpu_buffer_rsrc_t rf = q8_rsrc(a.moves + ((size_t)(place + g) * p.hv + head) * square, g > 0 ? 4 * square : 0);
#pragma unroll
        for (int t = 0; t < OWN; ++t) {
            const int row = 16 * (4 * t + tile0) + i;
#pragma unroll
            for (int k = 0; k < 2 * DKT; ++k) {
                const int c = 16 * k + 4 * gq;
                f[t][k] = fetch4<VEC>(rf, row < p.dk && c < p.dk ? 4u * (unsigned)(row * p.dk + c) : Q8_OOB, row < p.dk ? p.dk - c : 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) b[t][e] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(rb, at(t, e), 0, 0));
        }
    };
    fetch(0);
    for (int g = 0; g < n - 1; ++g) {                                       // (the last segment's end is nobody's start)
        if (g == 0) {
#pragma unroll
            for (int t = 0; t < OWN; ++t) st[t] = b[t];
        } else {
#pragma unroll
            for (int t = 0; t < OWN; ++t) {
                v4f x = b[t], y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 2 * DKT; ++k) {
                    const v4f z = *(const v4f *)(sS + lc * P + 16 * k + 4 * gq);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        x = __builtin_amdgcn_mfma_f32_16x16x4f32(f[t][k][e], z[e], x, 0, 0, 0);
                        y = __builtin_amdgcn_mfma_f32_16x16x4f32(f[t][k][e + 1], z[e + 1], y, 0, 0, 0);
                    }
                }
                st[t] = x + y;
            }
            const __amdgpu_buffer_rsrc_t rb = q8_rsrc(a.ends + ((size_t)(place + g) * p.hv + head) * size, 4 * size);
#pragma unroll
            for (int t = 0; t < OWN; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(st[t][e]), rb, at(t, e), 0, 0);
        }
        if (g + 2 >= n) break;
        fetch(g + 1);
        __syncthreads();                                                    // the state before has been read
#pragma unroll
        for (int t = 0; t < OWN; ++t) *(v4f *)(sS + lc * P + 16 * (4 * t + tile0) + 4 * gq) = st[t];
        __syncthreads();
    }
}

template <int DKT> static q8_status launch_sequence(q8_ctx *ctx, const DeltaSeqArgs &a)
{
    static Q8OncePerDevice once[6];
    constexpr size_t keys = 2 * 32 * 32 * DKT * sizeof(_Float16), whole = 2 * keys + delta_state_bytes<false>(DKT) + (4 * 32 * (DELTA_C + 4) + 6 * DELTA_C + 192) * sizeof(float),
                     move = keys + delta_state_bytes<true>(DKT) + (3 * 32 * (DELTA_C + 4) + 32 * 68 + 6 * DELTA_C + 256) * sizeof(float);
    auto carry = [&](void (*kernel)(DeltaSeqArgs), int form, int rows, int slices) {
        const size_t smem = form == 2 || form == 3 ? move : whole;
        const q8_status st = q8i_lds(ctx, once[form], (const void *)kernel, smem, "delta sequence");
        if (st) return st;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((size_t)rows * a.in.hv), slices), dim3(512), smem, ctx->stream, a);
        return q8i_launch_check(ctx, "delta sequence");
    };
    const int slices = (a.in.dv + 31) / 32;
    q8_status st;
    if (a.L > 0) {
        hipLaunchKernelGGL((a.vec_qk ? delta_chunk_kernel<DKT, true> : delta_chunk_kernel<DKT, false>), dim3((unsigned)((size_t)a.slots * a.in.hv)), dim3(256), 0, ctx->stream, a);
        if ((st = q8i_launch_check(ctx, "delta sequence"))) return st;
    }
    if (!a.seg) return a.vec ? carry(delta_carry_kernel<DKT, true, false, false>, 0, a.S, slices) : carry(delta_carry_kernel<DKT, false, false, false>, 1, a.S, slices);
    const int moves = (a.in.dv + 63) / 64 + (a.in.dk + 63) / 64;
    st = a.vec ? carry(delta_carry_kernel<DKT, true, true, true>, 2, a.segs, moves) : carry(delta_carry_kernel<DKT, false, true, true>, 3, a.segs, moves);
    if (st) return st;
    void (*const join)(DeltaSeqArgs) = a.in.dk % 4 == 0 ? delta_join_kernel<DKT, true> : delta_join_kernel<DKT, false>;
    hipLaunchKernelGGL(join, dim3((unsigned)((size_t)a.S * a.in.hv), slices), dim3(512), 0, ctx->stream, a);
    if ((st = q8i_launch_check(ctx, "delta sequence"))) return st;
    return a.vec ? carry(delta_carry_kernel<DKT, true, true, false>, 4, a.segs, slices) : carry(delta_carry_kernel<DKT, false, true, false>, 5, a.segs, slices);
}

static size_t delta_chunk_room(int L, int S, int hv) { return ((size_t)L / DELTA_C + S) * hv * DELTA_ROOM; }

// floats of the segments' ends and moves
static size_t delta_segment_room(int segs, int hv, int dk, int dv) { return (size_t)segs * hv * dk * ((size_t)dv + dk); }

static int delta_segments(int L, int S, int seg) { return L / (DELTA_C * seg) + S; }

size_t q8i_delta_room(int L, int S, int hv, int dk, int dv)
{
    const int seg = q8_delta_segment(L, S, hv, dk, dv);
    return (delta_chunk_room(L, S, hv) + (seg ? delta_segment_room(delta_segments(L, S, seg), hv, dk, dv) : 0)) * sizeof(float);
}

// ... of any call with up to L tokens and S sequences: fewer sequences may go in segments where S do not.  Segments are at most a part of the resident blocks for
// each sequence's heads and slices, and of four chunks at least, besides one for each sequence.
size_t q8i_delta_most_room(int L, int S, int hv, int dk, int dv)
{
    const int heads = hv * ((dv + 31) / 32);
    size_t room = delta_chunk_room(L, S, hv);
    if (heads <= Q8_DELTA_FEW && L >= 24 * DELTA_C) room += delta_segment_room(std::min(q8_delta_side(dk) / heads, L / (4 * DELTA_C)) + std::min(S, Q8_DELTA_FEW / heads), hv, dk, dv);
    return room * sizeof(float);
}

q8_status q8i_delta_sequence(q8_ctx *ctx, const q8_delta_inputs *in, int L, const int *off, int S, const float *state, float *state_out, float *out, int ldo, float *room)
{
    DeltaSeqArgs a = {*in, off, S, L, L / DELTA_C + S, room, state, state_out, out, ldo, 0, 0, q8_delta_segment(L, S, in->hv, in->dk, in->dv), 0, nullptr, nullptr};
    if (a.seg) {
        a.segs = delta_segments(L, S, a.seg);
        a.ends = room + delta_chunk_room(L, S, in->hv);
        a.moves = a.ends + (size_t)a.segs * in->hv * in->dk * in->dv;
    }
    a.vec_qk = in->dk % 4 == 0 && whole16(in->q, in->ldq) && whole16(in->k, in->ldk);
    a.vec = a.vec_qk && in->dv % 4 == 0 && whole16(in->v, in->ldv) && whole16(out, ldo);
    if (L <= 1) a.in.ldq = a.in.ldk = in->hk * in->dk, a.in.ldv = a.ldo = in->hv * in->dv;      // (a pitch that nothing uses, but bounds are formed with)
    if (in->dk <= 64) return launch_sequence<2>(ctx, a);
    if (in->dk <= 128) return launch_sequence<4>(ctx, a);
    return launch_sequence<8>(ctx, a);
}
