// q8_delta.hip -- the gated delta rule: per token and head S = a S, u = b (v - S^T k), S = S + k u^T, o = S^T q with a state S of
// dk x dv numbers; one token for n slots, and whole sequences laid end to end.
#include "q8_internal.h"

#include <math.h>

typedef float v4f __attribute__((ext_vector_type(4)));

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
// meet in LDS once.
template <int LPR, int R>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaStepArgs a)
{
    constexpr int GROUPS = 256 / LPR, WAVE_GROUPS = 64 / LPR > 0 ? 64 / LPR : 1;
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
#define DELTA_C 32
#define DELTA_ROOM (2 * DELTA_C * DELTA_C + 4 * DELTA_C)     // floats of a chunk and head: T, M, then exp(c) / |k|, exp(c) scale / |q|, exp(c_C - c) / |k|, exp(c_C)

struct DeltaSeqArgs {
    q8_delta_inputs in;
    const int *off;
    int S, L, slots;                 // chunk c of sequence s has place off[s] / 32 + s + c: no two the same, all below L / 32 + S
    float *room;
    const float *state;
    float *state_out, *out;
    int ldo, vec_qk, vec;
};

__device__ __forceinline__ int delta_first(const DeltaSeqArgs &a, int s) { return min(max(a.off[s], 0), a.L); }

// tokens of a sequence: offsets that are out of order or out of range give none or fewer
__device__ __forceinline__ int delta_length(const DeltaSeqArgs &a, int s, int first) { return max(min(max(a.off[s + 1], 0), a.L) - first, 0); }

template <int DKT>                   // dk in units of 32, rounded up
__global__ __launch_bounds__(256) void delta_chunk_kernel(DeltaSeqArgs a)
{
    constexpr int DKP = 32 * DKT, P = DKP + 4, PT = DELTA_C + 4;
    extern __shared__ __align__(16) float s_all[];
    float *sK = s_all, *sQ = sK + DELTA_C * P, *sA = sQ + DELTA_C * P, *sT = sA + DELTA_C * PT, *s_rk = sT + DELTA_C * PT, *s_rq = s_rk + DELTA_C, *s_b = s_rq + DELTA_C;
    double *s_c = (double *)(s_b + DELTA_C);
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, gq = lane >> 4;
    const int head = blockIdx.x % p.hv, slot = blockIdx.x / p.hv, kh = head / (p.hv / p.hk);
    // the last sequence whose places begin at or before this one
    int lo = 0, hi = a.S - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (delta_first(a, mid) / DELTA_C + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    const int first = delta_first(a, lo), length = delta_length(a, lo, first), t0 = (slot - (first / DELTA_C + lo)) * DELTA_C;
    if (t0 < 0 || t0 >= length) return;                                     // (a place that no chunk has)
    const int m = min(DELTA_C, length - t0);
    const size_t tok = (size_t)first + t0;
    for (int x = tid; x < DELTA_C * (DKP / 4); x += 256) {
        const int r = x / (DKP / 4), k = 4 * (x % (DKP / 4)), left = r < m ? p.dk - k : 0;
        *(v4f *)(sK + r * P + k) = load4(p.k + (tok + r) * p.ldk + (size_t)kh * p.dk + k, left, a.vec_qk);
        *(v4f *)(sQ + r * P + k) = load4(p.q + (tok + r) * p.ldq + (size_t)kh * p.dk + k, left, a.vec_qk);
    }
    if (tid < DELTA_C) {
        const float g = tid < m ? p.g[(tok + tid) * p.ldg + head] : 0.0f;
        s_c[tid] = g < (float)DELTA_LEAST ? DELTA_LEAST : (double)g;
        s_b[tid] = tid < m ? p.beta[(tok + tid) * p.ldb + head] : 0.0f;
    }
    __syncthreads();
    double c = 0.0;
    if (tid < DELTA_C)
        for (int t = 0; t <= tid; ++t) c += s_c[t];
    {
        const int r = tid >> 3, e0 = tid & 7;                               // eight threads a token
        float kk = 0.0f, qq = 0.0f;
        for (int k = 4 * e0; k < DKP; k += 32) {
            const v4f x = *(const v4f *)(sK + r * P + k), y = *(const v4f *)(sQ + r * P + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                kk = fmaf(x[e], x[e], kk);
                qq = fmaf(y[e], y[e], qq);
            }
        }
        for (int x = 1; x < 8; x *= 2) {
            kk += __shfl_xor(kk, x);
            qq += __shfl_xor(qq, x);
        }
        if (e0 == 0) {
            s_rk[r] = p.normalize ? unit_of(kk) : 1.0f;
            s_rq[r] = (p.normalize ? unit_of(qq) : 1.0f) * p.scale;
        }
    }
    __syncthreads();
    if (tid < DELTA_C) s_c[tid] = c;
    // products of 16 x 16 a wave: keys with keys and queries with keys
    const int mt = wave & 1, nt = wave >> 1;
    v4f akk = {0.0f, 0.0f, 0.0f, 0.0f}, aqk = akk;
    if (mt >= nt)
#pragma unroll
        for (int t = 0; t < DKP / 16; ++t) {
            const v4f x = *(const v4f *)(sK + (16 * mt + i) * P + 16 * t + 4 * gq), y = *(const v4f *)(sQ + (16 * mt + i) * P + 16 * t + 4 * gq);
            const v4f z = *(const v4f *)(sK + (16 * nt + i) * P + 16 * t + 4 * gq);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                akk = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], z[e], akk, 0, 0, 0);
                aqk = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], z[e], aqk, 0, 0, 0);
            }
        }
    __syncthreads();
    float *room = a.room + ((size_t)slot * p.hv + head) * DELTA_ROOM;
    const int col = 16 * nt + i;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = 16 * mt + 4 * gq + e;
        const float d = row >= col ? expf((float)(s_c[row] - s_c[col])) * s_rk[col] : 0.0f;
        sA[row * PT + col] = row > col ? s_b[row] * s_rk[row] * d * akk[e] : 0.0f;
        room[DELTA_C * DELTA_C + row * DELTA_C + col] = row >= col ? s_rq[row] * d * aqk[e] : 0.0f;
    }
    __syncthreads();
    // (I + A)^-1: the two diagonal blocks of 16 by substitution, a lane per column, then -T22 A21 T11
    if (tid < DELTA_C) {
        const int base = tid & 16, jc = tid & 15;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float v = r == jc ? 1.0f : 0.0f;
#pragma unroll
            for (int l = 0; l < r; ++l) v = fmaf(-sA[(base + r) * PT + base + l], x[l], v);
            x[r] = v;
            sT[(base + r) * PT + base + jc] = v;
        }
    }
    __syncthreads();
    {
        const int r = tid >> 4, cc = tid & 15;
        float v = 0.0f;
#pragma unroll
        for (int l = 0; l < 16; ++l) v = fmaf(sA[(16 + r) * PT + l], sT[l * PT + cc], v);
        sT[r * PT + 16 + cc] = v;                                           // (the upper right block holds it for now)
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int l = 0; l < 16; ++l) v = fmaf(sT[(16 + r) * PT + 16 + l], sT[l * PT + 16 + cc], v);
        sT[(16 + r) * PT + cc] = -v;
    }
    __syncthreads();
    for (int x = tid; x < DELTA_C * DELTA_C; x += 256) {
        const int r = x / DELTA_C, cc = x % DELTA_C;
        room[x] = r < 16 && cc >= 16 ? 0.0f : sT[r * PT + cc] * s_b[cc];
    }
    if (tid < DELTA_C) {
        float *v = room + 2 * DELTA_C * DELTA_C;
        const float e = expf((float)c);
        v[tid] = e * s_rk[tid];
        v[DELTA_C + tid] = e * s_rq[tid];
        v[2 * DELTA_C + tid] = expf((float)(s_c[DELTA_C - 1] - c)) * s_rk[tid];
        v[3 * DELTA_C + tid] = expf((float)s_c[DELTA_C - 1]);
    }
}

template <int DKT>
__global__ __launch_bounds__(256) void delta_carry_kernel(DeltaSeqArgs a)
{
    constexpr int DKP = 32 * DKT, P = DKP + 4, PT = DELTA_C + 4, PIECES = DELTA_C * (DKP / 4) / 256;
    extern __shared__ __align__(16) float s_all[];
    float *sK = s_all, *sQ = sK + DELTA_C * P, *sS = sQ + DELTA_C * P, *sR = sS + DELTA_C * P, *sU = sR + DELTA_C * PT;      // sS [column][row of the state], sR, sU [column][token]
    const q8_delta_inputs &p = a.in;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, gq = lane >> 4, mt = wave & 1, nt = wave >> 1;
    const int head = blockIdx.x % p.hv, s = blockIdx.x / p.hv, kh = head / (p.hv / p.hk), v0 = blockIdx.y * 32, col = v0 + 16 * nt + i;
    const int first = delta_first(a, s), length = delta_length(a, s, first);
    const bool live = col < p.dv;
    // rows 16 (2 t + mt) + 4 gq + e of column `col` of the state
    v4f st[DKT];
    const size_t at = ((size_t)s * p.hv + head) * p.dk * p.dv + col;
#pragma unroll
    for (int t = 0; t < DKT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = 16 * (2 * t + mt) + 4 * gq + e;
            st[t][e] = a.state && live && row < p.dk ? a.state[at + (size_t)row * p.dv] : 0.0f;
        }
    v4f pk[PIECES], pq[PIECES], pT[2], pM[2], pv, pe, pf, pd;
    float decay;
    auto fetch = [&](int t0) {
        const int m = min(DELTA_C, length - t0);
        const size_t tok = (size_t)first + t0;
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
            const int y = tid + 256 * x, r = y / (DKP / 4), k = 4 * (y % (DKP / 4)), left = r < m ? p.dk - k : 0;
            pk[x] = load4(p.k + (tok + r) * p.ldk + (size_t)kh * p.dk + k, left, a.vec_qk);
            pq[x] = load4(p.q + (tok + r) * p.ldq + (size_t)kh * p.dk + k, left, a.vec_qk);
        }
        const float *room = a.room + ((size_t)(first / DELTA_C + s + t0 / DELTA_C) * p.hv + head) * DELTA_ROOM;
        const float *vec = room + 2 * DELTA_C * DELTA_C;
        const int r0 = 16 * mt + 4 * gq;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            pT[t] = *(const v4f *)(room + (16 * mt + i) * DELTA_C + 16 * t + 4 * gq);
            pM[t] = *(const v4f *)(room + DELTA_C * DELTA_C + (16 * mt + i) * DELTA_C + 16 * t + 4 * gq);
        }
        pe = *(const v4f *)(vec + r0);
        pf = *(const v4f *)(vec + DELTA_C + r0);
        pd = *(const v4f *)(vec + 2 * DELTA_C + r0);
        decay = vec[3 * DELTA_C];
#pragma unroll
        for (int e = 0; e < 4; ++e) pv[e] = live && r0 + e < m ? p.v[(tok + r0 + e) * p.ldv + (size_t)head * p.dv + col] : 0.0f;
    };
    if (length > 0) fetch(0);
    for (int t0 = 0; t0 < length; t0 += DELTA_C) {
        const int m = min(DELTA_C, length - t0);
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
            const int y = tid + 256 * x, r = y / (DKP / 4), k = 4 * (y % (DKP / 4));
            *(v4f *)(sK + r * P + k) = pk[x];
            *(v4f *)(sQ + r * P + k) = pq[x];
        }
#pragma unroll
        for (int t = 0; t < DKT; ++t) *(v4f *)(sS + (16 * nt + i) * P + 16 * (2 * t + mt) + 4 * gq) = st[t];
        const v4f T[2] = {pT[0], pT[1]}, M[2] = {pM[0], pM[1]}, v = pv, ek = pe, eq = pf, el = pd;
        const float keep = decay;
        __syncthreads();
        if (t0 + DELTA_C < length) fetch(t0 + DELTA_C);
        v4f ks = {0.0f, 0.0f, 0.0f, 0.0f}, qs = ks;
#pragma unroll
        for (int t = 0; t < DKP / 16; ++t) {
            const v4f x = *(const v4f *)(sK + (16 * mt + i) * P + 16 * t + 4 * gq), y = *(const v4f *)(sQ + (16 * mt + i) * P + 16 * t + 4 * gq);
            const v4f z = *(const v4f *)(sS + (16 * nt + i) * P + 16 * t + 4 * gq);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ks = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], z[e], ks, 0, 0, 0);
                qs = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], z[e], qs, 0, 0, 0);
            }
        }
        // lane (i, gq): column i, tokens 16 mt + 4 gq + e
        *(v4f *)(sR + (16 * nt + i) * PT + 16 * mt + 4 * gq) = v - ek * ks;
        __syncthreads();
        v4f u = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v4f z = *(const v4f *)(sR + (16 * nt + i) * PT + 16 * t + 4 * gq);
#pragma unroll
            for (int e = 0; e < 4; ++e) u = __builtin_amdgcn_mfma_f32_16x16x4f32(T[t][e], z[e], u, 0, 0, 0);
        }
        // the state takes the updates times exp(c_C - c_j) / |k_j|, the results those themselves
        *(v4f *)(sU + (16 * nt + i) * PT + 16 * mt + 4 * gq) = u;
        __syncthreads();
        v4f *dst = (v4f *)(sR + (16 * nt + i) * PT + 16 * mt + 4 * gq);
        *dst = u * el;                                                      // (its readers are past the barrier)
        v4f o = eq * qs;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v4f z = *(const v4f *)(sU + (16 * nt + i) * PT + 16 * t + 4 * gq);
#pragma unroll
            for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(M[t][e], z[e], o, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 16 * mt + 4 * gq + e;
            if (live && r < m) a.out[((size_t)first + t0 + r) * a.ldo + (size_t)head * p.dv + col] = o[e];
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < DKT; ++t) st[t] *= keep;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v4f z = *(const v4f *)(sR + (16 * nt + i) * PT + 16 * t + 4 * gq);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int x = 0; x < DKT; ++x)
                    st[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(sK[(16 * t + 4 * gq + e) * P + 16 * (2 * x + mt) + i], z[e], st[x], 0, 0, 0);
        }
        __syncthreads();
    }
    if (a.state_out && live)
#pragma unroll
        for (int t = 0; t < DKT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * (2 * t + mt) + 4 * gq + e;
                if (row < p.dk) a.state_out[at + (size_t)row * p.dv] = st[t][e];
            }
}

template <int DKT> static q8_status launch_sequence(q8_ctx *ctx, const DeltaSeqArgs &a)
{
    static Q8OncePerDevice once[2];
    constexpr size_t row = (32 * DKT + 4) * sizeof(float), small = DELTA_C * (DELTA_C + 4) * sizeof(float);
    const size_t s1 = 2 * DELTA_C * row + 2 * small + 5 * DELTA_C * sizeof(float), s2 = 3 * DELTA_C * row + 2 * small;
    q8_status st = q8i_lds(ctx, once[0], (const void *)delta_chunk_kernel<DKT>, s1, "delta sequence");
    if (!st) st = q8i_lds(ctx, once[1], (const void *)delta_carry_kernel<DKT>, s2, "delta sequence");
    if (st) return st;
    if (a.L > 0) {
        hipLaunchKernelGGL(delta_chunk_kernel<DKT>, dim3((unsigned)((size_t)a.slots * a.in.hv)), dim3(256), s1, ctx->stream, a);
        st = q8i_launch_check(ctx, "delta sequence");
        if (st) return st;
    }
    hipLaunchKernelGGL(delta_carry_kernel<DKT>, dim3((unsigned)((size_t)a.S * a.in.hv), (a.in.dv + 31) / 32), dim3(256), s2, ctx->stream, a);
    return q8i_launch_check(ctx, "delta sequence");
}

size_t q8i_delta_room(int L, int S, int hv) { return ((size_t)L / DELTA_C + S) * hv * DELTA_ROOM * sizeof(float); }

q8_status q8i_delta_sequence(q8_ctx *ctx, const q8_delta_inputs *in, int L, const int *off, int S, const float *state, float *state_out, float *out, int ldo, float *room)
{
    DeltaSeqArgs a = {*in, off, S, L, L / DELTA_C + S, room, state, state_out, out, ldo, 0, 0};
    a.vec_qk = in->dk % 4 == 0 && whole16(in->q, in->ldq) && whole16(in->k, in->ldk);
    if (in->dk <= 32) return launch_sequence<1>(ctx, a);
    if (in->dk <= 64) return launch_sequence<2>(ctx, a);
    if (in->dk <= 128) return launch_sequence<4>(ctx, a);
    return launch_sequence<8>(ctx, a);
}
