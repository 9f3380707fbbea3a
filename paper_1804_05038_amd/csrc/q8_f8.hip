// q8_f8.hip -- 8-bit floating point with a scale per block: quantization of rows into e4m3 codes with one power of two per
// 128 columns, and the product of such codes, Y[j][i] = sum_b 2^(ew[i,b] + ex[j,b]) sum_{k in b} cw[i,k] cx[j,k] + bias[i].
#include "q8_internal.h"

#include <math.h>

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

#define F8_BLOCK 128                 // columns that share a scale

// ------------------------------------------------------------------------------ quantization ----

// The scale of a block whose largest finite magnitude is m: the smallest 2^e with m <= 448 * 2^e (448 = 1.75 * 2^8, the
// largest e4m3 value), from the bits of m; m < 2^-100: e = 0 and inv = 0, which makes every code 0.  Returns e + 127; inv = 2^-e.
__device__ __forceinline__ unsigned f8_scale_of(float m, float &inv)
{
    if (m < 0x1p-100f) { inv = 0.0f; return 127u; }
    const unsigned u = __float_as_uint(m);
    const unsigned e = (u >> 23) - 8u + ((u & 0x7fffffu) > 0x600000u ? 1u : 0u);
    inv = __uint_as_float((254u - e) << 23);
    return e;
}

__device__ __forceinline__ float f8_finite_abs(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; }

// Maximum over the 32 lanes of a half wave, in all of them.
__device__ __forceinline__ float f8_half_max(float v)
{
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_XOR1>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_XOR2>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_HALF_MIRROR>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_MIRROR>(__float_as_int(v))));
    return fmaxf(v, __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), SWZ_XOR16)));
}

// Four codes; the scaled values are at most 448 in magnitude or not finite (then the code is NaN).  The product with a power
// of two is exact, so the conversion's rounding (to nearest, ties to even) is the only one.  inv = 0: zeros without a sign.
__device__ __forceinline__ unsigned f8_codes4(float4 v, float inv)
{
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(v.x * inv, v.y * inv, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(v.z * inv, v.w * inv, p, true);
    return inv > 0.0f ? (unsigned)p : (unsigned)p & 0x7f7f7f7fu;
}

struct F8QuantArgs {
    const float *X;
    int rows, cols, ldx;
    uint8_t *codes;
    int ld;
    uint8_t *scale;
    int lds;
    int units_per_row;               // blocks of a row that have codes, pad bytes or a scale byte to write
    size_t units;
    int vec;                         // rows of X begin at 16-byte boundaries
};

#define F8_QUANT_PER_WAVE 8          // blocks that a wave takes, two at a time

// A half wave per block of 128 columns: four values a lane.  A wave asks for eight blocks before it waits.  Bound by memory:
// 50000 x 620 in 31.6 us, 4.9 TB/s read and written (a copy of 4 GiB: 4.8); 8 x 1024 in 4.3, a launch.
__global__ __launch_bounds__(256) void f8_quantize_kernel(F8QuantArgs a)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, i = lane & 31;
    const size_t wave = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const size_t u0 = wave * F8_QUANT_PER_WAVE;
    if (u0 >= a.units) return;
    size_t row = u0 / (unsigned)a.units_per_row;
    int b = (int)(u0 - row * (unsigned)a.units_per_row) + half;
    float4 v[F8_QUANT_PER_WAVE / 2];
    size_t rw[F8_QUANT_PER_WAVE / 2];
    int bl[F8_QUANT_PER_WAVE / 2];
#pragma unroll
    for (int t = 0; t < F8_QUANT_PER_WAVE / 2; ++t) {
        while (b >= a.units_per_row) { b -= a.units_per_row; ++row; }
        rw[t] = row;
        bl[t] = b;
        v[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const int k = b * F8_BLOCK + 4 * i;
        if (row < (size_t)a.rows && k < a.cols) {
            const float *x = a.X + row * (size_t)a.ldx + k;
            if (a.vec && k + 3 < a.cols) {
                v[t] = *(const float4 *)x;
            } else {
                v[t].x = x[0];
                if (k + 1 < a.cols) v[t].y = x[1];
                if (k + 2 < a.cols) v[t].z = x[2];
                if (k + 3 < a.cols) v[t].w = x[3];
            }
        }
        b += 2;
    }
#pragma unroll
    for (int t = 0; t < F8_QUANT_PER_WAVE / 2; ++t) {
        const float m = f8_half_max(fmaxf(fmaxf(f8_finite_abs(v[t].x), f8_finite_abs(v[t].y)), fmaxf(f8_finite_abs(v[t].z), f8_finite_abs(v[t].w))));
        float inv;
        const unsigned e = f8_scale_of(m, inv);
        const unsigned c = f8_codes4(v[t], inv);
        if (rw[t] < (size_t)a.rows) {
            const int k = bl[t] * F8_BLOCK + 4 * i;
            if (k < a.ld) *(unsigned *)(a.codes + rw[t] * (size_t)a.ld + k) = c;
            if (i == 0 && bl[t] < a.lds) a.scale[rw[t] * (size_t)a.lds + bl[t]] = (uint8_t)e;
        }
    }
}

q8_status q8i_quantize_f8(q8_ctx *ctx, const float *X, int rows, int cols, int ldx, uint8_t *codes, int ld, uint8_t *scale, int lds)
{
    F8QuantArgs a = {X, rows, cols, ldx, codes, ld, scale, lds, 0, 0, 0};
    const int nb = (ld + F8_BLOCK - 1) / F8_BLOCK;
    a.units_per_row = nb > lds ? nb : lds;
    a.units = (size_t)rows * a.units_per_row;
    a.vec = ldx % 4 == 0 && ((uintptr_t)X & 15) == 0;
    const size_t per_block = 4 * F8_QUANT_PER_WAVE, grid = (a.units + per_block - 1) / per_block;
    if (grid >= 1u << 24)                                                   // a launch has fewer than 2^32 threads
        return q8_fail(ctx, Q8_ERR_SHAPE, "quantize f8: %d rows of %d blocks are too many for a launch", rows, a.units_per_row);
    hipLaunchKernelGGL(f8_quantize_kernel, dim3((unsigned)grid), dim3(256), 0, ctx->stream, a);
    return q8i_launch_check(ctx, "quantize f8");
}

// ------------------------------------------------------------------------------- the product ----

struct F8GemmArgs {
    const uint8_t *W, *X;            // codes [rows x ldw], [n x ldx]
    const uint8_t *sw, *sx;          // scales [rows x ldsw], [n x ldsx]
    const float *bias;
    float *Y;
    int rows, n, cols, ldw, ldx, ldsw, ldsx, ldy;
    int row_tiles, col_tiles;
    unsigned magic, shift;
};

// The tile of a block.  Consecutive blocks run on different XCDs, each with an L2 cache of its own: each XCD gets a range of
// the tiles in a row, and these go through eight row tiles for each column tile, so that the tiles that run on an XCD at one
// time share rows and vectors.  (magic, shift: division by 8 col_tiles, see launch_f8.)
__device__ __forceinline__ void f8_tile_of(const F8GemmArgs &a, int &tr, int &tc)
{
    const unsigned block = blockIdx.x, total = gridDim.x, per = total / 8, over = total % 8, xcd = block % 8, idx = block / 8;
    const unsigned t = xcd * per + min(xcd, over) + idx, wide = 8u * (unsigned)a.col_tiles;
    const unsigned band = (unsigned)(((unsigned long long)t * a.magic) >> 32) >> a.shift, in = t - band * wide, height = (unsigned)a.row_tiles - 8u * band;
    if (height >= 8u) {
        tc = (int)(in >> 3);
        tr = (int)(8u * band + (in & 7u));
    } else {
        tc = (int)(in / height);
        tr = (int)(8u * band + in % height);
    }
}

// Sixteen codes times their block's scale as bf16, exactly: an e4m3 value has 4 significant bits, and the scale is a power of two.
__device__ __forceinline__ void f8_expand(v4i c, float s, v8bf &lo, v8bf &hi)
{
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        const v2bf p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[d], s, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[d], s, true);
        lo[4 * d] = p[0]; lo[4 * d + 1] = p[1]; lo[4 * d + 2] = q[0]; lo[4 * d + 3] = q[1];
        const v2bf r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 + d], s, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 + d], s, true);
        hi[4 * d] = r[0]; hi[4 * d + 1] = r[1]; hi[4 * d + 2] = t[0]; hi[4 * d + 3] = t[1];
    }
}

// Where a row's 16-byte pieces of a stage of 128 columns lie in LDS: exchanged by this number, so that the eight lanes that read
// together (eight rows) find theirs on different banks.
__device__ __forceinline__ int f8_twist(int row) { return row & 7; }

// Sixteen bytes a lane from memory to LDS at `at` + 16 lane (a wave's address), without passing through registers.
__device__ __forceinline__ void f8_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint8_t *at, unsigned offset, int step)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)at, 16, offset, step, 0, 0);
#endif
}

// Block of WM x WN waves, each with 32 TM rows x 32 TN vectors; stages of 128 columns go from memory to LDS without passing
// through registers, one on its way while the one before is multiplied.
// The codes are multiplied as bf16 values, because the matrix cores' own 8-bit floating point sums lose bits: products of a
// group are aligned to the largest and cut some 17 bits below it (two products of +-2^17.6 and 126 of 1 gave 120; Gaussian
// codes 1e-5 of the result in the 2-norm, bf16 3e-8).  They are converted on their way from LDS to the matrix cores: two codes
// an instruction, which the matrix cores' time covers (24 conversions beside 8 products of 32 x 32 x 16).  The order of k
// inside a block is the same for both operands, which is all that it has to be: lane half h takes the 16-byte pieces 2 j + h.
// KS > 1: KS such groups of waves take turns at the stages; their sums meet in LDS, in one order.
// 8192 x 8192 x 8192 in 850 to 875 us, 1.26 to 1.29 PFLOP/s (codes of zeros: 604, so that power bounds it; without results 826, without stages
// 749; the library's bf16 product of that size 1.20 PFLOP/s).  50000 x 512 x 1024 in 80 us: 205 MB of results, which alone take 50
// (4.1 TB/s), and products, which alone take 52, overlap in part.  As compiled every store waits for the one before: a wait for all memory
// operations, which the bias's load asks for, stands in front of each.
// PAST: the results go past the caches.
template <int WM, int WN, int TM, int TN, int KS, bool PAST>
__global__ __launch_bounds__(64 * WM * WN * KS) void f8_gemm_kernel(F8GemmArgs a)
{
    constexpr int ROWS = 32 * WM * TM, VECS = 32 * WN * TN, THREADS = 64 * WM * WN, STAGE = (ROWS + VECS) * F8_BLOCK;
    constexpr int LW = ROWS * 8 / THREADS, LX = VECS * 8 / THREADS;                    // 16-byte pieces a thread requests
    static_assert(ROWS * 8 % THREADS == 0 && VECS * 8 % THREADS == 0, "even shares of a stage");
    extern __shared__ __align__(16) uint8_t s_all[];                                   // [KS][2][STAGE]
    const int group = KS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS) : 0, tid = (int)threadIdx.x - group * THREADS;
    uint8_t *s_f8 = s_all + group * 2 * STAGE;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM, i = lane & 31, h = lane >> 5;
    int tr, tc;
    f8_tile_of(a, tr, tc);
    const int r0 = tr * ROWS, c0 = tc * VECS, steps = (a.cols + F8_BLOCK - 1) / F8_BLOCK, turns = (steps + KS - 1) / KS, kend = (a.cols + 15) & ~15;
    const int left_r = min(ROWS, a.rows - r0), left_c = min(VECS, a.n - c0);
    const __amdgpu_buffer_rsrc_t rw = q8_rsrc(a.W + (size_t)r0 * a.ldw, (size_t)left_r * a.ldw), rx = q8_rsrc(a.X + (size_t)c0 * a.ldx, (size_t)left_c * a.ldx);
    // piece p of a stage: row p / 8 (beyond the matrix: the last row again), the columns that the twist puts at place p % 8
    unsigned ow[LW], ox[LX];
#pragma unroll
    for (int u = 0; u < LW; ++u) {
        const int p = u * THREADS + tid, r = p >> 3;
        ow[u] = (unsigned)min(r, left_r - 1) * (unsigned)a.ldw + 16u * (unsigned)((p & 7) ^ f8_twist(r));
    }
#pragma unroll
    for (int u = 0; u < LX; ++u) {
        const int p = u * THREADS + tid, r = p >> 3;
        ox[u] = (unsigned)min(r, left_c - 1) * (unsigned)a.ldx + 16u * (unsigned)((p & 7) ^ f8_twist(r));
    }
    const int full = kend / F8_BLOCK;                                                  // stages that are all columns of the matrix
    auto request = [&](int step, int stage) {
        uint8_t *at = s_f8 + stage * STAGE + wave * 1024;
        if (step < full) {
#pragma unroll
            for (int u = 0; u < LW; ++u) f8_to_lds(rw, at + u * THREADS * 16, ow[u], step * F8_BLOCK);
#pragma unroll
            for (int u = 0; u < LX; ++u) f8_to_lds(rx, at + ROWS * F8_BLOCK + u * THREADS * 16, ox[u], step * F8_BLOCK);
        } else {                                                            // pieces past the columns: the row's first in their place
#pragma unroll
            for (int u = 0; u < LW; ++u) {
                const int p = u * THREADS + tid, c = 16 * ((p & 7) ^ f8_twist(p >> 3));
                f8_to_lds(rw, at + u * THREADS * 16, step * F8_BLOCK + c < kend ? ow[u] + step * F8_BLOCK : ow[u] - c, 0);
            }
#pragma unroll
            for (int u = 0; u < LX; ++u) {
                const int p = u * THREADS + tid, c = 16 * ((p & 7) ^ f8_twist(p >> 3));
                f8_to_lds(rx, at + ROWS * F8_BLOCK + u * THREADS * 16, step * F8_BLOCK + c < kend ? ox[u] + step * F8_BLOCK : ox[u] - c, 0);
            }
        }
    };
    // scales: four steps' bytes at a time
    const uint8_t *pw[TM], *px[TN];
#pragma unroll
    for (int t = 0; t < TM; ++t) pw[t] = a.sw + (size_t)min(r0 + 32 * (wm * TM + t) + i, a.rows - 1) * a.ldsw;
#pragma unroll
    for (int t = 0; t < TN; ++t) px[t] = a.sx + (size_t)min(c0 + 32 * (wn * TN + t) + i, a.n - 1) * a.ldsx;
    unsigned ew[TM], ex[TN];
    v16f acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][u][e] = 0.0f;
    const int lw = (32 * wm * TM + i) * F8_BLOCK, lx = ROWS * F8_BLOCK + (32 * wn * TN + i) * F8_BLOCK, twist = f8_twist(i);

    auto scales = [&](int step) {
#pragma unroll
        for (int t = 0; t < TM; ++t) ew[t] = *(const unsigned *)(pw[t] + (step & ~3));
#pragma unroll
        for (int t = 0; t < TN; ++t) ex[t] = *(const unsigned *)(px[t] + (step & ~3));
    };
    auto multiply = [&](int step, int stage) {
        const uint8_t *pw = s_f8 + stage * STAGE + lw, *px = s_f8 + stage * STAGE + lx;
        float fw[TM], fx[TN];
#pragma unroll
        for (int t = 0; t < TM; ++t) fw[t] = __uint_as_float(((ew[t] >> (8 * (step & 3))) & 255u) << 23);
#pragma unroll
        for (int t = 0; t < TN; ++t) fx[t] = __uint_as_float(((ex[t] >> (8 * (step & 3))) & 255u) << 23);
        v4i w[2][TM], x[2][TN];                                             // the next 32 columns are on their way while these are multiplied
        auto load = [&](int j) {
            const int piece = 16 * ((2 * j + h) ^ twist);
#pragma unroll
            for (int t = 0; t < TN; ++t) x[j & 1][t] = *(const v4i *)(px + t * 32 * F8_BLOCK + piece);
#pragma unroll
            for (int t = 0; t < TM; ++t) w[j & 1][t] = *(const v4i *)(pw + t * 32 * F8_BLOCK + piece);
        };
        load(0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j < 3) load(j + 1);
            __builtin_amdgcn_sched_barrier(0);
            v8bf xl[TN], xh[TN];
#pragma unroll
            for (int t = 0; t < TN; ++t) f8_expand(x[j & 1][t], fx[t], xl[t], xh[t]);
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                v8bf wl, wh;
                f8_expand(w[j & 1][t], fw[t], wl, wh);
#pragma unroll
                for (int u = 0; u < TN; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xl[u], wl, acc[t][u], 0, 0, 0);
#pragma unroll
                for (int u = 0; u < TN; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xh[u], wh, acc[t][u], 0, 0, 0);
            }
        }
    };
    if (group < steps) request(group, 0);
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
        const int step = turn * KS + group;
        if ((KS > 1 || (step & 3) == 0) && step < steps) scales(step);
        __syncthreads();                                                    // this turn's stages are there, the other ones are free
        if (step + KS < steps) request(step + KS, (turn + 1) & 1);
        if (turn == turns - 1 && full < steps) {                            // what lies past the columns counts as zeros
            if (step == full) {
#pragma unroll
                for (int u = 0; u < LW + LX; ++u) {
                    const int p = u * THREADS + tid;
                    if (step * F8_BLOCK + 16 * ((p & 7) ^ f8_twist(p >> 3)) >= kend) *(v4i *)(s_f8 + (turn & 1) * STAGE + 16 * p) = (v4i){0, 0, 0, 0};
                }
            }
            __syncthreads();
        }
        if (step < steps) multiply(step, turn & 1);
    }
    if constexpr (KS > 1) {
        // the groups' sums, one group's place per stage buffer: [wave][t][u][e][lane]
        static_assert(STAGE * 2 >= TM * TN * 16 * THREADS * 4, "a group's sums fit where its stages were");
        __syncthreads();
        float *mine = (float *)s_f8 + wave * TM * TN * 1024 + lane;
        if (group > 0) {
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int u = 0; u < TN; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) mine[((t * TN + u) * 16 + e) * 64] = acc[t][u][e];
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 1; g < KS; ++g) {
            const float *o = (const float *)(s_all + g * 2 * STAGE) + wave * TM * TN * 1024 + lane;
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int u = 0; u < TN; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[t][u][e] += o[((t * TN + u) * 16 + e) * 64];
        }
    }
    // lane (i, h): row i of each group, vectors 8 q + 4 h + (0 .. 3): 128 contiguous bytes of a vector a half wave.  Two groups of rows
    // trade halves: 64 rows of one vector, 256 contiguous bytes, a store.
    constexpr int PAIR = TM % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int t = 0; t < TM; t += PAIR) {
        const int row = r0 + 32 * (wm * TM + t) + (PAIR == 2 ? lane : i);
        const float b = a.bias && row < a.rows ? a.bias[row] : 0.0f;
#pragma unroll
        for (int u = 0; u < TN; ++u) {
            const int vec = c0 + 32 * (wn * TN + u) + (PAIR == 2 ? 0 : 4 * h);
            float *out = a.Y + (size_t)vec * a.ldy + row;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int v = 8 * (e >> 2) + (e & 3);
                float y[PAIR];
                if constexpr (PAIR == 2) {                                  // (by all lanes)
                    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_int(acc[t][u][e]), __float_as_int(acc[t + 1][u][e]), false, false);
                    y[0] = __int_as_float(p[0]);
                    y[1] = __int_as_float(p[1]);
                } else {
                    y[0] = acc[t][u][e];
                }
#pragma unroll
                for (int z = 0; z < PAIR; ++z) {
                    if (row >= a.rows || vec + v + 4 * z >= a.n) continue;
                    const float sum = a.bias ? y[z] + b : y[z];             // (y + 0 would turn -0 into 0)
                    if constexpr (PAST) __builtin_nontemporal_store(sum, &out[(size_t)(v + 4 * z) * a.ldy]);
                    else out[(size_t)(v + 4 * z) * a.ldy] = sum;
                }
            }
        }
    }
}

template <int WM, int WN, int TM, int TN, int KS = 1> static q8_status launch_f8(q8_ctx *ctx, F8GemmArgs &a)
{
    static Q8OncePerDevice once[2];
    const size_t smem = (size_t)KS * 2 * 32 * (WM * TM + WN * TN) * F8_BLOCK;
    a.row_tiles = (a.rows + 32 * WM * TM - 1) / (32 * WM * TM);
    a.col_tiles = (a.n + 32 * WN * TN - 1) / (32 * WN * TN);
    const size_t tiles = (size_t)a.row_tiles * a.col_tiles;
    // 50000 x 512 x 1024 77 against 92 us in the caches; but where blocks share the 64-byte pieces that memory takes, the caches put
    // them together: 6582 x 84 x 7068 43 us against 88 past them
    const bool past = a.ldy % 16 == 0 && ((uintptr_t)a.Y & 63) == 0;
    void (*const kernel)(F8GemmArgs) = past ? f8_gemm_kernel<WM, WN, TM, TN, KS, true> : f8_gemm_kernel<WM, WN, TM, TN, KS, false>;
    // t / d for t < 2^31 as (t magic / 2^32) / 2^shift: magic = ceil(2^(32 + shift) / d) with 2^shift < d <= 2^(shift + 1) is below 2^32, and
    // its excess over the quotient, less than 1, adds less than t / 2^(32 + shift) < 1 / d
    const unsigned long long d = 8ull * a.col_tiles;
    for (a.shift = 0; (2ull << a.shift) < d; ++a.shift) {}
    a.magic = (unsigned)(((1ull << (32 + a.shift)) + d - 1) / d);
    if (tiles * (64 * WM * WN * KS) > 0xffffffffu)                          // a launch has fewer than 2^32 threads
        return q8_fail(ctx, Q8_ERR_SHAPE, "f8 product: %d x %d results are too many for a launch", a.rows, a.n);
    const q8_status st = q8i_lds(ctx, once[past], (const void *)kernel, smem, "f8 product");
    if (st) return st;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(64 * WM * WN * KS), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product f8");
}

// Tiles by what each costs (us; rows x columns x vectors, the product alone): 256 x 256 and 128 x 128 where they are about one round of
// blocks or more, long enough that reading counts most, and the vectors fill them (8192 x 8192 x 8192 865, 986 and in 128 x 64 1146;
// 4096 x 1024 x 4096 43.3, 41.0 and 44.0; 50000 x 512 x 1024, four stages a tile, 110, 77.0 and 76.0); 128 x 32 for up to 32 vectors;
// 128 x 96 for 65 to 96 where they are one round (two blocks a compute unit) and the 128 x 64 ones, three a unit, are not, and longer than
// four stages (128 x 96, 128 x 64, 64 x 64 with 81 vectors: 47323 x 640 16.8, 14.7, 16.7; 50011 x 640 17.0, 17.0, 17.1; 63707 x 640 18.1,
// 19.6, 20.5; 67803 x 640 25.5, 20.3, 21.6; x 2048 31.8, 32.4, 35.8; 32.3, 38.6, 37.5; 34.6, 43.9, 44.8; 50.0, 47.0, 48.7; with 77 63644 x 256 11.9,
// 11.8, 12.1); 64 x 32 with four groups in turns at the stages where the others would leave compute units without any (1024 x 8192 x
// 64 22.9 against 35.1 in 64 x 64, 512 x 4096 x 17 10.2 against 17.2, 11807 x 1012 x 8 8.0 against 9.6 in 128 x 32); else 128 x 64 where
// these are more than a round, in eight waves (50000 x 640 x 320 35.0 against 39.7 in 64 x 64 and 39.1 in four waves), and 64 x 64
// (1024 x 2048 x 1024 11.9 against 14.3, 3117 x 4084 x 663 37.4 against 41.2).
static q8_status gemm_f8_tiles(q8_ctx *ctx, F8GemmArgs &a)
{
    auto tiles = [&](int r, int v) { return (long long)((a.rows + r - 1) / r) * ((a.n + v - 1) / v); };
    auto filled = [&](int v) { return (long long)((a.n + v - 1) / v) * v * 4 <= 5ll * a.n; };
    if (filled(256) && tiles(256, 256) >= 200 && a.cols >= 2048) return launch_f8<2, 4, 4, 2>(ctx, a);
    if (filled(128) && tiles(128, 128) >= 500 && a.cols >= 1024) return launch_f8<2, 4, 2, 1>(ctx, a);
    if (a.cols >= 512 && (a.n <= 32 ? tiles(128, 32) < 256 : tiles(64, 64) < 128)) return launch_f8<2, 1, 1, 1, 4>(ctx, a);
    if (a.n <= 32) return launch_f8<4, 1, 1, 1>(ctx, a);
    if (a.n > 64 && a.n <= 96 && a.cols > 512 && tiles(128, 96) <= 512 && tiles(128, 64) > 768) return launch_f8<4, 1, 1, 3>(ctx, a);
    if (tiles(128, 64) >= 320) return launch_f8<4, 2, 1, 1>(ctx, a);
    return launch_f8<2, 2, 1, 1>(ctx, a);
}

// ------------------------------------------------------------------------- few vectors ----

struct F8StreamArgs {
    F8GemmArgs g;
    const float *Xf;                 // the vectors in fp32 [n x ldxf], quantized here; or NULL: g.X, g.sx
    int ldxf, vec;                   // vec: the vectors begin at 16-byte boundaries
    int nb, pitch;                   // blocks of 128 columns; bytes of a vector in LDS
    int split, span;                 // waves for a row's columns, blocks of columns of each
};

// Up to 16 vectors: the weights go from memory to registers once, requested before anything else is waited for and again as
// soon as they are multiplied (as compiled into other registers, which are waited for and moved at a turn's end); the vectors lie in LDS as bf16 values, put there by every block for itself.  A wave multiplies 16
// rows at a time; `split` waves share them, each with its range of the columns.  Lane (i, g) has row i and of every 128 columns
// the 16-byte pieces g and g + 4.  Bound by the weights' way: 50000 x 512 x 5 in 8.9 us (26.9 MB, 3.0 TB/s; the kernel 8.0, of which
// a launch, the vectors' quantization and the last stores are some 3.5), 250000 x 1024 x 8 in 43 (5.9 TB/s; 52 with the weights out of
// every cache).
__global__ __launch_bounds__(512) void f8_stream_kernel(F8StreamArgs a)
{
    extern __shared__ __align__(16) uint8_t s_x[];                          // [n][pitch], then the waves' sums [waves][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, i = lane & 15, g = lane >> 4;
    const F8GemmArgs &m = a.g;
    const int split = a.split, part = wave & (split - 1), tiles = (m.rows + 15) >> 4, per = waves / split, stride = gridDim.x * per;
    const int kend = (m.cols + 15) & ~15, n = m.n, b0 = part * a.span, b1 = min(b0 + a.span, a.nb);
    int tile = blockIdx.x + gridDim.x * (wave / split), b = b0;
    __amdgpu_buffer_rsrc_t rw, rs;
    unsigned row_at, scale_at;
    float bias;
    auto rows_of = [&](int t) {                                             // no rows: every access past the end
        const int r0 = 16 * min(t, tiles - 1), left = t < tiles && b0 < b1 ? min(16, m.rows - r0) : 0;
        rw = q8_rsrc(m.W + (size_t)r0 * m.ldw, (size_t)left * m.ldw);
        rs = q8_rsrc(m.sw + (size_t)r0 * m.ldsw, (size_t)left * m.ldsw);
        row_at = i < left ? (unsigned)i * (unsigned)m.ldw + 16 * g : Q8_OOB;
        scale_at = i < left ? (unsigned)i * (unsigned)m.ldsw : Q8_OOB;
        bias = m.bias && i < left ? m.bias[r0 + i] : 0.0f;
    };
    v4i w[8];
    unsigned e;
    auto codes = [&](int s) {                                               // four blocks of columns, 64 columns each time
        const int k = (b + (s >> 1)) * F8_BLOCK + 64 * (s & 1);
        return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(b + (s >> 1) < b1 && k + 16 * g < kend && row_at != Q8_OOB ? row_at + k : Q8_OOB), 0, 0));
    };
    auto scale = [&] { return __builtin_amdgcn_raw_buffer_load_b32(rs, (int)(scale_at == Q8_OOB ? Q8_OOB : scale_at + b), 0, 0); };
    rows_of(tile);
#pragma unroll
    for (int s = 0; s < 8; ++s) w[s] = codes(s);
    e = scale();

    // ---- the vectors, a half wave per block of 128 columns, four values a lane
    const int q = lane & 31, units = n * a.nb, halves = 2 * waves;
    for (int u0 = tid >> 5; u0 < units; u0 += 2 * halves) {
        float4 v[2];
        unsigned c[2], se[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int u = u0 + halves * t, j = u / a.nb, k = (u - j * a.nb) * F8_BLOCK + 4 * q;
            v[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            c[t] = 0;
            se[t] = 127;
            if (u >= units) continue;
            if (a.Xf) {
                const float *x = a.Xf + (size_t)j * a.ldxf + k;
                if (k + 3 < m.cols) {
                    if (a.vec) v[t] = *(const float4 *)x;
                    else v[t] = make_float4(x[0], x[1], x[2], x[3]);
                } else {
                    if (k < m.cols) v[t].x = x[0];
                    if (k + 1 < m.cols) v[t].y = x[1];
                    if (k + 2 < m.cols) v[t].z = x[2];
                }
            } else {
                if (k < kend) c[t] = *(const unsigned *)(m.X + (size_t)j * m.ldx + k);
                se[t] = m.sx[(size_t)j * m.ldsx + u - j * a.nb];
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int u = u0 + halves * t, j = u / a.nb, k = (u - j * a.nb) * F8_BLOCK + 4 * q;
            if (u >= units) continue;                                       // (a half wave as one)
            if (a.Xf) {
                const float top = f8_half_max(fmaxf(fmaxf(f8_finite_abs(v[t].x), f8_finite_abs(v[t].y)), fmaxf(f8_finite_abs(v[t].z), f8_finite_abs(v[t].w))));
                float inv;
                se[t] = f8_scale_of(top, inv);
                c[t] = f8_codes4(v[t], inv);
            }
            const float s = __uint_as_float(se[t] << 23);
            union { v2bf h[2]; unsigned long long d; } p;
            p.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[t], s, false);
            p.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[t], s, true);
            *(unsigned long long *)(s_x + (size_t)j * a.pitch + 2 * k) = p.d;
        }
    }
    __syncthreads();

    v4f *s_sum = (v4f *)(s_x + (size_t)n * a.pitch);
    v4f acc[2];                                                             // two chains: a dependent matrix operation waits longer
    acc[0] = acc[1] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    const v8bf none = {};
    const uint8_t *px = s_x + (size_t)min(i, n - 1) * a.pitch + 32 * g;
    while (tile < tiles) {
        const int at = b, from = tile, left = max(b1 - at, 0);
        const unsigned es = left < 4 ? e & ((1u << 8 * left) - 1u) : e;     // (bytes past the columns: anything, 255 would make their zeros NaN)
        const float add = bias;
        b += 4;
        const bool last = b >= b1;
        if (last) {
            b = b0;
            tile += stride;
            rows_of(tile);
        }
        e = scale();
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            v8bf wl, wh, xl = none, xh = none;
            f8_expand(w[s], __uint_as_float(((es >> (8 * (s >> 1))) & 255u) << 23), wl, wh);
            w[s] = codes(s);
            if (i < n && at + (s >> 1) < b1) {
                const uint8_t *x = px + 2 * (at * F8_BLOCK + 64 * s);
                xl = *(const v8bf *)x;
                xh = *(const v8bf *)(x + 16);
            }
            acc[s & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xl, wl, acc[s & 1], 0, 0, 0);
            acc[s & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xh, wh, acc[s & 1], 0, 0, 0);
        }
        if (!last) continue;
        const v4f sum = acc[0] + acc[1];
        acc[0] = acc[1] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        if (split > 1) { s_sum[wave * 64 + lane] = sum; break; }
        // lane (i, g): row i, vectors 4 g + (0 .. 3)
        const int r = 16 * from + i;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (r < m.rows && 4 * g + v < n) m.Y[(size_t)(4 * g + v) * m.ldy + r] = m.bias ? sum[v] + add : sum[v];
    }
    if (split == 1) return;
    __syncthreads();                                                        // the ranges' sums, in one order
    const int from = blockIdx.x + gridDim.x * (wave / split), r = 16 * from + i;
    if (part || r >= m.rows) return;
    v4f sum = s_sum[wave * 64 + lane];
    for (int p = 1; p < split; ++p) sum += s_sum[(wave + p) * 64 + lane];
    const float add = m.bias ? m.bias[r] : 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (4 * g + v < n) m.Y[(size_t)(4 * g + v) * m.ldy + r] = m.bias ? sum[v] + add : sum[v];
}

// split: waves for a row's columns, a power of two, at most `waves`.  A part is a multiple of four blocks of columns, so that the last ones
// may have none (of 9 to 12 blocks in 4 parts one, of 17 to 20 in 8 three): their sums are zeros.
static q8_status launch_stream(q8_ctx *ctx, F8StreamArgs &a, int waves, int split)
{
    a.split = split;
    a.span = ((a.nb + split - 1) / split + 3) / 4 * 4;
    const int tiles = (a.g.rows + 15) / 16, per = waves / split;
    int blocks = (tiles + per - 1) / per;
    if (split == 1 && blocks > 256) blocks = 256;
    hipLaunchKernelGGL(f8_stream_kernel, dim3(blocks), dim3(64 * waves), (size_t)a.g.n * a.pitch + (split > 1 ? 1024 * waves : 0), ctx->stream, a);
    return q8i_launch_check(ctx, "product f8");
}

// Every block turns the vectors into bf16 values for itself, which saves a launch and costs time with their number (us; here and in
// two launches with 128 x 32 or 64 x 32 tiles): 50000 x 512 x 8 8.3 and 8.4, x 16 9.7 and 8.9; 300 x 300 x 16 5.5 and 7.5;
// 2048 x 2048 x 3 7.2 and 9.2; 512 x 8192 x 1 9.4 and 19.0, x 2 11.3 and 19.0; 1024 x 1024 x 16 9.3 and 8.1.
static bool gemm_f8_streams(int n, int nb) { return n <= 16 && (long long)n * nb <= (n <= 4 ? 160 : 56); }

// X in codes, or Xf [n x ldxf] in fp32 with X the room for its codes (rows, cols, ld, lds and memory), used where they are needed.
q8_status q8i_gemm_f8(q8_ctx *ctx, const q8_mat_f8 *W, const q8_mat_f8 *X, const float *Xf, int ldxf, const float *bias, float *Y, int ldy)
{
    F8GemmArgs a = {W->data, X->data, W->scale, X->scale, bias, Y, W->rows, X->rows, W->cols, W->ld, X->ld, W->lds, X->lds, ldy, 0, 0, 0, 0};
    const int nb = (a.cols + F8_BLOCK - 1) / F8_BLOCK;
    const bool streams = gemm_f8_streams(a.n, nb);
    // (results over the vectors: these are quantized first, as a whole)
    const uintptr_t x0 = (uintptr_t)Xf, x1 = x0 + 4 * ((size_t)(a.n - 1) * ldxf + a.cols), y0 = (uintptr_t)Y, y1 = y0 + 4 * ((size_t)(a.n - 1) * ldy + a.rows);
    if (Xf && (!streams || (x0 < y1 && y0 < x1))) {
        const q8_status st = q8i_quantize_f8(ctx, Xf, a.n, a.cols, ldxf, (uint8_t *)X->data, X->ld, (uint8_t *)X->scale, X->lds);
        if (st) return st;
        Xf = nullptr;
    }
    if (streams) {
        F8StreamArgs s = {a, Xf, ldxf, 0, nb, 0, 0, 0};
        s.vec = ldxf % 4 == 0 && ((uintptr_t)Xf & 15) == 0;
        s.pitch = s.nb * 2 * F8_BLOCK + 16;
        // the columns in parts where the rows alone make few waves: 512 x 8192 x 1 9.4 in 8 parts against 23.3 us, 16384 x 2048 x 3
        // 10.1 in two against 11.0 and 11.9 in four; blocks of four waves spread few rows wider (768 x 256 x 1 3.7 against 4.4)
        const int tiles = (a.rows + 15) / 16;
        int split = 1;
        while (split < 8 && s.nb > 4 * split && tiles * split < 2048) split *= 2;
        const int waves = tiles < 1024 && split == 1 ? 4 : 8;
        return launch_stream(ctx, s, waves, split);
    }
    return gemm_f8_tiles(ctx, a);
}

// ------------------------------------------------------------ statistics of the logits' tiles ----

// (max, sum of exp) of every 16 logits of a row, for the selection of the k best (q8i_select_logits).
__global__ __launch_bounds__(256) void f8_tile_stats_kernel(const float *__restrict__ logits, int n, int V, int ntiles, float *part_max, double *part_sum)
{
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (size_t)n * ntiles) return;
    const size_t j = idx / (unsigned)ntiles;
    const int r0 = (int)(idx - j * (unsigned)ntiles) * 16, rows = min(16, V - r0);
    const float *x = logits + j * (size_t)V + r0;
    float v[16], m = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        v[r] = r < rows ? x[r] : -INFINITY;
        m = fmaxf(m, v[r]);
    }
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (v[r] > -INFINITY) s += (double)exp_le0(v[r] - m);
    part_max[idx] = m;
    part_sum[idx] = s;
}

q8_status q8i_tile_stats(q8_ctx *ctx, const float *logits, int n, int V, float *part_max, double *part_sum)
{
    const int nt = q8i_out_tiles(V);
    const size_t total = (size_t)n * nt;
    hipLaunchKernelGGL(f8_tile_stats_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, ctx->stream, logits, n, V, nt, part_max, part_sum);
    return q8i_launch_check(ctx, "logit statistics");
}
