// q8_f8.hip -- 8-bit floating point with a scale per block: quantization of rows into e4m3 codes with one power of two per
// 128 columns, and the product of such codes, Y[j][i] = sum_b 2^(ew[i,b] + ex[j,b]) sum_{k in b} cw[i,k] cx[j,k] + bias[i].
#include "q8_internal.h"

#include <math.h>
#include <type_traits>

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
// of two is exact, so the conversion's rounding (to nearest, ties to even) is the only one.
__device__ __forceinline__ unsigned f8_codes4(float4 v, float inv)
{
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(v.x * inv, v.y * inv, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(v.z * inv, v.w * inv, p, true);
    return (unsigned)p;
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

// A half wave per block of 128 columns: four values a lane.
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
    const size_t per_block = 4 * F8_QUANT_PER_WAVE;
    hipLaunchKernelGGL(f8_quantize_kernel, dim3((unsigned)((a.units + per_block - 1) / per_block)), dim3(256), 0, ctx->stream, a);
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
    int vec;                         // results in whole 16-byte pieces
};

// The tile of a block.  Consecutive blocks run on different XCDs, each with an L2 cache of its own: each XCD gets a range of
// the tiles in a row, and these go through eight row tiles for each column tile, so that the tiles that run on an XCD at one
// time share rows and vectors.
__device__ __forceinline__ void f8_tile_of(unsigned block, int row_tiles, int col_tiles, int &tr, int &tc)
{
    const unsigned total = gridDim.x, per = total / 8, over = total % 8, xcd = block % 8, idx = block / 8;
    const unsigned t = xcd * per + min(xcd, over) + idx;
    const unsigned band = t / (8u * (unsigned)col_tiles), in = t - band * 8u * (unsigned)col_tiles, height = min(8u, (unsigned)row_tiles - 8u * band);
    tc = (int)(in / height);
    tr = (int)(8u * band + in % height);
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
// together (rows 0-3 and 16-19 of a group of 32, or 4-7 and 20-23, ...) find theirs on different banks.
__device__ __forceinline__ int f8_twist(int row) { return (row & 3) | ((row >> 2) & 4); }
// The row of a group of 32 that lane i multiplies: then lane (i, h) ends up with the results of 16 rows in a row, 16 h ...
__device__ __forceinline__ int f8_row(int i) { return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3); }

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
template <int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void f8_gemm_kernel(F8GemmArgs a)
{
    constexpr int ROWS = 32 * WM * TM, VECS = 32 * WN * TN, THREADS = 64 * WM * WN, STAGE = (ROWS + VECS) * F8_BLOCK;
    constexpr int LW = ROWS * 8 / THREADS, LX = VECS * 8 / THREADS;                    // 16-byte pieces a thread requests
    static_assert(ROWS * 8 % THREADS == 0 && VECS * 8 % THREADS == 0, "even shares of a stage");
    extern __shared__ __align__(16) uint8_t s_f8[];                                    // [2][STAGE]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM, i = lane & 31, h = lane >> 5;
    int tr, tc;
    f8_tile_of(blockIdx.x, a.row_tiles, a.col_tiles, tr, tc);
    const int r0 = tr * ROWS, c0 = tc * VECS, steps = (a.cols + F8_BLOCK - 1) / F8_BLOCK, kend = (a.cols + 15) & ~15;
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
        // (of the last one's pieces that lie past the columns, the row's first piece takes the place)
        auto past = [&](int p) { return step >= full && step * F8_BLOCK + 16 * ((p & 7) ^ f8_twist(p >> 3)) >= kend ? 16u * (unsigned)((p & 7) ^ f8_twist(p >> 3)) + step * F8_BLOCK : 0u; };
#pragma unroll
        for (int u = 0; u < LW; ++u)
            f8_to_lds(rw, at + u * THREADS * 16, ow[u] - past(u * THREADS + tid), step * F8_BLOCK);
#pragma unroll
        for (int u = 0; u < LX; ++u)
            f8_to_lds(rx, at + ROWS * F8_BLOCK + u * THREADS * 16, ox[u] - past(u * THREADS + tid), step * F8_BLOCK);
    };
    // scales: four steps' bytes at a time
    const uint8_t *pw[TM], *px[TN];
#pragma unroll
    for (int t = 0; t < TM; ++t) pw[t] = a.sw + (size_t)min(r0 + 32 * (wm * TM + t) + f8_row(i), a.rows - 1) * a.ldsw;
#pragma unroll
    for (int t = 0; t < TN; ++t) px[t] = a.sx + (size_t)min(c0 + 32 * (wn * TN + t) + f8_row(i), a.n - 1) * a.ldsx;
    unsigned ew[TM], ex[TN];
    v16f acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][u][e] = 0.0f;
    const int lw = (32 * wm * TM + f8_row(i)) * F8_BLOCK, lx = ROWS * F8_BLOCK + (32 * wn * TN + f8_row(i)) * F8_BLOCK, twist = f8_twist(f8_row(i));

    auto scales = [&](int step) {
        if ((step & 3) == 0) {
#pragma unroll
            for (int t = 0; t < TM; ++t) ew[t] = *(const unsigned *)(pw[t] + step);
#pragma unroll
            for (int t = 0; t < TN; ++t) ex[t] = *(const unsigned *)(px[t] + step);
        }
    };
    auto multiply = [&](int step, auto cut) {
        const uint8_t *st = s_f8 + (step & 1) * STAGE;
        float fw[TM], fx[TN];
#pragma unroll
        for (int t = 0; t < TM; ++t) fw[t] = __uint_as_float(((ew[t] >> (8 * (step & 3))) & 255u) << 23);
#pragma unroll
        for (int t = 0; t < TN; ++t) fx[t] = __uint_as_float(((ex[t] >> (8 * (step & 3))) & 255u) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v4i w[TM], x[TN];
            const int piece = 16 * ((2 * j + h) ^ twist);
#pragma unroll
            for (int t = 0; t < TM; ++t) w[t] = *(const v4i *)(st + lw + t * 32 * F8_BLOCK + piece);
#pragma unroll
            for (int t = 0; t < TN; ++t) x[t] = *(const v4i *)(st + lx + t * 32 * F8_BLOCK + piece);
            if constexpr (decltype(cut)::value) {                           // what lies past the columns counts as zeros
                const int keep = step * F8_BLOCK + 16 * (2 * j + h) < kend ? -1 : 0;
#pragma unroll
                for (int t = 0; t < TM; ++t) w[t] &= keep;
#pragma unroll
                for (int t = 0; t < TN; ++t) x[t] &= keep;
            }
            v8bf xl[TN], xh[TN];
#pragma unroll
            for (int t = 0; t < TN; ++t) f8_expand(x[t], fx[t], xl[t], xh[t]);
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                v8bf wl, wh;
                f8_expand(w[t], fw[t], wl, wh);
#pragma unroll
                for (int u = 0; u < TN; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wl, xl[u], acc[t][u], 0, 0, 0);
#pragma unroll
                for (int u = 0; u < TN; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wh, xh[u], acc[t][u], 0, 0, 0);
            }
        }
    };
    request(0, 0);
    for (int step = 0; step < full; ++step) {
        scales(step);
        __syncthreads();                                                    // this step's stage is there, the other one is free
        if (step + 1 < steps) request(step + 1, (step + 1) & 1);
        multiply(step, std::false_type());
    }
    if (full < steps) {
        scales(full);
        __syncthreads();
        multiply(full, std::true_type());
    }
    // lane (i, h): rows 16 h + (0 .. 15) of each group, vector f8_row(i)
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int row = r0 + 32 * (wm * TM + t) + 16 * h;
        float b[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) b[e] = a.bias && row + e < a.rows ? a.bias[row + e] : 0.0f;
#pragma unroll
        for (int u = 0; u < TN; ++u) {
            const int vec = c0 + 32 * (wn * TN + u) + f8_row(i);
            if (vec >= a.n) continue;
            float *out = a.Y + (size_t)vec * a.ldy + row;
            const bool plain = !a.bias;                                     // (y + 0 would turn -0 into 0)
            if (a.vec && row + 15 < a.rows) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float4 y = make_float4(acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]);
                    if (!plain) y = make_float4(y.x + b[4 * q], y.y + b[4 * q + 1], y.z + b[4 * q + 2], y.w + b[4 * q + 3]);
                    *(float4 *)(out + 4 * q) = y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (row + e < a.rows) out[e] = plain ? acc[t][u][e] : acc[t][u][e] + b[e];
            }
        }
    }
}

template <int WM, int WN, int TM, int TN> static q8_status launch_f8(q8_ctx *ctx, F8GemmArgs &a)
{
    static Q8OncePerDevice once;
    const size_t smem = (size_t)2 * 32 * (WM * TM + WN * TN) * F8_BLOCK;
    a.row_tiles = (a.rows + 32 * WM * TM - 1) / (32 * WM * TM);
    a.col_tiles = (a.n + 32 * WN * TN - 1) / (32 * WN * TN);
    const size_t tiles = (size_t)a.row_tiles * a.col_tiles;
    if (tiles > 0x7fffffffu) return q8_fail(ctx, Q8_ERR_SHAPE, "f8 product: %d x %d results are too many for a launch", a.rows, a.n);
    const q8_status st = q8i_lds(ctx, once, (const void *)f8_gemm_kernel<WM, WN, TM, TN>, smem, "f8 product");
    if (st) return st;
    hipLaunchKernelGGL((f8_gemm_kernel<WM, WN, TM, TN>), dim3((unsigned)tiles), dim3(64 * WM * WN), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product f8");
}

q8_status q8i_gemm_f8(q8_ctx *ctx, const q8_mat_f8 *W, const q8_mat_f8 *X, const float *bias, float *Y, int ldy)
{
    F8GemmArgs a = {W->data, X->data, W->scale, X->scale, bias, Y, W->rows, X->rows, W->cols, W->ld, X->ld, W->lds, X->lds, ldy, 0, 0, 0};
    a.vec = ldy % 4 == 0 && ((uintptr_t)Y & 15) == 0;
    const size_t big = (size_t)((a.rows + 255) / 256) * ((a.n + 255) / 256);
    if (big >= 200 && a.cols > 1024) return launch_f8<2, 4, 4, 2>(ctx, a);
    if (a.n <= 64) return launch_f8<4, 1, 1, 2>(ctx, a);
    return launch_f8<2, 2, 2, 2>(ctx, a);
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
