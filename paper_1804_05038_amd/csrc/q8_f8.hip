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
    int row_tiles;
    int vec;                         // results in whole 16-byte pieces
};

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

#define F8_TILE 64
#define F8_PITCH 144                 // bytes of a row of a stage in LDS: 16 lanes' reads fall on different banks

// Block of four waves: 64 rows x 64 vectors, a stage of 128 columns at a time; wave (wm, wn) has 32 x 32 results.
// The codes are multiplied as bf16 values, because the matrix cores' own 8-bit floating point sums lose bits: products of a
// group are aligned to the largest and cut some 17 bits below it (two products of +-2^17.6 and 126 of 1 gave 120; Gaussian
// codes 1e-5 of the result in the 2-norm, bf16 3e-8).  The order of k inside a block is the same for both operands, which is
// all that it has to be: lane half h takes the 16-byte pieces 2 j + h.
__global__ __launch_bounds__(256) void f8_gemm_kernel(F8GemmArgs a)
{
    __shared__ __align__(16) uint8_t s_w[F8_TILE * F8_PITCH], s_x[F8_TILE * F8_PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave & 1, wn = wave >> 1, i = lane & 31, h = lane >> 5;
    const int r0 = (int)(blockIdx.x % (unsigned)a.row_tiles) * F8_TILE, c0 = (int)(blockIdx.x / (unsigned)a.row_tiles) * F8_TILE;
    v16f acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    const int wrow = r0 + 32 * wm + i, xrow = c0 + 32 * wn + i;
    for (int k0 = 0, b = 0; k0 < a.cols; k0 += F8_BLOCK, ++b) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int e = u * 256 + tid, r = e >> 3, k = k0 + 16 * (e & 7);
            v4i w = {0, 0, 0, 0}, x = {0, 0, 0, 0};
            if (r0 + r < a.rows && k < a.ldw) w = *(const v4i *)(a.W + (size_t)(r0 + r) * a.ldw + k);
            if (c0 + r < a.n && k < a.ldx) x = *(const v4i *)(a.X + (size_t)(c0 + r) * a.ldx + k);
            *(v4i *)(s_w + r * F8_PITCH + 16 * (e & 7)) = w;
            *(v4i *)(s_x + r * F8_PITCH + 16 * (e & 7)) = x;
        }
        const unsigned ew = wrow < a.rows ? a.sw[(size_t)wrow * a.ldsw + b] : 127u, ex = xrow < a.n ? a.sx[(size_t)xrow * a.ldsx + b] : 127u;
        __syncthreads();
        const float fw = __uint_as_float(ew << 23), fx = __uint_as_float(ex << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v4i w = *(const v4i *)(s_w + (32 * wm + i) * F8_PITCH + 16 * (2 * j + h)), x = *(const v4i *)(s_x + (32 * wn + i) * F8_PITCH + 16 * (2 * j + h));
            v8bf wl, wh, xl, xh;
            f8_expand(w, fw, wl, wh);
            f8_expand(x, fx, xl, xh);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wl, xl, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wh, xh, acc, 0, 0, 0);
        }
        __syncthreads();
    }
    // lane (i, h) has rows 8 q + 4 h + (0 .. 3) of vector i
    if (xrow >= a.n) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int row = r0 + 32 * wm + 8 * q + 4 * h;
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = acc[4 * q + e];
            if (a.bias && row + e < a.rows) y[e] = y[e] + a.bias[row + e];
        }
        float *out = a.Y + (size_t)xrow * a.ldy + row;
        if (a.vec && row + 3 < a.rows) {
            *(float4 *)out = make_float4(y[0], y[1], y[2], y[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row + e < a.rows) out[e] = y[e];
        }
    }
}

q8_status q8i_gemm_f8(q8_ctx *ctx, const q8_mat_f8 *W, const q8_mat_f8 *X, const float *bias, float *Y, int ldy)
{
    F8GemmArgs a = {W->data, X->data, W->scale, X->scale, bias, Y, W->rows, X->rows, W->cols, W->ld, X->ld, W->lds, X->lds, ldy, 0, 0};
    a.row_tiles = (a.rows + F8_TILE - 1) / F8_TILE;
    a.vec = ldy % 4 == 0 && ((uintptr_t)Y & 15) == 0;
    const size_t tiles = (size_t)a.row_tiles * ((a.n + F8_TILE - 1) / F8_TILE);
    if (tiles > 0x7fffffffu) return q8_fail(ctx, Q8_ERR_SHAPE, "f8 product: %d x %d results are too many for a launch", a.rows, a.n);
    hipLaunchKernelGGL(f8_gemm_kernel, dim3((unsigned)tiles), dim3(256), 0, ctx->stream, a);
    return q8i_launch_check(ctx, "product f8");
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
