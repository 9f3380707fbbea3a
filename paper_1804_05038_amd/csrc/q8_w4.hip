// q8_w4.hip -- 4-bit weights with a scale and a zero point per group of 32, 64 or 128 columns of a row: quantization, and the
// product with fp32 vectors, Y[j][i] = sum_g s[i,g] sum_{k in g} (c[i,k] - z[i,g]) X[j][k] + bias[i].
#include "q8_internal.h"
#include "q8_parts.h"

#include <math.h>

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

#define W4_BLOCK 128                 // columns of a block: 64 bytes of codes, one, two or four groups
#define W4_SPLIT 512                 // bytes of a block of a vector in its two fp16 parts

// ------------------------------------------------------------------------------ quantization ----

struct W4QuantArgs {
    const float *X;
    int rows, cols, ldx, vec;        // vec: rows begin at 16-byte boundaries
    uint8_t *codes;
    int ld;
    unsigned *scale;
    int lds;
    int units_per_row;               // blocks of a row that have codes, pad bytes or scale words to write
    size_t units;
};

// Maximum over groups of `lanes` (8, 16 or 32) consecutive lanes, in all of them.
template <int LANES>
__device__ __forceinline__ float w4_group_max(float v)
{
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_XOR1>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_XOR2>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_HALF_MIRROR>(__float_as_int(v))));
    if (LANES >= 16) v = fmaxf(v, __int_as_float(dpp_mov_i<DPP_MIRROR>(__float_as_int(v))));
    if (LANES >= 32) v = fmaxf(v, __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), SWZ_XOR16)));
    return v;
}

// A half wave per block of 128 columns, four a lane.  Per group lo = min(0, least), hi = max(0, largest finite value);
// s = (hi - lo) / 15 rounded up to 8 significant bits, so that 15 s covers the range and s is the upper half of an fp32 number;
// z = rint(-lo / s), code = rint(x / s) + z within 0 .. 15, quotients as fp32 division rounds them.  (hi - lo is formed at a
// sixteenth: it may pass fp32's range.)  A run once per model: 50000 x 620 in groups of 32 takes some 40 us.
template <int G>
__global__ __launch_bounds__(256) void w4_quantize_kernel(W4QuantArgs a)
{
    const int half = threadIdx.x >> 5, q = threadIdx.x & 31;
    const size_t unit = (size_t)blockIdx.x * 8 + half;
    const size_t row = unit / (unsigned)a.units_per_row;
    const int b = (int)(unit - row * (unsigned)a.units_per_row), k = b * W4_BLOCK + 4 * q;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (unit < a.units && k < a.cols) {
        const float *x = a.X + row * (size_t)a.ldx + k;
        if (a.vec && k + 3 < a.cols) {
            const float4 f = *(const float4 *)x;
            v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = k + e < a.cols ? x[e] : 0.0f;
        }
    }
    float hi = 0.0f, neg = 0.0f;                                            // neg = -lo
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (fabsf(v[e]) < INFINITY) {
            hi = fmaxf(hi, v[e]);
            neg = fmaxf(neg, -v[e]);
        }
    hi = w4_group_max<G / 4>(hi);
    neg = w4_group_max<G / 4>(neg);
    float s = 1.0f;
    if (fmaxf(hi, neg) >= 0x1p-100f)
        s = __uint_as_float((__float_as_uint((hi * 0.0625f + neg * 0.0625f) / 15.0f * 16.0f) + 0xffffu) & 0xffff0000u);
    else
        neg = 0.0f;
    const float z = rintf(neg / s);
    unsigned c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {                                           // column 2 j + e of eight in bits 4 j + 16 e
        const float x = fmaxf(hi, neg) >= 0x1p-100f && v[e] == v[e] ? v[e] : 0.0f;
        const float f = fminf(fmaxf(rintf(x / s) + z, 0.0f), 15.0f);
        c |= (unsigned)f << (4 * (e >> 1) + 16 * (e & 1));
    }
    if (q & 1) c <<= 8;
    c |= (unsigned)dpp_mov_i<DPP_XOR1>((int)c);
    if (unit >= a.units) return;
    // columns 32 t + 8 g + (0 .. 7) of a block are word 4 g + t of its 16
    if (!(q & 1) && b * 64 < a.ld) *(unsigned *)(a.codes + row * (size_t)a.ld + b * 64 + 16 * ((q >> 1) & 3) + 4 * (q >> 3)) = c;
    const int w = b * (W4_BLOCK / G) + q / (G / 4);
    if (q % (G / 4) == 0 && w < a.lds) a.scale[row * (size_t)a.lds + w] = __float_as_uint(s) | (unsigned)z;
}

q8_status q8i_quantize_w4(q8_ctx *ctx, const float *X, int rows, int cols, int ldx, const q8_mat_w4 *out)
{
    W4QuantArgs a = {X, rows, cols, ldx, 0, (uint8_t *)out->data, out->ld, (unsigned *)out->scale, out->lds, 0, 0};
    const int per = W4_BLOCK / out->group, nb = out->ld / 64, ns = (out->lds + per - 1) / per;
    a.vec = ldx % 4 == 0 && ((uintptr_t)X & 15) == 0;
    a.units_per_row = nb > ns ? nb : ns;
    a.units = (size_t)rows * a.units_per_row;
    const size_t grid = (a.units + 7) / 8;
    if (grid >= 1u << 24)                                                   // a launch has fewer than 2^32 threads
        return q8_fail(ctx, Q8_ERR_SHAPE, "quantize w4: %d rows of %d blocks are too many for a launch", rows, a.units_per_row);
    void (*const kernel)(W4QuantArgs) = out->group == 32 ? w4_quantize_kernel<32> : out->group == 64 ? w4_quantize_kernel<64> : w4_quantize_kernel<128>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, ctx->stream, a);
    return q8i_launch_check(ctx, "quantize w4");
}

// ------------------------------------------------------------------------------- the product ----

// The matrix cores multiply fp16 values and sum in fp32.  A weight c - z is a whole number of at most 15 in magnitude: exact.  A
// vector's value times a power of two that puts the largest of its block (or of its vector) below 2^14 is the sum of two
// fp16 values, hi + lo, within 2^-22 of itself (2^-38 of the largest where that is more): two products instead of one, each exact
// in fp32, and what is lost is below what sums in fp32 lose.  A group's sum is formed in whole numbers and fractions of X alone and
// multiplied by its scale once.

// Eight weights c - z from a word of codes.  A code in the fraction of 1024.0 is 1024 + c, one four bits higher 1024 + 16 c.
// z1 = -(1024 + z), z2 = -(64 + z), twice each.
__device__ __forceinline__ v8h w4_expand(unsigned c, v2h z1, v2h z2)
{
    const v2h sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const unsigned d = c >> 8;
    const v2h a = __builtin_bit_cast(v2h, (c & 0x000f000fu) | 0x64006400u) + z1;
    const v2h b = __builtin_elementwise_fma(__builtin_bit_cast(v2h, (c & 0x00f000f0u) | 0x64006400u), sixteenth, z2);
    const v2h e = __builtin_bit_cast(v2h, (d & 0x000f000fu) | 0x64006400u) + z1;
    const v2h f = __builtin_elementwise_fma(__builtin_bit_cast(v2h, (d & 0x00f000f0u) | 0x64006400u), sixteenth, z2);
    return (v8h){a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]};
}

__device__ __forceinline__ void w4_zeros(unsigned word, v2h &z1, v2h &z2)
{
    const unsigned z = word & 15u, a = 0xe400u | z, b = 0xd400u + (z << 4);
    z1 = __builtin_bit_cast(v2h, a | a << 16);
    z2 = __builtin_bit_cast(v2h, b | b << 16);
}

struct W4GemmArgs {
    const uint8_t *W;
    const unsigned *sw;
    const float *X;                  // fp32 vectors [n x ldx]
    const uint8_t *parts;            // their parts [n][nb][hi 128 | lo 128] fp16 and scales, of the tiles
    const float *sx;
    const float *bias;
    float *Y;
    int rows, n, cols, ldw, lds, ng, ldx, ldy, nb;
    int vec;                         // the vectors begin at 16-byte boundaries
    int pitch, split, span;          // few vectors: bytes of a vector in LDS; waves for a row's columns, blocks of columns of each
    int row_tiles, col_tiles;
};

// ------------------------------------------------------------------------- few vectors ----

#define W4_STREAM_BLOCKS 128         // blocks of all vectors together, at most: their parts, pitches, scales and the waves' sums fit
#define W4_STREAM_LDS (W4_STREAM_BLOCKS * W4_SPLIT + 16 * 16 + 64 * W4_STREAM_BLOCKS + 1024 * 8)

// Up to 16 vectors: the codes go from memory to registers once; the vectors lie in LDS in parts, put there by every block for
// itself.  A wave multiplies 16 rows at a time, four blocks of columns a turn; `split` waves share the rows, each with its range of
// the columns.  Lane (i, g) has row i and of every block the 16-byte piece g, whose word t belongs to columns 32 t + 8 g + (0 .. 7):
// a matrix operation takes 32 columns in a row, so that groups of 32 have their sums too.
template <int PER>                   // groups of a block
__global__ __launch_bounds__(512) void w4_stream_kernel(W4GemmArgs a)
{
    extern __shared__ __align__(16) uint8_t s_x[];                          // [n][pitch], scales [nb][16], the waves' sums [waves][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, i = lane & 15, g = lane >> 4;
    const int n = a.n, split = a.split, part = wave & (split - 1), tiles = (a.rows + 15) >> 4, per = waves / split, stride = gridDim.x * per;
    const int b0 = part * a.span, b1 = min(b0 + a.span, a.nb);
    int tile = blockIdx.x + gridDim.x * (wave / split), b = b0;
    __amdgpu_buffer_rsrc_t rw, rs;
    unsigned row_at, scale_at;
    float bias;
    auto rows_of = [&](int t) {                                             // no rows: every access past the end
        const int r0 = 16 * min(t, tiles - 1), left = t < tiles && b0 < b1 ? min(16, a.rows - r0) : 0;
        rw = q8_rsrc(a.W + (size_t)r0 * a.ldw, (size_t)left * a.ldw);
        rs = q8_rsrc(a.sw + (size_t)r0 * a.lds, (size_t)left * a.lds * 4);
        row_at = i < left ? (unsigned)i * (unsigned)a.ldw + 16 * g : Q8_OOB;
        scale_at = i < left ? (unsigned)i * (unsigned)a.lds * 4 : Q8_OOB;
        bias = a.bias && i < left ? a.bias[r0 + i] : 0.0f;
    };
    v4u w[4], sc[PER];
    auto codes = [&](int s) {
        return __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(b + s < b1 && row_at != Q8_OOB ? row_at + 64 * (b + s) : Q8_OOB), 0, 0));
    };
    auto scales = [&](int p) {                                              // words 4 p .. 4 p + 3 of the turn's
        return __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(b * PER + 4 * p < a.lds && scale_at != Q8_OOB ? scale_at + 4 * (b * PER + 4 * p) : Q8_OOB), 0, 0));
    };
    rows_of(tile);
#pragma unroll
    for (int s = 0; s < 4; ++s) w[s] = codes(s);
#pragma unroll
    for (int p = 0; p < PER; ++p) sc[p] = scales(p);

    // ---- the vectors, a half wave per block of columns, four values a lane
    float *s_scale = (float *)(s_x + (size_t)n * a.pitch);
    const int q = lane & 31, units = n * a.nb, halves = 2 * waves;
    for (int u = tid >> 5; u < units; u += halves) {
        const int j = u / a.nb, blk = u - j * a.nb, k = blk * W4_BLOCK + 4 * q;
        const float *x = a.X + (size_t)j * a.ldx + k;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k + 3 < a.cols) {
            if (a.vec) v = *(const float4 *)x;
            else v = make_float4(x[0], x[1], x[2], x[3]);
        } else {
            if (k < a.cols) v.x = x[0];
            if (k + 1 < a.cols) v.y = x[1];
            if (k + 2 < a.cols) v.z = x[2];
        }
        const float top = w4_group_max<32>(fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))));
        float inv;
        const float sx = parts_scale(top, inv);
        uint2 hi, lo;
        parts4(v.x, v.y, v.z, v.w, inv, hi, lo);
        uint8_t *at = s_x + (size_t)j * a.pitch + blk * W4_SPLIT + 8 * q;
        *(uint2 *)at = hi;
        *(uint2 *)(at + W4_SPLIT / 2) = lo;
        if (q == 0) s_scale[blk * 16 + j] = sx;
    }
    __syncthreads();

    v4f *s_sum = (v4f *)(s_scale + 16 * a.nb);
    v4f total = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *px = s_x + (size_t)min(i, n - 1) * a.pitch + 16 * g;
    while (tile < tiles) {
        const int at = b, from = tile;
        const float add = bias;
        v4u cw[4], cs[PER];
#pragma unroll
        for (int s = 0; s < 4; ++s) cw[s] = w[s];
#pragma unroll
        for (int p = 0; p < PER; ++p) cs[p] = sc[p];
        b += 4;
        const bool last = b >= b1;
        if (last) {
            b = b0;
            tile += stride;
            rows_of(tile);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] = codes(s);
#pragma unroll
        for (int p = 0; p < PER; ++p) sc[p] = scales(p);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (at + s >= b1) break;
            const uint8_t *x = px + (at + s) * W4_SPLIT;
            const v4f sx = *(const v4f *)(s_scale + (at + s) * 16 + 4 * g);
            v4f hi, lo;
            v2h z1, z2;
            float sw = 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t % (4 / PER) == 0) {                                   // a group begins (past the last one: anything)
                    const int word = s * PER + t / (4 / PER);
                    const unsigned e = (at + s) * PER + t / (4 / PER) < a.ng ? cs[word >> 2][word & 3] : 0u;
                    w4_zeros(e, z1, z2);
                    sw = __uint_as_float(e & 0xffff0000u);
                    hi = lo = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
                }
                const v8h wv = w4_expand(cw[s][t], z1, z2);
                hi = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)(x + 64 * t), wv, hi, 0, 0, 0);
                lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)(x + 64 * t + W4_SPLIT / 2), wv, lo, 0, 0, 0);
                if (t % (4 / PER) == 4 / PER - 1) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) total[v] = fmaf((hi[v] + lo[v]) * sw, sx[v], total[v]);      // (sw sx alone may pass fp32's range)
                }
            }
        }
        if (!last) continue;
        const v4f sum = total;
        total = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        if (split > 1) { s_sum[wave * 64 + lane] = sum; break; }
        // lane (i, g): row i, vectors 4 g + (0 .. 3)
        const int r = 16 * from + i;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (r < a.rows && 4 * g + v < n) a.Y[(size_t)(4 * g + v) * a.ldy + r] = a.bias ? sum[v] + add : sum[v];
    }
    if (split == 1) return;
    __syncthreads();                                                        // the ranges' sums, in one order
    const int from = blockIdx.x + gridDim.x * (wave / split), r = 16 * from + i;
    if (part || r >= a.rows) return;
    v4f sum = s_sum[wave * 64 + lane];
    for (int p = 1; p < split; ++p)
        if (p * a.span < a.nb) sum += s_sum[(wave + p) * 64 + lane];
    const float add = a.bias ? a.bias[r] : 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (4 * g + v < n) a.Y[(size_t)(4 * g + v) * a.ldy + r] = a.bias ? sum[v] + add : sum[v];
}

// split: waves for a row's columns, a power of two, at most `waves`.  A part is a multiple of four blocks of columns, so that the last ones
// may have none: these leave no sums, and none are added.
static q8_status launch_stream_w4(q8_ctx *ctx, W4GemmArgs &a, int per_block, int waves, int split)
{
    static Q8OncePerDevice once[3];
    a.split = split;
    a.span = ((a.nb + split - 1) / split + 3) / 4 * 4;
    a.pitch = a.nb * W4_SPLIT + 16;
    const int tiles = (a.rows + 15) / 16, per = waves / split;
    int blocks = (tiles + per - 1) / per;
    if (split == 1 && blocks > 512) blocks = 512;
    const size_t smem = (size_t)a.n * a.pitch + 64 * a.nb + (split > 1 ? 1024 * waves : 0);
    void (*const kernel)(W4GemmArgs) = per_block == 4 ? w4_stream_kernel<4> : per_block == 2 ? w4_stream_kernel<2> : w4_stream_kernel<1>;
    const q8_status st = smem > 65536 ? q8i_lds(ctx, once[per_block >> 1], (const void *)kernel, W4_STREAM_LDS, "w4 product") : Q8_OK;
    if (st) return st;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product w4");
}

// ------------------------------------------------------------------------------ many vectors ----

// A vector's parts and scale, a block per vector.
__global__ __launch_bounds__(256) void w4_parts_kernel(const float *X, int cols, int ldx, int vec, int nb, uint8_t *parts, float *sx)
{
    __shared__ float s_max[4];
    const int j = blockIdx.x, tid = threadIdx.x;
    const float *x = X + (size_t)j * ldx;
    auto load = [&](int k) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k + 3 < cols && vec) return *(const float4 *)(x + k);
        if (k < cols) v.x = x[k];
        if (k + 1 < cols) v.y = x[k + 1];
        if (k + 2 < cols) v.z = x[k + 2];
        if (k + 3 < cols) v.w = x[k + 3];
        return v;
    };
    float4 keep[2];                                                         // the first 2048 columns stay in registers
    float m = 0.0f;
    for (int t = 0; t * 1024 < nb * W4_BLOCK; ++t) {
        const float4 v = load(t * 1024 + 4 * tid);
        if (t == 0) keep[0] = v;
        if (t == 1) keep[1] = v;
        m = fmaxf(m, fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))));
    }
    m = wave_max_f(m);
    if ((tid & 63) == 0) s_max[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    float inv;
    const float s = parts_scale(m, inv);
    if (tid == 0) sx[j] = s;
    for (int t = 0; t * 1024 < nb * W4_BLOCK; ++t) {
        const int k = t * 1024 + 4 * tid;
        if (k >= nb * W4_BLOCK) break;
        const float4 v = t == 0 ? keep[0] : t == 1 ? keep[1] : load(k);
        uint2 hi, lo;
        parts4(v.x, v.y, v.z, v.w, inv, hi, lo);
        uint8_t *at = parts + ((size_t)j * nb + (k >> 7)) * W4_SPLIT + 2 * (k & 127);
        *(uint2 *)at = hi;
        *(uint2 *)(at + W4_SPLIT / 2) = lo;
    }
}

// Sixteen bytes a lane from memory to LDS at `at` + 16 lane (a wave's address), without passing through registers.
__device__ __forceinline__ void w4_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint8_t *at, unsigned offset, int step)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)at, 16, offset, step, 0, 0);
#endif
}

// Block of WM x WN waves, each with 32 TM rows x 32 TN vectors; the vectors' parts come in stages of 128 columns (half a kilobyte a vector)
// from memory to LDS, one on its way while the one before is multiplied; each wave reads its rows' codes (64 bytes a stage) by itself.
// Lane (i, h) of a row tile has the 16-byte pieces h and 2 + h of row i: word t of piece 2 p + h belongs to columns 32 t + 16 p + 8 h + (0 .. 7),
// operation (t, p) of a stage to columns 32 t + 16 p + (0 .. 15).  In LDS a vector's 32 pieces of 16 bytes are exchanged by its number mod 8, so that
// lanes that read together find theirs on different banks.
template <int PER, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void w4_gemm_kernel(W4GemmArgs a)
{
    constexpr int VECS = 32 * WN * TN, THREADS = 64 * WM * WN, STAGE = VECS * W4_SPLIT, LX = VECS * 32 / THREADS;
    static_assert(VECS * 32 % THREADS == 0, "even shares of a stage");
    extern __shared__ __align__(16) uint8_t s_x[];                          // [2][STAGE]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM, i = lane & 31, h = lane >> 5;
    const int tr = blockIdx.x / a.col_tiles, tc = blockIdx.x % a.col_tiles;
    const int r0 = 32 * TM * (tr * WM + wm), c0 = tc * VECS, left = min(VECS, a.n - c0);
    const __amdgpu_buffer_rsrc_t rx = q8_rsrc(a.parts + (size_t)c0 * a.nb * W4_SPLIT, (size_t)left * a.nb * W4_SPLIT);
    unsigned ox[LX];                                                        // piece p of a stage: vector p / 32 (beyond the last: the last again)
#pragma unroll
    for (int u = 0; u < LX; ++u) {
        const int p = u * THREADS + tid, v = p >> 5;
        ox[u] = (unsigned)min(v, left - 1) * (unsigned)(a.nb * W4_SPLIT) + 16u * (unsigned)((p & 31) ^ (v & 7));
    }
    auto request = [&](int b, int stage) {
        uint8_t *at = s_x + stage * STAGE + wave * 1024;
#pragma unroll
        for (int u = 0; u < LX; ++u) w4_to_lds(rx, at + u * THREADS * 16, ox[u], b * W4_SPLIT);
    };
    const uint8_t *pw[TM];
    const unsigned *ps[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const size_t row = (size_t)min(r0 + 32 * t + i, a.rows - 1);
        pw[t] = a.W + row * a.ldw + 16 * h;
        ps[t] = a.sw + row * a.lds;
    }
    v4u w[TM][2];
    unsigned sc[TM][PER];
    auto codes = [&](int b) {
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            w[t][0] = *(const v4u *)(pw[t] + 64 * b);
            w[t][1] = *(const v4u *)(pw[t] + 64 * b + 32);
#pragma unroll
            for (int p = 0; p < PER; ++p) sc[t][p] = b * PER + p < a.ng ? ps[t][b * PER + p] : 0u;
        }
    };
    v16f acc[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][u][e] = 0.0f;
    const int twist = i & 7, lx = (32 * wn * TN + i) * W4_SPLIT;
    codes(0);
    request(0, 0);
#pragma unroll 1
    for (int b = 0; b < a.nb; ++b) {
        __syncthreads();                                                    // this stage is there, the other one is free
        if (b + 1 < a.nb) request(b + 1, (b + 1) & 1);
        v4u cw[TM][2];
        unsigned cs[TM][PER];
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            cw[t][0] = w[t][0];
            cw[t][1] = w[t][1];
#pragma unroll
            for (int p = 0; p < PER; ++p) cs[t][p] = sc[t][p];
        }
        if (b + 1 < a.nb) codes(b + 1);
        const uint8_t *px = s_x + (b & 1) * STAGE + lx;
        v16f sum[TM][TN];
        v2h z1[TM], z2[TM];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t % (4 / PER) == 0) {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    w4_zeros(cs[m][t / (4 / PER)], z1[m], z2[m]);
#pragma unroll
                    for (int u = 0; u < TN; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum[m][u][e] = 0.0f;
                }
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int piece = 4 * t + 2 * p + h;
                v8h xh[TN], xl[TN];
#pragma unroll
                for (int u = 0; u < TN; ++u) {
                    xh[u] = *(const v8h *)(px + u * 32 * W4_SPLIT + 16 * (piece ^ twist));
                    xl[u] = *(const v8h *)(px + u * 32 * W4_SPLIT + 16 * ((16 + piece) ^ twist));
                }
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const v8h wv = w4_expand(cw[m][p][t], z1[m], z2[m]);
#pragma unroll
                    for (int u = 0; u < TN; ++u) sum[m][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xh[u], wv, sum[m][u], 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < TN; ++u) sum[m][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xl[u], wv, sum[m][u], 0, 0, 0);
                }
            }
            if (t % (4 / PER) == 4 / PER - 1) {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const float sw = __uint_as_float(cs[m][t / (4 / PER)] & 0xffff0000u);
#pragma unroll
                    for (int u = 0; u < TN; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[m][u][e] = fmaf(sum[m][u][e], sw, acc[m][u][e]);
                }
            }
        }
    }
    // lane (i, h): row i of a row tile, vectors 8 q + 4 h + (0 .. 3) of a tile of vectors
    float bias[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) bias[t] = a.bias ? a.bias[min(r0 + 32 * t + i, a.rows - 1)] : 0.0f;
#pragma unroll
    for (int u = 0; u < TN; ++u) {
        const int v0 = c0 + 32 * (wn * TN + u) + 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int v = v0 + 8 * (e >> 2) + (e & 3);
            const float s = a.sx[min(v, a.n - 1)];
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                const int row = r0 + 32 * t + i;
                const float y = acc[t][u][e] * s;
                if (row < a.rows && v < a.n) a.Y[(size_t)v * a.ldy + row] = a.bias ? y + bias[t] : y;
            }
        }
    }
}

template <int PER, int WM, int WN, int TM, int TN> static q8_status launch_w4(q8_ctx *ctx, W4GemmArgs &a)
{
    static Q8OncePerDevice once;
    const size_t smem = (size_t)2 * 32 * WN * TN * W4_SPLIT;
    a.row_tiles = (a.rows + 32 * WM * TM - 1) / (32 * WM * TM);
    a.col_tiles = (a.n + 32 * WN * TN - 1) / (32 * WN * TN);
    const size_t tiles = (size_t)a.row_tiles * a.col_tiles;
    if (tiles * (64 * WM * WN) > 0xffffffffu)                               // a launch has fewer than 2^32 threads
        return q8_fail(ctx, Q8_ERR_SHAPE, "w4 product: %d x %d results are too many for a launch", a.rows, a.n);
    const q8_status st = q8i_lds(ctx, once, (const void *)w4_gemm_kernel<PER, WM, WN, TM, TN>, smem, "w4 product");
    if (st) return st;
    hipLaunchKernelGGL((w4_gemm_kernel<PER, WM, WN, TM, TN>), dim3((unsigned)tiles), dim3(64 * WM * WN), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product w4");
}

template <int PER> static q8_status gemm_w4_tiles(q8_ctx *ctx, W4GemmArgs &a)
{
    if (a.n <= 32) return launch_w4<PER, 4, 1, 1, 1>(ctx, a);
    return launch_w4<PER, 4, 1, 1, 2>(ctx, a);
}

// Every block makes the vectors' parts for itself, which saves a launch and costs time with their number.
static bool gemm_w4_streams(int n, int nb) { return n <= 16 && (long long)n * nb <= W4_STREAM_BLOCKS; }

size_t q8i_gemm_w4_parts(int n, int cols) { return (size_t)n * ((cols + W4_BLOCK - 1) / W4_BLOCK) * W4_SPLIT; }

q8_status q8i_gemm_w4(q8_ctx *ctx, const q8_mat_w4 *W, const float *X, int n, int ldx, const float *bias, float *Y, int ldy, uint8_t *parts, float *sx)
{
    W4GemmArgs a = {W->data, W->scale, X, parts, sx, bias, Y, W->rows, n, W->cols, W->ld, W->lds, (W->cols + W->group - 1) / W->group, ldx, ldy,
                    (W->cols + W4_BLOCK - 1) / W4_BLOCK, 0, 0, 0, 0, 0, 0};
    a.vec = ldx % 4 == 0 && ((uintptr_t)X & 15) == 0;
    const int per = W4_BLOCK / W->group;
    // (results over the vectors: these are read first, as a whole)
    const uintptr_t x0 = (uintptr_t)X, x1 = x0 + 4 * ((size_t)(n - 1) * ldx + a.cols), y0 = (uintptr_t)Y, y1 = y0 + 4 * ((size_t)(n - 1) * ldy + a.rows);
    if (gemm_w4_streams(n, a.nb) && !(x0 < y1 && y0 < x1)) {
        const int tiles = (a.rows + 15) / 16;
        int split = 1;
        while (split < 8 && a.nb > 4 * split && tiles * split < 2048) split *= 2;
        return launch_stream_w4(ctx, a, per, tiles < 1024 && split == 1 ? 4 : 8, split);
    }
    hipLaunchKernelGGL(w4_parts_kernel, dim3(n), dim3(256), 0, ctx->stream, X, a.cols, ldx, a.vec, a.nb, parts, sx);
    const q8_status st = q8i_launch_check(ctx, "parts w4");
    if (st) return st;
    return per == 4 ? gemm_w4_tiles<4>(ctx, a) : per == 2 ? gemm_w4_tiles<2>(ctx, a) : gemm_w4_tiles<1>(ctx, a);
}
