// q8_w4.hip -- 4-bit weights with a scale and a zero point per group of 32, 64 or 128 columns of a row: quantization, and the
// product with fp32 vectors, Y[j][i] = sum_g s[i,g] sum_{k in g} (c[i,k] - z[i,g]) X[j][k] + bias[i].
#include "q8_internal.h"
#include "q8_parts.h"
#include "q8_route.h"

#include <math.h>
#include <type_traits>

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

#define W4_BLOCK 128                 // columns of a block: 64 bytes of codes, one, two or four groups
#define W4_SPLIT 512                 // bytes of a block of a vector in its two fp16 parts
// A group's sum without scales is below 2^25 (128 weights of 15, parts below 2^14).  Words of scales above this (s = 2^93; its low bits are the zero point) could
// take the sums of 512 groups past fp32's range before the vector's power of two brings them back: these go another way.
#define W4_LARGE 0x6e000000u

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
// sixteenth: it may pass fp32's range.)  Run once per model: 63644 x 620 in groups of 32 in 57 us (183 MB read and written,
// 3.2 TB/s), 50000 x 512 in groups of 128 in 37.
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
// z1 = -(1024 + z), z2 = -(64 + z), twice each; magic = 1024.0 twice, in a register of the lanes: and-or takes one number of
// the wave's registers, which the mask is, and none of its own code.
__device__ __forceinline__ v8h w4_expand(unsigned c, v2h z1, v2h z2, unsigned magic)
{
    const v2h sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const unsigned d = c >> 8;
    const v2h a = __builtin_bit_cast(v2h, (c & 0x000f000fu) | magic) + z1;
    const v2h b = __builtin_elementwise_fma(__builtin_bit_cast(v2h, (c & 0x00f000f0u) | magic), sixteenth, z2);
    const v2h e = __builtin_bit_cast(v2h, (d & 0x000f000fu) | magic) + z1;
    const v2h f = __builtin_elementwise_fma(__builtin_bit_cast(v2h, (d & 0x00f000f0u) | magic), sixteenth, z2);
    return (v8h){a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]};
}

__device__ __forceinline__ unsigned w4_magic()
{
    unsigned m = 0x64006400u;
    asm("" : "+v"(m));
    return m;
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
    int pitch, split, span;          // few vectors: bytes of a vector in LDS; waves for a row's columns, blocks of columns of each
    int row_tiles, col_tiles;
};

// ------------------------------------------------------------------------- few vectors ----

#define W4_STREAM_BLOCKS Q8_W4_STREAM_BLOCKS      // of all vectors together, at most: their parts, pitches, scales (a vector has at least a block) and the waves' sums fit
#define W4_STREAM_LDS (W4_STREAM_BLOCKS * W4_SPLIT + 16 * 16 + 64 * W4_STREAM_BLOCKS + 1024 * 16)

// Up to 16 vectors (at 16-byte boundaries): the codes go from memory to registers once; the vectors lie in LDS in parts, put there by every block for
// itself.  A wave multiplies 16 rows at a time, four blocks of columns a turn; `split` waves share the rows, each with its range of
// the columns.  Lane (i, g) has row i and of every block the 16-byte piece g, whose word t belongs to columns 32 t + 8 g + (0 .. 7):
// a matrix operation takes 32 columns in a row, so that groups of 32 have their sums too.
// 50000 x 512 x 5 in 6.9 us (14.6 MB, 3.1 us at a copy's rate; the smallest call takes 3.5): a chain of the vectors' way, their parts, a barrier, the
// codes' expansion (nine instructions for eight weights) and the stores.  With the codes asked for before the vectors 8.7, as loads come back in order; vectors first
// 8.1, and-or in one instruction 7.7, the vectors' loads under no condition 7.2, stores under none 6.9 (a branch waits for what is in flight).  2048 x 8192 x 1 in 7.9: 128 blocks of 16 rows, half of the compute units idle.
template <int PER, int AHEAD>        // groups of a block; blocks of the vectors that a half wave asks for before anything else
__global__ __launch_bounds__(1024) void w4_stream_kernel(W4GemmArgs a)
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
        bias = a.bias && left > 0 ? a.bias[min(r0 + i, a.rows - 1)] : -0.0f;     // (y + -0 is y)
    };
    v4u w[4], sc[PER];
    auto codes = [&](int s) {
        return __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(b + s < b1 && row_at != Q8_OOB ? row_at + 64 * (b + s) : Q8_OOB), 0, 0));
    };
    auto scales = [&](int p) {                                              // words 4 p .. 4 p + 3 of the turn's
        return __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(b * PER + 4 * p < a.lds && scale_at != Q8_OOB ? scale_at + 4 * (b * PER + 4 * p) : Q8_OOB), 0, 0));
    };
    // ---- the vectors, a half wave per block of columns, four values a lane; the first ones are asked for before the codes, which come from farther
    // away: loads come back in order
    float *s_scale = (float *)(s_x + (size_t)n * a.pitch);
    const int q = lane & 31, units = n * a.nb, halves = 2 * waves;
    const __amdgpu_buffer_rsrc_t rx = q8_rsrc(a.X, 4 * ((size_t)(n - 1) * a.ldx + a.cols));
    auto load = [&](int u) {
        const int j = u / a.nb, k = (u - j * a.nb) * W4_BLOCK + 4 * q;
        const unsigned off = 4u * ((unsigned)j * (unsigned)a.ldx + k);
        v4u v = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)(u < units && k + 3 < a.cols ? off : Q8_OOB), 0, 0));
        if (a.cols & 3) {                                                   // the row's last piece
#pragma unroll
            for (int e = 0; e < 3; ++e) v[e] |= __builtin_amdgcn_raw_buffer_load_b32(rx, (int)(u < units && k + 3 >= a.cols && k + e < a.cols ? off + 4 * e : Q8_OOB), 0, 0);
        }
        return __builtin_bit_cast(v4f, v);
    };
    auto put = [&](int u, v4f v) {
        if (u >= units) return;                                             // (a half wave as one)
        const int j = u / a.nb, blk = u - j * a.nb;
        const float top = w4_group_max<32>(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
        float inv;
        const float sx = parts_scale(top, inv);
        uint2 hi, lo;
        parts4(v[0], v[1], v[2], v[3], inv, hi, lo);
        uint8_t *at = s_x + (size_t)j * a.pitch + blk * W4_SPLIT + 8 * q;
        *(uint2 *)at = hi;
        *(uint2 *)(at + W4_SPLIT / 2) = lo;
        if (q == 0) s_scale[blk * 16 + j] = sx;
    };
    const int u0 = tid >> 5;
    v4f xv[AHEAD];
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) xv[t] = load(u0 + t * halves);
    rows_of(tile);
#pragma unroll
    for (int s = 0; s < 4; ++s) w[s] = codes(s);
#pragma unroll
    for (int p = 0; p < PER; ++p) sc[p] = scales(p);
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) put(u0 + t * halves, xv[t]);
    for (int u = u0 + AHEAD * halves; u < units; u += halves) put(u, load(u));
    __syncthreads();

    v4f *s_sum = (v4f *)(s_scale + 16 * a.nb);
    const unsigned magic = w4_magic();
    v4f total = {0.0f, 0.0f, 0.0f, 0.0f};
    unsigned most = 0;                                                      // the largest word of scales of this lane's rows
    const uint8_t *px = s_x + (size_t)min(i, n - 1) * a.pitch + 16 * g;
    // rows r0 .. r0 + 15 of all vectors, dropped past the end instead of branches (pitches are at most 2^24)
    auto store = [&](int r0, v4f y, float add) {
        const int some = min(16, a.rows - r0);
        const __amdgpu_buffer_rsrc_t ry = q8_rsrc(a.Y + r0, 4 * ((size_t)(n - 1) * a.ldy + some));
        const unsigned at = i < some ? 4u * i : Q8_OOB;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(y[v] + add), ry, (int)(4 * g + v < n ? at + 4u * (unsigned)(4 * g + v) * (unsigned)a.ldy : Q8_OOB), 0, 0);
    };
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
                    most = max(most, e);
                }
                const v8h wv = w4_expand(cw[s][t], z1, z2, magic);
                const v4f none = {0.0f, 0.0f, 0.0f, 0.0f};
                const uint8_t *x = px + (at + s) * W4_SPLIT + 64 * t;
                hi = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)x, wv, t % (4 / PER) == 0 ? none : hi, 0, 0, 0);
                lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)(x + W4_SPLIT / 2), wv, t % (4 / PER) == 0 ? none : lo, 0, 0, 0);
                if (t % (4 / PER) == 4 / PER - 1) {
                    const v4f sx = *(const v4f *)(s_scale + (at + s) * 16 + 4 * g);
#pragma unroll
                    for (int v = 0; v < 4; ++v) total[v] = fmaf((hi[v] + lo[v]) * sw, sx[v], total[v]);      // (sw sx alone may pass fp32's range)
                }
            }
        }
        if (!last) continue;
        if (__builtin_expect(__any(most > W4_LARGE), 0)) {
            // scales so large that a sum times one may have passed fp32's range: these rows' columns again, the vectors' powers of two first where they are below one
            total = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
            const size_t row = (size_t)min(16 * from + i, a.rows - 1);
            const uint8_t *pw = a.W + row * a.ldw + 16 * g;
            const unsigned *ps = a.sw + row * a.lds;
#pragma unroll 1
            for (int k = b0; k < b1; ++k) {
                const v4u c = *(const v4u *)(pw + 64 * k);
                const v4f sx = *(const v4f *)(s_scale + k * 16 + 4 * g);
                v4f hi = {0.0f, 0.0f, 0.0f, 0.0f}, lo = hi;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int word = k * PER + t / (4 / PER);
                    const unsigned e = word < a.ng ? ps[word] : 0u;
                    v2h z1, z2;
                    w4_zeros(e, z1, z2);
                    const v8h wv = w4_expand(c[t], z1, z2, magic);
                    const uint8_t *x = px + k * W4_SPLIT + 64 * t;
                    hi = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)x, wv, hi, 0, 0, 0);
                    lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const v8h *)(x + W4_SPLIT / 2), wv, lo, 0, 0, 0);
                    if (t % (4 / PER) != 4 / PER - 1) continue;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        total[v] = fmaf((hi[v] + lo[v]) * fminf(sx[v], 1.0f) * __uint_as_float(e & 0xffff0000u), fmaxf(sx[v], 1.0f), total[v]);
                        hi[v] = lo[v] = 0.0f;
                    }
                }
            }
        }
        most = 0;
        const v4f sum = total;
        total = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        if (split > 1) { s_sum[wave * 64 + lane] = sum; break; }
        // lane (i, g): row i, vectors 4 g + (0 .. 3)
        store(16 * from, sum, add);
    }
    if (split == 1) return;
    __syncthreads();                                                        // the ranges' sums, in one order
    const int from = blockIdx.x + gridDim.x * (wave / split);
    if (part || from >= tiles) return;
    v4f sum = s_sum[wave * 64 + lane];
    for (int p = 1; p < split; ++p)
        if (p * a.span < a.nb) sum += s_sum[(wave + p) * 64 + lane];
    store(16 * from, sum, a.bias ? a.bias[min(16 * from + i, a.rows - 1)] : -0.0f);
}

// split: waves for a row's columns, a power of two, at most `waves`.  A part is a multiple of four blocks of columns, so that the last ones
// may have none: these leave zeros, which are not added.
template <int PER> static q8_status launch_stream_w4(q8_ctx *ctx, W4GemmArgs &a, int waves, int split)
{
    static Q8OncePerDevice once;
    a.split = split;
    a.span = ((a.nb + split - 1) / split + 3) / 4 * 4;
    a.pitch = a.nb * W4_SPLIT + 16;
    const int tiles = (a.rows + 15) / 16, per = waves / split;
    int blocks = (tiles + per - 1) / per;
    if (split == 1 && blocks > 512) blocks = 512;
    const size_t smem = (size_t)a.n * a.pitch + 64 * a.nb + (split > 1 ? 1024 * waves : 0);
    // one block of a vector is all that a half wave has: 768 x 256 x 1 3.6 against 3.8; three ahead 2048 x 8192 x 1 8.0 against 9.1 one by one
    void (*const kernel)(W4GemmArgs) = a.n * a.nb <= 2 * waves ? w4_stream_kernel<PER, 1> : w4_stream_kernel<PER, 3>;
    const q8_status st = smem > 65536 ? q8i_lds(ctx, once, (const void *)w4_stream_kernel<PER, 3>, W4_STREAM_LDS, "w4 product") : Q8_OK;
    if (st) return st;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product w4");
}

// ------------------------------------------------------------------------------ many vectors ----

// A vector's parts and scale, a block per vector.
__global__ __launch_bounds__(256) void w4_parts_kernel(const float *X, int cols, int ldx, int nb, uint8_t *parts, float *sx)
{
    __shared__ float s_max[4];
    const int j = blockIdx.x, tid = threadIdx.x;
    const float *x = X + (size_t)j * ldx;
    auto load = [&](int k) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (k + 3 < cols) return *(const float4 *)(x + k);
        if (k < cols) v.x = x[k];
        if (k + 1 < cols) v.y = x[k + 1];
        if (k + 2 < cols) v.z = x[k + 2];
        return v;
    };
    float4 keep[2];                                                         // the first 2048 columns stay in registers
    float m = 0.0f;
    for (int t = 0; t * 1024 < nb * W4_BLOCK; ++t) {
        const float4 v = load(t * 1024 + 4 * tid);
        if (t == 0) keep[0] = v;
        if (t == 1) keep[1] = v;
        m = fmaxf(m, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
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

// The tile of a block.  Consecutive blocks run on different XCDs, each with an L2 cache of its own: each XCD gets a range of the tiles in a row, those
// of the same rows one after the other, so that it reads its rows' codes from memory once.
__device__ __forceinline__ unsigned w4_tile_of()
{
    const unsigned total = gridDim.x, per = total / 8, over = total % 8, xcd = blockIdx.x % 8, idx = blockIdx.x / 8;
    return xcd * per + min(xcd, over) + idx;
}

template <int PER> struct W4Words;                                          // a block's words of a row, in one load
template <> struct W4Words<1> { typedef unsigned type; };
template <> struct W4Words<2> { typedef v2u type; };
template <> struct W4Words<4> { typedef v4u type; };

// Block of WM x WN waves, each with 32 TM rows x 32 TN vectors; the vectors' parts come in stages of 64 columns (256 bytes a vector) from memory to
// LDS, one on its way while the one before is multiplied; each wave reads its rows' codes (64 bytes for two stages) by itself, the next ones ahead.
// Lane (i, h) of a row tile has the 16-byte pieces h and 2 + h of row i: word t of piece 2 p + h belongs to columns 32 t + 16 p + 8 h + (0 .. 7),
// operation (t, p) of a block to columns 32 t + 16 p + (0 .. 15).  In LDS a vector's 16 pieces (hi, lo) are exchanged by its number mod 16, so that
// lanes that read together find theirs on different banks.
// KS > 1: KS such groups of waves take turns at the blocks of columns; their sums meet in LDS, in one order.  PAST: the results go past the caches.
// 50000 x 512 x 1024 in 104 us (least of 20 launches; the median 111), 112 with the parts' launch in calls among others: 105 GFLOP in two products, 1.0 PFLOP/s where the
// library's largest fp16 product has 1.09, beside 205 MB of results; 140 while each store stood in a branch of its own and waited for the one before.  63644 x 620 x 77 in
// 21.7 (45 MB).
template <int PER, int WM, int WN, int TM, int TN, int KS, bool PAST>
__global__ __launch_bounds__(64 * WM * WN * KS, TM * TN <= 4 ? 2 : 1) void w4_gemm_kernel(W4GemmArgs a)
{
    constexpr int VECS = 32 * WN * TN, THREADS = 64 * WM * WN, STAGE = VECS * 256, LX = VECS * 16 / THREADS, EACH = 4 / PER;      // EACH: operations t of a group
    static_assert(VECS * 16 % THREADS == 0, "even shares of a stage");
    typedef typename W4Words<PER>::type Words;
    extern __shared__ __align__(16) uint8_t s_all[];                        // [KS][2][STAGE]
    const int ks = KS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS) : 0, tid = (int)threadIdx.x - ks * THREADS;
    uint8_t *s_x = s_all + ks * 2 * STAGE;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM, i = lane & 31, h = lane >> 5;
    const unsigned tile = w4_tile_of(), tr = tile / (unsigned)a.col_tiles, tc = tile % (unsigned)a.col_tiles;
    const int r0 = 32 * TM * ((int)tr * WM + wm), c0 = (int)tc * VECS, left = min(VECS, a.n - c0);
    const __amdgpu_buffer_rsrc_t rx = q8_rsrc(a.parts + (size_t)c0 * a.nb * W4_SPLIT, (size_t)left * a.nb * W4_SPLIT);
    unsigned ox[LX];                                                        // place p of a stage: vector p / 16 (beyond the last: the last again)
#pragma unroll
    for (int u = 0; u < LX; ++u) {
        const int p = u * THREADS + tid, v = p >> 4, piece = (p & 15) ^ (v & 15);
        ox[u] = (unsigned)min(v, left - 1) * (unsigned)(a.nb * W4_SPLIT) + (piece >> 3) * (W4_SPLIT / 2) + 16u * (piece & 7);
    }
    auto request = [&](int stage) {
        uint8_t *at = s_x + (stage & 1) * STAGE + wave * 1024;
#pragma unroll
        for (int u = 0; u < LX; ++u) q8_to_lds(rx, at + u * THREADS * 16, ox[u], (stage >> 1) * W4_SPLIT + (stage & 1) * 128);
    };
    const uint8_t *pw[TM];
    const unsigned *ps[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const size_t row = (size_t)min(r0 + 32 * t + i, a.rows - 1);
        pw[t] = a.W + row * a.ldw + 16 * h;
        ps[t] = a.sw + row * a.lds;
    }
    v4u w[TM][2], cw[TM][2];
    Words sc[TM];
    unsigned cs[TM][PER];
    auto codes = [&](int b) {
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            w[t][0] = *(const v4u *)(pw[t] + 64 * b);
            w[t][1] = *(const v4u *)(pw[t] + 64 * b + 32);
            sc[t] = *(const Words *)(ps[t] + b * PER);
        }
    };
    v16f acc[TM][TN], sum[TM][TN];
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][u][e] = 0.0f;
    const int lx = (32 * wn * TN + i) * 256, twist = i & 15;
    v2h z1[TM], z2[TM];
    unsigned most = 0;                                                      // the largest word of scales of this lane's rows
    const unsigned magic = w4_magic();
    // half a block: operations t = 2 half, 2 half + 1
    auto multiply = [&](auto half_) {
        constexpr int half = decltype(half_)::value;
        const uint8_t *px = s_x + half * STAGE + lx;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            constexpr int t0 = 2 * half;
            const int t = t0 + q, group = t / EACH;
            const bool begins = t % EACH == 0;
            if (begins) {
#pragma unroll
                for (int m = 0; m < TM; ++m) w4_zeros(cs[m][group], z1[m], z2[m]);
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int piece = 4 * q + 2 * p + h;
                v8h xh[TN], xl[TN];
#pragma unroll
                for (int u = 0; u < TN; ++u) {
                    xh[u] = *(const v8h *)(px + u * 32 * 256 + 16 * (piece ^ twist));
                    xl[u] = *(const v8h *)(px + u * 32 * 256 + 16 * ((8 + piece) ^ twist));
                }
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const v8h wv = w4_expand(cw[m][p][t], z1[m], z2[m], magic);
                    const v16f none = {};
#pragma unroll
                    for (int u = 0; u < TN; ++u) sum[m][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xh[u], wv, begins && p == 0 ? none : sum[m][u], 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < TN; ++u) sum[m][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xl[u], wv, sum[m][u], 0, 0, 0);
                }
            }
            if (t % EACH == EACH - 1) {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const float sw = __uint_as_float(cs[m][group] & 0xffff0000u);
#pragma unroll
                    for (int u = 0; u < TN; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[m][u][e] = fmaf(sum[m][u][e], sw, acc[m][u][e]);
                }
            }
        }
    };
    const int turns = (a.nb + KS - 1) / KS;
    if (ks < a.nb) {
        codes(ks);
        request(2 * ks);
    }
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
        const int b = turn * KS + ks;
        const bool more = b + KS < a.nb;
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            cw[t][0] = w[t][0];
            cw[t][1] = w[t][1];
#pragma unroll
            for (int p = 0; p < PER; ++p) {                                 // (past the last group: anything)
                unsigned word;
                if constexpr (PER == 1) word = sc[t];
                else word = sc[t][p];
                cs[t][p] = b * PER + p < a.ng ? word : 0u;
                most = max(most, cs[t][p]);
            }
        }
        q8_stores_performed();                                              // (what this wave asked for is in LDS: the barrier alone does not wait for it)
        __syncthreads();                                                    // this stage is there, the other one is free
        if (b < a.nb) request(2 * b + 1);
        if (more) codes(b + KS);
        if (b < a.nb) multiply(std::integral_constant<int, 0>());
        q8_stores_performed();
        __syncthreads();
        if (more) request(2 * (b + KS));
        if (b < a.nb) multiply(std::integral_constant<int, 1>());
    }
    if constexpr (KS > 1) {
        // the groups' sums, a group's where its stages were: [wave][t][u][e][lane], and its largest words: [thread]
        constexpr int WORDS = TM * TN * 16 * THREADS;
        static_assert(STAGE * 2 >= (WORDS + THREADS) * 4, "a group's sums fit where its stages were");
        __syncthreads();
        float *mine = (float *)s_x + wave * TM * TN * 1024 + lane;
        if (ks > 0) {
            ((unsigned *)s_x)[WORDS + tid] = most;
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int u = 0; u < TN; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) mine[((t * TN + u) * 16 + e) * 64] = acc[t][u][e];
        }
        __syncthreads();
        if (ks > 0) return;
#pragma unroll
        for (int g = 1; g < KS; ++g) {
            const float *o = (const float *)(s_all + g * 2 * STAGE) + wave * TM * TN * 1024 + lane;
            most = max(most, ((const unsigned *)(s_all + g * 2 * STAGE))[WORDS + tid]);
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int u = 0; u < TN; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[t][u][e] += o[((t * TN + u) * 16 + e) * 64];
        }
    }
    // Scales so large that sums may have passed fp32's range before the vectors' powers of two: this wave's tile again, by the wave for itself and with the parts
    // from memory, each group's sums times both, the power of two first where it is below one.  (A tile of vectors at a time: no more registers than the loop above.)
    const bool again = __any(most > W4_LARGE);
    if (__builtin_expect(again, 0)) {
#pragma unroll
        for (int u = 0; u < TN; ++u) {
            const uint8_t *pv = a.parts + (size_t)min(c0 + 32 * (wn * TN + u) + i, a.n - 1) * a.nb * W4_SPLIT + 16 * h;
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[m][u] = (v16f){};
#pragma unroll 1
            for (int b = 0; b < a.nb; ++b, pv += W4_SPLIT) {
                codes(b);
#pragma unroll
                for (int m = 0; m < TM; ++m)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        unsigned word;                                      // (past the last group: anything)
                        if constexpr (PER == 1) word = sc[m];
                        else word = sc[m][t / EACH];
                        word = b * PER + t / EACH < a.ng ? word : 0u;
                        w4_zeros(word, z1[m], z2[m]);
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const v8h wv = w4_expand(w[m][p][t], z1[m], z2[m], magic);
                            const v16f none = {};
                            sum[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const v8h *)(pv + 64 * t + 32 * p), wv, t % EACH == 0 && p == 0 ? none : sum[0][0], 0, 0, 0);
                            sum[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const v8h *)(pv + W4_SPLIT / 2 + 64 * t + 32 * p), wv, sum[0][0], 0, 0, 0);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        if (t % EACH != EACH - 1) continue;
                        const float sw = __uint_as_float(word & 0xffff0000u);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const v4f f = *(const v4f *)(a.sx + c0 + 32 * (wn * TN + u) + 8 * q + 4 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[m][u][4 * q + e] = fmaf(sum[0][0][4 * q + e] * fminf(f[e], 1.0f) * sw, fmaxf(f[e], 1.0f), acc[m][u][4 * q + e]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
    }
    // lane (i, h): row i of a row tile, vectors 8 q + 4 h + (0 .. 3) of a tile of vectors.
    // (All loads first, and stores that are dropped past the end of eight vectors instead of branches: a branch would wait for the store before.)
    const int row = r0 + i;
    v4f sx[TN][4];                                                          // the vectors' scales (room for whole tiles is there)
#pragma unroll
    for (int u = 0; u < TN; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const v4f f = *(const v4f *)(a.sx + c0 + 32 * (wn * TN + u) + 8 * q + 4 * h), one = {1.0f, 1.0f, 1.0f, 1.0f};
            sx[u][q] = again ? one : f;
        }
    float bias[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) bias[t] = a.bias ? a.bias[min(row + 32 * t, a.rows - 1)] : -0.0f;       // (y + -0 is y)
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const unsigned at = row + 32 * t < a.rows ? 4u * i : Q8_OOB;        // (pitches are at most 2^25: eight vectors lie below 2^30 bytes)
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v0 = c0 + 32 * (wn * TN + u) + 8 * q, some = min(8, a.n - v0), first = r0 + 32 * t;
                const __amdgpu_buffer_rsrc_t ry = q8_rsrc(a.Y + (size_t)v0 * a.ldy + first, some > 0 && first < a.rows ? 4 * ((size_t)(some - 1) * a.ldy + min(32, a.rows - first)) : 0);
#pragma unroll
                for (int e = 0; e < 4; ++e)                                 // (y times the power of two is exact but for the range)
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_int(fmaf(acc[t][u][4 * q + e], sx[u][q][e], bias[t])), ry,
                                                          (int)(at + 4u * (unsigned)(4 * h + e) * (unsigned)a.ldy), 0, PAST ? 2 : 0);
            }
    }
}

template <int PER, int WM, int WN, int TM, int TN, int KS = 1> static q8_status launch_w4(q8_ctx *ctx, W4GemmArgs &a)
{
    constexpr size_t smem = (size_t)KS * 2 * 32 * WN * TN * 256;
    a.row_tiles = (a.rows + 32 * WM * TM - 1) / (32 * WM * TM);
    a.col_tiles = (a.n + 32 * WN * TN - 1) / (32 * WN * TN);
    const size_t tiles = (size_t)a.row_tiles * a.col_tiles;
    if (tiles * (64 * WM * WN * KS) > 0xffffffffu)                          // a launch has fewer than 2^32 threads
        return q8_fail(ctx, Q8_ERR_SHAPE, "w4 product: %d x %d results are too many for a launch", a.rows, a.n);
    // past the caches where blocks do not share the 64-byte pieces that memory takes, which the caches put together
    const bool past = a.ldy % 16 == 0 && ((uintptr_t)a.Y & 63) == 0;
    void (*const kernel)(W4GemmArgs) = past ? w4_gemm_kernel<PER, WM, WN, TM, TN, KS, true> : w4_gemm_kernel<PER, WM, WN, TM, TN, KS, false>;
    static Q8OncePerDevice once[2];
    const q8_status st = q8i_lds(ctx, once[past], (const void *)kernel, smem, "w4 product");
    if (st) return st;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(64 * WM * WN * KS), smem, ctx->stream, a);
    return q8i_launch_check(ctx, "product w4");
}

// (the rule: q8_route.h)
template <int PER> static q8_status gemm_w4_tiles(q8_ctx *ctx, W4GemmArgs &a, int route)
{
    if constexpr (PER < 4) {
        if (route == Q8_W4_256X64) return launch_w4<PER, 4, 1, 2, 2>(ctx, a);
    }
    switch (route) {
    case Q8_W4_32X32_FOUR: return launch_w4<PER, 1, 1, 1, 1, 4>(ctx, a);
    case Q8_W4_64X32_FOUR: return launch_w4<PER, 2, 1, 1, 1, 4>(ctx, a);
    case Q8_W4_64X32_TWO: return launch_w4<PER, 2, 1, 1, 1, 2>(ctx, a);
    case Q8_W4_128X96: return launch_w4<PER, 4, 1, 1, 3>(ctx, a);
    case Q8_W4_128X64: return launch_w4<PER, 4, 1, 1, 2>(ctx, a);
    default: return launch_w4<PER, 4, 1, 1, 1>(ctx, a);
    }
}

size_t q8i_gemm_w4_scales(int n) { return ((size_t)n + 255) / 256 * 256; }

size_t q8i_gemm_w4_parts(int n, int cols) { return (size_t)n * ((cols + W4_BLOCK - 1) / W4_BLOCK) * W4_SPLIT; }

template <int PER> static q8_status gemm_w4(q8_ctx *ctx, W4GemmArgs &a, int route)
{
    if (route != Q8_W4_STREAM) return gemm_w4_tiles<PER>(ctx, a, route);
    const int tiles = (a.rows + 15) / 16;
    int split = 1;
    while (split < 8 && a.nb > 4 * split && tiles * split < 2048) split *= 2;
    int waves = tiles < 1024 && split == 1 ? 4 : 8;
    if (split == 8 && a.nb > 32 && tiles <= 256) waves = split = 16;
    return launch_stream_w4<PER>(ctx, a, waves, split);
}

q8_status q8i_gemm_w4(q8_ctx *ctx, const q8_mat_w4 *W, const float *X, int n, int ldx, const float *bias, float *Y, int ldy, uint8_t *parts, float *sx)
{
    W4GemmArgs a = {W->data, W->scale, X, parts, sx, bias, Y, W->rows, n, W->cols, W->ld, W->lds, (W->cols + W->group - 1) / W->group, ldx, ldy,
                    (W->cols + W4_BLOCK - 1) / W4_BLOCK, 0, 0, 0, 0, 0};
    const int per = W4_BLOCK / W->group;
    if (n == 1) a.ldx = a.cols, a.ldy = a.rows;                             // (pitches that nothing uses, but bounds are formed with)
    // (results over the vectors: these are read first, as a whole)
    const uintptr_t x0 = (uintptr_t)X, x1 = x0 + 4 * ((size_t)(n - 1) * ldx + a.cols), y0 = (uintptr_t)Y, y1 = y0 + 4 * ((size_t)(n - 1) * ldy + a.rows);
    const int route = q8_w4_route(W->rows, W->cols, n, W->group, ldx <= 1 << 24 && a.ldy <= 1 << 24 && !(x0 < y1 && y0 < x1));
    if (route != Q8_W4_STREAM) {
        hipLaunchKernelGGL(w4_parts_kernel, dim3(n), dim3(256), 0, ctx->stream, X, a.cols, ldx, a.nb, parts, sx);
        const q8_status st = q8i_launch_check(ctx, "parts w4");
        if (st) return st;
    }
    return per == 4 ? gemm_w4<4>(ctx, a, route) : per == 2 ? gemm_w4<2>(ctx, a, route) : gemm_w4<1>(ctx, a, route);
}
