// Rotary positions with one or several axes, on plain rows or fused with the write of K/V
// into the pool (bf16 in, fp32 products, bf16 out), for gfx950.
//
// Pair j of a token's head turns by positions[axis_j] * inv_freq[j]. Angles of far
// positions lose their phase in fp32 (position 10^6 keeps 2^-4 of a radian), so the turn is
// formed and reduced in fp64, in whole revolutions: r = position * (inv_freq / 2 pi),
// minus its nearest integer, and cos and sin of the rest are taken in fp32.
#include <math.h>

#include "pcr_internal.h"

namespace pcr {
namespace {

typedef unsigned short u16;

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxAxes = 4;

// The rotation, in the launch's arguments.
struct RopeArgs {
    double turns[kMaxPairs];      // revolutions per position step
    uint8_t axis[kMaxPairs];
    int32_t half;                 // pairs
    int32_t interleaved;
    float scale, sin_scale;       // of cos and of sin (negated: transposed)
};

__device__ __forceinline__ float to_f32(u16 v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ u16 to_bf16(float v) { return __builtin_bit_cast(u16, (__bf16)v); }

__device__ __forceinline__ void turn(const RopeArgs &ra, const int32_t *positions, int64_t pos_stride, int64_t t, int j,
                                     float *c, float *s)
{
    double r = (double)positions[ra.axis[j] * pos_stride + t] * ra.turns[j];
    r -= rint(r);
    sincospif(2.f * (float)r, s, c);
    *c *= ra.scale;
    *s *= ra.sin_scale;
}

// Element x of a head's row after the rotation.
__device__ __forceinline__ u16 rotated(const u16 *row, int x, const RopeArgs &ra, const int32_t *positions,
                                       int64_t pos_stride, int64_t t)
{
    if (x >= 2 * ra.half) return row[x];
    const int j = ra.interleaved ? x >> 1 : x % ra.half;
    const bool second = ra.interleaved ? x & 1 : x >= ra.half;
    const int i1 = ra.interleaved ? 2 * j : j, i2 = ra.interleaved ? 2 * j + 1 : j + ra.half;
    float c, s;
    turn(ra, positions, pos_stride, t, j, &c, &s);
    const float a = to_f32(row[i1]), b = to_f32(row[i2]);
    return to_bf16(second ? b * c + a * s : a * c - b * s);
}

// One workgroup per token; the whole token is read before any of it is written (in place).
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(const RopeArgs ra, const u16 *x, int64_t x_stride,
                                                             const int32_t *__restrict__ positions, int64_t pos_stride,
                                                             int32_t H, int32_t D, u16 *out, int64_t out_stride)
{
    const int64_t t = blockIdx.x;
    for (int h = 0; h < H; ++h) {
        const u16 *row = x + t * x_stride + (int64_t)h * D;
        u16 *orow = out + t * out_stride + (int64_t)h * D;
        const int e = threadIdx.x;
        const u16 v = e < D ? rotated(row, e, ra, positions, pos_stride, t) : (u16)0;
        __syncthreads();
        if (e < D) orow[e] = v;
    }
}

__global__ __launch_bounds__(kThreads) void rope_append_kernel(
    const RopeArgs ra, u16 *__restrict__ pool_k, u16 *__restrict__ pool_v, int32_t num_blocks, int32_t Hkv, int32_t D,
    const u16 *__restrict__ k_new, int64_t k_stride, const u16 *__restrict__ v_new, int64_t v_stride,
    const int32_t *__restrict__ positions, int64_t pos_stride, const int32_t *__restrict__ slot_mapping)
{
    const int64_t t = blockIdx.x;
    const int32_t slot = slot_mapping[t];
    if (slot < 0 || slot / kBlockSize >= num_blocks) return;
    const int64_t blk = slot / kBlockSize;
    const int o = slot % kBlockSize;
    for (int i = threadIdx.x; i < Hkv * D; i += kThreads) {
        const int g = i / D, e = i % D;
        pool_k[((blk * Hkv + g) * kBlockSize + o) * D + e] =
            rotated(k_new + t * k_stride + (int64_t)g * D, e, ra, positions, pos_stride, t);
        pool_v[((blk * Hkv + g) * D + e) * kBlockSize + o] = v_new[t * v_stride + i];
    }
}

// The checks of a rotation, and its launch arguments.
pcr_status rope_args(const pcr_rope *rope, int32_t head_dim, int32_t inverse, const char *who, RopeArgs *ra)
{
    if (!rope || !rope->inv_freq) return fail(PCR_ERR_INVALID_ARG, "%s: rope or its inv_freq is NULL", who);
    if (rope->rotary_dim <= 0 || rope->rotary_dim % 16 || rope->rotary_dim > head_dim)
        return fail(PCR_ERR_UNSUPPORTED, "%s: rotary_dim %d is not a positive multiple of 16 up to head_dim %d", who,
                    rope->rotary_dim, head_dim);
    if (rope->num_axes < 1 || rope->num_axes > kMaxAxes)
        return fail(PCR_ERR_INVALID_ARG, "%s: num_axes must be 1 to %d", who, kMaxAxes);
    if (!isfinite(rope->scale)) return fail(PCR_ERR_INVALID_ARG, "%s: scale is not finite", who);
    ra->half = rope->rotary_dim / 2;
    ra->interleaved = rope->interleaved != 0;
    ra->scale = rope->scale;
    ra->sin_scale = inverse ? -rope->scale : rope->scale;
    for (int j = 0; j < ra->half; ++j) {
        const int32_t a = rope->pair_axis ? rope->pair_axis[j] : 0;
        if (a < 0 || a >= rope->num_axes)
            return fail(PCR_ERR_INVALID_ARG, "%s: pair %d has axis %d of %d", who, j, a, rope->num_axes);
        if (!isfinite(rope->inv_freq[j])) return fail(PCR_ERR_INVALID_ARG, "%s: inv_freq[%d] is not finite", who, j);
        ra->axis[j] = (uint8_t)a;
        ra->turns[j] = (double)rope->inv_freq[j] / (2.0 * M_PI);
    }
    return PCR_OK;
}

// T rows of `width` elements at `stride` (multiples of 8 elements, 16-byte aligned).
pcr_status check_rows(const void *x, int64_t stride, int64_t width, const char *what, const char *who)
{
    if (!x) return fail(PCR_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    if ((uintptr_t)x & 15) return fail(PCR_ERR_INVALID_ARG, "%s: %s must be 16-byte aligned", who, what);
    if (stride < width || stride % 8 || stride > (int64_t)1 << 40)
        return fail(PCR_ERR_INVALID_ARG, "%s: %s stride %lld is not a multiple of 8 of at least %lld", who, what,
                    (long long)stride, (long long)width);
    return PCR_OK;
}

bool rows_overlap(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int32_t T, int64_t width)
{
    const uintptr_t a0 = (uintptr_t)a, a1 = a0 + ((uintptr_t)(T - 1) * a_stride + width) * 2;
    const uintptr_t b0 = (uintptr_t)b, b1 = b0 + ((uintptr_t)(T - 1) * b_stride + width) * 2;
    return a0 < b1 && b0 < a1;
}

hipError_t launch_rows(const RopeArgs &ra, const void *x, int64_t x_stride, const int32_t *positions,
                       int64_t pos_stride, int32_t T, int32_t H, int32_t D, void *out, int64_t out_stride,
                       hipStream_t s)
{
    hipLaunchKernelGGL(rope_rows_kernel, dim3(T), dim3(kThreads), 0, s, ra, static_cast<const u16 *>(x), x_stride,
                       positions, pos_stride, H, D, static_cast<u16 *>(out), out_stride);
    return hipGetLastError();
}

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_rope_append_kv(const pcr_rope *rope, const pcr_kv_pool *pool, const void *q, int64_t q_stride,
                              const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                              const int32_t *positions, int64_t pos_stride, const int32_t *slot_mapping, int32_t T,
                              int32_t num_q_heads, void *q_out, void *stream)
{
    clear_error();
    const char *who = "pcr_rope_append_kv";
    pcr_status st = check_pool(pool, who);
    if (st) return st;
    RopeArgs ra;
    st = rope_args(rope, pool->head_dim, 0, who, &ra);
    if (st) return st;
    if (T < 0 || num_q_heads < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative T or num_q_heads", who);
    if (num_q_heads % pool->num_kv_heads != 0)
        return fail(PCR_ERR_UNSUPPORTED, "%s: num_q_heads %d is not a multiple of num_kv_heads %d", who, num_q_heads,
                    pool->num_kv_heads);
    if (T == 0) return PCR_OK;
    const int64_t kv_width = (int64_t)pool->num_kv_heads * pool->head_dim;
    const int64_t q_width = (int64_t)num_q_heads * pool->head_dim;
    if (!positions || !slot_mapping) return fail(PCR_ERR_INVALID_ARG, "%s: NULL positions or slot_mapping", who);
    if (pos_stride < T && rope->num_axes > 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: pos_stride %lld < T", who, (long long)pos_stride);
    st = check_rows(k_new, k_stride, kv_width, "k_new", who);
    if (!st) st = check_rows(v_new, v_stride, kv_width, "v_new", who);
    if (!st && num_q_heads > 0) st = check_rows(q, q_stride, q_width, "q", who);
    if (!st && num_q_heads > 0) st = check_rows(q_out, q_width, q_width, "q_out", who);
    if (st) return st;
    if (num_q_heads > 0) {
        if (!(q == q_out && q_stride == q_width) && rows_overlap(q, q_stride, q_out, q_width, T, q_width))
            return fail(PCR_ERR_INVALID_ARG, "%s: q and q_out overlap (and are not one array)", who);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (num_q_heads > 0)
        e = launch_rows(ra, q, q_stride, positions, pos_stride, T, num_q_heads, pool->head_dim, q_out, q_width, s);
    if (e == hipSuccess) {
        hipLaunchKernelGGL(rope_append_kernel, dim3(T), dim3(kThreads), 0, s, ra, static_cast<u16 *>(pool->k),
                           static_cast<u16 *>(pool->v), pool->num_blocks, pool->num_kv_heads, pool->head_dim,
                           static_cast<const u16 *>(k_new), k_stride, static_cast<const u16 *>(v_new), v_stride,
                           positions, pos_stride, slot_mapping);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return hip_fail(e, "pcr_rope_append_kv: launch");
    return PCR_OK;
}

pcr_status pcr_rope_rows(const pcr_rope *rope, const void *x, int64_t x_stride, const int32_t *positions,
                         int64_t pos_stride, int32_t T, int32_t num_heads, int32_t head_dim, int32_t inverse,
                         void *out, int64_t out_stride, void *stream)
{
    clear_error();
    const char *who = "pcr_rope_rows";
    if (T < 0 || num_heads <= 0) return fail(PCR_ERR_INVALID_ARG, "%s: T < 0 or num_heads <= 0", who);
    if (head_dim <= 0 || head_dim % 16 || head_dim > 2 * kMaxPairs)
        return fail(PCR_ERR_UNSUPPORTED, "%s: head_dim %d is not a multiple of 16 up to %d", who, head_dim,
                    2 * kMaxPairs);
    RopeArgs ra;
    pcr_status st = rope_args(rope, head_dim, inverse, who, &ra);
    if (st || T == 0) return st;
    if (!positions) return fail(PCR_ERR_INVALID_ARG, "%s: positions is NULL", who);
    if (pos_stride < T && rope->num_axes > 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: pos_stride %lld < T", who, (long long)pos_stride);
    const int64_t width = (int64_t)num_heads * head_dim;
    st = check_rows(x, x_stride, width, "x", who);
    if (!st) st = check_rows(out, out_stride, width, "out", who);
    if (st) return st;
    if (!(x == out && x_stride == out_stride) && rows_overlap(x, x_stride, out, out_stride, T, width))
        return fail(PCR_ERR_INVALID_ARG, "%s: x and out overlap (and are not one array)", who);
    const hipError_t e = launch_rows(ra, x, x_stride, positions, pos_stride, T, num_heads, head_dim, out, out_stride,
                                     static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "pcr_rope_rows: launch");
    return PCR_OK;
}

}  // extern "C"
