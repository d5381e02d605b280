// Cross attention to an encoder's cached states for gfx950 (bf16 in, fp32 accumulate, bf16
// out): every query row of a sequence attends all n of its encoder's keys, K/V read from
// the paged pool through the block table.
//
// The s * G query rows of one (sequence, kv head) see the same keys, so they are packed
// (row r = token r / G, head-in-group r % G). A wave takes 16 packed rows as the columns of
// the decode routine's tiles (decode_wave.h) and walks all keys.
#include "decode_wave.h"
#include "pcr_internal.h"

namespace pcr {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCols = decode_wave::kMaxCols;

// Grid (row tiles of the longest sequence, Hkv, B), one wave.
template <int D>
__global__ __launch_bounds__(64) void cross_kernel(const u16 *__restrict__ q, const u16 *__restrict__ pool_k,
                                                   const u16 *__restrict__ pool_v, int32_t num_blocks, int32_t Hkv,
                                                   const int32_t *__restrict__ block_tables, int32_t max_blocks,
                                                   const int32_t *__restrict__ key_lens,
                                                   const int32_t *__restrict__ cu_q, int32_t T, int32_t Hq,
                                                   float scale_log2, u16 *__restrict__ out)
{
    constexpr int MT = D / 16;
    const int lane = threadIdx.x, c = lane & 15, q4 = lane >> 4;
    const int g = blockIdx.y, b = blockIdx.z, G = Hq / Hkv;
    const int t0 = cu_q[b], t1 = min(cu_q[b + 1], T);
    const int64_t rows = (int64_t)(t1 - t0) * G, row0 = (int64_t)blockIdx.x * kCols;
    if (t0 < 0 || row0 >= rows) return;
    const bool col = row0 + c < rows;
    const int64_t r = col ? row0 + c : row0;
    const int64_t qrow = (t0 + r / G) * Hq + g * G + r % G;
    const int n = (int)min((int64_t)key_lens[b], (int64_t)max_blocks * kBlockSize);
    f32x4 o[MT];
    float m_run = decode_wave::kNoMax, l_run = 0.f;
    if (n > 0)
        decode_wave::chunk<D, 3, true>(q + qrow * D + 8 * q4, col, pool_k, pool_v, num_blocks, Hkv, g,
                                       block_tables + (int64_t)b * max_blocks, (n - 1) >> 4, 0, n, scale_log2, o, m_run,
                                       l_run);
    else
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = l_run + __shfl_xor(l_run, 16);
    l += __shfl_xor(l, 32);
    if (!col) return;
    const float inv = n > 0 ? 1.f / l : 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const bf16x4 v = __builtin_convertvector(o[mt] * inv, bf16x4);
        *reinterpret_cast<u32x2 *>(out + qrow * D + 16 * mt + 4 * q4) = __builtin_bit_cast(u32x2, v);
    }
}

pcr_status check_heads(int32_t num_q_heads, int32_t num_kv_heads, const char *who)
{
    if (num_q_heads <= 0 || num_q_heads % num_kv_heads != 0)
        return fail(PCR_ERR_UNSUPPORTED, "%s: num_q_heads %d is not a positive multiple of num_kv_heads %d", who,
                    num_q_heads, num_kv_heads);
    return PCR_OK;
}

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_cross_attn_workspace_size(int32_t B, int32_t total_rows, int32_t num_q_heads, int32_t num_kv_heads,
                                         int32_t head_dim, int32_t max_keys, int64_t *bytes)
{
    clear_error();
    const char *who = "pcr_cross_attn_workspace_size";
    if (!bytes) return fail(PCR_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    *bytes = 0;
    pcr_status st = check_layout(kBlockSize, num_kv_heads, head_dim, who);
    if (!st) st = check_heads(num_q_heads, num_kv_heads, who);
    if (st) return st;
    if (B < 0 || total_rows < 0 || max_keys < 0)
        return fail(PCR_ERR_INVALID_ARG, "%s: negative B, total_rows or max_keys", who);
    return PCR_OK;
}

pcr_status pcr_cross_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                          const int32_t *key_lens, const int32_t *cu_q, const int32_t *host_key_lens,
                          const int32_t *host_cu_q, int32_t B, int32_t num_q_heads, float sm_scale, void *out,
                          void *workspace, int64_t workspace_bytes, void *stream)
{
    clear_error();
    const char *who = "pcr_cross_attn";
    (void)workspace;
    (void)workspace_bytes;
    pcr_status st = check_pool(pool, who);
    if (st) return st;
    if (B < 0) return fail(PCR_ERR_INVALID_ARG, "%s: B < 0", who);
    if (B == 0) return PCR_OK;
    if (!host_key_lens || !host_cu_q) return fail(PCR_ERR_INVALID_ARG, "%s: NULL host length arrays", who);
    st = check_heads(num_q_heads, pool->num_kv_heads, who);
    if (st) return st;
    if (!(sm_scale > 0.f) || !(sm_scale < 1e30f)) return fail(PCR_ERR_INVALID_ARG, "%s: bad sm_scale", who);
    if (host_cu_q[0] != 0) return fail(PCR_ERR_INVALID_ARG, "%s: cu_q[0] must be 0", who);
    const int D = pool->head_dim, G = num_q_heads / pool->num_kv_heads;
    int64_t most = 0;
    for (int32_t b = 0; b < B; ++b) {
        const int64_t s = (int64_t)host_cu_q[b + 1] - host_cu_q[b];
        if (s < 0 || host_key_lens[b] < 0)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d has a negative length", who, b);
        if (s > 0 && ((int64_t)host_key_lens[b] + kBlockSize - 1) / kBlockSize > max_blocks)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d needs more blocks than max_blocks %d", who, b,
                        max_blocks);
        most = s > most ? s : most;
    }
    const int64_t T = host_cu_q[B];
    if (T == 0) return PCR_OK;
    if (T > INT32_MAX / num_q_heads) return fail(PCR_ERR_INVALID_ARG, "%s: too many rows", who);
    if (!q || !out || !block_tables || !key_lens || !cu_q)
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL device argument", who);
    if (((uintptr_t)q | (uintptr_t)out) & 15)
        return fail(PCR_ERR_INVALID_ARG, "%s: q/out must be 16-byte aligned", who);
    const uintptr_t qa = (uintptr_t)q, oa = (uintptr_t)out, bytes = (uintptr_t)T * num_q_heads * D * 2;
    if (qa < oa + bytes && oa < qa + bytes) return fail(PCR_ERR_INVALID_ARG, "%s: q and out overlap", who);
    if (B > 65535 || pool->num_kv_heads > 65535) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
    const dim3 grid((unsigned)((most * G + kCols - 1) / kCols), pool->num_kv_heads, B);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(64), 0, static_cast<hipStream_t>(stream), static_cast<const u16 *>(q),
                           static_cast<const u16 *>(pool->k), static_cast<const u16 *>(pool->v), pool->num_blocks,
                           pool->num_kv_heads, block_tables, max_blocks, key_lens, cu_q, (int32_t)T, num_q_heads,
                           sm_scale * kLog2e, static_cast<u16 *>(out));
    };
    if (D == 128) launch(cross_kernel<128>);
    else launch(cross_kernel<64>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "pcr_cross_attn: launch");
    return PCR_OK;
}

}  // extern "C"
