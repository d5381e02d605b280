// Attention of a tree of drafted tokens over the paged cache for gfx950 (bf16 in, fp32 accumulate,
// bf16 out): row i of a sequence sees the cached tokens and the nodes of its own words (itself and its
// ancestors, as pcr_draft_tree leaves them), K/V read through the block table.
//
// The rows of one (sequence, kv head) share its keys, so they are packed (row r = node r / G,
// head-in-group r % G) and taken in groups of up to 32, the columns of a wave's matrix tiles
// (tree_wave.h): K and V go from memory into registers once for all of them. A workgroup takes
// one group; its waves share out the keys and merge in LDS.
#include <algorithm>
#include <type_traits>

#include "pcr_internal.h"
#include "tree_wave.h"

namespace pcr {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStepKeys = tree_wave::kStepKeys;

struct TreeArgs {
    int32_t num_blocks, Hkv, Hq, max_blocks, B, T, words;
    float scale_log2;
};

// Grid (row groups, kv heads, sequences).
template <int D, int NC, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(1))) void tree_rows_kernel(
    const TreeArgs a, const u16 *__restrict__ q, const u16 *__restrict__ pool_k, const u16 *__restrict__ pool_v,
    const int32_t *__restrict__ block_tables, const int32_t *__restrict__ prefix_lens,
    const int32_t *__restrict__ cu_nodes, const uint64_t *__restrict__ visible, u16 *__restrict__ out)
{
    constexpr int MT = D / 16;
    __shared__ f32x4 part_o[WAVES - 1][NC][MT][64];
    __shared__ f32x2 part_ml[WAVES - 1][NC][64];
    const int lane = threadIdx.x & 63, c = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int g = blockIdx.y, b = blockIdx.z, G = a.Hq / a.Hkv;
    const int t0 = cu_nodes[b], nodes = min(cu_nodes[b + 1], a.T) - t0, prefix = prefix_lens[b];
    if (t0 < 0 || nodes <= 0 || prefix < 0) return;
    tree_wave::Rows rw{visible + (int64_t)t0 * a.words, a.words, prefix, nodes, (int)blockIdx.x * 16 * NC, 0, G};
    rw.rows = nodes * G - rw.row0;
    if (rw.rows <= 0) return;
    const int n_keys = (int)min((int64_t)prefix + nodes, (int64_t)a.max_blocks * kBlockSize);
    const int steps = (n_keys + kStepKeys - 1) / kStepKeys, per = (steps + WAVES - 1) / WAVES;
    const int kbeg = wave * per * kStepKeys, kend = min(n_keys, kbeg + per * kStepKeys);
    f32x4 o[NC][MT];
    float m[NC], l[NC];
    if (kbeg < kend) {
        tree_wave::chunk<D, NC, 2, true>(q + ((int64_t)t0 * a.Hq + g * G) * D, (int64_t)a.Hq * D, rw, pool_k, pool_v,
                                         a.num_blocks, a.Hkv, g, block_tables + (int64_t)b * a.max_blocks,
                                         (n_keys - 1) >> 4, kbeg, kend, a.scale_log2, o, m, l);
    } else {
#pragma unroll
        for (int t = 0; t < NC; ++t) {
            m[t] = tree_wave::kNoMax;
            l[t] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
    }
    // Waves 1.. leave O (lane layout), max and sum in LDS; wave 0 merges.
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < NC; ++t) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) part_o[wave - 1][t][mt][lane] = o[t][mt];
            part_ml[wave - 1][t][lane] = f32x2{m[t], l[t]};
        }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        float M = m[t];
        for (int w = 0; w < WAVES - 1; ++w) M = fmaxf(M, part_ml[w][t][lane][0]);
        const float a0 = __builtin_amdgcn_exp2f(m[t] - M);
        float L = l[t] * a0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[t][mt] *= a0;
        for (int w = 0; w < WAVES - 1; ++w) {
            const f32x2 ml = part_ml[w][t][lane];
            const float aw = __builtin_amdgcn_exp2f(ml[0] - M);
            L += aw * ml[1];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[t][mt] += aw * part_o[w][t][mt][lane];
        }
        const int r = 16 * t + c;
        if (r >= rw.rows) continue;
        const int pr = rw.row0 + r, node = pr / G, h = pr - node * G;
        const float inv = L == 0.f ? 0.f : 1.f / L;     // a row that sees nothing is zeros
        u16 *orow = out + ((int64_t)(t0 + node) * a.Hq + g * G + h) * D + 4 * q4;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const bf16x4 v = __builtin_convertvector(o[t][mt] * inv, bf16x4);
            *reinterpret_cast<u32x2 *>(orow + 16 * mt) = __builtin_bit_cast(u32x2, v);
        }
    }
}

constexpr int32_t kMaxKeys = 1 << 30;       // positions past a sequence's end still fit int32

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

pcr_status pcr_tree_attn_workspace_size(int32_t B, int32_t total_nodes, int32_t num_q_heads, int32_t num_kv_heads,
                                        int32_t head_dim, int32_t max_keys, int64_t *bytes)
{
    clear_error();
    const char *who = "pcr_tree_attn_workspace_size";
    if (!bytes) return fail(PCR_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    *bytes = 0;
    pcr_status st = check_layout(kBlockSize, num_kv_heads, head_dim, who);
    if (!st) st = check_heads(num_q_heads, num_kv_heads, who);
    if (st) return st;
    if (B < 0 || total_nodes < 0 || max_keys < 0)
        return fail(PCR_ERR_INVALID_ARG, "%s: negative B, total_nodes or max_keys", who);
    return PCR_OK;
}

pcr_status pcr_tree_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                         const int32_t *prefix_lens, const int32_t *cu_nodes, const int32_t *host_prefix_lens,
                         const int32_t *host_cu_nodes, int32_t B, const uint64_t *visible, int32_t mask_words,
                         int32_t num_q_heads, float sm_scale, void *out, void *workspace, int64_t workspace_bytes,
                         void *stream)
{
    clear_error();
    const char *who = "pcr_tree_attn";
    pcr_status st = check_pool(pool, who);
    if (st) return st;
    if (B < 0) return fail(PCR_ERR_INVALID_ARG, "%s: B < 0", who);
    if (B == 0) return PCR_OK;
    if (!host_prefix_lens || !host_cu_nodes) return fail(PCR_ERR_INVALID_ARG, "%s: NULL host length arrays", who);
    st = check_heads(num_q_heads, pool->num_kv_heads, who);
    if (st) return st;
    if (!(sm_scale > 0.f) || !(sm_scale < 1e30f)) return fail(PCR_ERR_INVALID_ARG, "%s: bad sm_scale", who);
    if (mask_words < 1 || mask_words > kMaxMaskWords)
        return fail(PCR_ERR_UNSUPPORTED, "%s: mask_words %d is not in 1 .. %d", who, mask_words, kMaxMaskWords);
    if (host_cu_nodes[0] != 0) return fail(PCR_ERR_INVALID_ARG, "%s: cu_nodes[0] must be 0", who);
    const int D = pool->head_dim, G = num_q_heads / pool->num_kv_heads;
    if (B > 65535 || pool->num_kv_heads > 65535) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
    int64_t most = 0;                       // packed rows of a sequence, at most
    for (int32_t b = 0; b < B; ++b) {
        const int64_t n = (int64_t)host_cu_nodes[b + 1] - host_cu_nodes[b];
        if (n < 0 || host_prefix_lens[b] < 0)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d has a negative length", who, b);
        if (n > 64 * mask_words)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d has more nodes than the %d of its words", who, b,
                        64 * mask_words);
        if (n > 0 && host_prefix_lens[b] + n > kMaxKeys)
            return fail(PCR_ERR_UNSUPPORTED, "%s: sequence %d has more than 2^30 keys", who, b);
        if (n > 0 && (host_prefix_lens[b] + n + kBlockSize - 1) / kBlockSize > max_blocks)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d needs more blocks than max_blocks %d", who, b,
                        max_blocks);
        most = std::max(most, n * G);
    }
    const int64_t T = host_cu_nodes[B];
    if (T == 0) return PCR_OK;
    if (T > INT32_MAX / num_q_heads) return fail(PCR_ERR_INVALID_ARG, "%s: too many rows", who);
    if (!q || !out || !block_tables || !prefix_lens || !cu_nodes || !visible)
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL device argument", who);
    if (((uintptr_t)q | (uintptr_t)out) & 15)
        return fail(PCR_ERR_INVALID_ARG, "%s: q/out must be 16-byte aligned", who);
    if ((uintptr_t)visible & 7) return fail(PCR_ERR_INVALID_ARG, "%s: visible must be 8-byte aligned", who);
    const uintptr_t qa = (uintptr_t)q, oa = (uintptr_t)out, bytes = (uintptr_t)T * num_q_heads * D * 2;
    if (qa < oa + bytes && oa < qa + bytes) return fail(PCR_ERR_INVALID_ARG, "%s: q and out overlap", who);
    TreeArgs a{pool->num_blocks, pool->num_kv_heads, num_q_heads, max_blocks, B, (int32_t)T, mask_words,
               sm_scale * kLog2e};
    auto go = [&](auto dim, auto tiles) {
        constexpr int DD = decltype(dim)::value, NC = decltype(tiles)::value;
        const dim3 grid((unsigned)((most + 16 * NC - 1) / (16 * NC)), pool->num_kv_heads, B);
        hipLaunchKernelGGL((tree_rows_kernel<DD, NC, 4>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), a,
                           static_cast<const u16 *>(q), static_cast<const u16 *>(pool->k),
                           static_cast<const u16 *>(pool->v), block_tables, prefix_lens, cu_nodes, visible,
                           static_cast<u16 *>(out));
        return hipGetLastError();
    };
    auto go_d = [&](auto dim) {
        if (most <= 16) return go(dim, std::integral_constant<int, 1>{});
        return go(dim, std::integral_constant<int, 2>{});
    };
    const hipError_t e = D == 128 ? go_d(std::integral_constant<int, 128>{}) : go_d(std::integral_constant<int, 64>{});
    if (e != hipSuccess) return hip_fail(e, "pcr_tree_attn: launch");
    return PCR_OK;
}

}  // extern "C"
