// Attention of a tree of drafted tokens over the paged cache for gfx950 (bf16 in, fp32 accumulate,
// bf16 out): row i of a sequence sees the cached tokens and the nodes of its own words (itself and its
// ancestors, as pcr_draft_tree leaves them), K/V read through the block table.
//
// The rows of one (sequence, kv head) share its keys, so they are packed (row r = node r / G,
// head-in-group r % G). Batches whose sequences have up to 32 packed rows each are bound by reading K and
// V: the rows are the columns of a wave's matrix tiles (tree_wave.h), K and V go from memory into
// registers once for all of them, and the keys of all sequences are shared out as those of cross attention
// are (rows_kernel.h). Any other batch runs on the row tiles of the prefill kernel (attn.hip) with bits
// for the causal bound.
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

constexpr int32_t kMaxKeys = 1 << 30;       // positions past a sequence's end still fit int32
// Packed rows of a sequence up to which waves hold them as columns. Rows kernel / row tiles, 32 / 8 heads of 128, 64
// sequences: 16 rows over 4096 keys 166 / 195 us, 32 rows 168 / 194, 32 rows over 500-4096 keys 134 / 124, 64 rows over
// 2100-4352 (four tiles of columns, which spill) 303 / 167; 32 rows of 128 sequences of up to 1000 keys, 8 / 8 heads of 64,
// 33 / 58. (Row tiles of 32 sequences of 64 nodes over 7000-8000 keys, 64 / 8 heads of 128: 456 us, 1122 TFLOP/s.)
constexpr int kMaxRows = kTreeMaxCols;

// 32-key steps of n keys (tree_wave.h).
int64_t key_steps(int64_t n) { return (n + 31) / 32; }

}  // namespace

// Constants for two sets of registers where cross attention has three (one sequence, four nodes of 32 / 8
// heads of 128 over 500 and 2000 keys: whole pairs 13.5 and 26.9 us, eight parts 13.8 and 15.2; 8 / 8 heads of
// 64 over 1000 and 4000: 11.5 and 24.1, 14.3 and 13.9). Two tiles of columns leave twice the partial
// results (64 ragged sequences of up to 4096 keys, eight nodes of 32 / 8 heads: even runs 142 us, whole pairs 133). Eight waves of a pair, as cross
// attention has with 64 dims, merge longer than they save: 8 / 8 heads over 2000 keys 16.4 us, four 15.2.
CrossRowsPlan tree_rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t cols,
                             int32_t n_cu)
{
    return rows_plan(steps, pairs, longest, head_dim, n_cu,
                     {head_dim == 128 ? 0.29f : 0.15f, 11.f, cols > 16 ? 1.25f : 1.f, 4});
}

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
    if (B == 0 || total_nodes == 0 || max_keys == 0) return PCR_OK;
    int32_t n_cu = 0;
    st = device_cu_count(&n_cu, who);
    if (st) return st;
    const int64_t rows = (int64_t)total_nodes * (num_q_heads / num_kv_heads);
    const int32_t cols = (int32_t)std::min<int64_t>(rows, kMaxRows);
    // (sequences without nodes count: a plan of parts has slots for them too)
    const int64_t steps = (int64_t)B * num_kv_heads * key_steps(max_keys);
    *bytes = cross_rows_workspace_bytes(std::min(steps, cross_rows_max_slots(head_dim, n_cu)), cols, head_dim);
    if (rows > kMaxRows) *bytes = std::max(*bytes, cross_tiles_workspace_bytes());
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
    if ((int64_t)B * pool->num_kv_heads > (int64_t)1 << 22)
        return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
    int64_t most = 0;                       // packed rows of a sequence, at most
    int64_t steps = 0;                      // 32-key steps of all (sequence, kv head) pairs with rows
    int64_t longest = 0;                    // of one of them, at most
    int64_t tiles = 0;                      // row tiles of one kv head
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
        if (n > 0) {
            const int64_t st_b = key_steps(host_prefix_lens[b] + n);
            steps += st_b * pool->num_kv_heads;
            longest = std::max(longest, st_b);
        }
        tiles += (n * G + attn_rows_per_workgroup(D) - 1) / attn_rows_per_workgroup(D);
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
    int32_t n_cu = 0;
    st = device_cu_count(&n_cu, who);
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (most <= kMaxRows) {
        if (steps > INT32_MAX) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
        const CrossRowsPlan plan =
            tree_rows_plan(steps, (int64_t)B * pool->num_kv_heads, longest, D, (int32_t)most, n_cu);
        bool cut = plan.parts > 1;          // some (sequence, kv head) lies in two runs
        int64_t x = 0;
        for (int32_t b = 0; b < B && !cut && !plan.parts; ++b) {
            const int64_t n = host_cu_nodes[b + 1] - host_cu_nodes[b];
            const int64_t st_b = n > 0 ? key_steps(host_prefix_lens[b] + n) : 0;
            for (int32_t g = 0; st_b > 0 && g < pool->num_kv_heads && !cut; ++g, x += st_b)
                cut = cross_rows_run(plan, steps, x) != cross_rows_run(plan, steps, x + st_b - 1);
        }
        st = check_workspace(cut ? cross_rows_workspace_bytes(plan.slots, (int32_t)most, D) : 0, workspace,
                             workspace_bytes, who);
        if (st) return st;
        e = launch_tree_rows(q, *pool, block_tables, max_blocks, prefix_lens, cu_nodes, B, visible, mask_words,
                             num_q_heads, (int32_t)T, (int32_t)most, steps, plan, cut, sm_scale, out, workspace, s);
    } else {
        if (tiles * pool->num_kv_heads > (int64_t)1 << 22) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
        // The partial results of a key split, asked for whether or not this batch takes one, as the size
        // query, which does not know the lengths, does.
        st = check_workspace(cross_tiles_workspace_bytes(), workspace, workspace_bytes, who);
        if (st) return st;
        e = launch_tree_tiles(q, *pool, block_tables, max_blocks, host_prefix_lens, host_cu_nodes, B, visible,
                              mask_words, num_q_heads, (int32_t)T, sm_scale, out, workspace, s, n_cu);
    }
    if (e != hipSuccess) return hip_fail(e, "pcr_tree_attn: launch");
    return PCR_OK;
}

}  // extern "C"
