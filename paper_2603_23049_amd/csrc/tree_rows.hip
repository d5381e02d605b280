// Attention of small trees of drafted tokens (up to 32 packed rows of a sequence and kv head) for gfx950:
// the rows kernel (rows_kernel.h) with one or two tiles of columns.
#include "rows_kernel.h"

namespace pcr {

hipError_t launch_tree_rows(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                            const int32_t *prefix_lens, const int32_t *cu_nodes, int32_t B, const uint64_t *visible,
                            int32_t mask_words, int32_t num_q_heads, int32_t T, int32_t cols, int64_t steps,
                            const CrossRowsPlan &plan, bool combine, float sm_scale, void *out, void *workspace,
                            hipStream_t s)
{
    auto go = [&](auto launch) {
        return launch(q, pool, block_tables, max_blocks, prefix_lens, cu_nodes, B, num_q_heads, T, cols, steps, plan,
                      combine, sm_scale, out, workspace, s, visible, mask_words);
    };
    if (cols <= 16) return go(launch_rows<1>);
    return go(launch_rows<2>);
}

}  // namespace pcr
