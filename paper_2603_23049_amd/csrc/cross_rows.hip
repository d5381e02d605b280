// Cross attention of few query rows per sequence (decode steps, beams) for gfx950: how the work is
// cut, and its launch (rows_kernel.h).
#include <algorithm>

#include "rows_kernel.h"

namespace pcr {

// How the steps are cut, by an estimate in us fitted to 330 batches (1 to 300 sequences of 20 to
// 16000 keys, equal and ragged, 1 to 16 kv heads, inputs out of the caches): memory takes bw for
// all steps at the rate of a full device, a compute unit cu for one step (its own limit, about
// 40 GB/s), and the constants are what the launches take with nothing to read. Measured, one run a
// pair / some runs a pair / even runs: one token of 187 sequences of 1064 keys (16 / 2 heads of 128)
// 42 / - / 44, of 2 of 2438 (28 / 4) 32 / 12 / 17, of 53 of 1034-8276 (64 / 8) 212 / - / 163 and
// of 45 of 828-6627 161 / - / 115. (The decode entry point's plan, chunks of one size for the
// whole batch, takes 48, 12, 252 and 184 there. Over the 330 this choice takes 8% less than that
// plan, 37% at best; the worst, a call of 14 us, 14% more.)
CrossRowsPlan cross_rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t n_cu)
{
    return rows_plan(steps, pairs, longest, head_dim, n_cu, {head_dim == 128 ? 0.41f : 0.22f, 9.5f, 1.f, 8});
}

CrossRowsPlan rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t n_cu,
                        const RowsCost &cost)
{
    CrossRowsPlan p{};
    if (steps <= 0) return p;
    const bool wide = head_dim == 128;
    const int64_t waves = (int64_t)n_cu * (wide ? 4 : 8);   // that are resident (registers)
    auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    const float bw = steps * (wide ? 0.0024f : 0.0012f) * 256.f / n_cu, cu = cost.cu;
    // The longest pairs run on with the device emptying around them for `tail`.
    const float mean = (float)steps / pairs, tail = cu * (longest - mean);
    // one run a pair: a compute unit's share of the pairs, one of them the longest
    const float whole = 6.f + tail + std::max(bw, cu * ceil_div(pairs, n_cu) * mean);
    // k runs of four waves a pair, of eight steps or more, all resident at once
    const int64_t k = std::max<int64_t>(1, std::min(ceil_div(longest, 8), waves / 4 / pairs));
    const float parts =
        cost.parts + std::max(bw + tail / k, cu * ceil_div(pairs * k, n_cu) * ceil_div(longest, k)) + 0.03f * k;
    // even runs of all steps: single waves, or four together where a pair had too many parts to merge
    const int64_t single = std::max<int64_t>(1, std::min(waves, steps / 2));
    const bool four = single > 32 * pairs;
    const float even = (four ? 13.5f : 11.f + 3.f * std::min(1.f, single / 600.f)) + bw * cost.even;
    if (whole <= even && (k == 1 || whole <= parts)) {
        p.parts = 1;
        p.waves = !wide && cost.waves == 8 && pairs * 8 <= waves ? 8 : pairs * 4 <= waves ? 4 : pairs * 2 <= waves ? 2 : 1;
        // more pairs than waves: long ones are shared all the same, so that the last ends earlier
        if (p.waves == 1 && longest >= (wide ? 64 : 20)) p.waves = 4;
        p.runs = (int32_t)pairs;
    } else if (k > 1 && parts <= even) {
        p.parts = (int32_t)k;
        p.waves = 4;
        p.runs = (int32_t)(pairs * k);
    } else {
        p.waves = four ? 4 : 1;
        p.runs = (int32_t)(four ? std::max<int64_t>(1, std::min(waves / 4, steps / 8)) : single);
    }
    p.slots = p.parts ? p.runs : 2 * p.runs;
    return p;
}

int64_t cross_rows_max_slots(int32_t head_dim, int32_t n_cu) { return (int64_t)2 * n_cu * (head_dim == 128 ? 4 : 8); }

int64_t cross_rows_workspace_bytes(int64_t slots, int32_t cols, int32_t head_dim)
{
    return slots * cols * (head_dim + 2) * 4;
}

hipError_t launch_cross_rows(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                             const int32_t *key_lens, const int32_t *cu_q, int32_t B, int32_t num_q_heads, int32_t T,
                             int32_t cols, int64_t steps, const CrossRowsPlan &plan, bool combine, float sm_scale,
                             void *out, void *workspace, hipStream_t s)
{
    return launch_rows<0>(q, pool, block_tables, max_blocks, key_lens, cu_q, B, num_q_heads, T, cols, steps, plan,
                          combine, sm_scale, out, workspace, s, nullptr, 0);
}

}  // namespace pcr
