// Cross attention to an encoder's cached states for gfx950 (bf16 in, fp32 accumulate, bf16
// out): every query row of a sequence attends all n of its encoder's keys, K/V read from
// the paged pool through the block table.
//
// The s * G query rows of one (sequence, kv head) see the same keys, so they are packed
// (row r = token r / G, head-in-group r % G). A batch whose sequences have up to 16 packed rows
// each (decode steps, beams) is bound by reading K and V: its waves hold the packed rows as the
// columns of one matrix tile and share out the keys of all sequences (cross_rows.hip). Any other
// runs on the row tiles of the prefill kernel (attn.hip) without their causal bound; its
// sequences of few rows take a decode workgroup in the same launch. Rows of sequences without
// keys are zeros that a kernel of their own writes.
//
// Scores, maxima, sums, partial results and their merges are fp32. The weights are rounded to bf16, as
// in every attention here, since the matrix instructions take V^T and P^T in one type; the rows are
// divided by the sum of the rounded weights. Against 64 bits an output is off by 0.0020-0.0023 of its
// size (root mean square; 0.0016-0.0017 with fp32 weights, from its own rounding alone). To carry
// the weights' rest in a second product would add half to the row tiles' matrix work, which
// bounds them; the few-rows kernels, which reads bound, keep the same rounding, so that a
// sequence's rows depend on the form by the order of their sums only.
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Zero rows of the sequences without keys. Grid (B, slices).
constexpr int kZeroThreads = 256;
constexpr int64_t kZeroSlice = 64 << 10;    // bytes of the longest such sequence per workgroup
__global__ __launch_bounds__(kZeroThreads) void cross_zero_kernel(const int32_t *__restrict__ key_lens,
                                                                  const int32_t *__restrict__ cu_q, int32_t T,
                                                                  int64_t row_vecs, u32x4 *__restrict__ out)
{
    const int b = blockIdx.x;
    if (key_lens[b] > 0) return;
    const int64_t v0 = max(cu_q[b], 0) * row_vecs, v1 = min(cu_q[b + 1], T) * row_vecs;
    for (int64_t v = v0 + (int64_t)blockIdx.y * kZeroThreads + threadIdx.x; v < v1; v += (int64_t)gridDim.y * kZeroThreads)
        out[v] = u32x4{0u, 0u, 0u, 0u};
}

constexpr int32_t kMaxKeys = 1 << 30;       // positions past a sequence's end still fit int32

// 32-key steps of n keys (decode_wave.h).
int64_t key_steps(int32_t n) { return ((int64_t)n + 31) / 32; }

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
    if (B == 0 || total_rows == 0 || max_keys == 0) return PCR_OK;
    int32_t n_cu = 0;
    st = device_cu_count(&n_cu, who);
    if (st) return st;
    const int64_t rows = (int64_t)total_rows * (num_q_heads / num_kv_heads);
    const int32_t cols = (int32_t)std::min<int64_t>(rows, decode_max_cols());
    // (sequences without rows count: a plan of parts has slots for them too)
    const int64_t steps = (int64_t)B * num_kv_heads * key_steps(max_keys);
    *bytes = cross_rows_workspace_bytes(std::min(steps, cross_rows_max_slots(head_dim, n_cu)), cols, head_dim);
    if (rows > decode_max_cols()) *bytes = std::max(*bytes, cross_tiles_workspace_bytes());
    return PCR_OK;
}

pcr_status pcr_cross_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                          const int32_t *key_lens, const int32_t *cu_q, const int32_t *host_key_lens,
                          const int32_t *host_cu_q, int32_t B, int32_t num_q_heads, float sm_scale, void *out,
                          void *workspace, int64_t workspace_bytes, void *stream)
{
    clear_error();
    const char *who = "pcr_cross_attn";
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
    if ((int64_t)B * pool->num_kv_heads > (int64_t)1 << 22)
        return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
    int64_t most = 0;                       // packed rows of a sequence, at most
    int64_t most_zero = 0;                  // tokens of one without keys, at most
    int64_t steps = 0;                      // 32-key steps of all (sequence, kv head) pairs with rows
    int64_t longest = 0;                    // of one of them, at most
    for (int32_t b = 0; b < B; ++b) {
        const int64_t s = (int64_t)host_cu_q[b + 1] - host_cu_q[b];
        if (s < 0 || host_key_lens[b] < 0)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d has a negative length", who, b);
        if (((int64_t)host_key_lens[b] + kBlockSize - 1) / kBlockSize > max_blocks)
            return fail(PCR_ERR_INVALID_ARG, "%s: sequence %d needs more blocks than max_blocks %d", who, b,
                        max_blocks);
        if (host_key_lens[b] > kMaxKeys)
            return fail(PCR_ERR_UNSUPPORTED, "%s: sequence %d has more than 2^30 keys", who, b);
        most = std::max(most, s * G);
        if (host_key_lens[b] == 0) most_zero = std::max(most_zero, s);
        if (s > 0) {
            steps += key_steps(host_key_lens[b]) * pool->num_kv_heads;
            longest = std::max(longest, key_steps(host_key_lens[b]));
        }
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
    int32_t n_cu = 0;
    st = device_cu_count(&n_cu, who);
    if (st) return st;
    const bool few = most <= decode_max_cols();
    CrossRowsPlan plan{};
    bool cut = false;                       // some (sequence, kv head) lies in two runs
    if (few) {
        if (steps > INT32_MAX) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
        plan = cross_rows_plan(steps, (int64_t)B * pool->num_kv_heads, longest, D, n_cu);
        cut = plan.parts > 1;
        int64_t x = 0;
        for (int32_t b = 0; b < B && !cut && !plan.parts; ++b) {
            const int64_t n = host_cu_q[b + 1] > host_cu_q[b] ? key_steps(host_key_lens[b]) : 0;
            for (int32_t g = 0; n > 0 && g < pool->num_kv_heads && !cut; ++g, x += n)
                cut = cross_rows_run(plan, steps, x) != cross_rows_run(plan, steps, x + n - 1);
        }
        st = check_workspace(cut ? cross_rows_workspace_bytes(plan.slots, (int32_t)most, D) : 0, workspace,
                             workspace_bytes, who);
    } else {
        int64_t tiles = 0;
        for (int32_t b = 0; b < B; ++b)
            tiles += ((int64_t)(host_cu_q[b + 1] - host_cu_q[b]) * G + attn_rows_per_workgroup(D) - 1) /
                     attn_rows_per_workgroup(D);
        if (tiles * pool->num_kv_heads > (int64_t)1 << 22)
            return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
        // The partial results of a key split, asked for whether or not this batch takes one, as the
        // size query, which does not know the lengths, does. (Without keys only zero rows are written.)
        st = check_workspace(steps > 0 ? cross_tiles_workspace_bytes() : 0, workspace, workspace_bytes, who);
    }
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (most_zero > 0) {
        const int64_t row_vecs = (int64_t)num_q_heads * D / 8;
        const int64_t slices = (most_zero * row_vecs * 16 + kZeroSlice - 1) / kZeroSlice;
        hipLaunchKernelGGL(cross_zero_kernel, dim3((unsigned)B, (unsigned)std::min<int64_t>(slices, 256)),
                           dim3(kZeroThreads), 0, s, key_lens, cu_q, (int32_t)T, row_vecs, static_cast<u32x4 *>(out));
        e = hipGetLastError();
    }
    if (e == hipSuccess && steps > 0)
        e = few ? launch_cross_rows(q, *pool, block_tables, max_blocks, key_lens, cu_q, B, num_q_heads, (int32_t)T,
                                    (int32_t)most, steps, plan, cut, sm_scale, out, workspace, s)
                : launch_cross_tiles(q, *pool, block_tables, max_blocks, host_key_lens, host_cu_q, B, num_q_heads,
                                     (int32_t)T, sm_scale, out, workspace, s, n_cu);
    if (e != hipSuccess) return hip_fail(e, "pcr_cross_attn: launch");
    return PCR_OK;
}

}  // extern "C"
