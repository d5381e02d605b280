// Internal declarations shared by the libpcr translation units (not installed).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/pcr.h"

namespace pcr {

constexpr int kBlockSize = 16;   // tokens per pool block (the serving engine's block, Sec. 5)

// Records a formatted message as this thread's last error and returns `st`.
pcr_status fail(pcr_status st, const char *fmt, ...);
// Turns a HIP error into PCR_ERR_HIP with the call site named.
pcr_status hip_fail(hipError_t e, const char *what);
void clear_error();
// The checks every entry point makes of a block layout and of a pool (errors name `who`).
pcr_status check_layout(int32_t block_size, int32_t num_kv_heads, int32_t head_dim, const char *who);
pcr_status check_pool(const pcr_kv_pool *pool, const char *who);
// Query heads of a pool with num_kv_heads, and a caller's workspace of which `need` bytes are needed.
pcr_status check_heads(int32_t num_q_heads, int32_t num_kv_heads, const char *who);
pcr_status check_workspace(int64_t need, const void *workspace, int64_t bytes, const char *who);

// Up to this many (src, dst) block pairs travel in one pull-kernel launch as
// kernel arguments (so no device copy of the host lists is needed).
constexpr int kPullPairsPerLaunch = 480;

struct PullArgs {
    int32_t n;
    int32_t src[kPullPairsPerLaunch];
    int32_t dst[kPullPairsPerLaunch];
};

// Kernel launchers (kv_move.hip).
hipError_t launch_append_kv(const pcr_kv_pool &pool, const void *k_new, const void *v_new,
                            const int32_t *slot_mapping, int32_t T, hipStream_t s);
hipError_t launch_gather_kv(const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                            const int32_t *starts, const int32_t *cu_out, int32_t B, int32_t total,
                            void *k_out, void *v_out, hipStream_t s);
hipError_t launch_pull_blocks(const void *host_k, const void *host_v, int64_t host_blocks,
                              void *pool_k, void *pool_v, int32_t pool_blocks, int64_t block_bytes,
                              const PullArgs &args, hipStream_t s);
hipError_t launch_device_blocks(const void *src_k, const void *src_v, int64_t src_blocks, void *dst_k, void *dst_v,
                                int64_t dst_blocks, int64_t block_bytes, const PullArgs &args, hipStream_t s);
hipError_t launch_push_blocks(const void *pool_k, const void *pool_v, int32_t pool_blocks, void *host_k,
                              void *host_v, int64_t host_blocks, int64_t block_bytes, const PullArgs &args,
                              hipStream_t s);

// Attention launcher (attn.hip).
// The lengths travel in the launches' arguments (the work map), taken from the host
// copies, which the caller guarantees equal the device arrays.
hipError_t launch_prefix_prefill_attn(const void *q, const pcr_kv_pool &pool,
                                      const int32_t *block_tables, int32_t max_blocks,
                                      const int32_t *host_prefix_lens, const int32_t *host_cu_suffix,
                                      int32_t B, int32_t num_q_heads, int32_t T, float sm_scale, void *out,
                                      hipStream_t s, int auto_schedule, int n_cu);
// Cross attention by row tiles (attn.hip): every row of a sequence sees its host_key_lens[b] keys;
// rows of sequences without keys are left.
// workspace: cross_tiles_workspace_bytes() for a key split, or NULL for none.
int64_t cross_tiles_workspace_bytes();
hipError_t launch_cross_tiles(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                              const int32_t *host_key_lens, const int32_t *host_cu_q, int32_t B, int32_t num_q_heads,
                              int32_t T, float sm_scale, void *out, void *workspace, hipStream_t s, int n_cu);
// Parts of a kv head's items that the XCDs sharing it take in a launch on row tiles of rpw rows over the sequences
// seq[0..n), n <= 128, longest context first (slot_order); 1: the given order.
int32_t prefill_attn_parts(const int32_t *seq, int32_t n, const int32_t *prefix_lens, const int32_t *cu_suffix,
                           int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t rpw, int32_t n_cu);
// Tree attention by row tiles (attn.hip), of any number of rows; workspace as for cross attention.
hipError_t launch_tree_tiles(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                             const int32_t *host_prefix_lens, const int32_t *host_cu_nodes, int32_t B,
                             const uint64_t *visible, int32_t mask_words, int32_t num_q_heads, int32_t T,
                             float sm_scale, void *out, void *workspace, hipStream_t s, int n_cu);
// Compute units of the current device (queried once per device).
pcr_status device_cu_count(int32_t *n_cu, const char *who);

// Decode attention (decode.hip). The key range of each (sequence, kv head) is cut
// into chunks of `chunk` keys, at most n_split per sequence. Without the context
// lengths (or when it does not shorten the chunks) the chunk follows from the
// largest context; with them, from the total count of keys (a ragged batch then
// gives its long sequences more chunks than its short ones). lds_merge: every
// sequence has n_split <= 4 chunks and they merge in LDS; otherwise chunks of one
// sequence merge through the workspace. bound_workspace_bytes covers every batch of
// B sequences with contexts up to max_context, under either rule.
struct DecodePlan {
    int32_t n_split;
    int32_t chunk;
    int32_t lds_merge;
    int32_t ws_wg_waves;   // waves per workgroup when chunks merge through the workspace
    int32_t sub;           // waves that share one chunk (chunks merging through the workspace)
    int32_t k_streamed;    // every sequence of one length: K loads non-temporal
    int64_t workspace_bytes;
    int64_t bound_workspace_bytes;
};
// ctx: the host context lengths (NULL: plan from max_context alone); the rule by total
// keys is taken only when its workspace fits ws_limit bytes.
DecodePlan decode_plan(int32_t B, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                       int32_t max_context, int32_t n_cu, const int32_t *ctx = nullptr, int64_t ws_limit = 0);
int decode_max_cols();
hipError_t launch_decode_attn(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables,
                              int32_t max_blocks, const int32_t *context_lens, int32_t B, int32_t num_q_heads,
                              const DecodePlan &plan, float sm_scale, void *out, void *workspace, hipStream_t s);
// Cross attention of sequences with few packed query rows each (cross_rows.hip): how the 32-key
// steps of all (sequence, kv head) pairs with rows and keys are cut into `runs` workgroups.
struct CrossRowsPlan {
    int32_t runs, waves;   // workgroups, and waves of each
    int32_t parts;         // runs of a pair, whatever its length; 0: even runs over all steps
    int32_t slots;         // partial results in the workspace (where some pair is cut)
};
// pairs: of all sequences (those without steps too); longest: steps of one pair, at most.
CrossRowsPlan cross_rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t n_cu);
// The same with the estimate's constants: us of a compute unit for a step, what parts take with nothing to
// read, how much longer than other cuts even runs take to read, and the most waves of a whole pair.
struct RowsCost {
    float cu, parts, even;
    int32_t waves;
};
CrossRowsPlan rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t n_cu,
                        const RowsCost &cost);
// Tree attention's (tree.hip), of up to cols packed rows a sequence.
CrossRowsPlan tree_rows_plan(int64_t steps, int64_t pairs, int64_t longest, int32_t head_dim, int32_t cols,
                             int32_t n_cu);
// Most slots of any plan (none has more than its steps, either).
int64_t cross_rows_max_slots(int32_t head_dim, int32_t n_cu);
// The run of an even cut that holds step x.
inline int64_t cross_rows_run(const CrossRowsPlan &p, int64_t steps, int64_t x)
{
    const int64_t base = steps / p.runs, rem = steps % p.runs, big = rem * (base + 1);
    return x < big ? x / (base + 1) : rem + (x - big) / base;
}
int64_t cross_rows_workspace_bytes(int64_t slots, int32_t cols, int32_t head_dim);
// cols: packed rows of a sequence, at most (up to decode_max_cols); combine: some pair is cut
// between runs. The rows of sequences without keys are left.
hipError_t launch_cross_rows(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                             const int32_t *key_lens, const int32_t *cu_q, int32_t B, int32_t num_q_heads, int32_t T,
                             int32_t cols, int64_t steps, const CrossRowsPlan &plan, bool combine, float sm_scale,
                             void *out, void *workspace, hipStream_t s);
// The same of trees (tree_rows.hip): keys are the cached tokens and then the nodes, cols up to kTreeMaxCols.
constexpr int kTreeMaxCols = 32;
hipError_t launch_tree_rows(const void *q, const pcr_kv_pool &pool, const int32_t *block_tables, int32_t max_blocks,
                            const int32_t *prefix_lens, const int32_t *cu_nodes, int32_t B, const uint64_t *visible,
                            int32_t mask_words, int32_t num_q_heads, int32_t T, int32_t cols, int64_t steps,
                            const CrossRowsPlan &plan, bool combine, float sm_scale, void *out, void *workspace,
                            hipStream_t s);
// Trees of drafted tokens (draft.hip, verify.hip, tree.hip).
constexpr int32_t kMaxMaskWords = 16;        // 64-bit words of a node's visible set
constexpr int32_t kMaxTreeSeqs = 1 << 21;    // a workgroup of up to 1024 threads each: below 2^32 threads
constexpr int32_t kMaxTreeNodes = 1 << 27;
constexpr int32_t kMaxVocab = 1 << 30;
constexpr int64_t kMaxRowStride = (int64_t)1 << 32;   // elements; times the rows, below 2^62 bytes
// How a verification of B sequences with T rows in all is cut up (verify.hip).
struct VerifyPlan {
    int32_t tiles, pieces;   // of a row, and of a tile
    int32_t rounds, wgs;     // launches before the last one, and their workgroups per sequence
    int64_t bytes;           // of workspace
};
VerifyPlan verify_plan(int32_t B, int32_t T, int32_t V, bool drawn);
// Size of the allocation-free decode entry point's per-device scratch (decode.hip),
// and its device address on the current device (taken with hipGetSymbolAddress on the
// first call per device, then reused).
constexpr int64_t kDecodeScratchBytes = PCR_DECODE_NOALLOC_SCRATCH_BYTES;
hipError_t decode_noalloc_scratch(void **ptr);

// The staged host-to-pool load (every check of pcr_load_kv_layer_staged) with its two
// halves on two streams: the copy-engine transfers into the workspace on dma_stream,
// then dma_done is recorded there, scatter_stream waits for it and runs the scatter
// into the pool. The workspace is free again once the scatter has run.
pcr_status load_staged_split(const pcr_host_kv *src, const int32_t *src_blocks, const pcr_kv_pool *dst,
                             const int32_t *dst_blocks, int32_t n, void *workspace, int64_t workspace_bytes,
                             hipStream_t dma_stream, hipStream_t scatter_stream, hipEvent_t dma_done);

// Size in bytes of one pool block of K (or V): block_size * num_kv_heads * head_dim bf16.
inline int64_t kv_block_bytes(int32_t block_size, int32_t num_kv_heads, int32_t head_dim)
{
    return (int64_t)block_size * num_kv_heads * head_dim * 2;
}

// Pool-to-host offload with any method (the staged one takes the workspace); used by
// the pipeline, which chooses the method per call.
pcr_status offload_with(const pcr_kv_pool *src, const int32_t *src_blocks, const pcr_host_kv *dst,
                        const int32_t *dst_blocks, int32_t n, pcr_load_method method, void *workspace,
                        int64_t workspace_bytes, void *stream);

// pcr_prefix_prefill_attn with a schedule preference: when the process-wide schedule
// is PCR_ATTN_SCHEDULE_AUTO, auto_schedule PCR_ATTN_SCHEDULE_KEY_HALVES takes key
// halves, unless row halves are estimated to be faster and their items all fit the compute
// units at once (PCR_ATTN_SCHEDULE_AUTO: the rule without that limit, and the key split).
pcr_status prefix_prefill_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables,
                               int32_t max_blocks, const int32_t *prefix_lens, const int32_t *cu_suffix,
                               const int32_t *host_prefix_lens, const int32_t *host_cu_suffix, int32_t B,
                               int32_t num_q_heads, float sm_scale, void *out, void *stream, int auto_schedule);

// Rows of packed (token, head-in-group) queries one attention workgroup handles with
// key halves (the most row tiles any schedule launches per sequence).
int attn_rows_per_workgroup(int head_dim);
// Process-wide attention schedule (PCR_ATTN_SCHEDULE_*), read at each launch.
void attn_set_schedule(int schedule);
hipError_t attn_hold_scratch(int n, int *free_entries);

// Every argument check of pcr_prefix_prefill_attn, with no launch (errors name `who`);
// on success *T_out is the suffix token count (0: nothing to do).
pcr_status attn_check(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                      const int32_t *prefix_lens, const int32_t *cu_suffix, const int32_t *host_prefix_lens,
                      const int32_t *host_cu_suffix, int32_t B, int32_t num_q_heads, float sm_scale,
                      const void *out, const char *who, int64_t *T_out);

}  // namespace pcr
