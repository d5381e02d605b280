/*
 * pcr.h -- C ABI of libpcr: the per-layer prefix-reuse prefill step on MI355X (gfx950).
 *
 * The operation (PCR, Sec. 2.2, 4.3 and 5; Alg. 1): a request's tokens split
 * into a cached prefix of p tokens, whose K/V already exist in pinned host
 * memory, and an uncached suffix of s tokens. For every layer, the prefix K/V
 * blocks are copied into a paged GPU KV pool (Sec. 5: fixed 16-token blocks
 * mapped through a per-sequence block table, one pool per layer), the
 * suffix's new K/V rows are written into the pool, and causal attention runs
 * for the s suffix rows over all p + s keys. With exact prefix matching the
 * result equals full prefill's output for those rows (Sec. 2.2). A two-stream
 * pipeline overlaps layer l's compute with the loads of later layers
 * (Sec. 4.3: only about one layer's load stays exposed when per-layer compute
 * exceeds per-layer load).
 *
 * Conventions for every entry point:
 *   - Ownership: the caller owns every buffer. Device buffers are plain
 *     device pointers (e.g. from hipMalloc or a framework allocator); host
 *     KV stores must be pinned (hipHostMalloc). The library keeps no pointer
 *     after a call returns.
 *   - Asynchrony: calls that take a stream only enqueue work on it and do
 *     not synchronise (pcr_pipeline_run with timing output is the one
 *     exception). Inputs must stay alive until the stream has passed the work.
 *   - Streams are hipStream_t values passed as void*; NULL is the default stream.
 *   - Errors: argument checks run on the host before anything is enqueued and
 *     return a negative pcr_status; pcr_last_error() then holds a message
 *     (per thread). Faults inside kernels surface at the caller's next
 *     synchronisation. No C++ exception crosses this interface.
 *   - Supported shapes: bf16 K/V/Q, block_size 16, head_dim 64 or 128,
 *     num_q_heads a multiple of num_kv_heads. Anything else returns
 *     PCR_ERR_UNSUPPORTED. (pcr_rope_rows, which touches no pool, takes more head_dims.)
 *   - Empty work (n = 0 pairs, T = 0 tokens, a sequence with s = 0) is a no-op
 *     returning PCR_OK.
 *
 * KV block layout (one layer; K and V are separate arrays of num_blocks blocks;
 * each block holds num_kv_heads payloads of block_size * head_dim bf16):
 *   K of (block blk, kv head g, slot o, dim x) at ((blk*Hkv + g)*bs + o)*d + x
 *   V of (block blk, kv head g, slot o, dim x) at ((blk*Hkv + g)*d + x)*bs + o
 * Host stores use the same per-block layout, so a load is a bitwise block copy.
 * Logical token t of sequence b is slot t % bs of pool block block_tables[b][t / bs].
 * Query head h attends with kv head h / (num_q_heads / num_kv_heads).
 */
#ifndef PCR_H_
#define PCR_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pcr_status {
    PCR_OK = 0,
    PCR_ERR_INVALID_ARG = -1,  /* null pointer, bad size, id out of range, inconsistent shapes */
    PCR_ERR_UNSUPPORTED = -2,  /* valid but unsupported shape (head_dim, block_size, ...) */
    PCR_ERR_NOT_PINNED = -3,   /* a host KV store is not pinned, device-accessible memory */
    PCR_ERR_HIP = -4           /* a HIP runtime call failed while enqueuing */
} pcr_status;

/* One layer's paged KV pool in device memory. */
typedef struct pcr_kv_pool {
    void *k;
    void *v;
    int32_t num_blocks;
    int32_t block_size;
    int32_t num_kv_heads;
    int32_t head_dim;
} pcr_kv_pool;

/* One layer's host KV store (pinned host memory, same per-block layout). */
typedef struct pcr_host_kv {
    const void *k;
    const void *v;
    int64_t num_blocks;
    int32_t block_size;
    int32_t num_kv_heads;
    int32_t head_dim;
} pcr_host_kv;

/* How pcr_load_kv_layer moves blocks over the host link. */
typedef enum pcr_load_method {
    PCR_LOAD_AUTO = 0,          /* the library's default (the measured fastest) */
    PCR_LOAD_DMA_BATCH = 1,     /* one hipMemcpyBatchAsync per call; runs of consecutive
                                   blocks merged into one copy */
    PCR_LOAD_DMA_PER_BLOCK = 2, /* one hipMemcpyAsync per block and per K/V (the
                                   block-by-block baseline of Sec. 5) */
    PCR_LOAD_KERNEL_PULL = 3,   /* a copy kernel on the given stream reads the pinned host
                                   pages directly and writes the pool blocks */
    PCR_LOAD_DMA_STAGED = 4     /* through a device workspace: the copy engines move whole
                                   runs of consecutive host blocks over the host link and a
                                   kernel scatters (load) or gathers (offload) the pool blocks
                                   at HBM speed; only with the *_staged entry points */
} pcr_load_method;

/*
 * pcr_plan -- host-side planning of one batch (Alg. 1, planning loop:
 * each cached block of a scheduled request goes on the host-to-GPU list;
 * only the unmatched tokens are computed).
 *
 * In (host arrays):
 *   prefix_lens[B], suffix_lens[B]        cached and new token counts (>= 0)
 *   block_tables[B][max_blocks]           pool block of every logical block; entries
 *                                         past ceil((p+s)/bs) are ignored
 *   host_blocks[B][max_host_blocks]       host-store block of every logical prefix
 *                                         block; entries past ceil(p/bs) are ignored
 * Out (host arrays, caller-allocated):
 *   src_blocks[cap_pairs], dst_blocks[cap_pairs], *n_pairs
 *       the load list, sequence by sequence, logical block ascending; a pair equal
 *       to an earlier one (a prefix block shared between sequences) is listed once.
 *       cap_pairs = sum_b ceil(p_b / bs) always suffices.
 *   slot_mapping[sum_b s_b]   pool slot (block*bs + offset) of each new token,
 *                             sequences in order
 *   cu_suffix[B+1]            prefix sums of suffix_lens
 * Errors (PCR_ERR_INVALID_ARG): a needed block id < 0; a pool block named as the
 * destination of two different host blocks; a new token's slot already taken, or
 * inside a pool block another sequence loads; capacity too small.
 * Touches no GPU.
 */
pcr_status pcr_plan(int32_t B, const int32_t *prefix_lens, const int32_t *suffix_lens,
                    const int32_t *block_tables, int32_t max_blocks,
                    const int32_t *host_blocks, int32_t max_host_blocks, int32_t block_size,
                    int32_t *src_blocks, int32_t *dst_blocks, int32_t cap_pairs, int32_t *n_pairs,
                    int32_t *slot_mapping, int32_t *cu_suffix);

/*
 * pcr_load_kv_layer -- enqueue the host-to-pool copy of one layer's cached blocks
 * (Sec. 5: one chunk's blocks land in non-consecutive pool blocks; Alg. 1
 * "LayerwiseUpload"). For each i < n: pool block dst_blocks[i] of dst (K and V,
 * all kv heads) becomes a bitwise copy of host block src_blocks[i] of src.
 * src_blocks / dst_blocks are host arrays, range-checked on the host; dst ids
 * must be distinct. src must be pinned (PCR_ERR_NOT_PINNED otherwise). Shapes of
 * src and dst must match. The caller records an event on copy_stream after the
 * call to order later compute behind the copy.
 */
pcr_status pcr_load_kv_layer(const pcr_host_kv *src, const int32_t *src_blocks,
                             const pcr_kv_pool *dst, const int32_t *dst_blocks, int32_t n,
                             void *copy_stream);

/* The same, with the copy method chosen by the caller. */
pcr_status pcr_load_kv_layer_method(const pcr_host_kv *src, const int32_t *src_blocks,
                                    const pcr_kv_pool *dst, const int32_t *dst_blocks, int32_t n,
                                    pcr_load_method method, void *copy_stream);

/*
 * pcr_plan_offload -- the GPU-to-host list of one batch (Alg. 1: a chunk of a
 * scheduled request that no cache tier holds is computed, then goes on the
 * GPU-to-CPU list, "LayerwiseDownload"). For each sequence b, every whole chunk of
 * chunk_tokens tokens (aligned to multiples of chunk_tokens from the sequence
 * start) that lies entirely inside the computed range [prefix_lens[b],
 * prefix_lens[b] + suffix_lens[b]) is listed block by block, sequences in order:
 * src_blocks[i] is its pool block (from block_tables) and dst_blocks[i] =
 * first_dst_block + i (host-store blocks in consecutive order, ready to become the
 * chunks' cache entries). A trailing partial chunk is not offloaded.
 *   chunk_tokens   a positive multiple of block_size
 *   cap            capacity of src_blocks / dst_blocks; *n_pairs receives the count
 * Errors: PCR_ERR_INVALID_ARG for negative lengths, a chunk size that is not a
 * multiple of the block size, a missing pool block (-1 or past max_blocks), or
 * more pairs than cap (nothing useful is written then).
 */
pcr_status pcr_plan_offload(int32_t B, const int32_t *prefix_lens, const int32_t *suffix_lens,
                            const int32_t *block_tables, int32_t max_blocks, int32_t block_size,
                            int32_t chunk_tokens, int32_t first_dst_block,
                            int32_t *src_blocks, int32_t *dst_blocks, int32_t cap, int32_t *n_pairs);

/*
 * pcr_offload_kv_layer -- enqueue the pool-to-host copy of one layer's new blocks
 * (Alg. 1 "LayerwiseDownload"; Sec. 4.3: offloading a layer starts as soon as
 * that layer's computation ends; Sec. 5: on a stream of its own). For each i < n:
 * host block dst_blocks[i] of dst becomes a bitwise copy of pool block
 * src_blocks[i] of src (K and V, all kv heads). Host arrays, range-checked on the
 * host; dst ids must be distinct; dst must be pinned (PCR_ERR_NOT_PINNED
 * otherwise). The caller orders the call after the compute that wrote the
 * blocks (an event from the compute stream).
 * Methods: PCR_LOAD_AUTO and PCR_LOAD_KERNEL_PULL select the copy kernel, which
 * here reads the pool and writes the pinned host pages directly;
 * PCR_LOAD_DMA_PER_BLOCK issues one hipMemcpyAsync per block and per K/V;
 * PCR_LOAD_DMA_BATCH one batched copy (PCR_ERR_UNSUPPORTED without it).
 */
pcr_status pcr_offload_kv_layer(const pcr_kv_pool *src, const int32_t *src_blocks,
                                const pcr_host_kv *dst, const int32_t *dst_blocks, int32_t n,
                                void *stream);
pcr_status pcr_offload_kv_layer_method(const pcr_kv_pool *src, const int32_t *src_blocks,
                                       const pcr_host_kv *dst, const int32_t *dst_blocks, int32_t n,
                                       pcr_load_method method, void *stream);

/*
 * The staged forms of the two copies (PCR_LOAD_DMA_STAGED). workspace: device
 * memory owned by the caller, 16-byte aligned, at least 2 * n * block bytes
 * (block bytes = block_size * num_kv_heads * head_dim * 2); its contents are
 * scratch. Work on one stream is ordered, so one workspace serves every call on
 * that stream; calls on different streams that may overlap need their own.
 * Offload: a kernel gathers the listed pool blocks into the workspace, then one
 * copy-engine transfer per run of consecutive dst host blocks. Load: one transfer
 * per run of consecutive src host blocks into the workspace, then a kernel
 * scatters the blocks into the pool. The long host-link transfers then occupy no
 * compute unit (a kernel that writes host memory directly slows kernels running
 * beside it far more than the copy engines do). PCR_ERR_INVALID_ARG if the
 * workspace is missing or too small.
 */
pcr_status pcr_offload_kv_layer_staged(const pcr_kv_pool *src, const int32_t *src_blocks,
                                       const pcr_host_kv *dst, const int32_t *dst_blocks, int32_t n,
                                       void *workspace, int64_t workspace_bytes, void *stream);
pcr_status pcr_load_kv_layer_staged(const pcr_host_kv *src, const int32_t *src_blocks,
                                    const pcr_kv_pool *dst, const int32_t *dst_blocks, int32_t n,
                                    void *workspace, int64_t workspace_bytes, void *stream);

/*
 * pcr_append_kv -- write the new tokens' K/V into the pool (the KV write that
 * computing the uncached tokens implies, Sec. 4.3).
 *   k_new, v_new   device, bf16 [T][Hkv][d] (row-major, contiguous)
 *   slot_mapping   device, int32 [T]: pool slot of token t (block*bs + offset);
 *                  slots must be distinct; a token whose slot is negative or
 *                  outside the pool is skipped by the kernel (no error is
 *                  reported: the values live in device memory)
 * When a prefix ends inside a block, that block must be loaded before this call
 * (the load copies the whole block; the append then fills its free slots).
 */
pcr_status pcr_append_kv(const pcr_kv_pool *pool, const void *k_new, const void *v_new,
                         const int32_t *slot_mapping, int32_t T, void *stream);

/*
 * pcr_prefix_prefill_attn -- causal GQA attention of the suffix rows over the
 * cached prefix plus the suffix, read through the block table (Sec. 2.2, 5).
 * For sequence b, query head h, suffix row i (absolute position p_b + i), and
 * keys j in [0, p_b + i]:  out = sum_j softmax_j(sm_scale * <q, k_j>) v_j.
 *   q              device bf16 [T][Hq][d]; T = cu_suffix[B]
 *   block_tables   device int32 [B][max_blocks]
 *   prefix_lens    device int32 [B];  cu_suffix device int32 [B+1]
 *   host_prefix_lens, host_cu_suffix   host copies of the same; they must equal the
 *                  device arrays. The launch takes the lengths from these (they size it
 *                  and travel in its arguments); the device arrays must be valid
 *                  (non-NULL) but are not read.
 *   out            device bf16 [T][Hq][d]; fp32 accumulation, rounded to nearest even
 *   sm_scale       finite and > 0 (else PCR_ERR_INVALID_ARG)
 * Numerics: scores <q, k_j> and their scaling are fp32; the probabilities enter the
 * product with V rounded to bf16 and each row is normalised by the sum of those
 * rounded values, so the weights sum to one for any softmax sharpness. Per output
 * element the error is about 2^-8 max_j |v_j - out| plus half a bf16 ulp of out.
 * Every key position j <= p_b + s_b - 1 must hold valid data (loaded or appended);
 * slots past p_b + s_b are never read into the result.
 * Mixed batches: a sequence with s_b = 1 (a decode row) and Hq / Hkv <= 16 is
 * computed in the same launch by a decode workgroup (the key range split over its
 * waves, the same numerics as pcr_decode_attn), and such rows are spread over the
 * prefill row tiles of the launch so that they run beside them.
 * Small launches: when a launch has too few workgroups for the device's compute units
 * and long keys (a short suffix on a long prefix), the keys of each row tile are cut into
 * chunks processed in parallel and merged by a second kernel on the same stream, with
 * the same numerics. The partial results go to scratch the library holds per device
 * (eight launches' worth, about 140 MB, until the process ends); a launch takes its
 * part when it runs and gives it back, so calls on any streams and threads and replays
 * of captured graphs may overlap. (Calls that overlap may write one out only if they
 * write equal values, as ever; each still has its own scratch.) The chunks follow
 * from the lengths alone, so repeated calls give identical bits; a launch that finds
 * eight others holding the scratch runs without chunks (same numerics, other roundings).
 */
pcr_status pcr_prefix_prefill_attn(const void *q, const pcr_kv_pool *pool,
                                   const int32_t *block_tables, int32_t max_blocks,
                                   const int32_t *prefix_lens, const int32_t *cu_suffix,
                                   const int32_t *host_prefix_lens, const int32_t *host_cu_suffix,
                                   int32_t B, int32_t num_q_heads, float sm_scale, void *out,
                                   void *stream);

/*
 * pcr_prefill_attn_set_schedule -- how pcr_prefix_prefill_attn (and the pipelines'
 * attention, pcr_cross_attn with more than 16 packed rows in a sequence and pcr_tree_attn with more than 32) divides a launch
 * among workgroups; a tuning and testing control, not part of the method. Every schedule
 * computes the same result (Sec. 2.2).
 *   PCR_ATTN_SCHEDULE_AUTO (the default): row halves from two of their workgroups per
 *     compute unit on, below it key halves, unless the other of the two is estimated to take
 *     4% less time; launches that leave compute units idle take key halves with the keys
 *     cut into chunks. pcr_pipeline_run and pcr_pipeline_run_offload, whose pull-kernel
 *     loads share the compute units with the attention, take key halves unless row halves
 *     are estimated so and their workgroups all fit the compute units at once (shorter
 *     workgroups let the copy workgroups onto a compute unit sooner), and never cut the
 *     keys;
 *   PCR_ATTN_SCHEDULE_KEY_HALVES: 128 packed query rows per workgroup, the two
 *     wave groups on the two halves of the key range, merged at the end;
 *   PCR_ATTN_SCHEDULE_ROW_HALVES: 256 packed query rows per workgroup, each wave
 *     group on 128 of them over the whole key range, both reading one copy of
 *     each K/V tile (half the workgroups, each with one start-up and no merge for
 *     twice the work, and half the tile loads per row).
 * A batch with more than 128 sequences with new tokens runs as consecutive launches
 * on the stream, the sequences (longest context first) dealt round robin so that
 * every launch gets the same mix; the schedule is chosen per launch.
 * Process-wide; takes effect at the next launch. PCR_ERR_INVALID_ARG for an
 * unknown value.
 */
#define PCR_ATTN_SCHEDULE_AUTO 0
#define PCR_ATTN_SCHEDULE_KEY_HALVES 1
#define PCR_ATTN_SCHEDULE_ROW_HALVES 2
pcr_status pcr_prefill_attn_set_schedule(int32_t schedule);

/*
 * pcr_prefill_attn_hold_scratch -- a testing control, not part of the method: gives back
 * the parts of the current device's key-split scratch that an earlier call holds, then
 * holds n of the eight, so that launches find fewer or none. *free_entries is the number
 * of launches that could register now: 64 with nothing running or held, the first eight
 * of them with scratch. Synchronises the device; no other launch may be running.
 */
pcr_status pcr_prefill_attn_hold_scratch(int32_t n, int32_t *free_entries);

/*
 * pcr_decode_attn -- one decode step: attention of one new query token per
 * sequence over every key of that sequence (Sec. 2.2 with a one-token suffix:
 * the output equals the last row of a full prefill of the sequence).
 * For sequence b, query head h and keys j in [0, n_b):
 *     out = sum_j softmax_j(sm_scale * <q, k_j>) v_j
 * where n_b = context_lens[b] counts the cached tokens plus the token being
 * decoded, whose K/V must already be in the pool (pcr_append_kv).
 *   q                  device bf16 [B][Hq][d], 16-byte aligned
 *   block_tables       device int32 [B][max_blocks]; entries past ceil(n_b/bs) are not read
 *   context_lens       device int32 [B]; host_context_lens: host copy of the same
 *                      (sizes the launch; the two must be equal)
 *   out                device bf16 [B][Hq][d], 16-byte aligned; fp32 accumulation,
 *                      rounded to nearest even
 *   workspace          device memory owned by the caller, 16-byte aligned, of
 *                      pcr_decode_attn_workspace_size(B, Hq, Hkv, d, max_b n_b) bytes
 *                      (NULL when that is 0); its contents are scratch. One workspace
 *                      serves every call ordered on one stream; calls that may overlap
 *                      need their own.
 * The key range of each (sequence, kv head) is split into chunks processed in
 * parallel and merged exactly (in LDS, or through the workspace and a second
 * kernel on the same stream), so the result does not depend on the split beyond
 * fp32 rounding. The chunk size follows the total count of keys when that gives
 * shorter chunks than the largest context alone (ragged batches: long sequences
 * get more chunks than short ones) and the workspace holds that plan; otherwise
 * it follows the largest context, which needs at most the workspace that
 * pcr_decode_attn_workspace_size reported before ragged plans existed (the error
 * message names the size needed). The plan depends only on the host context
 * lengths and the workspace size, so repeated calls give identical bits. Numerics as for
 * pcr_prefix_prefill_attn (fp32 scores, bf16 probabilities, rows normalised by
 * the rounded values); sm_scale must be finite and > 0.
 * Errors: PCR_ERR_UNSUPPORTED if Hq/Hkv > 16 (pcr_prefix_prefill_attn with
 * one-token suffixes covers that case); PCR_ERR_INVALID_ARG if some n_b < 1,
 * ceil(n_b/bs) > max_blocks, or the workspace is missing or too small (the
 * message names the size needed). B = 0 is a no-op.
 */
pcr_status pcr_decode_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables,
                           int32_t max_blocks, const int32_t *context_lens, const int32_t *host_context_lens,
                           int32_t B, int32_t num_q_heads, float sm_scale, void *out, void *workspace,
                           int64_t workspace_bytes, void *stream);

/*
 * pcr_decode_attn_noalloc -- pcr_decode_attn without a workspace argument, for
 * callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc). Same arguments, result and
 * numerics as pcr_decode_attn; the partial results of the chunk merge go to a
 * scratch array of PCR_DECODE_NOALLOC_SCRATCH_BYTES (16 MiB) that the library
 * holds per device until the process ends (its address is taken on the first call
 * on each device). The call allocates nothing and calls no allocating routine.
 * With a workspace of pcr_decode_attn_workspace_size bytes, pcr_decode_attn makes
 * the same plan as this entry point and gives the same bits.
 * Every call on one device shares that device's scratch, which keeps the last
 * call's contents (nothing needs clearing: each call writes every entry it reads
 * back), so calls on one device that may overlap (different streams, or host
 * threads without ordering) race; order them on one stream.
 * Errors: as pcr_decode_attn, and PCR_ERR_UNSUPPORTED when the batch would need
 * more scratch than the maximum (the plan by the largest context needs at most
 * about 11 MiB for any batch on a 256-compute-unit GPU, and the plan by total keys
 * is taken only when it fits); the message names both sizes.
 */
#define PCR_DECODE_NOALLOC_SCRATCH_BYTES (16 << 20)
pcr_status pcr_decode_attn_noalloc(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables,
                                   int32_t max_blocks, const int32_t *context_lens,
                                   const int32_t *host_context_lens, int32_t B, int32_t num_q_heads,
                                   float sm_scale, void *out, void *stream);

/*
 * pcr_decode_attn_workspace_size -- bytes of workspace with which pcr_decode_attn
 * takes its best plan on the current device for any batch of B sequences whose
 * context lengths are at most max_context (0 when every such batch is handled
 * without one); never decreases as max_context grows, and never exceeds
 * PCR_DECODE_NOALLOC_SCRATCH_BYTES beyond what the plan by the largest context
 * needs. Queries the device's compute-unit count; PCR_ERR_HIP when no device is
 * usable.
 */
pcr_status pcr_decode_attn_workspace_size(int32_t B, int32_t num_q_heads, int32_t num_kv_heads,
                                          int32_t head_dim, int32_t max_context, int64_t *bytes);

/*
 * pcr_gather_kv -- read tokens back out of the pool in logical order (the
 * staging step of a layer-wise offload, Sec. 4.3; also a test aid).
 * For each sequence b, tokens starts[b] .. starts[b]+lens[b]-1 go to rows
 * cu_out[b] .. of k_out / v_out (device bf16 [total][Hkv][d]).
 *   block_tables device [B][max_blocks]; starts, lens, cu_out device int32
 *   total = host copy of cu_out[B] (sizes the launch)
 */
pcr_status pcr_gather_kv(const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                         const int32_t *starts, const int32_t *cu_out, int32_t B, int32_t total,
                         void *k_out, void *v_out, void *stream);

/*
 * pcr_assign_blocks -- block tables and slot list of one step, built on the GPU from
 * the lengths (the device-side counterpart of pcr_plan's table and slot part: Sec. 5's
 * paged blocks; nothing is read back to the host, and nothing is copied to the device).
 * For sequence b with p_b = prefix_lens[b] tokens in the pool and s_b = suffix_lens[b] new
 * ones, held_b = ceil(p_b/bs) entries of its table row hold blocks already; new blocks
 * fill the entries up to need_b = ceil((p_b+s_b)/bs), taken from the top of the stack
 * of free block ids free_blocks[0 .. free_count): with new_b = need_b - held_b and off_b
 * the sum of new over the sequences before b,
 *     block_tables[b][held_b + i] = free_blocks[free_count - 1 - (off_b + i)],  i < new_b
 * and every new token t of b, at position pos = p_b + t, gets
 *     slot = block_tables[b][pos / bs] * bs + pos % bs
 * at row cu_suffix[b] + t, where cu_suffix are the prefix sums of s.
 * Served sequences: b is served when, for it and every sequence before it, the lengths
 * are not negative, the row has room (need <= max_blocks), and the new blocks and the
 * new tokens up to it fit (sum of new <= free_count, sum of s <= slots_cap). From the
 * first sequence that is not, none is: they take no block and have no rows (s counts 0).
 * Device arrays:
 *   prefix_lens[B], suffix_lens[B]   read
 *   free_blocks[free_cap]            read; free_count[1] read, held to [0, free_cap]
 *   block_tables[B][max_blocks]      only the new entries are written
 *   slot_mapping[slots_cap]          rows of tokens as above; -1 (which pcr_append_kv and
 *                                    pcr_rope_append_kv skip) in the rows after the last
 *                                    token, and for a table entry outside [0, num_blocks)
 *   positions[slots_cap]             pos of each row's token, 0 after the last; may be NULL
 *   cu_suffix[B+1]                   written
 *   context_lens[B]                  p_b + s_b (p_b where not served); may be prefix_lens itself
 *   free_count_out[1]                free_count less the blocks taken; may be free_count itself
 *   status[3]                        sequences served, blocks taken, tokens (cu_suffix[B])
 * The entry points that take host copies of the lengths (attention, cross attention) need them as
 * the device has them after this call: the caller's own lengths where it knows that every
 * sequence fits, else with s = 0 for the sequences from status[0] on, which it reads back.
 * Otherwise the arrays must not overlap. num_blocks: blocks of the pool. The call allocates
 * nothing and may be captured into a graph; with lengths and counts updated in place each
 * replay is the next step.
 * Errors: PCR_ERR_UNSUPPORTED for a block_size other than 16, max_blocks or num_blocks from
 * 2^27 on (token numbers are int32), or B, free_cap or slots_cap beyond 2^30;
 * PCR_ERR_INVALID_ARG for negative counts, NULL arrays, or max_blocks or num_blocks < 1.
 * B = 0 is a no-op only when slots_cap = 0 too; otherwise every row is marked as padding.
 */
pcr_status pcr_assign_blocks(int32_t B, const int32_t *prefix_lens, const int32_t *suffix_lens,
                             int32_t *block_tables, int32_t max_blocks, int32_t block_size, int32_t num_blocks,
                             const int32_t *free_blocks, int32_t free_cap, const int32_t *free_count,
                             int32_t *slot_mapping, int32_t *positions, int32_t slots_cap, int32_t *cu_suffix,
                             int32_t *context_lens, int32_t *free_count_out, int32_t *status, void *stream);

/*
 * pcr_release_blocks -- the reverse: blocks of ended or shortened sequences go back on
 * the stack of free ids (the pool side of dropping a request, or the rejected tokens of
 * a speculative step). Sequence b keeps its first keep_lens[b] of lens[b] tokens: its
 * entries ceil(keep/bs) .. ceil(len/bs) - 1 are handed back (none if keep >= len; a
 * negative keep counts as 0, a len beyond the row as its end). Blocks that other sequences
 * share must lie below keep. With N blocks in all, the k-th in order of (sequence, entry)
 * goes to free_blocks[free_count + N - 1 - k], so releasing what one pcr_assign_blocks call
 * took restores the stack. If the N ids do not fit (N > free_cap - free_count) nothing
 * is released.
 * Device arrays: lens[B], keep_lens[B], block_tables[B][max_blocks] read (entries keep their
 * values; the row's length says which count); free_blocks[free_cap] written at and above
 * free_count; free_count[1] read, held to [0, free_cap]; free_count_out[1] written, may be
 * free_count itself; status[3]: sequences handled (B, or 0 when nothing was released),
 * blocks released, N (2^31 - 1 if more). No other overlap. An entry outside [0, num_blocks)
 * is put on the stack as it is; pcr_assign_blocks gives its tokens no slot.
 * Errors as pcr_assign_blocks. B = 0 writes the count and the status only.
 */
pcr_status pcr_release_blocks(int32_t B, const int32_t *lens, const int32_t *keep_lens, const int32_t *block_tables,
                              int32_t max_blocks, int32_t block_size, int32_t num_blocks, int32_t *free_blocks,
                              int32_t free_cap, const int32_t *free_count, int32_t *free_count_out, int32_t *status,
                              void *stream);

/*
 * Rotary positions with one or several axes (text position; time, height and width of
 * image and video patches). Pair j of a head is the dims (j, j + rotary_dim/2), or
 * (2j, 2j + 1) when interleaved; it belongs to axis pair_axis[j] and turns by
 * angle = positions[pair_axis[j]][t] * inv_freq[j] for token t:
 *     (x1, x2) -> scale * (x1 cos - x2 sin, x2 cos + x1 sin)
 * Dims from rotary_dim on are passed through. inv_freq and pair_axis are host arrays, read
 * during the call only (they travel in the launch's arguments).
 *   rotary_dim   a positive multiple of 16, at most head_dim (else PCR_ERR_UNSUPPORTED)
 *   num_axes     1 to 4
 *   scale        finite (1 for a pure rotation)
 * Numerics: the angle is reduced in fp64 (error about |angle| * 2^-52, so positions over
 * the whole int32 range keep their phase), cos and sin are fp32 (off by at most 2^-22), the
 * products fp32, one rounding to bf16 (nearest even) at the end; the same bits for a token
 * whatever else is in the call.
 */
typedef struct pcr_rope {
    const float *inv_freq;      /* host [rotary_dim / 2], finite */
    const int32_t *pair_axis;   /* host [rotary_dim / 2], each 0 .. num_axes - 1; NULL: all 0 */
    int32_t rotary_dim;
    int32_t num_axes;
    int32_t interleaved;        /* 0: pairs (j, j + rotary_dim/2); 1: pairs (2j, 2j + 1) */
    float scale;
} pcr_rope;

/*
 * pcr_rope_append_kv -- rotates the new tokens' Q and K and writes K and V into the pool:
 * the position encoding that the attention entry points expect of their inputs (cached K
 * is position-encoded, Sec. 2.2 and 4.2) and pcr_append_kv in one pass over the data.
 *   q, k_new, v_new  device bf16, token t's heads contiguous at t * stride elements:
 *                    [Hq][d], [Hkv][d], [Hkv][d] (so the three may be parts of one fused
 *                    projection's rows); 16-byte aligned, strides multiples of 8 and at
 *                    least the heads' size
 *   positions        device int32 [num_axes][T], axis a at a * pos_stride (>= T) elements
 *   slot_mapping     device int32 [T], as pcr_append_kv: a token whose slot is negative or
 *                    outside the pool has no K/V written (its Q row is rotated all the same)
 *   q_out            device bf16 [T][Hq][d] contiguous, 16-byte aligned; may be q itself
 *                    when q_stride is Hq * d, otherwise the two must not overlap
 *   num_q_heads      0: no Q (q and q_out are not read)
 * k_new and v_new must not overlap q_out, none of the three the pool. Errors: as pcr_append_kv;
 * PCR_ERR_INVALID_ARG for the stride, alignment, overlap and rope conditions above;
 * PCR_ERR_UNSUPPORTED beyond 2^27 tokens, 2^32 threads (about one per 16 dims of 4 query heads)
 * or 2^48 bytes from the first row of an array to its last.
 */
pcr_status pcr_rope_append_kv(const pcr_rope *rope, const pcr_kv_pool *pool, const void *q, int64_t q_stride,
                              const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                              const int32_t *positions, int64_t pos_stride, const int32_t *slot_mapping, int32_t T,
                              int32_t num_q_heads, void *q_out, void *stream);

/*
 * pcr_rope_rows -- the same rotation of plain rows: x [T][num_heads][head_dim] bf16 at
 * x_stride elements per token, out likewise at out_stride (an encoder's heads, or Q and K
 * that go to no pool). inverse != 0 applies the transposed map (sin negated): the gradient
 * with respect to x of a gradient with respect to out, and with scale 1 the undoing.
 *   head_dim  a multiple of 16 up to 256 (else PCR_ERR_UNSUPPORTED)
 * out may be x itself when the strides are equal, otherwise they must not overlap (with equal
 * strides they may be different parts of the same rows); both
 * 16-byte aligned, strides multiples of 8 and at least num_heads * head_dim. T = 0 is a no-op.
 * PCR_ERR_UNSUPPORTED beyond 2^27 tokens, or 2^48 bytes from the first row of an array to its last.
 */
pcr_status pcr_rope_rows(const pcr_rope *rope, const void *x, int64_t x_stride, const int32_t *positions,
                         int64_t pos_stride, int32_t T, int32_t num_heads, int32_t head_dim, int32_t inverse,
                         void *out, int64_t out_stride, void *stream);

/*
 * pcr_cross_attn -- cross attention: every query row of sequence b attends all n_b =
 * key_lens[b] states of an encoder (of a length of their own), whose K/V lie in the pool
 * like any other tokens (written once by pcr_append_kv or loaded from the host store, then
 * read by every later step). For row t of [cu_q[b], cu_q[b+1]), head h, keys j in [0, n_b):
 *     out = sum_j softmax_j(sm_scale * <q, k_j>) v_j;   n_b = 0: the rows are zeros
 * No causal bound and no position encoding. Several row runs over one set of states (beams,
 * samples) are rows of one sequence; text that sees different images in different parts is
 * one sequence per part, their table rows naming the images' blocks (blocks may be shared).
 *   q, out           device bf16 [cu_q[B]][Hq][d], 16-byte aligned, not overlapping; fp32
 *                    accumulation, rounded to nearest even. Rows from cu_q[B] on are left.
 *   block_tables     device int32 [B][max_blocks]; entries past ceil(n_b/bs) are not read;
 *                    an id outside the pool reads block 0
 *   key_lens[B], cu_q[B+1]   device int32, and host copies of the same (they size the launch
 *                    and must be equal)
 *   workspace        device memory owned by the caller, 16-byte aligned, of
 *                    pcr_cross_attn_workspace_size bytes (NULL when that is 0); scratch. One
 *                    workspace serves every call ordered on one stream; calls that may
 *                    overlap (captured graphs that may run together among them) need their own.
 * Numerics as for pcr_prefix_prefill_attn; slots past n_b are never read into the result.
 * The split of the work follows from the host lengths, the device's compute units and the
 * schedule that is set, so repeated calls give identical bits.
 * Errors: as pcr_prefix_prefill_attn, PCR_ERR_UNSUPPORTED beyond 2^30 keys in a sequence or
 * 2^22 pairs of sequence and kv head, and PCR_ERR_INVALID_ARG when q and out overlap or the
 * workspace is missing, misaligned or too small (the message names the size needed).
 */
pcr_status pcr_cross_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                          const int32_t *key_lens, const int32_t *cu_q, const int32_t *host_key_lens,
                          const int32_t *host_cu_q, int32_t B, int32_t num_q_heads, float sm_scale, void *out,
                          void *workspace, int64_t workspace_bytes, void *stream);

/*
 * pcr_cross_attn_workspace_size -- bytes of workspace that serve every pcr_cross_attn call on
 * the current device of at most B sequences with at most total_rows query rows in all and at
 * most max_keys keys each. PCR_ERR_HIP when no device is usable.
 */
pcr_status pcr_cross_attn_workspace_size(int32_t B, int32_t total_rows, int32_t num_q_heads, int32_t num_kv_heads,
                                         int32_t head_dim, int32_t max_keys, int64_t *bytes);

/*
 * Trees of drafted tokens: a speculative step. Sequence b's nodes are the rows
 * cu_nodes[b] .. cu_nodes[b+1] - 1 of every array over nodes (n_b of them, numbered from 0
 * inside the sequence). Node 0 is the last token of the text, whose K/V the pool does not hold yet; the
 * others are drafted. parents[i] of node i is the node that it follows, 0 <= parents[i] < i, or -1:
 * it follows the p_b cached tokens. Node k's K/V lie at logical position p_b + k (the slots that
 * pcr_assign_blocks gives n_b new tokens), whatever its position in the text. A step in turn:
 *   pcr_assign_blocks, pcr_draft_tree; per layer pcr_rope_append_kv (with the tree's positions)
 *   and pcr_tree_attn; pcr_verify_drafts; pcr_compact_kv; pcr_release_blocks (lens p_b + n_b,
 *   keep_lens the context_lens of pcr_verify_drafts).
 * The calls allocate nothing and may be captured into a graph. cu_nodes ascends; rows from
 * cu_nodes[B] on are neither read nor written.
 */

/*
 * pcr_draft_tree -- what every node sees and where it stands. Bit k % 64 of word k / 64 of
 * visible row i is set when node k of the sequence is i itself or an ancestor of it; the
 * position is p_b plus the ancestors' count. A node whose parent is outside [-1, i), whose
 * ancestor's is, or with i >= 64 * mask_words is not part of the tree (padding, say): no bits, position p_b.
 *   cu_nodes[B+1], parents[T], prefix_lens[B]   device int32, read; T: rows of the arrays,
 *                  at least cu_nodes[B]
 *   visible        device uint64 [T][mask_words], 8-byte aligned; mask_words 1 to 16
 *   positions      device int32 [T]
 * No output may overlap another array. Errors: PCR_ERR_UNSUPPORTED for other mask_words, more than 2^21
 * sequences or 2^27 nodes; PCR_ERR_INVALID_ARG for negative counts, NULL arrays, a
 * misaligned visible.
 */
pcr_status pcr_draft_tree(int32_t B, const int32_t *cu_nodes, const int32_t *parents, const int32_t *prefix_lens,
                          int32_t T, int32_t mask_words, uint64_t *visible, int32_t *positions, void *stream);

/*
 * pcr_tree_attn -- attention of a tree's rows: node i of sequence b attends the p_b cached
 * tokens and the nodes of its visible words, keys S = [0, p_b) and p_b + k for every bit k < n_b:
 *     out = sum_{j in S} softmax_j(sm_scale * <q, k_j>) v_j;   S empty: zeros
 *   q, out           device bf16 [cu_nodes[B]][Hq][d], 16-byte aligned, not overlapping; fp32
 *                    accumulation, rounded to nearest even
 *   block_tables     device int32 [B][max_blocks]; entries past ceil((p_b + n_b)/bs) are not read;
 *                    an id outside the pool reads block 0
 *   prefix_lens[B], cu_nodes[B+1]   device int32, and host copies of the same (they size the
 *                    launch and must be equal)
 *   visible          device uint64 [cu_nodes[B]][mask_words] (pcr_draft_tree, or any other words: a
 *                    row need not see itself), 8-byte aligned; n_b <= 64 * mask_words
 *   workspace        as pcr_cross_attn's, of pcr_tree_attn_workspace_size bytes
 * What a row does not see does not reach it: slots of hidden nodes and past p_b + n_b may hold
 * anything, infinities and NaN too. Numerics as for pcr_prefix_prefill_attn. The split of the
 * work follows from the host lengths, the device's compute units and the schedule that is set,
 * so repeated calls give identical bits.
 * Errors: as pcr_cross_attn; PCR_ERR_INVALID_ARG for a sequence of more than 64 * mask_words nodes;
 * PCR_ERR_UNSUPPORTED for mask_words outside 1 .. 16 or more than 2^30 keys in a sequence.
 */
pcr_status pcr_tree_attn(const void *q, const pcr_kv_pool *pool, const int32_t *block_tables, int32_t max_blocks,
                         const int32_t *prefix_lens, const int32_t *cu_nodes, const int32_t *host_prefix_lens,
                         const int32_t *host_cu_nodes, int32_t B, const uint64_t *visible, int32_t mask_words,
                         int32_t num_q_heads, float sm_scale, void *out, void *workspace, int64_t workspace_bytes,
                         void *stream);

/*
 * pcr_tree_attn_workspace_size -- bytes of workspace that serve every pcr_tree_attn call on the
 * current device of at most B sequences with at most total_nodes nodes in all and at most
 * max_keys keys (p_b + n_b) each. PCR_ERR_HIP when no device is usable.
 */
pcr_status pcr_tree_attn_workspace_size(int32_t B, int32_t total_nodes, int32_t num_q_heads, int32_t num_kv_heads,
                                        int32_t head_dim, int32_t max_keys, int64_t *bytes);

/*
 * pcr_verify_drafts -- which drafted tokens stay, and the token after them (speculative sampling, over a
 * tree). The tokens of a step are distributed as the target's if, with draft_probs, the drafted children of
 * a node u were drawn from q_u independently of each other (with replacement: two may be the same token);
 * children drawn without replacement, or the best of q_u, are not so, and in general neither are the tokens. Without
 * draft_probs they are, however the children were chosen, provided that what was chosen does not
 * depend on the uniforms. The walk of
 * sequence b starts on node u = 0. With p_u the target's distribution behind node u, q_u the one
 * that u's drafted children were drawn from, and a = 0, Z = 1, the children of u (nodes i >= 1 with
 * parents[i] = u) are tried in their order: with x = tokens[i] and w = max(p_u(x) - a q_u(x), 0)
 *     uniforms[i] * q_u(x) * Z < w:  i stays, and the walk goes on from u = i, with a = 0, Z = 1;
 *     else a becomes a + Z, and then Z = sum_v max(p_u(v) - a q_u(v), 0).
 * Without q (draft_probs NULL) every child was proposed for certain (a draft's best tokens): w = p_u(x),
 * or 0 if a refused child of u had the same token; it stays if uniforms[i] * Z < w, else Z
 * becomes Z - w and x leaves the distribution. On the last node r(v) is what is left,
 * max(p_u(v) - a q_u(v), 0), or p_u without the refused tokens; with S = sum r the next token is the
 * least v with r(0) + .. + r(v) > uniforms[0] * S (the last v with r(v) > 0 if rounding leaves
 * none). If S = 0, r = p_u takes its place. The walk ends too once path_cap nodes stay.
 *   cu_nodes[B+1], parents[T], tokens[T], prefix_lens[B]   device int32, read; T as for
 *                  pcr_draft_tree. A token outside [0, vocab) never stays and refuses nothing.
 *   target_probs   device fp32: row t (node t's) at t * target_stride elements, vocab of them
 *   draft_probs    likewise, or NULL. Row t may be read wherever node t has a child with a token in
 *                  [0, vocab), whether or not the walk comes there, and is not read elsewhere; what
 *                  rows of nodes hold that the walk does not come to changes nothing
 *   uniforms       device fp32 [T], in [0, 1)
 *   path           device int32 [B][path_cap], written: the nodes that stay, node 0 first, -1 after
 *   accepted_lens  device int32 [B]: how many (1 + the drafted tokens that stay; 0 if n_b = 0)
 *   next_tokens    device int32 [B]: the drawn token, -1 if n_b = 0
 *   context_lens   device int32 [B]: prefix_lens[b] + accepted_lens[b]; may be prefix_lens itself
 *   workspace      device memory owned by the caller, 16-byte aligned, of
 *                  pcr_verify_drafts_workspace_size bytes (NULL when that is 0); scratch. One
 *                  workspace serves every call ordered on one stream; calls that may overlap
 *                  (captured graphs that may run together among them) need their own.
 * A remainder r(v) that is negative or NaN counts as 0; rows need not sum to one exactly. Sums are
 * fp64, products and differences rounded one by one, in an order that the vocabulary alone fixes:
 * repeated calls, and a sequence alone or among others, give the same tokens. No other overlap of outputs. Errors: PCR_ERR_INVALID_ARG for
 * negative counts, vocab or path_cap < 1, strides below vocab, NULL arrays, a workspace that is
 * missing, misaligned or too small; PCR_ERR_UNSUPPORTED beyond 2^21 sequences, 2^27 nodes, a
 * vocabulary of 2^30 or strides of 2^32.
 */
pcr_status pcr_verify_drafts(int32_t B, const int32_t *cu_nodes, const int32_t *parents, const int32_t *tokens,
                             int32_t T, int32_t vocab, const float *target_probs, int64_t target_stride,
                             const float *draft_probs, int64_t draft_stride, const float *uniforms,
                             const int32_t *prefix_lens, int32_t path_cap, int32_t *path, int32_t *accepted_lens,
                             int32_t *next_tokens, int32_t *context_lens, void *workspace, int64_t workspace_bytes,
                             void *stream);

/*
 * pcr_verify_drafts_workspace_size -- bytes of workspace that serve every pcr_verify_drafts call on
 * the current device of at most B sequences with at most T rows and this vocabulary.
 */
pcr_status pcr_verify_drafts_workspace_size(int32_t B, int32_t T, int32_t vocab, int64_t *bytes);

/*
 * pcr_compact_kv -- moves the nodes that stay into consecutive slots, in every layer: for i <
 * accepted_lens[b], the K/V at logical position p_b + path[b][i] go to position p_b + i (bitwise; as
 * if all were read before any is written). What lay there, and the slots behind the kept
 * tokens, are then free for other tokens (pcr_release_blocks hands whole blocks back).
 *   pools          host array of n_layers pools of one shape; their K and V arrays must all be
 *                  apart. Read during the call only.
 *   block_tables   device int32 [B][max_blocks]; the blocks from position p_b on belong to b alone
 *   prefix_lens[B], path[B][path_cap], accepted_lens[B]   device int32 (pcr_verify_drafts);
 *                  an accepted_lens beyond path_cap counts as path_cap
 * A path is strictly ascending from 0 or above, as every way down a tree is. An entry path[b][i] = i is in
 * its place: nothing moves, and its slot is not looked at. The moves of a sequence end before the first
 * entry that does not ascend, or that moves from or to a position past the table's row or in a block
 * outside the pool; none are made for a negative prefix.
 * Errors: as pcr_append_kv for each pool; PCR_ERR_INVALID_ARG for negative counts, pools of
 * different shapes or that overlap, max_blocks or path_cap < 1, NULL arrays; PCR_ERR_UNSUPPORTED beyond
 * 256 layers, 65535 sequences or 2^27 blocks. n_layers = 0 or B = 0 is a no-op.
 */
pcr_status pcr_compact_kv(const pcr_kv_pool *pools, int32_t n_layers, const int32_t *block_tables, int32_t max_blocks,
                          const int32_t *prefix_lens, const int32_t *path, int32_t path_cap,
                          const int32_t *accepted_lens, int32_t B, void *stream);

/* Per-layer device inputs and outputs for pcr_pipeline_run. */
typedef struct pcr_layer_io {
    pcr_host_kv host;     /* this layer's pinned host store */
    pcr_kv_pool pool;     /* this layer's pool */
    const void *q;        /* device bf16 [T][Hq][d] */
    const void *k_new;    /* device bf16 [T][Hkv][d] */
    const void *v_new;    /* device bf16 [T][Hkv][d] */
    void *out;            /* device bf16 [T][Hq][d] */
} pcr_layer_io;

/* The batch structure shared by every layer (from pcr_plan). */
typedef struct pcr_batch {
    const int32_t *src_blocks;        /* host [n_pairs] */
    const int32_t *dst_blocks;        /* host [n_pairs] */
    int32_t n_pairs;
    const int32_t *slot_mapping;      /* device [T] */
    int32_t T;
    const int32_t *block_tables;      /* device [B][max_blocks] */
    int32_t max_blocks;
    const int32_t *prefix_lens;       /* device [B] */
    const int32_t *cu_suffix;         /* device [B+1] */
    const int32_t *host_prefix_lens;  /* host [B] */
    const int32_t *host_cu_suffix;    /* host [B+1] */
    int32_t B;
    int32_t num_q_heads;
    float sm_scale;
} pcr_batch;

/*
 * pcr_pipeline_run -- the layer-wise overlapped step (Sec. 4.3; Alg. 1
 * "LayerwiseUpload" and "WaitForUploadEvents"). Every layer's load goes on
 * copy_stream, each followed by an event; compute_stream waits on layer l's
 * event, then runs layer l's append and attention. The host queues layer by
 * layer (load l, then compute l), so the copy stream runs the loads back to back
 * while the compute stream starts as soon as the first load is done. Layers are
 * independent here (each layer's Q and new K/V are inputs).
 * timing_ms: NULL, or host float[4*n_layers + 2]. When given, the call waits for
 * the last layer and fills, per layer l: [4l] load ms, [4l+1] compute ms
 * (append + attention), [4l+2] compute-stream wait before the layer (exposed
 * load), [4l+3] end of the layer's compute relative to the pipeline start; then
 * [4n] the whole pipeline ms and [4n+1] the sum of compute ms.
 * Overlap needs copy_stream and compute_stream on different hardware queues:
 * HIP maps a process's streams, in creation order, onto GPU_MAX_HW_QUEUES
 * hardware queues (4 unless the environment sets it), and two streams on one
 * queue run in series. Create these streams before others, or raise
 * GPU_MAX_HW_QUEUES before HIP starts (the same holds for the three streams of
 * pcr_pipeline_run_offload).
 * Every layer must have its own pool: nothing orders a later layer's load (copy
 * stream) after an earlier layer's attention (compute stream), so layers sharing
 * pool memory would race. Pool K/V base pointers repeated across layers (or a
 * layer's K equal to its V) are refused with PCR_ERR_INVALID_ARG; pools that
 * overlap at different base addresses are not detected and are the caller's error.
 * Errors: the pools' distinctness and the attention arguments of every layer
 * (batch-wide lengths, heads, sm_scale, block table size; each layer's pool, q
 * and out) are checked before anything is queued, and an error there leaves the
 * streams untouched. A later
 * error (a load's block list or unpinned host memory, found when that layer's
 * load is queued; a failed launch) returns with the earlier layers' work still
 * queued: it runs to completion, and the pools' contents are then unspecified.
 */
pcr_status pcr_pipeline_run(const pcr_layer_io *layers, int32_t n_layers, const pcr_batch *batch,
                            pcr_load_method method, void *copy_stream, void *compute_stream,
                            float *timing_ms);

/*
 * pcr_pipeline_run_staged -- pcr_pipeline_run with every layer's load staged
 * (Sec. 5: the layer's blocks go over the host link as batched copy-engine
 * transfers on their own stream). Layer l's host blocks batch->src_blocks are
 * moved by the copy engines into a workspace slot on copy_stream (one transfer
 * per run of consecutive host blocks, K then V), then a kernel on scatter_stream
 * writes them to pool blocks batch->dst_blocks; compute_stream waits for that
 * scatter, then runs layer l's append and attention. The transfers hold no
 * compute unit while attention runs beside them. workspace: device memory,
 * 16-byte aligned, of workspace_bytes >= one slot = 2 * n_pairs * block_size *
 * num_kv_heads * head_dim * 2 bytes (pcr_load_kv_layer_staged's workspace); it
 * holds floor(workspace_bytes / slot) slots (at most n_layers), layer l using
 * slot l mod slots, and the transfer into a slot waits for the scatter that last
 * read it: with two or more slots, layer l+1's transfer runs while layer l is
 * scattered. The workspace must not be used by other work until the pipeline has
 * run; the first transfers wait for the work already queued on scatter_stream
 * and compute_stream, and the first scatter for compute_stream. The three
 * streams must differ (and overlap only on different hardware queues, as for
 * pcr_pipeline_run). Every layer's pool must have the same block shape.
 * timing_ms and errors as pcr_pipeline_run; [4l] (load ms) spans the layer's
 * transfers and scatter. PCR_ERR_INVALID_ARG for a missing, misaligned or too
 * small workspace or equal streams, before anything is queued.
 * Choice of form: when a layer's compute takes at least as long as its load,
 * this form leaves the attention its whole device and exposes less of the loads
 * than pcr_pipeline_run's pull kernel; when the loads are longer (the host link
 * sets the time) the pull kernel, which needs no scatter, is as fast or faster.
 */
pcr_status pcr_pipeline_run_staged(const pcr_layer_io *layers, int32_t n_layers, const pcr_batch *batch,
                                   void *workspace, int64_t workspace_bytes, void *copy_stream,
                                   void *scatter_stream, void *compute_stream, float *timing_ms);

/*
 * pcr_pipeline_run_offload -- the three-stream form (Sec. 5: upload, compute and
 * download streams; Sec. 4.3: offloading a layer starts when its computation
 * ends). As pcr_pipeline_run, and in addition, after layer l's compute,
 * offload_stream waits for it and copies pool blocks off_src[i] of layer l into
 * host blocks off_dst[i] of offload_dst[l] (i < n_off, host arrays, the same list
 * for every layer) with offload_method. offload_dst: host array of n_layers pinned
 * stores. workspace / workspace_bytes: the staging memory of the offload stream
 * when offload_method is PCR_LOAD_DMA_STAGED (else unused, may be NULL / 0).
 * Before its first load the copy stream also waits for the work already queued on
 * offload_stream, so a load never overwrites a pool an earlier offload is still
 * reading. The three streams must differ.
 * timing_ms: NULL, or host float[6*n_layers + 3]; when given the call waits for
 * the last offload and fills, per layer l: [6l] load ms, [6l+1] compute ms,
 * [6l+2] compute-stream wait before the layer, [6l+3] end of the layer's compute
 * and [6l+5] end of its offload (both relative to the pipeline start), [6l+4]
 * offload ms; then [6n] the whole pipeline ms (to the last offload end), [6n+1]
 * the sum of compute ms, [6n+2] the end of the last compute.
 */
pcr_status pcr_pipeline_run_offload(const pcr_layer_io *layers, const pcr_host_kv *offload_dst,
                                    int32_t n_layers, const pcr_batch *batch, const int32_t *off_src,
                                    const int32_t *off_dst, int32_t n_off, pcr_load_method method,
                                    pcr_load_method offload_method, void *workspace, int64_t workspace_bytes,
                                    void *copy_stream, void *compute_stream, void *offload_stream,
                                    float *timing_ms);

/*
 * pcr_pipeline_run_offload_staged -- pcr_pipeline_run_offload with the loads
 * staged as in pcr_pipeline_run_staged: four streams (copy-engine transfers into
 * load_workspace slots on copy_stream, the scatter into the pool on
 * scatter_stream, append and attention on compute_stream, the offload of layer l
 * after its compute on offload_stream with offload_method and offload_workspace).
 * load_workspace follows pcr_pipeline_run_staged's workspace rules;
 * offload_workspace pcr_pipeline_run_offload's; the two must not overlap. Besides
 * the waits of both forms, the first scatter also waits for the work already
 * queued on offload_stream (an earlier offload may still read a pool). The four
 * streams must differ. timing_ms and errors as pcr_pipeline_run_offload; [6l]
 * (load ms) spans the layer's transfers and scatter.
 */
pcr_status pcr_pipeline_run_offload_staged(const pcr_layer_io *layers, const pcr_host_kv *offload_dst,
                                           int32_t n_layers, const pcr_batch *batch, const int32_t *off_src,
                                           const int32_t *off_dst, int32_t n_off, pcr_load_method offload_method,
                                           void *offload_workspace, int64_t offload_workspace_bytes,
                                           void *load_workspace, int64_t load_workspace_bytes, void *copy_stream,
                                           void *scatter_stream, void *compute_stream, void *offload_stream,
                                           float *timing_ms);

/*
 * The SSD tier of the chunk cache (Sec. 4.4 queue-based prefetch and asynchronous
 * write-back; Sec. 5 dedicated prefetch thread). A store is one file of fixed-size
 * chunk slots (chunk id c at byte c * chunk_bytes) served by io_threads host
 * threads in submission order. The file is created (truncated) at open. Buffers
 * belong to the caller and must stay untouched until the chunk's task completes;
 * page-aligned buffers (e.g. pinned host memory) with a page-multiple chunk size
 * bypass the page cache (O_DIRECT). No GPU work is involved.
 *   pcr_store_write_async   queue chunk_bytes from src as chunk chunk_id
 *   pcr_store_read_async    queue a read of chunk chunk_id into dst; PCR_ERR_INVALID_ARG
 *                           if the chunk was never written
 * Tasks of one chunk run one at a time, in submission order: both submit calls
 * first block until the chunk's earlier tasks are done (tasks of other chunks run
 * concurrently on the I/O threads).
 *   pcr_store_wait          block until chunk_id's tasks (or, for chunk_id < 0, all
 *                           tasks) are done; reports the first I/O error, if any
 *   pcr_store_poll          *done = 1 if nothing is pending for chunk_id (or at all)
 *   pcr_store_stats         bytes moved so far; whether the file is open for O_DIRECT;
 *                           and how many page-aligned transfers O_DIRECT refused (host
 *                           memory the GPU driver mapped, such as hipHostMalloc pinned
 *                           memory) and the page cache served instead
 * Any output pointer of pcr_store_stats may be NULL.
 *   pcr_store_close         drain the queue, stop the threads, close the file
 */
typedef struct pcr_chunk_store pcr_chunk_store;
pcr_status pcr_store_open(const char *path, int64_t chunk_bytes, int32_t io_threads, pcr_chunk_store **out);
pcr_status pcr_store_write_async(pcr_chunk_store *store, int64_t chunk_id, const void *src);
pcr_status pcr_store_read_async(pcr_chunk_store *store, int64_t chunk_id, void *dst);
pcr_status pcr_store_wait(pcr_chunk_store *store, int64_t chunk_id);
pcr_status pcr_store_poll(pcr_chunk_store *store, int64_t chunk_id, int32_t *done);
pcr_status pcr_store_stats(pcr_chunk_store *store, int64_t *bytes_read, int64_t *bytes_written, int32_t *direct,
                           int64_t *direct_fallbacks);
pcr_status pcr_store_close(pcr_chunk_store *store);

/* Message of the last failed call on this thread ("" if none). */
const char *pcr_last_error(void);

/* Library version string. */
const char *pcr_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PCR_H_ */
