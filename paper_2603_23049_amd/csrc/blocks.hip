// Block tables, slot lists and the stack of free blocks on the GPU (Sec. 5's paged blocks;
// the device-side counterpart of pcr_plan), for gfx950.
//
// Assignment is two prefix sums over the sequences (new blocks, new tokens) and then one
// independent piece of work per token: the sequence it lies in (a binary search of the
// token sums), its block (an entry the row holds already, or an id off the stack) and its
// slot. The token at a block's first slot writes the block's table entry: a new block's
// first token is always one of the new tokens.
//
// Sums saturate at 2^31 - 1 (a saturating sum of non-negative numbers does not depend on
// the grouping), so no length, however wrong, wraps around into a fit.
#include "pcr_internal.h"

namespace pcr {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kSumMax = 0x7FFFFFFFu;
constexpr int32_t kMaxCount = 1 << 30;      // sequences, free ids, rows: below the saturated sum

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kSumMax); }

// Blocks that hold n tokens (n >= 0, up to 2^31 - 1 and beyond it for a sum of two).
__device__ __forceinline__ int64_t blocks_of(int64_t n) { return (n + kBlockSize - 1) / kBlockSize; }

// Inclusive saturating sums of v over the workgroup's threads; *total gets the sum of all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *wave_sum, uint32_t *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t u = __shfl_up(v, off);
        if (lane >= off) v = sat_add(v, u);
    }
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t u = wave_sum[w];
        before = w < wave ? sat_add(before, u) : before;
        all = sat_add(all, u);
    }
    __syncthreads();
    *total = all;
    return sat_add(before, v);
}

// One workgroup: sequences in chunks of its threads, each chunk's sums first, then its tokens.
__global__ __launch_bounds__(kThreads) void assign_kernel(
    int32_t B, const int32_t *prefix_lens, const int32_t *__restrict__ suffix_lens,
    int32_t *block_tables, int32_t max_blocks, int32_t num_blocks, const int32_t *__restrict__ free_blocks,
    int32_t free_cap, const int32_t *free_count, int32_t *__restrict__ slot_mapping, int32_t *__restrict__ positions,
    int32_t slots_cap, int32_t *__restrict__ cu_suffix, int32_t *context_lens, int32_t *free_count_out,
    int32_t *__restrict__ status)
{
    __shared__ uint32_t wave_sum[kWaves];
    __shared__ int32_t first_bad;
    __shared__ int32_t tok0[kThreads + 1];      // first token of each of the chunk's sequences
    __shared__ int32_t prefix[kThreads];
    __shared__ int32_t blk0[kThreads];          // blocks taken before each
    const int tid = threadIdx.x;
    const int32_t count = min(max(*free_count, 0), free_cap);
    uint32_t blocks = 0, tokens = 0;            // of the chunks so far
    int32_t served = 0;
    bool open = true;                           // no sequence refused so far
    if (tid == 0) cu_suffix[0] = 0;
    for (int32_t b0 = 0; b0 < B; b0 += kThreads) {
        const int32_t b = b0 + tid;
        const int32_t p = b < B ? prefix_lens[b] : 0, s = b < B ? suffix_lens[b] : 0;
        const bool lens_ok = p >= 0 && s >= 0;
        const int64_t held = lens_ok ? blocks_of(p) : 0, need = lens_ok ? blocks_of((int64_t)p + s) : 0;
        uint32_t all_n, all_s;
        const uint32_t nb = (uint32_t)(need - held);
        const uint32_t incl_n = sat_add(blocks, block_scan(nb, wave_sum, &all_n));
        const uint32_t incl_s = sat_add(tokens, block_scan(lens_ok ? (uint32_t)s : 0u, wave_sum, &all_s));
        const bool fits = lens_ok && need <= max_blocks && incl_n <= (uint32_t)count && incl_s <= (uint32_t)slots_cap;
        if (tid == 0) first_bad = open ? kThreads : 0;
        __syncthreads();
        if (!fits && b < B) atomicMin(&first_bad, tid);
        __syncthreads();
        const int n_seq = min(min(B - b0, kThreads), first_bad);   // served in this chunk
        open = n_seq == min(B - b0, kThreads);
        served += n_seq;
        const bool mine = tid < n_seq;
        if (mine) {
            prefix[tid] = p;
            tok0[tid + 1] = (int32_t)incl_s;
            blk0[tid] = (int32_t)(incl_n - nb);
        }
        if (tid == 0) tok0[0] = (int32_t)tokens;
        __syncthreads();
        const int32_t end = tok0[n_seq];
        if (b < B) {
            cu_suffix[b + 1] = mine ? (int32_t)incl_s : end;
            context_lens[b] = mine ? p + s : p;
        }
        for (int32_t t = tok0[0] + tid; t < end; t += kThreads) {
            int lo = 0, hi = n_seq - 1;         // the last sequence that starts at or before t
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (tok0[mid] <= t) lo = mid; else hi = mid - 1;
            }
            const int32_t pb = prefix[lo], pos = pb + (t - tok0[lo]);
            const int32_t entry = pos / kBlockSize, held_b = (int32_t)blocks_of(pb);
            int32_t *row = block_tables + (int64_t)(b0 + lo) * max_blocks;
            int32_t id;
            if (entry < held_b) {
                id = row[entry];
            } else {
                id = free_blocks[count - 1 - (blk0[lo] + (entry - held_b))];
                if (pos % kBlockSize == 0) row[entry] = id;
            }
            slot_mapping[t] = id >= 0 && id < num_blocks ? id * kBlockSize + pos % kBlockSize : -1;
            if (positions) positions[t] = pos;
        }
        if (tid == n_seq - 1) wave_sum[0] = incl_n;   // blocks taken up to the last served one
        __syncthreads();
        if (n_seq) blocks = wave_sum[0];
        tokens = (uint32_t)end;
        __syncthreads();
    }
    for (int32_t t = (int32_t)tokens + tid; t < slots_cap; t += kThreads) {
        slot_mapping[t] = -1;
        if (positions) positions[t] = 0;
    }
    if (tid == 0) {
        *free_count_out = count - (int32_t)blocks;
        status[0] = served;
        status[1] = (int32_t)blocks;
        status[2] = (int32_t)tokens;
    }
}

__device__ __forceinline__ void released(const int32_t *lens, const int32_t *keep_lens, int32_t b, int32_t B,
                                         int32_t max_blocks, int32_t *first, uint32_t *n)
{
    *first = 0;
    *n = 0;
    if (b >= B) return;
    const int64_t f = blocks_of(max(keep_lens[b], 0));
    const int64_t l = blocks_of(min((int64_t)lens[b], (int64_t)max_blocks * kBlockSize));
    *first = (int32_t)f;
    *n = l > f ? (uint32_t)(l - f) : 0u;
}

__global__ __launch_bounds__(kThreads) void release_kernel(
    int32_t B, const int32_t *__restrict__ lens, const int32_t *__restrict__ keep_lens,
    const int32_t *__restrict__ block_tables, int32_t max_blocks, int32_t *__restrict__ free_blocks, int32_t free_cap,
    const int32_t *free_count, int32_t *free_count_out, int32_t *__restrict__ status)
{
    __shared__ uint32_t wave_sum[kWaves];
    __shared__ uint32_t upto[kThreads];         // blocks up to and with each of the chunk's sequences
    __shared__ int32_t first_e[kThreads];
    const int tid = threadIdx.x;
    const int32_t count = min(max(*free_count, 0), free_cap);
    uint32_t total = 0;
    for (int32_t b0 = 0; b0 < B; b0 += kThreads) {
        int32_t f;
        uint32_t n, all;
        released(lens, keep_lens, b0 + tid, B, max_blocks, &f, &n);
        (void)block_scan(n, wave_sum, &all);
        total = sat_add(total, all);
    }
    const bool ok = total <= (uint32_t)(free_cap - count);
    uint32_t before = 0;
    for (int32_t b0 = 0; ok && b0 < B; b0 += kThreads) {
        int32_t f;
        uint32_t n, all;
        released(lens, keep_lens, b0 + tid, B, max_blocks, &f, &n);
        upto[tid] = block_scan(n, wave_sum, &all);
        first_e[tid] = f;
        __syncthreads();
        for (uint32_t k = tid; k < all; k += kThreads) {
            int lo = 0, hi = kThreads - 1;      // the first sequence whose blocks reach beyond k
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (upto[mid] > k) hi = mid; else lo = mid + 1;
            }
            const uint32_t start = lo ? upto[lo - 1] : 0u;
            const int32_t id = block_tables[(int64_t)(b0 + lo) * max_blocks + first_e[lo] + (int32_t)(k - start)];
            free_blocks[count + (int64_t)total - 1 - (before + k)] = id;
        }
        before += all;
        __syncthreads();
    }
    if (tid == 0) {
        *free_count_out = ok ? count + (int32_t)total : count;
        status[0] = ok ? B : 0;
        status[1] = ok ? (int32_t)total : 0;
        status[2] = (int32_t)total;
    }
}

pcr_status check_tables(int32_t B, int32_t max_blocks, int32_t block_size, int32_t num_blocks, int32_t free_cap,
                        const char *who)
{
    if (B < 0 || free_cap < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative B or free_cap", who);
    if (block_size <= 0) return fail(PCR_ERR_INVALID_ARG, "%s: block_size must be positive", who);
    if (block_size != kBlockSize)
        return fail(PCR_ERR_UNSUPPORTED, "%s: block_size %d unsupported (only %d)", who, block_size, kBlockSize);
    if (max_blocks < 1 || num_blocks < 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: max_blocks and num_blocks must be positive", who);
    if (num_blocks > INT32_MAX / kBlockSize || max_blocks > INT32_MAX / kBlockSize)
        return fail(PCR_ERR_UNSUPPORTED, "%s: tokens of %d blocks overflow int32", who,
                    num_blocks > max_blocks ? num_blocks : max_blocks);
    if (B > kMaxCount || free_cap > kMaxCount) return fail(PCR_ERR_UNSUPPORTED, "%s: more than 2^30 entries", who);
    return PCR_OK;
}

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_assign_blocks(int32_t B, const int32_t *prefix_lens, const int32_t *suffix_lens,
                             int32_t *block_tables, int32_t max_blocks, int32_t block_size, int32_t num_blocks,
                             const int32_t *free_blocks, int32_t free_cap, const int32_t *free_count,
                             int32_t *slot_mapping, int32_t *positions, int32_t slots_cap, int32_t *cu_suffix,
                             int32_t *context_lens, int32_t *free_count_out, int32_t *status, void *stream)
{
    clear_error();
    const char *who = "pcr_assign_blocks";
    pcr_status st = check_tables(B, max_blocks, block_size, num_blocks, free_cap, who);
    if (st) return st;
    if (slots_cap < 0) return fail(PCR_ERR_INVALID_ARG, "%s: slots_cap < 0", who);
    if (slots_cap > kMaxCount) return fail(PCR_ERR_UNSUPPORTED, "%s: more than 2^30 rows", who);
    if (B == 0 && slots_cap == 0) return PCR_OK;
    if (!free_count || !cu_suffix || !free_count_out || !status || (slots_cap > 0 && !slot_mapping) ||
        (free_cap > 0 && !free_blocks) || (B > 0 && (!prefix_lens || !suffix_lens || !block_tables || !context_lens)))
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL argument", who);
    hipLaunchKernelGGL(assign_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), B, prefix_lens,
                       suffix_lens, block_tables, max_blocks, num_blocks, free_blocks, free_cap, free_count,
                       slot_mapping, positions, slots_cap, cu_suffix, context_lens, free_count_out, status);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "pcr_assign_blocks: launch");
    return PCR_OK;
}

pcr_status pcr_release_blocks(int32_t B, const int32_t *lens, const int32_t *keep_lens, const int32_t *block_tables,
                              int32_t max_blocks, int32_t block_size, int32_t num_blocks, int32_t *free_blocks,
                              int32_t free_cap, const int32_t *free_count, int32_t *free_count_out, int32_t *status,
                              void *stream)
{
    clear_error();
    const char *who = "pcr_release_blocks";
    pcr_status st = check_tables(B, max_blocks, block_size, num_blocks, free_cap, who);
    if (st) return st;
    if (!free_count || !free_count_out || !status || (free_cap > 0 && !free_blocks) ||
        (B > 0 && (!lens || !keep_lens || !block_tables)))
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL argument", who);
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), B, lens,
                       keep_lens, block_tables, max_blocks, free_blocks, free_cap, free_count, free_count_out, status);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "pcr_release_blocks: launch");
    return PCR_OK;
}

}  // extern "C"
