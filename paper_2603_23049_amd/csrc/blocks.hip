// Block tables, slot lists and the stack of free blocks on the GPU (Sec. 5's paged blocks;
// the device-side counterpart of pcr_plan), for gfx950.
//
// Assignment is two prefix sums over the sequences (new blocks, new tokens) and then one
// independent piece of work per token: the sequence it lies in (a binary search of the
// token sums), its block (an entry the row holds already, or an id off the stack) and its
// slot. The token at a block's first slot writes the block's table entry: a new block's
// first token is always one of the new tokens.
//
// Every workgroup forms the sums of all sequences itself (they are few, and their lengths stay
// in the caches) and takes one tile of the rows: no workgroup waits for another, nothing is
// kept between launches. The step's state (sums, lengths, counts) is written by the first
// workgroup, unless it is updated in place while others still read it: then by a launch of
// one workgroup after them.
//
// Sums saturate at 2^31 - 1 (a saturating sum of non-negative numbers does not depend on
// the grouping), so no length, however wrong, wraps around into a fit.
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

constexpr uint32_t kSumMax = 0x7FFFFFFFu;
constexpr int32_t kMaxCount = 1 << 30;      // sequences, free ids, rows: below the saturated sum

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kSumMax); }

// Blocks that hold n tokens.
__device__ __forceinline__ int64_t blocks_of(int64_t n) { return (n + kBlockSize - 1) / kBlockSize; }

// Inclusive saturating sums of N values over the workgroup's threads. One barrier; wave_sum
// must not be written again before the next one.
template <int THREADS, int N>
__device__ __forceinline__ void block_scan(uint32_t (&v)[N], uint32_t (*wave_sum)[THREADS / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        uint32_t u[N];
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = __shfl_up(v[i], off);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lane >= off ? sat_add(v[i], u[i]) : v[i];
    }
    if (lane == 63) {
#pragma unroll
        for (int i = 0; i < N; ++i) wave_sum[i][wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t before = 0;
        for (int w = 0; w < THREADS / 64; ++w) before = w < wave ? sat_add(before, wave_sum[i][w]) : before;
        v[i] = sat_add(before, v[i]);
    }
}

struct AssignArgs {
    const int32_t *prefix_lens, *suffix_lens, *free_blocks, *free_count;
    int32_t *block_tables, *slot_mapping, *positions, *cu_suffix, *context_lens, *free_count_out, *status;
    int32_t B, max_blocks, num_blocks, free_cap, slots_cap;
    int32_t tile;                               // rows per workgroup
    int32_t state;                              // the first workgroup writes the state
};

// Sequences in chunks of the workgroup's threads: each chunk's sums, then its rows of the tile.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void assign_kernel(const AssignArgs a)
{
    __shared__ uint32_t wave_sum[2][THREADS / 64];
    __shared__ int32_t wave_bad[THREADS / 64];  // first thread of each wave whose sequence does not fit
    __shared__ int32_t tok[THREADS + 1];        // tokens, and blocks taken, before each of the chunk's sequences
    __shared__ int32_t blk[THREADS + 1];
    __shared__ int32_t prefix[THREADS];
    const int tid = threadIdx.x;
    const bool state = a.state && blockIdx.x == 0;
    const int32_t t_lo = (int32_t)min((int64_t)blockIdx.x * a.tile, (int64_t)a.slots_cap);
    const int32_t t_hi = min(t_lo + a.tile, a.slots_cap);
    const int32_t count = min(max(*a.free_count, 0), a.free_cap);
    int32_t blocks = 0, tokens = 0, served = 0; // of the chunks so far
    bool open = true;                           // no sequence refused so far
    if (state && tid == 0) a.cu_suffix[0] = 0;
    for (int32_t b0 = 0; b0 < a.B; b0 += THREADS) {
        const int32_t b = b0 + tid, here = min(a.B - b0, THREADS);
        const int32_t p = b < a.B ? a.prefix_lens[b] : 0, s = b < a.B ? a.suffix_lens[b] : 0;
        const bool lens_ok = p >= 0 && s >= 0;
        const int64_t held = lens_ok ? blocks_of(p) : 0, need = lens_ok ? blocks_of((int64_t)p + s) : 0;
        uint32_t sum[2] = {(uint32_t)(need - held), lens_ok ? (uint32_t)s : 0u};
        block_scan<THREADS>(sum, wave_sum);
        const uint32_t n = sat_add((uint32_t)blocks, sum[0]), t = sat_add((uint32_t)tokens, sum[1]);
        const bool fits = b >= a.B || (lens_ok && need <= a.max_blocks && n <= (uint32_t)count && t <= (uint32_t)a.slots_cap);
        const uint64_t bad = __builtin_amdgcn_ballot_w64(!fits);
        if ((tid & 63) == 0) wave_bad[tid >> 6] = bad ? tid + (int)__builtin_ctzll(bad) : THREADS;
        if (tid == 0) {
            tok[0] = tokens;
            blk[0] = blocks;
        }
        tok[tid + 1] = (int32_t)t;
        blk[tid + 1] = (int32_t)n;
        prefix[tid] = p;
        __syncthreads();
        int n_seq = open ? here : 0;            // served in this chunk
        for (int w = 0; w < THREADS / 64; ++w) n_seq = min(n_seq, wave_bad[w]);
        open = n_seq == here;
        const int32_t end = tok[n_seq];
        if (state && b < a.B) {
            a.cu_suffix[b + 1] = min(tok[tid + 1], end);
            a.context_lens[b] = tid < n_seq ? p + s : p;
        }
        for (int32_t r = max(t_lo, tokens) + tid; r < min(t_hi, end); r += THREADS) {
            int lo = 0, hi = n_seq - 1;         // the last sequence that starts at or before r
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (tok[mid] <= r) lo = mid; else hi = mid - 1;
            }
            const int32_t pb = prefix[lo], pos = pb + (r - tok[lo]);
            const int32_t entry = pos / kBlockSize, held_b = (int32_t)blocks_of(pb);
            int32_t *row = a.block_tables + (int64_t)(b0 + lo) * a.max_blocks;
            int32_t id;
            if (entry < held_b) {
                id = row[entry];
            } else {
                id = a.free_blocks[count - 1 - (blk[lo] + (entry - held_b))];
                if (pos % kBlockSize == 0) row[entry] = id;
            }
            a.slot_mapping[r] = id >= 0 && id < a.num_blocks ? id * kBlockSize + pos % kBlockSize : -1;
            if (a.positions) a.positions[r] = pos;
        }
        tokens = end;
        blocks = blk[n_seq];
        served += n_seq;
        __syncthreads();                        // the next chunk writes the arrays again
    }
    for (int32_t r = max(t_lo, tokens) + tid; r < t_hi; r += THREADS) {
        a.slot_mapping[r] = -1;
        if (a.positions) a.positions[r] = 0;
    }
    if (state && tid == 0) {
        *a.free_count_out = count - blocks;
        a.status[0] = served;
        a.status[1] = blocks;
        a.status[2] = tokens;
    }
}

struct ReleaseArgs {
    const int32_t *lens, *keep_lens, *block_tables, *free_count;
    int32_t *free_blocks, *free_count_out, *status;
    int32_t B, max_blocks, free_cap;
    int32_t tile;                               // ids per workgroup
    int32_t state;                              // the first workgroup writes the state
};

// First entry that sequence b hands back, and how many.
__device__ __forceinline__ void released(const ReleaseArgs &a, int32_t b, int32_t &first, uint32_t &n)
{
    first = 0;
    n = 0;
    if (b >= a.B) return;
    const int64_t f = blocks_of(max(a.keep_lens[b], 0));
    const int64_t l = blocks_of(min((int64_t)a.lens[b], (int64_t)a.max_blocks * kBlockSize));
    first = (int32_t)f;
    n = l > f ? (uint32_t)(l - f) : 0u;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void release_kernel(const ReleaseArgs a)
{
    __shared__ uint32_t wave_sum[1][THREADS / 64];
    __shared__ uint32_t upto[THREADS + 1];      // ids of the chunk's sequences before each
    __shared__ int32_t first_e[THREADS];
    const int tid = threadIdx.x;
    const int32_t count = min(max(*a.free_count, 0), a.free_cap);
    uint32_t total = 0, sum[1];
    int32_t first = 0;
    const bool once = a.B <= THREADS;           // one chunk: its sums serve both passes
    for (int32_t b0 = 0; b0 < a.B; b0 += THREADS) {
        released(a, b0 + tid, first, sum[0]);
        block_scan<THREADS>(sum, wave_sum);
        for (int w = 0; w < THREADS / 64; ++w) total = sat_add(total, wave_sum[0][w]);
        __syncthreads();
    }
    const bool ok = total <= (uint32_t)(a.free_cap - count);
    const uint32_t k_lo = blockIdx.x * (uint32_t)a.tile;      // (k < 2^30: the grid ends with the free list)
    const uint32_t k_hi = ok ? min(k_lo + (uint32_t)a.tile, total) : 0u;
    uint32_t before = 0;
    for (int32_t b0 = 0; b0 < a.B && before < k_hi; b0 += THREADS) {
        if (!once) {
            released(a, b0 + tid, first, sum[0]);
            block_scan<THREADS>(sum, wave_sum);
        }
        if (tid == 0) upto[0] = before;
        upto[tid + 1] = before + sum[0];        // (no saturation: below the total)
        first_e[tid] = first;
        __syncthreads();
        const uint32_t end = upto[THREADS];
        for (uint32_t k = max(k_lo, before) + tid; k < min(k_hi, end); k += THREADS) {
            int lo = 0, hi = THREADS - 1;       // the first sequence whose ids reach beyond k
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (upto[mid + 1] > k) hi = mid; else lo = mid + 1;
            }
            a.free_blocks[count + (int64_t)total - 1 - k] =
                a.block_tables[(int64_t)(b0 + lo) * a.max_blocks + first_e[lo] + (int32_t)(k - upto[lo])];
        }
        before = end;
        __syncthreads();
    }
    if (a.state && blockIdx.x == 0 && tid == 0) {
        *a.free_count_out = ok ? count + (int32_t)total : count;
        a.status[0] = ok ? a.B : 0;
        a.status[1] = ok ? (int32_t)total : 0;
        a.status[2] = (int32_t)total;
    }
}

// Sequences up to which workgroups have 256 threads (a chunk of sequences each), 1024 above.
constexpr int kBigBatch = 256;
// Rows (ids) per thread where one workgroup takes them all for a state updated in place, at most
// (500 rows of one sequence 3.2 us; a second launch adds about 2.5). Otherwise each thread
// takes one: the rows' dependent loads are what a workgroup waits for (200 prompts in 131072 rows
// 4.0 us, 4.7 with two rows a thread, 6.3 with four, 130 with one workgroup; 160 thousand released ids
// of 500 rows 4.7, 5.4, 6.9 and 134; a decode step of 64 3.0).
constexpr int kPerThread = 4;
// Chunks of sequences from which a tile has more than one row per thread: every workgroup scans all
// chunks, so tiles grow with them, and the work of a call with it instead of with its square
// (262144 sequences: release of a million ids 2006 -> 537 us, a token each in 1262144 rows
// 2648 -> 559; 65536 alike; a line of 4 chunks takes up to 16% more).
constexpr int kManyChunks = 16;

// One launch, or two where the state is updated in place and several workgroups read it.
template <class Args>
hipError_t launch_tiles(void (*small)(Args), void (*big)(Args), Args a, int64_t rows, bool in_place, hipStream_t s)
{
    const int threads = a.B <= kBigBatch ? 256 : 1024;
    const int64_t chunks = ((int64_t)a.B + threads - 1) / threads;
    a.tile = in_place && rows <= threads * kPerThread ? threads * kPerThread
                                                      : threads * (int32_t)std::max<int64_t>(1, chunks / kManyChunks);
    const int64_t wgs = rows > a.tile ? (rows + a.tile - 1) / a.tile : 1;
    auto kernel = a.B <= kBigBatch ? small : big;
    a.state = wgs == 1 || !in_place;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(threads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.state) return e;
    a.tile = 0;
    a.state = 1;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(threads), 0, s, a);
    return hipGetLastError();
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
    AssignArgs a{prefix_lens, suffix_lens, free_blocks, free_count, block_tables, slot_mapping, positions, cu_suffix,
                 context_lens, free_count_out, status, B, max_blocks, num_blocks, free_cap, slots_cap, 0, 0};
    const bool in_place = context_lens == prefix_lens || free_count_out == free_count;
    const hipError_t e = launch_tiles(assign_kernel<256>, assign_kernel<1024>, a, slots_cap, in_place,
                                      static_cast<hipStream_t>(stream));
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
    ReleaseArgs a{lens, keep_lens, block_tables, free_count, free_blocks, free_count_out, status, B, max_blocks,
                  free_cap, 0, 0};
    // (no more ids than the rows hold, or than fit the stack)
    const int64_t ids = (int64_t)B * max_blocks < free_cap ? (int64_t)B * max_blocks : free_cap;
    const hipError_t e = launch_tiles(release_kernel<256>, release_kernel<1024>, a, ids, free_count_out == free_count,
                                      static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "pcr_release_blocks: launch");
    return PCR_OK;
}

}  // extern "C"
