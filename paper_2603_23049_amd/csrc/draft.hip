// Trees of drafted tokens for gfx950: which tokens every node of a tree sees and at which
// position it stands, and the move of the kept nodes' K/V into consecutive slots of the paged
// pools (the pool side of a speculative step; Sec. 5's paged blocks).
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16;

// Node i sees itself and its ancestors: bit k of its words for every k on the way to the root. One wave per
// sequence takes 64 nodes at a time: a lane's ancestors among the 64 by doubling (six rounds of "what my
// next ancestor has found, I have found too"), and from the first ancestor before them, whose row the
// wave wrote earlier, the words, the depth and whether it is part of the tree. Dependent steps
// bound it, not bytes: a thread per word that followed the parents one by one took 50 us for 500 trees of up to 256
// nodes, this 6.7 (2.8 for 64 trees of 16).
__global__ __launch_bounds__(64) void draft_tree_kernel(
    const int32_t *__restrict__ cu_nodes, const int32_t *__restrict__ parents, const int32_t *__restrict__ prefix_lens,
    int32_t T, int32_t words, uint64_t *visible, int32_t *positions)
{
    const int lane = threadIdx.x, b = blockIdx.x;
    const int32_t t0 = min(max(cu_nodes[b], 0), T), n = min(cu_nodes[b + 1], T) - t0;
    if (n <= 0) return;
    const int32_t p = prefix_lens[b];
    uint64_t *rows = visible + (int64_t)t0 * words;
    int32_t *pos = positions + t0;
    int32_t parent = lane < n ? parents[t0 + lane] : -1;
    for (int32_t c = 0; 64 * (int64_t)c < n; ++c) {
        const int32_t i = 64 * c + lane;
        const int32_t ahead = i + 64 < n ? parents[t0 + i + 64] : -1;   // the next 64's
        uint64_t m = 1ull << lane;                              // ancestors among the 64
        int32_t next = parent >= -1 && parent < i ? parent : -2;    // the first one not among them (-1: none)
#pragma unroll
        for (int r = 0; r < 6; ++r) {
            const bool inside = next >= 64 * c;
            const int src = inside ? next - 64 * c : lane;
            const uint64_t found = __shfl(m, src);
            const int32_t further = __shfl(next, src);
            m |= inside ? found : 0ull;
            next = inside ? further : next;
        }
        parent = ahead;
        if (i < n) {
            uint64_t *row = rows + (int64_t)i * words;
            const uint64_t *from = rows + (int64_t)max(next, 0) * words;
            bool in = next == -1 && c < words;
            int32_t depth = __builtin_popcountll(m);
            if (next >= 0 && c < words) {
                in = (from[next >> 6] >> (next & 63)) & 1;      // (a node of the tree sees itself)
                depth += pos[next] - p + 1;
            }
            for (int32_t w = 0; w < words; ++w) {
                const uint64_t before = in && w < c && next >= 0 ? from[w] : 0ull;
                row[w] = w == c && in ? m : before;
            }
            pos[i] = in ? p + depth - 1 : p;
        }
        __threadfence_block();                                  // the rows are read by other lanes next
    }
}

// Pools of one launch: they travel in its arguments.
constexpr int kLayersPerLaunch = 128;
constexpr int kMaxLayers = 256;
struct CompactArgs {
    u16 *k[kLayersPerLaunch], *v[kLayersPerLaunch];
    const int32_t *block_tables, *prefix_lens, *path, *accepted_lens;
    int32_t max_blocks, num_blocks, Hkv, path_cap;
};

constexpr int kCompactThreads = 256;
constexpr int kBatch = 8;      // tokens of a path moved at a time

// Grid (slices of the kv heads, sequences, layers). The path is strictly increasing and path[i] >= i, so
// that no token of a batch reads a slot that an earlier batch wrote; inside a batch every read
// comes before every write. A thread takes 16 bytes of one head's K row, and one head's V of one dim.
// V's layout bounds it: a token's V of one head is D values 32 bytes apart, so a move touches the whole payload of
// its blocks. 64 sequences that keep up to 8 of 32 nodes in 80 layers of 8 heads of 128 (204 tokens moved, 134 MB of
// K and V in and out): 269 MB read, 215 MB written, 120-124 us, 4.0 TB/s where a large copy reaches 4.9. (V's target
// rows read, changed and written whole: 124 us; two, four or eight layers a workgroup, with all their loads
// before their stores: 124-133.)
template <int D>
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(const CompactArgs a)
{
    constexpr int kHeads = kCompactThreads / D;             // of a workgroup
    constexpr int kPieces = D / 8;                          // of a K row
    constexpr int kTokens = kCompactThreads / (kHeads * kPieces);   // K rows of all the heads at a time
    constexpr int kRounds = kBatch / kTokens;
    __shared__ int32_t slot_s[kBatch], slot_d[kBatch];      // -1: not moved
    const int tid = threadIdx.x, b = blockIdx.y, layer = blockIdx.z, g0 = blockIdx.x * kHeads;
    const int32_t len = min(a.accepted_lens[b], a.path_cap), p = a.prefix_lens[b];
    if (len <= 0 || p < 0) return;
    const int32_t *path = a.path + (int64_t)b * a.path_cap, *row = a.block_tables + (int64_t)b * a.max_blocks;
    u16 *kp = a.k[layer], *vp = a.v[layer];
    auto slot = [&](int64_t pos) -> int32_t {               // of a position, -1 where there is none
        if (pos >= (int64_t)a.max_blocks * kBlockSize) return -1;
        const int32_t id = row[pos / kBlockSize];
        return (uint32_t)id < (uint32_t)a.num_blocks ? id * kBlockSize + (int32_t)(pos % kBlockSize) : -1;
    };
    bool open = true;
    for (int32_t i0 = 0; i0 < len && open; i0 += kBatch) {
        const int32_t here = min(len - i0, kBatch);
        // The first entry that is not in order, or has no slot, ends the moves.
        if (tid < 64) {
            const int32_t i = i0 + tid;
            int32_t s = -1, d = -1;
            bool bad = false;
            if (tid < here) {
                const int32_t x = path[i], before = i > 0 ? path[i - 1] : -1;
                bad = x <= before || x < i;
                if (!bad && x != i) {
                    s = slot((int64_t)p + x);
                    d = slot((int64_t)p + i);
                    bad = s < 0 || d < 0;
                }
            }
            const uint64_t stop = __builtin_amdgcn_ballot_w64(bad);
            const int first = stop ? (int)__builtin_ctzll(stop) : kBatch;
            if (tid < kBatch) {
                slot_s[tid] = tid < first ? s : -1;
                slot_d[tid] = tid < first ? d : (stop ? -2 : -1);
            }
        }
        __syncthreads();
        open = slot_d[kBatch - 1] != -2;
        u32x4 kr[kRounds];
        const int kg = g0 + tid / kPieces % kHeads, kx = tid % kPieces, kt = tid / (kPieces * kHeads);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int32_t s = slot_s[r * kTokens + kt];
            if (s >= 0 && kg < a.Hkv)
                kr[r] = *reinterpret_cast<const u32x4 *>(
                    kp + (((int64_t)(s / kBlockSize) * a.Hkv + kg) * kBlockSize + s % kBlockSize) * D + 8 * kx);
        }
        u16 vr[kBatch];
        const int vg = g0 + tid / D, x = tid % D;
#pragma unroll
        for (int r = 0; r < kBatch; ++r) {
            const int32_t s = slot_s[r];
            if (s >= 0 && vg < a.Hkv) vr[r] = vp[(((int64_t)(s / kBlockSize) * a.Hkv + vg) * D + x) * kBlockSize + s % kBlockSize];
        }
        __syncthreads();                                    // K rows of a batch are other threads' too
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int32_t d = slot_d[r * kTokens + kt];
            if (d >= 0 && kg < a.Hkv)
                *reinterpret_cast<u32x4 *>(
                    kp + (((int64_t)(d / kBlockSize) * a.Hkv + kg) * kBlockSize + d % kBlockSize) * D + 8 * kx) = kr[r];
        }
#pragma unroll
        for (int r = 0; r < kBatch; ++r) {
            const int32_t d = slot_d[r];
            if (d >= 0 && vg < a.Hkv) vp[(((int64_t)(d / kBlockSize) * a.Hkv + vg) * D + x) * kBlockSize + d % kBlockSize] = vr[r];
        }
        __syncthreads();                                    // the next batch writes the slots again
    }
}

constexpr int32_t kMaxSeqs = 65535;   // of compact_kv: a dimension of the grid

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_draft_tree(int32_t B, const int32_t *cu_nodes, const int32_t *parents, const int32_t *prefix_lens,
                          int32_t T, int32_t mask_words, uint64_t *visible, int32_t *positions, void *stream)
{
    clear_error();
    const char *who = "pcr_draft_tree";
    if (B < 0 || T < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative B or T", who);
    if (mask_words < 1 || mask_words > kMaxMaskWords)
        return fail(PCR_ERR_UNSUPPORTED, "%s: mask_words %d is not in 1 .. %d", who, mask_words, kMaxMaskWords);
    if (B > kMaxTreeSeqs || T > kMaxTreeNodes) return fail(PCR_ERR_UNSUPPORTED, "%s: batch too large", who);
    if (B == 0 || T == 0) return PCR_OK;
    if (!cu_nodes || !parents || !prefix_lens || !visible || !positions)
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL argument", who);
    if ((uintptr_t)visible & 7) return fail(PCR_ERR_INVALID_ARG, "%s: visible must be 8-byte aligned", who);
    hipLaunchKernelGGL(draft_tree_kernel, dim3(B), dim3(64), 0, static_cast<hipStream_t>(stream), cu_nodes,
                       parents, prefix_lens, T, mask_words, visible, positions);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "pcr_draft_tree: launch");
    return PCR_OK;
}

pcr_status pcr_compact_kv(const pcr_kv_pool *pools, int32_t n_layers, const int32_t *block_tables, int32_t max_blocks,
                          const int32_t *prefix_lens, const int32_t *path, int32_t path_cap,
                          const int32_t *accepted_lens, int32_t B, void *stream)
{
    clear_error();
    const char *who = "pcr_compact_kv";
    if (B < 0 || n_layers < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative B or n_layers", who);
    if (n_layers > kMaxLayers) return fail(PCR_ERR_UNSUPPORTED, "%s: more than %d layers", who, kMaxLayers);
    if (B > kMaxSeqs) return fail(PCR_ERR_UNSUPPORTED, "%s: more than %d sequences", who, kMaxSeqs);
    if (n_layers > 0 && !pools) return fail(PCR_ERR_INVALID_ARG, "%s: pools is NULL", who);
    // [start, end) of every array, to be told apart
    uintptr_t at[2 * kMaxLayers];
    for (int32_t l = 0; l < n_layers; ++l) {
        const pcr_status st = check_pool(pools + l, who);
        if (st) return st;
        if (pools[l].num_kv_heads != pools[0].num_kv_heads || pools[l].head_dim != pools[0].head_dim ||
            pools[l].num_blocks != pools[0].num_blocks)
            return fail(PCR_ERR_INVALID_ARG, "%s: layer %d's pool has another shape than the first's", who, l);
        at[2 * l] = (uintptr_t)pools[l].k;
        at[2 * l + 1] = (uintptr_t)pools[l].v;
    }
    if (n_layers > 0) {
        if (pools[0].num_blocks > INT32_MAX / kBlockSize)
            return fail(PCR_ERR_UNSUPPORTED, "%s: tokens of %d blocks overflow int32", who, pools[0].num_blocks);
        const uintptr_t bytes = (uintptr_t)pools[0].num_blocks *
                                kv_block_bytes(kBlockSize, pools[0].num_kv_heads, pools[0].head_dim);
        std::sort(at, at + 2 * n_layers);
        for (int32_t i = 1; i < 2 * n_layers; ++i)
            if (at[i] - at[i - 1] < bytes) return fail(PCR_ERR_INVALID_ARG, "%s: two layers' K or V overlap", who);
    }
    if (max_blocks < 1 || path_cap < 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: max_blocks and path_cap must be positive", who);
    if (B == 0 || n_layers == 0) return PCR_OK;
    if (!block_tables || !prefix_lens || !path || !accepted_lens)
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL device argument", who);
    const int D = pools[0].head_dim, heads = kCompactThreads / D;
    CompactArgs a{};
    a.block_tables = block_tables;
    a.prefix_lens = prefix_lens;
    a.path = path;
    a.accepted_lens = accepted_lens;
    a.max_blocks = max_blocks;
    a.num_blocks = pools[0].num_blocks;
    a.Hkv = pools[0].num_kv_heads;
    a.path_cap = path_cap;
    for (int32_t l0 = 0; l0 < n_layers; l0 += kLayersPerLaunch) {
        const int32_t here = std::min(n_layers - l0, kLayersPerLaunch);
        for (int32_t l = 0; l < here; ++l) {
            a.k[l] = static_cast<u16 *>(pools[l0 + l].k);
            a.v[l] = static_cast<u16 *>(pools[l0 + l].v);
        }
        const dim3 grid((a.Hkv + heads - 1) / heads, B, here);
        hipLaunchKernelGGL(D == 128 ? compact_kernel<128> : compact_kernel<64>, grid, dim3(kCompactThreads), 0,
                           static_cast<hipStream_t>(stream), a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "pcr_compact_kv: launch");
    }
    return PCR_OK;
}

}  // extern "C"
