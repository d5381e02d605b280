// Which of a tile's tokens one append workgroup writes, and how their V leaves it; shared by the
// append kernel (kv_move.hip) and the one that rotates K first (rope.hip).
//
// A workgroup takes about TILE new tokens. Tokens that go on inside the pool block of the token
// before the tile belong to the tile before, so a tile leaves out up to 15 tokens at its start
// and takes up to 15 after its end: no block is written by two workgroups. V is written
// d-major: a run of tokens inside one aligned chunk of 8 slots is one 16-byte store per dim where
// it fills the chunk.
#pragma once

#include "pcr_internal.h"

namespace pcr {
namespace append_tile {

constexpr int kExt = kBlockSize - 1;           // tokens after the tile it may take

// One wave, all 64 lanes. sl: the slot of token tok0 + lane if it is this tile's (else -1);
// follows: whether it follows the slot of the token before; last: one past the tile's last row.
template <int TILE>
__device__ __forceinline__ void own_slots(const int32_t *__restrict__ slot_mapping, int32_t T, int32_t num_blocks,
                                          int tok0, int32_t &sl, bool &follows, int &last)
{
    constexpr int ROWS = TILE + kExt;
    static_assert(ROWS < 64, "one wave ranks the chunk runs");
    static_assert(TILE >= kBlockSize, "a tile starts a block");
    const int tid = threadIdx.x & 63;
    sl = -1;
    // Lane 63 reads the slot of the token before the tile (all slots in one load).
    const int t = tid == 63 ? tok0 - 1 : tok0 + tid;
    if ((tid < ROWS || tid == 63) && t >= 0 && t < T) {
        sl = slot_mapping[t];
        if (sl < 0 || sl / kBlockSize >= num_blocks) sl = -1;
    }
    // the slot of the token before this one (the wave rotated by one lane: DPP wave_ror:1)
    const int32_t before = __builtin_amdgcn_update_dpp(sl, sl, 0x13C, 0xf, 0xf, false);
    if (tid == 63) sl = -1;
    follows = sl >= 0 && before >= 0 && sl == before + 1;
    // heads: tokens that do not go on inside the block of the token before them. The
    // tile's own tokens run from its first head to the first head at or after its end
    // (both within 15 tokens: a block has 16 slots).
    const uint64_t heads = ~__builtin_amdgcn_ballot_w64(follows && sl % kBlockSize != 0);
    const uint64_t rest = heads >> TILE;
    const int first = (int)__builtin_ctzll(heads);
    last = rest ? min(ROWS, TILE + (int)__builtin_ctzll(rest)) : ROWS;
    if (tid < first || tid >= last) sl = -1;
}

// One wave, with own_slots' results: runs[i] = (first row << 8) | rows of the i-th chunk run.
__device__ __forceinline__ void chunk_runs(int32_t sl, bool follows, int32_t *runs, int32_t &n_runs)
{
    const int tid = threadIdx.x & 63;
    // A token starts a chunk run when its slot is valid and either opens an aligned chunk
    // of 8 slots or does not follow the previous token's slot; the run goes on over the
    // following tokens until the next start or invalid slot (a continuing token's slot
    // is its predecessor's plus one, inside the same chunk).
    const bool valid = sl >= 0;
    const bool start = valid && (tid == 0 || sl % 8 == 0 || !follows);
    const uint64_t starts = __builtin_amdgcn_ballot_w64(start);
    const uint64_t stops = starts | ~__builtin_amdgcn_ballot_w64(valid);   // bits past the rows are stops
    if (start) {
        const uint64_t after = tid == 63 ? 0ull : stops >> (tid + 1);
        const int len = after ? 1 + __builtin_ctzll(after) : 64 - tid;
        const int idx = __builtin_popcountll(starts & ((1ull << tid) - 1ull));
        runs[idx] = (tid << 8) | len;
    }
    if (tid == 0) n_runs = __builtin_popcountll(starts);
}

// The workgroup (256 threads): V rows in LDS (kv head g) into the pool. Task = (run, dim).
template <int D, int STRIDE>
__device__ __forceinline__ void put_v(const unsigned short (*vs)[STRIDE], const int32_t *slots, const int32_t *runs,
                                      int n_runs, unsigned short *__restrict__ pool_v, int32_t Hkv, int g)
{
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    const int nr = n_runs;
    for (int task = threadIdx.x; task < nr * D; task += 256) {
        const int k = task / D, x = task % D;
        const int rv = runs[k], r0 = rv >> 8, len = rv & 0xff;
        const int32_t s0 = slots[r0];
        const int64_t blk = s0 / kBlockSize, o = s0 % kBlockSize;
        unsigned short *dst = pool_v + ((blk * Hkv + g) * D + x) * kBlockSize + o;
        if (len == 8) {   // a whole aligned chunk (a run of 8 starts at a multiple of 8)
            unsigned short e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = vs[r0 + j][x];
            u32x4 w;
            w.x = e[0] | ((unsigned)e[1] << 16);
            w.y = e[2] | ((unsigned)e[3] << 16);
            w.z = e[4] | ((unsigned)e[5] << 16);
            w.w = e[6] | ((unsigned)e[7] << 16);
            *reinterpret_cast<u32x4 *>(dst) = w;
        } else {
            for (int j = 0; j < len; ++j) dst[j] = vs[r0 + j][x];
        }
    }
}

}  // namespace append_tile
}  // namespace pcr
