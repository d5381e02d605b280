// One wave's part of tree attention: the keys [kbeg, kend) of one (sequence, kv head) for up to
// 16 NC of its packed query rows (row r = node r / G, head-in-group r % G), as in decode_wave.h but with
// NC column tiles of 16 rows, all fed from one copy of K and V in registers:
//   S^T[key][row] = K Q^T     A = 16 key rows x 32 dims of K,  B = Q^T (registers)
//   O^T[d][row]  += V^T P^T   A = 16 dims x 32 keys of V^T,    B = P^T (registers)
// Lane (c, q4) holds row c of each tile and keys 8 q4 .. 8 q4 + 7 of a 32-key step.
//
// Keys below `prefix` are seen by every row. Key prefix + k is node k, seen by the rows whose words
// have bit k. What a row does not see does not reach it, whatever the slot holds: its score
// becomes -inf (a NaN of K goes with it), and V entries of nodes that are infinite or NaN enter
// the product as 0, since 0 * inf is NaN; the rows that do see such an entry get it added apart.
#pragma once

#include "pcr_internal.h"

namespace pcr {
namespace tree_wave {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16;

constexpr int kStepKeys = 32;   // keys per step: two pool blocks
// The running max before any finite score (decode_wave.h).
constexpr float kNoMax = -__FLT_MAX__;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

template <int D>
struct StepRegs {
    u32x4 k[2][D / 32];   // K operands of the two products (row group r, dims 32*kk ..)
    u32x4 v[D / 16];      // V^T operands (dims 16*mt ..)
};

// Bits [d, d + 8) of a row's words (the first of them in a register), where bits below 0 are set and those
// from n on are not.
__device__ __forceinline__ unsigned seen8(const uint64_t *__restrict__ words, uint64_t first, int32_t n_words, int d, int n)
{
    const int lo = max(d, 0), w = lo >> 6, sh = lo & 63;
    uint64_t x = w == 0 ? first >> sh : 0ull;
    if (n_words > 1) {                                  // wave-uniform
        if (w > 0 && w < n_words) x = words[w] >> sh;
        if (sh > 56 && w + 1 < n_words) x |= words[w + 1] << (64 - sh);
    }
    const int cached = min(lo - d, 8);                  // bits below 0
    unsigned bits = cached == 8 ? 0xFFu : (((unsigned)x << cached) | ((1u << cached) - 1)) & 0xFFu;
    if (d + 8 > n) bits &= n > d ? (1u << (n - d)) - 1 : 0u;
    return bits;
}

// What a wave needs to know of its sequence and rows.
struct Rows {
    const uint64_t *visible;      // words of the sequence's first node
    int32_t n_words;
    int32_t prefix, nodes;
    int32_t rows;                 // packed rows, up to 16 NC
    int32_t G;
};

// q: the sequence's first node's first head of this kv head; q_stride: elements from node to node.
// bt_row: the sequence's block-table row; last_blk: its last block with a key.
template <int D, int NC, bool K_CACHED>
__device__ __forceinline__ void chunk(const u16 *__restrict__ q, int64_t q_stride, const Rows &rw,
                                      const u16 *__restrict__ pool_k, const u16 *__restrict__ pool_v,
                                      int32_t num_blocks, int32_t Hkv, int g, const int32_t *__restrict__ bt_row,
                                      int last_blk, int kbeg, int kend, float scale_log2, f32x4 (&o)[NC][D / 16],
                                      float (&m_run)[NC], float (&l_run)[NC])
{
    constexpr int KK = D / 32, MT = D / 16;
    const int lane = (int)(threadIdx.x & 63);
    const int c = lane & 15, q4 = lane >> 4;

    // Q^T operands: lane (c, q4) holds dims 32*kk + 8*q4 .. +7 of its row (zero past the last).
    u32x4 qf[NC][KK];
    uint64_t first[NC];           // the rows' first words, asked for here: a load in the step waits a microsecond
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        const int r = 16 * t + c;
        const bool col = r < rw.rows;
        const int pr = col ? r : 0, node = pr / rw.G, h = pr - node * rw.G;
        first[t] = rw.visible[(int64_t)node * rw.n_words];
        const u16 *qrow = q + (int64_t)node * q_stride + h * D + 8 * q4;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const u32x4 raw = *reinterpret_cast<const u32x4 *>(qrow + 32 * kk);
            qf[t][kk] = col ? raw : u32x4{0u, 0u, 0u, 0u};
        }
    }

    auto block_id = [&](int li) __attribute__((always_inline)) -> int32_t {
        const int32_t id = bt_row[min(li, last_blk)];
        return (uint32_t)id < (uint32_t)num_blocks ? id : 0;   // a bad entry reads block 0, never outside
    };
    const int krow = 8 * ((c >> 2) & 1) + (c & 3);    // slot of row group 0; row group 1 is 4 slots on
    auto load_v = [&](int step, StepRegs<D> &R) __attribute__((always_inline)) {
        const int li = (kbeg + step * kStepKeys) >> 4;
        const int32_t b0 = block_id(li), b1 = block_id(li + 1);
        const int32_t vb = (q4 >> 1) ? b1 : b0;
        const u16 *vp = pool_v + ((int64_t)vb * Hkv + g) * (kBlockSize * D) + c * kBlockSize + 8 * (q4 & 1);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            R.v[mt] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + 16 * mt * kBlockSize));
    };
    auto load_step = [&](int step, StepRegs<D> &R) __attribute__((always_inline)) {
        const int li = (kbeg + step * kStepKeys) >> 4;
        const int32_t b0 = block_id(li), b1 = block_id(li + 1);
        const int32_t kb = (c >> 3) ? b1 : b0;
        const u16 *kp = pool_k + ((int64_t)kb * Hkv + g) * (kBlockSize * D) + krow * D + 8 * q4;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const u32x4 *kq = reinterpret_cast<const u32x4 *>(kp + 4 * r * D + 32 * kk);
                if constexpr (K_CACHED)
                    R.k[r][kk] = *kq;
                else
                    R.k[r][kk] = __builtin_nontemporal_load(kq);
            }
        load_v(step, R);
    };

#pragma unroll
    for (int t = 0; t < NC; ++t) {
        m_run[t] = kNoMax;
        l_run[t] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Scores of tile t and their softmax: P^T operand, running max and sum, O rescaled.
    // P is rounded to bf16, as the matrix instruction takes it beside V: the result is off by 0.0020-0.0023 of
    // its size where weights of 32 bits leave 0.0016-0.0017 (most of it the output's own rounding). The rest of P in a
    // second product would take MT more per step. The sum adds what was rounded, so the weights sum to one.
    auto probabilities = [&](int t, const StepRegs<D> &R, unsigned seen, bool masked) __attribute__((always_inline)) -> bf16x8 {
        f32x4 s[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                s[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(R.k[r][kk]), as_bf16x8(qf[t][kk]), s[r],
                                                               0, 0, 0);
        }
        if (masked) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!((seen >> (4 * r + i)) & 1)) s[r][i] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                         fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run[t], mx * scale_log2);   // at least kNoMax: finite also where mx is -inf
        const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        bf16x8 pb;
        float ps = 0.f;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][i], scale_log2, -m_new));
                pb[4 * r + i] = (__bf16)p;
                ps += (float)pb[4 * r + i];     // the rounded value the product weights V with
            }
        l_run[t] = l_run[t] * alpha + ps;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {   // the max rose in some row
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[t][mt] *= alpha;
        }
        return pb;
    };

    // A step of cached keys only.
    auto process = [&](const StepRegs<D> &R) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < NC; ++t) {
            const bf16x8 pb = probabilities(t, R, 0xFFu, false);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(R.v[mt]), pb, o[t][mt], 0, 0, 0);
        }
    };
    // A step with nodes, or with keys from kend on.
    auto process_masked = [&](int step, StepRegs<D> &R) __attribute__((always_inline)) {
        const int k0 = kbeg + step * kStepKeys + 8 * q4;     // this lane's 8 keys
        const int cached = rw.prefix - k0;                   // of them, the first `cached` are cached tokens
        // V's infinite and NaN entries of nodes cleared.
        uint32_t odd = 0;
#pragma unroll
        for (int wd = 0; wd < 4; ++wd) {
            const uint32_t lo = 2 * wd >= cached ? 0x7F80u : 0xFFFFFFFFu, hi = 2 * wd + 1 >= cached ? 0x7F800000u : 0xFFFFFFFFu;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint32_t x = R.v[mt][wd];
                const uint32_t gone = ((x & 0x7F80u) == lo ? 0xFFFFu : 0u) | ((x & 0x7F800000u) == hi ? 0xFFFF0000u : 0u);
                odd |= gone;
                R.v[mt][wd] = x & ~gone;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        bf16x8 pb[NC];
#pragma unroll
        for (int t = 0; t < NC; ++t) {
            const int r = 16 * t + c;
            const int node = (r < rw.rows ? r : 0) / rw.G;
            unsigned seen = seen8(rw.visible + (int64_t)node * rw.n_words, first[t], rw.n_words, k0 - rw.prefix, rw.nodes);
            if (kend - k0 < 8) seen &= kend > k0 ? (1u << (kend - k0)) - 1 : 0u;
            __builtin_amdgcn_sched_barrier(0);
            pb[t] = probabilities(t, R, seen, true);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(R.v[mt]), pb[t], o[t][mt], 0, 0, 0);
        }
        if (__builtin_amdgcn_ballot_w64(odd != 0)) {
            load_v(step, R);                                 // as it was
            // How many +inf, -inf and NaN entries each row sees with a weight, by a product of
            // ones; they end in O as the sum that has them.
#pragma unroll
            for (int t = 0; t < NC; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) pb[t][e] = (float)pb[t][e] > 0.f ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll 1
            for (int kind = 0; kind < 3; ++kind) {
                const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
                // (the bit patterns in numbers of the kind: as comparisons by kind they all left the loop, 400 spills)
                const uint32_t flip = kind == 1 ? 0x8000u : 0u, keep = kind == 2 ? 0x7FFFu : 0xFFFFu;
                const uint32_t first = kind == 2 ? 0x7F81u : 0x7F80u, span = kind == 2 ? 0x7Eu : 0u;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    bf16x8 is;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t x = (R.v[mt][e / 2] >> (16 * (e & 1))) & 0xFFFFu;
                        const bool hit = ((x ^ flip) & keep) - first <= span;
                        is[e] = hit && e >= cached ? (__bf16)1.f : (__bf16)0.f;
                    }
#pragma unroll
                    for (int t = 0; t < NC; ++t) {
                        const f32x4 n =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, pb[t], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[t][mt][i] += n[i] > 0.f ? add : 0.f;
                    }
                    __builtin_amdgcn_sched_barrier(0);     // (no eight products' comparisons at a time)
                }
            }
        }
    };

    // Every load is unconditional (a step index past the end rereads the last step). Full steps of cached
    // keys first, the two sets of registers taking turns; then the others, one at a time. (A third set, as in
    // decode_wave.h, took more: one node's four heads of 64 sequences of 500-4096 keys 123 us with two sets and 127
    // with three, two tiles of columns 141 and 172.)
    const int n_steps = (kend - kbeg + kStepKeys - 1) / kStepKeys;
    const int n_plain = max(0, min(kend, rw.prefix) - kbeg) / kStepKeys;
    auto load = [&](int j, StepRegs<D> &R) __attribute__((always_inline)) { load_step(min(j, n_steps - 1), R); };
    StepRegs<D> ra, rb;
    load(0, ra);
    int j = 0;
    for (; j + 2 <= n_plain; j += 2) {
        load(j + 1, rb);
        process(ra);
        load(j + 2, ra);
        process(rb);
    }
    if (j < n_plain) {
        load(++j, rb);
        process(ra);
        ra = rb;
    }
#pragma unroll 1
    for (; j < n_steps; ++j) {
        load(j + 1, rb);
        process_masked(j, ra);
        ra = rb;
    }
}

}  // namespace tree_wave
}  // namespace pcr
