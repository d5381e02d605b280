// Cross attention of few query rows per sequence (decode steps, beams) for gfx950: bound by
// reading K and V of every (sequence, kv head) once.
//
// The work is the 32-key steps of all pairs (sequence, kv head). A workgroup takes a run of them,
// cut in one of three ways (cross_rows_plan):
//   a run is a whole pair: one launch, nothing to merge through memory;
//   a run is one of k equal parts of a pair: few pairs of long keys;
//   the steps of all pairs laid end to end are shared out evenly, whatever pair they belong to:
//     ragged batches and counts of pairs that leave compute units idle otherwise.
// Inside a run each pair's part (a segment) is cut once more among the workgroup's waves, which
// hold the up to 16 packed rows of the pair as matrix columns (decode_wave.h) and merge in LDS. A
// segment that is its whole pair writes the rows; the others leave (O, max, sum) in the
// workspace, at most two of a run (its first and its last), and cross_rows_combine_kernel
// merges the parts of each pair. K loads go past the caches, except in whole pairs, whose waves
// end at different times (one token each, 32 / 8 heads of 128, ordinary loads and past the caches:
// 64 ragged sequences of up to 6404 keys in even runs 187 and 181 us, as whole pairs 186 and 207;
// one sequence of 6404 keys, in parts, 14.9 and 14.1 us).
#include <algorithm>
#include <type_traits>

#include "decode_wave.h"
#include "pcr_internal.h"

namespace pcr {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16;

// What a run is (see above).
enum Cut { kWhole, kParts, kEven };

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStepKeys = decode_wave::kStepKeys;

// (Pointers are kernel parameters of their own: what is read carries __restrict__, without which
// the block ids would not be scalar loads but wait, in order, for the K/V loads before them.)
struct CrossArgs {
    int32_t num_blocks, Hkv, Hq, max_blocks, B, T;
    int32_t cols;                 // packed rows of a sequence, at most
    int32_t steps;                // of all pairs
    int32_t runs;
    int32_t base, rem;            // steps of a run (run_begin); even cut only
    int32_t parts;                // runs of a pair; cut by pairs only
    float scale_log2;
};

// Steps of one pair of sequence b (0: no rows or no keys, nothing to read).
__device__ __forceinline__ int pair_steps(const CrossArgs &a, const int32_t *__restrict__ key_lens,
                                          const int32_t *__restrict__ cu_q, int b, int &n_keys, int &t0, int &rows)
{
    t0 = cu_q[b];
    rows = min((min(cu_q[b + 1], a.T) - t0) * (a.Hq / a.Hkv), a.cols);
    n_keys = (int)min((int64_t)key_lens[b], (int64_t)a.max_blocks * kBlockSize);
    return t0 < 0 || rows <= 0 || n_keys <= 0 ? 0 : (n_keys + kStepKeys - 1) / kStepKeys;
}

// First step of run u: the first `rem` runs have base + 1 steps, the others base.
__device__ __forceinline__ int run_begin(const CrossArgs &a, int u) { return u * a.base + min(u, a.rem); }
// The run that holds step x.
__device__ __forceinline__ int run_of(const CrossArgs &a, int x)
{
    const int big = a.rem * (a.base + 1);
    return x < big ? x / (a.base + 1) : a.rem + (x - big) / a.base;
}

// Where a wave stands: sequence b, its first step, its steps per pair, keys and rows.
struct At {
    int b, first, st, n_keys, t0, rows;
};

// The sequence that holds step x (all lanes of a wave); false where there is none (device lengths
// shorter than the host's).
__device__ __forceinline__ bool find_sequence(const CrossArgs &a, const int32_t *__restrict__ key_lens,
                                              const int32_t *__restrict__ cu_q, int x, At &at)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int n = 0, t0 = 0, rows = 0, st = 0;
        if (b0 + lane < a.B) st = pair_steps(a, key_lens, cu_q, b0 + lane, n, t0, rows);
        int v = st * a.Hkv;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int u = __shfl_up(v, off);
            if (lane >= off) v += u;
        }
        const uint64_t over = __builtin_amdgcn_ballot_w64(before + v > x);
        if (over) {
            const int l = (int)__builtin_ctzll(over);
            at.b = b0 + l;
            at.st = __builtin_amdgcn_readlane(st, l);
            at.first = before + __builtin_amdgcn_readlane(v, l) - at.st * a.Hkv;
            at.n_keys = __builtin_amdgcn_readlane(n, l);
            at.t0 = __builtin_amdgcn_readlane(t0, l);
            at.rows = __builtin_amdgcn_readlane(rows, l);
            return true;
        }
        before += __builtin_amdgcn_readlane(v, 63);
    }
    return false;
}

template <int D, int WAVES, int CUT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(1))) void cross_rows_kernel(
    const CrossArgs a, const u16 *__restrict__ q, const u16 *__restrict__ pool_k, const u16 *__restrict__ pool_v,
    const int32_t *__restrict__ block_tables, const int32_t *__restrict__ key_lens, const int32_t *__restrict__ cu_q,
    u16 *__restrict__ out, float *__restrict__ ws_o, float *__restrict__ ws_ml)
{
    constexpr int MT = D / 16;
    __shared__ f32x4 part_o[WAVES > 1 ? WAVES - 1 : 1][MT][64];
    __shared__ f32x2 part_ml[WAVES > 1 ? WAVES - 1 : 1][64];
    const int lane = threadIdx.x & 63, c = lane & 15, q4 = lane >> 4;
    const int wave = WAVES > 1 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) : 0;
    const int run = blockIdx.x;
    const int G = a.Hq / a.Hkv, ct = c / G, cg = c - ct * G;
    int x0, x1;
    At at;
    if constexpr (CUT != kEven) {                      // part `run % parts` of pair `run / parts`
        const int pair = run / a.parts, part = run - pair * a.parts;
        at.b = pair / a.Hkv;
        at.st = pair_steps(a, key_lens, cu_q, at.b, at.n_keys, at.t0, at.rows);
        at.first = 0;
        const int per = (at.st + a.parts - 1) / a.parts, begin = (pair - at.b * a.Hkv) * at.st;
        x0 = begin + min(at.st, part * per);
        x1 = begin + min(at.st, (part + 1) * per);
    } else {
        x0 = run_begin(a, run);
        x1 = run_begin(a, run + 1);
        if (!find_sequence(a, key_lens, cu_q, x0, at)) return;
    }
    for (int x = x0; x < x1;) {
        while (CUT == kEven && x >= at.first + at.st * a.Hkv) {   // on to the next sequence with steps
            at.first += at.st * a.Hkv;
            if (++at.b >= a.B) return;
            at.st = pair_steps(a, key_lens, cu_q, at.b, at.n_keys, at.t0, at.rows);
        }
        const int b = at.b, st = at.st, n_keys = at.n_keys, t0 = at.t0, rows = at.rows;
        const int g = (x - at.first) / st, s0 = (x - at.first) - g * st;
        const int s1 = min(st, s0 + (x1 - x));         // the segment: steps [s0, s1) of the pair
        const bool whole = s0 == 0 && s1 == st;
        const int per = (s1 - s0 + WAVES - 1) / WAVES;
        const int kbeg = (s0 + wave * per) * kStepKeys;
        const int kend = min(n_keys, min(s1, s0 + (wave + 1) * per) * kStepKeys);
        const bool col = c < rows;
        const int64_t row = (int64_t)(t0 + ct) * a.Hq + g * G + cg;
        f32x4 o[MT];
        float m = decode_wave::kNoMax, l = 0.f;
        if (kbeg < kend) {
            const u16 *qrow = q + (col ? row : (int64_t)t0 * a.Hq + g * G) * D + 8 * q4;
            decode_wave::chunk<D, 3, CUT == kWhole>(qrow, col, pool_k, pool_v, a.num_blocks, a.Hkv, g,
                                               block_tables + (int64_t)b * a.max_blocks, (n_keys - 1) >> 4, kbeg, kend,
                                               a.scale_log2, o, m, l);
        } else {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if constexpr (WAVES > 1) {
            // Waves 1.. leave O (lane layout), max and sum in LDS; wave 0 merges. A part past the
            // segment's end, or without a finite score, has max kNoMax, sum 0, O 0.
            if (wave > 0) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) part_o[wave - 1][mt][lane] = o[mt];
                part_ml[wave - 1][lane] = f32x2{m, l};
            }
            __syncthreads();
            if (wave == 0) {
                float M = m;
                for (int w = 0; w < WAVES - 1; ++w) M = fmaxf(M, part_ml[w][lane][0]);
                const float a0 = __builtin_amdgcn_exp2f(m - M);
                l *= a0;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[mt] *= a0;
                for (int w = 0; w < WAVES - 1; ++w) {
                    const f32x2 ml = part_ml[w][lane];
                    const float aw = __builtin_amdgcn_exp2f(ml[0] - M);
                    l += aw * ml[1];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) o[mt] += aw * part_o[w][mt][lane];
                }
                m = M;
            }
        }
        if (wave == 0 && col) {
            if (whole) {
                const float inv = 1.f / l;
                u16 *orow = out + row * D + 4 * q4;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const bf16x4 v = __builtin_convertvector(o[mt] * inv, bf16x4);
                    *reinterpret_cast<u32x2 *>(orow + 16 * mt) = __builtin_bit_cast(u32x2, v);
                }
            } else if (ws_o) {                         // (device lengths that are not the host's may cut more pairs)
                const int64_t part = (int64_t)(CUT != kEven ? run : 2 * run + (x == x0 ? 0 : 1)) * a.cols + c;
                float *po = ws_o + part * D + 4 * q4;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4 *>(po + 16 * mt) = o[mt];
                if (q4 == 0) *reinterpret_cast<f32x2 *>(ws_ml + 2 * part) = f32x2{m, l};
            }
        }
        x += s1 - s0;
        if constexpr (WAVES > 1 && CUT == kEven) __syncthreads();   // the next segment writes the parts again
    }
}

// out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p with M = max_p m_p, over the parts p of a pair
// cut between runs, in their order. One wave per (pair, column) of a batch cut by pairs. In an even
// cut one per (run from the second on, column): of a pair that is cut one run is the first to begin
// inside it, and that run's wave merges it. So the waves are bounded by the runs, and the time
// grows with the sequences as one scan of them does. A wave per pair, each of which sums the
// sequences before its own, took time with their square and at 2^22 pairs of 16 columns more
// threads than a launch has (16 / 4 heads of 64, sequences of 30-60 keys and one of 3000: 16384 of them
// 1648 us that way, 424 this; 4096 169 and 111; 300 15.5 and 15.8; 64 ragged ones alike).
constexpr int kCombineWaves = 4;
template <int D, int CUT>
__global__ __launch_bounds__(64 * kCombineWaves) void cross_rows_combine_kernel(
    const CrossArgs a, const int32_t *__restrict__ key_lens, const int32_t *__restrict__ cu_q,
    const float *__restrict__ ws_o, const float *__restrict__ ws_ml, u16 *__restrict__ out)
{
    constexpr int E = D / 64;     // output elements per lane
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int task = blockIdx.x * kCombineWaves + wave;
    const int nth = task / a.cols, c = task - nth * a.cols;
    int g, t0, rows;              // kv head of the pair, first row and packed rows of its sequence
    int slot0, odd = 0, parts;    // slot of the first part (plus odd), slots from part to part, parts
    constexpr int kStride = CUT == kParts ? 1 : 2;
    if constexpr (CUT == kParts) {
        const int b = nth / a.Hkv;
        g = nth - b * a.Hkv;
        if (b >= a.B) return;
        int n;
        const int st = pair_steps(a, key_lens, cu_q, b, n, t0, rows);
        if (st == 0) return;
        const int per = (st + a.parts - 1) / a.parts;
        parts = (st + per - 1) / per;
        slot0 = nth * a.parts;
    } else {
        const int u0 = nth, x1 = run_begin(a, u0 + 1);   // does run u0 + 1 begin inside a pair that u0 begins?
        At at;
        if (u0 + 1 >= a.runs || !find_sequence(a, key_lens, cu_q, x1, at)) return;
        if ((uint32_t)(x1 - at.first) >= (uint32_t)(at.st * a.Hkv)) return;   // (device lengths that are not the host's)
        g = (x1 - at.first) / at.st;
        const int x = at.first + g * at.st;              // the pair's first step
        if (x == x1 || x < run_begin(a, u0)) return;
        if (x + at.st > a.steps) return;                 // (device lengths longer than the host's)
        t0 = at.t0;
        rows = at.rows;
        parts = run_of(a, x + at.st - 1) - u0 + 1;
        slot0 = 2 * u0;
        odd = run_begin(a, u0) == x ? 0 : 1;             // its run's last segment, or its first
    }
    if (c >= rows || parts == 1) return;                 // (one part: written by its run)
    auto slot = [&](int p) { return (int64_t)(slot0 + kStride * p + (p == 0 ? odd : 0)) * a.cols + c; };
    float M = -INFINITY, L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int p0 = 0; p0 < parts; p0 += 64) {            // up to 64 parts' maxima and sums at a time
        const int np = min(64, parts - p0);
        f32x2 ml = f32x2{-INFINITY, 0.f};
        if (lane < np) ml = *reinterpret_cast<const f32x2 *>(ws_ml + 2 * slot(p0 + lane));
        float mb = ml[0];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) mb = fmaxf(mb, __shfl_xor(mb, off));
        const float Mn = fmaxf(M, mb);                  // finite: every part's max is
        const float r = __builtin_amdgcn_exp2f(M - Mn);
        M = Mn;
        const float w = __builtin_amdgcn_exp2f(ml[0] - M);
        float lw = w * ml[1];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) lw += __shfl_xor(lw, off);
        L = L * r + lw;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= r;
        for (int j0 = 0; j0 < np; j0 += 8) {            // O rows eight at a time, loads before uses
            float po[8][E];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float *src = ws_o + slot(p0 + min(j0 + i, np - 1)) * D + E * lane;
#pragma unroll
                for (int e = 0; e < E; ++e) po[i][e] = src[e];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float wi = __builtin_bit_cast(
                    float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), min(j0 + i, 63)));
                const float wv = j0 + i < np ? wi : 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += wv * po[i][e];
            }
        }
    }
    const float inv = 1.f / L;
    const int G = a.Hq / a.Hkv;
    u16 *orow = out + ((int64_t)(t0 + c / G) * a.Hq + g * G + c % G) * D + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) orow[e] = __builtin_bit_cast(u16, (__bf16)(acc[e] * inv));
}

}  // namespace

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
    CrossRowsPlan p{};
    if (steps <= 0) return p;
    const bool wide = head_dim == 128;
    const int64_t waves = (int64_t)n_cu * (wide ? 4 : 8);   // that are resident (registers)
    auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    const float bw = steps * (wide ? 0.0024f : 0.0012f) * 256.f / n_cu, cu = wide ? 0.41f : 0.22f;
    // The longest pairs run on with the device emptying around them for `tail`.
    const float mean = (float)steps / pairs, tail = cu * (longest - mean);
    // one run a pair: a compute unit's share of the pairs, one of them the longest
    const float whole = 6.f + tail + std::max(bw, cu * ceil_div(pairs, n_cu) * mean);
    // k runs of four waves a pair, of eight steps or more, all resident at once
    const int64_t k = std::max<int64_t>(1, std::min(ceil_div(longest, 8), waves / 4 / pairs));
    const float parts =
        9.5f + std::max(bw + tail / k, cu * ceil_div(pairs * k, n_cu) * ceil_div(longest, k)) + 0.03f * k;
    // even runs of all steps: single waves, or four together where a pair had too many parts to merge
    const int64_t single = std::max<int64_t>(1, std::min(waves, steps / 2));
    const bool four = single > 32 * pairs;
    const float even = (four ? 13.5f : 11.f + 3.f * std::min(1.f, single / 600.f)) + bw;
    if (whole <= even && (k == 1 || whole <= parts)) {
        p.parts = 1;
        p.waves = !wide && pairs * 8 <= waves ? 8 : pairs * 4 <= waves ? 4 : pairs * 2 <= waves ? 2 : 1;
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
    // (where no pair is cut nothing is written there: no workspace, whatever its size, reaches the kernel)
    auto *ws_o = combine ? static_cast<float *>(workspace) : nullptr;
    float *ws_ml = ws_o ? ws_o + (int64_t)plan.slots * cols * pool.head_dim : nullptr;
    auto *oo = static_cast<u16 *>(out);
    CrossArgs a{};
    a.num_blocks = pool.num_blocks;
    a.Hkv = pool.num_kv_heads;
    a.Hq = num_q_heads;
    a.max_blocks = max_blocks;
    a.B = B;
    a.T = T;
    a.cols = cols;
    a.steps = (int32_t)steps;
    a.runs = plan.runs;
    a.parts = plan.parts;
    a.base = (int32_t)(steps / plan.runs);
    a.rem = (int32_t)(steps % plan.runs);
    a.scale_log2 = sm_scale * kLog2e;
    auto go = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto rows = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(plan.runs), dim3(64 * plan.waves), 0, s, a,
                               static_cast<const u16 *>(q), static_cast<const u16 *>(pool.k),
                               static_cast<const u16 *>(pool.v), block_tables, key_lens, cu_q, oo, ws_o, ws_ml);
        };
        if (plan.parts > 1) {
            rows(cross_rows_kernel<D, 4, kParts>);
        } else if (!plan.parts) {
            if (plan.waves == 4) rows(cross_rows_kernel<D, 4, kEven>);
            else rows(cross_rows_kernel<D, 1, kEven>);
        } else if (plan.waves == 4) {
            rows(cross_rows_kernel<D, 4, kWhole>);
        } else if (plan.waves == 2) {
            rows(cross_rows_kernel<D, 2, kWhole>);
        } else if (plan.waves == 1) {
            rows(cross_rows_kernel<D, 1, kWhole>);
        } else if constexpr (D == 64) {
            rows(cross_rows_kernel<D, 8, kWhole>);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !combine) return e;
        // (runs are no more than the waves resident at once: no grid comes near its limit)
        const int64_t tasks = (plan.parts ? (int64_t)B * pool.num_kv_heads : plan.runs - 1) * cols;
        auto merge = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((tasks + kCombineWaves - 1) / kCombineWaves)),
                               dim3(64 * kCombineWaves), 0, s, a, key_lens, cu_q, ws_o, ws_ml, oo);
        };
        if (plan.parts) merge(cross_rows_combine_kernel<D, kParts>);
        else merge(cross_rows_combine_kernel<D, kEven>);
        return hipGetLastError();
    };
    if (pool.head_dim == 128) return go(std::integral_constant<int, 128>{});
    return go(std::integral_constant<int, 64>{});
}

}  // namespace pcr
