// Verification of drafted tokens for gfx950: a walk down each sequence's tree that keeps a drafted
// token with the probability that makes the kept tokens distributed as the target's, and the draw of
// the token after them, from the target's (and the draft's) probabilities and given random numbers.
//
// At a node u with the target's row p and the draft's row q, drafted children are tried in their order.
// After k of them were refused the target's distribution that is left is, up to its sum, r_k = max(p - a_k q, 0):
// r_0 = p, and r_{k+1} = max(r_k / Z_k - q, 0) with Z_k = sum r_k is the same as a_{k+1} = a_k + Z_k.
// So two numbers (a, Z) hold the state of a walk, and a refusal costs one pass over the rows for the
// next Z. A draft without probabilities proposes each token for certain (q is 1 there): a refusal
// takes the token out of p, and Z falls by its share without a pass. Sums are in 64 bits: a
// row's cumulated sum decides between neighbouring tokens.
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

struct VerifyArgs {
    const int32_t *cu_nodes, *parents, *tokens, *prefix_lens;
    const float *target, *draft, *uniforms;
    int64_t target_stride, draft_stride;
    int32_t *path, *accepted_lens, *next_tokens, *context_lens;
    int32_t T, V, path_cap;
};

// What is left of a row. (The product and the difference are rounded each by itself: a fused one would
// leave other residues where p and q are equal.)
__device__ __forceinline__ double left(float p, float q, double a)
{
#pragma clang fp contract(off)
    const double aq = a * (double)q;
    const double r = (double)p - aq;
    return r > 0.0 ? r : 0.0;          // (NaN counts as 0)
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    return x;
}

// One workgroup per sequence.
__global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyArgs a)
{
    __shared__ double part[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const int32_t t0 = min(max(a.cu_nodes[b], 0), a.T), n = min(a.cu_nodes[b + 1], a.T) - t0;
    int32_t *path = a.path + (int64_t)b * a.path_cap;
    const int32_t *parents = a.parents + t0, *tokens = a.tokens + t0;
    int32_t at = 0, kept = n > 0 ? 1 : 0, refused = 0;      // the walk's node; refused children of it (their last)
    double shift = 0.0, Z = 1.0;
    const float *p = a.target + (int64_t)t0 * a.target_stride;
    const float *q = a.draft ? a.draft + (int64_t)t0 * a.draft_stride : nullptr;
    // Tokens of the refused children are out of the row (a draft without probabilities).
    auto out = [&](int32_t v) {
        for (int32_t i = at + 1; i <= refused; ++i)
            if (parents[i] == at && tokens[i] == v) return true;
        return false;
    };
    auto value = [&](int32_t v) -> double {
        if (q) return left(p[v], q[v], shift);
        const double r = left(p[v], 0.f, 0.0);
        return refused > at && r > 0.0 && out(v) ? 0.0 : r;
    };
    auto total = [&](int32_t lo, int32_t hi) -> double {    // sum of [lo, hi), on all threads
        double s = 0.0;
        for (int32_t v = lo + tid; v < hi; v += kThreads) s += value(v);
        s = wave_sum(s);
        __syncthreads();
        if (lane == 0) part[wave] = s;
        __syncthreads();
        s = 0.0;
        for (int w = 0; w < kWaves; ++w) s += part[w];
        return s;
    };
    if (tid == 0 && n > 0) path[0] = 0;
    for (int32_t i = 1; i < n && kept < a.path_cap; ++i) {
        if (parents[i] != at) continue;
        const int32_t x = tokens[i];
        if ((uint32_t)x >= (uint32_t)a.V) continue;         // no token: never kept, nothing refused
        const double u = (double)a.uniforms[t0 + i];
        const double w = value(x);
        const bool yes = q ? u * (double)q[x] * Z < w : u * Z < w;
        if (yes) {
            at = refused = i;
            if (tid == 0) path[kept] = i;
            ++kept;
            shift = 0.0;
            Z = 1.0;
            p = a.target + (int64_t)(t0 + i) * a.target_stride;
            if (q) q = a.draft + (int64_t)(t0 + i) * a.draft_stride;
        } else {
            refused = i;
            if (q) {
                shift += Z;
                Z = total(0, a.V);
            } else {
                Z -= w;
            }
        }
    }
    if (tid == 0) {
        a.accepted_lens[b] = kept;
        a.context_lens[b] = a.prefix_lens[b] + kept;
    }
    for (int32_t i = kept + tid; i < a.path_cap; i += kThreads) path[i] = -1;
    if (n <= 0) {
        if (tid == 0) a.next_tokens[b] = -1;
        return;
    }
    // The draw: the first token whose cumulated sum passes u * S. Waves take one part of the row each.
    double S = total(0, a.V);
    if (!(S > 0.0)) {                                       // nothing is left: the target's own row
        q = nullptr;
        refused = at;
        S = total(0, a.V);
    }
    double t = (double)a.uniforms[t0] * S;
    int32_t lo = 0, hi = a.V;
    while (hi - lo > 64) {                                  // sixteen parts of [lo, hi): the one that holds t
        const int32_t size = ((hi - lo + kWaves - 1) / kWaves + 63) / 64 * 64;
        const int32_t w0 = min(lo + wave * size, hi), w1 = min(w0 + size, hi);
        double s = 0.0;
        for (int32_t v = w0 + lane; v < w1; v += 64) s += value(v);
        s = wave_sum(s);
        __syncthreads();
        if (lane == 0) part[wave] = s;
        __syncthreads();
        double cum = 0.0, before = 0.0;
        int pick = -1;
        for (int w = 0; w < kWaves && pick < 0; ++w) {
            if (cum + part[w] > t) {
                pick = w;
                before = cum;
            }
            cum += part[w];
        }
        for (int w = kWaves - 1; w >= 0 && pick < 0; --w)   // (rounding: the last part with anything)
            if (part[w] > 0.0) {
                pick = w;
                before = -1e300;                            // its last token, below
            }
        pick = max(pick, 0);
        t = before == -1e300 ? 1e300 : t - before;
        lo = min(lo + pick * size, hi);
        hi = min(lo + size, hi);
    }
    if (wave == 0) {
        const double r = lo + lane < hi ? value(lo + lane) : 0.0;
        double c = r;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double o = __shfl_up(c, off);
            if (lane >= off) c += o;
        }
        const uint64_t over = __builtin_amdgcn_ballot_w64(c > t), some = __builtin_amdgcn_ballot_w64(r > 0.0);
        const int32_t end = some ? 63 - (int)__builtin_clzll(some) : 0;   // the last with anything
        const int32_t l = over ? min((int32_t)__builtin_ctzll(over), end) : end;
        if (lane == 0) a.next_tokens[b] = lo + l;
    }
}

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_verify_drafts_workspace_size(int32_t B, int32_t T, int32_t vocab, int64_t *bytes)
{
    clear_error();
    const char *who = "pcr_verify_drafts_workspace_size";
    if (!bytes) return fail(PCR_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    *bytes = 0;
    if (B < 0 || T < 0 || vocab < 1) return fail(PCR_ERR_INVALID_ARG, "%s: negative B or T, or vocab < 1", who);
    return PCR_OK;
}

pcr_status pcr_verify_drafts(int32_t B, const int32_t *cu_nodes, const int32_t *parents, const int32_t *tokens,
                             int32_t T, int32_t vocab, const float *target_probs, int64_t target_stride,
                             const float *draft_probs, int64_t draft_stride, const float *uniforms,
                             const int32_t *prefix_lens, int32_t path_cap, int32_t *path, int32_t *accepted_lens,
                             int32_t *next_tokens, int32_t *context_lens, void *workspace, int64_t workspace_bytes,
                             void *stream)
{
    clear_error();
    const char *who = "pcr_verify_drafts";
    if (B < 0 || T < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative B or T", who);
    if (vocab < 1 || path_cap < 1) return fail(PCR_ERR_INVALID_ARG, "%s: vocab and path_cap must be positive", who);
    if (B > kMaxTreeSeqs || T > kMaxTreeNodes || vocab > kMaxVocab)
        return fail(PCR_ERR_UNSUPPORTED, "%s: batch or vocabulary too large", who);
    if (target_stride < vocab || (draft_probs && draft_stride < vocab))
        return fail(PCR_ERR_INVALID_ARG, "%s: rows of fewer than vocab elements", who);
    if (target_stride > kMaxRowStride || (draft_probs && draft_stride > kMaxRowStride))
        return fail(PCR_ERR_UNSUPPORTED, "%s: row stride too large", who);
    if (B == 0) return PCR_OK;
    if (!cu_nodes || !prefix_lens || !path || !accepted_lens || !next_tokens || !context_lens ||
        (T > 0 && (!parents || !tokens || !target_probs || !uniforms)))
        return fail(PCR_ERR_INVALID_ARG, "%s: NULL argument", who);
    const VerifyArgs a{cu_nodes, parents, tokens, prefix_lens, target_probs, draft_probs, uniforms, target_stride,
                       draft_stride, path, accepted_lens, next_tokens, context_lens, T, vocab, path_cap};
    hipLaunchKernelGGL(verify_kernel, dim3(B), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "pcr_verify_drafts: launch");
    return PCR_OK;
}

}  // extern "C"
