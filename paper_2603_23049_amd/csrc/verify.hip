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
//
// The passes read all there is to read, so they are what has to fill the device: a round is a launch in
// which several workgroups per sequence each walk as far as the walk goes without a new sum (the
// walk itself is a few dependent loads) and then sum their tiles of the row it needs. The last
// launch, one workgroup per sequence, ends the walk (with passes of its own where a walk needs more
// rounds than were launched) and draws: the tile sums lead to the tile, which is read once more. (64 chains of
// 4 over 128000 tokens: a round 13.0 us, of which the rows' 57 MB take 9 and the walk before them four
// dependent loads; the draw 7.4, dependent loads too.)
#include <algorithm>

#include "pcr_internal.h"

namespace pcr {
namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // rows start anywhere

constexpr int kRoundThreads = 256;
constexpr int kRoundWaves = kRoundThreads / 64;
constexpr int kFinalThreads = 1024;
constexpr int kPiece = 1024;             // elements of a tile, times VerifyArgs::pieces; a wave sums a tile
constexpr int kVecs = kPiece / 256;      // vectors of four of a lane and piece
constexpr int kMaxTiles = 4096;

// Where a walk stands between launches.
enum Need { kNextZ, kSum, kNothing };    // a pass for Z, for the sum of the last row, or its tile sums are there
struct State {
    double a, Z;
    int32_t at, next;                    // node, and the first node not tried yet
    int32_t kept, need;
    int32_t buf, fresh;                  // where the tile sums are, and whether they are those of (at, a)
};

struct VerifyArgs {
    const int32_t *cu_nodes, *parents, *tokens, *prefix_lens;
    const float *target, *draft, *uniforms;
    int64_t target_stride, draft_stride;
    int32_t *path, *accepted_lens, *next_tokens, *context_lens;
    int32_t B, T, V, path_cap;
    int32_t tiles, pieces, rounds;
    State *states;                       // [2][B]
    double *sums;                        // [2][B][tiles]
};

// What is left of a row's element. (The product and the difference are rounded each by itself: a fused
// one would leave other residues where p and q are equal.)
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

__device__ __forceinline__ float lane_of(float x, int l)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
}

// A sequence's part of the arrays.
struct Seq {
    int32_t t0, n;
    const int32_t *parents, *tokens;
    const float *uniforms;
    int32_t *path;
};
__device__ __forceinline__ Seq sequence(const VerifyArgs &a, int b)
{
    Seq s;
    s.t0 = min(max(a.cu_nodes[b], 0), a.T);
    s.n = max(min(a.cu_nodes[b + 1], a.T) - s.t0, 0);
    s.parents = a.parents + s.t0;
    s.tokens = a.tokens + s.t0;
    s.uniforms = a.uniforms + s.t0;
    s.path = a.path + (int64_t)b * a.path_cap;
    return s;
}

// Goes on with a walk until it needs a sum (all lanes of one wave; the state is the same in each). Children
// are tried in ascending order and follow their parents, so one pass over the nodes does: 64 at a
// time, with the elements of the rows that their tests need.
__device__ __forceinline__ void walk(const VerifyArgs &a, const Seq &s, State &st, bool lead)
{
    const int lane = threadIdx.x & 63;
    while (st.next < s.n && st.kept < a.path_cap) {
        const int32_t c0 = st.next & ~63, i = c0 + lane;
        const bool in = i < s.n;
        const int32_t parent = in ? s.parents[i] : -1, x = in ? s.tokens[i] : -1;
        const float u = in ? s.uniforms[i] : 0.f;
        const bool ok = parent >= 0 && parent < i && (uint32_t)x < (uint32_t)a.V;   // else never kept, and refuses nothing
        float p = 0.f, q = 0.f;
        if (__builtin_amdgcn_ballot_w64(ok && i >= st.next && parent == st.at) && ok) {   // (some child here)
            p = a.target[(int64_t)(s.t0 + parent) * a.target_stride + x];
            if (a.draft) q = a.draft[(int64_t)(s.t0 + parent) * a.draft_stride + x];
        }
        while (st.kept < a.path_cap) {
            const uint64_t children = __builtin_amdgcn_ballot_w64(ok && i >= st.next && parent == st.at);
            if (!children) break;
            const int l = (int)__builtin_ctzll(children);
            const double ul = lane_of(u, l);
            const float pl = lane_of(p, l), ql = lane_of(q, l);
            double w = left(pl, ql, st.a);
            if (!a.draft) {                     // 0 where a refused child had the same token
                const int32_t xl = __builtin_amdgcn_readlane(x, l);
                uint64_t again = __builtin_amdgcn_ballot_w64(ok && lane < l && parent == st.at && x == xl);
                for (int32_t j0 = st.at + 1; j0 < c0; j0 += 64) {
                    const int32_t j = j0 + lane;
                    again |= __builtin_amdgcn_ballot_w64(j < c0 && s.parents[j] == st.at && s.tokens[j] == xl);
                }
                w = again ? 0.0 : w;
            }
            const bool stays = (a.draft ? ul * (double)ql * st.Z : ul * st.Z) < w;
            st.next = c0 + l + 1;
            if (stays) {
                st.at = c0 + l;
                if (lead && lane == 0) s.path[st.kept] = st.at;
                ++st.kept;
                st.a = 0.0;
                st.Z = 1.0;
                st.fresh = 0;
            } else if (a.draft) {
                st.a += st.Z;
                // Behind the last child the walk ends here: the sum is the draw's, not a test's.
                const bool ends = (children & (children - 1)) == 0 && c0 + 64 >= s.n;
                st.need = ends ? kSum : kNextZ;
                return;
            } else {
                st.Z -= w;
            }
        }
        if (st.kept >= a.path_cap) break;
        st.next = c0 + 64;
    }
    st.need = st.fresh ? kNothing : kSum;
}

// What a pass reads.
struct Row {
    const float *p, *q;
    double a;
    const int32_t *parents, *tokens;     // of the refused tokens that are out of p, if any: children of `at`
    int32_t at, end;                     // among the nodes (at, end)
    int32_t out0;                        // this lane's of the first 64 of them (-1: none)
};
__device__ __forceinline__ int32_t refused(const Row &r, int32_t j)
{
    return j < r.end && r.parents[j] == r.at ? r.tokens[j] : -1;
}
__device__ __forceinline__ Row row_of(const VerifyArgs &a, const Seq &s, const State &st)
{
    Row r;
    r.p = a.target + (int64_t)(s.t0 + st.at) * a.target_stride;
    r.q = a.draft && st.a != 0.0 ? a.draft + (int64_t)(s.t0 + st.at) * a.draft_stride : nullptr;
    r.a = st.a;
    r.parents = s.parents;
    r.tokens = s.tokens;
    r.at = st.at;
    r.end = a.draft ? st.at + 1 : min(st.next, s.n);
    r.out0 = refused(r, st.at + 1 + (int32_t)(threadIdx.x & 63));
    return r;
}

// The four elements at v of the rows.
struct Four {
    f32x4u p, q;
};
__device__ __forceinline__ Four load(const Row &r, int32_t V, int32_t v)
{
    Four x{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if (v + 3 < V) {
        x.p = *reinterpret_cast<const f32x4u *>(r.p + v);
        if (r.q) x.q = *reinterpret_cast<const f32x4u *>(r.q + v);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v + k < V) {
                x.p[k] = r.p[v + k];
                if (r.q) x.q[k] = r.q[v + k];
            }
    }
    return x;
}

// What is left of them (0 from hi on); base: of the wave's first lane.
__device__ __forceinline__ void values(const Row &r, const Four &x, int32_t base, int32_t v, int32_t hi, double (&e)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = v + k < hi ? left(x.p[k], x.q[k], r.a) : 0.0;
    // Refused tokens: 64 nodes at a time, those among the wave's 256 elements.
    for (int32_t j0 = r.at + 1; j0 < r.end; j0 += 64) {
        const int32_t y = j0 == r.at + 1 ? r.out0 : refused(r, j0 + (int32_t)(threadIdx.x & 63));
        uint64_t hits = __builtin_amdgcn_ballot_w64(y >= base && y - base < 256);
        while (hits) {
            const int32_t at = __builtin_amdgcn_readlane(y, (int)__builtin_ctzll(hits)) - v;
            hits &= hits - 1;
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = at == k ? 0.0 : e[k];
        }
    }
}

// Sum of what is left of the vectors v .. of a piece (all lanes of a wave).
template <int N>
__device__ __forceinline__ double piece_sum(const VerifyArgs &a, const Row &r, int32_t base, const Four (&x)[N])
{
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        double e[4];
        const int32_t at = base + k * 256;
        values(r, x[k], at, at + 4 * (int32_t)(threadIdx.x & 63), a.V, e);
        s += (e[0] + e[1]) + (e[2] + e[3]);
    }
    return s;
}
template <int N>
__device__ __forceinline__ void load_piece(const VerifyArgs &a, const Row &r, int32_t base, Four (&x)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = load(r, a.V, base + k * 256 + 4 * (int32_t)(threadIdx.x & 63));
}
// First element of a tile's piece (the row's end where it lies past it: no element of it).
__device__ __forceinline__ int32_t piece_begin(const VerifyArgs &a, int32_t t, int32_t piece)
{
    return (int32_t)min(((int64_t)t * a.pieces + piece) * kPiece, (int64_t)a.V);
}

// A wave's share of a pass: the tiles first, first + step, .. in pieces. AHEAD: the next piece's loads are in flight
// while one is added (a workgroup alone on its compute unit); else many waves hide them.
template <bool AHEAD>
__device__ __forceinline__ void tile_sums(const VerifyArgs &a, const Row &r, int32_t first, int32_t step, double *sums)
{
    const int lane = threadIdx.x & 63;
    if constexpr (!AHEAD) {
        for (int32_t t = first; t < a.tiles; t += step) {
            double s = 0.0;
            for (int32_t piece = 0; piece < a.pieces; ++piece) {
                Four x[kVecs];
                const int32_t base = piece_begin(a, t, piece);
                load_piece(a, r, base, x);
                s += piece_sum(a, r, base, x);
            }
            s = wave_sum(s);
            if (lane == 0) sums[t] = s;
        }
    } else {
        if (first >= a.tiles) return;
        Four x[kVecs], y[kVecs];
        load_piece(a, r, piece_begin(a, first, 0), x);
        double s = 0.0;
        for (int32_t t = first, piece = 0; t < a.tiles;) {
            const bool ends = piece + 1 == a.pieces;
            const int32_t t2 = ends ? t + step : t, piece2 = ends ? 0 : piece + 1;
            if (t2 < a.tiles) load_piece(a, r, piece_begin(a, t2, piece2), y);
            s += piece_sum(a, r, piece_begin(a, t, piece), x);
            if (ends) {
                s = wave_sum(s);
                if (lane == 0) sums[t] = s;
                s = 0.0;
            }
#pragma unroll
            for (int k = 0; k < kVecs; ++k) x[k] = y[k];
            t = t2;
            piece = piece2;
        }
    }
}

// Sum of all tiles, in one order whoever adds them.
__device__ __forceinline__ double add_tiles(const double *sums, int32_t tiles)
{
    double s = 0.0;
    for (int32_t t = threadIdx.x & 63; t < tiles; t += 64) s += sums[t];
    return wave_sum(s);
}

__device__ __forceinline__ State start(const Seq &s, bool lead)
{
    State st{0.0, 1.0, 0, 1, s.n > 0 ? 1 : 0, kSum, 0, 0};
    if (lead && s.n > 0 && (threadIdx.x & 63) == 0) s.path[0] = 0;
    return st;
}

// Grid (workgroups of a sequence, sequences).
__global__ __launch_bounds__(kRoundThreads) void verify_round_kernel(const VerifyArgs a, int round)
{
    __shared__ State sh;
    const int tid = threadIdx.x, b = blockIdx.y;
    const Seq s = sequence(a, b);
    State st;                                    // (read beside the lengths, whatever it is for an empty sequence)
    if (round > 0) st = a.states[(int64_t)((round - 1) & 1) * a.B + b];
    if (s.n == 0) return;
    const bool lead = blockIdx.x == 0;
    if (tid < 64) {
        if (round == 0) {
            st = start(s, lead);
            walk(a, s, st, lead);
        } else {
            if (st.need == kNextZ) {
                st.Z = add_tiles(a.sums + ((int64_t)st.buf * a.B + b) * a.tiles, a.tiles);
                st.fresh = 1;
                walk(a, s, st, lead);
            } else {
                st.need = kNothing;              // the last round's pass was the last row's
            }
        }
        if (st.need != kNothing) st.buf = round & 1;
        if (tid == 0) {
            sh = st;
            if (lead) a.states[(int64_t)(round & 1) * a.B + b] = st;
        }
    }
    __syncthreads();
    st = sh;
    if (st.need == kNothing) return;
    tile_sums<false>(a, row_of(a, s, st), kRoundWaves * blockIdx.x + (tid >> 6), kRoundWaves * gridDim.x,
              a.sums + ((int64_t)st.buf * a.B + b) * a.tiles);
}

// Inclusive sums of a wave's lanes.
__device__ __forceinline__ double wave_scan(double c)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(c, off);
        if (lane >= off) c += o;
    }
    return c;
}

// The first token whose cumulated sum passes t (all lanes of one wave): the tile, then its pieces. Where
// rounding leaves none it is the last token with anything, as in each step of the search.
__device__ __forceinline__ int32_t draw(const VerifyArgs &a, const Row &r, const double *sums, double t)
{
    const int lane = threadIdx.x & 63;
    int32_t tile = -1, some = 0;                            // some: the last tile with anything
    double before = 0.0;
    for (int32_t t0 = 0; t0 < a.tiles && tile < 0; t0 += 64) {
        const double x = t0 + lane < a.tiles ? sums[t0 + lane] : 0.0, c = wave_scan(x);
        const uint64_t any = __builtin_amdgcn_ballot_w64(x > 0.0);
        const uint64_t over = __builtin_amdgcn_ballot_w64(x > 0.0 && before + c > t);
        if (any) some = t0 + 63 - (int32_t)__builtin_clzll(any);
        if (over) {
            const int l = (int)__builtin_ctzll(over);
            tile = t0 + l;
            before += __shfl(c, l) - __shfl(x, l);
        } else {
            before += __shfl(c, 63);
        }
    }
    t = tile < 0 ? INFINITY : t - before;
    tile = tile < 0 ? some : tile;
    before = 0.0;
    int32_t token = -1, last = 0;                           // the token, and the last one with anything
    for (int32_t piece = 0; piece < a.pieces && token < 0; ++piece) {
        const int32_t base = (int32_t)min(((int64_t)tile * a.pieces + piece) * kPiece, (int64_t)a.V);
        Four x[kVecs];
#pragma unroll
        for (int k = 0; k < kVecs; ++k) x[k] = load(r, a.V, base + k * 256 + 4 * lane);
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            double e[4];
            values(r, x[k], base + k * 256, base + k * 256 + 4 * lane, a.V, e);
            const double y = (e[0] + e[1]) + (e[2] + e[3]), c = wave_scan(y);
            const uint64_t any = __builtin_amdgcn_ballot_w64(y > 0.0);
            const uint64_t over = __builtin_amdgcn_ballot_w64(y > 0.0 && before + c > t);
            if (any && token < 0) {
                const int l = over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(any);
                double z = before + (c - y);
                int32_t m = -1, end = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z += e[i];
                    if (m < 0 && e[i] > 0.0 && z > t) m = i;
                    if (e[i] > 0.0) end = i;
                }
                last = base + k * 256 + 4 * l + __shfl(over && m >= 0 ? m : end, l);
                if (over) token = last;
            }
            before += __shfl(c, 63);
        }
    }
    return token < 0 ? last : token;
}

// One workgroup per sequence.
__global__ __launch_bounds__(kFinalThreads) void verify_final_kernel(const VerifyArgs a)
{
    __shared__ State sh;
    __shared__ double sums[kMaxTiles];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const Seq s = sequence(a, b);
    const float u0 = s.n > 0 ? s.uniforms[0] : 0.f;
    State st;
    if (wave == 0) {
        // (state and, with one round, sums are read beside the lengths, whatever they are for an empty sequence)
        if (a.rounds > 0) st = a.states[(int64_t)((a.rounds - 1) & 1) * a.B + b];
        if (a.rounds == 0 || s.n == 0) {
            st = start(s, true);
            walk(a, s, st, true);
        } else {
            const double *from = a.sums + ((int64_t)(a.rounds == 1 ? 0 : st.buf) * a.B + b) * a.tiles;
            for (int32_t t = lane; t < a.tiles; t += 64) sums[t] = from[t];
            if (st.need == kNextZ) {
                st.Z = add_tiles(sums, a.tiles);
                st.fresh = 1;
                walk(a, s, st, true);
            } else {
                st.need = kNothing;
            }
        }
        if (lane == 0) sh = st;
    }
    __syncthreads();
    st = sh;
    while (s.n > 0 && st.need != kNothing) {
        tile_sums<true>(a, row_of(a, s, st), wave, kFinalThreads / 64, sums);
        __syncthreads();
        if (wave == 0) {
            if (st.need == kNextZ) {
                st.Z = add_tiles(sums, a.tiles);
                st.fresh = 1;
                walk(a, s, st, true);
            } else {
                st.need = kNothing;
            }
            if (lane == 0) sh = st;
        }
        __syncthreads();
        st = sh;
    }
    for (int32_t i = st.kept + tid; i < a.path_cap; i += kFinalThreads) s.path[i] = -1;
    if (tid == 0) {
        a.accepted_lens[b] = st.kept;
        a.context_lens[b] = a.prefix_lens[b] + st.kept;
        if (s.n == 0) a.next_tokens[b] = -1;
    }
    if (s.n == 0) return;
    Row r = row_of(a, s, st);
    double S = add_tiles(sums, a.tiles);
    if (!(S > 0.0)) {                                       // nothing is left: the target's own row
        r.q = nullptr;
        r.a = 0.0;
        r.end = r.at + 1;
        __syncthreads();
        tile_sums<true>(a, r, wave, kFinalThreads / 64, sums);
        __syncthreads();
        S = add_tiles(sums, a.tiles);
    }
    if (wave > 0) return;
    const int32_t token = draw(a, r, sums, (double)u0 * S);
    if (lane == 0) a.next_tokens[b] = token;
}

constexpr int32_t kRoundSeqs = 1024;      // sequences up to which there are rounds

}  // namespace

// How a call is cut up. A round, idle, costs 2 us among other launches. A pass over 128000 tokens takes about 15 us in
// the last launch, with one workgroup a sequence, and 5 or less in a round. With 0, 1, 2 and 4 rounds, us:
//   chains of 4, 128000 tokens, 64 of them     28.7  20.5  22.4  26.3      8 of them  25.7  12.4  14.3  18.9
//   one chain of 5, 32001 tokens               12.0  11.4  14.3  19.4
//   64 chains of 8, 128000 tokens              29.8  22.1  24.1  27.9      of 16      30.5  23.7  25.4  29.6
//   trees of 13 nodes, 128 of 128000 tokens    91.5  93.6  86.3  64.2      (three 75.9, five 66.7)
//   64 trees of 9 nodes, 128000 tokens         73.3  66.2  55.4  40.6      of 5       73.6  65.5  54.2  39.3
//   64 trees of 13, 8192 tokens                17.9  21.2  23.4            9217       20.4  23.2  25.0
//                   16384                      20.5  23.2  24.4  27.4      40960      31.4  32.3  30.6  30.4
//                   49152                      39.2  38.6  36.2  31.7
//   48 trees, no probabilities, 50001 tokens   18.2  15.0  17.0  21.3
//   512 trees of 4, 32000 tokens               45.6  48.7  46.5            1024       81.8  85.8  83.6
// So none up to 8 tiles, and where the sequences alone fill the device; one for a draft without probabilities (it
// needs one sum), below 48 tiles, and for few nodes; four for many, two between. What a walk needs
// follows from its refusals, so from siblings, which the host does not know and the mean number of nodes stands
// for: long chains pay idle rounds, and small trees take passes in the last launch.
VerifyPlan verify_plan(int32_t B, int32_t T, int32_t V, bool drawn)
{
    VerifyPlan p{};
    p.pieces = (int32_t)(((int64_t)V + (int64_t)kPiece * kMaxTiles - 1) / ((int64_t)kPiece * kMaxTiles));
    const int64_t size = (int64_t)p.pieces * kPiece;
    p.tiles = (int32_t)((V + size - 1) / size);
    const int64_t nodes = ((int64_t)T + std::max(B, 1) - 1) / std::max(B, 1);
    p.rounds = p.tiles <= 8 || B > kRoundSeqs ? 0 : !drawn || nodes <= 5 || p.tiles < 48 ? 1 : nodes <= 9 ? 2 : 4;
    // Two tiles a wave where the sequences fill the device that way, one where they are fewer, more where they
    // are many (one, two and four, us: 64 chains of 4 of 128000 tokens 22.5, 20.4, 21.8; 16 of them 14.0, 15.4, 19.0; 256 of
    // 50000 29.3, 28.6, 27.3; 128 trees of 13 nodes of 128000 91.4, 91.5, 101).
    const int64_t seqs = std::max(B, 1), one = (p.tiles + kRoundWaves - 1) / kRoundWaves, two = (one + 1) / 2;
    p.wgs = (int32_t)std::max<int64_t>(1, std::min(one, std::max(1024 / seqs, std::min(two, 4096 / seqs))));
    p.bytes = p.rounds ? (int64_t)2 * B * (sizeof(State) + 8 * p.tiles) : 0;
    return p;
}

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
    if (B > 0) *bytes = verify_plan(std::min(B, kRoundSeqs), T, vocab, true).bytes;
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
    const VerifyPlan plan = verify_plan(B, T, vocab, draft_probs != nullptr);
    const pcr_status st = check_workspace(plan.bytes, workspace, workspace_bytes, who);
    if (st) return st;
    State *states = static_cast<State *>(workspace);
    const VerifyArgs a{cu_nodes, parents, tokens, prefix_lens, target_probs, draft_probs, uniforms, target_stride,
                       draft_stride, path, accepted_lens, next_tokens, context_lens, B, T, vocab, path_cap, plan.tiles,
                       plan.pieces, plan.rounds, states, reinterpret_cast<double *>(states + 2 * (int64_t)B)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    for (int r = 0; r < plan.rounds && e == hipSuccess; ++r) {
        hipLaunchKernelGGL(verify_round_kernel, dim3(plan.wgs, B), dim3(kRoundThreads), 0, s, a, r);
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(verify_final_kernel, dim3(B), dim3(kFinalThreads), 0, s, a);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return hip_fail(e, "pcr_verify_drafts: launch");
    return PCR_OK;
}

}  // extern "C"
