// Rotary positions with one or several axes, on plain rows or fused with the write of K/V
// into the pool (bf16 in, fp32 products, bf16 out), for gfx950.
//
// Pair j of a token's head turns by positions[axis_j] * inv_freq[j]. Angles of far
// positions lose their phase in fp32 (position 10^6 keeps 2^-4 of a radian), so the turn is
// formed and reduced in fp64, in whole revolutions: r = position * (inv_freq / 2 pi),
// minus its nearest integer, and cos and sin of the rest come from v_cos_f32 and v_sin_f32,
// which take revolutions (off by at most 2^-22.9 on 2^28 arguments of [-1/2, 1/2], against
// fp64; the library's sincospif, 2^-24.2, takes about twice the instructions).
//
// Bound by moving the rows. A thread takes one unit of a token, 8 pairs = two 16-byte
// chunks of each head, computes their cos and sin once and walks the heads with them in
// registers. With few tokens the heads are dealt to more workgroups, each of which
// computes the angles again.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "append_tile.h"
#include "pcr_internal.h"

namespace pcr {
namespace {

typedef unsigned short u16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxAxes = 4;
constexpr int32_t kMaxTokens = 1 << 27;   // 2^31 threads at most for plain rows (launch_append checks its own)
constexpr int kUnit = 8;          // pairs of a unit
constexpr int kTile = 32;         // new tokens of a K/V workgroup (append_tile.h)

// The rotation, in the launch's arguments.
struct RopeArgs {
    double turns[kMaxPairs];      // revolutions per position step
    uint8_t axis[kMaxPairs];
    int32_t half;                 // pairs
    int32_t axes;
    int32_t interleaved;
    float scale, sin_scale;       // of cos and of sin (negated: transposed)
};

// NT: past the caches.
template <bool NT>
__device__ __forceinline__ u32x4 load16(const u16 *p)
{
    auto *v = reinterpret_cast<const u32x4 *>(p);
    if constexpr (NT) return __builtin_nontemporal_load(v);
    return *v;
}
template <bool NT>
__device__ __forceinline__ void store16(u16 *p, u32x4 x)
{
    if constexpr (NT) __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<u32x4 *>(p) = x;
}

// One unit of one token: where its two chunks lie in a head's row, and its cos and sin.
struct Unit {
    int32_t at[2];                // element offsets
    bool turned;                  // false: dims past the rotation, copied
    float c[kUnit], s[kUnit];
};

__device__ __forceinline__ void place_unit(const RopeArgs &ra, int u, Unit &un)
{
    const int n = ra.half / kUnit;                     // turned units of a head
    un.turned = u < n;
    if (un.turned && !ra.interleaved) {
        un.at[0] = kUnit * u;
        un.at[1] = ra.half + kUnit * u;
    } else {                                           // 16 dims back to back
        un.at[0] = 2 * kUnit * u;
        un.at[1] = un.at[0] + kUnit;
    }
}

__device__ __forceinline__ void turn_unit(const RopeArgs &ra, const int32_t *__restrict__ positions,
                                          int64_t pos_stride, int64_t t, int u, Unit &un)
{
    if (!un.turned) return;
    int32_t p[kMaxAxes];
#pragma unroll
    for (int a = 0; a < kMaxAxes; ++a) p[a] = a < ra.axes ? positions[a * pos_stride + t] : 0;
    const uint64_t axis = *reinterpret_cast<const uint64_t *>(ra.axis + kUnit * u);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
        const int a = (int)(axis >> (8 * j)) & 3;
        const int32_t pa = a & 2 ? (a & 1 ? p[3] : p[2]) : (a & 1 ? p[1] : p[0]);
        double r = (double)pa * ra.turns[kUnit * u + j];
        r -= rint(r);
        un.c[j] = __builtin_amdgcn_cosf((float)r) * ra.scale;
        un.s[j] = __builtin_amdgcn_sinf((float)r) * ra.sin_scale;
    }
}

__device__ __forceinline__ f32x8 widen(u32x4 v) { return __builtin_convertvector(__builtin_bit_cast(bf16x8, v), f32x8); }
__device__ __forceinline__ u32x4 narrow(f32x8 v) { return __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8)); }

// One pair: the sums written as fused products, so that every kernel (and every size of call)
// rounds them alike.
__device__ __forceinline__ void turn_pair(float x, float y, float c, float s, float &r, float &w)
{
    r = __builtin_fmaf(x, c, -(y * s));
    w = __builtin_fmaf(y, c, x * s);
}

// The unit's two chunks of one head, rotated (fp32 products, rounded once).
template <bool IL>
__device__ __forceinline__ void rotate(const Unit &un, u32x4 &a, u32x4 &b)
{
    const f32x8 x = widen(a), y = widen(b);
    float r[8], w[8];
    if constexpr (IL) {                                // chunk a holds pairs 0..3, b pairs 4..7
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            turn_pair(x[2 * j], x[2 * j + 1], un.c[j], un.s[j], r[2 * j], r[2 * j + 1]);
            turn_pair(y[2 * j], y[2 * j + 1], un.c[4 + j], un.s[4 + j], w[2 * j], w[2 * j + 1]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) turn_pair(x[j], y[j], un.c[j], un.s[j], r[j], w[j]);
    }
    const f32x8 rv = {r[0], r[1], r[2], r[3], r[4], r[5], r[6], r[7]};
    const f32x8 wv = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
    a = un.turned ? narrow(rv) : a;
    b = un.turned ? narrow(wv) : b;
}

// Heads [h0, h1) of the tokens of one workgroup. Threads past the last whole token idle.
// (A thread reads a unit before it writes it, and no other touches it: in place is safe.)
template <bool IL, int THREADS, int W, bool NT>
__device__ __forceinline__ void rotate_rows(const RopeArgs &ra, const u16 *x, int64_t x_stride,
                                            const int32_t *__restrict__ positions, int64_t pos_stride, int32_t T,
                                            int32_t D, int tile, int h0, int h1, u16 *out, int64_t out_stride)
{
    const int units = D / (2 * kUnit), per = THREADS / units;
    const int tl = threadIdx.x / units, u = threadIdx.x - tl * units;
    const int64_t t = (int64_t)tile * per + tl;
    if (tl >= per || t >= T) return;
    Unit un;
    place_unit(ra, u, un);
    const u16 *src = x + t * x_stride;
    u16 *dst = out + t * out_stride;
    u32x4 a[W], b[W];                                  // W heads in flight
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int hh = min(h + i, h1 - 1);         // (past the end: the last one again, not written)
            a[i] = load16<NT>(src + (int64_t)hh * D + un.at[0]);
            b[i] = load16<NT>(src + (int64_t)hh * D + un.at[1]);
        }
    };
    load(h0);                                          // in flight while the angles are formed
    turn_unit(ra, positions, pos_stride, t, u, un);
    for (int h = h0;;) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            rotate<IL>(un, a[i], b[i]);
            if (h + i < h1) {
                store16<NT>(dst + (int64_t)(h + i) * D + un.at[0], a[i]);
                store16<NT>(dst + (int64_t)(h + i) * D + un.at[1], b[i]);
            }
        }
        h += W;
        if (h >= h1) break;
        load(h);
    }
}

// Grid (token tiles, head groups of `heads`).
template <bool IL, int W, bool NT>
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(const RopeArgs ra, const u16 *x, int64_t x_stride,
                                                             const int32_t *__restrict__ positions, int64_t pos_stride,
                                                             int32_t T, int32_t H, int32_t D, int32_t heads, u16 *out,
                                                             int64_t out_stride)
{
    const int h0 = blockIdx.y * heads;
    rotate_rows<IL, kThreads, W, NT>(ra, x, x_stride, positions, pos_stride, T, D, blockIdx.x, h0, min(H, h0 + heads), out,
                                 out_stride);
}

// What the K/V and Q workgroups of one launch share out.
struct AppendArgs {
    u16 *pool_k, *pool_v;
    const u16 *k_new, *v_new, *q;
    u16 *q_out;
    int64_t k_stride, v_stride, q_stride, pos_stride;
    const int32_t *positions, *slot_mapping;
    int32_t num_blocks, Hkv, Hq, T;
    int32_t kv_heads, kv_groups, kv_wgs;      // kv heads of a workgroup, groups of them, K/V workgroups
    int32_t q_heads, q_groups;                // the same of Q
};

// K and V of kv heads [g0, g1) of one tile of new tokens: K rotated in registers and written
// by rows, V through LDS into its d-major chunks (two buffers, so a head costs one barrier). The
// next head's rows are requested before this one's V leaves LDS.
template <int D, bool IL, bool NT>
__device__ __forceinline__ void append_heads(const RopeArgs &ra, const AppendArgs &aa, int tile, int g0, int g1)
{
    constexpr int ROWS = kTile + append_tile::kExt, CPR = D / 8, UNITS = D / (2 * kUnit);
    constexpr int NK = (ROWS * UNITS + kThreads - 1) / kThreads, NV = (ROWS * CPR + kThreads - 1) / kThreads;
    __shared__ __attribute__((aligned(16))) u16 vs[2][ROWS][D + 8];   // +8 elements: stagger rows across banks
    __shared__ int32_t slots[ROWS];            // -1: no slot, or another tile's
    __shared__ int32_t runs[ROWS];
    __shared__ int32_t n_runs;
    const int tid = threadIdx.x, tok0 = tile * kTile;
    Unit un[NK];
    bool k_on[NK], v_on[NV];                   // rows this thread loads of
    u32x4 ka[NK], kb[NK], vv[NV];
    auto load = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            if (!k_on[i]) continue;
            const u16 *src = aa.k_new + (int64_t)(tok0 + (tid + kThreads * i) / UNITS) * aa.k_stride + g * D;
            ka[i] = load16<NT>(src + un[i].at[0]);
            kb[i] = load16<NT>(src + un[i].at[1]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = tid + kThreads * i;
            if (v_on[i])
                vv[i] = load16<NT>(aa.v_new + (int64_t)(tok0 + c / CPR) * aa.v_stride + g * D + c % CPR * 8);
        }
    };
#pragma unroll
    for (int i = 0; i < NK; ++i) place_unit(ra, (tid + kThreads * i) % UNITS, un[i]);
    if (tid < 64) {
        int32_t sl;
        bool follows;
        int last;
        append_tile::own_slots<kTile>(aa.slot_mapping, aa.T, aa.num_blocks, tok0, sl, follows, last);
        if (tid < ROWS) slots[tid] = sl;
        append_tile::chunk_runs(sl, follows, runs, n_runs);
    }
    __syncthreads();
    int64_t k_dst[NK];
#pragma unroll
    for (int i = 0; i < NK; ++i) {
        const int r = (tid + kThreads * i) / UNITS;
        const int32_t slot = r < ROWS ? slots[r] : -1;
        k_on[i] = slot >= 0;
        k_dst[i] = ((int64_t)(slot / kBlockSize) * aa.Hkv * kBlockSize + slot % kBlockSize) * D;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = (tid + kThreads * i) / CPR;
        v_on[i] = r < ROWS && slots[r] >= 0;
    }
    load(g0);                                  // in flight while the angles are formed
#pragma unroll
    for (int i = 0; i < NK; ++i) {
        const int c = tid + kThreads * i;
        if (k_on[i]) turn_unit(ra, aa.positions, aa.pos_stride, tok0 + c / UNITS, c % UNITS, un[i]);
    }
    for (int g = g0; g < g1; ++g) {
        u16(*buf)[D + 8] = vs[(g - g0) & 1];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = tid + kThreads * i;
            if (v_on[i]) *reinterpret_cast<u32x4 *>(&buf[c / CPR][c % CPR * 8]) = vv[i];
        }
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            if (!k_on[i]) continue;
            rotate<IL>(un[i], ka[i], kb[i]);
            u16 *dst = aa.pool_k + k_dst[i] + (int64_t)g * kBlockSize * D;
            *reinterpret_cast<u32x4 *>(dst + un[i].at[0]) = ka[i];
            *reinterpret_cast<u32x4 *>(dst + un[i].at[1]) = kb[i];
        }
        if (g + 1 < g1) load(g + 1);
        __syncthreads();                       // (and every wave is through with the other buffer)
        append_tile::put_v<D>(buf, slots, runs, n_runs, aa.pool_v, aa.Hkv, g);
    }
}

// The first kv_wgs workgroups append (they take longest), the others rotate Q.
template <int D, bool IL, bool NT>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeArgs ra, const AppendArgs aa)
{
    if ((int)blockIdx.x < aa.kv_wgs) {
        const int tile = blockIdx.x / aa.kv_groups, g0 = (blockIdx.x - tile * aa.kv_groups) * aa.kv_heads;
        append_heads<D, IL, NT>(ra, aa, tile, g0, min(aa.Hkv, g0 + aa.kv_heads));
    } else {
        const int w = blockIdx.x - aa.kv_wgs, tile = w / aa.q_groups, h0 = (w - tile * aa.q_groups) * aa.q_heads;
        rotate_rows<IL, kThreads, 4, NT>(ra, aa.q, aa.q_stride, aa.positions, aa.pos_stride, aa.T, D, tile, h0,
                                         min(aa.Hq, h0 + aa.q_heads), aa.q_out, (int64_t)aa.Hq * D);
    }
}

// The same for few tokens, which wait on latency: single waves, one unit of one (token, head) a
// thread, V in 2-byte stores straight from the registers. No barrier, and the stores of many
// one-token sequences, each 2 bytes of a line of its own, come from many compute units.
constexpr int kRowThreads = 64;
template <int D, bool IL>
__global__ __launch_bounds__(kRowThreads) void rope_append_rows_kernel(const RopeArgs ra, const AppendArgs aa)
{
    constexpr int UNITS = D / (2 * kUnit), PER = kRowThreads / UNITS;
    if ((int)blockIdx.x < aa.kv_wgs) {
        const int64_t pair = (int64_t)blockIdx.x * PER + threadIdx.x / UNITS;   // heads of a token side by side
        const int u = threadIdx.x % UNITS, t = (int)(pair / aa.Hkv), g = (int)(pair - (int64_t)t * aa.Hkv);
        if (t >= aa.T) return;
        Unit un;
        place_unit(ra, u, un);
        const int32_t slot = aa.slot_mapping[t];
        const u16 *ks = aa.k_new + t * aa.k_stride + g * D, *vs = aa.v_new + t * aa.v_stride + g * D + 16 * u;
        u32x4 a = *reinterpret_cast<const u32x4 *>(ks + un.at[0]), b = *reinterpret_cast<const u32x4 *>(ks + un.at[1]);
        u32x4 v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const u32x4 *>(vs + 8 * i);
        turn_unit(ra, aa.positions, aa.pos_stride, t, u, un);
        if (slot < 0 || slot / kBlockSize >= aa.num_blocks) return;
        const int64_t payload = ((int64_t)(slot / kBlockSize) * aa.Hkv + g) * kBlockSize * D;
        const int o = slot % kBlockSize;
        rotate<IL>(un, a, b);
        *reinterpret_cast<u32x4 *>(aa.pool_k + payload + o * D + un.at[0]) = a;
        *reinterpret_cast<u32x4 *>(aa.pool_k + payload + o * D + un.at[1]) = b;
        u16 *dst = aa.pool_v + payload + 16 * u * kBlockSize + o;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                dst[(8 * i + j) * kBlockSize] = (u16)(v[i][j >> 1] >> (16 * (j & 1)));
    } else {
        const int w = blockIdx.x - aa.kv_wgs, tile = w / aa.Hq, h = w - tile * aa.Hq;
        rotate_rows<IL, kRowThreads, 1, false>(ra, aa.q, aa.q_stride, aa.positions, aa.pos_stride, aa.T, D, tile, h, h + 1,
                                        aa.q_out, (int64_t)aa.Hq * D);
    }
}

// Heads of a workgroup that walks several (rotate_rows): one batch of loads. Bytes in flight
// come from many workgroups rather than from long ones: 18480 tokens of 32 query heads of 128
// took 78 us with 4 heads, 82 with 8, 94 with 16 (16000 of 64 heads 109, 113, 127). Where that
// gives fewer than kMinWgs workgroups every head has one of its own (300 rows of 64 heads of
// 128: 3.8 us, 4.2 with twice the line).
constexpr int kHeads = 4;
constexpr int kMinWgs = 256;
constexpr int kMaxGridY = 65535;  // more head groups are not launched: they take more heads
// K/V workgroups wanted; a tile's kv heads are dealt to as many as that takes (2048 to 8192 alike).
constexpr int kKvWgs = 2048;
// Bytes of K and Q up to which a call runs as rows (rope_append_rows_kernel). One token of each
// of 64 sequences, 32 query / 8 kv heads of 128: 3.4 us as rows, 8.3 in tiles; 64 of one
// sequence 3.4 and 4.9; 200 4.8 and 9.5, 4.4 and 5.1; 400 (the line) 7.2 and 11.2, 6.2 and 5.8;
// 800 12.0 and 13.4, 10.9 and 7.3. With 8 / 1 heads 1600 tokens 5.3 and 10.0, 3.5 and 5.5.
constexpr int64_t kRowsBytes = 4ll << 20;
// Bytes of input above which it is read, and Q written, past the caches: input and output no
// longer fit the 256 MB cache together. 18480 tokens as above (227 MB in) 92 -> 78 us =
// 5.8 TB/s, with input in or out of the caches; 16384 rows of 40 heads of 128 (168 MB) 69 -> 64
// out of them, 65 -> 63 in them. Below the line it depends on where the input is. Past the caches
// it takes less time where the input is out of them (8000 tokens, 98 MB, 43 -> 38; 4000 24.8 -> 21.3; 4096
// rows of 40 heads of 128 21.4 -> 16.7) and more where the pass before has just written it (33.8 ->
// 37.9, 18.6 -> 20.2, 13.2 -> 14.2), which is how a layer's step finds its projections; 2000 tokens
// alone gain either way (13.2 -> 10.9, 9.8 -> 8.6). Only where each chunk's wave stores whole
// lines (runs of 64 pairs, or more of them back to back): 8065 rows of 80 dims would take 15
// instead of 12 us out of the caches. So adjacent pairs and heads turned in part stay with the caches
// at every size: 18480 tokens take 92 us with either.
constexpr int64_t kNtBytes = 128ll << 20;
bool whole_lines(const RopeArgs &ra) { return !ra.interleaved && ra.half % 64 == 0; }

// The checks of a rotation, and its launch arguments.
pcr_status rope_args(const pcr_rope *rope, int32_t head_dim, int32_t inverse, const char *who, RopeArgs *ra)
{
    if (!rope || !rope->inv_freq) return fail(PCR_ERR_INVALID_ARG, "%s: rope or its inv_freq is NULL", who);
    if (rope->rotary_dim <= 0 || rope->rotary_dim % 16 || rope->rotary_dim > head_dim)
        return fail(PCR_ERR_UNSUPPORTED, "%s: rotary_dim %d is not a positive multiple of 16 up to head_dim %d", who,
                    rope->rotary_dim, head_dim);
    if (rope->num_axes < 1 || rope->num_axes > kMaxAxes)
        return fail(PCR_ERR_INVALID_ARG, "%s: num_axes must be 1 to %d", who, kMaxAxes);
    if (!isfinite(rope->scale)) return fail(PCR_ERR_INVALID_ARG, "%s: scale is not finite", who);
    ra->half = rope->rotary_dim / 2;
    ra->axes = rope->num_axes;
    ra->interleaved = rope->interleaved != 0;
    ra->scale = rope->scale;
    ra->sin_scale = inverse ? -rope->scale : rope->scale;
    for (int j = 0; j < ra->half; ++j) {
        const int32_t a = rope->pair_axis ? rope->pair_axis[j] : 0;
        if (a < 0 || a >= rope->num_axes)
            return fail(PCR_ERR_INVALID_ARG, "%s: pair %d has axis %d of %d", who, j, a, rope->num_axes);
        if (!isfinite(rope->inv_freq[j])) return fail(PCR_ERR_INVALID_ARG, "%s: inv_freq[%d] is not finite", who, j);
        ra->axis[j] = (uint8_t)a;
        ra->turns[j] = (double)rope->inv_freq[j] / (2.0 * M_PI);
    }
    return PCR_OK;
}

// T rows of `width` elements at `stride` (multiples of 8 elements, 16-byte aligned).
constexpr int64_t kMaxSpan = 1ll << 47;   // elements: all 48-bit addresses
pcr_status check_rows(const void *x, int32_t T, int64_t stride, int64_t width, const char *what, const char *who)
{
    if (!x) return fail(PCR_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    if ((uintptr_t)x & 15) return fail(PCR_ERR_INVALID_ARG, "%s: %s must be 16-byte aligned", who, what);
    if (width > (int64_t)1 << 30) return fail(PCR_ERR_UNSUPPORTED, "%s: rows of more than 2^30 elements", who);
    if (stride < width || stride % 8 || stride > (int64_t)1 << 40)
        return fail(PCR_ERR_INVALID_ARG, "%s: %s stride %lld is not a multiple of 8 of at least %lld", who, what,
                    (long long)stride, (long long)width);
    if (stride > kMaxSpan / T)
        return fail(PCR_ERR_UNSUPPORTED, "%s: %d rows of %s at stride %lld reach past all addresses", who, T, what,
                    (long long)stride);
    return PCR_OK;
}

bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}
// Bytes from the first element of T rows to the last (2^48 and a row at most: check_rows).
int64_t span(int32_t T, int64_t stride, int64_t width) { return ((int64_t)(T - 1) * stride + width) * 2; }

bool rows_overlap(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int32_t T, int64_t width)
{
    if (!overlap(a, span(T, a_stride, width), b, span(T, b_stride, width))) return false;
    if (a_stride != b_stride) return true;
    // Parts of the same rows: the distance within a row says it.
    const uint64_t row = (uint64_t)a_stride * 2, bytes = (uint64_t)width * 2;
    const uint64_t d = (a > b ? (uintptr_t)a - (uintptr_t)b : (uintptr_t)b - (uintptr_t)a) % row;
    return d < bytes || row - d < bytes;
}

hipError_t launch_rows(const RopeArgs &ra, const void *x, int64_t x_stride, const int32_t *positions,
                       int64_t pos_stride, int32_t T, int32_t H, int32_t D, void *out, int64_t out_stride,
                       hipStream_t s)
{
    const int per = kThreads / (D / (2 * kUnit));
    const int64_t tiles = ((int64_t)T + per - 1) / per;
    int32_t heads = H >= kHeads && tiles * ((H + kHeads - 1) / kHeads) >= kMinWgs ? kHeads : 1;
    heads = std::max(heads, (H + kMaxGridY - 1) / kMaxGridY);
    const dim3 grid((unsigned)tiles, (unsigned)((H + heads - 1) / heads));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, ra, static_cast<const u16 *>(x), x_stride, positions,
                           pos_stride, T, H, D, heads, static_cast<u16 *>(out), out_stride);
    };
    if (whole_lines(ra) && (int64_t)T * H * D * 2 > kNtBytes) launch(rope_rows_kernel<false, 4, true>);
    else if (heads > 1 && ra.interleaved) launch(rope_rows_kernel<true, 4, false>);
    else if (heads > 1) launch(rope_rows_kernel<false, 4, false>);
    else if (ra.interleaved) launch(rope_rows_kernel<true, 1, false>);
    else launch(rope_rows_kernel<false, 1, false>);
    return hipGetLastError();
}

pcr_status launched(hipError_t e) { return e == hipSuccess ? PCR_OK : hip_fail(e, "pcr_rope_append_kv: launch"); }

pcr_status launch_append(const RopeArgs &ra, AppendArgs aa, int D, hipStream_t s)
{
    if ((int64_t)aa.T * (aa.Hkv + aa.Hq) * D * 2 <= kRowsBytes) {
        const int rows = kRowThreads / (D / (2 * kUnit));
        aa.kv_wgs = (int32_t)(((int64_t)aa.T * aa.Hkv + rows - 1) / rows);
        const dim3 grid((unsigned)(aa.kv_wgs + (aa.T + rows - 1) / rows * aa.Hq));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, s, ra, aa); };
        if (D == 128) {
            if (ra.interleaved) go(rope_append_rows_kernel<128, true>);
            else go(rope_append_rows_kernel<128, false>);
        } else {
            if (ra.interleaved) go(rope_append_rows_kernel<64, true>);
            else go(rope_append_rows_kernel<64, false>);
        }
        return launched(hipGetLastError());
    }
    const int per = kThreads / (D / (2 * kUnit));
    const int64_t kv_tiles = ((int64_t)aa.T + kTile - 1) / kTile, q_tiles = ((int64_t)aa.T + per - 1) / per;
    const int64_t kv_groups = (kKvWgs + kv_tiles - 1) / kv_tiles;
    aa.kv_heads = (int32_t)((aa.Hkv + kv_groups - 1) / kv_groups);
    aa.kv_groups = (aa.Hkv + aa.kv_heads - 1) / aa.kv_heads;
    aa.kv_wgs = (int32_t)(kv_tiles * aa.kv_groups);
    aa.q_heads = kHeads;
    aa.q_groups = (aa.Hq + aa.q_heads - 1) / aa.q_heads;
    const int64_t in_bytes = (int64_t)aa.T * (aa.Hq + 2 * aa.Hkv) * D * 2;
    const int64_t wgs = aa.kv_wgs + q_tiles * aa.q_groups;
    if (wgs * kThreads > (int64_t)UINT32_MAX)
        return fail(PCR_ERR_UNSUPPORTED, "pcr_rope_append_kv: %d tokens of %d query heads take 2^32 threads or more",
                    aa.T, aa.Hq);
    const dim3 grid((unsigned)wgs);
    auto launch = [&](auto dim) {
        constexpr int DD = decltype(dim)::value;
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, ra, aa); };
        if constexpr (DD == 128) {            // (64 dims have no 64 pairs)
            if (whole_lines(ra) && in_bytes > kNtBytes) return go(rope_append_kernel<DD, false, true>);
        }
        if (ra.interleaved) go(rope_append_kernel<DD, true, false>);
        else go(rope_append_kernel<DD, false, false>);
    };
    if (D == 128) launch(std::integral_constant<int, 128>{});
    else launch(std::integral_constant<int, 64>{});
    return launched(hipGetLastError());
}

}  // namespace
}  // namespace pcr

using namespace pcr;

extern "C" {

pcr_status pcr_rope_append_kv(const pcr_rope *rope, const pcr_kv_pool *pool, const void *q, int64_t q_stride,
                              const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                              const int32_t *positions, int64_t pos_stride, const int32_t *slot_mapping, int32_t T,
                              int32_t num_q_heads, void *q_out, void *stream)
{
    clear_error();
    const char *who = "pcr_rope_append_kv";
    pcr_status st = check_pool(pool, who);
    if (st) return st;
    RopeArgs ra;
    st = rope_args(rope, pool->head_dim, 0, who, &ra);
    if (st) return st;
    if (T < 0 || num_q_heads < 0) return fail(PCR_ERR_INVALID_ARG, "%s: negative T or num_q_heads", who);
    if (T > kMaxTokens) return fail(PCR_ERR_UNSUPPORTED, "%s: more than 2^27 tokens", who);
    if (num_q_heads % pool->num_kv_heads != 0)
        return fail(PCR_ERR_UNSUPPORTED, "%s: num_q_heads %d is not a multiple of num_kv_heads %d", who, num_q_heads,
                    pool->num_kv_heads);
    if (T == 0) return PCR_OK;
    const int64_t kv_width = (int64_t)pool->num_kv_heads * pool->head_dim;
    const int64_t q_width = (int64_t)num_q_heads * pool->head_dim;
    if (!positions || !slot_mapping) return fail(PCR_ERR_INVALID_ARG, "%s: NULL positions or slot_mapping", who);
    if (pos_stride < T && rope->num_axes > 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: pos_stride %lld < T", who, (long long)pos_stride);
    st = check_rows(k_new, T, k_stride, kv_width, "k_new", who);
    if (!st) st = check_rows(v_new, T, v_stride, kv_width, "v_new", who);
    if (!st && num_q_heads > 0) st = check_rows(q, T, q_stride, q_width, "q", who);
    if (!st && num_q_heads > 0) st = check_rows(q_out, T, q_width, q_width, "q_out", who);
    if (st) return st;
    if (num_q_heads > 0) {
        if (!(q == q_out && q_stride == q_width) && rows_overlap(q, q_stride, q_out, q_width, T, q_width))
            return fail(PCR_ERR_INVALID_ARG, "%s: q and q_out overlap (and are not one array)", who);
    }
    const int64_t k_span = span(T, k_stride, kv_width), v_span = span(T, v_stride, kv_width);
    const int64_t q_span = num_q_heads > 0 ? T * q_width * 2 : 0;
    if (overlap(k_new, k_span, q_out, q_span) || overlap(v_new, v_span, q_out, q_span))
        return fail(PCR_ERR_INVALID_ARG, "%s: q_out overlaps k_new or v_new", who);
    const int64_t pool_bytes = pool->num_blocks * kv_block_bytes(pool->block_size, pool->num_kv_heads, pool->head_dim);
    for (const void *x : {pool->k, pool->v})
        if (overlap(x, pool_bytes, k_new, k_span) || overlap(x, pool_bytes, v_new, v_span) ||
            overlap(x, pool_bytes, q_out, q_span))
            return fail(PCR_ERR_INVALID_ARG, "%s: k_new, v_new or q_out overlaps the pool", who);
    AppendArgs aa{};
    aa.pool_k = static_cast<u16 *>(pool->k);
    aa.pool_v = static_cast<u16 *>(pool->v);
    aa.k_new = static_cast<const u16 *>(k_new);
    aa.v_new = static_cast<const u16 *>(v_new);
    aa.q = static_cast<const u16 *>(q);
    aa.q_out = static_cast<u16 *>(q_out);
    aa.k_stride = k_stride;
    aa.v_stride = v_stride;
    aa.q_stride = q_stride;
    aa.pos_stride = pos_stride;
    aa.positions = positions;
    aa.slot_mapping = slot_mapping;
    aa.num_blocks = pool->num_blocks;
    aa.Hkv = pool->num_kv_heads;
    aa.Hq = num_q_heads;
    aa.T = T;
    return launch_append(ra, aa, pool->head_dim, static_cast<hipStream_t>(stream));
}

pcr_status pcr_rope_rows(const pcr_rope *rope, const void *x, int64_t x_stride, const int32_t *positions,
                         int64_t pos_stride, int32_t T, int32_t num_heads, int32_t head_dim, int32_t inverse,
                         void *out, int64_t out_stride, void *stream)
{
    clear_error();
    const char *who = "pcr_rope_rows";
    if (T < 0 || num_heads <= 0) return fail(PCR_ERR_INVALID_ARG, "%s: T < 0 or num_heads <= 0", who);
    if (head_dim <= 0 || head_dim % 16 || head_dim > 2 * kMaxPairs)
        return fail(PCR_ERR_UNSUPPORTED, "%s: head_dim %d is not a multiple of 16 up to %d", who, head_dim,
                    2 * kMaxPairs);
    RopeArgs ra;
    pcr_status st = rope_args(rope, head_dim, inverse, who, &ra);
    if (st || T == 0) return st;
    if (T > kMaxTokens) return fail(PCR_ERR_UNSUPPORTED, "%s: more than 2^27 tokens", who);
    if (!positions) return fail(PCR_ERR_INVALID_ARG, "%s: positions is NULL", who);
    if (pos_stride < T && rope->num_axes > 1)
        return fail(PCR_ERR_INVALID_ARG, "%s: pos_stride %lld < T", who, (long long)pos_stride);
    const int64_t width = (int64_t)num_heads * head_dim;
    st = check_rows(x, T, x_stride, width, "x", who);
    if (!st) st = check_rows(out, T, out_stride, width, "out", who);
    if (st) return st;
    if (!(x == out && x_stride == out_stride) && rows_overlap(x, x_stride, out, out_stride, T, width))
        return fail(PCR_ERR_INVALID_ARG, "%s: x and out overlap (and are not one array)", who);
    const hipError_t e = launch_rows(ra, x, x_stride, positions, pos_stride, T, num_heads, head_dim, out, out_stride,
                                     static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "pcr_rope_rows: launch");
    return PCR_OK;
}

}  // extern "C"
