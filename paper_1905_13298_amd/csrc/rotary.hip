// Query and key heads, normed and turned by their tokens' positions in one pass, and the gradient.
//
// A head's vector x of `dim` elements: n = x / sqrt(mean(x^2) + eps), u = n * weight (without a weight
// u = x), then pair i of u is turned by the angle position * frequency[i]:
//   (a, b) -> (a cos - b sin, b cos + a sin),
// pairs (i, i + pairs) or, interleaved, (2 i, 2 i + 1); elements past the pairs stay. With several axes
// the first pairs go by the first axis' positions, the next ones by the second's, and so on.
//
// The gradient turns dy back, g = R^T dy, and goes through the norm: with d = g * weight,
// dx = (d - n * mean(d * n)) / sqrt(mean(x^2) + eps), dweight = sum over tokens and heads of g * n.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "conv_plan.hpp"
#include "fastdiv.hpp"
#include "fp8.hpp"

namespace ds {

namespace {

constexpr int kMaxAxes = 4;

struct RotaryParams {
    const int *positions;
    const void *frequencies;
    int64_t pa, pb, pt;                // strides of the positions: axis, sequence, token
    int64_t in[2][3], out[2][3], grad[2][3];   // of q and k, their results, and (gradient) what comes in: sequence, token, head
    int rows;                          // batch * tokens
    FastDiv tokens;
    int heads[2], dim, pairs, interleaved, wide;     // wide: the frequencies have 64 bits
    int until[kMaxAxes];               // the pair that an axis ends before
    float eps;
    int per, chunks;                   // groups of heads that a wave takes, and how many times that q has
    int blocks;                        // of the gradient's launch, those of q
};

// A lane's 16 elements of a vector: 8 pairs from pair 8 * lane on. Pairs past `pairs`, of the elements
// that are not turned, are made up likewise; turn() leaves those as they are. RUN: so many of the lane's first (and second) elements
// lie together: 8, 4 or 1.
template <int RUN>
struct Lane {
    int j0, half, pairs, rest, interleaved;
    __device__ __forceinline__ Lane(const RotaryParams &p, int lane)
    {
        half = p.dim / 2;
        pairs = p.pairs;
        rest = half - pairs;
        interleaved = p.interleaved;
        j0 = lane * 8;
    }
    // The element of a pair.
    __device__ __forceinline__ int where(int j, int which) const
    {
        if (interleaved) return 2 * j + which;
        return j < pairs ? j + which * pairs : pairs + j + which * rest;
    }
    // Pair i turned by its angle, back where SIGN is -1. (An element that stays is chosen, not multiplied by 1 and 0: its made-up
    // partner may be infinite or NaN.)
    template <int SIGN>
    __device__ __forceinline__ void turn(int i, float cosine, float sine, float &a, float &b) const
    {
        const float x = a, y = b, s = SIGN * sine;
        const bool turned = j0 + i < pairs;
        a = turned ? fmaf(x, cosine, -(y * s)) : x;
        b = turned ? fmaf(y, cosine, x * s) : y;
    }
    // The pairs' elements a[i], b[i].
    template <typename T>
    __device__ __forceinline__ void load(const T *p, float (&a)[8], float (&b)[8]) const
    {
        if constexpr (RUN == 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                a[i] = j0 + i < half ? float(p[where(j0 + i, 0)]) : 0.f;
                b[i] = j0 + i < half ? float(p[where(j0 + i, 1)]) : 0.f;
            }
        } else {
            // Two pieces of RUN elements for RUN pairs.
            T x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; i += RUN) {
                if (RUN < 8 && j0 + i >= half) {
#pragma unroll
                    for (int e = 0; e < RUN; ++e) x[i + e] = y[i + e] = T(0.f);
                    continue;
                }
                __builtin_memcpy(x + i, p + where(j0 + i, 0), RUN * sizeof(T));
                __builtin_memcpy(y + i, p + (interleaved ? 2 * (j0 + i) + RUN : where(j0 + i, 1)), RUN * sizeof(T));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int of = i / RUN * RUN, in = i % RUN * 2;        // (interleaved: place in the two pieces)
                const T e = in < RUN ? x[of + in % RUN] : y[of + in % RUN], o = in < RUN ? x[of + in % RUN + 1] : y[of + in % RUN + 1];
                a[i] = float(interleaved ? e : x[i]);
                b[i] = float(interleaved ? o : y[i]);
            }
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T *p, const float (&a)[8], const float (&b)[8]) const
    {
        if constexpr (RUN == 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (j0 + i >= half) continue;
                p[where(j0 + i, 0)] = T(a[i]);
                p[where(j0 + i, 1)] = T(b[i]);
            }
        } else {
            T x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int of = i / RUN * RUN, in = i % RUN;
                const float lo = in & 1 ? b[of + in / 2] : a[of + in / 2], hi = in & 1 ? b[of + RUN / 2 + in / 2] : a[of + RUN / 2 + in / 2];
                x[i] = T(interleaved ? lo : a[i]);
                y[i] = T(interleaved ? hi : b[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; i += RUN) {
                if (RUN < 8 && j0 + i >= half) continue;
                __builtin_memcpy(p + where(j0 + i, 0), x + i, RUN * sizeof(T));
                __builtin_memcpy(p + (interleaved ? 2 * (j0 + i) + RUN : where(j0 + i, 1)), y + i, RUN * sizeof(T));
            }
        }
    }
};

// Cosine and sine of 2 pi t. The angle is taken in quarter turns from the nearest one, in 64 bits: three roundings (1 / 2 pi, its
// product with the frequency, that with the position), at most 3 * 2^-53 of the angle (2^-31 at a million radians), whatever the
// position. What remains, up to pi / 4, is rounded to 32 bits and goes through the Taylor polynomials up to x^9 and x^10, whose next terms
// are 2.2e-9 of x and 1.1e-10: in 32 bits, off by 2^-22 at most, as what they multiply has 24 bits itself.
__device__ __forceinline__ void turn_of(double t, float &cosine, float &sine)
{
    const double quarters = t * 4, near = rint(quarters);
    const float x = float(quarters - near) * 1.57079632679489662f, z = x * x;
    const int q = int(near - 4 * rint(near * 0.25));
    const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float u = q & 1 ? s : c, w = q & 1 ? c : s;
    cosine = (q + 1) & 2 ? -u : u;
    sine = q & 2 ? -w : w;
}

// The angles of a lane's pairs for one token. The wave's lanes work each out once and hand them on to the lanes
// of all its heads (every lane for itself: 55 us instead of 37 where a wave has one group of heads of 4 x 2001 tokens).
template <int LPV, int RUN>
__device__ __forceinline__ void angles(const RotaryParams &p, const Lane<RUN> &lane, int b, int t, float (&cosine)[8], float (&sine)[8])
{
    constexpr int kEach = LPV > 8 ? LPV / 8 : 1;         // pairs of a lane: those from 8 l + kEach * sub on
    const int l = lane.j0 / 8, sub = int(threadIdx.x & 63) / LPV;
    const int *at = p.positions + b * p.pb + t * p.pt;
    float c[kEach], s[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int j = lane.j0 + (sub * kEach + i) % 8;
        c[i] = 1.f;
        s[i] = 0.f;
        if (j >= p.pairs) continue;
        const int axis = (j >= p.until[0]) + (j >= p.until[1]) + (j >= p.until[2]);
        const double f = p.wide ? static_cast<const double *>(p.frequencies)[j] : double(static_cast<const float *>(p.frequencies)[j]);
        turn_of(double(at[axis * p.pa]) * (f * 0.15915494309189533577), c[i], s[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cosine[i] = __shfl(c[i % kEach], i / kEach * LPV + l);
        sine[i] = __shfl(s[i % kEach], i / kEach * LPV + l);
    }
}

// A wave has one token and LPV lanes for each of 64 / LPV heads of q or k at once, a group; it takes up to 4 groups of its
// token, where there are tokens enough, so that angles and weight are found once for them. Bound by bandwidth: 4 x 2001 tokens
// of 32 + 8 heads of 128, 164 MB, 30.1 us (5.4 TB/s, some of it from the caches); 8 x 1 tokens 3.2 us, the launch's trip.
template <typename T, typename W, int LPV, int RUN>
__global__ void __launch_bounds__(256)
rotary_kernel(const T *__restrict__ q, const T *__restrict__ k, const W *__restrict__ qw, const W *__restrict__ kw, T *__restrict__ qo,
              T *__restrict__ ko, const RotaryParams p)
{
    constexpr int kHeads = 64 / LPV;
    const int lane = int(threadIdx.x & 63), sub = lane / LPV;
    const int row = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * 4 + int(threadIdx.x >> 6));
    if (row >= p.rows) return;
    const int b = fdiv(row, p.tokens), t = row - b * int(p.tokens.d);
    const Lane<RUN> me(p, lane % LPV);
    const bool some = me.j0 < me.half;
    const int which = int(blockIdx.y) >= p.chunks, first = (int(blockIdx.y) - which * p.chunks) * p.per * kHeads, heads = p.heads[which];
    const W *const weight = which ? kw : qw;
    const T *const src = (which ? k : q) + b * p.in[which][0] + t * p.in[which][1];
    T *const dst = (which ? ko : qo) + b * p.out[which][0] + t * p.out[which][1];
    float cosine[8], sine[8], wa[8] = {}, wb[8] = {};
    if (weight && some) me.load(weight, wa, wb);
    angles<LPV>(p, me, b, t, cosine, sine);
    const float inv = 1.f / float(p.dim);
    for (int h0 = first; h0 < min(first + p.per * kHeads, heads); h0 += kHeads) {
        const int h = h0 + sub;
        const bool mine = some && h < heads;
        float x[8] = {}, y[8] = {};
        if (mine) me.load(src + h * p.in[which][2], x, y);
        if (weight) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
            const float r = 1.f / sqrtf(fmaf(lanes_sum<LPV>(sum), inv, p.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] *= r * wa[e];
                y[e] *= r * wb[e];
            }
        }
        if (!mine) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) me.template turn<1>(e, cosine[e], sine[e], x[e], y[e]);
        me.store(dst + h * p.out[which][2], x, y);
    }
}

// The gradient: a block has q or k; its waves go through every so many tokens' chunks and keep their sums for the
// weight, which they add up in LDS, in a fixed order, into the block's row of `part`. Bound by bandwidth: 4 x 2048 tokens of 32 + 8
// heads of 128, 252 MB, 52 us (4.8 TB/s) and 4 of adding up the rows.
template <typename T, typename W, int LPV, int RUN>
__global__ void __launch_bounds__(256)
rotary_grad_kernel(const T *__restrict__ dq, const T *__restrict__ dk, const T *__restrict__ q, const T *__restrict__ k,
                   const W *__restrict__ qw, const W *__restrict__ kw, T *__restrict__ dqo, T *__restrict__ dko, float *__restrict__ part,
                   const RotaryParams p)
{
    constexpr int kHeads = 64 / LPV;
    __shared__ float red[4][LPV * 16];
    const int lane = int(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), sub = lane / LPV;
    const Lane<RUN> me(p, lane % LPV);
    const bool some = me.j0 < me.half;
    const float inv = 1.f / float(p.dim);
    const int which = int(blockIdx.x) >= p.blocks, at = int(blockIdx.x) - which * p.blocks, blocks = which ? int(gridDim.x) - p.blocks : p.blocks;
    const int heads = p.heads[which], chunk = p.per * kHeads, chunks = (heads + chunk - 1) / chunk;
    const W *const weight = which ? kw : qw;
    float wa[8] = {}, wb[8] = {}, da[8] = {}, db[8] = {};
    if (weight && some) me.load(weight, wa, wb);
    for (int64_t unit = at * 4 + wave; unit < int64_t(p.rows) * chunks; unit += blocks * 4) {
        const int row = chunks == 1 ? int(unit) : int(unit / chunks), first = chunks == 1 ? 0 : int(unit - int64_t(row) * chunks) * chunk;
        const int b = fdiv(row, p.tokens), t = row - b * int(p.tokens.d);
        const T *const dy = (which ? dk : dq) + b * p.grad[which][0] + t * p.grad[which][1];
        const T *const src = (which ? k : q) + b * p.in[which][0] + t * p.in[which][1];
        T *const dst = (which ? dko : dqo) + b * p.out[which][0] + t * p.out[which][1];
        float cosine[8], sine[8];
        angles<LPV>(p, me, b, t, cosine, sine);
        for (int h0 = first; h0 < min(first + chunk, heads); h0 += kHeads) {
            const int h = h0 + sub;
            const bool mine = some && h < heads;
            float u[8] = {}, v[8] = {}, x[8] = {}, y[8] = {};
            if (mine) {
                me.load(dy + h * p.grad[which][2], u, v);
                if (weight) me.load(src + h * p.in[which][2], x, y);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) me.template turn<-1>(i, cosine[i], sine[i], u[i], v[i]);
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
                // (A lane without elements adds 0 to the weight's sums, also where eps is 0 and its root has no inverse.)
                const float root = sqrtf(fmaf(lanes_sum<LPV>(sum), inv, p.eps)), r = mine ? 1.f / root : 0.f;
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= r;
                    y[i] *= r;
                    da[i] = fmaf(u[i], x[i], da[i]);
                    db[i] = fmaf(v[i], y[i], db[i]);
                    u[i] *= wa[i];
                    v[i] *= wb[i];
                    sum = fmaf(u[i], x[i], fmaf(v[i], y[i], sum));
                }
                const float mean = lanes_sum<LPV>(sum) * inv;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    u[i] = r * (u[i] - x[i] * mean);
                    v[i] = r * (v[i] - y[i] * mean);
                }
            }
            if (mine) me.store(dst + h * p.out[which][2], u, v);
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float s = e ? db[i] : da[i];
#pragma unroll
            for (int o = LPV; o < 64; o <<= 1) s += __shfl_xor(s, o);
            if (sub == 0) red[wave][(lane * 2 + e) * 8 + i] = s;
        }
    __syncthreads();
    const int i = int(threadIdx.x), j = i / 16 * 8 + i % 8;
    if (i < LPV * 16 && j < me.half)
        part[int64_t(blockIdx.x) * p.dim + me.where(j, i / 8 % 2)] = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
}

// dweight = the sum over the rows of part that the blocks of q (or of k, behind them) have written: a block adds 32
// columns, 32 threads each.
template <typename W>
__global__ void __launch_bounds__(1024)
rotary_grad_weight_kernel(const float *__restrict__ part, W *__restrict__ dqw, W *__restrict__ dkw, int q_rows, int k_rows, int dim)
{
    __shared__ float red[32][33];
    const int x = int(threadIdx.x & 31), y = int(threadIdx.x >> 5), which = int(blockIdx.y), c = int(blockIdx.x) * 32 + x;
    W *const dst = which ? dkw : dqw;
    if (!dst) return;
    float sum = 0.f;
    if (c < dim) {
#pragma unroll 8
        for (int i = (which ? q_rows : 0) + y; i < q_rows + (which ? k_rows : 0); i += 32) sum += part[int64_t(i) * dim + c];
    }
    red[y][x] = sum;
    __syncthreads();
    sum = red[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 32);
    const int out = int(blockIdx.x) * 32 + y;
    if (x == 0 && out < dim) dst[out] = W(sum);
}

// f with the element type, the weights' (the same or float32), the lanes of a vector (8 pairs each) and
// how many of a lane's elements lie together.
template <typename F>
void for_layout(const RotaryParams &p, int32_t type, int32_t wtype, F &&f)
{
    const int apart = p.interleaved ? p.dim / 2 : p.pairs | p.dim / 2;
    const auto layout = [&](auto t, auto w) {
        const auto lanes = [&](auto l) {
            if (apart % 8 == 0) f(t, w, l, std::integral_constant<int, 8>{});
            else if (apart % 4 == 0) f(t, w, l, std::integral_constant<int, 4>{});
            else f(t, w, l, std::integral_constant<int, 1>{});
        };
        if (p.dim <= 64) lanes(std::integral_constant<int, 4>{});
        else if (p.dim <= 128) lanes(std::integral_constant<int, 8>{});
        else lanes(std::integral_constant<int, 16>{});
    };
    const auto weights = [&](auto t) {
        if (wtype == DS_TYPE_F32) layout(t, float{});
        else layout(t, t);
    };
    if (type == DS_TYPE_F32) weights(float{});
    else if (type == DS_TYPE_F16) weights(_Float16{});
    else weights(__bf16{});
}

// Heads of a group: those that a wave has at once.
int heads_at_once(int64_t dim) { return dim <= 64 ? 16 : dim <= 128 ? 8 : 4; }

struct Split {
    int per, chunks[2];                // groups of heads that a wave takes; chunks of q and of k
    int blocks[2];                     // of the gradient's launch: a row of the weights' sums each
};

// A wave takes up to 4 groups of a token (4 x 2001 tokens of 4 + 1 groups: 30.1 us, with 2 33.4, with 1 39.9), as long as 4096
// waves have work (2 x 1221 tokens of 2 + 2 groups: 2 each 6.9 us, 1 each 8.1). The gradient has up to 1024 blocks, four a CU,
// shared between q and k by their groups: 4 x 2048 tokens 56.2 us, with 768 56.9, with 512 66.0, with 256 103.
Split split_heads(int64_t rows, int64_t heads, int64_t kv_heads, int64_t dim)
{
    Split a;
    const int64_t once = heads_at_once(dim), groups = (heads + once - 1) / once, kv_groups = (kv_heads + once - 1) / once;
    a.per = int(std::max<int64_t>(1, std::min<int64_t>(4, rows * (groups + kv_groups) / 4096)));
    a.chunks[0] = int((groups + a.per - 1) / a.per);
    a.chunks[1] = int((kv_groups + a.per - 1) / a.per);
    for (int i = 0; i < 2; ++i) {
        const int64_t share = std::max<int64_t>(1, 1024 * (i ? kv_groups : groups) / (groups + kv_groups));
        a.blocks[i] = int(std::min<int64_t>((rows * a.chunks[i] + 3) / 4, share));
    }
    return a;
}

// What both directions check; bytes: those that q and k, and their results, span.
ds_status rotary_params(RotaryParams &p, int64_t batch, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim, int64_t pairs,
                        int64_t axes, const int32_t *sections, int32_t interleaved, float eps, int32_t type, int32_t weight_type,
                        int32_t frequency_type)
{
    if (batch < 0 || tokens < 0 || heads <= 0 || kv_heads < 0 || dim <= 0 || pairs <= 0 || axes <= 0)
        return fail(DS_ERR_INVALID_SHAPE, "batch, tokens and kv_heads must be >= 0; heads, dim, pairs and axes > 0");
    if (dim % 2 || dim > 256) return fail(DS_ERR_UNSUPPORTED, "dim must be even, at most 256");
    if (pairs > dim / 2) return fail(DS_ERR_INVALID_SHAPE, "more pairs than half of dim");
    if (axes > kMaxAxes) return fail(DS_ERR_UNSUPPORTED, "more than %d axes", kMaxAxes);
    if (axes > 1 && !sections) return fail(DS_ERR_NULL_POINTER, "several axes need sections");
    if (!float_bytes(type)) return fail(DS_ERR_INVALID_ARG, "type must be DS_TYPE_F32, DS_TYPE_F16 or DS_TYPE_BF16");
    if (weight_type != type && weight_type != DS_TYPE_F32) return fail(DS_ERR_INVALID_ARG, "weights must have q's type or float32");
    if (frequency_type != DS_TYPE_F32 && frequency_type != DS_TYPE_F64)
        return fail(DS_ERR_INVALID_ARG, "frequencies must be DS_TYPE_F32 or DS_TYPE_F64");
    if (!(eps >= 0.f)) return fail(DS_ERR_INVALID_ARG, "eps must be >= 0");
    if (heads > 65535 || kv_heads > 65535 || batch > kMaxElems || tokens > kMaxElems || batch * tokens > kMaxElems - 4096)
        return fail(DS_ERR_UNSUPPORTED, "too many heads or tokens");
    p = RotaryParams{};
    p.rows = int(batch * tokens);
    p.tokens = make_fastdiv(uint32_t(std::max<int64_t>(tokens, 1)));
    p.heads[0] = int(heads);
    p.heads[1] = int(kv_heads);
    p.dim = int(dim);
    p.pairs = int(pairs);
    p.interleaved = interleaved != 0;
    p.wide = frequency_type == DS_TYPE_F64;
    p.eps = eps;
    int64_t until = 0;
    for (int i = 0; i < kMaxAxes; ++i) {
        if (axes > 1 && i < axes) {
            if (sections[i] < 0) return fail(DS_ERR_INVALID_ARG, "sections must be >= 0");
            until += sections[i];
        }
        p.until[i] = axes == 1 || i >= axes - 1 ? int(pairs) : int(std::min<int64_t>(until, pairs));
    }
    if (axes > 1 && until != pairs) return fail(DS_ERR_INVALID_ARG, "the sections' sum is not the number of pairs");
    return DS_SUCCESS;
}

ds_status take_strides(int64_t (&to)[3], const int64_t *from)
{
    for (int i = 0; i < 3; ++i) {
        if (from[i] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        to[i] = from[i];
    }
    return DS_SUCCESS;
}

}  // namespace

}  // namespace ds

using namespace ds;

extern "C" ds_status ds_rotary_norm(const void *q, const void *k, const int32_t *positions, const void *frequencies,
                                    const void *q_weight, const void *k_weight, void *q_out, void *k_out, int64_t batch,
                                    int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim, int64_t pairs, int64_t axes,
                                    const int32_t *sections, const int64_t *q_strides, const int64_t *k_strides,
                                    const int64_t *position_strides, const int64_t *q_out_strides, const int64_t *k_out_strides,
                                    int32_t interleaved, float eps, int32_t type, int32_t weight_type, int32_t frequency_type,
                                    void *stream)
{
    if (batch != 0 && tokens != 0 &&
        (!q || !positions || !frequencies || !q_out || !q_strides || !position_strides || !q_out_strides ||
         (kv_heads != 0 && (!k || !k_out || !k_strides || !k_out_strides))))
        return fail(DS_ERR_NULL_POINTER, "a required pointer is NULL");
    RotaryParams p;
    if (ds_status st = rotary_params(p, batch, tokens, heads, kv_heads, dim, pairs, axes, sections, interleaved, eps, type, weight_type, frequency_type))
        return st;
    const int64_t blocks = (int64_t(p.rows) + 3) / 4;
    if (!grid_fits(blocks, 256)) return fail(DS_ERR_UNSUPPORTED, "too many tokens for a launch");
    if (p.rows == 0) return ok();
    int64_t ps[3];
    if (ds_status st = take_strides(ps, position_strides)) return st;
    p.pa = ps[0], p.pb = ps[1], p.pt = ps[2];
    p.positions = positions;
    p.frequencies = frequencies;
    const int64_t es = float_bytes(type), wb = dim * float_bytes(weight_type);
    int64_t in[2] = {}, out[2] = {};
    for (int i = 0; i < (kv_heads ? 2 : 1); ++i) {
        if (ds_status st = take_strides(p.in[i], i ? k_strides : q_strides)) return st;
        if (ds_status st = take_strides(p.out[i], i ? k_out_strides : q_out_strides)) return st;
        in[i] = span(batch, tokens, p.heads[i], p.in[i], dim, es);
        out[i] = span(batch, tokens, p.heads[i], p.out[i], dim, es);
    }
    if (!kv_heads) k = k_weight = nullptr, k_out = nullptr;
    if (ds_status st = check_tensors({{q, in[0], "q", false}, {k, in[1], "k", false},
                                      {positions, span(axes, batch, tokens, ps, 1, 4), "positions", false},
                                      {frequencies, pairs * (p.wide ? 8 : 4), "frequencies", false}, {q_weight, wb, "q_weight", false},
                                      {k_weight, wb, "k_weight", false}, {q_out, out[0], "q_out", true}, {k_out, out[1], "k_out", true}}))
        return st;
    const Split a = split_heads(p.rows, heads, kv_heads, dim);
    p.per = a.per;
    p.chunks = a.chunks[0];
    for_layout(p, type, weight_type, [&](auto t, auto w, auto lanes, auto run) {
        using T = decltype(t);
        using W = decltype(w);
        hipLaunchKernelGGL((rotary_kernel<T, W, decltype(lanes)::value, decltype(run)::value>), dim3(uint32_t(blocks), uint32_t(a.chunks[0] + a.chunks[1])), dim3(256), 0,
                           static_cast<hipStream_t>(stream), static_cast<const T *>(q), static_cast<const T *>(k),
                           static_cast<const W *>(q_weight), static_cast<const W *>(k_weight), static_cast<T *>(q_out),
                           static_cast<T *>(k_out), p);
    });
    return launched("ds_rotary_norm");
}

extern "C" int64_t ds_rotary_norm_backward_scratch_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim)
{
    if (batch <= 0 || tokens <= 0 || heads <= 0 || kv_heads < 0 || heads > 65535 || kv_heads > 65535 || dim <= 0 || dim > 256 || batch > kMaxElems ||
        tokens > kMaxElems || batch * tokens > kMaxElems)
        return 0;
    const Split a = split_heads(batch * tokens, heads, kv_heads, dim);
    return int64_t(a.blocks[0] + a.blocks[1]) * dim * 4;
}

extern "C" ds_status ds_rotary_norm_backward(const void *dq_out, const void *dk_out, const void *q, const void *k, const int32_t *positions,
                                             const void *frequencies, const void *q_weight, const void *k_weight, void *dq, void *dk,
                                             void *dq_weight, void *dk_weight, int64_t batch, int64_t tokens, int64_t heads,
                                             int64_t kv_heads, int64_t dim, int64_t pairs, int64_t axes, const int32_t *sections,
                                             const int64_t *dq_out_strides, const int64_t *dk_out_strides, const int64_t *q_strides,
                                             const int64_t *k_strides, const int64_t *position_strides, const int64_t *dq_strides,
                                             const int64_t *dk_strides, int32_t interleaved, float eps, int32_t type,
                                             int32_t weight_type, int32_t frequency_type, void *scratch, int64_t scratch_bytes,
                                             void *stream)
{
    if (batch != 0 && tokens != 0 &&
        (!dq_out || !positions || !frequencies || !dq || !dq_out_strides || !position_strides || !dq_strides ||
         (q_weight && (!q || !q_strides)) ||
         (kv_heads != 0 && (!dk_out || !dk || !dk_out_strides || !dk_strides || (k_weight && (!k || !k_strides))))))
        return fail(DS_ERR_NULL_POINTER, "a required pointer is NULL");
    RotaryParams p;
    if (ds_status st = rotary_params(p, batch, tokens, heads, kv_heads, dim, pairs, axes, sections, interleaved, eps, type, weight_type, frequency_type))
        return st;
    if (!kv_heads) dk_out = k = k_weight = nullptr, dk = nullptr;
    if ((dq_weight && !q_weight) || (dk_weight && !k_weight && kv_heads))
        return fail(DS_ERR_INVALID_ARG, "a gradient of a weight that is not given");
    const int64_t es = float_bytes(type), wb = dim * float_bytes(weight_type);
    const bool sums = dq_weight || dk_weight;
    const int64_t need = sums ? ds_rotary_norm_backward_scratch_bytes(batch, tokens, heads, kv_heads, dim) : 0;
    if (need > 0 && !scratch) return fail(DS_ERR_NULL_POINTER, "gradients of weights need scratch");
    if (need > scratch_bytes) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    if (p.rows == 0 && !sums) return ok();
    int64_t ps[3] = {}, in[2] = {}, out[2] = {}, grad[2] = {};
    if (p.rows > 0) {
        if (ds_status st = take_strides(ps, position_strides)) return st;
        for (int i = 0; i < (kv_heads ? 2 : 1); ++i) {
            if (ds_status st = take_strides(p.grad[i], i ? dk_out_strides : dq_out_strides)) return st;
            if (ds_status st = take_strides(p.out[i], i ? dk_strides : dq_strides)) return st;
            grad[i] = span(batch, tokens, p.heads[i], p.grad[i], dim, es);
            out[i] = span(batch, tokens, p.heads[i], p.out[i], dim, es);
            if (!(i ? k_weight : q_weight)) continue;
            if (ds_status st = take_strides(p.in[i], i ? k_strides : q_strides)) return st;
            in[i] = span(batch, tokens, p.heads[i], p.in[i], dim, es);
        }
    }
    p.pa = ps[0], p.pb = ps[1], p.pt = ps[2];
    p.positions = positions;
    p.frequencies = frequencies;
    if (ds_status st = check_tensors({{dq_out, grad[0], "dq_out", false}, {dk_out, grad[1], "dk_out", false},
                                      {q_weight ? q : nullptr, in[0], "q", false}, {k_weight ? k : nullptr, in[1], "k", false},
                                      {positions, p.rows ? span(axes, batch, tokens, ps, 1, 4) : 0, "positions", false},
                                      {frequencies, p.rows ? pairs * (p.wide ? 8 : 4) : 0, "frequencies", false},
                                      {q_weight, wb, "q_weight", false}, {k_weight, wb, "k_weight", false}, {dq, out[0], "dq", true},
                                      {dk, out[1], "dk", true}, {dq_weight, wb, "dq_weight", true}, {dk_weight, wb, "dk_weight", true},
                                      {need ? scratch : nullptr, need, "scratch", true}}))
        return st;
    const Split a = split_heads(p.rows, heads, kv_heads, dim);
    const int blocks = a.blocks[0] + a.blocks[1];           // (0 without tokens)
    p.per = a.per;
    p.blocks = a.blocks[0];
    const auto s = static_cast<hipStream_t>(stream);
    for_layout(p, type, weight_type, [&](auto t, auto w, auto lanes, auto run) {
        using T = decltype(t);
        using W = decltype(w);
        if (blocks > 0)
            hipLaunchKernelGGL((rotary_grad_kernel<T, W, decltype(lanes)::value, decltype(run)::value>), dim3(uint32_t(blocks)), dim3(256), 0, s,
                               static_cast<const T *>(dq_out), static_cast<const T *>(dk_out), static_cast<const T *>(q),
                               static_cast<const T *>(k), static_cast<const W *>(q_weight), static_cast<const W *>(k_weight),
                               static_cast<T *>(dq), static_cast<T *>(dk), sums ? static_cast<float *>(scratch) : nullptr, p);
        if (sums)
            hipLaunchKernelGGL(rotary_grad_weight_kernel<W>, dim3(uint32_t((dim + 31) / 32), 2), dim3(1024), 0, s,
                               static_cast<const float *>(scratch), static_cast<W *>(dq_weight), static_cast<W *>(dk_weight), a.blocks[0], a.blocks[1], int(dim));
    });
    return launched("ds_rotary_norm_backward");
}
