// A paged cache of keys and values in 4 bits, the way back to floats, and the attention that
// reads it.
//
// A number is E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two a byte, the first in the
// low half, with one E8M0 scale for each token, head and 32 elements. A token has its scales for
// itself, so that what a page holds never changes when others follow. Keys are rows
// [page][head][token][dim]; values lie in pieces of 16 bytes, 4 tokens x 8 dimensions
// [page][head][token / 4][dim / 8][token % 4], which is what a lane turns into an operand of the second
// product (it contracts tokens); scales are [page][head][dim / 32][token], so that those of neighbouring
// tokens are one load. Scales lie in 2^-23 .. 2^13, where every number is a 16-bit float exactly.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention.hpp"
#include "conv_plan.hpp"
#include "fastdiv.hpp"

namespace ds {

namespace {

constexpr int kBlock4 = 32;                       // elements that share a scale
constexpr int kLow4 = 127 - 23, kHigh4 = 127 + 13, kNan4 = 255;

int64_t blocks4(int64_t dim) { return (dim + kBlock4 - 1) / kBlock4; }

// ---------------------------------------------------------------------------
// To and from the cache.

struct CacheParams {
    const int *table, *start, *count;
    int64_t ldt;
    int columns, pages, tokens, heads, dim, page_shift, blocks, per;      // per: workgroups of a sequence
    FastDiv lanes, by_head;            // threads of a vector (8 elements each, whole scale blocks), heads
    int64_t sb[2], st[2], sh[2];       // strides of k and v: sequence, token, head
};

// A thread's share of k or v: 8 elements of N tokens, where N is 4 those of one multiple of 4 positions, whose values
// and scales lie together in the cache. Which they are, and where the cache has them.
template <int N>
struct Place {
    int b, t, h, lane, slot;           // t, slot: of the first of the N (t may be negative)
    int low, high;                     // the tokens t + low .. t + high - 1 are meant
    int64_t at;                        // page and head, -1: nowhere
    __device__ __forceinline__ Place(const CacheParams &p)
    {
        b = int(blockIdx.x) / p.per;
        const int i = (int(blockIdx.x) - b * p.per) * 256 + int(threadIdx.x), vec = fdiv(i, p.lanes), nth = fdiv(vec, p.by_head);
        lane = i - vec * int(p.lanes.d);
        h = vec - nth * p.heads;
        const int start = p.start[b], n = p.count ? min(max(p.count[b], 0), p.tokens) : p.tokens;     // (n - t stays a 32-bit number)
        t = nth * N - (start & (N - 1));
        low = max(-t, 0);
        high = min(n - t, N);
        at = -1;
        slot = 0;
        if (start < 0 || high <= low) return;
        const uint32_t pos = uint32_t(start) - uint32_t(start & (N - 1)) + uint32_t(nth) * N, col = pos >> p.page_shift;
        if (col >= uint32_t(p.columns)) return;
        const int pid = p.table[b * p.ldt + col];
        if (unsigned(pid) >= unsigned(p.pages)) return;
        at = int64_t(pid) * p.heads + h;
        slot = int(pos) & ((1 << p.page_shift) - 1);
    }
    // The bytes of the first token's codes (keys: the next ones dim / 2 further; values: 4), and of the scales.
    __device__ __forceinline__ int64_t codes(const CacheParams &p, bool values) const
    {
        return (at << p.page_shift) * (p.dim / 2) + (values ? (slot >> 2) * 2 * p.dim + lane * 16 + (slot & 3) * 4 : slot * (p.dim / 2) + lane * 4);
    }
    __device__ __forceinline__ int64_t scale(const CacheParams &p) const
    {
        return ((at * p.blocks + (lane >> 2)) << p.page_shift) + slot;
    }
};

// 2^(e - 127) of the scale byte e for the conversions, which look at the exponent's bits alone
// (255: NaN).
__device__ __forceinline__ float scale4(uint32_t e) { return __uint_as_float(e << 23); }

// The same of scale byte i of a word (the conversions do not look at the sign and the mantissa).
__device__ __forceinline__ float scale_of(uint32_t word, int i)
{
    return __uint_as_float(i == 0 ? word << 23 : i == 1 ? word << 15 : i == 2 ? word << 7 : word >> 1);
}

// The scale byte of the least power of two that brings `amax` (finite, >= 0) to at most 6 = 1.5 * 2^2:
// a mantissa above 1.5 carries into the exponent.
__device__ __forceinline__ int scale_byte4(float amax)
{
    return min(max(int((__float_as_uint(amax) + 0x3fffffu) >> 23) - 2, kLow4), kHigh4);
}

// The largest of four neighbouring lanes' values (>= 0, or infinite), in all four.
__device__ __forceinline__ float max_of_4(float v)
{
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true)));       // lanes 1, 0, 3, 2
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true)));    // lanes 2, 3, 0, 1
}

// New tokens into their pages: 8 elements of N tokens a thread, 4 threads a scale. An element that is no finite
// number makes its block NaN (scale byte 255, codes 0). Bound by bandwidth: 4 x 2001 tokens of 8 heads of 128 in 16 bits,
// 42 MB, 11.5 us (3.6 TB/s, the launch's 2 us among them); 64 x 1 3.2.
template <typename T, int N>
__global__ void __launch_bounds__(256)
append4_kernel(const T *__restrict__ k, const T *__restrict__ v, uint8_t *__restrict__ kc, uint8_t *__restrict__ vc,
               uint8_t *__restrict__ ks, uint8_t *__restrict__ vs, const CacheParams p)
{
    const int which = int(blockIdx.y);
    const Place<N> at(p);
    const bool mine = at.at >= 0 && at.lane * 8 < p.dim;
    const T *const src = (which ? v : k) + at.b * p.sb[which] + at.t * p.st[which] + at.h * p.sh[which] + at.lane * 8;
    Eight<T> x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        x[j].clear();
        if (mine && j >= at.low && j < at.high) __builtin_memcpy(x[j].v, src + j * p.st[which], sizeof x[j].v);
    }
    uint32_t q[N], scales = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        bool fine = true;
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            fine = fine && fabsf(x[j].at(i)) < __builtin_inff();
            top = fmaxf(top, fabsf(x[j].at(i)));
        }
        top = max_of_4(fine ? top : __builtin_inff());
        fine = top < __builtin_inff();
        const uint32_t e = fine ? uint32_t(scale_byte4(top)) : uint32_t(kNan4);
        const float s = scale4(e);
        q[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[j].at(0), x[j].at(1), s, 0);
        q[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[j], x[j].at(2), x[j].at(3), s, 1);
        q[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[j], x[j].at(4), x[j].at(5), s, 2);
        q[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[j], x[j].at(6), x[j].at(7), s, 3);
        q[j] = fine ? q[j] : 0u;
        scales |= e << (8 * j);
    }
    if (!mine) return;
    uint8_t *const codes = (which ? vc : kc) + at.codes(p, which), *const e = (which ? vs : ks) + at.scale(p);
    const bool whole = N == 4 && at.low == 0 && at.high == 4;
    if (which && whole) {
        __builtin_memcpy(__builtin_assume_aligned(codes, 4 * N), q, sizeof q);
    } else {
        const int step = which ? 4 : p.dim / 2;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j >= at.low && j < at.high) *reinterpret_cast<uint32_t *>(codes + j * step) = q[j];
    }
    if ((at.lane & 3) != 0) return;
    if (whole) {
        *reinterpret_cast<uint32_t *>(e) = scales;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j >= at.low && j < at.high) e[j] = uint8_t(scales >> (8 * j));
    }
}

// Eight numbers of a scale, exactly (2^-24 .. 6 * 2^13: 16-bit floats; NaN of scale byte 255).
__device__ __forceinline__ void widen4(uint32_t codes, float s, float (&x)[8])
{
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// Tokens of a cache as floats [sequence][token][head][dim], 0 where there is none: 8 elements of N tokens a
// thread. Bound by bandwidth: 6 x 20000 tokens of 8 heads of 128 to 16 bits, 608 MB, 115 us (5.3 TB/s).
template <typename T, int N>
__global__ void __launch_bounds__(256)
read4_kernel(T *__restrict__ k, T *__restrict__ v, const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
             const uint8_t *__restrict__ ks, const uint8_t *__restrict__ vs, const CacheParams p)
{
    const int which = int(blockIdx.y);
    const Place<N> at(p);
    if (at.lane * 8 >= p.dim) return;
    uint32_t q[N] = {}, scales = 0;
    if (at.at >= 0) {
        const uint8_t *const codes = (which ? vc : kc) + at.codes(p, which);
        if (which) {
            __builtin_memcpy(q, __builtin_assume_aligned(codes, 4 * N), sizeof q);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) q[j] = *reinterpret_cast<const uint32_t *>(codes + j * (p.dim / 2));
        }
        const uint8_t *const e = (which ? vs : ks) + at.scale(p);
        scales = N == 4 ? *reinterpret_cast<const uint32_t *>(e) : *e;
    }
    T *const dst = (which ? v : k) + at.b * p.sb[which] + at.t * p.st[which] + at.h * p.sh[which] + at.lane * 8;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (at.t + j < 0 || at.t + j >= p.tokens) continue;
        float x[8] = {};
        if (at.at >= 0 && j >= at.low && j < at.high) widen4(q[j], scale_of(scales, j), x);
        store8(dst + j * p.st[which], 8, x);
    }
}

// ---------------------------------------------------------------------------
// Attention. A kv head's queries are its `rows` = tokens x group vectors, and a wave
// handles 16 of them at a time with 64 keys:
//
//   S^T = K Q^T (the matrix instruction's rows are keys, its columns queries), so that a
//   lane holds 16 consecutive keys of one query;
//   t = S * scale * log2(e), p = 2^(t - m), m such that the largest p of a row is from 2^9 to 2^15;
//   O^T += V^T P (rows: dimensions, columns: queries), l += p.
//
// The key of row r of a 16-key tile t is 4 r + t: lane group g (lane / 16) holds the products of keys
// 16 g .. 16 g + 15, and those are the ones that it contracts in the second product, 8 at a time; and a
// lane's four keys of the first product have their scales side by side. Dimension r of tile j of
// the second product is 8 r + j (of heads of up to 64: 4 r + j; above 128 there are two such sets), so that a lane's
// dimensions are neighbours in memory too. Keys become numbers of the queries' type exactly, with their scales; p and the values
// are 16-bit floats with 10 bits of mantissa: values exactly, p rounded once, to 2^-11 of itself down to
// 2^-23 of the row's largest and to 2^-34 of that one below (l has all of it in 32 bits). That rounding buys one matrix
// instruction of 16-bit floats where p as a sum of two of them needs two: 2 x 1000 queries over 8000 keys 243 us for 331, 32 x 5
// over up to 4000 34.2 for 38.4, one over 131072 34.3 for 35.5 (float16 results 2.2e-4 of their size off instead of 2.1e-4).

// Eight numbers as an operand.
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type operand4(uint32_t codes, float s)
{
    if constexpr (__is_same(T, _Float16)) {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 1);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 3);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
}

// 0x80 in each byte of x that is 255, the scale that is NaN. A weight of 0 does not keep a NaN out of a
// sum: where some queries see a step's keys and others do not, such scales are taken out, and come back
// as NaN in the results of the queries that see them (a product of where they are with what is seen).
__device__ __forceinline__ uint32_t nan_scales(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & x & 0x80808080u; }

// Two dimensions (byte `sel` of each) of 8 tokens, the numbers of a dimension together: 4 tokens a
// piece, a word each, scales s.
template <int SEL>
__device__ __forceinline__ void turn4(const i32x4 &a, const i32x4 &b, const float (&s)[8], f16x8 &even, f16x8 &odd)
{
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(uint32_t(i < 4 ? a[i] : b[i - 4]), s[i], SEL);
        x[i] = __builtin_bit_cast(uint32_t, y);
    }
    i32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = int(__builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u));
        hi[i] = int(__builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u));
    }
    even = __builtin_bit_cast(f16x8, lo);
    odd = __builtin_bit_cast(f16x8, hi);
}

// f(0) .. f(N - 1) with the number as a constant.
template <int FROM, int TO, typename F>
__device__ __forceinline__ void unroll(F &&f)
{
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        unroll<FROM + 1, TO>(f);
    }
}

// Up to 16 TILES queries of a kv head at a time (tokens being decoded): a block of 4 waves takes a share of the keys, each wave
// every fourth 64 of it straight from memory to registers (no two waves share any), and joins them at its end.
// Bound by reading the cache once, and by the blocks' starts and ends: 131072 keys of 8 heads of 128, 143 MB, 30.3 us
// (4.7 TB/s) and 3.4 of joining; its VALU instructions, a third of them conversions, would take 38 % of that. Heads
// above 128 need 369 registers and have one block a CU: as many bytes in 4 heads of 256 47 us in all.
template <typename T, int DP, int TILES>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1)
attention4_few_kernel(const AttentionParams p, int blocks)
{
    constexpr int kWaves = 4;
    constexpr int QC = DP / 32;            // chunks of 32 of the first product's contraction, words of a lane's part of a key
    constexpr int DT = DP / 16;            // tiles of 16 dimensions of the second product
    constexpr int NS = DP == 256 ? 2 : 1;  // scale blocks of a lane's part of a key, or value
    typedef typename Vec8<T>::type v8;
    __shared__ float ml[2][kWaves][16];
    __shared__ f32x4 osum[kWaves][DT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const int split = int(blockIdx.x), bh = int(blockIdx.y), b = bh / p.heads, h = bh - b * p.heads;
    const int D = p.dim, page = 1 << p.page_shift, row0 = int(blockIdx.z) * 16 * TILES;
    const Sequence seq(p, b);
    // Keys that some query sees lie in [tlo, thi); every query that sees any sees [alo, ahi).
    const int t1 = min(seq.count, p.tokens) - 1, t0 = min(max(-seq.first, 0), max(t1, 0));      // the first query that is not before the first key
    const int thi = t1 >= t0 ? min(max(seq.first + t1 + 1, 0), seq.keys) : 0, ahi = min(max(seq.first + t0 + 1, 0), seq.keys);
    const int tlo = p.window ? max(seq.first + t0 + 1 - p.window, 0) : 0, alo = p.window ? max(seq.first + t1 + 1 - p.window, 0) : 0;
    const int s0 = thi > tlo ? tlo / kStep : 0, s1 = thi > tlo ? (thi + kStep - 1) / kStep : 0;
    const int each = max((s1 - s0 + p.splits - 1) / p.splits, p.least);
    const int from = s0 + split * each, to = min(s1, from + each);
    auto part_of = [&](int row) { return p.part + ((int64_t(bh) * p.rows + row) * p.splits + split) * (D + 2); };
    if (p.part && from >= to) {      // nothing here: no results, only that there are none
        if (int(threadIdx.x) < min(16 * TILES, p.rows - row0)) {
            float *const part = part_of(row0 + int(threadIdx.x));
            part[D] = -__builtin_inff();
            part[D + 1] = 0.f;
        }
        return;
    }

    f32x4 acc[TILES][DT];
    float m[TILES], l[TILES];
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        m[u] = -__builtin_inff();
        l[u] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[u][d] = f32x4{};
    }
    // Page of the 16 keys from `key` on (they share it), or -1 where there is none.
    auto page_of = [&](int key) {
        const int col = key >> p.page_shift;
        const int pid = key < thi ? p.table[b * p.ldt + col] : -1;
        return unsigned(pid) < unsigned(p.pages) ? pid : -1;
    };
    // What a lane reads of a step: a quarter of the dimensions of keys 4 r .. 4 r + 3, and of the values 16 tokens
    // x 8 dimensions (of heads of up to 64 half of that counts, of more than 128 it is twice as much). Where there is no page, page 0
    // is read instead, and what lies past `dim` somewhere inside.
    struct Step {
        uint32_t k[4][QC], ks[NS], vs[NS][4];
        i32x4 v[NS][4];
        int vp;
    };
    uint32_t koff[QC / 2], kso[NS], voff[NS], vso[NS];
#pragma unroll
    for (int c = 0; c < QC / 2; ++c) koff[c] = uint32_t(min(g * (DP / 4) + c * 16, D - 16) / 2 + (r & 3) * 4 * (D / 2));
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int d = min(DP == 64 ? r * 4 : i * 128 + r * 8, D - 8);
        kso[i] = uint32_t(min(g * (DP / 4) / 32 + i, blocks - 1) * page + (r & 3) * 4);
        voff[i] = uint32_t(d / 8 * 16);
        vso[i] = uint32_t(d / 32 * page);
    }
    auto fetch = [&](int step, int kp, int vp, Step &x) {
        const int kslot = (step * kStep + (r >> 2) * 16) & (page - 1), vslot = (step * kStep + g * 16) & (page - 1);
        const int64_t kat = int64_t(max(kp, 0)) * p.heads + h, vat = int64_t(max(vp, 0)) * p.heads + h;
        const uint8_t *const k = p.kc + (kat * page + kslot) * (D / 2), *const ks = p.ks + kat * blocks * page + kslot;
        const uint8_t *const v = p.vc + (vat * page + vslot) * (D / 2), *const vs = p.vs + vat * blocks * page + vslot;
        if (DP > 64 && D == DP) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < QC; c += 4) {
                    const i32x4 y = *reinterpret_cast<const i32x4 *>(k + koff[c / 2] + t * (DP / 2));
#pragma unroll
                    for (int w = 0; w < 4; ++w) x.k[t][(c + w) % QC] = uint32_t(y[w]);
                }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < QC; c += 2) {
                    const i32x2 y = *reinterpret_cast<const i32x2 *>(k + koff[c / 2] + t * (D / 2));
                    const bool in = g * (DP / 4) + c * 8 < D;
                    x.k[t][c] = in ? uint32_t(y[0]) : 0u;
                    x.k[t][c + 1] = in ? uint32_t(y[1]) : 0u;
                }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            x.ks[i] = *reinterpret_cast<const uint32_t *>(ks + kso[i]);
#pragma unroll
            for (int q = 0; q < 4; ++q) x.v[i][q] = *reinterpret_cast<const i32x4 *>(v + voff[i] + q * 2 * D);
            const i32x4 e = *reinterpret_cast<const i32x4 *>(vs + vso[i]);
#pragma unroll
            for (int q = 0; q < 4; ++q) x.vs[i][q] = uint32_t(e[q]);
        }
        x.vp = vp;
    };
    // The next step's pages are looked up while this one's keys and values are worked on. (Those themselves a step
    // ahead: 38.1 us instead of 35.2 for 131072 keys, 64.7 and 61.1 for 48 x 1: registers for a third wave of a SIMD.)
    int kp = -1, vp = -1;
    auto look = [&](int step) {
        kp = page_of(step * kStep + (r >> 2) * 16);
        vp = page_of(step * kStep + g * 16);
    };
    look(from + wave);
    v8 qf[TILES][QC];
    int low[TILES], high[TILES];
    bool none[TILES];
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        load_query<T, DP, 8, DP / 4, QC>(p, seq, b, h, row0 + u * 16 + r, g, low[u], high[u], qf[u]);
        // A row that sees no key, and is 0 in the end, takes part as if it saw every one, which costs less.
        none[u] = high[u] == 0;
        if (none[u]) high[u] = 0x7fffffff;
    }
    for (int step = from + wave; step < to; step += kWaves) {
        Step x;
        const int base = step * kStep, vrun = base + g * 16;
        fetch(step, kp, vp, x);
        look(step + kWaves);
        const bool there = x.vp >= 0;
        f32x4 products[TILES][4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                const v8 key = operand4<T>(x.k[t][c], scale_of(x.ks[c * NS / QC], t));
#pragma unroll
                for (int u = 0; u < TILES; ++u) products[u][t] = mma(key, qf[u][c], c == 0 ? f32x4{} : products[u][t]);
            }
        f16x8 pf[TILES][2];
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            f32x4 (&s)[4] = products[u];
            // Element i of s[t]: key vrun + 4 i + t.
            if (!__all(there && vrun >= low[u] && vrun + 16 <= high[u])) {
                int run = vrun;
                asm volatile("" : "+v"(run));         // (what follows is not worked out where it is not needed)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = run + (i & 3) * 4 + (i >> 2);
                    s[i >> 2][i & 3] = there && key >= low[u] && key < high[u] ? s[i >> 2][i & 3] : -__builtin_inff();
                }
            }
            const float sub = or_zero(m[u]);
            float e[16], top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] = fmaf(s[i & 3][i >> 2], p.scale, -sub);        // (key vrun + i)
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(e[i], e[i + 1]));
            raise(m[u], l[u], max_over_32(max_over_16(top)),
                  [&](float by) {
#pragma unroll
                      for (int i = 0; i < 16; ++i) e[i] -= by;
                  },
                  [&](float alpha) {
#pragma unroll
                      for (int d = 0; d < DT; ++d) acc[u][d] *= alpha;
                  });
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                e[i] = __builtin_amdgcn_exp2f(e[i]);
                l[u] += e[i];
                pf[u][i >> 3][i & 7] = _Float16(e[i]);
            }
        }
        if (!__all(there && base + kStep <= thi && base >= tlo)) {
            // Keys that no query sees may hold anything: their values count as 0 (whatever the code, 2^-127
            // of it is 0 as a 16-bit float).
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < NS; ++i) x.vs[i][q] &= uint32_t(there ? key_mask(vrun + 4 * q, tlo, thi) : 0);
        }
        if (base + kStep > ahi || base < alo) {
            uint32_t nan = 0;
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) nan |= nan_scales(x.vs[i][q]);
            if (__any(nan != 0)) {
                int run = vrun;
                asm volatile("" : "+v"(run));
                f32x4 n[TILES][NS];
#pragma unroll
                for (int u = 0; u < TILES; ++u) {
                    f16x8 seen[2];
#pragma unroll
                    for (int i = 0; i < 16; ++i) seen[i >> 3][i & 7] = _Float16(there && run + i >= low[u] && run + i < high[u] ? 1.f : 0.f);
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        n[u][i] = f32x4{};
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            f16x8 where;
#pragma unroll
                            for (int j = 0; j < 8; ++j) where[j] = _Float16((x.vs[i][2 * c + j / 4] >> (8 * (j & 3)) & 255u) == 255u ? 1.f : 0.f);
                            n[u][i] = mma(where, seen[c], n[u][i]);
                        }
                        // A lane's dimensions have their scale in common: the same in all of their tiles.
#pragma unroll
                        for (int d = i * (DT / NS); d < (i + 1) * (DT / NS); ++d)
#pragma unroll
                            for (int w = 0; w < 4; ++w) acc[u][d][w] += n[u][i][w] > 0.f ? __builtin_nanf("") : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < NS; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) x.vs[i][q] &= ~((nan_scales(x.vs[i][q]) >> 7) * 0xffu);
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                i32x4 va = x.v[i][2 * c], vb = x.v[i][2 * c + 1];
                if (DP == 64 && (r & 1)) {         // the other half of the pieces' dimensions
                    va >>= 16;
                    vb >>= 16;
                }
                float sv[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) sv[j] = scale_of(x.vs[i][2 * c + j / 4], j & 3);
                auto pair = [&](auto sel) {
                    constexpr int SEL = decltype(sel)::value;
                    f16x8 even, odd;
                    turn4<SEL>(va, vb, sv, even, odd);
#pragma unroll
                    for (int u = 0; u < TILES; ++u) {
                        f32x4 &a = acc[u][i * (DT / NS) + 2 * SEL], &b = acc[u][i * (DT / NS) + 2 * SEL + 1];
                        a = mma(even, pf[u][c], a);
                        b = mma(odd, pf[u][c], b);
                    }
                };
                pair(std::integral_constant<int, 0>{});
                pair(std::integral_constant<int, 1>{});
                if constexpr (DP > 64) {
                    pair(std::integral_constant<int, 2>{});
                    pair(std::integral_constant<int, 3>{});
                }
            }
    }
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        if (u > 0) __syncthreads();
        const int row = row0 + u * 16 + r;
        if (none[u]) {
            m[u] = -__builtin_inff();
            l[u] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[u][d] = f32x4{};
        }
        // The waves' sums together: a lane's l is its own keys'.
        l[u] += __shfl_xor(l[u], 16);
        l[u] += __shfl_xor(l[u], 32);
        if (g == 0) {
            ml[0][wave][r] = m[u];
            ml[1][wave][r] = l[u];
        }
        __syncthreads();
        float top = ml[0][0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[0][w][r]);
        const float sub = or_zero(top), mine = __builtin_amdgcn_exp2f(m[u] - sub);
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total = fmaf(ml[1][w][r], __builtin_amdgcn_exp2f(ml[0][w][r] - sub), total);
        // Four dimensions that are neighbours, tiles 4 d .. 4 d + 3 of one row, a piece.
#pragma unroll
        for (int d = 0; d < DT; d += 4)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                osum[wave][d + w][lane] = f32x4{acc[u][d][w], acc[u][d + 1][w], acc[u][d + 2][w], acc[u][d + 3][w]} * mine;
        __syncthreads();
        if (row >= p.rows) continue;
        float *const part = p.part ? part_of(row) : nullptr;
        if (part && wave == 0 && g == 0) {
            part[D] = top;
            part[D + 1] = total;
        }
        const float inv = inverse(total);
        for (int d = wave; d < DT; d += kWaves) {
            // Tiles d & -4 .. + 3 of row 4 g + d % 4.
            const int line = g * 4 + (d & 3), tile = d & -4;
            const int dim = DP == 64 ? line * 4 : tile / 8 * 128 + line * 8 + (tile & 4);
            if (dim >= D) continue;
            f32x4 o = osum[0][d][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) o += osum[w][d][lane];
            store_row<T>(p, b, h, row, part, dim, o, inv);
        }
    }
}

// Many queries of a kv head: a block's four waves have 32 of them each and share the keys, 64 at a
// time. A wave reads its part of them a step ahead, turns them into 16-bit floats, once for
// the whole block, and puts them into LDS: keys as rows [key][dim], values as rows [dim][key],
// the 16-byte pieces of a row in an order of its own, so that the lanes of a read (0-3, 12-15,
// 20-27 at once, and so on) meet in no bank.
//
// The products are 32 x 32: one query a lane and 32 keys of it, 8 of each 16. Row 8 w + 4 hf + e of tile
// tt is key 32 tt + 16 (w / 2) + 8 hf + 4 (w % 2) + e: lane half hf then holds the keys that it
// contracts in the second product.
//
// Bound by the matrix instructions and the exponentials between them, which two waves of a SIMD overlap in
// part, and by turning keys and values into floats (without it 217 us): 2 x 1000 queries of 32 heads over up to 8000
// keys of 8 heads of 128 take 243-246 us, 980 TFLOP/s. (Blocks of eight waves, which turn half as much each, 281.) Heads of 65 to
// 128 spill 11 registers, those above, which leave one wave a SIMD, 57: 4 x 300 queries of 256 over up to 4000 221 us, 420 TFLOP/s.
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 256 ? 1 : 2)
attention4_many_kernel(const AttentionParams p, int blocks, int bhs)
{
    constexpr int kWaves = 4, QC = DP / 16, DT = DP / 32;
    constexpr int kWords = DP / 32;            // words (8 codes) of a lane's part of a run's keys, and of its values' tokens
    constexpr int NS = DP == 256 ? 2 : 1;      // scale blocks of it
    constexpr int kKeys = kStep * DP * 2;      // bytes of a step's keys, or values
    typedef typename Vec8<T>::type v8;
    __shared__ __align__(16) uint8_t lds[2][2 * kKeys];
    __shared__ int nans[2][kWaves];             // whether a wave's part of the values has any
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 31, hf = lane >> 5, g = lane >> 4;
    // An eighth of the work to each XCD, a head's blocks together, so that they read its
    // keys through one L2, the same head of every sequence next, whose lengths may differ; the
    // last rows, which see the most keys, first.
    const int per = p.row_tiles * p.splits, all = bhs * per, share = (all + 7) >> 3;
    const int at = (int(blockIdx.x) & 7) * share + (int(blockIdx.x) >> 3);
    if ((int(blockIdx.x) >> 3) >= share || at >= all) return;
    const int unit = at / per, rest = at - unit * per, tile = p.row_tiles - 1 - rest / p.splits, split = rest % p.splits;
    const int batch = bhs / p.heads, h = unit / batch, b = unit - h * batch, bh = b * p.heads + h;
    const int D = p.dim, page = 1 << p.page_shift;
    const Sequence seq(p, b);
    v8 qf[QC];
    int low, high;
    const int row = (tile * kWaves + wave) * 32 + r;
    const bool live = load_query<T, DP, 16, 8, QC>(p, seq, b, h, row, hf, low, high, qf);
    // A row without a query sees every key, which costs less than no key, and is 0 in the end.
    if (!live) high = 0x7fffffff;
    // The block's keys: from the first that its first query sees to its last query's own.
    const int t0 = tile * kWaves * 32 / p.group, t1 = min(((tile + 1) * kWaves * 32 - 1) / p.group, seq.count - 1);
    const int thi = t0 < seq.count ? min(max(seq.first + t1 + 1, 0), seq.keys) : 0;
    const int tlo = p.window ? max(max(seq.first + t0 + 1, 0) - p.window, 0) : 0;
    // Steps of which one of its queries does not see every key.
    const int alo = p.window ? max(max(seq.first + t1 + 1, 0) - p.window, 0) : 0, ahi = min(max(seq.first + t0 + 1, 0), seq.keys);
    auto mixed = [&](int step) { return step * kStep < alo || step * kStep + kStep > ahi; };
    const int s0 = thi > tlo ? tlo / kStep : 0, s1 = thi > tlo ? (thi + kStep - 1) / kStep : 0;
    const int each = (s1 - s0 + p.splits - 1) / p.splits;
    const int from = s0 + split * each, to = min(s1, from + each);

    f32x16 acc[DT];
    float m = -__builtin_inff(), l = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x16{};
    // The table's entry of the g-th 16 keys of a step; a page of the cache or -1.
    const int *const table = p.table + b * p.ldt;
    auto entry = [&](int step) {
        const int key = step * kStep + g * 16;
        return step < to && key < thi ? table[key >> p.page_shift] : -1;
    };
    auto on_page = [&](int pid) { return unsigned(pid) < unsigned(p.pages) ? pid : -1; };
    auto on_pages = [&](int pids) { return bool(__all(pids >= 0)); };
    // A lane's part of a run of 16 keys: a quarter of the dimensions of one key, and of the values 4 tokens x 8 dimensions
    // (of heads of up to 64 half of them, of more than 128 two such pieces). What lies past `dim` is read somewhere
    // inside. Where there is no page, page 0 is read instead. Which lane has which part is such that lanes which
    // write to LDS at once, 128 bytes of them, meet in no bank (with neighbours in a row half of the writes' cycles
    // were conflicts: 250.9 us for 249.4; 4 x 300 queries of heads of 256 over 4000 keys 229.8 for 221.1).
    const int bit2 = (lane >> 2) & 1, bit3 = (lane >> 3) & 1, high2 = lane >> 4;
    const int kkey = DP == 64 ? high2 * 4 + bit2 * 2 + bit3 : DP == 128 ? high2 * 4 + ((lane >> 1) & 3) : bit2 * 8 + bit3 * 4 + (lane & 3);
    const int quarter = DP == 64 ? lane & 3 : DP == 128 ? bit3 * 2 + (lane & 1) : high2, kdim = quarter * (DP / 4);
    const int quad = (lane >> 5) * 2 + (lane & 1), vgroup = ((lane >> 4) & 1) * 8 + ((lane >> 1) & 7);
    uint32_t kraw[kWords], kse[NS], vse[NS];
    i32x4 vraw[NS];
    uint32_t koff[kWords / 2], kso[NS], voff[NS], vso[NS];
#pragma unroll
    for (int i = 0; i < kWords / 2; ++i) koff[i] = uint32_t(kkey * (D / 2) + min(kdim + i * 16, D - 16) / 2);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int d = min(DP == 64 ? vgroup * 4 : i * 128 + vgroup * 8, D - 8);
        kso[i] = uint32_t(min(kdim / 32 + i, blocks - 1) * page + kkey);
        voff[i] = uint32_t(quad * 2 * D + d / 8 * 16);
        vso[i] = uint32_t(d / 32 * page + quad * 4);
    }
    const int64_t head_bytes = int64_t(D / 2) * page, head_scales = int64_t(blocks) * page;
    const uint8_t *const kh = p.kc + h * head_bytes, *const vh = p.vc + h * head_bytes;
    const uint8_t *const ksh = p.ks + h * head_scales, *const vsh = p.vs + h * head_scales;
    const int64_t page_bytes = p.heads * head_bytes, page_scales = p.heads * head_scales;
    auto fetch = [&](int step, int pids) {
        const int pid = max(__builtin_amdgcn_readlane(pids, wave * 16), 0), slot = (step * kStep + wave * 16) & (page - 1);
        const uint8_t *k = kh + pid * page_bytes + slot * (D / 2), *v = vh + pid * page_bytes + slot * (D / 2);
        const uint8_t *ks = ksh + pid * page_scales + slot, *vs = vsh + pid * page_scales + slot;
        if (kWords >= 4 && D == DP) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const i32x4 x = *reinterpret_cast<const i32x4 *>(k + koff[2 * i]);
#pragma unroll
                for (int w = 0; w < 4; ++w) kraw[4 * i + w] = uint32_t(x[w]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 2; ++i) {
                const i32x2 x = *reinterpret_cast<const i32x2 *>(k + koff[i]);
                kraw[2 * i] = uint32_t(x[0]);
                kraw[2 * i + 1] = uint32_t(x[1]);
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            vraw[i] = *reinterpret_cast<const i32x4 *>(v + voff[i]);
            kse[i] = ks[kso[i]];
            vse[i] = *reinterpret_cast<const uint32_t *>(vs + vso[i]);
        }
    };
    // The order of a key's pieces: its row in a tile, from 16 on again (rows of 128 bytes share a bank row
    // by twos); of a dimension's pieces: such that both a read's 16 dimensions and a write's, every
    // fourth or eighth of 8, are spread.
    auto order = [](int key) { return ((key & 3) | ((key >> 3) & 1) << 2 | ((key >> 2) & 1) << 3) >> (DP < 128 ? 1 : 0); };
    auto vorder = [](int d) { return ((d >> 1) ^ (d >> 4)) & 7; };
    // Keys that no query sees may hold anything: their values count as 0 (whatever the code, 2^-127 of it is
    // 0 as a 16-bit float). So does what was read of a key past `dim`.
    auto clear = [&](int step, int pids) {
        if (__builtin_expect(D == DP && step * kStep >= tlo && step * kStep + kStep <= thi && on_pages(pids), 1)) return;
        const bool there = __builtin_amdgcn_readlane(pids, wave * 16) >= 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) vse[i] &= uint32_t(there ? key_mask(step * kStep + wave * 16 + 4 * quad, tlo, thi) : 0);
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            if (kdim + i * 8 >= D) kraw[i] = 0;
    };
    auto note_nans = [&](int step, int buf) {
        if (!mixed(step)) return;
        uint32_t nan = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) nan |= nan_scales(vse[i]);
        nans[buf][wave] = __any(nan != 0);
    };
    // Part u of what fetch() read, to LDS: 8 dimensions of a key, or 2 of 4 tokens' values, turned
    // around. A part's place differs from the first one's in bits that are 0 there or are exclusive-ored by the
    // order; it is formed anew each time, since registers are short.
    constexpr int kParts = kWords * 2;
    int kput = (wave * 16 + kkey) * DP * 2 + ((quarter * kWords) ^ order(kkey)) * 16;
    int vput = kKeys + vgroup * (DP == 64 ? 4 : 8) * 128 + ((wave * 2 + (quad >> 1)) ^ vorder(vgroup * (DP == 64 ? 4 : 8))) * 16 + (quad & 1) * 8;
    auto put = [&](auto part, int buf) {
        constexpr int u = decltype(part)::value;
        constexpr int c = u / 2;
        if constexpr (u % 2 == 0) {
            *reinterpret_cast<v8 *>(lds[buf] + (kput ^ c * 16)) = operand4<T>(kraw[c], scale4(kse[c * NS / kWords]));
        } else {
            constexpr int i = DP == 256 ? c / 4 : 0, sel = c % 4;
            uint32_t x[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t w = uint32_t(vraw[i][t]);
                const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(DP == 64 ? w >> (16 * (vgroup & 1)) : w, scale_of(vse[i], t), sel);
                x[t] = __builtin_bit_cast(uint32_t, y);
            }
            uint8_t *const to = lds[buf] + ((vput ^ sel * 16) + (i * 128 + sel * 2) * 128);
            *reinterpret_cast<i32x2 *>(to) = i32x2{int(__builtin_amdgcn_perm(x[1], x[0], 0x05040100u)), int(__builtin_amdgcn_perm(x[3], x[2], 0x05040100u))};
            *reinterpret_cast<i32x2 *>(to + 128) = i32x2{int(__builtin_amdgcn_perm(x[1], x[0], 0x07060302u)), int(__builtin_amdgcn_perm(x[3], x[2], 0x07060302u))};
        }
    };
    // Pages of this step and the next, and the table's entry of the one after.
    int pid0 = -1, pid1 = -1, next = -1;
    if (from < to) {
        pid1 = on_page(entry(from));
        fetch(from, pid1);
        next = entry(from + 1);
        clear(from, pid1);
        note_nans(from, 0);
        unroll<0, kParts>([&](auto u) { put(u, 0); });
        pid0 = pid1;
        pid1 = on_page(next);
        next = entry(from + 2);
        fetch(from + 1, pid1);
    }
    // A step mixes what does not depend on each other, product by product (each is issued in
    // a few clocks and takes 32): into the first products the transfer of the next step's keys
    // to LDS, into the second ones the weights that the products after them need. What they
    // read from LDS is read four products ahead (eight: 249 us for 246, heads of 256 269 for 230: registers).
    // A wave goes first while it has its first products, so that the two of a SIMD come to do different
    // things (246 us, without 261).
    constexpr int kFirst = 2 * QC, kSecond = 4 * DT, kAhead = 4;
    const int krow = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);     // row r's key in tile 0
    auto body = [&](int step, auto which_buf) {
        constexpr int buf = decltype(which_buf)::value;
        const int base = step * kStep;
        asm("" : "+v"(kput), "+v"(vput));
        wait_lds();
        barrier();
        const uint8_t *const kt = lds[buf] + krow * DP * 2, *const vt = lds[buf] + kKeys + r * 128;
        auto key_part = [&](int n) { return *reinterpret_cast<const v8 *>(kt + (n % 2) * 32 * DP * 2 + ((n / 2 * 2 + hf) ^ order(krow)) * 16); };
        auto value_part = [&](int n) {
            return *reinterpret_cast<const f16x8 *>(vt + n % DT * 32 * 128 + ((n / DT * 2 + hf) ^ vorder(n % DT * 32 + r)) * 16);
        };
        if (mixed(step)) {
            int nan = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) nan |= nans[buf][w];
            if (__builtin_amdgcn_readfirstlane(nan)) {      // the same in every wave
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    f32x16 n{};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const bool there = __builtin_amdgcn_readlane(pid0, q * 16) >= 0;
                        const f16x8 v = value_part(q * DT + d);
                        f16x8 where, seen;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int key = base + q * 16 + hf * 8 + i;
                            where[i] = _Float16(v[i] != v[i] ? 1.f : 0.f);
                            seen[i] = _Float16(there && key >= low && key < high ? 1.f : 0.f);
                        }
                        n = mma32(where, seen, n);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] += n[i] > 0.f ? __builtin_nanf("") : 0.f;
                    __builtin_amdgcn_sched_barrier(0);
                }
                wait_lds();
                barrier();
                for (int i = int(threadIdx.x); i < kKeys / 16; i += 64 * kWaves) {
                    f16x8 *const at = reinterpret_cast<f16x8 *>(lds[buf] + kKeys + i * 16);
                    f16x8 v = *at;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = v[e] != v[e] ? _Float16(0.f) : v[e];
                    *at = v;
                }
                wait_lds();
                barrier();
            }
        }
        v8 kf[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) kf[n] = key_part(n);
        const bool held = on_pages(pid0);
        const int now = pid0;
        if (step + 1 < to) {
            clear(step + 1, pid1);
            note_nans(step + 1, buf ^ 1);
        }
        f32x16 s[2];
        __builtin_amdgcn_s_setprio(1);
        unroll<0, kFirst>([&](auto nth) {
            constexpr int n = decltype(nth)::value;
            s[n % 2] = mma32(kf[n % kAhead], qf[n / 2], n < 2 ? f32x16{} : s[n % 2]);
            if constexpr (n + kAhead < kFirst) kf[n % kAhead] = key_part(n + kAhead);
            unroll<n * kParts / kFirst, (n + 1) * kParts / kFirst>([&](auto u) { put(u, buf ^ 1); });
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
        f16x8 vf[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) vf[n] = value_part(n);
        pid0 = pid1;
        if (step + 1 < to) {
            pid1 = on_page(next);
            next = entry(step + 3);
            fetch(step + 2, pid1);
        }
        // Element i of s[t]: key 16 (2 t + i / 8) + 8 hf + i % 8.
        if (!held || !__all(base >= low && base + kStep <= high)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool there = __builtin_amdgcn_readlane(now, q * 16) >= 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = base + q * 16 + hf * 8 + i;
                    float &v = reinterpret_cast<float *>(&s[q >> 1])[(q & 1) * 8 + i];
                    v = there && key >= low && key < high ? v : -__builtin_inff();
                }
            }
        }
        float top = -__builtin_inff();
        const float sub = or_zero(m);
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i / 16][i % 16] = fmaf(s[i / 16][i % 16], p.scale, -sub);
#pragma unroll
        for (int i = 0; i < 32; i += 2) top = fmaxf(top, fmaxf(s[i / 16][i % 16], s[i / 16][i % 16 + 1]));
        raise(m, l, max_over_32(top),
              [&](float by) {
#pragma unroll
                  for (int i = 0; i < 32; ++i) s[i / 16][i % 16] -= by;
              },
              [&](float alpha) {
#pragma unroll
                  for (int d = 0; d < DT; ++d) acc[d] *= alpha;
              });
        f16x8 pf[4];
        float sum[4] = {};
        auto weigh = [&](int q, int i) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float e = __builtin_amdgcn_exp2f(s[q >> 1][(q & 1) * 8 + i + k]);
                sum[q] += e;
                pf[q][i + k] = _Float16(e);
            }
        };
#pragma unroll
        for (int i = 0; i < 8; i += 2) weigh(0, i);
#pragma unroll
        for (int n = 0; n < kSecond; ++n) {
            const int q = n / DT, d = n % DT;
            acc[d] = mma32(vf[n % kAhead], pf[q], acc[d]);
            if (n + kAhead < kSecond) vf[n % kAhead] = value_part(n + kAhead);
            if (q < 3) {
#pragma unroll
                for (int i = d * 4 / DT * 2; i < (d + 1) * 4 / DT * 2; i += 2) weigh(q + 1, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    for (int step = from; step < to; step += 2) {
        body(step, std::integral_constant<int, 0>{});
        if (step + 1 < to) body(step + 1, std::integral_constant<int, 1>{});
    }
    l += __shfl_xor(l, 32);
    if (row >= p.rows) return;
    if (!live || high == 0) {
        m = -__builtin_inff();
        l = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f32x16{};
    }
    float *part = p.part ? p.part + ((int64_t(bh) * p.rows + row) * p.splits + split) * (D + 2) : nullptr;
    if (part && hf == 0) {
        part[D] = m;
        part[D + 1] = l;
    }
    const float inv = inverse(l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int at = d * 32 + w * 8 + hf * 4;
            if (at < D) store_row<T>(p, b, h, row, part, at, f32x4{acc[d][4 * w], acc[d][4 * w + 1], acc[d][4 * w + 2], acc[d][4 * w + 3]}, inv);
        }
}

// The splits of a row together, in one trip: a block of 4 waves per row, LANES lanes (4 dimensions each) per split,
// which keep a running maximum, and the groups' sums together in LDS. 64 splits of 32 rows 3.4 us behind the launch that
// writes them (4.1 where the maximum is looked for first; 4 of 1536 rows 3.4 and 4.7). A split without keys has no results, only its
// maximum of -inf.
template <typename T, int LANES>
__global__ void __launch_bounds__(256)
attention4_join_kernel(const AttentionParams p)
{
    constexpr int kAtOnce = 256 / LANES;
    __shared__ float ml[2][kAtOnce];
    __shared__ f32x4 sums[256];
    const int64_t at = blockIdx.x;
    const int D = p.dim, lane = int(threadIdx.x % LANES), mine = int(threadIdx.x) / LANES, d = min(lane * 4, D - 4);
    const float *const part = p.part + at * p.splits * (D + 2);
    float m = -__builtin_inff(), l = 0.f;
    f32x4 o{};
#pragma unroll 4
    for (int s = mine; s < p.splits; s += kAtOnce) {
        const float *const from = part + s * (D + 2);
        const float sm = from[D], sl = from[D + 1];
        f32x4 x;
        __builtin_memcpy(&x, from + d, 16);
        const float top = fmaxf(m, sm), sub = or_zero(top), a = __builtin_amdgcn_exp2f(m - sub), b = __builtin_amdgcn_exp2f(sm - sub);
        m = top;
        l = fmaf(l, a, sl * b);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], a, sm == -__builtin_inff() ? 0.f : x[i] * b);
    }
    if (lane == 0) {
        ml[0][mine] = m;
        ml[1][mine] = l;
    }
    sums[threadIdx.x] = o;
    __syncthreads();
    if (mine != 0 || lane * 4 >= D) return;
    float top = ml[0][0], total = 0.f;
#pragma unroll
    for (int i = 1; i < kAtOnce; ++i) top = fmaxf(top, ml[0][i]);
    const float sub = or_zero(top);
    f32x4 sum{};
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[0][i] - sub);
        total = fmaf(ml[1][i], f, total);
        sum += sums[i * LANES + lane] * f;
    }
    const int64_t bh = at / p.rows;
    store_row<T>(p, int(bh / p.heads), int(bh % p.heads), int(at - bh * p.rows), nullptr, lane * 4, sum, inverse(total));
}

// How a call is split: over the rows first, then over the keys until 512 blocks (two a CU, of heads above 128 in two rounds) have at
// least 8 steps of 64 keys each. Measured (8 heads of 128, 4 query heads each; us): one query over 131072 keys 34.7,
// with 768 blocks 36.9, with 1024 43; 16 x 1 over up to 8192 23.5, 22.7 and 28. Where sequences and heads alone
// make more than 256 blocks of few queries, whose lengths may differ, until 1536 have at least 16 steps each: 48 x 1 over
// up to 8192 55.5, until 512 60.4, with 8 splits each 70; 64 x 1 over up to 16000 131, 16 splits each 170. (Splits have the same
// number of steps, so that a sequence much longer than 63 others is what a call waits for.) Few queries whose
// splits would not give every CU a block have splits of 4 steps: 1 x 1 over 2000 8.7, of 8 10.1.
// (Lengths and windows are the device's: the splits go by the table's width. In a table for 131072 keys 1 x 1 over 2000 takes 11.9
// for 8.1, and with a window of 4096 over 131072 11.9 for the 8.2 of 4096 alone: few of the splits have keys then.)
// Up to 64 rows run attention4_few_kernel, from 17 on in blocks of 32 rows (of heads above 128: 16): 32 x 5 queries over
// up to 4000 keys 34.1, through LDS 63.8; 32 x 16 62.1 and 72.1, of heads of 256 (8 x 16) 53.5 and 63.8, of 64 58.6 and 65.0;
// 5 x 3 of 7 heads each 12.8 and 14.5; 1 x 16 over 8000 15.0 and 22.2. Above, 32 x 32 queries would take 105 for 84.
Plan plan_attention4(int64_t batch, int64_t tokens, int64_t heads, int64_t group, int64_t dim, int64_t columns, int64_t page)
{
    Plan a;
    a.rows = tokens * group;
    a.waves = a.rows <= 64 ? 0 : 4;
    const int tile = a.waves ? 32 * a.waves : dim <= 128 && a.rows > 16 ? 32 : 16;
    a.row_tiles = int((a.rows + tile - 1) / tile);
    const int64_t blocks = std::max<int64_t>(batch * heads * a.row_tiles, 1), steps = (columns * page + kStep - 1) / kStep;
    const bool uneven = a.waves == 0 && blocks > 256;
    a.least = uneven ? 16 : 8;
    const int64_t most = uneven ? (1535 + blocks) / blocks : a.waves ? 512 / blocks : (511 + blocks) / blocks;
    const auto split = [&] { a.splits = int(std::max<int64_t>(1, std::min<int64_t>({most, (steps + a.least - 1) / a.least, 256}))); };
    split();
    if (a.waves == 0 && a.splits > 1 && blocks * a.splits < 256) {
        a.least = 4;
        split();
    }
    return a;
}

template <typename T, int DP>
void run_attention4(const AttentionParams &p, const Plan &a, int64_t batch, hipStream_t s)
{
    const int bhs = int(batch * p.heads);
    const int blocks = int(blocks4(p.dim));
    if (a.waves == 0) {
        constexpr int most = DP <= 128 ? 2 : 1;
        hipLaunchKernelGGL((a.rows <= 16 ? attention4_few_kernel<T, DP, 1> : attention4_few_kernel<T, DP, most>), dim3(a.splits, bhs, a.row_tiles), dim3(256), 0, s, p, blocks);
    } else {
        const dim3 grid(uint32_t((int64_t(bhs) * a.row_tiles * a.splits + 7) / 8 * 8));
        hipLaunchKernelGGL((attention4_many_kernel<T, DP>), grid, dim3(64 * a.waves), 0, s, p, blocks, bhs);
    }
    if (a.splits > 1)
        hipLaunchKernelGGL((attention4_join_kernel<T, DP / 4>), dim3(uint32_t(bhs * a.rows)), dim3(256), 0, s, p);
}

template <typename T>
void run_attention4(const AttentionParams &p, const Plan &a, int64_t batch, hipStream_t s)
{
    if (p.dim <= 64) run_attention4<T, 64>(p, a, batch, s);
    else if (p.dim <= 128) run_attention4<T, 128>(p, a, batch, s);
    else run_attention4<T, 256>(p, a, batch, s);
}

int page_shift(int64_t page)
{
    int shift = 4;
    while ((int64_t(1) << shift) < page) ++shift;
    return shift;
}

// Whether a thread has 4 tokens, where that leaves work for the whole chip. Append and read of 4 x 2001 tokens (8 heads
// of 128, pages of 64) 20.2 us, with 1 24.4; 2000 (dim 80) 8.6 and 9.1; 64 x 4 5.9 and 5.4; 64 x 1 5.3 and 4.5; a read
// of 6 x 20000 116 and 183.
bool four_tokens(int64_t batch, int64_t tokens, int64_t heads, int64_t dim)
{
    return tokens > 1 && double(batch) * double(tokens) * double(heads) * double(dim) >= (1 << 20);
}

// What an append and a read have in common; bytes: those that k and v span.
ds_status cache_params(bool four, CacheParams &p, int64_t (&bytes)[2], const int32_t *table, const int32_t *start, const int32_t *count, int64_t batch,
                       int64_t tokens, int64_t heads, int64_t dim, int64_t page, int64_t pages, int64_t columns, int64_t ldt,
                       const int64_t *k_strides, const int64_t *v_strides, int64_t es)
{
    const int64_t lanes = blocks4(dim) * 4, shares = four ? (tokens + 2) / 4 + 1 : tokens;        // (a sequence's start is any)
    if (shares * heads > (kMaxElems - 255) / lanes) return fail(DS_ERR_UNSUPPORTED, "too many vectors of a sequence in one call");
    const int64_t per = (shares * heads * lanes + 255) / 256;
    if (!grid_fits(batch * per, 256)) return fail(DS_ERR_UNSUPPORTED, "too many vectors in one call");
    p = CacheParams{table, start, count, ldt, int(columns), int(pages), int(tokens), int(heads), int(dim), page_shift(page),
                    int(blocks4(dim)), int(per), make_fastdiv(uint32_t(lanes)), make_fastdiv(uint32_t(heads)), {}, {}, {}};
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? v_strides : k_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        p.sb[i] = s[0];
        p.st[i] = s[1];
        p.sh[i] = s[2];
        bytes[i] = span(batch, tokens, heads, s, dim, es);
    }
    return DS_SUCCESS;
}

// Cache and scale addresses for whole words.
ds_status check_aligned(const uint8_t *k_cache, const uint8_t *v_cache, const uint8_t *k_scales, const uint8_t *v_scales)
{
    for (const void *p : {k_cache, v_cache, k_scales, v_scales})
        if (reinterpret_cast<uintptr_t>(p) % 16) return fail(DS_ERR_INVALID_ARG, "a cache and its scales must begin on 16 bytes");
    return DS_SUCCESS;
}

}  // namespace

}  // namespace ds

using namespace ds;

extern "C" ds_status ds_kv_cache_fp4_append(const void *k, const void *v, uint8_t *k_cache, uint8_t *v_cache, uint8_t *k_scales,
                                            uint8_t *v_scales, const int32_t *table, const int32_t *start, const int32_t *count,
                                            int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int64_t page, int64_t pages,
                                            int64_t columns, int64_t ldt, const int64_t *k_strides, const int64_t *v_strides,
                                            int32_t type, void *stream)
{
    if (batch != 0 && tokens != 0 &&
        (!k || !v || !k_cache || !v_cache || !k_scales || !v_scales || !table || !start || !k_strides || !v_strides))
        return fail(DS_ERR_NULL_POINTER, "a required pointer is NULL");
    if (ds_status st = check_cache(batch, tokens, heads, dim, page, pages, columns, ldt)) return st;
    const int64_t es = float_bytes(type);
    if (!es) return fail(DS_ERR_INVALID_ARG, "type must be DS_TYPE_F32, DS_TYPE_F16 or DS_TYPE_BF16");
    if (batch == 0 || tokens == 0) return ok();
    if (ds_status st = check_aligned(k_cache, v_cache, k_scales, v_scales)) return st;
    const bool four = four_tokens(batch, tokens, heads, dim);
    CacheParams p;
    int64_t bytes[2];
    if (ds_status st = cache_params(four, p, bytes, table, start, count, batch, tokens, heads, dim, page, pages, columns, ldt, k_strides, v_strides, es))
        return st;
    const int64_t cb = pages * heads * page * dim / 2, sb = pages * heads * page * blocks4(dim);
    if (ds_status st = check_tensors({{k, bytes[0], "k", false}, {v, bytes[1], "v", false}, {table, span(batch, ldt, columns, 4), "table", false},
                                      {start, batch * 4, "start", false}, {count, batch * 4, "count", false},
                                      {k_cache, cb, "k_cache", true}, {v_cache, cb, "v_cache", true},
                                      {k_scales, sb, "k_scales", true}, {v_scales, sb, "v_scales", true}}))
        return st;
    const auto go = [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((four ? append4_kernel<T, 4> : append4_kernel<T, 1>), dim3(uint32_t(batch * p.per), 2), dim3(256), 0, static_cast<hipStream_t>(stream),
                           static_cast<const T *>(k), static_cast<const T *>(v), k_cache, v_cache, k_scales, v_scales, p);
    };
    if (type == DS_TYPE_F32) go(float{});
    else if (type == DS_TYPE_F16) go(_Float16{});
    else go(__bf16{});
    return launched("ds_kv_cache_fp4_append");
}

extern "C" ds_status ds_kv_cache_fp4_read(const uint8_t *k_cache, const uint8_t *v_cache, const uint8_t *k_scales, const uint8_t *v_scales,
                                          const int32_t *table, const int32_t *start, const int32_t *count, void *k, void *v,
                                          int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int64_t page, int64_t pages,
                                          int64_t columns, int64_t ldt, const int64_t *k_strides, const int64_t *v_strides,
                                          int32_t type, void *stream)
{
    if (batch != 0 && tokens != 0 &&
        (!k || !v || !k_cache || !v_cache || !k_scales || !v_scales || !table || !start || !k_strides || !v_strides))
        return fail(DS_ERR_NULL_POINTER, "a required pointer is NULL");
    if (ds_status st = check_cache(batch, tokens, heads, dim, page, pages, columns, ldt)) return st;
    const int64_t es = float_bytes(type);
    if (!es) return fail(DS_ERR_INVALID_ARG, "type must be DS_TYPE_F32, DS_TYPE_F16 or DS_TYPE_BF16");
    if (batch == 0 || tokens == 0) return ok();
    if (ds_status st = check_aligned(k_cache, v_cache, k_scales, v_scales)) return st;
    const bool four = four_tokens(batch, tokens, heads, dim);
    CacheParams p;
    int64_t bytes[2];
    if (ds_status st = cache_params(four, p, bytes, table, start, count, batch, tokens, heads, dim, page, pages, columns, ldt, k_strides, v_strides, es))
        return st;
    const int64_t cb = pages * heads * page * dim / 2, sb = pages * heads * page * blocks4(dim);
    if (ds_status st = check_tensors({{k_cache, cb, "k_cache", false}, {v_cache, cb, "v_cache", false}, {k_scales, sb, "k_scales", false},
                                      {v_scales, sb, "v_scales", false}, {table, span(batch, ldt, columns, 4), "table", false},
                                      {start, batch * 4, "start", false}, {count, batch * 4, "count", false},
                                      {k, bytes[0], "k", true}, {v, bytes[1], "v", true}}))
        return st;
    const auto go = [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((four ? read4_kernel<T, 4> : read4_kernel<T, 1>), dim3(uint32_t(batch * p.per), 2), dim3(256), 0, static_cast<hipStream_t>(stream),
                           static_cast<T *>(k), static_cast<T *>(v), k_cache, v_cache, k_scales, v_scales, p);
    };
    if (type == DS_TYPE_F32) go(float{});
    else if (type == DS_TYPE_F16) go(_Float16{});
    else go(__bf16{});
    return launched("ds_kv_cache_fp4_read");
}

extern "C" int64_t ds_attention_fp4_scratch_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t group, int64_t dim,
                                                  int64_t page, int64_t columns)
{
    if (batch <= 0 || tokens <= 0 || heads <= 0 || group <= 0 || dim <= 0 || page <= 0 || columns <= 0) return 0;
    return 4 * part_floats(plan_attention4(batch, tokens, heads, group, dim, columns, page), batch, heads, dim);
}

extern "C" ds_status ds_attention_fp4(const void *q, const uint8_t *k_cache, const uint8_t *v_cache, const uint8_t *k_scales,
                                      const uint8_t *v_scales, const int32_t *table, const int32_t *length,
                                      const int32_t *count, void *o, int64_t batch, int64_t tokens, int64_t heads,
                                      int64_t group, int64_t dim, int64_t page, int64_t pages, int64_t columns, int64_t ldt,
                                      const int64_t *q_strides, const int64_t *o_strides, float scale, int64_t window,
                                      int32_t type, void *scratch, int64_t scratch_bytes, void *stream)
{
    if (batch != 0 && tokens != 0 &&
        (!q || !k_cache || !v_cache || !k_scales || !v_scales || !table || !length || !o || !q_strides || !o_strides))
        return fail(DS_ERR_NULL_POINTER, "a required pointer is NULL");
    if (ds_status st = check_cache(batch, tokens, heads, dim, page, pages, columns, ldt)) return st;
    if (group <= 0) return fail(DS_ERR_INVALID_SHAPE, "group must be > 0");
    if (type != DS_TYPE_F16 && type != DS_TYPE_BF16) return fail(DS_ERR_INVALID_ARG, "type must be DS_TYPE_F16 or DS_TYPE_BF16");
    if (window < 0 || window > kMaxElems) return fail(DS_ERR_INVALID_ARG, "window must be in [0, 2^31)");
    if (!std::isfinite(scale)) return fail(DS_ERR_INVALID_ARG, "scale must be finite");
    if (batch == 0 || tokens == 0) return ok();
    if (ds_status st = check_aligned(k_cache, v_cache, k_scales, v_scales)) return st;
    if (batch * heads > 65535) return fail(DS_ERR_UNSUPPORTED, "more than 65535 sequences times heads");
    if (group > 65535 || tokens * group > kMaxElems / 64) return fail(DS_ERR_UNSUPPORTED, "too many queries of a head");
    const Plan a = plan_attention4(batch, tokens, heads, group, dim, columns, page);
    if (batch * heads * a.rows * a.splits > kMaxElems / 2) return fail(DS_ERR_UNSUPPORTED, "too many queries");
    int64_t bytes[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? o_strides : q_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        bytes[i] = span(batch, tokens, heads * group, s, dim, 2);
    }
    const int64_t cb = pages * heads * page * dim / 2, sb = pages * heads * page * blocks4(dim), need = 4 * part_floats(a, batch, heads, dim);
    if (need > 0 && !scratch) return fail(DS_ERR_NULL_POINTER, "scratch must not be NULL");
    if (need > scratch_bytes) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    if (ds_status st = check_tensors({{q, bytes[0], "q", false}, {k_cache, cb, "k_cache", false}, {v_cache, cb, "v_cache", false},
                                      {k_scales, sb, "k_scales", false}, {v_scales, sb, "v_scales", false},
                                      {table, span(batch, ldt, columns, 4), "table", false}, {length, batch * 4, "length", false},
                                      {count, batch * 4, "count", false}, {o, bytes[1], "o", true},
                                      {need ? scratch : nullptr, need, "scratch", true}}))
        return st;
    // (The factor is above 0: a key that is not seen has -inf, which stays that.)
    const AttentionParams p{q, k_cache, v_cache, k_scales, v_scales, table, length, count, o,
                            need ? static_cast<float *>(scratch) : nullptr, ldt, q_strides[0], q_strides[1], q_strides[2],
                            o_strides[0], o_strides[1], o_strides[2], int(columns), int(pages), int(tokens), int(heads),
                            int(group), int(dim), page_shift(page), int(window), a.splits, int(a.rows), a.row_tiles,
                            std::max(std::fabs(scale) * 1.44269504f, 0x1p-126f), scale < 0, a.least};
    const auto s = static_cast<hipStream_t>(stream);
    if (type == DS_TYPE_F16) run_attention4<_Float16>(p, a, batch, s);
    else run_attention4<__bf16>(p, a, batch, s);
    return launched("ds_attention_fp4");
}
