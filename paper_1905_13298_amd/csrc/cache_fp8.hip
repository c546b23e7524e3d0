// A paged cache of keys and values in 8 bits, and the attention that reads it.
//
// Layout: keys [page][head][token][dim], values [page][head][dim][token] (the order in
// which the second product of an attention contracts them), both E4M3, with one E8M0
// scale for each page and head. A sequence's pages are listed in a row of a table.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention.hpp"
#include "conv_plan.hpp"
#include "fastdiv.hpp"

namespace ds {

namespace {

// Scales of a cache lie in 2^-48 .. 2^48: the attention adds terms of pages with
// different scales in one sum, and within these bounds no term that counts can leave
// the range of its 32-bit numbers.
constexpr int kCacheLow = 127 - 48, kCacheHigh = 127 + 48;

struct AppendParams {
    const int *table, *start, *count;
    int64_t ldt;
    int columns, pages, tokens, heads, dim, page;
    FastDiv vecs;                      // of a token's vector, 8 elements each
    int64_t sb[2], st[2], sh[2];       // strides of k and v: sequence, token, head
};

// One page's new tokens of one head: its scale, the rounding of what it holds already
// to a larger scale, and the tokens. Every (page, head) is one block's alone. A thread keeps
// its first HELD vectors of 8 elements from the search for the scale (of 8 a page of 128 x 128
// or 64 x 256 elements; 4 or 1 where that is all, for more blocks a CU: 16 x 2001 tokens, 8 heads
// of 128, pages of 32 take 48 us with 4, 62 with 8, 51 with 1; single tokens 5.4 with 1, 5.9 with 8);
// values go through LDS, where they change from tokens to dimensions. Bound by bandwidth: 4 x 2001 tokens
// in 16 bits, 49 MB, 14.2 us (3.5 TB/s, the launch's 2 us among them).
template <typename T, int HELD>
__global__ void __launch_bounds__(256)
append_kernel(const T *__restrict__ k, const T *__restrict__ v, uint8_t *__restrict__ kc, uint8_t *__restrict__ vc,
              uint8_t *__restrict__ ks, uint8_t *__restrict__ vs, const AppendParams p, int touched)
{
    __shared__ float red[4];
    extern __shared__ __align__(16) uint8_t tile[];       // values: [token, from a multiple of 8 on][dim + 4]
    const int b = int(blockIdx.x) / touched, j = int(blockIdx.x) - b * touched, h = int(blockIdx.y), which = int(blockIdx.z);
    const int start = p.start[b], n = p.count ? min(p.count[b], p.tokens) : p.tokens;
    if (start < 0 || n <= 0) return;
    const int col = start / p.page + j;
    const int64_t c0 = int64_t(col) * p.page;
    const int lo = int(max(int64_t(start), c0) - c0), hi = int(min(int64_t(start) + n, c0 + p.page) - c0);
    if (hi <= lo || col >= p.columns) return;
    const int pid = p.table[b * p.ldt + col];
    if (pid < 0 || pid >= p.pages) return;
    const T *src = (which ? v : k) + b * p.sb[which] + (c0 + lo - start) * p.st[which] + h * p.sh[which];
    const int64_t st = p.st[which], at = int64_t(pid) * p.heads + h;
    uint8_t *cache = (which ? vc : kc) + at * p.page * p.dim, *scale = (which ? vs : ks) + at;
    const int D = p.dim, vecs = D / 8, total = (hi - lo) * vecs;
    const int before = min(max(int(*scale), kCacheLow), kCacheHigh);
    Eight<T> held[HELD];
    auto load = [&](int i) {
        Eight<T> x;
        const int tok = fdiv(i, p.vecs);
        x.template load<true>(src + tok * st, uint32_t(i - tok * vecs) * 8, 8);
        return x;
    };
    float amax = 0.f;
    auto look = [&](const Eight<T> &x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(x.at(e)));
    };
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (int(threadIdx.x) + q * 256 < total) held[q] = load(int(threadIdx.x) + q * 256);
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (int(threadIdx.x) + q * 256 < total) look(held[q]);
    for (int i = int(threadIdx.x) + HELD * 256; i < total; i += 256) look(load(i));
    amax = lanes_max<64>(amax);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    int e = amax == 0.f ? kCacheLow : min(max(scale_byte(amax), kCacheLow), kCacheHigh);
    if (lo > 0) e = max(e, before);
    const float s = power_of_two(254 - e);
    if (lo > 0 && e != before) {
        // What the page holds moves to the larger scale: tokens 0 .. lo - 1.
        const float f = power_of_two(uint32_t(127 + before - e));
        for (int i = threadIdx.x; i < lo * D; i += 256) {
            const int tok = which ? i % lo : i / D, d = which ? i / lo : i % D;
            uint8_t *q = cache + (which ? d * p.page + tok : tok * D + d);
            *q = uint8_t(to_fp8x4(__builtin_amdgcn_cvt_f32_fp8(int(*q), 0) * f, 0.f, 0.f, 0.f));
        }
    }
    // A finite element beyond the largest scale's range is held as the largest number.
    auto fit = [&](float x) { return fabsf(x) < __builtin_inff() ? fminf(fmaxf(x * s, -448.f), 448.f) : __builtin_nanf(""); };
    const int pitch = D + 4, skew = lo & 7;
    auto put = [&](int i, const Eight<T> &x) {
        const int tok = fdiv(i, p.vecs), d = (i - tok * vecs) * 8;
        i32x2 q;
        q[0] = to_fp8x4(fit(x.at(0)), fit(x.at(1)), fit(x.at(2)), fit(x.at(3)));
        q[1] = to_fp8x4(fit(x.at(4)), fit(x.at(5)), fit(x.at(6)), fit(x.at(7)));
        if (which) {
            *reinterpret_cast<int *>(tile + (skew + tok) * pitch + d) = q[0];
            *reinterpret_cast<int *>(tile + (skew + tok) * pitch + d + 4) = q[1];
        } else {
            *reinterpret_cast<i32x2 *>(cache + (lo + tok) * D + d) = q;
        }
    };
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (int(threadIdx.x) + q * 256 < total) put(int(threadIdx.x) + q * 256, held[q]);
    for (int i = int(threadIdx.x) + HELD * 256; i < total; i += 256) put(i, load(i));
    if (threadIdx.x == 0) *scale = uint8_t(e);
    if (!which) return;
    __syncthreads();
    // Eight tokens (an eighth's: what lies before lo or from hi on is not written) of four
    // dimensions a thread.
    const int first = lo / 8, eighths = (hi + 7) / 8 - first;
    for (int i = threadIdx.x; i < eighths * (D / 4); i += 256) {
        const int dg = i / eighths, t = i - dg * eighths, from = (first + t) * 8;
        uint32_t in[8];
        uint64_t out[4];
#pragma unroll
        for (int q = 0; q < 8; ++q) in[q] = *reinterpret_cast<const uint32_t *>(tile + (t * 8 + q) * pitch + dg * 4);
        turn(in, out);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint8_t *o = cache + (dg * 4 + q) * p.page + from;
            if (from >= lo && from + 8 <= hi) {
                *reinterpret_cast<uint64_t *>(o) = out[q];
            } else {
                for (int x = max(lo - from, 0); x < min(hi - from, 8); ++x) o[x] = uint8_t(out[q] >> (8 * x));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Attention. A kv head's queries are its `rows` = tokens x group vectors, and a wave
// handles 16 of them at a time with 64 keys:
//
//   S^T = K Q^T (the matrix instruction's rows are keys, its columns queries), so that a
//   lane holds 16 consecutive keys of one query;
//   t = S * 2^ek * scale * log2(e) + log2(2^ev): the value scale ev of the keys' page goes
//   into the exponent, so that p = 2^(t - m) weighs the 8-bit values themselves; m is such that
//   the largest p of a row is from 2^9 to 2^15;
//   O^T += V^T P (rows: dimensions, columns: queries), l += p * 2^-ev.
//
// The two layouts agree, so that p goes from the first product to the second in place:
// the key of row r of a 16-key tile t is chosen as (r / 4) * 16 + t * 4 + r % 4, which
// leaves lane group g (lane / 16) with keys 16 g .. 16 g + 15, and those are the ones that
// it contracts in the second product, 8 at a time. Keys become numbers of the queries'
// type exactly; p and the values are 16-bit floats with 10 bits of mantissa: values exactly, p
// rounded once, to 2^-11 of itself down to 2^-23 of the row's largest and to 2^-34 of that one
// below (l has all of it in 32 bits). The largest is of t, thus of weights times their page's value
// scale: where pages' scales are 2^d apart, weights on the smaller one keep their bits down to
// 2^(d - 23) of the largest, and what 10^4 of them lose below that is less than the larger page's
// values were rounded by when they became 8 bits (unless those are exactly 0).

template <typename T>
__device__ __forceinline__ typename Vec8<T>::type widen(int lo, int hi)
{
    if constexpr (sizeof(T) == 2 && __is_same(T, _Float16)) {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
        return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
}

// The factors of a page's scales: of its keys' products (times the softmax scale, > 0), the
// logarithm of its values', and one over that.
struct PageScale {
    float sk, lv, iv;
};

__device__ __forceinline__ PageScale page_scale(int ek, int ev, float scale)
{
    ek = min(max(ek, kCacheLow), kCacheHigh);
    ev = min(max(ev, kCacheLow), kCacheHigh);
    return PageScale{fmaxf(power_of_two(uint32_t(ek)) * scale, 0x1p-126f), float(ev - 127), power_of_two(uint32_t(254 - ev))};
}

// The weights of 64 keys for one query a lane (16 of the keys in this lane): s holds the
// products, key `run` + i in [low, high) counts.
template <typename Rescale>
__device__ __forceinline__ void weights(f32x4 (&s)[4], float &m, float &l, const PageScale &ps, bool page, int run, int low, int high,
                                        f16x8 (&pf)[2], Rescale &&rescale)
{
    if (!__all(page && run >= low && run + 16 <= high)) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            s[i >> 2][i & 3] = page && run + i >= low && run + i < high ? s[i >> 2][i & 3] : -__builtin_inff();
    }
    const float off = ps.lv - or_zero(m);
    float e[16], top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = fmaf(s[i >> 2][i & 3], ps.sk, off);
#pragma unroll
    for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(e[i], e[i + 1]));
    raise(m, l, max_over_32(max_over_16(top)),
          [&](float by) {
#pragma unroll
              for (int i = 0; i < 16; ++i) e[i] -= by;
          },
          rescale);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        e[i] = __builtin_amdgcn_exp2f(e[i]);
        sum += e[i];
        pf[i >> 3][i & 7] = _Float16(e[i]);
    }
    l = fmaf(sum, ps.iv, l);
}

// 0x80 in each byte of x that is an E4M3 NaN. A weight of 0 does not keep a NaN out of a sum: where
// some queries see a step's keys and others do not, values that are NaN are taken out, and come back
// as NaN in the results of the queries that see them (a product of where they are with what is seen).
__device__ __forceinline__ uint32_t nan_bytes(int x) { return ((uint32_t(x) & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Up to 16 queries of a kv head (tokens being decoded): a block of 4 waves takes a share of
// the keys, each wave every fourth 64 of it straight from memory to registers (no two waves
// share any, so LDS would only add a trip), and joins them at its end. Bound by reading the
// cache once: 131072 keys of 8 heads of 128, 268 MB, 57 us with the join (4.7 TB/s). ONE: of one token,
// whose query heads all see the same keys (16 x 1 over up to 8192: 40.5 us, with the code for values
// that are NaN 41.3).
template <typename T, int DP, bool ONE>
__global__ void __launch_bounds__(256)
attention_few_kernel(const AttentionParams p)
{
    constexpr int kWaves = 4;
    constexpr int QC = DP / 32;            // chunks of 32 of the first product's contraction
    constexpr int KB = DP / 64;            // 16-byte loads of a lane's part of a key
    constexpr int DT = DP / 16;            // tiles of 16 dimensions of the second product
    typedef typename Vec8<T>::type v8;
    __shared__ float ml[2][kWaves][16];
    __shared__ f32x4 osum[kWaves][DT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const int split = int(blockIdx.x), bh = int(blockIdx.y), b = bh / p.heads, h = bh - b * p.heads;
    const int D = p.dim, page = 1 << p.page_shift;
    const Sequence seq(p, b);
    v8 qf[QC];
    int low, high;
    load_query<T, DP, 8, DP / 4, QC>(p, seq, b, h, r, g, low, high, qf);
    int tlo = high > 0 ? low : 0x7fffffff, thi = high;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
        tlo = min(tlo, __shfl_xor(tlo, o));
        thi = max(thi, __shfl_xor(thi, o));
    }
    tlo = __builtin_amdgcn_readfirstlane(tlo);
    thi = __builtin_amdgcn_readfirstlane(thi);
    // Keys that some query sees: [tlo, thi), others are masked in the values themselves; that every one
    // sees: [alo, ahi).
    const int alo = p.window ? max(max(seq.first + seq.count, 0) - p.window, 0) : 0, ahi = min(max(seq.first + 1, 0), seq.keys);
    const int s0 = thi > 0 ? tlo / kStep : 0, s1 = (thi + kStep - 1) / kStep;
    const int each = (s1 - s0 + p.splits - 1) / p.splits;
    const int from = s0 + split * each, to = min(s1, from + each);

    f32x4 acc[DT];
    float m = -__builtin_inff(), l = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
    // Page of the 16 keys from `key` on (they share it), or -1 where there is none.
    auto page_of = [&](int key) {
        const int col = key >> p.page_shift;
        const int pid = key < thi ? p.table[b * p.ldt + col] : -1;
        return unsigned(pid) < unsigned(p.pages) ? pid : -1;
    };
    int kp = page_of((from + wave) * kStep + (r >> 2) * 16), vp = page_of((from + wave) * kStep + g * 16);
    for (int step = from + wave; step < to; step += kWaves) {
        const int base = step * kStep;
        const int krun = base + (r >> 2) * 16, vrun = base + g * 16;
        const int64_t kat = (int64_t(max(kp, 0)) * p.heads + h) * page, vat = int64_t(max(vp, 0)) * p.heads + h;
        const uint8_t *krow = p.kc + (kat + (krun & (page - 1)) + (r & 3)) * D;
        const uint8_t *vrow = p.vc + (vat * D + r) * page + (vrun & (page - 1));
        i32x4 kraw[4][KB], vraw[DT];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                const int d = g * (DP / 4) + i * 16;
                kraw[t][i] = kp >= 0 && d < D ? *reinterpret_cast<const i32x4 *>(krow + t * 4 * D + d) : i32x4{};
            }
        const int ek = p.ks[vat], ev = p.vs[vat];
#pragma unroll
        for (int d = 0; d < DT; ++d)
            vraw[d] = vp >= 0 && d * 16 < D ? *reinterpret_cast<const i32x4 *>(vrow + d * 16 * page) : i32x4{};
        const bool held = vp >= 0;
        kp = page_of(krun + kWaves * kStep);
        vp = page_of(vrun + kWaves * kStep);
        f32x4 s[4];
#pragma unroll
        for (int c = 0; c < QC; ++c)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                s[t] = mma(widen<T>(kraw[t][c >> 1][(c & 1) * 2], kraw[t][c >> 1][(c & 1) * 2 + 1]), qf[c], c == 0 ? f32x4{} : s[t]);
        const PageScale ps = page_scale(ek, ev, p.scale);
        f16x8 pf[2];
        weights(s, m, l, ps, held, vrun, low, high, pf, [&](float alpha) {
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= alpha;
        });
        if (base + kStep > thi || base < tlo) {
            // Keys that no query sees may hold anything: their values count as 0.
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int mask = key_mask(vrun + 4 * w, tlo, thi);
#pragma unroll
                for (int d = 0; d < DT; ++d) vraw[d][w] &= mask;
            }
        }
        if (!ONE && (base + kStep > ahi || base < alo)) {
            uint32_t nan = 0;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int w = 0; w < 4; ++w) nan |= nan_bytes(vraw[d][w]);
            if (__any(nan != 0)) {
                f16x8 seen[2];
#pragma unroll
                for (int i = 0; i < 16; ++i) seen[i >> 3][i & 7] = _Float16(held && vrun + i >= low && vrun + i < high ? 1.f : 0.f);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    i32x4 where;                  // 1 for NaN
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        asm("" : "+v"(vraw[d][w]));     // (not kept from above: registers)
                        const uint32_t z = nan_bytes(vraw[d][w]) >> 7;
                        where[w] = int(z * 0x38u);
                        vraw[d][w] &= int(~(z * 0xffu));
                    }
                    f32x4 n{};
#pragma unroll
                    for (int c = 0; c < 2; ++c) n = mma(widen<_Float16>(where[2 * c], where[2 * c + 1]), seen[c], n);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[d][i] += n[i] > 0.f ? __builtin_nanf("") : 0.f;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = mma(widen<_Float16>(vraw[d][2 * c], vraw[d][2 * c + 1]), pf[c], acc[d]);
    }
    if (high == 0) {      // a row that sees no key, whatever the others see
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
    }
    // The waves' sums together: a lane's l is its own keys'.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        ml[0][wave][r] = m;
        ml[1][wave][r] = l;
    }
    __syncthreads();
    float top = ml[0][0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[0][w][r]);
    const float sub = or_zero(top), mine = __builtin_amdgcn_exp2f(m - sub);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total = fmaf(ml[1][w][r], __builtin_amdgcn_exp2f(ml[0][w][r] - sub), total);
#pragma unroll
    for (int d = 0; d < DT; ++d) osum[wave][d][lane] = acc[d] * mine;
    __syncthreads();
    if (r >= p.rows) return;
    float *part = p.part ? p.part + ((int64_t(bh) * p.rows + r) * p.splits + split) * (D + 2) : nullptr;
    if (part && wave == 0 && g == 0) {
        part[D] = top;
        part[D + 1] = total;
    }
    const float inv = inverse(total);
    for (int d = wave; d < DT; d += kWaves) {
        if (d * 16 >= D) continue;
        f32x4 o = osum[0][d][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) o += osum[w][d][lane];
        store_row<T>(p, b, h, r, part, d * 16 + g * 4, o, inv);
    }
}

// Many queries of a kv head: a block's waves have 32 of them each and share the keys, 64 at a
// time. A wave reads its part of them a step ahead, turns them into 16-bit floats, once for
// the whole block, and puts them into LDS: keys as rows [key][dim], values as rows [dim][key],
// the 16-byte pieces of a row in an order of its own, so that the lanes of a read (0-3, 12-15,
// 20-27 at once, and so on) meet in no bank.
//
// The products are 32 x 32: one query a lane and 32 keys of it, 8 of each 16, and twice the
// work an instruction, which one wave can issue without a pause (it issues at most one 16 x 16
// x 32 in 32 clocks where two waves reach one in 16). Row 8 w + 4 hf + e of tile tt is key
// 32 tt + 16 (w / 2) + 8 hf + 4 (w % 2) + e: lane half hf then holds the keys that it
// contracts in the second product.
//
// Bound by the matrix instructions and the exponentials between them, which do not overlap in one
// wave: 2 x 1000 queries of 32 heads over up to 8000 keys of 8 heads of 128 take 254 to 270 us, pages
// of 16 tokens as long as those of 64 (the products alone take 203 us at the rate of a large 16-bit
// product).
template <typename T, int DP, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, DP <= 128 ? 2 : 1)
attention_many_kernel(const AttentionParams p, int bhs)
{
    constexpr int QC = DP / 16, DT = DP / 32, kLoads = DP / 64, kRuns = 4 / WAVES, kScales = 4;
    constexpr int kKeys = kStep * DP * 2;      // bytes of a step's keys, or values
    typedef typename Vec8<T>::type v8;
    __shared__ __align__(16) uint8_t lds[2][2 * kKeys];
    __shared__ int nans[2][WAVES];             // whether a wave's part of the values has any
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 31, hf = lane >> 5, g = lane >> 4;
    // An eighth of the work to each XCD, a head's blocks together, so that they read its
    // keys through one L2, the same head of every sequence next, whose lengths may differ; the
    // last rows, which see the most keys, first.
    const int per = p.row_tiles * p.splits, blocks = bhs * per, share = (blocks + 7) >> 3;
    const int at = (int(blockIdx.x) & 7) * share + (int(blockIdx.x) >> 3);
    if ((int(blockIdx.x) >> 3) >= share || at >= blocks) return;
    const int unit = at / per, rest = at - unit * per, tile = p.row_tiles - 1 - rest / p.splits, split = rest % p.splits;
    const int batch = bhs / p.heads, h = unit / batch, b = unit - h * batch, bh = b * p.heads + h;
    const int D = p.dim, page = 1 << p.page_shift;
    const Sequence seq(p, b);
    v8 qf[QC];
    int low, high;
    const int row = (tile * WAVES + wave) * 32 + r;
    const bool live = load_query<T, DP, 16, 8, QC>(p, seq, b, h, row, hf, low, high, qf);
    // A row without a query sees every key, which costs less than no key, and is 0 in the end.
    if (!live) high = 0x7fffffff;
    // The block's keys: from the first that its first query sees to its last query's own.
    const int t0 = tile * WAVES * 32 / p.group, t1 = min(((tile + 1) * WAVES * 32 - 1) / p.group, seq.count - 1);
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
    i32x4 kraw[kRuns][kLoads], vraw[kRuns][kLoads];
    // This wave's runs of 16 keys of a step: of the values dimension `lane`, of the keys a
    // piece of 16 dimensions of one key (what lies past `dim` is read somewhere inside). Where
    // there is no page, page 0 is read instead.
    uint32_t koff[kLoads], voff[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        koff[i] = uint32_t((i * 64 + lane) / (DP / 16) * D + min(lane % (DP / 16) * 16, D - 16));
        voff[i] = uint32_t(min(i * 64 + lane, D - 1) * page);
    }
    const uint8_t *const kh = p.kc + int64_t(h) * D * page, *const vh = p.vc + int64_t(h) * D * page;
    const int64_t page_bytes = int64_t(p.heads) * D * page;
    auto fetch = [&](int step, int pids) {
#pragma unroll
        for (int q = 0; q < kRuns; ++q) {
            const int which = wave * kRuns + q, pid = __builtin_amdgcn_readlane(pids, which * 16);
            const int slot = (step * kStep + which * 16) & (page - 1);
            const int64_t at = max(pid, 0) * page_bytes;
            const uint8_t *k = kh + at + slot * D, *v = vh + at + slot;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                kraw[q][i] = *reinterpret_cast<const i32x4 *>(k + koff[i]);
                vraw[q][i] = *reinterpret_cast<const i32x4 *>(v + voff[i]);
            }
        }
    };
    // The order of a key's pieces: its row in a tile, from 16 on again. Rows of 128 bytes
    // share a bank row by twos.
    auto order = [](int key) { return ((key & 3) | ((key >> 3) & 1) << 2 | ((key >> 2) & 1) << 3) >> (DP < 128 ? 1 : 0); };
    // Keys that no query sees may hold anything: their values count as 0. So does what was
    // read of a key past `dim`.
    auto clear = [&](int step, int pids) {
        if (__builtin_expect(D == DP && step * kStep >= tlo && step * kStep + kStep <= thi && on_pages(pids), 1)) return;
#pragma unroll
        for (int q = 0; q < kRuns; ++q) {
            const int which = wave * kRuns + q, run = step * kStep + which * 16;
            const bool there = __builtin_amdgcn_readlane(pids, which * 16) >= 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int mask = there ? key_mask(run + 4 * w, tlo, thi) : 0;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    vraw[q][i][w] &= mask;
                    if (lane % (DP / 16) * 16 >= D) kraw[q][i][w] = 0;
                }
            }
        }
    };
    auto note_nans = [&](int step, int buf) {
        if (!mixed(step)) return;
        uint32_t nan = 0;
#pragma unroll
        for (int q = 0; q < kRuns; ++q)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int w = 0; w < 4; ++w) nan |= nan_bytes(vraw[q][i][w]);
        nans[buf][wave] = __any(nan != 0);
    };
    // Part u of what fetch() read, to LDS: 8 keys or values a lane.
    constexpr int kParts = kRuns * kLoads * 4;
    auto put = [&](int u, int buf) {
        const int q = u / (kLoads * 4), i = u / 4 % kLoads, c = u / 2 % 2, which = wave * kRuns + q;
        uint8_t *const ks = lds[buf], *const vs = ks + kKeys;
        if (u % 2 == 0) {
            const int key = which * 16 + (i * 64 + lane) / (DP / 16), piece = (lane % (DP / 16)) * 2;
            *reinterpret_cast<v8 *>(ks + key * DP * 2 + ((piece + c) ^ order(key)) * 16) = widen<T>(kraw[q][i][2 * c], kraw[q][i][2 * c + 1]);
        } else {
            const int d = i * 64 + lane;
            *reinterpret_cast<f16x8 *>(vs + d * 128 + ((which * 2 + c) ^ ((d >> 1) & 7)) * 16) = widen<_Float16>(vraw[q][i][2 * c], vraw[q][i][2 * c + 1]);
        }
    };
    // Pages of this step and the next, the table's entry of the one after, and this step's
    // scales. Those of the next step are read before its successor's keys, so that waiting
    // for them waits for nothing else.
    int pid0 = -1, pid1 = -1, next = -1, ek = 0, ev = 0;
    auto look_ahead = [&](int step) {
        const int64_t at = int64_t(max(pid1, 0)) * p.heads + h;
        ek = p.ks[at];
        ev = p.vs[at];
        next = entry(step);
        asm volatile("" : : : "memory");
    };
    if (from < to) {
        pid1 = on_page(entry(from));
        fetch(from, pid1);
        look_ahead(from + 1);
        clear(from, pid1);
        note_nans(from, 0);
#pragma unroll
        for (int u = 0; u < kParts; ++u) put(u, 0);
        pid0 = pid1;
        pid1 = on_page(next);
        next = entry(from + 2);
        fetch(from + 1, pid1);
    }
    // A step mixes what does not depend on each other, product by product (each is issued in
    // a few clocks and takes 32): into the first products the transfer of the next step's keys
    // to LDS, into the second ones the weights that the products after them need. What they
    // read from LDS is read eight products ahead.
    constexpr int kFirst = 2 * QC, kSecond = 4 * DT, kAhead = 8;
    const int krow = (r >> 4) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);     // row r's key in tile 0
    auto body = [&](int step, auto which_buf) {
        constexpr int buf = decltype(which_buf)::value;
        const int base = step * kStep;
        wait_lds();
        barrier();
        const uint8_t *const kt = lds[buf] + krow * DP * 2, *const vt = lds[buf] + kKeys + r * 128;
        auto key_part = [&](int n) { return *reinterpret_cast<const v8 *>(kt + (n % 2) * 32 * DP * 2 + ((n / 2 * 2 + hf) ^ order(krow)) * 16); };
        auto value_part = [&](int n) {
            return *reinterpret_cast<const f16x8 *>(vt + n % DT * 32 * 128 + ((n / DT * 2 + hf) ^ ((r >> 1) & 7)) * 16);
        };
        if (mixed(step)) {
            int nan = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) nan |= nans[buf][w];
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
                for (int i = int(threadIdx.x); i < kKeys / 16; i += 64 * WAVES) {
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
        const PageScale ps = page_scale(ek, ev, p.scale);
        const bool held = on_pages(pid0);
        const int now = pid0;
        if (step + 1 < to) {
            clear(step + 1, pid1);
            note_nans(step + 1, buf ^ 1);
        }
        f32x16 s[2];
#pragma unroll
        for (int n = 0; n < kFirst; ++n) {
            s[n % 2] = mma32(kf[n % kAhead], qf[n / 2], n < 2 ? f32x16{} : s[n % 2]);
            if (n + kAhead < kFirst) kf[n % kAhead] = key_part(n + kAhead);
#pragma unroll
            for (int u = n * kParts / kFirst; u < (n + 1) * kParts / kFirst; ++u) put(u, buf ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        f16x8 vf[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) vf[n] = value_part(n);
        pid0 = pid1;
        if (step + 1 < to) {
            const int pid2 = on_page(next);
            look_ahead(step + 3);
            pid1 = pid2;
            fetch(step + 2, pid2);
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
        float sk[kScales], lv[kScales], iv[kScales], top = -__builtin_inff();
        const float sub = or_zero(m);
#pragma unroll
        for (int j = 0; j < kScales; ++j) {
            auto of = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), j * 16)); };
            sk[j] = of(ps.sk);
            lv[j] = of(ps.lv);
            iv[j] = of(ps.iv);
            constexpr int kN = 32 / kScales;
            const float off = lv[j] - sub;
#pragma unroll
            for (int i = j * kN; i < (j + 1) * kN; ++i) s[i / 16][i % 16] = fmaf(s[i / 16][i % 16], sk[j], off);
#pragma unroll
            for (int i = j * kN; i < (j + 1) * kN; i += 2) top = fmaxf(top, fmaxf(s[i / 16][i % 16], s[i / 16][i % 16 + 1]));
        }
        raise(m, l, max_over_32(top),
              [&](float by) {
#pragma unroll
                  for (int i = 0; i < 32; ++i) s[i / 16][i % 16] -= by;
              },
              [&](float alpha) {
#pragma unroll
                  for (int d = 0; d < DT; ++d) acc[d] *= alpha;
              });
        // (The sum is of the 32-bit weights: of a page whose scale is far below the largest one's
        // nothing may be left in 16 bits, but its weights count all the same.)
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
#pragma unroll
        for (int q = 0; q < 4; ++q) l = fmaf(sum[q], iv[q * kScales / 4], l);
    };
    for (int step = from; step < to; step += 2) {
        body(step, std::integral_constant<int, 0>{});
        if (step + 1 < to) body(step + 1, std::integral_constant<int, 1>{});
    }
    l += __shfl_xor(l, 32);
    if (row >= p.rows) return;
    if (!live) {
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

// The splits of a row together: a block of 4 waves per row, LANES lanes (4 dimensions each)
// per split, so that 16 or 8 or 4 splits are read at once. A few us (64 splits of 32 rows: 3), behind
// the launch that writes them.
template <typename T, int LANES>
__global__ void __launch_bounds__(256)
attention_join_kernel(const AttentionParams p)
{
    constexpr int kAtOnce = 256 / LANES;
    __shared__ float red[2][4];
    __shared__ f32x4 sums[256];
    const int64_t at = blockIdx.x;
    const int D = p.dim, d = int(threadIdx.x % LANES) * 4, mine = int(threadIdx.x) / LANES;
    const float *part = p.part + at * p.splits * (D + 2);
    float top = -__builtin_inff();
    for (int s = threadIdx.x; s < p.splits; s += 256) top = fmaxf(top, part[s * (D + 2) + D]);
    top = lanes_max<64>(top);
    if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = top;
    __syncthreads();
    const float sub = or_zero(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])));
    float total = 0.f;
    for (int s = threadIdx.x; s < p.splits; s += 256)
        total = fmaf(part[s * (D + 2) + D + 1], __builtin_amdgcn_exp2f(part[s * (D + 2) + D] - sub), total);
    total = lanes_sum<64>(total);
    if ((threadIdx.x & 63) == 0) red[1][threadIdx.x >> 6] = total;
    f32x4 o{};
    if (d < D) {
#pragma unroll 4
        for (int s = mine; s < p.splits; s += kAtOnce) {
            const float f = __builtin_amdgcn_exp2f(part[s * (D + 2) + D] - sub);
            f32x4 x;
            __builtin_memcpy(&x, part + s * (D + 2) + d, 16);
            o += x * f;
        }
    }
    sums[threadIdx.x] = o;
    __syncthreads();
    if (mine != 0 || d >= D) return;
#pragma unroll
    for (int i = 1; i < kAtOnce; ++i) o += sums[i * LANES + threadIdx.x];
    const int64_t bh = at / p.rows;
    store_row<T>(p, int(bh / p.heads), int(bh % p.heads), int(at - bh * p.rows), nullptr, d, o, inverse(red[1][0] + red[1][1] + red[1][2] + red[1][3]));
}

// How a call is split: over the rows first, then over the keys until 512 blocks (two a CU) have at
// least 8 steps of 64 keys each. Measured (8 heads of 128, 4 query heads each; us): one query over 131072
// keys 57, with 256 blocks 61, with 1024 61, unsplit 1202; 16 x 1 over up to 8192 40, 55, 43 and, with 2048,
// 48; 48 x 1 (384 blocks, two splits each, since lengths differ) 94, with 1024 91, unsplit 108; 100 queries
// over 32768 keys 95, with 256 blocks 116, with 1024 115. Up to 16 rows run attention_few_kernel (48 x 1: 94,
// the other 238; 32 x 16 of 1 query head over 4096 keys 56 and 79). From 17 to 64 rows blocks of two waves:
// 32 x 16 queries over 4096 keys 90, of four 98, of 2 query heads 81 and 88; above, of four: 2 x 1000
// queries 270, of two 410. (Splits go by the table's width, not by lengths: 64 sequences of 8 heads are
// not split, and one of them that is much longer than the others is what a call waits for.)
Plan plan_attention(int64_t batch, int64_t tokens, int64_t heads, int64_t group, int64_t columns, int64_t page)
{
    Plan a;
    a.rows = tokens * group;
    a.waves = a.rows <= 16 ? 0 : a.rows <= 64 ? 2 : 4;
    a.row_tiles = a.waves ? int((a.rows + 32 * a.waves - 1) / (32 * a.waves)) : 1;
    const int64_t blocks = std::max<int64_t>(batch * heads * a.row_tiles, 1), steps = (columns * page + kStep - 1) / kStep;
    a.splits = int(std::max<int64_t>(1, std::min<int64_t>({a.waves ? 512 / blocks : (511 + blocks) / blocks, (steps + 7) / 8, 256})));
    return a;
}

template <typename T, int DP>
void run_attention(const AttentionParams &p, const Plan &a, int64_t batch, hipStream_t s)
{
    const int bhs = int(batch * p.heads);
    const dim3 many(uint32_t((int64_t(bhs) * a.row_tiles * a.splits + 7) / 8 * 8));
    if (a.waves == 0) {
        hipLaunchKernelGGL((p.tokens == 1 ? attention_few_kernel<T, DP, true> : attention_few_kernel<T, DP, false>), dim3(a.splits, bhs),
                           dim3(256), 0, s, p);
    } else {
        hipLaunchKernelGGL((a.waves == 2 ? attention_many_kernel<T, DP, 2> : attention_many_kernel<T, DP, 4>), many, dim3(64 * a.waves), 0, s, p, bhs);
    }
    if (a.splits > 1)
        hipLaunchKernelGGL((attention_join_kernel<T, DP / 4>), dim3(uint32_t(bhs * a.rows)), dim3(256), 0, s, p);
}

template <typename T>
void run_attention(const AttentionParams &p, const Plan &a, int64_t batch, hipStream_t s)
{
    if (p.dim <= 64) run_attention<T, 64>(p, a, batch, s);
    else if (p.dim <= 128) run_attention<T, 128>(p, a, batch, s);
    else run_attention<T, 256>(p, a, batch, s);
}

}  // namespace

}  // namespace ds

using namespace ds;

extern "C" ds_status ds_kv_cache_append(const void *k, const void *v, uint8_t *k_cache, uint8_t *v_cache, uint8_t *k_scales,
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
    AppendParams p{table, start, count, ldt, int(columns), int(pages), int(tokens), int(heads), int(dim), int(page), make_fastdiv(uint32_t(dim / 8)), {}, {}, {}};
    int64_t bytes[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? v_strides : k_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        p.sb[i] = s[0];
        p.st[i] = s[1];
        p.sh[i] = s[2];
        bytes[i] = span(batch, tokens, heads, s, dim, es);
    }
    const int64_t cb = pages * heads * page * dim, sb = pages * heads;
    const int touched = int((tokens + page - 2) / page + 1);
    if (!grid_fits(batch * touched, 256)) return fail(DS_ERR_UNSUPPORTED, "too many pages in one call");
    if (ds_status st = check_tensors({{k, bytes[0], "k", false}, {v, bytes[1], "v", false}, {table, span(batch, ldt, columns, 4), "table", false},
                                      {start, batch * 4, "start", false}, {count, batch * 4, "count", false},
                                      {k_cache, cb, "k_cache", true}, {v_cache, cb, "v_cache", true},
                                      {k_scales, sb, "k_scales", true}, {v_scales, sb, "v_scales", true}}))
        return st;
    const dim3 grid(uint32_t(batch * touched), uint32_t(heads), 2);
    // (Tokens from a multiple of 8 to a multiple of 8.)
    const size_t lds = size_t(std::min(page, (tokens + 14) / 8 * 8)) * size_t(dim + 4);
    const auto s = static_cast<hipStream_t>(stream);
    const auto go = [&](auto t) {
        using T = decltype(t);
        const int64_t each = (std::min(page, tokens) * dim / 8 + 255) / 256;
        const auto kernel = each <= 1 ? append_kernel<T, 1> : each <= 4 ? append_kernel<T, 4> : append_kernel<T, 8>;
        hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, static_cast<const T *>(k), static_cast<const T *>(v),
                           k_cache, v_cache, k_scales, v_scales, p, touched);
    };
    if (type == DS_TYPE_F32) go(float{});
    else if (type == DS_TYPE_F16) go(_Float16{});
    else go(__bf16{});
    return launched("ds_kv_cache_append");
}

extern "C" int64_t ds_attention_fp8_scratch_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t group, int64_t dim,
                                                  int64_t page, int64_t columns)
{
    if (batch <= 0 || tokens <= 0 || heads <= 0 || group <= 0 || dim <= 0 || page <= 0 || columns <= 0) return 0;
    return 4 * part_floats(plan_attention(batch, tokens, heads, group, columns, page), batch, heads, dim);
}

extern "C" ds_status ds_attention_fp8(const void *q, const uint8_t *k_cache, const uint8_t *v_cache, const uint8_t *k_scales,
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
    if (batch * heads > 65535) return fail(DS_ERR_UNSUPPORTED, "more than 65535 sequences times heads");
    if (group > 65535 || tokens * group > kMaxElems / 64) return fail(DS_ERR_UNSUPPORTED, "too many queries of a head");
    const Plan a = plan_attention(batch, tokens, heads, group, columns, page);
    if (batch * heads * a.rows * a.splits > kMaxElems / 2) return fail(DS_ERR_UNSUPPORTED, "too many queries");
    int64_t bytes[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? o_strides : q_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        bytes[i] = span(batch, tokens, heads * group, s, dim, 2);
    }
    const int64_t cb = pages * heads * page * dim, sb = pages * heads, need = 4 * part_floats(a, batch, heads, dim);
    if (need > 0 && !scratch) return fail(DS_ERR_NULL_POINTER, "scratch must not be NULL");
    if (need > scratch_bytes) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    if (ds_status st = check_tensors({{q, bytes[0], "q", false}, {k_cache, cb, "k_cache", false}, {v_cache, cb, "v_cache", false},
                                      {k_scales, sb, "k_scales", false}, {v_scales, sb, "v_scales", false},
                                      {table, span(batch, ldt, columns, 4), "table", false}, {length, batch * 4, "length", false},
                                      {count, batch * 4, "count", false}, {o, bytes[1], "o", true},
                                      {need ? scratch : nullptr, need, "scratch", true}}))
        return st;
    int shift = 4;
    while ((int64_t(1) << shift) < page) ++shift;
    const AttentionParams p{q, k_cache, v_cache, k_scales, v_scales, table, length, count, o,
                            need ? static_cast<float *>(scratch) : nullptr, ldt, q_strides[0], q_strides[1], q_strides[2],
                            o_strides[0], o_strides[1], o_strides[2], int(columns), int(pages), int(tokens), int(heads),
                            int(group), int(dim), shift, int(window), a.splits, int(a.rows), a.row_tiles,
                            std::fabs(scale) * 1.44269504f, scale < 0};
    const auto s = static_cast<hipStream_t>(stream);
    if (type == DS_TYPE_F16) run_attention<_Float16>(p, a, batch, s);
    else run_attention<__bf16>(p, a, batch, s);
    return launched("ds_attention_fp8");
}
