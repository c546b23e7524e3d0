// A paged cache of keys and values in 8 bits, and the attention that reads it.
//
// Layout: keys [page][head][token][dim], values [page][head][dim][token] (the order in
// which the second product of an attention contracts them), both E4M3, with one E8M0
// scale for each page and head. A sequence's pages are listed in a row of a table.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "conv_plan.hpp"
#include "fp8.hpp"

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
    int64_t sb[2], st[2], sh[2];       // strides of k and v: sequence, token, head
};

// One page's new tokens of one head: its scale, the rounding of what it holds already
// to a larger scale, and the tokens. Every (page, head) is one block's alone.
template <typename T>
__global__ void __launch_bounds__(256)
append_kernel(const T *__restrict__ k, const T *__restrict__ v, uint8_t *__restrict__ kc, uint8_t *__restrict__ vc,
              uint8_t *__restrict__ ks, uint8_t *__restrict__ vs, const AppendParams p, int touched)
{
    __shared__ float red[4];
    extern __shared__ uint8_t tile[];       // values: [token][dim + 4]
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
    float amax = 0.f;
    for (int i = threadIdx.x; i < total; i += 256) {
        float x[8];
        load8(src + (i / vecs) * st + (i % vecs) * 8, 8, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(x[e]));
    }
    amax = lanes_max<64>(amax);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    const int before = min(max(int(*scale), kCacheLow), kCacheHigh);
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
    auto held = [&](float x) { return fabsf(x) < __builtin_inff() ? fminf(fmaxf(x * s, -448.f), 448.f) : __builtin_nanf(""); };
    const int pitch = D + 4;
    for (int i = threadIdx.x; i < total; i += 256) {
        const int tok = i / vecs, d = (i % vecs) * 8;
        float x[8];
        load8(src + tok * st + d, 8, x);
        i32x2 q;
        q[0] = to_fp8x4(held(x[0]), held(x[1]), held(x[2]), held(x[3]));
        q[1] = to_fp8x4(held(x[4]), held(x[5]), held(x[6]), held(x[7]));
        if (which) {
            *reinterpret_cast<int *>(tile + tok * pitch + d) = q[0];
            *reinterpret_cast<int *>(tile + tok * pitch + d + 4) = q[1];
        } else {
            *reinterpret_cast<i32x2 *>(cache + int64_t(lo + tok) * D + d) = q;
        }
    }
    if (threadIdx.x == 0) *scale = uint8_t(e);
    if (!which) return;
    __syncthreads();
    // Four tokens of one dimension a thread, from the tile's columns.
    const int q0 = lo / 4, quads = (hi + 3) / 4 - q0;
    for (int i = threadIdx.x; i < quads * D; i += 256) {
        const int d = i / quads, q = q0 + i % quads;
        uint8_t *o = cache + int64_t(d) * p.page + 4 * q;
        uint32_t w = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int tok = 4 * q + t - lo;
            if (tok >= 0 && tok < hi - lo) w |= uint32_t(tile[tok * pitch + d]) << (8 * t);
        }
        if (4 * q >= lo && 4 * q + 4 <= hi) {
            *reinterpret_cast<uint32_t *>(o) = w;
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (4 * q + t >= lo && 4 * q + t < hi) o[t] = uint8_t(w >> (8 * t));
        }
    }
}

// ---------------------------------------------------------------------------
// Attention. A kv head's queries are its `rows` = tokens x group vectors, and a wave
// handles MT x 16 of them with 64 keys at a time:
//
//   S^T = K Q^T (the matrix instruction's rows are keys, its columns queries), so that a
//   lane holds 16 consecutive keys of one query;
//   t = S * 2^ek * scale * log2(e) + log2(2^ev): the value scale ev of the keys' page goes
//   into the exponent, so p = 2^(t - m), m the running maximum of t, is at most 1 and
//   weighs the 8-bit values themselves;
//   O^T += V^T P (rows: dimensions, columns: queries), l += p * 2^-ev.
//
// The two layouts agree, so that p goes from the first product to the second in place:
// the key of row r of a 16-key tile t is chosen as (r / 4) * 16 + t * 4 + r % 4, which
// leaves lane group g (lane / 16) with keys 16 g .. 16 g + 15, and those are the ones that
// it contracts in the second product, 8 at a time. Keys become numbers of the queries'
// type exactly; p and the values are 16-bit floats with 10 bits of mantissa (values
// exactly, p rounded once to 2^-11).

constexpr int kStep = 64;       // keys of a step

struct AttentionParams {
    const void *q;
    const uint8_t *kc, *vc, *ks, *vs;
    const int *table, *length, *count;
    void *o;
    float *part;                 // [row of all][split][dim + 2], or NULL
    int64_t ldt, qb, qt, qh, ob, ot, oh;
    int columns, pages, tokens, heads, group, dim, page_shift;
    int window, splits, rows, row_tiles;
    float scale;                 // softmax scale * log2(e)
};

template <typename T> struct Vec8;
template <> struct Vec8<_Float16> { typedef f16x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };

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

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// v if it is finite or +inf, 0 for -inf: what a row without keys subtracts.
__device__ __forceinline__ float or_zero(float v) { return v == -__builtin_inff() ? 0.f : v; }

// Block: 4 waves, the same rows, every fourth step of the block's share of the keys.
template <typename T, int DP, int MT>
__global__ void __launch_bounds__(256)
attention_kernel(const AttentionParams p)
{
    constexpr int kWaves = 4;
    constexpr int QC = DP / 32;            // chunks of 32 of the first product's contraction
    constexpr int KB = DP / 64;            // 16-byte loads of a lane's part of a key
    constexpr int DT = DP / 16;            // tiles of 16 dimensions of the second product
    typedef typename Vec8<T>::type v8;
    __shared__ float ml[2][kWaves][MT * 16];
    __shared__ f32x4 osum[kWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const int split = int(blockIdx.x), tile = int(blockIdx.y), bh = int(blockIdx.z), b = bh / p.heads, h = bh - b * p.heads;
    const int D = p.dim, page = 1 << p.page_shift;
    const int64_t held = int64_t(p.columns) * page;
    const int length = int(min(int64_t(max(p.length[b], 0)), held));
    const int count = min(p.count ? max(p.count[b], 0) : p.tokens, min(p.tokens, length));
    const int first = length - count;      // position of the first query

    // This lane's queries, one of each tile: the keys [low, high) they see.
    v8 qf[MT][QC];
    int low[MT], high[MT];
    int tlo = 0x7fffffff, thi = 0;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = (tile * MT + mt) * 16 + r, t = row / p.group, hq = h * p.group + row - t * p.group;
        const bool live = row < p.rows && t < count;
        high[mt] = live ? first + t + 1 : 0;
        low[mt] = live && p.window ? max(high[mt] - p.window, 0) : 0;
        if (live) {
            tlo = min(tlo, low[mt]);
            thi = max(thi, high[mt]);
        }
        const T *src = static_cast<const T *>(p.q) + b * p.qb + (live ? t * p.qt + hq * p.qh : 0);
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            const int d = g * (DP / 4) + c * 8;
            v8 x{};
            if (live && d < D) __builtin_memcpy(&x, src + d, 16);
            qf[mt][c] = x;
        }
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
        tlo = min(tlo, __shfl_xor(tlo, o));
        thi = max(thi, __shfl_xor(thi, o));
    }
    tlo = __builtin_amdgcn_readfirstlane(tlo);
    thi = __builtin_amdgcn_readfirstlane(thi);
    const int s0 = thi > 0 ? tlo / kStep : 0, s1 = (thi + kStep - 1) / kStep;
    const int each = (s1 - s0 + p.splits - 1) / p.splits;
    const int from = s0 + split * each, to = min(s1, from + each);

    f32x4 acc[MT][DT];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -__builtin_inff();
        l[mt] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[mt][d] = f32x4{};
    }
    // Page of the 16 keys from `key` on (they share it), or -1 where there is none.
    auto page_of = [&](int key) {
        const int col = key >> p.page_shift;
        const int pid = key < thi ? p.table[b * p.ldt + col] : -1;
        return unsigned(pid) < unsigned(p.pages) ? pid : -1;
    };
    for (int step = from + wave; step < to; step += kWaves) {
        const int base = step * kStep;
        const int krun = base + (r >> 2) * 16, vrun = base + g * 16;
        const int kp = page_of(krun), vp = page_of(vrun);
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
#pragma unroll
        for (int d = 0; d < DT; ++d)
            vraw[d] = vp >= 0 && d * 16 < D ? *reinterpret_cast<const i32x4 *>(vrow + d * 16 * page) : i32x4{};
        const int ek = min(max(int(p.ks[vat]), kCacheLow), kCacheHigh), ev = min(max(int(p.vs[vat]), kCacheLow), kCacheHigh);
        const float sk = power_of_two(uint32_t(ek)) * p.scale, lv = float(ev - 127), iv = power_of_two(uint32_t(254 - ev));
        if (base + kStep > thi || base < tlo) {
            // Keys that no query sees may hold anything: their values count as 0.
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int upto = thi - vrun - 4 * w, past = tlo - vrun - 4 * w;
                uint32_t mask = upto >= 4 ? 0xffffffffu : upto <= 0 ? 0u : (1u << (8 * upto)) - 1u;
                if (past > 0) mask &= past >= 4 ? 0u : 0xffffffffu << (8 * past);
#pragma unroll
                for (int d = 0; d < DT; ++d) vraw[d][w] &= int(mask);
            }
        }
        f32x4 s[MT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s[mt][t] = f32x4{};
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                const v8 kf = widen<T>(kraw[t][c >> 1][(c & 1) * 2], kraw[t][c >> 1][(c & 1) * 2 + 1]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) s[mt][t] = mma(kf, qf[mt][c], s[mt][t]);
            }
        }
        f16x8 pf[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const bool whole = vp >= 0 && vrun >= low[mt] && vrun + 16 <= high[mt];
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float t = fmaf(s[mt][i >> 2][i & 3], sk, lv);
                if (!whole) t = vp >= 0 && vrun + i >= low[mt] && vrun + i < high[mt] ? t : -__builtin_inff();
                s[mt][i >> 2][i & 3] = t;
                top = fmaxf(top, t);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float mn = fmaxf(m[mt], top), sub = or_zero(mn), alpha = __builtin_amdgcn_exp2f(m[mt] - sub);
            m[mt] = mn;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(s[mt][i >> 2][i & 3] - sub);
                sum += e;
                pf[mt][i >> 3][i & 7] = _Float16(e);
            }
            l[mt] = fmaf(l[mt], alpha, sum * iv);
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[mt][d] *= alpha;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const f16x8 vf = widen<_Float16>(vraw[d][2 * c], vraw[d][2 * c + 1]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[mt][d] = mma(vf, pf[mt][c], acc[mt][d]);
            }
    }
    // The waves' sums together: a lane's l is its own keys'.
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        l[mt] += __shfl_xor(l[mt], 16);
        l[mt] += __shfl_xor(l[mt], 32);
        if (g == 0) {
            ml[0][wave][mt * 16 + r] = m[mt];
            ml[1][wave][mt * 16 + r] = l[mt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = (tile * MT + mt) * 16 + r, t = row / p.group, hq = h * p.group + row - t * p.group;
        float top = ml[0][0][mt * 16 + r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[0][w][mt * 16 + r]);
        const float sub = or_zero(top), mine = __builtin_amdgcn_exp2f(m[mt] - sub);
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total = fmaf(ml[1][w][mt * 16 + r], __builtin_amdgcn_exp2f(ml[0][w][mt * 16 + r] - sub), total);
        const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
        float *part = p.part + ((int64_t(bh) * p.rows + min(row, p.rows - 1)) * p.splits + split) * (D + 2);
        if (p.part && row < p.rows && wave == 0 && g == 0) {
            part[D] = top;
            part[D + 1] = total;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            osum[wave][lane] = acc[mt][d] * mine;
            __syncthreads();
            if (wave == (d & (kWaves - 1)) && row < p.rows && d * 16 + g * 4 < D) {
                f32x4 o = osum[0][lane];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) o += osum[w][lane];
                if (p.part) {
                    __builtin_memcpy(part + d * 16 + g * 4, &o, 16);
                } else {
                    T *out = static_cast<T *>(p.o) + b * p.ob + t * p.ot + hq * p.oh + d * 16 + g * 4;
                    T x[4] = {T(o[0] * inv), T(o[1] * inv), T(o[2] * inv), T(o[3] * inv)};
                    __builtin_memcpy(out, x, 8);
                }
            }
            __syncthreads();
        }
    }
}

// The splits of a row together: a wave per row.
template <typename T>
__global__ void __launch_bounds__(256)
attention_join_kernel(const AttentionParams p, int64_t rows_of_all)
{
    const int lane = threadIdx.x & 63;
    const int64_t at = int64_t(blockIdx.x) * 4 + int(threadIdx.x >> 6);
    if (at >= rows_of_all) return;
    const int D = p.dim;
    const float *part = p.part + at * p.splits * (D + 2);
    float top = -__builtin_inff();
    for (int s = lane; s < p.splits; s += 64) top = fmaxf(top, part[s * (D + 2) + D]);
    const float sub = or_zero(lanes_max<64>(top));
    float total = 0.f;
    f32x4 o{};
    for (int s = 0; s < p.splits; ++s) {
        const float *q = part + s * (D + 2), f = __builtin_amdgcn_exp2f(q[D] - sub);
        total = fmaf(q[D + 1], f, total);
        if (f != 0.f && lane * 4 < D) {
            f32x4 x;
            __builtin_memcpy(&x, q + lane * 4, 16);
            o += x * f;
        }
    }
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
    const int64_t bh = at / p.rows;
    const int row = int(at - bh * p.rows), t = row / p.group, b = int(bh / p.heads), hq = int(bh - int64_t(b) * p.heads) * p.group + row - t * p.group;
    if (lane * 4 >= D) return;
    T *out = static_cast<T *>(p.o) + b * p.ob + t * p.ot + hq * p.oh + lane * 4;
    T x[4] = {T(o[0] * inv), T(o[1] * inv), T(o[2] * inv), T(o[3] * inv)};
    __builtin_memcpy(out, x, 8);
}

bool page_ok(int64_t page) { return page == 16 || page == 32 || page == 64 || page == 128; }

ds_status check_cache(int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int64_t page, int64_t pages, int64_t columns,
                      int64_t ldt)
{
    if (batch < 0 || tokens < 0 || heads <= 0 || dim <= 0 || pages <= 0 || columns <= 0)
        return fail(DS_ERR_INVALID_SHAPE, "batch and tokens must be >= 0; heads, dim, pages and columns > 0");
    if (dim % 16 || dim > 256) return fail(DS_ERR_UNSUPPORTED, "dim must be a multiple of 16, at most 256");
    if (!page_ok(page)) return fail(DS_ERR_UNSUPPORTED, "a page must have 16, 32, 64 or 128 tokens");
    if (ldt < columns) return fail(DS_ERR_INVALID_ARG, "a row of the table is shorter than its columns");
    if (heads > 65535 || batch > (1 << 20) || tokens > (1 << 24) || pages > kMaxElems || columns * page > kMaxElems)
        return fail(DS_ERR_UNSUPPORTED, "too many heads, sequences, tokens or pages");
    return DS_SUCCESS;
}

struct Plan {
    int mt, splits, row_tiles;
    int64_t rows;
};

// How a call is split. MT: 16 rows a wave, more where there are more rows.
Plan plan_attention(int64_t batch, int64_t tokens, int64_t heads, int64_t group, int64_t dim, int64_t columns, int64_t page)
{
    Plan a;
    a.rows = tokens * group;
    a.mt = a.rows <= 16 ? 1 : a.rows <= 32 || dim > 128 ? 2 : 4;
    a.row_tiles = int((a.rows + 16 * a.mt - 1) / (16 * a.mt));
    const int64_t blocks = std::max<int64_t>(batch * heads * a.row_tiles, 1), steps = (columns * page + kStep - 1) / kStep;
    a.splits = int(std::max<int64_t>(1, std::min<int64_t>({2048 / blocks, (steps + 7) / 8, 256})));
    return a;
}

int64_t part_floats(const Plan &a, int64_t batch, int64_t heads, int64_t dim)
{
    return a.splits == 1 ? 0 : batch * heads * a.rows * a.splits * (dim + 2);
}

template <typename T, int DP>
void run_attention(const AttentionParams &p, const Plan &a, int64_t batch, hipStream_t s)
{
    const dim3 grid(uint32_t(a.splits), uint32_t(a.row_tiles), uint32_t(batch * p.heads));
    if (a.mt == 1) hipLaunchKernelGGL((attention_kernel<T, DP, 1>), grid, dim3(256), 0, s, p);
    else if (a.mt == 2 || DP > 128) hipLaunchKernelGGL((attention_kernel<T, DP, 2>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attention_kernel<T, DP, (DP > 128 ? 2 : 4)>), grid, dim3(256), 0, s, p);
    if (a.splits > 1) {
        const int64_t rows = batch * p.heads * a.rows;
        hipLaunchKernelGGL(attention_join_kernel<T>, dim3(uint32_t((rows + 3) / 4)), dim3(256), 0, s, p, rows);
    }
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
    AppendParams p{table, start, count, ldt, int(columns), int(pages), int(tokens), int(heads), int(dim), int(page), {}, {}, {}};
    int64_t bytes[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? v_strides : k_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        p.sb[i] = s[0];
        p.st[i] = s[1];
        p.sh[i] = s[2];
        bytes[i] = ((batch - 1) * s[0] + (tokens - 1) * s[1] + (heads - 1) * s[2] + dim) * es;
    }
    const int64_t cb = pages * heads * page * dim, sb = pages * heads;
    const int touched = int((tokens + page - 2) / page + 1);
    if (batch * touched > kMaxElems) return fail(DS_ERR_UNSUPPORTED, "too many pages in one call");
    if (ds_status st = check_tensors({{k, bytes[0], "k", false}, {v, bytes[1], "v", false}, {table, span(batch, ldt, columns) * 4, "table", false},
                                      {start, batch * 4, "start", false}, {count, batch * 4, "count", false},
                                      {k_cache, cb, "k_cache", true}, {v_cache, cb, "v_cache", true},
                                      {k_scales, sb, "k_scales", true}, {v_scales, sb, "v_scales", true}}))
        return st;
    const dim3 grid(uint32_t(batch * touched), uint32_t(heads), 2);
    const size_t lds = size_t(std::min(page, tokens)) * size_t(dim + 4);
    const auto s = static_cast<hipStream_t>(stream);
    const auto go = [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(append_kernel<T>, grid, dim3(256), lds, s, static_cast<const T *>(k), static_cast<const T *>(v),
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
    return 4 * part_floats(plan_attention(batch, tokens, heads, group, dim, columns, page), batch, heads, dim);
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
    const Plan a = plan_attention(batch, tokens, heads, group, dim, columns, page);
    if (a.row_tiles > 65535) return fail(DS_ERR_UNSUPPORTED, "too many queries of a head");
    int64_t bytes[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *s = i ? o_strides : q_strides;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0) return fail(DS_ERR_INVALID_ARG, "strides must be >= 0");
        bytes[i] = ((batch - 1) * s[0] + (tokens - 1) * s[1] + (heads * group - 1) * s[2] + dim) * 2;
    }
    const int64_t cb = pages * heads * page * dim, sb = pages * heads, need = 4 * part_floats(a, batch, heads, dim);
    if (need > 0 && !scratch) return fail(DS_ERR_NULL_POINTER, "scratch must not be NULL");
    if (need > scratch_bytes) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    if (ds_status st = check_tensors({{q, bytes[0], "q", false}, {k_cache, cb, "k_cache", false}, {v_cache, cb, "v_cache", false},
                                      {k_scales, sb, "k_scales", false}, {v_scales, sb, "v_scales", false},
                                      {table, span(batch, ldt, columns) * 4, "table", false}, {length, batch * 4, "length", false},
                                      {count, batch * 4, "count", false}, {o, bytes[1], "o", true},
                                      {need ? scratch : nullptr, need, "scratch", true}}))
        return st;
    int shift = 4;
    while ((int64_t(1) << shift) < page) ++shift;
    const AttentionParams p{q, k_cache, v_cache, k_scales, v_scales, table, length, count, o,
                            need ? static_cast<float *>(scratch) : nullptr, ldt, q_strides[0], q_strides[1], q_strides[2],
                            o_strides[0], o_strides[1], o_strides[2], int(columns), int(pages), int(tokens), int(heads),
                            int(group), int(dim), shift, int(window), a.splits, int(a.rows), a.row_tiles,
                            scale * 1.44269504f};
    const auto s = static_cast<hipStream_t>(stream);
    if (type == DS_TYPE_F16) run_attention<_Float16>(p, a, batch, s);
    else run_attention<__bf16>(p, a, batch, s);
    return launched("ds_attention_fp8");
}
