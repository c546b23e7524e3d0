// What the attentions over paged caches share: how queries and keys are found, the running
// maximum of a softmax, and the results' way out.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "fp8.hpp"

namespace ds {

// (Of each source that includes it.)
namespace {

constexpr int kStep = 64;       // keys of a step

// Key positions are 32-bit numbers, those of some steps past a table's last one among them.
constexpr int64_t kMaxKeys = (int64_t(1) << 31) - 4096;

struct AttentionParams {
    const void *q;
    const uint8_t *kc, *vc, *ks, *vs;
    const int *table, *length, *count;
    void *o;
    float *part;                 // [row of all][split][dim + 2], or NULL
    int64_t ldt, qb, qt, qh, ob, ot, oh;
    int columns, pages, tokens, heads, group, dim, page_shift;
    int window, splits, rows, row_tiles;
    float scale;                 // |softmax scale| * log2(e)
    int negative;                // the scale is: the queries are taken with the other sign
    int least;                   // steps of a split, where it has any
};

template <typename T> struct Vec8;
template <> struct Vec8<_Float16> { typedef f16x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x16 mma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// v if it is finite or +inf, 0 for -inf: what a row without keys subtracts.
__device__ __forceinline__ float or_zero(float v) { return v == -__builtin_inff() ? 0.f : v; }

// A row's reference m lies kBias below the largest exponent that it was set by and moves only when
// it is passed by more than kBias + kSlack, so that the sums are hardly ever rescaled: the exponents
// are formed with the old one, and where none is above that they stay. Weights reach 2^15 at
// most, the upper end of a 16-bit float's range (65504), and have the rest of it below them. What the
// bias gains there the slack loses in time: 2 x 1000 queries over up to 8000 keys take 256.8 us, with
// 7 and 8 255.2, with 11 and 4 260.7 (heads of 64, 4000 keys: 94.4, 93.6 and 97.9).
constexpr float kBias = 9.f, kSlack = 6.f;

// `top`: the largest of a row's new exponents, relative to the reference (0 in its place where
// there is none yet). Moves the reference where it has to, in a branch that is rarely taken: then
// shift(by) takes `by` off the exponents and rescale(alpha) multiplies the sums.
template <typename Shift, typename Rescale>
__device__ __forceinline__ void raise(float &m, float &l, float top, Shift &&shift, Rescale &&rescale)
{
    const bool none = m == -__builtin_inff(), grown = none ? top > m : top > kBias + kSlack;
    if (__any(grown)) {
        const float by = grown ? top - kBias : 0.f, alpha = grown ? (none ? 0.f : __builtin_amdgcn_exp2f(-by)) : 1.f;
        m = none ? (grown ? by : m) : m + by;
        l *= alpha;
        shift(by);
        rescale(alpha);
    }
}

// The larger of a lane's value and that of the lane 32 (16) further, in both.
__device__ __forceinline__ float max_over_32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float max_over_16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Bytes of the 4 keys from `key` on that lie in [low, high).
__device__ __forceinline__ int key_mask(int key, int low, int high)
{
    const int upto = high - key, past = low - key;
    uint32_t mask = upto >= 4 ? 0xffffffffu : upto <= 0 ? 0u : (1u << (8 * upto)) - 1u;
    if (past > 0) mask &= past >= 4 ? 0u : 0xffffffffu << (8 * past);
    return int(mask);
}

// A sequence's queries and the position of the first, which a length beyond the table does not
// move (and which is negative where there are more queries than tokens); the keys that have a column.
struct Sequence {
    int count, first, keys;
    __device__ __forceinline__ Sequence(const AttentionParams &p, int b)
    {
        const int length = max(p.length[b], 0);
        count = p.count ? min(max(p.count[b], 0), p.tokens) : p.tokens;
        first = length - count;
        keys = int(min(int64_t(length), int64_t(p.columns) << p.page_shift));
    }
};

// A lane's query: row `row` of head h, its keys [low, high) (0, 0 where it sees none), its elements as
// the first product's second operand (chunk c: elements c * CHUNK + g * GROUP .. + 7).
template <typename T, int DP, int CHUNK, int GROUP, int N>
__device__ __forceinline__ bool load_query(const AttentionParams &p, const Sequence &seq, int b, int h, int row, int g, int &low, int &high,
                                           typename Vec8<T>::type (&qf)[N])
{
    const int t = row / p.group, hq = h * p.group + row - t * p.group;
    const bool live = row < p.rows && t < seq.count;
    const int upto = live ? seq.first + t + 1 : 0;
    high = min(max(upto, 0), seq.keys);
    low = p.window ? max(max(upto, 0) - p.window, 0) : 0;
    if (low >= high) low = high = 0;
    const T *src = static_cast<const T *>(p.q) + b * p.qb + (live ? t * p.qt + hq * p.qh : 0);
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int d = c * CHUNK + g * GROUP;
        typename Vec8<T>::type x{};
        if (live && d < p.dim) __builtin_memcpy(&x, src + d, 16);
        qf[c] = p.negative ? -x : x;
    }
    return live;
}

// Four of a row's results, to o or (unnormalised) to the split's part.
template <typename T>
__device__ __forceinline__ void store_row(const AttentionParams &p, int b, int h, int row, float *part, int d, f32x4 o, float inv)
{
    if (part) {
        __builtin_memcpy(part + d, &o, 16);
        return;
    }
    const int t = row / p.group, hq = h * p.group + row - t * p.group;
    T *out = static_cast<T *>(p.o) + b * p.ob + t * p.ot + hq * p.oh + d;
    T x[4] = {T(o[0] * inv), T(o[1] * inv), T(o[2] * inv), T(o[3] * inv)};
    __builtin_memcpy(out, x, 8);
}

__device__ __forceinline__ float inverse(float total) { return total > 0.f ? 1.f / total : total == 0.f ? 0.f : total; }

bool page_ok(int64_t page) { return page == 16 || page == 32 || page == 64 || page == 128; }

ds_status check_cache(int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int64_t page, int64_t pages, int64_t columns,
                      int64_t ldt)
{
    if (batch < 0 || tokens < 0 || heads <= 0 || dim <= 0 || pages <= 0 || columns <= 0)
        return fail(DS_ERR_INVALID_SHAPE, "batch and tokens must be >= 0; heads, dim, pages and columns > 0");
    if (dim % 16 || dim > 256) return fail(DS_ERR_UNSUPPORTED, "dim must be a multiple of 16, at most 256");
    if (!page_ok(page)) return fail(DS_ERR_UNSUPPORTED, "a page must have 16, 32, 64 or 128 tokens");
    if (ldt < columns) return fail(DS_ERR_INVALID_ARG, "a row of the table is shorter than its columns");
    if (heads > 65535 || batch > (1 << 20) || tokens > (1 << 24) || pages > kMaxElems || columns > kMaxKeys / page)
        return fail(DS_ERR_UNSUPPORTED, "too many heads, sequences, tokens or pages");
    return DS_SUCCESS;
}

struct Plan {
    int waves, splits, row_tiles;      // waves 0: few queries of a head
    int64_t rows;
    int least = 1;                     // steps of a split, where it has any
};

int64_t part_floats(const Plan &a, int64_t batch, int64_t heads, int64_t dim)
{
    return a.splits == 1 ? 0 : batch * heads * a.rows * a.splits * (dim + 2);
}

}  // namespace

}  // namespace ds
