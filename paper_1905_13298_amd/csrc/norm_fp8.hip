// Root-mean-square norm with the residual's addition and an 8-bit output, its
// gradient, and the quantisers: of activations (with or without a SiLU gate), of
// weight matrices, and of shift codes.
//
// All are streaming passes bound by memory bandwidth: every input is read once and
// every output written once. A thread holds 8 consecutive elements, so 16 lanes hold
// the 128 elements that share a scale and its maximum is four steps between lanes.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "conv_plan.hpp"
#include "fastdiv.hpp"
#include "fp8.hpp"

namespace ds {

namespace {

// ---------------------------------------------------------------------------
// Norm. h = x + residual (rounded to x's type, as it is stored), rstd = 1 / sqrt(mean
// h^2 + eps), y = h * rstd * weight, in 8 bits or in x's type.

struct NormParams {
    int64_t rows, ldx, ldr, ldh, ldy, lds;
    int cols;
    float eps;
};

// Sum of `v` over the TPR threads of a row; `red` holds a float per wave.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red)
{
    v = lanes_sum<64>(v);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) v += red[i];
    }
    return v;
}

template <int TPR>
constexpr int row_block() { return TPR < 256 ? 256 : TPR; }

// TPR threads hold a row in registers, NV vectors of 8 elements each. WHOLE: rows of a
// multiple of 8 elements. Weights are read with the row, not behind its sum. Bound by bandwidth
// where rows are many (8192 x 4096 with residual, 235 MB: 39.7 us, 5.9 TB/s with part of it still in
// the caches), by the launch and one trip to memory where they are few (8 x 4096: 3.3 us).
template <typename T, typename W, int TPR, int NV, bool QUANT, bool WHOLE>
__global__ void __launch_bounds__(row_block<TPR>())
norm_kernel(const T *__restrict__ x, const T *__restrict__ residual, const W *__restrict__ weight, void *__restrict__ y,
            uint8_t *__restrict__ scales, T *__restrict__ h, float *__restrict__ rstd, const NormParams p)
{
    __shared__ float red[row_block<TPR>() / 64];
    constexpr int kRowsPerBlock = row_block<TPR>() / TPR;
    const int t = int(threadIdx.x) % TPR;
    const int64_t row = int64_t(blockIdx.x) * kRowsPerBlock + __builtin_amdgcn_readfirstlane(int(threadIdx.x) / TPR);
    if (kRowsPerBlock > 1 && row >= p.rows) return;    // whole waves: no barrier follows
    const T *const xr = x + row * p.ldx, *const rr = residual + row * p.ldr;
    T *const hr = h + row * p.ldh;
    Eight<T> v[NV], r8[NV];
    Eight<W> w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8, n = p.cols - c;
        v[i].clear();
        r8[i].clear();
        w[i].clear();
        if (n <= 0) continue;
        v[i].template load<WHOLE>(xr, c, n);
        if (residual) r8[i].template load<WHOLE>(rr, c, n);
        w[i].template load<WHOLE>(weight, c, n);
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8, n = p.cols - c;
        if (residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i].v[e] = T(v[i].at(e) + r8[i].at(e));
            if (n > 0) v[i].template store<WHOLE>(hr, c, n);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(v[i].at(e), v[i].at(e), sum);
    }
    sum = row_sum<TPR>(sum, red);
    const float r = 1.f / sqrtf(sum / float(p.cols) + p.eps);
    if (rstd && t == 0) rstd[row] = r;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8, n = p.cols - c;
        float o[8], amax = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = WHOLE || e < n ? v[i].at(e) * r * w[i].at(e) : 0.f;      // (r may be no number)
            amax = fmaxf(amax, finite_abs(o[e]));
        }
        if constexpr (QUANT) {
            const int e = block_scale(lanes_max<16>(amax));
            const float s = power_of_two(254 - e);
            if (n > 0) {
                i32x2 q;
                q[0] = to_fp8x4(o[0] * s, o[1] * s, o[2] * s, o[3] * s);
                q[1] = to_fp8x4(o[4] * s, o[5] * s, o[6] * s, o[7] * s);
                *reinterpret_cast<i32x2 *>(static_cast<uint8_t *>(y) + row * p.ldy + c) = q;
                if ((t & 15) == 0) scales[row * p.lds + c / kScaleBlock] = uint8_t(e);
            }
        } else if (n > 0) {
            store8(static_cast<T *>(y) + row * p.ldy + c, WHOLE ? 8 : n, o);
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient. With n = h * rstd and g = dy * weight: dx = rstd * (g - n * mean(g * n)) +
// dh (the gradient of x and of the residual alike), dweight = sum over rows of dy * n.
// The rounding to 8 bits counts as the identity. A block takes every `gridDim.x`-th
// row (or group of rows) and keeps its share of dweight in registers; the shares are
// added by a second launch, always in the same order. Bound by bandwidth: 8192 x 4096 elements in
// 16 bits with dh, 268 MB, 46 us (5.8 TB/s).

struct NormGradParams {
    int64_t rows, lddy, ldh, lddh, lddx;
    int cols;
};

// WHOLE: rows of a multiple of 8 elements. (Without the loads of single elements the wide
// rows' 128 registers a thread are enough.)
template <typename T, typename W, int TPR, int NV, bool WHOLE>
__global__ void __launch_bounds__(row_block<TPR>(), NV == 1 && TPR > 64 ? 4 : 1)
norm_grad_kernel(const T *__restrict__ dy, const T *__restrict__ h, const W *__restrict__ weight,
                 const float *__restrict__ rstd, const T *__restrict__ dh, T *__restrict__ dx, float *__restrict__ part,
                 const NormGradParams p)
{
    constexpr int kRowsPerBlock = row_block<TPR>() / TPR;
    __shared__ float red[2][row_block<TPR>() / 64];
    const int t = int(threadIdx.x) % TPR, sub = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / TPR);
    Eight<W> w[NV];
    float dw[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8, n = p.cols - c;
        w[i].clear();
        if (n > 0) w[i].template load<WHOLE>(weight, c, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = 0.f;
    }
    const float inv = 1.f / float(p.cols);
    const int64_t step = int64_t(gridDim.x) * kRowsPerBlock, first = int64_t(blockIdx.x) * kRowsPerBlock + sub;
    // The next row's elements are on their way while this one's are reduced; they stay as they
    // were stored, in half the registers. What lies past the columns stays 0. (Two rows ahead:
    // the same time.)
    struct Row {
        Eight<T> dy[NV], h[NV], dh[NV];
        float r;
    };
    Row next;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        next.dy[i].clear();
        next.h[i].clear();
        next.dh[i].clear();
    }
    next.r = 0.f;
    auto fetch = [&](int64_t row) {
        if (row >= p.rows) return;
        next.r = rstd[row];
        const T *const dyr = dy + row * p.lddy, *const hr = h + row * p.ldh, *const dhr = dh + row * p.lddh;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * 8, n = p.cols - c;
            if (n <= 0) continue;
            next.dy[i].template load<WHOLE>(dyr, c, n);
            next.h[i].template load<WHOLE>(hr, c, n);
            if (dh) next.dh[i].template load<WHOLE>(dhr, c, n);
        }
    };
    fetch(first);
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += step, turn ^= 1) {
        const Row x = next;
        fetch(row + step);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x.dy[i].at(e), n = x.h[i].at(e) * x.r;
                dw[i][e] = fmaf(d, n, dw[i][e]);
                sum = fmaf(d * w[i].at(e), n, sum);
            }
        sum = lanes_sum<64>(sum);
        if constexpr (TPR > 64) {
            // Two sets of sums in turn: a wave is at most one row ahead of the slowest.
            if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = sum;
            wait_lds();
            barrier();
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < TPR / 64; ++i) sum += red[turn][i];
        }
        const float mean = sum * inv;
        T *const out = dx + row * p.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * 8, n = p.cols - c;
            if (n <= 0) continue;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                o[e] = fmaf(x.r, x.dy[i].at(e) * w[i].at(e) - x.h[i].at(e) * x.r * mean, x.dh[i].at(e));
            store8(out + uint32_t(c), WHOLE ? 8 : n, o);
        }
    }
    if (!part) return;
    const int64_t base = (int64_t(blockIdx.x) * kRowsPerBlock + sub) * p.cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8, n = p.cols - c;
        if (n > 0) store8(part + base + c, n, dw[i]);
    }
}

// dweight[c] = sum over `parts` rows of part: a block adds 32 columns, 32 threads a column.
template <typename W>
__global__ void __launch_bounds__(1024)
norm_grad_weight_kernel(const float *__restrict__ part, W *__restrict__ dweight, int parts, int cols)
{
    __shared__ float red[32][33];
    const int x = int(threadIdx.x & 31), y = int(threadIdx.x >> 5), c = int(blockIdx.x) * 32 + x;
    float sum = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int i = y; i < parts; i += 32) sum += part[int64_t(i) * cols + c];
    }
    red[y][x] = sum;
    __syncthreads();
    // Column y of the block, its 32 sums across half a wave.
    sum = red[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 32);
    const int out = int(blockIdx.x) * 32 + y;
    if (x == 0 && out < cols) dweight[out] = W(sum);
}

// ---------------------------------------------------------------------------
// Quantisers.

struct QuantParams {
    int64_t ldx, ldg, ldy, lds;
    int cols, blocks;            // blocks of 128 in the whole tensor
    FastDiv per_row;             // blocks of a row
};

// x, or silu(gate) * x, in 8 bits: 16 lanes per block of 128. Bound by bandwidth: 4099 x 11000
// gated, 226 MB, 50 us (4.5 TB/s); 16 x 8192 by the launch, 3.4 us.
template <typename T, bool GATE>
__global__ void __launch_bounds__(256)
quantize_kernel(const T *__restrict__ x, const T *__restrict__ gate, uint8_t *__restrict__ y, uint8_t *__restrict__ scales,
                const QuantParams p)
{
    const int b = int(blockIdx.x) * 16 + int(threadIdx.x >> 4);
    const int bc = min(b, p.blocks - 1);
    const int64_t row = fdiv(bc, p.per_row);
    const int blk = bc - int(row) * int(p.per_row.d);
    const int c = blk * kScaleBlock + int(threadIdx.x & 15) * 8, n = p.cols - c;
    float v[8] = {};
    if (n > 0) {
        load8(x + row * p.ldx + c, n, v);
        if constexpr (GATE) {
            float g[8];
            load8(gate + row * p.ldg + c, n, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = g[e] / (1.f + __expf(-g[e])) * v[e];     // (exact to 2^-22 + |g| 2^-24, the result to 2^-4)
        }
    }
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(v[e]));
    const int e = block_scale(lanes_max<16>(amax));
    if (b >= p.blocks || n <= 0) return;
    const float s = power_of_two(254 - e);
    i32x2 q;
    q[0] = to_fp8x4(v[0] * s, v[1] * s, v[2] * s, v[3] * s);
    q[1] = to_fp8x4(v[4] * s, v[5] * s, v[6] * s, v[7] * s);
    *reinterpret_cast<i32x2 *>(y + row * p.ldy + c) = q;
    if ((threadIdx.x & 15) == 0) scales[row * p.lds + blk] = uint8_t(e);
}

// A weight matrix in 8 bits, a scale for each 128 x 128 elements: one block each, a
// thread 8 rows' 8 elements (rows threadIdx / 16 + 16 i).
template <typename T>
__global__ void __launch_bounds__(256)
quantize_weights_kernel(const T *__restrict__ w, uint8_t *__restrict__ y, uint8_t *__restrict__ scales, int rows, int cols,
                        int64_t ldw, int64_t ldy, int64_t lds)
{
    __shared__ float red[4];
    const int c = int(blockIdx.x) * kScaleBlock + int(threadIdx.x & 15) * 8, n = cols - c;
    const int r0 = int(blockIdx.y) * kScaleBlock + int(threadIdx.x >> 4);
    float v[8][8];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        if (r < rows && n > 0) load8(w + r * ldw + c, n, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(v[i][e]));
    }
    amax = lanes_max<64>(amax);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    __syncthreads();
    const int e = block_scale(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float s = power_of_two(254 - e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        if (r >= rows || n <= 0) continue;
        i32x2 q;
        q[0] = to_fp8x4(v[i][0] * s, v[i][1] * s, v[i][2] * s, v[i][3] * s);
        q[1] = to_fp8x4(v[i][4] * s, v[i][5] * s, v[i][6] * s, v[i][7] * s);
        *reinterpret_cast<i32x2 *>(y + r * ldy + c) = q;
    }
    if (threadIdx.x == 0) scales[int64_t(blockIdx.y) * lds + blockIdx.x] = uint8_t(e);
}

// Shift codes as E5M2 numbers, which hold +-2^0 .. +-2^-14 and 0 exactly (2^-14 is
// the least normal one): exponent field 15 - shift, mantissa 0. 8 codes a thread.
__global__ void __launch_bounds__(256)
shift_to_fp8_kernel(const uint32_t *__restrict__ wp, uint8_t *__restrict__ y, int cols, int wpr, int64_t ldy, const CodeFmt fmt)
{
    const int64_t row = blockIdx.y;
    const uint32_t c = (blockIdx.x * 256 + threadIdx.x) * 8, n = uint32_t(cols);      // (c: up to 2^31)
    if (c >= n) return;
    uint32_t q[2] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t code = c + i < n ? fmt.at(wp + row * wpr, int(c + i)) : 15u, sh = code & 15u;
        const uint32_t byte = sh == 15u ? 0u : (code >> 4) << 7 | (15u - sh) << 2;
        q[i >> 2] |= byte << (8 * (i & 3));
    }
    *reinterpret_cast<i32x2 *>(y + row * ldy + c) = i32x2{int(q[0]), int(q[1])};
}

// ---------------------------------------------------------------------------

// Threads and vectors per row: a wave holds rows of up to 1024 elements, four waves
// up to 2048, eight up to 16384, sixteen up to 65536. Norm with residual, 16 bits to 8: 16384 rows of
// 512 take 11.4 us, by four waves 19.8; 8192 of 1024 11.6 and 13.2 (8 of 1000: 3.5 and 3.1); 8192 of
// 2048 19.5, by one wave 21.6; 8 of 4096 3.3, by four waves 3.7 (8192 of them 39.7 and 38.7); 4096 of
// 8192 38.8, by sixteen 41.6 (of 16384: 87 and 84).
template <typename F>
bool for_row_layout(int64_t cols, F &&f)
{
#define DS_TRY(TPR, NV) \
    if (cols <= int64_t(TPR) * NV * 8) return f(std::integral_constant<int, TPR>{}, std::integral_constant<int, NV>{}), true
    DS_TRY(64, 1);
    DS_TRY(64, 2);
    DS_TRY(256, 1);
    DS_TRY(512, 1);
    DS_TRY(512, 2);
    DS_TRY(512, 4);
    DS_TRY(1024, 4);
    DS_TRY(1024, 8);
#undef DS_TRY
    return false;
}
constexpr int64_t kMaxCols = 65536;

// f with the element type of `type`, and of weights (x's type or float32).
template <typename F>
void for_type(int32_t type, F &&f)
{
    if (type == DS_TYPE_F32) f(float{});
    else if (type == DS_TYPE_F16) f(_Float16{});
    else f(__bf16{});
}

template <typename F>
void for_types(int32_t type, int32_t wtype, F &&f)
{
    for_type(type, [&](auto t) {
        if (wtype == DS_TYPE_F32) f(t, float{});
        else f(t, t);
    });
}

ds_status check_rows(int64_t rows, int64_t cols, int32_t type)
{
    if (rows < 0 || cols <= 0) return fail(DS_ERR_INVALID_SHAPE, "rows must be >= 0 and cols > 0");
    if (!float_bytes(type)) return fail(DS_ERR_INVALID_ARG, "type must be DS_TYPE_F32, DS_TYPE_F16 or DS_TYPE_BF16");
    if (rows > kMaxElems || cols > kMaxElems || prod({std::max<int64_t>(rows, 1), cols}) > (int64_t(1) << 40))
        return fail(DS_ERR_UNSUPPORTED, "2^31 or more rows or columns, or over 2^40 elements");
    return DS_SUCCESS;
}

// An 8-bit matrix: rows that begin on 16 bytes (and so are readable to a multiple of 16).
ds_status check_rows8(const void *p, int64_t cols, int64_t ld, int64_t lds, int64_t blocks)
{
    if (ld < (cols + 15) / 16 * 16 || ld % 16 || reinterpret_cast<uintptr_t>(p) % 16)
        return fail(DS_ERR_INVALID_ARG, "8-bit rows must begin on 16 bytes and be a multiple of 16 apart, at least the columns");
    if (lds < blocks) return fail(DS_ERR_INVALID_ARG, "fewer scales in a row than blocks of 128");
    return DS_SUCCESS;
}

int64_t blocks_of(int64_t cols) { return (cols + kScaleBlock - 1) / kScaleBlock; }

// Blocks of the gradient's launch, a row of dweight's shares each (times the rows that
// a block takes at once): one a CU. 8192 x 4096 elements 46 us, with 512 blocks 51, 1024 55; 16384 x
// 1024 29, 32 and 41.
int norm_grad_blocks(int64_t rows, int64_t cols)
{
    const int64_t per = cols <= 1024 ? 4 : 1;
    return int(std::min<int64_t>((rows + per - 1) / per, 256));
}

}  // namespace

}  // namespace ds

using namespace ds;

extern "C" ds_status ds_rms_norm(const void *x, const void *residual, const void *weight, void *y, uint8_t *scales, void *h,
                                 float *rstd, int64_t rows, int64_t cols, int64_t ldx, int64_t ldr, int64_t ldh,
                                 int64_t ldy, int64_t lds, float eps, int32_t type, int32_t weight_type, int32_t y_type,
                                 void *stream)
{
    if (rows != 0 && (!x || !weight || !y || (residual && !h)))
        return fail(DS_ERR_NULL_POINTER, "x, weight, y (and h with a residual) must not be NULL");
    if (rows != 0 && h && !residual) return fail(DS_ERR_INVALID_ARG, "h is written with a residual only");
    if (ds_status st = check_rows(rows, cols, type)) return st;
    if (cols > kMaxCols) return fail(DS_ERR_UNSUPPORTED, "more than %lld columns", (long long)kMaxCols);
    if (weight_type != type && weight_type != DS_TYPE_F32) return fail(DS_ERR_INVALID_ARG, "weight must have x's type or float32");
    if (y_type != type && y_type != DS_TYPE_F8E4M3) return fail(DS_ERR_INVALID_ARG, "y must have x's type or DS_TYPE_F8E4M3");
    if (!(eps >= 0.f)) return fail(DS_ERR_INVALID_ARG, "eps must be >= 0");
    const bool quant = y_type == DS_TYPE_F8E4M3;
    if (ldx < cols || (residual && (ldr < cols || ldh < cols)) || (!quant && ldy < cols))
        return fail(DS_ERR_INVALID_ARG, "a row's stride is shorter than the row");
    if (quant) {
        if (rows != 0 && !scales) return fail(DS_ERR_NULL_POINTER, "an 8-bit y needs scales");
        if (ds_status st = check_rows8(y, cols, ldy, lds, blocks_of(cols))) return st;
    }
    bool fits = true;
    for_row_layout(cols, [&](auto tpr, auto) {
        constexpr int block = row_block<decltype(tpr)::value>(), per = block / decltype(tpr)::value;
        fits = grid_fits((rows + per - 1) / per, block);
    });
    if (!fits) return fail(DS_ERR_UNSUPPORTED, "too many rows for a launch");
    if (rows == 0) return ok();
    const int64_t es = float_bytes(type);
    if (ds_status st = check_tensors({{x, span(rows, ldx, cols, es), "x", false},
                                      {residual, span(rows, ldr, cols, es), "residual", false},
                                      {weight, cols * float_bytes(weight_type), "weight", false},
                                      {y, quant ? span(rows, ldy, (cols + 7) / 8 * 8) : span(rows, ldy, cols, es), "y", true},
                                      {quant ? scales : nullptr, span(rows, lds, blocks_of(cols)), "scales", true},
                                      {h, span(rows, ldh, cols, es), "h", true},
                                      {rstd, rows * 4, "rstd", true}}))
        return st;
    const NormParams p{rows, ldx, ldr, ldh, ldy, lds, int(cols), eps};
    for_types(type, weight_type, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        for_row_layout(cols, [&](auto tpr, auto nv) {
            constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
            const auto k = cols % 8 ? (quant ? norm_kernel<T, W, TPR, NV, true, false> : norm_kernel<T, W, TPR, NV, false, false>)
                                    : (quant ? norm_kernel<T, W, TPR, NV, true, true> : norm_kernel<T, W, TPR, NV, false, true>);
            constexpr int block = row_block<TPR>(), per = block / TPR;
            hipLaunchKernelGGL(k, dim3(uint32_t((rows + per - 1) / per)), dim3(block), 0, static_cast<hipStream_t>(stream),
                               static_cast<const T *>(x), static_cast<const T *>(residual), static_cast<const W *>(weight), y,
                               scales, static_cast<T *>(h), rstd, p);
        });
    });
    return launched("ds_rms_norm");
}

extern "C" int64_t ds_rms_norm_backward_scratch_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || cols > kMaxCols) return 0;
    return int64_t(norm_grad_blocks(rows, cols)) * (cols <= 1024 ? 4 : 1) * cols * 4;
}

extern "C" ds_status ds_rms_norm_backward(const void *dy, const void *h, const void *weight, const float *rstd, const void *dh,
                                          void *dx, void *dweight, int64_t rows, int64_t cols, int64_t lddy, int64_t ldh,
                                          int64_t lddh, int64_t lddx, int32_t type, int32_t weight_type, void *scratch,
                                          int64_t scratch_bytes, void *stream)
{
    if (rows != 0 && (!dy || !h || !weight || !rstd || !dx))
        return fail(DS_ERR_NULL_POINTER, "dy, h, weight, rstd and dx must not be NULL");
    if (ds_status st = check_rows(rows, cols, type)) return st;
    if (cols > kMaxCols) return fail(DS_ERR_UNSUPPORTED, "more than %lld columns", (long long)kMaxCols);
    if (weight_type != type && weight_type != DS_TYPE_F32) return fail(DS_ERR_INVALID_ARG, "weight must have dy's type or float32");
    if (lddy < cols || ldh < cols || (dh && lddh < cols) || lddx < cols)
        return fail(DS_ERR_INVALID_ARG, "a row's stride is shorter than the row");
    const int64_t need = dweight ? ds_rms_norm_backward_scratch_bytes(rows, cols) : 0;
    if (need > 0 && !scratch) return fail(DS_ERR_NULL_POINTER, "dweight needs scratch");
    if (need > scratch_bytes) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    const int64_t es = float_bytes(type);
    if (ds_status st = check_tensors({{dy, span(rows, lddy, cols, es), "dy", false},
                                      {h, span(rows, ldh, cols, es), "h", false},
                                      {weight, cols * float_bytes(weight_type), "weight", false},
                                      {rstd, rows * 4, "rstd", false},
                                      {dh, span(rows, lddh, cols, es), "dh", false},
                                      {dx, span(rows, lddx, cols, es), "dx", true},
                                      {dweight, cols * float_bytes(weight_type), "dweight", true},
                                      {need ? scratch : nullptr, need, "scratch", true}}))
        return st;
    const auto s = static_cast<hipStream_t>(stream);
    const int blocks = norm_grad_blocks(rows, cols), parts = blocks * (cols <= 1024 ? 4 : 1);
    const NormGradParams p{rows, lddy, ldh, lddh, lddx, int(cols)};
    for_types(type, weight_type, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        if (rows > 0)
            for_row_layout(cols, [&](auto tpr, auto nv) {
                constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
                const auto k = cols % 8 ? norm_grad_kernel<T, W, TPR, NV, false> : norm_grad_kernel<T, W, TPR, NV, true>;
                hipLaunchKernelGGL(k, dim3(blocks), dim3(row_block<TPR>()), 0, s, static_cast<const T *>(dy), static_cast<const T *>(h),
                                   static_cast<const W *>(weight), rstd, static_cast<const T *>(dh), static_cast<T *>(dx),
                                   dweight ? static_cast<float *>(scratch) : nullptr, p);
            });
        if (dweight)
            hipLaunchKernelGGL(norm_grad_weight_kernel<W>, dim3(uint32_t((cols + 31) / 32)), dim3(1024), 0, s,
                               static_cast<const float *>(scratch), static_cast<W *>(dweight), rows > 0 ? parts : 0, int(cols));
    });
    return launched("ds_rms_norm_backward");
}

extern "C" ds_status ds_quantize_fp8(const void *x, const void *gate, uint8_t *y, uint8_t *scales, int64_t rows, int64_t cols,
                                     int64_t ldx, int64_t ldg, int64_t ldy, int64_t lds, int32_t type, void *stream)
{
    if (rows != 0 && (!x || !y || !scales)) return fail(DS_ERR_NULL_POINTER, "x, y and scales must not be NULL");
    if (ds_status st = check_rows(rows, cols, type)) return st;
    if (ldx < cols || (gate && ldg < cols)) return fail(DS_ERR_INVALID_ARG, "a row's stride is shorter than the row");
    const int64_t nb = blocks_of(cols);
    if (ds_status st = check_rows8(y, cols, ldy, lds, nb)) return st;
    if (!grid_fits((rows * nb + 15) / 16, 256)) return fail(DS_ERR_UNSUPPORTED, "2^28 or more scales");
    if (rows == 0) return ok();
    const int64_t es = float_bytes(type);
    if (ds_status st = check_tensors({{x, span(rows, ldx, cols, es), "x", false},
                                      {gate, span(rows, ldg, cols, es), "gate", false},
                                      {y, span(rows, ldy, (cols + 7) / 8 * 8), "y", true},
                                      {scales, span(rows, lds, nb), "scales", true}}))
        return st;
    const QuantParams p{ldx, ldg, ldy, lds, int(cols), int(rows * nb), make_fastdiv(uint32_t(nb))};
    for_type(type, [&](auto t) {
        using T = decltype(t);
        const auto k = gate ? quantize_kernel<T, true> : quantize_kernel<T, false>;
        hipLaunchKernelGGL(k, dim3(uint32_t((rows * nb + 15) / 16)), dim3(256), 0, static_cast<hipStream_t>(stream),
                           static_cast<const T *>(x), static_cast<const T *>(gate), y, scales, p);
    });
    return launched("ds_quantize_fp8");
}

extern "C" ds_status ds_quantize_weights_fp8(const void *w, uint8_t *w8, uint8_t *scales, int64_t rows, int64_t cols,
                                             int64_t ldw, int64_t ldw8, int64_t lds, int32_t type, void *stream)
{
    if (!w || !w8 || !scales) return fail(DS_ERR_NULL_POINTER, "w, w8 and scales must not be NULL");
    if (rows == 0) return fail(DS_ERR_INVALID_SHAPE, "rows must be > 0");
    if (ds_status st = check_rows(rows, cols, type)) return st;
    if (ldw < cols) return fail(DS_ERR_INVALID_ARG, "a row's stride is shorter than the row");
    const int64_t nb = blocks_of(cols), rb = blocks_of(rows);
    if (ds_status st = check_rows8(w8, cols, ldw8, lds, nb)) return st;
    if (rb > 65535 || !grid_fits(nb, 256)) return fail(DS_ERR_UNSUPPORTED, "more than 65535 x 128 rows, or 2^24 or more x 128 columns");
    const int64_t es = float_bytes(type);
    if (ds_status st = check_tensors({{w, span(rows, ldw, cols, es), "w", false},
                                      {w8, span(rows, ldw8, (cols + 7) / 8 * 8), "w8", true},
                                      {scales, span(rb, lds, nb), "scales", true}}))
        return st;
    for_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(quantize_weights_kernel<T>, dim3(uint32_t(nb), uint32_t(rb)), dim3(256), 0,
                           static_cast<hipStream_t>(stream), static_cast<const T *>(w), w8, scales, int(rows), int(cols), ldw,
                           ldw8, lds);
    });
    return launched("ds_quantize_weights_fp8");
}

extern "C" ds_status ds_shift_weights_to_fp8(const uint32_t *w_packed, uint8_t *w8, int64_t rows, int64_t cols, int64_t ldw8,
                                             uint32_t flags, void *stream)
{
    if (!w_packed || !w8) return fail(DS_ERR_NULL_POINTER, "w_packed and w8 must not be NULL");
    if (rows <= 0 || cols <= 0) return fail(DS_ERR_INVALID_SHAPE, "rows and cols must be > 0");
    if (flags & ~0xF00u) return fail(DS_ERR_INVALID_ARG, "unknown flags 0x%x", flags);
    const int bits = flags_code_bits(flags);
    if (bits < 0) return fail(DS_ERR_INVALID_ARG, "DS_CODE_BITS must be 2..5 (or 0 for 5)");
    if (prod({rows, cols}) < 0 || prod({rows, cols}) > kMaxElems || rows > 65535)
        return fail(DS_ERR_UNSUPPORTED, "2^31 or more weights, or more than 65535 rows");
    if (ds_status st = check_rows8(w8, cols, ldw8, 0, 0)) return st;
    const int64_t wpr = row_words_bits(cols, bits);
    if (ds_status st = check_tensors({{w_packed, rows * wpr * 4, "w_packed", false},
                                      {w8, span(rows, ldw8, (cols + 7) / 8 * 8), "w8", true}}))
        return st;
    hipLaunchKernelGGL(shift_to_fp8_kernel, dim3(uint32_t((cols + 2047) / 2048), uint32_t(rows)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), w_packed, w8, int(cols), int(wpr), ldw8, code_fmt(bits));
    return launched("ds_shift_weights_to_fp8");
}
