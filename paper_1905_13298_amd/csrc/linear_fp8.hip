// The product of 8-bit matrices with power-of-two block scales, and its input gradient.
//
//   y[m][n] = bias[n] + sum over blocks b of 128 of
//             2^(xs[m][b] + ws[n / 128][b] - 254) * sum_{k in b} x8[m][k] * w8[n][k]
//
// x8 in E4M3 with a scale for each row and 128 elements, w8 in E4M3 or E5M2 with a
// scale for each 128 x 128 elements. The scales are the matrix instruction's own block
// scale operands, so they cost no instruction and the sums stay in 32-bit accumulators
// from the first element to the last.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "conv_plan.hpp"
#include "fp8.hpp"

namespace ds {

namespace {

struct LinearParams {
    const uint8_t *x, *xs, *w, *ws;
    const float *bias;
    void *y;
    int m, n, k, kblocks;
    int64_t ldx, ldxs, ldw, ldws, ldy;
};

// 16 bytes of a row from element k on; bytes past `cols` are 0 (the row's first bytes
// are read in place of a piece that begins past the end).
__device__ __forceinline__ i32x4 row16(const uint8_t *row, int k, int cols)
{
    const int n = cols - k;
    i32x4 v = *reinterpret_cast<const i32x4 *>(row + (n > 0 ? k : 0));
    if (n < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int left = n - 4 * i;
            v[i] = left >= 4 ? v[i] : left <= 0 ? 0 : v[i] & int((1u << (8 * left)) - 1u);
        }
    }
    return v;
}

__device__ __forceinline__ i32x8 whole32(const uint8_t *p)
{
    const i32x4 a = *reinterpret_cast<const i32x4 *>(p), b = *reinterpret_cast<const i32x4 *>(p + 16);
    return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

__device__ __forceinline__ i32x8 row32(const uint8_t *row, int k, int cols)
{
    const i32x4 a = row16(row, k, cols), b = row16(row, k + 16, cols);
    return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// 8 of a lane's 32 elements as 16-bit floats, exactly (WF 0: E4M3, 1: E5M2).
template <int WF>
__device__ __forceinline__ f16x8 widen(i32x8 v, int i)
{
    f16x8 o;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        f16x2 a, b;
        if constexpr (WF == 0) {
            a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * i + j], 1.f, false);
            b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * i + j], 1.f, true);
        } else {
            a = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(v[2 * i + j], 1.f, false);
            b = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(v[2 * i + j], 1.f, true);
        }
        o[4 * j] = a[0];
        o[4 * j + 1] = a[1];
        o[4 * j + 2] = b[0];
        o[4 * j + 3] = b[1];
    }
    return o;
}

// c + one block's products. The 8-bit instruction aligns the products of each 8 elements with
// the largest of them and drops what lies 2^-14 below it. For normal inputs, 128 to 11008 elements
// of them, that is 2.8e-5 of the outputs' root mean square (E4M3 weights) or 6.5e-5 (E5M2) without a
// bias: a 60th or a 25th of what rounding to bfloat16 costs, an 8th or a third for a 16-bit float. An
// output of 32 bits would show it: it (FULL) is formed from the same numbers as 16-bit floats, whose
// products and sums keep 24 bits, the scales applied afterwards.
// The scales are byte BYTE of ws and xs.
template <int WF, bool FULL, int BYTE = 0>
__device__ __forceinline__ f32x4 mma(i32x8 w, i32x8 x, f32x4 c, int ws, int xs)
{
    if constexpr (FULL) {
        f32x4 part{};
#pragma unroll
        for (int i = 0; i < 4; ++i) part = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<WF>(w, i), widen<0>(x, i), part, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] += ldexpf(part[i], (ws >> (8 * BYTE) & 255) + (xs >> (8 * BYTE) & 255) - 254);
        return c;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, WF, 0, BYTE, ws, BYTE, xs);
    }
}

// Four scale bytes of a row, of blocks b .. b + 3 (those past the last hold anything): as
// they are read, and in place once they are there.
__device__ __forceinline__ uint32_t load_scales4(const uint8_t *row, int b, int blocks)
{
    uint32_t v = 0;
    if (blocks >= 4) {
        __builtin_memcpy(&v, row + min(b, blocks - 4), 4);
    } else {
        for (int i = 0; i < blocks; ++i) v |= uint32_t(row[i]) << (8 * i);
    }
    return v;
}

__device__ __forceinline__ uint32_t place_scales4(uint32_t v, int b, int blocks)
{
    return blocks >= 4 ? v >> (8 * max(b - (blocks - 4), 0)) : v;
}

// Whether one of the first n scale bytes of a word is 255, no number. The 8-bit instruction makes
// products of NaN of it by itself; sums of 16-bit products (FULL) are struck out once for the
// word's blocks, in a branch (a test in every block took 9 % of 1000 x 4096 outputs of 4096).
__device__ __forceinline__ bool no_number(uint32_t word, int n)
{
    const uint32_t z = ~word | (n >= 4 ? 0u : 0xffffffffu << (8 * n));
    return ((z - 0x01010101u) & ~z & 0x80808080u) != 0;
}

// Few rows of x: the weights go from memory to registers, once. A block takes 16 rows of
// w and MT x 16 rows of x; each of its waves takes a share of the reduction, in blocks of 128,
// and they add their sums in LDS. The weights are the instruction's first operand, so that a
// lane ends up with four consecutive outputs of one row of y. Bound by the latency of reading
// w: 8 x 4096 outputs of 4096, 17 MB, 6.6 us (2.6 TB/s; the launch and the sums' exchange are about 3
// of them); with more rows by the loads of x, which every block repeats.
template <typename O, int WF, int MT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
linear_rows_kernel(const LinearParams p)
{
    __shared__ f32x4 sums[WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int n0 = int(blockIdx.x) * 16, m0 = int(blockIdx.y) * 16 * MT;
    const uint8_t *wrow = p.w + int64_t(min(n0 + r, p.n - 1)) * p.ldw;
    const uint8_t *wsrow = p.ws + int64_t(n0 / kScaleBlock) * p.ldws;
    const uint8_t *xrow[MT], *xsrow[MT];
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = min(m0 + t * 16 + r, p.m - 1);
        xrow[t] = p.x + m * p.ldx;
        xsrow[t] = p.xs + m * p.ldxs;
        acc[t] = f32x4{};
    }
    // Four whole blocks at a time, their loads before their products and their scales as one
    // word (bytes by themselves took a fifth of the time at 64 rows); others one by one.
    const int full = p.k / kScaleBlock, each = (p.kblocks + WAVES - 1) / WAVES, end = min(p.kblocks, (wave + 1) * each);
    for (int b = wave * each; b < end;) {
        if (b + 4 <= min(end, full)) {
            i32x8 w[4], x[4][MT];
            uint32_t ws = load_scales4(wsrow, b, p.kblocks), xs[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) xs[t] = load_scales4(xsrow[t], b, p.kblocks);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int k = (b + u) * kScaleBlock + g * 32;
                w[u] = whole32(wrow + k);
#pragma unroll
                for (int t = 0; t < MT; ++t) x[u][t] = whole32(xrow[t] + k);
            }
            ws = place_scales4(ws, b, p.kblocks);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const uint32_t s = place_scales4(xs[t], b, p.kblocks);
                acc[t] = mma<WF, sizeof(O) == 4, 0>(w[0], x[0][t], acc[t], int(ws), int(s));
                acc[t] = mma<WF, sizeof(O) == 4, 1>(w[1], x[1][t], acc[t], int(ws), int(s));
                acc[t] = mma<WF, sizeof(O) == 4, 2>(w[2], x[2][t], acc[t], int(ws), int(s));
                acc[t] = mma<WF, sizeof(O) == 4, 3>(w[3], x[3][t], acc[t], int(ws), int(s));
                if (sizeof(O) == 4 && (no_number(ws, 4) || no_number(s, 4))) acc[t] += __builtin_nanf("");
            }
            b += 4;
        } else {
            const int k = b * kScaleBlock + g * 32;
            const i32x8 w = row32(wrow, k, p.k);
            const int ws = wsrow[b];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int s = xsrow[t][b];
                acc[t] = mma<WF, sizeof(O) == 4>(w, row32(xrow[t], k, p.k), acc[t], ws, s);
                if (sizeof(O) == 4 && max(ws, s) == 255) acc[t] += __builtin_nanf("");
            }
            ++b;
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < MT; t += WAVES) {
        f32x4 s = sums[0][t][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) s += sums[i][t][lane];
        const int m = m0 + t * 16 + r, n = n0 + g * 4;
        if (m >= p.m) continue;
        O *y = static_cast<O *>(p.y) + m * p.ldy + n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.n) y[i] = O(s[i] + (p.bias ? p.bias[n + i] : 0.f));
    }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t *p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, int(bytes), 0x00020000);
}

// Where a lane's 16 bytes of a step are, or, past the reduction's end, an offset outside every
// buffer: zeros are put there. A step is sent for in the same way whether it is whole, the last
// or past it, since a branch in the loop would have the compiler move products behind it.
__device__ __forceinline__ int inside(int offset, bool in) { return in ? offset : 0x7ffffff0; }

// The scalar offset of a step: the last step's for those past it. The range check takes it off the
// buffer's size, which may be as little as one row, so it has to stay within that.
__device__ __forceinline__ int step_offset(int step, int steps) { return min(step, steps - 1) * 128; }

// A reduction that ends inside a lane's 16 bytes: the bytes past its end, in LDS.
__device__ __forceinline__ void clear_past(uint8_t *at, int left)
{
    if (left <= 0 || left >= 16) return;
    i32x4 v = *reinterpret_cast<const i32x4 *>(at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = left - 4 * i;
        v[i] = n >= 4 ? v[i] : n <= 0 ? 0 : v[i] & int((1u << (8 * n)) - 1u);
    }
    *reinterpret_cast<i32x4 *>(at) = v;
}

// Four consecutive outputs of a row of y.
template <typename O>
__device__ __forceinline__ void store_outputs(const LinearParams &p, int m, int n, f32x4 v)
{
    O *y = static_cast<O *>(p.y) + m * p.ldy + n;
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += p.bias[min(n + i, p.n - 1)];
    }
    O o[4] = {O(v[0]), O(v[1]), O(v[2]), O(v[3])};
    if (n + 4 <= p.n) {
        __builtin_memcpy(y, o, sizeof o);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.n) y[i] = o[i];
    }
}

// Many rows of x: a block forms BN outputs of BM rows of y, 128 elements of the reduction
// at a time, which go from memory to LDS without registers, STAGES - 1 steps ahead of the
// products. A row's eight 16-byte pieces are kept in an order of its own, so that the
// lanes of a read find theirs in different banks. Bound by the transfers' latency where
// there is one round of blocks (128 x 4096 outputs of 4096, tiles of 64: 12.8 us for 32 steps), by LDS reads
// where there are more (tiles of 128, 2900 x 6000 outputs of 4096: 84 us, 1.7 PFLOP/s).
template <typename O, int WF, int BN, int BM, int WN, int WM, int STAGES>
__global__ void __launch_bounds__(64 * WN * WM, 1)
linear_tile_kernel(const LinearParams p, int tiles_n, int tiles_m)
{
    constexpr int kWaves = WN * WM, NT = BN / WN / 16, MT = BM / WM / 16;
    constexpr int kStage = (BN + BM) * 128, kLoadsW = BN / 8 / kWaves, kLoadsX = BM / 8 / kWaves, kGroup = 8;
    constexpr int kGroups = 16;                  // of 4 steps, whose scales are in LDS together
    constexpr int kWeights = (BN + 127) / 128;    // scales of w a step
    __shared__ __align__(16) uint8_t lds[STAGES * kStage];
    __shared__ uint32_t scales[kGroups][BM + kWeights];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    // Blocks are dealt to the 8 XCDs in turn: each takes a run of tiles, kGroup rows of
    // tiles at a time, so that those in flight share their inputs in its L2.
    const int tiles = tiles_n * tiles_m, share = (tiles + 7) >> 3, at = (int(blockIdx.x) & 7) * share + (int(blockIdx.x) >> 3);
    if ((int(blockIdx.x) >> 3) >= share || at >= tiles) return;
    const int band = at / (kGroup * tiles_n), in = at - band * kGroup * tiles_n, deep = min(kGroup, tiles_m - band * kGroup);
    const int n0 = in / deep * BN, m0 = (band * kGroup + in % deep) * BM;
    const int wn = wave % WN, wm = wave / WN;

    const uint8_t *wbase = p.w + n0 * p.ldw, *xbase = p.x + m0 * p.ldx;
    const int krow = (p.k + 15) & ~15;
    const __amdgpu_buffer_rsrc_t wr = rows_rsrc(wbase, (min(BN, p.n - n0) - 1) * p.ldw + krow);
    const __amdgpu_buffer_rsrc_t xr = rows_rsrc(xbase, (min(BM, p.m - m0) - 1) * p.ldx + krow);
    const int ldw = int(p.ldw), ldx = int(p.ldx);
    const int lrow = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;
    int wv[kLoadsW], xv[kLoadsX];      // rows past the last read it instead
#pragma unroll
    for (int i = 0; i < kLoadsW; ++i) wv[i] = min(i * kWaves * 8 + lrow, p.n - 1 - n0) * ldw + piece;
#pragma unroll
    for (int i = 0; i < kLoadsX; ++i) xv[i] = min(i * kWaves * 8 + lrow, p.m - 1 - m0) * ldx + piece;
    const uint32_t base_lds = __builtin_amdgcn_readfirstlane(lds_address(lds));
    auto stage = [&](int step, int buf) {
        const int k = step_offset(step, p.kblocks);
        const bool in = step * 128 + piece < p.k;
#pragma unroll
        for (int i = 0; i < kLoadsW; ++i)
            to_lds16(base_lds + buf * kStage + (i * kWaves + wave) * 1024, wr, inside(wv[i], in), k);
#pragma unroll
        for (int i = 0; i < kLoadsX; ++i)
            to_lds16(base_lds + buf * kStage + (BN / 8 + i * kWaves + wave) * 1024, xr, inside(xv[i], in), k);
    };
    // The scales of the block's rows (of w's, by 128) for 64 steps from `step` on, four a word.
    auto fetch_scales = [&](int step) {
        constexpr int kRows = BM + kWeights;
        const int groups = min(kGroups, (p.kblocks - step + 3) / 4);
#pragma unroll 4
        for (int i = threadIdx.x; i < kRows * groups; i += 64 * kWaves) {
            const int gr = i / kRows, row = i - gr * kRows, at = step + 4 * gr;
            const uint8_t *src = row < BM ? p.xs + min(m0 + row, p.m - 1) * p.ldxs : p.ws + min(n0 / 128 + row - BM, (p.n - 1) / 128) * p.ldws;
            scales[gr][row] = place_scales4(load_scales4(src, at, p.kblocks), at, p.kblocks);
        }
    };
    uint32_t xs[MT], ws;
    f32x4 acc[NT][MT];
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < MT; ++b) acc[a][b] = f32x4{};

#pragma unroll
    for (int i = 0; i < STAGES; ++i) stage(i, i);
    fetch_scales(0);
    wait_all();
    barrier();
    const int so = r * 128 + (g ^ (r >> 1)) * 16, s1 = so ^ 64;      // pieces g and g + 4
    auto frag = [&](const uint8_t *base, int t) {
        const i32x4 a = *reinterpret_cast<const i32x4 *>(base + t * 2048 + so), b = *reinterpret_cast<const i32x4 *>(base + t * 2048 + s1);
        return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    };
    const uint8_t *const wt = lds + wn * NT * 2048, *const xt = lds + BN * 128 + wm * MT * 2048;
    i32x8 wf[NT], x;
#pragma unroll
    for (int a = 0; a < NT; ++a) wf[a] = frag(wt, a);
    x = frag(xt, 0);
    // A step: rows of tiles of x one after the other, the next one's elements read ahead.
    // Before the last row's products every element of this step has been read: one barrier
    // says so and that the next step's have arrived. Behind it, the step after the next is
    // sent for, and each of the last products is followed by the read of the next step's
    // weights into the registers that it leaves.
    const bool partial = p.k % 16 != 0;
    for (int step = 0; step < p.kblocks; ++step) {
        const int buf = step % STAGES, following = buf + 1 < STAGES ? buf + 1 : 0;
        if (partial && step + 1 == p.kblocks) {
#pragma unroll
            for (int i = 0; i < kLoadsW + kLoadsX; ++i)
                clear_past(lds + buf * kStage + (i * kWaves + wave) * 1024 + lane * 16, p.k - step * 128 - piece);
            wait_lds();
            barrier();
#pragma unroll
            for (int a = 0; a < NT; ++a) wf[a] = frag(wt + buf * kStage, a);
            x = frag(xt + buf * kStage, 0);
        }
        if ((step & 3) == 0) {
            if ((step & (4 * kGroups - 1)) == 0 && step > 0) {
                barrier();
                fetch_scales(step);
                wait_lds();
                barrier();
            }
            const uint32_t *from = scales[(step >> 2) & (kGroups - 1)];
#pragma unroll
            for (int t = 0; t < MT; ++t) xs[t] = from[(wm * MT + t) * 16 + r];
            ws = from[BM + wn * NT / 8];
            if constexpr (sizeof(O) == 4) {
                bool out = no_number(ws, p.kblocks - step);
#pragma unroll
                for (int t = 0; t < MT; ++t) out = out || no_number(xs[t], p.kblocks - step);
                if (__any(out)) {
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        const float by = no_number(ws, p.kblocks - step) || no_number(xs[t], p.kblocks - step) ? __builtin_nanf("") : 0.f;
#pragma unroll
                        for (int a = 0; a < NT; ++a) acc[a][t] += by;
                    }
                }
            }
        }
        const uint8_t *const xb = xt + buf * kStage, *const wnext = wt + following * kStage;
#pragma unroll
        for (int b = 0; b + 1 < MT; ++b) {
            const i32x8 ahead = frag(xb, b + 1);
#pragma unroll
            for (int a = 0; a < NT; ++a) acc[a][b] = mma<WF, sizeof(O) == 4>(wf[a], x, acc[a][b], int(ws), int(xs[b]));
            x = ahead;
            __builtin_amdgcn_sched_barrier(0);
        }
        // The transfers of the steps behind the next one may be on their way.
        wait_but<(STAGES - 2) * (kLoadsW + kLoadsX)>();
        barrier();
        stage(step + STAGES, buf);
        // (After the last step these reads are of LDS that nothing uses any more.)
        const i32x8 ahead = frag(xt + following * kStage, 0);
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            acc[a][MT - 1] = mma<WF, sizeof(O) == 4>(wf[a], x, acc[a][MT - 1], int(ws), int(xs[MT - 1]));
            wf[a] = frag(wnext, a);
            __builtin_amdgcn_sched_barrier(0);
        }
        x = ahead;
        ws >>= 8;
#pragma unroll
        for (int t = 0; t < MT; ++t) xs[t] >>= 8;
    }
    wait_all();     // no transfer may outlive the block's LDS
#pragma unroll
    for (int b = 0; b < MT; ++b) {
        const int m = m0 + (wm * MT + b) * 16 + r;
        if (m >= p.m) continue;
#pragma unroll
        for (int a = 0; a < NT; ++a) store_outputs<O>(p, m, n0 + (wn * NT + a) * 16 + g * 4, acc[a][b]);
    }
}

// A large product: 256 x 256 outputs a block, 128 x 128 a wave, as linear_tile_kernel with
// more of the reduction on its way. A step's elements of x come in two halves (the first
// four tiles of 16 rows of every wave, and the last four), which go through five places in
// turn; those of w go through two and into registers before their step. A half's place is
// free when its last elements have been read, so there are two barriers a step: from the last
// products of the first half on, the next but one step's second half and weights are sent
// for, among those of the second half's last row the first half of the step after that, a transfer
// behind every two or three products (all at once: 247 us for 233). What a step waits for was
// sent for about a step before (a step takes 1.1 us at the least, memory behind the L2 answers
// after up to 2). Bound by the matrix instructions, at
// the clock that the card holds while they run, and by a block's start and end, which nothing
// overlaps: 8192 x 8192 outputs of 4096 in 229 to 236 us (2.4 PFLOP/s).
template <typename O, int WF>
__global__ void __launch_bounds__(256, 1)
linear_wide_kernel(const LinearParams p, int tiles_n, int tiles_m)
{
    constexpr int B = 256, NT = 8, MT = 8, kW = B * 128, kHalf = kW / 2, kPlaces = 5, kGroup = 4, kGroups = 8;
    __shared__ __align__(16) uint8_t lds[2 * kW + kPlaces * kHalf];
    __shared__ uint32_t scales[kGroups][B + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const int tiles = tiles_n * tiles_m, share = (tiles + 7) >> 3, at = (int(blockIdx.x) & 7) * share + (int(blockIdx.x) >> 3);
    if ((int(blockIdx.x) >> 3) >= share || at >= tiles) return;
    const int band = at / (kGroup * tiles_n), in = at - band * kGroup * tiles_n, deep = min(kGroup, tiles_m - band * kGroup);
    const int n0 = in / deep * B, m0 = (band * kGroup + in % deep) * B;
    const int wn = wave & 1, wm = wave >> 1;

    const uint8_t *wbase = p.w + n0 * p.ldw, *xbase = p.x + m0 * p.ldx;
    const int krow = (p.k + 15) & ~15, nlast = min(B, p.n - n0) - 1, mlast = min(B, p.m - m0) - 1;
    const __amdgpu_buffer_rsrc_t wr = rows_rsrc(wbase, nlast * p.ldw + krow), xr = rows_rsrc(xbase, mlast * p.ldx + krow);
    const int lrow = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;
    // Load i of a wave: rows i * 32 + lrow of w; row i * 32 + lrow of a half of x is row 64 (i /
    // 2) past it (a wave's half has 64 rows), and 64 more in the second half. Rows past the last
    // read it instead.
    auto xrow = [&](int half, int i) { return min(i / 2 * 128 + i % 2 * 32 + half * 64 + lrow, mlast); };
    int wv[8], xv[2][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) wv[i] = min(i * 32 + lrow, nlast) * int(p.ldw) + piece;
#pragma unroll
    for (int i = 0; i < 8; ++i) xv[i / 4][i % 4] = xrow(i / 4, i % 4) * int(p.ldx) + piece;
    const uint32_t base_lds = __builtin_amdgcn_readfirstlane(lds_address(lds));
    // Load i of a step's weights, or of a half of its elements of x.
    auto fetch_w = [&](int step, int i) {
        to_lds16(base_lds + (step & 1) * kW + (i * 4 + wave) * 1024, wr, inside(wv[i], step * 128 + piece < p.k),
                 step_offset(step, p.kblocks));
    };
    auto fetch_x = [&](int step, int half, int place, int i) {
        to_lds16(base_lds + 2 * kW + place * kHalf + (i * 4 + wave) * 1024, xr, inside(xv[half][i], step * 128 + piece < p.k),
                 step_offset(step, p.kblocks));
    };
    // The scales of the block's rows (of w's, by 128) for 32 steps from `step` on, four a word.
    auto fetch_scales = [&](int step) {
        const int groups = min(kGroups, (p.kblocks - step + 3) / 4);
#pragma unroll 1
        for (int i = threadIdx.x; i < (B + 2) * groups; i += 256) {
            const int gr = i / (B + 2), row = i - gr * (B + 2), at = step + 4 * gr;
            const uint8_t *src = row < B ? p.xs + min(m0 + row, p.m - 1) * p.ldxs : p.ws + min(n0 / 128 + row - B, (p.n - 1) / 128) * p.ldws;
            scales[gr][row] = place_scales4(load_scales4(src, at, p.kblocks), at, p.kblocks);
        }
    };
    f32x4 acc[NT][MT];
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < MT; ++b) acc[a][b] = f32x4{};

#pragma unroll
    for (int i = 0; i < kPlaces * 4; ++i) fetch_x(i / 8, i / 4 % 2, i / 4, i % 4);
#pragma unroll
    for (int i = 0; i < 16; ++i) fetch_w(i / 8, i % 8);
    fetch_scales(0);
    wait_all();
    barrier();
    const int so = r * 128 + (g ^ (r >> 1)) * 16, s1 = so ^ 64;      // pieces g and g + 4
    auto frag = [&](const uint8_t *base, int t) {
        const i32x4 a = *reinterpret_cast<const i32x4 *>(base + t * 2048 + so), b = *reinterpret_cast<const i32x4 *>(base + t * 2048 + s1);
        return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    };
    const uint8_t *const wt = lds + wn * NT * 2048, *const xt = lds + 2 * kW + wm * kHalf / 2;
    i32x8 wf[NT], x;
#pragma unroll
    for (int a = 0; a < NT; ++a) wf[a] = frag(wt, a);
    x = frag(xt, 0);
    uint32_t xs[MT], ws;
    int place = 0;                                  // of this step's first half
    auto past = [&](int by) { const int q = place + by; return q >= kPlaces ? q - kPlaces : q; };
    const bool partial = p.k % 16 != 0;
    for (int step = 0; step < p.kblocks; ++step) {
        if (partial && step + 1 == p.kblocks) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                clear_past(lds + (step & 1) * kW + (i * 4 + wave) * 1024 + lane * 16, p.k - step * 128 - piece);
                clear_past(lds + 2 * kW + past(i / 4) * kHalf + (i % 4 * 4 + wave) * 1024 + lane * 16, p.k - step * 128 - piece);
            }
            wait_lds();
            barrier();
#pragma unroll
            for (int a = 0; a < NT; ++a) wf[a] = frag(wt + (step & 1) * kW, a);
            x = frag(xt + place * kHalf, 0);
        }
        if ((step & 3) == 0) {
            if ((step & (4 * kGroups - 1)) == 0 && step > 0) {
                barrier();
                fetch_scales(step);
                wait_lds();
                barrier();
            }
            const uint32_t *from = scales[(step >> 2) & (kGroups - 1)];
#pragma unroll
            for (int t = 0; t < MT; ++t) xs[t] = from[(wm * MT + t) * 16 + r];
            ws = from[B + wn];
        }
        const uint8_t *const x0 = xt + place * kHalf, *const x1 = xt + past(1) * kHalf, *const x2 = xt + past(2) * kHalf;
#pragma unroll
        for (int b = 0; b + 1 < MT; ++b) {
            if (b == MT / 2 - 1) {
                wait_lds();
                barrier();
            }
            const i32x8 ahead = b + 1 < MT / 2 ? frag(x0, b + 1) : frag(x1, b + 1 - MT / 2);
#pragma unroll
            for (int a = 0; a < NT; ++a) {
                acc[a][b] = mma<WF, false>(wf[a], x, acc[a][b], int(ws), int(xs[b]));
                // A load behind each two or three products: 12 in the last four rows but one.
                if (b >= MT / 2 - 1 && (a == 1 || a == 4 || a == 7)) {
                    const int i = (b - (MT / 2 - 1)) * 3 + a / 3;
                    if (i < 4) fetch_x(step + 2, 1, place, i);
                    else fetch_w(step + 2, i - 4);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            x = ahead;
            __builtin_amdgcn_sched_barrier(0);
        }
        // Behind the next step's weights: the first half of step + 2, its second half and weights.
        wait_but<16>();
        barrier();
        // (After the last step these reads are of LDS that nothing uses any more.)
        const i32x8 ahead = frag(x2, 0);
        const uint8_t *const wnext = wt + ((step + 1) & 1) * kW;
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            acc[a][MT - 1] = mma<WF, false>(wf[a], x, acc[a][MT - 1], int(ws), int(xs[MT - 1]));
            wf[a] = frag(wnext, a);
            if (a % 2) fetch_x(step + 3, 0, past(1), a / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        x = ahead;
        ws >>= 8;
#pragma unroll
        for (int t = 0; t < MT; ++t) xs[t] >>= 8;
        place = past(2);
    }
    wait_all();     // no transfer may outlive the block's LDS
#pragma unroll
    for (int b = 0; b < MT; ++b) {
        const int m = m0 + (wm * MT + b) * 16 + r;
        if (m >= p.m) continue;
#pragma unroll
        for (int a = 0; a < NT; ++a) store_outputs<O>(p, m, n0 + (wn * NT + a) * 16 + g * 4, acc[a][b]);
    }
}

// w8 [n][k] to [k][n] (rows of ldt bytes, filled up with zeros) and its scales [n / 128][k /
// 128] to [k / 128][blocks of n]: 128 x 64 bytes a block, 8 x 4 of them a thread. The gradient
// contracts over w's rows and the matrix instruction wants them consecutive in a lane; turned
// around once in scratch they go through the forward product's kernels (2048 columns by 1000
// rows: 4.2 of the gradient's 16 us).
__global__ void __launch_bounds__(256)
transpose8_kernel(const uint8_t *__restrict__ w, const uint8_t *__restrict__ ws, uint8_t *__restrict__ t, uint8_t *__restrict__ ts, int n,
                  int k, int64_t ldw, int64_t ldws, int64_t ldt)
{
    __shared__ __align__(16) uint8_t tile[128][68];
    const int k0 = int(blockIdx.x) * 64, n0 = int(blockIdx.y) * 128, row = int(threadIdx.x >> 1), piece = int(threadIdx.x & 1) * 32;
    i32x4 v[2] = {};
    if (n0 + row < n) {
        v[0] = row16(w + (n0 + row) * ldw, k0 + piece, k);
        v[1] = row16(w + (n0 + row) * ldw, k0 + piece + 16, k);
    }
    if (threadIdx.x == 0 && k0 % 128 == 0) ts[k0 / 128 * int64_t(gridDim.y) + blockIdx.y] = ws[blockIdx.y * ldws + k0 / 128];
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<int *>(&tile[row][piece + 4 * i]) = v[i / 4][i % 4];
    __syncthreads();
    const int ng = int(threadIdx.x & 15) * 8, kg = int(threadIdx.x >> 4) * 4;
    uint32_t in[8];
    uint64_t out[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = *reinterpret_cast<const uint32_t *>(&tile[ng + i][kg]);
    turn(in, out);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k0 + kg + i < k && n0 + ng < ldt) *reinterpret_cast<uint64_t *>(t + (k0 + kg + i) * ldt + n0 + ng) = out[i];
}

template <typename O, int WF, int BN, int BM, int WN, int WM, int STAGES>
void run_tiles(const LinearParams &p, hipStream_t s)
{
    const int tn = (p.n + BN - 1) / BN, tm = (p.m + BM - 1) / BM;
    hipLaunchKernelGGL((linear_tile_kernel<O, WF, BN, BM, WN, WM, STAGES>), dim3(uint32_t((int64_t(tn) * tm + 7) / 8 * 8)), dim3(64 * WN * WM), 0, s, p, tn, tm);
}

// Rows further apart are out of the tiles' reach, whose 32-bit offsets span 256 of them.
constexpr int64_t kReach = 1 << 22;

// Which kernel a product runs on. (Up to 32 bits' offsets only: further apart, rows go through
// linear_rows_kernel.)
template <typename O, int WF>
void run_linear(const LinearParams &p, hipStream_t s)
{
    const bool reach = p.ldx <= kReach && p.ldw <= kReach;
    // Few rows: linear_rows_kernel, whose time goes with its groups of 16 outputs times 16 rows, where those
    // are few. k = 4096, us, tiles behind: 8 x 8192 outputs (512 groups) 9.7 and 12.1, 8 x 11000 (688) 12.6 and
    // 12.4; 32 x 4096 (512) 9.1 and 12.2, 32 x 5504 (688) 14.9 and 12.3; 64 x 2048 (512) 12.9 and 12.0.
    // Outputs in 32 bits, whose products are more instructions in either: 8 x 11000 13.0 and 22.1, 64 x 4096
    // 14.3 and 22.3, 128 x 4096 26.1 and 22.6.
    const int64_t groups = int64_t((p.n + 15) / 16) * (p.m <= 16 ? 1 : p.m <= 32 ? 2 : 4);
    constexpr bool wide_sums = sizeof(O) == 4;
    if ((p.m > (wide_sums ? 64 : 32) || groups > (wide_sums ? 1200 : 512)) && reach) {
        const int64_t t256 = int64_t((p.n + 255) / 256) * ((p.m + 255) / 256), t128 = int64_t((p.n + 127) / 128) * ((p.m + 127) / 128);
        if constexpr (sizeof(O) == 2) {
            // Whichever takes less by what its rounds take (in 10 ns): of 256 tiles of 256, or, two a CU,
            // of half as many CUs' tiles of 128. Measured (tiles of 256 and of 128, us): k = 4096, 2500 x 4096
            // outputs 52 and 55; 2048 x 4096 52 and 38; 2900 x 6000 105 and 84; 5000 x 5000 108 and 116;
            // 4096 x 4096 60 and 70; 8192 x 8192 236 and 311; k = 128, 5698 x 4352 31 and 24, 4096 x 4096 17 and
            // 17; k = 1024, 5698 x 4352 48 and 39, 8192 x 8192 92 and 101.
            const int64_t wide = (t256 + 255) / 256 * (1300 + 120 * p.kblocks), two = (t128 + 255) / 256 * (350 + 43 * p.kblocks);
            if (t128 > 256 && wide <= two) {
                const int tn = (p.n + 255) / 256, tm = (p.m + 255) / 256;
                hipLaunchKernelGGL((linear_wide_kernel<O, WF>), dim3(uint32_t((t256 + 7) / 8 * 8)), dim3(256), 0, s, p, tn, tm);
                return;
            }
        }
        // Up to two blocks a CU of 64 x 64: a step's products and reads are a quarter as many, and it is
        // their time that a lone block waits for (us, tiles of 128 behind; 128 x 4096 outputs of 4096: 12.8 and
        // 19.5; 6383 x 80 of 2822: 11.7 and 17.0; 512 x 4096 of 128, 1024, 4096, 11008: 5.3 and 6.0, 7.7 and 9.1,
        // 16.9 and 19.9, 38.9 and 42.4. More blocks, 1024 x 4096 of the first three: 8.7 and 6.7, 13.5 and 10.6,
        // 30 and 21; 2005 x 2048 of 1000: 17.0 and 12.3).
        const int64_t t64 = int64_t((p.n + 63) / 64) * ((p.m + 63) / 64);
        if (t64 <= 512) return run_tiles<O, WF, 64, 64, 2, 2, 4>(p, s);
        // One block of 128 x 128 a CU at most: eight waves, four steps in LDS (1024 x 4096 outputs of 4096:
        // 21.5 us, four waves with two steps 26.3; 2005 x 2048 of 1000: 12.3 and 13.4). More: two blocks of four
        // waves share a CU (5000 x 5000 outputs of 4096: 113 us, eight waves and four steps 130).
        if (t128 <= 256) return run_tiles<O, WF, 128, 128, 2, 4, 4>(p, s);
        return run_tiles<O, WF, 128, 128, 2, 2, 2>(p, s);
    }
    const auto rows = [&](auto mt) {
        constexpr int MT = decltype(mt)::value, WAVES = 8;
        const dim3 grid(uint32_t((p.n + 15) / 16), uint32_t((p.m + 16 * MT - 1) / (16 * MT)));
        hipLaunchKernelGGL((linear_rows_kernel<O, WF, MT, WAVES>), grid, dim3(64 * WAVES), 0, s, p);
    };
    if (p.m <= 16) rows(std::integral_constant<int, 1>{});
    else if (p.m <= 32) rows(std::integral_constant<int, 2>{});
    else rows(std::integral_constant<int, 4>{});
}

template <typename O>
void run_linear(const LinearParams &p, bool e5m2, hipStream_t s)
{
    if (e5m2) run_linear<O, 1>(p, s);
    else run_linear<O, 0>(p, s);
}

// Whether a product whose rows are too far apart for the tiles has few enough for linear_rows_kernel's
// grid, whose second axis takes 65535 times 64 of them.
bool rows_fit(int64_t m, int64_t ldx, int64_t ldw) { return (ldx <= kReach && ldw <= kReach) || m <= 64 * 65535; }

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t blocks_of(int64_t v) { return (v + kScaleBlock - 1) / kScaleBlock; }

ds_status check_linear(const char *a, int64_t m, int64_t n, int64_t k, int64_t in, int64_t out, const void *x8, const void *w8,
                       int64_t ldx, int64_t ldxs, int64_t ldw, int64_t ldws, int64_t ldy, int32_t w_type, int32_t y_type)
{
    if (m < 0 || n <= 0 || k <= 0) return fail(DS_ERR_INVALID_SHAPE, "m must be >= 0, n and k > 0");
    if (m > kMaxElems / 64 || n > kMaxElems / 64 || k > kMaxElems / 64)
        return fail(DS_ERR_UNSUPPORTED, "2^25 or more rows or columns");
    if (w_type != DS_TYPE_F8E4M3 && w_type != DS_TYPE_F8E5M2) return fail(DS_ERR_INVALID_ARG, "w_type must be DS_TYPE_F8E4M3 or DS_TYPE_F8E5M2");
    if (!float_bytes(y_type)) return fail(DS_ERR_INVALID_ARG, "y_type must be DS_TYPE_F32, DS_TYPE_F16 or DS_TYPE_BF16");
    if (ldx < up(in, 16) || ldx % 16 || reinterpret_cast<uintptr_t>(x8) % 16 || ldw < up(k, 16) || ldw % 16 ||
        reinterpret_cast<uintptr_t>(w8) % 16)
        return fail(DS_ERR_INVALID_ARG, "8-bit rows must begin on 16 bytes and be a multiple of 16 apart, at least the columns");
    if (ldxs < blocks_of(in) || ldws < blocks_of(k)) return fail(DS_ERR_INVALID_ARG, "fewer scales in a row than blocks of 128");
    if (ldy < out) return fail(DS_ERR_INVALID_ARG, "a row of %s is shorter than its columns", a);
    return DS_SUCCESS;
}

void launch(const LinearParams &p, int32_t w_type, int32_t y_type, hipStream_t s)
{
    const bool e5m2 = w_type == DS_TYPE_F8E5M2;
    if (y_type == DS_TYPE_F32) run_linear<float>(p, e5m2, s);
    else if (y_type == DS_TYPE_F16) run_linear<_Float16>(p, e5m2, s);
    else run_linear<__bf16>(p, e5m2, s);
}

}  // namespace

}  // namespace ds

using namespace ds;

extern "C" ds_status ds_linear_fp8(const uint8_t *x8, const uint8_t *x_scales, const uint8_t *w8, const uint8_t *w_scales,
                                   const float *bias, void *y, int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldxs,
                                   int64_t ldw, int64_t ldws, int64_t ldy, int32_t w_type, int32_t y_type, void *stream)
{
    if (m != 0 && (!x8 || !x_scales || !w8 || !w_scales || !y))
        return fail(DS_ERR_NULL_POINTER, "x8, w8, their scales and y must not be NULL");
    if (ds_status st = check_linear("y", m, n, k, k, n, x8, w8, ldx, ldxs, ldw, ldws, ldy, w_type, y_type)) return st;
    if (!rows_fit(m, ldx, ldw)) return fail(DS_ERR_UNSUPPORTED, "more than 64 x 65535 rows, some more than 4 MiB apart");
    if (m == 0) return ok();
    const int64_t es = float_bytes(y_type);
    if (ds_status st = check_tensors({{x8, span(m, ldx, up(k, 16)), "x8", false},
                                      {x_scales, span(m, ldxs, blocks_of(k)), "x_scales", false},
                                      {w8, span(n, ldw, up(k, 16)), "w8", false},
                                      {w_scales, span(blocks_of(n), ldws, blocks_of(k)), "w_scales", false},
                                      {bias, n * 4, "bias", false},
                                      {y, span(m, ldy, n, es), "y", true}}))
        return st;
    const LinearParams p{x8, x_scales, w8, w_scales, bias, y, int(m), int(n), int(k), int(blocks_of(k)), ldx, ldxs, ldw, ldws, ldy};
    launch(p, w_type, y_type, static_cast<hipStream_t>(stream));
    return launched("ds_linear_fp8");
}

extern "C" int64_t ds_linear_fp8_backward_data_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m <= 0 || n <= 0 || k <= 0 || n > kMaxElems / 64 || k > kMaxElems / 64) return 0;
    return up(k * up(n, 16), 256) + up(blocks_of(k) * blocks_of(n), 256);
}

extern "C" ds_status ds_linear_fp8_backward_data(const uint8_t *dy8, const uint8_t *dy_scales, const uint8_t *w8,
                                                 const uint8_t *w_scales, void *dx, int64_t m, int64_t n, int64_t k,
                                                 int64_t lddy, int64_t lddys, int64_t ldw, int64_t ldws, int64_t lddx,
                                                 int32_t w_type, int32_t dx_type, void *scratch, int64_t scratch_bytes,
                                                 void *stream)
{
    if (m != 0 && (!dy8 || !dy_scales || !w8 || !w_scales || !dx))
        return fail(DS_ERR_NULL_POINTER, "dy8, w8, their scales and dx must not be NULL");
    if (ds_status st = check_linear("dx", m, n, k, n, k, dy8, w8, lddy, lddys, ldw, ldws, lddx, w_type, dx_type)) return st;
    if (!rows_fit(m, lddy, up(n, 16))) return fail(DS_ERR_UNSUPPORTED, "more than 64 x 65535 rows, some more than 4 MiB apart");
    if (m == 0) return ok();
    const int64_t need = ds_linear_fp8_backward_data_scratch_bytes(m, n, k), es = float_bytes(dx_type);
    if (!scratch) return fail(DS_ERR_NULL_POINTER, "scratch must not be NULL");
    if (scratch_bytes < need) return fail(DS_ERR_BUFFER_TOO_SMALL, "scratch has %lld bytes, %lld are needed", (long long)scratch_bytes, (long long)need);
    if (reinterpret_cast<uintptr_t>(scratch) % 256) return fail(DS_ERR_INVALID_ARG, "scratch is not 256-byte aligned");
    if (ds_status st = check_tensors({{dy8, span(m, lddy, up(n, 16)), "dy8", false},
                                      {dy_scales, span(m, lddys, blocks_of(n)), "dy_scales", false},
                                      {w8, span(n, ldw, up(k, 16)), "w8", false},
                                      {w_scales, span(blocks_of(n), ldws, blocks_of(k)), "w_scales", false},
                                      {dx, span(m, lddx, k, es), "dx", true},
                                      {scratch, need, "scratch", true}}))
        return st;
    const auto s = static_cast<hipStream_t>(stream);
    const int64_t ldt = up(n, 16);
    uint8_t *wt = static_cast<uint8_t *>(scratch), *wst = wt + up(k * ldt, 256);
    const int nb = int(blocks_of(n));
    if (nb > 65535) return fail(DS_ERR_UNSUPPORTED, "more than 65535 x 128 rows of w8");
    hipLaunchKernelGGL(transpose8_kernel, dim3(uint32_t((k + 63) / 64), uint32_t(nb)), dim3(256), 0, s, w8, w_scales, wt, wst, int(n), int(k),
                       ldw, ldws, ldt);
    const LinearParams p{dy8, dy_scales, wt, wst, nullptr, dx, int(m), int(k), int(n), nb, lddy, lddys, ldt, int64_t(nb), lddx};
    launch(p, w_type, dx_type, s);
    return launched("ds_linear_fp8_backward_data");
}
