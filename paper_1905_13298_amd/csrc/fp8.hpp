// What the 8-bit operators share: float8 numbers with power-of-two block scales.
//
// A block of numbers y is held as bytes q and one scale byte e (E8M0, a biased
// exponent): y = q * 2^(e - 127). A power of two costs the matrix instructions
// nothing (their block scale operand applies it), is exact in every format here,
// and moving a block to another scale is a change of its elements' exponents.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.hpp"

namespace ds {

constexpr int kScaleBlock = 128;   // elements of a row that share a scale

// The element types of the unquantised tensors.
inline int float_bytes(int32_t type) { return type == DS_TYPE_F32 ? 4 : type == DS_TYPE_F16 || type == DS_TYPE_BF16 ? 2 : 0; }

// The status of a call whose launches are enqueued.
inline ds_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return ok();
    return fail(DS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Whether a launch can have that many blocks: a grid's first axis has fewer than 2^32 threads.
inline bool grid_fits(int64_t blocks, int64_t threads) { return blocks <= int64_t(0xffffffff) / threads; }

// Bytes of so many elements, -1 for more than 2^62.
inline int64_t bytes_of(__int128 elements, int64_t size)
{
    const __int128 bytes = elements * size;
    return bytes > __int128(1) << 62 ? -1 : int64_t(bytes);
}

// Bytes that `rows` rows of `row` elements span when they begin `ld` elements apart.
inline int64_t span(int64_t rows, int64_t ld, int64_t row, int64_t size = 1)
{
    return rows <= 0 ? 0 : bytes_of(__int128(rows - 1) * ld + row, size);
}

// Bytes that vectors [a][b][c][row] of the given strides span.
inline int64_t span(int64_t a, int64_t b, int64_t c, const int64_t *strides, int64_t row, int64_t size)
{
    return bytes_of(__int128(a - 1) * strides[0] + __int128(b - 1) * strides[1] + __int128(c - 1) * strides[2] + row, size);
}

// A tensor of a call: checked to lie in device memory; an output overlaps no other.
struct Tensor {
    const void *p;
    int64_t bytes;
    const char *name;
    bool out;
};

inline ds_status check_tensors(std::initializer_list<Tensor> list)
{
    for (const Tensor &t : list)
        if (t.p && t.bytes < 0) return fail(DS_ERR_UNSUPPORTED, "%s spans more than 2^62 bytes", t.name);
    for (const Tensor &t : list) {
        if (!t.out || !t.p) continue;
        for (const Tensor &o : list)
            if (&o != &t && overlap(t.p, t.bytes, o.p, o.bytes))
                return fail(DS_ERR_INVALID_ARG, "%s overlaps %s", t.name, o.name);
    }
    // (A call's small tensors often lie in one allocation, which is looked up once, 0.1 us.)
    uintptr_t base[4] = {};
    uint64_t size[4] = {};
    int known = 0;
    for (const Tensor &t : list) {
        if (!t.p || t.bytes <= 0) continue;
        const auto p = reinterpret_cast<uintptr_t>(t.p);
        const auto in = [&](int i) { return p >= base[i] && p - base[i] + uint64_t(t.bytes) <= size[i]; };
        bool ok = false;
        for (int i = 0; i < std::min(known, 4) && !ok; ++i) ok = in(i);
        if (!ok) {
            const int at = known++ & 3;
            ok = device_allocation(t.p, base[at], size[at]) && in(at);
        }
        if (!ok) return fail(DS_ERR_INVALID_ARG, "%s is not a device buffer of %lld bytes", t.name, (long long)t.bytes);
    }
    return DS_SUCCESS;
}

#if defined(__HIPCC__)

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 2^(e - 127) for e in 1 .. 254.
__device__ __forceinline__ float power_of_two(uint32_t e) { return __uint_as_float(e << 23); }

// The scale byte of the least power of two that brings `amax` (finite, >= 0) to at
// most 448 = 1.75 * 2^8, the largest E4M3 number: a mantissa above 1.75 carries into
// the exponent. Not limited to a byte from below: the caller does that.
__device__ __forceinline__ int scale_byte(float amax) { return int((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8; }

// The scale byte of a block of activations or weights: 2^0 for a block of zeros.
__device__ __forceinline__ int block_scale(float amax) { return amax == 0.f ? 127 : max(scale_byte(amax), 1); }

// |v|, or 0 where v is infinite or NaN: such an element is held as NaN and has no
// say in its block's scale.
__device__ __forceinline__ float finite_abs(float v)
{
    const float a = fabsf(v);
    return a < __builtin_inff() ? a : 0.f;
}

// Four floats as E4M3 bytes, rounded to nearest even (beyond +-448, infinite or NaN: NaN).
__device__ __forceinline__ int to_fp8x4(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// 8 rows of 4 bytes turned around: out[i] holds byte i of the 8 rows, first to last.
__device__ __forceinline__ void turn(const uint32_t (&in)[8], uint64_t (&out)[4])
{
    uint32_t half[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t *q = in + 4 * k;
            // Bytes 0, 1 of two rows, then 2, 3; then two pairs of rows together.
        const uint32_t lo0 = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), lo1 = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);
        const uint32_t hi0 = __builtin_amdgcn_perm(q[1], q[0], 0x07030602u), hi1 = __builtin_amdgcn_perm(q[3], q[2], 0x07030602u);
        half[k][0] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100u);
        half[k][1] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302u);
        half[k][2] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100u);
        half[k][3] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = uint64_t(half[1][i]) << 32 | half[0][i];
}

// Eight consecutive elements as floats. Rows may begin anywhere (16-byte loads need no
// alignment on this machine); `n` < 8 reads the first n, the others are 0.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (n >= 8) {
        T t[8];
        __builtin_memcpy(t, p, sizeof t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? float(p[i]) : 0.f;
    }
}

// Eight consecutive elements as they are stored.
template <typename T>
struct Eight {
    T v[8];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = T(0.f);
    }
    __device__ __forceinline__ float at(int i) const { return float(v[i]); }
    // The first n (or all, as always where WHOLE) of those at p + at.
    template <bool WHOLE>
    __device__ __forceinline__ void load(const T *p, uint32_t at, int n)
    {
        if (WHOLE || n >= 8) {
            __builtin_memcpy(v, p + at, sizeof v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) v[i] = p[at + i];
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void store(T *p, uint32_t at, int n) const
    {
        if (WHOLE || n >= 8) {
            __builtin_memcpy(p + at, v, sizeof v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[at + i] = v[i];
        }
    }
};

template <typename T>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = T(v[i]);
        __builtin_memcpy(p, t, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = T(v[i]);
    }
}

// 16 bytes a lane from a buffer to LDS, the lanes' pieces one after the other from `to` on
// (an LDS address, the same in every lane). No register takes part: the data have arrived
// behind wait_all() and, for other waves, a barrier. In assembly, since the compiler takes
// every later read of LDS to need what such a load brings, and waits for it there.
__device__ __forceinline__ void to_lds16(uint32_t to, __amdgpu_buffer_rsrc_t from, int lane_offset, int offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(to), "v"(lane_offset), "s"(from), "s"(offset)
                 : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return uint32_t(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void *)p));
}

// Everything that the wave has loaded and read is there.
__device__ __forceinline__ void wait_all()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0) lgkmcnt(0)
    asm volatile("" : : : "memory");
}

// The same but for its last N loads.
template <int N>
__device__ __forceinline__ void wait_but()
{
    static_assert(N < 64, "what the counter holds");
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    asm volatile("" : : : "memory");
}

// What the wave has written to LDS is there; loads from memory may be on their way.
__device__ __forceinline__ void wait_lds()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
    asm volatile("" : : : "memory");
}

// The waves' barrier, without the wait for memory that __syncthreads() implies.
__device__ __forceinline__ void barrier()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// Sum / maximum over aligned groups of N lanes (N a power of two up to 64), in every lane.
template <int N>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

template <int N>
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

#endif  // __HIPCC__

}  // namespace ds
