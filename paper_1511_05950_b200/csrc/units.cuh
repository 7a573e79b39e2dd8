// Units of eight elements of a row: one or two 16-byte vectors of activations (bf16 or fp32), one 8-byte vector of codes; four neighbouring
// lanes hold the 32 columns that share a scale.  A unit whose address or length does not allow vectors is taken element by element.
#pragma once

#include "packed.cuh"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace softsync {

constexpr int kUnit = 8;                  // elements
constexpr int kPackBlock = 32;            // columns that share a scale
constexpr unsigned kAllLanes = 0xffffffffu;

// A kernel of these waits for the one before it on the stream before it touches memory, and lets the next one start: launched as dependent, kernels prepare themselves
// under the end of their predecessor.  So they are there while the predecessor still writes, and none of them may read by way of the non-coherent cache
// (__ldg, ld.global.nc), whose values have to stand still from a kernel's start to its end.
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- eight elements ----------------------------------------------------------------------------------------------------
struct alignas(16) Unit {
    float v[kUnit];
    __device__ __forceinline__ float2 pair(int k) const { return make_float2(v[2 * k], v[2 * k + 1]); }
    __device__ __forceinline__ void set(int k, float2 x) { v[2 * k] = x.x; v[2 * k + 1] = x.y; }
};
constexpr int kUnitPairs = kUnit / 2;

__device__ __forceinline__ float unit_value(const float *p) { return *p; }
__device__ __forceinline__ float unit_value(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

__device__ __forceinline__ uint4 load_stream16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// A unit as it lies in memory, so that loads are under way before anything is computed.
template <typename T> struct RawUnit;
template <> struct RawUnit<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const void *p) { a = load_stream16(p); }
    __device__ __forceinline__ void take(const void *p) { a = *static_cast<const uint4 *>(p); }
    __device__ __forceinline__ Unit values() const
    {
        Unit u;
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { u.v[2 * k] = __uint_as_float(w[k] << 16); u.v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
        return u;
    }
};
template <> struct RawUnit<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const void *p) { a = load_stream16(p); b = load_stream16(static_cast<const char *>(p) + 16); }
    __device__ __forceinline__ void take(const void *p) { a = static_cast<const uint4 *>(p)[0]; b = static_cast<const uint4 *>(p)[1]; }
    __device__ __forceinline__ Unit values() const
    {
        return Unit{{__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                     __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)}};
    }
};

__device__ __forceinline__ unsigned bf16_pair(float lo, float hi)
{
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Elements [0, n) of a unit (n <= 8; zeros beyond); whole: all eight, from an address that allows vectors.
template <typename T>
__device__ __forceinline__ void load_unit(RawUnit<T> &raw, const T *p, int n, bool whole)
{
    if (whole) {
        raw.load(p);
        return;
    }
    T part[kUnit];
#pragma unroll
    for (int k = 0; k < kUnit; ++k) part[k] = k < n ? p[k] : T(0.f);
    unsigned *w = reinterpret_cast<unsigned *>(&raw);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __bfloat16_as_ushort(part[2 * k]) | static_cast<unsigned>(__bfloat16_as_ushort(part[2 * k + 1])) << 16;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(part[k]);
    }
}

template <typename T>
__device__ __forceinline__ void store_unit(T *p, const Unit &u, int n, bool whole)
{
    if constexpr (sizeof(T) == 2) {
        if (whole) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(bf16_pair(u.v[0], u.v[1]), bf16_pair(u.v[2], u.v[3]), bf16_pair(u.v[4], u.v[5]), bf16_pair(u.v[6], u.v[7]));
            return;
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) if (k < n) p[k] = __float2bfloat16_rn(u.v[k]);
    } else {
        if (whole) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(u.v[0], u.v[1], u.v[2], u.v[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(u.v[4], u.v[5], u.v[6], u.v[7]);
            return;
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) if (k < n) p[k] = u.v[k];
    }
}

// Stores of rows that allow no vectors: a warp's 32 units (256 neighbouring elements of a row) go through shared memory, so that neighbouring lanes write
// neighbouring elements; unit by unit, a store of two bytes touched as many sectors as one of sixteen (5003 x 1100, bf16: 22 us).
template <typename T> struct WarpDesk { alignas(16) T v[32 * kUnit]; };

// This lane's unit of a row, by all lanes of a warp that has 32 neighbouring units.
template <bool ALIGNED, typename T>
__device__ __forceinline__ void store_row(T *row, int unit, int cols, const Unit &u, WarpDesk<T> *desk)
{
    const int lane = threadIdx.x & 31, left = cols - unit * kUnit;
    if constexpr (ALIGNED) {
        if (left > 0) store_unit(row + unit * kUnit, u, left, left >= kUnit);
    } else {
        T *v = desk[threadIdx.x >> 5].v;
        store_unit(v + lane * kUnit, u, kUnit, true);
        __syncwarp();
        const int first = (unit - lane) * kUnit + lane;
#pragma unroll
        for (int k = 0; k < kUnit; ++k) if (first + k * 32 < cols) row[first + k * 32] = v[lane + k * 32];
        __syncwarp();
    }
}
template <typename T> __device__ __forceinline__ float2 rounded(float2 x);
template <> __device__ __forceinline__ float2 rounded<float>(float2 x) { return x; }
template <> __device__ __forceinline__ float2 rounded<__nv_bfloat16>(float2 x)
{
    const unsigned w = bf16_pair(x.x, x.y);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// ---- 8 bits with a scale -----------------------------------------------------------------------------------------------
// The byte s of a block stands for the unit 2^(s - 127) = 2^(floor(log2 max|x|) - 6), at least 2^-126; 255 for a block with an infinity or a
// NaN, whose codes are zero and whose values are NaN (zero times infinity).  Taken from the bits, so there is no rounding but the code's own.
__device__ __forceinline__ unsigned block_scale(unsigned max_bits)
{
    const unsigned e = max_bits >> 23;
    return e == 255u ? 255u : e > 7u ? e - 6u : 1u;
}
__device__ __forceinline__ float scale_unit(unsigned s) { return __uint_as_float(s << 23); }

__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight codes from the eight values of this lane; the four lanes of a block have to call it together.
__device__ __forceinline__ uint2 pack_unit(const Unit &u, unsigned &scale)
{
    float top = max_or_nan(fabsf(u.v[0]), fabsf(u.v[1]));
#pragma unroll
    for (int k = 2; k < kUnit; ++k) top = max_or_nan(top, fabsf(u.v[k]));
    unsigned m = __float_as_uint(top);                      // a NaN is above every number, an infinity above every finite one
    m = max(m, __shfl_xor_sync(kAllLanes, m, 1));
    m = max(m, __shfl_xor_sync(kAllLanes, m, 2));
    scale = block_scale(m);
    // x / unit + 1.5 * 2^23 rounds to nearest, ties to even (the product is exact: the sum is rounded once): |x| / unit is below 128, so the code is in the low byte.
    // Only a block whose largest is 127.5 units or more has codes to cut: its mantissa tells.
    constexpr float middle = 12582912.f;
    const float inv = __uint_as_float((254u - scale) << 23);
    Unit b;
#pragma unroll
    for (int k = 0; k < kUnitPairs; ++k) b.set(k, fma2(u.pair(k), make_float2(inv, inv), make_float2(middle, middle)));
    if ((m & 0x7fffffu) >= 0x7f0000u) {
        if (scale == 255u) return make_uint2(0, 0);
#pragma unroll
        for (int k = 0; k < kUnit; ++k) b.v[k] = fminf(fmaxf(b.v[k], middle - 127.f), middle + 127.f);
    }
    if (scale == 255u) return make_uint2(0, 0);
    const auto bytes = [&](int k) {
        return __byte_perm(__byte_perm(__float_as_uint(b.v[k]), __float_as_uint(b.v[k + 1]), 0x0040), __byte_perm(__float_as_uint(b.v[k + 2]), __float_as_uint(b.v[k + 3]), 0x0040), 0x5410);
    };
    return make_uint2(bytes(0), bytes(4));
}

// The values of eight codes: exact (a code has 7 bits and the unit is a power of two).  With b = code + 128 in the low byte of the float 2^23 + b, minus 2^23 + 128,
// times the unit: two codes an instruction, and none of the slow conversions.
__device__ __forceinline__ Unit unpack_unit(uint2 codes, unsigned scale)
{
    const float unit = scale_unit(scale);
    const unsigned w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
    Unit u;
#pragma unroll
    for (int k = 0; k < kUnitPairs; ++k) {
        const unsigned b = w[k / 2], lo = __byte_perm(b, 0x4b000000u, 0x7440 + 2 * (k & 1)), hi = __byte_perm(b, 0x4b000000u, 0x7441 + 2 * (k & 1));
        u.set(k, mul2(add2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), make_float2(-8388736.f, -8388736.f)), make_float2(unit, unit)));
    }
    return u;
}

__device__ __forceinline__ Unit load_gain(const void *gain, int is_bf16, int col, int n, bool whole)
{
    if (!gain) return Unit{{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}};
    Unit u;
    if (is_bf16) {
        const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(gain) + col;
        if (whole) {
            RawUnit<__nv_bfloat16> raw;
            raw.a = *reinterpret_cast<const uint4 *>(p);
            return raw.values();
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] = k < n ? unit_value(p + k) : 0.f;
    } else {
        const float *p = static_cast<const float *>(gain) + col;
        if (whole) {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            return Unit{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
        }
#pragma unroll
        for (int k = 0; k < kUnit; ++k) u.v[k] = k < n ? p[k] : 0.f;
    }
    return u;
}

}  // namespace softsync
