// Device-side values in 8 bits: vectors of BFloat16 or Float32 values from any address, their largest magnitude, and their codes.  With m the
// largest magnitude of the values that share a scale,  scale = m / 127,  code = round(x * (127 / m)),  Float32 operations rounded to nearest
// even.  Shared by the checkpoints of activations (ktanh_keep8.hip) and by the rows of matrix products (ktanh_q8_rows.hip, ktanh_q8_product.hip).
#pragma once
#include "ktanh_device.h"

namespace ktanh_device {

// ELEM: uint16_t (BFloat16) or uint32_t (Float32).  A lane has one 128-bit vector of values and as many codes.
template <class ELEM> constexpr unsigned kPerLane = 16 / sizeof(ELEM);

// ------------------------------------------------------------------------------------ accesses
// `count` (of kPerLane) elements from p, zeros behind them.  A whole vector comes with one access, also from an address that is only
// aligned to its elements; only the last lane with values of a tensor or row has fewer.
template <bool ALIGNED, bool NEAR = false, class ELEM>
__device__ __forceinline__ uint4 load_values(const ELEM *p, unsigned count)
{
    if (count == kPerLane<ELEM>) return load_vec<ALIGNED, NEAR>(reinterpret_cast<const char *>(p));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    for (unsigned i = 0; i < kPerLane<ELEM>; ++i)
        if (i < count) w[i * sizeof(ELEM) / 4] |= (uint32_t)p[i] << (8 * (i * sizeof(ELEM) % 4));
    return uint4{w[0], w[1], w[2], w[3]};
}

template <bool ALIGNED, bool KEEP, class ELEM>
__device__ __forceinline__ void store_values(ELEM *p, uint4 v, unsigned count)
{
    if (count == kPerLane<ELEM>) {
        if constexpr (ALIGNED) store_stream<KEEP>(reinterpret_cast<uint4 *>(p), v);
        else *reinterpret_cast<u32x4_anywhere *>(p) = u32x4{v.x, v.y, v.z, v.w};
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    for (unsigned i = 0; i < kPerLane<ELEM>; ++i)
        if (i < count) p[i] = (ELEM)(w[i * sizeof(ELEM) / 4] >> (8 * (i * sizeof(ELEM) % 4)));
}

// ------------------------------------------------------------------------------------ accesses of codes
typedef u32x2 u32x2_anywhere __attribute__((aligned(1)));
typedef uint32_t u32_anywhere __attribute__((aligned(1)));

// Codes, one byte each: two words a lane (BFloat16) or one.
template <bool ALIGNED, class ELEM>
__device__ __forceinline__ uint2 load_codes(const int8_t *p, unsigned count)
{
    if (count == kPerLane<ELEM>) {
        if constexpr (sizeof(ELEM) == 2) {
            u32x2 t;
            if constexpr (ALIGNED) t = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(p));
            else t = *reinterpret_cast<const u32x2_anywhere *>(p);
            return uint2{t.x, t.y};
        } else {
            if constexpr (ALIGNED) return uint2{__builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p)), 0u};
            else return uint2{*reinterpret_cast<const u32_anywhere *>(p), 0u};
        }
    }
    uint32_t w[2] = {0u, 0u};
    for (unsigned i = 0; i < kPerLane<ELEM>; ++i)
        if (i < count) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
    return uint2{w[0], w[1]};
}

template <bool ALIGNED, class ELEM>
__device__ __forceinline__ void store_codes(int8_t *p, uint2 c, unsigned count)
{
    if (count == kPerLane<ELEM>) {
        if constexpr (sizeof(ELEM) == 2) {
            if constexpr (ALIGNED) __builtin_nontemporal_store(u32x2{c.x, c.y}, reinterpret_cast<u32x2 *>(p));
            else *reinterpret_cast<u32x2_anywhere *>(p) = u32x2{c.x, c.y};
        } else {
            if constexpr (ALIGNED) __builtin_nontemporal_store(c.x, reinterpret_cast<uint32_t *>(p));
            else *reinterpret_cast<u32_anywhere *>(p) = c.x;
        }
        return;
    }
    const uint32_t w[2] = {c.x, c.y};
    for (unsigned i = 0; i < kPerLane<ELEM>; ++i)
        if (i < count) p[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
}

// ------------------------------------------------------------------------------------ codes
// The vector's values in Float32.
template <class ELEM>
__device__ __forceinline__ void widen(uint4 v, float (&x)[kPerLane<ELEM>])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) {
        if constexpr (sizeof(ELEM) == 2) {
            x[2 * i] = widen_lo(w[i]);
            x[2 * i + 1] = widen_hi(w[i]);
        } else {
            x[i] = __uint_as_float(w[i]);
        }
    }
}

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The bits of the largest finite magnitude of a lane's values, as a Float32.  Magnitudes order like their bits.
template <class ELEM>
__device__ __forceinline__ uint32_t largest_of_lane(uint4 v, bool &odd)
{
    if constexpr (sizeof(ELEM) == 2) {
        const uint32_t a = v.x & kMag2, b = v.y & kMag2, c = v.z & kMag2, d = v.w & kMag2;
        const uint32_t m2 = max_pair(max_pair(a, b), max_pair(c, d));
        const uint32_t m = larger(m2 & 0xFFFFu, m2 >> 16);
        odd = m >= 0x7F80u;
        return m << 16;
    } else {
        const uint32_t m = larger(larger(v.x & 0x7FFFFFFFu, v.y & 0x7FFFFFFFu), larger(v.z & 0x7FFFFFFFu, v.w & 0x7FFFFFFFu));
        odd = m >= 0x7F800000u;
        return m;
    }
}

// Below it 127 / m leaves Float32: such values are taken as zeros, with the scale 0.
constexpr float kTiny = 0x1p-120f;
__device__ __forceinline__ float inverse_of(float top) { return top < kTiny ? 0.f : 127.0f / top; }
__device__ __forceinline__ float scale_of(float top) { return top < kTiny ? 0.f : top / 127.0f; }

// A code in the low byte.  x * inverse is at most 127 (1 + 2^-23); 1.5 * 2^23 added to it rounds it to an integer, to nearest even, whose
// two's complement is in the sum's low bits.
__device__ __forceinline__ uint32_t rounded_code(float x, float inverse) { return __float_as_uint(x * inverse + 12582912.0f); }

__device__ __forceinline__ uint32_t four_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

}  // namespace ktanh_device
