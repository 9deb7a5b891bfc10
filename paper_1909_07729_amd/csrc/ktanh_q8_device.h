// Device-side pieces of the products in 8-bit integers: operands from memory, results scaled and stored.
#pragma once
#include "ktanh_device.h"

namespace ktanh_q8 {

using namespace ktanh_device;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_anywhere __attribute__((aligned(1)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Operands {
    const int8_t *x, *w;
    unsigned long long x_row, w_row;
    const float *x_scale, *w_scale, *bias;
    void *out;
    unsigned long long out_row;
    unsigned rows, outer, inner;
};

// 16 integers from p.
template <bool ALIGNED>
__device__ __forceinline__ i32x4 load16(const int8_t *p)
{
    if constexpr (ALIGNED) return *reinterpret_cast<const i32x4 *>(p);
    else return *reinterpret_cast<const i32x4_anywhere *>(p);
}
// The same of a row of `inner` integers, `count` of which are from p on (any number; zeros behind them), in two steps, so that the first can be far ahead of
// the second.  The row's last integers come with one load that ends where the row does, and are then moved to their place.
__device__ __forceinline__ i32x4 ask16(const int8_t *p, int count, unsigned inner)
{
    i32x4 v = {0, 0, 0, 0};
    if (count > 0 && inner >= 16) v = load16<false>(count >= 16 ? p : p - (16 - inner % 16));
    return v;
}
__device__ __forceinline__ i32x4 take16(i32x4 v, const int8_t *p, int count, unsigned inner)
{
    if (count <= 0 || count >= 16) return v;
    if (inner < 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < count) v[i / 4] |= (int)(uint8_t)p[i] << (8 * (i % 4));
        return v;
    }
    const unsigned by = 16 - inner % 16;    // bytes that come too early: alike in all lanes
    if (by & 8) v = i32x4{v[2], v[3], 0, 0};
    if (by & 4) v = i32x4{v[1], v[2], v[3], 0};
    auto moved = [&](int high, int low) { return (int)__builtin_amdgcn_alignbyte((uint32_t)high, (uint32_t)low, by & 3); };
    return i32x4{moved(v[1], v[0]), moved(v[2], v[1]), moved(v[3], v[2]), moved(0, v[3])};
}
__device__ __forceinline__ i32x4 load16(const int8_t *p, int count, unsigned inner) { return take16(ask16(p, count, inner), p, count, inner); }

// What leaves a block: results, or (SUMS) the sums of its part of the inner dimension, as the bits of Float32.
enum Out { BF16 = 0, F32 = 1, SUMS = 2 };

// Results leave by rows, 16 bytes of a lane's at once, to any address of an element's alignment.
template <Out OUT> struct Result {
    typedef float type;
    typedef u32x4 anywhere __attribute__((aligned(4)));
    static constexpr unsigned kEach = 4;    // of a 16-byte chunk
};
template <> struct Result<BF16> {
    typedef uint16_t type;
    typedef u32x4 anywhere __attribute__((aligned(2)));
    static constexpr unsigned kEach = 8;
};

template <Out OUT>
__device__ __forceinline__ void store_chunk(const Operands &a, unsigned t, unsigned o, u32x4 v)
{
    typedef typename Result<OUT>::type T;
    if (t >= a.rows || o >= a.outer) return;
    T *to = static_cast<T *>(a.out) + t * a.out_row + o;
    if (o + Result<OUT>::kEach <= a.outer) {
        *reinterpret_cast<typename Result<OUT>::anywhere *>(to) = v;
        return;
    }
    const T *from = reinterpret_cast<const T *>(&v);
    for (unsigned i = 0; i < Result<OUT>::kEach - 1; ++i)
        if (o + i < a.outer) to[i] = from[i];
}

// Scales, or biases, of channels o .. o + 3; past the last channel the last one's.
__device__ __forceinline__ f32x4 four_of(const float *p, unsigned o, unsigned outer)
{
    typedef f32x4 anywhere __attribute__((aligned(4)));
    if (o + 4 <= outer) return *reinterpret_cast<const anywhere *>(p + o);
    auto at = [&](unsigned i) { return p[i < outer ? i : outer - 1]; };
    return f32x4{at(o), at(o + 1), at(o + 2), at(o + 3)};
}

__device__ __forceinline__ f32x4 scaled(i32x4 sum, float row, f32x4 channel, f32x4 bias, bool biased)
{
    f32x4 y;
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) {
        y[i] = ((float)sum[i] * row) * channel[i];
        if (biased) y[i] = y[i] + bias[i];
    }
    return y;
}

// Four neighbouring results into LDS.
template <Out OUT>
__device__ __forceinline__ void put_four(char *to, f32x4 y)
{
    if constexpr (OUT != BF16) *reinterpret_cast<f32x4 *>(to) = y;
    else *reinterpret_cast<u32x2 *>(to) = u32x2{narrow_pair(y[0], y[1]), narrow_pair(y[2], y[3])};
}

// A block's OT channels by TT rows from its W wavefronts' sums in LDS.
template <unsigned OT, unsigned TT, unsigned W, Out OUT>
__device__ __forceinline__ void store_joined(const Operands &a, unsigned o0, unsigned t0, const int (&part)[W][TT][OT + 4])
{
    constexpr unsigned E = Result<OUT>::kEach;
    for (unsigned e = threadIdx.x; e < TT * OT / E; e += 64 * W) {
        const unsigned t = e / (OT / E), o = e % (OT / E) * E;
        if (t0 + t >= a.rows || o0 + o >= a.outer) continue;
        const float row = a.x_scale[t0 + t];
        u32x4 out;
#pragma unroll
        for (unsigned h = 0; h < E / 4; ++h) {
            i32x4 v = *reinterpret_cast<const i32x4 *>(&part[0][t][o + 4 * h]);
#pragma unroll
            for (unsigned i = 1; i < W; ++i) v += *reinterpret_cast<const i32x4 *>(&part[i][t][o + 4 * h]);
            const unsigned c = o0 + o + 4 * h;
            const bool biased = a.bias != nullptr;
            const f32x4 y = scaled(v, row, four_of(a.w_scale, c, a.outer), biased ? four_of(a.bias, c, a.outer) : f32x4{0, 0, 0, 0}, biased);
            put_four<OUT>(reinterpret_cast<char *>(&out) + 8 * h, y);
        }
        store_chunk<OUT>(a, t0 + t, o0 + o, out);
    }
}

}  // namespace ktanh_q8
