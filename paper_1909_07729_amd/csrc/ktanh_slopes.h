// Device-side slopes of the activations, shared by the gradients from a forward output or input (ktanh_backward.hip) and by those from
// an input kept in 8 bits (ktanh_keep8.hip).
#pragma once
#include "ktanh_device.h"

namespace ktanh_device {

// Which slope multiplies dy.  TanH and Sigmoid take it from the forward OUTPUT (no table involved);
// Swish and GELU rebuild the K-TanH value from the forward INPUT with the device functions the
// forward kernels use:
//   TanH'    = 1 - y^2                      Sigmoid' = s * (1 - s)
//   Swish'   = s + x * (s * (1 - s)),                                       s = Sigmoid(x)
//   GELU'    = 0.5 * (1 + t) + (0.5 * x) * ((1 - t^2) * (c * (1 + 3a * x^2))),   t = K(c * (x + a x^3))
// Float32, one rounding per written operation.
enum Grad { GRAD_TANH = 0, GRAD_SIGMOID = 1, GRAD_SWISH = 2, GRAD_GELU = 3 };

// The slope from Float32 values: v is the forward output (TanH, Sigmoid) or the input with its
// K-TanH-derived value k already formed (s for Swish, t for GELU).
template <int GRAD>
__device__ __forceinline__ float slope_of(float v, float k)
{
    if constexpr (GRAD == GRAD_TANH) {
        const float sq = v * v;
        return 1.0f - sq;
    } else if constexpr (GRAD == GRAD_SIGMOID) {
        const float one_minus = 1.0f - v;
        return v * one_minus;
    } else if constexpr (GRAD == GRAD_SWISH) {
        const float one_minus = 1.0f - k;
        const float bell = k * one_minus;
        const float xbell = v * bell;
        return k + xbell;
    } else {
        const float a3 = 0.134145f;  // 3a
        const float c = 0.7978845608028654f;
        const float one_plus = 1.0f + k;
        const float left = 0.5f * one_plus;
        const float tsq = k * k;
        const float sech2 = 1.0f - tsq;
        const float sq = v * v;
        const float a3sq = a3 * sq;
        const float poly = 1.0f + a3sq;
        const float du = c * poly;
        const float chain = sech2 * du;
        const float half_x = 0.5f * v;
        const float right = half_x * chain;
        return left + right;
    }
}

// The argument of K inside GELU: c * (x + a * x^3).
__device__ __forceinline__ float gelu_argument(float x)
{
    const float a = 0.044715f;
    const float c = 0.7978845608028654f;
    const float sq = x * x;
    const float cube = sq * x;
    const float acube = a * cube;
    const float inner = x + acube;
    return c * inner;
}

// One 32-bit word of each stream: a packed BFloat16 pair (ELEM = uint16_t) or one Float32
// (ELEM = uint32_t, `hi` unused).  A single BFloat16 element travels in the low half of the word.
struct Slopes {
    float lo, hi;
};

// k: the K-TanH-derived values that the slopes were formed with (lo, hi).
template <class ELEM, int GRAD, bool WIDE>
__device__ __forceinline__ Slopes slopes_of_word(uint32_t v_w, const LaneTable &tab, float (&k)[2])
{
    if constexpr (sizeof(ELEM) == 2) {
        const float v[2] = {widen_lo(v_w), widen_hi(v_w)};
        if constexpr (GRAD == GRAD_SWISH) {
            ksigmoid_f32_pair<false, WIDE>(v_w, tab, k[0], k[1]);  // a NaN x reaches the slope through x itself
        } else if constexpr (GRAD == GRAD_GELU) {
            const uint32_t t2 = ktanh_pair<false, WIDE>(narrow_pair(gelu_argument(v[0]), gelu_argument(v[1])), tab);
            k[0] = widen_lo(t2);
            k[1] = widen_hi(t2);
        }
        return Slopes{slope_of<GRAD>(v[0], k[0]), slope_of<GRAD>(v[1], k[1])};
    } else {
        const float v = __uint_as_float(v_w);
        if constexpr (GRAD == GRAD_SWISH) {
            // 0.5 * t is exact for every K output t that can change the sum, so the multiply-add may fuse
            const float t = __uint_as_float(ktanh_f32_one<WIDE>(__float_as_uint(0.5f * v), tab));
            k[0] = __builtin_fmaf(0.5f, t, 0.5f);
        } else if constexpr (GRAD == GRAD_GELU) {
            k[0] = __uint_as_float(ktanh_f32_one<WIDE>(__float_as_uint(gelu_argument(v)), tab));
        }
        return Slopes{slope_of<GRAD>(v, k[0]), 0.f};
    }
}

template <class ELEM, int GRAD, bool WIDE>
__device__ __forceinline__ Slopes slopes_of_word(uint32_t v_w, const LaneTable &tab)
{
    float k[2] = {0.f, 0.f};
    return slopes_of_word<ELEM, GRAD, WIDE>(v_w, tab, k);
}

template <class ELEM>
__device__ __forceinline__ uint32_t grad_word(uint32_t dy_w, const Slopes &s)
{
    if constexpr (sizeof(ELEM) == 2) return narrow_pair(widen_lo(dy_w) * s.lo, widen_hi(dy_w) * s.hi);
    else return __float_as_uint(__uint_as_float(dy_w) * s.lo);
}

}  // namespace ktanh_device
