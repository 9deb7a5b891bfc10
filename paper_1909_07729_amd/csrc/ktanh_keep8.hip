// libktanh: Swish and GELU that keep their input in 8 bits for the backward pass, and that pass.
//
// What the backward pass of Swish and GELU needs is the forward input.  Kept as it is it costs 2 or 4 bytes a value from the forward to
// the backward pass; here it costs one, and 4 bytes for each 128 consecutive values (a group): with m the largest finite magnitude of
// the group
//   scale = m / 127,   code = round(x * (127 / m)),   and what the code stands for is code * scale, rounded to the tensor's type
// (the scale is held below where that is infinite).
// The gradient is that of kswish_backward and kgelu_backward at the values that the codes stand for, operation for operation.  The code -128 stands
// for an infinity or a NaN, whose gradient is a NaN in those calls too (Swish and GELU multiply it by a slope of zero); it is left out
// of m, so that its neighbours keep their values.
//
// Bound by memory: forward 5 bytes a BFloat16 value and 1/32 (8192 x 16384 in 103 us, 6.5 TB/s), backward 5 (113 us, 6.0 TB/s), and 2 more where the
// activation is rebuilt (4096 x 16384 in 70 us, 6.9 TB/s); Float32 13 bytes with it (20 million values in 38 us, 6.9 TB/s).  A wavefront to a block: there is
// nothing to share beyond a group.
#include "ktanh_codes.h"
#include "ktanh_slopes.h"
#include "ktanh_stream_impl.h"

#include <type_traits>

using namespace ktanh_device;

namespace {

constexpr unsigned kGroup = KTANH_KEEP8_GROUP;

// A lane has one 128-bit vector of values and as many codes, a wavefront 512 (BFloat16) or 256 (Float32) values, which are whole groups
// of 16 or 32 lanes: the largest magnitude is found with cross-lane moves, and no group is shared between wavefronts.
template <class ELEM> constexpr unsigned kGroupLanes = kGroup / kPerLane<ELEM>;

// ------------------------------------------------------------------------------------ codes
// The largest of a group's lanes, in all of them: four moves within a row of 16 lanes, and one to the other row for groups of 32.
template <unsigned LANES>
__device__ __forceinline__ uint32_t largest_of_group(uint32_t m)
{
    m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xF, 0xF, false));  // row_ror:8
    m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xF, 0xF, false));
    m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x122, 0xF, 0xF, false));
    m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x121, 0xF, 0xF, false));
    if constexpr (LANES == 32) m = larger(m, (uint32_t)__builtin_amdgcn_ds_swizzle((int)m, 0x401F));  // lane ^ 16
    return m;
}

// 127 times it is the last Float32 but one: a group with the last, which stands for masked places, would have a scale whose 127-fold is infinite, and so NaNs
// for gradients.
constexpr float kMostScale = 0x1.020406p121f;

// The codes of a lane's vector, and its group's scale.
template <class ELEM>
__device__ __forceinline__ uint2 codes_of(uint4 v, float &scale)
{
    constexpr unsigned N = kPerLane<ELEM>;
    float x[N];
    widen<ELEM>(v, x);
    bool odd;
    uint32_t m = largest_of_lane<ELEM>(v, odd);
    const bool any_odd = __any(odd);  // the wavefront has an infinity or a NaN
    if (any_odd) {
        m = 0;
#pragma unroll
        for (unsigned i = 0; i < N; ++i) {
            const uint32_t mag = __float_as_uint(x[i]) & 0x7FFFFFFFu;
            m = larger(m, mag < 0x7F800000u ? mag : 0u);
        }
    }
    const float top = __uint_as_float(largest_of_group<kGroupLanes<ELEM>>(m));
    const float inverse = inverse_of(top);
    scale = scale_of(top);
    if constexpr (sizeof(ELEM) == 4) scale = __builtin_fminf(scale, kMostScale);
    uint32_t q[N];
#pragma unroll
    for (unsigned i = 0; i < N; ++i) q[i] = rounded_code(x[i], inverse);
    if (any_odd) {
#pragma unroll
        for (unsigned i = 0; i < N; ++i)
            if ((__float_as_uint(x[i]) & 0x7FFFFFFFu) >= 0x7F800000u) q[i] = 0x80u;
    }
    uint2 out{four_codes(q[0], q[1], q[2], q[3]), 0u};
    if constexpr (N == 8) out.y = four_codes(q[4], q[5], q[6], q[7]);
    return out;
}

// What four codes stand for, in Float32.
__device__ __forceinline__ void values_of(uint32_t codes, float scale, float (&x)[4])
{
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) x[i] = (float)(int8_t)(codes >> (8 * i)) * scale;
    // bytes equal to 0x80 leave a zero byte here; the lowest such byte is found exactly, and that is all that is asked
    const uint32_t d = codes ^ 0x80808080u;
    const bool odd = ((d - 0x01010101u) & ~d & 0x80808080u) != 0;
    if (__any(odd)) {
#pragma unroll
        for (unsigned i = 0; i < 4; ++i)
            if ((uint8_t)(codes >> (8 * i)) == 0x80u) x[i] = __builtin_nanf("");
    }
}

// ------------------------------------------------------------------------------------ forward
template <class ELEM, int OP, bool WIDE, bool ALIGNED, bool KEEP>
__global__ __launch_bounds__(kBlock) void keep8_kernel(const ELEM *in, ELEM *out, int8_t *codes, float *scales, unsigned long long n,
                                                       KtLutPack pack)
{
    constexpr unsigned N = kPerLane<ELEM>;
    const LaneTable tab(pack);
    const unsigned long long at = ((unsigned long long)blockIdx.x * kBlock + threadIdx.x) * N;
    const unsigned count = at >= n ? 0u : n - at < N ? (unsigned)(n - at) : N;
    uint4 v = uint4{0u, 0u, 0u, 0u};
    if (count != 0) v = load_values<ALIGNED>(in + at, count);
    float scale;
    const uint2 c = codes_of<ELEM>(v, scale);
    if (count != 0) {
        store_codes<ALIGNED, ELEM>(codes + at, c, count);
        if (threadIdx.x % kGroupLanes<ELEM> == 0) scales[at / kGroup] = scale;
    }
    if constexpr (sizeof(ELEM) == 2) v = apply_vec_bf16<OP, WIDE>(v, tab);
    else v = apply_vec_f32<OP, WIDE>(v, tab);
    if (count != 0) store_values<ALIGNED, KEEP>(out + at, v, count);
}

// ------------------------------------------------------------------------------------ backward
// The activation itself from x and the K value that slope_of takes: x s, and (x / 2)(1 + t), which rounds like x (0.5 + 0.5 t).
template <int GRAD>
__device__ __forceinline__ float value_of(float x, float k)
{
    if constexpr (GRAD == GRAD_SWISH) return x * k;
    else return x * __builtin_fmaf(0.5f, k, 0.5f);
}

template <class ELEM, int GRAD, bool WIDE, bool ALIGNED, bool KEEP, bool REBUILD>
__global__ __launch_bounds__(kBlock) void keep8_backward_kernel(const ELEM *dy, const int8_t *codes, const float *scales, ELEM *dx,
                                                                unsigned long long n, ELEM *y, KtLutPack pack)
{
    constexpr unsigned N = kPerLane<ELEM>;
    const LaneTable tab(pack);
    const unsigned long long at = ((unsigned long long)blockIdx.x * kBlock + threadIdx.x) * N;
    const unsigned count = at >= n ? 0u : n - at < N ? (unsigned)(n - at) : N;
    uint2 c{0u, 0u};
    uint4 d = uint4{0u, 0u, 0u, 0u};
    float scale = 0.f;
    if (count != 0) {
        c = load_codes<ALIGNED, ELEM>(codes + at, count);
        scale = scales[at / kGroup];
        d = load_values<ALIGNED>(dy + at, count);
    }
    float x[N];
    values_of(c.x, scale, reinterpret_cast<float(&)[4]>(x[0]));
    if constexpr (N == 8) values_of(c.y, scale, reinterpret_cast<float(&)[4]>(x[4]));
    const uint32_t dw[4] = {d.x, d.y, d.z, d.w};
    uint32_t gw[4], yw[4];
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) {
        float k[2] = {0.f, 0.f};
        if constexpr (sizeof(ELEM) == 2) {
            const uint32_t w = narrow_pair(x[2 * i], x[2 * i + 1]);
            const Slopes s = slopes_of_word<ELEM, GRAD, WIDE>(w, tab, k);
            gw[i] = grad_word<ELEM>(dw[i], s);
            yw[i] = narrow_pair(value_of<GRAD>(widen_lo(w), k[0]), value_of<GRAD>(widen_hi(w), k[1]));
        } else {
            const Slopes s = slopes_of_word<ELEM, GRAD, WIDE>(__float_as_uint(x[i]), tab, k);
            gw[i] = grad_word<ELEM>(dw[i], s);
            yw[i] = __float_as_uint(value_of<GRAD>(x[i], k[0]));
        }
    }
    if (count != 0) {
        store_values<ALIGNED, KEEP>(dx + at, uint4{gw[0], gw[1], gw[2], gw[3]}, count);
        if constexpr (REBUILD) store_values<ALIGNED, KEEP>(y + at, uint4{yw[0], yw[1], yw[2], yw[3]}, count);
    }
}

// ------------------------------------------------------------------------------------ host side
// Bits of the addresses that are below the width of the accesses.
template <class ELEM>
bool on_the_grid(const void *a, const void *b, const void *c, const void *codes)
{
    const uintptr_t values = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c);
    return values % 16 == 0 && reinterpret_cast<uintptr_t>(codes) % kPerLane<ELEM> == 0;
}

template <class ELEM>
ktanh_status_t check_call(const void *a, const void *b, const void *c, const void *codes, const void *scales, size_t n, unsigned *tiles)
{
    if (a == nullptr || b == nullptr || codes == nullptr || scales == nullptr) return KT_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c)) % sizeof(ELEM) != 0 ||
        reinterpret_cast<uintptr_t>(scales) % 4 != 0)
        return KT_ERR_ALIGN;
    constexpr unsigned long long kTile = kBlock * kPerLane<ELEM>;
    if (n > kMaxTiles * kTile) return KT_ERR_SHAPE;
    *tiles = (unsigned)((n + kTile - 1) / kTile);
    return KT_OK;
}

template <class ELEM, int OP, class Lut>
ktanh_status_t launch_keep8(const void *in, void *out, int8_t *codes, float *scales, size_t n, const Lut *lut, ktanh_stream_t stream)
{
    constexpr bool WIDE = is_wide(static_cast<const Lut *>(nullptr));
    if (n == 0) return KT_OK;
    unsigned tiles;
    ktanh_status_t st = check_call<ELEM>(in, out, nullptr, codes, scales, n, &tiles);
    if (st != KT_OK) return st;
    KtLutPack pack;
    st = pack_for(lut, sizeof(ELEM) == 4, &pack);
    if (st != KT_OK) return st;
    auto launch = [&](auto kernel) {
        return launch_checked(kernel, tiles, kBlock, stream, static_cast<const ELEM *>(in), static_cast<ELEM *>(out), codes, scales,
                              (unsigned long long)n, pack);
    };
    if (!on_the_grid<ELEM>(in, out, nullptr, codes)) return launch(keep8_kernel<ELEM, OP, WIDE, false, true>);
    return stays_cached(n * sizeof(ELEM)) ? launch(keep8_kernel<ELEM, OP, WIDE, true, true>) : launch(keep8_kernel<ELEM, OP, WIDE, true, false>);
}

template <class ELEM, int GRAD, class Lut>
ktanh_status_t launch_keep8_backward(const void *dy, const int8_t *codes, const float *scales, void *dx, void *y, size_t n, const Lut *lut,
                                     ktanh_stream_t stream)
{
    constexpr bool WIDE = is_wide(static_cast<const Lut *>(nullptr));
    if (n == 0) return KT_OK;
    unsigned tiles;
    ktanh_status_t st = check_call<ELEM>(dy, dx, y, codes, scales, n, &tiles);
    if (st != KT_OK) return st;
    KtLutPack pack;
    st = pack_for(lut, sizeof(ELEM) == 4, &pack);
    if (st != KT_OK) return st;
    if (y == dx) return KT_ERR_SHAPE;
    auto launch = [&](auto kernel) {
        return launch_checked(kernel, tiles, kBlock, stream, static_cast<const ELEM *>(dy), codes, scales, static_cast<ELEM *>(dx),
                              (unsigned long long)n, static_cast<ELEM *>(y), pack);
    };
    auto with = [&](auto aligned, auto kept) {
        constexpr bool ALIGNED = decltype(aligned)::value, KEEP = decltype(kept)::value;
        return y != nullptr ? launch(keep8_backward_kernel<ELEM, GRAD, WIDE, ALIGNED, KEEP, true>)
                            : launch(keep8_backward_kernel<ELEM, GRAD, WIDE, ALIGNED, KEEP, false>);
    };
    if (!on_the_grid<ELEM>(dy, dx, y, codes)) return with(std::false_type(), std::true_type());
    return stays_cached(n * sizeof(ELEM)) ? with(std::true_type(), std::true_type()) : with(std::true_type(), std::false_type());
}

}  // namespace

#define KEEP8(name, ELEM, CTYPE, OP, GRAD, LUT)                                                                                  \
    extern "C" ktanh_status_t name##_keep8(const CTYPE *in, CTYPE *out, int8_t *codes, float *scales, size_t n, const LUT *lut,  \
                                           ktanh_stream_t stream)                                                                \
    {                                                                                                                            \
        return launch_keep8<ELEM, OP>(in, out, codes, scales, n, lut, stream);                                                   \
    }                                                                                                                            \
    extern "C" ktanh_status_t name##_keep8_backward(const CTYPE *dy, const int8_t *codes, const float *scales, CTYPE *dx,        \
                                                    CTYPE *y, size_t n, const LUT *lut, ktanh_stream_t stream)                   \
    {                                                                                                                            \
        return launch_keep8_backward<ELEM, GRAD>(dy, codes, scales, dx, y, n, lut, stream);                                      \
    }
KEEP8(kswish, uint16_t, uint16_t, OP_SWISH, GRAD_SWISH, ktanh_lut_t)
KEEP8(kgelu, uint16_t, uint16_t, OP_GELU, GRAD_GELU, ktanh_lut_t)
KEEP8(kswish_f32, uint32_t, float, OP_SWISH, GRAD_SWISH, ktanh_lut_t)
KEEP8(kgelu_f32, uint32_t, float, OP_GELU, GRAD_GELU, ktanh_lut_t)
KEEP8(kswish64, uint16_t, uint16_t, OP_SWISH, GRAD_SWISH, ktanh_lut64_t)
KEEP8(kgelu64, uint16_t, uint16_t, OP_GELU, GRAD_GELU, ktanh_lut64_t)
KEEP8(kswish64_f32, uint32_t, float, OP_SWISH, GRAD_SWISH, ktanh_lut64_t)
KEEP8(kgelu64_f32, uint32_t, float, OP_GELU, GRAD_GELU, ktanh_lut64_t)
