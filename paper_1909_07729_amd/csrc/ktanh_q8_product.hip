// libktanh: products of rows in 8-bit integers with weights in 8-bit integers, scaled by row and by output channel.
//
//   out[t][o] = (float(sum over i of x[t][i] * w[o][i]) * x_scale[t]) * w_scale[o] + bias[o]
//
// The sums are exact (32-bit integers); the scaling is Float32, one rounding per operation.
#include <type_traits>

#include "ktanh_device.h"
#include "ktanh_q8.h"

using namespace ktanh_device;
using namespace ktanh_q8;

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_anywhere __attribute__((aligned(1)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

struct Operands {
    const int8_t *x, *w;
    unsigned long long x_row, w_row;
    const float *x_scale, *w_scale, *bias;
    void *out;
    unsigned long long out_row;
    unsigned rows, outer, inner;
};

// 16 integers from p, of which the first `count` are there (the rest zeros): at the end of a row.
template <bool ALIGNED>
__device__ __forceinline__ i32x4 load16(const int8_t *p)
{
    if constexpr (ALIGNED) return *reinterpret_cast<const i32x4 *>(p);
    else return *reinterpret_cast<const i32x4_anywhere *>(p);
}
template <bool ALIGNED>
__device__ __forceinline__ i32x4 load16(const int8_t *p, int count)
{
    if (count >= 16) return load16<ALIGNED>(p);
    i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < count) v[i / 4] |= (int)(uint8_t)p[i] << (8 * (i % 4));
    return v;
}

// The result at (t, o .. o + 3), as far as it is inside.
template <bool F32, bool WHOLE>
__device__ __forceinline__ void store_scaled(const Operands &a, unsigned t, unsigned o, const int (&sum)[4])
{
    if (t >= a.rows || o >= a.outer) return;
    const float row = a.x_scale[t];
    float y[4];
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) {
        const unsigned at = WHOLE || o + i < a.outer ? o + i : o;
        y[i] = ((float)sum[i] * row) * a.w_scale[at];
        if (a.bias != nullptr) y[i] = y[i] + a.bias[at];
    }
    const unsigned long long at = t * a.out_row + o;
    if constexpr (F32) {
        float *to = static_cast<float *>(a.out) + at;
        if constexpr (WHOLE) *reinterpret_cast<f32x4 *>(to) = f32x4{y[0], y[1], y[2], y[3]};
        else
            for (unsigned i = 0; i < 4; ++i)
                if (o + i < a.outer) to[i] = y[i];
    } else {
        uint16_t *to = static_cast<uint16_t *>(a.out) + at;
        const uint32_t lo = narrow_pair(y[0], y[1]), hi = narrow_pair(y[2], y[3]);
        if constexpr (WHOLE) *reinterpret_cast<u32x2 *>(to) = u32x2{lo, hi};
        else {
            const uint32_t w[2] = {lo, hi};
            for (unsigned i = 0; i < 4; ++i)
                if (o + i < a.outer) to[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
        }
    }
}

// A block has OT output channels and TT rows, and its W wavefronts share the inner dimension in steps of 64 integers: wavefront s takes the steps
// s, s + W, ..., so that the block reads whole cache lines.  Operands go from memory to the matrix cores' registers; the wavefronts' sums
// meet in LDS.
template <unsigned OT, unsigned TT, unsigned W, bool F32, bool ALIGNED, bool WHOLE>
__global__ __launch_bounds__(64 * W) void q8_shared_inner_kernel(Operands a)
{
    constexpr unsigned OI = OT / 16, TI = TT / 16;
    __shared__ int part[W][TT][OT + 4];
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned o0 = blockIdx.x * OT, t0 = blockIdx.y * TT;
    // rows past the last are read as the last, and not stored
    const int8_t *w[OI], *x[TI];
    const unsigned k = lane / 16 * 16;
#pragma unroll
    for (unsigned i = 0; i < OI; ++i) {
        const unsigned o = o0 + 16 * i + lane % 16;
        w[i] = a.w + (o < a.outer ? o : a.outer - 1) * a.w_row + k;
    }
#pragma unroll
    for (unsigned i = 0; i < TI; ++i) {
        const unsigned t = t0 + 16 * i + lane % 16;
        x[i] = a.x + (t < a.rows ? t : a.rows - 1) * a.x_row + k;
    }
    i32x4 sum[OI][TI];
#pragma unroll
    for (unsigned i = 0; i < OI; ++i)
#pragma unroll
        for (unsigned j = 0; j < TI; ++j) sum[i][j] = i32x4{0, 0, 0, 0};
    auto multiply = [&](const i32x4 (&wf)[OI], const i32x4 (&xf)[TI]) {
#pragma unroll
        for (unsigned i = 0; i < OI; ++i)
#pragma unroll
            for (unsigned j = 0; j < TI; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[i], xf[j], sum[i][j], 0, 0, 0);
    };
    const unsigned whole = a.inner / 64;
    constexpr unsigned U = OI + TI > 4 ? 2 : 8;
    unsigned s = wave;
    for (; s + (U - 1) * W < whole; s += U * W) {
        i32x4 wf[U][OI], xf[U][TI];
#pragma unroll
        for (unsigned u = 0; u < U; ++u) {
#pragma unroll
            for (unsigned i = 0; i < OI; ++i) wf[u][i] = load16<ALIGNED>(w[i] + (s + u * W) * 64ull);
#pragma unroll
            for (unsigned i = 0; i < TI; ++i) xf[u][i] = load16<ALIGNED>(x[i] + (s + u * W) * 64ull);
        }
#pragma unroll
        for (unsigned u = 0; u < U; ++u) multiply(wf[u], xf[u]);
    }
    for (; s * 64 < a.inner; s += W) {
        const int there = (int)a.inner - (int)(s * 64 + k);
        i32x4 wf[OI], xf[TI];
#pragma unroll
        for (unsigned i = 0; i < OI; ++i) wf[i] = load16<ALIGNED>(w[i] + s * 64ull, there);
#pragma unroll
        for (unsigned i = 0; i < TI; ++i) xf[i] = load16<ALIGNED>(x[i] + s * 64ull, there);
        multiply(wf, xf);
    }
    // a lane has 4 neighbouring channels of a row
#pragma unroll
    for (unsigned i = 0; i < OI; ++i)
#pragma unroll
        for (unsigned j = 0; j < TI; ++j)
            *reinterpret_cast<i32x4 *>(&part[wave][16 * j + lane % 16][16 * i + lane / 16 * 4]) = sum[i][j];
    __syncthreads();
    for (unsigned e = threadIdx.x; e < TT * OT / 4; e += 64 * W) {
        const unsigned t = e / (OT / 4), o = e % (OT / 4) * 4;
        i32x4 v = *reinterpret_cast<const i32x4 *>(&part[0][t][o]);
#pragma unroll
        for (unsigned i = 1; i < W; ++i) v += *reinterpret_cast<const i32x4 *>(&part[i][t][o]);
        const int four[4] = {v.x, v.y, v.z, v.w};
        store_scaled<F32, WHOLE>(a, t0 + t, o0 + o, four);
    }
}

}  // namespace

namespace ktanh_q8 {

// Arguments have been checked.
ktanh_status_t launch_product(const kq8_shape_t &s, const int8_t *x, size_t x_row, const float *x_scale, const int8_t *w, const float *w_scale,
                              const float *bias, void *out, ktanh_stream_t stream)
{
    Operands a;
    a.x = x;
    a.w = w;
    a.x_row = stride(s.rows, x_row);
    a.w_row = stride(s.outer, s.w_row);
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.bias = bias;
    a.out = out;
    a.out_row = stride(s.rows, s.out_row);
    a.rows = (unsigned)s.rows;
    a.outer = (unsigned)s.outer;
    a.inner = (unsigned)s.inner;
    const bool aligned = !off(x, 16) && a.x_row % 16 == 0 && !off(w, 16) && a.w_row % 16 == 0;
    // four neighbouring results are stored at once
    const bool whole = s.outer % 4 == 0 && a.out_row % 4 == 0 && !off(out, s.out_f32 ? 16 : 8);
    auto launch = [&](auto kernel, unsigned threads, unsigned ot, unsigned tt) {
        const size_t over = (s.outer + ot - 1) / ot, across = (s.rows + tt - 1) / tt;
        if (over * threads >= (1ull << 32) || across > 65535) return KT_ERR_SHAPE;
        void *args[] = {&a};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)over, (unsigned)across), dim3(threads), args, 0,
                               static_cast<hipStream_t>(stream)) == hipSuccess ? KT_OK : KT_ERR_HIP;
    };
    auto sized = [&](auto f32, auto on_grid, auto fours) {
        constexpr bool F = decltype(f32)::value, A = decltype(on_grid)::value, H = decltype(fours)::value;
        if (s.rows <= 16) return launch(q8_shared_inner_kernel<16, 16, 8, F, A, H>, 512, 16, 16);
        if (s.rows <= 32) return launch(q8_shared_inner_kernel<32, 32, 4, F, A, H>, 256, 32, 32);
        return launch(q8_shared_inner_kernel<64, 64, 4, F, A, H>, 256, 64, 64);
    };
    auto stored = [&](auto f32, auto on_grid) { return whole ? sized(f32, on_grid, std::true_type()) : sized(f32, on_grid, std::false_type()); };
    auto typed = [&](auto f32) { return aligned ? stored(f32, std::true_type()) : stored(f32, std::false_type()); };
    return s.out_f32 ? typed(std::true_type()) : typed(std::false_type());
}

}  // namespace ktanh_q8

namespace {

// What a product needs besides its rows.
ktanh_status_t check_weights(const kq8_shape_t *s, const int8_t *w, const float *w_scale, const float *bias, const void *out)
{
    if (w_scale == nullptr || out == nullptr || (s->inner != 0 && w == nullptr)) return KT_ERR_NULL;
    if (off(w_scale, 4) || off(bias, 4) || off(out, s->out_f32 ? 4 : 2)) return KT_ERR_ALIGN;
    return KT_OK;
}

template <class Lut>
ktanh_status_t linear_entry(const kq8_shape_t *s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, void *workspace,
                            const Lut *lut, ktanh_stream_t stream)
{
    ktanh_status_t st = check_rows(s);
    if (st == KT_OK) st = check_product(s);
    if (st != KT_OK) return st;
    if (s->rows == 0 || s->outer == 0) return KT_OK;
    if (workspace == nullptr || (s->inner != 0 && x == nullptr)) return KT_ERR_NULL;
    st = check_weights(s, w, w_scale, bias, out);
    if (st != KT_OK) return st;
    if (off(x, s->x_f32 ? 4 : 2) || off(workspace, 16)) return KT_ERR_ALIGN;
    int8_t *codes = static_cast<int8_t *>(workspace);
    const size_t row = padded(s->inner);
    float *scales = reinterpret_cast<float *>(codes + s->rows * row);
    if constexpr (is_wide(static_cast<const Lut *>(nullptr))) st = kq8_rows64(s, x, codes, row, scales, lut, stream);
    else st = kq8_rows(s, x, codes, row, scales, lut, stream);
    if (st != KT_OK) return st;
    return launch_product(*s, codes, row, scales, w, w_scale, bias, out, stream);
}

}  // namespace

extern "C" ktanh_status_t kq8_product(const kq8_shape_t *shape, const int8_t *codes, const float *scales, const int8_t *w, const float *w_scale,
                                      const float *bias, void *out, ktanh_stream_t stream)
{
    ktanh_status_t st = check_product(shape);
    if (st != KT_OK) return st;
    if (shape->rows == 0 || shape->outer == 0) return KT_OK;
    if (scales == nullptr || (shape->inner != 0 && codes == nullptr)) return KT_ERR_NULL;
    st = check_weights(shape, w, w_scale, bias, out);
    if (st != KT_OK) return st;
    if (off(scales, 4)) return KT_ERR_ALIGN;
    return launch_product(*shape, codes, shape->x_row, scales, w, w_scale, bias, out, stream);
}

extern "C" size_t kq8_linear_workspace(const kq8_shape_t *shape)
{
    if (check_rows(shape) != KT_OK || check_product(shape) != KT_OK) return 0;
    return shape->rows * (padded(shape->inner) + sizeof(float));
}

extern "C" ktanh_status_t kq8_linear(const kq8_shape_t *shape, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out,
                                     void *workspace, const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return linear_entry(shape, x, w, w_scale, bias, out, workspace, lut, stream);
}
extern "C" ktanh_status_t kq8_linear64(const kq8_shape_t *shape, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out,
                                       void *workspace, const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return linear_entry(shape, x, w, w_scale, bias, out, workspace, lut, stream);
}
