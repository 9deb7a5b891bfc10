// libktanh: rows to 8-bit integers and their product in one launch, for the few rows of a decoding step.
//
// Every block brings the rows to integers for itself, in LDS, while its first weights are on their way: a second launch, and a trip of the codes
// through memory, cost more than that as long as the rows are few and short.
#include <type_traits>

#include "ktanh_codes.h"
#include "ktanh_q8.h"
#include "ktanh_q8_device.h"
#include "ktanh_stream_impl.h"

using namespace ktanh_device;
using namespace ktanh_q8;

namespace {

constexpr unsigned kWaves = 8, kMostRows8 = 8, kMostValues = 16384, kSteps = 8;

// ROWS (a power of two) rows, kWaves / ROWS wavefronts to each; then 16 output channels by all of them, the inner dimension shared among the wavefronts
// as in q8_shared_inner_kernel.
template <class ELEM, int ACT, bool WIDE, Out OUT, unsigned ROWS>
__global__ __launch_bounds__(64 * kWaves) void q8_few_kernel(Operands a, const ELEM *x, unsigned long long x_row, KtLutPack pack)
{
    constexpr unsigned N = kPerLane<ELEM>, kEach = kWaves / ROWS, kVectors = kMostValues / kWaves / 64 / N;
    __shared__ __align__(16) int8_t codes[kMostValues + kMostRows8 * 80];
    __shared__ int part[kWaves][16][20];
    __shared__ uint32_t tops[kWaves];
    __shared__ float scales[16];
    const LaneTable tab(pack);
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned o0 = blockIdx.x * 16, k = lane / 16 * 16;
    const unsigned o = o0 + lane % 16;
    const int8_t *w = a.w + (o < a.outer ? o : a.outer - 1) * a.w_row + k;
    const unsigned steps = a.inner / 64, mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    i32x4 wf[kSteps];
#pragma unroll
    for (unsigned u = 0; u < kSteps; ++u)
        if (u < mine) wf[u] = load16<true>(w + (wave + u * kWaves) * 64);

    // the rows: a row's pitch moves neighbouring ones to other banks
    const unsigned pitch = (a.inner + 63) / 64 * 64 + 16, row = wave / kEach, slice = wave % kEach;
    const ELEM *from = x + (row < a.rows ? row : a.rows - 1) * x_row;
    auto place = [&](unsigned v) { return ((v * kEach + slice) * 64 + lane) * N; };
    auto count = [&](unsigned at) { return at >= a.inner ? 0u : a.inner - at < N ? a.inner - at : N; };
    uint4 v[kVectors];
    uint32_t m = 0;
    bool odd;
#pragma unroll
    for (unsigned i = 0; i < kVectors; ++i) {
        v[i] = uint4{0u, 0u, 0u, 0u};
        if (i * kEach * 64 * N < a.inner) {
            const unsigned at = place(i), n = count(at);
            if (n != 0) v[i] = load_values<false, true>(from + at, n);
            if constexpr (ACT != KQ8_NONE) {        // the table reads need all lanes
                if constexpr (sizeof(ELEM) == 2) v[i] = apply_vec_bf16<ACT == KQ8_GELU ? OP_GELU : OP_SWISH, WIDE>(v[i], tab);
                else v[i] = apply_vec_f32<ACT == KQ8_GELU ? OP_GELU : OP_SWISH, WIDE>(v[i], tab);
            }
            m = larger(m, largest_of_lane<ELEM>(v[i], odd));
        }
    }
    for (int by = 1; by < 64; by *= 2) m = larger(m, (uint32_t)__shfl_xor((int)m, by));
    if (lane == 0) tops[wave] = m;
    __syncthreads();
    m = tops[row * kEach];
#pragma unroll
    for (unsigned i = 1; i < kEach; ++i) m = larger(m, tops[row * kEach + i]);
    const bool finite = m < 0x7F800000u;
    const float top = __uint_as_float(m), inverse = inverse_of(top);
    if (lane == 0 && slice == 0) scales[row] = finite ? scale_of(top) : __builtin_nanf("");
#pragma unroll
    for (unsigned i = 0; i < kVectors; ++i) {
        const unsigned at = place(i);
        if (at + N > pitch - 16) continue;          // up to a whole step, zeros behind the row
        float f[N];
        widen<ELEM>(v[i], f);
        uint32_t q[N];
#pragma unroll
        for (unsigned e = 0; e < N; ++e) q[e] = finite ? rounded_code(f[e], inverse) : 0u;
        int8_t *to = codes + row * pitch + at;
        if constexpr (N == 8) *reinterpret_cast<u32x2 *>(to) = u32x2{four_codes(q[0], q[1], q[2], q[3]), four_codes(q[4], q[5], q[6], q[7])};
        else *reinterpret_cast<uint32_t *>(to) = four_codes(q[0], q[1], q[2], q[3]);
    }
    __syncthreads();

    const int8_t *xf = codes + (lane % 16 < ROWS ? lane % 16 : 0) * pitch + k;
    i32x4 sum = {0, 0, 0, 0};
    auto multiply = [&](const i32x4 &wv, unsigned step) {
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, *reinterpret_cast<const i32x4 *>(xf + step * 64), sum, 0, 0, 0);
    };
    for (unsigned first = 0; first < mine; first += kSteps) {
#pragma unroll
        for (unsigned u = 0; u < kSteps; ++u)
            if (first + u < mine) multiply(wf[u], wave + (first + u) * kWaves);
#pragma unroll
        for (unsigned u = 0; u < kSteps; ++u)
            if (first + kSteps + u < mine) wf[u] = load16<true>(w + (wave + (first + kSteps + u) * kWaves) * 64);
    }
    if (steps % kWaves == wave && a.inner % 64 != 0) multiply(load16(w + steps * 64, (int)a.inner - (int)(steps * 64 + k), a.inner), steps);
    *reinterpret_cast<i32x4 *>(&part[wave][lane % 16][lane / 16 * 4]) = sum;
    __syncthreads();
    a.x_scale = scales;
    store_joined<16, 16, kWaves, OUT>(a, o0, 0, part);
}

template <class ELEM, int ACT, bool WIDE>
ktanh_status_t launch_with(const kq8_shape_t &s, const void *x, const Operands &a, const KtLutPack &pack, ktanh_stream_t stream)
{
    const unsigned blocks = (a.outer + 15) / 16;
    auto launch = [&](auto kernel) {
        return launch_checked(kernel, blocks, 64 * kWaves, stream, a, static_cast<const ELEM *>(x), (unsigned long long)stride(s.rows, s.x_row), pack);
    };
    auto of = [&](auto out) {
        constexpr Out O = decltype(out)::value;
        if (a.rows == 1) return launch(q8_few_kernel<ELEM, ACT, WIDE, O, 1>);
        if (a.rows == 2) return launch(q8_few_kernel<ELEM, ACT, WIDE, O, 2>);
        if (a.rows <= 4) return launch(q8_few_kernel<ELEM, ACT, WIDE, O, 4>);
        return launch(q8_few_kernel<ELEM, ACT, WIDE, O, 8>);
    };
    return s.out_f32 ? of(std::integral_constant<Out, F32>()) : of(std::integral_constant<Out, BF16>());
}

// Every block of a CU makes the integers again, so at most one block to a CU, and at most 16384 values, half as many behind an activation.  us of rows in
// BFloat16, two launches | one:  1 x 4096 x 4096 8.2 | 7.2, 4 x 2048 x 4096 7.2 | 6.0, 4 x 4096 x 4096 8.8 | 8.5, 8 x 4096 x 4096 9.2 | 10.6, 1 x 2048 x 16384
// 11.6 | 12.9;  behind GELU  2 x 4096 x 4096 9.3 | 8.6, 4 x 4096 x 4096 9.6 | 10.4.  (Between launches that are not in a graph the host's time is saved as well.)
bool worth(const kq8_shape_t &s)
{
    if (s.rows > kMostRows8 || s.inner == 0 || s.inner > kMostValues || s.outer > 4096) return false;
    const size_t power = s.rows <= 2 ? s.rows : s.rows <= 4 ? 4 : 8, values = power * ((s.inner + 63) / 64 * 64);
    return values <= kMostValues / (s.activation == KQ8_NONE ? 1 : 2);
}

}  // namespace

namespace ktanh_q8 {

ktanh_status_t launch_few(const kq8_shape_t &s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, const ktanh_lut_t *lut,
                          const ktanh_lut64_t *lut64, bool wide, ktanh_stream_t stream, bool *done)
{
    *done = worth(s) && !off(w, 16) && stride(s.outer, s.w_row) % 16 == 0;
    if (!*done) return KT_OK;
    Operands a;
    a.x = nullptr;
    a.w = w;
    a.x_row = 0;
    a.w_row = stride(s.outer, s.w_row);
    a.x_scale = nullptr;
    a.w_scale = w_scale;
    a.bias = bias;
    a.out = out;
    a.out_row = stride(s.rows, s.out_row);
    a.rows = (unsigned)s.rows;
    a.outer = (unsigned)s.outer;
    a.inner = (unsigned)s.inner;
    KtLutPack pack;
    const bool none = s.activation == KQ8_NONE;
    const ktanh_status_t st = wide && !none ? pack_for(lut64, s.x_f32 != 0, &pack) : pack_for(none ? nullptr : lut, s.x_f32 != 0, &pack);
    if (st != KT_OK) return st;
    auto typed = [&](auto act, auto table) {
        constexpr int ACT = decltype(act)::value;
        constexpr bool WIDE = decltype(table)::value;
        return s.x_f32 ? launch_with<uint32_t, ACT, WIDE>(s, x, a, pack, stream) : launch_with<uint16_t, ACT, WIDE>(s, x, a, pack, stream);
    };
    auto tabled = [&](auto act) { return wide ? typed(act, std::true_type()) : typed(act, std::false_type()); };
    if (none) return typed(std::integral_constant<int, KQ8_NONE>(), std::false_type());
    return s.activation == KQ8_SWISH ? tabled(std::integral_constant<int, KQ8_SWISH>()) : tabled(std::integral_constant<int, KQ8_GELU>());
}

}  // namespace ktanh_q8
