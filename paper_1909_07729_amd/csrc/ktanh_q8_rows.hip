// libktanh: rows of values, or of an activation's outputs, in 8-bit integers with a scale for each row.
//
// One pass: a row is held in registers between the search for its largest magnitude and its rounding (rows beyond 32768 BFloat16 or 16384
// Float32 values are read twice).  Bound by memory: 3 bytes a BFloat16 value; 8192 rows of 16384 take 72 us (5.6 TB/s), behind GELU 85.  A block to a
// row, of as many lanes as keep it in 8 vectors each: what a lane holds it needs again, and its rounding waits for the whole row's largest.
#include "ktanh_codes.h"
#include "ktanh_q8.h"
#include "ktanh_stream_impl.h"

#include <type_traits>

using namespace ktanh_device;
using namespace ktanh_q8;

namespace {

// The largest of a block's lanes, in all of them.  `part`: a word for each wavefront in LDS.
template <unsigned THREADS>
__device__ __forceinline__ uint32_t largest_of_block(uint32_t m, uint32_t *part)
{
#pragma unroll
    for (int step = 1; step < 64; step *= 2) m = larger(m, (uint32_t)__shfl_xor((int)m, step));
    if constexpr (THREADS > 64) {
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
        __syncthreads();
        m = part[0];
#pragma unroll
        for (unsigned i = 1; i < THREADS / 64; ++i) m = larger(m, part[i]);
    }
    return m;
}

template <class ELEM, int ACT, bool WIDE>
__device__ __forceinline__ uint4 activated(uint4 v, const LaneTable &tab)
{
    if constexpr (ACT == KQ8_NONE) return v;
    else if constexpr (sizeof(ELEM) == 2) return apply_vec_bf16<ACT == KQ8_GELU ? OP_GELU : OP_SWISH, WIDE>(v, tab);
    else return apply_vec_f32<ACT == KQ8_GELU ? OP_GELU : OP_SWISH, WIDE>(v, tab);
}

// A row to a block of THREADS lanes, R vectors of each lane (0: any number, read twice).  The table reads of the activations need every
// lane enabled: bounds predicate the accesses alone.
template <class ELEM, int ACT, bool WIDE, bool ALIGNED, unsigned THREADS, unsigned R>
__global__ __launch_bounds__(THREADS) void q8_rows_kernel(const ELEM *x, unsigned long long x_row, unsigned cols, int8_t *codes,
                                                          unsigned long long codes_row, float *scales, KtLutPack pack)
{
    constexpr unsigned N = kPerLane<ELEM>, kInf = 0x7F800000u;
    __shared__ uint32_t part[THREADS / 64];
    const LaneTable tab(pack);
    const ELEM *from = x + blockIdx.x * x_row;
    int8_t *to = codes + blockIdx.x * codes_row;
    auto count_at = [&](unsigned at) { return at >= cols ? 0u : cols - at < N ? cols - at : N; };
    auto load = [&](unsigned at) {
        const unsigned count = count_at(at);
        uint4 v = uint4{0u, 0u, 0u, 0u};
        if (count != 0) v = load_values<ALIGNED, true>(from + at, count);
        return v;
    };
    bool odd;
    uint32_t m = 0;
    uint4 v[R == 0 ? 1 : R];
    if constexpr (R == 0) {
        for (unsigned at = 0; at < cols; at += THREADS * N)
            m = larger(m, largest_of_lane<ELEM>(activated<ELEM, ACT, WIDE>(load(at + threadIdx.x * N), tab), odd));
    } else {
#pragma unroll
        for (unsigned r = 0; r < R; ++r) v[r] = load((r * THREADS + threadIdx.x) * N);
#pragma unroll
        for (unsigned r = 0; r < R; ++r) {
            v[r] = activated<ELEM, ACT, WIDE>(v[r], tab);
            m = larger(m, largest_of_lane<ELEM>(v[r], odd));
            // one after the other: all at once take 193 registers a lane where these take 64 (8192 rows of 16384 behind GELU 152 us against 85)
            if constexpr (ACT != KQ8_NONE) __builtin_amdgcn_sched_barrier(0);
        }
    }
    m = largest_of_block<THREADS>(m, part);
    const bool finite = m < kInf;
    const float top = __uint_as_float(m), inverse = inverse_of(top);
    if (threadIdx.x == 0) scales[blockIdx.x] = finite ? scale_of(top) : __builtin_nanf("");
    auto store = [&](unsigned at, uint4 w) {
        float f[N];
        widen<ELEM>(w, f);
        uint32_t q[N];
#pragma unroll
        for (unsigned i = 0; i < N; ++i) q[i] = finite ? rounded_code(f[i], inverse) : 0u;
        uint2 c{four_codes(q[0], q[1], q[2], q[3]), 0u};
        if constexpr (N == 8) c.y = four_codes(q[4], q[5], q[6], q[7]);
        const unsigned count = count_at(at);
        if (count != 0) store_codes<ALIGNED, ELEM>(to + at, c, count);
    };
    if constexpr (R == 0) {
        for (unsigned at = 0; at < cols; at += THREADS * N) {
            const uint4 w = activated<ELEM, ACT, WIDE>(load(at + threadIdx.x * N), tab);
            store(at + threadIdx.x * N, w);
        }
    } else {
#pragma unroll
        for (unsigned r = 0; r < R; ++r) store((r * THREADS + threadIdx.x) * N, v[r]);
    }
}

template <class ELEM, int ACT, class Lut>
ktanh_status_t launch_rows(const kq8_shape_t &s, const void *x, int8_t *codes, size_t codes_row, float *scales, const Lut *lut, ktanh_stream_t stream)
{
    constexpr bool WIDE = is_wide(static_cast<const Lut *>(nullptr));
    constexpr size_t N = kPerLane<ELEM>;
    KtLutPack pack;
    const ktanh_status_t st = pack_for(ACT == KQ8_NONE ? nullptr : lut, sizeof(ELEM) == 4, &pack);
    if (st != KT_OK) return st;
    const size_t x_row = stride(s.rows, s.x_row);
    codes_row = stride(s.rows, codes_row);
    const Memory in = matrix(x, s.rows, s.inner, x_row, sizeof(ELEM)), out = matrix(codes, s.rows, s.inner, codes_row, 1),
                 scaling = vector(scales, s.rows * sizeof(float));
    if (!apart(in, out) || !apart(in, scaling) || !apart(out, scaling)) return KT_ERR_SHAPE;
    const bool aligned = !off(x, 16) && x_row % N == 0 && !off(codes, N) && codes_row % N == 0;
    // a launch has fewer than 2^32 lanes
    auto launch = [&](auto kernel, unsigned threads) {
        const size_t most = kMostLanes / threads;
        for (size_t first = 0; first < s.rows; first += most) {
            const size_t rows = s.rows - first < most ? s.rows - first : most;
            const ktanh_status_t done =
                launch_checked(kernel, (unsigned)rows, threads, stream, static_cast<const ELEM *>(x) + first * x_row, (unsigned long long)x_row, (unsigned)s.inner,
                               codes + first * codes_row, (unsigned long long)codes_row, scales + first, pack);
            if (done != KT_OK) return done;
        }
        return KT_OK;
    };
    auto of = [&](auto on_grid) {
        constexpr bool ALIGNED = decltype(on_grid)::value;
        const size_t vectors = (s.inner + N - 1) / N;
        if (vectors <= 64) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 64, 1>, 64);
        // 8192 rows of 1024: 6.7 us, behind GELU 8.9; with the next blocks 8.1 and 12.9
        if (vectors <= 128) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 128, 1>, 128);
        if (vectors <= 256) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 256, 1>, 256);
        if (vectors <= 512) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 256, 2>, 256);
        if (vectors <= 1024) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 256, 4>, 256);
        if (vectors <= 2048) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 256, 8>, 256);
        if (vectors <= 4096) return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 1024, 4>, 1024);
        return launch(q8_rows_kernel<ELEM, ACT, WIDE, ALIGNED, 1024, 0>, 1024);
    };
    return aligned ? of(std::true_type()) : of(std::false_type());
}

template <class Lut>
ktanh_status_t rows_entry(const kq8_shape_t *s, const void *x, int8_t *codes, size_t codes_row, float *scales, const Lut *lut, ktanh_stream_t stream)
{
    const ktanh_status_t st = check_rows(s);
    if (st != KT_OK) return st;
    if (s->rows == 0) return KT_OK;
    if (scales == nullptr || (s->inner != 0 && (x == nullptr || codes == nullptr))) return KT_ERR_NULL;
    if (off(x, s->x_f32 ? 4 : 2) || off(scales, 4)) return KT_ERR_ALIGN;
    if (codes_row > kMostStride || (s->rows > 1 && codes_row < s->inner)) return KT_ERR_SHAPE;
    auto launch = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        return s->x_f32 ? launch_rows<uint32_t, ACT>(*s, x, codes, codes_row, scales, lut, stream)
                        : launch_rows<uint16_t, ACT>(*s, x, codes, codes_row, scales, lut, stream);
    };
    if (s->activation == KQ8_NONE) {  // no table: one instance for both widths
        const ktanh_lut_t *none = nullptr;
        return s->x_f32 ? launch_rows<uint32_t, KQ8_NONE>(*s, x, codes, codes_row, scales, none, stream)
                        : launch_rows<uint16_t, KQ8_NONE>(*s, x, codes, codes_row, scales, none, stream);
    }
    return s->activation == KQ8_SWISH ? launch(std::integral_constant<int, KQ8_SWISH>()) : launch(std::integral_constant<int, KQ8_GELU>());
}

}  // namespace

extern "C" ktanh_status_t kq8_rows(const kq8_shape_t *shape, const void *x, int8_t *codes, size_t codes_row, float *scales, const ktanh_lut_t *lut,
                                   ktanh_stream_t stream)
{
    return rows_entry(shape, x, codes, codes_row, scales, lut, stream);
}
extern "C" ktanh_status_t kq8_rows64(const kq8_shape_t *shape, const void *x, int8_t *codes, size_t codes_row, float *scales, const ktanh_lut64_t *lut,
                                     ktanh_stream_t stream)
{
    return rows_entry(shape, x, codes, codes_row, scales, lut, stream);
}
