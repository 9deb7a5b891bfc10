// libktanh: the choice of a token of each row of logits, by temperature, top-k, top-p and min-p from a given uniform number.
//
// With z the logits (capped through K-TanH where asked), tokens ranked by z, the lowest index first among equals, and weights
// w = exp((z - max) / T), all four choices are questions about the mass G(r) of the first r tokens:
//   top-k  keeps k tokens;  top-p the smallest r with G(r) >= p G(k);  min-p as many as have w >= min_p;  of the kept n the token is the
//   first with G(r) > u G(n).
// No sort of the row is needed for them.  A row is cut into bins of z, the bins' counts and masses are summed, and only the tokens of the bins that
// hold an answer are collected and sorted: all bins up to it where these are few tokens (one question answers the others then), else one bin at a
// time.  Within a bin weights are summed as integers, multiples of 2^-43 of the weight at the bin's start: such sums do not depend on
// the order in which lanes add to them; sums over bins and over sorted tokens are doubles in a fixed order.
#include "ktanh_codes.h"
#include "ktanh_stream_impl.h"

#include <cmath>
#include <type_traits>

using namespace ktanh_device;

namespace {

constexpr unsigned kThreads = 1024, kBins = kThreads;   // a bin for each lane of a block
constexpr unsigned kListed = 2048;                      // tokens that a block sorts
constexpr double kFar = 51.0;                           // KSAMPLE_MOST exp(-kFar) < 2^-53: what lies beyond does not reach a sum of doubles
constexpr double kOne = 8796093022208.0;                // 2^43: KSAMPLE_MOST of them fit 64 bits
constexpr uint32_t kNan = 0xFFFFFFFFu, kNothing = 0x007FFFFFu;   // keys of a NaN and of -infinity

typedef unsigned long long u64;

// Float32 values in their order as integers; one zero, and NaNs above all.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return kNan;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

// Rank order as one number: the higher logit first, the lower index among equals.
__device__ __forceinline__ u64 place_of(uint32_t key, uint32_t index) { return (u64)(~key) << 32 | index; }

struct Settings {
    double inverse;     // of the temperature
    double top_p, u;
    double reach;       // -log of min_p
    uint32_t top_k;
    bool greedy;
};

struct SampleArgs {
    const void *logits;
    u64 row;
    unsigned vocabulary;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    float one_temperature, one_top_p, one_min_p;
    uint32_t one_top_k;
    float cap;
    long long *tokens;
};

__device__ __forceinline__ float in_unit(float v, float otherwise) { return v >= 0.f ? (v < 1.f ? v : 1.f) : v < 0.f ? 0.f : otherwise; }

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, unsigned row)
{
    Settings s;
    const float t = a.temperature != nullptr ? a.temperature[row] : a.one_temperature;
    s.greedy = !(t > 0.f);
    s.inverse = s.greedy ? 0.0 : 1.0 / (double)t;
    s.top_p = in_unit(a.top_p != nullptr ? a.top_p[row] : a.one_top_p, 1.f);
    const float min_p = in_unit(a.min_p != nullptr ? a.min_p[row] : a.one_min_p, 0.f);
    s.reach = min_p > 0.f ? -log((double)min_p) : (double)INFINITY;
    s.u = in_unit(a.uniform[row], 0.f);
    const int32_t k = a.top_k != nullptr ? a.top_k[row] : (int32_t)a.one_top_k;
    s.top_k = k <= 0 || (uint32_t)k > a.vocabulary ? a.vocabulary : (uint32_t)k;
    return s;
}

// How far z is below the largest logit, as a power of e of the weight.
__device__ __forceinline__ double depth_of(float z, float top, double inverse)
{
    const double a = z == top ? 0.0 : ((double)top - (double)z) * inverse;
    return a < kFar ? a : (double)INFINITY;     // also a NaN, of -infinity at an infinite temperature
}

// A row of logits, its table and its cap.
template <class ELEM, bool CAP, bool WIDE, bool ALIGNED>
struct Row {
    const ELEM *from;
    unsigned size;
    float cap;
    const LaneTable &tab;

    // f(z, index, inside) for every token, by every lane of a block at once: the table reads need all lanes.
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        constexpr unsigned N = kPerLane<ELEM>;
        for (unsigned base = 0; base < size; base += kThreads * N) {
            const unsigned at = base + threadIdx.x * N;
            const unsigned count = at >= size ? 0u : size - at < N ? size - at : N;
            uint4 v = uint4{0u, 0u, 0u, 0u};
            if (count != 0) v = load_values<ALIGNED, true>(from + at, count);
            float z[N];
            widen<ELEM>(v, z);
#pragma unroll
            for (unsigned i = 0; i < N; ++i) {
                if constexpr (CAP) {
                    const float t = __uint_as_float(ktanh_f32_one<WIDE>(__float_as_uint(z[i] / cap), tab));
                    z[i] = z[i] == -INFINITY ? z[i] : cap * t;      // a masked token stays masked
                }
                f(z[i], at + i, i < count);
            }
        }
    }
};

// ------------------------------------------------------------------------------------ sums over a block
struct Mass {
    uint32_t count;
    double mass;
};
__device__ __forceinline__ Mass operator+(Mass a, Mass b) { return Mass{a.count + b.count, a.mass + b.mass}; }

struct Shared {
    Mass part[kThreads / 64];
    u64 best[kThreads / 64];
    uint32_t low[kThreads / 64];
    uint32_t count[kBins];
    u64 mass[kBins];
    u64 list[kListed];
    uint32_t listed;
    uint32_t found;
    Mass before, at;
    u64 low_place, high_place;
};

// Sum of the lanes up to and with this one; `total` is that of all.
__device__ __forceinline__ Mass sum_up_to(Mass v, Shared &sh, Mass &total)
{
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    Mass run = v;
#pragma unroll
    for (unsigned by = 1; by < 64; by *= 2) {
        const Mass other{(uint32_t)__shfl_up((int)run.count, by), __shfl_up(run.mass, by)};
        if (lane >= by) run = run + other;
    }
    __syncthreads();        // the last use of part
    if (lane == 63) sh.part[wave] = run;
    __syncthreads();
    Mass first{0, 0};
    total = Mass{0, 0};
#pragma unroll
    for (unsigned i = 0; i < kThreads / 64; ++i) {
        if (i < wave) first = first + sh.part[i];
        total = total + sh.part[i];
    }
    return first + run;
}

// ------------------------------------------------------------------------------------ one row
// Sorts sh.list[0 .. n), n <= kListed; what is behind it up to a power of two is overwritten.
__device__ __forceinline__ void sort_list(Shared &sh, unsigned n)
{
    unsigned size = 64;
    while (size < n) size *= 2;
    for (unsigned i = n + threadIdx.x; i < size; i += kThreads) sh.list[i] = ~0ull;
    for (unsigned k = 2; k <= size; k *= 2)
        for (unsigned j = k / 2; j > 0; j /= 2) {
            __syncthreads();
            const unsigned a = (threadIdx.x / j) * 2 * j + threadIdx.x % j, b = a + j;
            if (b < size) {
                const u64 x = sh.list[a], y = sh.list[b];
                if ((x > y) == ((a & k) == 0)) {
                    sh.list[a] = y;
                    sh.list[b] = x;
                }
            }
        }
    __syncthreads();
}

template <class ROW>
struct Sampler {
    const ROW &row;
    const Settings &s;
    Shared &sh;
    float top, spread;      // the largest logit; bins a unit of z
    double width;           // of a bin, as a power of e

    __device__ __forceinline__ unsigned bin_of(float z) const
    {
        const float d = z == top ? 0.f : (top - z) * spread;
        return d < (float)(kBins - 1) ? (unsigned)d : kBins - 1;
    }

    // A token's part of its bin's mass.
    __device__ __forceinline__ u64 part_of(double depth, unsigned bin) const { return (u64)(exp(bin * width - depth) * kOne + 0.5); }
    __device__ __forceinline__ double unit_of(unsigned bin) const { return exp(-(bin * width)) / kOne; }

    // Counts and masses of the bins into sh.count and sh.mass; how many tokens min-p keeps.
    __device__ __forceinline__ uint32_t fill_bins()
    {
        sh.count[threadIdx.x] = 0;
        sh.mass[threadIdx.x] = 0;
        __syncthreads();
        uint32_t kept = 0;
        row.each([&](float z, unsigned, bool inside) {
            const double depth = depth_of(z, top, s.inverse);
            if (!inside || !(depth < kFar)) return;
            const unsigned b = bin_of(z);
            atomicAdd(&sh.count[b], 1u);
            atomicAdd(&sh.mass[b], part_of(depth, b));
            kept += depth <= s.reach;
        });
        Mass total;
        sum_up_to(Mass{kept, 0.0}, sh, total);
        return total.count;
    }

    // Tokens of bins lo .. hi with places first .. last into sh.list, sorted; how many.
    __device__ __forceinline__ unsigned collect(unsigned lo, unsigned hi, u64 first, u64 last)
    {
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        row.each([&](float z, unsigned i, bool inside) {
            if (!inside) return;
            const unsigned b = bin_of(z);
            if (b < lo || b > hi) return;
            const u64 p = place_of(key_of(z), i);
            if (p < first || p > last || !(depth_of(z, top, s.inverse) < kFar)) return;
            const unsigned at = atomicAdd(&sh.listed, 1u);
            if (at < kListed) sh.list[at] = p;
        });
        __syncthreads();
        const unsigned n = sh.listed;
        if (n <= kListed) sort_list(sh, n);
        return n;
    }

    __device__ __forceinline__ double listed_weight(unsigned i, unsigned n) const
    {
        return i < n ? exp(-depth_of(value_of_key(~(uint32_t)(sh.list[i] >> 32)), top, s.inverse)) : 0.0;
    }

    // The first listed token for which `reached(count, mass)` holds, of all tokens up to it (the last one if for none): its index in the list and,
    // in `kept`, that count and mass.  `before`: what ranks before the list.
    template <class F>
    __device__ __forceinline__ unsigned first_listed(unsigned n, Mass before, F reached, Mass &kept)
    {
        const unsigned i = threadIdx.x * 2;
        const double w0 = listed_weight(i, n), w1 = listed_weight(i + 1, n);
        Mass total;
        const Mass m1 = before + sum_up_to(Mass{(i < n ? 1u : 0u) + (i + 1 < n ? 1u : 0u), w0 + w1}, sh, total);
        const Mass m0{m1.count - (i + 1 < n ? 1u : 0u), m1.mass - w1};
        __syncthreads();
        if (threadIdx.x == 0) sh.found = n - 1;
        __syncthreads();
        if (i < n && reached(m0.count, m0.mass)) atomicMin(&sh.found, i);
        else if (i + 1 < n && reached(m1.count, m1.mass)) atomicMin(&sh.found, i + 1);
        __syncthreads();
        const unsigned at = sh.found;
        if (i == at) sh.at = m0;
        else if (i + 1 == at) sh.at = m1;
        __syncthreads();
        kept = sh.at;
        return at;
    }

    // The same for the bins in sh.count and sh.mass that have tokens, whose masses are multiples of `unit` (of the lane's bin): the bin, and what
    // is before it and with it.
    template <class F>
    __device__ __forceinline__ unsigned first_bin(Mass before, double unit, F reached, Mass &found, Mass &with)
    {
        const Mass own{sh.count[threadIdx.x], (double)sh.mass[threadIdx.x] * unit};
        Mass total;
        const Mass m1 = before + sum_up_to(own, sh, total);
        const bool some = own.count != 0, last = some && m1.count == before.count + total.count;
        __syncthreads();
        if (threadIdx.x == 0) sh.found = kBins;
        __syncthreads();
        if (some && (last || reached(m1.count, m1.mass))) atomicMin(&sh.found, threadIdx.x);
        __syncthreads();
        const unsigned at = sh.found;
        if (threadIdx.x == at) {
            sh.before = Mass{m1.count - own.count, m1.mass - own.mass};
            sh.at = m1;
        }
        __syncthreads();
        found = sh.before;
        with = sh.at;
        return at;
    }

    // The answer within a bin of more tokens than a list holds: bins of places inside it, until they are few.  Leaves them listed.
    template <class F>
    __device__ __forceinline__ unsigned narrow(unsigned bin, Mass &before, F reached)
    {
        __syncthreads();
        if (threadIdx.x == 0) {
            sh.low_place = ~0ull;
            sh.high_place = 0;
        }
        __syncthreads();
        row.each([&](float z, unsigned i, bool inside) {
            if (!inside || bin_of(z) != bin || !(depth_of(z, top, s.inverse) < kFar)) return;
            const u64 p = place_of(key_of(z), i);
            atomicMin(&sh.low_place, p);
            atomicMax(&sh.high_place, p);
        });
        __syncthreads();
        u64 first = sh.low_place, last = sh.high_place;
        for (;;) {
            const u64 step = (last - first) / kBins + 1;
            __syncthreads();
            sh.count[threadIdx.x] = 0;
            sh.mass[threadIdx.x] = 0;
            __syncthreads();
            row.each([&](float z, unsigned i, bool inside) {
                if (!inside || bin_of(z) != bin) return;
                const u64 p = place_of(key_of(z), i);
                const double depth = depth_of(z, top, s.inverse);
                if (p < first || p > last || !(depth < kFar)) return;
                const unsigned b = (unsigned)((p - first) / step);
                atomicAdd(&sh.count[b], 1u);
                atomicAdd(&sh.mass[b], part_of(depth, bin));
            });
            __syncthreads();
            Mass with;
            const unsigned b = first_bin(before, unit_of(bin), reached, before, with);
            first += b * step;
            if (last - first >= step) last = first + step - 1;
            if (with.count - before.count <= kListed) return collect(bin, bin, first, last);     // a step of 1 holds one token
        }
    }

    // Lists what is needed to answer in `bin`, of which `before` is before it and `with` includes it.
    template <class F>
    __device__ __forceinline__ unsigned list_bin(unsigned bin, Mass &before, Mass with, F reached)
    {
        if (with.count - before.count <= kListed) return collect(bin, bin, 0, ~0ull);
        const uint32_t count = sh.count[threadIdx.x];       // the bins of the row, which the narrower ones overwrite
        const u64 mass = sh.mass[threadIdx.x];
        const unsigned n = narrow(bin, before, reached);
        __syncthreads();
        sh.count[threadIdx.x] = count;
        sh.mass[threadIdx.x] = mass;
        __syncthreads();
        return n;
    }

    // The first `kept.count` tokens are kept so far: the ones up to the first of all for which `reached` holds, from the bins of the row.
    template <class F>
    __device__ __forceinline__ Mass resolved(double unit, F reached)
    {
        const Mass none{0, 0.0};
        Mass before, with, kept;
        const unsigned bin = first_bin(none, unit, reached, before, with);
        const unsigned n = list_bin(bin, before, with, reached);
        first_listed(n, before, reached, kept);
        return kept;
    }

    __device__ __forceinline__ long long choose()
    {
        const uint32_t by_min = fill_bins();
        const double unit = unit_of(threadIdx.x);
        const Mass none{0, 0.0};
        auto has_k = [&](uint32_t count, double) { return count >= s.top_k; };
        Mass before, kept;
        unsigned bin = first_bin(none, unit, has_k, before, kept);      // top-k's, and what it keeps if not part of that bin
        if (kept.count <= kListed) {
            const unsigned n = collect(0, bin, 0, ~0ull);
            first_listed(n, none, has_k, kept);
            return choose_listed(n, kept, by_min);
        }
        if (s.top_k < kept.count) kept = resolved(unit, has_k);
        if (s.top_p < 1.0) {
            const double wanted = s.top_p * kept.mass;
            const uint32_t most = kept.count;
            auto has_p = [&](uint32_t count, double mass) { return mass >= wanted || count >= most; };
            Mass with;
            bin = first_bin(none, unit, has_p, before, with);
            if (with.count <= kListed) return choose_listed(collect(0, bin, 0, ~0ull), kept, by_min);
            kept = resolved(unit, has_p);
        }
        if (by_min < kept.count) kept = resolved(unit, [&](uint32_t count, double) { return count >= by_min; });
        const double target = s.u * kept.mass;
        auto has_u = [&](uint32_t count, double mass) { return mass > target || count >= kept.count; };
        Mass with;
        bin = first_bin(none, unit, has_u, before, with);
        const unsigned n = list_bin(bin, before, with, has_u);
        return token_listed(first_listed(n, before, has_u, with));
    }

    __device__ __forceinline__ long long token_listed(unsigned i) const { return (long long)(uint32_t)sh.list[i]; }

    // top-p, min-p and the choice where the first n tokens by rank are listed and they hold the answers; `kept` is what top-k keeps.
    __device__ __forceinline__ long long choose_listed(unsigned n, Mass kept, uint32_t by_min)
    {
        const Mass none{0, 0.0};
        if (s.top_p < 1.0) {
            const double wanted = s.top_p * kept.mass;
            const uint32_t most = kept.count;
            first_listed(n, none, [&](uint32_t count, double mass) { return mass >= wanted || count >= most; }, kept);
        }
        if (by_min < kept.count) first_listed(n, none, [&](uint32_t count, double) { return count >= by_min; }, kept);
        const double target = s.u * kept.mass;
        Mass with;
        return token_listed(first_listed(n, none, [&](uint32_t count, double mass) { return mass > target || count >= kept.count; }, with));
    }
};

template <class ELEM, bool CAP, bool WIDE, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Row<ELEM, CAP, WIDE, ALIGNED> row{static_cast<const ELEM *>(a.logits) + blockIdx.x * a.row, a.vocabulary, a.cap, tab};
    const Settings s = settings_of(a, blockIdx.x);
    // the first token by rank, and the smallest logit that is not masked
    u64 best = ~0ull;
    uint32_t low = kNan;
    row.each([&](float z, unsigned i, bool inside) {
        if (!inside) return;
        const uint32_t k = key_of(z);
        const u64 p = place_of(k, i);
        best = p < best ? p : best;
        if (k > kNothing) low = k < low ? k : low;
    });
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const u64 p = __shfl_xor(best, step);
        const uint32_t k = (uint32_t)__shfl_xor((int)low, step);
        best = p < best ? p : best;
        low = k < low ? k : low;
    }
    if (threadIdx.x % 64 == 0) {
        sh.best[threadIdx.x / 64] = best;
        sh.low[threadIdx.x / 64] = low;
    }
    __syncthreads();
#pragma unroll
    for (unsigned i = 0; i < kThreads / 64; ++i) {
        best = sh.best[i] < best ? sh.best[i] : best;
        low = sh.low[i] < low ? sh.low[i] : low;
    }
    const uint32_t key = ~(uint32_t)(best >> 32);
    long long token = (long long)(uint32_t)best;
    if (key == kNan || key <= kNothing) token = -1;     // a NaN, or nothing to choose from
    else if (!s.greedy && s.top_k != 1) {
        const float top = value_of_key(key), far = (float)(kFar / s.inverse), down = top - value_of_key(low);
        const float range = down < far ? down : far, spread = range > 0.f ? (float)kBins / range : 0.f;
        const double width = spread > 0.f ? s.inverse / (double)spread : 0.0;
        Sampler<Row<ELEM, CAP, WIDE, ALIGNED>> sampler{row, s, sh, top, spread, width < kFar ? width : 0.0};
        token = sampler.choose();
    }
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = token;
}

// ------------------------------------------------------------------------------------ host side
bool in_range(double v, double most) { return v >= 0.0 && v <= most; }

template <class Lut>
ktanh_status_t sample_entry(const ksample_shape_t *s, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                            const float *top_p, const float *min_p, int64_t *tokens, const Lut *lut, ktanh_stream_t stream)
{
    constexpr bool WIDE = is_wide(static_cast<const Lut *>(nullptr));
    if (s == nullptr) return KT_ERR_NULL;
    if (s->rows > (size_t)1 << 30 || s->vocabulary == 0 || s->vocabulary > KSAMPLE_MOST || s->row > (size_t)1 << 40 ||
        !in_range(s->temperature, 3e38) || !in_range(s->top_p, 1.0) || !in_range(s->min_p, 1.0) || !in_range(s->cap, 3e38) ||
        (s->cap > 0.0 && s->cap < 1e-30))
        return KT_ERR_SHAPE;
    if (s->rows == 0) return KT_OK;
    if (logits == nullptr || uniform == nullptr || tokens == nullptr) return KT_ERR_NULL;
    auto off = [](const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
    if (off(logits, s->f32 ? 4 : 2) || off(uniform, 4) || off(temperature, 4) || off(top_k, 4) || off(top_p, 4) || off(min_p, 4) || off(tokens, 8))
        return KT_ERR_ALIGN;
    KtLutPack pack;
    const ktanh_status_t st = pack_for(lut, true, &pack);
    if (st != KT_OK) return st;
    SampleArgs a;
    a.logits = logits;
    a.row = s->rows > 1 ? s->row : 0;
    a.vocabulary = (unsigned)s->vocabulary;
    a.uniform = uniform;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.one_temperature = (float)s->temperature;
    a.one_top_k = s->top_k > s->vocabulary ? 0u : (uint32_t)s->top_k;
    a.one_top_p = (float)s->top_p;
    a.one_min_p = (float)s->min_p;
    a.cap = (float)s->cap;
    a.tokens = reinterpret_cast<long long *>(tokens);
    const bool aligned = !off(logits, 16) && a.row % (s->f32 ? 4 : 8) == 0;
    auto launch = [&](auto kernel) { return launch_checked(kernel, (unsigned)s->rows, kThreads, stream, a, pack); };
    auto placed = [&](auto elem, auto capped) {
        typedef decltype(elem) ELEM;
        constexpr bool CAP = decltype(capped)::value, W = CAP && WIDE;
        return aligned ? launch(sample_kernel<ELEM, CAP, W, true>) : launch(sample_kernel<ELEM, CAP, W, false>);
    };
    if (s->f32) return s->cap > 0.0 ? placed(uint32_t(), std::true_type()) : placed(uint32_t(), std::false_type());
    return s->cap > 0.0 ? placed(uint16_t(), std::true_type()) : placed(uint16_t(), std::false_type());
}

}  // namespace

extern "C" ktanh_status_t ksample(const ksample_shape_t *shape, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                                  const float *top_p, const float *min_p, int64_t *tokens, const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return sample_entry(shape, logits, uniform, temperature, top_k, top_p, min_p, tokens, lut, stream);
}
extern "C" ktanh_status_t ksample64(const ksample_shape_t *shape, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                                    const float *top_p, const float *min_p, int64_t *tokens, const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return sample_entry(shape, logits, uniform, temperature, top_k, top_p, min_p, tokens, lut, stream);
}
