// libktanh: the choice of a token of each row of logits, by temperature, top-k, top-p and min-p from a given uniform number.
//
// With z the logits (capped through K-TanH where asked), tokens ranked by z, the lowest index first among equals, and weights
// w = exp((z - max) / T), all four choices are questions about the mass G(r) of the first r tokens:
//   top-k  keeps k tokens;  top-p the smallest r with G(r) >= p G(k);  min-p as many as have w >= min_p;  of the kept n the token is the
//   first with G(r) > u G(n).
// No sort of the row is needed for them.  The row is cut into bins of z, some bins to a factor of two of the weight, whose counts and masses
// say which bins hold the answers; the tokens of these alone are listed and sorted, in most rows once.
//
// Within a bin weights are summed as integers, multiples of 2^-32 of the power of two above: such sums do not depend on the order in which
// lanes add to them.  Sums over bins and over sorted tokens are doubles in a fixed order.
//
// A block holds up to 32768 logits in registers.  Rows of no more take one launch, and are read once.  Longer ones are cut into chunks of that size
// and take four: the chunks' largest logits, their bins, their tokens of the bins that hold answers, and one block for the answers.
#include "ktanh_codes.h"
#include "ktanh_stream_impl.h"

#include <cmath>
#include <type_traits>

using namespace ktanh_device;

namespace {

constexpr unsigned kThreads = 1024, kBins = kThreads;   // a bin for each lane of a block
constexpr unsigned kListed = 2048;                      // tokens that a block sorts
constexpr unsigned kChunk = 32 * kThreads;
constexpr unsigned kSteps = 7;                          // log2 of the finest bins to a factor of two
constexpr double kFar = 73.5;                           // KSAMPLE_MOST 2^-kFar < 2^-53: what lies beyond does not reach a sum of doubles
constexpr double kLog2e = 1.4426950408889634;
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

struct SampleArgs {
    const void *logits;
    u64 row;
    unsigned vocabulary, chunks;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    float one_temperature, one_top_p, one_min_p;
    uint32_t one_top_k;
    float cap;
    long long *tokens;
    // of rows in chunks: by row and chunk, and by row
    u64 *best, *bins, *list;
    uint32_t *low, *by_min, *listed;
};

// A value that all lanes have alike, in scalar registers: the vector ones hold the logits.
template <class T>
__device__ __forceinline__ T uniform(T v)
{
    static_assert(sizeof(T) % 4 == 0, "words");
    uint32_t w[sizeof(T) / 4];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    __builtin_memcpy(&v, w, sizeof(T));
    return v;
}

struct Settings {
    double scale;       // log2(e) / temperature
    double top_p, u;
    double reach;       // -log2 of min_p
    uint32_t top_k;
    bool greedy;
};

__device__ __forceinline__ float in_unit(float v, float otherwise) { return v >= 0.f ? (v < 1.f ? v : 1.f) : v < 0.f ? 0.f : otherwise; }

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, unsigned row)
{
    Settings s;
    const float t = a.temperature != nullptr ? a.temperature[row] : a.one_temperature;
    const int32_t k = a.top_k != nullptr ? a.top_k[row] : (int32_t)a.one_top_k;
    s.top_k = k <= 0 || (uint32_t)k > a.vocabulary ? a.vocabulary : (uint32_t)k;
    s.greedy = !(t > 0.f) || s.top_k == 1;
    s.scale = s.greedy ? 0.0 : uniform(kLog2e / (double)t);
    s.top_p = (double)in_unit(a.top_p != nullptr ? a.top_p[row] : a.one_top_p, 1.f);
    const float min_p = in_unit(a.min_p != nullptr ? a.min_p[row] : a.one_min_p, 0.f);
    s.reach = uniform(min_p > 0.f ? -log2((double)min_p) : (double)INFINITY);
    s.top_p = uniform(s.top_p);
    s.u = uniform((double)in_unit(a.uniform[row], 0.f));
    return s;
}

// ------------------------------------------------------------------------------------ logits
template <class ELEM>
__device__ __forceinline__ uint4 load_logits(const ELEM *from, unsigned at, unsigned end)
{
    constexpr unsigned N = kPerLane<ELEM>;
    const unsigned count = at >= end ? 0u : end - at < N ? end - at : N;
    uint4 v = uint4{0u, 0u, 0u, 0u};
    if (count != 0) v = load_values<false, true>(from + at, count);
    return v;
}
template <class ELEM, bool CAP, bool WIDE>
__device__ __forceinline__ void logits_of(uint4 v, unsigned at, unsigned end, float cap, const LaneTable &tab, float (&z)[kPerLane<ELEM>])
{
    widen<ELEM>(v, z);
#pragma unroll
    for (unsigned i = 0; i < kPerLane<ELEM>; ++i) {
        if constexpr (CAP) {    // the table reads need all lanes
            const float t = __uint_as_float(ktanh_f32_one<WIDE>(__float_as_uint(z[i] / cap), tab));
            z[i] = z[i] == -INFINITY ? z[i] : cap * t;      // a masked token stays masked
        }
        if (at + i >= end) z[i] = -INFINITY;                // what is behind the row is like masked tokens
    }
}

// Logits of `first` .. `end` - 1 in a block's registers, E to a lane.
template <class ELEM, bool CAP, bool WIDE, unsigned E>
struct Held {
    static constexpr unsigned N = kPerLane<ELEM>;
    float z[E / N][N];
    unsigned first;

    __device__ __forceinline__ Held(const ELEM *from, unsigned first, unsigned end, float cap, const LaneTable &tab) : first(first)
    {
        uint4 raw[E / N];
#pragma unroll
        for (unsigned v = 0; v < E / N; ++v) raw[v] = load_logits(from, place(v), end);
#pragma unroll
        for (unsigned v = 0; v < E / N; ++v) {
            logits_of<ELEM, CAP, WIDE>(raw[v], place(v), end, cap, tab, z[v]);
            if constexpr (CAP) {    // one vector at a time: all at once do not fit the registers
#pragma unroll
                for (unsigned i = 0; i < N; ++i) asm volatile("" : "+v"(z[v][i]));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    __device__ __forceinline__ unsigned place(unsigned v) const { return first + (v * kThreads + threadIdx.x) * N; }
    // f(z, index) for each, by every lane of a block.  What f makes of a logit is made again in the next pass, and not kept.
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
#pragma unroll
        for (unsigned v = 0; v < E / N; ++v) {
#pragma unroll
            for (unsigned i = 0; i < N; ++i) asm volatile("" : "+v"(z[v][i]));
#pragma unroll
            for (unsigned i = 0; i < N; ++i) {
                f(z[v][i], place(v) + i);
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
};

// The same from memory, each time.
template <class ELEM, bool CAP, bool WIDE>
struct Read {
    const ELEM *from;
    unsigned end;
    float cap;
    const LaneTable &tab;

    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        constexpr unsigned N = kPerLane<ELEM>;
        for (unsigned base = 0; base < end; base += kThreads * N) {
            const unsigned at = base + threadIdx.x * N;
            float z[N];
            logits_of<ELEM, CAP, WIDE>(load_logits(from, at, end), at, end, cap, tab, z);
#pragma unroll
            for (unsigned i = 0; i < N; ++i) f(z[i], at + i);
        }
    }
};

// ------------------------------------------------------------------------------------ a block's memory and sums
struct Mass {
    uint32_t count;
    double mass;
};
__device__ __forceinline__ Mass operator+(Mass a, Mass b) { return Mass{a.count + b.count, a.mass + b.mass}; }

struct Shared {
    Mass part[kThreads / 64];
    u64 best[kThreads / 64];
    uint32_t low[kThreads / 64];
    double power[1u << kSteps];     // 2^(-j / 128)
    u64 bins[kBins];                // count << 48 | mass
    Mass own[kBins], upto[kBins];   // of each bin, and of all up to it: a lane's own, which its registers have no room for
    uint32_t flags[kBins / 32];     // bins whose tokens are listed
    uint32_t starts[kBins];         // of the flagged bins in the list
    u64 list[kListed];
    uint32_t listed, found;
    Mass before, at;
    u64 low_place, high_place;
};

// Sums over the first lanes of a wavefront.
template <unsigned LANES>
__device__ __forceinline__ Mass scanned(Mass v)
{
    const unsigned lane = threadIdx.x % LANES;
#pragma unroll
    for (unsigned by = 1; by < LANES; by *= 2) {
        const Mass other{(uint32_t)__shfl_up((int)v.count, by), __shfl_up(v.mass, by)};
        if (lane >= by) v = v + other;
    }
    return v;
}

// Sum of the lanes up to and with this one; `total` is that of all.
__device__ __forceinline__ Mass sum_up_to(Mass v, Shared &sh, Mass &total)
{
    constexpr unsigned kWaves = kThreads / 64;
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const Mass run = scanned<64>(v);
    __syncthreads();        // the last use of part
    if (lane == 63) sh.part[wave] = run;
    __syncthreads();
    const Mass parts = scanned<kWaves>(sh.part[lane % kWaves]);
    total = Mass{(uint32_t)__shfl((int)parts.count, kWaves - 1), __shfl(parts.mass, kWaves - 1)};
    const Mass first{(uint32_t)__shfl((int)parts.count, (int)wave - 1), __shfl(parts.mass, (int)wave - 1)};
    return wave != 0 ? first + run : run;
}

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

// The first token by rank of a source, and the smallest logit that is not masked, as its key.
template <class SOURCE>
__device__ __forceinline__ void ends_of(SOURCE &source, Shared &sh, u64 &best, uint32_t &low)
{
    best = ~0ull;
    low = kNan;
    source.each([&](float z, unsigned i) {
        const uint32_t k = key_of(z);
        const u64 p = place_of(k, i);
        best = p < best ? p : best;
        if (k > kNothing) low = k < low ? k : low;
    });
    auto meet = [&](int lanes) {
        for (int step = 1; step < lanes; step *= 2) {
            const u64 p = __shfl_xor(best, step);
            const uint32_t k = (uint32_t)__shfl_xor((int)low, step);
            best = p < best ? p : best;
            low = k < low ? k : low;
        }
    };
    meet(64);
    if (threadIdx.x % 64 == 0) {
        sh.best[threadIdx.x / 64] = best;
        sh.low[threadIdx.x / 64] = low;
    }
    __syncthreads();
    best = sh.best[threadIdx.x % (kThreads / 64)];
    low = sh.low[threadIdx.x % (kThreads / 64)];
    meet(kThreads / 64);
}

// ------------------------------------------------------------------------------------ weights and bins
// Depth: how far a logit is below the largest, as the power of two that its weight is below 1.
struct Weights {
    float top;
    double scale;
    unsigned shift;     // kSteps less the log2 of the bins to a factor of two

    __device__ __forceinline__ Weights(uint32_t top_key, uint32_t low_key, double scale) : top(uniform(value_of_key(top_key))), scale(scale)
    {
        const double down = ((double)top - (double)value_of_key(low_key)) * scale, range = down < kFar ? down : kFar;
        unsigned by = 0;    // kBins = 8 << kSteps
        while (by < 4 && range > (double)(7u << by)) ++by;
        shift = uniform(by);
    }
    __device__ __forceinline__ double depth_of(float z) const
    {
        const double d = z == top ? 0.0 : ((double)top - (double)z) * scale;
        return d < kFar ? d : (double)INFINITY;     // also a NaN, of -infinity at an infinite temperature
    }
    // A depth below kFar in steps of 2^-kSteps, and the weight as a part of the power of two above it: 2^-(steps % 128 / 128) 2^-r, |r| <= 2^-8, by a table and
    // four terms of the exponential series (the fifth is below 2e-15).
    __device__ __forceinline__ double part_of(double depth, const double *power, unsigned &steps) const
    {
        constexpr double kMagic = 0x1.8p45;     // its last place is 2^-kSteps
        const double y = depth + kMagic, r = (depth - (y - kMagic)) * -0.6931471805599453;
        steps = (unsigned)__double_as_longlong(y);
        const double series = __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(r, 1.0 / 24, 1.0 / 6), r, 0.5), r, 1.0), r, 1.0);
        return power[steps & 127u] * series;
    }
    __device__ __forceinline__ double weight_of(float z, const double *power) const
    {
        const double depth = depth_of(z);
        if (!(depth < kFar)) return 0.0;
        unsigned steps;
        const double part = part_of(depth, power, steps);
        return ldexp(part, -(int)(steps >> kSteps));
    }
    __device__ __forceinline__ unsigned bin_of(unsigned steps) const
    {
        const unsigned b = steps >> shift;
        return b < kBins - 1 ? b : kBins - 1;
    }
    __device__ __forceinline__ unsigned steps_of(double depth) const { return (unsigned)__double_as_longlong(depth + 0x1.8p45); }
    // The power of two that a bin's mass is held in.
    __device__ __forceinline__ double unit_of(unsigned bin) const { return ldexp(1.0, -32 - (int)(bin >> (kSteps - shift))); }
};

constexpr u64 kOneToken = 1ull << 48, kMassBits = kOneToken - 1;

__device__ __forceinline__ void fill_powers(Shared &sh)
{
    if (threadIdx.x < 1u << kSteps) sh.power[threadIdx.x] = exp2(-(double)threadIdx.x / (1u << kSteps));
}

// A token's count and mass for its bin.
__device__ __forceinline__ u64 packed(double part)
{
    return ((u64)__double_as_longlong(__builtin_fma(part, 0x1p32, 0x1p52)) & 0xFFFFFFFFFFFFFull) | kOneToken;     // part <= 1.003
}

// Bins of a source of at most kChunk logits into sh.bins; how many tokens min-p keeps.
template <class SOURCE>
__device__ __forceinline__ uint32_t fill_bins(SOURCE &source, const Weights &w, double reach, Shared &sh)
{
    sh.bins[threadIdx.x] = 0;
    fill_powers(sh);
    __syncthreads();
    uint32_t kept = 0;
    source.each([&](float z, unsigned) {
        const double depth = w.depth_of(z);
        if (!(depth < kFar)) return;
        unsigned steps;
        const double part = w.part_of(depth, sh.power, steps);
        atomicAdd(&sh.bins[w.bin_of(steps)], packed(part));
        kept += depth <= reach;
    });
    Mass total;
    sum_up_to(Mass{kept, 0.0}, sh, total);
    return uniform(total.count);
}

// Tokens of the flagged bins into sh.list, unsorted.
template <class SOURCE>
__device__ __forceinline__ void list_flagged(SOURCE &source, const Weights &w, Shared &sh)
{
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    source.each([&](float z, unsigned i) {
        const double depth = w.depth_of(z);
        if (!(depth < kFar)) return;
        const unsigned b = w.bin_of(w.steps_of(depth));
        if ((sh.flags[b / 32] >> (b % 32) & 1u) == 0) return;
        const unsigned at = atomicAdd(&sh.listed, 1u);
        if (at < kListed) sh.list[at] = place_of(key_of(z), i);
    });
    __syncthreads();
}

// ------------------------------------------------------------------------------------ questions
// The first token with which the count or the mass is reached.
struct Question {
    uint32_t count;
    double mass;
    bool above;     // more than the mass, not as much
    __device__ __forceinline__ bool reached(Mass m) const { return m.count >= count || (above ? m.mass > mass : m.mass >= mass); }
};

struct Bin {
    unsigned at;
    Mass before, with;
};

struct Questions {
    const Weights &w;
    const Settings &s;
    Shared &sh;
    Mass total;

    __device__ __forceinline__ Questions(const Weights &w, const Settings &s, Shared &sh, uint32_t count, u64 mass) : w(w), s(s), sh(sh)
    {
        const Mass own{count, (double)mass * w.unit_of(threadIdx.x)};
        sh.own[threadIdx.x] = own;
        sh.upto[threadIdx.x] = sum_up_to(own, sh, total);
        total = Mass{uniform(total.count), uniform(total.mass)};
    }

    // The first bin with tokens at whose end `q` is reached, or the last with tokens.
    __device__ __forceinline__ Bin find(const Question &q, Mass own, Mass upto, uint32_t last)
    {
        __syncthreads();
        if (threadIdx.x == 0) sh.found = kBins;
        __syncthreads();
        if (own.count != 0 && (upto.count == last || q.reached(upto))) atomicMin(&sh.found, threadIdx.x);
        __syncthreads();
        const unsigned at = sh.found;
        if (threadIdx.x == at) {
            sh.before = Mass{upto.count - own.count, upto.mass - own.mass};
            sh.at = upto;
        }
        __syncthreads();
        return Bin{uniform(at), {uniform(sh.before.count), uniform(sh.before.mass)}, {uniform(sh.at.count), uniform(sh.at.mass)}};
    }
    __device__ __forceinline__ Bin find(const Question &q) { return find(q, sh.own[threadIdx.x], sh.upto[threadIdx.x], total.count); }

    __device__ __forceinline__ bool flagged(unsigned bin) const { return (sh.flags[bin / 32] >> (bin % 32) & 1u) != 0; }

    // Flags bins lo .. hi, and says where each flagged bin starts in the list; how many tokens are flagged.
    __device__ __forceinline__ uint32_t flag(unsigned lo, unsigned hi, bool more)
    {
        const bool mine = (threadIdx.x >= lo && threadIdx.x <= hi) || (more && flagged(threadIdx.x));
        const u64 wave = __ballot(mine);
        __syncthreads();
        if (threadIdx.x % 32 == 0) sh.flags[threadIdx.x / 32] = (uint32_t)(wave >> (threadIdx.x % 64));
        Mass all;
        const uint32_t count = mine ? sh.own[threadIdx.x].count : 0u;
        const Mass end = sum_up_to(Mass{count, 0.0}, sh, all);
        sh.starts[threadIdx.x] = end.count - count;
        __syncthreads();
        return uniform(all.count);
    }

    // Flags the bins that, as far as the bins tell, hold the answers: all up to the last of them where these are few tokens.
    __device__ __forceinline__ void plan(uint32_t by_min)
    {
        uint32_t listed = flag(1, 0, false);
        Mass low = total, high = total;     // what is kept, at the least and at the most
        auto add = [&](const Bin &b) {
            if (b.with.count <= kListed) {
                flag(0, b.at, false);
                return true;
            }
            const uint32_t tokens = b.with.count - b.before.count;
            if (!flagged(b.at) && listed + tokens <= kListed) listed = flag(b.at, b.at, true);
            if (b.before.count < low.count) low = b.before;
            if (b.with.count < high.count) high = b.with;
            return false;
        };
        if (s.top_k < total.count && add(find(Question{s.top_k, (double)INFINITY, false}))) return;
        if (s.top_p < 1.0) {
            const double most = s.top_p * high.mass, least = s.top_p * low.mass;
            if (add(find(Question{high.count, most, false}))) return;
            if (least < most && add(find(Question{high.count, least, false}))) return;
        }
        if (by_min < high.count && add(find(Question{by_min, (double)INFINITY, false}))) return;
        const Bin first = find(Question{high.count, s.u * low.mass, true}), last = find(Question{high.count, s.u * high.mass, true});
        if (last.with.count <= kListed) {
            flag(0, last.at, false);
            return;
        }
        if (listed + last.with.count - first.before.count <= kListed) flag(first.at, last.at, true);
    }

    // Of n listed tokens from `start` on, before which `before` ranks: the first with which `q` is reached (the last if it never is), and what is
    // kept with it.
    __device__ __forceinline__ unsigned find_listed(const Question &q, unsigned start, unsigned n, Mass before, Mass &kept)
    {
        const unsigned i = threadIdx.x * 2;
        auto weight = [&](unsigned at) { return at < n ? w.weight_of(value_of_key(~(uint32_t)(sh.list[start + at] >> 32)), sh.power) : 0.0; };
        const double w0 = weight(i), w1 = weight(i + 1);
        Mass all;
        const Mass m1 = before + sum_up_to(Mass{(i < n ? 1u : 0u) + (i + 1 < n ? 1u : 0u), w0 + w1}, sh, all);
        const Mass m0{m1.count - (i + 1 < n ? 1u : 0u), m1.mass - w1};
        __syncthreads();
        if (threadIdx.x == 0) sh.found = n - 1;
        __syncthreads();
        if (i < n && q.reached(m0)) atomicMin(&sh.found, i);
        else if (i + 1 < n && q.reached(m1)) atomicMin(&sh.found, i + 1);
        __syncthreads();
        const unsigned at = sh.found;
        if (i == at) sh.at = m0;
        else if (i + 1 == at) sh.at = m1;
        __syncthreads();
        kept = Mass{uniform(sh.at.count), uniform(sh.at.mass)};
        return start + at;
    }

    // Lists the tokens of a bin of more than kListed that are near the answer: bins of places inside it, until they are few.
    template <class SOURCE>
    __device__ __forceinline__ unsigned narrow(const SOURCE &source, const Question &q, unsigned bin, Mass &before)
    {
        auto each = [&](auto f) {
            source.each([&](float z, unsigned i) {
                const double depth = w.depth_of(z);
                if (depth < kFar && w.bin_of(w.steps_of(depth)) == bin) f(z, depth, place_of(key_of(z), i));
            });
        };
        __syncthreads();
        if (threadIdx.x == 0) {
            sh.low_place = ~0ull;
            sh.high_place = 0;
        }
        __syncthreads();
        each([&](float, double, u64 p) {
            atomicMin(&sh.low_place, p);
            atomicMax(&sh.high_place, p);
        });
        __syncthreads();
        u64 first = sh.low_place, last = sh.high_place;
        for (;;) {
            // counts and masses apart: a bin may hold more tokens than a chunk
            const u64 step = (last - first) / kBins + 1;
            __syncthreads();
            sh.bins[threadIdx.x] = 0;
            sh.starts[threadIdx.x] = 0;
            __syncthreads();
            each([&](float, double depth, u64 p) {
                if (p < first || p > last) return;
                unsigned steps;
                const unsigned b = (unsigned)((p - first) / step);
                atomicAdd(&sh.bins[b], packed(w.part_of(depth, sh.power, steps)) & kMassBits);
                atomicAdd(&sh.starts[b], 1u);
            });
            __syncthreads();
            const Mass mine{sh.starts[threadIdx.x], (double)sh.bins[threadIdx.x] * w.unit_of(bin)};
            Mass all;
            const Mass end = before + sum_up_to(mine, sh, all);
            const Bin b = find(q, mine, end, before.count + all.count);
            before = b.before;
            first += b.at * step;
            if (last - first >= step) last = first + step - 1;
            if (b.with.count - b.before.count <= kListed) break;    // a step of 1 holds one token
        }
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        each([&](float, double, u64 p) {
            if (p < first || p > last) return;
            const unsigned at = atomicAdd(&sh.listed, 1u);
            if (at < kListed) sh.list[at] = p;
        });
        __syncthreads();
        sort_list(sh, sh.listed);
        return sh.listed;
    }

    // The answer: its index in the list, and what is kept with it.
    template <class SOURCE>
    __device__ __forceinline__ unsigned ask(const SOURCE &source, const Question &q, Mass &kept)
    {
        const Bin b = find(q);
        Mass before = b.before;
        unsigned start = 0, n = b.with.count - b.before.count;
        if (flagged(b.at)) {
            start = sh.starts[b.at];
        } else if (n <= kListed) {
            flag(b.at, b.at, false);
            list_flagged(source, w, sh);
            sort_list(sh, n);
        } else {
            n = narrow(source, q, b.at, before);
            flag(1, 0, false);
        }
        return find_listed(q, start, n, before, kept);
    }

    // The token, where the tokens of the flagged bins are listed and sorted.
    template <class SOURCE>
    __device__ __forceinline__ long long choose(const SOURCE &source, uint32_t by_min)
    {
        Mass kept = total;
        unsigned at = 0;
#pragma unroll 1
        for (unsigned turn = 0; turn < 4; ++turn) {     // top-k, top-p, min-p, the choice
            Question q{kept.count, (double)INFINITY, turn == 3};
            bool needed = true;
            if (turn == 0) {
                needed = s.top_k < kept.count;
                q.count = s.top_k;
            } else if (turn == 1) {
                needed = s.top_p < 1.0;
                q.mass = s.top_p * kept.mass;
            } else if (turn == 2) {
                needed = by_min < kept.count;
                q.count = by_min;
            } else {
                q.mass = s.u * kept.mass;
            }
            if (needed) at = ask(source, q, kept);
        }
        return (long long)(uint32_t)sh.list[at];
    }
};

// A row's token where it takes no weights: none in a row with a NaN or without tokens, or the first by rank.
__device__ __forceinline__ bool is_simple(u64 best, const Settings &s, long long &token)
{
    const uint32_t key = ~(uint32_t)(best >> 32);
    token = key == kNan || key <= kNothing ? -1 : (long long)(uint32_t)best;
    return token < 0 || s.greedy;
}

// ------------------------------------------------------------------------------------ kernels
// A row to a block.
template <class ELEM, bool CAP, bool WIDE, unsigned E>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Settings s = settings_of(a, blockIdx.x);
    Held<ELEM, CAP, WIDE, E> held(static_cast<const ELEM *>(a.logits) + blockIdx.x * a.row, 0, a.vocabulary, a.cap, tab);
    u64 best;
    uint32_t low;
    ends_of(held, sh, best, low);
    long long token;
    if (!is_simple(best, s, token)) {
        const Weights w(~(uint32_t)(best >> 32), low, s.scale);
        const uint32_t by_min = fill_bins(held, w, s.reach, sh);
        const u64 mine = sh.bins[threadIdx.x];
        Questions questions(w, s, sh, (uint32_t)(mine >> 48), mine & kMassBits);
        questions.plan(by_min);
        list_flagged(held, w, sh);
        sort_list(sh, sh.listed);
        // another list than the plan's, if one is needed, comes from memory: the registers are the questions'
        const Read<ELEM, CAP, WIDE> read{static_cast<const ELEM *>(a.logits) + blockIdx.x * a.row, a.vocabulary, a.cap, tab};
        token = questions.choose(read, by_min);
    }
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = token;
}

// Rows in chunks.  Blocks have a chunk each but for the last launch.
struct Where {
    unsigned row, first, end;
};
__device__ __forceinline__ Where chunk_of(const SampleArgs &a)
{
    const unsigned row = blockIdx.x / a.chunks, first = blockIdx.x % a.chunks * kChunk;
    return Where{row, first, a.vocabulary - first < kChunk ? a.vocabulary : first + kChunk};
}

// The row's ends from those of its chunks.
__device__ __forceinline__ void row_ends(const SampleArgs &a, unsigned row, u64 &best, uint32_t &low)
{
    best = ~0ull;
    low = kNan;
    for (unsigned c = 0; c < a.chunks; ++c) {
        const u64 p = a.best[row * (u64)a.chunks + c];
        const uint32_t k = a.low[row * (u64)a.chunks + c];
        best = p < best ? p : best;
        low = k < low ? k : low;
    }
}

// This lane's bin of the row.
__device__ __forceinline__ Questions row_questions(const SampleArgs &a, unsigned row, const Weights &w, const Settings &s, Shared &sh, uint32_t &by_min)
{
    uint32_t count = 0;
    u64 mass = 0;
    by_min = 0;
    for (unsigned c = 0; c < a.chunks; ++c) {
        const u64 at = row * (u64)a.chunks + c, v = a.bins[at * kBins + threadIdx.x];
        count += (uint32_t)(v >> 48);
        mass += v & kMassBits;
        by_min += a.by_min[at];
    }
    return Questions(w, s, sh, count, mass);
}

template <class ELEM, bool CAP, bool WIDE>
__global__ __launch_bounds__(kThreads) void sample_ends_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of(a);
    Held<ELEM, CAP, WIDE, 32> held(static_cast<const ELEM *>(a.logits) + at.row * a.row, at.first, at.end, a.cap, tab);
    u64 best;
    uint32_t low;
    ends_of(held, sh, best, low);
    if (threadIdx.x == 0) {
        a.best[blockIdx.x] = best;
        a.low[blockIdx.x] = low;
        if (at.first == 0) a.listed[at.row] = 0;
    }
}

template <class ELEM, bool CAP, bool WIDE>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of(a);
    const Settings s = settings_of(a, at.row);
    u64 best;
    uint32_t low;
    row_ends(a, at.row, best, low);
    long long token;
    if (is_simple(best, s, token)) return;
    Held<ELEM, CAP, WIDE, 32> held(static_cast<const ELEM *>(a.logits) + at.row * a.row, at.first, at.end, a.cap, tab);
    const uint32_t by_min = fill_bins(held, Weights(~(uint32_t)(best >> 32), low, s.scale), s.reach, sh);
    a.bins[blockIdx.x * (u64)kBins + threadIdx.x] = sh.bins[threadIdx.x];
    if (threadIdx.x == 0) a.by_min[blockIdx.x] = by_min;
}

template <class ELEM, bool CAP, bool WIDE>
__global__ __launch_bounds__(kThreads) void sample_list_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of(a);
    const Settings s = settings_of(a, at.row);
    u64 best;
    uint32_t low;
    row_ends(a, at.row, best, low);
    long long token;
    if (is_simple(best, s, token)) return;
    const Weights w(~(uint32_t)(best >> 32), low, s.scale);
    uint32_t by_min;
    Questions questions = row_questions(a, at.row, w, s, sh, by_min);
    questions.plan(by_min);
    Held<ELEM, CAP, WIDE, 32> held(static_cast<const ELEM *>(a.logits) + at.row * a.row, at.first, at.end, a.cap, tab);
    list_flagged(held, w, sh);
    const unsigned n = sh.listed;       // at most kListed: the plan's
    if (threadIdx.x == 0) sh.found = atomicAdd(&a.listed[at.row], n);
    __syncthreads();
    const unsigned start = sh.found;
    for (unsigned i = threadIdx.x; i < n; i += kThreads)
        if (start + i < kListed) a.list[at.row * (u64)kListed + start + i] = sh.list[i];
}

template <class ELEM, bool CAP, bool WIDE>
__global__ __launch_bounds__(kThreads) void sample_answer_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const unsigned row = blockIdx.x;
    const Settings s = settings_of(a, row);
    u64 best;
    uint32_t low;
    row_ends(a, row, best, low);
    long long token;
    if (!is_simple(best, s, token)) {
        const Weights w(~(uint32_t)(best >> 32), low, s.scale);
        fill_powers(sh);
        uint32_t by_min;
        Questions questions = row_questions(a, row, w, s, sh, by_min);
        questions.plan(by_min);
        const unsigned n = a.listed[row];
        for (unsigned i = threadIdx.x; i < n && i < kListed; i += kThreads) sh.list[i] = a.list[row * (u64)kListed + i];
        sort_list(sh, n < kListed ? n : kListed);
        const Read<ELEM, CAP, WIDE> read{static_cast<const ELEM *>(a.logits) + row * a.row, a.vocabulary, a.cap, tab};
        token = questions.choose(read, by_min);
    }
    if (threadIdx.x == 0) a.tokens[row] = token;
}

// ------------------------------------------------------------------------------------ host side
bool in_range(double v, double most) { return v >= 0.0 && v <= most; }

ktanh_status_t check_shape(const ksample_shape_t *s)
{
    if (s == nullptr) return KT_ERR_NULL;
    if (s->rows > (size_t)1 << 24 || s->vocabulary == 0 || s->vocabulary > KSAMPLE_MOST || s->row > (size_t)1 << 40 ||
        !in_range(s->temperature, 3e38) || !in_range(s->top_p, 1.0) || !in_range(s->min_p, 1.0) || !in_range(s->cap, 3e38) ||
        (s->cap > 0.0 && s->cap < 1e-30))
        return KT_ERR_SHAPE;
    return KT_OK;
}

size_t chunks_of(size_t vocabulary) { return (vocabulary + kChunk - 1) / kChunk; }

template <class Lut>
ktanh_status_t sample_entry(const ksample_shape_t *s, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                            const float *top_p, const float *min_p, int64_t *tokens, void *workspace, const Lut *lut, ktanh_stream_t stream)
{
    constexpr bool WIDE = is_wide(static_cast<const Lut *>(nullptr));
    ktanh_status_t st = check_shape(s);
    if (st != KT_OK) return st;
    if (s->rows == 0) return KT_OK;
    if (logits == nullptr || uniform == nullptr || tokens == nullptr) return KT_ERR_NULL;
    auto off = [](const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
    if (off(logits, s->f32 ? 4 : 2) || off(uniform, 4) || off(temperature, 4) || off(top_k, 4) || off(top_p, 4) || off(min_p, 4) || off(tokens, 8) ||
        off(workspace, 16))
        return KT_ERR_ALIGN;
    KtLutPack pack;
    st = pack_for(lut, true, &pack);
    if (st != KT_OK) return st;
    SampleArgs a;
    a.logits = logits;
    a.row = s->rows > 1 ? s->row : 0;
    a.vocabulary = (unsigned)s->vocabulary;
    a.chunks = (unsigned)chunks_of(s->vocabulary);
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
    a.best = a.bins = a.list = nullptr;
    a.low = a.by_min = a.listed = nullptr;
    const size_t rows = s->rows, blocks = rows * a.chunks;
    if (a.chunks > 1) {
        if (workspace == nullptr) return KT_ERR_NULL;
        a.bins = static_cast<u64 *>(workspace);
        a.list = a.bins + blocks * kBins;
        a.best = a.list + rows * kListed;
        a.low = reinterpret_cast<uint32_t *>(a.best + blocks);
        a.by_min = a.low + blocks;
        a.listed = a.by_min + blocks;
    }
    if (blocks * kThreads >= (size_t)1 << 32) return KT_ERR_SHAPE;
    auto launch = [&](auto kernel, size_t n) { return launch_checked(kernel, (unsigned)n, kThreads, stream, a, pack); };
    auto of = [&](auto elem, auto capped) {
        typedef decltype(elem) ELEM;
        constexpr bool CAP = decltype(capped)::value, W = CAP && WIDE;
        if (s->vocabulary <= 8 * kThreads) return launch(sample_kernel<ELEM, CAP, W, 8>, rows);
        if (a.chunks == 1) return launch(sample_kernel<ELEM, CAP, W, 32>, rows);
        ktanh_status_t done = launch(sample_ends_kernel<ELEM, CAP, W>, blocks);
        if (done == KT_OK) done = launch(sample_bins_kernel<ELEM, CAP, W>, blocks);
        if (done == KT_OK) done = launch(sample_list_kernel<ELEM, CAP, W>, blocks);
        return done == KT_OK ? launch(sample_answer_kernel<ELEM, CAP, W>, rows) : done;
    };
    if (s->f32) return s->cap > 0.0 ? of(uint32_t(), std::true_type()) : of(uint32_t(), std::false_type());
    return s->cap > 0.0 ? of(uint16_t(), std::true_type()) : of(uint16_t(), std::false_type());
}

}  // namespace

extern "C" size_t ksample_workspace(const ksample_shape_t *shape)
{
    if (check_shape(shape) != KT_OK) return 0;
    const size_t chunks = chunks_of(shape->vocabulary), blocks = shape->rows * chunks;
    return chunks == 1 ? 0 : blocks * (kBins * sizeof(u64) + sizeof(u64) + 2 * sizeof(uint32_t)) + shape->rows * (kListed * sizeof(u64) + sizeof(uint32_t));
}
extern "C" ktanh_status_t ksample(const ksample_shape_t *shape, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                                  const float *top_p, const float *min_p, int64_t *tokens, void *workspace, const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return sample_entry(shape, logits, uniform, temperature, top_k, top_p, min_p, tokens, workspace, lut, stream);
}
extern "C" ktanh_status_t ksample64(const ksample_shape_t *shape, const void *logits, const float *uniform, const float *temperature, const int32_t *top_k,
                                    const float *top_p, const float *min_p, int64_t *tokens, void *workspace, const ktanh_lut64_t *lut,
                                    ktanh_stream_t stream)
{
    return sample_entry(shape, logits, uniform, temperature, top_k, top_p, min_p, tokens, workspace, lut, stream);
}
