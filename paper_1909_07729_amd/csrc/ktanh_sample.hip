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
// A block holds up to 32768 logits in registers.  Rows of no more take one launch, and are read once.  Longer ones are cut into chunks and take
// three: the chunks' largest logits, their bins, and their tokens of the bins that hold answers, among which the row's last block chooses.
// Sums over the bins and over the listed tokens are formed once, with barriers; questions are then searches that every wavefront makes for
// itself, with none.  Where top-k leaves few tokens they are all listed, and nothing else is needed.
//
// What bounds it: in a row of its own the steps' latencies, one behind the other (one row of 32000: top-k 50 and top-p 0.95 in 10.9 us, top-p alone in 21.6, greedy in
// 6.5); in many the vector instructions, 20 a logit for its cap alone (64 rows of 131072: 41 us uncapped, 57 capped: ends 13.6, bins 18.2, answers 28.4).  The
// logits themselves, 17 or 34 MB, are 3 to 5 us of each pass.
#include "ktanh_codes.h"
#include "ktanh_stream_impl.h"

#include <cmath>
#include <type_traits>

using namespace ktanh_device;

namespace {

constexpr unsigned kThreads = 1024, kBins = kThreads;   // a bin for each lane of a block
constexpr unsigned kListed = 2048;                      // tokens that a block sorts
constexpr unsigned kRanked = 512;                       // of these, how many by counting
constexpr unsigned kMost = 32, kFew = 8;                // logits of a lane
constexpr unsigned kSteps = 7;                          // log2 of the finest bins to a factor of two
constexpr double kFar = 73.5;                           // KSAMPLE_MOST 2^-kFar < 2^-53: what lies beyond does not reach a sum of doubles
constexpr double kLog2e = 1.4426950408889634;
constexpr float kHottest = 3e38f;                       // the highest temperature

typedef unsigned long long u64;

// Float32 values in their order as integers, with one zero.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);
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
    u64 *bins, *list;
    float4 *ends;       // the largest logit, the smallest, the largest magnitude (the bits of a NaN if there is one), the index of the largest
    uint32_t *by_min, *listed, *arrived;
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
    float t = a.temperature != nullptr ? a.temperature[row] : a.one_temperature;
    t = t > kHottest ? kHottest : t;
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
// What is behind the row is like masked tokens, which the cap leaves masked.  The table reads need all lanes.
template <bool CAP, bool WIDE>
__device__ __forceinline__ float logit_of(float z, bool inside, float cap, const LaneTable &tab)
{
    if constexpr (CAP) {
        const float t = __uint_as_float(ktanh_f32_one<WIDE>(__float_as_uint(z / cap), tab));
        z = z == -INFINITY ? z : cap * t;
    }
    return inside ? z : -INFINITY;
}

// Which logits can be among the first: (top - z) * by < limit, in Float32 operations, which keep the order of logits.  by == 0: all.
struct Near {
    float top, by, limit;
    __device__ __forceinline__ bool all() const { return by == 0.f; }
    __device__ __forceinline__ bool operator()(float z) const { return (top - z) * by < limit; }
};
constexpr Near kAll{0.f, 0.f, 1.f};

// Logits of `first` .. `end` - 1 for a block, E to a lane, asked for.
template <class ELEM, unsigned E>
struct OnTheWay {
    static constexpr unsigned N = kPerLane<ELEM>;
    uint4 v[E / N];
    unsigned first, end;

    OnTheWay() = default;
    __device__ __forceinline__ OnTheWay(const ELEM *from, unsigned first, unsigned end) : first(first), end(end)
    {
#pragma unroll
        for (unsigned i = 0; i < E / N; ++i) v[i] = load_logits(from, first + (i * kThreads + threadIdx.x) * N, end);
    }
};

// The same in a block's registers.
template <class ELEM, bool CAP, bool WIDE, unsigned E>
struct Held {
    static constexpr unsigned N = kPerLane<ELEM>;
    float z[E / N][N];
    unsigned first;

    __device__ __forceinline__ Held(const OnTheWay<ELEM, E> &raw, float cap, const LaneTable &tab) : first(raw.first)
    {
#pragma unroll
        for (unsigned v = 0; v < E / N; ++v) {
            widen<ELEM>(raw.v[v], z[v]);
#pragma unroll
            for (unsigned i = 0; i < N; ++i) z[v][i] = logit_of<CAP, WIDE>(z[v][i], place(v) + i < raw.end, cap, tab);
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
            unsigned at = place(v);
            asm volatile("" : "+v"(at));
#pragma unroll
            for (unsigned i = 0; i < N; ++i) asm volatile("" : "+v"(z[v][i]));
#pragma unroll
            for (unsigned i = 0; i < N; ++i) {
                f(z[v][i], at + i);
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
};

// The same from memory, each time: for the few rows whose answers are not where the sums of bins say.
template <class ELEM, bool CAP, bool WIDE>
struct Read {
    const ELEM *from;
    unsigned end;
    float cap;
    const LaneTable &tab;

    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 1
        for (unsigned base = 0; base < end; base += kThreads) {
            const unsigned at = base + threadIdx.x;
            uint32_t u = at < end ? (uint32_t)from[at] : 0u;
            if constexpr (sizeof(ELEM) == 2) u <<= 16;
            const float z = logit_of<CAP, WIDE>(__uint_as_float(u), at < end, cap, tab);
            f(z, at);
        }
    }
};

// ------------------------------------------------------------------------------------ a block's memory and sums
struct Mass {
    uint32_t count;
    double mass;
};
__device__ __forceinline__ Mass operator+(Mass a, Mass b) { return Mass{a.count + b.count, a.mass + b.mass}; }
__device__ __forceinline__ Mass uniform(Mass m) { return Mass{uniform(m.count), uniform(m.mass)}; }

constexpr unsigned kWaves = kThreads / 64;

struct Shared {
    Mass part[kWaves];
    float top[kWaves], low[kWaves];
    uint32_t widest[kWaves], first[kWaves];
    unsigned from[4], to[4];        // bins that the plan lists
    double power[1u << kSteps];     // 2^(32 - j / 128)
    u64 bins[kBins];                // count << 48 | mass
    uint32_t count[kBins];          // of all bins up to each
    double mass[kBins];
    uint32_t flags[kBins / 32];     // bins whose tokens are listed
    uint32_t starts[kBins];         // of the flagged bins in the list
    u64 list[kListed];
    double list_mass[kListed];      // of all listed tokens up to each
    uint32_t ranks[kRanked];
    uint32_t listed, by_min;
    u64 low_place, high_place;
    // a question that is not answered by the list
    uint32_t asked;
    unsigned asked_bin;
    uint32_t asked_count, asked_above;
    double asked_mass;
    Mass asked_before, asked_with;
};

// Moves between the lanes of a wavefront; lanes that none moves to get 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true); }
template <int CTRL, int ROWS>
__device__ __forceinline__ Mass moved(Mass m)
{
    const u64 v = (u64)__double_as_longlong(m.mass);
    const u64 to = (u64)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v);
    return Mass{moved<CTRL, ROWS>(m.count), __longlong_as_double((long long)to)};
}
// Sums of a wavefront's lanes up to and with each: within rows of 16 lanes, then from row to row.
__device__ __forceinline__ Mass scanned(Mass v)
{
    v = v + moved<0x111, 0xF>(v);   // row_shr
    v = v + moved<0x112, 0xF>(v);
    v = v + moved<0x114, 0xF>(v);
    v = v + moved<0x118, 0xF>(v);
    v = v + moved<0x142, 0xA>(v);   // row_bcast:15
    return v + moved<0x143, 0xC>(v);
}

// Sum of the block's lanes up to and with this one.
__device__ __forceinline__ Mass sum_up_to(Mass v, Shared &sh)
{
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const Mass run = scanned(v);
    __syncthreads();        // the last use of part
    if (lane == 63) sh.part[wave] = run;
    __syncthreads();
    const Mass parts = scanned(lane < kWaves ? sh.part[lane] : Mass{0, 0.0});
    const Mass before{(uint32_t)__shfl((int)parts.count, (int)wave - 1), __shfl(parts.mass, (int)wave - 1)};
    return wave != 0 ? before + run : run;
}

// The first of n (at most 64 * 64) for which `holds`, n if for none: a search by a wavefront whose lanes look at 64 places at once.  `holds` stays true once
// it is.
template <class F>
__device__ __forceinline__ unsigned first_where(unsigned n, F holds)
{
    const unsigned lane = threadIdx.x % 64, step = (n + 63) / 64;
    auto at = [&](unsigned i) { return i < n && holds(i); };
    const unsigned end = (lane + 1) * step - 1;
    const u64 ends = __ballot(end < n ? holds(end) : lane * step < n && holds(n - 1));
    if (ends == 0) return n;
    const unsigned first = (unsigned)__builtin_ctzll(ends) * step;
    if (n <= 64) return first;
    const u64 inside = __ballot(lane < step && at(first + lane));
    return inside == 0 ? n - 1 : first + (unsigned)__builtin_ctzll(inside);
}

// Sorts sh.list[0 .. n), n <= kListed; what is behind it up to a power of two is overwritten.  Few by counting for each how many are below it, shared
// out among all lanes (64 tokens: 4 comparisons a lane); many by a bitonic network.
__device__ __forceinline__ void sort_list(Shared &sh, unsigned n)
{
    __syncthreads();
    if (n <= kRanked) {
        unsigned lg = 6;
        while ((1u << lg) < n) ++lg;
        const unsigned i = threadIdx.x & ((1u << lg) - 1), slice = threadIdx.x >> lg, slices = kThreads >> lg;
        if (threadIdx.x < kRanked) sh.ranks[threadIdx.x] = 0;
        const u64 mine = i < n ? sh.list[i] : 0;
        __syncthreads();
        uint32_t below = 0;
        for (unsigned j = slice; j < n; j += slices) below += sh.list[j] < mine;
        if (i < n && below != 0) atomicAdd(&sh.ranks[i], below);
        __syncthreads();
        if (threadIdx.x < n) sh.list[sh.ranks[i]] = mine;
        __syncthreads();
        return;
    }
    unsigned lg = 10;
    while ((1u << lg) < n) ++lg;
    const unsigned size = 1u << lg;
    for (unsigned i = n + threadIdx.x; i < size; i += kThreads) sh.list[i] = ~0ull;
    for (unsigned lk = 1; lk <= lg; ++lk)
        for (unsigned lj = lk; lj-- > 0;) {
            // up to a distance of 64 a wavefront stays within its own 128 places
            if (lk == 1 || lj > 6 || (lj == 6 && lk > 7)) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const unsigned a = (threadIdx.x >> lj) << (lj + 1) | (threadIdx.x & ((1u << lj) - 1)), b = a | 1u << lj;
            if (b < size) {
                const u64 x = sh.list[a], y = sh.list[b];
                if ((x > y) == ((a >> lk & 1u) == 0)) {
                    sh.list[a] = y;
                    sh.list[b] = x;
                }
            }
        }
    __syncthreads();
}

// What a source's logits tell before any weight: the largest, the smallest that is not masked (infinity if all are), and whether there is a NaN.
struct Ends {
    float top, low;
    uint32_t widest;    // magnitude, as bits
    __device__ __forceinline__ void meet(float t, float l, uint32_t m)
    {
        top = __builtin_fmaxf(top, t);
        low = __builtin_fminf(low, l);
        widest = m > widest ? m : widest;
    }
    __device__ __forceinline__ bool strange() const { return widest > 0x7F800000u; }
    // A row without a token to choose from.
    __device__ __forceinline__ bool empty() const { return strange() || top == -INFINITY; }
};
constexpr Ends kNoEnds{-INFINITY, INFINITY, 0};

template <int CTRL, int ROWS>
__device__ __forceinline__ void meet_moved(Ends &e)     // lanes that none moves to meet themselves
{
    auto bits = [](uint32_t u) { return (uint32_t)__builtin_amdgcn_update_dpp((int)u, (int)u, CTRL, ROWS, 0xF, false); };
    auto other = [&](float v) { return __uint_as_float(bits(__float_as_uint(v))); };
    e.meet(other(e.top), other(e.low), bits(e.widest));
}
// Of all lanes of a wavefront, in all of them.
__device__ __forceinline__ Ends met(Ends e)
{
    meet_moved<0x111, 0xF>(e);
    meet_moved<0x112, 0xF>(e);
    meet_moved<0x114, 0xF>(e);
    meet_moved<0x118, 0xF>(e);
    meet_moved<0x142, 0xA>(e);
    meet_moved<0x143, 0xC>(e);
    auto last = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); };
    return Ends{__uint_as_float(last(__float_as_uint(e.top))), __uint_as_float(last(__float_as_uint(e.low))), last(e.widest)};
}

template <class SOURCE>
__device__ __forceinline__ Ends ends_of(SOURCE &source, float &lane_top, Shared &sh)
{
    Ends e = kNoEnds;
    source.each([&](float z, unsigned) { e.meet(z, z == -INFINITY ? INFINITY : z, __float_as_uint(z) & 0x7FFFFFFFu); });
    lane_top = e.top;
    e = met(e);
    if (threadIdx.x % 64 == 0) {
        sh.top[threadIdx.x / 64] = e.top;
        sh.low[threadIdx.x / 64] = e.low;
        sh.widest[threadIdx.x / 64] = e.widest;
    }
    __syncthreads();
    const unsigned part = threadIdx.x % kWaves;
    return met(Ends{sh.top[part], sh.low[part], sh.widest[part]});
}

// The lowest index of a logit equal to `top`, or what is above all indices.
template <class SOURCE>
__device__ __forceinline__ uint32_t first_of(SOURCE &source, float top, Shared &sh)
{
    uint32_t first = ~0u;
    source.each([&](float z, unsigned i) {
        if (z == top && i < first) first = i;
    });
    for (int step = 1; step < 64; step *= 2) {
        const uint32_t other = (uint32_t)__shfl_xor((int)first, step);
        first = other < first ? other : first;
    }
    if (threadIdx.x % 64 == 0) sh.first[threadIdx.x / 64] = first;
    __syncthreads();
    first = sh.first[0];
    for (unsigned i = 1; i < kWaves; ++i) first = sh.first[i] < first ? sh.first[i] : first;
    return first;
}

// ------------------------------------------------------------------------------------ weights and bins
// Depth: how far a logit is below the largest, as the power of two that its weight is below 1.
struct Weights {
    float top;
    bool infinite;      // the largest logit is: only its like have a weight
    double scale;
    unsigned shift;     // kSteps less the log2 of the bins to a factor of two
    // In scalar registers: as literals they would be moved to vector ones for every logit.
    double magic = 0x1.8p45;        // its last place is 2^-kSteps
    double series[4] = {-0.69314718055994530942, 0.24022650695910071233, -0.05550410866482157995, 0.00961812910762847716};

    __device__ __forceinline__ Weights(const Ends &e, double scale) : top(e.top), infinite(e.top == INFINITY), scale(scale)
    {
        const double down = ((double)e.top - (double)e.low) * scale, range = down < kFar ? down : kFar;
        unsigned by = 0;    // kBins = 8 << kSteps
        while (by < 4 && range > (double)(7u << by)) ++by;
        shift = uniform(by);
        asm volatile("" : "+s"(magic), "+s"(series[0]), "+s"(series[1]), "+s"(series[2]), "+s"(series[3]));
    }
    // Not below kFar, or a NaN: no weight.
    __device__ __forceinline__ double depth_of(float z) const
    {
        if (infinite) return z == top ? 0.0 : (double)INFINITY;
        return ((double)top - (double)z) * scale;
    }
    // A depth below kFar in steps of 2^-kSteps, and the weight in 2^-32 of the power of two above it, as the product of 2^(32 - steps % 128 / 128) from a table and
    // 2^-r, |r| <= 2^-8, by four terms of its series (the fifth is below 2e-15).
    __device__ __forceinline__ double part_of(double depth, unsigned &steps) const
    {
        const double y = depth + magic, r = depth - (y - magic);
        steps = (unsigned)__double_as_longlong(y);
        return __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(r, series[3], series[2]), r, series[1]), r, series[0]), r, 1.0);
    }
    __device__ __forceinline__ double weight_of(float z, const double *power) const
    {
        const double depth = depth_of(z);
        if (!(depth < kFar)) return 0.0;
        unsigned steps;
        const double part = part_of(depth, steps);
        return ldexp(power[steps & 127u] * part, -32 - (int)(steps >> kSteps));
    }
    __device__ __forceinline__ unsigned bin_of(unsigned steps) const
    {
        const unsigned b = steps >> shift;
        return b < kBins - 1 ? b : kBins - 1;
    }
    __device__ __forceinline__ unsigned steps_of(double depth) const { return (unsigned)__double_as_longlong(depth + magic); }
    // The power of two that a bin's mass is held in.
    __device__ __forceinline__ double unit_of(unsigned bin) const { return ldexp(1.0, -32 - (int)(bin >> (kSteps - shift))); }
};

constexpr u64 kOneToken = 1ull << 48, kMassBits = kOneToken - 1;

// 2^(32 - j / 128), by the bits of j: 2^(-1/128), 2^(-1/64) and so on.
__device__ __forceinline__ void fill_powers(Shared &sh)
{
    constexpr double kPowers[kSteps] = {0.99459942348363317565, 0.98922801319397548413, 0.97857206208770013453, 0.95760328069857364694,
                                        0.91700404320467123174, 0.84089641525371454303, 0.70710678118654752440};
    if (threadIdx.x >= 1u << kSteps) return;
    double v = 0x1p32;
#pragma unroll
    for (unsigned i = 0; i < kSteps; ++i) v *= threadIdx.x >> i & 1u ? kPowers[i] : 1.0;
    sh.power[threadIdx.x] = v;
}

// A token's count and mass for its bin.
__device__ __forceinline__ u64 packed(double power, double part)
{
    return ((u64)__double_as_longlong(__builtin_fma(power, part, 0x1p52)) & 0xFFFFFFFFFFFFFull) | kOneToken;      // at most 1.003 2^32
}

// The largest logits of lanes as a source: the k-th largest of them is no larger than the k-th largest of all.
struct Tops {
    float z;
    template <class F>
    __device__ __forceinline__ void each(F f) const { f(z, 0u); }
};

// Which tokens may be among the first k, and how many these are: by counts alone, which cost less than weights where they are few (one row of 32000: 50
// in 12.8 us, 20.3 by weights; 1000 in 28.1, by weights 24.3).
template <class SOURCE>
__device__ __forceinline__ Near nearest(SOURCE &source, const Ends &e, uint32_t k, uint32_t &tokens, Shared &sh)
{
    tokens = ~0u;
    const float width = e.top - e.low;
    if (!(width > 0x1p-110f && width < 3e38f)) return kAll;     // all alike, too near each other for a quotient in Float32, or an infinity
    const float by = (float)(kBins - 1) / width;
    sh.count[threadIdx.x] = 0;
    __syncthreads();
    source.each([&](float z, unsigned) {
        const float d = (e.top - z) * by;
        if (d < (float)kBins) atomicAdd(&sh.count[(unsigned)d], 1u);
    });
    __syncthreads();
    const uint32_t upto = sum_up_to(Mass{sh.count[threadIdx.x], 0.0}, sh).count;
    __syncthreads();
    sh.count[threadIdx.x] = upto;
    __syncthreads();
    const unsigned last = first_where(kBins, [&](unsigned i) { return sh.count[i] >= k; });
    tokens = uniform(sh.count[last < kBins ? last : kBins - 1]);
    return uniform(Near{e.top, by, (float)(last + 1)});      // bins 0 .. last; all if the tokens are fewer than k
}

// Bins of a source of at most 32768 logits into sh.bins, and how many tokens min-p keeps into sh.by_min.
template <class SOURCE>
__device__ __forceinline__ void fill_bins(SOURCE &source, const Weights &w, double reach, Shared &sh)
{
    sh.bins[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.by_min = 0;
    fill_powers(sh);
    __syncthreads();
    uint32_t kept = 0;
    source.each([&](float z, unsigned) {
        const double depth = w.depth_of(z);
        if (!(depth < kFar)) return;
        unsigned steps;
        const double part = w.part_of(depth, steps);
        atomicAdd(&sh.bins[w.bin_of(steps)], packed(sh.power[steps & 127u], part));
        kept += depth <= reach;
    });
    const Mass all = scanned(Mass{kept, 0.0});
    if (threadIdx.x % 64 == 63) atomicAdd(&sh.by_min, all.count);
    __syncthreads();
}

// Tokens of the flagged bins, all of whose logits are between `low` and `high`, into sh.list, unsorted.
template <class SOURCE>
__device__ __forceinline__ void list_flagged(SOURCE &source, const Weights &w, float low, float high, Shared &sh)
{
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    source.each([&](float z, unsigned i) {
        if (!(z >= low && z <= high)) return;
        const double depth = w.depth_of(z);
        if (!(depth < kFar)) return;
        const unsigned b = w.bin_of(w.steps_of(depth));
        if ((sh.flags[b / 32] >> (b % 32) & 1u) == 0) return;
        const unsigned at = atomicAdd(&sh.listed, 1u);
        if (at < kListed) sh.list[at] = place_of(key_of(z), i);
    });
    __syncthreads();
}

// The near tokens into sh.list, unsorted, as far as they are at most kListed; sh.listed: how many they are.
template <class SOURCE>
__device__ __forceinline__ void list_near(SOURCE &source, const Weights &w, const Near &near, Shared &sh)
{
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    source.each([&](float z, unsigned i) {
        if (!near(z) || !(w.depth_of(z) < kFar)) return;
        const unsigned at = atomicAdd(&sh.listed, 1u);
        if (at < kListed) sh.list[at] = place_of(key_of(z), i);
    });
    __syncthreads();
}

// Sorts n listed tokens and sums their weights.
__device__ __forceinline__ void finish_list(const Weights &w, unsigned n, Shared &sh)
{
    sort_list(sh, n);
    const unsigned i = threadIdx.x * 2;
    auto weight = [&](unsigned at) { return at < n ? w.weight_of(value_of_key(~(uint32_t)(sh.list[at] >> 32)), sh.power) : 0.0; };
    const double w0 = weight(i), w1 = weight(i + 1);
    const double upto = sum_up_to(Mass{0, w0 + w1}, sh).mass;
    sh.list_mass[i] = upto - w1;
    sh.list_mass[i + 1] = upto;
    __syncthreads();
}

// The token where all that can be chosen are listed and sorted, n of them: no bins are needed.  The first wavefront's work.
__device__ __forceinline__ long long choose_listed(const Weights &w, const Settings &s, unsigned n, const Shared &sh)
{
    if (s.top_k < n) n = s.top_k;
    if (s.top_p < 1.0) {
        const double most = s.top_p * sh.list_mass[n - 1];
        const unsigned i = uniform(first_where(n, [&](unsigned i) { return sh.list_mass[i] >= most; }));
        n = i < n ? i + 1 : n;
    }
    if (s.reach < kFar) n = uniform(first_where(n, [&](unsigned i) { return w.depth_of(value_of_key(~(uint32_t)(sh.list[i] >> 32))) > s.reach; }));
    const double most = s.u * sh.list_mass[n - 1];
    const unsigned i = uniform(first_where(n, [&](unsigned i) { return sh.list_mass[i] > most; }));
    return (long long)(uint32_t)sh.list[i < n ? i : n - 1];
}

// ------------------------------------------------------------------------------------ questions
// The first token with which the count or the mass is reached.
struct Question {
    uint32_t count;
    double mass;
    bool above;     // more than the mass, not as much
    __device__ __forceinline__ bool reached(uint32_t c, double m) const { return c >= count || (above ? m > mass : m >= mass); }
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
    uint32_t by_min;
    float low_logit, high_logit;    // of the tokens that the plan lists

    __device__ __forceinline__ Questions(const Weights &w, const Settings &s, Shared &sh, uint32_t by_min) : w(w), s(s), sh(sh), by_min(by_min) {}

    // Sums of the bins, of which a lane has one.
    __device__ __forceinline__ void add_up(uint32_t count, u64 mass)
    {
        const Mass upto = sum_up_to(Mass{count, (double)mass * w.unit_of(threadIdx.x)}, sh);
        sh.count[threadIdx.x] = upto.count;
        sh.mass[threadIdx.x] = upto.mass;
        __syncthreads();
        total = uniform(Mass{sh.count[kBins - 1], sh.mass[kBins - 1]});
    }

    // The first of bins with tokens, by their sums, at whose end `q` is reached.  The last such bin is if no other.
    __device__ __forceinline__ Bin find(Question q, const uint32_t *count, const double *mass) const
    {
        const uint32_t all = count[kBins - 1];
        if (q.count > all) q.count = all;
        unsigned at = first_where(kBins, [&](unsigned i) { return q.reached(count[i], mass[i]); });
        if (count[at] == (at != 0 ? count[at - 1] : 0u))    // an empty one, where sums differ by a rounding
            at = first_where(kBins, [&](unsigned i) { return count[i] > count[at]; });
        const Mass before = at != 0 ? Mass{count[at - 1], mass[at - 1]} : Mass{0, 0.0};
        return Bin{uniform(at), uniform(before), uniform(Mass{count[at], mass[at]})};
    }
    __device__ __forceinline__ Bin find(const Question &q) const { return find(q, sh.count, sh.mass); }

    __device__ __forceinline__ bool flagged(unsigned bin) const { return (sh.flags[bin / 32] >> (bin % 32) & 1u) != 0; }

    // Flags this lane's bin or not, and says where each flagged bin starts in the list.
    __device__ __forceinline__ void flag(bool mine)
    {
        const u64 wave = __ballot(mine);
        if (threadIdx.x % 32 == 0) sh.flags[threadIdx.x / 32] = (uint32_t)(wave >> (threadIdx.x % 64));
        const uint32_t count = mine ? sh.count[threadIdx.x] - (threadIdx.x != 0 ? sh.count[threadIdx.x - 1] : 0u) : 0u;
        sh.starts[threadIdx.x] = sum_up_to(Mass{count, 0.0}, sh).count - count;
        __syncthreads();
    }

    // Flags the bins that hold the answers as far as the sums of bins tell: what one question leaves open between the ends of its bin is carried to the
    // next, from `low` to `high`.  The first wavefront's work.
    __device__ __forceinline__ void plan()
    {
        if (threadIdx.x < 64) {
            uint32_t listed = 0;
            Mass low = total, high = total;
            unsigned asked = 0;
            auto add = [&](const Question &least, const Question &most) {
                const Bin to = find(most), from = least.count == most.count && least.mass == most.mass ? to : find(least);
                low = from.before;
                high = to.with;
                const uint32_t tokens = high.count - low.count;
                const bool fits = listed + tokens <= kListed;
                if (fits) listed += tokens;
                if (threadIdx.x == 0) {
                    sh.from[asked] = fits ? from.at : kBins;
                    sh.to[asked] = to.at;
                }
                ++asked;
            };
            constexpr double kAny = (double)INFINITY;
            auto some = [](uint32_t count) { return count != 0 ? count : 1u; };
            if (s.top_k < total.count) add(Question{s.top_k, kAny, false}, Question{s.top_k, kAny, false});
            if (s.top_p < 1.0) add(Question{some(low.count), s.top_p * low.mass, false}, Question{high.count, s.top_p * high.mass, false});
            if (by_min < high.count) add(Question{by_min < low.count ? by_min : some(low.count), kAny, false}, Question{by_min, kAny, false});
            add(Question{some(low.count), s.u * low.mass, true}, Question{high.count, s.u * high.mass, true});
            for (; asked < 4; ++asked)
                if (threadIdx.x == 0) sh.from[asked] = kBins;
        }
        __syncthreads();
        bool mine = false;
        unsigned first = kBins, last = 0;
        for (unsigned i = 0; i < 4; ++i) {
            const unsigned from = sh.from[i], to = sh.to[i];
            mine = mine || (threadIdx.x >= from && threadIdx.x <= to);
            if (from >= kBins) continue;
            first = from < first ? from : first;
            last = to > last ? to : last;
        }
        flag(mine);
        // logits of bins `first` to `last`, and of one more on either side
        const double step = 1.0 / ((double)(1u << (kSteps - w.shift)) * w.scale);
        high_logit = (float)((double)w.top - ((double)first - 1.0) * step);
        low_logit = last < kBins - 2 ? (float)((double)w.top - ((double)last + 2.0) * step) : -INFINITY;
        if (w.infinite || !(step < 1e30)) {
            high_logit = INFINITY;
            low_logit = -INFINITY;
        }
        high_logit = uniform(high_logit);
        low_logit = uniform(low_logit);
    }

    // Lists the tokens of a bin of more than kListed that are near the answer: bins of places inside it, until they are few.  `before` moves up to them.
    template <class SOURCE>
    __device__ __forceinline__ unsigned narrow(SOURCE &source, const Question &q, unsigned bin, Mass &before)
    {
        auto each = [&](auto f) {
            source.each([&](float z, unsigned i) {
                const double depth = w.depth_of(z);
                if (depth < kFar && w.bin_of(w.steps_of(depth)) == bin) f(depth, place_of(key_of(z), i));
            });
        };
        __syncthreads();
        if (threadIdx.x == 0) {
            sh.low_place = ~0ull;
            sh.high_place = 0;
        }
        __syncthreads();
        each([&](double, u64 p) {
            atomicMin(&sh.low_place, p);
            atomicMax(&sh.high_place, p);
        });
        __syncthreads();
        u64 first = sh.low_place, last = sh.high_place;
        uint32_t *const count = reinterpret_cast<uint32_t *>(sh.list);      // sums of the bins of places
        double *const mass = sh.list_mass;
        for (;;) {
            const u64 step = (last - first) / kBins + 1;
            __syncthreads();
            sh.bins[threadIdx.x] = 0;       // counts and masses apart: a bin may hold more tokens than a chunk
            sh.starts[threadIdx.x] = 0;
            __syncthreads();
            each([&](double depth, u64 p) {
                if (p < first || p > last) return;
                unsigned steps;
                const unsigned b = (unsigned)((p - first) / step);
                const double part = w.part_of(depth, steps);
                atomicAdd(&sh.bins[b], packed(sh.power[steps & 127u], part) & kMassBits);
                atomicAdd(&sh.starts[b], 1u);
            });
            __syncthreads();
            const Mass upto = before + sum_up_to(Mass{sh.starts[threadIdx.x], (double)sh.bins[threadIdx.x] * w.unit_of(bin)}, sh);
            count[threadIdx.x] = upto.count - before.count;
            mass[threadIdx.x] = upto.mass;
            __syncthreads();
            Question here = q;
            here.count = q.count > before.count ? q.count - before.count : 1u;
            const Bin b = find(here, count, mass);
            if (b.at != 0) before = Mass{before.count + b.before.count, b.before.mass};
            first += b.at * step;
            if (last - first >= step) last = first + step - 1;
            if (b.with.count - b.before.count <= kListed) break;    // a step of 1 holds one token
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        each([&](double, u64 p) {
            if (p < first || p > last) return;
            const unsigned at = atomicAdd(&sh.listed, 1u);
            if (at < kListed) sh.list[at] = p;
        });
        __syncthreads();
        return uniform(sh.listed);
    }

    // Top-k, top-p, min-p, the choice; whether it is asked at all.
    __device__ __forceinline__ bool question(unsigned turn, const Mass &kept, Question &q) const
    {
        q = Question{kept.count, (double)INFINITY, turn == 3};
        if (turn == 0) {
            q.count = s.top_k;
            return s.top_k < kept.count;
        }
        if (turn == 1) {
            q.mass = s.top_p * kept.mass;
            return s.top_p < 1.0;
        }
        if (turn == 2) {
            q.count = by_min;
            return by_min < kept.count;
        }
        q.mass = s.u * kept.mass;
        return true;
    }

    // The token (in the first wavefront, which asks the questions), where the tokens of the flagged bins are listed and sorted.  All lanes list others
    // where a question needs them.
    template <class SOURCE>
    __device__ __forceinline__ long long choose(SOURCE &source)
    {
        Mass kept = total, before{0, 0.0};
        unsigned turn = 0, at = 0, n = 0;
        bool relisted = false;      // for the question that is asked next, n tokens behind `before`
        for (;;) {
            if (threadIdx.x < 64) {
                bool open = false;
                for (; turn < 4 && !open; ) {
                    Question q;
                    if (question(turn, kept, q)) {
                        unsigned start = 0;
                        if (!relisted) {
                            const Bin b = find(q);
                            before = b.before;
                            n = b.with.count - b.before.count;
                            open = !flagged(b.at);
                            if (!open) {
                                start = uniform(sh.starts[b.at]);
                            } else if (threadIdx.x == 0) {
                                sh.asked_bin = b.at;
                                sh.asked_count = q.count;
                                sh.asked_above = q.above;
                                sh.asked_mass = q.mass;
                                sh.asked_before = b.before;
                                sh.asked_with = b.with;
                            }
                        }
                        if (!open) {
                            const double base = before.mass - (start != 0 ? sh.list_mass[start - 1] : 0.0);
                            const unsigned i = first_where(n, [&](unsigned i) { return q.reached(before.count + i + 1, base + sh.list_mass[start + i]); });
                            at = uniform(start + (i < n ? i : n - 1));
                            kept = uniform(Mass{before.count + at - start + 1, base + sh.list_mass[at]});
                            relisted = false;
                        }
                    }
                    if (!open) ++turn;
                }
                if (threadIdx.x == 0) sh.asked = open;
            }
            __syncthreads();
            if (uniform(sh.asked) == 0) break;
            const unsigned bin = uniform(sh.asked_bin);
            before = uniform(sh.asked_before);
            n = uniform(sh.asked_with.count) - before.count;
            __syncthreads();
            if (n <= kListed) {
                flag(threadIdx.x == bin);
                list_flagged(source, w, -INFINITY, INFINITY, sh);
            } else {
                n = narrow(source, Question{uniform(sh.asked_count), uniform(sh.asked_mass), sh.asked_above != 0}, bin, before);
                flag(false);
            }
            finish_list(w, n, sh);
            relisted = true;
        }
        return (long long)(uint32_t)sh.list[at];
    }
};

// ------------------------------------------------------------------------------------ kernels
// A row to a block.
template <class ELEM, bool CAP, bool WIDE, unsigned E>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const OnTheWay<ELEM, E> raw(static_cast<const ELEM *>(a.logits) + blockIdx.x * a.row, 0, a.vocabulary);
    const Settings s = settings_of(a, blockIdx.x);
    Held<ELEM, CAP, WIDE, E> held(raw, a.cap, tab);
    float lane_top;
    const Ends e = ends_of(held, lane_top, sh);
    long long token = -1;
    if (!e.empty()) {
        if (s.greedy) {
            token = first_of(held, e.top, sh);
        } else {
            const Weights w(e, s.scale);
            fill_powers(sh);
            // Where all that top-k leaves, with what is near its last, are at most kRanked tokens, they are listed, and nothing else is needed.
            bool few = false;
            if (s.top_k <= kRanked / 2 && s.top_k < a.vocabulary) {
                uint32_t tokens;
                if (E == kMost) {
                    // counting the lanes' largest alone mostly leaves little more than is asked for (one row of 32000: 50 in 11.0 us, 200 in 15.3; with all
                    // logits counted 12.8 and 16.5; rows with few logits for each lane would be counted twice)
                    Tops tops{lane_top};
                    const Near near = nearest(tops, e, s.top_k, tokens, sh);
                    if (!near.all()) {
                        list_near(held, w, near, sh);
                        few = uniform(sh.listed) <= kRanked;
                    }
                }
                if (!few) {
                    const Near near = nearest(held, e, s.top_k, tokens, sh);
                    few = tokens <= kRanked;
                    if (few) list_near(held, w, near, sh);
                }
            }
            Questions questions(w, s, sh, 0);
            if (!few) {
                fill_bins(held, w, s.reach, sh);
                questions.by_min = uniform(sh.by_min);
                questions.add_up((uint32_t)(sh.bins[threadIdx.x] >> 48), sh.bins[threadIdx.x] & kMassBits);
                questions.plan();
                list_flagged(held, w, questions.low_logit, questions.high_logit, sh);
            }
            const unsigned n = uniform(sh.listed);
            finish_list(w, n, sh);
            // another list than the plan's, if one is needed, comes from memory: the registers are the questions'
            Read<ELEM, CAP, WIDE> read{static_cast<const ELEM *>(a.logits) + blockIdx.x * a.row, a.vocabulary, a.cap, tab};
            if (!few) token = questions.choose(read);
            else if (threadIdx.x < 64) token = choose_listed(w, s, n, sh);
        }
    }
    if (threadIdx.x == 0) a.tokens[blockIdx.x] = token;
}

// Rows in chunks of E logits a lane.  Blocks have a chunk each but for the last launch.
struct Where {
    unsigned row, first, end;
};
template <unsigned E>
__device__ __forceinline__ Where chunk_of(const SampleArgs &a)
{
    constexpr unsigned kChunk = E * kThreads;
    const unsigned row = blockIdx.x / a.chunks, first = blockIdx.x % a.chunks * kChunk;
    return Where{row, first, a.vocabulary - first < kChunk ? a.vocabulary : first + kChunk};
}

// The row's ends from those of its chunks.
__device__ __forceinline__ Ends row_ends(const SampleArgs &a, unsigned row)
{
    Ends e = kNoEnds;
#pragma unroll 4
    for (unsigned c = 0; c < a.chunks; ++c) {
        const float4 v = a.ends[row * (u64)a.chunks + c];
        e.meet(v.x, v.y, __float_as_uint(v.z));
    }
    return e;
}

// The row's bins added up from those of its chunks, and the plan.
__device__ __forceinline__ void add_up_row(const SampleArgs &a, unsigned row, Questions &questions)
{
    uint32_t count = 0, by_min = 0;
    u64 mass = 0;
#pragma unroll 4
    for (unsigned c = 0; c < a.chunks; ++c) {
        const u64 at = row * (u64)a.chunks + c, v = a.bins[at * kBins + threadIdx.x];
        count += (uint32_t)(v >> 48);
        mass += v & kMassBits;
        by_min += a.by_min[at];
    }
    questions.by_min = by_min;
    questions.add_up(count, mass);
    questions.plan();
}

template <class ELEM, bool CAP, bool WIDE, unsigned E>
__global__ __launch_bounds__(kThreads) void sample_ends_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of<E>(a);
    const OnTheWay<ELEM, E> raw(static_cast<const ELEM *>(a.logits) + at.row * a.row, at.first, at.end);
    Held<ELEM, CAP, WIDE, E> held(raw, a.cap, tab);
    float lane_top;
    const Ends e = ends_of(held, lane_top, sh);
    const uint32_t first = settings_of(a, at.row).greedy ? first_of(held, e.top, sh) : 0u;
    if (threadIdx.x == 0) {
        a.ends[blockIdx.x] = float4{e.top, e.low, __uint_as_float(e.widest), __uint_as_float(first)};
        if (at.first == 0) a.listed[at.row] = a.arrived[at.row] = 0;
    }
}

template <class ELEM, bool CAP, bool WIDE, unsigned E>
__global__ __launch_bounds__(kThreads, 8) void sample_bins_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of<E>(a);
    const OnTheWay<ELEM, E> raw(static_cast<const ELEM *>(a.logits) + at.row * a.row, at.first, at.end);
    const Settings s = settings_of(a, at.row);
    const Ends e = row_ends(a, at.row);
    if (e.empty() || s.greedy) return;
    Held<ELEM, CAP, WIDE, E> held(raw, a.cap, tab);
    fill_bins(held, Weights(e, s.scale), s.reach, sh);
    a.bins[blockIdx.x * (u64)kBins + threadIdx.x] = sh.bins[threadIdx.x];
    if (threadIdx.x == 0) a.by_min[blockIdx.x] = sh.by_min;
}

// The chunks' tokens of the bins that hold answers; the block that is the row's last to have listed its own has them all, and answers.  None waits for
// another.
template <class ELEM, bool CAP, bool WIDE, unsigned E>
__global__ __launch_bounds__(kThreads, 8) void sample_answer_kernel(SampleArgs a, KtLutPack pack)
{
    __shared__ Shared sh;
    const LaneTable tab(pack);
    const Where at = chunk_of<E>(a);
    const ELEM *const from = static_cast<const ELEM *>(a.logits) + at.row * a.row;
    // asked for before all else, where the registers are enough for that and for two blocks on a CU
    constexpr bool kEarly = sizeof(ELEM) * E <= 64;
    OnTheWay<ELEM, E> raw;
    if constexpr (kEarly) raw = OnTheWay<ELEM, E>(from, at.first, at.end);
    const Settings s = settings_of(a, at.row);
    const Ends e = row_ends(a, at.row);
    if (e.empty() || s.greedy) {
        if (at.first != 0 || threadIdx.x != 0) return;
        long long token = -1;
        for (unsigned c = a.chunks; c-- > 0 && !e.empty();) {   // the first chunk with the largest logit
            const float4 v = a.ends[at.row * (u64)a.chunks + c];
            if (v.x == e.top) token = (long long)__float_as_uint(v.w);
        }
        a.tokens[at.row] = token;
        return;
    }
    const Weights w(e, s.scale);
    fill_powers(sh);
    Questions questions(w, s, sh, 0);
    add_up_row(a, at.row, questions);
    {
        if constexpr (!kEarly) raw = OnTheWay<ELEM, E>(from, at.first, at.end);
        Held<ELEM, CAP, WIDE, E> held(raw, a.cap, tab);
        list_flagged(held, w, questions.low_logit, questions.high_logit, sh);
    }
    const unsigned mine = uniform(sh.listed);       // at most kListed: the plan's
    if (threadIdx.x == 0) sh.asked_bin = atomicAdd(&a.listed[at.row], mine);
    __syncthreads();
    u64 *const list = a.list + at.row * (u64)kListed;
    for (unsigned i = threadIdx.x; i < mine; i += kThreads)
        if (sh.asked_bin + i < kListed) __hip_atomic_store(&list[sh.asked_bin + i], sh.list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // These stores go to where all dies see them, and are there before the block counts as arrived: on gfx950 agent-scope stores and
    // loads carry sc1, with which they do not stop at the L2 of their die, and vmcnt counts a store until it is done.  The order rests on that and on the barrier, not on
    // release and acquire: a fence of the whole GPU would write every L2 back, each wavefront's once more (64 rows of 131072 took 145 us with them).
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) sh.asked = atomicAdd(&a.arrived[at.row], 1u) + 1 == a.chunks;
    __syncthreads();
    if (uniform(sh.asked) == 0) return;
    const unsigned listed = uniform(__hip_atomic_load(&a.listed[at.row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)), n = listed < kListed ? listed : kListed;
    for (unsigned i = threadIdx.x; i < n; i += kThreads) sh.list[i] = __hip_atomic_load(&list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    finish_list(w, n, sh);
    Read<ELEM, CAP, WIDE> read{from, a.vocabulary, a.cap, tab};
    const long long token = questions.choose(read);
    if (threadIdx.x == 0) a.tokens[at.row] = token;
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

// Logits of a lane, and chunks of a row.
struct Cut {
    unsigned each;
    size_t chunks;
};
Cut cut_of(size_t rows, size_t vocabulary)
{
    auto chunks = [&](unsigned each) { return (vocabulary + each * kThreads - 1) / (each * kThreads); };
    if (vocabulary <= kFew * kThreads) return Cut{kFew, 1};
    if (vocabulary <= kMost * kThreads) return Cut{kMost, 1};
    // chunks of 8192 where each has a CU (32 rows of 50000: 27 us, 33 with chunks of 32768), of 32768 beyond (32 rows of 131072: 37 us against 51)
    return rows * chunks(kFew) <= 256 ? Cut{kFew, chunks(kFew)} : Cut{kMost, chunks(kMost)};
}

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
    const Cut cut = cut_of(s->rows, s->vocabulary);
    a.chunks = (unsigned)cut.chunks;
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
    a.bins = a.list = nullptr;
    a.ends = nullptr;
    a.by_min = a.listed = a.arrived = nullptr;
    const size_t rows = s->rows, blocks = rows * a.chunks;
    if (a.chunks > 1) {
        if (workspace == nullptr) return KT_ERR_NULL;
        a.bins = static_cast<u64 *>(workspace);
        a.list = a.bins + blocks * kBins;
        a.ends = reinterpret_cast<float4 *>(a.list + rows * kListed);
        a.by_min = reinterpret_cast<uint32_t *>(a.ends + blocks);
        a.listed = a.by_min + blocks;
        a.arrived = a.listed + rows;
    }
    if (blocks * kThreads >= (size_t)1 << 32) return KT_ERR_SHAPE;
    auto launch = [&](auto kernel, size_t n) { return launch_checked(kernel, (unsigned)n, kThreads, stream, a, pack); };
    auto of = [&](auto elem, auto capped) {
        typedef decltype(elem) ELEM;
        constexpr bool CAP = decltype(capped)::value, W = CAP && WIDE;
        if (a.chunks == 1) return cut.each == kFew ? launch(sample_kernel<ELEM, CAP, W, kFew>, rows) : launch(sample_kernel<ELEM, CAP, W, kMost>, rows);
        auto chunked = [&](auto each) {
            constexpr unsigned E = decltype(each)::value;
            ktanh_status_t done = launch(sample_ends_kernel<ELEM, CAP, W, E>, blocks);
            if (done == KT_OK) done = launch(sample_bins_kernel<ELEM, CAP, W, E>, blocks);
            return done == KT_OK ? launch(sample_answer_kernel<ELEM, CAP, W, E>, blocks) : done;
        };
        return cut.each == kFew ? chunked(std::integral_constant<unsigned, kFew>()) : chunked(std::integral_constant<unsigned, kMost>());
    };
    if (s->f32) return s->cap > 0.0 ? of(uint32_t(), std::true_type()) : of(uint32_t(), std::false_type());
    return s->cap > 0.0 ? of(uint16_t(), std::true_type()) : of(uint16_t(), std::false_type());
}

}  // namespace

extern "C" size_t ksample_workspace(const ksample_shape_t *shape)
{
    if (check_shape(shape) != KT_OK) return 0;
    const size_t chunks = cut_of(shape->rows, shape->vocabulary).chunks, blocks = shape->rows * chunks;
    return chunks == 1 ? 0 : blocks * (kBins * sizeof(u64) + sizeof(float4) + sizeof(uint32_t)) + shape->rows * (kListed * sizeof(u64) + 2 * sizeof(uint32_t));
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
