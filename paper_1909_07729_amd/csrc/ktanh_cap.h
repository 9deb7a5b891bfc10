// Attention with scores capped through K-TanH: what its kernels share.
//
//   s = q . k,   t = K(s * scale / cap),   y = cap * t,   p = softmax of y over the keys that a query sees
//
// K is the Float32 form of Algorithm 1 (arXiv:1909.07729).  On one interval of the table it is a line,
//   K(x) = A x + B for x > 0,   A = 2^(E - E_i - r),   B = 2^(E - 127) (1 - 2^-r + b/128),
// which the kernels evaluate with one fused multiply-add: what the shift of Algorithm 1 drops below the last
// place of a Float32 is kept.  128 lines are held in LDS, indexed by the three low exponent bits and the four
// high mantissa bits of |x| clamped to [0.25 - 2^-26, 16]: the identity below 0.25, saturation from 4 on and
// the table in between need no comparisons, and tables of 32 and of 64 intervals run the same code.
//
// |y| <= cap, and caps are at most 64, so e^y stays within e^-64 .. e^64 and the softmax needs no running
// maximum: the weights are summed as they are, which also lets parts of a row be joined by adding.
//
// Matrix products use v_mfma_f32_32x32x16_bf16.  Scores are formed so that the lane that holds a weight holds
// it where the next product wants it: an accumulator's lane l has column l & 31 and the rows (r & 3) + 8 (r >>
// 2) + 4 (l >> 5), r = 0..15; packed to BFloat16, registers 8 i .. 8 i + 7 are the second operand of a product
// over 16 of those rows in the order  8 i' + 4 (l >> 5) + (j & 3),  and the first operand is read from LDS in
// that same order by transposing reads of 4 rows x 16 columns (ds_read_b64_tr_b16).  No weight crosses lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ktanh_pack.h"

namespace ktanh_cap {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_at8 __attribute__((ext_vector_type(4), aligned(8)));  // 16 bytes anywhere that eight may be

constexpr int kThreads = 256, kWaves = 4;
// A wavefront has 32 rows.  The four of a block go over the tiles of the other tensor together, with 128 rows,
// or the same 64 or 32 rows of two or four heads that share that tensor; or (SPLIT) all four have the same 32
// rows, each goes over every fourth tile on its own, and their sums are joined at the end.
constexpr int kRows = 128;
constexpr float kLog2e = 1.44269504088896340736f;

// A tensor [rows][heads][dim], dim contiguous.
struct Rows {
    const uint16_t *at;
    long long row, head;  // strides in elements
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

__device__ __forceinline__ bf16x8 pack8(const float *v)
{
    return __builtin_bit_cast(bf16x8, u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])});
}

__device__ __forceinline__ float sum_of(bf16x2 pair, float sum)
{
    return __builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
}

// The same, with the sum of the rounded values.  Outputs are divided by the sum of the weights as the product
// has them: the roundings of one weight in numerator and denominator cancel (o is off by 0.0018 of its norm
// instead of 0.0023, 0.0017 of it the rounding of o itself).
__device__ __forceinline__ bf16x8 pack8(const float *v, float *sum)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 pair = __builtin_convertvector(f32x2{v[2 * i], v[2 * i + 1]}, bf16x2);
        *sum = sum_of(pair, *sum);
        w[i] = __builtin_bit_cast(uint32_t, pair);
    }
    return __builtin_bit_cast(bf16x8, w);
}

// ------------------------------------------------------------------------------------------ the cap
// lines[i], i = low three exponent bits << 4 | high four mantissa bits, times `unit`.
template <int THREADS = kThreads>
__device__ __forceinline__ void spread_lines(f32x2 *lines, const KtCapPack &pack, float unit)
{
    for (int i = threadIdx.x; i < 128; i += THREADS) {
        const int e = i >> 4, slot = i & 63;
        const float a = e == 4 ? 1.0f : (e >= 1 && e <= 3) ? 0.0f : pack.a[slot];
        const float b = e == 4 ? 0.0f : (e >= 1 && e <= 3) ? 1.0f : pack.b[slot];
        lines[i] = f32x2{a * unit, b * unit};
    }
}

// unit * K(x).  A NaN stays one.  Everything below 0.25 reads one line, so that lanes of small scores share an
// address: table reads at many are what the LDS unit has least time for.
__device__ __forceinline__ f32x2 line_of(float x, const f32x2 *lines)
{
    const uint32_t key = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fabsf(x), 0x1.fffffep-3f, 16.0f));
    return *reinterpret_cast<const f32x2 *>(reinterpret_cast<const char *>(lines) + ((key >> 16) & 0x3F8u));
}

__device__ __forceinline__ float on_line(float x, f32x2 line) { return __builtin_copysignf(__builtin_fmaf(line.x, __builtin_fabsf(x), line.y), x); }

__device__ __forceinline__ float capped(float x, const f32x2 *lines) { return on_line(x, line_of(x, lines)); }

// Which accumulator rows of a lane, numbered from 0 at `at`, lie in [first, last): others become zero.  In a
// branch of its own (the statement keeps the compiler from testing every tile).
struct Span {
    uint32_t from, count;
    __device__ __forceinline__ Span(int first, int last, int at)
        : from((uint32_t)(at + 4 * (int)((threadIdx.x & 63) >> 5) - first)), count((uint32_t)max(last - first, 0))
    {
    }
    __device__ __forceinline__ bool has(int r) const { return from + (uint32_t)((r & 3) + 8 * (r >> 2)) < count; }
};

__device__ __forceinline__ void keep(float *p, Span span)
{
    asm volatile("" : "+v"(span.count));
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = span.has(r) ? p[r] : 0.0f;
}

// ------------------------------------------------------------------------------------- tiles in LDS
// Rows of D BFloat16 values, 16 bytes apart, in an order in which the two low bits of a row's number change
// places with the two above them.  Both ways of reading then run without bank conflicts, eight rows at one
// 16-byte chunk (ds_read_b128) and 64 bytes of four consecutive rows (transposing reads), and all reads of a
// lane are one address and constant offsets.
template <int D> constexpr int kPitch = 2 * D + 16;

template <int D>
__device__ __forceinline__ int chunk_at(int row, int chunk)  // byte offset
{
    return ((row & ~15) | (row & 3) << 2 | (row >> 2 & 3)) * kPitch<D> + 16 * chunk;
}

// Operand of 32 rows of the tile (from `row0`, a multiple of 32) over values 16 k .. 16 k + 15 of each.
template <int D>
__device__ __forceinline__ bf16x8 rows_of(const char *tile, int row0, int k)
{
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const bf16x8 *>(tile + chunk_at<D>(lane & 31, lane >> 5) + row0 * kPitch<D> + 32 * k);
}

// Operand of columns 32 c .. 32 c + 31 of the tile over its rows row0 .. row0 + 15 in the order of a packed
// accumulator.
template <int D>
__device__ __forceinline__ bf16x8 columns_of(const char *tile, int row0, int c)
{
    typedef __attribute__((address_space(3))) s16x4 *lds4;
    const int lane = threadIdx.x & 63;
    const char *at = tile + chunk_at<D>((lane >> 5) * 4 + (lane >> 2 & 3), 0) + (lane >> 4 & 1) * 32 + (lane & 3) * 8 + row0 * kPitch<D> + 64 * c;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 2 * kPitch<D>));  // eight rows on
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// 32 rows of D BFloat16 values as direct loads bring them (each instruction of a wavefront writes 1 KiB in the
// order of its lanes):
// row m lies in stretch m % kStretches, m / kStretches rows into it.  The stretches start such that, again,
// eight rows at one 16-byte chunk and 64 bytes of four consecutive rows lie in different banks, and all reads
// of a lane are one address and constants.
template <int D>
struct Keys32 {
    static constexpr int kStretches = D / 16, kDeep = 32 / kStretches, kChunks = D / 8;
    static constexpr int kBytes = D == 128 ? 8 * 1088 + 32 : 4 * 1104;

    __device__ __forceinline__ static int stretch_at(int g) { return D == 128 ? g * 1088 + (g >> 2) * 16 : g * 1104; }
    __device__ __forceinline__ static int row_at(int m) { return stretch_at(m % kStretches) + m / kStretches * (2 * D); }
    // The row and the chunk of it that a lane loads into stretch g.
    __device__ __forceinline__ static int row_of_lane(int g) { return g + (int)(threadIdx.x & 63) / kChunks * kStretches; }
    __device__ __forceinline__ static int chunk_of_lane() { return threadIdx.x % kChunks; }

    // Operand of the 32 rows over values 16 k .. 16 k + 15 of each.
    __device__ __forceinline__ static bf16x8 rows(const char *tile, int k)
    {
        const int lane = threadIdx.x & 63;
        return *reinterpret_cast<const bf16x8 *>(tile + row_at(lane & 31) + 16 * (lane >> 5) + 32 * k);
    }
    // Operand of columns 32 c .. 32 c + 31 over rows 16 i .. 16 i + 15 in the order of a packed accumulator.
    __device__ __forceinline__ static bf16x8 columns(const char *tile, int i, int c)
    {
        typedef __attribute__((address_space(3))) s16x4 *lds4;
        const int lane = threadIdx.x & 63;
        const char *at = tile + row_at((lane >> 5) * 4 + (lane >> 2 & 3)) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 16 / kStretches * i * (2 * D) + 64 * c));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + (16 * i + 8) / kStretches * (2 * D) + 64 * c));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// 16 bytes of each lane from memory to LDS, at `to` + 16 * lane, with no register between.
__device__ __forceinline__ void load_direct(const void *from, char *to)
{
    typedef const __attribute__((address_space(1))) void *global;
    typedef __attribute__((address_space(3))) void *local;
    __builtin_amdgcn_global_load_lds((global)from, (local)to, 16, 0, 0);
}

// This wavefront's loads, direct ones among them, have arrived.
__device__ __forceinline__ void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// A tile in LDS is complete, and what was in the place of the next one has been read: behind the block's
// barrier where its wavefronts share it, else behind this wavefront's own reads and writes.
template <bool SPLIT>
__device__ __forceinline__ void tile_complete()
{
    if constexpr (SPLIT) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    else __syncthreads();
}

// 32 rows of D BFloat16 values to memory by whole rows, through `tile` of LDS: a wavefront's own, or (SPLIT)
// the block's, of which each wavefront has a fourth of the columns.  quad(i) are values 8 i + 4 (lane / 32) ..
// + 3 of row lane & 31, from the wavefront's first column on.  Straight from the accumulator each store touches
// 32 rows, 16 bytes of each: 16 documents of 256 tokens, 32 heads of 128, take 46 us so, and 30 this way.
// Chunks of 16 bytes change places with the low bits of their row's number against bank conflicts.
template <int D, bool SPLIT, class Quad>
__device__ __forceinline__ void store_rows(char *tile, uint16_t *to, long long row, int there, Quad quad)
{
    constexpr int kChunks = D / 8, kMine = SPLIT ? kChunks / kWaves : kChunks, kLanes = SPLIT ? kThreads : 64;
    const int lane = threadIdx.x & 63, first = SPLIT ? (int)(threadIdx.x >> 6) * kMine : 0;
    const int member = SPLIT ? (int)threadIdx.x : lane, chunk = member % kChunks;
    auto complete = [] {
        if constexpr (SPLIT) __syncthreads();
        else tile_complete<true>();
    };
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        *reinterpret_cast<u32x2 *>(tile + (lane & 31) * 2 * D + 16 * (((first + i) ^ lane) % kChunks) + 8 * (lane >> 5)) = quad(i);
    complete();
#pragma unroll
    for (int n = 0; n < 32 * kChunks / kLanes; ++n) {
        const int at = member / kChunks + n * (kLanes / kChunks);
        const u32x4 v = *reinterpret_cast<const u32x4 *>(tile + at * 2 * D + 16 * ((chunk ^ at) % kChunks));
        if (at < there) *reinterpret_cast<u32x4_at8 *>(to + at * row + 8 * chunk) = v;
    }
    complete();
}

// The same of a wavefront's D Float32 values, in two halves: `tile` has 64 D bytes, as for the other.
template <int D, class Quad>
__device__ __forceinline__ void store_rows_wide(char *tile, float *to, long long row, int there, Quad quad)
{
    constexpr int kChunks = D / 8, kQuads = D / 16;  // of half a row
    const int lane = threadIdx.x & 63, chunk = lane % kChunks;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < kQuads; ++i)
            *reinterpret_cast<f32x4 *>(tile + (lane & 31) * 2 * D + 16 * (((2 * i + (lane >> 5)) ^ lane) % kChunks)) = quad(kQuads * half + i);
        tile_complete<true>();
#pragma unroll
        for (int n = 0; n < kChunks / 2; ++n) {
            const int at = lane / kChunks + n * (64 / kChunks);
            const f32x4 v = *reinterpret_cast<const f32x4 *>(tile + at * 2 * D + 16 * ((chunk ^ at) % kChunks));
            if (at < there) *reinterpret_cast<f32x4 *>(to + at * row + D / 2 * half + 4 * chunk) = v;
        }
        tile_complete<true>();
    }
}

// Tiles of 32 rows of two tensors on their way to LDS, one behind the other, and of each the stretches that
// wavefront `wave` of LOADERS brings; a row behind the last one is read as the last.  One address for all lanes
// and 32 bits of offset for each (strides are below 2^24).
template <int D, int LOADERS, int STEP = 32>
struct Stream {
    typedef Keys32<D> Tile;
    static constexpr int kShare = Tile::kStretches / LOADERS;
    const uint16_t *a_rows, *b_rows;
    long long a_row, b_row;
    int last, wave;
    const char *a, *b;  // the next tile's first row of this wavefront
    uint32_t a_off, b_off;

    __device__ __forceinline__ Stream(const uint16_t *a_rows, long long a_row, const uint16_t *b_rows, long long b_row,
                                      int last, int wave, int at)
        : a_rows(a_rows), b_rows(b_rows), a_row(a_row), b_row(b_row), last(last), wave(wave)
    {
        const uint32_t row = Tile::row_of_lane(0), chunk = 16 * Tile::chunk_of_lane();
        a_off = row * 2 * (uint32_t)a_row + chunk;
        b_off = row * 2 * (uint32_t)b_row + chunk;
        start(at);
    }
    __device__ __forceinline__ void start(int at)
    {
        a = reinterpret_cast<const char *>(a_rows + (at + wave * kShare) * a_row);
        b = reinterpret_cast<const char *>(b_rows + (at + wave * kShare) * b_row);
    }
    // Loads rows at .. at + 31, which are next; the ones after begin STEP on.
    __device__ __forceinline__ void next(int at, char *a_tile, char *b_tile)
    {
        const bool there = at + 32 <= last + 1;
        // Of two stretches each chooses its addresses, eight are in the code twice: with the second form for
        // two 16384 tokens in 32 heads of 128 take 2360 us instead of 2310, with the first for eight 2048 in 8
        // heads 29.7 instead of 25.9.
        if constexpr (kShare <= 2) {
#pragma unroll
            for (int n = 0; n < kShare; ++n) {
                const int g = wave * kShare + n;
                uint32_t a_at = a_off, b_at = b_off;
                const char *a_from = a + n * 2 * a_row, *b_from = b + n * 2 * b_row;
                if (!there) {
                    const uint32_t row = min(Tile::row_of_lane(g), last - at), chunk = 16 * Tile::chunk_of_lane();
                    a_from = reinterpret_cast<const char *>(a_rows + at * a_row);
                    b_from = reinterpret_cast<const char *>(b_rows + at * b_row);
                    a_at = row * 2 * (uint32_t)a_row + chunk;
                    b_at = row * 2 * (uint32_t)b_row + chunk;
                }
                load_direct(a_from + a_at, a_tile + Tile::stretch_at(g));
                load_direct(b_from + b_at, b_tile + Tile::stretch_at(g));
            }
        } else if (there) {
#pragma unroll
            for (int n = 0; n < kShare; ++n) {
                const int g = wave * kShare + n;
                load_direct(a + n * 2 * a_row + a_off, a_tile + Tile::stretch_at(g));
                load_direct(b + n * 2 * b_row + b_off, b_tile + Tile::stretch_at(g));
            }
        } else {
            const char *a_from = reinterpret_cast<const char *>(a_rows + at * a_row), *b_from = reinterpret_cast<const char *>(b_rows + at * b_row);
            const uint32_t chunk = 16 * Tile::chunk_of_lane();
#pragma unroll
            for (int n = 0; n < kShare; ++n) {
                const int g = wave * kShare + n;
                const uint32_t row = min(Tile::row_of_lane(g), last - at);
                load_direct(a_from + (row * 2 * (uint32_t)a_row + chunk), a_tile + Tile::stretch_at(g));
                load_direct(b_from + (row * 2 * (uint32_t)b_row + chunk), b_tile + Tile::stretch_at(g));
            }
        }
        a += STEP * 2 * a_row;
        b += STEP * 2 * b_row;
    }
};

// ------------------------------------------------------------------------------------------- blocks
// What a block has to do: a stretch of rows, by its rank in work, for one key/value head, one of the parts that
// it is cut into, and one of the `members` that share its keys (query heads of the group).
struct Unit {
    int kv_head, rank, part, member;
};

// Blocks for all units; behind them come the blocks that clear.
__host__ __device__ __forceinline__ unsigned long long unit_blocks(unsigned long long tiles, int kv_heads, int parts, int members)
{
    return (tiles * kv_heads * parts + 7) / 8 * 8 * members;
}

// Consecutive blocks go to the eight dies in turn.  The members of a unit come to one die, and share its
// second-level cache; where the key/value heads are a multiple of eight, all units of a head do, eight heads
// after the other; else the heads take turns, so that in either case each die has as much of the long stretches
// as of the short ones and of those that are empty (pieces of 500 tokens of eight sequences, 12 heads on 4:
// 268 us; with half of a head's ranks to each die 392).  False: nothing to do.
__device__ __forceinline__ bool unit_of_block(unsigned block, unsigned tiles, int kv_heads, int parts, int members, Unit *unit)
{
    const unsigned i = block >> 3, n = i / members * 8 + (block & 7), turns = kv_heads % 8 == 0 ? 8 : kv_heads, of_head = n / turns;
    if (n >= tiles * kv_heads * parts) return false;
    unit->member = (int)(i % members);
    unit->part = (int)(of_head % parts);
    unit->rank = (int)(of_head / parts % tiles);
    unit->kv_head = (int)(of_head / parts / tiles * turns + n % turns);
    return true;
}

// A stretch of 2^shift rows of a document.  There are at most rows >> shift and documents in sum, known without
// reading the offsets.
// Offsets outside [0, rows] are taken as the nearest in range, so that a wrong one reads nothing out of bounds.
struct Stretch {
    int doc, begin, end, first;  // rows of the document, and the first of the stretch; first >= end: nothing to do
    int other_begin, others;     // rows of the other tensor that belong to the document
};

struct Others {
    int begin, count;
};

__device__ __forceinline__ int offset_at(const int *offsets, int d, int rows)
{
    return offsets == nullptr ? min(d, rows) : min(max(offsets[d], 0), rows);
}

// The last document for which `starts` (true up to some document, false behind it) holds; 0 if none.  By whole
// wavefronts.
template <class Starts>
__device__ __forceinline__ int last_document(int docs, Starts starts)
{
    int before = 0;
    if (docs > 1) {
        for (int base = 0; base < docs; base += 64) {
            const int d = base + (int)(threadIdx.x & 63);
            const int n = __builtin_popcountll(__ballot(d < docs && starts(d)));
            before += n;
            if (n < 64) break;
        }
    }
    return __builtin_amdgcn_readfirstlane(max(before, 1) - 1);
}

// The sum over the wavefront, and over the lanes before this one, of numbers below 2^bits.
__device__ __forceinline__ int lanes_sum(int v, int bits)
{
    int sum = 0;
    for (int b = 0; b < bits; ++b) sum += __builtin_popcountll(__ballot(v >> b & 1)) << b;
    return sum;
}

__device__ __forceinline__ int lanes_before(int v, int bits)
{
    int sum = 0;
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot(v >> b & 1);
        sum += __builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0)) << b;
    }
    return sum;
}

// The stretch of 2^shift rows that is the rank-th in work, the most first: blocks start in this order, and the
// last ones to start are short (in the order of the rows sixteen documents of 8192 tokens keep the chip 79 %
// busy, like this 94).  By whole wavefronts.
// `others_of(d)`: rows of the other tensor that document d has; asked for together with the document's own.
// Work, in units of as many rows: those rows if all are seen; if causal, the number of the stretch and the rows
// before the document's first (`rising`: queries, over keys), or its number from the end (keys, over queries).
// More than 64 documents stay in the order of their rows.
template <class OthersOf>
__device__ __forceinline__ Stretch stretch_of(int shift, int rank, const int *offsets, int docs, int rows, bool causal,
                                              bool rising, OthersOf others_of)
{
    Stretch s;
    if (docs > 64) {
        const int tile = causal && rising ? (rows >> shift) + docs - 1 - rank : rank;
        s.doc = last_document(docs, [&](int d) { return (offset_at(offsets, d, rows) >> shift) + d <= tile; });
        s.begin = offset_at(offsets, s.doc, rows);
        s.end = max(offset_at(offsets, s.doc + 1, rows), s.begin);
        const int number = tile - ((s.begin >> shift) + s.doc);  // below 0: rows before the first document
        s.first = number >= 0 ? s.begin + (number << shift) : s.end;
        const Others others = others_of(s.doc);
        s.other_begin = others.begin;
        s.others = others.count;
        return s;
    }
    const int d = (int)(threadIdx.x & 63), my_doc = min(d, docs - 1);
    const Others others = others_of(my_doc);
    const int begin = offset_at(offsets, my_doc, rows), end = d < docs ? max(offset_at(offsets, my_doc + 1, rows), begin) : begin;
    const int up = (1 << shift) - 1, count = (end - begin + up) >> shift;
    int number;  // of the stretch in its document
    if (docs == 1) {
        s.doc = 0;
        number = causal && rising ? count - 1 - rank : rank;
        if (rank >= count) number = count;
    } else {
        const int least = !causal ? (others.count + up) >> shift : rising ? max(others.count - (end - begin), 0) >> shift : 0;
        // stretches of this document with more work than w
        auto above = [&](int w) { return causal ? min(max(least + count - 1 - w, 0), count) : least > w ? count : 0; };
        int bits = 0, top = 0;
        while (__ballot(count >> bits) != 0) ++bits;
        while (__ballot((causal ? least + count : least) >> top) != 0) ++top;
        int low = -1, high = 1 << top;  // fewer than or as many as `rank` have more work than `high`, more have more than `low`
        if (lanes_sum(count, bits) <= rank) {
            s.doc = s.begin = s.end = s.first = s.other_begin = s.others = 0;
            return s;
        }
        while (high - low > 1) {
            const int middle = low + (high - low) / 2;
            if (lanes_sum(above(middle), bits) <= rank) high = middle;
            else low = middle;
        }
        const int equal = above(high - 1) - above(high), nth = rank - lanes_sum(above(high), bits), before = lanes_before(equal, bits);
        s.doc = __builtin_ctzll(__ballot(before <= nth && nth < before + equal));
        number = !causal ? nth - before : rising ? high - least : count - 1 - (high - least);
    }
    s.doc = __builtin_amdgcn_readfirstlane(s.doc);
    s.begin = __builtin_amdgcn_readlane(begin, s.doc);
    s.end = __builtin_amdgcn_readlane(end, s.doc);
    s.first = s.begin + (__builtin_amdgcn_readlane(number, s.doc) << shift);
    s.other_begin = __builtin_amdgcn_readlane(others.begin, s.doc);
    s.others = __builtin_amdgcn_readlane(others.count, s.doc);
    return s;
}

// Rows [begin, end) of a document in the other tensor.
__device__ __forceinline__ Others rows_in(const int *offsets, int doc, int rows)
{
    const int begin = offset_at(offsets, doc, rows);
    return Others{begin, max(offset_at(offsets, doc + 1, rows) - begin, 0)};
}

// Rows of one head that no document covers (documents follow each other, so they lie before the first and
// behind the last) of a dense tensor [rows][heads][D] become zero; by one block.
template <int D, class Also>
__device__ __forceinline__ void clear_rows(uint16_t *tensor, const int *offsets, int docs, int rows, int heads, int head, Also also)
{
    const int first = offset_at(offsets, 0, rows), last = max(offset_at(offsets, docs, rows), first);
    const int count = first + rows - last;
    for (long long i = threadIdx.x; i < (long long)count * (D / 4); i += kThreads) {
        const int n = (int)(i / (D / 4)), row = n < first ? n : n - first + last;
        *reinterpret_cast<u32x2 *>(tensor + ((long long)row * heads + head) * D + 4 * (i % (D / 4))) = u32x2{0, 0};
        if (i % (D / 4) == 0) also(row);
    }
}

}  // namespace ktanh_cap
