// libktanh: gradients of the capped attention.
//
//   P = e^(y - lse),  dP = dO V^T,  delta = rowsum(dO * O),  dS = P (dP - delta) (1 - t^2),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// 1 - t^2 is the library's derivative identity of TanH at K-TanH's value.  Scores are formed again in two
// kernels, each summing what it owns in registers, so that no gradient is added to by two blocks and results do
// not depend on their order:
//   cap_dq_kernel    32 queries for each wavefront (or for all), over their keys; also forms delta
//   cap_dkdv_kernel  32 keys for each wavefront (or for all) of a key/value head, over the queries of the heads that share them
//
// P and dS are rounded to BFloat16 where they become operands: dq and dk are then off by 0.0025 of their norm,
// of which 0.0017 is the rounding of the results themselves.  A second term would double the instructions of
// three of the seven products.
//
// What bounds it: six documents of 8192 tokens in all, 32 heads of 128 on 8, causal: dq 320 us, dk and dv 455
// in blocks of 32 rows (medians of ten passes from an idle card; the least 290 and 409, in blocks of 128 then
// 380 and 46 to join four parts).  A tile of 32 x 32 takes 24 (32) matrix and 220 (235) vector instructions, in
// 197 (247) registers, so that two wavefronts share a SIMD: its matrix unit is busy 34 (33) % of the time and
// its vector unit 46 (38) %, and the rest is waiting for one another and for LDS, which is busy 35 (43) %.  Two
// tiles behind one barrier, or all operands of a tile read ahead, changed less than 2 %.
#include "ktanh_cap_args.h"

using namespace ktanh_cap;

namespace {

struct BackwardArgs {
    CapShape s;
    const int *q_offsets, *k_offsets;
    Rows o, rest, d_o;          // dense o and rest, d_o with any strides
    const float *lse;           // [heads][q_rows]
    float *delta;               // [heads][q_rows]
    uint16_t *dq, *dk, *dv;     // dense
    float *dk_parts, *dv_parts; // [parts][k_rows][kv_heads][dim], NULL where one block sums all heads of a group
    unsigned tiles;
    int shift;  // of the rows of a stretch
    int parts;
};

constexpr int kTile = 32;  // rows of a tile in LDS

// Of the rows that this wavefront loaded, those behind the last become zero in both tiles: what they hold is
// not the document's.
template <int D, int LOADERS>
__device__ __forceinline__ void clear_behind(char *a_tile, char *b_tile, int wave, int there)
{
    constexpr int kShare = Keys32<D>::kStretches / LOADERS;
#pragma unroll
    for (int n = 0; n < kShare; ++n) {
        const int g = wave * kShare + n, at = Keys32<D>::stretch_at(g) + 16 * (threadIdx.x & 63);
        if (Keys32<D>::row_of_lane(g) >= there)
            *reinterpret_cast<u32x4 *>(a_tile + at) = *reinterpret_cast<u32x4 *>(b_tile + at) = u32x4{0, 0, 0, 0};
    }
}

__device__ __forceinline__ Rows of_head(const Rows &t, int head) { return Rows{t.at + head * t.head, t.row, t.head}; }

// A lane's share of one row as second operands: values 16 k + 8 (lane / 32) .. + 7.
template <int D>
__device__ __forceinline__ void load_row(bf16x8 (&to)[D / 16], const Rows &from, int row)
{
    const uint16_t *at = from.at + row * from.row + 8 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) to[k] = *reinterpret_cast<const bf16x8 *>(at + 16 * k);
}

// Values 4 i .. 4 i + 3 of every 32 of an accumulator [dim][32 rows], a lane's row.
__device__ __forceinline__ f32x4 quad(const f32x16 *acc, int i)
{
    const f32x16 &c = acc[i / 4];
    return f32x4{c[4 * (i % 4)], c[4 * (i % 4) + 1], c[4 * (i % 4) + 2], c[4 * (i % 4) + 3]};
}

__device__ __forceinline__ void store4(uint16_t *to, f32x4 v)
{
    *reinterpret_cast<u32x2 *>(to) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}
__device__ __forceinline__ void store4(float *to, f32x4 v) { *reinterpret_cast<f32x4 *>(to) = v; }

// An accumulator as the wavefront's rows (first `to`, `next` apart, `there` of them) of a dense tensor, times
// `by`.  SPLIT: the sum of all wavefronts' in their order, a fourth of the columns by each; by all threads, and
// `sums` is free once more behind the next barrier.  BY_ROWS: by way of `tile`, LDS that nobody reads any more
// but the sums' readers.
template <int D, bool SPLIT, bool BY_ROWS, class T, class Sums>
__device__ __forceinline__ void store_acc(T *to, long long next, int there, const f32x16 (&acc)[D / 32], float by, Sums &sums, char *tile)
{
    constexpr int kQuads = D / 8, kMine = SPLIT ? kQuads / kWaves : kQuads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = SPLIT ? wave * kMine : 0;
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) sums[wave][i][lane] = quad(acc, i);
        __syncthreads();
    }
    f32x4 v[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if constexpr (SPLIT) {
            v[i] = sums[0][first + i][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v[i] += sums[w][first + i][lane];
        } else {
            v[i] = quad(acc, i);
        }
    }
    if constexpr (BY_ROWS && sizeof(T) == 2) {
        if constexpr (SPLIT) __syncthreads();
        store_rows<D, SPLIT>(tile, to, next, there, [&](int i) {
            const f32x4 w = v[i] * by;
            return u32x2{pack2(w[0], w[1]), pack2(w[2], w[3])};
        });
    } else if constexpr (BY_ROWS && !SPLIT) {
        store_rows_wide<D>(tile, to, next, there, [&](int i) { return v[i] * by; });
    } else {
        to += (lane & 31) * next + 4 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if ((lane & 31) < there) store4(to + 8 * (first + i), v[i] * by);
    }
}

template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void cap_dq_kernel(BackwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    constexpr int kLoaders = SPLIT ? 1 : kWaves, kTiles = SPLIT ? kWaves : 1, kStep = kTile * kTiles;  // a tile's wavefronts; tiles at once
    constexpr int kBuffers = SPLIT ? 1 : 2;  // two blocks to a compute unit hide each other's loads
    struct Tiles {
        char k[kBuffers][kBytes], v[kBuffers][kBytes];
    };
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        union {
            Tiles tiles[kTiles];
            f32x4 sums[SPLIT ? kWaves : 1][SPLIT ? D / 8 : 1][64];  // of each wavefront, at the end
        };
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    // heads of a block, as a power of two; blocks that share keys
    const int together = SPLIT ? 0 : 7 - a.shift, members = a.s.group >> together;
    const unsigned blocks = (unsigned)unit_blocks(a.tiles, a.s.kv_heads, 1, members);
    if (blockIdx.x >= blocks) {
        clear_rows<D>(a.dq, a.q_offsets, a.s.docs, a.s.q_rows, a.s.heads, (int)(blockIdx.x - blocks), [](int) {});
        return;
    }
    Unit work;
    if (!unit_of_block(blockIdx.x, a.tiles, a.s.kv_heads, 1, members, &work)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv_head = work.kv_head, head = kv_head * a.s.group + (work.member << together) + (wave & ((1 << together) - 1));
    auto keys_of = [&](int doc) { return rows_in(a.k_offsets, doc, a.s.k_rows); };
    const Stretch at = stretch_of(a.shift, work.rank, a.q_offsets, a.s.docs, a.s.q_rows, a.s.causal, true, keys_of);
    if (at.first >= at.end) return;
    const int k_begin = at.other_begin, n_keys = at.others;
    Rows keys = of_head(a.s.k, kv_head), values = of_head(a.s.v, kv_head);
    keys.at += k_begin * keys.row;
    values.at += k_begin * values.row;

    const int shift = n_keys - (at.end - at.begin);
    const int row0 = at.first + (SPLIT ? 0 : 32 * (wave >> together)), row = row0 + (lane & 31), row_there = min(row, at.end - 1);
    const int place0 = row0 - at.begin + shift, my_place = row - at.begin + shift;
    const int block_first = at.first - at.begin + shift;
    const int block_last = min(at.first + (1 << a.shift), at.end) - 1 - at.begin + shift;
    const int key_end = a.s.causal ? min(n_keys, block_last + 1) : n_keys;
    const int key_begin = a.s.window > 0 ? max(0, block_first - a.s.window + 1) & ~(kTile - 1) : 0;
    const int first_seen = a.s.window > 0 ? max(0, my_place - a.s.window + 1) : 0, last_seen = a.s.causal ? min(n_keys, my_place + 1) : n_keys;
    // What is loaded first is what takes longest; the lines are there behind the first tile's barrier.
    const int loader = SPLIT ? 0 : wave, j_begin = key_begin + (SPLIT ? kTile * wave : 0);  // this wavefront's first tile
    Tiles &tiles = shared.tiles[SPLIT ? wave : 0];
    Stream<D, kLoaders, kStep> stream(keys.at, keys.row, values.at, values.row, n_keys - 1, loader, j_begin);
    if (j_begin < key_end) stream.next(j_begin, tiles.k[0], tiles.v[0]);
    bf16x8 q[kSteps], d_o[kSteps];
    load_row<D>(q, of_head(a.s.q, head), row_there);
    load_row<D>(d_o, of_head(a.d_o, head), row_there);
    float delta = 0.0f;
    {
        bf16x8 o[kSteps], rest[kSteps];
        load_row<D>(o, of_head(a.o, head), row_there);
        if (a.rest.at != nullptr) {
            load_row<D>(rest, of_head(a.rest, head), row_there);
        } else {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) rest[k] = bf16x8{};
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = __builtin_fmaf((float)d_o[k][i], (float)o[k][i] + (float)rest[k][i], delta);
        delta += __shfl_xor(delta, 32);
    }
    spread_lines(lines, pack, 1.0f);
    if constexpr (SPLIT) __syncthreads();
    const long long sum_at = (long long)head * a.s.q_rows + row;
    if (row < at.end && lane < 32 && (!SPLIT || wave == 0)) a.delta[sum_at] = delta;
    const float lse2 = a.lse[(long long)head * a.s.q_rows + row_there] * kLog2e;
    const float unit = a.s.cap * kLog2e;

    f32x16 dq[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) dq[c] = f32x16{0};
    // tiles that every query of the block sees whole
    const int whole_from = a.s.window > 0 ? block_last - a.s.window + 1 : 0, whole_to = a.s.causal ? min(n_keys, block_first + 1) : n_keys;
    const bool idle = row0 >= at.end;
    auto step = [&](int j0, char *__restrict__ k_tile, char *__restrict__ v_tile, char *__restrict__ next_k, char *__restrict__ next_v) {
        wait_for_loads();
        const bool whole = j0 >= whole_from && j0 + kTile <= whole_to;
        if (j0 + kTile > n_keys) clear_behind<D, kLoaders>(k_tile, v_tile, loader, n_keys - j0);
        // Behind this barrier the tile is complete and all are done with the one before, whose place the next
        // one takes.
        tile_complete<SPLIT>();
        if (!SPLIT && j0 + kStep < key_end) stream.next(j0 + kStep, next_k, next_v);
        if (idle) return;
        if (!whole && ((a.s.causal && j0 > place0 + 31) || (a.s.window > 0 && j0 + kTile - 1 <= place0 - a.s.window))) return;
        f32x16 s = f32x16{0}, dp = f32x16{0};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s = mfma(Keys32<D>::rows(k_tile, k), q[k], s);
        // the products of dP between the weights' instructions
        constexpr int kEach = 16 / kSteps;
        float x[16], ds[16];
        f32x2 line[16];
        bf16x8 v_rows = Keys32<D>::rows(v_tile, 0);
        auto weigh = [&](int r) {
            const float t = on_line(x[r], line[r]);
            ds[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(t, unit, -lse2)) * __builtin_fmaf(-t, t, 1.0f);
        };
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            dp = mfma(v_rows, d_o[k], dp);
            if (k + 1 < kSteps) v_rows = Keys32<D>::rows(v_tile, k + 1);
#pragma unroll
            for (int r = k * kEach; r < (k + 1) * kEach; ++r) {
                x[r] = s[r] * a.s.to_x;
                line[r] = line_of(x[r], lines);
                if (r >= kEach) weigh(r - kEach);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 16 - kEach; r < 16; ++r) weigh(r);
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] *= dp[r] - delta;
        if (!whole) keep(ds, Span(first_seen, last_seen, j0));
        const bf16x8 shares[2] = {pack8(ds), pack8(ds + 8)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) dq[c] = mfma(Keys32<D>::columns(k_tile, i, c), shares[i], dq[c]);
    };
    if constexpr (SPLIT) {
        for (int j0 = j_begin; j0 < key_end; j0 += kStep) {
            step(j0, tiles.k[0], tiles.v[0], nullptr, nullptr);
            tile_complete<SPLIT>();
            if (j0 + kStep < key_end) stream.next(j0 + kStep, tiles.k[0], tiles.v[0]);
        }
    } else {
        for (int j0 = j_begin; j0 < key_end; j0 += 2 * kStep) {
            step(j0, tiles.k[0], tiles.v[0], tiles.k[1], tiles.v[1]);
            if (j0 + kStep < key_end) step(j0 + kStep, tiles.k[1], tiles.v[1], tiles.k[0], tiles.v[0]);
        }
    }
    __syncthreads();
    // At 64 its registers would leave room for three wavefronts instead of four: 8192 tokens 748 us, 730 without.
    constexpr bool kByRows = SPLIT || D == 128;
    store_acc<D, SPLIT, kByRows>(a.dq + ((long long)row0 * a.s.heads + head) * D, (long long)a.s.heads * D, at.end - row0, dq,
                                 a.s.scale, shared.sums, shared.tiles[0].k[0] + (SPLIT ? 0 : wave * kBytes));
}

template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void cap_dkdv_kernel(BackwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    constexpr int kLoaders = SPLIT ? 1 : kWaves, kTiles = SPLIT ? kWaves : 1;  // a tile's wavefronts; tiles at once
    constexpr int kBuffers = SPLIT ? 1 : 2;  // two blocks to a compute unit hide each other's loads
    struct Tiles {
        char q[kBuffers][kBytes], d_o[kBuffers][kBytes];
        float sums[kBuffers][2 * kTile];  // lse * log2 e | delta of a tile's rows
    };
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        // the wavefronts' 32 rows of values: registers for them would leave one wavefront to a SIMD
        char v[SPLIT ? 1 : kWaves][kBytes];
        union {
            Tiles tiles[kTiles];
            f32x4 sums[SPLIT ? kWaves : 1][SPLIT ? D / 8 : 1][64];  // of each wavefront, at the end
        };
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    const unsigned blocks = (unsigned)unit_blocks(a.tiles, a.s.kv_heads, a.parts, 1);
    if (blockIdx.x >= blocks) {  // where there are parts, the kernel that joins them clears
        const int head = (int)(blockIdx.x - blocks);
        clear_rows<D>(a.dk, a.k_offsets, a.s.docs, a.s.k_rows, a.s.kv_heads, head, [](int) {});
        clear_rows<D>(a.dv, a.k_offsets, a.s.docs, a.s.k_rows, a.s.kv_heads, head, [](int) {});
        return;
    }
    Unit work;
    if (!unit_of_block(blockIdx.x, a.tiles, a.s.kv_heads, a.parts, 1, &work)) return;
    const int part = work.part, kv_head = work.kv_head;
    auto queries_of = [&](int doc) { return rows_in(a.q_offsets, doc, a.s.q_rows); };
    const Stretch at = stretch_of(a.shift, work.rank, a.k_offsets, a.s.docs, a.s.k_rows, a.s.causal, false, queries_of);
    if (at.first >= at.end) return;
    const int q_begin = at.other_begin, n_queries = at.others;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shift = (at.end - at.begin) - n_queries;  // query i is key i + shift
    const int row0 = at.first + (SPLIT ? 0 : 32 * wave), row = row0 + (lane & 31), row_there = min(row, at.end - 1);
    const int key0 = row0 - at.begin, key = row_there - at.begin;
    const int block_first = at.first - at.begin, block_last = min(at.first + (1 << a.shift), at.end) - 1 - at.begin;
    // queries that see some key of the block
    const int from = a.s.causal ? max(0, block_first - shift) & ~(kTile - 1) : 0;
    const int to = a.s.window > 0 ? min((long long)n_queries, max(0ll, (long long)block_last - shift + a.s.window)) : n_queries;
    // queries that see this lane's key
    const int first_seen = a.s.causal ? max(0, key - shift) : 0;
    const int last_seen = a.s.window > 0 ? (int)min((long long)n_queries, max(0ll, (long long)key - shift + a.s.window)) : n_queries;
    const float unit = a.s.cap * kLog2e;

    bf16x8 k[kSteps];
    load_row<D>(k, of_head(a.s.k, kv_head), row_there);
    char *values = shared.v[SPLIT ? 0 : wave];
    {
        const Rows v = of_head(a.s.v, kv_head);
        constexpr int kShare = Keys32<D>::kStretches / kTiles;
#pragma unroll
        for (int n = 0; n < kShare; ++n) {
            const int g = SPLIT ? wave * kShare + n : n;
            load_direct(v.at + min(row0 + Keys32<D>::row_of_lane(g), at.end - 1) * v.row + 8 * Keys32<D>::chunk_of_lane(),
                        values + Keys32<D>::stretch_at(g));
        }
    }
    f32x16 dk[kBlocks], dv[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) dk[c] = dv[c] = f32x16{0};

    const int heads = a.s.group / a.parts, head0 = kv_head * a.s.group + part * heads;
    // tiles of queries that all see every key of the block
    const int whole_from = a.s.causal ? block_last - shift : 0;
    const int whole_to = a.s.window > 0 ? (int)min((long long)n_queries, (long long)block_first - shift + a.s.window) : n_queries;
    const bool idle = row0 >= at.end;
    const long long first_query = q_begin;
    const Rows q = of_head(a.s.q, head0), d_o = of_head(a.d_o, head0);
    // Tiles of queries, heads one behind the other: this wavefront's first one and the one that it loads next.
    const int loader = SPLIT ? 0 : wave, each = max((to - from + kTile - 1) / kTile, 0), tiles = each * heads;  // of a head; of all
    struct Where {
        int tile, head, query;
    };
    auto advance = [&](Where &w) {
        w.tile += kTiles;
        w.query += kTiles * kTile;
        while (w.query >= to && w.tile < tiles) {
            w.query -= each * kTile;
            ++w.head;
        }
    };
    Where now{SPLIT ? wave : 0, 0, from + (SPLIT ? wave * kTile : 0)};
    now.tile -= kTiles;
    now.query -= kTiles * kTile;
    advance(now);
    Where next = now;
    Stream<D, kLoaders, kTiles * kTile> stream(q.at + first_query * q.row + next.head * q.head, q.row,
                                               d_o.at + first_query * d_o.row + next.head * d_o.head, d_o.row,
                                               n_queries - 1, loader, next.query);
    // Where wavefronts share a tile, one brings 16 of its 64 sums.
    const int sum_lanes = SPLIT ? 64 : 16, sum_row = SPLIT ? lane & 31 : 16 * (wave >> 1) + (lane & 15);
    const bool is_delta = SPLIT ? lane >= 32 : (wave & 1) != 0;
    const float *sum_from = (is_delta ? a.delta : a.lse) + (long long)head0 * a.s.q_rows + q_begin;
    float next_sum = 0.0f;
    auto load = [&](char *q_tile, char *do_tile) {
        stream.next(next.query, q_tile, do_tile);
        next_sum = sum_from[(long long)next.head * a.s.q_rows + min(next.query + sum_row, n_queries - 1)];
        const int head = next.head;
        advance(next);
        if (next.head != head) {
            stream.a_rows = q.at + first_query * q.row + next.head * q.head;
            stream.b_rows = d_o.at + first_query * d_o.row + next.head * d_o.head;
            stream.start(next.query);
        }
    };
    auto step = [&](int i0, const char *__restrict__ v_tile, char *__restrict__ q_tile, char *__restrict__ do_tile,
                    float *__restrict__ sums, char *__restrict__ next_q, char *__restrict__ next_do) {
        wait_for_loads();
        if (i0 + kTile > n_queries) clear_behind<D, kLoaders>(q_tile, do_tile, loader, n_queries - i0);
        if (lane < sum_lanes) sums[(is_delta ? kTile : 0) + sum_row] = is_delta ? next_sum : next_sum * kLog2e;
        tile_complete<SPLIT>();
        if (!SPLIT && next.tile < tiles) load(next_q, next_do);
        const int first = i0 + shift;  // the place of the tile's first query
        const bool whole = i0 >= whole_from && i0 + kTile <= whole_to;
        if (idle || (!whole && ((a.s.causal && first + kTile - 1 < key0) || (a.s.window > 0 && first > key0 + 31 + a.s.window - 1)))) return;
        // the scores' weights, their product, and only then dP: fewer registers at once
        f32x16 s = f32x16{0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = mfma(Keys32<D>::rows(q_tile, i), k[i], s);
        float p[16], slope[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 lse2 = *reinterpret_cast<const f32x4 *>(sums + 8 * g + 4 * (lane >> 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                const float t = capped(s[r] * a.s.to_x, lines);
                p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(t, unit, -lse2[e]));
                slope[r] = p[r] * __builtin_fmaf(-t, t, 1.0f);
            }
        }
        if (!whole) {
            const Span seen(first_seen, last_seen, i0);
            keep(p, seen);
            keep(slope, seen);
        }
        const bf16x8 weights[2] = {pack8(p), pack8(p + 8)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) dv[c] = mfma(Keys32<D>::columns(do_tile, i, c), weights[i], dv[c]);
        f32x16 dp = f32x16{0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) dp = mfma(Keys32<D>::rows(do_tile, i), Keys32<D>::rows(v_tile, i), dp);
        float ds[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 delta = *reinterpret_cast<const f32x4 *>(sums + kTile + 8 * g + 4 * (lane >> 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) ds[4 * g + e] = slope[4 * g + e] * (dp[4 * g + e] - delta[e]);
        }
        const bf16x8 shares[2] = {pack8(ds), pack8(ds + 8)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) dk[c] = mfma(Keys32<D>::columns(q_tile, i, c), shares[i], dk[c]);
    };
    Tiles &mine = shared.tiles[SPLIT ? wave : 0];
    if (next.tile < tiles) load(mine.q[0], mine.d_o[0]);
    spread_lines(lines, pack, 1.0f);  // there behind the first tile's barrier
    if constexpr (SPLIT) {
        wait_for_loads();
        __syncthreads();
    }
    while (now.tile < tiles) {
        if constexpr (SPLIT) {
            step(now.query, values, mine.q[0], mine.d_o[0], mine.sums[0], nullptr, nullptr);
            tile_complete<SPLIT>();
            if (next.tile < tiles) load(mine.q[0], mine.d_o[0]);
        } else {
            step(now.query, values, mine.q[0], mine.d_o[0], mine.sums[0], mine.q[1], mine.d_o[1]);
            advance(now);
            if (now.tile >= tiles) break;
            step(now.query, values, mine.q[1], mine.d_o[1], mine.sums[1], mine.q[0], mine.d_o[0]);
        }
        advance(now);
    }
    const long long first_at = ((long long)row0 * a.s.kv_heads + kv_head) * D, to_next = (long long)a.s.kv_heads * D;
    // The wavefront's rows of values are free behind its last tile.  A block that no query sees has had none,
    // and has not waited for those rows yet.
    if constexpr (SPLIT) {
        __syncthreads();
    } else {
        wait_for_loads();
        tile_complete<true>();
    }
    auto store = [&](auto *dk_to, auto *dv_to) {
        store_acc<D, SPLIT, true>(dk_to + first_at, to_next, at.end - row0, dk, a.s.scale, shared.sums, values);
        if constexpr (SPLIT) __syncthreads();
        store_acc<D, SPLIT, true>(dv_to + first_at, to_next, at.end - row0, dv, 1.0f, shared.sums, values);
    };
    if (a.dk_parts == nullptr) {
        store(a.dk, a.dv);
    } else {
        const long long part_at = (long long)part * a.s.k_rows * a.s.kv_heads * D;
        store(a.dk_parts + part_at, a.dv_parts + part_at);
    }
}

// The parts of shared heads added up in their order, zero for rows of no document: 8 values of dk or dv for
// each thread.
__global__ __launch_bounds__(kThreads) void cap_join_grads_kernel(BackwardArgs a, long long width)
{
    const long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * 8, each = a.s.k_rows * width;
    if (i >= each) return;
    const int first = offset_at(a.k_offsets, 0, a.s.k_rows), row = (int)(i / width);
    const float *from = blockIdx.y == 0 ? a.dk_parts : a.dv_parts;
    float v[8] = {};
    if (row >= first && row < offset_at(a.k_offsets, a.s.docs, a.s.k_rows))
        for (int p = 0; p < a.parts; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(from + p * each + i + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * h + e] += w[e];
            }
    *reinterpret_cast<bf16x8 *>((blockIdx.y == 0 ? a.dk : a.dv) + i) = pack8(v);
}

size_t delta_bytes(const kcap_shape_t &s) { return (s.heads * s.q_rows * 4 + 127) / 128 * 128; }

template <class Lut>
ktanh_status_t backward(const kcap_shape_t *shape, const uint16_t *d_o, size_t do_row, size_t do_head, const uint16_t *q,
                        const uint16_t *k, const uint16_t *v, const uint16_t *o, const uint16_t *rest, const float *lse,
                        const int32_t *q_offsets, const int32_t *k_offsets, uint16_t *dq, uint16_t *dk, uint16_t *dv,
                        void *workspace, const Lut *lut, ktanh_stream_t stream)
{
    if (shape == nullptr) return KT_ERR_NULL;
    if (shape->docs == 0 || (shape->q_rows == 0 && shape->k_rows == 0)) return KT_OK;
    const bool queries = shape->q_rows != 0, keys = shape->k_rows != 0;
    if (q_offsets == nullptr || k_offsets == nullptr || workspace == nullptr) return KT_ERR_NULL;
    if (queries && (d_o == nullptr || q == nullptr || o == nullptr || lse == nullptr || dq == nullptr)) return KT_ERR_NULL;
    if (keys && (k == nullptr || v == nullptr || dk == nullptr || dv == nullptr)) return KT_ERR_NULL;
    BackwardArgs a{};
    ktanh_status_t st = read_shape(shape, q, k, v, &a.s);
    if (st != KT_OK) return st;
    if (do_row % 8 != 0 || do_head % 8 != 0) return KT_ERR_ALIGN;
    for (const void *at : {(const void *)d_o, (const void *)o, (const void *)rest, (const void *)dq, (const void *)dk, (const void *)dv,
                           (const void *)workspace})
        if (!aligned16(at)) return KT_ERR_ALIGN;
    for (const void *at : {(const void *)lse, (const void *)q_offsets, (const void *)k_offsets})
        if (reinterpret_cast<uintptr_t>(at) % 4 != 0) return KT_ERR_ALIGN;
    if (do_row >= (size_t)1 << 24 || do_head >= (size_t)1 << 24) return KT_ERR_SHAPE;
    KtCapPack pack;
    if ((st = pack_lines(lut, &pack)) != KT_OK) return st;
    const long long dim = (long long)shape->dim;
    a.q_offsets = q_offsets;
    a.k_offsets = k_offsets;
    a.o = Rows{o, a.s.heads * dim, dim};
    a.rest = Rows{rest, a.s.heads * dim, dim};
    a.d_o = Rows{d_o, (long long)do_row, (long long)do_head};
    a.lse = lse;
    a.delta = static_cast<float *>(workspace);
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    const KeysPlan plan = keys_plan(*shape);
    a.parts = plan.parts;
    const long long each = (long long)a.s.k_rows * a.s.kv_heads * dim;
    if (a.parts > 1) {
        a.dk_parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + delta_bytes(*shape));
        a.dv_parts = a.dk_parts + a.parts * each;
    }
    const bool split_keys = split_tiles(*shape);
    const int q_shift = rows_shift(a.s, split_keys), k_shift = plan.split ? 5 : 7;
    const unsigned long long q_tiles = stretches(shape->q_rows, shape->docs, q_shift), k_tiles = stretches(shape->k_rows, shape->docs, k_shift);
    const unsigned long long q_blocks = unit_blocks(q_tiles, a.s.kv_heads, 1, split_keys ? a.s.group : a.s.group >> (7 - q_shift)) + a.s.heads;
    const unsigned long long k_blocks = unit_blocks(k_tiles, a.s.kv_heads, a.parts, 1) + (a.parts == 1 ? a.s.kv_heads : 0);
    const unsigned long long joins = (unsigned long long)(each + kThreads * 8 - 1) / (kThreads * 8);
    if (q_blocks > kMaxBlocks || k_blocks > kMaxBlocks || joins > kMaxBlocks) return KT_ERR_SHAPE;

    const auto on = static_cast<hipStream_t>(stream);
    if (queries) {
        a.tiles = (unsigned)q_tiles;
        a.shift = q_shift;
        auto *kernel = split_keys ? dim == 64 ? &cap_dq_kernel<64, true> : &cap_dq_kernel<128, true>
                                   : dim == 64 ? &cap_dq_kernel<64, false> : &cap_dq_kernel<128, false>;
        kernel<<<dim3((unsigned)q_blocks), dim3(kThreads), 0, on>>>(a, pack);
        if ((st = launched()) != KT_OK) return st;
    }
    if (!keys) return KT_OK;
    a.tiles = (unsigned)k_tiles;
    a.shift = k_shift;
    auto *kernel = plan.split ? dim == 64 ? &cap_dkdv_kernel<64, true> : &cap_dkdv_kernel<128, true>
                            : dim == 64 ? &cap_dkdv_kernel<64, false> : &cap_dkdv_kernel<128, false>;
    kernel<<<dim3((unsigned)k_blocks), dim3(kThreads), 0, on>>>(a, pack);
    if ((st = launched()) != KT_OK) return st;
    if (a.parts > 1) {
        cap_join_grads_kernel<<<dim3((unsigned)joins, 2), dim3(kThreads), 0, on>>>(a, a.s.kv_heads * dim);
        st = launched();
    }
    return st;
}

}  // namespace

extern "C" size_t kcap_attention_backward_workspace(const kcap_shape_t *shape)
{
    if (shape == nullptr || shape->kv_heads == 0 || shape->heads < shape->kv_heads || shape->heads > 65536 || shape->dim > 128 ||
        shape->q_rows > 1u << 30 || shape->k_rows > 1u << 30 || shape->docs > 1u << 30)
        return 0;
    const size_t parts = (size_t)keys_plan(*shape).parts;
    return delta_bytes(*shape) + 128 + (parts > 1 ? 2 * parts * shape->k_rows * shape->kv_heads * shape->dim * 4 : 0);
}

extern "C" ktanh_status_t kcap_attention_backward(const kcap_shape_t *shape, const uint16_t *d_o, size_t do_row, size_t do_head, const uint16_t *q,
                                                  const uint16_t *k, const uint16_t *v, const uint16_t *o, const uint16_t *rest, const float *lse, const int32_t *q_offsets,
                                                  const int32_t *k_offsets, uint16_t *dq, uint16_t *dk, uint16_t *dv, void *workspace,
                                                  const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return backward(shape, d_o, do_row, do_head, q, k, v, o, rest, lse, q_offsets, k_offsets, dq, dk, dv, workspace, lut, stream);
}

extern "C" ktanh_status_t kcap_attention64_backward(const kcap_shape_t *shape, const uint16_t *d_o, size_t do_row, size_t do_head, const uint16_t *q,
                                                    const uint16_t *k, const uint16_t *v, const uint16_t *o, const uint16_t *rest, const float *lse, const int32_t *q_offsets,
                                                    const int32_t *k_offsets, uint16_t *dq, uint16_t *dk, uint16_t *dv, void *workspace,
                                                    const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return backward(shape, d_o, do_row, do_head, q, k, v, o, rest, lse, q_offsets, k_offsets, dq, dk, dv, workspace, lut, stream);
}
