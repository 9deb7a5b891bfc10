// libktanh: gradients of the capped attention.
//
//   P = e^(y - lse),  dP = dO V^T,  delta = rowsum(dO * O),  dS = P (dP - delta) (1 - t^2),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// 1 - t^2 is the library's derivative identity of TanH at K-TanH's value.  Scores are formed again in two kernels, each
// summing what it owns in registers, so that no gradient is added to by two blocks and results do not depend on their order:
//   cap_dq_kernel    128 queries of a head, over their keys; also forms delta
//   cap_dkdv_kernel  128 keys of a key/value head, over the queries of the heads that share them
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
    int parts;
};

constexpr int kTile = 32;  // rows of a tile in LDS

// Of the rows that this wavefront loaded, those behind the last become zero in both tiles: what they hold is not the document's.
template <int D>
__device__ __forceinline__ void clear_behind(char *a_tile, char *b_tile, int wave, int there)
{
#pragma unroll
    for (int n = 0; n < Stream<D>::kShare; ++n) {
        const int g = wave * Stream<D>::kShare + n, at = Keys32<D>::stretch_at(g) + 16 * (threadIdx.x & 63);
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

// An accumulator [dim][32 rows] as a lane's row of a dense tensor, times `by`.
template <int D>
__device__ __forceinline__ void store_row(uint16_t *row, const f32x16 (&acc)[D / 32], float by)
{
    row += 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x2 *>(row + 32 * c + 8 * i) =
                u32x2{pack2(acc[c][4 * i] * by, acc[c][4 * i + 1] * by), pack2(acc[c][4 * i + 2] * by, acc[c][4 * i + 3] * by)};
}

template <int D>
__device__ __forceinline__ void store_row(float *row, const f32x16 (&acc)[D / 32], float by)
{
    row += 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4 *>(row + 32 * c + 8 * i) =
                f32x4{acc[c][4 * i] * by, acc[c][4 * i + 1] * by, acc[c][4 * i + 2] * by, acc[c][4 * i + 3] * by};
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void cap_dq_kernel(BackwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        char k[2][kBytes], v[2][kBytes];
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    const unsigned total = a.tiles * (unsigned)a.s.heads;
    if (blockIdx.x >= padded(total)) {
        clear_rows<D>(a.dq, a.q_offsets, a.s.docs, a.s.q_rows, a.s.heads, (int)(blockIdx.x - padded(total)), [](int) {});
        return;
    }
    const unsigned place = place_of_block(blockIdx.x, total);
    if (place >= total) return;
    const int in_group = place % a.s.group;
    const int kv_head = place / a.s.group / a.tiles, head = kv_head * a.s.group + in_group;
    auto keys_of = [&](int doc) { return rows_in(a.k_offsets, doc, a.s.k_rows); };
    const Stretch at = stretch_of((int)(place / a.s.group % a.tiles), a.q_offsets, a.s.docs, a.s.q_rows, a.s.causal, true, keys_of);
    if (at.first >= at.end) return;
    const int k_begin = at.other_begin, n_keys = at.others;
    Rows keys = of_head(a.s.k, kv_head), values = of_head(a.s.v, kv_head);
    keys.at += k_begin * keys.row;
    values.at += k_begin * values.row;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shift = n_keys - (at.end - at.begin);
    const int row0 = at.first + 32 * wave, row = row0 + (lane & 31), row_there = min(row, at.end - 1);
    const int place0 = row0 - at.begin + shift, my_place = row - at.begin + shift;
    const int block_first = at.first - at.begin + shift;
    const int block_last = min(at.first + kRows, at.end) - 1 - at.begin + shift;
    const int key_end = a.s.causal ? min(n_keys, block_last + 1) : n_keys;
    const int key_begin = a.s.window > 0 ? max(0, block_first - a.s.window + 1) & ~(kTile - 1) : 0;
    const int first_seen = a.s.window > 0 ? max(0, my_place - a.s.window + 1) : 0, last_seen = a.s.causal ? min(n_keys, my_place + 1) : n_keys;
    // What is loaded first is what takes longest; the lines are there behind the first tile's barrier.
    Stream<D> stream(keys.at, keys.row, values.at, values.row, n_keys - 1, wave, key_begin);
    if (key_begin < key_end) stream.next(key_begin, shared.k[0], shared.v[0]);
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
    const long long sum_at = (long long)head * a.s.q_rows + row;
    if (row < at.end && lane < 32) a.delta[sum_at] = delta;
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
        if (j0 + kTile > n_keys) clear_behind<D>(k_tile, v_tile, wave, n_keys - j0);
        // Behind this barrier the tile is complete and all are done with the one before, whose place the next one takes.
        __syncthreads();
        if (j0 + kTile < key_end) stream.next(j0 + kTile, next_k, next_v);
        if (idle || (!whole && ((a.s.causal && j0 > place0 + 31) || (a.s.window > 0 && j0 + kTile - 1 <= place0 - a.s.window)))) return;
        f32x16 s = f32x16{0}, dp = f32x16{0};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s = mfma(Keys32<D>::rows(k_tile, k), q[k], s);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) dp = mfma(Keys32<D>::rows(v_tile, k), d_o[k], dp);
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float t = capped(s[r] * a.s.to_x, lines);
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(t, unit, -lse2));
            ds[r] = p * (dp[r] - delta) * __builtin_fmaf(-t, t, 1.0f);
        }
        if (!whole) keep(ds, Span(first_seen, last_seen, j0));
        const bf16x8 shares[2] = {pack8(ds), pack8(ds + 8)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) dq[c] = mfma(Keys32<D>::columns(k_tile, i, c), shares[i], dq[c]);
    };
    for (int j0 = key_begin; j0 < key_end; j0 += 2 * kTile) {
        step(j0, shared.k[0], shared.v[0], shared.k[1], shared.v[1]);
        if (j0 + kTile < key_end) step(j0 + kTile, shared.k[1], shared.v[1], shared.k[0], shared.v[0]);
    }
    if (row < at.end) store_row<D>(a.dq + ((long long)row * a.s.heads + head) * D, dq, a.s.scale);
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void cap_dkdv_kernel(BackwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        char q[2][kBytes], d_o[2][kBytes];
        char v[kWaves][kBytes];   // each wavefront's 32 rows of values: registers for them would leave one wavefront to a SIMD
        float sums[2][2 * kTile];  // lse * log2 e | delta of a tile's rows
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    const unsigned total = a.tiles * (unsigned)(a.s.kv_heads * a.parts);
    if (blockIdx.x >= padded(total)) {  // where there are parts, the kernel that joins them clears
        const int head = (int)(blockIdx.x - padded(total));
        clear_rows<D>(a.dk, a.k_offsets, a.s.docs, a.s.k_rows, a.s.kv_heads, head, [](int) {});
        clear_rows<D>(a.dv, a.k_offsets, a.s.docs, a.s.k_rows, a.s.kv_heads, head, [](int) {});
        return;
    }
    const unsigned place = place_of_block(blockIdx.x, total);
    if (place >= total) return;
    const int part = place % a.parts, kv_head = place / a.parts / a.tiles;
    auto queries_of = [&](int doc) { return rows_in(a.q_offsets, doc, a.s.q_rows); };
    const Stretch at = stretch_of((int)(place / a.parts % a.tiles), a.k_offsets, a.s.docs, a.s.k_rows, a.s.causal, false, queries_of);
    if (at.first >= at.end) return;
    const int q_begin = at.other_begin, n_queries = at.others;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shift = (at.end - at.begin) - n_queries;  // query i is key i + shift
    const int row0 = at.first + 32 * wave, row = row0 + (lane & 31), row_there = min(row, at.end - 1);
    const int key0 = row0 - at.begin, key = row_there - at.begin;
    const int block_first = at.first - at.begin, block_last = min(at.first + kRows, at.end) - 1 - at.begin;
    // queries that see some key of the block
    const int from = a.s.causal ? max(0, block_first - shift) & ~(kTile - 1) : 0;
    const int to = a.s.window > 0 ? min((long long)n_queries, max(0ll, (long long)block_last - shift + a.s.window)) : n_queries;
    // queries that see this lane's key
    const int first_seen = a.s.causal ? max(0, key - shift) : 0;
    const int last_seen = a.s.window > 0 ? (int)min((long long)n_queries, max(0ll, (long long)key - shift + a.s.window)) : n_queries;
    const float unit = a.s.cap * kLog2e;

    bf16x8 k[kSteps];
    load_row<D>(k, of_head(a.s.k, kv_head), row_there);
    {
        const Rows v = of_head(a.s.v, kv_head);
#pragma unroll
        for (int g = 0; g < Keys32<D>::kStretches; ++g)
            load_direct(v.at + min(row0 + Keys32<D>::row_of_lane(g), at.end - 1) * v.row + 8 * Keys32<D>::chunk_of_lane(), shared.v[wave] + Keys32<D>::stretch_at(g));
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
    Stream<D> stream(q.at + first_query * q.row, q.row, d_o.at + first_query * d_o.row, d_o.row, n_queries - 1, wave, from);
    // a wavefront brings 16 of a tile's 64 sums
    const float *sum_from = ((wave & 1) == 0 ? a.lse : a.delta) + (long long)head0 * a.s.q_rows + q_begin;
    float next_sum = 0.0f;
    int left = from < to ? heads : 0, next_query = from;  // heads not loaded to their end, and where
    auto load = [&](char *q_tile, char *do_tile) {  // the next tile: heads one behind the other
        stream.next(next_query, q_tile, do_tile);
        next_sum = sum_from[min(next_query + 16 * (wave >> 1) + (lane & 15), n_queries - 1)];
        next_query += kTile;
        if (next_query >= to) {
            next_query = from;
            --left;
            stream.a_rows += q.head;
            stream.b_rows += d_o.head;
            stream.start(from);
            sum_from += a.s.q_rows;
        }
    };
    auto step = [&](int i0, const char *__restrict__ v_tile, char *__restrict__ q_tile, char *__restrict__ do_tile, float *__restrict__ sums, char *__restrict__ next_q,
                    char *__restrict__ next_do) {
        wait_for_loads();
        if (i0 + kTile > n_queries) clear_behind<D>(q_tile, do_tile, wave, n_queries - i0);
        if (lane < 16) sums[(wave & 1) * kTile + 16 * (wave >> 1) + lane] = (wave & 1) == 0 ? next_sum * kLog2e : next_sum;
        __syncthreads();
        if (left > 0) load(next_q, next_do);
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
    const int tiles = left * ((to - from + kTile - 1) / kTile);
    if (left > 0) load(shared.q[0], shared.d_o[0]);
    spread_lines(lines, pack, 1.0f);  // there behind the first tile's barrier
    int i0 = from;
    for (int n = 0; n < tiles; n += 2) {
        step(i0, shared.v[wave], shared.q[0], shared.d_o[0], shared.sums[0], shared.q[1], shared.d_o[1]);
        i0 = i0 + kTile < to ? i0 + kTile : from;
        if (n + 1 == tiles) break;
        step(i0, shared.v[wave], shared.q[1], shared.d_o[1], shared.sums[1], shared.q[0], shared.d_o[0]);
        i0 = i0 + kTile < to ? i0 + kTile : from;
    }
    if (row >= at.end) return;
    const long long to_row = ((long long)row * a.s.kv_heads + kv_head) * D;
    if (a.dk_parts == nullptr) {
        store_row<D>(a.dk + to_row, dk, a.s.scale);
        store_row<D>(a.dv + to_row, dv, 1.0f);
    } else {
        const long long part_at = (long long)part * a.s.k_rows * a.s.kv_heads * D + to_row;
        store_row<D>(a.dk_parts + part_at, dk, a.s.scale);
        store_row<D>(a.dv_parts + part_at, dv, 1.0f);
    }
}

// The parts of shared heads added up in their order, zero for rows of no document: 8 values of dk or dv for each thread.
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

// Blocks over 128 keys of a key/value head, all heads of its group one behind the other, where those blocks are many; else one head each.
int parts_of(const kcap_shape_t &s)
{
    const size_t group = s.heads / s.kv_heads;
    return (s.k_rows / kRows + s.docs) * s.kv_heads >= 2048 ? 1 : (int)group;
}

size_t delta_bytes(const kcap_shape_t &s) { return (s.heads * s.q_rows * 4 + 127) / 128 * 128; }

template <class Lut>
ktanh_status_t backward(const kcap_shape_t *shape, const uint16_t *d_o, size_t do_row, size_t do_head, const uint16_t *q, const uint16_t *k,
                        const uint16_t *v, const uint16_t *o, const uint16_t *rest, const float *lse, const int32_t *q_offsets, const int32_t *k_offsets, uint16_t *dq,
                        uint16_t *dk, uint16_t *dv, void *workspace, const Lut *lut, ktanh_stream_t stream)
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
    if (do_row % 8 != 0 || do_head % 8 != 0 || !aligned16(d_o) || !aligned16(o) || !aligned16(rest) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(workspace) ||
        reinterpret_cast<uintptr_t>(lse) % 4 != 0 || reinterpret_cast<uintptr_t>(q_offsets) % 4 != 0 || reinterpret_cast<uintptr_t>(k_offsets) % 4 != 0)
        return KT_ERR_ALIGN;
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
    a.parts = parts_of(*shape);
    const long long each = (long long)a.s.k_rows * a.s.kv_heads * dim;
    if (a.parts > 1) {
        a.dk_parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + delta_bytes(*shape));
        a.dv_parts = a.dk_parts + a.parts * each;
    }
    const unsigned long long q_tiles = shape->q_rows / kRows + shape->docs, k_tiles = shape->k_rows / kRows + shape->docs;
    const unsigned long long q_blocks = (q_tiles * a.s.heads + 7) / 8 * 8 + a.s.heads;
    const unsigned long long k_blocks = (k_tiles * a.s.kv_heads * a.parts + 7) / 8 * 8 + (a.parts == 1 ? a.s.kv_heads : 0);
    const unsigned long long joins = (unsigned long long)(each + kThreads * 8 - 1) / (kThreads * 8);
    if (q_blocks > kMaxBlocks || k_blocks > kMaxBlocks || joins > kMaxBlocks) return KT_ERR_SHAPE;

    const auto on = static_cast<hipStream_t>(stream);
    if (queries) {
        a.tiles = (unsigned)q_tiles;
        auto *kernel = dim == 64 ? &cap_dq_kernel<64> : &cap_dq_kernel<128>;
        kernel<<<dim3((unsigned)q_blocks), dim3(kThreads), 0, on>>>(a, pack);
        if ((st = launched()) != KT_OK) return st;
    }
    if (!keys) return KT_OK;
    a.tiles = (unsigned)k_tiles;
    auto *kernel = dim == 64 ? &cap_dkdv_kernel<64> : &cap_dkdv_kernel<128>;
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
    const size_t parts = (size_t)parts_of(*shape);
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
