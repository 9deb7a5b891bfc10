// libktanh: attention with scores capped through K-TanH over many queries: packed documents, and pieces of
// prompts over a paged cache.
//
// A wavefront holds 32 queries in its registers, a block 128 of one document, or the same 64 or 32 of two or
// four heads that share keys, and goes once over the keys that they see in tiles of 32, double-buffered in LDS
// by direct loads.  Where blocks are few (SPLIT) all four wavefronts hold the same 32 queries of one head, each
// goes over every fourth tile with a place in LDS of its own, and the four sums are joined at the end.
//   S^T = K Q^T (keys x queries), p = e^(cap K(x)) in the accumulator, O^T += V^T P^T with P^T as it lies.
//
// What bounds it: 16384 tokens, 32 heads of 128, causal, take 2290 us, 960 TFLOP/s.  The matrix instructions
// alone take 1430 (1.54 PFLOP/s, what the card's clock allows a large product too), reading their operands from
// LDS 160 more, bringing the tiles 310, the cap, the exponentials and the sums, about 130 vector instructions
// for 16 matrix instructions, 430.  Three wavefronts share a SIMD because the tile's 32 keys and the direct
// loads leave 160 registers enough: with 64 keys to a tile, through registers, and two wavefronts 2736; with 32
// keys through registers 2620.
#include <type_traits>

#include "ktanh_cap_args.h"

using namespace ktanh_cap;

namespace {

// Rows j of keys and values.
template <bool PAGED>
struct Keys {
    const uint16_t *k, *v;  // of this document (or cache) and head
    long long k_row, v_row;
    int last;               // a row that is there, in place of all behind it
    // PAGED
    const int *pages;
    int shift, count;
    uint32_t k_page, v_page;

    __device__ __forceinline__ int page(int j) const
    {
        if constexpr (!PAGED) return 0;
        // a page that does not exist is read as one that does
        return min(max(pages[min(j, last) >> shift], 0), count - 1);
    }
    __device__ __forceinline__ const uint16_t *k_at(int j, int page) const
    {
        j = min(j, last);
        if constexpr (!PAGED) return k + j * k_row;
        return k + wide(page, k_page) + wide(j & ((1 << shift) - 1), (uint32_t)k_row);
    }
    __device__ __forceinline__ const uint16_t *v_at(int j, int page) const
    {
        j = min(j, last);
        if constexpr (!PAGED) return v + j * v_row;
        return v + wide(page, v_page) + wide(j & ((1 << shift) - 1), (uint32_t)v_row);
    }
};

constexpr int kKeys = 32;  // of a tile

// The same for keys and values in pages: the pages of a tile's rows are looked up one tile ahead.
template <int D, int LOADERS, int STEP>
struct PagedStream {
    typedef Keys32<D> Tile;
    static constexpr int kShare = Tile::kStretches / LOADERS;
    const Keys<true> &keys;
    const int wave;
    int pages[kShare];

    __device__ __forceinline__ PagedStream(const Keys<true> &keys, int wave, int at) : keys(keys), wave(wave) { start(at); }
    __device__ __forceinline__ void start(int at)
    {
#pragma unroll
        for (int n = 0; n < kShare; ++n) pages[n] = keys.page(at + Tile::row_of_lane(wave * kShare + n));
    }
    __device__ __forceinline__ void next(int at, char *k_tile, char *v_tile)
    {
        const int chunk = Tile::chunk_of_lane();
#pragma unroll
        for (int n = 0; n < kShare; ++n) {
            const int g = wave * kShare + n, row = Tile::row_of_lane(g);
            load_direct(keys.k_at(at + row, pages[n]) + 8 * chunk, k_tile + Tile::stretch_at(g));
            load_direct(keys.v_at(at + row, pages[n]) + 8 * chunk, v_tile + Tile::stretch_at(g));
        }
        start(at + STEP);
    }
};

template <int D, int LOADERS, int STEP>
__device__ __forceinline__ Stream<D, LOADERS, STEP> stream_of(const Keys<false> &keys, int wave, int at)
{
    return Stream<D, LOADERS, STEP>(keys.k, keys.k_row, keys.v, keys.v_row, keys.last, wave, at);
}
template <int D, int LOADERS, int STEP>
__device__ __forceinline__ PagedStream<D, LOADERS, STEP> stream_of(const Keys<true> &keys, int wave, int at)
{
    return PagedStream<D, LOADERS, STEP>(keys, wave, at);
}

// Infinities and NaN become zero.
__device__ __forceinline__ void take_special(u32x4 *v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = ((*v)[i] & 0x7F80u) == 0x7F80u, hi = ((*v)[i] & 0x7F800000u) == 0x7F800000u;
        (*v)[i] &= (lo ? 0xFFFF0000u : ~0u) & (hi ? 0xFFFFu : ~0u);
    }
}

// Of the rows that this wavefront loaded: values behind the last key become zero, as infinities and NaN do.
// Their weights are zero, and the product would not be.
template <int D, int LOADERS>
__device__ __forceinline__ void clean_values(char *v_tile, int wave, int there)
{
    constexpr int kShare = Keys32<D>::kStretches / LOADERS;
#pragma unroll
    for (int n = 0; n < kShare; ++n) {
        const int g = wave * kShare + n;
        u32x4 *at = reinterpret_cast<u32x4 *>(v_tile + Keys32<D>::stretch_at(g) + 16 * (threadIdx.x & 63));
        u32x4 w = *at;
        if (Keys32<D>::row_of_lane(g) >= there) w = u32x4{0, 0, 0, 0};
        else take_special(&w);
        *at = w;
    }
}

struct ForwardArgs {
    CapShape s;
    const int *q_offsets, *k_offsets;
    uint16_t *o, *rest;
    float *lse;
    CapPages p;
    unsigned tiles;
    int shift;  // of the rows of a stretch
    // PAGED: blocks of a stretch that share its keys, with sums [parts][q_rows][heads] and numerators
    // [parts][q_rows][heads][dim] in Float32
    int parts;
    float *part_sums, *part_values;
};

// SUMS: with log-sums.
template <int D, bool PAGED, bool SUMS, bool SPLIT>
__global__ __launch_bounds__(kThreads, SPLIT ? 2 : 3) void cap_forward_kernel(ForwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    constexpr int kLoaders = SPLIT ? 1 : kWaves, kTiles = SPLIT ? kWaves : 1, kStep = kKeys * kTiles;  // a tile's wavefronts; tiles at once
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
        float weights[SPLIT ? kWaves : 1][SPLIT ? 64 : 1];
        int special[kWaves];  // whether the wavefront has numerators that are not finite
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    // heads of a block, as a power of two; blocks that share keys
    const int together = SPLIT ? 0 : 7 - a.shift, members = a.s.group >> together;
    const unsigned blocks = (unsigned)unit_blocks(a.tiles, a.s.kv_heads, a.parts, members);
    if (blockIdx.x >= blocks) {
        const int head = (int)(blockIdx.x - blocks);
        clear_rows<D>(a.o, a.q_offsets, a.s.docs, a.s.q_rows, a.s.heads, head, [&](int row) {
            if (SUMS) a.lse[(long long)head * a.s.q_rows + row] = -__builtin_inff();
        });
        return;
    }
    Unit work;
    if (!unit_of_block(blockIdx.x, a.tiles, a.s.kv_heads, PAGED ? a.parts : 1, members, &work)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv_head = work.kv_head, part = work.part;
    const int head = kv_head * a.s.group + (work.member << together) + (wave & ((1 << together) - 1));
    auto keys_of = [&](int doc) {
        if constexpr (PAGED) return Others{0, keys_in_pages(a.p, doc)};
        else return rows_in(a.k_offsets, doc, a.s.k_rows);
    };
    const Stretch at = stretch_of(a.shift, work.rank, a.q_offsets, a.s.docs, a.s.q_rows, a.s.causal, true, keys_of);
    if (at.first >= at.end) return;

    Keys<PAGED> keys;
    const int n_keys = at.others;
    if constexpr (PAGED) {
        keys.k = a.s.k.at + kv_head * a.s.k.head;
        keys.v = a.s.v.at + kv_head * a.s.v.head;
        keys.pages = a.p.pages + at.doc * a.p.row;
        keys.shift = a.p.shift;
        keys.count = a.p.count;
        keys.k_page = a.p.k_page;
        keys.v_page = a.p.v_page;
    } else {
        keys.k = a.s.k.at + at.other_begin * a.s.k.row + kv_head * a.s.k.head;
        keys.v = a.s.v.at + at.other_begin * a.s.v.row + kv_head * a.s.v.head;
    }
    keys.k_row = a.s.k.row;
    keys.v_row = a.s.v.row;
    keys.last = max(n_keys - 1, 0);  // a sequence without keys looks up its first page, and reads none

    const int shift = n_keys - (at.end - at.begin);            // query i is key i + shift
    const int row0 = at.first + (SPLIT ? 0 : 32 * (wave >> together));       // this wavefront's first query
    const int row = row0 + (lane & 31);                        // this lane's
    const int place0 = row0 - at.begin + shift, my_place = row - at.begin + shift;
    const int block_first = at.first - at.begin + shift;
    const int block_last = min(at.first + (1 << a.shift), at.end) - 1 - at.begin + shift;
    int key_end = a.s.causal ? min(n_keys, block_last + 1) : n_keys;
    int key_begin = a.s.window > 0 ? max(0, block_first - a.s.window + 1) & ~(kKeys - 1) : 0;
    if (PAGED && a.parts > 1) {  // this block's share of them, in whole tiles
        const int share = (max(key_end - key_begin, 0) + a.parts * kKeys - 1) / (a.parts * kKeys) * kKeys;
        key_begin = min(key_begin + part * share, max(key_end, key_begin));
        key_end = min(key_end, key_begin + share);
    }

    // What is loaded first is what takes longest; the lines are there behind the first tile's barrier.
    const int loader = SPLIT ? 0 : wave, j_begin = key_begin + (SPLIT ? kKeys * wave : 0);  // this wavefront's first tile
    Tiles &tiles = shared.tiles[SPLIT ? wave : 0];
    auto stream = stream_of<D, kLoaders, kStep>(keys, loader, j_begin);
    if (j_begin < key_end) stream.next(j_begin, tiles.k[0], tiles.v[0]);
    bf16x8 q[kSteps];
    {
        const uint16_t *from = a.s.q.at + min(row, at.end - 1) * a.s.q.row + head * a.s.q.head + 8 * (lane >> 5);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) q[k] = *reinterpret_cast<const bf16x8 *>(from + 16 * k);
    }
    f32x16 o[kBlocks];
    spread_lines(lines, pack, a.s.cap * kLog2e);
    if constexpr (SPLIT) __syncthreads();
    float sum, rounded_sum;  // of the weights, and of the weights as the product has them

    // Tiles that every query of the block sees whole.  In the others a weight may be zero because its key is
    // hidden, and the product with an infinite or NaN value would not be: a block whose numerators are not all
    // finite goes over its keys once more, and then takes such values out of these tiles and adds them behind
    // the loop where they are seen.  (Looking for them in every such tile took 4 to 7 % of the time over
    // documents of some hundred tokens and windows.)
    const int whole_from = a.s.window > 0 ? block_last - a.s.window + 1 : 0, whole_to = a.s.causal ? min(n_keys, block_first + 1) : n_keys;
    auto whole = [&](int j0) { return j0 >= whole_from && j0 + kKeys <= whole_to; };
    const int first_seen = a.s.window > 0 ? max(0, my_place - a.s.window + 1) : 0, last_seen = a.s.causal ? min(n_keys, my_place + 1) : n_keys;
    const bool idle = row0 >= at.end;
    auto add_tile = [&](int j0, const char *__restrict__ k_tile, const char *__restrict__ v_tile, bool masked) {
        f32x16 s = f32x16{0};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s = mfma(Keys32<D>::rows(k_tile, k), q[k], s);
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(capped(s[r] * a.s.to_x, lines));
        if (masked) keep(p, Span(first_seen, last_seen, j0));
        if constexpr (SUMS) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += p[r];
        }
        const bf16x8 weights[2] = {pack8(p, &rounded_sum), pack8(p + 8, &rounded_sum)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) o[c] = mfma(Keys32<D>::columns(v_tile, i, c), weights[i], o[c]);
    };
    auto step = [&](auto careful, int j0, char *__restrict__ k_tile, char *__restrict__ v_tile, char *__restrict__ next_k, char *__restrict__ next_v) {
        wait_for_loads();
        const bool is_whole = whole(j0);
        if (careful.value && !is_whole) clean_values<D, kLoaders>(v_tile, loader, n_keys - j0);
        // Behind this barrier the tile is complete and all are done with the one before, whose place the next
        // one takes.
        tile_complete<SPLIT>();
        if (!SPLIT && j0 + kStep < key_end) stream.next(j0 + kStep, next_k, next_v);
        if (is_whole ? !idle : !idle && !(a.s.causal && j0 > place0 + 31) && !(a.s.window > 0 && j0 + kKeys - 1 <= place0 - a.s.window))
            add_tile(j0, k_tile, v_tile, !is_whole);
    };
    auto add_all = [&](auto careful) {
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) o[c] = f32x16{0};
        sum = rounded_sum = 0.0f;
        if constexpr (SPLIT) {
            for (int j0 = j_begin; j0 < key_end; j0 += kStep) {
                step(careful, j0, tiles.k[0], tiles.v[0], nullptr, nullptr);
                tile_complete<SPLIT>();
                if (j0 + kStep < key_end) stream.next(j0 + kStep, tiles.k[0], tiles.v[0]);
            }
        } else {
            for (int j0 = j_begin; j0 < key_end; j0 += 2 * kStep) {
                step(careful, j0, tiles.k[0], tiles.v[0], tiles.k[1], tiles.v[1]);
                if (j0 + kStep < key_end) step(careful, j0 + kStep, tiles.k[1], tiles.v[1], tiles.k[0], tiles.v[0]);
            }
        }
    };
    add_all(std::false_type{});
    float probe = 0.0f;  // NaN if a numerator is not finite
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) probe = __builtin_fmaf(o[c][r], 0.0f, probe);
    shared.special[wave] = __ballot(probe != probe) != 0;
    __syncthreads();
    if (shared.special[0] | shared.special[1] | shared.special[2] | shared.special[3]) {
        stream.start(j_begin);
        if (j_begin < key_end) stream.next(j_begin, tiles.k[0], tiles.v[0]);
        add_all(std::true_type{});
        __syncthreads();
        for (int j0 = j_begin; j0 < key_end; j0 += kStep) {
            if (whole(j0)) continue;
            for (int j = j0; j < min(j0 + kKeys, n_keys); ++j) {
                if (row >= at.end || j < first_seen || j >= last_seen) continue;
                const uint16_t *value = keys.v_at(j, keys.page(j)) + 4 * (lane >> 5);
#pragma unroll
                for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t v = value[32 * c + 8 * (r >> 2) + (r & 3)];
                        if ((v & 0x7F80u) == 0x7F80u) o[c][r] += __uint_as_float(v << 16);
                    }
            }
        }
    }

    sum += __shfl_xor(sum, 32);
    rounded_sum += __shfl_xor(rounded_sum, 32);
    // Numerators 4 i .. 4 i + 3 of every 32: a wavefront's own, or (SPLIT) a fourth of all, joined in the order
    // of the wavefronts.
    constexpr int kQuads = D / 8, kMine = SPLIT ? kQuads / kWaves : kQuads;
    const int quad0 = SPLIT ? wave * kMine : 0;
    f32x4 n[kMine];
    auto quad = [&](int i) {
        const f32x16 &c = o[i / 4];
        return f32x4{c[4 * (i % 4)], c[4 * (i % 4) + 1], c[4 * (i % 4) + 2], c[4 * (i % 4) + 3]};
    };
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) shared.sums[wave][i][lane] = quad(i);
        shared.weights[wave][lane] = lane < 32 ? rounded_sum : sum;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) n[i] = f32x4{0, 0, 0, 0};
        sum = rounded_sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) n[i] += shared.sums[w][quad0 + i][lane];
            rounded_sum += shared.weights[w][lane & 31];
            sum += shared.weights[w][32 + (lane & 31)];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) n[i] = quad(i);
    }
    const bool writes_sums = lane < 32 && (!SPLIT || wave == 0) && row < at.end;
    if (SUMS && writes_sums)
        a.lse[(long long)head * a.s.q_rows + row] = sum > 0.0f ? __builtin_logf(sum) : sum == 0.0f ? -__builtin_inff() : sum;
    const int first_value = 8 * quad0 + 4 * (lane >> 5);
    if (PAGED && a.parts > 1) {
        const long long at_row = ((long long)part * a.s.q_rows + row0) * a.s.heads + head;
        if (writes_sums) a.part_sums[at_row + (long long)(lane & 31) * a.s.heads] = rounded_sum;
        if constexpr (SPLIT) {
            if (row >= at.end) return;
            float *values = a.part_values + (at_row + (long long)(lane & 31) * a.s.heads) * D + first_value;
#pragma unroll
            for (int i = 0; i < kMine; ++i) *reinterpret_cast<f32x4 *>(values + 8 * i) = n[i];
        } else {
            store_rows_wide<D>(shared.tiles[0].k[0] + wave * kBytes, a.part_values + at_row * D, (long long)a.s.heads * D,
                               at.end - row0, [&](int i) { return n[i]; });
        }
        return;
    }
    const float to_mean = rounded_sum == 0.0f ? 0.0f : 1.0f / rounded_sum;
    auto rounded = [&](int i) { return u32x2{pack2(n[i][0] * to_mean, n[i][1] * to_mean), pack2(n[i][2] * to_mean, n[i][3] * to_mean)}; };
    auto dropped = [&](int i) {  // by rounding
        const u32x2 kept = rounded(i);
        float rest[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) rest[e] = n[i][e] * to_mean - __uint_as_float(e & 1 ? kept[e / 2] & 0xFFFF0000u : kept[e / 2] << 16);
        return u32x2{pack2(rest[0], rest[1]), pack2(rest[2], rest[3])};
    };
    if constexpr (PAGED && !SPLIT) {  // by whole rows 33 registers would spill
        if (row >= at.end) return;
        const long long to = ((long long)row * a.s.heads + head) * D + first_value;
#pragma unroll
        for (int i = 0; i < kMine; ++i) *reinterpret_cast<u32x2 *>(a.o + to + 8 * i) = rounded(i);
    } else {
        // all tiles are free since the barrier behind them, and the sums behind this one
        if constexpr (SPLIT) __syncthreads();
        char *tile = shared.tiles[0].k[0] + (SPLIT ? 0 : wave * kBytes);
        const long long to = ((long long)row0 * a.s.heads + head) * D, to_next = (long long)a.s.heads * D;
        store_rows<D, SPLIT>(tile, a.o + to, to_next, at.end - row0, rounded);
        if (a.rest != nullptr) store_rows<D, SPLIT>(tile, a.rest + to, to_next, at.end - row0, dropped);
    }
}

// The parts of a row added up in their order: four values of one row and head for each thread.
template <int D>
__global__ __launch_bounds__(kThreads) void cap_join_parts_kernel(ForwardArgs a)
{
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x, rows = (long long)a.s.q_rows * a.s.heads, at = i / (D / 4);
    if (at >= rows) return;
    const int first = offset_at(a.q_offsets, 0, a.s.q_rows), row = (int)(at / a.s.heads);
    f32x4 n = f32x4{0, 0, 0, 0};
    float total = 0.0f;
    if (row >= first && row < offset_at(a.q_offsets, a.s.docs, a.s.q_rows))
        for (int part = 0; part < a.parts; ++part) {
            n += *reinterpret_cast<const f32x4 *>(a.part_values + (part * rows + at) * D + 4 * (i % (D / 4)));
            total += a.part_sums[part * rows + at];
        }
    const float to_mean = total == 0.0f ? 0.0f : 1.0f / total;
    *reinterpret_cast<u32x2 *>(a.o + 4 * i) = u32x2{pack2(n[0] * to_mean, n[1] * to_mean), pack2(n[2] * to_mean, n[3] * to_mean)};
}

template <bool PAGED, bool SUMS>
ktanh_status_t launch_forward(const ForwardArgs &a, size_t dim, bool split, const KtCapPack &pack, ktanh_stream_t stream)
{
    const int members = split ? a.s.group : a.s.group >> (7 - a.shift);
    const unsigned long long blocks = unit_blocks(a.tiles, a.s.kv_heads, a.parts, members) + (a.parts == 1 ? a.s.heads : 0);
    const unsigned long long joins = ((unsigned long long)a.s.q_rows * a.s.heads * dim / 4 + kThreads - 1) / kThreads;
    if (blocks > kMaxBlocks || (a.parts > 1 && joins > kMaxBlocks)) return KT_ERR_SHAPE;
    auto *kernel = split ? dim == 64 ? &cap_forward_kernel<64, PAGED, SUMS, true> : &cap_forward_kernel<128, PAGED, SUMS, true>
                         : dim == 64 ? &cap_forward_kernel<64, PAGED, SUMS, false> : &cap_forward_kernel<128, PAGED, SUMS, false>;
    kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a, pack);
    ktanh_status_t st = launched();
    if constexpr (PAGED) {
        if (st == KT_OK && a.parts > 1) {
            auto *join = dim == 64 ? &cap_join_parts_kernel<64> : &cap_join_parts_kernel<128>;
            join<<<dim3((unsigned)joins), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
            st = launched();
        }
    }
    return st;
}

template <class Lut>
ktanh_status_t attention(const kcap_shape_t *shape, const uint16_t *q, const uint16_t *k, const uint16_t *v, const int32_t *q_offsets,
                         const int32_t *k_offsets, uint16_t *o, uint16_t *rest, float *lse, const Lut *lut, ktanh_stream_t stream)
{
    if (shape == nullptr) return KT_ERR_NULL;
    if (shape->q_rows == 0 || shape->docs == 0) return KT_OK;
    if (q == nullptr || q_offsets == nullptr || k_offsets == nullptr || o == nullptr) return KT_ERR_NULL;
    if ((k == nullptr || v == nullptr) && shape->k_rows != 0) return KT_ERR_NULL;
    ForwardArgs a{};
    ktanh_status_t st = read_shape(shape, q, k, v, &a.s);
    if (st != KT_OK) return st;
    if (reinterpret_cast<uintptr_t>(o) % 8 != 0 || reinterpret_cast<uintptr_t>(rest) % 8 != 0 || reinterpret_cast<uintptr_t>(lse) % 4 != 0 ||
        reinterpret_cast<uintptr_t>(q_offsets) % 4 != 0 || reinterpret_cast<uintptr_t>(k_offsets) % 4 != 0) return KT_ERR_ALIGN;
    KtCapPack pack;
    if ((st = pack_lines(lut, &pack)) != KT_OK) return st;
    a.q_offsets = q_offsets;
    a.k_offsets = k_offsets;
    a.o = o;
    a.rest = rest;
    a.lse = lse;
    a.parts = 1;
    const bool split = split_tiles(*shape);
    a.shift = rows_shift(a.s, split);
    a.tiles = (unsigned)stretches(shape->q_rows, shape->docs, a.shift);
    return lse != nullptr ? launch_forward<false, true>(a, shape->dim, split, pack, stream)
                          : launch_forward<false, false>(a, shape->dim, split, pack, stream);
}

}  // namespace

// How many blocks share the keys of a stretch, and of which kind they are: the least time of all, by what a
// block takes for a tile and around its tiles, how many a compute unit holds, and the launch that joins parts
// written and read at 4 TB/s.  Only the longest text is known here; texts are taken to be spread evenly up to
// it, so that the time is that of the longest or that of all on average.
// Four pieces of 512 tokens behind texts of up to 6000, 32 heads of 128: 253 us in one part, 261 in two, 228 in
// three (of 6000 each: 260, 304, 277).
// 8 tokens behind 16384 of four sequences: 143 us in blocks of 128 rows, 96 in blocks of 32; 512 behind 512 of
// eight: 58 and 107.
ktanh_cap::ForwardPlan ktanh_cap::forward_plan(const kcap_shape_t &s, const kcap_pages_t &p)
{
    ForwardPlan best{false, 1};
    if (s.docs == 0 || s.q_rows == 0 || s.kv_heads == 0 || s.heads < s.kv_heads) return best;
    const double docs = (double)s.docs, each = std::ceil((double)s.q_rows / docs), spread = (docs + 1.0) / (2.0 * docs);
    const double cached = (double)p.most * (double)p.page_size, part_us = (double)s.q_rows * (double)s.heads * (double)s.dim * 8.0 / 4e6;
    double least = 0.0;
    for (const bool split : {false, true}) {
        const size_t together = split ? 1 : (size_t)heads_together(s.heads / s.kv_heads);
        const double rows = split ? 32.0 : (double)(kRows / together), blocks = std::ceil(each / rows) * docs * (double)(s.heads / together);
        const double keys = s.window > 0 ? std::min(cached, (double)s.window + std::min(rows, each)) : cached;
        // Microseconds of 32 keys with 128 rows, or 128 with 32, by how many blocks a compute unit holds, up to
        // as many as it can.
        const double full_us[4] = {0.0, 1.2, 1.45, 1.85}, split_us[3] = {0.0, 1.75, 2.6};
        const double *tile_us = split ? split_us : full_us;
        const int most = split ? 2 : 3;
        for (int parts = 1; parts <= 64 && (parts == 1 || keys >= 256.0 * parts); ++parts) {
            const double tiles = keys / (split ? 128.0 : 32.0) / parts, held = std::ceil(blocks * parts / 256.0), rounds = std::floor(held / most);
            const double all_us = rounds * tile_us[most] + tile_us[(int)(held - rounds * most)];
            const double t = tiles * std::max(tile_us[1], spread * all_us) + 4.0 * std::ceil(held / most) + (parts > 1 ? 5.0 + part_us * parts : 0.0);
            if (least == 0.0 || t < least) {
                least = t;
                best = ForwardPlan{split, parts};
            }
        }
    }
    return best;
}

ktanh_status_t ktanh_cap::launch_forward_paged(const CapShape &s, const CapPages &p, const int *q_offsets, uint16_t *o,
                                               int dim, ForwardPlan plan, float *workspace, const KtCapPack &pack,
                                               ktanh_stream_t stream)
{
    ForwardArgs a{};
    a.s = s;
    a.p = p;
    a.q_offsets = q_offsets;
    a.o = o;
    a.parts = plan.parts;
    a.part_sums = workspace;
    a.part_values = workspace + forward_sums(plan.parts, s.q_rows, s.heads);
    a.shift = rows_shift(s, plan.split);
    a.tiles = (unsigned)stretches(s.q_rows, s.docs, a.shift);
    return launch_forward<true, false>(a, (size_t)dim, plan.split, pack, stream);
}

extern "C" ktanh_status_t kcap_attention(const kcap_shape_t *shape, const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                         const int32_t *q_offsets, const int32_t *k_offsets, uint16_t *o, uint16_t *rest, float *lse,
                                         const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return attention(shape, q, k, v, q_offsets, k_offsets, o, rest, lse, lut, stream);
}

extern "C" ktanh_status_t kcap_attention64(const kcap_shape_t *shape, const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                           const int32_t *q_offsets, const int32_t *k_offsets, uint16_t *o, uint16_t *rest, float *lse,
                                           const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return attention(shape, q, k, v, q_offsets, k_offsets, o, rest, lse, lut, stream);
}
