// libktanh: attention with scores capped through K-TanH over many queries: packed documents, and pieces of
// prompts over a paged cache.
//
// A block holds 128 queries of one head and one document, 32 in each wavefront's registers, and goes once over the
// keys that they see in tiles of 32, double-buffered in LDS by direct loads.
//   S^T = K Q^T (keys x queries), p = e^(cap K(x)) in the accumulator, O^T += V^T P^T with P^T as it lies.
//
// What bounds it: a wavefront's 16 matrix and about 150 vector instructions of a tile take some 340 ns side by side with two
// others' (269 the matrix instructions alone), and three wavefronts share a SIMD because the tile's 32 keys and the direct loads leave
// 160 registers enough.  16384 tokens, 32 heads of 128, causal: 2331 us, 943 TFLOP/s; with 64 keys to a tile, through registers, and
// two wavefronts 2736; with 32 keys through registers 2620.
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
template <int D>
struct PagedStream {
    typedef Keys32<D> Tile;
    static constexpr int kShare = Tile::kStretches / kWaves;
    const Keys<true> &keys;
    const int wave;
    int pages[kShare];

    __device__ __forceinline__ PagedStream(const Keys<true> &keys, int wave, int at) : keys(keys), wave(wave) { look_up(at); }
    __device__ __forceinline__ void look_up(int at)
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
        look_up(at + kKeys);
    }
};

template <int D>
__device__ __forceinline__ Stream<D> stream_of(const Keys<false> &keys, int wave, int at)
{
    return Stream<D>(keys.k, keys.k_row, keys.v, keys.v_row, keys.last, wave, at);
}
template <int D>
__device__ __forceinline__ PagedStream<D> stream_of(const Keys<true> &keys, int wave, int at) { return PagedStream<D>(keys, wave, at); }

// Infinities and NaN become zero.  Returns whether there was one.
__device__ __forceinline__ bool take_special(u32x4 *v)
{
    bool found = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = ((*v)[i] & 0x7F80u) == 0x7F80u, hi = ((*v)[i] & 0x7F800000u) == 0x7F800000u;
        (*v)[i] &= (lo ? 0xFFFF0000u : ~0u) & (hi ? 0xFFFFu : ~0u);
        found |= lo || hi;
    }
    return found;
}

// Of the rows that this wavefront loaded: values behind the last key become zero, as infinities and NaN do.  Their weights are zero,
// and the product would not be.
template <int D>
__device__ __forceinline__ bool clean_values(char *v_tile, int wave, int there)
{
    bool found = false;
#pragma unroll
    for (int n = 0; n < Stream<D>::kShare; ++n) {
        const int g = wave * Stream<D>::kShare + n;
        u32x4 *at = reinterpret_cast<u32x4 *>(v_tile + Keys32<D>::stretch_at(g) + 16 * (threadIdx.x & 63));
        u32x4 w = *at;
        if (Keys32<D>::row_of_lane(g) >= there) w = u32x4{0, 0, 0, 0};
        else found |= take_special(&w);
        *at = w;
    }
    return found;
}

struct ForwardArgs {
    CapShape s;
    const int *q_offsets, *k_offsets;
    uint16_t *o, *rest;
    float *lse;
    CapPages p;
    unsigned tiles;
    // PAGED: blocks of a stretch that share its keys, with sums [parts][q_rows][heads] and numerators [parts][q_rows][heads][dim] in Float32
    int parts;
    float *part_sums, *part_values;
};

// SUMS: with log-sums.
template <int D, bool PAGED, bool SUMS>
__global__ __launch_bounds__(kThreads, 3) void cap_forward_kernel(ForwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = Keys32<D>::kBytes, kSteps = D / 16, kBlocks = D / 32;
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        char k[2][kBytes], v[2][kBytes];
        int special[kWaves];  // whether the wavefront took a value out of a tile
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    const unsigned total = a.tiles * (unsigned)(a.s.heads * a.parts);
    if (blockIdx.x >= padded(total)) {
        const int head = (int)(blockIdx.x - padded(total));
        clear_rows<D>(a.o, a.q_offsets, a.s.docs, a.s.q_rows, a.s.heads, head, [&](int row) {
            if (SUMS) a.lse[(long long)head * a.s.q_rows + row] = -__builtin_inff();
        });
        return;
    }
    const unsigned place = place_of_block(blockIdx.x, total);
    if (place >= total) return;
    // heads that share keys side by side, then the stretches by their work
    const int in_group = place % a.s.group, part = PAGED ? place / a.s.group % a.parts : 0;
    const unsigned stretch = place / a.s.group / a.parts;
    const int kv_head = stretch / a.tiles, head = kv_head * a.s.group + in_group;
    auto keys_of = [&](int doc) {
        if constexpr (PAGED) return Others{0, keys_in_pages(a.p, doc)};
        else return rows_in(a.k_offsets, doc, a.s.k_rows);
    };
    const Stretch at = stretch_of((int)(stretch % a.tiles), a.q_offsets, a.s.docs, a.s.q_rows, a.s.causal, true, keys_of);
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

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shift = n_keys - (at.end - at.begin);            // query i is key i + shift
    const int row0 = at.first + 32 * wave;                     // this wavefront's first query
    const int row = row0 + (lane & 31);                        // this lane's
    const int place0 = row0 - at.begin + shift, my_place = row - at.begin + shift;
    const int block_first = at.first - at.begin + shift;
    const int block_last = min(at.first + kRows, at.end) - 1 - at.begin + shift;
    int key_end = a.s.causal ? min(n_keys, block_last + 1) : n_keys;
    int key_begin = a.s.window > 0 ? max(0, block_first - a.s.window + 1) & ~(kKeys - 1) : 0;
    if (PAGED && a.parts > 1) {  // this block's share of them, in whole tiles
        const int share = (max(key_end - key_begin, 0) + a.parts * kKeys - 1) / (a.parts * kKeys) * kKeys;
        key_begin = min(key_begin + part * share, max(key_end, key_begin));
        key_end = min(key_end, key_begin + share);
    }

    // What is loaded first is what takes longest; the lines are there behind the first tile's barrier.
    auto stream = stream_of<D>(keys, wave, key_begin);
    if (key_begin < key_end) stream.next(key_begin, shared.k[0], shared.v[0]);
    bf16x8 q[kSteps];
    {
        const uint16_t *from = a.s.q.at + min(row, at.end - 1) * a.s.q.row + head * a.s.q.head + 8 * (lane >> 5);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) q[k] = *reinterpret_cast<const bf16x8 *>(from + 16 * k);
    }
    f32x16 o[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) o[c] = f32x16{0};
    spread_lines(lines, pack, a.s.cap * kLog2e);
    shared.special[wave] = 0;
    float sum = 0.0f, rounded_sum = 0.0f;  // of the weights, and of the weights as the product has them

    // Tiles that every query of the block sees whole.  In the others a weight may be zero because its key is hidden, and the product
    // with an infinite or NaN value would not be: such values are taken out, and added behind the loop where they are seen.
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
    auto step = [&](int j0, char *__restrict__ k_tile, char *__restrict__ v_tile, char *__restrict__ next_k, char *__restrict__ next_v) {
        wait_for_loads();
        const bool is_whole = whole(j0);
        if (!is_whole && clean_values<D>(v_tile, wave, n_keys - j0)) shared.special[wave] = 1;
        // Behind this barrier the tile is complete and all are done with the one before, whose place the next one takes.
        __syncthreads();
        if (j0 + kKeys < key_end) stream.next(j0 + kKeys, next_k, next_v);
        if (is_whole ? !idle : !idle && !(a.s.causal && j0 > place0 + 31) && !(a.s.window > 0 && j0 + kKeys - 1 <= place0 - a.s.window))
            add_tile(j0, k_tile, v_tile, !is_whole);
    };
    for (int j0 = key_begin; j0 < key_end; j0 += 2 * kKeys) {
        step(j0, shared.k[0], shared.v[0], shared.k[1], shared.v[1]);
        if (j0 + kKeys < key_end) step(j0 + kKeys, shared.k[1], shared.v[1], shared.k[0], shared.v[0]);
    }

    __syncthreads();
    if (shared.special[0] | shared.special[1] | shared.special[2] | shared.special[3]) {
        for (int j0 = key_begin; j0 < key_end; j0 += kKeys) {
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
    if (row >= at.end) return;
    if (SUMS && lane < 32)
        a.lse[(long long)head * a.s.q_rows + row] = sum > 0.0f ? __builtin_logf(sum) : sum == 0.0f ? -__builtin_inff() : sum;
    if (PAGED && a.parts > 1) {
        const long long at_row = ((long long)part * a.s.q_rows + row) * a.s.heads + head;
        if (lane < 32) a.part_sums[at_row] = rounded_sum;
        float *values = a.part_values + at_row * D + 4 * (lane >> 5);
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4 *>(values + 32 * c + 8 * i) = f32x4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
        return;
    }
    const float to_mean = rounded_sum == 0.0f ? 0.0f : 1.0f / rounded_sum;
    const long long to = ((long long)row * a.s.heads + head) * D + 4 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float w[4], rest[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = o[c][4 * i + e] * to_mean;
            const u32x2 rounded = {pack2(w[0], w[1]), pack2(w[2], w[3])};
            *reinterpret_cast<u32x2 *>(a.o + to + 32 * c + 8 * i) = rounded;
            if (a.rest != nullptr) {
#pragma unroll
                for (int e = 0; e < 4; ++e) rest[e] = w[e] - __uint_as_float(e & 1 ? rounded[e / 2] & 0xFFFF0000u : rounded[e / 2] << 16);
                *reinterpret_cast<u32x2 *>(a.rest + to + 32 * c + 8 * i) = u32x2{pack2(rest[0], rest[1]), pack2(rest[2], rest[3])};
            }
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
ktanh_status_t launch_forward(const ForwardArgs &a, size_t dim, const KtCapPack &pack, ktanh_stream_t stream)
{
    const unsigned long long blocks = ((unsigned long long)a.tiles * a.s.heads * a.parts + 7) / 8 * 8 + (a.parts == 1 ? a.s.heads : 0);
    const unsigned long long joins = ((unsigned long long)a.s.q_rows * a.s.heads * dim / 4 + kThreads - 1) / kThreads;
    if (blocks > kMaxBlocks || (a.parts > 1 && joins > kMaxBlocks)) return KT_ERR_SHAPE;
    auto *kernel = dim == 64 ? &cap_forward_kernel<64, PAGED, SUMS> : &cap_forward_kernel<128, PAGED, SUMS>;
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
    if (q == nullptr || q_offsets == nullptr || k_offsets == nullptr || o == nullptr || ((k == nullptr || v == nullptr) && shape->k_rows != 0)) return KT_ERR_NULL;
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
    a.tiles = (unsigned)(shape->q_rows / kRows + shape->docs);
    return lse != nullptr ? launch_forward<false, true>(a, shape->dim, pack, stream) : launch_forward<false, false>(a, shape->dim, pack, stream);
}

}  // namespace

// How many blocks share the keys of a stretch.  768 blocks run at once (three to a compute unit); one takes about 1.2 us for a tile of 32
// keys and 4 us around them, and joining costs a launch and the parts written and read at 4 TB/s.  By that the least of
// all rounds: four pieces of 512 tokens in 32 heads are 512 blocks, which take 253 us by themselves, 261 in two parts (two rounds of
// half the keys) and 228 in three; one piece of a long text needs many.
int ktanh_cap::forward_parts(const kcap_shape_t &s, const kcap_pages_t &p)
{
    if (s.docs == 0 || s.q_rows == 0) return 1;
    const double stretches = (double)s.docs * (double)(((s.q_rows + s.docs - 1) / s.docs + kRows - 1) / kRows);  // of sequences alike
    const double blocks = stretches * (double)s.heads, keys = (double)p.most * (double)p.page_size;
    const double part_us = (double)s.q_rows * (double)s.heads * (double)s.dim * 8.0 / 4e6;
    int best = 1;
    double least = 0.0;
    for (int parts = 1; parts <= 64 && (parts == 1 || keys >= 256.0 * parts); ++parts) {
        const double us = std::ceil(blocks * parts / 768.0) * (keys / 32.0 * 1.2 / parts + 4.0) + (parts > 1 ? 5.0 + part_us * parts : 0.0);
        if (parts == 1 || us < least) {
            least = us;
            best = parts;
        }
    }
    return best;
}

ktanh_status_t ktanh_cap::launch_forward_paged(const CapShape &s, const CapPages &p, const int *q_offsets, uint16_t *o, int dim, int parts,
                                               float *workspace, const KtCapPack &pack, ktanh_stream_t stream)
{
    ForwardArgs a{};
    a.s = s;
    a.p = p;
    a.q_offsets = q_offsets;
    a.o = o;
    a.parts = parts;
    a.part_sums = workspace;
    a.part_values = workspace + forward_sums(parts, s.q_rows, s.heads);
    a.tiles = (unsigned)(s.q_rows / kRows + s.docs);
    return launch_forward<true, false>(a, (size_t)dim, pack, stream);
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
