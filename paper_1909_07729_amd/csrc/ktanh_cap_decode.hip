// libktanh: capped attention over a paged cache, one query for each sequence.
//
// What it costs is reading the keys and values once.  All tiles of 32 keys of all sequences and key/value heads
// form one row, which is cut into equal shares, one for each wavefront that the chip holds: however the lengths
// differ, all are done at the same time, and none waits for a first load but at its start.  A wavefront works
// for up to 32 query heads that share keys, with the tile in LDS of its own (no barriers), the next one on its
// way in registers and the pages of the one behind it looked up.  Weights need no maximum (|y| <= cap), so what
// several wavefronts have of a sequence is joined by adding numerators and denominators; a sequence within one
// share is finished there.  Weights go into the product as two BFloat16 terms, 15 bits in all: the matrix unit
// idles, so the second term costs nothing, and the output is as far off as its own rounding.  Both terms have
// the weight's sign: of opposite ones, or with a zero among them, an infinite value would come out as NaN.
//
// What bounds it: memory.  64 texts of up to 8192 tokens, 32 heads of 128 on 8: 1.04 GB in 178 us, 5.9 TB/s (a
// wide read of as much memory reaches 6.9); two of 131071: 175 us, 6.1.  One text of 777 tokens: 10 us, half of
// it the second launch.
#include "ktanh_cap_args.h"

using namespace ktanh_cap;

namespace {

constexpr int kKeys = 32;  // of a tile

struct DecodeArgs {
    CapShape s;
    CapPages p;
    uint16_t *o;
    // what a wavefront has of the first and of the last sequence of its share, if others have the rest:
    // [shares][2][rows] and [..][rows][dim]
    float *sums, *parts;
    int shares, rows, row_blocks, slices;
};

__device__ __forceinline__ int first_key(const CapShape &s, int n_keys) { return s.window > 0 ? max(0, n_keys - s.window) : 0; }

__device__ __forceinline__ int tiles_of(const DecodeArgs &a, int seq)
{
    const int n_keys = keys_in_pages(a.p, seq);
    return (n_keys + kKeys - 1) / kKeys - first_key(a.s, n_keys) / kKeys;
}

// The row of tiles: sequence by sequence, in each head by head (or 32 heads by 32).
struct Row {
    int total, share;  // tiles in all, and of a wavefront
    int seq, before;   // the sequence that holds the first tile of share `at_share` (or, from 0 on, `given`), and the tiles before it
    __device__ __forceinline__ Row(const DecodeArgs &a, int at_share, int given) : total(0), share(1), seq(max(given, 0)), before(0)
    {
        const int heads = a.s.kv_heads * a.row_blocks, lane = (int)(threadIdx.x & 63);
        int count = 0, bits = 0;  // tiles of the sequences that the lanes look at, for one head
        auto look_at = [&](int base) {
            count = base + lane < a.s.docs ? tiles_of(a, base + lane) : 0;
            for (bits = 0; bits < 31 && __ballot(count >> bits) != 0;) ++bits;
        };
        for (int base = 0; base < a.s.docs; base += 64) {
            look_at(base);
            total += lanes_sum(count, bits) * heads;
        }
        share = max((total + a.shares - 1) / a.shares, 1);
        const int at = at_share * share;
        for (int base = 0, sum = 0; base < a.s.docs; base += 64) {
            if (a.s.docs > 64) look_at(base);
            const int mine = sum + lanes_before(count, bits) * heads;
            const unsigned long long here = __ballot(given >= 0 ? base + lane == given : mine <= at && at < mine + count * heads);
            if (here != 0) {
                const int at_lane = __builtin_ctzll(here);
                seq = base + at_lane;
                before = __builtin_amdgcn_readlane(mine, at_lane);
                break;
            }
            sum += lanes_sum(count, bits) * heads;
        }
    }
};

// A tile's place: scalars.
struct Place {
    int seq, head, j0, n_keys, first;  // head counts key/value heads by blocks of 32 query heads

    __device__ __forceinline__ void enter(const DecodeArgs &a)
    {
        n_keys = __builtin_amdgcn_readfirstlane(keys_in_pages(a.p, seq));
        first = first_key(a.s, n_keys);
        j0 = first & ~(kKeys - 1);
    }
    __device__ __forceinline__ void advance(const DecodeArgs &a)
    {
        j0 += kKeys;
        if (j0 < n_keys) return;
        j0 = first & ~(kKeys - 1);
        if (++head < a.s.kv_heads * a.row_blocks) return;
        head = 0;
        do {
            ++seq;
            enter(a);
        } while (n_keys == 0 && seq + 1 < a.s.docs);
    }
};

template <int D>
__global__ __launch_bounds__(64, 2) void cap_decode_kernel(DecodeArgs a, KtCapPack pack)
{
    constexpr int kBytes = kKeys * kPitch<D>, kSteps = D / 16, kBlocks = D / 32;
    constexpr int kChunks = D / 8, kLoads = kKeys * kChunks / 64;  // 16-byte loads of a lane for each of K and V
    struct Shared {
        f32x2 lines[128];  // first: the offset of a line is its address
        char k[kBytes], v[kBytes];
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    const int lane = threadIdx.x;
    const Row all(a, (int)blockIdx.x, -1);
    const int start = (int)blockIdx.x * all.share, end = min(all.total, start + all.share);
    if (start >= end) return;
    Place now;
    now.seq = __builtin_amdgcn_readfirstlane(all.seq);
    now.enter(a);
    {
        const int tiles = (now.n_keys + kKeys - 1) / kKeys - now.first / kKeys, in_seq = start - __builtin_amdgcn_readfirstlane(all.before);
        now.head = in_seq / tiles;
        now.j0 += in_seq % tiles * kKeys;
    }
    // The page of key j0 + (lane & 31), handed to the lanes that load the row one tile later.
    auto page_for = [&](const Place &at) {
        return min(max(a.p.pages[at.seq * a.p.row + (min(at.j0 + (lane & 31), at.n_keys - 1) >> a.p.shift)], 0), a.p.count - 1);
    };
    u32x4 next_k[kLoads], next_v[kLoads];
    auto load = [&](const Place &at, int page) {
        const int kv_head = at.head / a.row_blocks;
        const uint16_t *k = a.s.k.at + kv_head * a.s.k.head, *v = a.s.v.at + kv_head * a.s.v.head;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int row = lane / kChunks + n * (64 / kChunks), j = min(at.j0 + row, at.n_keys - 1);
            const int in_page = j & ((1 << a.p.shift) - 1), p = __shfl(page, row);
            // read once: with the hint a batch takes 200 us instead of 222
            next_k[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(
                k + wide(p, a.p.k_page) + wide(in_page, (uint32_t)a.s.k.row) + 8 * (lane % kChunks)));
            next_v[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(
                v + wide(p, a.p.v_page) + wide(in_page, (uint32_t)a.s.v.row) + 8 * (lane % kChunks)));
        }
    };
    bf16x8 q[kSteps];
    f32x16 o[kBlocks];
    float sum = 0.0f;
    int head0 = 0, heads = 0;  // query heads of the present sequence and key/value head
    auto begin = [&](const Place &at) {
        const int kv_head = at.head / a.row_blocks, row_block = at.head % a.row_blocks;
        head0 = kv_head * a.s.group + 32 * row_block;
        heads = min(32, a.s.group - 32 * row_block);
        const uint16_t *from = a.s.q.at + at.seq * a.s.q.row + (head0 + min(lane & 31, heads - 1)) * a.s.q.head + 8 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const bf16x8 *>(from + 16 * i);
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) o[c] = f32x16{0};
        sum = 0.0f;
    };

    Place next = now, pages = now;
    int page = page_for(now);
    load(now, page);
    if (start + 1 < end) {
        next.advance(a);
        page = page_for(next);
        pages = next;
    }
    begin(now);
    spread_lines<64>(lines, pack, a.s.cap * kLog2e);
    int segment = start;  // the first tile of the present sequence and head in this share
    __syncthreads();      // lines
    for (int n = start; n < end; ++n) {
        const int j0 = now.j0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = lane / kChunks + i * (64 / kChunks), chunk = lane % kChunks;
            const bool seen = j0 + row >= now.first && j0 + row < now.n_keys;  // a value that is not seen may be an infinity
            *reinterpret_cast<u32x4 *>(shared.k + chunk_at<D>(row, chunk)) = next_k[i];
            *reinterpret_cast<u32x4 *>(shared.v + chunk_at<D>(row, chunk)) = seen ? next_v[i] : u32x4{0, 0, 0, 0};
        }
        if (n + 1 < end) {
            load(next, page);
            if (n + 2 < end) {
                pages.advance(a);
                page = page_for(pages);
            }
        }
        // the tile is this wavefront's own: its LDS accesses are served in order
        __builtin_amdgcn_wave_barrier();
        f32x16 s = f32x16{0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = mfma(rows_of<D>(shared.k, 0, i), q[i], s);
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(capped(s[r] * a.s.to_x, lines));
        if (j0 < now.first || j0 + kKeys > now.n_keys) keep(p, Span(now.first, now.n_keys, j0));
        // The matrix units wait for memory here: weights go in as two BFloat16 values each, 15 bits of them at
        // least, and are summed as they go in.
        // Both are positive where the weight is, so that an infinite value stays one: the first is the weight
        // cut off, the second what is left of 1 + 2^-16 times it, and never zero.
        u32x4 cut[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the high halves of two weights
            const uint32_t pair = __builtin_amdgcn_perm(__float_as_uint(p[2 * i + 1]), __float_as_uint(p[2 * i]), 0x07060302u);
            sum = sum_of(__builtin_bit_cast(bf16x2, pair), sum);
            cut[i / 4][i % 4] = pair;
        }
        const bf16x8 weights[2] = {__builtin_bit_cast(bf16x8, cut[0]), __builtin_bit_cast(bf16x8, cut[1])};
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_fmaf(p[r], 1.0f + 0x1p-16f, -__uint_as_float(__float_as_uint(p[r]) & 0xFFFF0000u));
        const bf16x8 rests[2] = {pack8(p, &sum), pack8(p + 8, &sum)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) {
                const bf16x8 columns = columns_of<D>(shared.v, 16 * i, c);
                o[c] = mfma(columns, weights[i], o[c]);
                o[c] = mfma(columns, rests[i], o[c]);
            }
        __builtin_amdgcn_wave_barrier();

        const bool last = j0 + kKeys >= now.n_keys;  // of this sequence and head
        if (last || n + 1 == end) {
            const float all_keys = sum + __shfl_xor(sum, 32);
            const int tiles = (now.n_keys + kKeys - 1) / kKeys - now.first / kKeys;
            const bool whole = last && n + 1 - segment == tiles;
            const int row = lane & 31;
            if (row < heads) {
                if (whole) {
                    const float to_mean = all_keys == 0.0f ? 0.0f : 1.0f / all_keys;
                    uint16_t *to = a.o + ((long long)now.seq * a.s.heads + head0 + row) * D + 4 * (lane >> 5);
#pragma unroll
                    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<u32x2 *>(to + 32 * c + 8 * i) =
                                u32x2{pack2(o[c][4 * i] * to_mean, o[c][4 * i + 1] * to_mean), pack2(o[c][4 * i + 2] * to_mean, o[c][4 * i + 3] * to_mean)};
                } else {
                    const long long at = ((long long)blockIdx.x * 2 + (segment == start ? 0 : 1)) * a.rows + row;
                    if (lane < 32) a.sums[at] = all_keys;
                    float *to = a.parts + at * D + 4 * (lane >> 5);
#pragma unroll
                    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<f32x4 *>(to + 32 * c + 8 * i) = f32x4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
                }
            }
            if (n + 1 < end) {
                begin(next);
                segment = n + 1;
            }
        }
        now = next;
        next = pages;
    }
}

// The parts of a sequence and key/value head added up: four values of a row for each thread, the shares dealt
// to as many threads as there are for them in turn, and what those have joined in their order.  Where sequences
// are few eight blocks take a slice of the values each:
// two texts of 131071 tokens 174 us with slices, 188 without, 32 texts of up to 2000 37 and 33, 96 of up to 300
// in 8 heads 38 and 17.
constexpr int kJoinThreads = 256;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void cap_join_kernel(DecodeArgs a)
{
    __shared__ f32x4 parts[kJoinThreads];
    __shared__ float sums[kJoinThreads];
    const int pairs = a.s.kv_heads * a.row_blocks, slice = blockIdx.x % a.slices;
    const int seq = blockIdx.x / a.slices / pairs, pair = blockIdx.x / a.slices % pairs;
    const int head0 = pair / a.row_blocks * a.s.group + 32 * (pair % a.row_blocks), heads = min(32, a.s.group - 32 * (pair % a.row_blocks));
    const Row all(a, 0, seq);
    const int tiles = tiles_of(a, seq), from = all.before + pair * tiles;
    const int first = from / all.share, last = tiles > 0 ? (from + tiles - 1) / all.share : first;
    if (tiles > 0 && first == last) return;  // finished by that wavefront
    const int across = heads * (D / 4) / a.slices, deep = kJoinThreads / across, at_deep = threadIdx.x / across;
    const int item = slice * across + threadIdx.x % across, row = item / (D / 4), d = item % (D / 4) * 4;
    f32x4 n = f32x4{0, 0, 0, 0};
    float total = 0.0f;
    if (tiles > 0 && at_deep < deep) {
#pragma unroll 4
        for (int share = first + at_deep; share <= last; share += deep) {
            const long long at = ((long long)share * 2 + (from <= share * all.share ? 0 : 1)) * a.rows + row;
            n += *reinterpret_cast<const f32x4 *>(a.parts + at * D + d);
            total += a.sums[at];
        }
    }
    parts[threadIdx.x] = n;
    sums[threadIdx.x] = total;
    __syncthreads();
    if (at_deep != 0) return;
    for (int i = 1; i < deep; ++i) {
        n += parts[threadIdx.x + i * across];
        total += sums[threadIdx.x + i * across];
    }
    const float to_mean = total == 0.0f ? 0.0f : 1.0f / total;
    *reinterpret_cast<u32x2 *>(a.o + ((long long)seq * a.s.heads + head0 + row) * D + d) =
        u32x2{pack2(n[0] * to_mean, n[1] * to_mean), pack2(n[2] * to_mean, n[3] * to_mean)};
}

// Wavefronts: as many as the chip holds (eight to a compute unit at dim 128, twelve at 64), at most one for
// each tile that the table has room for.
// 64 texts of up to 8192 tokens, with four, eight and sixteen to a compute unit 223, 177 and 185 us at dim 128,
// with six, twelve and eighteen 112, 101 and 103 at 64.
struct Shares {
    unsigned long long tiles, shares, rows, row_blocks;
    Shares(const kcap_shape_t &s, const kcap_pages_t &p)
    {
        const unsigned long long group = s.kv_heads > 0 ? s.heads / s.kv_heads : 0;
        row_blocks = (group + 31) / 32;
        rows = group < 32 ? group : 32;
        tiles = ((unsigned long long)p.most * p.page_size + kKeys - 1) / kKeys * s.docs * s.kv_heads * row_blocks;
        const unsigned long long most = 256 * (s.dim == 64 ? 12 : 8);
        shares = tiles < most ? tiles : most;
    }
    // Bytes of the sums in front of the numerators, which start on a cache line.
    unsigned long long sums_bytes() const { return (shares * 2 * rows * 4 + 127) / 128 * 128; }
};

template <class Lut>
ktanh_status_t attention_paged(const kcap_shape_t *shape, const kcap_pages_t *cache, const uint16_t *q, const uint16_t *k_cache,
                               const uint16_t *v_cache, const int32_t *pages, const int32_t *lengths, const int32_t *q_offsets, uint16_t *o,
                               void *workspace, const Lut *lut, ktanh_stream_t stream)
{
    if (shape == nullptr || cache == nullptr) return KT_ERR_NULL;
    if (shape->q_rows == 0 || shape->docs == 0) return KT_OK;
    if (q == nullptr || o == nullptr) return KT_ERR_NULL;
    kcap_shape_t in_cache = *shape;
    in_cache.k_rows = 0;
    in_cache.causal = 1;
    in_cache.k_row = cache->k_slot;
    in_cache.k_head = cache->k_head;
    in_cache.v_row = cache->v_slot;
    in_cache.v_head = cache->v_head;
    CapPages p;
    ktanh_status_t st = read_pages(cache, pages, lengths, k_cache, v_cache, &p);
    if (st != KT_OK) return st;
    DecodeArgs a{};
    if ((st = read_shape(&in_cache, q, k_cache, v_cache, &a.s)) != KT_OK) return st;
    if (reinterpret_cast<uintptr_t>(o) % 8 != 0 || reinterpret_cast<uintptr_t>(q_offsets) % 4 != 0) return KT_ERR_ALIGN;
    KtCapPack pack;
    if ((st = pack_lines(lut, &pack)) != KT_OK) return st;
    if (q_offsets != nullptr) {
        const ForwardPlan plan = forward_plan(*shape, *cache);
        if (plan.parts > 1 && workspace == nullptr) return KT_ERR_NULL;
        if (plan.parts > 1 && !aligned16(workspace)) return KT_ERR_ALIGN;
        return launch_forward_paged(a.s, p, q_offsets, o, (int)shape->dim, plan, static_cast<float *>(workspace), pack, stream);
    }

    if (shape->q_rows != shape->docs) return KT_ERR_SHAPE;
    const Shares cut(*shape, *cache);
    const unsigned long long joins = shape->docs * shape->kv_heads * cut.row_blocks;
    if (cut.tiles > 0x7FFFFFFF - 65536 || joins > kMaxBlocks / 8) return KT_ERR_SHAPE;
    if (workspace == nullptr) return KT_ERR_NULL;
    if (!aligned16(workspace)) return KT_ERR_ALIGN;
    a.p = p;
    a.o = o;
    a.shares = (int)cut.shares;
    a.rows = (int)cut.rows;
    a.row_blocks = (int)cut.row_blocks;
    a.sums = static_cast<float *>(workspace);
    a.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + cut.sums_bytes());
    const auto on = static_cast<hipStream_t>(stream);
    auto *kernel = shape->dim == 64 ? &cap_decode_kernel<64> : &cap_decode_kernel<128>;
    kernel<<<dim3((unsigned)cut.shares), dim3(64), 0, on>>>(a, pack);
    if ((st = launched()) != KT_OK) return st;
    auto *join = shape->dim == 64 ? &cap_join_kernel<64> : &cap_join_kernel<128>;
    a.slices = joins >= 256 && a.rows * (int)shape->dim / 4 <= kJoinThreads ? 1 : 8;  // a slice is no more than a block's threads
    join<<<dim3((unsigned)(joins * a.slices)), dim3(kJoinThreads), 0, on>>>(a);
    return launched();
}

}  // namespace

extern "C" size_t kcap_attention_paged_workspace(const kcap_shape_t *shape, const kcap_pages_t *cache, int single)
{
    if (shape == nullptr || cache == nullptr || shape->docs == 0 || cache->page_size == 0 || cache->page_size > 1u << 20 ||
        cache->most == 0 || cache->most > 1u << 30 || shape->docs > 1u << 30 || shape->q_rows > 1u << 30 ||
        shape->heads > 65536 || shape->kv_heads > 65536 || shape->dim > 128)
        return 0;
    if (!single) {
        const size_t parts = (size_t)forward_plan(*shape, *cache).parts;
        return parts > 1 ? (forward_sums(parts, shape->q_rows, shape->heads) + parts * shape->q_rows * shape->heads * shape->dim) * 4 : 0;
    }
    const Shares cut(*shape, *cache);
    return (size_t)(cut.sums_bytes() + cut.shares * 2 * cut.rows * shape->dim * 4);
}

extern "C" ktanh_status_t kcap_attention_paged(const kcap_shape_t *shape, const kcap_pages_t *cache, const uint16_t *q, const uint16_t *k_cache,
                                               const uint16_t *v_cache, const int32_t *pages, const int32_t *lengths, const int32_t *q_offsets,
                                               uint16_t *o, void *workspace, const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return attention_paged(shape, cache, q, k_cache, v_cache, pages, lengths, q_offsets, o, workspace, lut, stream);
}

extern "C" ktanh_status_t kcap_attention64_paged(const kcap_shape_t *shape, const kcap_pages_t *cache, const uint16_t *q, const uint16_t *k_cache,
                                                 const uint16_t *v_cache, const int32_t *pages, const int32_t *lengths, const int32_t *q_offsets,
                                                 uint16_t *o, void *workspace, const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return attention_paged(shape, cache, q, k_cache, v_cache, pages, lengths, q_offsets, o, workspace, lut, stream);
}
