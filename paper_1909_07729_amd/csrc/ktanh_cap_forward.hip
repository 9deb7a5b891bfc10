// libktanh: attention with scores capped through K-TanH over many queries: packed documents, and pieces of
// prompts over a paged cache.
//
// A block holds 128 queries of one head and one document, 32 in each wavefront's registers, and goes once over the
// keys that they see in tiles of 64, double-buffered in LDS (the next tile travels through registers while this one is used).
//   S^T = K Q^T (keys x queries), p = e^(cap K(x)) in the accumulator, O^T += V^T P^T with P^T as it lies.
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
    long long k_page, v_page;

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
        return k + page * k_page + (j & ((1 << shift) - 1)) * k_row;
    }
    __device__ __forceinline__ const uint16_t *v_at(int j, int page) const
    {
        j = min(j, last);
        if constexpr (!PAGED) return v + j * v_row;
        return v + page * v_page + (j & ((1 << shift) - 1)) * v_row;
    }
};

// One thread's share of a tile: chunk threadIdx % (D / 8) of the rows threadIdx / (D / 8) + n * kStep.
template <int D>
struct Share {
    static constexpr int kChunks = D / 8, kStep = kThreads / kChunks, kCount = kTile / kStep;
    u32x4 k[kCount], v[kCount];
};

template <int D, bool PAGED>
__device__ __forceinline__ void pages_of(const Keys<PAGED> &keys, int j0, int (&pages)[Share<D>::kCount])
{
#pragma unroll
    for (int n = 0; n < Share<D>::kCount; ++n) pages[n] = keys.page(j0 + (int)threadIdx.x / Share<D>::kChunks + n * Share<D>::kStep);
}

template <int D, bool PAGED>
__device__ __forceinline__ void load_share(Share<D> &share, const Keys<PAGED> &keys, int j0, const int (&pages)[Share<D>::kCount])
{
    const int chunk = threadIdx.x % Share<D>::kChunks;
#pragma unroll
    for (int n = 0; n < Share<D>::kCount; ++n) {
        const int j = j0 + (int)threadIdx.x / Share<D>::kChunks + n * Share<D>::kStep;
        share.k[n] = *reinterpret_cast<const u32x4 *>(keys.k_at(j, pages[n]) + 8 * chunk);
        share.v[n] = *reinterpret_cast<const u32x4 *>(keys.v_at(j, pages[n]) + 8 * chunk);
    }
}

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

// Values of rows from `end` on are zero: their weights are, and zero times an infinity would not be.
template <int D>
__device__ __forceinline__ void store_share(const Share<D> &share, char *k_tile, char *v_tile, int j0, int end)
{
    const int chunk = threadIdx.x % Share<D>::kChunks;
#pragma unroll
    for (int n = 0; n < Share<D>::kCount; ++n) {
        const int row = threadIdx.x / Share<D>::kChunks + n * Share<D>::kStep;
        *reinterpret_cast<u32x4 *>(k_tile + chunk_at<D>(row, chunk)) = share.k[n];
        *reinterpret_cast<u32x4 *>(v_tile + chunk_at<D>(row, chunk)) = j0 + row < end ? share.v[n] : u32x4{0, 0, 0, 0};
    }
}

struct ForwardArgs {
    CapShape s;
    const int *q_offsets, *k_offsets;
    uint16_t *o, *rest;
    float *lse;
    CapPages p;
    unsigned tiles;
};

template <int D, bool PAGED>
__global__ __launch_bounds__(kThreads, 2) void cap_forward_kernel(ForwardArgs a, KtCapPack pack)
{
    constexpr int kBytes = kTile * D * 2, kSteps = D / 16, kBlocks = D / 32;
    __shared__ __align__(16) char k_tiles[2][kBytes];
    __shared__ __align__(16) char v_tiles[2][kBytes];
    __shared__ f32x2 lines[128];
    __shared__ int special;  // whether a value was taken out of a tile

    const unsigned total = a.tiles * (unsigned)a.s.heads;
    if (blockIdx.x >= padded(total)) {
        const int head = (int)(blockIdx.x - padded(total));
        clear_rows<D>(a.o, a.q_offsets, a.s.docs, a.s.q_rows, a.s.heads, head, [&](int row) {
            if (a.lse != nullptr) a.lse[(long long)head * a.s.q_rows + row] = -__builtin_inff();
        });
        return;
    }
    const unsigned place = place_of_block(blockIdx.x, total);
    if (place >= total) return;
    // heads that share keys side by side, then the stretches from the last (the longest, if causal) to the first
    const int in_group = place % a.s.group;
    const int tile = (int)(a.tiles - 1 - place / a.s.group % a.tiles);
    const int kv_head = place / a.s.group / a.tiles, head = kv_head * a.s.group + in_group;
    const Stretch at = stretch_of(tile, a.q_offsets, a.s.docs, a.s.q_rows, kRows);
    if (at.first >= at.end) return;

    Keys<PAGED> keys;
    int n_keys;
    if constexpr (PAGED) {
        n_keys = keys_in_pages(a.p, at.doc);
        keys.k = a.s.k.at + kv_head * a.s.k.head;
        keys.v = a.s.v.at + kv_head * a.s.v.head;
        keys.pages = a.p.pages + at.doc * a.p.row;
        keys.shift = a.p.shift;
        keys.count = a.p.count;
        keys.k_page = a.p.k_page;
        keys.v_page = a.p.v_page;
    } else {
        const int begin = offset_at(a.k_offsets, at.doc, a.s.k_rows);
        n_keys = max(offset_at(a.k_offsets, at.doc + 1, a.s.k_rows) - begin, 0);
        keys.k = a.s.k.at + begin * a.s.k.row + kv_head * a.s.k.head;
        keys.v = a.s.v.at + begin * a.s.v.row + kv_head * a.s.v.head;
    }
    keys.k_row = a.s.k.row;
    keys.v_row = a.s.v.row;
    keys.last = n_keys - 1;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int shift = n_keys - (at.end - at.begin);            // query i is key i + shift
    const int row0 = at.first + 32 * wave;                     // this wavefront's first query
    const int row = row0 + (lane & 31);                        // this lane's
    const int place0 = row0 - at.begin + shift, my_place = row - at.begin + shift;
    const int block_first = at.first - at.begin + shift;
    const int block_last = min(at.first + kRows, at.end) - 1 - at.begin + shift;
    const int key_end = a.s.causal ? min(n_keys, block_last + 1) : n_keys;
    const int key_begin = a.s.window > 0 ? max(0, block_first - a.s.window + 1) & ~(kTile - 1) : 0;

    if (threadIdx.x == 0) special = 0;
    const float unit = a.s.cap * kLog2e;
    spread_lines(lines, pack, unit);
    __syncthreads();

    bf16x8 q[kSteps];
    {
        const uint16_t *from = a.s.q.at + min(row, at.end - 1) * a.s.q.row + head * a.s.q.head + 8 * (lane >> 5);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) q[k] = *reinterpret_cast<const bf16x8 *>(from + 16 * k);
    }
    f32x16 o[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) o[c] = f32x16{0};
    float sum = 0.0f, rounded_sum = 0.0f;  // of the weights, and of the weights as the product has them

    Share<D> share;
    int pages[Share<D>::kCount];
    if (key_begin < key_end) {
        pages_of<D>(keys, key_begin, pages);
        load_share<D>(share, keys, key_begin, pages);
        if constexpr (PAGED) pages_of<D>(keys, key_begin + kTile, pages);
    }
    // Whether some query of the block does not see all of the tile.  There a weight may be zero because its key is hidden, and
    // the product with an infinite or NaN value would not be: such values are taken out, and added behind the loop where they are seen.
    auto mixed = [&](int j0) {
        return j0 + kTile > n_keys || (a.s.causal && j0 + kTile - 1 > block_first) || (a.s.window > 0 && j0 <= block_last - a.s.window);
    };
    auto seen = [&](int j) { return (j < n_keys) & (!a.s.causal | (j <= my_place)) & ((a.s.window == 0) | (j > my_place - a.s.window)); };
    int buffer = 0;
    for (int j0 = key_begin; j0 < key_end; j0 += kTile, buffer ^= 1) {
        char *k_tile = k_tiles[buffer], *v_tile = v_tiles[buffer];
        if (mixed(j0)) {
            bool found = false;
#pragma unroll
            for (int n = 0; n < Share<D>::kCount; ++n) found |= take_special(&share.v[n]);
            if (found) special = 1;
        }
        store_share<D>(share, k_tile, v_tile, j0, n_keys);
        // Another wavefront may still read the other buffer, which is next written behind this barrier's successor.
        __syncthreads();
        if (j0 + kTile < key_end) {
            load_share<D>(share, keys, j0 + kTile, pages);
            if constexpr (PAGED) pages_of<D>(keys, j0 + 2 * kTile, pages);
        }
        const bool none = (a.s.causal && j0 > place0 + 31) || (a.s.window > 0 && j0 + kTile - 1 <= place0 - a.s.window) || row0 >= at.end;
        if (none) continue;
        const bool partial = j0 + kTile > n_keys || (a.s.causal && j0 + kTile - 1 > place0) ||
                             (a.s.window > 0 && j0 <= place0 + 31 - a.s.window);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            f32x16 s = f32x16{0};
#pragma unroll
            for (int k = 0; k < kSteps; ++k) s = mfma(rows_of<D>(k_tile, 32 * sub, k), q[k], s);
            float p[16];
            if (any_capped(s, a.s.to_x)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(capped(s[r] * a.s.to_x, lines));
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] * a.s.to_x * unit);
            }
            if (partial) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = j0 + 32 * sub + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
                    p[r] = seen(j) ? p[r] : 0.0f;
                }
            }
            if (a.lse != nullptr) {
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += p[r];
            }
            const bf16x8 weights[2] = {pack8(p, &rounded_sum), pack8(p + 8, &rounded_sum)};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) o[c] = mfma(columns_of<D>(v_tile, 32 * sub + 16 * i, c), weights[i], o[c]);
        }
    }

    __syncthreads();
    if (special) {
        for (int j0 = key_begin; j0 < key_end; j0 += kTile) {
            if (!mixed(j0)) continue;
            for (int j = j0; j < min(j0 + kTile, n_keys); ++j) {
                if (row >= at.end || !seen(j)) continue;
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
    if (a.lse != nullptr && lane < 32)
        a.lse[(long long)head * a.s.q_rows + row] = sum > 0.0f ? __builtin_logf(sum) : sum == 0.0f ? -__builtin_inff() : sum;
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

template <bool PAGED>
ktanh_status_t launch_forward(const ForwardArgs &a, size_t dim, const KtCapPack &pack, ktanh_stream_t stream)
{
    const unsigned long long blocks = ((unsigned long long)a.tiles * a.s.heads + 7) / 8 * 8 + a.s.heads;
    if (blocks > kMaxBlocks) return KT_ERR_SHAPE;
    auto *kernel = dim == 64 ? &cap_forward_kernel<64, PAGED> : &cap_forward_kernel<128, PAGED>;
    kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a, pack);
    return launched();
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
    a.tiles = (unsigned)(shape->q_rows / kRows + shape->docs);
    return launch_forward<false>(a, shape->dim, pack, stream);
}

}  // namespace

ktanh_status_t ktanh_cap::launch_forward_paged(const CapShape &s, const CapPages &p, const int *q_offsets, uint16_t *o, int dim,
                                               const KtCapPack &pack, ktanh_stream_t stream)
{
    ForwardArgs a{};
    a.s = s;
    a.p = p;
    a.q_offsets = q_offsets;
    a.o = o;
    a.tiles = (unsigned)(s.q_rows / kRows + s.docs);
    return launch_forward<true>(a, (size_t)dim, pack, stream);
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
