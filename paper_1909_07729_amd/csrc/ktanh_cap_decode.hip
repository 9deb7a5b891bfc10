// libktanh: capped attention over a paged cache, one query for each sequence.
//
// What it costs is reading the keys and values once.  The keys of a sequence and key/value head are cut into spans, a block
// for each; a wavefront takes every fourth tile of 32 keys for up to 32 query heads that share them, with the tile in LDS of its own
// (no barrier in the loop) and the next one on its way in registers.  Weights need no maximum (|y| <= cap),
// so wavefronts and spans are joined by adding numerators and denominators.
#include "ktanh_cap_args.h"

using namespace ktanh_cap;

namespace {

constexpr int kKeys = 32;  // of a wavefront's tile

struct DecodeArgs {
    CapShape s;
    CapPages p;
    uint16_t *o;
    float *sums, *parts;  // [docs][spans][heads], [docs][spans][heads][dim]: NULL where one span holds all keys
    int span, spans, row_blocks;
};

__device__ __forceinline__ int first_key(const CapShape &s, int n_keys) { return s.window > 0 ? max(0, n_keys - s.window) : 0; }

template <int D>
__global__ __launch_bounds__(kThreads, 2) void cap_decode_kernel(DecodeArgs a, KtCapPack pack)
{
    constexpr int kBytes = kKeys * kPitch<D>, kSteps = D / 16, kBlocks = D / 32;
    constexpr int kChunks = D / 8, kLoads = kKeys * kChunks / 64;  // 16-byte loads of a lane for each of K and V
    struct Shared {
        f32x2 lines[128];                 // first: the offset of a line is its address
        char tiles[kWaves][2 * kBytes];   // keys | values; at the end 32 x D numerators
        float sums[kWaves][32];
    };
    __shared__ __align__(16) Shared shared;
    f32x2 *lines = shared.lines;

    // heads and sequences first: the empty spans behind short sequences come last
    const int row_block = (int)(blockIdx.x % a.row_blocks), kv_head = (int)(blockIdx.x / a.row_blocks % a.s.kv_heads);
    const int seq = (int)(blockIdx.x / a.row_blocks / a.s.kv_heads % a.s.docs), span = (int)(blockIdx.x / a.row_blocks / a.s.kv_heads / a.s.docs);
    const int n_keys = keys_in_pages(a.p, seq), begin = max(first_key(a.s, n_keys), span * a.span), end = min(n_keys, (span + 1) * a.span);
    if (begin >= end && a.parts != nullptr) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head0 = kv_head * a.s.group + 32 * row_block, heads = min(32, a.s.group - 32 * row_block);
    const int *pages = a.p.pages + seq * a.p.row;
    const uint16_t *k = a.s.k.at + kv_head * a.s.k.head, *v = a.s.v.at + kv_head * a.s.v.head;
    char *k_tile = shared.tiles[wave], *v_tile = shared.tiles[wave] + kBytes;
    spread_lines(lines, pack, a.s.cap * kLog2e);

    bf16x8 q[kSteps];
    {
        const uint16_t *from = a.s.q.at + seq * a.s.q.row + (head0 + min(lane & 31, heads - 1)) * a.s.q.head + 8 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const bf16x8 *>(from + 16 * i);
    }
    f32x16 o[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) o[c] = f32x16{0};
    float sum = 0.0f;

    // The page of key j0 + (lane & 31): loaded two tiles ahead, handed to the lanes that load the row one tile ahead.
    auto page_for = [&](int j0) { return min(max(pages[min(j0 + (lane & 31), n_keys - 1) >> a.p.shift], 0), a.p.count - 1); };
    u32x4 next_k[kLoads], next_v[kLoads];
    auto load = [&](int j0, int page) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int row = lane / kChunks + n * (64 / kChunks), j = min(j0 + row, n_keys - 1);
            const long long in_page = j & ((1 << a.p.shift) - 1), p = __shfl(page, row);
            // read once: with the hint a batch takes 200 us instead of 222
            next_k[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(k + p * a.p.k_page + in_page * a.s.k.row + 8 * (lane % kChunks)));
            next_v[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(v + p * a.p.v_page + in_page * a.s.v.row + 8 * (lane % kChunks)));
        }
    };
    constexpr int kStride = kWaves * kKeys;
    int j0 = (begin & ~(kKeys - 1)) + wave * kKeys;
    int page = 0;
    if (j0 < end) {
        load(j0, page_for(j0));
        page = page_for(j0 + kStride);
    }
    __syncthreads();  // lines
    for (; j0 < end; j0 += kStride) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int row = lane / kChunks + n * (64 / kChunks), chunk = lane % kChunks;
            const bool seen = j0 + row >= begin && j0 + row < end;  // a value that is not seen may be an infinity
            *reinterpret_cast<u32x4 *>(k_tile + chunk_at<D>(row, chunk)) = next_k[n];
            *reinterpret_cast<u32x4 *>(v_tile + chunk_at<D>(row, chunk)) = seen ? next_v[n] : u32x4{0, 0, 0, 0};
        }
        if (j0 + kStride < end) {
            load(j0 + kStride, page);
            page = page_for(j0 + 2 * kStride);
        }
        // the tile is this wavefront's own: its LDS accesses are served in order
        __builtin_amdgcn_wave_barrier();
        f32x16 s = f32x16{0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = mfma(rows_of<D>(k_tile, 0, i), q[i], s);
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(capped(s[r] * a.s.to_x, lines));
        if (j0 < begin || j0 + kKeys > end) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int j = j0 + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
                p[r] = j >= begin && j < end ? p[r] : 0.0f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += p[r];
        // The matrix units wait for memory here: weights go in as two BFloat16 values each, 16 bits of them.
        const bf16x8 weights[2] = {pack8(p), pack8(p + 8)};
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] -= (float)weights[r / 8][r % 8];
        const bf16x8 rests[2] = {pack8(p), pack8(p + 8)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) {
                const bf16x8 columns = columns_of<D>(v_tile, 16 * i, c);
                o[c] = mfma(columns, weights[i], o[c]);
                o[c] = mfma(columns, rests[i], o[c]);
            }
        __builtin_amdgcn_wave_barrier();
    }

    // numerators [32][D] of each wavefront where its tile was, and their sums over the wavefronts
    __syncthreads();
    sum += __shfl_xor(sum, 32);
    if (lane < 32) shared.sums[wave][lane] = sum;
    if ((lane & 31) < heads) {
        float *mine = reinterpret_cast<float *>(shared.tiles[wave]) + (lane & 31) * D + 4 * (lane >> 5);
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4 *>(mine + 32 * c + 8 * i) = f32x4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < heads * (D / 4); i += kThreads) {
        const int h = i / (D / 4), d = i % (D / 4) * 4;
        f32x4 n = f32x4{0, 0, 0, 0};
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            n += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(shared.tiles[w]) + h * D + d);
            total += shared.sums[w][h];
        }
        if (a.parts == nullptr) {
            const float to_mean = total == 0.0f ? 0.0f : 1.0f / total;
            *reinterpret_cast<u32x2 *>(a.o + ((long long)seq * a.s.heads + head0 + h) * D + d) =
                u32x2{pack2(n[0] * to_mean, n[1] * to_mean), pack2(n[2] * to_mean, n[3] * to_mean)};
        } else {
            const long long at = ((long long)seq * a.spans + span) * a.s.heads + head0 + h;
            *reinterpret_cast<f32x4 *>(a.parts + at * D + d) = n;
            if (d == 0) a.sums[at] = total;
        }
    }
}

// The spans of a sequence and head added up: four values of one head for each thread, spans dealt to 16 or 32 threads in turn and
// those joined in their order.
constexpr int kJoinThreads = 1024;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void cap_join_kernel(DecodeArgs a)
{
    constexpr int kAcross = D / 4, kDeep = kJoinThreads / kAcross;
    __shared__ f32x4 parts[kDeep][kAcross];
    __shared__ float sums[kDeep];
    const int seq = blockIdx.x / a.s.heads, head = blockIdx.x % a.s.heads;
    const int n_keys = keys_in_pages(a.p, seq), begin = first_key(a.s, n_keys);
    const int across = threadIdx.x % kAcross, deep = threadIdx.x / kAcross;
    f32x4 n = f32x4{0, 0, 0, 0};
    float total = 0.0f;
    for (int span = begin / a.span + deep; span * a.span < n_keys; span += kDeep) {
        const long long at = ((long long)seq * a.spans + span) * a.s.heads + head;
        n += *reinterpret_cast<const f32x4 *>(a.parts + at * D + 4 * across);
        total += a.sums[at];
    }
    parts[deep][across] = n;
    if (across == 0) sums[deep] = total;
    __syncthreads();
    if (deep != 0) return;
#pragma unroll
    for (int i = 1; i < kDeep; ++i) {
        n += parts[i][across];
        total += sums[i];
    }
    const float to_mean = total == 0.0f ? 0.0f : 1.0f / total;
    *reinterpret_cast<u32x2 *>(a.o + ((long long)seq * a.s.heads + head) * D + 4 * across) =
        u32x2{pack2(n[0] * to_mean, n[1] * to_mean), pack2(n[2] * to_mean, n[3] * to_mean)};
}

// Keys of a span: a power of two between one round of the four wavefronts and 1024 keys, such that all sequences' spans
// fill the chip several times over if they are as long as the table allows.
int span_of(const kcap_shape_t &s, const kcap_pages_t &p)
{
    const unsigned long long keys = (unsigned long long)p.most * p.page_size, across = (unsigned long long)s.docs * s.kv_heads;
    int span = 1024;
    while (span > kWaves * kKeys && across * ((keys + span - 1) / span) < 2048) span /= 2;
    return span;
}

unsigned long long spans_of(const kcap_pages_t &p, int span) { return ((unsigned long long)p.most * p.page_size + span - 1) / span; }

// Bytes of the sums in front of the numerators, which start on a cache line.
unsigned long long sums_bytes(const kcap_shape_t &s, unsigned long long spans) { return (s.docs * spans * s.heads * 4 + 127) / 128 * 128; }

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
        const int parts = forward_parts(*shape, *cache);
        if (parts > 1 && workspace == nullptr) return KT_ERR_NULL;
        if (parts > 1 && !aligned16(workspace)) return KT_ERR_ALIGN;
        return launch_forward_paged(a.s, p, q_offsets, o, (int)shape->dim, parts, static_cast<float *>(workspace), pack, stream);
    }

    if (shape->q_rows != shape->docs) return KT_ERR_SHAPE;
    a.p = p;
    a.o = o;
    a.span = span_of(*shape, *cache);
    const unsigned long long spans = spans_of(*cache, a.span);
    a.row_blocks = (a.s.group + 31) / 32;
    const unsigned long long blocks = spans * shape->docs * shape->kv_heads * a.row_blocks, joins = shape->docs * shape->heads;
    if (blocks > kMaxBlocks || joins > kMaxBlocks / (kJoinThreads / kThreads)) return KT_ERR_SHAPE;
    a.spans = (int)spans;
    if (spans > 1) {
        if (workspace == nullptr) return KT_ERR_NULL;
        if (!aligned16(workspace)) return KT_ERR_ALIGN;
        a.sums = static_cast<float *>(workspace);
        a.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + sums_bytes(*shape, spans));
    }
    const auto on = static_cast<hipStream_t>(stream);
    auto *kernel = shape->dim == 64 ? &cap_decode_kernel<64> : &cap_decode_kernel<128>;
    kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, on>>>(a, pack);
    if ((st = launched()) != KT_OK || spans == 1) return st;
    auto *join = shape->dim == 64 ? &cap_join_kernel<64> : &cap_join_kernel<128>;
    join<<<dim3((unsigned)joins), dim3(kJoinThreads), 0, on>>>(a);
    return launched();
}

}  // namespace

extern "C" size_t kcap_attention_paged_workspace(const kcap_shape_t *shape, const kcap_pages_t *cache, int single)
{
    if (shape == nullptr || cache == nullptr || shape->docs == 0 || cache->page_size == 0 || cache->page_size > 1u << 20 ||
        cache->most == 0 || cache->most > 1u << 30 || shape->docs > 1u << 30 || shape->heads > 65536 || shape->kv_heads > 65536 || shape->dim > 128 || shape->q_rows > 1u << 30)
        return 0;
    if (!single) {
        const size_t parts = (size_t)forward_parts(*shape, *cache);
        return parts > 1 ? (forward_sums(parts, shape->q_rows, shape->heads) + parts * shape->q_rows * shape->heads * shape->dim) * 4 : 0;
    }
    const unsigned long long spans = spans_of(*cache, span_of(*shape, *cache));
    if (spans <= 1) return 0;
    return (size_t)(sums_bytes(*shape, spans) + shape->docs * spans * shape->heads * shape->dim * 4);
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
