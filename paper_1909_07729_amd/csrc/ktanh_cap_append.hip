// libktanh: new tokens into a paged cache, keys rotated on the way, values as they are, and the queries
// rotated.
//
// Moves each value once.  A lane takes units of 16 values of one head, two 16-byte pieces: both halves of eight
// rotated pairs, or what is behind the rotated part.  A wavefront works for one token, so that its place
// (document, length, page: three loads one behind the other) is looked up once, while the values are on their
// way.
//
// What bounds it: memory.  16384 tokens of 32 heads of 128 on 8: 411 MB in 69 us, 6.0 TB/s; 64 tokens take 5
// us, a launch and two latencies.
#include "ktanh_cap_args.h"

using namespace ktanh_cap;

namespace {

struct AppendArgs {
    Rows q, k, v;
    uint16_t *q_out, *k_cache, *v_cache;
    CapPages p;
    long long k_slot, k_head, v_slot, v_head;
    const int *q_offsets;
    const float *cos, *sin;
    int docs, tokens, heads, kv_heads, dim, positions, angles, interleaved, waves_per_token;
};

__device__ __forceinline__ void unpack8(u32x4 w, float *v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ u32x4 packed8(const float *v) { return __builtin_bit_cast(u32x4, pack8(v)); }

constexpr int kUnits = 2;  // of a lane: 16384 tokens in 69.3 us, with one 70.0, with four 76.4

__global__ __launch_bounds__(kThreads) void cap_append_kernel(AppendArgs a)
{
    const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    const int token = (int)(wave / a.waves_per_token), lane = threadIdx.x & 63;
    if (token >= a.tokens) return;

    // The values are asked for first: nothing of their address depends on where they go.
    const int pieces = a.dim / 16;  // of a head, 16 values each
    const int rows = a.heads + 2 * a.kv_heads;
    int row[kUnits], piece[kUnits], lo[kUnits], hi[kUnits];
    u32x4 out_lo[kUnits], out_hi[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int unit = ((int)(wave % a.waves_per_token) * kUnits + u) * 64 + lane;
        row[u] = unit / pieces;
        piece[u] = unit % pieces;
        const int at = min(row[u], rows - 1);
        const bool is_q = at < a.heads, is_v = at >= a.heads + a.kv_heads;
        const Rows &in = is_q ? a.q : is_v ? a.v : a.k;
        const uint16_t *from = in.at + token * in.row + (is_q ? at : (at - a.heads) % a.kv_heads) * in.head;
        const bool halves = !is_v && 8 * piece[u] < a.angles && !a.interleaved;
        lo[u] = halves ? 8 * piece[u] : 16 * piece[u];
        hi[u] = halves ? lo[u] + a.angles : lo[u] + 8;
        // read once: with the hint 16384 tokens take 69 us instead of 79
        out_lo[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + lo[u]));
        out_hi[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + hi[u]));
    }

    const int doc = a.q_offsets == nullptr ? token : last_document(a.docs, [&](int d) { return offset_at(a.q_offsets, d, a.tokens) <= token; });
    const int first = offset_at(a.q_offsets, doc, a.tokens);
    if (token < first || token >= offset_at(a.q_offsets, doc + 1, a.tokens)) return;  // in no sequence
    const int position = (int)min((long long)max(a.p.lengths[doc], 0) + (token - first), 0x7FFFFFFFll);
    const bool has_angles = position < a.positions;
    const int slot = position >> a.p.shift;
    const int page = has_angles && slot < a.p.most ? a.p.pages[doc * a.p.row + slot] : -1;
    const long long in_page = position & ((1 << a.p.shift) - 1);

#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        if (row[u] >= rows) continue;
        const bool is_q = row[u] < a.heads, is_v = row[u] >= a.heads + a.kv_heads;
        const int head = is_q ? row[u] : (row[u] - a.heads) % a.kv_heads;
        if (!is_q && (page < 0 || page >= a.p.count)) continue;
        uint16_t *to = is_q   ? a.q_out + ((long long)token * a.heads + head) * a.dim
                       : is_v ? a.v_cache + wide(page, a.p.v_page) + in_page * a.v_slot + head * a.v_head
                              : a.k_cache + wide(page, a.p.k_page) + in_page * a.k_slot + head * a.k_head;
        if (!is_v && 8 * piece[u] < a.angles) {
            float x[16], cos[8], sin[8];
            unpack8(out_lo[u], x);
            unpack8(out_hi[u], x + 8);
            const long long angle = (long long)min(position, a.positions - 1) * a.angles + 8 * piece[u];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<f32x4 *>(cos + 4 * i) = *reinterpret_cast<const f32x4 *>(a.cos + angle + 4 * i);
                *reinterpret_cast<f32x4 *>(sin + 4 * i) = *reinterpret_cast<const f32x4 *>(a.sin + angle + 4 * i);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at_a = a.interleaved ? 2 * i : i, at_b = a.interleaved ? 2 * i + 1 : i + 8;
                const float v = x[at_a], w = x[at_b];
                x[at_a] = v * cos[i] - w * sin[i];
                x[at_b] = w * cos[i] + v * sin[i];
            }
            out_lo[u] = packed8(x);
            out_hi[u] = packed8(x + 8);
        }
        if (is_q && !has_angles) out_lo[u] = out_hi[u] = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        *reinterpret_cast<u32x4 *>(to + lo[u]) = out_lo[u];
        *reinterpret_cast<u32x4 *>(to + hi[u]) = out_hi[u];
    }
}

}  // namespace

extern "C" ktanh_status_t kcap_append(const kcap_shape_t *shape, const kcap_pages_t *cache, const uint16_t *q, const uint16_t *k,
                                      const uint16_t *v, uint16_t *q_out, uint16_t *k_cache, uint16_t *v_cache, const int32_t *pages,
                                      const int32_t *lengths, const int32_t *q_offsets, const float *cos, const float *sin, size_t positions,
                                      size_t angles, int interleaved, ktanh_stream_t stream)
{
    if (shape == nullptr || cache == nullptr) return KT_ERR_NULL;
    if (shape->q_rows == 0 || shape->docs == 0) return KT_OK;
    if (q == nullptr || k == nullptr || v == nullptr || q_out == nullptr || cos == nullptr || sin == nullptr) return KT_ERR_NULL;
    kcap_shape_t plain = *shape;
    plain.k_rows = 0;
    plain.scale = plain.cap = 1.0;  // not read
    plain.window = 0;
    CapShape s;
    AppendArgs a{};
    ktanh_status_t st = read_pages(cache, pages, lengths, k_cache, v_cache, &a.p);
    if (st != KT_OK || (st = read_shape(&plain, q, k, v, &s)) != KT_OK) return st;
    if (!aligned16(q_out) || !aligned16(cos) || !aligned16(sin) || reinterpret_cast<uintptr_t>(q_offsets) % 4 != 0) return KT_ERR_ALIGN;
    if (angles % 8 != 0 || 2 * angles > shape->dim || angles == 0 || positions == 0 || positions > 0x7FFFFFFF) return KT_ERR_SHAPE;
    if (q_offsets == nullptr && shape->q_rows != shape->docs) return KT_ERR_SHAPE;
    a.q = s.q;
    a.k = s.k;
    a.v = s.v;
    a.q_out = q_out;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.k_slot = (long long)cache->k_slot;
    a.k_head = (long long)cache->k_head;
    a.v_slot = (long long)cache->v_slot;
    a.v_head = (long long)cache->v_head;
    a.q_offsets = q_offsets;
    a.cos = cos;
    a.sin = sin;
    a.docs = s.docs;
    a.tokens = s.q_rows;
    a.heads = s.heads;
    a.kv_heads = s.kv_heads;
    a.dim = (int)shape->dim;
    a.positions = (int)positions;
    a.angles = (int)angles;
    a.interleaved = interleaved != 0;
    a.waves_per_token = ((s.heads + 2 * s.kv_heads) * (a.dim / 16) + 64 * kUnits - 1) / (64 * kUnits);
    const unsigned long long blocks = ((unsigned long long)a.tokens * a.waves_per_token + kWaves - 1) / kWaves;
    if (blocks > kMaxBlocks) return KT_ERR_SHAPE;  // wavefronts are numbered in 32 bits
    cap_append_kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
    return launched();
}
