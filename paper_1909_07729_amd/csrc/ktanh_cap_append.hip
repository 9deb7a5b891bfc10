// libktanh: new tokens into a paged cache, keys rotated on the way, values as they are, and the queries rotated.
//
// Moves each value once.  A lane takes 16 values of one head, two 16-byte pieces: both halves of eight rotated pairs, or
// what is behind the rotated part.  A wavefront works for one token, so that its place is looked up once.
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

__global__ __launch_bounds__(kThreads) void cap_append_kernel(AppendArgs a)
{
    const long long wave = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int token = (int)(wave / a.waves_per_token), lane = threadIdx.x & 63;
    if (token >= a.tokens) return;
    const int doc = a.q_offsets == nullptr ? token : last_document(a.docs, [&](int d) { return offset_at(a.q_offsets, d, a.tokens) <= token; });
    const int first = offset_at(a.q_offsets, doc, a.tokens);
    if (token < first || token >= offset_at(a.q_offsets, doc + 1, a.tokens)) return;  // in no sequence
    const int position = (int)min((long long)max(a.p.lengths[doc], 0) + (token - first), 0x7FFFFFFFll);

    const int pieces = a.dim / 16;  // of a head, 16 values each
    const int unit = (int)(wave % a.waves_per_token) * 64 + lane, row = unit / pieces, piece = unit % pieces;
    if (row >= a.heads + 2 * a.kv_heads) return;
    const bool is_q = row < a.heads, is_v = row >= a.heads + a.kv_heads;
    const int head = is_q ? row : (row - a.heads) % a.kv_heads;
    const bool has_angles = position < a.positions;

    uint16_t *to;
    if (is_q) {
        to = a.q_out + ((long long)token * a.heads + head) * a.dim;
    } else {
        const int slot = position >> a.p.shift;
        if (!has_angles || slot >= a.p.most) return;
        const int page = a.p.pages[doc * a.p.row + slot];
        if (page < 0 || page >= a.p.count) return;
        const long long in_page = position & ((1 << a.p.shift) - 1);
        to = is_v ? a.v_cache + page * a.p.v_page + in_page * a.v_slot + head * a.v_head
                  : a.k_cache + page * a.p.k_page + in_page * a.k_slot + head * a.k_head;
    }
    const Rows &in = is_q ? a.q : is_v ? a.v : a.k;
    const uint16_t *from = in.at + token * in.row + head * in.head;

    const bool turned = !is_v && 8 * piece < a.angles;
    const bool halves = turned && !a.interleaved;
    const int lo = halves ? 8 * piece : 16 * piece, hi = halves ? lo + a.angles : lo + 8;
    u32x4 out_lo = *reinterpret_cast<const u32x4 *>(from + lo), out_hi = *reinterpret_cast<const u32x4 *>(from + hi);
    if (turned) {
        float x[16], cos[8], sin[8];
        unpack8(out_lo, x);
        unpack8(out_hi, x + 8);
        const long long angle = (long long)min(position, a.positions - 1) * a.angles + 8 * piece;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<f32x4 *>(cos + 4 * i) = *reinterpret_cast<const f32x4 *>(a.cos + angle + 4 * i);
            *reinterpret_cast<f32x4 *>(sin + 4 * i) = *reinterpret_cast<const f32x4 *>(a.sin + angle + 4 * i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at_a = a.interleaved ? 2 * i : i, at_b = a.interleaved ? 2 * i + 1 : i + 8;
            const float u = x[at_a], w = x[at_b];
            x[at_a] = u * cos[i] - w * sin[i];
            x[at_b] = w * cos[i] + u * sin[i];
        }
        out_lo = packed8(x);
        out_hi = packed8(x + 8);
    }
    if (is_q && !has_angles) out_lo = out_hi = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
    *reinterpret_cast<u32x4 *>(to + lo) = out_lo;
    *reinterpret_cast<u32x4 *>(to + hi) = out_hi;
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
    a.waves_per_token = ((s.heads + 2 * s.kv_heads) * (a.dim / 16) + 63) / 64;
    const unsigned long long blocks = ((unsigned long long)a.tokens * a.waves_per_token + kWaves - 1) / kWaves;
    if (blocks > kMaxBlocks) return KT_ERR_SHAPE;
    cap_append_kernel<<<dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
    return launched();
}
