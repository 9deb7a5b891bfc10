// Internal to libktanh: arguments of the capped-attention kernels and the checks that their entry points share.
#pragma once
#include <cmath>

#include "ktanh_cap.h"
#include "ktanh_cap_plan.h"

namespace ktanh_cap {

// A launch holds fewer than 2^32 work-items.
constexpr unsigned long long kMaxBlocks = (1ull << 32) / kThreads - 8;

struct CapShape {
    int docs, q_rows, k_rows, heads, kv_heads, group;
    int causal, window;
    float scale, to_x, cap;  // to_x = scale / cap, formed in double and rounded once
    Rows q, k, v;
};

inline bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Checks what every entry point takes and fills `out`.
inline ktanh_status_t read_shape(const kcap_shape_t *s, const uint16_t *q, const uint16_t *k, const uint16_t *v, CapShape *out)
{
    constexpr size_t kMost = 1u << 30;  // places of rows and sums of two of them fit 32 bits
    if (s->dim != 64 && s->dim != 128) return KT_ERR_SHAPE;
    if (s->heads == 0 || s->kv_heads == 0 || s->heads % s->kv_heads != 0) return KT_ERR_SHAPE;
    if (s->docs > kMost || s->q_rows > kMost || s->k_rows > kMost || s->heads > 65536) return KT_ERR_SHAPE;
    if (!(s->cap > 0.0 && s->cap <= KCAP_MAX)) return KT_ERR_SHAPE;
    if (!std::isfinite((float)s->scale) || !std::isfinite((float)(s->scale / s->cap))) return KT_ERR_SHAPE;
    for (size_t stride : {s->q_row, s->q_head, s->k_row, s->k_head, s->v_row, s->v_head}) {
        if (stride % 8 != 0) return KT_ERR_ALIGN;
        if (stride >= (size_t)1 << 24) return KT_ERR_SHAPE;
    }
    if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return KT_ERR_ALIGN;
    out->docs = (int)s->docs;
    out->q_rows = (int)s->q_rows;
    out->k_rows = (int)s->k_rows;
    out->heads = (int)s->heads;
    out->kv_heads = (int)s->kv_heads;
    out->group = (int)(s->heads / s->kv_heads);
    out->causal = s->causal != 0;
    out->window = s->window > kMost ? 0 : (int)s->window;  // wider than any row of keys: none
    out->scale = (float)s->scale;
    out->to_x = (float)(s->scale / s->cap);
    out->cap = (float)s->cap;
    out->q = Rows{q, (long long)s->q_row, (long long)s->q_head};
    out->k = Rows{k, (long long)s->k_row, (long long)s->k_head};
    out->v = Rows{v, (long long)s->v_row, (long long)s->v_head};
    return KT_OK;
}

inline ktanh_status_t launched() { return hipGetLastError() == hipSuccess ? KT_OK : KT_ERR_HIP; }

inline ktanh_status_t pack_lines(const ktanh_lut_t *lut, KtCapPack *pack) { return kt_pack_cap(lut, pack); }
inline ktanh_status_t pack_lines(const ktanh_lut64_t *lut, KtCapPack *pack) { return kt_pack_cap64(lut, pack); }

// Keys and values in pages: key j of sequence s is row j % 2^shift of page pages[s * row + (j >> shift)].
struct CapPages {
    const int *pages;
    const int *lengths;  // keys of each sequence
    long long row;
    int most, shift, count;
    uint32_t k_page, v_page;  // strides in elements
};

// Products of two 32-bit numbers in 64 bits: one instruction, where strides of 64 bits take five.
__device__ __forceinline__ unsigned long long wide(int a, uint32_t b) { return (unsigned long long)(uint32_t)a * b; }

__device__ __forceinline__ int keys_in_pages(const CapPages &p, int sequence)
{
    return min(max(p.lengths[sequence], 0), p.most << p.shift);
}

// Checks a page table and its cache; the tensors of the cache themselves may be NULL where there are no pages.
inline ktanh_status_t read_pages(const kcap_pages_t *p, const int32_t *pages, const int32_t *lengths, const uint16_t *k, const uint16_t *v,
                                 CapPages *out)
{
    if (pages == nullptr || lengths == nullptr || k == nullptr || v == nullptr) return KT_ERR_NULL;
    if (p->page_size == 0 || (p->page_size & (p->page_size - 1)) != 0 || p->page_size > 1u << 20) return KT_ERR_SHAPE;
    if (p->page_count == 0 || p->page_count > 0x7FFFFFFF || p->table_row > (size_t)1 << 40) return KT_ERR_SHAPE;
    if (p->most == 0 || p->most > (1u << 30) / p->page_size) return KT_ERR_SHAPE;
    for (size_t stride : {p->k_page, p->k_slot, p->k_head, p->v_page, p->v_slot, p->v_head}) {
        if (stride % 8 != 0) return KT_ERR_ALIGN;
        if (stride >= (size_t)1 << 31) return KT_ERR_SHAPE;
    }
    if (!aligned16(k) || !aligned16(v)) return KT_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(pages) % 4 != 0 || reinterpret_cast<uintptr_t>(lengths) % 4 != 0) return KT_ERR_ALIGN;
    out->pages = pages;
    out->lengths = lengths;
    out->row = (long long)p->table_row;
    out->most = (int)p->most;
    out->shift = __builtin_ctzll(p->page_size);
    out->count = (int)p->page_count;
    out->k_page = (uint32_t)p->k_page;
    out->v_page = (uint32_t)p->v_page;
    return KT_OK;
}

// Rows of a stretch, as a power of two: of a block whose wavefronts share tiles, or of one with as many query
// heads of a group together as its four wavefronts can have.  16 documents of 8192 tokens, 32 heads of 128 on
// 8: 108.7 us with one head, 102.4 with four; 4 tokens each behind up to 2000 of 64 sequences 109 and 70.
inline int rows_shift(const CapShape &s, bool split) { return split ? 5 : 7 - __builtin_ctz((unsigned)heads_together((size_t)s.group)); }
inline unsigned long long stretches(size_t rows, size_t docs, int shift) { return (rows >> shift) + docs; }

// Many queries of each sequence over the cache (ktanh_cap_forward.hip).  Where parts are above 1 the workspace
// holds forward_sums Float32 sums and as many times dim numerators.
struct ForwardPlan {
    bool split;
    int parts;
};
ForwardPlan forward_plan(const kcap_shape_t &s, const kcap_pages_t &p);
inline size_t forward_sums(size_t parts, size_t rows, size_t heads) { return (parts * rows * heads + 31) / 32 * 32; }
ktanh_status_t launch_forward_paged(const CapShape &s, const CapPages &p, const int *q_offsets, uint16_t *o, int dim,
                                    ForwardPlan plan, float *workspace, const KtCapPack &pack, ktanh_stream_t stream);

}  // namespace ktanh_cap
