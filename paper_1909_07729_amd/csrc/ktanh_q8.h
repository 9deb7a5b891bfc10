// Internal to libktanh: checks of the calls on rows and products in 8-bit integers.  Plain C++.
#pragma once
#include <stdint.h>

#include "ktanh.h"

namespace ktanh_q8 {

constexpr size_t kMostRows = (size_t)1 << 30;       // rows, and output channels
constexpr size_t kMostInner = 131071;               // 128 * 128 * 131071 < 2^31: every sum of products fits 32 bits
constexpr size_t kMostStride = (size_t)1 << 40;

inline bool off(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
inline size_t stride(size_t rows, size_t step) { return rows > 1 ? step : 0; }     // that of a single row means nothing

inline ktanh_status_t check_rows(const kq8_shape_t *s)
{
    if (s == nullptr) return KT_ERR_NULL;
    if (s->activation < KQ8_NONE || s->activation > KQ8_GELU || s->rows > kMostRows || s->inner > kMostRows || s->x_row > kMostStride)
        return KT_ERR_SHAPE;
    return KT_OK;
}

inline ktanh_status_t check_product(const kq8_shape_t *s)
{
    if (s == nullptr) return KT_ERR_NULL;
    if (s->rows > kMostRows || s->outer > kMostRows || s->inner > kMostInner || s->x_row > kMostStride || s->w_row > kMostStride ||
        s->out_row > kMostStride || (s->rows > 1 && s->out_row < s->outer))
        return KT_ERR_SHAPE;
    return KT_OK;
}

// Codes of a call that makes its own: rows of a multiple of 16 bytes, then the scales.
inline size_t padded(size_t inner) { return (inner + 15) / 16 * 16; }

}  // namespace ktanh_q8
