// Internal to libktanh: checks of the calls on rows and products in 8-bit integers.  Plain C++.
#pragma once
#include <stdint.h>

#include "ktanh.h"

namespace ktanh_q8 {

constexpr size_t kMostRows = (size_t)1 << 30;       // rows, and output channels
constexpr size_t kMostInner = 131071;               // 128 * 128 * 131071 < 2^31: every sum of products fits 32 bits
constexpr size_t kMostStride = (size_t)1 << 40;
constexpr size_t kMostLanes = ((size_t)1 << 32) - 1;    // of a launch

inline bool off(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
inline size_t stride(size_t rows, size_t step) { return rows > 1 ? step : 0; }     // that of a single row means nothing

// Memory that a call reads or writes: rows of `bytes`, `step` bytes apart.
struct Memory {
    const void *at;
    size_t rows, bytes, step;
};
inline Memory vector(const void *p, size_t bytes) { return Memory{p, 1, bytes, 0}; }
inline Memory matrix(const void *p, size_t rows, size_t row, size_t step, size_t size)
{
    return step == 0 || rows == 1 ? vector(p, row * size) : Memory{p, rows, row * size, step * size};
}

// Whether no byte is in both.  Where their spans cross, of those that are known to be apart by their columns: rows of one stride (or a single row), each
// beside the other's.  Blocks of a launch read while others write, so that no shared byte would be safe.
inline bool apart(const Memory &a, const Memory &b)
{
    if (a.at == nullptr || b.at == nullptr || a.rows == 0 || b.rows == 0 || a.bytes == 0 || b.bytes == 0) return true;
    typedef unsigned __int128 wide;
    const wide a0 = reinterpret_cast<uintptr_t>(a.at), b0 = reinterpret_cast<uintptr_t>(b.at);
    if (a0 + (wide)(a.rows - 1) * a.step + a.bytes <= b0 || b0 + (wide)(b.rows - 1) * b.step + b.bytes <= a0) return true;
    if (a.rows == 1 && b.rows == 1) return false;
    const size_t step = a.rows == 1 ? b.step : a.step;
    if (b.rows != 1 && b.step != step) return false;
    const size_t ahead = (size_t)((b0 % step + step - a0 % step) % step);       // of a row of b behind the nearest start of one of a's
    return ahead >= a.bytes && ahead + b.bytes <= step;
}

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

// Which blocks a product is cut into.  Tiles through LDS (channels by rows), of which `parts` blocks share the inner dimension and leave sums that a second
// launch joins; or blocks of 16 by 16 whose wavefronts share it (SHARED), for few results and short rows.
//
// The plan is the one that takes least by a model of what steps, rounds of blocks, memory and launches cost.  Its numbers are measured, us of calls on
// weights out of the cache, by the model's choice | the others:
//     1 x 4096 x 4096   SHARED 5.9 | 64x64 10.7                  128 x 4096 x 16384   128x64 23.7 | 64x64 26.9, 128x128 27.9, SHARED 139
//    16 x 16384 x 4096  SHARED 23.3 | 64x64 in 4 parts 22.4,     256 x 4096 x 4096    64x64 11.8 | 128x64 14.3, 128x128 19.3
//                       in one 35.5                              512 x 4096 x 4096    128x64 17.2 | 64x64 18.0, 128x128 21.5
//    24 x 2048 x 50000  128x32 23.8 | 128x64 24.9, 64x64 26.5    512 x 16384 x 1024   128x64 in 4 parts 23.6 | in one 54.2
//    64 x 1024 x 1024   SHARED 3.4 | 64x64 5.1                  1024 x 4096 x 4096    128x128 25.3 | 128x64 31.3, 256x256 61.4
//    64 x 4096 x 16384  64x64 19.2 | 128x64 22.9, SHARED 74.5   2048 x 4096 x 4096    128x128 41.1 | 192x256 52.9, 128x64 57.1
//   128 x 4096 x 4096   64x64 11.1 | 128x64 14.0, SHARED 35.5   2048 x 4096 x 6144    192x256 54.2 | 256x256 65.5, 128x128 73.6
//   128 x 1024 x 512    SHARED 3.4 | 64x64 5.1                  8192 x 16384 x 4096   256x256 481 | 128x128 536
// What the model leaves out is the end of rows that fill no tile, with its two barriers and four steps that nothing hides: 777 x 1001 x 2003 takes 11.2 us where it says 6.3.
// Between 128 and 1024 rows its choices are 1.7 to 2.6 times what memory and the matrix cores need: a block of four wavefronts to a CU is one to a SIMD, and nothing runs
// while it waits for LDS and for its tile.
enum Kind { T256, T192, T128, T128_64, T64, T128_32, SHARED };
struct Tile {
    unsigned over, across;      // output channels, rows
    double alone, together;     // us of a step of 128 integers of a block by itself on a CU, and of each of two
};
constexpr Tile kTiles[] = {{256, 256, 1.85, 1.9}, {192, 256, 1.45, 1.48}, {128, 128, 0.94, 0.59}, {128, 64, 0.35, 0.41}, {64, 64, 0.22, 0.216}, {128, 32, 0.22, 0.216}, {16, 16, 0, 0}};
constexpr double kRoomy = 0.71;     // of a T128 block with three places, where every block has a CU of its own

struct Plan {
    Kind kind;
    unsigned parts;
};

inline double blocks_of(Kind kind, size_t rows, size_t outer, unsigned parts)
{
    const Tile &t = kTiles[kind];
    return (double)((outer + t.over - 1) / t.over) * (double)((rows + t.across - 1) / t.across) * parts;
}

inline double us_of(Kind kind, unsigned parts, size_t rows, size_t inner, size_t outer)
{
    const Tile &t = kTiles[kind];
    const double blocks = blocks_of(kind, rows, outer, parts);
    const double rounds = blocks <= 256 ? 1 : (double)(size_t)((blocks + 255) / 256), pairs = (double)(size_t)(rounds / 2);
    double us;
    if (kind == SHARED) us = rounds * (0.5 + 0.48 * (double)((inner + 511) / 512));
    else us = (double)((inner + 128 * parts - 1) / (128 * parts)) * (pairs * 2 * t.together + (rounds - pairs * 2) * (kind == T128 && blocks <= 256 ? kRoomy : t.alone));
    // memory at 5 TB/s, less where not every CU has a block or tiles are read past the last row
    double memory = ((double)rows + (double)outer) * (double)inner / 5e6 * (blocks < 256 ? 1 + (256 - blocks) / 512 : 1);
    memory *= 1.2 - 0.2 * (double)rows / (double)((rows + t.across - 1) / t.across * t.across);
    if (us < memory) us = memory;
    us += kind == SHARED ? 2.5 : 3.5;
    if (parts > 1) us += 2.5 + (double)parts * (double)rows * (double)outer * 8 / 4e6;
    return us;
}

inline Plan plan_of(size_t rows, size_t inner, size_t outer)
{
    Plan best{SHARED, 1};
    double least = us_of(SHARED, 1, rows, inner, outer);
    for (int kind = T256; kind < SHARED; ++kind)
        for (unsigned parts = 1; parts <= 8; parts *= 2) {
            if (parts > 1 && (kind <= T192 || inner / 128 < 4 * parts)) break;      // four tiles for each at least
            const double us = us_of((Kind)kind, parts, rows, inner, outer);
            if (us < least) {
                least = us;
                best = Plan{(Kind)kind, parts};
            }
        }
    return best;
}

// The kernel that a product takes: tiles; or, where operands are off the 16-byte grid or a tile's offsets would leave 32 bits, blocks of 16 by 16 or of 64 by 64 whose
// wavefronts share the inner dimension.  Large ones from two of the small ones on each CU on (300 x 300 x 300 6.3 us against 10.5, 2000 x 200 x 5000 258 against 41).
enum Way { TILES, SHARED16, SHARED64 };
inline Way way_of(const Plan &plan, size_t rows, size_t outer, bool aligned, size_t x_row, size_t w_row)
{
    if (aligned && plan.kind != SHARED && x_row < (size_t)1 << 23 && w_row < (size_t)1 << 23) return TILES;
    return plan.kind == SHARED || rows <= 32 || ((rows + 15) / 16) * ((outer + 15) / 16) <= 512 ? SHARED16 : SHARED64;
}

// Rows and channels of one launch: fewer than 2^32 lanes, and where the grid has two dimensions at most 65535 blocks of rows.
struct Piece {
    size_t rows, outer;
};
inline Piece piece_of(Way way, const Plan &plan, size_t rows, size_t outer)
{
    const size_t over = way == TILES ? kTiles[plan.kind].over : way == SHARED16 ? 16 : 64, across = way == TILES ? kTiles[plan.kind].across : over;
    const size_t most = kMostLanes / (way == SHARED16 ? 512 : 256) / (way == TILES ? plan.parts : 1);
    size_t channels = (outer + over - 1) / over;
    if (channels > most) channels = most;
    const size_t row_blocks = way == TILES ? most / channels : 65535;
    return Piece{rows < row_blocks * across ? rows : row_blocks * across, outer < channels * over ? outer : channels * over};
}

// A call's workspace: codes that it makes itself (rows of a multiple of 16 bytes, then the scales), and the sums of parts.
inline size_t padded(size_t inner) { return (inner + 15) / 16 * 16; }
inline size_t rows_bytes(const kq8_shape_t &s) { return (s.rows * (padded(s.inner) + sizeof(float)) + 15) / 16 * 16; }
inline size_t sums_bytes(const kq8_shape_t &s)
{
    if (s.rows == 0 || s.outer == 0) return 0;
    const unsigned parts = plan_of(s.rows, s.inner, s.outer).parts;
    return parts > 1 ? s.rows * s.outer * sizeof(int32_t) * parts : 0;
}

// Few short rows and their product in one launch, where that is the faster way (*done), with either table.
ktanh_status_t launch_few(const kq8_shape_t &s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, const ktanh_lut_t *lut,
                          const ktanh_lut64_t *lut64, bool wide, ktanh_stream_t stream, bool *done);

}  // namespace ktanh_q8
