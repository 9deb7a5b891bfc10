// Internal to libktanh: how the work of the capped attention over documents is cut into blocks.  Host code,
// from what is known on the host: numbers of documents, rows and heads, but not how the rows are dealt to the
// documents.
#pragma once
#include <algorithm>
#include <cmath>

#include "ktanh.h"

namespace ktanh_cap {

// Query heads of a group that a block has together.
inline int heads_together(size_t group) { return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1; }

// Whether blocks hold 32 queries, their wavefronts sharing the tiles of keys, rather than 32 in each: the
// shorter time of the block that takes longest, or of all blocks, by what they take for a tile alone, a compute
// unit with all that it holds, and around their tiles.  Documents count as 1.2 times as long as the average.
// Output, then gradients, causal, in us, wavefronts of their own rows | sharing the tiles:
//    1024 rows,  8 heads of 128 on 8        36  63 |  15  39
//    4096 rows,  8 heads of 128 on 8       128 245 |  65 179
//    1500 rows, 32 heads of 128 on 8        51 130 |  45 128
//    2048 rows, 32 heads of 128 on 8        68 218 |  72 229
//    eight documents of 256, 32 heads on 8  17  50 |  39  82
//    8192 rows,  5 heads of 128 on 1       249 561 | 144 459
//    a document of 32 rows, 8 heads of 64  4.7 10.3 | 5.0 11.3
// and the output alone:
//    four documents of 1250, 16 heads on 4      52 |  84
//    four of 700, 16 heads of 128 on 16         33 |  41
//    four of 700, 8 heads of 64 on 2            24 |  16
//    20 at random, 10000 rows, 5 heads on 1     65 |  52
inline bool split_tiles(const kcap_shape_t &s)
{
    if (s.k_rows <= 32 * s.docs) return false;  // one tile cannot be shared
    const double docs = (double)s.docs, queries = (double)s.q_rows / docs, keys = (double)s.k_rows / docs;
    const bool narrow = s.window > 0 && (double)s.window + 128.0 < keys;
    const double seen = narrow ? (double)s.window + 128.0 : keys, mean = s.causal && !narrow ? 0.5 : 1.0;
    const double longest = docs > 1.0 && !narrow ? 1.2 : 1.0;
    const double together = heads_together(s.heads / s.kv_heads);
    const double own_blocks = std::ceil(queries * together / 128.0) * docs * (double)s.heads / together, own_tiles = seen / 32.0;
    const double sharing_blocks = std::ceil(queries / 32.0) * docs * (double)s.heads, sharing_tiles = seen / 128.0;
    const double rounds = (s.dim == 64 ? 0.6 : 1.0) / 256.0;  // of heads of 64 a compute unit holds more
    return std::max(5.0 + 1.35 * longest * sharing_tiles, rounds * sharing_blocks * (0.85 * mean * sharing_tiles + 3.2)) <
           std::max(3.0 + 1.03 * longest * own_tiles, rounds * own_blocks * (0.57 * mean * own_tiles + 3.5));
}

// How the blocks over keys are cut: their rows, and into how many parts the query heads that share a key/value
// head are dealt, each with a block and sums in Float32 of its own that another kernel adds up.
struct KeysPlan {
    bool split;
    int parts;
};

// The least time of all: of the block that takes longest, or of all blocks with some of that one's at their
// end, by what a block takes for a tile alone, and a compute unit with all that it holds, and around its tiles;
// and of the parts written and read.  Documents count as 1.6 times as long as the average.  Fitted to 754 calls
// with 5 to 40 heads and held against 523 more: 1.5 % above the best plan on average (documents alike or only
// one 1.2, of evenly spread lengths 0.8, cut at random 2.7), 1.4 % of them more than 20 % above.  Gradients
// causal, in us with four | two | one part | one part in blocks of 32 rows:
//    six documents, 8192 rows at random, 32 heads of 128 on 8    934 |  988 | 1338 |  905
//    64 documents of 256                                         526 |  413 |  334 |  413
//    32 documents of 256                                         283 |  228 |  185 |  245
//    16 documents of 256                                         140 |  114 |  121 |  111
//    eight documents of 2048                                    1411 | 1291 | 1267 | 1341
//    one of 8192                                                2100 | 2198 | 2700 | 2291
//    64 documents of 256, 8 heads of 64 on 2                      74 |   67 |   77 |   53
inline KeysPlan keys_plan(const kcap_shape_t &s)
{
    KeysPlan best{false, 1};
    if (s.docs == 0 || s.kv_heads == 0 || s.heads < s.kv_heads) return best;
    const int group = (int)(s.heads / s.kv_heads);
    const double docs = (double)s.docs, queries = (double)s.q_rows / docs, keys = (double)s.k_rows / docs;
    double least = 0.0;
    for (const bool split : {false, true}) {
        if (split && s.q_rows <= 32 * s.docs) break;  // one tile cannot be shared
        const double rows = split ? 32.0 : 128.0, at_once = split ? 4.0 : 1.0, alone_us = split ? 2.3 : 1.8;
        const double all_us = s.dim == 64 ? 0.9 : split ? 1.2 : 1.05, around_us = (split ? 12.0 : 6.0) * (s.dim == 64 ? 0.5 : 1.0);
        const bool narrow = s.window > 0 && (double)s.window + rows < queries;
        const double tiles = (narrow ? (double)s.window + rows : queries) / 32.0 / at_once, mean = s.causal && !narrow ? tiles / 2.0 : tiles;
        for (int parts = 1; parts <= group; ++parts) {
            if (group % parts != 0) continue;
            const double heads = group / parts, blocks = std::ceil(keys / rows) * docs * (double)s.kv_heads * parts;
            const double longest = heads * tiles * (s.docs > 1 && !narrow ? 1.6 : 1.0) * alone_us;
            const double all = blocks * heads * mean * all_us / 256.0 + around_us * blocks / 512.0;
            const double join = parts > 1 ? 5.0 + parts * (double)s.k_rows * (double)s.kv_heads * (double)s.dim * 16.0 / 6e6 : 0.0;
            const double t = std::max(longest, all + 0.3 * longest) + join;
            if (least == 0.0 || t < least) {
                least = t;
                best = KeysPlan{split, parts};
            }
        }
    }
    return best;
}

}  // namespace ktanh_cap
