// Which kernel a product takes and how it is cut into launches: reads lines "rows inner outer aligned x_row w_row", writes "way tile-channels tile-rows parts
// piece-rows piece-channels" for each.
#include <cstdio>

#include "ktanh_q8.h"

int main()
{
    using namespace ktanh_q8;
    size_t rows, inner, outer, x_row, w_row;
    int aligned;
    while (std::scanf("%zu %zu %zu %d %zu %zu", &rows, &inner, &outer, &aligned, &x_row, &w_row) == 6) {
        const Plan plan = plan_of(rows, inner, outer);
        const Way way = way_of(plan, rows, outer, aligned != 0, x_row, w_row);
        const Piece piece = piece_of(way, plan, rows, outer);
        const Tile &t = kTiles[plan.kind];
        std::printf("%d %u %u %u %zu %zu\n", (int)way, t.over, t.across, plan.parts, piece.rows, piece.outer);
    }
    return 0;
}
