// The plans of products in 8-bit integers: reads lines "rows inner outer", writes "kind over across parts bytes-of-sums" for each.
#include <cstdio>

#include "ktanh_q8.h"

int main()
{
    kq8_shape_t s{};
    while (std::scanf("%zu %zu %zu", &s.rows, &s.inner, &s.outer) == 3) {
        const ktanh_q8::Plan plan = ktanh_q8::plan_of(s.rows, s.inner, s.outer);
        const ktanh_q8::Tile &t = ktanh_q8::kTiles[plan.kind];
        std::printf("%d %u %u %u %zu\n", (int)plan.kind, t.over, t.across, plan.parts, ktanh_q8::sums_bytes(s));
    }
    return 0;
}
