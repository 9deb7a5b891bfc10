// The plans of calls over documents: reads lines "docs rows heads kv_heads dim causal window", writes "split_tiles, keys' split, keys' parts" for each.
#include <cstdio>

#include "ktanh_cap_plan.h"

int main()
{
    kcap_shape_t s{};
    while (std::scanf("%zu %zu %zu %zu %zu %d %zu", &s.docs, &s.q_rows, &s.heads, &s.kv_heads, &s.dim, &s.causal, &s.window) == 7) {
        s.k_rows = s.q_rows;
        const ktanh_cap::KeysPlan plan = ktanh_cap::keys_plan(s);
        std::printf("%d %d %d\n", ktanh_cap::split_tiles(s), plan.split, plan.parts);
    }
    return 0;
}
