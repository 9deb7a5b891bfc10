// Whether two pieces of memory of a call on 8-bit integers are apart: reads lines "at rows bytes step at rows bytes step", writes 1 or 0 for each.
#include <cstdio>

#include "ktanh_q8.h"

int main()
{
    ktanh_q8::Memory m[2];
    unsigned long long at[2];
    while (std::scanf("%llu %zu %zu %zu %llu %zu %zu %zu", &at[0], &m[0].rows, &m[0].bytes, &m[0].step, &at[1], &m[1].rows, &m[1].bytes, &m[1].step) == 8) {
        for (int i = 0; i < 2; ++i) m[i].at = reinterpret_cast<const void *>(at[i]);
        std::printf("%d\n", ktanh_q8::apart(m[0], m[1]));
    }
    return 0;
}
