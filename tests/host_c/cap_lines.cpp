// The lines that kt_pack_cap and kt_pack_cap64 form, against shift and add on every interval's ends.
#include <cmath>
#include <cstdio>

#include "ktanh_pack.h"

static int bad = 0;

static void check(const KtCapPack &pack, int intervals, const uint8_t *E, const uint8_t *r, const int8_t *b)
{
    for (int t = 0; t < 64; ++t) {
        const int u = intervals == 64 ? t : t >> 1, e_in = 125 + (((t >> 4) - 125) & 3);
        for (int m = (t & 15) * 8; m < (t & 15) * 8 + 8; ++m) {
            const double x = std::ldexp(1.0 + m / 128.0, e_in - 127);
            // with the bits that the shift drops
            const double want = std::ldexp(1.0 + m / 128.0 * std::ldexp(1.0, -r[u]) + b[u] / 128.0, E[u] - 127);
            if ((double)pack.a[t] * x + (double)pack.b[t] != want) ++bad;
        }
    }
}

int main()
{
    KtCapPack pack, same;
    ktanh_lut_t t32 = *ktanh_default_lut();
    ktanh_lut64_t t64;
    if (kt_pack_cap(nullptr, &pack) != KT_OK || kt_pack_cap(&t32, &same) != KT_OK) return 1;
    check(pack, 32, t32.E, t32.r, t32.b);
    check(same, 32, t32.E, t32.r, t32.b);
    ktanh_fit_lut64(&t64);
    if (kt_pack_cap64(nullptr, &pack) != KT_OK || kt_pack_cap64(&t64, &same) != KT_OK) return 1;
    check(pack, 64, t64.E, t64.r, t64.b);
    check(same, 64, t64.E, t64.r, t64.b);
    ktanh_fit_lut_bmin0(&t32);
    if (kt_pack_cap(&t32, &pack) != KT_OK) return 1;
    check(pack, 32, t32.E, t32.r, t32.b);
    t32.E[0] = 127;  // K above 1
    if (kt_pack_cap(&t32, &pack) != KT_ERR_LUT) return 1;
    t32.r[0] = 8;    // no valid table
    if (kt_pack_cap(&t32, &pack) != KT_ERR_LUT) return 1;
    std::puts(bad == 0 ? "lines agree" : "lines differ");
    return bad != 0;
}
