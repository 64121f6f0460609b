// Prints, for each codebook read from stdin (bits, then 2^bits levels), the
// values that attention's forms of it stand for, level by level: two and three
// digits (build_value_digits), one and two fp16 parts (build_half_levels, with
// the error it reports first).
#include <cmath>
#include <cstdio>
#include <cstring>

#include "isoq_internal.h"

static int digit(const isoq::ValueDigits &v, int t, int at)
{
    return (int)reinterpret_cast<const signed char *>(v.tab[t])[at];
}

static double half(const isoq::HalfLevels &h, int t, int at)
{
    const uint16_t bits = (uint16_t)(reinterpret_cast<const uint8_t *>(h.tab[t])[at] |
                                     reinterpret_cast<const uint8_t *>(h.tab[t + 1])[at] << 8);
    _Float16 v;
    std::memcpy(&v, &bits, 2);
    return (double)v;
}

int main()
{
    int bits;
    while (std::scanf("%d", &bits) == 1) {
        const int K = 1 << bits;
        float lev[16];
        for (int k = 0; k < K; k++)
            if (std::scanf("%f", lev + k) != 1)
                return 1;
        for (int digits = 2; digits <= 3; digits++) {
            isoq::ValueDigits v;
            isoq::build_value_digits(bits, lev, digits, v);
            for (int k = 0; k < K; k++) {
                // 4 bits: magnitude k - 8, or the complement of magnitude 7 - k
                const int at = bits < 4 ? k : k >= 8 ? k - 8 : 7 - k;
                long n = 0;
                for (int t = digits - 1; t >= 0; t--) {
                    const int d = digit(v, t, at);
                    n = 256 * n + (bits == 4 && k < 8 ? ~d : d);
                }
                const double offset = bits < 4 ? 0.0 : digits == 2 ? 128.5 : 32896.5;
                std::printf("%.17g ", ((double)n + offset) * v.scale);
            }
            std::printf("\n");
        }
        for (int pair = 0; pair < 2; pair++) {
            isoq::HalfLevels h;
            std::printf("%.17g ", isoq::build_half_levels(bits, lev, pair, h));
            for (int k = 0; k < K; k++) {
                const int at = bits < 4 ? k : k >= 8 ? k - 8 : 7 - k;
                const double v = (half(h, 0, at) + (pair ? half(h, 2, at) : 0.0)) * h.scale;
                std::printf("%.17g ", bits == 4 && k < 8 ? -v : v);
            }
            std::printf("\n");
        }
    }
    return 0;
}
