// Prints, for each codebook read from stdin (bits, then 2^bits levels), the
// values that attention's forms of it stand for, level by level: two and three
// digits (build_value_digits), in fp16 (build_half_levels, with the error it
// reports first), with what that leaves in e4m3, and in e4m3.
#include <cmath>
#include <cstdio>
#include <cstring>

#include "isoq_attn_tables.h"

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

static double byte(const isoq::HalfLevels &h, int t, int at)
{
    const int v = reinterpret_cast<const uint8_t *>(h.tab[t])[at], e = v >> 3 & 15, m = v & 7;
    const double x = e == 0 ? std::ldexp(m, -9) : std::ldexp(8 + m, e - 10);
    return (v & 127) == 127 ? NAN : v & 128 ? -x : x;
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
        isoq::HalfLevels h;
        const double off = isoq::build_half_levels(bits, lev, h);
        for (int form = 0; form < 3; form++) {
            if (form == 0)
                std::printf("%.17g ", off);
            for (int k = 0; k < K; k++) {
                const int at = bits < 4 ? k : k >= 8 ? k - 8 : 7 - k;
                const double v = form == 2   ? byte(h, 2, at)
                                 : form == 1 ? half(h, 0, at) + std::ldexp(byte(h, 3, at), -isoq::kLevelRest)
                                             : half(h, 0, at);
                std::printf("%.17g ", (bits == 4 && k < 8 ? -v : v) * h.scale);
            }
            std::printf("\n");
        }
    }
    return 0;
}
