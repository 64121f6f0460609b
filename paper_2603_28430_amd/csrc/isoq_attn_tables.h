// The codebook in the forms that attention multiplies with, built on the host
// once per handle, by its first attention.
#pragma once

#include <cstdint>

namespace isoq {

// The codebook as 8-bit digits for the weighted sums of attention (isoq_attn_m.h):
// byte k of tab[t] is digit t (least significant first) of level k's integer,
// n_k = d_0 + 256 d_1 (+ 65536 d_2), and scale n_k the level.  At 4 bits of the
// positive level of magnitude k, which is scale (n_k + half), half = (1 + 256 (+
// 65536)) / 2: the complement of the digits then stands for its mirror image.
struct ValueDigits {
    uint32_t tab[3][2];
    float scale;
};

// The codebook in fp16 for attention of many rows (isoq_attn_c.h): byte k of
// tab[0] and tab[1] are the low and high byte of level k's fp16 value in units of
// scale, of tab[2] its e4m3 value, of tab[3] that of 2^kLevelRest times what fp16
// leaves of it, and of tab[4] and tab[5] the bytes of that in fp16.  At 4 bits of
// the positive level of magnitude k.
struct HalfLevels {
    uint32_t tab[6][2];
    float scale;
};

// The levels as integers of `digits` (2 or 3) balanced 8-bit digits.  The scale
// is searched for the least sum of squared errors over the levels; the largest
// level's integer is at least half of what the digits hold.
void build_value_digits(int bits, const float *levels, int digits, ValueDigits &out);
// The levels in units searched for the least sum of the squares of what fp16
// leaves of them (the largest level is 1 .. 2).  Returns the most that it leaves
// of a level, relative to it.
double build_half_levels(int bits, const float *levels, HalfLevels &out);
// What is multiplied of what fp16 leaves of the keys' levels (isoq_attn_c.h):
// nothing where that is 2^-20 of them at most; in e4m3, times the query in e4m3,
// which leaves 2^-4.8 of it, where it is 2^-14.8 (Lloyd-Max levels of 3 bits: 2^-15);
// else in fp16 (of 4 bits: 2^-11.8).
enum { kRestNone, kRestBytes, kRestHalves };
constexpr double kLeftNone = 0x1p-20, kLeftBytes = 0x1.2p-15;
// (2^-11 at most, so 2^8 in e4m3, whose largest is 448)
constexpr int kLevelRest = 19;

struct AttnTables {
    ValueDigits vd[2];   // of two digits (fp16 queries), three (fp32)
    HalfLevels half;
    int key_rest;        // the form of what fp16 leaves of the keys' (kRestNone ..)
};

}  // namespace isoq
