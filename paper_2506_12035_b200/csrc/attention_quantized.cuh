// What the two attention kernels over the 8-bit cache share: the units of their sums.
//
// O is summed up from weights p vs, rounded to fp16 relative to a power of two, the unit, and p is relative to a reference, 2^(x - ref).  Ordinarily
// the unit lies above all value scales met so far and the reference is the row's largest logit (or near it).  Value scales that lie far apart break
// that: a key with a scale far above the others' may have no weight, and beside it theirs would be nothing.  A sample and head whose scales are more
// than 2^spread apart is wide from the tile on in which that shows:
//   the reference of a row is its largest x + log2(vs / unit), so that its largest product is the unit's; but not more than 2^kBelow below a key's own
//   logit, so that the sum of weights, which is relative to it as well, stays in fp32's range;
//   the unit, which all rows share, stays at most 2^kAboveLow above the smallest scale and at most 2^kBelowTop below the largest.  When it rises by
//   2^d, the references fall by d: products over the unit, and with them O, stay as they are, and the sums of weights rise by 2^d.
// Scales of 16-bit numbers that lie up to 2^125 apart keep to both: a row's largest product is at least 2^-5 of what fp16 holds, and sums of weights
// stay between 2^-85 and 2^125.
// Samples that are not wide pay for finding that out (a running minimum per tile): one token over 4 x 65521 keys at most 88.9 -> 90.5 us, 128 x 43 rows
// over 320 keys 65.5 us before and after.  A wide one pays 2 to 4 % in the mma.sync kernel, half again as much in the tcgen05 one (64 logarithms a row and tile).
#pragma once

#include "common.cuh"

namespace marche {
namespace attq {

constexpr int kAboveLow = 50, kBelowTop = 75;
constexpr float kBelow = 45.f;

MARCHE_DEVINL float pow2(int biased_exponent) { return __int_as_float(biased_exponent << 23); }
MARCHE_DEVINL uint32_t magnitude(float scale) { return __float_as_uint(scale) & 0x7fffffffu; }
MARCHE_DEVINL float lg2_approx(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Magnitudes of two 16-bit numbers at once: the larger ones, and the smaller ones that are not 0, less 1.
MARCHE_DEVINL uint32_t larger2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
MARCHE_DEVINL uint32_t smaller2_less_1(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("{\n.reg .b32 t;\nadd.u16x2 t, %2, %3;\nmin.u16x2 %0, %1, t;\n}" : "=r"(r) : "r"(a), "r"(b), "r"(0xffffffffu));
  return r;
}
// Of both halves of a word the larger one that is a finite bf16 number's magnitude, or 0.
MARCHE_DEVINL uint32_t finite_of(uint32_t w) {
  const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
  return max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u);
}

// The largest value scale so far by magnitude and the unit, as biased exponents, and a lane's smallest scale so far that is not 0.
struct Units {
  int top = 14, unit = 14;                                 // (14: the lowest whose factors exist)
  uint32_t low = 0xffffffffu;                              // as bits less 1
  bool wide = false;
  // Takes in a tile's largest scale and the smallest that is not 0 of the lane's, less 1 (0xffffffff: none), as magnitudes' bits, which order as
  // integers; NaN counts as the largest number.
  MARCHE_DEVINL void see(uint32_t largest, uint32_t smallest_less_1) {
    top = max(top, min((int)(largest >> 23), 254));
    low = min(low, smallest_less_1);
  }
  // The sample is wide if any lane's scales are apart.  Once they are, they stay so.
  template <int SPREAD> MARCHE_DEVINL bool apart() const { return low < (uint32_t)max(top - SPREAD, 0) << 23; }
  // The unit for what has been seen, by all lanes of the warp; returns by how many powers of two it rises.
  MARCHE_DEVINL int move(bool is_wide, bool first) {
    wide = is_wide;
    const int before = first ? top : unit;
    int d = top - before;
    if (__builtin_expect(wide, 0)) {
      const int lowest = max((int)((__reduce_min_sync(0xffffffffu, low) + 1u) >> 23) + kAboveLow, 14);
      d = min(max(max(min(before, lowest), top - kBelowTop) - before, -100), 100);
    }
    unit = before + d;
    return first ? 0 : d;
  }
};
// What O is multiplied by when the unit rises by d and the references stay (where it rises this far, O is nothing beside it).
MARCHE_DEVINL float step_of(int d) { return d > 126 ? 0.f : pow2(127 - d); }
// What a key's logit counts for its row's reference in a wide sample: log2 of its scale over the unit, at least -kBelow.
MARCHE_DEVINL float counts(float scale_over_unit) { return fmaxf(lg2_approx(fabsf(scale_over_unit)), -kBelow); }

// unit / l as two factors that leave fp32's range neither by themselves nor multiplied one after the other: 1 / l's mantissa, and the powers of two
// (what of them is too small for one number goes to the first).  l 0 (no key): zeros; NaN stays.
MARCHE_DEVINL float2 unit_over(float l, int biased_unit) {
  const int power = biased_unit + 127 - (int)(__float_as_uint(l) >> 23);
  const float inv = 1.0f / __int_as_float((__float_as_int(l) & 0x7fffff) | 0x3f800000);
  return make_float2(l > 0.f ? inv * pow2(127 + max(min(power - 1, 0), -100)) : l, pow2(min(max(power, 1), 254)));
}

}  // namespace attq
}  // namespace marche
