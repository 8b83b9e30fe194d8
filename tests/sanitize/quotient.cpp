// Host comparison of the appended rows' quotient with a division: every fraction of the
// scale, at a few exponents, times values at and beside each tie of E4M3's codes (normal
// and subnormal ones), and values at random: the codes, and the bits where no intermediate
// is below fp32's range.  Prints "ok <pairs>" or the first difference.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "quotient.hpp"

namespace {
long pairs = 0;
float of_bits(uint32_t b) {
  float f;
  std::memcpy(&f, &b, 4);
  return f;
}
// The value of a quotient's code: 2^-9 apart below 2^-6, three bits of fraction above.
float code(float q) {
  int e;
  std::frexp(q, &e);
  const int step = std::max(e - 4, -9);
  return std::ldexp(std::nearbyint(std::ldexp(q, -step)), step);
}
void compare(float y, float scale, float inverse) {
  const float want = y / scale, got = splash::quotient<true>(y, scale, inverse), open = splash::quotient<false>(y, scale, inverse);
  ++pairs;
  if (std::fabs(want) > 449.f) return;  // (no value of a row: the scale is its largest over 448)
  const bool bits = scale >= 0x1p-90f && (std::fabs(want) >= 0x1p-11f || want == 0.f);
  if (std::memcmp(&got, &open, 4) || (bits && std::memcmp(&want, &got, 4)) || code(want) != code(got) || std::signbit(want) != std::signbit(got)) {
    std::printf("FAILED %a / %a: %a, not %a\n", y, scale, got, want);
    std::exit(1);
  }
}
}  // namespace

int main() {
  const int exponents[] = {-100, -90, 0, 100};
  const float ties[] = {17.f / 16, 19.f / 16, 21.f / 16, 23.f / 16, 25.f / 16, 27.f / 16, 29.f / 16, 31.f / 16, 0x1p-10f, 3 * 0x1p-10f, 448.f};
  std::mt19937 rng(3);
  for (uint32_t f = 0; f < 1u << 23; ++f) {
    const float scale = std::ldexp(of_bits(0x3f800000u | f), exponents[f & 3]), inverse = 1.f / scale;
    for (const float tie : ties) {
      const float y = (float)((double)tie * scale);
      compare(y, scale, inverse);
      compare(std::nextafterf(y, 0.f), scale, inverse);
      compare(-std::nextafterf(y, 3e38f), scale, inverse);
    }
    compare(std::ldexp(of_bits(0x3f800000u | (rng() & 0x7fffffu)), (int)(rng() % 20) - 11) * scale, scale, inverse);
    compare(f & 1 ? 0.f : -0.f, scale, inverse);
  }
  std::printf("ok %ld\n", pairs);
  return 0;
}
