// A rotation's frequencies as turns, on the host: rounded once, so that an angle is off by
// no more than the 64 bits that a frequency is held in.
#pragma once

#include <math.h>
#include <stdint.h>

namespace palq {

// The first 1216 binary places of 1 / (2 pi), the highest first.
constexpr uint64_t kTurnsOfRadian[19] = {
    0x28be60db9391054a, 0x7f09d5f47d4d3770, 0x36d8a5664f10e410, 0x7f9458eaf7aef158,
    0x6dc91b8e909374b8, 0x01924bba82746487, 0x3f877ac72c4a69cf, 0xba208d7d4baed121,
    0x3a671c09ad17df90, 0x4e64758e60d4ce7d, 0x272117e2ef7e4a0e, 0xc7fe25fff7816603,
    0xfbcbc462d6829b47, 0xdb4d9fb3c9f2c26d, 0xd3d18fd9a797fa8b, 0x5d49eeb1faf97c5e,
    0xcf41ce7de294a4ba, 0x9afed7ec47e35742, 0x1580cc11bf1edaea};

// freq / (2 pi) modulo 1 in 2^-64, to the nearest; freq finite.  With freq = m 2^e, m below 2^53, the places of 1 / (2 pi)
// up to the e-th give whole turns, and what is behind the next 192 is less than 2^-75 of the result's unit.
inline uint64_t turns_of(double freq) {
  int e;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(freq), &e), 53);
  e -= 53;
  const int whole = e > 0 ? e : 0, word = whole / 64, bit = whole % 64;
  uint64_t p[5] = {0, 0, 0, 0, 0};  // m times those 192 places, the lowest first
  unsigned __int128 sum = 0;
  for (int i = 0; i < 3; ++i) {
    const uint64_t *w = kTurnsOfRadian + word + 2 - i;
    sum += (unsigned __int128)m * (bit ? w[0] << bit | w[1] >> (64 - bit) : w[0]);
    p[i] = (uint64_t)sum;
    sum >>= 64;
  }
  p[3] = (uint64_t)sum;
  const int drop = 128 + whole - e;  // places behind the result's
  if (drop > 255) return 0;          // (m times them ends below 2^245)
  auto from = [&](int at) { return at % 64 ? p[at / 64] >> at % 64 | p[at / 64 + 1] << (64 - at % 64) : p[at / 64]; };
  const uint64_t t = from(drop) + (from(drop - 1) & 1);
  return freq < 0 ? 0 - t : t;
}

}  // namespace palq
