// Frequencies as fractions of a turn.  Host arithmetic only, apart from the call so that a test can compile it by itself.  Internal: not
// part of the C ABI.
#pragma once

#include <math.h>
#include <stdint.h>

// 2^64 frac(f / 2 pi), rounded, of a finite f below 2^64 in magnitude: f's 64 bits times the first 256 bits of 1 / 2 pi, so that the whole
// turns that come off take no bits of the fraction with them (divided in 64 bits, 10^6 radians keep 47 of the fraction's).
static inline uint64_t lq_turn_fraction(long double f) {
  static const uint64_t inv[4] = {0x28be60db9391054aull, 0x7f09d5f47d4d3770ull, 0x36d8a5664f10e410ull, 0x7f9458eaf7aef158ull};
  int x;
  const uint64_t m = (uint64_t)ldexpl(frexpl(fabsl(f), &x), 64);           // |f| = m 2^(x - 64)
  uint64_t w[6] = {};                                                      // m times those bits, lowest word first
  for (int i = 0; i < 4; ++i) {
    const unsigned __int128 v = (unsigned __int128)m * inv[3 - i] + w[i];
    w[i] = (uint64_t)v;
    w[i + 1] = (uint64_t)(v >> 64);
  }
  const int shift = 256 - x;                                               // the fraction's lowest bit; 192 or more
  if (shift > 320) return 0;
  const int at = shift / 64, off = shift % 64, below = shift - 1;
  uint64_t turn = w[at] >> off | (off ? w[at + 1] << (64 - off) : 0);
  turn += w[below / 64] >> (below % 64) & 1;
  return f < 0 ? 0 - turn : turn;
}
