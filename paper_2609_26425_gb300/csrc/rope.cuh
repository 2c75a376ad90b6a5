// rope.cuh -- the angle of a rotary position, for the kernels that turn by it.
#pragma once

#include "paged.cuh"

namespace qwm {

// (cos, sin) of pos * f, exact to the fp32 rounding of the reduced angle at every
// position.  The angle is taken in turns, as a 64-bit fraction whose whole turns fall
// off the top (after Payne and Hanek, who form only the bits of a product that a
// reduction keeps): f = m 2^e with a 24-bit m, f / (2 pi) = m 2^e C with C = 1 / (2 pi) to 128
// bits, cut below 2^-64 of a turn, times the position (2^-33 of a turn at 2^31).  What
// is left beside the nearest quarter turn is at most pi / 4 in fp32, where the fast sine
// and cosine are good to 2^-21: far below the output's 2^-9 or 2^-12.  An f of 2^24 or
// more, an infinity or a NaN gives NaN.
// FINE: with the full sine and cosine, for results that are rounded to less than they are good
// for: next to a border between two codes every bit counts.
template <bool FINE = false>
__device__ __forceinline__ float2 turn(int pos, float f, float sign) {
  constexpr uint64_t kC1 = 0x28BE60DB9391054Aull, kC0 = 0x7F09D5F47D4D3770ull;   // floor(2^128 / (2 pi))
  constexpr float kTurn = (float)(6.283185307179586476925286766559 / 18446744073709551616.0);
  const uint32_t w = __float_as_uint(f), ex = (w >> 23) & 255u;
  const uint64_t m = (w & 0x7FFFFFu) | (ex ? 0x800000u : 0u);
  const int down = 150 - (int)max(ex, 1u);         // -e
  const uint64_t c0 = __umul64hi(m, kC0), lo = m * kC1 + c0, hi = __umul64hi(m, kC1) + (lo < c0);
  const uint64_t g = down <= 0 ? lo : (down < 64 ? (lo >> down) | (hi << (64 - down)) : (down < 128 ? hi >> (down - 64) : 0));
  const uint64_t t = (uint64_t)(int64_t)pos * g;
  const uint64_t q = (t + (1ull << 61)) >> 62;      // quarter turns
  float sn, cs;
  const float left = (float)(int64_t)(t - (q << 62)) * kTurn;
  if (FINE) sincosf(left, &sn, &cs);
  else __sincosf(left, &sn, &cs);
  if (ex >= 127 + 24) cs = __uint_as_float(0x7FFFFFFFu);
  const float c = q & 1 ? sn : cs, d = q & 1 ? cs : sn;
  // a quarter turn on is (-sn, cs), and so forth
  const float sc = (q + 1) & 2 ? -c : c, ss = q & 2 ? -d : d;
  return make_float2(sc, (w >> 31) ? -(sign * ss) : sign * ss);
}

__device__ __forceinline__ int64_t wide(int a, int b) { return (int64_t)a * b; }

}  // namespace qwm
