// Rotary positions on the device: the cosine and sine of a position's angle.
#pragma once

#include "common.cuh"
#include "decode.h"

namespace ravel {

// amplitude * (cos, sin) of the angle that is f 2^-64 turns times the position.  The product modulo
// 2^64 is exact; its upper 32 bits less the nearest quarter turn, at most an eighth of a turn,
// go to fp32 with the 24 bits of that remainder, and the quarter turns change places and signs.
// (The same from a float angle loses position * 2^-24: half a turn at position 10^7.)
__device__ __forceinline__ float2 turn_of(unsigned long long f, long long position, float amplitude) {
  const unsigned long long t = f * (unsigned long long)position + 0x80000000ull;
  const uint32_t turn = (uint32_t)(t >> 32);
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float half_turns = (float)(int)(turn - (quarter << 30)) * 0x1p-31f;
  float s, c;
  sincospif(half_turns, &s, &c);
  float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
  if (quarter & 2) x = -x, y = -y;
  return make_float2(x * amplitude, y * amplitude);
}

// What one value of a pair becomes: own c - other s of the first, own c + other s of the second.
// (Written out, so that every kernel rounds alike.)
__device__ __forceinline__ float turned(float own, float other, float2 cs, bool first) {
  const float y = __fmul_rn(other, cs.y);
  return __fmaf_rn(own, cs.x, first ? -y : y);
}

}  // namespace ravel
