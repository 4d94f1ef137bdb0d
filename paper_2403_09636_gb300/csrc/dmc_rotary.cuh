// Position rotation: pair i of a head turns by position * frequency_i.
//
// Frequencies are kept as turns per token times 2^64. A phase is then a product of whole numbers modulo 2^64, exact for
// any position, where an angle in fp32 would be off by half a turn from positions of some millions on; what is left of
// its rounding is that of the angle itself to fp32, in half turns of [-1, 1) (9e-8).
#pragma once

#include "dmc_internal.cuh"

namespace dmc {

enum : int { kRotNone = 0, kRotHalf = 1, kRotPairs = 2 };  // pairs: none; dims i, i + D / 2; dims 2 i, 2 i + 1

// (cos, sin) of `at` tokens' turn of a pair. Pair 0 holds the gate and stays as it is: its callers give it no turns.
__device__ __forceinline__ float2 turn_of(unsigned long long turns, long long at) {
  const unsigned long long phase = turns * (unsigned long long)at;
  float2 cs;
  sincospif((float)(int)(phase >> 32) * 4.656612873077393e-10f, &cs.y, &cs.x);  // 2^-31: half turns
  return cs;
}

__device__ __forceinline__ unsigned long long turns_of_pair(const unsigned long long* turns, int pair) {
  return pair == 0 ? 0ull : __ldg(turns + pair);
}

// (x, y) turned.
__device__ __forceinline__ void turn(float2 cs, float& x, float& y) {
  const float a = x * cs.x - y * cs.y, b = y * cs.x + x * cs.y;
  x = a;
  y = b;
}

}  // namespace dmc
