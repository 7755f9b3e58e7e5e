// How the kernels read activations kept in 8 bits (pack8.hip).
#pragma once
#include "kernels.h"

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float step_of(int byte) {          // 2^e
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x400000u : (unsigned)byte << 23);
}
// the eight values of two words; (number + 128) * step - 128 * step in one operation would overflow in blocks of the largest numbers
__device__ __forceinline__ void unpack8_of(u32x2 q, int byte, float (&v)[8]) {
  const float step = step_of(byte);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned w = (h ? q.y : q.x) ^ 0x80808080u;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * h + k] = ((float)(w >> (8 * k) & 0xffu) - 128.f) * step;
  }
}
