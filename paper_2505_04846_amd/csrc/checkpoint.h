// Activations in 8 bits: 32 values of a row share a power of two, each is a whole number of at most 127 of it.
//
//   e = floor(log2 max |x|) - 6,   code = round(x / 2^e), ties to even, at most 127 in magnitude
// so that the largest of the 32 has a code of 64 to 127 and every value is off by at most 2^e / 2 (a largest one
// within 2^e / 2 of 2^(e + 7) by up to 2^e).  A code times its power of two has at most 7 significant bits: it is a
// number of the row's own type (e stays at or above fp16's smallest step, 2^-24, and 2^-126 for bf16), and what
// reads it back is exact.  exps holds e + 127; 255 stands for 32 values of which one was not finite: NaN.
#pragma once

#include "common.h"

namespace hpr {

template <class T>
__device__ __forceinline__ int checkpoint_least() {
  return T::kNarrow ? -24 : -126;
}

// 2^e of a stored exponent, NaN for 255.
__device__ __forceinline__ float checkpoint_step(uint32_t e) {
  return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23);
}

// Eight codes' values.  A code plus 128 is a byte, which one instruction converts.
__device__ __forceinline__ void code_values(uint2 codes, uint32_t e, float (&f)[8]) {
  const float step = checkpoint_step(e);
  const uint32_t w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    f[i] = ((float)((w[i >> 2] >> (8 * (i & 3))) & 255u) - 128.f) * step;
}

// Eight values in the 16-bit type, exactly.
template <class T>
__device__ __forceinline__ u32x4 unpack8(uint2 codes, uint32_t e) {
  float f[8];
  code_values(codes, e, f);
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = T::pack(f[2 * i], f[2 * i + 1]);
  return v;
}

}  // namespace hpr
