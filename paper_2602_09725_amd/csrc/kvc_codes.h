// Codes of 4 bits as pages hold them (include/kvc.h): from 16-bit values and back.
//
// A word has eight codes of a token, elements 8 w .. 8 w + 7 of a head: the even ones in its low half, the odd ones in its high half, so that
// (word >> 4 i) & 0x000f000f is the pair of elements 2 i, 2 i + 1 side by side.  A vector has the same word of four tokens that follow one another.
#pragma once

#include <hip/hip_runtime.h>

#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

typedef short s16x2 __attribute__((ext_vector_type(2)));

// 16-bit floating values as whole numbers of the same order, two at a time (the map is its own inverse): -inf and the negative NaNs lie at the low end,
// inf and the others at the high one.
__device__ __forceinline__ uint32_t as_ordered(uint32_t w) {
  const s16x2 sign = __builtin_bit_cast(s16x2, w) >> 15;
  return w ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}

// The least and the most of some values, as ordered numbers in the low halves.
struct Extremes {
  s16x2 low, high;
};
__device__ __forceinline__ void widen_to(Extremes& e, uint32_t ordered) {
  e.low = __builtin_elementwise_min(e.low, __builtin_bit_cast(s16x2, ordered));
  e.high = __builtin_elementwise_max(e.high, __builtin_bit_cast(s16x2, ordered));
}

// What a token's head is held with.
struct Pair {
  float mn, inv;
  uint32_t bits;  // scale and mn as stored
  bool wild;      // something is not finite: all of it reads back as NaN
};

template <int DT>
__device__ __forceinline__ Pair pair_of(short low, short high) {
  constexpr uint32_t kExp = DT == KVC_F16 ? 0x7c00u : 0x7f80u;  // infinity, and as an ordered number the least of what is not finite
  const uint32_t most = as_ordered((uint16_t)high), least = as_ordered((uint16_t)low);
  Pair r;
  r.mn = widen_bits<DT>(least & 0xffffu) + 0.0f;
  const float range = widen_bits<DT>(most & 0xffffu) - r.mn;
  r.wild = (int)high >= (int)kExp || (int)low <= ~(int)kExp || (__builtin_bit_cast(uint32_t, range) & 0x7f800000u) == 0x7f800000u;
  const float step = range / 15.0f;
  // rounded up to the type: the codes then reach the largest value, and no value is further than half a scale from what it is held as
  uint32_t scale;
  if constexpr (DT == KVC_F16) {
    scale = narrow_pair<DT>(step, 0.0f) & 0xffffu;
    scale += widen_bits<DT>(scale) < step;
  } else {
    scale = (__builtin_bit_cast(uint32_t, step) + 0xffffu) >> 16;
  }
  r.inv = scale ? 1.0f / widen_bits<DT>(scale) : 0.0f;
  const uint32_t mn = least == 0x8000u ? 0u : least & 0xffffu;
  r.bits = r.wild ? (DT == KVC_F16 ? 0x7e00u : 0x7fc0u) : scale | mn << 16;
  return r;
}

// Eight values -> a word.  code = rint((x - mn) * inv), which does not exceed 15: scale * 15 is at least the range, but for a rounding that rint takes
// back.  (Adding 1.5 * 2^23 rounds to whole numbers, half to even, and leaves them in the low bits.)
template <int DT>
__device__ __forceinline__ uint32_t word_of(u32x4 v, const Pair& p) {
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    widen_pair<DT>(v[i], a, b);
    const uint32_t even = __builtin_bit_cast(uint32_t, (a - p.mn) * p.inv + 12582912.0f) & 15u;
    const uint32_t odd = __builtin_bit_cast(uint32_t, (b - p.mn) * p.inv + 12582912.0f) & 15u;
    word |= even << (4 * i) | odd << (4 * i + 16);
  }
  return p.wild ? 0u : word;
}

// A word -> the eight values that it stands for, rounded to the type.  Where the scale's rounding has pushed the last code beyond the type's largest
// number, that number is taken.
template <int DT>
__device__ __forceinline__ u32x4 values_of(uint32_t word, uint32_t pair) {
  const float most = DT == KVC_F16 ? 65504.0f : 3.38953139e38f;
  const float scale = widen_bits<DT>(pair & 0xffffu), mn = widen_bits<DT>(pair >> 16);
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = fmaf((float)(word >> (4 * i) & 15u), scale, mn), b = fmaf((float)(word >> (4 * i + 16) & 15u), scale, mn);
    if (a > most) a = most;  // (a NaN stays one)
    if (b > most) b = most;
    v[i] = narrow_pair<DT>(a, b);
  }
  return v;
}

}  // namespace kvc
