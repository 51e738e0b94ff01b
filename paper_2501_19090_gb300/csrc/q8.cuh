// q8.cuh -- elements and scales of a paged cache in 8 bits (rope_q8.cu), and how attention takes them (attention_q8.cu, attention_tc.cu).
//
// Both products run on fp16: e4m3 numbers are fp16 numbers, and rows of Q are brought into its range by a power of two. Of
// the scales the keys' multiply the scores. The values' become part of the weights' exponents: with x_j the score of key j
// (times log2(e)) and t its value's scale,
//   w_j = 2^(x_j + log2 t - base - m),  O = sum_j w_j v_j,  l = sum_j w_j 2^(base - log2 t),  o = 2^base O / l
// so that a weight costs no operation more, and fp16's range is spent on what the weights contribute. `base`, whole, is near
// the largest log2 t so far: a larger one than base + 40 raises it, and O is brought into
// the new unit; smaller ones than base - 40 count as
// that, in w and in l alike, which puts an error of less than 2^-39 of the largest value into o. In between neither w nor l leaves
// fp32's range where it matters (a w below 2^-126 belongs to a weight of less than 2^-46 of the largest).
#ifndef PIFA_Q8_CUH_
#define PIFA_Q8_CUH_

#include <stdint.h>

#include <cuda_fp16.h>

namespace pifa {

// A running maximum is raised when a score passes it by 8 in the exponent, so that weights reach 2^8 of what it refers to, and fp16
// goes to 2^15: weights are held 2^7 times as large (m is the maximum less 7; O and l are both in those units, which o = O / l is
// rid of), and those below fp16's normal range are off by 2^-32 of the largest. They count: the tens of thousands of keys beside one
// that has all but a millionth of the weight, and a value near zero, are all of o. (Without it, those 2^-25 of the largest and less were in l alone.)
constexpr float LIFT = 7.0f, RISE = 8.0f + LIFT;
constexpr float UNLIFT = 0x1p-7f;  // pieces that are written to be added up leave these units: values may be near fp32's largest

constexpr float NO_BASE = -1000.0f;
constexpr float FAR = 40.0f;

// 2^e for e in [-126, 127].
__device__ __forceinline__ float exponent_of_2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The scale that a byte b stands for, 2^(b - 127); 255: NaN.
__device__ __forceinline__ float scale_of(int byte) {
  return byte == 0 ? __uint_as_float(0x00400000u) : byte == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float((uint32_t)byte << 23);
}

// What stands for the scale of a block that is not read (zeros do as its keys and values).
constexpr int NO_SCALE = 256;

// Sets `base` by the largest exponent (-1000: none) of the first blocks that have one, and raises it by that of later ones where
// it has to; returns by how much it has risen.
__device__ __forceinline__ float raise_base(int exponent, float& base) {
  if (exponent == -1000) return 0.0f;
  const float e = fmaxf((float)exponent, -126.0f);
  if (base != NO_BASE && e <= base + FAR) return 0.0f;
  const float up = base == NO_BASE ? 0.0f : e - base;
  base = e;
  return up;
}

struct ValueScale {
  float exponent, inverse;  // log2 t - base, and 2^ the negative of it
};
// A block's scale byte against `base`. A scale of NaN gives weights of NaN to the keys that are seen, and leaves l alone where
// none is. (Chunks make such a block's keys NaN instead, and its values zeros.)
__device__ __forceinline__ ValueScale value_scale(int byte, float base) {
  if (byte == 255) return {__uint_as_float(0x7fffffffu), 0.0f};
  if (byte == NO_SCALE) return {0.0f, 1.0f};
  const float e = fminf(fmaxf((float)(byte - 127) - base, -FAR), FAR);
  return {e, exponent_of_2(-(int)e)};
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Two e4m3 numbers as fp16, the lower byte's in the lower half.
__device__ __forceinline__ uint32_t halves_of(uint32_t e4m3x2) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)e4m3x2));
  return h;
}

// The power of two that brings a row of bf16 magnitudes up to `most` to [2^14, 2^15); what is that small that this would leave
// fp32's range, zeros and what is not finite are taken as they come.
__device__ __forceinline__ int row_exponent(float most) {
  const int e = (int)(__float_as_uint(most) >> 23) - 127;
  return most == 0.0f || e == 128 ? 0 : 14 - max(e, -100);
}

// Two e4m3 numbers times s in 16 bits, each rounded once; a finite product stays finite, at most the type's largest number.
template <bool F16>
__device__ __forceinline__ uint32_t scaled_from_e4m3x2(uint32_t two, float s) {
  const uint32_t h = halves_of(two);
  const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h));
  uint32_t r;
  if constexpr (F16) asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(p.y * s), "f"(p.x * s));
  else asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(p.y * s), "f"(p.x * s));
  return r;
}

}  // namespace pifa

#endif  // PIFA_Q8_CUH_
