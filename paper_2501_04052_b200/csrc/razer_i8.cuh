// Rounding to 8-bit integers with a scale, shared by the row quantizer and the cache writer.
//
//   s = fl32(a / 127), a = the largest magnitude; a quotient that rounds to 0 with a > 0 becomes the smallest subnormal
//   q = the exact quotient x / s to the nearest integer, ties to even, clamped to +-127
// A NaN or an infinity among the values makes the scale NaN and their codes 0, so that whatever is computed from them shows it.
//
// The quotient is never formed: q comes from x * (1 / s) by one FMA that rounds at the units place, and the remainder x - q s, which
// one FMA gives exactly (at most 24 bits: |x - q s| is at most about s / 2 and a multiple of the smaller of the two operands' last
// places), says whether it is the nearest.  It is off only where the quotient lies within 2^-16 of a border, so that a whole
// vector's remainders are looked at together; 5 instructions an element, against about 20 with a division.
#pragma once

#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>

namespace razer {

struct I8Step {
  float s, inv;      // the scale and about its reciprocal
  bool plain;        // scale in the range where the reciprocal and the remainders are good
};
constexpr float I8_MAGIC = 12582912.0f;            // 1.5 * 2^23: adding it rounds to an integer, which is then in the low bits

// bits: those of the largest magnitude, as FP32.
__device__ __forceinline__ float i8_scale(uint32_t bits) {
  if (bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float s = __fdiv_rn(__uint_as_float(bits), 127.0f);
  return s == 0.0f && bits ? __uint_as_float(1u) : s;
}
__device__ __forceinline__ I8Step i8_step(float s) {
  I8Step t;
  t.s = s;
  t.plain = s >= 7.9e-31f && s < 1e37f;            // 2^-100: below, remainders could lose bits to underflow
  t.inv = t.plain ? __frcp_rn(s) : 0.0f;
  return t;
}
// Any scale, one element; the double quotient of two 24-bit numbers never crosses a border that the exact one does not cross.
static __device__ __noinline__ int i8_round_any(float x, float s) {
  if (!(s > 0.0f) || !(fabsf(x) < __uint_as_float(0x7F800000u))) return 0;
  const double q = rint((double)x / (double)s);
  return (int)fmin(fmax(q, -127.0), 127.0);
}
// N elements, N a multiple of 4, to N / 4 words of codes.  |x| <= 127 s but for rounding, or the scale is not plain.
template <int N>
__device__ __forceinline__ void i8_round(const float (&x)[N], const I8Step& t, uint32_t (&out)[N / 4]) {
  float m[N];
  if (t.plain) {
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m[i] = __fmaf_rn(x[i], t.inv, I8_MAGIC);
      far = fmaxf(far, fabsf(__fmaf_rn(-(m[i] - I8_MAGIC), t.s, x[i])));
    }
    if (2.0f * far >= t.s) {                        // someone lies on a border, or was put on the wrong side of one
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float q = m[i] - I8_MAGIC;
        const float r = 2.0f * __fmaf_rn(-q, t.s, x[i]);
        const bool odd = __float_as_uint(m[i]) & 1u;
        if (r > t.s || (r == t.s && odd)) q += 1.0f;
        else if (r < -t.s || (r == -t.s && odd)) q -= 1.0f;
        m[i] = fminf(fmaxf(q, -127.0f), 127.0f) + I8_MAGIC;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = __uint_as_float((uint32_t)i8_round_any(x[i], t.s));
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint32_t lo = __byte_perm(__float_as_uint(m[4 * i]), __float_as_uint(m[4 * i + 1]), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(m[4 * i + 2]), __float_as_uint(m[4 * i + 3]), 0x0040);
    out[i] = __byte_perm(lo, hi, 0x5410);
  }
}

// The larger magnitude of bf16 pairs, as two 15-bit patterns: their order as integers is that of the values, NaN above infinity.
__device__ __forceinline__ uint32_t bf16_pair_max(uint32_t so_far, uint32_t pair) { return __vmaxu2(so_far, pair & 0x7FFF7FFFu); }
__device__ __forceinline__ uint32_t bf16_pair_top(uint32_t pair) { return max(pair >> 16, pair & 0xFFFFu) << 16; }
__device__ __forceinline__ float bf16_lo(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

}  // namespace razer
