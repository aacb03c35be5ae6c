// Operands on their way to the FP16 words of the products: what is to be packed, and where the words are.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace sgc {

constexpr int kPackScaleExp = 11;        // s: what Eq. sf_bounds leaves for the whole normal FP16 window
constexpr float kPackInvScale = 1.f / 2048.f;

// One matrix to pack: X, or (dz) the gradient in front of the activation, X[i] * act'(Z[i]).
struct PackJob {
  int rows, cols;
  const float* X;
  long long ldx;
  const float* Z;          // dz only
  long long ldz;
  uint16_t* hi;
  uint16_t* lo;
  long long ldh;           // a multiple of 8; the words up to it are written (zeros past cols)
  int* exp;                // p, written by the range kernel
  int vec;                 // X (and Z) take 16-byte loads
};

// 15 - e for the largest magnitude's bits: e is its unbiased exponent after rounding to an 11-bit
// significand, so the largest high word lands in the top normal FP16 binade and cannot overflow.
__device__ __forceinline__ int pack_exponent(uint32_t amax) {
  if (amax == 0) return 0;
  int adj = 0;
  if (amax < 0x00800000u) {                    // FP32 subnormal: normalise first (exact)
    amax = __float_as_uint(__fmul_rn(__uint_as_float(amax), 16777216.0f));
    adj = -24;
  }
  const int p = 15 - ((int)((amax + 0x1000u) >> 23) - 127 + adj);
  return p > 126 ? 126 : (p < -126 ? -126 : p);
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;             // inf and NaN do not set the scale
}

// Words of a packed operand (row-major, both with the leading dimension ld) and the device word with its exponent.
struct Packed {
  const uint16_t* hi;
  const uint16_t* lo;
  int64_t ld;
  const int* exp;
};

}  // namespace sgc
