// The operand split of one and of two elements: hi = fl16(x), lo = fl16((x - hi) * 2^s), both
// conversions round-to-nearest-even (paper Eq. recover_eqn, first two lines; Sec. 3.3; Sec. 4.2).
#pragma once

#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace sgc {

// One element.  x - hi is exact in FP32 and so is the power-of-two scaling (Sec. 3.3), so the
// only roundings are the two conversions.  FP16 subnormals are produced, never flushed.
__device__ __forceinline__ void split_one(float x, float scale, uint16_t& hi, uint16_t& lo) {
  const __half h = __float2half_rn(x);
  const float r = __fsub_rn(x, __half2float(h));
  const __half l = __float2half_rn(__fmul_rn(r, scale));
  hi = __half_as_ushort(h);
  lo = __half_as_ushort(l);
}

// Two elements packed: hi and lo words as f16x2 (element 0 in the low half).
__device__ __forceinline__ void split_two(float x0, float x1, float scale, uint32_t& hi2,
                                          uint32_t& lo2) {
  const __half2 h = __floats2half2_rn(x0, x1);
  const float2 hf = __half22float2(h);
  const float t0 = __fmul_rn(__fsub_rn(x0, hf.x), scale);
  const float t1 = __fmul_rn(__fsub_rn(x1, hf.y), scale);
  const __half2 l = __floats2half2_rn(t0, t1);
  hi2 = *reinterpret_cast<const uint32_t*>(&h);
  lo2 = *reinterpret_cast<const uint32_t*>(&l);
}

__device__ __forceinline__ float pow2f(int s) { return __int_as_float((127 + s) << 23); }

}  // namespace sgc
