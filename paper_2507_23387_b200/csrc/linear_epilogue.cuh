// What a linear layer does to a finished product element, and how a 32 x 128 register tile of them is
// stored.  Shared by the tensor-core kernel's epilogue, the split-K reduction and the few-row kernel.
//
//   z = 2^-(p_x + p_w) acc + b[col],   y = act(z) + R[row, col]
//
// acc is the FP32 product of the packed operands 2^p_x X and 2^p_w W; the way back is exact unless the
// result leaves the normal FP32 range.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace sgc {

enum Activation { kActNone = 0, kActRelu, kActGelu, kActGeluTanh, kActSilu };

// act(z), FP32 throughout.  The library's erff, tanhf and expf (about 2 ulp), not the fast
// approximations: the product in front is good to 2^-22 and the activation should not be what limits it.
__device__ __forceinline__ float act_value(int act, float z) {
  switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;                            // keeps NaN
    case kActGelu: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    case kActGeluTanh:
      return 0.5f * z * (1.f + tanhf(0.79788456080286536f * fmaf(0.044715f * z * z, z, z)));
    case kActSilu: return z / (1.f + expf(-z));
    default: return z;
  }
}

// act'(z).  relu'(0) = 0.  For z far below zero the products that vanish are cut off before a factor
// overflows (z^2 and exp(-z) leave the FP32 range, their products do not), so no 0 * inf appears.
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : (z == z ? 0.f : z);
    case kActGelu: {
      const float phi = 0.5f * (1.f + erff(z * 0.70710678118654752f));
      const float u = fminf(fabsf(z), 20.f);                            // exp(-200) = 0 in FP32
      return fmaf(copysignf(u, z) * 0.39894228040143268f, expf(-0.5f * u * u), phi);
    }
    case kActGeluTanh: {
      const float u = copysignf(fminf(fabsf(z), 20.f), z);              // tanh is +-1 from there on
      const float t = tanhf(0.79788456080286536f * fmaf(0.044715f * u * u, u, u));
      const float s = 0.5f * (1.f + t) +
                      0.5f * u * (1.f - t * t) * 0.79788456080286536f * fmaf(0.134145f * u, u, 1.f);
      return z == z ? s : z;
    }
    case kActSilu: {
      const float p = 1.f / (1.f + expf(-z));
      const float u = fmaxf(z, -110.f);                                 // p = 0 in FP32 from -104 on
      const float s = p * fmaf(u, 1.f - p, 1.f);
      return z == z ? s : z;
    }
    default: return 1.f;
  }
}

struct LinearEpilogue {
  const int* exp_a;       // exponents p of the two packed operands (device; null: 0)
  const int* exp_b;
  const float* bias;      // [N] or null
  const float* R;         // residual or null; may be Y itself
  long long ldr;
  float* Z;               // z is stored here too, or null
  long long ldz;
  int act;
  int vec;                // Y, Z and R take 16-byte accesses
};

// 2^-(p_a + p_b) as two FP32 factors (the sum of two exponents can leave the range of one).
struct PowerBack {
  float f0, f1;
  __device__ __forceinline__ float operator()(float v) const { return v * f0 * f1; }
};
__device__ __forceinline__ PowerBack power_back(const int* pa, const int* pb) {
  const int t = -((pa ? *pa : 0) + (pb ? *pb : 0));
  const int t0 = t > 127 ? 127 : (t < -126 ? -126 : t);
  return PowerBack{__int_as_float((127 + t0) << 23), __int_as_float((127 + t - t0) << 23)};
}

// One element whose z is known: stores z, returns y.
__device__ __forceinline__ float linear_finish(const LinearEpilogue& e, float z, long long row, int col) {
  if (e.Z) e.Z[row * e.ldz + col] = z;
  float y = act_value(e.act, z);
  if (e.R) y += e.R[row * e.ldr + col];
  return y;
}

// The 32 rows x 128 columns of one accumulate warp: lane l holds row `row0 + l`, columns col0 .. col0 + 127.
// 32 x 32 blocks go through the warp's 4 KB staging buffer (16-byte chunks XOR-swizzled by row: no bank
// conflicts either way), so that bias, residual and stores run along rows.  Aligned matrices: 16 bytes
// per lane, four rows an instruction.  Others (odd leading dimensions): 4 bytes per lane, a row an
// instruction, which keeps the accesses of a warp in one or two 128-byte lines.
__device__ __forceinline__ void linear_store_tile(const LinearEpilogue& e, float* Y, long long ldy, int M, int N,
                                                  const float (&S)[128], uint32_t stg, int row0, int col0,
                                                  int lane) {
  const PowerBack back = power_back(e.exp_a, e.exp_b);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stg + lane * 128 + ((q ^ (lane & 7)) << 4)),
                   "f"(S[g * 32 + 4 * q]), "f"(S[g * 32 + 4 * q + 1]), "f"(S[g * 32 + 4 * q + 2]),
                   "f"(S[g * 32 + 4 * q + 3])
                   : "memory");
    __syncwarp();
    if (e.vec) {
      const int q = lane & 7;
      const int col = col0 + g * 32 + q * 4;
      const bool full = col + 4 <= N;
      float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
      if (e.bias) {
        if (col < N) b.x = e.bias[col];
        if (col + 1 < N) b.y = e.bias[col + 1];
        if (col + 2 < N) b.z = e.bias[col + 2];
        if (col + 3 < N) b.w = e.bias[col + 3];
      }
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const int r = i * 4 + (lane >> 3);
        const int row = row0 + r;
        if (row >= M || col >= N) continue;
        float4 v;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                     : "r"(stg + r * 128 + ((q ^ (r & 7)) << 4))
                     : "memory");
        v.x = back(v.x) + b.x; v.y = back(v.y) + b.y; v.z = back(v.z) + b.z; v.w = back(v.w) + b.w;
        if (full) {
          float4 res = make_float4(0.f, 0.f, 0.f, 0.f);
          if (e.R) res = *reinterpret_cast<const float4*>(e.R + (long long)row * e.ldr + col);
          if (e.Z) *reinterpret_cast<float4*>(e.Z + (long long)row * e.ldz + col) = v;
          if (e.act != kActNone) {
            v.x = act_value(e.act, v.x); v.y = act_value(e.act, v.y);
            v.z = act_value(e.act, v.z); v.w = act_value(e.act, v.w);
          }
          if (e.R) { v.x += res.x; v.y += res.y; v.z += res.z; v.w += res.w; }
          *reinterpret_cast<float4*>(Y + (long long)row * ldy + col) = v;
        } else {
          const float z[4] = {v.x, v.y, v.z, v.w};
          for (int j = 0; j < 4 && col + j < N; ++j)
            Y[(long long)row * ldy + col + j] = linear_finish(e, z[j], row, col + j);
        }
      }
    } else {
      const int col = col0 + g * 32 + lane;
      const float b = (e.bias && col < N) ? e.bias[col] : 0.f;
#pragma unroll 1
      for (int r = 0; r < 32; ++r) {
        const int row = row0 + r;
        if (row >= M || col >= N) break;
        float v;
        asm volatile("ld.shared.f32 %0, [%1];"
                     : "=f"(v)
                     : "r"(stg + r * 128 + ((((lane >> 2) ^ (r & 7)) << 4) | ((lane & 3) << 2)))
                     : "memory");
        Y[(long long)row * ldy + col] = linear_finish(e, back(v) + b, row, col);
      }
    }
    __syncwarp();
  }
}

}  // namespace sgc
