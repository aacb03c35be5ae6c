// What a linear layer does to a finished product element, and how a tile of them is stored.  Shared by the
// tensor-core kernels' epilogues and the few-row kernels.
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

// exp and 1 / x on the special function unit (2^-22 and one ulp; exponentials below 2^-126 are zero).
__device__ __forceinline__ float fast_exp2(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  return e;
}
__device__ __forceinline__ float fast_exp(float x) { return fast_exp2(x * 1.4426950408889634f); }
__device__ __forceinline__ float fast_rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// s = 1 / (1 + exp(-z)), and s (1 - s) without the difference (which loses its bits where s is near 1).
__device__ __forceinline__ float sigmoid(float z, float& slope) {
  const float e = fast_exp(-fabsf(z));
  const float r = fast_rcp(1.f + e);
  slope = e * r * r;
  return z < 0.f ? e * r : r;
}

// Phi(z), the normal distribution function, and e = exp(-z^2 / 2):  erfc(x) / 2 = t Q(t) exp(-x^2) with
// t = 1 / (1 + 0.3 x) and Q of degree 8, fitted to exp(x^2) erfc(x) / t over 0 <= x <= 9.5 for the least relative error
// (2e-8), x = |z| / sqrt(2).  The lower tail is taken from it directly, not as a difference from 1, so it keeps its digits: in
// FP32 off by 4e-7 of itself at z = 0, 1.5e-6 at -3, 3e-6 at -5 (the rounding of z^2 in the exponent).  16 instructions where
// erff and expf take 45: with those the kernels around the product were bound by arithmetic, not by memory
// (8192 x 16384: 347 us for the pass that needs 164).
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float t = fast_rcp(fmaf(0.3f * 0.70710678118654752f, fabsf(z), 1.f));
  float q = fmaf(-0.0647170395f, t, 0.242548227f);
  q = fmaf(q, t, -0.255613238f);
  q = fmaf(q, t, 0.273197532f);
  q = fmaf(q, t, -0.04681563f);
  q = fmaf(q, t, 0.107218139f);
  q = fmaf(q, t, 0.0742412135f);
  q = fmaf(q, t, 0.0853459686f);
  q = fmaf(q, t, 0.0845948085f);
  e = fast_exp2(-0.5f * 1.4426950408889634f * z * z);
  q = q * t * e;
  return z < 0.f ? q : 1.f - q;
}

// sigmoid(2u) = (1 + tanh u) / 2 with the tanh form's u = sqrt(2 / pi) (z + 0.044715 z^3)
__device__ __forceinline__ float gelu_tanh_weight(float z, float& slope) {
  return sigmoid(1.5957691216057308f * fmaf(0.044715f * z * z, z, z), slope);
}

// act(z), good to 2^-21 (|z| + 1).
__device__ __forceinline__ float act_value(int act, float z) {
  float unused;
  switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;                            // keeps NaN
    case kActGelu: return z * normal_cdf(z, unused);
    case kActGeluTanh: return z * gelu_tanh_weight(z, unused);
    case kActSilu: return z * sigmoid(z, unused);
    default: return z;
  }
}

// act'(z), good to 2^-20.  relu'(0) = 0.  Where a factor overflows while the product vanishes, z is cut off first
// (no 0 * inf).
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : (z == z ? 0.f : z);
    case kActGelu: {
      float e;
      const float phi = normal_cdf(z, e);
      return fmaf(copysignf(fminf(fabsf(z), 20.f), z) * 0.39894228040143268f, e, phi);     // e = 0 from 20 on
    }
    case kActGeluTanh: {
      const float u = copysignf(fminf(fabsf(z), 20.f), z);              // the weight is 0 or 1 from there on
      float ds;
      const float w = gelu_tanh_weight(u, ds);
      const float d = 1.5957691216057308f * fmaf(0.134145f * u, u, 1.f);
      return z == z ? fmaf(u * ds, d, w) : z;
    }
    case kActSilu: {
      const float u = copysignf(fminf(fabsf(z), 110.f), z);             // s is 0 or 1 in FP32 from 104 on
      float ds;
      const float w = sigmoid(u, ds);
      return z == z ? fmaf(u, ds, w) : z;
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
  // Scratch tiles of 128 x 256 sums: two for every block, or (split-K) `ksplit` for every tile of Y.  Null: the
  // accumulate warps store to Y themselves.
  float* tiles;
};

// 2^-(p_a + p_b) as two FP32 factors (the sum of two exponents can leave the range of one).
struct PowerBack {
  float f0, f1;
  __device__ __forceinline__ float operator()(float v) const { return v * f0 * f1; }
};
__device__ __forceinline__ PowerBack power_back_of(int t) {       // 2^t
  const int t0 = t > 127 ? 127 : (t < -126 ? -126 : t);
  return PowerBack{__int_as_float((127 + t0) << 23), __int_as_float((127 + t - t0) << 23)};
}
__device__ __forceinline__ PowerBack power_back(const int* pa, const int* pb) {
  return power_back_of(-((pa ? *pa : 0) + (pb ? *pb : 0)));
}

// One element whose z is known: stores z, returns y.
__device__ __forceinline__ float linear_finish(const LinearEpilogue& e, float z, long long row, int col) {
  if (e.Z) e.Z[row * e.ldz + col] = z;
  float y = act_value(e.act, z);
  if (e.R) y += e.R[row * e.ldr + col];
  return y;
}

// A finished 128 x 256 tile of sums waits in the block's scratch as float4 [64][128]: four columns of a row, the 128
// rows next to each other, which is how the accumulate warps hold it (a thread has a row).
__device__ __forceinline__ float4* tile_slot(float* tile, int col4, int row) {
  return reinterpret_cast<float4*>(tile) + col4 * 128 + row;
}

template <int ACT, int N>
__device__ __forceinline__ void act_each(float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = act_value(ACT, v[i]);
}
template <int ACT>
__device__ __forceinline__ void act_four(float4& v) {
  v.x = act_value(ACT, v.x); v.y = act_value(ACT, v.y); v.z = act_value(ACT, v.z); v.w = act_value(ACT, v.w);
}

// Blocks of 32 rows x 16 columns of such a tile, from `first` on every `step`-th, to Y: lane = every eighth row x four
// columns, so that a warp reads whole lines and writes 64 bytes of every row.  `slices` tiles `stride` floats
// apart (split-K) are added in order.  Few warps do this and instructions are what bounds it: bias and addresses
// are taken once for the four rows of a lane, and a block inside N of aligned matrices tests nothing but rows.
// (One row at a time with everything tested took 18 us for a tile; the accumulate warps doing it on their
// 128 registers, with the tensor core waiting, 55 us: 8192 x 16384 x 4096 with gelu 4011 us, without 2388.)
__device__ __forceinline__ void linear_store_blocks(const LinearEpilogue& e, float* Y, long long ldy, int M, int N,
                                                    float* tile, int slices, long long stride, int row0, int col0,
                                                    int first, int step, int lane) {
  constexpr int U = 4;                                       // rows of a lane, 8 apart
  const PowerBack back = power_back(e.exp_a, e.exp_b);
  const float back_all = back.f0 * back.f1;
  const bool one_factor = fabsf(back_all) >= 1.17549435e-38f && fabsf(back_all) <= 1.7e38f;
  const int lr = lane >> 2, lc = lane & 3;
  const int blocks = (min(128, M - row0) + 8 * U - 1) / (8 * U) * 16;
#pragma unroll 1
  for (int b = first; b < blocks; b += step) {
    const int r0 = (b >> 4) * (8 * U) + lr;
    const int col = col0 + (b & 15) * 16 + lc * 4;
    if (col0 + (b & 15) * 16 >= N) continue;
    const bool full = e.vec && col0 + (b & 15) * 16 + 16 <= N;
    const int row = row0 + r0;
    const float4* src = tile_slot(tile, (b & 15) * 4 + lc, r0);
    float4 v[U], res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = __ldcg(src + 8 * u);
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
    if (e.bias) {
      if (col < N) bias.x = __ldg(e.bias + col);
      if (col + 1 < N) bias.y = __ldg(e.bias + col + 1);
      if (col + 2 < N) bias.z = __ldg(e.bias + col + 2);
      if (col + 3 < N) bias.w = __ldg(e.bias + col + 3);
    }
    if (e.R) {
      const float* r = e.R + row * e.ldr + col;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        res[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row + 8 * u < M) {
          const float* ru = r + 8 * u * e.ldr;
          if (full) {
            res[u] = *reinterpret_cast<const float4*>(ru);
          } else {
            if (col < N) res[u].x = ru[0];
            if (col + 1 < N) res[u].y = ru[1];
            if (col + 2 < N) res[u].z = ru[2];
            if (col + 3 < N) res[u].w = ru[3];
          }
        }
      }
    }
#pragma unroll 1
    for (int s = 1; s < slices; ++s) {
      const float4* more = src + s * (stride / 4);
      float4 f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] = __ldcg(more + 8 * u);
#pragma unroll
      for (int u = 0; u < U; ++u) { v[u].x += f[u].x; v[u].y += f[u].y; v[u].z += f[u].z; v[u].w += f[u].w; }
    }
    auto store = [&](float* out, long long ld) {
      out += row * ld + col;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (row + 8 * u >= M) break;
        float* o = out + 8 * u * ld;
        if (full) {
          *reinterpret_cast<float4*>(o) = v[u];
        } else {
          if (col < N) o[0] = v[u].x;
          if (col + 1 < N) o[1] = v[u].y;
          if (col + 2 < N) o[2] = v[u].z;
          if (col + 3 < N) o[3] = v[u].w;
        }
      }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (one_factor) {
        v[u].x = fmaf(v[u].x, back_all, bias.x); v[u].y = fmaf(v[u].y, back_all, bias.y);
        v[u].z = fmaf(v[u].z, back_all, bias.z); v[u].w = fmaf(v[u].w, back_all, bias.w);
      } else {
        v[u].x = back(v[u].x) + bias.x; v[u].y = back(v[u].y) + bias.y;
        v[u].z = back(v[u].z) + bias.z; v[u].w = back(v[u].w) + bias.w;
      }
    }
    if (e.Z) store(e.Z, e.ldz);
    switch (e.act) {
      case kActRelu:
#pragma unroll
        for (int u = 0; u < U; ++u) act_four<kActRelu>(v[u]);
        break;
      case kActGelu:
#pragma unroll
        for (int u = 0; u < U; ++u) act_four<kActGelu>(v[u]);
        break;
      case kActGeluTanh:
#pragma unroll
        for (int u = 0; u < U; ++u) act_four<kActGeluTanh>(v[u]);
        break;
      case kActSilu:
#pragma unroll
        for (int u = 0; u < U; ++u) act_four<kActSilu>(v[u]);
        break;
      default: break;
    }
    if (e.R) {
#pragma unroll
      for (int u = 0; u < U; ++u) { v[u].x += res[u].x; v[u].y += res[u].y; v[u].z += res[u].z; v[u].w += res[u].w; }
    }
    store(Y, ldy);
  }
}

// The same where Y, Z or R cannot be met with 16 bytes: the scratch tile is row-major, 256 columns, and a warp takes half
// of two rows at a time, lane = one column in 32, so that its accesses stay in one or two lines.
__device__ __forceinline__ void linear_store_rows(const LinearEpilogue& e, float* Y, long long ldy, int M, int N,
                                                  const float* tile, int slices, long long stride, int row0, int col0,
                                                  int first, int step, int lane) {
  constexpr int U = 2, C = 4;                                // rows, and columns of a lane
  const PowerBack back = power_back(e.exp_a, e.exp_b);
  const int blocks = (min(128, M - row0) + U - 1) / U * 2;
#pragma unroll 1
  for (int b = first; b < blocks; b += step) {
    const int r = (b >> 1) * U, row = row0 + r, c = (b & 1) * 128 + lane, col = col0 + c;
    if (col0 + (b & 1) * 128 >= N) continue;
    const float* src = tile + r * 256 + c;
    float v[U * C], res[U * C], bias[C];
#pragma unroll
    for (int i = 0; i < U * C; ++i) v[i] = __ldcg(src + (i / C) * 256 + (i % C) * 32);
#pragma unroll
    for (int q = 0; q < C; ++q) bias[q] = e.bias && col + q * 32 < N ? __ldg(e.bias + col + q * 32) : 0.f;
    if (e.R) {
#pragma unroll
      for (int i = 0; i < U * C; ++i)
        res[i] = row + i / C < M && col + (i % C) * 32 < N ? e.R[(row + i / C) * e.ldr + col + (i % C) * 32] : 0.f;
    }
#pragma unroll 1
    for (int s = 1; s < slices; ++s) {
      float f[U * C];
#pragma unroll
      for (int i = 0; i < U * C; ++i) f[i] = __ldcg(src + s * stride + (i / C) * 256 + (i % C) * 32);
#pragma unroll
      for (int i = 0; i < U * C; ++i) v[i] += f[i];
    }
    auto store = [&](float* out, long long ld) {
#pragma unroll
      for (int i = 0; i < U * C; ++i)
        if (row + i / C < M && col + (i % C) * 32 < N) out[(row + i / C) * ld + col + (i % C) * 32] = v[i];
    };
#pragma unroll
    for (int i = 0; i < U * C; ++i) v[i] = back(v[i]) + bias[i % C];
    if (e.Z) store(e.Z, e.ldz);
    switch (e.act) {
      case kActRelu: act_each<kActRelu>(v); break;
      case kActGelu: act_each<kActGelu>(v); break;
      case kActGeluTanh: act_each<kActGeluTanh>(v); break;
      case kActSilu: act_each<kActSilu>(v); break;
      default: break;
    }
    if (e.R) {
#pragma unroll
      for (int i = 0; i < U * C; ++i) v[i] += res[i];
    }
    store(Y, ldy);
  }
}

}  // namespace sgc
