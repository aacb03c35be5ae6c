// The logits' part in a softmax cross entropy, taken from a finished tile of the product X W: z = 2^-(p_x + p_w) acc + b.
// Of every row and every 64 columns the largest logit m and the sum of exp(z - m) are kept (8 bytes for 256), and the
// target's logit; the logits themselves are stored only where a gradient is going to be formed of them.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "linear_epilogue.cuh"

namespace sgc {

constexpr int kLossColumns = 64;       // columns that a pair (m, sum) stands for
constexpr float kLog2e = 1.4426950408889634f;

struct LossEpilogue {
  const int* exp_a;         // exponents of the packed operands (device)
  const int* exp_b;
  const float* bias;        // [N] or null
  const long long* targets; // [M]
  float* target_logit;      // [M]: written where a target is inside [0, N)
  float2* parts;            // [M][ldp]: (m, sum) of every 64 columns
  long long ldp;
  float* Z;                 // the logits, 16-byte aligned rows of at least N rounded up to 4, or null
  long long ldz;
  float* tiles;             // as in LinearEpilogue
};

// (m, sum) of a row's values, N of them in each of the lanes that differ in the bits of `mask`.  A row of -inf has
// (-inf, 0); NaN or +inf makes the sum NaN.
template <int N>
__device__ __forceinline__ float2 softmax_part(const float (&v)[N], int lanes) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
  for (int x = 1; x < lanes; x *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  const float base = m == -INFINITY ? 0.f : m;               // (the difference first: large logits keep their digits)
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s += fast_exp2((v[i] - base) * kLog2e);
  for (int x = 1; x < lanes; x *= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
  return make_float2(m, s);
}

// Pieces of 32 rows x 64 columns of a finished tile, from `first` on every `step`-th: a lane has four columns of every 16
// in four rows, 8 apart.
__device__ __forceinline__ void loss_store(const LossEpilogue& e, int M, int N, float* tile, int slices, long long stride,
                                           int row0, int col0, int first, int step, int lane) {
  const PowerBack back = power_back(e.exp_a, e.exp_b);
  const int lr = lane >> 2, lc = lane & 3;
  const int pieces = (min(128, M - row0) + 31) / 32 * 4;
#pragma unroll 1
  for (int b = first; b < pieces; b += step) {
    const int rb = (b >> 2) * 32, cb = (b & 3) * kLossColumns;
    if (col0 + cb >= N) continue;
    const int c = col0 + cb + lc * 4;
    float bias[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int col = c + (i >> 2) * 16 + (i & 3);
      bias[i] = e.bias && col < N ? __ldg(e.bias + col) : 0.f;
    }
#pragma unroll 1
    for (int u = 0; u < 4; ++u) {
      const int r = rb + lr + 8 * u;
      const long long row = row0 + r;
      const float4* src = tile_slot(tile, (cb >> 2) + lc, r);
      float v[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 f = __ldcg(src + i * 4 * 128);
#pragma unroll 1
        for (int s = 1; s < slices; ++s) {
          const float4 g = __ldcg(src + i * 4 * 128 + s * (stride / 4));
          f.x += g.x; f.y += g.y; f.z += g.z; f.w += g.w;
        }
        v[4 * i] = back(f.x); v[4 * i + 1] = back(f.y); v[4 * i + 2] = back(f.z); v[4 * i + 3] = back(f.w);
      }
      const long long target = row < M ? e.targets[row] : -1;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int col = c + (i >> 2) * 16 + (i & 3);
        v[i] += bias[i];
        if (col == target) e.target_logit[row] = v[i];
      }
      if (e.Z && row < M) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i * 16 < N)
            *reinterpret_cast<float4*>(e.Z + row * e.ldz + c + i * 16) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (c + (i >> 2) * 16 + (i & 3) >= N) v[i] = -INFINITY;
      const float2 part = softmax_part(v, 4);
      if (lc == 0 && row < M) e.parts[row * e.ldp + (col0 + cb) / kLossColumns] = part;
    }
  }
}

}  // namespace sgc
