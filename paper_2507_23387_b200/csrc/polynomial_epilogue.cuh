// One step of a matrix polynomial on packed operands: what becomes of a finished product of matrices that are kept as
// FP16 words throughout,
//
//   v = alpha acc + beta R[row, col],
//
// acc the product of the words, R a matrix of words (its way back from words is in beta, the product's in alpha), v
// stored as words of pre v, or as FP32 with a residual of its own.  A symmetric product (X X', the square of a symmetric
// matrix) is formed in the tiles that reach the lower triangle only, and every element below the diagonal is stored at its
// mirror image too: half of the products, and a result that is symmetric to the bit.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "elements.cuh"
#include "linear_epilogue.cuh"
#include "pack_job.cuh"
#include "split_math.cuh"

namespace sgc {

struct PolynomialEpilogue {
  float alpha, beta, pre;
  const uint16_t* r_hi;       // words of R, or null; ld a multiple of 8, 16-byte aligned, as all words here
  const uint16_t* r_lo;
  long long ldr;
  uint16_t* hi;               // the result's words, or null
  uint16_t* lo;
  long long ldw;
  float* Y;                   // where hi is null: Y = scale v + keep Y_old, FP32 of any alignment
  long long ldy;
  const float* kept;          // Y_old, or null; may be Y itself
  long long ldk;
  float scale, keep;
  int vec;                    // Y and the kept matrix take 16-byte accesses
  int symmetric;              // M == N, tiles that reach the lower triangle only; R is symmetric too
  float* tiles;               // as in LinearEpilogue
};

// Tiles of 128 x 256 (pairs: 256 x 256) that reach the lower triangle of a matrix with num_m tile rows, and the
// coordinates of tile `t` of them: row by row; a row of pairs has one tile more than the row before, a row of
// single tiles every second time.
__host__ __device__ inline long long lower_tiles(int num_m, bool pair) {
  if (pair) return (long long)num_m * (num_m + 1) / 2;
  const long long g = num_m / 2;
  return g * (g + 1) + (num_m % 2) * (g + 1);
}
__device__ __forceinline__ void lower_tile_coords(int t, bool pair, int& tm, int& tn) {
  if (pair) {
    int g = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((long long)g * (g + 1) / 2 > t) --g;                      // (the root is rounded)
    while ((long long)(g + 1) * (g + 2) / 2 <= t) ++g;
    tm = g;
    tn = t - (int)((long long)g * (g + 1) / 2);
  } else {
    int g = (int)((sqrtf(4.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((long long)g * (g + 1) > t) --g;
    while ((long long)(g + 1) * (g + 2) <= t) ++g;
    const int rest = t - (int)((long long)g * (g + 1));
    tm = 2 * g + (rest > g ? 1 : 0);
    tn = rest - (rest > g ? g + 1 : 0);
  }
}

__device__ __forceinline__ void unpack_words(const uint4& hi, const uint4& lo, float f, float (&v)[8]) {
  const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
  const float f_lo = f * kPackInvScale;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&l[i]));
    v[2 * i] = fmaf(f, a.x, fmaf(f_lo, b.x, v[2 * i]));
    v[2 * i + 1] = fmaf(f, a.y, fmaf(f_lo, b.y, v[2 * i + 1]));
  }
}
__device__ __forceinline__ void pack_words(const float (&v)[8], float pre, uint4& hi, uint4& lo) {
  const float scale = pow2f(kPackScaleExp);
  split_two(v[0] * pre, v[1] * pre, scale, hi.x, lo.x);
  split_two(v[2] * pre, v[3] * pre, scale, hi.y, lo.y);
  split_two(v[4] * pre, v[5] * pre, scale, hi.z, lo.z);
  split_two(v[6] * pre, v[7] * pre, scale, hi.w, lo.w);
}
// The same for four elements.
__device__ __forceinline__ void unpack_words(const uint2& hi, const uint2& lo, float f, float4& v) {
  const float f_lo = f * kPackInvScale;
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hi.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi.y));
  const float2 c = __half22float2(*reinterpret_cast<const __half2*>(&lo.x)), d = __half22float2(*reinterpret_cast<const __half2*>(&lo.y));
  v.x = fmaf(f, a.x, fmaf(f_lo, c.x, v.x)); v.y = fmaf(f, a.y, fmaf(f_lo, c.y, v.y));
  v.z = fmaf(f, b.x, fmaf(f_lo, d.x, v.z)); v.w = fmaf(f, b.y, fmaf(f_lo, d.y, v.w));
}
__device__ __forceinline__ void pack_words(const float4& v, float pre, uint2& hi, uint2& lo) {
  const float scale = pow2f(kPackScaleExp);
  split_two(v.x * pre, v.y * pre, scale, hi.x, lo.x);
  split_two(v.z * pre, v.w * pre, scale, hi.y, lo.y);
}
// Eight words to `at`, or those of them that `take` has a bit for.
__device__ __forceinline__ void store_words(uint16_t* at, const uint4& w, uint32_t take) {
  if (take == 0xFFu) {
    *reinterpret_cast<uint4*>(at) = w;
  } else {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (take >> q & 1) at[q] = (uint16_t)(v[q >> 1] >> (q & 1 ? 16 : 0));
  }
}

// Which of the elements (r, c .. c + 7) lie on or below the diagonal, and which of (r .. r + 7, c) strictly below it.
__device__ __forceinline__ uint32_t on_or_below(int r, int c) {
  const int under = r - c;
  return under >= 7 ? 0xFFu : (under < 0 ? 0u : (2u << under) - 1u);
}
__device__ __forceinline__ uint32_t strictly_below(int r, int c) {
  const int under = c - r;
  return under < 0 ? 0xFFu : (under >= 7 ? 0u : 0xFFu & ~((2u << under) - 1u));
}
// y = scale v + keep k for up to eight columns, `left` of them inside the matrix.
__device__ __forceinline__ void store_eight(float* y, const float* k, float scale, float keep, bool vec, int left, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] *= scale;
  if (vec && left >= 8) {
#pragma unroll
    for (int q = 0; q < 8; q += 4) {
      float4 o = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
      if (k) {
        const float4 old = *reinterpret_cast<const float4*>(k + q);
        o.x = fmaf(keep, old.x, o.x); o.y = fmaf(keep, old.y, o.y);
        o.z = fmaf(keep, old.z, o.z); o.w = fmaf(keep, old.w, o.w);
      }
      *reinterpret_cast<float4*>(y + q) = o;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < left) y[q] = k ? fmaf(keep, k[q], v[q]) : v[q];
  }
}

__device__ __forceinline__ void store_four(float* y, const float* k, float scale, float keep, bool vec, int left, float4 v) {
  v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
  if (vec && left >= 4) {
    if (k) {
      const float4 old = *reinterpret_cast<const float4*>(k);
      v.x = fmaf(keep, old.x, v.x); v.y = fmaf(keep, old.y, v.y); v.z = fmaf(keep, old.z, v.z); v.w = fmaf(keep, old.w, v.w);
    }
    *reinterpret_cast<float4*>(y) = v;
  } else {
    y[0] = k ? fmaf(keep, k[0], v.x) : v.x;
    if (left > 1) y[1] = k ? fmaf(keep, k[1], v.y) : v.y;
    if (left > 2) y[2] = k ? fmaf(keep, k[2], v.z) : v.z;
    if (left > 3) y[3] = k ? fmaf(keep, k[3], v.w) : v.w;
  }
}

// 2^p / (norm + eps) as two FP32 factors (1 / norm can leave the FP32 range while the entries times it do not).  A matrix of
// zeros with eps = 0 stays one; a norm that is not finite makes every entry NaN.
__device__ __forceinline__ void norm_factors(double squares, float eps, float pre, float& f0, float& f1) {
  const double norm = sqrt(squares) + (double)eps;
  const double scale = norm == 0.0 ? 0.0 : (isfinite(norm) ? 1.0 / norm : (double)NAN);
  const int e = scale != 0.0 && isfinite(scale) ? max(-126, min(126, ilogb(scale) / 2)) : 0;
  f0 = pow2f(e);
  f1 = (float)(scale * (double)pow2f(-e)) * pre;
}
// Words of f0 f1 G for eight columns, `left` of them inside the matrix (zeros behind them).
template <typename T>
__device__ __forceinline__ void normalise_eight(const T* at, bool vec, int left, float f0, float f1, uint16_t* hi, uint16_t* lo) {
  constexpr int V = Elem<T>::kVec;
  float v[8];
  if (vec && left >= 8) {
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
      float x[V];
      Elem<T>::unpack(*reinterpret_cast<const uint4*>(at + i * V), x);
#pragma unroll
      for (int q = 0; q < V; ++q) v[i * V + q] = x[q];
    }
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < left ? Elem<T>::get(at[q]) : 0.f;
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] *= f0;
  uint4 h, l;
  pack_words(v, f1, h, l);
  *reinterpret_cast<uint4*>(hi) = h;
  *reinterpret_cast<uint4*>(lo) = l;
}

// Blocks of 32 x 32 of a finished tile, from `first` on every `step`-th (linear_epilogue.cuh describes the tile).  A
// lane has eight columns of every eighth row; for the mirror image it has eight rows of four columns.
__device__ __forceinline__ void polynomial_store(const PolynomialEpilogue& e, int M, int N, float* tile, int slices,
                                                 long long stride, int row0, int col0, int first, int step, int lane) {
  const int blocks = (min(128, M - row0) + 31) / 32 * 8;
#pragma unroll 1
  for (int b = first; b < blocks; b += step) {
    const int rb = (b >> 3) * 32, cb = (b & 7) * 32;
    const int r_first = row0 + rb, c_first = col0 + cb;
    if (c_first >= N || (e.symmetric && r_first + 31 < c_first)) continue;
    {
      const int lr = lane >> 2, c = c_first + (lane & 3) * 8;
      const float4* src = tile_slot(tile, (cb >> 2) + (lane & 3) * 2, rb + lr);
#pragma unroll
      for (int half = 0; half < 2; ++half) {                 // two rows at a time, 8 apart
        float v[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float4 f = __ldcg(src + 8 * (2 * half + u) + q * 128);
            v[u][4 * q] = f.x; v[u][4 * q + 1] = f.y; v[u][4 * q + 2] = f.z; v[u][4 * q + 3] = f.w;
          }
#pragma unroll 1
        for (int s = 1; s < slices; ++s) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const float4 f = __ldcg(src + s * (stride / 4) + 8 * (2 * half + u) + q * 128);
              v[u][4 * q] += f.x; v[u][4 * q + 1] += f.y; v[u][4 * q + 2] += f.z; v[u][4 * q + 3] += f.w;
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const long long r = r_first + lr + 8 * (2 * half + u);
          if (r >= M || c >= N) continue;
#pragma unroll
          for (int q = 0; q < 8; ++q) v[u][q] *= e.alpha;
          if (e.r_hi)
            unpack_words(*reinterpret_cast<const uint4*>(e.r_hi + r * e.ldr + c),
                         *reinterpret_cast<const uint4*>(e.r_lo + r * e.ldr + c), e.beta, v[u]);
          if (e.hi) {
            uint4 h, l;
            pack_words(v[u], e.pre, h, l);
            const uint32_t take = e.symmetric ? on_or_below((int)r, c) : 0xFFu;     // the rest comes from the mirror image
            store_words(e.hi + r * e.ldw + c, h, take);
            store_words(e.lo + r * e.ldw + c, l, take);
          } else {
            store_eight(e.Y + r * e.ldy + c, e.kept ? e.kept + r * e.ldk + c : nullptr, e.scale, e.keep, e.vec != 0, N - c, v[u]);
          }
        }
      }
    }
    if (!e.symmetric || r_first + 31 <= c_first) continue;
    const int rl = (lane & 3) * 8, r = r_first + rl, c = c_first + (lane >> 2) * 4;
    const float4* src = tile_slot(tile, (cb >> 2) + (lane >> 2), rb + rl);
    float4 f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __ldcg(src + i);
#pragma unroll 1
    for (int s = 1; s < slices; ++s) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 g = __ldcg(src + s * (stride / 4) + i);
        f[i].x += g.x; f[i].y += g.y; f[i].z += g.z; f[i].w += g.w;
      }
    }
    if (r >= M) continue;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const long long at = c + q;                            // element (r + i, at) goes to (at, r + i)
      const uint32_t take = strictly_below(r, c + q);
      if (at >= N || take == 0u) continue;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = e.alpha * (q == 0 ? f[i].x : (q == 1 ? f[i].y : (q == 2 ? f[i].z : f[i].w)));
      if (e.r_hi)
        unpack_words(*reinterpret_cast<const uint4*>(e.r_hi + at * e.ldr + r),
                     *reinterpret_cast<const uint4*>(e.r_lo + at * e.ldr + r), e.beta, v);
      uint4 h, l;
      pack_words(v, e.pre, h, l);
      store_words(e.hi + at * e.ldw + r, h, take);
      store_words(e.lo + at * e.ldw + r, l, take);
    }
  }
}

}  // namespace sgc
