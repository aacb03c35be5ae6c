// Kernels around the product of a linear layer: packing an FP32 operand (power-of-two scaling found on
// the device, then the two-word split), the gradient in front of the activation, and the product for a
// few rows.
#pragma once

#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "linear_epilogue.cuh"
#include "pack_job.cuh"
#include "ptx_sm100.cuh"
#include "split_math.cuh"

namespace sgc {

// Block-wide largest value, then one atomic per block; the last block of the job turns the largest
// magnitude into the exponent and leaves the two words zero for the next call.  A maximum does not
// depend on the order of its operands, so the result is the same every time.
__device__ __forceinline__ void publish_amax(uint32_t m, unsigned int* amax_word, unsigned int* count_word,
                                             unsigned int blocks, int* exp_out) {
  __shared__ uint32_t warp_max[32];
  m = __reduce_max_sync(0xffffffffu, m);
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) warp_max[warp] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) m = max(m, warp_max[w]);
    atomicMax(amax_word, m);
    __threadfence();
    if (atomicAdd(count_word, 1u) == blocks - 1) {
      __threadfence();
      *exp_out = pack_exponent(atomicExch(amax_word, 0u));
      atomicExch(count_word, 0u);
    }
  }
}

// Largest finite magnitude of one or two matrices.  One read of each: 4 bytes per element.
// The first `blocks_a` blocks take job a.
__global__ void __launch_bounds__(256)
pack_range_kernel(PackJob a, PackJob b, unsigned int blocks_a, unsigned int* words) {
  const bool second = blockIdx.x >= blocks_a;
  const PackJob& j = second ? b : a;
  const unsigned int nblk = second ? gridDim.x - blocks_a : blocks_a;
  const unsigned int blk = second ? blockIdx.x - blocks_a : blockIdx.x;
  uint32_t m = 0;
  // Items are 4 elements of a row (vector) or single elements; every thread has four in flight.  Rows behind one another are one
  // vector, whatever their width; what lies in front of its first 16 bytes and behind its last is the first block's.
  const bool flat = j.ldx == j.cols, quads = flat || j.vec;
  const long long all = (long long)j.rows * j.cols;
  const int head = flat ? (int)min(all, (long long)((16 - (reinterpret_cast<uintptr_t>(j.X) & 15)) % 16 / 4)) : 0;
  const long long per_row = quads ? j.cols >> 2 : j.cols;
  const long long total = flat ? (all - head) >> 2 : (long long)j.rows * per_row;
  const long long stride = (long long)nblk * 256;
  if (flat && blk == 0) {
    if ((int)threadIdx.x < head) m = finite_bits(j.X[threadIdx.x]);
    if (head + 4 * total + threadIdx.x < all) m = max(m, finite_bits(j.X[head + 4 * total + threadIdx.x]));
  }
  auto at = [&](long long it) -> const float* {
    if (flat) return j.X + head + it * 4;
    const long long r = total < (1ll << 31) ? (long long)((uint32_t)it / (uint32_t)per_row) : it / per_row;
    return j.X + r * j.ldx + (it - r * per_row) * (j.vec ? 4 : 1);
  };
  long long it = (long long)blk * 256 + threadIdx.x;
  if (quads) {
    for (; it + 3 * stride < total; it += 4 * stride) {
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float4*>(at(it + u * stride));
#pragma unroll
      for (int u = 0; u < 4; ++u)
        m = max(m, max(max(finite_bits(v[u].x), finite_bits(v[u].y)), max(finite_bits(v[u].z), finite_bits(v[u].w))));
    }
    for (; it < total; it += stride) {
      const float4 v = *reinterpret_cast<const float4*>(at(it));
      m = max(m, max(max(finite_bits(v.x), finite_bits(v.y)), max(finite_bits(v.z), finite_bits(v.w))));
    }
  } else {
    for (; it + 3 * stride < total; it += 4 * stride) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *at(it + u * stride);
#pragma unroll
      for (int u = 0; u < 4; ++u) m = max(m, finite_bits(v[u]));
    }
    for (; it < total; it += stride) m = max(m, finite_bits(*at(it)));
  }
  publish_amax(m, words + (second ? 1 : 0), words + (second ? 3 : 2), nblk, j.exp);
}

// The gradient in front of the activation, dz = dY act'(Z), in one pass over dY and Z: its largest
// finite magnitude, and its column sums (the bias gradient) as one partial row per row chunk, added up
// in a fixed order by the kernel that splits dz.  Block: 128 columns x 8 rows a step, four columns a lane.
// grid (ceil(cols / 128), chunks).
template <int ACT>
__global__ void __launch_bounds__(256)
dz_range_kernel(PackJob j, float* __restrict__ col_part, int rows_per_chunk, unsigned int* words) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * 128;
  const int r_end = (int)min((long long)j.rows, (long long)(blockIdx.y + 1) * rows_per_chunk);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t m = 0;
  int col[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) col[q] = j.vec ? c0 + lane * 4 + q : c0 + q * 32 + lane;
  constexpr int U = 4;                                       // rows in flight per thread
  for (int r0 = blockIdx.y * rows_per_chunk + warp; r0 < r_end; r0 += 8 * U) {
    float dy[U][4], z[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + 8 * u;
      const float* x = j.X + (long long)r * j.ldx;
      const float* zp = ACT != kActNone ? j.Z + (long long)r * j.ldz : nullptr;
      if (j.vec) {                                           // cols % 4 == 0: a lane has all four or none
        const bool in = r < r_end && col[0] < j.cols;
        const float4 v = in ? *reinterpret_cast<const float4*>(x + col[0]) : make_float4(0.f, 0.f, 0.f, 0.f);
        dy[u][0] = v.x; dy[u][1] = v.y; dy[u][2] = v.z; dy[u][3] = v.w;
        if (ACT != kActNone) {
          const float4 w = in ? *reinterpret_cast<const float4*>(zp + col[0]) : make_float4(0.f, 0.f, 0.f, 0.f);
          z[u][0] = w.x; z[u][1] = w.y; z[u][2] = w.z; z[u][3] = w.w;
        }
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bool in = r < r_end && col[q] < j.cols;
          dy[u][q] = in ? x[col[q]] : 0.f;
          if (ACT != kActNone) z[u][q] = in ? zp[col[q]] : 0.f;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float d = dy[u][q];
        if (ACT != kActNone) d *= act_slope(ACT, z[u][q]);
        m = max(m, finite_bits(d));
        sum[q] += d;
      }
  }
  if (col_part) {
    __shared__ float part[8][128];
#pragma unroll
    for (int q = 0; q < 4; ++q) part[warp][col[q] - c0] = sum[q];
    __syncthreads();
    const int t = threadIdx.x;
    if (t < 128 && c0 + t < j.cols) {
      float s = part[0][t];
      for (int w = 1; w < 8; ++w) s += part[w][t];
      col_part[(long long)blockIdx.y * j.cols + c0 + t] = s;
    }
  }
  if (words) publish_amax(m, words, words + 2, gridDim.x * gridDim.y, j.exp);
}

// Eight elements of a row on any address, out of the three 16-byte words that hold them (both passes over 50001 x 1001 107 us; by
// elements 111, and 130 with the range pass by elements, too).  The caller sees that those lie in the matrix.
__device__ __forceinline__ void load_eight(const float* src, float (&v)[8]) {
  const uintptr_t addr = reinterpret_cast<uintptr_t>(src);
  const float4* words = reinterpret_cast<const float4*>(addr & ~uintptr_t(15));
  const bool one = addr & 4, two = addr & 8;
  const float4 a = words[0], b = words[1], c = words[2];
  const float w[12] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z, c.w};
  float s[11];
#pragma unroll
  for (int q = 0; q < 11; ++q) s[q] = one ? w[q + 1] : w[q];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = two ? s[q + 2] : s[q];
}

// The split of one or two matrices (or of dz): 2^p x as hi, lo words.  Item: 8 consecutive elements of a
// row.  Bytes per element: 4 (dz: 8) read, 4 written: bound by memory (16384 x 4096 81 us, 6.6 TB/s; the range pass
// before it 54, 5 TB/s beside the writing back of what the kernels before left in L2; dz of 8192 x 16384 with gelu
// 281, 5.7 TB/s, its range pass 224).
template <int ACT, bool DZ>
__device__ __forceinline__ void pack_items(const PackJob& j, long long first, long long stride) {
  const float pre = pow2f(*j.exp);
  const float scale = pow2f(kPackScaleExp);
  const int per_row = (j.cols + 7) >> 3;
  const long long total = (long long)j.rows * per_row;
  const float* end = j.X + (long long)(j.rows - 1) * j.ldx + j.cols;
  // From the end to the start: the range pass before read from start to end, so what it read last is
  // still in L2.
  for (long long it = total - 1 - first; it >= 0; it -= stride) {
    const long long r = total < (1ll << 31) ? (long long)((uint32_t)it / (uint32_t)per_row) : it / per_row;
    const int c = (int)(it - r * per_row) << 3;
    const float* src = j.X + r * j.ldx + c;
    float v[8];
    if (j.vec && c + 8 <= j.cols) {
      const float4 a = *reinterpret_cast<const float4*>(src);
      const float4 b = *reinterpret_cast<const float4*>(src + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else if (!DZ && c + 8 <= j.cols && src - j.X >= 3 && end - src >= 12) {
      load_eight(src, v);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = c + q < j.cols ? src[q] : 0.f;
    }
    if (DZ && ACT != kActNone) {
      const float* zp = j.Z + r * j.ldz + c;
      if (j.vec && c + 8 <= j.cols) {
        const float4 a = *reinterpret_cast<const float4*>(zp);
        const float4 b = *reinterpret_cast<const float4*>(zp + 4);
        v[0] *= act_slope(ACT, a.x); v[1] *= act_slope(ACT, a.y);
        v[2] *= act_slope(ACT, a.z); v[3] *= act_slope(ACT, a.w);
        v[4] *= act_slope(ACT, b.x); v[5] *= act_slope(ACT, b.y);
        v[6] *= act_slope(ACT, b.z); v[7] *= act_slope(ACT, b.w);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = c + q < j.cols ? v[q] * act_slope(ACT, zp[q]) : 0.f;
      }
    }
    uint4 h, l;
    split_two(v[0] * pre, v[1] * pre, scale, h.x, l.x);
    split_two(v[2] * pre, v[3] * pre, scale, h.y, l.y);
    split_two(v[4] * pre, v[5] * pre, scale, h.z, l.z);
    split_two(v[6] * pre, v[7] * pre, scale, h.w, l.w);
    *reinterpret_cast<uint4*>(j.hi + r * j.ldh + c) = h;
    *reinterpret_cast<uint4*>(j.lo + r * j.ldh + c) = l;
  }
}

__global__ void __launch_bounds__(256) pack_split_kernel(PackJob a, PackJob b, unsigned int blocks_a) {
  if (blockIdx.x < blocks_a)
    pack_items<kActNone, false>(a, (long long)blockIdx.x * 256 + threadIdx.x, (long long)blocks_a * 256);
  else
    pack_items<kActNone, false>(b, (long long)(blockIdx.x - blocks_a) * 256 + threadIdx.x,
                                (long long)(gridDim.x - blocks_a) * 256);
}

// The bias gradient from its partial rows, in chunk order.
__device__ __forceinline__ void add_column_parts(const float* part, int chunks, int cols, float* out, int col) {
  if (col >= cols) return;
  float s = part[col];
#pragma unroll 8
  for (int c = 1; c < chunks; ++c) s += part[(long long)c * cols + col];
  out[col] = s;
}
__global__ void __launch_bounds__(256)
column_parts_kernel(const float* __restrict__ part, int chunks, int cols, float* __restrict__ out) {
  add_column_parts(part, chunks, cols, out, blockIdx.x * 256 + threadIdx.x);
}

// Splits dz; the last `sum_blocks` blocks add up the bias gradient instead.
template <int ACT>
__global__ void __launch_bounds__(256)
dz_split_kernel(PackJob j, unsigned int sum_blocks, const float* __restrict__ part, int chunks,
                float* __restrict__ dbias) {
  const unsigned int split_blocks = gridDim.x - sum_blocks;
  if (blockIdx.x >= split_blocks)
    add_column_parts(part, chunks, j.cols, dbias, (blockIdx.x - split_blocks) * 256 + threadIdx.x);
  else
    pack_items<ACT, true>(j, (long long)blockIdx.x * 256 + threadIdx.x, (long long)split_blocks * 256);
}

// ---------------------------------------------------------------------------------- one launch for both
// Matrices that fit the registers of the blocks that are resident at once (32 elements a thread, 4.8 million in
// all) are packed in one cooperative launch: every block reads its part once, the blocks agree on the largest
// magnitude, and each splits what it holds: bound by the launch, one load and the blocks' meeting (777 x 1001 and
// 1001 x 2049 together 11 us, 16 in two launches; 1024 x 1024 8).
struct GridWords {             // zero between calls
  unsigned int amax[2];        // of up to two jobs
  unsigned int arrived, left;
};

// Publishes a block's largest magnitude for its job and waits for all blocks; returns the job's.  The last block to
// leave clears the words.  The launch is cooperative, so all blocks run; the wait is bounded all the same.
__device__ __forceinline__ bool agree_on_amax(uint32_t m, int job, GridWords* words, unsigned int* err, uint32_t& amax) {
  __shared__ uint32_t warp_max[32];
  __shared__ uint32_t result[2];
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) m = max(m, warp_max[w]);
    const unsigned int blocks = gridDim.x * gridDim.y;
    atomicMax(&words->amax[job], m);
    __threadfence();
    atomicAdd(&words->arrived, 1u);
    const long long t0 = clock64();
    unsigned int seen = 0;
    bool ok = true;
    while (true) {
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&words->arrived) : "memory");
      if (seen >= blocks) break;
      __nanosleep(32);                                   // the arrivals need the line, too
      if (clock64() - t0 > kWaitLimitClocks) { ok = false; break; }
    }
    if (ok) {
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(result[0]) : "l"(&words->amax[job]) : "memory");
      __threadfence();
      if (atomicAdd(&words->left, 1u) == blocks - 1) {
        words->amax[0] = words->amax[1] = 0u;
        words->arrived = words->left = 0u;
      }
    } else {
      atomicExch(err, (unsigned int)kErrPackWait);
    }
    result[1] = ok;
  }
  __syncthreads();
  amax = result[0];
  return result[1] != 0;
}

constexpr int kOnceItems = 4;  // of 8 elements, a thread

// The first `blocks_a` blocks take job a.
__global__ void __launch_bounds__(256, 4)
pack_once_kernel(PackJob a, PackJob b, unsigned int blocks_a, GridWords* words, unsigned int* err) {
  const bool second = blockIdx.x >= blocks_a;
  const PackJob& j = second ? b : a;
  const unsigned int nblk = second ? gridDim.x - blocks_a : blocks_a;
  const unsigned int blk = second ? blockIdx.x - blocks_a : blockIdx.x;
  constexpr int U = kOnceItems;
  const int per_row = (j.cols + 7) >> 3;
  const int total = j.rows * per_row;                    // within 32 bits: the matrix is small
  float v[U][8];
  int row[U], col[U];
  uint32_t m = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int it = ((int)blk + u * (int)nblk) * 256 + (int)threadIdx.x;
    row[u] = it < total ? it / per_row : -1;
    col[u] = (it - row[u] * per_row) << 3;
    if (row[u] < 0) col[u] = j.cols;
    const float* src = j.X + (long long)max(row[u], 0) * j.ldx + col[u];
    if (j.vec && col[u] + 8 <= j.cols) {
      const float4 f = *reinterpret_cast<const float4*>(src);
      const float4 g = *reinterpret_cast<const float4*>(src + 4);
      v[u][0] = f.x; v[u][1] = f.y; v[u][2] = f.z; v[u][3] = f.w;
      v[u][4] = g.x; v[u][5] = g.y; v[u][6] = g.z; v[u][7] = g.w;
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[u][q] = col[u] + q < j.cols ? src[q] : 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int q = 0; q < 8; ++q) m = max(m, finite_bits(v[u][q]));
  uint32_t amax;
  if (!agree_on_amax(m, second ? 1 : 0, words, err, amax)) return;
  const int p = pack_exponent(amax);
  if (blk == 0 && threadIdx.x == 0) *j.exp = p;
  const float pre = pow2f(p), scale = pow2f(kPackScaleExp);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] < 0) continue;
    uint4 h, l;
    split_two(v[u][0] * pre, v[u][1] * pre, scale, h.x, l.x);
    split_two(v[u][2] * pre, v[u][3] * pre, scale, h.y, l.y);
    split_two(v[u][4] * pre, v[u][5] * pre, scale, h.z, l.z);
    split_two(v[u][6] * pre, v[u][7] * pre, scale, h.w, l.w);
    *reinterpret_cast<uint4*>(j.hi + row[u] * j.ldh + col[u]) = h;
    *reinterpret_cast<uint4*>(j.lo + row[u] * j.ldh + col[u]) = l;
  }
}

// The same for dz with its column sums: a block holds 128 columns x 64 rows, a thread four columns of eight rows.
// grid (ceil(cols / 128), ceil(rows / 64)); the first row of blocks adds up the bias gradient.
constexpr int kOnceRows = 64;
template <int ACT>
__global__ void __launch_bounds__(256, 4)
dz_once_kernel(PackJob j, float* col_part, float* dbias, GridWords* words, unsigned int* err) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * 128 + lane * 4;
  constexpr int U = kOnceRows / 8;
  float v[U][4];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t m = 0;
  float z[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = blockIdx.y * kOnceRows + warp + 8 * u;
    const float* x = j.X + (long long)r * j.ldx + c0;
    const float* zp = ACT != kActNone ? j.Z + (long long)r * j.ldz + c0 : nullptr;
    if (j.vec && r < j.rows && c0 < j.cols) {            // cols % 4 == 0: a lane has all four or none
      const float4 f = *reinterpret_cast<const float4*>(x);
      v[u][0] = f.x; v[u][1] = f.y; v[u][2] = f.z; v[u][3] = f.w;
      if (ACT != kActNone) {
        const float4 g = *reinterpret_cast<const float4*>(zp);
        z[u][0] = g.x; z[u][1] = g.y; z[u][2] = g.z; z[u][3] = g.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bool in = r < j.rows && c0 + q < j.cols;
        v[u][q] = in ? x[q] : 0.f;
        if (ACT != kActNone) z[u][q] = in ? zp[q] : 0.f;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (ACT != kActNone) v[u][q] *= act_slope(ACT, z[u][q]);
      m = max(m, finite_bits(v[u][q]));
      sum[q] += v[u][q];
    }
  if (dbias) {
    __shared__ float part[8][128];
#pragma unroll
    for (int q = 0; q < 4; ++q) part[warp][lane * 4 + q] = sum[q];
    __syncthreads();
    const int t = threadIdx.x, c = blockIdx.x * 128 + t;
    if (t < 128 && c < j.cols) {
      float s = part[0][t];
      for (int w = 1; w < 8; ++w) s += part[w][t];
      col_part[(long long)blockIdx.y * j.cols + c] = s;
    }
    __threadfence();                                     // the partial rows, before the block arrives
    __syncthreads();
  }
  uint32_t amax;
  if (!agree_on_amax(m, 0, words, err, amax)) return;
  const int p = pack_exponent(amax);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *j.exp = p;
  const float pre = pow2f(p), scale = pow2f(kPackScaleExp);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = blockIdx.y * kOnceRows + warp + 8 * u;
    if (r >= j.rows || c0 >= ((j.cols + 7) & ~7)) continue;
    uint2 h, l;
    split_two(v[u][0] * pre, v[u][1] * pre, scale, h.x, l.x);
    split_two(v[u][2] * pre, v[u][3] * pre, scale, h.y, l.y);
    *reinterpret_cast<uint2*>(j.hi + r * j.ldh + c0) = h;
    *reinterpret_cast<uint2*>(j.lo + r * j.ldh + c0) = l;
  }
  if (dbias && blockIdx.y == 0 && threadIdx.x < 128) {
    const int c = blockIdx.x * 128 + threadIdx.x;
    if (c < j.cols) {
      float s = __ldcg(col_part + c);
#pragma unroll 8
      for (int k = 1; k < (int)gridDim.y; ++k) s += __ldcg(col_part + (long long)k * j.cols + c);
      dbias[c] = s;
    }
  }
}

// The empty inner dimension: y = act(b) + R.
__global__ void __launch_bounds__(256)
linear_empty_kernel(int M, int N, float* Y, long long ldy, LinearEpilogue e) {
  const long long total = (long long)M * N;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < total; it += (long long)gridDim.x * 256) {
    const long long r = it / N;
    const int c = (int)(it - r * N);
    Y[r * ldy + c] = linear_finish(e, e.bias ? e.bias[c] : 0.f, r, c);
  }
}

// ------------------------------------------------------------------------------------------ few rows
// Up to eight rows of X: the product is bound by the bytes of W (4 per weight, FP32 or two words), so W
// streams past the rows once and FP32 FMAs on the ordinary cores keep up; no tile is padded to 128 rows
// and an FP32 W needs no packing.  A packed weight is put together again as 2^-p (hi + 2^-11 lo) (22 bits), so that the
// products and the partial sums have the size of the result's own terms and not 2^p times that.
// One row of 4096 x 1024 packed 6.7 us, of 16384 x 4096 47 (5.7 TB/s); with more rows the loads of X and the FMAs
// take over (FP32 weight, 4 rows 75, 8 rows 155), which is where the tensor cores are asked instead.
struct FewRowsParams {
  int M, N, K;
  const float* X;
  long long ldx;
  const float* W;            // FP32, or null
  const uint16_t* Whi;
  const uint16_t* Wlo;
  long long ldw;
  float* Y;
  long long ldy;
  int xvec;                  // X takes 16-byte loads
  LinearEpilogue ep;         // exp_a null; exp_b for a packed W
};
enum FewRowsLoad { kLoadPacked = 0, kLoadF32Vec, kLoadF32 };
// Blocks an SM that their loads in flight leave registers for (one packed row of 16384 x 4096: four 46 us, three 57; and
// below, four FP32 rows of 4096 x 4096: 64 registers 25 us, the 48 of five blocks 37).
constexpr int few_rows_blocks(int rows) { return rows == 1 ? 4 : (rows == 4 ? 2 : 3); }

__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
// Two weights from their words: up = 2^-p, up_lo = 2^(-11-p), each twice in a register pair.
__device__ __forceinline__ void join_words(uint32_t h2, uint32_t l2, uint64_t up, uint64_t up_lo, float& w0, float& w1) {
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&h2));
  const float2 l = __half22float2(*reinterpret_cast<const __half2*>(&l2));
  uint64_t a, b;
  asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(h.x), "f"(h.y));
  asm("mov.b64 %0, {%1, %2};" : "=l"(b) : "f"(l.x), "f"(l.y));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a) : "l"(a), "l"(up));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(a) : "l"(b), "l"(up_lo), "l"(a));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(w0), "=f"(w1) : "l"(a));
}

// Sums that FP32 may have got wrong at the ends of its range are taken once more in FP64, by the whole warp for one
// output after the other: at the lower end, where products have lost bits to underflow (2^-150 each), and those
// that are not finite, since products or partial sums can overflow where the sum does not (what is infinite or NaN
// in FP64 too stays so).  A sum of exactly zero is kept: rows of zeros are common, and products that all vanish
// add up to less than K 2^-150, which is below the smallest normal number.
// Sums like that are not met in a working model; nothing else is slowed by this.
constexpr float kTinySum = 7.5e-37f;                   // 2^-120
constexpr float kLargestFloat = 3.402823466e38f;
template <int LOAD>
__device__ __noinline__ float few_rows_again(const FewRowsParams& p, unsigned int todo, float z, int m, int n, bool nk) {
  const int lane = threadIdx.x & 31;
  for (; todo; todo &= todo - 1) {
    const int who = __ffs(todo) - 1;
    const int row = __shfl_sync(0xffffffffu, m, who), col = __shfl_sync(0xffffffffu, n, who);
    double s = 0.0;
    for (int k = lane; k < p.K; k += 32) {
      const long long off = nk ? col * p.ldw + k : k * p.ldw + col;
      double w;
      if (LOAD == kLoadPacked)
        w = (double)__half2float(__ushort_as_half(p.Whi[off])) +
            (double)kPackInvScale * (double)__half2float(__ushort_as_half(p.Wlo[off]));
      else
        w = (double)p.W[off];
      s += (double)p.X[row * p.ldx + k] * w;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == who) z = (float)ldexp(s, LOAD == kLoadPacked ? -*p.ep.exp_b : 0);
  }
  return z;
}
// z, or what FP64 makes of it; the whole warp calls, `in` says whose z is an output.
template <int LOAD>
__device__ __forceinline__ float few_rows_checked(const FewRowsParams& p, bool in, float z, int m, int n, bool nk) {
  const bool sure = z == 0.f || (fabsf(z) >= kTinySum && fabsf(z) <= kLargestFloat);
  const unsigned int todo = __ballot_sync(0xffffffffu, in && !sure);
  return todo ? few_rows_again<LOAD>(p, todo, z, m, n, nk) : z;
}

// W stored outputs x inputs (rows contiguous along k).  A group of `ksplit` warps owns NR outputs; lanes
// run along k, eight weights of every output a step; the lanes' sums meet in shuffles and the warps' in
// shared memory, always in the same order.  MR: rows computed (>= M; rows past M repeat the last).
template <int MR, int NR, int LOAD>
__global__ void __launch_bounds__(256, few_rows_blocks(MR))
few_rows_nk_kernel(FewRowsParams p, int ksplit) {
  constexpr int E = 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = 8 / ksplit, group = warp / ksplit, slice = warp % ksplit;
  const int n0 = (blockIdx.x * groups + group) * NR;
  float acc[NR][MR];
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int m = 0; m < MR; ++m) acc[i][m] = 0.f;
  // what the last step needs, asked for now: this thread's output
  const int out_n = (blockIdx.x * groups + threadIdx.x / (NR * MR)) * NR + threadIdx.x % (NR * MR) / MR;
  const bool out_in = threadIdx.x < groups * NR * MR && out_n < p.N && threadIdx.x % MR < p.M;
  const float out_bias = out_in && p.ep.bias ? __ldg(p.ep.bias + out_n) : 0.f;
  uint64_t up = 0, up_lo = 0;
  if constexpr (LOAD == kLoadPacked) {
    const float f = pow2f(-__ldg(p.ep.exp_b)), f_lo = f * kPackInvScale;   // (2^-137 at the least: subnormal, not lost)
    asm("mov.b64 %0, {%1, %1};" : "=l"(up) : "f"(f));
    asm("mov.b64 %0, {%1, %1};" : "=l"(up_lo) : "f"(f_lo));
  }
  // element e of the lane's step at k0: k0 + lane * 8 + e, or k0 + lane + 32 e where loads are single words
  constexpr int LS = LOAD == kLoadF32 ? 1 : E, ES = LOAD == kLoadF32 ? 32 : 1;
  for (int k0 = slice * 32 * E; k0 < p.K; k0 += ksplit * 32 * E) {
    const int k = k0 + lane * LS;
    if (k >= p.K) break;
    float w[NR][E];
    if (LOAD == kLoadPacked) {
      uint4 h[NR], l[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const long long off = (long long)min(n0 + i, p.N - 1) * p.ldw + k;
        h[i] = ldg_stream(p.Whi + off);
        l[i] = ldg_stream(p.Wlo + off);
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        join_words(h[i].x, l[i].x, up, up_lo, w[i][0], w[i][1]);
        join_words(h[i].y, l[i].y, up, up_lo, w[i][2], w[i][3]);
        join_words(h[i].z, l[i].z, up, up_lo, w[i][4], w[i][5]);
        join_words(h[i].w, l[i].w, up, up_lo, w[i][6], w[i][7]);
      }
    } else if (LOAD == kLoadF32Vec) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float* src = p.W + (long long)min(n0 + i, p.N - 1) * p.ldw + k;
        const uint4 a = ldg_stream(src);
        const uint4 b = k + 4 < p.K ? ldg_stream(src + 4) : make_uint4(0, 0, 0, 0);
        w[i][0] = __uint_as_float(a.x); w[i][1] = __uint_as_float(a.y);
        w[i][2] = __uint_as_float(a.z); w[i][3] = __uint_as_float(a.w);
        w[i][4] = __uint_as_float(b.x); w[i][5] = __uint_as_float(b.y);
        w[i][6] = __uint_as_float(b.z); w[i][7] = __uint_as_float(b.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float* src = p.W + (long long)min(n0 + i, p.N - 1) * p.ldw;
#pragma unroll
        for (int e = 0; e < E; ++e) w[i][e] = k + e * ES < p.K ? src[k + e * ES] : 0.f;
      }
    }
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      const float* xr = p.X + (long long)min(m, p.M - 1) * p.ldx;
      float x[E];
      if (LOAD != kLoadF32 && p.xvec && k + E <= p.K) {
        const float4 a = *reinterpret_cast<const float4*>(xr + k);
        const float4 b = *reinterpret_cast<const float4*>(xr + k + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = k + e * ES < p.K ? xr[k + e * ES] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[i][m] = fmaf(w[i][e], x[e], acc[i][m]);
    }
  }
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[i][m] += __shfl_xor_sync(0xffffffffu, acc[i][m], o);
  __shared__ float part[8][NR * MR];
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int m = 0; m < MR; ++m) part[warp][i * MR + m] = acc[i][m];
  }
  __syncthreads();
  // thread t of the block: output t / MR of the block's groups * NR, row t % MR (at most 8 * 16 of them)
  static_assert(8 * NR * MR <= 256, "one output a thread");
  const int t = threadIdx.x, n = out_n, m = t % MR;
  float z = 0.f;
  if (out_in) {
    const int g = t / (NR * MR), i = t % (NR * MR) / MR;
    z = part[g * ksplit][i * MR + m];
    for (int s = 1; s < ksplit; ++s) z += part[g * ksplit + s][i * MR + m];
  }
  z = few_rows_checked<LOAD>(p, out_in, z, m, n, true);
  if (out_in) p.Y[(long long)m * p.ldy + n] = linear_finish(p.ep, z + out_bias, m, n);
}

// W stored inputs x outputs (rows contiguous along n).  A block owns 128 outputs, four a lane, and its
// eight warps take every eighth k of the block's k range; the grid's y dimension cuts k into slices of a
// cluster, whose sums meet in the first block's shared memory, warps and blocks in order.
template <int MR, int LOAD>
__global__ void __launch_bounds__(256, MR <= 4 ? 4 : 1)
few_rows_kn_kernel(FewRowsParams p, int k_per_block) {
  static_assert(LOAD != kLoadPacked, "packed weights of this layout go to the tensor cores");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n0 = blockIdx.x * 128;
  const int k_begin = blockIdx.y * k_per_block, k_end = min(p.K, k_begin + k_per_block);
  float acc[MR][4];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[m][q] = 0.f;
  // output q of a lane: n0 + lane * 4 + q, or n0 + q * 32 + lane where loads are single words
  constexpr int LS = LOAD == kLoadF32 ? 1 : 4, QS = LOAD == kLoadF32 ? 32 : 1;
  const int n = n0 + lane * LS;
  constexpr int U = 4;                                 // k in flight per warp
  for (int k0 = k_begin + warp; k0 < k_end; k0 += 8 * U) {
    float w[U][4];
    if (LOAD == kLoadF32Vec) {                         // N % 4 == 0
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = k0 + 8 * u < k_end && n < p.N;
        const float4 v = in ? __ldcs(reinterpret_cast<const float4*>(p.W + (long long)(k0 + 8 * u) * p.ldw + n))
                            : make_float4(0.f, 0.f, 0.f, 0.f);
        w[u][0] = v.x; w[u][1] = v.y; w[u][2] = v.z; w[u][3] = v.w;
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w[u][q] = (k0 + 8 * u < k_end && n + q * QS < p.N) ? p.W[(long long)(k0 + 8 * u) * p.ldw + n + q * QS] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + 8 * u >= k_end) break;
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const float x = p.X[(long long)min(m, p.M - 1) * p.ldx + k0 + 8 * u];
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[m][q] = fmaf(w[u][q], x, acc[m][q]);
      }
    }
  }
  extern __shared__ float sums[];                      // [8][MR][128], then [MR][128] in sums[0]
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[(warp * MR + m) * 128 + lane * LS + q * QS] = acc[m][q];
  __syncthreads();
  for (int t = threadIdx.x; t < MR * 128; t += 256) {
    float s = sums[t];
    for (int w = 1; w < 8; ++w) s += sums[w * MR * 128 + t];
    sums[t] = s;
  }
  const uint32_t slices = gridDim.y;
  if (slices > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  if (blockIdx.y == 0) {
    const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(sums));
    for (int t = threadIdx.x; t < MR * 128; t += 256) {  // (whole warps)
      const int m = t >> 7, c = n0 + (t & 127);
      const bool in = m < p.M && c < p.N;
      float z = 0.f;
      if (in) {
        z = sums[t];
        for (uint32_t s = 1; s < slices; ++s) {
          uint32_t remote;
          float v;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(base + t * 4), "r"(s));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
          z += v;
        }
      }
      z = few_rows_checked<LOAD>(p, in, z, m, c, false);
      if (in) p.Y[(long long)m * p.ldy + c] = linear_finish(p.ep, z + (p.ep.bias ? p.ep.bias[c] : 0.f), m, c);
    }
  }
  if (slices > 1)                                      // a block's sums stay until the first has read them
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace sgc
