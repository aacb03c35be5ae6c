// Softmax cross entropy of a linear layer's outputs over a large vocabulary, from the layer's inputs, and its gradients
// (contracts: include/sgemm_cube.h).
//
//   z = X W + b,  lse = log sum_j exp(z_j),  loss = lse - z_t,  dz = dloss (exp(z - lse) - 1[t]),
//   dX = dz W^T,  dW = X^T dz,  db = column sums of dz.
//
// Forward: the logits stay in the product's tiles; (largest, sum) of every 64 of them is what a tile leaves behind
// (loss_epilogue.cuh), and one pass over those pairs gives lse and the loss.  (Few rows: the linear layer's forms for them write the logits.)
// Gradients: a piece of the rows at a time.  Its logits (1 GiB at most) go to the workspace once and are turned into
// the FP16 words of dz (as much again), which both products read: three products in all.  (In pieces of the vocabulary a piece's logits would have to
// be formed a second time once lse is known: four products.)  The words' exponent is known before them, |dz| <= |dloss|.
#include "ctx.cuh"
#include "product_host.cuh"

namespace sgc {

constexpr int kFormLossKM = form_of(kFormKM, kEpiLoss), kFormLossKK = form_of(kFormKK, kEpiLoss);

struct LossJoinParams {
  int rows, vocab, per_row;
  const float2* parts;
  long long ldp;
  const long long* targets;
  const float* target_logit;
  float* loss;              // or null
  float* lse;               // or null
  float2* stats;            // (m, 1 / sum) of a row, or null
  const float* dloss;       // with the words below: the exponent of dz' words, |dz| <= |dloss| of a row with a target
  unsigned int* range;      // {largest so far, blocks that are through}, zero between calls
  int* exp;
  unsigned int* counts;     // cleared for the gradient's kernel, or null
  int n_counts;
};
// lse and loss of a row from its (largest, sum).  loss = (m - z_t) + log sum: the difference of two logits keeps its digits,
// whatever their size.
__device__ __forceinline__ void finish_row(const LossJoinParams& p, long long r, float2 acc, float target_logit) {
  const bool none = acc.x == -INFINITY && acc.y == 0.f;              // no logit above -inf
  const float log_sum = logf(acc.y);
  const long long t = p.targets[r];
  float loss = 0.f;
  if (t >= p.vocab) loss = NAN;
  else if (t >= 0) loss = none ? INFINITY : (acc.x - target_logit) + log_sum;
  if (p.loss) p.loss[r] = loss;
  if (p.lse) p.lse[r] = none ? -INFINITY : acc.x + log_sum;
  if (p.stats) p.stats[r] = make_float2(none ? 0.f : acc.x, none ? 0.f : 1.f / acc.y);
}
__device__ __forceinline__ float2 join_parts(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);              // both 0, or NaN
  return make_float2(m, a.y * expf(a.x - m) + b.y * expf(b.x - m));
}
// The largest |dloss| so far; the last of `blocks` makes the exponent of it and leaves zeros for the next call.
__device__ __forceinline__ void publish_weight(const LossJoinParams& p, uint32_t m, unsigned int blocks) {
  if (m) atomicMax(&p.range[0], m);
  __threadfence();
  if (atomicAdd(&p.range[1], 1u) == blocks - 1) {
    __threadfence();
    *p.exp = pack_exponent(atomicExch(&p.range[0], 0u));
    atomicExch(&p.range[1], 0u);
  }
}

// A block's (largest, sum), in thread 0: the threads' in a fixed tree.
template <int WARPS>
__device__ __forceinline__ float2 join_block(float2 acc) {
  for (int x = 16; x > 0; x >>= 1) {
    const float2 o = make_float2(__shfl_xor_sync(0xffffffffu, acc.x, x), __shfl_xor_sync(0xffffffffu, acc.y, x));
    acc = join_parts(acc, o);
  }
  __shared__ float2 warp_part[WARPS];
  if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = acc;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < WARPS; ++w) acc = join_parts(acc, warp_part[w]);
  return acc;
}

// lse and loss of a row from its pairs: a block a row, or (WARP) a warp a row where there are few pairs.  A thread joins its pairs
// in their order.
template <bool WARP>
__global__ void __launch_bounds__(128) loss_join_kernel(LossJoinParams p) {
  constexpr int T = WARP ? 32 : 128;
  const int t = threadIdx.x % T;
  if (p.counts)
    for (int i = blockIdx.x * 128 + threadIdx.x; i < p.n_counts; i += gridDim.x * 128) p.counts[i] = 0u;
  const long long r = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  float2 acc = make_float2(-INFINITY, 0.f);
  if (r < p.rows)
    for (int i0 = t; i0 < p.per_row; i0 += 4 * T) {
      float2 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i0 + u * T < p.per_row ? p.parts[r * p.ldp + i0 + u * T] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int u = 0; u < 4; ++u) acc = join_parts(acc, v[u]);
    }
  if constexpr (WARP) {
    for (int x = 16; x > 0; x >>= 1)
      acc = join_parts(acc, make_float2(__shfl_xor_sync(0xffffffffu, acc.x, x), __shfl_xor_sync(0xffffffffu, acc.y, x)));
  } else {
    acc = join_block<4>(acc);
  }
  if (t == 0 && r < p.rows) finish_row(p, r, acc, p.target_logit[r]);
  if (p.exp) {
    uint32_t m = t == 0 && r < p.rows && p.targets[r] >= 0 ? finite_bits(p.dloss[r]) : 0u;
    if constexpr (WARP) {
      __shared__ uint32_t most[4];
      if (t == 0) most[threadIdx.x >> 5] = m;
      __syncthreads();
      m = max(max(most[0], most[1]), max(most[2], most[3]));
    }
    if (threadIdx.x == 0) publish_weight(p, m, gridDim.x);
  }
}

// The same from logits that are there already (few rows: the linear layer's own forms wrote them, they are in L2): a
// cluster of blocks has a row, and its first block joins their pairs.  Rows start on 16 bytes.
constexpr int kRowThreads = 256;
__global__ void __launch_bounds__(kRowThreads) loss_rows_kernel(LossJoinParams p, const float* __restrict__ Z, long long ldz) {
  __shared__ float2 pairs[8];                                        // of the cluster's blocks, in the first
  const int ranks = (int)cluster_size(), rank = (int)cluster_ctarank();
  cluster_started();                                                 // waited for in front of the store to the first block
  if (p.counts)
    for (int i = blockIdx.x * kRowThreads + threadIdx.x; i < p.n_counts; i += gridDim.x * kRowThreads) p.counts[i] = 0u;
  const long long r = blockIdx.x / ranks;
  const float4* z = reinterpret_cast<const float4*>(Z + r * ldz);
  float2 acc = make_float2(-INFINITY, 0.f);
  constexpr int U = 4;
  const int quads = (p.vocab + 3) / 4, step = ranks * kRowThreads;
  for (int i0 = rank * kRowThreads + threadIdx.x; i0 < quads; i0 += U * step) {
    float v[4 * U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * step;
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (i < quads) q = z[i];
      const int left = p.vocab - 4 * i;                              // (what stands behind the row's end is not looked at)
      v[4 * u] = q.x;
      v[4 * u + 1] = left > 1 ? q.y : -INFINITY;
      v[4 * u + 2] = left > 2 ? q.z : -INFINITY;
      v[4 * u + 3] = left > 3 ? q.w : -INFINITY;
    }
    acc = join_parts(acc, softmax_part(v, 1));
  }
  acc = join_block<kRowThreads / 32>(acc);
  __syncwarp();
  cluster_wait_started();                                            // the first block runs before anyone writes to it
  if (threadIdx.x == 0) {
    const uint32_t at = mapa_u32(smem_u32(&pairs[rank]), 0);
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(acc.x), "f"(acc.y) : "memory");
  }
  __syncwarp();
  cluster_sync_all();
  if (rank == 0 && threadIdx.x == 0) {
    acc = pairs[0];
    for (int k = 1; k < ranks; ++k) acc = join_parts(acc, pairs[k]);
    const long long t = p.targets[r];
    finish_row(p, r, acc, t >= 0 && t < p.vocab ? Z[r * ldz + t] : 0.f);
    if (p.exp) publish_weight(p, t >= 0 ? finite_bits(p.dloss[r]) : 0u, (unsigned)p.rows);
  }
}

struct LossGradParams {
  int rows, vocab, rows_per_chunk;
  const float* Z;
  long long ldz;
  float* dz;                // dz in FP32 too, in the place of Z, or null
  const float2* stats;
  const float* dloss;
  const long long* targets;
  uint16_t* hi;             // words of dz, or null
  uint16_t* lo;
  long long ldw;
  const int* exp;
  float* col_part;          // [chunks][vocab] column sums of dz, or null
  unsigned int* counts;     // [blocks in x]: chunks that are there, zero before the launch
  float* dbias;             // the chunks' sums in their order, added to what is there for the second piece and on
  int add;
};
// dz = dloss (exp(z - m) / sum - 1[t]) of a piece of rows, as words, with its column sums.  A lane has eight columns; the warps
// of a block take every eighth row of its chunk, and the last block of a column adds the chunks' sums.  Bound by memory: 8 bytes
// a logit (2048 x 131072 343 us, 6.3 TB/s).
__global__ void __launch_bounds__(256) loss_grad_kernel(LossGradParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 256 + lane * 8;
  const int r_end = min(p.rows, (int)(blockIdx.y + 1) * p.rows_per_chunk);
  const float pre = p.hi ? pow2f(*p.exp) : 1.f;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  constexpr int U = 2;
  for (int r0 = blockIdx.y * p.rows_per_chunk + warp; r0 < r_end && c < p.vocab; r0 += 8 * U) {
    float4 a[U], b[U];
    float2 st[U];
    long long t[U];
    float g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + 8 * u, r_end - 1);
      const float* z = p.Z + (long long)r * p.ldz + c;               // (rows are 8 floats wide at least)
      a[u] = __ldcs(reinterpret_cast<const float4*>(z));
      b[u] = __ldcs(reinterpret_cast<const float4*>(z + 4));
      st[u] = p.stats[r];
      t[u] = p.targets[r];
      g[u] = p.dloss[r];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + 8 * u;
      if (r >= r_end) break;
      float weight = t[u] >= 0 ? g[u] : 0.f;
      if (t[u] >= p.vocab) weight = NAN;
      const bool none = st[u].y == 0.f;                              // nothing is allowed: no gradient
      const float w = none ? 0.f : weight * st[u].y;
      float d[8] = {a[u].x, a[u].y, a[u].z, a[u].w, b[u].x, b[u].y, b[u].z, b[u].w};
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        d[q] = c + q < p.vocab && t[u] >= 0 ? w * fast_exp2((d[q] - st[u].x) * kLog2e) : 0.f;
        if (c + q == t[u] && !none) d[q] -= weight;
        sum[q] += d[q];
      }
      if (p.dz) {
        float* out = p.dz + (long long)r * p.ldz + c;
        *reinterpret_cast<float4*>(out) = make_float4(d[0], d[1], d[2], d[3]);
        *reinterpret_cast<float4*>(out + 4) = make_float4(d[4], d[5], d[6], d[7]);
      }
      if (p.hi) {
        uint4 h, l;
        pack_words(d, pre, h, l);
        *reinterpret_cast<uint4*>(p.hi + (long long)r * p.ldw + c) = h;
        *reinterpret_cast<uint4*>(p.lo + (long long)r * p.ldw + c) = l;
      }
    }
  }
  if (p.col_part) {
    __shared__ float part[8][256];
#pragma unroll
    for (int q = 0; q < 8; ++q) part[warp][lane * 8 + q] = sum[q];
    __syncthreads();
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col < p.vocab) {
      float s = part[0][threadIdx.x];
      for (int w = 1; w < 8; ++w) s += part[w][threadIdx.x];
      p.col_part[(long long)blockIdx.y * p.vocab + col] = s;
    }
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&p.counts[blockIdx.x], 1u) == gridDim.y - 1;
    __syncthreads();
    if (last && col < p.vocab) {
      __threadfence();
      float s = p.add ? p.dbias[col] : 0.f;
#pragma unroll 8
      for (int i = 0; i < (int)gridDim.y; ++i) s += __ldcg(p.col_part + (long long)i * p.vocab + col);
      p.dbias[col] = s;
    }
  }
}

// Products of few rows with an FP32 matrix, in FP32, up to 16 rows at a time: Y[m, j] = sum over i of A[m, i] W(i, j).  The matrix streams
// past the rows once, and a long sum is shared by many blocks, whose parts are added in order.  4 bytes an entry of W, latency above
// a few rows (12 rows of 65536 x 1024 119 us, 2.3 TB/s: 64 sums a thread leave 16 warps an SM).  Used where the linear layer's forms for few rows have no
// work for all SMs (they share a sum among 8 blocks at most: dX of one row of 65536 x 1024 took 230 us, here 60), or would have to
// pack W first because its rows are not on 16 bytes.
struct FewProduct {
  int M, J, I;               // rows, outputs, length of the sums
  const float* A;
  long long lda;
  const float* W;
  long long ldw;
  int run;                   // of a block's sum; a multiple of 32
  float* part;               // [runs][M_all][J], at this group's first row
  long long part_stride;     // M_all * J
};
constexpr int kFewChunk = 256, kFewMost = 16;           // entries of a sum between two loads of A; rows

// W's rows are the summed index: a block has 128 outputs and a run of rows, a warp four rows in every 32, a lane four outputs.
template <int MR, bool VEC>
__global__ void __launch_bounds__(256) few_rows_sums_kernel(FewProduct p) {
  __shared__ __align__(16) float d[MR][kFewChunk];
  __shared__ __align__(16) float sums[8][4][128];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x * 128;
  const int n_first = (int)min((long long)p.I, (long long)blockIdx.y * p.run), n_end = (int)min((long long)p.I, (long long)(blockIdx.y + 1) * p.run);
  int col[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) col[q] = c0 + (VEC ? lane * 4 + q : q * 32 + lane);
  float acc[MR][4];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[m][q] = 0.f;
  for (int n0 = n_first; n0 < n_end; n0 += kFewChunk) {
    __syncthreads();
    for (int i = threadIdx.x; i < MR * kFewChunk; i += 256) {
      const int m = i / kFewChunk, n = n0 + i % kFewChunk;
      d[m][i % kFewChunk] = m < p.M && n < n_end ? p.A[m * p.lda + n] : 0.f;
    }
    __syncthreads();
    const int rows = min(kFewChunk, n_end - n0);
#pragma unroll 1
    for (int i = warp * 4; i < rows; i += 32) {
      float w[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* at = p.W + (long long)(n0 + i + j) * p.ldw;
        const bool in = i + j < rows;
        if (VEC) {
          const float4 v = in && col[0] < p.J ? __ldcs(reinterpret_cast<const float4*>(at + col[0])) : make_float4(0.f, 0.f, 0.f, 0.f);
          w[j][0] = v.x; w[j][1] = v.y; w[j][2] = v.z; w[j][3] = v.w;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) w[j][q] = in && col[q] < p.J ? __ldcs(at + col[q]) : 0.f;
        }
      }
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const float4 f = *reinterpret_cast<const float4*>(&d[m][i]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[m][q] = fmaf(f.x, w[0][q], fmaf(f.y, w[1][q], fmaf(f.z, w[2][q], fmaf(f.w, w[3][q], acc[m][q]))));
      }
    }
  }
#pragma unroll
  for (int m0 = 0; m0 < MR; m0 += 4) {
    __syncthreads();
#pragma unroll
    for (int m = m0; m < m0 + 4 && m < MR; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) sums[warp][m - m0][col[q] - c0] = acc[m][q];
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * 128; i += 256) {
      const int m = m0 + i / 128, c = c0 + i % 128;
      if (m >= p.M || c >= p.J || m >= MR) continue;
      float s = sums[0][i / 128][i % 128];
      for (int w = 1; w < 8; ++w) s += sums[w][i / 128][i % 128];
      p.part[blockIdx.y * p.part_stride + (long long)m * p.J + c] = s;
    }
  }
}

// W's rows are the outputs: a warp has four of them and a run of the sum, a lane every 32nd vector (or entry) of it.
template <int MR, bool VEC>
__global__ void __launch_bounds__(256) few_rows_dots_kernel(FewProduct p) {
  __shared__ __align__(16) float d[MR][kFewChunk];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long j0 = (long long)blockIdx.x * 32 + warp * 4;
  const int n_first = (int)min((long long)p.I, (long long)blockIdx.y * p.run), n_end = (int)min((long long)p.I, (long long)(blockIdx.y + 1) * p.run);
  float acc[MR][4];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[m][q] = 0.f;
  for (int n0 = n_first; n0 < n_end; n0 += kFewChunk) {
    __syncthreads();
    for (int i = threadIdx.x; i < MR * kFewChunk; i += 256) {
      const int m = i / kFewChunk, n = n0 + i % kFewChunk;
      d[m][i % kFewChunk] = m < p.M && n < n_end ? p.A[m * p.lda + n] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kFewChunk / 128; ++g) {                      // 128 entries of the sum: four a lane
      float w[4][4];
      const int at = VEC ? g * 128 + lane * 4 : g * 128 + lane;
      if (n0 + g * 128 >= n_end) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* row = p.W + (j0 + j) * p.ldw + n0;
        if (VEC) {
          const float4 v = j0 + j < p.J && n0 + at < n_end ? __ldcs(reinterpret_cast<const float4*>(row + at)) : make_float4(0.f, 0.f, 0.f, 0.f);
          w[j][0] = v.x; w[j][1] = v.y; w[j][2] = v.z; w[j][3] = v.w;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) w[j][q] = j0 + j < p.J && n0 + at + q * 32 < n_end ? __ldcs(row + at + q * 32) : 0.f;
        }
      }
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        float f[4];
        if (VEC) {
          const float4 v = *reinterpret_cast<const float4*>(&d[m][at]);
          f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) f[q] = d[m][at + q * 32];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[m][j] = fmaf(f[0], w[j][0], fmaf(f[1], w[j][1], fmaf(f[2], w[j][2], fmaf(f[3], w[j][3], acc[m][j]))));
      }
    }
  }
  // the lanes' sums of a row, in a fixed tree; lane j keeps output j's
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    float mine = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float s = acc[m][j];
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      if (lane == j) mine = s;
    }
    if (m < p.M && lane < 4 && j0 + lane < p.J) p.part[blockIdx.y * p.part_stride + (long long)m * p.J + j0 + lane] = mine;
  }
}
// An FP32 matrix copied to rows on 16 bytes (`quads` of them a row; zeros behind the end), where TMA can read it.  Blocks follow each other
// in memory (100001 x 999 122 us, 6.5 TB/s; threads a grid apart 143), from the end on: the product finds the matrix' start in L2.
constexpr int kRealignBlock = 1024;                    // 16-byte words that a block copies at a time
__global__ void __launch_bounds__(256)
realign_kernel(long long rows, int cols, const float* __restrict__ W, long long ldw, float4* __restrict__ out, int quads) {
  const long long total = rows * quads;
  constexpr int U = kRealignBlock / 256;
  for (long long i0 = (long long)(gridDim.x - 1 - blockIdx.x) * kRealignBlock + threadIdx.x; i0 < total; i0 += (long long)gridDim.x * kRealignBlock) {
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * 256;
      if (i >= total) break;
      const long long r = total < (1ll << 31) ? (long long)((uint32_t)i / (uint32_t)quads) : i / quads;
      const int c = (int)(i - r * quads) * 4;
      const float* at = W + r * ldw + c;
      v[u].x = __ldcs(at);
      v[u].y = c + 1 < cols ? __ldcs(at + 1) : 0.f;
      v[u].z = c + 2 < cols ? __ldcs(at + 2) : 0.f;
      v[u].w = c + 3 < cols ? __ldcs(at + 3) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * 256;
      if (i < total) out[i] = v[u];
    }
  }
}

// dW for few rows: out[r, c] = sum over m of a[m, r] b[m, c], in FP32, up to 64 of them.  A block has 256 rows and 128 columns of the
// result, a warp eight rows at a time, a lane four columns: bound by the result's bytes for few rows, then by FMA.
// (The tensor cores' tiles store a matrix with rows on odd addresses by elements, a row a thread: 8 rows, 100001 x 999, 560 us.)
constexpr int kOuterMost = 64, kOuterRows = 256;
template <int MOST, bool VEC>
__global__ void __launch_bounds__(256)
few_outer_kernel(int M, int R, int C, const float* __restrict__ a, long long lda, const float* __restrict__ b, long long ldb,
                 float* __restrict__ out, long long ldo) {
  constexpr int CHUNK = MOST <= 16 ? kOuterRows : 64;                // rows of the result between two loads of a
  __shared__ __align__(16) float bs[MOST][128];
  __shared__ __align__(16) float as[MOST][CHUNK];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x * 128;
  for (int i = threadIdx.x; i < M * 128; i += 256) {
    const int m = i / 128, c = i % 128;
    // (a lane's four columns next to each other in either layout)
    const int at = VEC ? c : (c % 32) * 4 + c / 32;
    bs[m][at] = c0 + c < C ? b[m * ldb + c0 + c] : 0.f;
  }
  const long long r_first = (long long)blockIdx.y * kOuterRows;
  const long long r_end = min((long long)R, r_first + kOuterRows);
  for (long long r0 = r_first; r0 < r_end; r0 += 64) {
    const int at = (int)(r0 - r_first) % CHUNK;
    if (at == 0) {
      __syncthreads();
      for (int i = threadIdx.x; i < M * CHUNK; i += 256) {
        const int m = i / CHUNK, r = i % CHUNK;
        as[m][r] = r0 + r < r_end ? a[m * lda + r0 + r] : 0.f;
      }
      __syncthreads();
    }
    float acc[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[j][q] = 0.f;
#pragma unroll 2
    for (int m = 0; m < M; ++m) {
      const float4 x = *reinterpret_cast<const float4*>(&as[m][at + warp * 8]);
      const float4 z = *reinterpret_cast<const float4*>(&as[m][at + warp * 8 + 4]);
      const float4 y = *reinterpret_cast<const float4*>(&bs[m][lane * 4]);
      const float xs[8] = {x.x, x.y, x.z, x.w, z.x, z.y, z.z, z.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[j][q] = fmaf(xs[j], ys[q], acc[j][q]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long long r = r0 + warp * 8 + j;
      if (r >= r_end) break;
      float* to = out + r * ldo + c0;
      if (VEC) {
        if (c0 + lane * 4 < C) __stcs(reinterpret_cast<float4*>(to + lane * 4), make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]));
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (c0 + q * 32 + lane < C) __stcs(to + q * 32 + lane, acc[j][q]);
      }
    }
  }
}

__global__ void __launch_bounds__(256)
sum_runs_kernel(int M, int J, const float* __restrict__ part, int runs, const float* __restrict__ bias, float* __restrict__ Y, long long ldy) {
  const int c = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  if (c >= J) return;
  float s = 0.f;
#pragma unroll 8
  for (int i = 0; i < runs; ++i) s += part[((long long)i * M + m) * J + c];
  Y[m * ldy + c] = bias ? s + bias[c] : s;
}

}  // namespace sgc

namespace {

using sgc::Carve;
using sgc::Packed;
using sgc::PackJob;

constexpr size_t kPieceBytes = (size_t)1 << 30;          // logits of a piece of rows
constexpr int kPieceRows = 1 << 22;                      // (small vocabularies)
constexpr int kGradRows = 256, kGradRowsLeast = 32;      // rows of a column sum's part

int loss_setup(sgemm_cube_ctx* h) {
  return sgc::product_setup<sgc::kFormLossKM, sgc::kFormLossKK>(h, h->loss_clusters);
}

template <int FORM>
int loss_product(sgemm_cube_ctx* h, int M, int N, int K, const Packed& X, const Packed& W, sgc::LossEpilogue ep, cudaStream_t st) {
  const int rc = loss_setup(h);
  if (rc) return rc;
  ep.exp_a = X.exp;
  ep.exp_b = W.exp;
  sgc::TcLossParams p;
  memset(&p, 0, sizeof(p));
  p.M = M; p.N = N; p.K = K;
  p.ep = ep;
  return sgc::run_product<FORM>(h, h->loss_clusters, X, W, p, true, st);
}

sgc::LossJoinParams join_params(int rows, int vocab, const sgc::LossEpilogue& ep, float* loss, float* lse) {
  sgc::LossJoinParams j;
  memset(&j, 0, sizeof(j));
  j.rows = rows; j.vocab = vocab; j.per_row = (vocab + sgc::kLossColumns - 1) / sgc::kLossColumns;
  j.parts = ep.parts; j.ldp = ep.ldp;
  j.targets = ep.targets; j.target_logit = ep.target_logit;
  j.loss = loss; j.lse = lse;
  return j;
}
int launch_join(sgemm_cube_ctx* h, const sgc::LossJoinParams& j, cudaStream_t st) {
  if (j.per_row <= 512) sgc::loss_join_kernel<true><<<(unsigned)((j.rows + 3) / 4), 128, 0, st>>>(j);
  else sgc::loss_join_kernel<false><<<(unsigned)j.rows, 128, 0, st>>>(j);
  return sgc::launched(h);
}
int launch_rows(sgemm_cube_ctx* h, const sgc::LossJoinParams& j, const float* Z, int64_t ldz, cudaStream_t st) {
  // blocks of a row: pieces of at least 4096 columns, while the SMs have room
  int ranks = 1;
  while (ranks < 8 && (long long)j.rows * ranks < 2 * h->sm_count && j.vocab / (2 * ranks) >= 4096) ranks *= 2;
  for (;; ranks = 1) {                           // clusters that cannot be scheduled: one block a row
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = (unsigned)ranks; a.val.clusterDim.y = 1; a.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(j.rows * ranks), 1, 1);
    cfg.blockDim = dim3(sgc::kRowThreads, 1, 1);
    cfg.stream = st;
    cfg.attrs = &a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, sgc::loss_rows_kernel, j, Z, (long long)ldz) == cudaSuccess) break;
    cudaGetLastError();
    if (ranks == 1) return SGEMM_CUBE_CUDA_ERROR;
  }
  h->launches++;
  return SGEMM_CUBE_OK;
}

// Products by the kernels above: how many runs the sums are cut into, about four blocks an SM.
int few_runs(const sgemm_cube_ctx* h, int J, int I, bool dots, int* run) {
  const int tiles = dots ? (int)(((long long)J + 31) / 32) : (int)(((long long)J + 127) / 128);
  int runs = (4 * h->sm_count + tiles - 1) / tiles;
  const int most = (I + 2 * sgc::kFewChunk - 1) / (2 * sgc::kFewChunk);
  if (runs > most) runs = most;
  *run = (int)round_up((size_t)(((long long)I + runs - 1) / runs), 32);
  return (int)(((long long)I + *run - 1) / *run);
}
size_t few_part(const sgemm_cube_ctx* h, int M, int J, int I, bool dots) {
  int run;
  return (size_t)few_runs(h, J, I, dots, &run) * M * J;
}
template <int MR, bool VEC>
int launch_few(sgemm_cube_ctx* h, const sgc::FewProduct& p, bool dots, int runs, cudaStream_t st) {
  if (dots) {
    const dim3 grid((unsigned)(((long long)p.J + 31) / 32), (unsigned)runs, 1);
    sgc::few_rows_dots_kernel<MR, VEC><<<grid, 256, 0, st>>>(p);
  } else {
    const dim3 grid((unsigned)(((long long)p.J + 127) / 128), (unsigned)runs, 1);
    sgc::few_rows_sums_kernel<MR, VEC><<<grid, 256, 0, st>>>(p);
  }
  return sgc::launched(h);
}
// (16 rows by single entries: 1.7 TB/s where 8 take 3.2)
template <bool VEC>
constexpr int few_most() { return VEC ? sgc::kFewMost : 8; }
template <bool VEC>
int launch_few(sgemm_cube_ctx* h, const sgc::FewProduct& p, bool dots, int runs, cudaStream_t st) {
  if (p.M == 1) return launch_few<1, VEC>(h, p, dots, runs, st);
  if (p.M == 2) return launch_few<2, VEC>(h, p, dots, runs, st);
  if (p.M <= 4) return launch_few<4, VEC>(h, p, dots, runs, st);
  if constexpr (few_most<VEC>() > 8) {
    if (p.M > 8) return launch_few<few_most<VEC>(), VEC>(h, p, dots, runs, st);
  }
  return launch_few<8, VEC>(h, p, dots, runs, st);
}
// Y (M x J) = A (M x I) W + bias; W's rows are the outputs (dots) or the summed index.
int few_product(sgemm_cube_ctx* h, int M, int J, int I, const float* A, int64_t lda, const float* W, int64_t ldw, bool dots, const float* bias,
                float* part, float* Y, int64_t ldy, cudaStream_t st) {
  sgc::FewProduct p;
  memset(&p, 0, sizeof(p));
  p.J = J; p.I = I;
  p.lda = lda;
  p.W = W; p.ldw = ldw;
  p.part_stride = (long long)M * J;
  const int runs = few_runs(h, J, I, dots, &p.run);
  const bool vec = aligned16(W) && ldw % 4 == 0 && (dots ? I : J) % 4 == 0;
  const int most = vec ? few_most<true>() : few_most<false>();
  for (int m0 = 0; m0 < M; m0 += most) {
    p.M = M - m0 < most ? M - m0 : most;
    p.A = A + m0 * lda;
    p.part = part + (long long)m0 * J;
    const int rc = vec ? launch_few<true>(h, p, dots, runs, st) : launch_few<false>(h, p, dots, runs, st);
    if (rc) return rc;
  }
  sgc::sum_runs_kernel<<<dim3((unsigned)(((long long)J + 255) / 256), (unsigned)M, 1), 256, 0, st>>>(M, J, part, runs, bias, Y, ldy);
  return sgc::launched(h);
}
bool on_16_bytes(const sgemm_cube_operand* W) { return aligned16(W->f32_dev) && W->ld % 4 == 0; }
// Logits: an FP32 weight whose rows are not on 16 bytes would be copied or packed first; up to 16 rows, eight at a time, read it as
// it is instead (100001 x 999: 8 rows 126 us, 370 packed; 14 rows 218, 275 copied and 345 packed).
bool few_logits(int M, const sgemm_cube_operand* W) { return W->f32_dev && M > 4 && M <= 16 && !on_16_bytes(W); }
// dX: the linear layer's forms have about J / 128 tiles of up to 8 blocks; where that leaves more than half of the SMs idle for every
// group of 16 rows, W is read once for each group instead (20 x 168 outputs of a sum of 78984: the call 335 -> 197 us; but 53 x 384
// of 27468 185 -> 210 without that bound).  On odd addresses up to 8 rows (16 of 45889 x 3664, all gradients: 997 us, 847 packed).
bool few_dx(const sgemm_cube_ctx* h, int M, int J, const sgemm_cube_operand* W) {
  if (!W->f32_dev) return false;
  if (M <= 8) return true;
  const int groups = (M + sgc::kFewMost - 1) / sgc::kFewMost, tiles = (J + 127) / 128, blocks = tiles * 2 <= h->sm_count ? tiles * 8 : tiles;
  return on_16_bytes(W) && J % 4 == 0 && M <= 4 * sgc::kFewMost && (groups == 1 || 2ll * groups * blocks < h->sm_count);
}
// dW: by FMA where memory bounds that, or the tensor cores' tiles would store by elements.
bool few_dw(int M, const float* dW, int64_t lddw) { return M <= (aligned16(dW) && lddw % 4 == 0 ? 32 : sgc::kOuterMost); }
int few_outer(sgemm_cube_ctx* h, int M, int R, int C, const float* a, int64_t lda, const float* b, int64_t ldb, float* out, int64_t ldo,
              cudaStream_t st) {
  // columns in x: the blocks that run at the same time write the same rows
  const long long rows = ((long long)R + sgc::kOuterRows - 1) / sgc::kOuterRows;
  const bool vec = aligned16(out) && ldo % 4 == 0 && C % 4 == 0;
  for (long long y0 = 0; y0 < rows; y0 += 65535) {       // (the grid's limit)
    const long long r0 = y0 * sgc::kOuterRows, some = rows - y0 < 65535 ? rows - y0 : 65535;
    const long long left = (long long)R - r0, here = left < some * sgc::kOuterRows ? left : some * sgc::kOuterRows;
    const dim3 grid((unsigned)(((long long)C + 127) / 128), (unsigned)some, 1);
    const auto kernel = M <= 16 ? (vec ? sgc::few_outer_kernel<16, true> : sgc::few_outer_kernel<16, false>)
                                : (vec ? sgc::few_outer_kernel<sgc::kOuterMost, true> : sgc::few_outer_kernel<sgc::kOuterMost, false>);
    kernel<<<grid, 256, 0, st>>>(M, (int)here, C, a + r0, lda, b, ldb, out + r0 * ldo, ldo);
    const int rc = sgc::launched(h);
    if (rc) return rc;
  }
  return SGEMM_CUBE_OK;
}

bool bad_layout(int layout) { return layout != SGEMM_CUBE_WEIGHT_KN && layout != SGEMM_CUBE_WEIGHT_NK; }

int check_loss(sgemm_cube_ctx* h, int M, int N, int K, const sgemm_cube_operand* X, const sgemm_cube_operand* W, int layout,
               const float* bias, const int64_t* targets, const float* loss, const float* lse) {
  if (!h || bad_dims(M, N, K) || N < 1 || K < 1 || bad_layout(layout)) return SGEMM_CUBE_INVALID_ARG;
  const bool nk = layout == SGEMM_CUBE_WEIGHT_NK;
  int rc = sgc::check_operand(X, M, K);
  if (rc) return rc;
  if ((rc = nk ? sgc::check_operand(W, N, K) : sgc::check_operand(W, K, N))) return rc;
  if (M > 0 && !targets) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(4, bias, loss, lse) || misplaced(8, targets)) return SGEMM_CUBE_INVALID_ARG;
  return SGEMM_CUBE_OK;
}

}  // namespace

extern "C" {

int sgemm_cube_cross_entropy(sgemm_cube_handle h, int M, int N, int K, const sgemm_cube_operand* X, const sgemm_cube_operand* W,
                             int weight_layout, const float* bias, const int64_t* targets, float* loss, float* lse, void* stream) {
  int rc = check_loss(h, M, N, K, X, W, weight_layout, bias, targets, loss, lse);
  if (rc) return rc;
  if (M == 0) return SGEMM_CUBE_OK;
  if (!loss && !lse) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool nk = weight_layout == SGEMM_CUBE_WEIGHT_NK;
  const bool few = !sgc::is_packed(X) && sgc::linear_takes_few(h, M, N, K, sgc::is_packed(W), nk);
  const int per_row = (N + sgc::kLossColumns - 1) / sgc::kLossColumns;
  sgc::LossEpilogue ep;
  memset(&ep, 0, sizeof(ep));
  ep.bias = bias;
  ep.targets = reinterpret_cast<const long long*>(targets);
  ep.ldp = per_row;
  float *Z = nullptr, *part = nullptr;
  const int64_t ldz = (int64_t)round_up((size_t)N, 8);
  const bool by_fma = few && few_logits(M, W);
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->loss_ws) : nullptr;
    if (few) {
      Z = c.take<float>((size_t)M * ldz);
      if (by_fma) part = c.take<float>(few_part(h, M, N, K, nk));
    } else {
      ep.parts = c.take<float2>((size_t)M * per_row);
      ep.target_logit = c.take<float>((size_t)M);
    }
    if (!pass && (rc = grow(h, &h->loss_ws, &h->loss_ws_bytes, c.used, st))) return rc;
  }
  if (few) {
    // few rows: kernels for them, whose logits stay in L2
    const int w_rows = nk ? N : K, w_cols = nk ? K : N, quads = (w_cols + 3) / 4;
    const sgemm_cube_operand* w = W;
    sgemm_cube_operand copy{nullptr, 4ll * quads, nullptr, nullptr, 0, nullptr};
    if (!by_fma && W->f32_dev && M > 8 && !on_16_bytes(W)) {
      // Rows on odd addresses: the layer would pack the weight, 12 bytes an entry and 4 to read the words; a copy that its kernel can
      // read by TMA moves 8 and 4.
      if ((rc = grow(h, &h->ws, &h->ws_bytes, (size_t)w_rows * quads * 16, st))) return rc;
      copy.f32_dev = static_cast<const float*>(h->ws);
      w = &copy;
      const long long pieces = ((long long)w_rows * quads + sgc::kRealignBlock - 1) / sgc::kRealignBlock;
      sgc::realign_kernel<<<(unsigned)(pieces < (1 << 24) ? pieces : 1 << 24), 256, 0, st>>>(w_rows, w_cols, W->f32_dev, W->ld,
                                                                                             static_cast<float4*>(h->ws), quads);
      if ((rc = sgc::launched(h))) return rc;
    }
    if (by_fma) rc = few_product(h, M, N, K, X->f32_dev, X->ld, W->f32_dev, W->ld, nk, bias, part, Z, ldz, st);
    else rc = sgemm_cube_linear(h, M, N, K, X, w, weight_layout, bias, nullptr, 0, SGEMM_CUBE_ACT_NONE, Z, ldz, nullptr, 0, stream);
    if (rc) return rc;
    return launch_rows(h, join_params(M, N, ep, loss, lse), Z, ldz, st);
  }
  PackJob jobs[2];
  int n_jobs = 0;
  int* exps = reinterpret_cast<int*>(h->err_dev + sgc::kExpWords);
  Packed px{}, pw{};
  for (int pass = 0; pass < 2; ++pass) {
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->ws) : nullptr;
    n_jobs = 0;
    px = sgc::words_of(X, M, K, c, exps, jobs, &n_jobs);
    pw = sgc::words_of(W, nk ? N : K, nk ? K : N, c, exps + 1, jobs, &n_jobs);
    if (!pass && c.used && (rc = grow(h, &h->ws, &h->ws_bytes, c.used, st))) return rc;
  }
  if (n_jobs && (rc = sgc::launch_pack(h, jobs, n_jobs, st))) return rc;
  rc = nk ? loss_product<sgc::kFormLossKK>(h, M, N, K, px, pw, ep, st) : loss_product<sgc::kFormLossKM>(h, M, N, K, px, pw, ep, st);
  if (rc) return rc;
  return launch_join(h, join_params(M, N, ep, loss, lse), st);
}

int sgemm_cube_cross_entropy_backward(sgemm_cube_handle h, int M, int N, int K, const sgemm_cube_operand* X,
                                      const sgemm_cube_operand* W, int weight_layout, const float* bias, const int64_t* targets,
                                      const float* dloss, float* loss, float* lse, float* dX, int64_t lddx, float* dW, int64_t lddw,
                                      float* dbias, void* stream) {
  int rc = check_loss(h, M, N, K, X, W, weight_layout, bias, targets, loss, lse);
  if (rc) return rc;
  const bool nk = weight_layout == SGEMM_CUBE_WEIGHT_NK;
  const int w_rows = nk ? N : K, w_cols = nk ? K : N;
  if ((M > 0 && !dloss) || (dX && lddx < K) || (dW && lddw < w_cols)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(4, dloss, dX, dW, dbias)) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (M == 0) {                                  // empty sums
    if (dW && cudaMemset2DAsync(dW, (size_t)lddw * 4, 0, (size_t)w_cols * 4, w_rows, st) != cudaSuccess) rc = SGEMM_CUBE_CUDA_ERROR;
    if (!rc && dbias && cudaMemsetAsync(dbias, 0, (size_t)N * 4, st) != cudaSuccess) rc = SGEMM_CUBE_CUDA_ERROR;
    if (rc) cudaGetLastError();
    return rc;
  }
  const int per_row = (N + sgc::kLossColumns - 1) / sgc::kLossColumns;
  const bool split = dX || dW;
  if (!split && !dbias)                          // nothing but the loss
    return loss || lse ? sgemm_cube_cross_entropy(h, M, N, K, X, W, weight_layout, bias, targets, loss, lse, stream) : SGEMM_CUBE_OK;
  const int64_t ldz = (int64_t)round_up((size_t)N, 8);
  // rows of a piece: whole tiles of pairs, pieces of about the same size
  long long most = (long long)(kPieceBytes / (4 * (size_t)ldz)) / 256 * 256;
  if (most > kPieceRows) most = kPieceRows;
  if (most < 256) most = 256;
  int piece = most < M ? (int)most : M;
  if (piece < M) {
    const long long pieces = ((long long)M + piece - 1) / piece;
    piece = (int)round_up((size_t)((M + pieces - 1) / pieces), 256);
  }
  // rows of a part: enough parts for eight blocks an SM
  int grad_rows = kGradRows;
  while (grad_rows > kGradRowsLeast && (long long)((N + 255) / 256) * ((piece + grad_rows - 1) / grad_rows) < 8 * h->sm_count) grad_rows /= 2;
  const int chunks = (piece + grad_rows - 1) / grad_rows, col_blocks = (N + 255) / 256;
  sgc::LossEpilogue ep;
  memset(&ep, 0, sizeof(ep));
  ep.bias = bias;
  ep.ldp = per_row;
  ep.ldz = ldz;
  float2* stats = nullptr;
  uint16_t *ghi = nullptr, *glo = nullptr;
  float* col_part = nullptr;
  unsigned int* counts = nullptr;
  float* target_logit = nullptr;
  // (before the sizes: what the forms for few rows are chosen by has to be known)
  const bool few = !sgc::is_packed(X) && sgc::linear_takes_few(h, M, N, K, sgc::is_packed(W), nk) &&
                   (!dX || sgc::linear_takes_few(h, M, K, N, sgc::is_packed(W), !nk));
  const bool fma_logits = few && few_logits(M, W), fma_dx = few && dX && few_dx(h, M, K, W), fma_dw = few && dW && few_dw(M, dW, lddw);
  float *sum_part = nullptr, *logit_part = nullptr;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->loss_ws) : nullptr;
    if (fma_dx) sum_part = c.take<float>(few_part(h, M, K, N, !nk));
    if (fma_logits) logit_part = c.take<float>(few_part(h, M, N, K, nk));
    ep.parts = c.take<float2>((size_t)piece * per_row);
    target_logit = c.take<float>((size_t)piece);
    stats = c.take<float2>((size_t)piece);
    ep.Z = c.take<float>((size_t)piece * ldz);
    if (split) {
      ghi = c.take<uint16_t>((size_t)piece * ldz);
      glo = c.take<uint16_t>((size_t)piece * ldz);
    }
    if (dbias) {
      col_part = c.take<float>((size_t)chunks * N);
      counts = c.take<unsigned int>((size_t)col_blocks);
    }
    if (!pass && (rc = grow(h, &h->loss_ws, &h->loss_ws_bytes, c.used, st))) return rc;
  }
  ep.target_logit = target_logit;
  PackJob jobs[2];
  int n_jobs = 0;
  int* exps = reinterpret_cast<int*>(h->err_dev + sgc::kExpWords);
  Packed px{}, pw{};
  const auto grad = [&](int r0, int rows, float* dz, bool words) {
    sgc::LossGradParams p;
    memset(&p, 0, sizeof(p));
    p.rows = rows; p.vocab = N; p.rows_per_chunk = grad_rows;
    p.Z = ep.Z; p.ldz = ldz;
    p.dz = dz;
    p.stats = stats;
    p.dloss = dloss + r0;
    p.targets = reinterpret_cast<const long long*>(targets) + r0;
    if (words) { p.hi = ghi; p.lo = glo; p.ldw = ldz; }
    p.exp = exps + 2;
    p.col_part = col_part; p.counts = counts;
    p.dbias = dbias; p.add = r0 > 0;
    sgc::loss_grad_kernel<<<dim3((unsigned)col_blocks, (unsigned)((rows + grad_rows - 1) / grad_rows), 1), 256, 0, st>>>(p);
    return sgc::launched(h);
  };
  const auto rows_of_join = [&](int r0, int rows) {
    sgc::LossJoinParams j = join_params(rows, N, ep, loss ? loss + r0 : nullptr, lse ? lse + r0 : nullptr);
    j.stats = stats;
    j.dloss = dloss + r0;
    j.range = h->err_dev + sgc::kRangeWords;
    j.exp = split ? exps + 2 : nullptr;
    j.counts = counts; j.n_counts = col_blocks;
    return j;
  };
  const auto weight_gradient = [&](const Packed& x, int rows, sgc::LinearEpilogue le) {
    const Packed dz{ghi, glo, ldz, exps + 2};
    return nk ? sgc::linear_product_any(sgc::kFormMM, h, N, K, rows, dz, x, dW, lddw, le, st)
              : sgc::linear_product_any(sgc::kFormMM, h, K, N, rows, x, dz, dW, lddw, le, st);
  };
  sgc::LinearEpilogue plain;
  memset(&plain, 0, sizeof(plain));
  // Few rows (one piece): the weight's bytes decide, so both products with it take forms that read it as it is, or, where a row of
  // it does not start on 16 bytes and more than a few rows of X ask for that, pack it once for both.
  const bool packed_w = sgc::is_packed(W);
  if (few) {
    // (nothing that follows has to pack the weight)
    const bool as_it_is = packed_w || on_16_bytes(W) || ((fma_logits || M <= 4) && (!dX || fma_dx || M <= 4));
    const bool words = dW && !fma_dw;              // of X and dz
    if (words || !as_it_is) {
      for (int pass = 0; pass < 2; ++pass) {
        Carve c;
        c.base = pass ? static_cast<uint8_t*>(h->ws) : nullptr;
        n_jobs = 0;
        if (!as_it_is) pw = sgc::words_of(W, w_rows, w_cols, c, exps + 1, jobs, &n_jobs);
        if (words) px = sgc::words_of(X, M, K, c, exps + 3, jobs, &n_jobs);
        if (!pass && (rc = grow(h, &h->ws, &h->ws_bytes, c.used, st))) return rc;
      }
      if ((rc = sgc::launch_pack(h, jobs, n_jobs, st))) return rc;
    }
    const sgemm_cube_operand packed{nullptr, 0, pw.hi, pw.lo, pw.ld, pw.exp};
    const sgemm_cube_operand* w = as_it_is ? W : &packed;
    if (fma_logits && as_it_is) rc = few_product(h, M, N, K, X->f32_dev, X->ld, W->f32_dev, W->ld, nk, bias, logit_part, ep.Z, ldz, st);
    else rc = sgemm_cube_linear(h, M, N, K, X, w, weight_layout, bias, nullptr, 0, SGEMM_CUBE_ACT_NONE, ep.Z, ldz, nullptr, 0, stream);
    if (rc) return rc;
    ep.targets = reinterpret_cast<const long long*>(targets);
    if ((rc = launch_rows(h, rows_of_join(0, M), ep.Z, ldz, st)) || (rc = grad(0, M, dX || fma_dw ? ep.Z : nullptr, words))) return rc;
    if (fma_dx) {
      rc = few_product(h, M, K, N, ep.Z, ldz, W->f32_dev, W->ld, !nk, nullptr, sum_part, dX, lddx, st);
    } else if (dX) {
      const sgemm_cube_operand dz{ep.Z, ldz, nullptr, nullptr, 0, nullptr};
      rc = sgemm_cube_linear(h, M, K, N, &dz, w, nk ? SGEMM_CUBE_WEIGHT_KN : SGEMM_CUBE_WEIGHT_NK, nullptr, nullptr, 0,
                             SGEMM_CUBE_ACT_NONE, dX, lddx, nullptr, 0, stream);
    }
    if (rc || !dW) return rc;
    if (!fma_dw) return weight_gradient(px, M, plain);
    return nk ? few_outer(h, M, N, K, ep.Z, ldz, X->f32_dev, X->ld, dW, lddw, st)
              : few_outer(h, M, K, N, X->f32_dev, X->ld, ep.Z, ldz, dW, lddw, st);
  }
  for (int pass = 0; pass < 2; ++pass) {
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->ws) : nullptr;
    n_jobs = 0;
    px = sgc::words_of(X, M, K, c, exps, jobs, &n_jobs);
    pw = sgc::words_of(W, w_rows, w_cols, c, exps + 1, jobs, &n_jobs);
    if (!pass && c.used && (rc = grow(h, &h->ws, &h->ws_bytes, c.used, st))) return rc;
  }
  if (n_jobs && (rc = sgc::launch_pack(h, jobs, n_jobs, st))) return rc;
  for (int r0 = 0; r0 < M; r0 += piece) {
    const int rows = M - r0 < piece ? M - r0 : piece;
    const Packed x{px.hi + (int64_t)r0 * px.ld, px.lo + (int64_t)r0 * px.ld, px.ld, px.exp};
    ep.targets = reinterpret_cast<const long long*>(targets) + r0;
    rc = nk ? loss_product<sgc::kFormLossKK>(h, rows, N, K, x, pw, ep, st) : loss_product<sgc::kFormLossKM>(h, rows, N, K, x, pw, ep, st);
    if (rc) return rc;
    if ((rc = launch_join(h, rows_of_join(r0, rows), st)) || (rc = grad(r0, rows, nullptr, split))) return rc;
    const Packed dz{ghi, glo, ldz, exps + 2};
    if (dX && (rc = sgc::linear_product_any(nk ? sgc::kFormKM : sgc::kFormKK, h, rows, K, N, dz, pw, dX + (int64_t)r0 * lddx, lddx, plain, st)))
      return rc;
    if (dW) {
      sgc::LinearEpilogue le = plain;
      if (r0 > 0) { le.R = dW; le.ldr = lddw; }
      if ((rc = weight_gradient(x, rows, le))) return rc;
    }
  }
  return SGEMM_CUBE_OK;
}

}  // extern "C"
