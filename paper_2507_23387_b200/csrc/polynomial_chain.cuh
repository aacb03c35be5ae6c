// All products of an orthogonalised update in one launch, for matrices whose products are too small to fill the device for
// long: fifteen launches of the tensor-core kernel took 18 to 38 us each whatever they multiplied (a start, cold
// instructions, two trips through L2 around the epilogue), here a product is a phase of a resident kernel.
//
//   |G|_F, X = G / (|G|_F + eps);  steps times:  A = X X^T | B = b A + c A A | X <- a X + B X      (| all blocks meet)
//
// One block an SM, cooperative, in clusters.  A unit is a 128 x 128 tile, or a slice of its k range: with S slices a tile (S
// divides the cluster) S blocks of a cluster read each other's sums from shared memory and each finishes 128 / S of its rows.  Warps 0-7 take the sums out of TMEM (k-blocks added in
// FP32, as in gemm_tc.cuh) and finish the tile through shared memory (the ring, which is idle by then), along rows and, for
// what is below the diagonal of a symmetric product, along columns; warp 8 loads by TMA, warp 9 issues the MMAs.
// Words are written by ordinary stores and read by TMA in the next phase: a proxy fence stands on both sides of the meeting.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "elements.cuh"
#include "polynomial_epilogue.cuh"
#include "ptx_sm100.cuh"

namespace sgc {

constexpr int kChainTile = 128, kChainBK = 64, kChainStages = 3;
constexpr int kChainThreads = 320, kChainEpiThreads = 256;
constexpr uint32_t kChainWords = kChainTile * kChainBK * 2;              // one word of one operand's tile
constexpr uint32_t kChainStageBytes = 4 * kChainWords;                   // A hi, A lo, B hi, B lo
constexpr uint32_t kChainRing = kChainStages * kChainStageBytes;
constexpr int kChainPitch = 132;                                         // finishing: rows of a tile, 132 floats apart, in the ring
static_assert(kChainTile * kChainPitch * 4 <= kChainRing, "a finished tile fits the ring");
constexpr uint32_t kChainSmem = kChainRing + 256 + 1024;
constexpr int kChainMostSteps = 64, kChainMostCluster = 16;

struct ChainStep {           // factors of a step's three products (powers of two for the words' exponents in them)
  float gram_alpha, gram_pre, square_alpha, square_beta, square_pre, update_alpha, update_beta, update_pre;
};
struct ChainSplit {          // tiles of a product, slices of a tile (a power of two), 64-deep stages of a slice
  int tiles, slices, per;
};
struct ChainParams {
  int rows, cols, tall, steps;
  const void* G;
  long long ldg;
  int vec;                   // G takes 16-byte accesses
  float eps, pre;            // pre: 2^p of X's words
  uint16_t *x_hi[2], *x_lo[2], *a_hi, *a_lo, *b_hi, *b_lo;
  long long ldx, lda;
  float* O;
  long long ldo;
  const float* R;
  long long ldr;
  float scale, keep;
  int vec_out;
  int chunk;                 // stages of a k-block
  ChainSplit gram, square, update;
  double* sums;              // [blocks]
  unsigned int* words;       // {arrived, left} of the grid, zero between calls
  unsigned int* err;
  ChainStep step[kChainMostSteps];
};
struct ChainMaps {
  CUtensorMap x[2][2], a[2], b[2];       // hi, lo; boxes of 64 x 64 words
};

__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }
// Relaxed: the fences around them stand alone (a releasing addition or acquiring loads in the loop each add one of their own).
__device__ __forceinline__ unsigned int load_relaxed(const unsigned int* p) {
  unsigned int v;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_relaxed(unsigned int* p) {
  asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(1u) : "memory");
}
// The 256 threads of the first eight warps meet; true if `ok` is for all of them.
__device__ __forceinline__ bool chain_agree(bool ok) {
  uint32_t all;
  __syncwarp();
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "barrier.cta.red.and.aligned.pred q, 1, 256, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(all) : "r"((uint32_t)ok) : "memory");
  return all != 0;
}
// Waits, bounded, until *p is at least `want`.
__device__ __forceinline__ bool chain_wait(const unsigned int* p, unsigned int want, volatile uint32_t* abort_flag, unsigned int* err) {
  const long long t0 = clock64();
  while (load_relaxed(p) < want) {
    if (*abort_flag) return false;
    if (clock64() - t0 > kWaitLimitClocks) {
      *abort_flag = 1u;
      atomicCAS(err, 0u, (unsigned int)kErrChainWait);
      __threadfence();
      return false;
    }
  }
  return true;
}
// All blocks of the grid meet for the `round`-th time (from 1); what they stored is there for loads and, behind a proxy
// fence of the thread that issues it, for TMA.  One thread's fences stand for the block's stores, which the barrier has put
// before them (every thread fencing for itself took 3000 to 5000 clocks a meeting).
// The answer is the first thread's, in a word that nobody writes before the next meeting: one for all threads.
__device__ __forceinline__ bool chain_meet(const ChainParams& p, unsigned int round, volatile uint32_t* abort_flag) {
  volatile uint32_t* met = abort_flag + 1;
  __syncthreads();
  if (threadIdx.x == 0) {
    bool ok = *abort_flag == 0u;
    if (ok) {
      __threadfence();
      fence_proxy_async_global();
      add_relaxed(&p.words[0]);
      ok = chain_wait(&p.words[0], round * gridDim.x, abort_flag, p.err);
      __threadfence();
    }
    *met = ok;
  }
  __syncthreads();
  return *met != 0u;
}

// All threads of the cluster meet, warp by warp (the barrier wants whole warps).
__device__ __forceinline__ void chain_cluster_meet() {
  __syncwarp();
  cluster_sync_all();
}
// Four floats of shared memory of a block of the cluster.
__device__ __forceinline__ float4 load_peer(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// Tile `t` of the lower triangle, row by row.
__device__ __forceinline__ void chain_tile(int t, bool symmetric, int tiles_n, int& tm, int& tn) {
  if (symmetric) {
    lower_tile_coords(t, true, tm, tn);
  } else {
    tm = t / tiles_n;
    tn = t - tm * tiles_n;
  }
}

template <typename T>
__global__ void __launch_bounds__(kChainThreads, 1)
polynomial_chain_kernel(const __grid_constant__ ChainMaps maps, const __grid_constant__ ChainParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* stage = reinterpret_cast<float*>(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kChainRing);
  uint64_t* full_bar = bars;                          // [stages]  TMA -> MMA
  uint64_t* empty_bar = bars + kChainStages;          // [stages]  MMA -> TMA
  uint64_t* tfull_bar = bars + 2 * kChainStages;      // [3]  MMA -> sums: hi*hi regions 0 and 1, corrections
  uint64_t* tempty_bar = tfull_bar + 3;               // [3]  sums -> MMA
  uint64_t* ring_bar = tempty_bar + 3;                // finishing -> TMA: the ring may be filled again
  uint64_t* drain_bar = ring_bar + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;      // and, behind it, chain_meet's word
  double* block_sums = reinterpret_cast<double*>(stage);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool tall = p.tall != 0;
  const int n = tall ? p.cols : p.rows, m = tall ? p.rows : p.cols;

  if (tid == 0) {
    for (int s = 0; s < kChainStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int r = 0; r < 3; ++r) {
      mbar_init(&tfull_bar[r], 1);
      mbar_init(&tempty_bar[r], kChainEpiThreads / 32);
    }
    mbar_init(ring_bar, kChainEpiThreads / 32);
    mbar_init(drain_bar, 1);
    *abort_flag = 0u;
    fence_mbar_init();
  }
  if (warp == 8 && lane < 8) {
    const CUtensorMap* all = maps.x[0];
    tma_prefetch_desc(all + lane);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;

  // ---------------------------------------------------------------------- X = G / (|G|_F + eps)
  // The sum of squares in FP64: gradients of any FP32 size neither overflow nor vanish.
  const T* G = static_cast<const T*>(p.G);
  unsigned int round = 0;
  bool go;
  {
    constexpr int V = Elem<T>::kVec;
    double s = 0.0;
    const int per_row = p.vec ? p.cols / V : p.cols;
    const long long total = (long long)p.rows * per_row, stride = (long long)gridDim.x * kChainThreads;
    for (long long it = (long long)blockIdx.x * kChainThreads + tid; it < total; it += stride) {
      const long long r = it / per_row;
      const T* at = G + r * p.ldg + (it - r * per_row) * (p.vec ? V : 1);
      if (p.vec) {
        float v[V];
        Elem<T>::unpack(*reinterpret_cast<const uint4*>(at), v);
#pragma unroll
        for (int q = 0; q < V; ++q) s += (double)v[q] * (double)v[q];
      } else {
        const double v = (double)Elem<T>::get(*at);
        s += v * v;
      }
    }
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    if (lane == 0) block_sums[warp] = s;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kChainThreads / 32; ++w) s += block_sums[w];
      p.sums[blockIdx.x] = s;
    }
    go = chain_meet(p, ++round, abort_flag);
  }
  if (go) {
    double s = 0.0;                                          // every warp adds all blocks' sums in the same order
    for (int i = lane; i < (int)gridDim.x; i += 32) s += __ldcg(p.sums + i);
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    float f0, f1;
    norm_factors(s, p.eps, p.pre, f0, f1);
    const int per_row = (p.cols + 7) >> 3;
    const long long total = (long long)p.rows * per_row, stride = (long long)gridDim.x * kChainThreads;
    for (long long it = (long long)blockIdx.x * kChainThreads + tid; it < total; it += stride) {
      const long long r = it / per_row;
      const int c = (int)(it - r * per_row) << 3;
      normalise_eight(G + r * p.ldg + c, p.vec != 0, p.cols - c, f0, f1, p.x_hi[0] + r * p.ldx + c, p.x_lo[0] + r * p.ldx + c);
    }
    go = chain_meet(p, ++round, abort_flag);
  }

  // ---------------------------------------------------------------------- the products
  uint32_t it = 0;                                           // stages: producer and MMA thread each count them
  uint32_t chunks_done = 0, units_done = 0;                  // k-blocks and units: MMA thread and sums
  const int phases = 3 * p.steps;
  int phase = 0;
  for (; phase < phases && go; ++phase) {
    const int step = phase / 3, kind = phase - 3 * step;
    const ChainStep& f = p.step[step];
    const ChainSplit split = kind == 0 ? p.gram : (kind == 1 ? p.square : p.update);
    const bool symmetric = kind != 2;
    const int cur = step & 1;
    const int M = symmetric ? n : p.rows, N = symmetric ? n : p.cols, K = kind == 0 ? m : n;
    const int tiles_n = (N + kChainTile - 1) / kChainTile, num_kb = (K + kChainBK - 1) / kChainBK;
    const int units = split.tiles * split.slices;
    auto unit_of = [&](int unit, int& tm, int& tn, int& slice, int& kb0, int& kb1) {
      const int tile = unit / split.slices;
      slice = unit - tile * split.slices;
      chain_tile(tile, symmetric, tiles_n, tm, tn);
      kb0 = slice * split.per;
      kb1 = min(num_kb, kb0 + split.per);
    };
    // With slices every block has at most one unit; the cluster meets once, when all sums of its tiles are in shared memory.
    const bool sliced = split.slices > 1;
    // A's and B's rows (or, MN-major, columns) of a tile and their k, by majorness
    const bool a_mn = kind == 0 && tall, b_mn = (kind == 0 && tall) || (kind == 2 && !tall);
    if (warp < 8) {
      // ------------------------------------------------------------------ sums, and what becomes of them
      const int quarter = warp & 3, half = warp >> 2;
      const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16) + half * 64;
      const float alpha = kind == 0 ? f.gram_alpha : (kind == 1 ? f.square_alpha : f.update_alpha);
      const float beta = kind == 0 ? 0.f : (kind == 1 ? f.square_beta : f.update_beta);
      const bool last = phase == phases - 1;
      const float pre = kind == 0 ? f.gram_pre : (kind == 1 ? f.square_pre : f.update_pre);
      const uint16_t* r_hi = kind == 0 ? nullptr : (kind == 1 ? p.a_hi : p.x_hi[cur]);
      const uint16_t* r_lo = kind == 1 ? p.a_lo : p.x_lo[cur];
      uint16_t* w_hi = kind == 0 ? p.a_hi : (kind == 1 ? p.b_hi : p.x_hi[cur ^ 1]);
      uint16_t* w_lo = kind == 0 ? p.a_lo : (kind == 1 ? p.b_lo : p.x_lo[cur ^ 1]);
      const long long ld = symmetric ? p.lda : p.ldx;
      // Rows of a tile that a block finishes.
      const int share = kChainTile / split.slices;
      const int filled = (num_kb + split.per - 1) / split.per;       // slices that hold sums
      for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int tm, tn, slice, kb0, kb1;
        unit_of(unit, tm, tn, slice, kb0, kb1);
        const int r0 = slice * share;
        const int unit_chunks = (kb1 - kb0 + p.chunk - 1) / p.chunk;
        float S[64];
        bool ok = true;
        for (int c = 0; c < unit_chunks && ok; ++c, ++chunks_done) {
          const uint32_t r = chunks_done & 1;
          ok = mbar_wait_bounded(&tfull_bar[r], (chunks_done >> 1) & 1, abort_flag, p.err, kErrEpiTmemFullWait);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(t_lane + r * kChainTile + g * 32, v);
            tmem_ld_wait();
            if (c == 0) {
#pragma unroll
              for (int j = 0; j < 32; ++j) S[g * 32 + j] = __uint_as_float(v[j]);
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) S[g * 32 + j] = __fadd_rn(S[g * 32 + j], __uint_as_float(v[j]));
            }
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tempty_bar[r]);
        }
        const bool empty = kb0 >= kb1;                       // a slice behind the end: its block finishes rows all the same
        if (ok && !empty) {
          ok = mbar_wait_bounded(&tfull_bar[2], units_done & 1, abort_flag, p.err, kErrEpiTmemFullWait);
          ok = __all_sync(0xffffffffu, ok);
        }
        if (!empty) ++units_done;
        if (ok && !empty) {
          tc_fence_after_sync();
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(t_lane + 2 * kChainTile + g * 32, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) S[g * 32 + j] = __fmaf_rn(__uint_as_float(v[j]), kPackInvScale, S[g * 32 + j]);
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tempty_bar[2]);
        }
        if (ok && !empty) {
          float* out = stage + (quarter * 32 + lane) * kChainPitch + half * 64;
#pragma unroll
          for (int c = 0; c < 64; c += 4) *reinterpret_cast<float4*>(out + c) = make_float4(S[c], S[c + 1], S[c + 2], S[c + 3]);
        }
        // A lane has four columns of a row, a warp every eighth row, four of them at a time; R's words come one turn ahead.
        // Loops, not straight lines: what a block runs through once a phase comes from the instruction cache's far end (16 rows
        // unrolled took four times as long).
        const int cg = lane * 4, c = tn * kChainTile + cg;
        const bool mirror = symmetric && tm != tn;           // (a tile on the diagonal holds its own mirror image)
        const int row_end = min(share, M - tm * kChainTile - r0);
        int lr = c < N ? warp : kChainTile;
        long long at_r = (long long)(tm * kChainTile + r0 + lr) * ld + c;
        uint2 rh[4], rl[4];
        auto ask = [&](int row, long long at) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            rh[j] = rl[j] = make_uint2(0u, 0u);
            if (r_hi && row + 8 * j < row_end) {
              rh[j] = __ldcg(reinterpret_cast<const uint2*>(r_hi + at + 8 * j * ld));
              rl[j] = __ldcg(reinterpret_cast<const uint2*>(r_lo + at + 8 * j * ld));
            }
          }
        };
        ask(lr, at_r);
        if (sliced) chain_cluster_meet();
        ok = chain_agree(ok);
        if (!ok) break;
        const uint32_t first_peer = cluster_ctarank() & ~(uint32_t)(split.slices - 1);
#pragma unroll 1
        for (; lr < row_end; lr += 32, at_r += 32 * ld) {
          float* at = stage + (r0 + lr) * kChainPitch + cg;
          float4 v[4];
          if (!sliced) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float4*>(at + 8 * j * kChainPitch);   // (the ring goes on behind the tile)
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            int from = slice < filled ? slice : slice % filled;      // in a fixed order; a block begins with its own, so that
#pragma unroll 4
            for (int s = 0; s < filled; ++s) {                       // they do not all read one
              const uint32_t peer = mapa_u32(smem_u32(at), first_peer + from);
              from = from + 1 < filled ? from + 1 : 0;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (lr + 8 * j < row_end) {
                  const float4 t = load_peer(peer + 8 * j * kChainPitch * 4);
                  v[j].x += t.x; v[j].y += t.y; v[j].z += t.z; v[j].w += t.w;
                }
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j].x *= alpha; v[j].y *= alpha; v[j].z *= alpha; v[j].w *= alpha;
            unpack_words(rh[j], rl[j], beta, v[j]);
          }
          ask(lr + 32, at_r + 32 * ld);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (lr + 8 * j >= row_end) break;
            if (mirror) *reinterpret_cast<float4*>(at + 8 * j * kChainPitch) = v[j];
            if (last) {
              const long long r = tm * kChainTile + r0 + lr + 8 * j;
              store_four(p.O + r * p.ldo + c, p.R ? p.R + r * p.ldr + c : nullptr, p.scale, p.keep, p.vec_out != 0, N - c, v[j]);
            } else {
              uint2 h, l;
              pack_words(v[j], pre, h, l);
              *reinterpret_cast<uint2*>(w_hi + at_r + 8 * j * ld) = h;
              *reinterpret_cast<uint2*>(w_lo + at_r + 8 * j * ld) = l;
            }
          }
        }
        if (mirror) {
          chain_agree(true);
          // eight rows of a column, to the row of that number
          // (up to four of a warp's lanes next to each other: 64 bytes of a row, and its reads meet in few banks)
          const int groups = share >> 3, wide = groups < 2 ? 0 : (groups < 4 ? 1 : 2);
#pragma unroll 1
          for (int i = tid; i < groups * kChainTile; i += kChainEpiThreads) {
            const int col = (i >> wide) & (kChainTile - 1), g = ((i & ((1 << wide) - 1)) + ((i >> wide) / kChainTile << wide)) * 8;
            const int row = tn * kChainTile + col;
            if (row < N && g < row_end) {
              float v[8];
#pragma unroll
              for (int q = 0; q < 8; ++q) v[q] = stage[(r0 + g + q) * kChainPitch + col];
              uint4 h, l;
              pack_words(v, pre, h, l);
              const long long to = (long long)row * ld + tm * kChainTile + r0 + g;
              *reinterpret_cast<uint4*>(w_hi + to) = h;
              *reinterpret_cast<uint4*>(w_lo + to) = l;
            }
          }
        }
        // (the ring's next user is TMA: the accesses above are put before it)
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0 && !empty) mbar_arrive(ring_bar);
      }
      if (sliced && (int)blockIdx.x >= units) chain_cluster_meet();
    } else if (warp == 8) {
      // ------------------------------------------------------------------ TMA producer
      if (lane == 0) {
        fence_proxy_async_global();
        const CUtensorMap* a = kind == 0 ? maps.x[cur] : (kind == 1 ? maps.a : (tall ? maps.x[cur] : maps.b));
        const CUtensorMap* b = kind == 0 ? maps.x[cur] : (kind == 1 ? maps.a : (tall ? maps.b : maps.x[cur]));
        bool ok = true;
        for (int unit = blockIdx.x; unit < units && ok; unit += gridDim.x) {
          int tm, tn, slice, kb0, kb1;
          unit_of(unit, tm, tn, slice, kb0, kb1);
          if (kb0 >= kb1) break;
          ok = mbar_wait_bounded(ring_bar, (units_done & 1) ^ 1, abort_flag, p.err, kErrProducerEmptyWait);
          ++units_done;
          for (int kb = kb0; kb < kb1 && ok; ++kb, ++it) {
            const uint32_t s = it % kChainStages;
            ok = mbar_wait_bounded(&empty_bar[s], ((it / kChainStages) & 1) ^ 1, abort_flag, p.err, kErrProducerEmptyWait);
            if (!ok) break;
            uint8_t* dst = smem + s * kChainStageBytes;
            mbar_arrive_expect_tx(&full_bar[s], kChainStageBytes);
            const int k0 = kb * kChainBK;
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int ra = tm * kChainTile + i * 64, rb = tn * kChainTile + i * 64;
                tma_load_2d(dst + w * kChainWords + i * (kChainWords / 2), a + w, a_mn ? ra : k0, a_mn ? k0 : ra, &full_bar[s]);
                tma_load_2d(dst + (2 + w) * kChainWords + i * (kChainWords / 2), b + w, b_mn ? rb : k0, b_mn ? k0 : rb, &full_bar[s]);
              }
          }
        }
        if (!ok)                                             // copies in flight, before the block ends
          for (uint32_t d = 1; d <= kChainStages && d <= it; ++d)
            mbar_wait_clocks(&full_bar[(it - d) % kChainStages], ((it - d) / kChainStages) & 1, kAbortDrainClocks);
      }
      if (sliced) chain_cluster_meet();
    } else {
      // ------------------------------------------------------------------ MMA issuer
      if (lane == 0) {
        const uint32_t idesc = umma_idesc_f16(kChainTile, kChainTile, a_mn, b_mn);
        // K-major: rows of 128 bytes, eight of them 1024 further; MN-major: eight k-rows 1024, the next 64 columns 8192 further
        constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | ((uint32_t)kSwizzle128 << 29);
        const uint32_t a_lo0 = ((a_mn ? 8192u : 16u) >> 4) << 16, b_lo0 = ((b_mn ? 8192u : 16u) >> 4) << 16;
        const uint32_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
        auto desc = [](uint32_t lo) -> uint64_t {
          uint64_t d;
          asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(desc_hi));
          return d;
        };
        bool ok = true;
        for (int unit = blockIdx.x; unit < units && ok; unit += gridDim.x, ++units_done) {
          int tm, tn, slice, kb0, kb1;
          unit_of(unit, tm, tn, slice, kb0, kb1);
          if (kb0 >= kb1) break;
          const uint32_t d_x = tmem_base + 2 * kChainTile;
          for (int c0 = kb0; c0 < kb1 && ok; c0 += p.chunk, ++chunks_done) {
            const uint32_t r = chunks_done & 1, d_main = tmem_base + r * kChainTile;
            ok = mbar_wait_bounded(&tempty_bar[r], ((chunks_done >> 1) & 1) ^ 1, abort_flag, p.err, kErrMmaTmemEmptyWait);
            if (ok && c0 == kb0)
              ok = mbar_wait_bounded(&tempty_bar[2], (units_done & 1) ^ 1, abort_flag, p.err, kErrMmaTmemEmptyWait);
            if (!ok) break;
            tc_fence_after_sync();
            const int c1 = min(kb1, c0 + p.chunk);
            for (int kb = c0; kb < c1; ++kb, ++it) {
              const uint32_t s = it % kChainStages;
              ok = mbar_wait_bounded(&full_bar[s], (it / kChainStages) & 1, abort_flag, p.err, kErrMmaFullWait);
              if (!ok) break;
              tc_fence_after_sync();
              const uint32_t st = (smem_u32(smem + s * kChainStageBytes) & 0x3FFFFu) >> 4;    // (without the rank in the cluster)
              const uint32_t a_hi = a_lo0 + st, a_lo = a_hi + (kChainWords >> 4);
              const uint32_t b_hi = b_lo0 + st + 2 * (kChainWords >> 4), b_lo = b_hi + (kChainWords >> 4);
#pragma unroll
              for (int j = 0; j < kChainBK / 16; ++j) {
                umma_f16_ss(d_x, desc(a_lo + a_step * j), desc(b_hi + b_step * j), idesc, kb == kb0 && j == 0 ? 0u : 1u);
                umma_f16_ss(d_main, desc(a_hi + a_step * j), desc(b_hi + b_step * j), idesc, kb == c0 && j == 0 ? 0u : 1u);
                umma_f16_ss(d_x, desc(a_hi + a_step * j), desc(b_lo + b_step * j), idesc, 1u);
              }
              umma_commit(&empty_bar[s]);
            }
            if (!ok) break;
            umma_commit(&tfull_bar[r]);
          }
          if (ok) umma_commit(&tfull_bar[2]);
        }
      }
      if (sliced) chain_cluster_meet();
    }
    if (phase + 1 < phases) go = chain_meet(p, ++round, abort_flag);
  }

  // A wait ran out: the block has nothing more to do, but others of its cluster may be through that wait and read its shared memory
  // yet.  It stays, and meets them as often as they meet it, so that no phase's meeting is taken for another one's.
#pragma unroll 1
  for (; phase < phases; ++phase) {
    const int kind = phase % 3;
    if ((kind == 0 ? p.gram : (kind == 1 ? p.square : p.update)).slices > 1) chain_cluster_meet();
  }

  // ---------------------------------------------------------------------- teardown
  if (warp == 9 && lane == 0) {                              // everything issued has retired before TMEM is freed
    umma_commit(drain_bar);
    mbar_wait_bounded(drain_bar, 0, nullptr, p.err, kErrDrainWait);
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
  chain_cluster_meet();                                      // (no block ends while another of its cluster may read its sums)
  if (tid == 0 && *abort_flag == 0u) {
    if (atomicAdd(&p.words[1], 1u) == gridDim.x - 1) p.words[0] = p.words[1] = 0u;      // the last one clears both
  }
}

}  // namespace sgc
