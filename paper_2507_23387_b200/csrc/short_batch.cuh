// The linear layer for a short batch (a few rows to some hundred): Y^T = W X^T on the tensor cores, one launch.
//
// The weight's 4 bytes per element are what bounds it, so the weight takes the 128-row side of the tile and the few rows
// of X the narrow one (16, 32 or 64 columns): a stage holds 32 KB of the weight and little else, and four to six of
// them are in flight in every SM (16384 x 4096 packed, 24 rows: 48 to 50 us in a chain of launches, 5.4 TB/s, 54 called
// one by one; its 128 tiles leave 20 SMs idle, and the MMA thread needs 1100 clocks of the 1500 that a block of 64 k
// takes).  A block takes one tile, so other widths fit worse: 86 tiles leave 62 SMs idle, 149 take two turns.  An
// FP32 weight comes in FP32 and is split here too, by eight warps, which then bound the kernel (86 us where packing and
// the product on packed words took 200).  X is not packed by a launch of its own: warps of this kernel turn 64 columns of it
// into words as they are needed, each such block with an exponent of its own (15 - e_max, as in packing; the more
// local scale keeps at least as many bits).  The warps that take the sums of a block out of TMEM bring them to the
// smallest exponent so far, like the running maximum of a softmax: all factors are powers of two, and what they push
// below FP32's range is nothing beside the block that caused it.
//
// A cluster of up to eight blocks shares a tile's k range where there are fewer tiles than SMs; their sums meet
// in shared memory, added in the order of the slices.
#pragma once

#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "linear_epilogue.cuh"
#include "linear_kernels.cuh"
#include "ptx_sm100.cuh"
#include "split_math.cuh"

namespace sgc {

constexpr int kShortThreads = 512;
constexpr int kShortK = 64;                  // k of a stage, of an exponent and of a stay in TMEM
constexpr int kShortN = 128;                 // outputs of a tile

struct ShortBatchParams {
  int M, N, K;
  int row_tiles;                             // of NT rows; neighbouring blocks take the same part of the weight
  const float* X;
  long long ldx;
  int xvec;
  float* Y;
  long long ldy;
  int ksplit, kslice_blocks;
  unsigned int* err;
  LinearEpilogue ep;                         // exp_b: the weight's exponent
};

template <int NT, bool W_F32>
struct ShortBatchCfg {
  static constexpr uint32_t W_TILE = kShortN * kShortK * 2, X_TILE = NT * kShortK * 2;
  static constexpr uint32_t STAGE_BYTES = 2 * (W_TILE + X_TILE), F32_BYTES = kShortN * kShortK * 4;
  // FP32 weights: two stages of words, and as many of FP32 as fit
  static constexpr int STAGES = W_F32 ? 2 : 221184 / STAGE_BYTES;
  static constexpr int F32_STAGES = W_F32 ? (221184 - STAGES * STAGE_BYTES) / F32_BYTES : 1;
  static constexpr uint32_t RING_BYTES = STAGES * STAGE_BYTES + (W_F32 ? F32_STAGES * F32_BYTES : 0);
  static constexpr uint32_t SMEM_BYTES = RING_BYTES + 1024 /*align*/ + 1024 /*barriers, exponents*/;
  static_assert(STAGES <= 6, "the ring of 16 exponents covers what is under way: STAGES + 2 blocks");
  static_assert(NT * kShortN * 4 <= RING_BYTES, "the sums lie where the stages were");
};

// split_two of x pre, two elements at a time: (x - hi) 2^s as one packed FMA, which is exact like the difference.
__device__ __forceinline__ void split_two_by(float x0, float x1, float pre, uint32_t& hi2, uint32_t& lo2) {
  uint64_t x, p, a, big, h2;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(x0), "f"(x1));
  asm("mov.b64 %0, {%1, %1};" : "=l"(p) : "f"(pre));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a) : "l"(x), "l"(p));
  float a0, a1;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(a));
  const __half2 h = __floats2half2_rn(a0, a1);
  const float2 hf = __half22float2(h);
  asm("mov.b64 %0, {%1, %1};" : "=l"(p) : "f"(pow2f(kPackScaleExp)));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(big) : "l"(a), "l"(p));
  asm("mov.b64 %0, {%1, %1};" : "=l"(p) : "f"(-pow2f(kPackScaleExp)));
  asm("mov.b64 %0, {%1, %2};" : "=l"(h2) : "f"(hf.x), "f"(hf.y));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(a) : "l"(h2), "l"(p), "l"(big));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(a));
  const __half2 l = __floats2half2_rn(a0, a1);
  hi2 = *reinterpret_cast<const uint32_t*>(&h);
  lo2 = *reinterpret_cast<const uint32_t*>(&l);
}
// The largest finite magnitude's bits of N x 4 elements.
template <int N>
__device__ __forceinline__ uint32_t largest_finite(const float4 (&v)[N]) {
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < N; ++u)
    m = fmaxf(fmaxf(m, fmaxf(fabsf(v[u].x), fabsf(v[u].y))), fmaxf(fabsf(v[u].z), fabsf(v[u].w)));
  if (m < INFINITY) return __float_as_uint(m);             // NaN loses against every number
  uint32_t b = 0;
#pragma unroll
  for (int u = 0; u < N; ++u)
    b = max(max(b, max(finite_bits(v[u].x), finite_bits(v[u].y))), max(finite_bits(v[u].z), finite_bits(v[u].w)));
  return b;
}

__device__ __forceinline__ int block_exponent(uint32_t amax) {
  return amax == 0 ? 126 : pack_exponent(amax);            // nothing but zeros: no reason to bring other blocks down
}
// Four elements of a row of which `left` are there.
__device__ __forceinline__ float4 load_four(const float* src, int left, int vec) {
  if (vec && left >= 4) return __ldg(reinterpret_cast<const float4*>(src));
  return make_float4(left > 0 ? __ldg(src) : 0.f, left > 1 ? __ldg(src + 1) : 0.f, left > 2 ? __ldg(src + 2) : 0.f,
                     left > 3 ? __ldg(src + 3) : 0.f);
}

// 2^d for d <= 0, zero where FP32 has no normal number for it.
__device__ __forceinline__ float pow2_down(int d) { return d < -126 ? 0.f : pow2f(d); }

template <int NT, bool W_MN, bool W_F32>
__global__ void __launch_bounds__(kShortThreads, 1)
short_batch_kernel(const __grid_constant__ CUtensorMap tm_hi, const __grid_constant__ CUtensorMap tm_lo,
                   const ShortBatchParams p) {
  using Cfg = ShortBatchCfg<NT, W_F32>;
  constexpr int STAGES = Cfg::STAGES, F32_STAGES = Cfg::F32_STAGES, kRing = 16, kGroups = 4;
  // two TMEM regions: hi*hi and hi*lo sums (2 NT columns), lo*hi sums (NT columns, at 2 NT)
  constexpr uint32_t kRegion = 4 * NT, kTmem = 2 * kRegion;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + Cfg::RING_BYTES);    // TMA and converters -> MMA
  uint64_t* empty_bar = full_bar + STAGES;                                     // MMA -> TMA and converters
  uint64_t* tfull_bar = empty_bar + STAGES;                                    // [2] MMA -> accumulate warps
  uint64_t* tempty_bar = tfull_bar + 2;                                        // [2] accumulate warps -> MMA
  uint64_t* pair_bar = tempty_bar + 2;                                         // [kGroups] between two converter warps
  uint64_t* full32_bar = pair_bar + kGroups;                                   // FP32 weights: TMA -> converters
  uint64_t* empty32_bar = full32_bar + F32_STAGES;                             // and back
  uint64_t* drain_bar = empty32_bar + F32_STAGES;                              // the MMA thread's last wait
  int* block_exp = reinterpret_cast<int*>(drain_bar + 1);                      // [kRing]
  uint32_t* part_max = reinterpret_cast<uint32_t*>(block_exp + kRing);         // [2][8 warps][X, weight]
  int* slice_exp = reinterpret_cast<int*>(part_max + 32);                      // [8] of the cluster's blocks
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(slice_exp + 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  static_assert((2 * STAGES + 5 + kGroups + 2 * F32_STAGES) * 8 + (kRing + 32 + 8 + 2) * 4 <= 1024, "barrier block");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ranks = p.ksplit, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int tile = (int)(blockIdx.x / (unsigned)ranks);
  const int n0 = tile / p.row_tiles * kShortN, m0 = tile % p.row_tiles * NT, rows = min(NT, p.M - m0);
  const int num_kb = (p.K + kShortK - 1) / kShortK;
  const int kb0 = rank * p.kslice_blocks, count = min(num_kb, kb0 + p.kslice_blocks) - kb0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], W_F32 ? 8 : 3);                // all converter warps; or two of them and the TMA thread
      mbar_init(&empty_bar[s], 1);
    }
    for (int r = 0; r < 2; ++r) {
      mbar_init(&tfull_bar[r], 1);
      mbar_init(&tempty_bar[r], 4);
    }
    mbar_init(drain_bar, 1);
    for (int g = 0; g < kGroups; ++g) mbar_init(&pair_bar[g], W_F32 ? 8 : 2);
    for (int s = 0; s < F32_STAGES; ++s) {
      mbar_init(&full32_bar[s], 1);
      mbar_init(&empty32_bar[s], 8);
    }
    *abort_flag = 0u;
    fence_mbar_init();
    tma_prefetch_desc(&tm_hi);
    tma_prefetch_desc(&tm_lo);
  }
  if (warp == 1) { tmem_alloc(tmem_slot, kTmem); tmem_relinquish(); }
  tc_fence_before_sync();
  __syncthreads();
  if (ranks > 1) cluster_sync_all();                         // the peers run before anyone writes to them
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA: the weight's words, or the FP32 weight
    if (lane == 0) {
      bool ok = true;
      for (int i = 0; i < count; ++i) {
        if constexpr (W_F32) {
          const int s = i % F32_STAGES;
          if (!mbar_wait_bounded(&empty32_bar[s], ((i / F32_STAGES) & 1) ^ 1, abort_flag, p.err, kErrProducerEmptyWait)) {
            ok = false;
            break;
          }
          uint8_t* st = smem + STAGES * Cfg::STAGE_BYTES + s * Cfg::F32_BYTES;
          const int k0 = (kb0 + i) * kShortK;
          mbar_arrive_expect_tx(&full32_bar[s], Cfg::F32_BYTES);
          if (W_MN) tma_load_2d(st, &tm_hi, n0, k0, &full32_bar[s]);         // 64 rows of 128 outputs
          else tma_load_2d(st, &tm_hi, k0, n0, &full32_bar[s]);              // 128 rows of 64 k
          continue;
        }
        const int s = i % STAGES;
        if (!mbar_wait_bounded(&empty_bar[s], ((i / STAGES) & 1) ^ 1, abort_flag, p.err, kErrProducerEmptyWait)) {
          ok = false;
          break;
        }
        uint8_t* st = smem + s * Cfg::STAGE_BYTES;
        const int k0 = (kb0 + i) * kShortK;
        mbar_arrive_expect_tx(&full_bar[s], 2 * Cfg::W_TILE);
        if constexpr (W_MN) {                                // boxes of 64 outputs x 64 k rows
          for (int a = 0; a < 2; ++a) {
            tma_load_2d(st + a * 8192, &tm_hi, n0 + a * 64, k0, &full_bar[s]);
            tma_load_2d(st + Cfg::W_TILE + a * 8192, &tm_lo, n0 + a * 64, k0, &full_bar[s]);
          }
        } else {                                             // one box of 64 k x 128 outputs
          tma_load_2d(st, &tm_hi, k0, n0, &full_bar[s]);
          tma_load_2d(st + Cfg::W_TILE, &tm_lo, k0, n0, &full_bar[s]);
        }
      }
      if (!ok) {                                             // copies may be under way: let them land
        const long long t0 = clock64();
        while (clock64() - t0 < kAbortDrainClocks) {}
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      // An MMA of 128 rows and 16 k takes about 120 clocks however few columns it has, so hi and lo words of X, which lie
      // one behind the other, are the columns of one: hi*hi and hi*lo next to each other.  lo*hi has columns of its own,
      // since only MMAs of the same shape are sure to follow one another on the same sums.  (With three MMAs a k16 step
      // they bound the kernel: 1440 clocks a block.)
      constexpr uint32_t idesc_both = umma_idesc_f16(kShortN, 2 * NT, W_MN, false), idesc = umma_idesc_f16(kShortN, NT, W_MN, false);
      // Descriptors: everything but the address (low word, 16-byte units) is constant, and an MMA's costs one addition.
      // A single lane issues them all.
      constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | ((uint32_t)kSwizzle128 << 29);
      constexpr uint32_t w_lo0 = ((W_MN ? 8192u : 16u) >> 4) << 16, x_lo0 = (16u >> 4) << 16;
      constexpr uint32_t w_step = (W_MN ? 2048u : 32u) >> 4, x_step = 32u >> 4;    // from one k16 step to the next
      constexpr uint32_t w_words = Cfg::W_TILE >> 4;   // from hi to lo words
      const uint32_t ring = (smem_u32(smem) & 0x3FFFFu) >> 4;                      // (a cluster's rank bits cut off)
      auto desc = [](uint32_t lo) {
        uint64_t d;
        asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(desc_hi));
        return d;
      };
      int s = 0;
      uint32_t phase = 0;
      for (int i = 0; i < count; ++i) {
        const int r = i & 1;
        if (!mbar_wait_bounded(&full_bar[s], phase, abort_flag, p.err, kErrMmaFullWait)) break;
        if (!mbar_wait_bounded(&tempty_bar[r], ((i >> 1) & 1) ^ 1, abort_flag, p.err, kErrMmaTmemEmptyWait)) break;
        tc_fence_after_sync();
        const uint32_t w = ring + s * (Cfg::STAGE_BYTES >> 4) + w_lo0;
        const uint32_t x = ring + s * (Cfg::STAGE_BYTES >> 4) + 2 * w_words + x_lo0;
        const uint32_t d = tmem + r * kRegion;
#pragma unroll
        for (int j = 0; j < kShortK / 16; ++j) {
          umma_f16_ss(d, desc(w + j * w_step), desc(x + j * x_step), idesc_both, j != 0);
          umma_f16_ss(d + 2 * NT, desc(w + w_words + j * w_step), desc(x + j * x_step), idesc, j != 0);
        }
        umma_commit(&empty_bar[s]);
        umma_commit(&tfull_bar[r]);
        if (++s == STAGES) { s = 0; phase ^= 1; }
      }
      // whether the loop came to its end or not: everything issued has been done before TMEM is freed
      umma_commit(drain_bar);
      mbar_wait_bounded(drain_bar, 0, nullptr, p.err, kErrDrainWait);
    }
  } else if (W_F32 && warp >= 8) {
    // ------------------------------------------------------------------ converters: weight and X to words
    // All eight warps on every block: a thread has four neighbouring elements of 8 places of the weight and of NT / 16
    // of X; those of the next block's X are on their way meanwhile.  The next block is read and its maxima exchanged
    // right behind the conversion of the present one (in front of it: 16384 x 4096 with 16 rows 112 us, 86 so).
    constexpr int UW = kShortN * kShortK / 4 / 256, UX = NT * kShortK / 4 / 256;
    const int t = threadIdx.x - 256, q = t & 15;
    float4 w[UW], w_next[UW], x[UX], x_next[UX];
    auto fetch_x = [&](int i) {
      const int k = (kb0 + i) * kShortK + q * 4;
#pragma unroll
      for (int u = 0; u < UX; ++u) {
        const int row = (u * 256 + t) >> 4;
        x_next[u] = load_four(p.X + (m0 + row) * p.ldx + k, row < rows ? p.K - k : 0, p.xvec);
      }
    };
    auto put = [](uint8_t* hi_at, uint32_t lo_off, float4 v, float pre) {
      uint2 hi, lo;
      split_two_by(v.x, v.y, pre, hi.x, lo.x);
      split_two_by(v.z, v.w, pre, hi.y, lo.y);
      *reinterpret_cast<uint2*>(hi_at) = hi;
      *reinterpret_cast<uint2*>(hi_at + lo_off) = lo;
    };
    auto read_block = [&](int i) {                           // block i to w_next; its maxima, with x_next's, to all warps
      const int s32 = i % F32_STAGES;
      const bool ok = mbar_wait_bounded(&full32_bar[s32], (i / F32_STAGES) & 1, abort_flag, p.err, kErrConvFullWait);
      if (!__all_sync(0xffffffffu, ok)) return false;
      const float4* src = reinterpret_cast<const float4*>(smem + STAGES * Cfg::STAGE_BYTES + s32 * Cfg::F32_BYTES) + t;
#pragma unroll
      for (int u = 0; u < UW; ++u) w_next[u] = src[u * 256];
      const uint32_t mx = __reduce_max_sync(0xffffffffu, largest_finite(x_next));
      const uint32_t mw = __reduce_max_sync(0xffffffffu, largest_finite(w_next));
      if (lane == 0) {
        mbar_arrive(&empty32_bar[s32]);
        *reinterpret_cast<uint2*>(part_max + (i & 1) * 16 + (warp - 8) * 2) = make_uint2(mx, mw);
        mbar_arrive(&pair_bar[0]);
      }
      return true;
    };
    fetch_x(0);
    bool ok = read_block(0);
    for (int i = 0; i < count && ok; ++i) {
      const int s = i % STAGES;
#pragma unroll
      for (int u = 0; u < UW; ++u) w[u] = w_next[u];
#pragma unroll
      for (int u = 0; u < UX; ++u) x[u] = x_next[u];
      if (i + 1 < count) fetch_x(i + 1);
      ok = mbar_wait_bounded(&pair_bar[0], i & 1, abort_flag, p.err, kErrConvFullWait) &&
           mbar_wait_bounded(&empty_bar[s], ((i / STAGES) & 1) ^ 1, abort_flag, p.err, kErrConvEmptyWait);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      uint32_t mx = 0, mw = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint2 m = *reinterpret_cast<const uint2*>(part_max + (i & 1) * 16 + j * 2);
        mx = max(mx, m.x);
        mw = max(mw, m.y);
      }
      const int ex = block_exponent(mx), ew = block_exponent(mw);
      if (t == 0) block_exp[i % kRing] = ex + ew;
      const float pre_x = pow2f(ex), pre_w = pow2f(ew);
      uint8_t* words = smem + s * Cfg::STAGE_BYTES;
#pragma unroll
      for (int u = 0; u < UW; ++u) {
        const int at = u * 256 + t;                          // 128-byte rows: an output's 64 k, or 64 outputs of a k
        const int row = W_MN ? at >> 5 : at >> 4, half = W_MN ? (at >> 4) & 1 : 0;
        put(words + half * 8192 + row * 128 + (((q >> 1) ^ (row & 7)) << 4) + (q & 1) * 8, Cfg::W_TILE, w[u], pre_w);
      }
      words += 2 * Cfg::W_TILE;
#pragma unroll
      for (int u = 0; u < UX; ++u) {
        const int row = (u * 256 + t) >> 4;
        put(words + row * 128 + (((q >> 1) ^ (row & 7)) << 4) + (q & 1) * 8, Cfg::X_TILE, x[u], pre_x);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full_bar[s]);
      if (i + 1 < count) ok = read_block(i + 1);
    }
  } else if (warp >= 8) {
    // ------------------------------------------------------------------ converters: X to words
    // Two warps take every fourth block of 64 columns; a thread has eight neighbouring elements of NT / 8 rows.
    constexpr int U = NT / 8;
    const int group = (warp - 8) >> 1, t = threadIdx.x & 63;
    const int chunk = t & 7, row0 = t >> 3;
    for (int i = group; i < count; i += kGroups) {
      const int s = i % STAGES, k = (kb0 + i) * kShortK + chunk * 8;
      float4 v[2 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = row0 + 8 * u, left = row < rows ? p.K - k : 0;
        const float* src = p.X + (m0 + row) * p.ldx + k;
        v[2 * u] = load_four(src, left, p.xvec);
        v[2 * u + 1] = load_four(src + 4, left - 4, p.xvec);
      }
      uint32_t m = largest_finite(v);
      m = __reduce_max_sync(0xffffffffu, m);
      uint32_t* both = part_max + ((i / kGroups) & 1) * 2 * kGroups + group * 2;
      if (lane == 0) {
        both[warp & 1] = m;
        mbar_arrive(&pair_bar[group]);
      }
      bool ok = mbar_wait_bounded(&pair_bar[group], (i / kGroups) & 1, abort_flag, p.err, kErrConvFullWait);
      m = max(both[0], both[1]);
      const int e = block_exponent(m);
      const float pre = pow2f(e);
      ok = ok && mbar_wait_bounded(&empty_bar[s], ((i / STAGES) & 1) ^ 1, abort_flag, p.err, kErrConvEmptyWait);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (t == 0) block_exp[i % kRing] = e;
      uint8_t* words = smem + s * Cfg::STAGE_BYTES + 2 * Cfg::W_TILE;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = row0 + 8 * u;
        uint4 hi, lo;
        split_two_by(v[2 * u].x, v[2 * u].y, pre, hi.x, lo.x);
        split_two_by(v[2 * u].z, v[2 * u].w, pre, hi.y, lo.y);
        split_two_by(v[2 * u + 1].x, v[2 * u + 1].y, pre, hi.z, lo.z);
        split_two_by(v[2 * u + 1].z, v[2 * u + 1].w, pre, hi.w, lo.w);
        uint8_t* at = words + row * 128 + ((chunk ^ (row & 7)) << 4);        // 128-byte swizzle
        *reinterpret_cast<uint4*>(at) = hi;
        *reinterpret_cast<uint4*>(at + Cfg::X_TILE) = lo;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full_bar[s]);
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ accumulate: one output a thread
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    float S[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) S[j] = 0.f;
    int e = 252;                                             // above every block's
    for (int i = 0; i < count; ++i) {
      const int r = i & 1;
      const bool ok = mbar_wait_bounded(&tfull_bar[r], (i >> 1) & 1, abort_flag, p.err, kErrEpiTmemFullWait);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after_sync();
      const int now = block_exp[i % kRing];
      if (now < e) {
        const float down = pow2_down(now - e);
#pragma unroll
        for (int j = 0; j < NT; ++j) S[j] *= down;
        e = now;
      }
      const float f = pow2_down(e - now);
#pragma unroll
      for (int g = 0; g < NT / 16; ++g) {
        uint32_t v[3][16];
#pragma unroll
        for (int a = 0; a < 3; ++a) tmem_ld_32x32b_x16(mine + r * kRegion + a * NT + g * 16, v[a]);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float cross = __uint_as_float(v[1][j]) + __uint_as_float(v[2][j]);
          S[g * 16 + j] = fmaf(fmaf(cross, kPackInvScale, __uint_as_float(v[0][j])), f, S[g * 16 + j]);
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty_bar[r]);
    }
    // every stage has been multiplied: the sums go where the first of them was
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int j = 0; j < NT; ++j) sums[j * kShortN + (warp & 3) * 32 + lane] = S[j];
    if (warp == 4 && lane < ranks)
      asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(ranks > 1 ? mapa_u32(smem_u32(slice_exp + rank), (uint32_t)lane)
                                                                      : smem_u32(slice_exp)), "r"(e) : "memory");
  }
  tc_fence_before_sync();
  __syncthreads();
  if (ranks > 1) cluster_sync_all();

  // ---------------------------------------------------------------------- all warps: rows rank, rank + ranks, ... of Y
  {
    constexpr int U = 4;
    const int f = (warp & 3) * 32 + lane, n = n0 + f;
    const bool in = n < p.N;
    int least = slice_exp[0];
    for (int s = 1; s < ranks; ++s) least = min(least, slice_exp[s]);
    const PowerBack back = power_back_of(-(least + (W_F32 ? 0 : *p.ep.exp_b)));
    const float bias = p.ep.bias && in ? __ldg(p.ep.bias + n) : 0.f;
    const uint32_t sums = smem_u32(smem) + f * 4;
#pragma unroll 1
    for (int i = warp >> 2; rank + ranks * i < rows; i += 4 * U) {
      float v[U], res[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = rank + ranks * (i + 4 * u);
        v[u] = 0.f;
        res[u] = p.ep.R && in && row < rows ? p.ep.R[(m0 + row) * p.ep.ldr + n] : 0.f;
      }
#pragma unroll 1
      for (int s = 0; s < ranks; ++s) {
        const float scale = pow2_down(least - slice_exp[s]);
        const uint32_t from = ranks > 1 ? mapa_u32(sums, (uint32_t)s) : sums;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int row = min(rank + ranks * (i + 4 * u), rows - 1);
          float x;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(from + row * (kShortN * 4)) : "memory");
          v[u] = fmaf(x, scale, v[u]);
        }
      }
      auto store = [&](float* out, long long ld) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int row = rank + ranks * (i + 4 * u);
          if (in && row < rows) out[(m0 + row) * ld + n] = v[u];
        }
      };
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = back(v[u]) + bias;
      if (p.ep.Z) store(p.ep.Z, p.ep.ldz);
      switch (p.ep.act) {
        case kActRelu: act_each<kActRelu>(v); break;
        case kActGelu: act_each<kActGelu>(v); break;
        case kActGeluTanh: act_each<kActGeluTanh>(v); break;
        case kActSilu: act_each<kActSilu>(v); break;
        default: break;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) if (p.ep.R) v[u] += res[u];
      store(p.Y, p.ldy);
    }
  }
  if (ranks > 1) cluster_sync_all();                         // a block's sums stay until every other has read them
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(tmem, kTmem);
  }
}

}  // namespace sgc
