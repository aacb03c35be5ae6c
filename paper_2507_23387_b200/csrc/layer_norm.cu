// Layer normalisation and its gradients (contracts: include/sgemm_cube.h).
//
//   forward    mean = sum x / n;  var = sum (x - mean)^2 / n;  y = (x - mean) rstd w + b
//              The sum and its division leave mean off by some units in its last place, which is much where the
//              spread is small beside it.  So what the first mean m0 is off by is found as well:
//              c = sum (x - m0) / n,  mean = m0 + c,  var = sum (x - m0)^2 / n - c^2,  y = (x - m0 - c) rstd w + b
//   backward   u = dy w;  n = (x - mean) rstd;  dx = rstd (u - mean(u) - n mean(u n))
//              dw = sum over rows of dy n;  db = sum over rows of dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx, each once (8192 x 4096 FP32
// 44 us and 69, 6.1 and 5.9 TB/s; BF16 rows by instructions as well, 6000 x 2048 12 and 23, 4.1 and 3.2 TB/s).  A row
// lives in the registers of one group of warps between its load and its store, so the second moment is
// taken about the first mean (no cancellation of squares) without a second read.  Blocks are persistent: a
// group asks for its next rows before it works on the present one, and keeps its columns' weights (forward)
// or running sums of dw and db (backward) in registers all the way.
//
// Rows of an odd length start anywhere between two 16-byte boundaries and are read element by element, except by the
// backward kernel where all tensors agree in where a row starts: then the vectors are laid on the boundaries
// (kShifted), and a group's rows are a multiple of 8 (FP32: 4) apart, so that they all start equally far behind one
// and a thread's columns stay the same (4000 x 7001 BF16 51 us, 83 by elements).
#include <atomic>

#include "ctx.cuh"
#include "elements.cuh"

namespace sgc {

constexpr int kPT = 16;         // elements of a row a thread holds

// Aligned rows pass through shared memory: this many rows of a block's groups have slots there (three where they fit,
// so that two are under way beside the present one).
template <typename T, int WARPS>
constexpr int slot_stages(int tensors) {
  const size_t row = (size_t)tensors * kPT * sizeof(T) * (WARPS > 8 ? WARPS * 32 : 256);
  // FP32 rows of 8 warps (2049 to 4096 columns, three blocks an SM) come two deep, which is the faster over their whole
  // range (2 and 3 deep: 8192 x 2052 29.9 and 31.6 us, x 2560 29.8 and 30.9, x 3584 37.9 and 40.3, x 4096 45.9 and
  // 48.8; 1000 x 4096 7.8 and 8.3).
  if (tensors == 1 && WARPS == 8 && sizeof(T) == 4) return 2;
  return 3 * row <= 200 * 1024 ? 3 : (2 * row <= 200 * 1024 ? 2 : 1);
}
template <typename T, int WARPS, bool VEC, int TENSORS>
constexpr int kStages = VEC ? slot_stages<T, WARPS>(TENSORS) : 0;
template <typename T, int WARPS, bool VEC, int TENSORS>
constexpr size_t kSlotBytes = (size_t)kStages<T, WARPS, VEC, TENSORS> * TENSORS * kPT * sizeof(T) * (WARPS > 8 ? WARPS * 32 : 256);

__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
// Warps' sums added over a row's group of warps.  The caller takes two buffers in turn, so one barrier a sum is enough.
// (16 and 32 warps by shuffles: 2048 x 16384 BF16 32 us, 34.5 with every thread adding up; 4 and 8 are faster that way.)
template <int WARPS, int N>
__device__ __forceinline__ void join_warps(float (&s)[N], float* buf, int group, int warp_in_group, int bar_threads) {
  if constexpr (WARPS > 1) {
    float* b = buf + group * WARPS * N;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) b[warp_in_group * N + i] = s[i];
    }
    if (bar_threads == 0) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(bar_threads) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (WARPS >= 16) {                       // a warp's sum a lane
        s[i] = b[(threadIdx.x & (WARPS - 1)) * N + i];
#pragma unroll
        for (int o = WARPS / 2; o > 0; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
      } else {
        float t = b[i];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) t += b[w * N + i];
        s[i] = t;
      }
    }
  }
}
template <int WARPS, int N>
__device__ __forceinline__ void group_sum(float (&s)[N], float* buf, int group, int warp_in_group, int bar_threads) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = warp_sum(s[i]);
  join_warps<WARPS>(s, buf, group, warp_in_group, bar_threads);
}

struct NormParams {
  int rows, cols;
  const void* X;
  long long ldx;
  const void* dY;
  long long lddy;
  void* out;               // Y or dX
  long long ldo;
  const float* weight;
  const float* bias;
  float eps;
  float* mean;
  float* rstd;
  const float* mean_in;
  const float* rstd_in;
  float* part;             // backward: [blocks][2][cols] partial sums of dw and db, or null
  int period;              // backward: rows this far apart start equally far behind a 16-byte boundary
};

// rstd from the mean square about the first mean and that mean's correction; the difference of the two may fall below
// zero by rounding (a NaN stays).  1 / sqrt as the approximate one (2^-22) with a Newton step, good to 2 units; the step is
// left out where it would multiply 0 by infinity.
__device__ __forceinline__ float norm_rstd(float square, float c, float eps) {
  const float var = fmaf(-c, c, square), v = (var < 0.f ? 0.f : var) + eps;
  const float r = rsqrtf(v), e = fmaf(-v * r, r, 1.f);
  return fabsf(e) < 1.f ? fmaf(0.5f * r, e, r) : r;
}

// Blocks an SM the registers are cut for: with three, single elements and groups that meet at barriers of their own run
// out of them (6001 x 2047 BF16 21.4 us, 14.5 with two; 6000 x 2048 13.8 and 12.1; but 8192 x 4096 26.5 and 27.5).
constexpr int forward_blocks(int warps, bool vec) { return warps > 8 ? 1 : (vec && warps == 8 ? 3 : 2); }

// WARPS warps a row, 8 / WARPS rows a block (one for WARPS >= 8).
template <typename T, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS > 8 ? WARPS * 32 : 256, forward_blocks(WARPS, VEC)) norm_forward_kernel(NormParams p) {
  constexpr int kGroups = WARPS >= 8 ? 1 : 8 / WARPS, kThreads = WARPS * 32;
  __shared__ float buf[kGroups * WARPS], buf2[kGroups * WARPS * 2];
  const int group = threadIdx.x / kThreads, t = threadIdx.x % kThreads, wg = t >> 5;
  const int bar = kGroups == 1 ? 0 : kThreads;         // groups meet at their own barriers
  const float inv_n = 1.f / (float)p.cols;
  const long long step = (long long)gridDim.x * kGroups;
  long long row = (long long)blockIdx.x * kGroups + group;
  if (row >= p.rows) return;
  constexpr int kBlock = WARPS > 8 ? WARPS * 32 : 256, kWords = VEC ? kPT / Elem<T>::kVec : 1;
  constexpr int kRing = kStages<T, WARPS, VEC, 1>, kAhead = kRing - 1;
  static_assert(!VEC || kRing >= 2, "forward rows always fit twice");
  extern __shared__ uint4 ring[];                      // [kRing][kWords][kBlock]
  RowRegs<T, VEC ? 1 : kPT> next;                      // (not for vectors)
  auto ask = [&](long long r, int s) {                 // an empty group past the end
    if (r < p.rows)
      RowSlots<T, kPT>::ask(ring + s * kWords * kBlock + threadIdx.x, kBlock, static_cast<const T*>(p.X) + r * p.ldx,
                            p.cols, t, kThreads);
    async_commit();
  };
  int stage = 0;
  if constexpr (VEC) {
    for (int a = 0; a < kAhead; ++a) ask(row + a * step, a);
  } else {
    next.fetch(static_cast<const T*>(p.X) + row * p.ldx, p.cols, t, kThreads);
  }
  float w[kPT], b[kPT];
  load_params<T, kPT, VEC>(p.weight, 1.f, p.cols, t, kThreads, w);
  load_params<T, kPT, VEC>(p.bias, 0.f, p.cols, t, kThreads, b);
  // FP32 rows are summed a second time for the correction.  A warp's 512 elements of a 16-bit type have so few bits
  // that their sum loses next to nothing in FP32; there its difference to count * mean serves.
  constexpr bool kTwice = sizeof(T) == 4;
  int columns = 0;                                     // of this warp
#pragma unroll
  for (int i = 0; i < kPT; ++i) columns += row_column<T, VEC>(i, t, kThreads) < p.cols;
  [[maybe_unused]] const float count = (float)__reduce_add_sync(0xffffffffu, columns);
  for (; row < p.rows; row += step) {
    float v[kPT];
    if constexpr (VEC) {
      ask(row + kAhead * step, stage == 0 ? kAhead : stage - 1);
      async_wait<kAhead>();
      RowSlots<T, kPT>::get(ring + stage * kWords * kBlock + threadIdx.x, kBlock, v);
      stage = stage == kAhead ? 0 : stage + 1;
    } else {
      next.get(v);
      if (row + step < p.rows) next.fetch(static_cast<const T*>(p.X) + (row + step) * p.ldx, p.cols, t, kThreads);
    }
    float s[1] = {0.f}, d[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kPT; ++i) s[0] += v[i];
    const float own = s[0] = warp_sum(s[0]);
    join_warps<WARPS>(s, buf, group, wg, bar);
    const float mean = s[0] * inv_n;
#pragma unroll
    for (int i = 0; i < kPT; ++i) {
      v[i] -= mean;
      const float in = row_column<T, VEC>(i, t, kThreads) < p.cols ? v[i] : 0.f;
      d[0] = fmaf(v[i], in, d[0]);
      if constexpr (kTwice) d[1] += in;
    }
    d[0] = warp_sum(d[0]);
    d[1] = kTwice ? warp_sum(d[1]) : fmaf(-mean, count, own);
    join_warps<WARPS>(d, buf2, group, wg, bar);
    const float c = d[1] * inv_n, rstd = norm_rstd(d[0] * inv_n, c, p.eps), shift = -c * rstd;
#pragma unroll
    for (int i = 0; i < kPT; ++i) v[i] = fmaf(fmaf(v[i], rstd, shift), w[i], b[i]);
    store_row<T, kPT, VEC>(static_cast<T*>(p.out) + row * p.ldo, p.cols, t, kThreads, v);
    if (t == 0) {
      if (p.mean) p.mean[row] = mean + c;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

// Rows too long for the registers of one block: three passes, the later ones from L2.
template <typename T>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(NormParams p) {
  __shared__ float buf[32], buf2[64];
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.X) + row * p.ldx;
  T* y = static_cast<T*>(p.out) + row * p.ldo;
  const int t = threadIdx.x;
  float s[1] = {0.f};
  for (int c = t; c < p.cols; c += 1024) s[0] += Elem<T>::get(x[c]);
  group_sum<32>(s, buf, 0, t >> 5, 0);
  const float mean = s[0] / (float)p.cols;
  float sd[2] = {0.f, 0.f};
  for (int c = t; c < p.cols; c += 1024) {
    const float d = Elem<T>::get(x[c]) - mean;
    sd[0] = fmaf(d, d, sd[0]);
    sd[1] += d;
  }
  group_sum<32>(sd, buf2, 0, t >> 5, 0);
  const float more = sd[1] / (float)p.cols, rstd = norm_rstd(sd[0] / (float)p.cols, more, p.eps), shift = -more * rstd;
  for (int c = t; c < p.cols; c += 1024) {
    float n = fmaf(Elem<T>::get(x[c]) - mean, rstd, shift);
    if (p.weight) n *= p.weight[c];
    if (p.bias) n += p.bias[c];
    y[c] = Elem<T>::put(n);
  }
  if (t == 0) {
    if (p.mean) p.mean[row] = mean + more;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// dx, and the block's partial sums of dw and db: a thread holds the same columns of every row.  The longest aligned
// rows (1024 threads, 64 registers each) stay in their slots and are read twice from there, for the sums and for dx;
// shorter ones are held in registers with the weights (2048 x 16384 FP32 260 us held, 110 read twice; 8192 x 4096
// 81 held, 90 read twice).
enum RowAccess { kElements = 0, kAligned, kShifted };

template <typename T, int WARPS, RowAccess ACCESS>
__global__ void __launch_bounds__(WARPS > 8 ? WARPS * 32 : 256, WARPS > 8 ? 1 : 2) norm_backward_kernel(NormParams p) {
  constexpr bool VEC = ACCESS != kElements, SHIFT = ACCESS == kShifted;
  constexpr int kGroups = WARPS >= 8 ? 1 : 8 / WARPS, kThreads = WARPS * 32;
  __shared__ float buf[2][kGroups * WARPS * 2];
  const int group = threadIdx.x / kThreads, t = threadIdx.x % kThreads, wg = t >> 5;
  const int bar = kGroups == 1 ? 0 : kThreads;
  const float inv_n = 1.f / (float)p.cols;
  const long long step = (long long)gridDim.x * kGroups;
  long long row = (long long)blockIdx.x * kGroups + group;
  float dw[kPT], db[kPT];
#pragma unroll
  for (int i = 0; i < kPT; ++i) dw[i] = db[i] = 0.f;
  int slot = 0;
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch_stats = [&](long long r) {
    next_mean = __ldg(p.mean_in + r);
    next_rstd = __ldg(p.rstd_in + r);
  };
  if (row < p.rows) fetch_stats(row);
  // the thread's first column, and the column of its element i
  int first = VEC ? t * Elem<T>::kVec : t;
  if constexpr (SHIFT)
    first -= (int)((reinterpret_cast<uintptr_t>(static_cast<const T*>(p.X) + row * p.ldx) & 15u) / sizeof(T));
  auto column = [&](int i) {
    constexpr int V = VEC ? Elem<T>::kVec : 1;
    return i / V * kThreads * V + first + i % V;
  };
  auto inside = [&](int c) { return (unsigned)c < (unsigned)p.cols; };
  if constexpr (VEC) {
    constexpr int V = Elem<T>::kVec, kWords = kPT / V, kBlock = WARPS > 8 ? WARPS * 32 : 256;
    constexpr int kRing = kStages<T, WARPS, VEC, 2>;
    extern __shared__ uint4 ring[];                    // [kRing][2][kWords][kBlock]
    auto ask = [&](long long r, int s) {               // an empty group past the end
      if (r < p.rows) {
        uint4* to = ring + s * 2 * kWords * kBlock + threadIdx.x;
        const T* x = static_cast<const T*>(p.X) + r * p.ldx;
        const T* g = static_cast<const T*>(p.dY) + r * p.lddy;
        if constexpr (SHIFT) {
          ShiftedSlots<T, kPT>::ask(to, kBlock, x, p.cols, first, kThreads, r == 0);
          ShiftedSlots<T, kPT>::ask(to + kWords * kBlock, kBlock, g, p.cols, first, kThreads, r == 0);
        } else {
          RowSlots<T, kPT>::ask(to, kBlock, x, p.cols, t, kThreads);
          RowSlots<T, kPT>::ask(to + kWords * kBlock, kBlock, g, p.cols, t, kThreads);
        }
      }
      async_commit();
    };
    constexpr bool kHold = WARPS <= 16;
    const bool wvec = !SHIFT && (reinterpret_cast<uintptr_t>(p.weight) & 15u) == 0;
    float w[kHold ? kPT : 1];
    if constexpr (kHold && SHIFT) {
#pragma unroll
      for (int i = 0; i < kPT; ++i) w[i] = p.weight && inside(column(i)) ? __ldg(p.weight + column(i)) : 1.f;
    } else if constexpr (kHold) {
      load_params<T, kPT, VEC>(p.weight, 1.f, p.cols, t, kThreads, w);
    }
    // n, dy and u = dy w of vector i of a row
    auto vector_of = [&](const uint4* from, int i, float mean, float rstd, float (&n)[V], float (&g)[V], float (&u)[V]) {
      if constexpr (SHIFT) {
        ShiftedSlots<T, kPT>::vector(from, kBlock, i, first, n);
        ShiftedSlots<T, kPT>::vector(from + kWords * kBlock, kBlock, i, first, g);
      } else {
        Elem<T>::unpack(from[i * kBlock], n);
        Elem<T>::unpack(from[(kWords + i) * kBlock], g);
      }
      const int c = column(i * V);
#pragma unroll
      for (int q = 0; q < V; ++q) n[q] = (n[q] - mean) * rstd;
      if constexpr (kHold) {
#pragma unroll
        for (int q = 0; q < V; ++q) u[q] = g[q] * w[i * V + q];
      } else if (p.weight && c < p.cols) {
        if (wvec) {
#pragma unroll
          for (int q = 0; q < V; q += 4) {
            const float4 w = __ldg(reinterpret_cast<const float4*>(p.weight + c + q));
            u[q] = g[q] * w.x; u[q + 1] = g[q + 1] * w.y; u[q + 2] = g[q + 2] * w.z; u[q + 3] = g[q + 3] * w.w;
          }
        } else {
#pragma unroll
          for (int q = 0; q < V; ++q) u[q] = !SHIFT || inside(c + q) ? g[q] * __ldg(p.weight + c + q) : 0.f;
        }
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q) u[q] = g[q];       // columns past the end: g = 0
      }
    };
    int stage = 0;
    for (int a = 0; a < (kRing > 1 ? kRing - 1 : 1); ++a) ask(row + a * step, a);
    for (; row < p.rows; row += step) {
      const float mean = next_mean, rstd = next_rstd;
      if (kRing > 1) ask(row + (kRing - 1) * step, stage == 0 ? kRing - 1 : stage - 1);
      if (row + step < p.rows) fetch_stats(row + step);
      async_wait<(kRing > 1 ? kRing - 1 : 0)>();
      const uint4* from = ring + stage * 2 * kWords * kBlock + threadIdx.x;
      float s[2] = {0.f, 0.f};
      float held_n[kHold ? kWords : 1][V], held_u[kHold ? kWords : 1][V];
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        float lone_n[V], lone_u[V], g[V];
        float (&n)[V] = kHold ? held_n[kHold ? i : 0] : lone_n;
        float (&u)[V] = kHold ? held_u[kHold ? i : 0] : lone_u;
        vector_of(from, i, mean, rstd, n, g, u);
#pragma unroll
        for (int q = 0; q < V; ++q) {
          dw[i * V + q] = fmaf(g[q], n[q], dw[i * V + q]);
          db[i * V + q] += g[q];
          s[0] += u[q];
          s[1] = fmaf(u[q], n[q], s[1]);
        }
      }
      if (p.out) {
        group_sum<WARPS>(s, buf[slot], group, wg, bar);
        slot ^= 1;
        const float mu = s[0] * inv_n, mun = s[1] * inv_n;
        T* out = static_cast<T*>(p.out) + row * p.ldo;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
          float lone_n[V], lone_u[V], g[V];
          float (&n)[V] = kHold ? held_n[kHold ? i : 0] : lone_n;
          float (&u)[V] = kHold ? held_u[kHold ? i : 0] : lone_u;
          if (!kHold) vector_of(from, i, mean, rstd, n, g, u);
#pragma unroll
          for (int q = 0; q < V; ++q) u[q] = rstd * (u[q] - mu - n[q] * mun);
          const int c = column(i * V);
          if constexpr (SHIFT) ShiftedSlots<T, kPT>::store(out, p.cols, c, u);
          else if (c < p.cols) *reinterpret_cast<uint4*>(out + c) = Elem<T>::pack(u);
        }
      }
      if (kRing == 1) ask(row + step, 0);              // the thread has read its slots for the last time
      stage = stage + 1 >= kRing ? 0 : stage + 1;
    }
  } else {
    RowRegs<T, kPT> next_x, next_g;
    auto fetch = [&](long long r) {
      next_x.fetch(static_cast<const T*>(p.X) + r * p.ldx, p.cols, t, kThreads);
      next_g.fetch(static_cast<const T*>(p.dY) + r * p.lddy, p.cols, t, kThreads);
    };
    if (row < p.rows) fetch(row);
    for (; row < p.rows; row += step) {
      float x[kPT], g[kPT];
      next_x.get(x);
      next_g.get(g);
      const float mean = next_mean, rstd = next_rstd;
      if (row + step < p.rows) {
        fetch(row + step);
        fetch_stats(row + step);
      }
      float s[2] = {0.f, 0.f};
      {
        float w[kPT];                                  // from L1: registers are short here
        load_params<T, kPT, VEC>(p.weight, 1.f, p.cols, t, kThreads, w);
#pragma unroll
        for (int i = 0; i < kPT; ++i) {
          x[i] = (x[i] - mean) * rstd;                 // n; columns past the end have g = 0
          dw[i] = fmaf(g[i], x[i], dw[i]);
          db[i] += g[i];
          g[i] *= w[i];
          s[0] += g[i];
          s[1] = fmaf(g[i], x[i], s[1]);
        }
      }
      if (!p.out) continue;
      group_sum<WARPS>(s, buf[slot], group, wg, bar);
      slot ^= 1;
      const float mu = s[0] * inv_n, mun = s[1] * inv_n;
#pragma unroll
      for (int i = 0; i < kPT; ++i) g[i] = rstd * (g[i] - mu - x[i] * mun);
      store_row<T, kPT, VEC>(static_cast<T*>(p.out) + row * p.ldo, p.cols, t, kThreads, g);
    }
  }
  if (!p.part) return;
  float* pw = p.part + (long long)blockIdx.x * 2 * p.cols;
  if constexpr (kGroups == 1) {
#pragma unroll
    for (int i = 0; i < kPT; ++i) {
      const int c = column(i);
      if (inside(c)) { pw[c] = dw[i]; pw[p.cols + c] = db[i]; }
    }
  } else {                                             // the block's groups first, in order
    __shared__ float sum[2][kThreads * kPT];
    for (int g = 0; g < kGroups; ++g) {
      if (g == group) {
#pragma unroll
        for (int i = 0; i < kPT; ++i) {
          const int at = SHIFT ? column(i) : i * kThreads + t;       // shifted groups hold their columns elsewhere
          if (SHIFT && !inside(at)) continue;
          sum[0][at] = (g ? sum[0][at] : 0.f) + dw[i];
          sum[1][at] = (g ? sum[1][at] : 0.f) + db[i];
        }
      }
      __syncthreads();
    }
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < kPT; ++i) {
        const int c = column(i), at = SHIFT ? c : i * kThreads + t;
        if (inside(c)) { pw[c] = sum[0][at]; pw[p.cols + c] = sum[1][at]; }
      }
    }
  }
}

// Long rows: dx in two passes; dw and db by column tiles.
template <typename T>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(NormParams p) {
  __shared__ float buf[64];
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.X) + row * p.ldx;
  const T* dy = static_cast<const T*>(p.dY) + row * p.lddy;
  T* dx = static_cast<T*>(p.out) + row * p.ldo;
  const float mean = p.mean_in[row], rstd = p.rstd_in[row];
  const int t = threadIdx.x;
  float s[2] = {0.f, 0.f};
  for (int c = t; c < p.cols; c += 1024) {
    const float u = Elem<T>::get(dy[c]) * (p.weight ? p.weight[c] : 1.f);
    s[0] += u;
    s[1] = fmaf(u, (Elem<T>::get(x[c]) - mean) * rstd, s[1]);
  }
  group_sum<32>(s, buf, 0, t >> 5, 0);
  const float mu = s[0] / (float)p.cols, mun = s[1] / (float)p.cols;
  for (int c = t; c < p.cols; c += 1024) {
    const float u = Elem<T>::get(dy[c]) * (p.weight ? p.weight[c] : 1.f);
    dx[c] = Elem<T>::put(rstd * (u - mu - (Elem<T>::get(x[c]) - mean) * rstd * mun));
  }
}
// grid (ceil(cols / 32), blocks); thread (lane, warp): column lane, every eighth row of the block's chunk.
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormParams p, int rows_per_block) {
  __shared__ float sum[2][8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  const long long r_end = min((long long)p.rows, (long long)(blockIdx.y + 1) * rows_per_block);
  float dw = 0.f, db = 0.f;
  if (c < p.cols)
    for (long long r = (long long)blockIdx.y * rows_per_block + warp; r < r_end; r += 8) {
      const float g = Elem<T>::get(static_cast<const T*>(p.dY)[r * p.lddy + c]);
      const float n = (Elem<T>::get(static_cast<const T*>(p.X)[r * p.ldx + c]) - p.mean_in[r]) * p.rstd_in[r];
      dw = fmaf(g, n, dw);
      db += g;
    }
  sum[0][warp][lane] = dw;
  sum[1][warp][lane] = db;
  __syncthreads();
  if (warp < 2 && c < p.cols) {
    float s = sum[warp][0][lane];
    for (int w = 1; w < 8; ++w) s += sum[warp][w][lane];
    p.part[((long long)blockIdx.y * 2 + warp) * p.cols + c] = s;
  }
}

// Adds the blocks' partial rows in a fixed order: 32 columns a block, 16 warps over the partial rows, eight
// loads of a thread in flight.  grid (ceil(cols / 32), 2): dw, db.
__global__ void __launch_bounds__(512)
norm_parts_kernel(const float* __restrict__ part, int parts, int cols, float* dweight, float* dbias) {
  __shared__ float sum[16][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  float s = 0.f;
  if (c < cols) {
    const float* src = part + (long long)blockIdx.y * cols + c;
    const long long ld = 2ll * cols;
#pragma unroll 8
    for (int i = warp; i < parts; i += 16) s += src[i * ld];
  }
  sum[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    for (int w = 1; w < 16; ++w) s += sum[w][lane];
    out[c] = s;
  }
}

}  // namespace sgc

namespace {

using sgc::NormParams;

int done(sgemm_cube_ctx* h) {
  h->launches++;
  return cudaGetLastError() == cudaSuccess ? SGEMM_CUBE_OK : SGEMM_CUBE_CUDA_ERROR;
}

// Blocks of a persistent kernel: one per `groups` rows, at most what is resident at once.  `KERNEL` is asked for its
// occupancy once a device.
template <auto KERNEL>
int persistent_blocks(sgemm_cube_ctx* h, int threads, size_t smem, int rows, int period, int groups, int* blocks) {
  static std::atomic<int> known[64];                   // blocks an SM, per device; 0: not asked yet
  std::atomic<int>* entry = h->device < 64 ? &known[h->device] : nullptr;
  auto kernel = KERNEL;
  int per_sm = entry ? entry->load(std::memory_order_relaxed) : 0;
  if (per_sm == 0 && ((smem > 32 * 1024 &&                              // (48 KB with the static arrays is where the limit starts)
       cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) ||
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess || per_sm < 1)) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  if (entry) entry->store(per_sm, std::memory_order_relaxed);
  const long long want = ((long long)rows + groups - 1) / groups, cap = (long long)per_sm * h->sm_count;
  const long long turn = period > groups ? period / groups : 1;      // blocks that take `period` rows, or more
  *blocks = (int)(want <= cap ? want : (cap > turn ? cap / turn * turn : turn));
  return SGEMM_CUBE_OK;
}

template <typename T, int WARPS, bool VEC>
int forward_rows(sgemm_cube_ctx* h, const NormParams& p, cudaStream_t st) {
  constexpr int groups = WARPS >= 8 ? 1 : 8 / WARPS, threads = WARPS > 8 ? WARPS * 32 : 256;
  int blocks = 0;
  constexpr size_t smem = sgc::kSlotBytes<T, WARPS, VEC, 1>;
  const int rc = persistent_blocks<sgc::norm_forward_kernel<T, WARPS, VEC>>(h, threads, smem, p.rows, 1, groups, &blocks);
  if (rc) return rc;
  sgc::norm_forward_kernel<T, WARPS, VEC><<<(unsigned)blocks, threads, smem, st>>>(p);
  return done(h);
}
template <typename T, bool VEC>
int forward_typed(sgemm_cube_ctx* h, const NormParams& p, cudaStream_t st) {
  if (p.cols <= 1 * 32 * sgc::kPT) return forward_rows<T, 1, VEC>(h, p, st);
  if (p.cols <= 2 * 32 * sgc::kPT) return forward_rows<T, 2, VEC>(h, p, st);
  if (p.cols <= 4 * 32 * sgc::kPT) return forward_rows<T, 4, VEC>(h, p, st);
  if (p.cols <= 8 * 32 * sgc::kPT) return forward_rows<T, 8, VEC>(h, p, st);
  if (p.cols <= 16 * 32 * sgc::kPT) return forward_rows<T, 16, VEC>(h, p, st);
  if (p.cols <= 32 * 32 * sgc::kPT) return forward_rows<T, 32, VEC>(h, p, st);
  sgc::norm_forward_long_kernel<T><<<(unsigned)p.rows, 1024, 0, st>>>(p);
  return done(h);
}

template <typename T, int WARPS, sgc::RowAccess ACCESS>
int backward_rows(sgemm_cube_ctx* h, NormParams p, float* dweight, float* dbias, cudaStream_t st) {
  constexpr int groups = WARPS >= 8 ? 1 : 8 / WARPS, threads = WARPS > 8 ? WARPS * 32 : 256;
  int blocks = 0;
  constexpr size_t smem = sgc::kSlotBytes<T, WARPS, ACCESS != sgc::kElements, 2>;
  int rc = persistent_blocks<sgc::norm_backward_kernel<T, WARPS, ACCESS>>(h, threads, smem, p.rows, p.period, groups, &blocks);
  if (rc) return rc;
  if (dweight || dbias) {
    rc = grow(h, &h->part_ws, &h->part_ws_bytes, (size_t)blocks * 2 * p.cols * 4, st);
    if (rc) return rc;
    p.part = static_cast<float*>(h->part_ws);
  }
  sgc::norm_backward_kernel<T, WARPS, ACCESS><<<(unsigned)blocks, threads, smem, st>>>(p);
  rc = done(h);
  if (rc || !p.part) return rc;
  sgc::norm_parts_kernel<<<dim3((unsigned)((p.cols + 31) / 32), 2), 512, 0, st>>>(p.part, blocks, p.cols, dweight, dbias);
  return done(h);
}
template <typename T>
int backward_long(sgemm_cube_ctx* h, NormParams p, float* dweight, float* dbias, cudaStream_t st) {
  int rc = SGEMM_CUBE_OK;
  if (dweight || dbias) {                              // before dx, which may overwrite dy
    const int tiles = (p.cols + 31) / 32;
    int blocks = (16 * h->sm_count + tiles - 1) / tiles;
    if (blocks > (p.rows + 31) / 32) blocks = (p.rows + 31) / 32;
    const int per = (p.rows + blocks - 1) / blocks;
    blocks = (p.rows + per - 1) / per;
    if ((rc = grow(h, &h->part_ws, &h->part_ws_bytes, (size_t)blocks * 2 * p.cols * 4, st))) return rc;
    p.part = static_cast<float*>(h->part_ws);
    sgc::norm_columns_kernel<T><<<dim3((unsigned)tiles, (unsigned)blocks), 256, 0, st>>>(p, per);
    if ((rc = done(h))) return rc;
    sgc::norm_parts_kernel<<<dim3((unsigned)tiles, 2), 512, 0, st>>>(p.part, blocks, p.cols, dweight, dbias);
    if ((rc = done(h))) return rc;
  }
  if (!p.out) return rc;
  sgc::norm_backward_long_kernel<T><<<(unsigned)p.rows, 1024, 0, st>>>(p);
  return done(h);
}
template <typename T, sgc::RowAccess ACCESS>
int backward_as(sgemm_cube_ctx* h, const NormParams& p, float* dw, float* db, cudaStream_t st) {
  if (p.cols <= 1 * 32 * sgc::kPT) return backward_rows<T, 1, ACCESS>(h, p, dw, db, st);
  if (p.cols <= 2 * 32 * sgc::kPT) return backward_rows<T, 2, ACCESS>(h, p, dw, db, st);
  if (p.cols <= 4 * 32 * sgc::kPT) return backward_rows<T, 4, ACCESS>(h, p, dw, db, st);
  if (p.cols <= 8 * 32 * sgc::kPT) return backward_rows<T, 8, ACCESS>(h, p, dw, db, st);
  if (p.cols <= 16 * 32 * sgc::kPT) return backward_rows<T, 16, ACCESS>(h, p, dw, db, st);
  if (p.cols <= 32 * 32 * sgc::kPT) return backward_rows<T, 32, ACCESS>(h, p, dw, db, st);
  return backward_long<T>(h, p, dw, db, st);
}

template <typename T>
int backward_typed(sgemm_cube_ctx* h, NormParams p, float* dw, float* db, cudaStream_t st) {
  constexpr int v = sgc::Elem<T>::kVec;
  p.period = 1;
  if (sgc::rows_take_vectors(p.X, p.ldx, p.cols, sizeof(T)) && sgc::rows_take_vectors(p.dY, p.lddy, p.cols, sizeof(T)) &&
      (!p.out || sgc::rows_take_vectors(p.out, p.ldo, p.cols, sizeof(T))))
    return backward_as<T, sgc::kAligned>(h, p, dw, db, st);
  // All rows start alike, and what the first vector lays in front costs no more warps a row.
  const auto start = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16; };
  bool alike = start(p.X) == start(p.dY) && (p.ldx - p.lddy) % v == 0;
  if (p.out) alike = alike && start(p.X) == start(p.out) && (p.ldx - p.ldo) % v == 0;
  int limit = 32 * sgc::kPT;
  while (limit < p.cols) limit *= 2;
  if (alike && p.cols >= v && p.cols + v - 1 <= limit && limit <= 32 * 32 * sgc::kPT) {
    if (p.ldx % v) p.period = v;
    return backward_as<T, sgc::kShifted>(h, p, dw, db, st);
  }
  return backward_as<T, sgc::kElements>(h, p, dw, db, st);
}

size_t elem_size(int dtype) { return dtype == SGEMM_CUBE_F32 ? 4 : 2; }
bool bad_dtype(int dtype) { return dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16; }

}  // namespace

extern "C" {

int sgemm_cube_layer_norm(sgemm_cube_handle h, int rows, int cols, int dtype, const void* X, int64_t ldx,
                          const float* weight, const float* bias, float eps, void* Y, int64_t ldy, float* mean,
                          float* rstd, void* stream) {
  if (!h || bad_dims(rows, cols) || cols < 1 || bad_dtype(dtype) || !(eps >= 0.f) || ldx < cols || ldy < cols)
    return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!X || !Y || misplaced(elem_size(dtype), X, Y) || misplaced(4, weight, bias, mean, rstd)) return SGEMM_CUBE_INVALID_ARG;
  if (X == Y && ldx != ldy && rows > 1) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  NormParams p;
  memset(&p, 0, sizeof(p));
  p.rows = rows; p.cols = cols;
  p.X = X; p.ldx = ldx;
  p.out = Y; p.ldo = ldy;
  p.weight = weight; p.bias = bias; p.eps = eps;
  p.mean = mean; p.rstd = rstd;
  const size_t e = elem_size(dtype);
  const bool vec = sgc::rows_take_vectors(X, ldx, cols, e) && sgc::rows_take_vectors(Y, ldy, cols, e);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SGEMM_CUBE_F32) return vec ? forward_typed<float, true>(h, p, st) : forward_typed<float, false>(h, p, st);
  if (dtype == SGEMM_CUBE_F16) return vec ? forward_typed<__half, true>(h, p, st) : forward_typed<__half, false>(h, p, st);
  return vec ? forward_typed<__nv_bfloat16, true>(h, p, st) : forward_typed<__nv_bfloat16, false>(h, p, st);
}

int sgemm_cube_layer_norm_backward(sgemm_cube_handle h, int rows, int cols, int dtype, const void* dY, int64_t lddy,
                                   const void* X, int64_t ldx, const float* weight, const float* mean,
                                   const float* rstd, void* dX, int64_t lddx, float* dweight, float* dbias,
                                   void* stream) {
  if (!h || bad_dims(rows, cols) || cols < 1 || bad_dtype(dtype) || ldx < cols || lddy < cols || (dX && lddx < cols))
    return SGEMM_CUBE_INVALID_ARG;
  if (rows > 0 && (!dY || !X || !mean || !rstd)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(elem_size(dtype), dY, X, dX) || misplaced(4, weight, mean, rstd, dweight, dbias)) return SGEMM_CUBE_INVALID_ARG;
  if (dX == dY && lddx != lddy && rows > 1) return SGEMM_CUBE_INVALID_ARG;
  if (!dX && !dweight && !dbias) return SGEMM_CUBE_OK;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    for (float* p : {dweight, dbias})
      if (p && cudaMemsetAsync(p, 0, (size_t)cols * 4, st) != cudaSuccess) {
        cudaGetLastError();
        return SGEMM_CUBE_CUDA_ERROR;
      }
    return SGEMM_CUBE_OK;
  }
  NormParams p;
  memset(&p, 0, sizeof(p));
  p.rows = rows; p.cols = cols;
  p.X = X; p.ldx = ldx;
  p.dY = dY; p.lddy = lddy;
  p.out = dX; p.ldo = lddx;
  p.weight = weight;
  p.mean_in = mean; p.rstd_in = rstd;
  if (dtype == SGEMM_CUBE_F32) return backward_typed<float>(h, p, dweight, dbias, st);
  if (dtype == SGEMM_CUBE_F16) return backward_typed<__half>(h, p, dweight, dbias, st);
  return backward_typed<__nv_bfloat16>(h, p, dweight, dbias, st);
}

}  // extern "C"
