// Log probabilities of given tokens under softmax(scale * x), with entropy and the largest alternatives, and
// the gradient of the logits (contracts: include/sgemm_cube.h).
//
// Forward, one pass over a row with a running maximum m and, relative to it, the sums
//   Z = sum exp(scale (x - m)),   S = sum exp(scale (x - m)) scale (x - m);
// when m grows to m' both shrink by r = exp(scale (m - m')) and S also takes r scale (m - m') Z.  Then
//   lse = scale m + log Z,   log p_t = scale (x_t - m) - log Z,   H = log Z - S / Z.
// Bound by reading the logits once (2048 x 65536 FP32 85 us, 6.3 TB/s); with 16-bit logits by the instructions as much as
// by waiting for the loads, so the instructions are counted (1000 x 50001 BF16 24 us, 4.2 TB/s; 31 with eight
// alternatives, half of the issue slots used).
// Exponentials run in base 2, a = scale log2 e: t = x a - M, M = fl(m a), is one FMA; what the rounding of M does to
// every term alike (at most 1 while |M| < 2^25) is taken out of a thread's sums at the end.  Logits are cut at -2^60
// (2^-30 <= scale <= 2^30), so that -inf gives a weight of zero and no 0 * inf.  A thread whose largest logit has
// |m a| >= 2^25 (masked with the type's lowest value, or a large scale), or had one before that m does not dwarf, sums its
// columns again in the form (x - m) a, which neither overflows nor is cut.
#include <type_traits>

#include "ctx.cuh"
#include "elements.cuh"

namespace sgc {

constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kTopMax = 32;
constexpr int kCandidates = 256;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kNoWeight = -160.f;      // 2^-160 is zero in FP32: exponents are cut there where they are factors
constexpr float kLowestLogit = -1152921504606846976.f;    // -2^60
constexpr float kFarTerm = 33554432.f;                    // 2^25, so near logits lie within 2^55 of zero, well above the cut

// 2^t, zero below 2^-126: in a sum such weights are nothing beside the row's largest, which is 1, and keeping them
// takes three more instructions.
__device__ __forceinline__ float ex2(float t) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}
// 2^t down to the subnormal numbers, for the gradient, where each element stands alone.
__device__ __forceinline__ float ex2_gradual(float t) {
  float e;
  asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(t));
  return e;
}
__device__ __forceinline__ uint32_t cluster_rank_x() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_address(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(a) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  return a;
}
__device__ __forceinline__ float remote_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t remote_u64(uint32_t a) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

struct LogprobParams {
  int rows, vocab;
  const void* X;
  long long ld;
  const long long* tokens;
  float scale, a;                // a = scale log2 e
  float* logp;
  float* entropy;
  float* stats;
  int top_k;
  float* top_logp;
  long long* top_index;
};

// Two FP32 values in one register pair: the packed instructions round each like the scalar ones.
struct Two {
  uint64_t p;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two t;
  asm("mov.b64 %0, {%1, %2};" : "=l"(t.p) : "f"(a), "f"(b));
  return t;
}
__device__ __forceinline__ void parts_of(Two t, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(t.p)); }
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two c;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(c.p) : "l"(a.p), "l"(b.p));
  return c;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two c;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(c.p) : "l"(a.p), "l"(b.p));
  return c;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.p) : "l"(a.p), "l"(b.p), "l"(c.p));
  return d;
}

// Running sums of a part of a row; S in base-2 units.
struct Running {
  float m, Z, S;
};
__device__ __forceinline__ void join(Running& r, Running o, float a) {
  if (o.m > r.m) { const Running x = r; r = o; o = x; }
  // r has the larger m; an -inf part has empty sums, or NaN ones, which stay
  if (o.m == -INFINITY) { r.Z += o.Z; r.S += o.S; return; }
  const float d = (o.m - r.m) * a;
  const float f = ex2(d);
  r.Z = fmaf(o.Z, f, r.Z);
  r.S += f * fmaf(fmaxf(d, kNoWeight), o.Z, o.S);
}
// join over groups of N neighbouring lanes; the first lane of each ends up with the sum
template <int N>
__device__ __forceinline__ void join_lanes(Running& r, float a) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) {
    Running other;
    other.m = __shfl_down_sync(0xffffffffu, r.m, o);
    other.Z = __shfl_down_sync(0xffffffffu, r.Z, o);
    other.S = __shfl_down_sync(0xffffffffu, r.S, o);
    join(r, other, a);
  }
}

// The same for one thread while it goes through its columns: even and odd elements apart, so that the packed
// instructions apply.  M = fl(m a), 0 while m is far from zero: -inf and other cut logits then weigh nothing.
struct ThreadSums {
  float m, M;
  Two Z, S;
  bool lost;               // a largest logit far from zero was followed by a near one that does not dwarf it
  static __device__ __forceinline__ bool near(float m, float a) { return fabsf(m * a) < kFarTerm; }
  __device__ __forceinline__ void raise(float top, float a) {            // top > m
    const float to = near(top, a) ? top * a : 0.f;
    const float d = fmaxf(M - to, kNoWeight);
    const float f = near(m, a) ? ex2(d) : 0.f;         // 0 times the sums, not 0: NaN stays
    lost = lost || (!near(m, a) && (m - top) * a > kNoWeight);
    S = fma2(two(d, d), Z, S) * two(f, f);
    Z = Z * two(f, f);
    m = top;
    M = to;
  }
  // x >= kLowestLogit or NaN
  __device__ __forceinline__ void add(float x0, float x1, Two a, Two minus_m) {
    const Two t = fma2(two(x0, x1), a, minus_m);
    float t0, t1;
    parts_of(t, t0, t1);
    const Two e = two(ex2(t0), ex2(t1));
    Z = Z + e;
    S = fma2(e, t, S);
  }
  // with the rounding of M taken out: t is too large by lo = m a - M
  __device__ __forceinline__ Running sum(float a) const {
    float z0, z1, s0, s1;
    parts_of(Z, z0, z1);
    parts_of(S, s0, s1);
    const float lo = near(m, a) ? fmaf(m, a, -M) : 0.f;
    const float f = ex2(-lo), z = z0 + z1;
    return Running{m, z * f, fmaf(-lo, z, s0 + s1) * f};
  }
};
// A logit as ThreadSums takes it; NaN stays.
__device__ __forceinline__ float cut_logit(float x) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(kLowestLogit));
  return y;
}
// The same for a word of elements, where the type allows it (FP16 has no -2^60: its elements are cut one by one).
template <typename T>
__device__ __forceinline__ uint32_t cut_word(uint32_t w) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const uint32_t low = 0xDD80DD80u;                                       // -2^60 twice
    const __nv_bfloat162 m =
        __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&w), *reinterpret_cast<const __nv_bfloat162*>(&low));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  return w;
}

// The largest of the elements in a word, or of two words element by element; a NaN loses against a number.
template <typename T>
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b) {
  if constexpr (sizeof(T) == 4) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  } else if constexpr (std::is_same<T, __half>::value) {
    const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  } else {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
}
template <typename T>
__device__ __forceinline__ float max_of_word(uint32_t w) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(w);
  } else if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return fmaxf(f.x, f.y);
  } else {
    return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
}

// Four 32-bit words of -inf elements.
template <typename T>
__device__ __forceinline__ uint4 no_logits() {
  const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : (std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u);
  return make_uint4(w, w, w, w);
}

// Order of the alternatives: larger logit first, then the lower column, as one unsigned number; 0 is none.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t col) {
  const uint32_t u = __float_as_uint(x + 0.f);                        // -0 counts as 0
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return x == x ? ((uint64_t)o << 32) | (0xFFFFFFFFu - col) : 0ull;
}
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ uint32_t key_column(uint64_t k) { return 0xFFFFFFFFu - (uint32_t)k; }

// Bitonic networks over the 32 lanes, descending.
__device__ __forceinline__ uint64_t lane_exchange(uint64_t k, int stride, bool keep_max) {
  const uint64_t o = __shfl_xor_sync(0xffffffffu, k, stride);
  return keep_max ? (k > o ? k : o) : (k < o ? k : o);
}
__device__ __forceinline__ uint64_t sort_lanes(uint64_t k, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int stride = size >> 1; stride > 0; stride >>= 1)
      k = lane_exchange(k, stride, ((lane & stride) == 0) == ((lane & size) == 0 || size == 32));
  return k;
}
// Two descending lists, the second given in reverse: the 32 largest of both, descending.
__device__ __forceinline__ uint64_t merge_lanes(uint64_t a, uint64_t b_reversed, int lane) {
  uint64_t k = a > b_reversed ? a : b_reversed;
#pragma unroll
  for (int stride = 16; stride > 0; stride >>= 1) k = lane_exchange(k, stride, (lane & stride) == 0);
  return k;
}

// A block's columns [0, n) of a row, x pointing at the first: up to one vector of single elements in front of
// the first 16-byte boundary, whole vectors, and the rest.  Thread t takes element t of the front, the vectors
// t, t + threads, ... and element t of the rest.
template <typename T>
struct Piece {
  const T* x;
  int n, head, vecs, tail;
  __device__ __forceinline__ Piece(const T* p, int count) : x(p), n(count) {
    constexpr int V = Elem<T>::kVec;
    const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    head = min(n, (V - off) % V);
    vecs = (n - head) / V;
    tail = n - head - vecs * V;
  }
  __device__ __forceinline__ const uint4* vec(int v) const { return reinterpret_cast<const uint4*>(x + head) + v; }
  __device__ __forceinline__ int owner(int c) const {                     // the thread that takes column c
    constexpr int V = Elem<T>::kVec;
    if (c < head) return c;
    c -= head;
    return c < vecs * V ? c / V % kLpThreads : c - vecs * V;
  }
};

// Calls f(key) for the columns above `bound` that the owners of the first `count` keys of `list` hold, these keys
// themselves left out; the work is spread over `threads` threads, which all make the same calls (key 0: nothing
// there), so that f may use the whole warp.
template <typename T, typename F>
__device__ __forceinline__ void for_columns_above(const Piece<T>& piece, int c0, const uint64_t* list, int count,
                                                  uint64_t bound, int t, int threads, F f) {
  constexpr int V = Elem<T>::kVec;
  auto call = [&](float x, int c, uint64_t own, bool in) {
    const uint64_t k = in ? order_key(x, (uint32_t)(c0 + c)) : 0ull;
    f(k > bound && k != own ? k : 0ull);
  };
  for (int i0 = 0; i0 < 2 * count; i0 += threads) {      // the elements in front and at the end
    const int i = i0 + t;
    const uint64_t own = i < 2 * count ? list[i >> 1] : 0ull;
    const int w = own ? piece.owner((int)key_column(own) - c0) : 0;
    const int c = (i & 1) ? piece.head + piece.vecs * V + w : w;
    const bool in = own != 0 && w < ((i & 1) ? piece.tail : piece.head);
    call(in ? Elem<T>::get(piece.x[c]) : 0.f, c, own, in);
  }
  const int each = (piece.vecs + kLpThreads - 1) / kLpThreads;
  for (int i0 = 0; i0 < count * each; i0 += threads) {
    const int i = i0 + t, j = i / each;
    const uint64_t own = j < count ? list[j] : 0ull;
    const int v = (own ? piece.owner((int)key_column(own) - c0) : 0) + (i - j * each) * kLpThreads;
    const bool in = own != 0 && v < piece.vecs;
    float e[V];
    Elem<T>::unpack(in ? __ldg(piece.vec(v)) : no_logits<T>(), e);
#pragma unroll
    for (int q = 0; q < V; ++q) call(e[q], piece.head + v * V + q, own, in);
  }
}

// A thread's sums where its largest logit m, or an earlier one that still counts, is far from zero.
template <typename T>
__device__ __forceinline__ Running sum_far(const Piece<T>& piece, int t, float m, float a) {
  constexpr int V = Elem<T>::kVec;
  Running r{m, 0.f, 0.f};
  auto add = [&](float x) {
    const float d = (x - m) * a;
    const float e = ex2(d);
    r.Z += e;
    r.S = fmaf(e, fmaxf(d, kNoWeight), r.S);
  };
  if (t < piece.head) add(Elem<T>::get(piece.x[t]));
  for (int v = t; v < piece.vecs; v += kLpThreads) {
    float e[V];
    Elem<T>::unpack(__ldg(piece.vec(v)), e);
#pragma unroll
    for (int q = 0; q < V; ++q) add(e[q]);
  }
  if (t < piece.tail) add(Elem<T>::get(piece.x[piece.head + piece.vecs * V + t]));
  return r;
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads) token_logprobs_kernel(LogprobParams p) {
  constexpr int V = Elem<T>::kVec, U = 4;                // 64 bytes of a thread are a batch, another is in flight
  __shared__ Running parts[kLpWarps];
  __shared__ Running block_sum;
  __shared__ uint64_t list[TOP ? kLpWarps : 1][32];
  __shared__ uint64_t more[TOP ? kCandidates : 1];
  __shared__ uint64_t best[32];
  __shared__ int more_count;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const uint32_t ranks = cluster_size(), rank = cluster_rank_x();
  const long long row = blockIdx.x / ranks;
  const T* x_row = static_cast<const T*>(p.X) + row * p.ld;
  const long long per = ((long long)p.vocab + ranks - 1) / ranks;
  const int c0 = (int)min((long long)p.vocab, rank * per), c1 = (int)min((long long)p.vocab, c0 + per);
  const Piece<T> piece(x_row + c0, c1 - c0);

  // the target's logit, long before it is needed
  long long target = -1;
  float target_logit = 0.f;
  if (t == 0 && rank == 0 && p.logp) {
    target = p.tokens[row];
    if (target >= 0 && target < p.vocab) target_logit = Elem<T>::get(x_row[target]);
  }

  ThreadSums r{-INFINITY, 0.f, two(0.f, 0.f), two(0.f, 0.f), false};
  const Two a2 = two(p.a, p.a);
  auto add_single = [&](float x) { r.add(cut_logit(x), kLowestLogit, a2, two(-r.M, -r.M)); };
  int at = -1;                                           // where m was met: -1 nowhere, 0 front, 1 + batch, then the rest
  const int batches = (piece.vecs + kLpThreads * U - 1) / (kLpThreads * U);
  uint4 next[U];
  auto fetch = [&](int b, uint4 (&raw)[U]) {             // the vectors of batch b, -inf past the end
    const int v0 = b * kLpThreads * U + t;
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = v0 + u * kLpThreads < piece.vecs ? __ldg(piece.vec(v0 + u * kLpThreads)) : no_logits<T>();
  };
  fetch(0, next);
  if (t < piece.head) {
    const float x = Elem<T>::get(piece.x[t]);
    if (x > r.m) { r.raise(x, p.a); at = 0; }
    add_single(x);
  }
  for (int b = 0; b < batches; ++b) {
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
    if (b + 1 < batches) fetch(b + 1, next);
    uint32_t w = raw[0].x;
#pragma unroll
    for (int u = 0; u < U; ++u)
      w = max_words<T>(w, max_words<T>(max_words<T>(raw[u].x, raw[u].y), max_words<T>(raw[u].z, raw[u].w)));
    const float top = max_of_word<T>(w);
    if (top > r.m) { r.raise(top, p.a); at = 1 + b; }
    const Two minus = two(-r.M, -r.M);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[V];
      raw[u].x = cut_word<T>(raw[u].x); raw[u].y = cut_word<T>(raw[u].y);
      raw[u].z = cut_word<T>(raw[u].z); raw[u].w = cut_word<T>(raw[u].w);
      Elem<T>::unpack(raw[u], v);
      constexpr bool cut = std::is_same<T, __nv_bfloat16>::value;
#pragma unroll
      for (int q = 0; q < V; q += 2)
        r.add(cut ? v[q] : cut_logit(v[q]), cut ? v[q + 1] : cut_logit(v[q + 1]), a2, minus);
    }
  }
  if (t < piece.tail) {
    const float x = Elem<T>::get(piece.x[piece.head + piece.vecs * V + t]);
    if (x > r.m) { r.raise(x, p.a); at = 1 + batches; }
    add_single(x);
  }
  Running sum = r.sum(p.a);
  if ((r.lost || !ThreadSums::near(r.m, p.a)) && r.m != -INFINITY) sum = sum_far(piece, t, r.m, p.a);   // NaN for +inf

  if constexpr (TOP) {
    // The k largest of the threads' maxima bound the k largest elements from below, and hold every thread
    // that owns one of them: an element among the k largest is not above its thread's maximum.
    int c = -1;                                          // column of the own maximum, the lowest if it is met again
    if (at > 0 && at <= batches) {
      uint4 raw[U];
      fetch(at - 1, raw);
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        float e[V];
        Elem<T>::unpack(raw[u], e);
#pragma unroll
        for (int q = V - 1; q >= 0; --q)
          if (e[q] == r.m) c = piece.head + ((at - 1) * kLpThreads * U + t + u * kLpThreads) * V + q;
      }
    } else if (at > batches) {
      c = piece.head + piece.vecs * V + t;
    } else if (t < piece.head) {                         // in front, or nothing above -inf: the first column
      c = t;
    } else if (t < piece.vecs) {
      c = piece.head + t * V;
    } else if (t < piece.tail) {
      c = piece.head + piece.vecs * V + t;
    }
    if (t == 0) more_count = 0;
    list[warp][lane] = sort_lanes(c >= 0 ? order_key(r.m, (uint32_t)(c0 + c)) : 0ull, lane);
    __syncthreads();
    for (int s = kLpWarps / 2; s > 0; s >>= 1) {         // warp w takes over list w + s, which nobody else reads
      if (warp < s) list[warp][lane] = merge_lanes(list[warp][lane], list[warp + s][31 - lane], lane);
      __syncthreads();
    }
    const uint64_t bound = list[0][p.top_k - 1];
    // what else these threads own above the bound
    for_columns_above(piece, c0, list[0], p.top_k, bound, t, kLpThreads, [&](uint64_t k) {
      if (k) {
        const int slot = atomicAdd(&more_count, 1);
        if (slot < kCandidates) more[slot] = k;
      }
    });
    __syncthreads();
    if (warp == 0) {
      uint64_t k = list[0][lane];
      auto add = [&](uint64_t o) {
        o = sort_lanes(o, lane);
        k = merge_lanes(k, __shfl_sync(0xffffffffu, o, 31 - lane), lane);
      };
      if (more_count <= kCandidates) {
        for (int i = 0; i < more_count; i += 32) add(i + lane < more_count ? more[i + lane] : 0ull);
      } else {                                           // many in a few threads: straight from the row
        for_columns_above(piece, c0, list[0], p.top_k, bound, lane, 32, [&](uint64_t o) {
          if (__any_sync(0xffffffffu, o != 0)) add(o);
        });
      }
      best[lane] = k;
    }
  }

  join_lanes<32>(sum, p.a);
  if (lane == 0) parts[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    sum = lane < kLpWarps ? parts[lane] : Running{-INFINITY, 0.f, 0.f};
    join_lanes<kLpWarps>(sum, p.a);
    if (lane == 0) block_sum = sum;
  }
  if (ranks > 1) {
    cluster_meet();
    if (rank == 0 && warp == 0) {
      if (lane > 0 && lane < ranks) {
        const uint32_t a = remote_address(&block_sum, lane);
        sum = Running{remote_f32(a), remote_f32(a + 4), remote_f32(a + 8)};
      } else if (lane > 0) {
        sum = Running{-INFINITY, 0.f, 0.f};
      }
      join_lanes<8>(sum, p.a);
      if constexpr (TOP) {
        uint64_t k = best[lane], o[7];
#pragma unroll
        for (int i = 0; i < 7; ++i) o[i] = i + 1 < (int)ranks ? remote_u64(remote_address(&best[31 - lane], i + 1)) : 0ull;
#pragma unroll
        for (int i = 0; i < 7; ++i)
          if (i + 1 < (int)ranks) k = merge_lanes(k, o[i], lane);
        __syncwarp();
        best[lane] = k;
      }
    }
  }
  if (rank == 0 && warp == 0) {
    sum.m = __shfl_sync(0xffffffffu, sum.m, 0);
    sum.Z = __shfl_sync(0xffffffffu, sum.Z, 0);
    sum.S = __shfl_sync(0xffffffffu, sum.S, 0);
    const bool none = sum.m == -INFINITY && sum.Z == 0.f;  // every logit is -inf
    const float log_z = logf(sum.Z);
    if (lane == 0) {
      if (p.stats) { p.stats[2 * row] = sum.m; p.stats[2 * row + 1] = sum.Z; }
      if (p.entropy) p.entropy[row] = none ? 0.f : log_z - sum.S / sum.Z * kLn2;
      if (p.logp) {
        float lp = 0.f;
        if (target >= p.vocab) lp = NAN;
        else if (target >= 0) lp = none ? -INFINITY : (target_logit - sum.m) * p.scale - log_z;
        p.logp[row] = lp;
      }
    }
    if (TOP && lane < p.top_k) {
      const uint64_t k = best[lane];
      p.top_logp[row * p.top_k + lane] = none ? -INFINITY : (k ? (key_logit(k) - sum.m) * p.scale - log_z : NAN);
      p.top_index[row * p.top_k + lane] = k ? (long long)key_column(k) : lane;
    }
  }
  if (ranks > 1) cluster_meet();                         // a block's sums stay until the first has read them
}

struct LogprobGradParams {
  int rows, vocab;
  const void* X;
  long long ld;
  const long long* tokens;
  float scale, a;
  const float* stats;
  const float* entropy;
  const float* dlogp;
  const float* dentropy;
  void* dX;
  long long lddx;
  int chunks, vec;
};

// dx_j = e_j (A + B t_j) + [j == target] scale g with e_j = exp2(t_j), t_j = (x_j - m) a:
//   p_j = e_j / Z,  log p_j = ln2 t_j - log Z,
//   A = -scale (g + h (H - log Z)) / Z,  B = -scale h ln2 / Z      (g, h the two incoming gradients)
// Reads and writes every logit once (4096 x 65536 FP32 323 us, 6.6 TB/s; BF16 163 us, 6.6 TB/s).  A block takes chunk `blockIdx % chunks` of a row, then the same of the
// row `gridDim / chunks` further.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) token_logprobs_grad_kernel(LogprobGradParams p) {
  constexpr int V = Elem<T>::kVec, U = 16 / V;
  const int chunk = blockIdx.x % p.chunks;
  const long long per = ((p.vocab - 1) / p.chunks + 16) / 16 * 16;
  const int c0 = (int)min((long long)p.vocab, chunk * per), c1 = (int)min((long long)p.vocab, c0 + per);
  for (long long row = blockIdx.x / p.chunks; row < p.rows; row += gridDim.x / p.chunks) {
    const T* x = static_cast<const T*>(p.X) + row * p.ld;
    T* dx = static_cast<T*>(p.dX) + row * p.lddx;
    const float m = p.stats[2 * row], Z = p.stats[2 * row + 1];
    const bool none = m == -INFINITY && Z == 0.f;
    const long long target = p.dlogp ? p.tokens[row] : -1;
    float g = target >= 0 ? p.dlogp[row] : 0.f;
    if (target >= p.vocab) g = NAN;
    const float h = p.dentropy ? p.dentropy[row] : 0.f;
    const float base = none ? 0.f : m;
    const float c = none ? 0.f : 1.f / Z;
    const float H = p.dentropy && !none ? p.entropy[row] - logf(Z) : 0.f;
    const float A = -c * p.scale * fmaf(h, H, g), B = -c * p.scale * h * kLn2;
    const float hit = none ? 0.f : p.scale * g;
    const int tc = (target >= c0 && target < c1) ? (int)target : -1;
    auto grad = [&](float v, int col) {
      const float t = (v - base) * p.a;
      const float d = ex2_gradual(t) * fmaf(B, fmaxf(t, kNoWeight), A);
      return col == tc ? d + hit : d;
    };
    if (VEC) {
      // single elements up to the first 16-byte boundary (the same in both rows), vectors, single elements
      const int off = (int)((reinterpret_cast<uintptr_t>(x + c0) & 15u) / sizeof(T));
      const int head = min(c1 - c0, (V - off) % V);
      const int b0 = c0 + head, b1 = b0 + (c1 - b0) / V * V;
      if ((int)threadIdx.x < head) dx[c0 + threadIdx.x] = Elem<T>::put(grad(Elem<T>::get(x[c0 + threadIdx.x]), c0 + threadIdx.x));
      if ((int)threadIdx.x < c1 - b1) dx[b1 + threadIdx.x] = Elem<T>::put(grad(Elem<T>::get(x[b1 + threadIdx.x]), b1 + threadIdx.x));
      for (int v0 = b0 + threadIdx.x * V; v0 < b1; v0 += 256 * V * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (v0 + u * 256 * V < b1) raw[u] = __ldcs(reinterpret_cast<const uint4*>(x + v0 + u * 256 * V));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int col = v0 + u * 256 * V;
          if (col >= b1) break;
          float e[V];
          Elem<T>::unpack(raw[u], e);
#pragma unroll
          for (int q = 0; q < V; ++q) e[q] = grad(e[q], col + q);
          __stcs(reinterpret_cast<uint4*>(dx + col), Elem<T>::pack(e));
        }
      }
    } else {
      for (int col = c0 + threadIdx.x; col < c1; col += 256) dx[col] = Elem<T>::put(grad(Elem<T>::get(x[col]), col));
    }
  }
}

}  // namespace sgc

namespace {

template <typename T, bool TOP>
int launch_logprobs(sgemm_cube_ctx* h, const sgc::LogprobParams& p, cudaStream_t st) {
  // Few rows: a cluster of blocks shares a row, its pieces at least 4096 columns.  (Two blocks a row for more rows
  // than that, or blocks of 128 threads, measured slower: 1000 x 50001 BF16 with eight alternatives 54 and 34 us
  // against 34, 512 x 131072 45 and 44 against 38.)
  int ranks = 1;
  while (ranks < 8 && (long long)p.rows * ranks < 2 * h->sm_count && p.vocab / (2 * ranks) >= 4096) ranks *= 2;
  for (;; ranks = 1) {                                    // clusters that cannot be scheduled: one block a row
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = (unsigned)ranks; a.val.clusterDim.y = 1; a.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(p.rows * ranks), 1, 1);
    cfg.blockDim = dim3(sgc::kLpThreads, 1, 1);
    cfg.stream = st;
    cfg.attrs = &a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, sgc::token_logprobs_kernel<T, TOP>, p) == cudaSuccess) break;
    cudaGetLastError();
    if (ranks == 1) return SGEMM_CUBE_CUDA_ERROR;
  }
  h->launches++;
  return SGEMM_CUBE_OK;
}

template <typename T>
int launch_grad(sgemm_cube_ctx* h, sgc::LogprobGradParams p, cudaStream_t st) {
  p.chunks = (p.vocab - 1) / 16384 + 1;
  const long long units = (long long)p.rows * p.chunks, cap = (long long)h->sm_count * 64 / p.chunks * p.chunks;
  const unsigned blocks = (unsigned)(units < cap ? units : (cap > p.chunks ? cap : p.chunks));
  if (p.vec) sgc::token_logprobs_grad_kernel<T, true><<<blocks, 256, 0, st>>>(p);
  else sgc::token_logprobs_grad_kernel<T, false><<<blocks, 256, 0, st>>>(p);
  h->launches++;
  return cudaGetLastError() == cudaSuccess ? SGEMM_CUBE_OK : SGEMM_CUBE_CUDA_ERROR;
}

size_t elem_size(int dtype) { return dtype == SGEMM_CUBE_F32 ? 4 : 2; }
bool bad_dtype(int dtype) { return dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16; }
bool bad_scale(float s) { return !(s >= 0x1p-30f && s <= 0x1p30f); }

}  // namespace

extern "C" {

int sgemm_cube_token_logprobs(sgemm_cube_handle h, int rows, int vocab, int dtype, const void* logits, int64_t ld,
                              const int64_t* tokens, float scale, float* logp, float* entropy, float* stats,
                              int top_k, float* top_logp, int64_t* top_index, void* stream) {
  if (!h || bad_dims(rows, vocab) || vocab < 1 || ld < vocab || bad_dtype(dtype) || bad_scale(scale)) return SGEMM_CUBE_INVALID_ARG;
  if (top_k < 0 || top_k > sgc::kTopMax || top_k > vocab) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!logits || misplaced(elem_size(dtype), logits)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(4, logp, entropy, stats, top_logp) || misplaced(8, tokens, top_index)) return SGEMM_CUBE_INVALID_ARG;
  if ((logp != nullptr) != (tokens != nullptr)) return SGEMM_CUBE_INVALID_ARG;
  if ((top_k > 0) != (top_logp != nullptr) || (top_k > 0) != (top_index != nullptr)) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  sgc::LogprobParams p;
  memset(&p, 0, sizeof(p));
  p.rows = rows; p.vocab = vocab;
  p.X = logits; p.ld = ld;
  p.tokens = reinterpret_cast<const long long*>(tokens);
  p.scale = scale;
  p.a = (float)((double)scale * 1.4426950408889634);
  p.logp = logp; p.entropy = entropy; p.stats = stats;
  p.top_k = top_k; p.top_logp = top_logp;
  p.top_index = reinterpret_cast<long long*>(top_index);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SGEMM_CUBE_F32)
    return top_k ? launch_logprobs<float, true>(h, p, st) : launch_logprobs<float, false>(h, p, st);
  if (dtype == SGEMM_CUBE_F16)
    return top_k ? launch_logprobs<__half, true>(h, p, st) : launch_logprobs<__half, false>(h, p, st);
  return top_k ? launch_logprobs<__nv_bfloat16, true>(h, p, st) : launch_logprobs<__nv_bfloat16, false>(h, p, st);
}

int sgemm_cube_token_logprobs_backward(sgemm_cube_handle h, int rows, int vocab, int dtype, const void* logits,
                                       int64_t ld, const int64_t* tokens, float scale, const float* stats,
                                       const float* entropy, const float* dlogp, const float* dentropy,
                                       void* dlogits, int64_t lddl, void* stream) {
  if (!h || bad_dims(rows, vocab) || vocab < 1 || ld < vocab || lddl < vocab || bad_dtype(dtype) || bad_scale(scale))
    return SGEMM_CUBE_INVALID_ARG;
  if (!dlogp && !dentropy) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!logits || !dlogits || !stats || misplaced(elem_size(dtype), logits, dlogits)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(4, stats, entropy, dlogp, dentropy) || misplaced(8, tokens)) return SGEMM_CUBE_INVALID_ARG;
  if (logits == dlogits && ld != lddl && rows > 1) return SGEMM_CUBE_INVALID_ARG;
  if ((dlogp && !tokens) || (dentropy && !entropy)) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  sgc::LogprobGradParams p;
  memset(&p, 0, sizeof(p));
  p.rows = rows; p.vocab = vocab;
  p.X = logits; p.ld = ld;
  p.tokens = reinterpret_cast<const long long*>(tokens);
  p.scale = scale;
  p.a = (float)((double)scale * 1.4426950408889634);
  p.stats = stats; p.entropy = entropy;
  p.dlogp = dlogp; p.dentropy = dentropy;
  p.dX = dlogits; p.lddx = lddl;
  const size_t e = elem_size(dtype);
  // vectors where the two rows meet 16-byte boundaries at the same columns
  p.vec = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(dlogits)) % 16 == 0 && (ld - lddl) * e % 16 == 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SGEMM_CUBE_F32) return launch_grad<float>(h, p, st);
  if (dtype == SGEMM_CUBE_F16) return launch_grad<__half>(h, p, st);
  return launch_grad<__nv_bfloat16>(h, p, st);
}

}  // extern "C"
