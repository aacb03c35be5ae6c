// Log probabilities of given tokens under softmax(scale * x), with entropy and the largest alternatives, and
// the gradient of the logits (contracts: include/sgemm_cube.h).
//
// Forward, one pass over a row with a running maximum m and, relative to it, the sums
//   Z = sum exp(scale (x - m)),   S = sum exp(scale (x - m)) scale (x - m);
// when m grows to m' both shrink by r = exp(scale (m - m')) and S also takes r scale (m - m') Z.  Then
//   lse = scale m + log Z,   log p_t = scale (x_t - m) - log Z,   H = log Z - S / Z.
// Bound by reading the logits once.  Exponentials run in base 2, t = (x - m) a with a = scale log2 e.  The difference
// is taken first: one FMA with fl(m a) would save an instruction, but overflows where masked logits hold the
// type's lowest value, and puts the rounding of m a into every term.
#include "ctx.cuh"
#include "elements.cuh"

namespace sgc {

constexpr int kLpThreads = 512;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kTopMax = 32;
constexpr int kCandidates = 256;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kNoWeight = -160.f;      // 2^-160 is zero in FP32: exponents are cut there where they are factors

__device__ __forceinline__ float ex2(float t) {
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

// Running sums of a part of a row; S in base-2 units.
struct Running {
  float m, Z, S;
};
__device__ __forceinline__ void raise(Running& r, float m, float a) {   // m > r.m
  const float d = (r.m - m) * a;
  const float f = ex2(d);                      // zero when r.m is -inf
  r.S = f * fmaf(fmaxf(d, kNoWeight), r.Z, r.S);
  r.Z *= f;
  r.m = m;
}
// `m` is r.m, or 0 while that is -inf (then x is -inf or NaN)
__device__ __forceinline__ void add_one(Running& r, float x, float m, float a) {
  const float t = (x - m) * a;
  const float e = ex2(t);
  r.Z += e;
  r.S = fmaf(e, fmaxf(t, kNoWeight), r.S);
}
__device__ __forceinline__ float finite_max(const Running& r) { return r.m == -INFINITY ? 0.f : r.m; }
__device__ __forceinline__ void join(Running& r, Running o, float a) {
  if (o.m > r.m) { const Running x = r; r = o; o = x; }
  // r has the larger m; an -inf part has empty sums, or NaN ones, which stay
  if (o.m == -INFINITY) { r.Z += o.Z; r.S += o.S; return; }
  const float d = (o.m - r.m) * a;
  const float f = ex2(d);
  r.Z = fmaf(o.Z, f, r.Z);
  r.S += f * fmaf(fmaxf(d, kNoWeight), o.Z, o.S);
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
  // element e of thread t's own sequence (front, vectors, rest), as a column of the piece; -1 past its end
  __device__ __forceinline__ int column(int t, int e) const {
    constexpr int V = Elem<T>::kVec;
    if (t < head) {
      if (e == 0) return t;
      --e;
    }
    const int mine = vecs > t ? (vecs - t + kLpThreads - 1) / kLpThreads * V : 0;
    if (e < mine) return head + (t + e / V * kLpThreads) * V + e % V;
    return (e == mine && t < tail) ? head + vecs * V + t : -1;
  }
  __device__ __forceinline__ int owner(int c) const {
    constexpr int V = Elem<T>::kVec;
    if (c < head) return c;
    c -= head;
    return c < vecs * V ? c / V % kLpThreads : c - vecs * V;
  }
};

template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads) token_logprobs_kernel(LogprobParams p) {
  constexpr int V = Elem<T>::kVec, U = 16 / V;           // 16 elements of a thread in flight
  __shared__ Running parts[kLpWarps];
  __shared__ Running block_sum;
  __shared__ uint64_t list[TOP ? kLpWarps : 1][32];
  __shared__ uint64_t more[TOP ? kCandidates : 1];
  __shared__ uint64_t best[TOP ? 32 : 1];
  __shared__ int more_count;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const uint32_t ranks = cluster_size(), rank = cluster_rank_x();
  const long long row = blockIdx.x / ranks;
  const T* x_row = static_cast<const T*>(p.X) + row * p.ld;
  const long long per = ((long long)p.vocab + ranks - 1) / ranks;
  const int c0 = (int)min((long long)p.vocab, rank * per), c1 = (int)min((long long)p.vocab, c0 + per);
  const Piece<T> piece(x_row + c0, c1 - c0);

  Running r{-INFINITY, 0.f, 0.f};
  int at = -1;                                           // where m was met: -1 nowhere, 0 front, 1 + batch, then the rest
  if (t < piece.head) {
    const float x = Elem<T>::get(piece.x[t]);
    if (x > r.m) { raise(r, x, p.a); at = 0; }
    add_one(r, x, finite_max(r), p.a);
  }
  const int batches = (piece.vecs + kLpThreads * U - 1) / (kLpThreads * U);
  for (int b = 0; b < batches; ++b) {
    uint4 raw[U];
    const int v0 = b * kLpThreads * U + t;
    const bool whole = (b + 1) * kLpThreads * U <= piece.vecs;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (whole || v0 + u * kLpThreads < piece.vecs) raw[u] = __ldg(piece.vec(v0 + u * kLpThreads));
    float v[U][V];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (whole || v0 + u * kLpThreads < piece.vecs) {
        Elem<T>::unpack(raw[u], v[u]);
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q) v[u][q] = -INFINITY;
      }
#pragma unroll
      for (int q = 0; q < V; ++q) top = fmaxf(top, v[u][q]);
    }
    if (top > r.m) { raise(r, top, p.a); at = 1 + b; }
    const float m = finite_max(r);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < V; ++q) add_one(r, v[u][q], m, p.a);
  }
  if (t < piece.tail) {
    const float x = Elem<T>::get(piece.x[piece.head + piece.vecs * V + t]);
    if (x > r.m) { raise(r, x, p.a); at = 1 + batches; }
    add_one(r, x, finite_max(r), p.a);
  }

  if (TOP) {
    // The k largest of the threads' maxima bound the k largest elements from below, and hold every thread
    // that owns one of them: an element among the k largest is not above its thread's maximum.
    uint64_t key = 0;
    int e0 = 0, e1 = 1;                                  // elements of the own sequence that hold the maximum
    if (at > 0 && at <= batches) { e0 = (t < piece.head) + (at - 1) * 16; e1 = e0 + 16; }
    else if (at > batches) { e0 = (t < piece.head) + (piece.vecs > t ? (piece.vecs - t + kLpThreads - 1) / kLpThreads * V : 0); e1 = e0 + 1; }
    for (int e = e0; e < e1; ++e) {
      const int c = piece.column(t, e);
      if (c < 0) break;
      const uint64_t k = order_key(Elem<T>::get(piece.x[c]), (uint32_t)(c0 + c));
      if (k > key) key = k;
    }
    if (t == 0) more_count = 0;
    list[warp][lane] = sort_lanes(key, lane);
    __syncthreads();
    for (int s = kLpWarps / 2; s > 0; s >>= 1) {
      uint64_t k = 0;
      if (warp < s) k = merge_lanes(list[warp][lane], list[warp + s][31 - lane], lane);
      __syncthreads();
      if (warp < s) list[warp][lane] = k;
      __syncthreads();
    }
    const uint64_t bound = list[0][p.top_k - 1];
    // what else these threads own above the bound
    for (int j = warp; j < p.top_k; j += kLpWarps) {
      const uint64_t own = list[0][j];
      if (own == 0) break;
      const int w = piece.owner((int)key_column(own) - c0);
      for (int e = lane;; e += 32) {
        const int c = piece.column(w, e);
        if (c >= 0) {
          const uint64_t k = order_key(Elem<T>::get(piece.x[c]), (uint32_t)(c0 + c));
          if (k > bound && k != own) {
            const int at_more = atomicAdd(&more_count, 1);
            if (at_more < kCandidates) more[at_more] = k;
          }
        }
        if (__all_sync(0xffffffffu, c < 0)) break;
      }
    }
    __syncthreads();
    if (warp == 0) {
      uint64_t k = list[0][lane];
      if (more_count <= kCandidates) {
        for (int i = 0; i < more_count; i += 32) {
          const uint64_t o = sort_lanes(i + lane < more_count ? more[i + lane] : 0ull, lane);
          k = merge_lanes(k, __shfl_sync(0xffffffffu, o, 31 - lane), lane);
        }
      } else {                                           // many in a few threads: straight from the row
        for (int j = 0; j < p.top_k; ++j) {
          const uint64_t own = list[0][j];
          if (own == 0) break;
          const int w = piece.owner((int)key_column(own) - c0);
          for (int e = lane;; e += 32) {
            const int c = piece.column(w, e);
            uint64_t o = 0;
            if (c >= 0) {
              o = order_key(Elem<T>::get(piece.x[c]), (uint32_t)(c0 + c));
              if (o <= bound || o == own) o = 0;
            }
            if (__any_sync(0xffffffffu, o != 0)) {
              o = sort_lanes(o, lane);
              k = merge_lanes(k, __shfl_sync(0xffffffffu, o, 31 - lane), lane);
            }
            if (__all_sync(0xffffffffu, c < 0)) break;
          }
        }
      }
      best[lane] = k;
    }
  }

#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Running other;
    other.m = __shfl_down_sync(0xffffffffu, r.m, o);
    other.Z = __shfl_down_sync(0xffffffffu, r.Z, o);
    other.S = __shfl_down_sync(0xffffffffu, r.S, o);
    join(r, other, p.a);
  }
  if (lane == 0) parts[warp] = r;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < kLpWarps; ++w) join(r, parts[w], p.a);
    block_sum = r;
  }
  if (ranks > 1) cluster_meet();
  else __syncthreads();
  if (rank == 0 && warp == 0) {
    r = block_sum;
    uint64_t k = TOP ? best[lane] : 0ull;
    for (uint32_t o = 1; o < ranks; ++o) {
      const uint32_t a = remote_address(&block_sum, o);
      Running other;
      other.m = remote_f32(a); other.Z = remote_f32(a + 4); other.S = remote_f32(a + 8);
      join(r, other, p.a);
      if (TOP) k = merge_lanes(k, remote_u64(remote_address(&best[31 - lane], o)), lane);
    }
    const bool none = r.m == -INFINITY && r.Z == 0.f;     // every logit is -inf
    const float log_z = logf(r.Z);
    if (lane == 0) {
      if (p.stats) { p.stats[2 * row] = r.m; p.stats[2 * row + 1] = r.Z; }
      if (p.entropy) p.entropy[row] = none ? 0.f : log_z - r.S / r.Z * kLn2;
      if (p.logp) {
        const long long target = p.tokens[row];
        float lp = 0.f;
        if (target >= p.vocab) lp = NAN;
        else if (target >= 0) lp = none ? -INFINITY : (Elem<T>::get(x_row[target]) - r.m) * p.scale - log_z;
        p.logp[row] = lp;
      }
    }
    if (TOP && lane < p.top_k) {
      p.top_logp[row * p.top_k + lane] = none ? -INFINITY : (k ? (key_logit(k) - r.m) * p.scale - log_z : NAN);
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
// Reads and writes every logit once.  A block takes chunk `blockIdx % chunks` of a row, then the same of the
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
      const float d = ex2(t) * fmaf(B, fmaxf(t, kNoWeight), A);
      return col == tc ? d + hit : d;
    };
    if (VEC) {
      for (int v0 = c0 + threadIdx.x * V; v0 < c1; v0 += 256 * V * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (v0 + u * 256 * V < c1) raw[u] = __ldcs(reinterpret_cast<const uint4*>(x + v0 + u * 256 * V));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int col = v0 + u * 256 * V;
          if (col >= c1) break;
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
  // Few rows: a cluster of blocks shares a row, its pieces at least 4096 columns.
  int ranks = 1;
  while (ranks < 8 && (long long)p.rows * ranks < 2 * h->sm_count && p.vocab / (2 * ranks) >= 4096) ranks *= 2;
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
  h->launches++;
  if (cudaLaunchKernelEx(&cfg, sgc::token_logprobs_kernel<T, TOP>, p) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
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
bool off_elem(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_size(dtype) != 0; }
bool bad_scale(float s) { return !(s > 0.f && s <= 3.0e38f); }

}  // namespace

extern "C" {

int sgemm_cube_token_logprobs(sgemm_cube_handle h, int rows, int vocab, int dtype, const void* logits, int64_t ld,
                              const int64_t* tokens, float scale, float* logp, float* entropy, float* stats,
                              int top_k, float* top_logp, int64_t* top_index, void* stream) {
  if (!h || rows < 0 || vocab < 1 || ld < vocab || bad_dtype(dtype) || bad_scale(scale)) return SGEMM_CUBE_INVALID_ARG;
  if (top_k < 0 || top_k > sgc::kTopMax || top_k > vocab) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!logits || off_elem(logits, dtype)) return SGEMM_CUBE_INVALID_ARG;
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
  if (!h || rows < 0 || vocab < 1 || ld < vocab || lddl < vocab || bad_dtype(dtype) || bad_scale(scale))
    return SGEMM_CUBE_INVALID_ARG;
  if (!dlogp && !dentropy) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!logits || !dlogits || !stats || off_elem(logits, dtype) || off_elem(dlogits, dtype)) return SGEMM_CUBE_INVALID_ARG;
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
  p.vec = sgc::rows_take_vectors(logits, ld, vocab, e) && sgc::rows_take_vectors(dlogits, lddl, vocab, e);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SGEMM_CUBE_F32) return launch_grad<float>(h, p, st);
  if (dtype == SGEMM_CUBE_F16) return launch_grad<__half>(h, p, st);
  return launch_grad<__nv_bfloat16>(h, p, st);
}

}  // extern "C"
