// Layer normalisation and its gradients (contracts: include/sgemm_cube.h).
//
//   forward    mean = sum x / n;  var = sum (x - mean)^2 / n;  y = (x - mean) rstd w + b
//   backward   u = dy w;  n = (x - mean) rstd;  dx = rstd (u - mean(u) - n mean(u n))
//              dw = sum over rows of dy n;  db = sum over rows of dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx, each once.  A row
// lives in the registers of one group of warps between its load and its store, so the second moment is
// taken about the mean (no cancellation of squares) without a second read.
#include "ctx.cuh"
#include "elements.cuh"

namespace sgc {

constexpr int kFwdPT = 32;      // elements a thread holds, forward
constexpr int kBwdPT = 16;      // backward: x, dy and two running sums for each

// Sums over a row's group of warps.  `slot` alternates between two buffers, so one barrier a sum is enough.
template <int WARPS, int N>
__device__ __forceinline__ void group_sum(float (&s)[N], float* buf, int group, int warp_in_group, int bar_threads) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
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
      float t = b[i];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) t += b[w * N + i];
      s[i] = t;
    }
  }
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
};

// WARPS warps a row, 8 / WARPS rows a block (one for WARPS >= 8).
template <typename T, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS > 8 ? WARPS * 32 : 256) norm_forward_kernel(NormParams p) {
  constexpr int kGroups = WARPS >= 8 ? 1 : 8 / WARPS, kThreads = WARPS * 32;
  __shared__ float buf[2][kGroups * WARPS];
  const int group = threadIdx.x / kThreads, t = threadIdx.x % kThreads, wg = t >> 5;
  const long long row = (long long)blockIdx.x * kGroups + group;
  if (row >= p.rows) return;                           // whole groups leave; groups meet at their own barriers
  const int bar = kGroups == 1 ? 0 : kThreads;
  float v[kFwdPT];
  load_row<T, kFwdPT, VEC>(static_cast<const T*>(p.X) + row * p.ldx, p.cols, t, kThreads, 0.f, v);
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < kFwdPT; ++i) s[0] += v[i];
  group_sum<WARPS>(s, buf[0], group, wg, bar);
  const float mean = s[0] / (float)p.cols;
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < kFwdPT; ++i) {
    const float d = row_column<T, VEC>(i, t, kThreads) < p.cols ? v[i] - mean : 0.f;
    s[0] = fmaf(d, d, s[0]);
  }
  group_sum<WARPS>(s, buf[1], group, wg, bar);
  const float rstd = 1.f / sqrtf(s[0] / (float)p.cols + p.eps);
#pragma unroll
  for (int i = 0; i < kFwdPT; ++i) {
    const int c = row_column<T, VEC>(i, t, kThreads);
    float n = (v[i] - mean) * rstd;
    if (c < p.cols) {
      if (p.weight) n *= __ldg(p.weight + c);
      if (p.bias) n += __ldg(p.bias + c);
    }
    v[i] = n;
  }
  store_row<T, kFwdPT, VEC>(static_cast<T*>(p.out) + row * p.ldo, p.cols, t, kThreads, v);
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Rows too long for the registers of one block: three passes, the later ones from L2.
template <typename T>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(NormParams p) {
  __shared__ float buf[2][32];
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.X) + row * p.ldx;
  T* y = static_cast<T*>(p.out) + row * p.ldo;
  const int t = threadIdx.x;
  float s[1] = {0.f};
  for (int c = t; c < p.cols; c += 1024) s[0] += Elem<T>::get(x[c]);
  group_sum<32>(s, buf[0], 0, t >> 5, 0);
  const float mean = s[0] / (float)p.cols;
  s[0] = 0.f;
  for (int c = t; c < p.cols; c += 1024) {
    const float d = Elem<T>::get(x[c]) - mean;
    s[0] = fmaf(d, d, s[0]);
  }
  group_sum<32>(s, buf[1], 0, t >> 5, 0);
  const float rstd = 1.f / sqrtf(s[0] / (float)p.cols + p.eps);
  for (int c = t; c < p.cols; c += 1024) {
    float n = (Elem<T>::get(x[c]) - mean) * rstd;
    if (p.weight) n *= p.weight[c];
    if (p.bias) n += p.bias[c];
    y[c] = Elem<T>::put(n);
  }
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// A persistent block walks over rows; a thread holds the same columns of every row, so its two running
// sums for dw and db stay in registers until the end, when the block writes one partial row of each.
template <typename T, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS > 8 ? WARPS * 32 : 256) norm_backward_kernel(NormParams p) {
  constexpr int kGroups = WARPS >= 8 ? 1 : 8 / WARPS, kThreads = WARPS * 32;
  __shared__ float buf[2][kGroups * WARPS * 2];
  const int group = threadIdx.x / kThreads, t = threadIdx.x % kThreads, wg = t >> 5;
  const int bar = kGroups == 1 ? 0 : kThreads;
  const float inv_n = 1.f / (float)p.cols;
  float dw[kBwdPT], db[kBwdPT];
#pragma unroll
  for (int i = 0; i < kBwdPT; ++i) dw[i] = db[i] = 0.f;
  int slot = 0;
  for (long long row = (long long)blockIdx.x * kGroups + group; row < p.rows; row += (long long)gridDim.x * kGroups) {
    float x[kBwdPT], g[kBwdPT];
    load_row<T, kBwdPT, VEC>(static_cast<const T*>(p.X) + row * p.ldx, p.cols, t, kThreads, 0.f, x);
    load_row<T, kBwdPT, VEC>(static_cast<const T*>(p.dY) + row * p.lddy, p.cols, t, kThreads, 0.f, g);
    const float mean = p.mean_in[row], rstd = p.rstd_in[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kBwdPT; ++i) {
      const int c = row_column<T, VEC>(i, t, kThreads);
      x[i] = (x[i] - mean) * rstd;                     // n; columns past the end have g = 0
      dw[i] = fmaf(g[i], x[i], dw[i]);
      db[i] += g[i];
      if (p.weight) g[i] *= c < p.cols ? __ldg(p.weight + c) : 0.f;
      s[0] += g[i];
      s[1] = fmaf(g[i], x[i], s[1]);
    }
    if (!p.out) continue;
    group_sum<WARPS>(s, buf[slot], group, wg, bar);
    slot ^= 1;
    const float mu = s[0] * inv_n, mun = s[1] * inv_n;
#pragma unroll
    for (int i = 0; i < kBwdPT; ++i) g[i] = rstd * (g[i] - mu - x[i] * mun);
    store_row<T, kBwdPT, VEC>(static_cast<T*>(p.out) + row * p.ldo, p.cols, t, kThreads, g);
  }
  if (!p.part) return;
  float* pw = p.part + (long long)blockIdx.x * 2 * p.cols;
  if constexpr (kGroups == 1) {
#pragma unroll
    for (int i = 0; i < kBwdPT; ++i) {
      const int c = row_column<T, VEC>(i, t, kThreads);
      if (c < p.cols) { pw[c] = dw[i]; pw[p.cols + c] = db[i]; }
    }
  } else {                                             // the block's groups first, in order
    __shared__ float sum[2][kThreads * kBwdPT];
    for (int g = 0; g < kGroups; ++g) {
      if (g == group) {
#pragma unroll
        for (int i = 0; i < kBwdPT; ++i) {
          sum[0][i * kThreads + t] = (g ? sum[0][i * kThreads + t] : 0.f) + dw[i];
          sum[1][i * kThreads + t] = (g ? sum[1][i * kThreads + t] : 0.f) + db[i];
        }
      }
      __syncthreads();
    }
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < kBwdPT; ++i) {
        const int c = row_column<T, VEC>(i, t, kThreads);
        if (c < p.cols) { pw[c] = sum[0][i * kThreads + t]; pw[p.cols + c] = sum[1][i * kThreads + t]; }
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

// Adds the blocks' partial rows in a fixed order: 32 columns a block, eight warps over the partial rows.
// grid (ceil(cols / 32), 2): dw, db.
__global__ void __launch_bounds__(256)
norm_parts_kernel(const float* __restrict__ part, int parts, int cols, float* dweight, float* dbias) {
  __shared__ float sum[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  float s = 0.f;
  if (c < cols)
    for (int i = warp; i < parts; i += 8) s += part[((long long)i * 2 + blockIdx.y) * cols + c];
  sum[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    for (int w = 1; w < 8; ++w) s += sum[w][lane];
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

template <typename T, int WARPS, bool VEC>
int forward_rows(sgemm_cube_ctx* h, const NormParams& p, cudaStream_t st) {
  constexpr int groups = WARPS >= 8 ? 1 : 8 / WARPS;
  sgc::norm_forward_kernel<T, WARPS, VEC>
      <<<(unsigned)((p.rows + groups - 1) / groups), WARPS > 8 ? WARPS * 32 : 256, 0, st>>>(p);
  return done(h);
}
template <typename T, bool VEC>
int forward_typed(sgemm_cube_ctx* h, const NormParams& p, cudaStream_t st) {
  if (p.cols <= 1 * 32 * sgc::kFwdPT) return forward_rows<T, 1, VEC>(h, p, st);
  if (p.cols <= 2 * 32 * sgc::kFwdPT) return forward_rows<T, 2, VEC>(h, p, st);
  if (p.cols <= 4 * 32 * sgc::kFwdPT) return forward_rows<T, 4, VEC>(h, p, st);
  if (p.cols <= 8 * 32 * sgc::kFwdPT) return forward_rows<T, 8, VEC>(h, p, st);
  if (p.cols <= 16 * 32 * sgc::kFwdPT) return forward_rows<T, 16, VEC>(h, p, st);
  if (p.cols <= 32 * 32 * sgc::kFwdPT) return forward_rows<T, 32, VEC>(h, p, st);
  sgc::norm_forward_long_kernel<T><<<(unsigned)p.rows, 1024, 0, st>>>(p);
  return done(h);
}

template <typename T, int WARPS, bool VEC>
int backward_rows(sgemm_cube_ctx* h, NormParams p, float* dweight, float* dbias, cudaStream_t st) {
  constexpr int groups = WARPS >= 8 ? 1 : 8 / WARPS, threads = WARPS > 8 ? WARPS * 32 : 256;
  int per_sm = 0;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, sgc::norm_backward_kernel<T, WARPS, VEC>, threads, 0) !=
      cudaSuccess || per_sm < 1) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  const long long want = ((long long)p.rows + groups - 1) / groups, cap = (long long)per_sm * h->sm_count;
  const int blocks = (int)(want < cap ? want : cap);
  if (dweight || dbias) {
    int rc = grow(&h->part_ws, &h->part_ws_bytes, (size_t)blocks * 2 * p.cols * 4);
    if (rc) return rc;
    p.part = static_cast<float*>(h->part_ws);
  }
  sgc::norm_backward_kernel<T, WARPS, VEC><<<(unsigned)blocks, threads, 0, st>>>(p);
  int rc = done(h);
  if (rc || !p.part) return rc;
  sgc::norm_parts_kernel<<<dim3((unsigned)((p.cols + 31) / 32), 2), 256, 0, st>>>(p.part, blocks, p.cols, dweight, dbias);
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
    if ((rc = grow(&h->part_ws, &h->part_ws_bytes, (size_t)blocks * 2 * p.cols * 4))) return rc;
    p.part = static_cast<float*>(h->part_ws);
    sgc::norm_columns_kernel<T><<<dim3((unsigned)tiles, (unsigned)blocks), 256, 0, st>>>(p, per);
    if ((rc = done(h))) return rc;
    sgc::norm_parts_kernel<<<dim3((unsigned)tiles, 2), 256, 0, st>>>(p.part, blocks, p.cols, dweight, dbias);
    if ((rc = done(h))) return rc;
  }
  if (!p.out) return rc;
  sgc::norm_backward_long_kernel<T><<<(unsigned)p.rows, 1024, 0, st>>>(p);
  return done(h);
}
template <typename T, bool VEC>
int backward_typed(sgemm_cube_ctx* h, const NormParams& p, float* dw, float* db, cudaStream_t st) {
  if (p.cols <= 1 * 32 * sgc::kBwdPT) return backward_rows<T, 1, VEC>(h, p, dw, db, st);
  if (p.cols <= 2 * 32 * sgc::kBwdPT) return backward_rows<T, 2, VEC>(h, p, dw, db, st);
  if (p.cols <= 4 * 32 * sgc::kBwdPT) return backward_rows<T, 4, VEC>(h, p, dw, db, st);
  if (p.cols <= 8 * 32 * sgc::kBwdPT) return backward_rows<T, 8, VEC>(h, p, dw, db, st);
  if (p.cols <= 16 * 32 * sgc::kBwdPT) return backward_rows<T, 16, VEC>(h, p, dw, db, st);
  if (p.cols <= 32 * 32 * sgc::kBwdPT) return backward_rows<T, 32, VEC>(h, p, dw, db, st);
  return backward_long<T>(h, p, dw, db, st);
}

size_t elem_size(int dtype) { return dtype == SGEMM_CUBE_F32 ? 4 : 2; }
bool bad_dtype(int dtype) { return dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16; }
bool off_elem(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_size(dtype) != 0; }

}  // namespace

extern "C" {

int sgemm_cube_layer_norm(sgemm_cube_handle h, int rows, int cols, int dtype, const void* X, int64_t ldx,
                          const float* weight, const float* bias, float eps, void* Y, int64_t ldy, float* mean,
                          float* rstd, void* stream) {
  if (!h || rows < 0 || cols < 1 || bad_dtype(dtype) || !(eps >= 0.f) || ldx < cols || ldy < cols)
    return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  if (!X || !Y || off_elem(X, dtype) || off_elem(Y, dtype)) return SGEMM_CUBE_INVALID_ARG;
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
  if (!h || rows < 0 || cols < 1 || bad_dtype(dtype) || ldx < cols || lddy < cols || (dX && lddx < cols))
    return SGEMM_CUBE_INVALID_ARG;
  if (rows > 0 && (!dY || !X || !mean || !rstd || off_elem(dY, dtype) || off_elem(X, dtype) || off_elem(dX, dtype)))
    return SGEMM_CUBE_INVALID_ARG;
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
  const size_t e = elem_size(dtype);
  const bool vec = sgc::rows_take_vectors(X, ldx, cols, e) && sgc::rows_take_vectors(dY, lddy, cols, e) &&
                   (!dX || sgc::rows_take_vectors(dX, lddx, cols, e));
  if (dtype == SGEMM_CUBE_F32)
    return vec ? backward_typed<float, true>(h, p, dweight, dbias, st) : backward_typed<float, false>(h, p, dweight, dbias, st);
  if (dtype == SGEMM_CUBE_F16)
    return vec ? backward_typed<__half, true>(h, p, dweight, dbias, st) : backward_typed<__half, false>(h, p, dweight, dbias, st);
  return vec ? backward_typed<__nv_bfloat16, true>(h, p, dweight, dbias, st)
             : backward_typed<__nv_bfloat16, false>(h, p, dweight, dbias, st);
}

}  // extern "C"
