// Softmax cross entropy of a linear layer's outputs over a large vocabulary, without the logits, and its gradients
// (contracts: include/sgemm_cube.h).
//
//   z = X W + b,  lse = log sum_j exp(z_j),  loss = lse - z_t,  dz = dloss (exp(z - lse) - 1[t]),
//   dX = dz W^T,  dW = X^T dz,  db = column sums of dz.
//
// Forward: the logits stay in the product's tiles; (largest, sum) of every 64 of them is what a tile leaves behind
// (loss_epilogue.cuh), and one pass over those pairs gives lse and the loss.
// Gradients: a piece of the rows at a time.  Its logits (1 GiB at most) go to the workspace once and are turned into
// the FP16 words of dz, which both products read: three products in all.  (In pieces of the vocabulary a piece's logits would have to
// be formed a second time once lse is known: four products.)  The words' exponent is known before them, |dz| <= |dloss|.
#include "ctx.cuh"
#include "product_host.cuh"

namespace sgc {

constexpr int kFormLossKM = form_of(kFormKM, kEpiLoss), kFormLossKK = form_of(kFormKK, kEpiLoss);

// The pairs of logits that are there already (few rows: the linear layer's own forms wrote them).  A warp takes 64
// columns of a row, two a lane.
__global__ void __launch_bounds__(256)
logit_parts_kernel(int rows, int vocab, const float* __restrict__ Z, long long ldz, const long long* __restrict__ targets,
                   float* __restrict__ target_logit, float2* __restrict__ parts, long long ldp) {
  const int lane = threadIdx.x & 31;
  const int per_row = (vocab + kLossColumns - 1) / kLossColumns;
  const long long total = (long long)rows * per_row;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += (long long)gridDim.x * 8) {
    const long long r = w / per_row;
    const int piece = (int)(w - r * per_row), c = piece * kLossColumns + lane * 2;
    const float* z = Z + r * ldz + c;
    float v[2];
    v[0] = c < vocab ? z[0] : -INFINITY;
    v[1] = c + 1 < vocab ? z[1] : -INFINITY;
    const long long t = targets[r];
    if (t >= c && t < c + 2 && t < vocab) target_logit[r] = v[t - c];
    const float2 part = softmax_part(v, 32);
    if (lane == 0) parts[r * ldp + piece] = part;
  }
}

struct LossJoinParams {
  int rows, vocab, per_row;
  const float2* parts;
  long long ldp;
  const long long* targets;
  const float* target_logit;
  float* loss;              // or null
  float* lse;               // or null
  float2* stats;            // (m, 1 / sum) of a row, or null
};
__device__ __forceinline__ float2 join_parts(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);              // both 0, or NaN
  return make_float2(m, a.y * expf(a.x - m) + b.y * expf(b.x - m));
}
// lse and loss of a row from its pairs; a block a row.  The pairs of a thread are joined in their order, the threads' in
// a fixed tree.  loss = (m - z_t) + log sum: the difference of two logits keeps its digits, whatever their size.
__global__ void __launch_bounds__(128) loss_join_kernel(LossJoinParams p) {
  const long long r = blockIdx.x;
  float2 acc = make_float2(-INFINITY, 0.f);
  for (int i = threadIdx.x; i < p.per_row; i += 128) acc = join_parts(acc, p.parts[r * p.ldp + i]);
  for (int x = 16; x > 0; x >>= 1) {
    const float2 o = make_float2(__shfl_xor_sync(0xffffffffu, acc.x, x), __shfl_xor_sync(0xffffffffu, acc.y, x));
    acc = join_parts(acc, o);
  }
  __shared__ float2 warp_part[4];
  if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) acc = join_parts(acc, warp_part[w]);
    const bool none = acc.x == -INFINITY && acc.y == 0.f;            // no logit above -inf
    const float log_sum = logf(acc.y);
    const long long t = p.targets[r];
    float loss = 0.f;
    if (t >= p.vocab) loss = NAN;
    else if (t >= 0) loss = none ? INFINITY : (acc.x - p.target_logit[r]) + log_sum;
    if (p.loss) p.loss[r] = loss;
    if (p.lse) p.lse[r] = none ? -INFINITY : acc.x + log_sum;
    if (p.stats) p.stats[r] = make_float2(none ? 0.f : acc.x, none ? 0.f : 1.f / acc.y);
  }
}

// The exponent of dz' words: |dz| <= |dloss| of a row with a target.  One block.
__global__ void __launch_bounds__(1024)
loss_exponent_kernel(int rows, const float* __restrict__ dloss, const long long* __restrict__ targets, int* exp) {
  uint32_t m = 0;
  for (int r = threadIdx.x; r < rows; r += 1024)
    if (targets[r] >= 0) m = max(m, finite_bits(dloss[r]));
  m = __reduce_max_sync(0xffffffffu, m);
  __shared__ uint32_t warp_max[32];
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x < 32) {
    m = __reduce_max_sync(0xffffffffu, warp_max[threadIdx.x]);
    if (threadIdx.x == 0) *exp = pack_exponent(m);
  }
}

struct LossGradParams {
  int rows, vocab, rows_per_chunk;
  const float* Z;
  long long ldz;
  const float2* stats;
  const float* dloss;
  const long long* targets;
  uint16_t* hi;             // words of dz, or null
  uint16_t* lo;
  long long ldw;
  const int* exp;
  float* col_part;          // [chunks][vocab] column sums of dz, or null
};
// dz = dloss (exp(z - m) / sum - 1[t]) of a piece of rows, as words, with its column sums.  A lane has eight columns; the warps
// of a block take every eighth row of its chunk.  Bound by memory: 8 bytes a logit.
__global__ void __launch_bounds__(256) loss_grad_kernel(LossGradParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 256 + lane * 8;
  const int r_end = min(p.rows, (int)(blockIdx.y + 1) * p.rows_per_chunk);
  const float pre = p.hi ? pow2f(*p.exp) : 1.f;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int r = blockIdx.y * p.rows_per_chunk + warp; r < r_end; r += 8) {
    if (c >= p.vocab) break;
    const float* z = p.Z + (long long)r * p.ldz + c;                 // rows are 8 floats wide at least, zeros behind the end
    const float4 a = __ldcs(reinterpret_cast<const float4*>(z));
    const float4 b = __ldcs(reinterpret_cast<const float4*>(z + 4));
    const float2 st = p.stats[r];
    const long long t = p.targets[r];
    float g = t >= 0 ? p.dloss[r] : 0.f;
    if (t >= p.vocab) g = NAN;
    const bool none = st.y == 0.f;                                   // nothing is allowed: no gradient
    const float w = none ? 0.f : g * st.y;
    float d[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      d[q] = c + q < p.vocab && t >= 0 ? w * fast_exp2((d[q] - st.x) * kLog2e) : 0.f;
      if (c + q == t && !none) d[q] -= g;
      sum[q] += d[q];
    }
    if (p.hi) {
      uint4 h, l;
      pack_words(d, pre, h, l);
      *reinterpret_cast<uint4*>(p.hi + (long long)r * p.ldw + c) = h;
      *reinterpret_cast<uint4*>(p.lo + (long long)r * p.ldw + c) = l;
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
  }
}

__global__ void __launch_bounds__(256)
loss_column_sums_kernel(const float* __restrict__ part, int chunks, int cols, float* __restrict__ out) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float s = part[c];
#pragma unroll 8
  for (int i = 1; i < chunks; ++i) s += part[(long long)i * cols + c];
  out[c] = s;
}

}  // namespace sgc

namespace {

using sgc::Carve;
using sgc::Packed;
using sgc::PackJob;

constexpr size_t kPieceBytes = (size_t)1 << 30;          // logits of a piece of rows
constexpr int kPieceRows = 1 << 22;                      // (small vocabularies)
constexpr int kGradRows = 256;                           // rows of a column sum's part

int loss_setup(sgemm_cube_ctx* h) {
  return sgc::product_setup<sgc::kFormLossKM, sgc::kFormLossKK>(h, h->loss_clusters);
}

struct LossCall {
  int M, N, K;
  bool nk;
  const float* bias;
  const int64_t* targets;
};

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

int launch_join(sgemm_cube_ctx* h, int rows, int vocab, const sgc::LossEpilogue& ep, float* loss, float* lse, float2* stats, cudaStream_t st) {
  sgc::LossJoinParams j;
  j.rows = rows; j.vocab = vocab; j.per_row = (vocab + sgc::kLossColumns - 1) / sgc::kLossColumns;
  j.parts = ep.parts; j.ldp = ep.ldp;
  j.targets = ep.targets; j.target_logit = ep.target_logit;
  j.loss = loss; j.lse = lse; j.stats = stats;
  sgc::loss_join_kernel<<<(unsigned)rows, 128, 0, st>>>(j);
  return sgc::launched(h);
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
  float* Z = nullptr;
  const int64_t ldz = (int64_t)round_up((size_t)N, 8);
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->loss_ws) : nullptr;
    ep.parts = c.take<float2>((size_t)M * per_row);
    ep.target_logit = c.take<float>((size_t)M);
    if (few) Z = c.take<float>((size_t)M * ldz);
    if (!pass && (rc = grow(h, &h->loss_ws, &h->loss_ws_bytes, c.used, st))) return rc;
  }
  if (few) {
    // few rows: the layer's kernels for them, whose logits stay in L2
    rc = sgemm_cube_linear(h, M, N, K, X, W, weight_layout, bias, nullptr, 0, SGEMM_CUBE_ACT_NONE, Z, ldz, nullptr, 0, stream);
    if (rc) return rc;
    sgc::logit_parts_kernel<<<sgc::blocks_for(h, (long long)M * per_row * 32), 256, 0, st>>>(
        M, N, Z, ldz, ep.targets, ep.target_logit, ep.parts, ep.ldp);
    if ((rc = sgc::launched(h))) return rc;
    return launch_join(h, M, N, ep, loss, lse, nullptr, st);
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
  return launch_join(h, M, N, ep, loss, lse, nullptr, st);
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
  int piece = most < 256 ? 256 : (most < M ? (int)most : M);
  if (piece < M) {
    const long long pieces = ((long long)M + piece - 1) / piece;
    piece = (int)round_up((size_t)((M + pieces - 1) / pieces), 256);
  }
  const int chunks = (M + kGradRows - 1) / kGradRows + (M + piece - 1) / piece;     // (every piece rounds up)
  sgc::LossEpilogue ep;
  memset(&ep, 0, sizeof(ep));
  ep.bias = bias;
  ep.ldp = per_row;
  ep.ldz = ldz;
  float2* stats = nullptr;
  uint16_t *ghi = nullptr, *glo = nullptr;
  float* col_part = nullptr;
  float* target_logit = nullptr;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->loss_ws) : nullptr;
    ep.parts = c.take<float2>((size_t)piece * per_row);
    target_logit = c.take<float>((size_t)piece);
    stats = c.take<float2>((size_t)piece);
    ep.Z = c.take<float>((size_t)piece * ldz);
    if (split) {
      ghi = c.take<uint16_t>((size_t)piece * ldz);
      glo = c.take<uint16_t>((size_t)piece * ldz);
    }
    if (dbias) col_part = c.take<float>((size_t)chunks * N);
    if (!pass && (rc = grow(h, &h->loss_ws, &h->loss_ws_bytes, c.used, st))) return rc;
  }
  ep.target_logit = target_logit;
  PackJob jobs[2];
  int n_jobs = 0;
  int* exps = reinterpret_cast<int*>(h->err_dev + sgc::kExpWords);
  Packed px{}, pw{};
  for (int pass = 0; pass < 2; ++pass) {
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->ws) : nullptr;
    n_jobs = 0;
    px = sgc::words_of(X, M, K, c, exps, jobs, &n_jobs);
    pw = sgc::words_of(W, w_rows, w_cols, c, exps + 1, jobs, &n_jobs);
    if (!pass && c.used && (rc = grow(h, &h->ws, &h->ws_bytes, c.used, st))) return rc;
  }
  if (n_jobs && (rc = sgc::launch_pack(h, jobs, n_jobs, st))) return rc;
  if (split) {
    sgc::loss_exponent_kernel<<<1, 1024, 0, st>>>(M, dloss, reinterpret_cast<const long long*>(targets), exps + 2);
    if ((rc = sgc::launched(h))) return rc;
  }
  int chunk0 = 0;
  for (int r0 = 0; r0 < M; r0 += piece) {
    const int rows = M - r0 < piece ? M - r0 : piece;
    const Packed x{px.hi + (int64_t)r0 * px.ld, px.lo + (int64_t)r0 * px.ld, px.ld, px.exp};
    ep.targets = reinterpret_cast<const long long*>(targets) + r0;
    rc = nk ? loss_product<sgc::kFormLossKK>(h, rows, N, K, x, pw, ep, st) : loss_product<sgc::kFormLossKM>(h, rows, N, K, x, pw, ep, st);
    if (rc) return rc;
    if ((rc = launch_join(h, rows, N, ep, loss ? loss + r0 : nullptr, lse ? lse + r0 : nullptr, stats, st))) return rc;
    sgc::LossGradParams p;
    memset(&p, 0, sizeof(p));
    p.rows = rows; p.vocab = N; p.rows_per_chunk = kGradRows;
    p.Z = ep.Z; p.ldz = ldz;
    p.stats = stats;
    p.dloss = dloss + r0;
    p.targets = ep.targets;
    p.hi = ghi; p.lo = glo; p.ldw = ldz;
    p.exp = exps + 2;
    p.col_part = dbias ? col_part + (size_t)chunk0 * N : nullptr;
    const int row_chunks = (rows + kGradRows - 1) / kGradRows;
    sgc::loss_grad_kernel<<<dim3((unsigned)((N + 255) / 256), (unsigned)row_chunks, 1), 256, 0, st>>>(p);
    if ((rc = sgc::launched(h))) return rc;
    chunk0 += row_chunks;
    const Packed dz{ghi, glo, ldz, exps + 2};
    sgc::LinearEpilogue le;
    memset(&le, 0, sizeof(le));
    if (dX && (rc = sgc::linear_product_any(nk ? sgc::kFormKM : sgc::kFormKK, h, rows, K, N, dz, pw, dX + (int64_t)r0 * lddx, lddx, le, st)))
      return rc;
    if (dW) {
      if (r0 > 0) { le.R = dW; le.ldr = lddw; }
      rc = nk ? sgc::linear_product_any(sgc::kFormMM, h, N, K, rows, dz, x, dW, lddw, le, st)
              : sgc::linear_product_any(sgc::kFormMM, h, K, N, rows, x, dz, dW, lddw, le, st);
      if (rc) return rc;
    }
  }
  if (dbias) {
    sgc::loss_column_sums_kernel<<<(unsigned)((N + 255) / 256), 256, 0, st>>>(col_part, chunk0, N, dbias);
    return sgc::launched(h);
  }
  return SGEMM_CUBE_OK;
}

}  // extern "C"
