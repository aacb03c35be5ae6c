// Entry points of the linear layer on the split product (contracts: include/sgemm_cube.h): packing of
// operands, the layer with bias, activation and residual, and its gradients.
#include "ctx.cuh"
#include "gemm_tc.cuh"
#include "linear_kernels.cuh"
#include "product_host.cuh"
#include "short_batch.cuh"

namespace {

using sgc::blocks_for;
using sgc::Carve;
using sgc::check_operand;
using sgc::is_packed;
using sgc::kExpWords;
using sgc::kGridWords;
using sgc::kRangeWords;
using sgc::launch_pack;
using sgc::launched;
using sgc::linear_config;
using sgc::linear_product_any;
using sgc::Packed;
using sgc::PackJob;
using sgc::words_of;

bool takes_vec4(const void* p, int64_t ld, int cols) { return aligned16(p) && ld % 4 == 0 && cols % 4 == 0; }

PackJob pack_job(int rows, int cols, const float* X, int64_t ldx, uint16_t* hi, uint16_t* lo, int64_t ldh, int* exp) {
  PackJob j;
  memset(&j, 0, sizeof(j));
  j.rows = rows; j.cols = cols; j.X = X; j.ldx = ldx;
  j.hi = hi; j.lo = lo; j.ldh = ldh; j.exp = exp;
  j.vec = takes_vec4(X, ldx, cols);
  return j;
}
long long elements(const PackJob& j) { return (long long)j.rows * j.cols; }

sgc::GridWords* grid_words(sgemm_cube_ctx* h) { return reinterpret_cast<sgc::GridWords*>(h->err_dev + kGridWords); }

template <typename K>
int resident_blocks(sgemm_cube_ctx* h, K kernel, int* cached) {
  if (*cached == 0) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, 256, 0) != cudaSuccess) { cudaGetLastError(); per_sm = 0; }
    *cached = per_sm > 0 ? per_sm * h->sm_count : -1;
  }
  return *cached;
}
template <typename... P, typename... A>
int launch_cooperative(sgemm_cube_ctx* h, void (*kernel)(P...), dim3 grid, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3(256, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute a;
  a.id = cudaLaunchAttributeCooperative;
  a.val.cooperative = 1;
  cfg.attrs = &a;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  h->launches++;
  return SGEMM_CUBE_OK;
}

}  // namespace

// Range and split of one job, or of two in the same launches (the blocks in proportion to the elements).
int sgc::launch_pack(sgemm_cube_ctx* h, const PackJob* jobs, int n, cudaStream_t st) {
  const long long ea = elements(jobs[0]), eb = n == 2 ? elements(jobs[1]) : 0;
  const PackJob& b = jobs[n == 2 ? 1 : 0];
  // one cooperative launch where the blocks that are resident at once hold everything
  const long long items_a = (long long)jobs[0].rows * ((jobs[0].cols + 7) / 8);
  const long long items_b = n == 2 ? (long long)b.rows * ((b.cols + 7) / 8) : 0;
  const int resident = resident_blocks(h, sgc::pack_once_kernel, &h->pack_once_blocks);
  long long once_a = (items_a + 255) / 256, once_b = (items_b + 255) / 256;
  if (once_a + once_b > resident && n == 2) {            // fewer blocks with more items each, in proportion
    once_b = (long long)((double)resident * (double)items_b / (double)(items_a + items_b) + 0.5);
    once_b = once_b < 1 ? 1 : (once_b > resident - 1 ? resident - 1 : once_b);
    once_a = resident - once_b;
  } else if (once_a > resident) {
    once_a = resident;
  }
  const long long held = 256ll * sgc::kOnceItems;
  if (resident >= 2 && items_a <= once_a * held && items_b <= once_b * held) {
    const int rc = launch_cooperative(h, sgc::pack_once_kernel, dim3((unsigned)(once_a + once_b), 1, 1), st, jobs[0], b,
                                      (unsigned)once_a, grid_words(h), h->err_dev);
    if (rc == SGEMM_CUBE_OK) return rc;                  // else: a device that is partly occupied by others
  }
  for (int phase = 0; phase < 2; ++phase) {
    int blocks = blocks_for(h, (ea + eb) / (phase == 0 ? 16 : 8) + 1), blocks_a = blocks;
    if (n == 2) {
      if (blocks < 2) blocks = 2;
      blocks_a = (int)((double)blocks * (double)ea / (double)(ea + eb) + 0.5);
      blocks_a = blocks_a < 1 ? 1 : (blocks_a > blocks - 1 ? blocks - 1 : blocks_a);
    }
    if (phase == 0)
      sgc::pack_range_kernel<<<blocks, 256, 0, st>>>(jobs[0], b, (unsigned)blocks_a, h->err_dev + kRangeWords);
    else
      sgc::pack_split_kernel<<<blocks, 256, 0, st>>>(jobs[0], b, (unsigned)blocks_a);
    const int rc = launched(h);
    if (rc) return rc;
  }
  return SGEMM_CUBE_OK;
}

namespace {

template <int NT, bool W_F32>
int short_batch_attrs() {
  constexpr int smem = (int)sgc::ShortBatchCfg<NT, W_F32>::SMEM_BYTES;
  constexpr cudaFuncAttribute a = cudaFuncAttributeMaxDynamicSharedMemorySize;
  if (cudaFuncSetAttribute(sgc::short_batch_kernel<NT, false, W_F32>, a, smem) != cudaSuccess ||
      cudaFuncSetAttribute(sgc::short_batch_kernel<NT, true, W_F32>, a, smem) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  return SGEMM_CUBE_OK;
}
int linear_setup(sgemm_cube_ctx* h) {
  sgc::ResidentClusters& k = h->linear_clusters;
  if (k.ready) return SGEMM_CUBE_OK;
  int rc;
  if ((rc = short_batch_attrs<16, false>()) || (rc = short_batch_attrs<32, false>()) || (rc = short_batch_attrs<64, false>()) ||
      (rc = short_batch_attrs<16, true>()) || (rc = short_batch_attrs<32, true>()) || (rc = short_batch_attrs<64, true>()))
    return rc;
  return sgc::product_setup<sgc::kFormKM, sgc::kFormKK, sgc::kFormMM>(h, k);
}

// C (M x N) = epilogue of A B on packed operands, termwise.
template <int FORM>
int linear_product(sgemm_cube_ctx* h, int M, int N, int K, const Packed& A, const Packed& B, float* Y, int64_t ldy,
                   sgc::LinearEpilogue ep, cudaStream_t st) {
  const int rc = linear_setup(h);
  if (rc) return rc;
  ep.exp_a = A.exp;
  ep.exp_b = B.exp;
  ep.vec = aligned16(Y) && ldy % 4 == 0 && (!ep.Z || (aligned16(ep.Z) && ep.ldz % 4 == 0)) &&
           (!ep.R || (aligned16(ep.R) && ep.ldr % 4 == 0));
  sgc::TcLinearParams p;
  memset(&p, 0, sizeof(p));
  p.M = M; p.N = N; p.K = K;
  p.D = Y; p.ldd = ldy;
  p.ep = ep;
  // Nothing but the way back to do: the accumulate warps store to Y themselves.
  const bool scratch = ep.bias || ep.R || ep.Z || ep.act != SGEMM_CUBE_ACT_NONE;
  return sgc::run_product<FORM>(h, h->linear_clusters, A, B, p, scratch, st);
}

}  // namespace

int sgc::linear_product_any(int form, sgemm_cube_ctx* h, int M, int N, int K, const Packed& A, const Packed& B, float* Y,
                            int64_t ldy, const LinearEpilogue& ep, cudaStream_t st) {
  if (form == sgc::kFormKM) return linear_product<sgc::kFormKM>(h, M, N, K, A, B, Y, ldy, ep, st);
  if (form == sgc::kFormKK) return linear_product<sgc::kFormKK>(h, M, N, K, A, B, Y, ldy, ep, st);
  return linear_product<sgc::kFormMM>(h, M, N, K, A, B, Y, ldy, ep, st);
}

namespace {

// ------------------------------------------------------------------------------------------ few rows
// Which calls the FMA kernels take: their arithmetic grows with the rows, the tensor cores' costs a longer start
// (cold cache, times with the launches' own).
//   packed, outputs x inputs: one row (16384 x 4096 57 us, 65 on the tensor cores; 1024 x 1024 10 and 14), and up to four
//   of a weight below 8 million elements (2048 x 2048 16 and 18; but 4096 x 4096 29 and 27); inputs x outputs: never
//   (one row of 1024 x 4096 33 and 18)
//   FP32: up to four rows (4096 x 4096 31 and 34), up to eight below 2 million elements (1024 x 1024 12 and 18; but 8 rows
//   of 2048 x 2048 28 and 23, of 16384 x 4096 164 and 86)
constexpr int kFewRows = 8;

bool use_few_rows(int M, int N, int K, bool packed, bool nk) {
  const long long weights = (long long)N * K;
  if (!packed) return M <= 4 || (M <= kFewRows && weights < (1ll << 21));
  return nk && (M == 1 || (M <= 4 && weights < (1ll << 23)));
}

template <int MR, int LOAD>
int launch_few_nk(sgemm_cube_ctx* h, const sgc::FewRowsParams& p, cudaStream_t st) {
  constexpr int NR = MR == 8 ? 2 : 4;
  const long long outs = (p.N + NR - 1) / NR;
  int ksplit = 1;
  while (ksplit < 8 && outs * ksplit < (long long)h->sm_count * 16 && ksplit * 2 * 256 <= p.K) ksplit *= 2;
  const int per_block = 8 / ksplit;
  sgc::few_rows_nk_kernel<MR, NR, LOAD><<<(unsigned)((outs + per_block - 1) / per_block), 256, 0, st>>>(p, ksplit);
  return launched(h);
}
template <int MR, int LOAD>
int launch_few_kn(sgemm_cube_ctx* h, const sgc::FewRowsParams& p, cudaStream_t st) {
  const int cols = (p.N + 127) / 128;
  int slices = 1;
  while (slices < 8 && (long long)cols * slices < 2 * h->sm_count && p.K / (slices * 2) >= 64) slices *= 2;
  for (;; slices = 1) {                                              // clusters that cannot be scheduled: whole k
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = 1; a.val.clusterDim.y = (unsigned)slices; a.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)cols, (unsigned)slices, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.dynamicSmemBytes = 8 * MR * 128 * sizeof(float);
    cfg.stream = st;
    cfg.attrs = &a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, sgc::few_rows_kn_kernel<MR, LOAD>, p, (p.K + slices - 1) / slices) == cudaSuccess) break;
    cudaGetLastError();
    if (slices == 1) return SGEMM_CUBE_CUDA_ERROR;
  }
  h->launches++;
  return SGEMM_CUBE_OK;
}
template <int LOAD>
int launch_few(sgemm_cube_ctx* h, const sgc::FewRowsParams& p, bool nk, cudaStream_t st) {
  if constexpr (LOAD == sgc::kLoadPacked) {
    if (p.M == 1) return launch_few_nk<1, LOAD>(h, p, st);
    return p.M == 2 ? launch_few_nk<2, LOAD>(h, p, st) : launch_few_nk<4, LOAD>(h, p, st);
  } else {
    if (p.M == 1) return nk ? launch_few_nk<1, LOAD>(h, p, st) : launch_few_kn<1, LOAD>(h, p, st);
    if (p.M == 2) return nk ? launch_few_nk<2, LOAD>(h, p, st) : launch_few_kn<2, LOAD>(h, p, st);
    if (p.M <= 4) return nk ? launch_few_nk<4, LOAD>(h, p, st) : launch_few_kn<4, LOAD>(h, p, st);
    return nk ? launch_few_nk<8, LOAD>(h, p, st) : launch_few_kn<8, LOAD>(h, p, st);
  }
}

// ------------------------------------------------------------------------------------------ short batches
// Rows and blocks of 64 k for which the short-batch kernel is the faster one (cold cache, times with the launches' own):
//   up to 64 rows always: 4096 x 4096 with 16 rows 29 us, 50 on the 128-row tiles; 16384 x 4096 with 64 rows 70 and 89;
//   up to 256 where its 64-row tiles fit the SMs at once and have little to do each: 128 rows of 4096 x 4096 (32 blocks)
//   43 and 52, 256 of 4096 x 1024 (16 blocks) 27 and 38; but 160 of 4096 x 4096 (64 blocks) 70 and 58, 65 of
//   16384 x 4096 (two turns of tiles) 129 and 89.
constexpr int kShortRows = 64, kShortMoreRows = 256, kShortMoreBlocks = 32;

bool use_short_batch(const sgemm_cube_ctx* h, int M, int N, int K, int* slices) {
  const int nt = M <= 16 ? 16 : (M <= 32 ? 32 : 64);
  const long long tiles = (long long)((N + sgc::kShortN - 1) / sgc::kShortN) * ((M + nt - 1) / nt);
  *slices = sgc::product_slices(h, h->linear_clusters, tiles, K, 2 * sgc::kShortK);
  if (M <= kShortRows) return true;
  const int blocks = (K + sgc::kShortK - 1) / sgc::kShortK;
  return M <= kShortMoreRows && tiles <= h->sm_count && (blocks + *slices - 1) / *slices <= kShortMoreBlocks;
}

template <int NT, bool W_MN, bool W_F32>
int launch_short(sgemm_cube_ctx* h, const sgemm_cube_operand& W, sgc::ShortBatchParams p, int slices, cudaStream_t st) {
  using Cfg = sgc::ShortBatchCfg<NT, W_F32>;
  constexpr CUtensorMapDataType f16 = CU_TENSOR_MAP_DATA_TYPE_FLOAT16, f32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
  constexpr CUtensorMapSwizzle swizzle = W_F32 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
  CUtensorMap tm[2];
  for (int w = 0; w < (W_F32 ? 1 : 2); ++w) {
    const void* words = W_F32 ? static_cast<const void*>(W.f32_dev) : (w ? W.lo_dev : W.hi_dev);
    const int64_t ld = W_F32 ? W.ld : W.ld16;
    const size_t size = W_F32 ? 4 : 2;
    const int rc = W_MN ? make_map(h, &tm[w], W_F32 ? f32 : f16, size, words, p.N, p.K, ld, W_F32 ? sgc::kShortN : 64, sgc::kShortK, swizzle)
                        : make_map(h, &tm[w], W_F32 ? f32 : f16, size, words, p.K, p.N, ld, sgc::kShortK, sgc::kShortN, swizzle);
    if (rc) return rc;
  }
  if (W_F32) tm[1] = tm[0];
  const int blocks = (p.K + sgc::kShortK - 1) / sgc::kShortK;
  p.row_tiles = (p.M + NT - 1) / NT;
  for (;; slices = 1) {                                              // clusters that cannot be scheduled: whole k
    p.kslice_blocks = (blocks + slices - 1) / slices;
    p.ksplit = (blocks + p.kslice_blocks - 1) / p.kslice_blocks;     // no slice is empty
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = linear_config(Cfg::SMEM_BYTES, (unsigned)p.ksplit, &attr, st);
    cfg.blockDim = dim3(sgc::kShortThreads, 1, 1);
    cfg.gridDim = dim3((unsigned)((p.N + sgc::kShortN - 1) / sgc::kShortN * p.row_tiles * p.ksplit), 1, 1);
    if (cudaLaunchKernelEx(&cfg, sgc::short_batch_kernel<NT, W_MN, W_F32>, tm[0], tm[1], p) == cudaSuccess) break;
    cudaGetLastError();
    if (slices == 1) return SGEMM_CUBE_CUDA_ERROR;
  }
  h->launches++;
  return SGEMM_CUBE_OK;
}
template <int NT>
int launch_short(sgemm_cube_ctx* h, const sgemm_cube_operand& W, const sgc::ShortBatchParams& p, bool nk, int slices, cudaStream_t st) {
  if (W.f32_dev)
    return nk ? launch_short<NT, false, true>(h, W, p, slices, st) : launch_short<NT, true, true>(h, W, p, slices, st);
  return nk ? launch_short<NT, false, false>(h, W, p, slices, st) : launch_short<NT, true, false>(h, W, p, slices, st);
}

// ------------------------------------------------------------------------------------------ arguments
}  // namespace

int sgc::check_operand(const sgemm_cube_operand* o, int rows, int cols) {
  if (!o) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0 || cols == 0) return SGEMM_CUBE_OK;              // an empty operand is not looked at
  if (o->f32_dev) return o->ld >= cols && !misplaced(4, o->f32_dev) ? SGEMM_CUBE_OK : SGEMM_CUBE_INVALID_ARG;
  if (!o->hi_dev || !o->lo_dev || !o->exp_dev || o->ld16 < cols || misplaced(4, o->exp_dev)) return SGEMM_CUBE_INVALID_ARG;
  if (!aligned16(o->hi_dev) || !aligned16(o->lo_dev) || o->ld16 % 8) return SGEMM_CUBE_MISALIGNED;
  return SGEMM_CUBE_OK;
}
namespace {

bool bad_layout(int layout) { return layout != SGEMM_CUBE_WEIGHT_KN && layout != SGEMM_CUBE_WEIGHT_NK; }
bool bad_act(int act) { return act < SGEMM_CUBE_ACT_NONE || act > SGEMM_CUBE_ACT_SILU; }

}  // namespace

// The words of an operand: its own, or (FP32) room in the workspace and a job that fills it.
sgc::Packed sgc::words_of(const sgemm_cube_operand* o, int rows, int cols, Carve& c, int* exp, PackJob* jobs, int* n_jobs) {
  if (is_packed(o)) return Packed{o->hi_dev, o->lo_dev, o->ld16, o->exp_dev};
  const int64_t ld = (int64_t)round_up((size_t)cols, 8);
  uint16_t* hi = c.take<uint16_t>((size_t)rows * ld);
  uint16_t* lo = c.take<uint16_t>((size_t)rows * ld);
  jobs[(*n_jobs)++] = pack_job(rows, cols, o->f32_dev, o->ld, hi, lo, ld, exp);
  return Packed{hi, lo, ld, exp};
}

bool sgc::linear_takes_few(sgemm_cube_ctx* h, int M, int N, int K, bool packed, bool nk) {
  int slices;
  return use_few_rows(M, N, K, packed, nk) || (linear_setup(h) == SGEMM_CUBE_OK && use_short_batch(h, M, N, K, &slices));
}

namespace {

template <int ACT>
int launch_dz(sgemm_cube_ctx* h, const PackJob& j, bool split, float* col_part, int chunks, int rows_per_chunk,
              float* dbias, cudaStream_t st) {
  const dim3 once((unsigned)((j.cols + 127) / 128), (unsigned)((j.rows + sgc::kOnceRows - 1) / sgc::kOnceRows), 1);
  if (split && (long long)once.x * once.y <= resident_blocks(h, sgc::dz_once_kernel<ACT>, &h->dz_once_blocks[ACT]) &&
      launch_cooperative(h, sgc::dz_once_kernel<ACT>, once, st, j, col_part, dbias, grid_words(h), h->err_dev) ==
          SGEMM_CUBE_OK)
    return SGEMM_CUBE_OK;
  const dim3 grid((unsigned)((j.cols + 127) / 128), (unsigned)chunks, 1);
  sgc::dz_range_kernel<ACT><<<grid, 256, 0, st>>>(j, col_part, rows_per_chunk, split ? h->err_dev + kRangeWords : nullptr);
  int rc = launched(h);
  if (rc) return rc;
  const int sum_blocks = dbias ? (j.cols + 255) / 256 : 0;
  if (split) {
    const int blocks = blocks_for(h, (long long)j.rows * ((j.cols + 7) / 8)) + sum_blocks;
    sgc::dz_split_kernel<ACT><<<blocks, 256, 0, st>>>(j, (unsigned)sum_blocks, col_part, chunks, dbias);
    return launched(h);
  }
  if (dbias) {
    sgc::column_parts_kernel<<<sum_blocks, 256, 0, st>>>(col_part, chunks, j.cols, dbias);
    return launched(h);
  }
  return SGEMM_CUBE_OK;
}

int zero_matrix(float* p, int64_t ld, int rows, int cols, cudaStream_t st) {
  if (!p || rows == 0 || cols == 0) return SGEMM_CUBE_OK;
  if (cudaMemset2DAsync(p, (size_t)ld * 4, 0, (size_t)cols * 4, rows, st) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  return SGEMM_CUBE_OK;
}

}  // namespace

extern "C" {

int sgemm_cube_pack(sgemm_cube_handle h, int rows, int cols, const float* X, int64_t ldx, uint16_t* hi, uint16_t* lo,
                    int64_t ld16, int32_t* exp, void* stream) {
  if (!h) return SGEMM_CUBE_INVALID_ARG;
  if (bad_dims(rows, cols) || ldx < cols || ld16 < cols) return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0 || cols == 0) return SGEMM_CUBE_OK;
  if (!X || !hi || !lo || !exp || misplaced(4, X, exp)) return SGEMM_CUBE_INVALID_ARG;
  if (!aligned16(hi) || !aligned16(lo) || ld16 % 8) return SGEMM_CUBE_MISALIGNED;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  const PackJob j = pack_job(rows, cols, X, ldx, hi, lo, ld16, exp);
  return launch_pack(h, &j, 1, static_cast<cudaStream_t>(stream));
}

int sgemm_cube_linear(sgemm_cube_handle h, int M, int N, int K, const sgemm_cube_operand* X,
                      const sgemm_cube_operand* W, int weight_layout, const float* bias, const float* R, int64_t ldr,
                      int activation, float* Y, int64_t ldy, float* Z, int64_t ldz, void* stream) {
  if (!h || bad_dims(M, N, K) || bad_layout(weight_layout) || bad_act(activation)) return SGEMM_CUBE_INVALID_ARG;
  const bool nk = weight_layout == SGEMM_CUBE_WEIGHT_NK;
  int rc = check_operand(X, M, K);
  if (rc) return rc;
  if ((rc = nk ? check_operand(W, N, K) : check_operand(W, K, N))) return rc;
  if (M == 0 || N == 0) return SGEMM_CUBE_OK;
  if (!Y || ldy < N || (R && ldr < N) || (Z && ldz < N)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(4, bias, R, Y, Z)) return SGEMM_CUBE_INVALID_ARG;
  if (Z && (Z == Y || Z == R)) return SGEMM_CUBE_INVALID_ARG;
  if (R == Y && ldr != ldy && M > 1) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  sgc::LinearEpilogue ep;
  memset(&ep, 0, sizeof(ep));
  ep.bias = bias;
  ep.R = R; ep.ldr = ldr;
  ep.Z = Z; ep.ldz = ldz;
  ep.act = activation;
  if (K == 0) {
    sgc::linear_empty_kernel<<<blocks_for(h, (long long)M * N), 256, 0, st>>>(M, N, Y, ldy, ep);
    return launched(h);
  }
  if (!is_packed(X) && use_few_rows(M, N, K, is_packed(W), nk)) {
    sgc::FewRowsParams p;
    memset(&p, 0, sizeof(p));
    p.M = M; p.N = N; p.K = K;
    p.X = X->f32_dev; p.ldx = X->ld;
    p.Y = Y; p.ldy = ldy;
    p.xvec = aligned16(p.X) && p.ldx % 4 == 0;
    p.ep = ep;
    if (is_packed(W)) {
      p.Whi = W->hi_dev; p.Wlo = W->lo_dev; p.ldw = W->ld16;
      p.ep.exp_b = W->exp_dev;
      return launch_few<sgc::kLoadPacked>(h, p, nk, st);
    }
    p.W = W->f32_dev; p.ldw = W->ld;
    if (takes_vec4(p.W, p.ldw, nk ? K : N)) return launch_few<sgc::kLoadF32Vec>(h, p, nk, st);
    return launch_few<sgc::kLoadF32>(h, p, nk, st);
  }
  PackJob jobs[2];
  int n_jobs = 0, slices = 1;
  int* exps = reinterpret_cast<int*>(h->err_dev + kExpWords);
  const int w_rows = nk ? N : K, w_cols = nk ? K : N;
  if ((rc = linear_setup(h))) return rc;                 // clusters that are resident: the choices below look at them
  const bool short_batch = !is_packed(X) && use_short_batch(h, M, N, K, &slices);
  Carve size;
  if (!short_batch) words_of(X, M, K, size, exps, jobs, &n_jobs);
  // An FP32 weight that TMA can read is split inside the kernel, by every tile of rows for itself: 128 rows of
  // 2048 x 2048 29 us, 34 with packing first; 256 rows of 1024 x 1024 21 and 26, of 4096 x 1024 43 and 40.
  const bool direct = short_batch && W->f32_dev && aligned16(W->f32_dev) && W->ld % 4 == 0;
  if (!direct) words_of(W, w_rows, w_cols, size, exps + 1, jobs, &n_jobs);
  if (size.used && (rc = grow(h, &h->ws, &h->ws_bytes, size.used, st))) return rc;
  Carve c;
  c.base = static_cast<uint8_t*>(h->ws);
  n_jobs = 0;
  Packed px{}, pw{};                                    // (what a form does not pack has no exponent)
  if (!short_batch) px = words_of(X, M, K, c, exps, jobs, &n_jobs);
  if (!direct) pw = words_of(W, w_rows, w_cols, c, exps + 1, jobs, &n_jobs);
  if (n_jobs && (rc = launch_pack(h, jobs, n_jobs, st))) return rc;
  if (short_batch) {
    sgc::ShortBatchParams p;
    memset(&p, 0, sizeof(p));
    p.M = M; p.N = N; p.K = K;
    p.X = X->f32_dev; p.ldx = X->ld;
    p.xvec = aligned16(p.X) && p.ldx % 4 == 0;
    p.Y = Y; p.ldy = ldy;
    p.err = h->err_dev;
    p.ep = ep;
    p.ep.exp_b = pw.exp;
    sgemm_cube_operand w = *W;
    if (!direct) w = sgemm_cube_operand{nullptr, 0, pw.hi, pw.lo, pw.ld, pw.exp};
    if (M <= 16) return launch_short<16>(h, w, p, nk, slices, st);
    return M <= 32 ? launch_short<32>(h, w, p, nk, slices, st) : launch_short<64>(h, w, p, nk, slices, st);
  }
  return linear_product_any(nk ? sgc::kFormKK : sgc::kFormKM, h, M, N, K, px, pw, Y, ldy, ep, st);
}

int sgemm_cube_linear_backward(sgemm_cube_handle h, int M, int N, int K, const float* dY, int64_t lddy, const float* Z,
                               int64_t ldz, int activation, const sgemm_cube_operand* X, const sgemm_cube_operand* W,
                               int weight_layout, float* dX, int64_t lddx, float* dW, int64_t lddw, float* dbias,
                               void* stream) {
  if (!h || bad_dims(M, N, K) || bad_layout(weight_layout) || bad_act(activation)) return SGEMM_CUBE_INVALID_ARG;
  const bool nk = weight_layout == SGEMM_CUBE_WEIGHT_NK;
  const int w_rows = nk ? N : K, w_cols = nk ? K : N;
  int rc;
  if (dW && (rc = check_operand(X, M, K))) return rc;
  if (dX && (rc = check_operand(W, w_rows, w_cols))) return rc;
  if ((dX && lddx < K) || (dW && lddw < w_cols) || misplaced(4, dX, dW, dbias)) return SGEMM_CUBE_INVALID_ARG;
  if (M > 0 && N > 0) {
    if (!dY || lddy < N || misplaced(4, dY)) return SGEMM_CUBE_INVALID_ARG;
    if (activation != SGEMM_CUBE_ACT_NONE && (!Z || ldz < N || misplaced(4, Z))) return SGEMM_CUBE_INVALID_ARG;
  }
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (M == 0 || N == 0) {                        // empty sums
    if ((rc = zero_matrix(dX, lddx, M, K, st))) return rc;
    if ((rc = zero_matrix(dW, lddw, w_rows, w_cols, st))) return rc;
    return zero_matrix(dbias, N, 1, N, st);
  }
  if (K == 0) dX = dW = nullptr;                 // no elements
  const bool split = dX || dW;
  if (!split && !dbias) return SGEMM_CUBE_OK;
  // Row chunks of the column sums: about eight blocks an SM in all, at least kOnceRows rows a chunk.  That is what
  // they have where the one-launch form fits (at most four blocks an SM), so both forms add in the same order.
  const int col_blocks = (N + 127) / 128;
  int chunks = (8 * h->sm_count + col_blocks - 1) / col_blocks;
  const int most = (M + sgc::kOnceRows - 1) / sgc::kOnceRows;
  if (chunks > most) chunks = most;
  const int rows_per_chunk = (int)round_up((size_t)((M + chunks - 1) / chunks), sgc::kOnceRows);
  chunks = (M + rows_per_chunk - 1) / rows_per_chunk;
  PackJob jobs[2];
  int n_jobs = 0;
  int* exps = reinterpret_cast<int*>(h->err_dev + kExpWords);
  const int64_t ldg = (int64_t)round_up((size_t)N, 8);
  Packed px{}, pw{};
  uint16_t *ghi = nullptr, *glo = nullptr;
  float* col_part = nullptr;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->ws) : nullptr;
    n_jobs = 0;
    if (dW) px = words_of(X, M, K, c, exps, jobs, &n_jobs);
    if (dX) pw = words_of(W, w_rows, w_cols, c, exps + 1, jobs, &n_jobs);
    if (split) {
      ghi = c.take<uint16_t>((size_t)M * ldg);
      glo = c.take<uint16_t>((size_t)M * ldg);
    }
    if (dbias) col_part = c.take<float>((size_t)chunks * N);
    if (!pass && (rc = grow(h, &h->ws, &h->ws_bytes, c.used, st))) return rc;
  }
  if (n_jobs && (rc = launch_pack(h, jobs, n_jobs, st))) return rc;
  PackJob j = pack_job(M, N, dY, lddy, ghi, glo, ldg, exps + 2);
  if (activation != SGEMM_CUBE_ACT_NONE) {
    j.Z = Z; j.ldz = ldz;
    j.vec = j.vec && takes_vec4(Z, ldz, N);
  }
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU: rc = launch_dz<sgc::kActRelu>(h, j, split, col_part, chunks, rows_per_chunk, dbias, st); break;
    case SGEMM_CUBE_ACT_GELU: rc = launch_dz<sgc::kActGelu>(h, j, split, col_part, chunks, rows_per_chunk, dbias, st); break;
    case SGEMM_CUBE_ACT_GELU_TANH: rc = launch_dz<sgc::kActGeluTanh>(h, j, split, col_part, chunks, rows_per_chunk, dbias, st); break;
    case SGEMM_CUBE_ACT_SILU: rc = launch_dz<sgc::kActSilu>(h, j, split, col_part, chunks, rows_per_chunk, dbias, st); break;
    default: rc = launch_dz<sgc::kActNone>(h, j, split, col_part, chunks, rows_per_chunk, dbias, st); break;
  }
  if (rc) return rc;
  const Packed pg{ghi, glo, ldg, exps + 2};
  sgc::LinearEpilogue ep;
  memset(&ep, 0, sizeof(ep));
  // dX (M x K) = dz W^T: dz contiguous along the contracted N; W contiguous along N (KN) or K (NK).
  if (dX && (rc = linear_product_any(nk ? sgc::kFormKM : sgc::kFormKK, h, M, K, N, pg, pw, dX, lddx, ep, st))) return rc;
  // dW = dz^T X (NK) or X^T dz (KN): the contracted index runs over rows of both.
  if (dW) {
    if (nk) return linear_product<sgc::kFormMM>(h, N, K, M, pg, px, dW, lddw, ep, st);
    return linear_product<sgc::kFormMM>(h, K, N, M, px, pg, dW, lddw, ep, st);
  }
  return SGEMM_CUBE_OK;
}

}  // extern "C"
