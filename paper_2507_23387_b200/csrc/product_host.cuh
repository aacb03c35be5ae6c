// Launching the forms of the tensor-core product that work on packed operands (the linear layer, the cross entropy's
// logits, the products of an orthogonalised update).  Host code; used by the translation units that instantiate them.
#pragma once

#include "ctx.cuh"
#include "gemm_tc.cuh"
#include "pack_job.cuh"

namespace sgc {

constexpr int kMaxSlices = 8;          // blocks of a portable cluster

inline int launched(sgemm_cube_ctx* h) {
  h->launches++;
  return cudaGetLastError() == cudaSuccess ? SGEMM_CUBE_OK : SGEMM_CUBE_CUDA_ERROR;
}
inline int blocks_for(const sgemm_cube_ctx* h, long long items) {
  const long long b = (items + 255) / 256, cap = (long long)h->sm_count * 16;
  return (int)(b < 1 ? 1 : (b < cap ? b : cap));
}

// Words of the handle's device scratch: running maxima and block counts of up to two packing jobs, exponents of operands
// that a call packs itself, and the words in which the blocks of a one-launch kernel meet.
// Every call leaves the first and the last four zero; after a kernel that gave up sgemm_cube_check does.
constexpr int kRangeWords = 20, kExpWords = 24, kGridWords = 28;

// Pieces of the handle's workspace, in the order they are asked for.
struct Carve {
  size_t used = 0;
  uint8_t* base = nullptr;
  template <typename T>
  T* take(size_t n) {
    T* p = reinterpret_cast<T*>(base + used);
    used += round_up(n * sizeof(T), 256);
    return p;
  }
};

// Of linear_api.cu: what an operand has to be, whether it is packed, its words (its own, or room in the workspace and a
// job that fills it), and running up to two jobs.
int check_operand(const sgemm_cube_operand* o, int rows, int cols);
inline bool is_packed(const sgemm_cube_operand* o) { return o->f32_dev == nullptr && o->hi_dev != nullptr; }
Packed words_of(const sgemm_cube_operand* o, int rows, int cols, Carve& c, int* exp, PackJob* jobs, int* n_jobs);
int launch_pack(sgemm_cube_ctx* h, const PackJob* jobs, int n, cudaStream_t st);
// C (M x N) = epilogue of A B on packed operands, termwise, in one of the linear layer's forms.
int linear_product_any(int form, sgemm_cube_ctx* h, int M, int N, int K, const Packed& A, const Packed& B, float* Y,
                       int64_t ldy, const LinearEpilogue& ep, cudaStream_t st);
// Whether sgemm_cube_linear multiplies an FP32 X of M rows in one of its forms for few rows or a short batch.
bool linear_takes_few(sgemm_cube_ctx* h, int M, int N, int K, bool packed, bool nk);

inline cudaLaunchConfig_t linear_config(size_t smem, unsigned cluster, cudaLaunchAttribute* attr, cudaStream_t st) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.blockDim = dim3(kLinearThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  if (cluster > 1) {
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = cluster; attr->val.clusterDim.y = 1; attr->val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  return cfg;
}
// Kernel attributes, and how many clusters of pairs and of 2 to 8 split-K blocks are resident at once (the fewest
// over the forms of a family).
template <int FORM, bool PAIR>
int product_attrs(const sgemm_cube_ctx* h, ResidentClusters& k) {
  auto kernel = tc_gemm_kernel<3, false, PAIR, false, FORM>;
  constexpr size_t smem = TcCfg<3, PAIR, false>::SMEM_BYTES;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  for (int c = 2; c <= (PAIR ? 2 : kMaxSlices); ++c) {
    cudaLaunchAttribute a;
    cudaLaunchConfig_t cfg = linear_config(smem, (unsigned)c, &a, nullptr);
    cfg.gridDim = dim3((unsigned)(c * h->sm_count), 1, 1);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
    int& least = PAIR ? k.pairs : k.slices[c];
    if (n < least) least = n;
  }
  return SGEMM_CUBE_OK;
}
template <int... FORMS>
int product_setup(const sgemm_cube_ctx* h, ResidentClusters& k) {
  if (k.ready) return SGEMM_CUBE_OK;
  k.pairs = h->sm_count;
  for (int& n : k.slices) n = h->sm_count;
  int rc = SGEMM_CUBE_OK;
  (void)((rc == SGEMM_CUBE_OK && ((rc = product_attrs<FORMS, false>(h, k)) || (rc = product_attrs<FORMS, true>(h, k)), true)) && ...);
  k.ready = rc == SGEMM_CUBE_OK;
  return rc;
}

// Tiles of a product: 128 x 256, or the 256 x 256 of a pair.
template <int FORM>
long long product_tiles(const TcParams<FORM>& p, bool pair) {
  const long long num_m = (p.M + (pair ? 2 : 1) * kBM - 1) / ((pair ? 2 : 1) * kBM), num_n = (p.N + kBN - 1) / kBN;
  if constexpr (epilogue_of(FORM) == kEpiPolynomial) {
    if (p.ep.symmetric) return lower_tiles((int)num_m, pair);
  }
  return num_m * num_n;
}

template <int FORM, bool PAIR>
int launch_product(sgemm_cube_ctx* h, const ResidentClusters& k, const Packed& A, const Packed& B, const TcParams<FORM>& p,
                   cudaStream_t st) {
  using Cfg = TcCfg<3, PAIR, false>;
  constexpr bool a_mn = layout_of(FORM) == kFormMM, b_mn = layout_of(FORM) != kFormKK;
  CUtensorMap tm[4];
  for (int w = 0; w < 2; ++w) {
    const uint16_t* a = w ? A.lo : A.hi;
    const uint16_t* b = w ? B.lo : B.hi;
    const CUtensorMapDataType t = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUtensorMapSwizzle z = CU_TENSOR_MAP_SWIZZLE_128B;
    int rc = a_mn ? make_map(h, &tm[w], t, 2, a, p.M, p.K, A.ld, 64, Cfg::BK, z)
                  : make_map(h, &tm[w], t, 2, a, p.K, p.M, A.ld, Cfg::BK, kBM, z);
    if (rc) return rc;
    rc = b_mn ? make_map(h, &tm[2 + w], t, 2, b, p.N, p.K, B.ld, 64, Cfg::BK, z)
              : make_map(h, &tm[2 + w], t, 2, b, p.K, p.N, B.ld, Cfg::BK, Cfg::BN_CTA, z);
    if (rc) return rc;
  }
  cudaLaunchAttribute attr;
  const unsigned cluster = PAIR ? 2u : (unsigned)p.ksplit;
  cudaLaunchConfig_t cfg = linear_config(Cfg::SMEM_BYTES, cluster, &attr, st);
  const long long tiles = product_tiles<FORM>(p, PAIR);
  const int cap = PAIR ? k.pairs : (cluster > 1 ? k.slices[cluster] : h->sm_count);
  cfg.gridDim = dim3(cluster * (unsigned)(tiles < cap ? tiles : cap), 1, 1);
  h->launches++;
  if (cudaLaunchKernelEx(&cfg, tc_gemm_kernel<3, false, PAIR, false, FORM>, tm[0], tm[1], tm[2], tm[3], p) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  return SGEMM_CUBE_OK;
}

// How many k slices, when the tiles leave half of the SMs idle: the clusters that are resident at once go
// through the tiles in turns, and a turn takes as long as its slice; the fewest slices among those that take the
// least time.  A slice is at least two k-blocks.
inline int product_slices(const sgemm_cube_ctx* h, const ResidentClusters& k, long long tiles, int K, int chunk_k) {
  if (!h->split_k) return 1;
  if (tiles * 2 > h->sm_count) return 1;
  const int chunks = (K + chunk_k - 1) / chunk_k;
  int best = 1;
  long long best_time = chunks;
  for (int s = 2; s <= kMaxSlices && 2 * s <= chunks; ++s) {
    const int per = (chunks + s - 1) / s, clusters = k.slices[s];
    if (clusters < 1 || (chunks + per - 1) / per != s) continue;      // the last slice would be empty
    const long long time = (tiles + clusters - 1) / clusters * per;
    if (time < best_time) { best_time = time; best = s; }
  }
  return best;
}

// A product on packed operands, termwise.  M, N, K and the epilogue come in `p`; `scratch`: its finished tiles go through
// the handle's scratch (the store warps have work to do on them).
template <int FORM>
int run_product(sgemm_cube_ctx* h, const ResidentClusters& k, const Packed& A, const Packed& B, TcParams<FORM>& p, bool scratch,
                cudaStream_t st) {
  constexpr int BK = TcCfg<3, false, false>::BK;
  int rc;
  p.order = SGEMM_CUBE_TERMWISE;
  p.kchunk_blocks = h->kblock_termwise / BK;
  p.inv_scale = kPackInvScale;
  p.scale = 1.f;
  p.err = h->err_dev;
  p.ksplit = 1;
  const long long tiles = product_tiles<FORM>(p, false);
  const int slices = product_slices(h, k, tiles, p.K, p.kchunk_blocks * BK);
  if (slices > 1) {
    rc = grow(h, &h->part_ws, &h->part_ws_bytes, (size_t)tiles * slices * kTileFloats * 4, st);
    if (rc) return rc;
    const int chunks = (p.K + p.kchunk_blocks * BK - 1) / (p.kchunk_blocks * BK);
    p.ksplit = slices;
    p.kslice_blocks = (chunks + slices - 1) / slices * p.kchunk_blocks;
    p.ep.tiles = static_cast<float*>(h->part_ws);
    rc = launch_product<FORM, false>(h, k, A, B, p, st);
    if (rc != SGEMM_CUBE_CUDA_ERROR) return rc;
    p.ksplit = 1;                                        // clusters that cannot be scheduled: whole k
    p.kslice_blocks = 0;
    p.ep.tiles = nullptr;
  }
  if (scratch) {
    rc = grow(h, &h->tile_ws, &h->tile_ws_bytes, (size_t)h->sm_count * 2 * kTileFloats * 4, st);
    if (rc) return rc;
    p.ep.tiles = static_cast<float*>(h->tile_ws);
  }
  const bool pair = (h->cta_pair == 2 ? p.M > kBM : h->cta_pair == 1) && k.pairs > 0;
  if (pair) {
    rc = launch_product<FORM, true>(h, k, A, B, p, st);
    if (rc != SGEMM_CUBE_CUDA_ERROR || h->cta_pair != 2) return rc;
  }
  return launch_product<FORM, false>(h, k, A, B, p, st);
}

}  // namespace sgc
