// A matrix brought near the closest one with orthonormal rows (columns, where it has more rows), by Newton-Schulz products
// (contract: include/sgemm_cube.h):
//
//   X = G / (|G|_F + eps);   steps times:  A = X X^T,  B = b A + c A A,  X <- a X + B X;   O = scale X + beta R
//
// (rows <= columns; else A = X^T X and X <- a X + X B).  X, A and B live as FP16 words from the first pass to the last, written by
// the epilogues of the products that make them (polynomial_epilogue.cuh): no pass of its own packs anything.  Their exponents
// are known beforehand: the singular values of X lie in [0, s] with s = 1 at the start and the polynomial's largest value
// on [0, s] after a step, and no entry of a matrix is larger than its largest singular value.
// A and B are symmetric: half of their tiles are formed.  (a X is added in FP32: as a diagonal of B it went through the tensor
// core's truncating sums, with 128 x 384 and five steps 2.8e-6 off where FP32 products are 1.7e-6.)
// Small matrices take all of it in one launch (polynomial_chain.cuh).
#include <cmath>
#include <type_traits>

#include "ctx.cuh"
#include "elements.cuh"
#include "polynomial_chain.cuh"
#include "product_host.cuh"

namespace sgc {

// Sum of squares of a block's share of G, in FP64: gradients of any FP32 size neither overflow nor vanish.
template <typename T>
__global__ void __launch_bounds__(256)
square_sums_kernel(int rows, int cols, const T* __restrict__ G, long long ldg, int vec, double* __restrict__ sums) {
  constexpr int V = Elem<T>::kVec;
  double s = 0.0;
  const int per_row = vec ? cols / V : cols;
  const long long total = (long long)rows * per_row, stride = (long long)gridDim.x * 256;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < total; it += stride) {
    const long long r = total < (1ll << 31) ? (long long)((uint32_t)it / (uint32_t)per_row) : it / per_row;
    const T* at = G + r * ldg + (it - r * per_row) * (vec ? V : 1);
    if (vec) {
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
  __shared__ double warp_sum[8];
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += warp_sum[w];
    sums[blockIdx.x] = s;
  }
}

// Words of 2^p G / (|G|_F + eps); every block adds the sums for itself, in the same order.
template <typename T>
__global__ void __launch_bounds__(256)
normalise_kernel(int rows, int cols, const T* __restrict__ G, long long ldg, int vec, const double* __restrict__ sums, int n_sums,
                 float eps, float pre, uint16_t* __restrict__ hi, uint16_t* __restrict__ lo, long long ldw) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n_sums; i += 256) s += sums[i];
  for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
  __shared__ double warp_sum[8];
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = s;
  __syncthreads();
  s = warp_sum[0];
  for (int w = 1; w < 8; ++w) s += warp_sum[w];
  float f0, f1;
  norm_factors(s, eps, pre, f0, f1);
  const int per_row = (cols + 7) >> 3;
  const long long total = (long long)rows * per_row, stride = (long long)gridDim.x * 256;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < total; it += stride) {
    const long long r = total < (1ll << 31) ? (long long)((uint32_t)it / (uint32_t)per_row) : it / per_row;
    const int c = (int)(it - r * per_row) << 3;
    normalise_eight(G + r * ldg + c, vec != 0, cols - c, f0, f1, hi + r * ldw + c, lo + r * ldw + c);
  }
}

constexpr int kFormPolyKM = form_of(kFormKM, kEpiPolynomial), kFormPolyKK = form_of(kFormKK, kEpiPolynomial),
              kFormPolyMM = form_of(kFormMM, kEpiPolynomial);

}  // namespace sgc

namespace {

using sgc::Carve;
using sgc::Packed;

struct Words {
  uint16_t* hi;
  uint16_t* lo;
  int64_t ld;
  Packed packed() const { return Packed{hi, lo, ld, nullptr}; }
};
Words take_words(Carve& c, int rows, int cols) {
  const int64_t ld = (int64_t)round_up((size_t)cols, 8);
  uint16_t* hi = c.take<uint16_t>((size_t)rows * ld);
  return Words{hi, c.take<uint16_t>((size_t)rows * ld), ld};
}

// Largest |f| on [0, s], f(x) = x^odd (k0 + k1 x^2 + k2 x^4): at the end, or where the derivative in x^2 vanishes.
double largest_on(double s, double k0, double k1, double k2, int odd) {
  const auto f = [&](double x) { return std::fabs((odd ? x : 1.0) * (k0 + x * x * (k1 + x * x * k2))); };
  double most = std::fmax(f(0.0), f(s));
  // odd: k0 + 3 k1 y + 5 k2 y^2 = 0, else k1 + 2 k2 y = 0, y = x^2
  const double q2 = odd ? 5.0 * k2 : 0.0, q1 = odd ? 3.0 * k1 : 2.0 * k2, q0 = odd ? k0 : k1;
  double roots[2];
  int n = 0;
  if (q2 != 0.0) {
    const double d = q1 * q1 - 4.0 * q2 * q0;
    if (d >= 0.0) {
      const double t = -0.5 * (q1 + std::copysign(std::sqrt(d), q1));
      roots[n++] = t / q2;
      if (t != 0.0) roots[n++] = q0 / t;
    }
  } else if (q1 != 0.0) {
    roots[n++] = -q0 / q1;
  }
  for (int i = 0; i < n; ++i)
    if (roots[i] > 0.0 && roots[i] < s * s) most = std::fmax(most, f(std::sqrt(roots[i])));
  return most;
}
// p with 2^p x below the largest FP16 number for |x| <= bound, a sixteenth of it left for rounding.  At most 60, which X and A do not
// reach: a smaller B vanishes beside a X (a step of B alone would leave less than the smallest singular value that is allowed), its
// words lose bits from 2^-95 on, and 2^p stays FP32's whatever the coefficients.
constexpr int kMostWordExponent = 60;
int word_exponent(double bound) {
  if (!(bound > 0.0)) return 0;                  // a matrix of zeros
  const double p = 15.0 - std::floor(std::log2(bound * 1.0625));
  return p < kMostWordExponent ? (int)p : kMostWordExponent;
}

template <typename T>
int normalise(sgemm_cube_ctx* h, int rows, int cols, const void* G, int64_t ldg, double* sums, int blocks, float eps, float pre,
              const Words& X, cudaStream_t st) {
  const T* g = static_cast<const T*>(G);
  const int vec = sgc::rows_take_vectors(G, ldg, cols, sizeof(T));
  sgc::square_sums_kernel<T><<<blocks, 256, 0, st>>>(rows, cols, g, ldg, vec, sums);
  int rc = sgc::launched(h);
  if (rc) return rc;
  sgc::normalise_kernel<T><<<sgc::blocks_for(h, (long long)rows * ((cols + 7) / 8)), 256, 0, st>>>(rows, cols, g, ldg, vec, sums, blocks,
                                                                                                 eps, pre, X.hi, X.lo, X.ld);
  return sgc::launched(h);
}

template <int FORM>
int polynomial_product(sgemm_cube_ctx* h, int M, int N, int K, const Words& A, const Words& B, const sgc::PolynomialEpilogue& ep,
                       cudaStream_t st) {
  sgc::TcPolynomialParams p;
  memset(&p, 0, sizeof(p));
  p.M = M; p.N = N; p.K = K;
  p.ep = ep;
  return sgc::run_product<FORM>(h, h->polynomial_clusters, A.packed(), B.packed(), p, true, st);
}

struct OrthogonalizeCall {
  int rows, cols, dtype;
  const void* G;
  int64_t ldg;
  int steps;
  float eps;
  const float* R;
  int64_t ldr;
  float scale, beta;
  float* O;
  int64_t ldo;
  bool tall;
  int n, m;                  // the shorter and the longer side
  float pre;                 // 2^p of the first X
  const sgc::ChainStep* step;
  cudaStream_t st;
  int vec_out() const { return aligned16(O) && ldo % 4 == 0 && (!R || (aligned16(R) && ldr % 4 == 0)); }
};

// One launch a product.
int run_products(sgemm_cube_ctx* h, const OrthogonalizeCall& c) {
  int rc = sgc::product_setup<sgc::kFormPolyKM, sgc::kFormPolyKK, sgc::kFormPolyMM>(h, h->polynomial_clusters);
  if (rc) return rc;
  const int blocks = sgc::blocks_for(h, (long long)c.rows * c.cols / 16 + 1);
  Words X[2], A, B;
  double* sums = nullptr;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve w;
    w.base = pass ? static_cast<uint8_t*>(h->poly_ws) : nullptr;
    sums = w.take<double>((size_t)blocks);
    X[0] = take_words(w, c.rows, c.cols);
    X[1] = c.steps > 1 ? take_words(w, c.rows, c.cols) : X[0];
    A = take_words(w, c.n, c.n);
    B = take_words(w, c.n, c.n);
    if (!pass && (rc = grow(h, &h->poly_ws, &h->poly_ws_bytes, w.used, c.st))) return rc;
  }
  rc = c.dtype == SGEMM_CUBE_F32   ? normalise<float>(h, c.rows, c.cols, c.G, c.ldg, sums, blocks, c.eps, c.pre, X[0], c.st)
       : c.dtype == SGEMM_CUBE_F16 ? normalise<__half>(h, c.rows, c.cols, c.G, c.ldg, sums, blocks, c.eps, c.pre, X[0], c.st)
                                   : normalise<__nv_bfloat16>(h, c.rows, c.cols, c.G, c.ldg, sums, blocks, c.eps, c.pre, X[0], c.st);
  if (rc) return rc;
  for (int i = 0; i < c.steps; ++i) {
    const Words &x = X[i & 1], &next = X[(i + 1) & 1];
    const sgc::ChainStep& f = c.step[i];
    sgc::PolynomialEpilogue ep;
    memset(&ep, 0, sizeof(ep));
    ep.alpha = f.gram_alpha;
    ep.hi = A.hi; ep.lo = A.lo; ep.ldw = A.ld;
    ep.pre = f.gram_pre;
    ep.symmetric = 1;
    rc = c.tall ? polynomial_product<sgc::kFormPolyMM>(h, c.n, c.n, c.m, x, x, ep, c.st)
                : polynomial_product<sgc::kFormPolyKK>(h, c.n, c.n, c.m, x, x, ep, c.st);
    if (rc) return rc;
    ep.alpha = f.square_alpha;
    ep.r_hi = A.hi; ep.r_lo = A.lo; ep.ldr = A.ld;
    ep.beta = f.square_beta;
    ep.hi = B.hi; ep.lo = B.lo; ep.ldw = B.ld;
    ep.pre = f.square_pre;
    if ((rc = polynomial_product<sgc::kFormPolyKK>(h, c.n, c.n, c.n, A, A, ep, c.st))) return rc;
    memset(&ep, 0, sizeof(ep));
    ep.alpha = f.update_alpha;
    ep.r_hi = x.hi; ep.r_lo = x.lo; ep.ldr = x.ld;
    ep.beta = f.update_beta;
    if (i + 1 < c.steps) {
      ep.hi = next.hi; ep.lo = next.lo; ep.ldw = next.ld;
      ep.pre = f.update_pre;
    } else {
      ep.Y = c.O; ep.ldy = c.ldo;
      ep.kept = c.R; ep.ldk = c.ldr; ep.scale = c.scale; ep.keep = c.beta;
      ep.vec = c.vec_out();
    }
    rc = c.tall ? polynomial_product<sgc::kFormPolyKK>(h, c.rows, c.cols, c.cols, x, B, ep, c.st)
                : polynomial_product<sgc::kFormPolyKM>(h, c.rows, c.cols, c.rows, B, x, ep, c.st);
    if (rc) return rc;
  }
  return SGEMM_CUBE_OK;
}

// Which matrices take the one launch: its tiles of 128 x 128 fetch twice as many bytes for a product as the larger kernel's pairs and
// have no next tile's products to hide their epilogue behind.  Five steps, one launch and a launch a product: 128 x 384 123 and
// 318 us, 2048 x 512 186 and 523, 1024 x 8192 758 and 933, 2048 x 2048 664 and 820; 3000 x 3000 2416 and 2036.
bool takes_chain(int n, int m) { return (double)n * n * m <= 1.2e10; }

// Slices of a product's tiles in a grid of clusters, and about how many clocks the product then takes: 1300 for a stage, 4000
// until the first sums are there, 1300 for every 32 rows of a block, and 1500 for the meeting of a cluster, 3000 of one of 16.
long long chain_split(long long tiles, int K, int blocks, int cluster, sgc::ChainSplit* split) {
  const int stages = (K + sgc::kChainBK - 1) / sgc::kChainBK;
  long long least = 0;
  for (int s = 1; s <= cluster; s *= 2) {
    const int per = (stages + s - 1) / s;
    if (s > 1 && tiles * s > blocks) continue;
    const long long turns = (tiles * s + blocks - 1) / blocks;
    const long long clocks = turns * (4000 + per * 1300ll + (s < 4 ? 4 / s : 1) * 1300ll) + (s > 8 ? 3000 : (s > 1 ? 1500 : 0));
    if (s == 1 || clocks < least) { least = clocks; *split = sgc::ChainSplit{(int)tiles, s, per}; }
  }
  return least;
}

cudaLaunchConfig_t chain_config(int blocks, int cluster, cudaLaunchAttribute* attr, cudaStream_t st) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(sgc::kChainThreads, 1, 1);
  cfg.dynamicSmemBytes = sgc::kChainSmem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}
// How many clusters of 1 to 16 blocks are resident at once.
template <typename T>
int chain_setup(sgemm_cube_ctx* h) {
  sgc::ResidentClusters& k = h->chain_clusters[sizeof(T) == 4 ? 0 : (std::is_same<T, __half>::value ? 1 : 2)];
  if (k.ready) return SGEMM_CUBE_OK;
  auto kernel = sgc::polynomial_chain_kernel<T>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sgc::kChainSmem) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    cudaGetLastError();
    return SGEMM_CUBE_CUDA_ERROR;
  }
  for (int c = 1; c <= sgc::kChainMostCluster; c *= 2) {
    cudaLaunchAttribute a[2];
    cudaLaunchConfig_t cfg = chain_config(c * h->sm_count, c, a, nullptr);
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
    k.slices[c] = n * c < h->sm_count ? n : h->sm_count / c;
  }
  k.ready = true;
  return SGEMM_CUBE_OK;
}

// All products in one cooperative launch; *done stays false where that cannot be had.
template <typename T>
int run_chain(sgemm_cube_ctx* h, const OrthogonalizeCall& c, bool* done) {
  int rc = chain_setup<T>(h);
  if (rc) return rc;
  const sgc::ResidentClusters& k = h->chain_clusters[sizeof(T) == 4 ? 0 : (std::is_same<T, __half>::value ? 1 : 2)];
  const long long side = (c.n + sgc::kChainTile - 1) / sgc::kChainTile, lower = side * (side + 1) / 2;
  const long long all = side * ((c.m + sgc::kChainTile - 1) / sgc::kChainTile);
  sgc::ChainParams p;
  memset(&p, 0, sizeof(p));
  // the cluster's size: larger ones share a tile among more blocks, smaller ones leave fewer SMs out
  int cluster = 0, blocks = 0;
  long long least = 0;
  for (int s = 1; s <= (h->split_k ? sgc::kChainMostCluster : 1); s *= 2) {      // (clusters are for slices of a k range)
    const int resident = k.slices[s] * s;
    if (resident == 0) continue;
    sgc::ChainSplit gram, square, update;
    const long long clocks = chain_split(lower, c.m, resident, s, &gram) + chain_split(lower, c.n, resident, s, &square) +
                             chain_split(all, c.n, resident, s, &update);
    if (cluster && clocks >= least) continue;
    least = clocks;
    cluster = s;
    p.gram = gram; p.square = square; p.update = update;
    // blocks: as many as the largest product has work for, and enough to read G
    long long units = (long long)c.rows * c.cols / (sgc::kChainThreads * 8) + 1;
    for (const sgc::ChainSplit* q : {&gram, &square, &update})
      if ((long long)q->tiles * q->slices > units) units = (long long)q->tiles * q->slices;
    blocks = (int)(units < resident ? (units + s - 1) / s * s : resident);
  }
  if (!cluster) return SGEMM_CUBE_OK;
  Words X[2], A, B;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve w;
    w.base = pass ? static_cast<uint8_t*>(h->poly_ws) : nullptr;
    p.sums = w.take<double>((size_t)blocks);
    X[0] = take_words(w, c.rows, c.cols);
    X[1] = c.steps > 1 ? take_words(w, c.rows, c.cols) : X[0];
    A = take_words(w, c.n, c.n);
    B = take_words(w, c.n, c.n);
    if (!pass && (rc = grow(h, &h->poly_ws, &h->poly_ws_bytes, w.used, c.st))) return rc;
  }
  sgc::ChainMaps maps;
  const auto map = [&](CUtensorMap* to, const Words& w, int rows, int cols) {
    const uint16_t* words[2] = {w.hi, w.lo};
    for (int i = 0; i < 2; ++i) {
      const int e = make_map(h, to + i, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, words[i], cols, rows, w.ld, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B);
      if (e) return e;
    }
    return (int)SGEMM_CUBE_OK;
  };
  if ((rc = map(maps.x[0], X[0], c.rows, c.cols)) || (rc = map(maps.x[1], X[1], c.rows, c.cols)) || (rc = map(maps.a, A, c.n, c.n)) ||
      (rc = map(maps.b, B, c.n, c.n)))
    return rc;
  p.rows = c.rows; p.cols = c.cols; p.tall = c.tall; p.steps = c.steps;
  p.G = c.G; p.ldg = c.ldg; p.vec = sgc::rows_take_vectors(c.G, c.ldg, c.cols, sizeof(T));
  p.eps = c.eps; p.pre = c.pre;
  for (int i = 0; i < 2; ++i) { p.x_hi[i] = X[i].hi; p.x_lo[i] = X[i].lo; }
  p.a_hi = A.hi; p.a_lo = A.lo; p.b_hi = B.hi; p.b_lo = B.lo;
  p.ldx = X[0].ld; p.lda = A.ld;
  p.O = c.O; p.ldo = c.ldo; p.R = c.R; p.ldr = c.ldr; p.scale = c.scale; p.keep = c.beta; p.vec_out = c.vec_out();
  p.chunk = h->kblock_termwise / sgc::kChainBK;
  p.words = h->err_dev + sgc::kGridWords + 2;
  p.err = h->err_dev;
  memcpy(p.step, c.step, (size_t)c.steps * sizeof(sgc::ChainStep));
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = chain_config(blocks, cluster, attr, c.st);
  if (cudaLaunchKernelEx(&cfg, sgc::polynomial_chain_kernel<T>, maps, p) != cudaSuccess) {
    cudaGetLastError();                          // a device that is partly occupied by others
    return SGEMM_CUBE_OK;
  }
  h->launches++;
  *done = true;
  return SGEMM_CUBE_OK;
}

constexpr int kMostSteps = sgc::kChainMostSteps;
constexpr double kMostBound = 0x1p20, kLeastBound = 0x1p-20;   // X's and A's exponents stay inside FP32's, squared and all; B's: word_exponent

}  // namespace

extern "C" int sgemm_cube_orthogonalize(sgemm_cube_handle h, int rows, int cols, int dtype, const void* G, int64_t ldg, int steps,
                                        const float* coefficients, float eps, float scale, const float* R, int64_t ldr, float beta,
                                        float* O, int64_t ldo, void* stream) {
  static const float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
  if (!h || bad_dims(rows, cols) || dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16) return SGEMM_CUBE_INVALID_ARG;
  if (steps < 1 || steps > kMostSteps || !(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(scale) || !std::isfinite(beta))
    return SGEMM_CUBE_INVALID_ARG;
  // what the words of X, A and B have to hold, step by step
  double s = 1.0, bound_a[kMostSteps], bound_b[kMostSteps], bound_x[kMostSteps + 1];
  float k[kMostSteps][3];
  bound_x[0] = s;
  for (int i = 0; i < steps; ++i) {
    for (int q = 0; q < 3; ++q) {
      k[i][q] = coefficients ? coefficients[3 * i + q] : kQuintic[q];
      if (!std::isfinite(k[i][q])) return SGEMM_CUBE_INVALID_ARG;
    }
    bound_a[i] = s * s;
    bound_b[i] = largest_on(s, 0.0, k[i][1], k[i][2], 0);
    s = largest_on(s, k[i][0], k[i][1], k[i][2], 1);
    bound_x[i + 1] = s;
    if (!(s <= kMostBound && bound_b[i] <= kMostBound && s >= kLeastBound)) return SGEMM_CUBE_INVALID_ARG;
  }
  if (rows == 0 || cols == 0) return SGEMM_CUBE_OK;
  const size_t elem = dtype == SGEMM_CUBE_F32 ? 4 : 2;
  if (!G || !O || ldg < cols || ldo < cols || (R && ldr < cols)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(elem, G) || misplaced(4, O, R)) return SGEMM_CUBE_INVALID_ARG;
  if (R == O && ldr != ldo && rows > 1) return SGEMM_CUBE_INVALID_ARG;
  if (G == O && (dtype != SGEMM_CUBE_F32 || (ldg != ldo && rows > 1))) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tall = rows > cols;
  const int n = tall ? cols : rows, m = tall ? rows : cols;
  // factors of the products, the words' exponents in them
  sgc::ChainStep step[kMostSteps];
  const int px0 = word_exponent(bound_x[0]);
  for (int i = 0, px = px0; i < steps; ++i) {
    const int pa = word_exponent(bound_a[i]), pb = word_exponent(bound_b[i]), pn = word_exponent(bound_x[i + 1]);
    step[i].gram_alpha = std::ldexp(1.f, -2 * px);
    step[i].gram_pre = std::ldexp(1.f, pa);
    step[i].square_alpha = k[i][2] * std::ldexp(1.f, -2 * pa);
    step[i].square_beta = k[i][1] * std::ldexp(1.f, -pa);
    step[i].square_pre = std::ldexp(1.f, pb);
    step[i].update_alpha = std::ldexp(1.f, -px - pb);
    step[i].update_beta = k[i][0] * std::ldexp(1.f, -px);
    step[i].update_pre = std::ldexp(1.f, pn);
    px = pn;
  }
  OrthogonalizeCall c{rows, cols, dtype, G, ldg, steps, eps, R, ldr, scale, beta, O, ldo, tall, n, m, std::ldexp(1.f, px0), step, st};
  bool done = false;
  int rc = SGEMM_CUBE_OK;
  if (takes_chain(n, m)) {
    rc = dtype == SGEMM_CUBE_F32   ? run_chain<float>(h, c, &done)
         : dtype == SGEMM_CUBE_F16 ? run_chain<__half>(h, c, &done)
                                   : run_chain<__nv_bfloat16>(h, c, &done);
  }
  return done || rc ? rc : run_products(h, c);
}
