// A matrix brought near the closest one with orthonormal rows (columns, where it has more rows), by Newton-Schulz products
// (contract: include/sgemm_cube.h):
//
//   X = G / (|G|_F + eps);   steps times:  A = X X^T,  P = a + b A + c A A,  X <- P X;   O = scale X + beta R
//
// (rows <= columns; else A = X^T X and X <- X P).  X, A and P live as FP16 words from the first pass to the last, written by the
// epilogues of the products that make them (polynomial_epilogue.cuh): no pass of its own packs anything.  Their exponents
// are known beforehand: the singular values of X lie in [0, s] with s = 1 at the start and the polynomial's largest value
// on [0, s] after a step, and no entry of a matrix is larger than its largest singular value.
// A and P are symmetric: half of their tiles are formed.
#include <cmath>

#include "ctx.cuh"
#include "elements.cuh"
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
  constexpr int V = Elem<T>::kVec;
  double s = 0.0;
  for (int i = threadIdx.x; i < n_sums; i += 256) s += sums[i];
  for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
  __shared__ double warp_sum[8];
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = s;
  __syncthreads();
  s = warp_sum[0];
  for (int w = 1; w < 8; ++w) s += warp_sum[w];
  const double norm = sqrt(s) + (double)eps;
  // (a matrix of zeros with eps = 0 stays one; a norm that is not finite makes every entry NaN)
  const double scale = norm == 0.0 ? 0.0 : (isfinite(norm) ? 1.0 / norm : (double)NAN);
  // two FP32 factors: 1 / norm can leave the FP32 range while the entries times it do not
  const int e = scale != 0.0 && isfinite(scale) ? max(-126, min(126, ilogb(scale) / 2)) : 0;
  const float f0 = pow2f(e), f1 = (float)(scale * (double)pow2f(-e)) * pre;
  const int per_row = (cols + 7) >> 3;
  const long long total = (long long)rows * per_row, stride = (long long)gridDim.x * 256;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < total; it += stride) {
    const long long r = total < (1ll << 31) ? (long long)((uint32_t)it / (uint32_t)per_row) : it / per_row;
    const int c = (int)(it - r * per_row) << 3;
    const T* at = G + r * ldg + c;
    float v[8];
    if (vec && c + 8 <= cols) {
#pragma unroll
      for (int i = 0; i < 8 / V; ++i) {
        float x[V];
        Elem<T>::unpack(*reinterpret_cast<const uint4*>(at + i * V), x);
#pragma unroll
        for (int q = 0; q < V; ++q) v[i * V + q] = x[q];
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = c + q < cols ? Elem<T>::get(at[q]) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= f0;
    uint4 h, l;
    pack_words(v, f1, h, l);
    *reinterpret_cast<uint4*>(hi + r * ldw + c) = h;
    *reinterpret_cast<uint4*>(lo + r * ldw + c) = l;
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
// p with 2^p x below the largest FP16 number for |x| <= bound, a sixteenth of it left for rounding.
int word_exponent(double bound) {
  return 15 - (int)std::floor(std::log2(bound * 1.0625));
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

constexpr int kMostSteps = 64;
constexpr double kMostBound = 0x1p20, kLeastBound = 0x1p-20;   // the words' exponents stay inside FP32's, squared and all

}  // namespace

extern "C" int sgemm_cube_orthogonalize(sgemm_cube_handle h, int rows, int cols, int dtype, const void* G, int64_t ldg, int steps,
                                        const float* coefficients, float eps, float scale, const float* R, int64_t ldr, float beta,
                                        float* O, int64_t ldo, void* stream) {
  static const float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
  if (!h || bad_dims(rows, cols) || dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16) return SGEMM_CUBE_INVALID_ARG;
  if (steps < 1 || steps > kMostSteps || !(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(scale) || !std::isfinite(beta))
    return SGEMM_CUBE_INVALID_ARG;
  // what the words of X, A and P have to hold, step by step
  double s = 1.0, bound_a[kMostSteps], bound_p[kMostSteps], bound_x[kMostSteps + 1];
  float k[kMostSteps][3];
  bound_x[0] = s;
  for (int i = 0; i < steps; ++i) {
    for (int q = 0; q < 3; ++q) {
      k[i][q] = coefficients ? coefficients[3 * i + q] : kQuintic[q];
      if (!std::isfinite(k[i][q])) return SGEMM_CUBE_INVALID_ARG;
    }
    bound_a[i] = s * s;
    bound_p[i] = largest_on(s, k[i][0], k[i][1], k[i][2], 0);
    s = largest_on(s, k[i][0], k[i][1], k[i][2], 1);
    bound_x[i + 1] = s;
    if (!(s <= kMostBound && bound_p[i] <= kMostBound && s >= kLeastBound)) return SGEMM_CUBE_INVALID_ARG;
  }
  if (rows == 0 || cols == 0) return SGEMM_CUBE_OK;
  const size_t elem = dtype == SGEMM_CUBE_F32 ? 4 : 2;
  if (!G || !O || ldg < cols || ldo < cols || (R && ldr < cols)) return SGEMM_CUBE_INVALID_ARG;
  if (misplaced(elem, G) || misplaced(4, O, R)) return SGEMM_CUBE_INVALID_ARG;
  if (R == O && ldr != ldo && rows > 1) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int rc = sgc::product_setup<sgc::kFormPolyKM, sgc::kFormPolyKK, sgc::kFormPolyMM>(h, h->polynomial_clusters);
  if (rc) return rc;
  const bool tall = rows > cols;
  const int n = tall ? cols : rows, m = tall ? rows : cols;
  const int blocks = sgc::blocks_for(h, (long long)rows * cols / 16 + 1);
  Words X[2], A, P;
  double* sums = nullptr;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->poly_ws) : nullptr;
    sums = c.take<double>((size_t)blocks);
    X[0] = take_words(c, rows, cols);
    X[1] = steps > 1 ? take_words(c, rows, cols) : X[0];
    A = take_words(c, n, n);
    P = take_words(c, n, n);
    if (!pass && (rc = grow(h, &h->poly_ws, &h->poly_ws_bytes, c.used, st))) return rc;
  }
  int px = word_exponent(bound_x[0]);
  const float pre = std::ldexp(1.f, px);
  rc = dtype == SGEMM_CUBE_F32   ? normalise<float>(h, rows, cols, G, ldg, sums, blocks, eps, pre, X[0], st)
       : dtype == SGEMM_CUBE_F16 ? normalise<__half>(h, rows, cols, G, ldg, sums, blocks, eps, pre, X[0], st)
                                 : normalise<__nv_bfloat16>(h, rows, cols, G, ldg, sums, blocks, eps, pre, X[0], st);
  if (rc) return rc;
  for (int i = 0; i < steps; ++i) {
    const Words &x = X[i & 1], &next = X[(i + 1) & 1];
    const int pa = word_exponent(bound_a[i]), pp = word_exponent(bound_p[i]), pn = word_exponent(bound_x[i + 1]);
    sgc::PolynomialEpilogue ep;
    // A = X X^T, or X^T X
    memset(&ep, 0, sizeof(ep));
    ep.alpha = std::ldexp(1.f, -2 * px);
    ep.hi = A.hi; ep.lo = A.lo; ep.ldw = A.ld;
    ep.pre = std::ldexp(1.f, pa);
    ep.symmetric = 1;
    rc = tall ? polynomial_product<sgc::kFormPolyMM>(h, n, n, m, x, x, ep, st)
              : polynomial_product<sgc::kFormPolyKK>(h, n, n, m, x, x, ep, st);
    if (rc) return rc;
    // P = a + b A + c A A
    ep.alpha = k[i][2] * std::ldexp(1.f, -2 * pa);
    ep.r_hi = A.hi; ep.r_lo = A.lo; ep.ldr = A.ld;
    ep.beta = k[i][1] * std::ldexp(1.f, -pa);
    ep.diagonal = k[i][0];
    ep.hi = P.hi; ep.lo = P.lo; ep.ldw = P.ld;
    ep.pre = std::ldexp(1.f, pp);
    if ((rc = polynomial_product<sgc::kFormPolyKK>(h, n, n, n, A, A, ep, st))) return rc;
    // X <- P X, or X P; the last one to O
    memset(&ep, 0, sizeof(ep));
    ep.alpha = std::ldexp(1.f, -px - pp);
    if (i + 1 < steps) {
      ep.hi = next.hi; ep.lo = next.lo; ep.ldw = next.ld;
      ep.pre = std::ldexp(1.f, pn);
    } else {
      ep.alpha *= scale;
      ep.Y = O; ep.ldy = ldo;
      ep.kept = R; ep.ldk = ldr; ep.keep = beta;
      ep.vec = aligned16(O) && ldo % 4 == 0 && (!R || (aligned16(R) && ldr % 4 == 0));
    }
    rc = tall ? polynomial_product<sgc::kFormPolyKK>(h, rows, cols, cols, x, P, ep, st)
              : polynomial_product<sgc::kFormPolyKM>(h, rows, cols, rows, P, x, ep, st);
    if (rc) return rc;
    px = pn;
  }
  return SGEMM_CUBE_OK;
}
