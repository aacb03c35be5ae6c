// What the entry points' translation units share: the handle, the device guard, workspace growth and
// tensor maps.  Host code only.
#pragma once

#include <cstdint>
#include <cstring>
#include <vector>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/sgemm_cube.h"

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct DeviceGuard {
  int prev = -1;
  bool ok = true, changed = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev == dev) return;
    changed = true;
    if (cudaSetDevice(dev) != cudaSuccess) ok = false;
  }
  ~DeviceGuard() {
    if (changed && prev >= 0) cudaSetDevice(prev);
  }
};

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
// Whether one of the pointers (null ones aside) is not a multiple of `size` bytes.
template <typename... P>
inline bool misplaced(size_t size, P... p) { return ((reinterpret_cast<uintptr_t>(p) % size != 0) || ...); }
// Whether one of an operator's dimensions is outside [0, 2^31 - 2^16]: the kernels count rows and columns in 32 bits and
// step past the end by a block's stride.
template <typename... D>
inline bool bad_dims(D... d) { return ((d < 0 || d > 0x7FFF0000) || ...); }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

namespace sgc {
// How many clusters of a family of product kernels are resident at once: pairs, and 2 to 8 (one-launch updates: 16) blocks with a k slice each.
struct ResidentClusters {
  bool ready = false;          // kernel attributes set, the counts below known
  int pairs = 0, slices[17] = {0};
};
}  // namespace sgc

struct sgemm_cube_ctx {
  int device = 0;
  int sm_count = 0;
  unsigned int* err_dev = nullptr;   // [0] error word; [4..13] scratch of sgemm_cube_exponent_window;
                                     // [16..19] clocks and nanoseconds of the last timed tensor-core kernel;
                                     // [20..31] ranges, exponents and meeting words of the linear layer's packing
  bool err_dev_has_clock = false;    // false for the static entry point's single error word
  void* ws = nullptr;          // unfused path: FP16 words of A and B, D_hh, D_x
  size_t ws_bytes = 0;
  void* part_ws = nullptr;     // split-K partial sums
  size_t part_ws_bytes = 0;
  int split_k = 1;             // 1: split the k range of few-tile problems over idle SMs; 0: never
  void* tile_ws = nullptr;     // linear forms: two 128 x 256 tiles for every block of the tensor-core kernel
  size_t tile_ws_bytes = 0;
  void* loss_ws = nullptr;     // cross entropy: logits of a piece of rows, words of their gradient, pairs
  size_t loss_ws_bytes = 0;
  void* poly_ws = nullptr;     // orthogonalised updates: words of X, of its Gram matrix and of the polynomial
  size_t poly_ws_bytes = 0;
  void* sort_ws = nullptr;     // embedding gradients: sorted tokens and their rows, partial sums
  size_t sort_ws_bytes = 0;
  void* host_ws = nullptr;     // host-buffer path: device copies of A, B, C
  size_t host_ws_bytes = 0;
  std::vector<void*> graph_ws; // buffers that captured calls have used, outgrown ones among them
  long long launches = 0;
  int kblock_termwise = 128;
  int kblock_elementwise = 64;
  int cta_pair = 2;            // 0/1: never/always 2-CTA clusters (cta_group::2); 2: see use_pair
  int strategy = 0;            // sgemm_cube: 0 auto, 1 fused kernel, 2 split kernel + 3-product kernel
  int time_kernel = 0;         // record events around the tensor-core kernel of sgemm_cube
  static constexpr int kTimedCalls = 128;           // event pairs kept (most recent calls)
  cudaEvent_t ev_ring[2 * kTimedCalls] = {};
  long long ev_calls = 0;      // timed calls since timing was switched on or last averaged
  // host-buffer path: copy streams and events of the panel pipeline (created on first use)
  static constexpr int kMaxPanels = 32;
  cudaStream_t s_in = nullptr, s_out = nullptr;
  cudaEvent_t ev_start = nullptr, ev_b = nullptr, ev_out = nullptr;
  cudaEvent_t ev_a[kMaxPanels] = {}, ev_c[kMaxPanels] = {};
  int max_pair_clusters[3] = {0, 0, 0};   // co-resident 2-CTA clusters: <1,false>, <3,false>, <3,true>
  EncodeTiledFn encode = nullptr;
  bool attrs_set = false;
  sgc::ResidentClusters linear_clusters, polynomial_clusters, loss_clusters, chain_clusters[3];   // (chain: by element type)
  int pack_once_blocks = 0, dz_once_blocks[5] = {0, 0, 0, 0, 0};   // resident blocks of the one-launch packing kernels
};

// Room of at least `want` bytes in one of the handle's buffers, for a call on `st`.  A buffer that grows is freed and
// allocated anew, unless a call that was captured has had it: the graph goes on using it whenever it is replayed, so
// such a buffer stays until the handle is destroyed.
inline int grow(sgemm_cube_ctx* h, void** buf, size_t* have, size_t want, cudaStream_t st) {
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  // (an error: the legacy stream while another one is captured; this call is not part of that)
  if (cudaStreamIsCapturing(st, &status) != cudaSuccess) { cudaGetLastError(); status = cudaStreamCaptureStatusNone; }
  const bool capturing = status != cudaStreamCaptureStatusNone;
  const auto in_graph = [&](void* p) {
    for (void* q : h->graph_ws)
      if (q == p) return true;
    return false;
  };
  if (*have < want) {
    const bool keep = *buf && (capturing || in_graph(*buf));
    if (*buf && !keep) {
      if (cudaFree(*buf) != cudaSuccess) return SGEMM_CUBE_CUDA_ERROR;
      *buf = nullptr;
      *have = 0;
    }
    void* fresh = nullptr;
    if (cudaMalloc(&fresh, want) != cudaSuccess) {
      cudaGetLastError();
      return SGEMM_CUBE_ALLOC_FAILED;
    }
    if (keep && !in_graph(*buf)) h->graph_ws.push_back(*buf);
    *buf = fresh;
    *have = want;
  }
  if (capturing && !in_graph(*buf)) h->graph_ws.push_back(*buf);
  return SGEMM_CUBE_OK;
}
inline void free_workspaces(sgemm_cube_ctx* h) {
  void* const current[] = {h->ws, h->part_ws, h->tile_ws, h->loss_ws, h->poly_ws, h->sort_ws, h->host_ws};
  for (void* p : h->graph_ws) {
    bool also = false;
    for (void* q : current) also = also || q == p;
    if (!also) cudaFree(p);
  }
  for (void* p : current)
    if (p) cudaFree(p);
}

// 2-D tensor map over a row-major matrix: dims {inner, outer}, row pitch in bytes.
inline int make_map(sgemm_cube_ctx* h, CUtensorMap* map, CUtensorMapDataType dt, size_t elem, const void* base,
             uint64_t inner, uint64_t outer, uint64_t ld_elems, uint32_t box_inner,
             uint32_t box_outer, CUtensorMapSwizzle swz) {
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {ld_elems * elem};
  cuuint32_t box[2] = {box_inner, box_outer};
  cuuint32_t estr[2] = {1, 1};
  CUresult r = h->encode(map, dt, 2, const_cast<void*>(base), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SGEMM_CUBE_OK : SGEMM_CUBE_CUDA_ERROR;
}
