// Embedding lookup with a scale, and the gradient of the table by sorted tokens (contracts: include/sgemm_cube.h).
//
//   Y[i] = scale E[t_i];   dE[v] = scale sum over i with t_i = v of dY[i]  (+ dE[v])
//
// Both only move memory.  The gradient sorts the tokens (stable, so a token's rows are added in their order and the result
// is the same every time), cuts the sorted list into pieces of equal length, and adds the rows of each piece, a run of equal
// tokens at a time: a frequent token's rows are shared by many blocks, and a run that leaves a piece goes through partial sums.
#include <cmath>

#include "ctx.cuh"
#include "elements.cuh"
#include "product_host.cuh"

namespace sgc {

// ------------------------------------------------------------------------------------------ lookup
struct LookupParams {
  long long rows;
  int vocab, cols, pieces;       // pieces of a row
  const long long* tokens;
  const void* table;
  long long ld;
  float scale;
  void* Y;
  long long ldy;
};
constexpr int kLookupThreads = 128, kLookupItems = 4;

// 16 bytes from an address that is a multiple of the element's size: the 4-byte words that hold them (each holds a byte of
// them, so none lies outside what may be read), shifted.
template <typename T>
__device__ __forceinline__ uint4 load_shifted(const T* at) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(at);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(a & ~uintptr_t(3));
  uint4 v = make_uint4(__ldg(w), __ldg(w + 1), __ldg(w + 2), __ldg(w + 3));
  if (sizeof(T) == 2 && (a & 2)) {
    const uint32_t x = __ldg(w + 4);
    v.x = __funnelshift_r(v.x, v.y, 16); v.y = __funnelshift_r(v.y, v.z, 16);
    v.z = __funnelshift_r(v.z, v.w, 16); v.w = __funnelshift_r(v.w, x, 16);
  }
  return v;
}

// A block copies a piece of a row in 16-byte vectors; where the two rows do not meet 16-byte boundaries at the same
// columns (VEC false) these lie on Y's boundaries, their source comes in 4-byte words, and what is left of the row at both
// ends goes by elements.  (All of it by elements: 30001 x 1001 FP16 40 us.)
// TH threads have a row's piece, the block's others rows of their own.
template <typename T, bool VEC, int TH>
__global__ void __launch_bounds__(kLookupThreads) embedding_kernel(LookupParams p) {
  constexpr int V = Elem<T>::kVec, U = kLookupItems;
  constexpr int side = kLookupThreads / TH;
  const int t_row = (int)threadIdx.x % TH;
  for (long long unit = (long long)blockIdx.x * side + (int)threadIdx.x / TH; unit < p.rows * p.pieces; unit += (long long)gridDim.x * side) {
    const long long row = p.pieces == 1 ? unit : unit / p.pieces;
    const int c0 = (int)(unit - row * p.pieces) * (TH * V * U) + t_row * V;
    const long long t = __ldg(p.tokens + row);
    const bool inside = t >= 0 && t < p.vocab;
    const T* src = static_cast<const T*>(p.table) + (inside ? t : 0) * p.ld;
    T* dst = static_cast<T*>(p.Y) + row * p.ldy;
    const float none = t < 0 ? 0.f : NAN;
    if constexpr (VEC) {
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * TH * V;
        if (inside && c < p.cols) raw[u] = __ldg(reinterpret_cast<const uint4*>(src + c));
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * TH * V;
        if (c >= p.cols) break;
        float e[V];
        Elem<T>::unpack(raw[u], e);
#pragma unroll
        for (int q = 0; q < V; ++q) e[q] = inside ? e[q] * p.scale : none;
        *reinterpret_cast<uint4*>(dst + c) = Elem<T>::pack(e);
      }
    } else {
      const int head = min(p.cols, (int)((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) % 16 / sizeof(T)));
      const int end = head + (p.cols - head) / V * V;
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = head + c0 + u * TH * V;
        if (inside && c < end) raw[u] = load_shifted(src + c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = head + c0 + u * TH * V;
        if (c >= end) break;
        float e[V];
        Elem<T>::unpack(raw[u], e);
#pragma unroll
        for (int q = 0; q < V; ++q) e[q] = inside ? e[q] * p.scale : none;
        *reinterpret_cast<uint4*>(dst + c) = Elem<T>::pack(e);
      }
      if (c0 < TH * V) {                         // the row's first piece: both ends
        const int i = t_row, c = i < head ? i : end + i - head;
        if (c < p.cols) dst[c] = Elem<T>::put(inside ? Elem<T>::get(src[c]) * p.scale : none);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------ sorting
constexpr int kSortThreads = 512, kSortItems = 4, kSortTile = kSortThreads * kSortItems;
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits;        // two passes for vocabularies up to 2^18
static_assert(kSortThreads == kSortBins, "a thread has a digit");
constexpr int kSortFew = 256;                                   // items that one block ranks by counting

struct SortParams {
  int n, vocab, passes;
  const long long* tokens;
  int* key[2];               // the pass reads from one and writes to the other; the first reads the tokens
  int* pos[2];
  int* hist;                 // [blocks][bins]
  unsigned char* met;        // [vocab rounded up to 16]: whether the token occurs, or null
  int clear;                 // the flags are cleared here first
  unsigned int* words;       // {arrived, left}, zero between calls
  unsigned int* err;
};

// All blocks of the grid meet for the `round`-th time (from 1).  Cooperative launch; bounded all the same.
__device__ __forceinline__ bool sort_meet(const SortParams& p, unsigned int round) {
  __shared__ unsigned int ok;
  if (gridDim.x == 1) {
    __syncthreads();
    return true;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();                                           // the block's stores, which the barrier has put before this
    asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(&p.words[0]), "r"(1u) : "memory");
    const unsigned int want = round * gridDim.x;
    const long long t0 = clock64();
    unsigned int seen = 0;
    ok = 1u;
    while (true) {
      asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&p.words[0]) : "memory");
      if (seen >= want) break;
      if (clock64() - t0 > kWaitLimitClocks) {
        atomicExch(p.err, (unsigned int)kErrSortWait);
        ok = 0u;
        break;
      }
    }
    __threadfence();
  }
  __syncthreads();
  return ok != 0u;
}

// Stable sort of (token, row) by token, 9 bits a pass from the lowest.  A block has a run of whole tiles; in a pass it counts
// its digits, meets the others, adds up for every digit what lies before its own first one, and
// moves its items in order.  Tokens outside [0, vocab) get the key `vocab` and end up behind all others.
// After a wait that ran out, until sgemm_cube_check has cleared the words, counts and items may be anything that the workspace held: places
// are looked at before they are written to, here, and tokens and rows before they are used, in the sums.
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(SortParams p) {
  __shared__ int base[kSortBins];                              // next place of a digit
  __shared__ int warp_hist[kSortThreads / 32][kSortBins];
  __shared__ int scan[kSortThreads / 32];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int tiles = (p.n + kSortTile - 1) / kSortTile;
  const int per_block = (tiles + gridDim.x - 1) / gridDim.x;
  const int first = min((long long)p.n, (long long)blockIdx.x * per_block * kSortTile);
  const int last = min((long long)p.n, ((long long)blockIdx.x + 1) * per_block * kSortTile);
  if (p.clear)
    for (long long v = (long long)blockIdx.x * kSortThreads + t; v < (p.vocab + 15) / 16; v += (long long)gridDim.x * kSortThreads)
      reinterpret_cast<uint4*>(p.met)[v] = make_uint4(0u, 0u, 0u, 0u);
  if (p.n <= kSortFew) {
    // One block: an item's place is the number of items that come before it.
    __shared__ int keys[kSortFew];
    for (int i = t; i < p.n; i += kSortThreads) {
      const long long v = p.tokens[i];
      keys[i] = v >= 0 && v < p.vocab ? (int)v : p.vocab;
    }
    __syncthreads();                                           // (the flags are cleared, too)
    for (int i = t; i < p.n; i += kSortThreads) {
      const int own = keys[i];
      int place = 0;
#pragma unroll 8
      for (int j = 0; j < p.n; ++j) place += keys[j] < own || (keys[j] == own && j < i) ? 1 : 0;
      p.key[p.passes & 1][place] = own;
      p.pos[p.passes & 1][place] = i;
      if (p.met && own < p.vocab) p.met[own] = 1;
    }
    return;
  }
  unsigned int round = 0;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * kSortBits;
    const int *key_in = p.key[pass & 1], *pos_in = p.pos[pass & 1];
    int *key_out = p.key[(pass & 1) ^ 1], *pos_out = p.pos[(pass & 1) ^ 1];
    auto key_of = [&](int i) -> int {
      if (pass) return __ldcg(key_in + i);
      const long long v = p.tokens[i];
      return v >= 0 && v < p.vocab ? (int)v : p.vocab;
    };
    base[t] = 0;
    __syncthreads();
    for (int i = first + t; i < last; i += kSortTile) {
      int key[kSortItems];
#pragma unroll
      for (int u = 0; u < kSortItems; ++u) key[u] = i + u * kSortThreads < last ? key_of(i + u * kSortThreads) : -1;
#pragma unroll
      for (int u = 0; u < kSortItems; ++u)
        if (key[u] >= 0) atomicAdd(&base[(key[u] >> shift) & (kSortBins - 1)], 1);
    }
    __syncthreads();
    p.hist[blockIdx.x * kSortBins + t] = base[t];
    if (!sort_meet(p, ++round)) return;
    // thread t: digit t's items in the blocks before this one, and in all of them
    int before = 0, all = 0;
    for (int b0 = 0; b0 < (int)gridDim.x; b0 += 8) {
      int c[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) c[u] = b0 + u < (int)gridDim.x ? __ldcg(p.hist + (b0 + u) * kSortBins + t) : 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        before += b0 + u < (int)blockIdx.x ? c[u] : 0;
        all += c[u];
      }
    }
    int incl = all;
    for (int x = 1; x < 32; x *= 2) {
      const int o = __shfl_up_sync(0xffffffffu, incl, x);
      if (lane >= x) incl += o;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += scan[w];
    base[t] = incl - all + before;
    __syncthreads();
    for (int tile = first; tile < last; tile += kSortTile) {
      // a warp has 128 items in a row, 32 at a time; an item's place among the warp's of its digit
      int key[kSortItems], place[kSortItems];
      for (int i = lane; i < kSortBins; i += 32) warp_hist[warp][i] = 0;
      __syncwarp();
#pragma unroll
      for (int u = 0; u < kSortItems; ++u) {
        const int i = tile + warp * (32 * kSortItems) + u * 32 + lane;
        key[u] = i < last ? key_of(i) : -1;
        const int digit = key[u] < 0 ? kSortBins : (key[u] >> shift) & (kSortBins - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        const int ahead = __popc(same & ((1u << lane) - 1u));
        int start = 0;
        if (digit < kSortBins) start = warp_hist[warp][digit];
        __syncwarp();
        if (digit < kSortBins && ahead == 0) warp_hist[warp][digit] = start + __popc(same);
        __syncwarp();
        place[u] = start + ahead;
      }
      __syncthreads();
      // thread t: where each warp's items of digit t begin
      int at = base[t];
      for (int w = 0; w < kSortThreads / 32; ++w) {
        const int c = warp_hist[w][t];
        warp_hist[w][t] = at;
        at += c;
      }
      __syncthreads();
      base[t] = at;
#pragma unroll
      for (int u = 0; u < kSortItems; ++u) {
        if (key[u] < 0) continue;
        const int i = tile + warp * (32 * kSortItems) + u * 32 + lane;
        const int to = warp_hist[warp][(key[u] >> shift) & (kSortBins - 1)] + place[u];
        if ((unsigned)to >= (unsigned)p.n) continue;
        key_out[to] = key[u];
        pos_out[to] = pass ? __ldcg(pos_in + i) : i;
        if (p.met && pass == p.passes - 1 && key[u] < p.vocab) p.met[key[u]] = 1;
      }
      __syncthreads();
    }
    if (pass + 1 < p.passes && !sort_meet(p, ++round)) return;
  }
  if (gridDim.x > 1 && t == 0) {
    if (atomicAdd(&p.words[1], 1u) == gridDim.x - 1) p.words[0] = p.words[1] = 0u;   // the last one clears both
  }
}

// ------------------------------------------------------------------------------------------ sums
// The same for a few thousand items without digits and meetings: an item's place is the number of items that come before it, and
// blocks count apart from each other.  A warp has four items, a lane four keys of every 128; keys in front of the warp's own 128 count when
// they are equal, too.  Bound by the n^2 comparisons and by every block's reading of all tokens (calls with the lookup, 512 columns: 1000 rows 39 us, one
// block counting 67; 4096 rows 50, by digits 58; 8192 63 and 65).
constexpr int kRankThreads = 512, kRankItems = 4, kRankBlock = kRankThreads / 32 * kRankItems, kRankMost = 8192;
__global__ void __launch_bounds__(kRankThreads) rank_tokens_kernel(SortParams p) {
  __shared__ __align__(16) int keys[kRankMost];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int* const key_out = p.passes & 1 ? p.key[1] : p.key[0];
  int* const pos_out = p.passes & 1 ? p.pos[1] : p.pos[0];
  const int chunks = (p.n + 127) / 128;
#pragma unroll 8
  for (int i = threadIdx.x; i < chunks * 128; i += kRankThreads) {
    const long long v = i < p.n ? p.tokens[i] : -1;
    keys[i] = i >= p.n ? INT_MAX : (v >= 0 && v < p.vocab ? (int)v : p.vocab);
  }
  __syncthreads();
  const int first = (int)blockIdx.x * kRankBlock + warp * kRankItems;
  if (first >= p.n) return;
  int own[kRankItems], place[kRankItems];
#pragma unroll
  for (int k = 0; k < kRankItems; ++k) {
    own[k] = keys[first + k];
    place[k] = 0;
  }
  const int4* quads = reinterpret_cast<const int4*>(keys) + lane;
  const int mid = first / 128;
#pragma unroll 2
  for (int c = 0; c < mid; ++c) {
    const int4 v = quads[c * 32];
#pragma unroll
    for (int k = 0; k < kRankItems; ++k) place[k] += (v.x <= own[k]) + (v.y <= own[k]) + (v.z <= own[k]) + (v.w <= own[k]);
  }
  {
    const int4 v = quads[mid * 32];
    const int j = mid * 128 + lane * 4;
#pragma unroll
    for (int k = 0; k < kRankItems; ++k) {
      const int i = first + k;
      place[k] += (v.x < own[k] || (v.x == own[k] && j < i)) + (v.y < own[k] || (v.y == own[k] && j + 1 < i)) +
                  (v.z < own[k] || (v.z == own[k] && j + 2 < i)) + (v.w < own[k] || (v.w == own[k] && j + 3 < i));
    }
  }
#pragma unroll 2
  for (int c = mid + 1; c < chunks; ++c) {
    const int4 v = quads[c * 32];
#pragma unroll
    for (int k = 0; k < kRankItems; ++k) place[k] += (v.x < own[k]) + (v.y < own[k]) + (v.z < own[k]) + (v.w < own[k]);
  }
#pragma unroll
  for (int k = 0; k < kRankItems; ++k) {
    const int to = __reduce_add_sync(0xffffffffu, place[k]);
    if (lane == k && first + k < p.n) {
      key_out[to] = own[k];
      pos_out[to] = first + k;
      if (p.met && own[k] < p.vocab) p.met[own[k]] = 1;
    }
  }
}

struct TableGradParams {
  int n, vocab, cols, piece, pieces;   // sorted items; items of a piece, pieces
  int tiles;                           // column tiles of a row
  const int* key;
  const int* pos;
  const unsigned char* met;            // null: nothing is cleared
  const void* dY;
  long long lddy;
  float scale;
  int accumulate;
  float* dE;
  long long ldd;
  float* part;                         // [2 pieces][ldp]: the run that a piece finds begun, and the one that it leaves open
  long long ldp;
  unsigned int sum_blocks;             // the blocks behind them clear the rows of tokens that do not occur
  int vec_out;                         // dE takes 16-byte accesses
};
constexpr int kGradThreads = 128, kClearPiece = 4096;   // threads; floats that a block clears at a time

__device__ __forceinline__ bool is_token(const TableGradParams& p, int key) { return (unsigned)key < (unsigned)p.vocab; }

// Column of the thread's element q in its tile of TH threads: consecutive ones where rows take vectors, else TH apart.
template <typename T, bool VEC, int TH>
__device__ __forceinline__ int grad_column(int tile, int q) {
  const int t = (int)threadIdx.x % TH;
  return tile * (TH * Elem<T>::kVec) + (VEC ? t * Elem<T>::kVec + q : q * TH + t);
}
template <typename T, bool VEC, int TH>
__device__ __forceinline__ void store_grad(const TableGradParams& p, int token, int tile, const float (&acc)[Elem<T>::kVec]) {
  constexpr int V = Elem<T>::kVec;
  float* out = p.dE + (long long)token * p.ldd;
  if (VEC && p.vec_out) {
    const int c = grad_column<T, VEC, TH>(tile, 0);
    if (c >= p.cols) return;
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      float4 o = make_float4(acc[q] * p.scale, acc[q + 1] * p.scale, acc[q + 2] * p.scale, acc[q + 3] * p.scale);
      if (p.accumulate) {
        const float4 old = *reinterpret_cast<const float4*>(out + c + q);
        o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w;
      }
      *reinterpret_cast<float4*>(out + c + q) = o;
    }
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const int c = grad_column<T, VEC, TH>(tile, q);
      if (c < p.cols) out[c] = p.accumulate ? out[c] + acc[q] * p.scale : acc[q] * p.scale;
    }
  }
}

// Zeros for `len` floats, by all threads of a block, 32 bytes at a time.
__device__ __forceinline__ void clear_run(float* out, int len) {
  const int head = min(len, (int)((32 - (reinterpret_cast<uintptr_t>(out) & 31)) % 32 / 4)), eights = (len - head) / 8;
  float* body = out + head;
#pragma unroll 4
  for (int i = threadIdx.x; i < eights; i += kGradThreads)
    asm volatile("st.global.v8.f32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(body + 8 * i), "f"(0.f) : "memory");
  if (threadIdx.x < head) out[threadIdx.x] = 0.f;
  if (threadIdx.x < len - head - 8 * eights) body[8 * eights + threadIdx.x] = 0.f;
}
// Zeros for the rows of tokens that do not occur.  A block has a piece of 16 KiB, and the pieces follow each other in memory as the
// blocks start: 71496 x 7509 with 9 tokens 298 us, 7.5 TB/s while it clears; blocks that stay and take every so many-th piece 325, eight
// whole rows at a time 382.  Pieces are cut at multiples of 128 bytes, since what two blocks write of one sector goes to memory twice.
// A warp looks at the flags of 32 rows; rows next to each other are one run.
__device__ __forceinline__ void clear_rows(const TableGradParams& p, unsigned int blk, unsigned int blocks) {
  const int lane = threadIdx.x & 31;
  const bool flat = p.ldd == p.cols;
  const long long total = (long long)p.vocab * p.cols;
  const int skew = (int)((reinterpret_cast<uintptr_t>(p.dE) >> 2) & 31);
  for (long long at = (long long)blk * kClearPiece - skew; at < total; at += (long long)blocks * kClearPiece) {
    const long long lo = max(at, 0ll), hi = min(at + kClearPiece, total);
    for (long long v0 = lo / p.cols; v0 * p.cols < hi; v0 += 32) {
      uint32_t left = __ballot_sync(0xffffffffu, v0 + lane < p.vocab && (v0 + lane) * p.cols < hi && p.met[v0 + lane] == 0);
      while (left) {
        const int first = __ffs(left) - 1;
        const uint32_t behind = ~(left >> first);                      // the run's first row that is not to be cleared
        const int run = flat ? (behind ? __ffs(behind) - 1 : 32) : 1;
        left &= run + first >= 32 ? (1u << first) - 1u : ~(((1u << run) - 1u) << first);
        const long long row = (v0 + first) * p.cols, begin = max(lo, row), end = min(hi, row + (long long)run * p.cols);
        clear_run(p.dE + (v0 + first) * p.ldd + (begin - row), (int)(end - begin));
      }
    }
  }
}

// TH threads add the rows of one piece in one tile of columns; a block has 128 / TH pieces side by side.  Rows come four at a time; a run that lies inside the piece
// is stored, the others' sums go to `part`.  The last blocks clear rows.
template <typename T, bool VEC, int TH>
__global__ void __launch_bounds__(kGradThreads) table_grad_kernel(TableGradParams p) {
  constexpr int V = Elem<T>::kVec, U = 4;
  if (blockIdx.x >= p.sum_blocks) {
    clear_rows(p, blockIdx.x - p.sum_blocks, gridDim.x - p.sum_blocks);
    return;
  }
  const int group = (int)(blockIdx.x / p.tiles), tile = (int)(blockIdx.x - (unsigned)group * p.tiles);
  const int piece = group * (kGradThreads / TH) + (int)threadIdx.x / TH;
  if (piece >= p.pieces) return;
  const int first = piece * p.piece, last = (int)min((long long)p.n, (long long)first + p.piece);
  float acc[V];
#pragma unroll
  for (int q = 0; q < V; ++q) acc[q] = 0.f;
  // tokens outside the vocabulary lie behind all others and have no row
  int run = __ldg(p.key + first);
  if (!is_token(p, run)) return;
  bool open = first > 0 && __ldg(p.key + first - 1) == run;          // begun in the piece before
  auto leave = [&](bool goes_on) {
    if (!open && !goes_on) {
      store_grad<T, VEC, TH>(p, run, tile, acc);
    } else {
      float* out = p.part + (2ll * piece + (open ? 0 : 1)) * p.ldp;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const int c = grad_column<T, VEC, TH>(tile, q);
        if (c < p.cols) out[c] = acc[q];
      }
    }
  };
  for (int i = first; i < last; i += U) {
    int key[U];
    uint4 raw[U];
    T one[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      key[u] = i + u < last ? __ldg(p.key + i + u) : p.vocab;
      if (is_token(p, key[u])) {
        const T* src = static_cast<const T*>(p.dY) + (long long)min((unsigned)__ldg(p.pos + i + u), (unsigned)(p.n - 1)) * p.lddy;
        if constexpr (VEC) {
          const int c = grad_column<T, VEC, TH>(tile, 0);
          raw[u] = c < p.cols ? __ldcs(reinterpret_cast<const uint4*>(src + c)) : make_uint4(0u, 0u, 0u, 0u);
        } else {
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const int c = grad_column<T, VEC, TH>(tile, q);
            one[u][q] = c < p.cols ? src[c] : Elem<T>::put(0.f);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!is_token(p, key[u])) break;
      if (key[u] != run) {
        leave(false);
        run = key[u];
        open = false;
#pragma unroll
        for (int q = 0; q < V; ++q) acc[q] = 0.f;
      }
      float e[V];
      if constexpr (VEC) {
        Elem<T>::unpack(raw[u], e);
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q) e[q] = Elem<T>::get(one[u][q]);
      }
#pragma unroll
      for (int q = 0; q < V; ++q) acc[q] += e[q];
    }
  }
  leave(last < p.n && __ldg(p.key + last) == run);
}

// Runs that reach over pieces: the block of the piece in which one begins adds the parts of the others, in order, eight loads
// at a time.  (Eight groups of threads with an eighth of the parts each, or eight pieces a block, are faster for a token in 2000
// of 30001 rows, 26 us as a plain loop, and slower where no token is in that many: 8192 rows 15 us where this takes 7.)
template <typename T, bool VEC, int TH>
__global__ void __launch_bounds__(TH) table_grad_join_kernel(TableGradParams p) {
  constexpr int V = Elem<T>::kVec;
  const int piece = (int)(blockIdx.x / p.tiles), tile = (int)(blockIdx.x - (unsigned)piece * p.tiles);
  const long long first = (long long)piece * p.piece, last = first + p.piece;
  if (last >= p.n) return;
  const int run = __ldg(p.key + last - 1), next = __ldg(p.key + last), start = __ldg(p.key + first);
  const int before = first > 0 ? __ldg(p.key + first - 1) : -1;
  if (!is_token(p, run) || next != run || (start == run && before == run)) return;     // ends here, or begun before
  int end = piece + 1;                                                                 // behind the pieces that find it begun
  while (true) {
    const int i = end + (int)threadIdx.x;
    const int found = __syncthreads_count(i < p.pieces && __ldg(p.key + (long long)i * p.piece) == run);
    end += found;
    if (found < TH) break;
  }
  float acc[V];
  int col[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    col[q] = grad_column<T, VEC, TH>(tile, q);
    acc[q] = col[q] < p.cols ? p.part[(2ll * piece + 1) * p.ldp + col[q]] : 0.f;
  }
  for (int i0 = piece + 1; i0 < end; i0 += 8) {
    float part[8][V];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int q = 0; q < V; ++q) part[u][q] = i0 + u < end && col[q] < p.cols ? p.part[2ll * (i0 + u) * p.ldp + col[q]] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int q = 0; q < V; ++q) acc[q] += part[u][q];
  }
  store_grad<T, VEC, TH>(p, run, tile, acc);
}

}  // namespace sgc

namespace {

using sgc::Carve;

size_t elem_size(int dtype) { return dtype == SGEMM_CUBE_F32 ? 4 : 2; }
bool bad_dtype(int dtype) { return dtype < SGEMM_CUBE_F32 || dtype > SGEMM_CUBE_BF16; }
bool bad_scale(float s) { return !std::isfinite(s); }

template <typename T, int TH>
int launch_lookup(sgemm_cube_ctx* h, sgc::LookupParams p, bool vec, cudaStream_t st) {
  const int span = TH * sgc::kLookupItems * sgc::Elem<T>::kVec, side = sgc::kLookupThreads / TH;
  p.pieces = (p.cols + span - 1) / span;
  const long long units = (p.rows * p.pieces + side - 1) / side, cap = 0x7FFFFFFF;
  const unsigned blocks = (unsigned)(units < cap ? units : cap);
  if (vec) sgc::embedding_kernel<T, true, TH><<<blocks, sgc::kLookupThreads, 0, st>>>(p);
  else sgc::embedding_kernel<T, false, TH><<<blocks, sgc::kLookupThreads, 0, st>>>(p);
  return sgc::launched(h);
}
// As few threads as have a vector each, 16 at least (both ends of a row that is off the boundaries are theirs too): 32768 rows of
// 128 FP32 10 us, 20 with 128 threads a row.
template <typename T>
int launch_lookup(sgemm_cube_ctx* h, const sgc::LookupParams& p, bool vec, cudaStream_t st) {
  constexpr int V = sgc::Elem<T>::kVec;
  if (p.cols <= 16 * V) return launch_lookup<T, 16>(h, p, vec, st);
  if (p.cols <= 32 * V) return launch_lookup<T, 32>(h, p, vec, st);
  return p.cols <= 64 * V ? launch_lookup<T, 64>(h, p, vec, st) : launch_lookup<T, 128>(h, p, vec, st);
}

template <typename T, int TH>
int launch_table_grad(sgemm_cube_ctx* h, sgc::TableGradParams p, bool vec, unsigned clear_blocks, cudaStream_t st) {
  constexpr int columns = TH * sgc::Elem<T>::kVec, side = sgc::kGradThreads / TH;
  p.tiles = (p.cols + columns - 1) / columns;
  const long long joins = (long long)p.pieces * p.tiles;
  if (joins > 0x3FFFFFFF) return SGEMM_CUBE_INVALID_ARG;
  p.sum_blocks = (unsigned)((long long)((p.pieces + side - 1) / side) * p.tiles);
  const unsigned blocks = p.sum_blocks + clear_blocks;
  if (vec) sgc::table_grad_kernel<T, true, TH><<<blocks, sgc::kGradThreads, 0, st>>>(p);
  else sgc::table_grad_kernel<T, false, TH><<<blocks, sgc::kGradThreads, 0, st>>>(p);
  int rc = sgc::launched(h);
  if (rc || p.pieces < 2) return rc;
  if (vec) sgc::table_grad_join_kernel<T, true, TH><<<(unsigned)joins, TH, 0, st>>>(p);
  else sgc::table_grad_join_kernel<T, false, TH><<<(unsigned)joins, TH, 0, st>>>(p);
  return sgc::launched(h);
}
template <typename T>
int launch_table_grad(sgemm_cube_ctx* h, const sgc::TableGradParams& p, bool vec, unsigned clear_blocks, cudaStream_t st) {
  constexpr int V = sgc::Elem<T>::kVec;
  if (p.cols <= 32 * V) return launch_table_grad<T, 32>(h, p, vec, clear_blocks, st);
  return p.cols <= 64 * V ? launch_table_grad<T, 64>(h, p, vec, clear_blocks, st) : launch_table_grad<T, 128>(h, p, vec, clear_blocks, st);
}

int launch_sort(sgemm_cube_ctx* h, const sgc::SortParams& p, int blocks, cudaStream_t st) {
  if (blocks > 1) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
    cfg.blockDim = dim3(sgc::kSortThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeCooperative;
    a.val.cooperative = 1;
    cfg.attrs = &a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, sgc::sort_tokens_kernel, p) == cudaSuccess) {
      h->launches++;
      return SGEMM_CUBE_OK;
    }
    cudaGetLastError();                          // a device that is partly occupied by others: one block does it
  }
  sgc::sort_tokens_kernel<<<1, sgc::kSortThreads, 0, st>>>(p);
  return sgc::launched(h);
}

}  // namespace

extern "C" {

int sgemm_cube_embedding(sgemm_cube_handle h, int rows, int vocab, int cols, int dtype, const int64_t* tokens, const void* table,
                         int64_t ld, float scale, void* Y, int64_t ldy, void* stream) {
  if (!h || bad_dims(rows, vocab, cols) || vocab < 1 || cols < 1 || ld < cols || ldy < cols || bad_dtype(dtype) || bad_scale(scale))
    return SGEMM_CUBE_INVALID_ARG;
  if (rows == 0) return SGEMM_CUBE_OK;
  const size_t e = elem_size(dtype);
  if (!tokens || !table || !Y || table == Y || misplaced(8, tokens) || misplaced(e, table, Y)) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  sgc::LookupParams p;
  memset(&p, 0, sizeof(p));
  p.rows = rows; p.vocab = vocab; p.cols = cols;
  p.tokens = reinterpret_cast<const long long*>(tokens);
  p.table = table; p.ld = ld;
  p.scale = scale;
  p.Y = Y; p.ldy = ldy;
  const bool vec = sgc::rows_take_vectors(table, ld, cols, e) && sgc::rows_take_vectors(Y, ldy, cols, e);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SGEMM_CUBE_F32) return launch_lookup<float>(h, p, vec, st);
  if (dtype == SGEMM_CUBE_F16) return launch_lookup<__half>(h, p, vec, st);
  return launch_lookup<__nv_bfloat16>(h, p, vec, st);
}

int sgemm_cube_embedding_backward(sgemm_cube_handle h, int rows, int vocab, int cols, int dtype, const int64_t* tokens,
                                  const void* dY, int64_t lddy, float scale, int accumulate, float* dtable, int64_t ldd,
                                  void* stream) {
  if (!h || bad_dims(rows, vocab, cols) || vocab < 1 || cols < 1 || lddy < cols || ldd < cols || bad_dtype(dtype) || bad_scale(scale))
    return SGEMM_CUBE_INVALID_ARG;
  if (accumulate != 0 && accumulate != 1) return SGEMM_CUBE_INVALID_ARG;
  const size_t e = elem_size(dtype);
  if (!dtable || misplaced(4, dtable)) return SGEMM_CUBE_INVALID_ARG;
  if (rows > 0 && (!tokens || !dY || misplaced(8, tokens) || misplaced(e, dY))) return SGEMM_CUBE_INVALID_ARG;
  DeviceGuard g(h->device);
  if (!g.ok) return SGEMM_CUBE_CUDA_ERROR;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {                               // empty sums
    if (accumulate) return SGEMM_CUBE_OK;
    if (cudaMemset2DAsync(dtable, (size_t)ldd * 4, 0, (size_t)cols * 4, vocab, st) != cudaSuccess) {
      cudaGetLastError();
      return SGEMM_CUBE_CUDA_ERROR;
    }
    return SGEMM_CUBE_OK;
  }
  // Pieces of 32 sorted rows; longer ones (fewer parts to join for a frequent token) where eight blocks an SM have one all the same,
  // and where there would be more than 4096: 32768 x 8192 BF16 in 60000 rows,
  // with the lookup, 644 us with pieces of 32, 627 with 256.
  int piece = rows <= 32 * 4096 ? 32 : (int)(((long long)rows + 4095) / 4096);
  const long long row_tiles = ((long long)cols * e + 2047) / 2048;       // about: 128 threads with 16 bytes each
  while (piece < 256 && rows / (2 * piece) * row_tiles >= 8 * h->sm_count) piece *= 2;
  sgc::TableGradParams p;
  memset(&p, 0, sizeof(p));
  p.n = rows; p.vocab = vocab; p.cols = cols;
  p.piece = piece; p.pieces = (rows + piece - 1) / piece;
  p.dY = dY; p.lddy = lddy;
  p.scale = scale;
  p.accumulate = accumulate;
  p.dE = dtable; p.ldd = ldd;
  p.ldp = (int64_t)round_up((size_t)cols, 4);
  p.vec_out = sgc::rows_take_vectors(dtable, ldd, cols, 4);
  const bool vec = sgc::rows_take_vectors(dY, lddy, cols, e);
  sgc::SortParams s;
  memset(&s, 0, sizeof(s));
  s.n = rows; s.vocab = vocab;
  for (s.passes = 1; s.passes < 4 && (vocab >> (s.passes * sgc::kSortBits)) != 0; ++s.passes) {}
  s.tokens = reinterpret_cast<const long long*>(tokens);
  s.words = h->err_dev + sgc::kGridWords + 2;
  s.err = h->err_dev;
  const bool ranked = rows > sgc::kSortFew && rows <= sgc::kRankMost;
  const int sort_tiles = (rows + sgc::kSortTile - 1) / sgc::kSortTile;
  const int blocks = sort_tiles < h->sm_count ? sort_tiles : h->sm_count;
  int rc;
  for (int pass = 0; pass < 2; ++pass) {         // sizes first, then pointers
    Carve c;
    c.base = pass ? static_cast<uint8_t*>(h->sort_ws) : nullptr;
    for (int i = 0; i < 2; ++i) {
      s.key[i] = c.take<int>((size_t)rows);
      s.pos[i] = c.take<int>((size_t)rows);
    }
    s.hist = c.take<int>((size_t)blocks * sgc::kSortBins);
    s.met = c.take<unsigned char>(round_up((size_t)vocab, 16));
    if (p.pieces > 1) p.part = c.take<float>((size_t)2 * p.pieces * p.ldp);
    if (!pass && (rc = grow(h, &h->sort_ws, &h->sort_ws_bytes, c.used, st))) return rc;
  }
  if (accumulate) s.met = nullptr;
  if (s.met) {                                   // 8 turns of the sort's blocks at the most, else a launch of its own
    s.clear = !ranked && (size_t)vocab <= (size_t)blocks * sgc::kSortThreads * 16 * 8;
    if (!s.clear && cudaMemsetAsync(s.met, 0, (size_t)vocab, st) != cudaSuccess) {
      cudaGetLastError();
      return SGEMM_CUBE_CUDA_ERROR;
    }
  }
  if (ranked) {
    sgc::rank_tokens_kernel<<<(unsigned)((rows + sgc::kRankBlock - 1) / sgc::kRankBlock), sgc::kRankThreads, 0, st>>>(s);
    if ((rc = sgc::launched(h))) return rc;
  } else if ((rc = launch_sort(h, s, blocks, st))) {
    return rc;
  }
  p.key = s.key[s.passes & 1];
  p.pos = s.pos[s.passes & 1];
  p.met = s.met;
  const long long clear_pieces = (long long)vocab * cols / sgc::kClearPiece + 2, clear_most = 1 << 24;      // (64 G floats; more take turns)
  const unsigned clear_blocks = accumulate ? 0u : (unsigned)(clear_pieces < clear_most ? clear_pieces : clear_most);
  if (dtype == SGEMM_CUBE_F32) return launch_table_grad<float>(h, p, vec, clear_blocks, st);
  if (dtype == SGEMM_CUBE_F16) return launch_table_grad<__half>(h, p, vec, clear_blocks, st);
  return launch_table_grad<__nv_bfloat16>(h, p, vec, clear_blocks, st);
}

}  // extern "C"
