// FP32, FP16 and BF16 elements for the kernels that work in FP32 whatever the storage type: 16-byte
// vectors and single elements, converted on load and rounded once (to nearest even) on store.
#pragma once

#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace sgc {

template <typename T>
struct Elem;

template <>
struct Elem<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};

template <>
struct Elem<__half> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};

template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};

// A thread of a group of `threads` holds PT elements of a row: 16-byte vectors, vector i at (i * threads + t) * kVec, or
// (rows that are not 16-byte aligned) single elements, element i at i * threads + t.  Either way a warp's accesses are
// contiguous, and columns past `cols` read as zero.
// Single elements of a row that is asked for (fetch) before it is needed (get): they wait in registers.
template <typename T, int PT>
struct RowRegs {
  T raw[PT];
  __device__ __forceinline__ void fetch(const T* row, int cols, int t, int threads) {
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int c = i * threads + t;
      raw[i] = c < cols ? row[c] : Elem<T>::put(0.f);
    }
  }
  __device__ __forceinline__ void get(float (&v)[PT]) const {
#pragma unroll
    for (int i = 0; i < PT; ++i) v[i] = Elem<T>::get(raw[i]);
  }
};
// The same through shared memory, for vectors: a thread's own 16-byte slots, filled by asynchronous copies of the
// thread itself, so nobody else has to be waited for, rows can be asked for several ahead, and the copies are under
// way whatever the compiler does with the loads around them (it moved the loads into registers behind the arithmetic,
// where registers were short).  `slots` is the thread's first of kWords, `pitch` uint4 apart.
template <typename T, int PT>
struct RowSlots {
  static constexpr int kWords = PT / Elem<T>::kVec;
  static __device__ __forceinline__ void ask(uint4* slots, int pitch, const T* row, int cols, int t, int threads) {
    constexpr int V = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int c = (i * threads + t) * V;
      const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(slots + i * pitch));
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"        // 0 bytes read: zeros
                   ::"r"(dst), "l"(row + (c < cols ? c : 0)), "r"(c < cols ? 16 : 0) : "memory");
    }
  }
  static __device__ __forceinline__ void get(const uint4* slots, int pitch, float (&v)[PT]) {
    constexpr int V = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      float e[V];
      Elem<T>::unpack(slots[i * pitch], e);
#pragma unroll
      for (int q = 0; q < V; ++q) v[i * V + q] = e[q];
    }
  }
};
// Vectors of rows that start `shift` elements behind a 16-byte boundary, laid on the boundaries: vector i of a thread at
// i * threads * kVec + first, first = t * kVec - shift.  The first and the last may reach outside the row, where the
// elements are zero.  What the first one brings from the row before is put to zero on the way out; row 0 has none
// before it (`lead`), and there the thread copies the elements itself.
template <typename T, int PT>
struct ShiftedSlots {
  static constexpr int V = Elem<T>::kVec, kWords = PT / V;
  static __device__ __forceinline__ void ask(uint4* slots, int pitch, const T* row, int cols, int first, int threads, bool lead) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int c = i * threads * V + first;
      if (i == 0 && c < 0 && lead) {
        T e[V];
#pragma unroll
        for (int q = 0; q < V; ++q) e[q] = c + q >= 0 ? row[c + q] : Elem<T>::put(0.f);
        *slots = *reinterpret_cast<const uint4*>(e);
        continue;
      }
      const int bytes = min(16, max(0, (cols - c) * (int)sizeof(T)));     // the rest of the slot becomes zero
      const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(slots + i * pitch));
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                   ::"r"(dst), "l"(row + (bytes > 0 ? c : first % V)), "r"(bytes) : "memory");
    }
  }
  static __device__ __forceinline__ void vector(const uint4* slots, int pitch, int i, int first, float (&e)[V]) {
    Elem<T>::unpack(slots[i * pitch], e);
    if (i == 0 && first < 0) {
#pragma unroll
      for (int q = 0; q < V; ++q) e[q] = first + q >= 0 ? e[q] : 0.f;
    }
  }
  static __device__ __forceinline__ void store(T* row, int cols, int c, const float (&e)[V]) {
    if (c >= 0 && c + V <= cols) {
      *reinterpret_cast<uint4*>(row + c) = Elem<T>::pack(e);
    } else if (c < cols) {
#pragma unroll
      for (int q = 0; q < V; ++q)
        if ((unsigned)(c + q) < (unsigned)cols) row[c + q] = Elem<T>::put(e[q]);
    }
  }
};
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The thread's entries of a vector of FP32 parameters, `fill` past the end or where there is none.  The vector is
// read in 16-byte pieces where the rows are and it is aligned itself.
template <typename T, int PT, bool VEC>
__device__ __forceinline__ void load_params(const float* p, float fill, int cols, int t, int threads, float (&v)[PT]) {
  constexpr int V = VEC ? Elem<T>::kVec : 1;
  const bool vec = VEC && (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
#pragma unroll
  for (int i = 0; i < PT / V; ++i) {
    const int c = (i * threads + t) * V;
    if (VEC && p && vec && c < cols) {
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(p + c + q));
        v[i * V + q] = f.x; v[i * V + q + 1] = f.y; v[i * V + q + 2] = f.z; v[i * V + q + 3] = f.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < V; ++q) v[i * V + q] = p && c + q < cols ? __ldg(p + c + q) : fill;
    }
  }
}
template <typename T, int PT, bool VEC>
__device__ __forceinline__ void store_row(T* row, int cols, int t, int threads, const float (&v)[PT]) {
  if constexpr (VEC) {
    constexpr int V = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < PT / V; ++i) {
      const int c = (i * threads + t) * V;
      float e[V];
#pragma unroll
      for (int q = 0; q < V; ++q) e[q] = v[i * V + q];
      if (c < cols) *reinterpret_cast<uint4*>(row + c) = Elem<T>::pack(e);
    }
  } else {
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int c = i * threads + t;
      if (c < cols) row[c] = Elem<T>::put(v[i]);
    }
  }
}
// Column of the thread's element i.
template <typename T, bool VEC>
__device__ __forceinline__ int row_column(int i, int t, int threads) {
  if constexpr (VEC) {
    constexpr int V = Elem<T>::kVec;
    return (i / V * threads + t) * V + i % V;
  } else {
    return i * threads + t;
  }
}

// Whether rows of `ld` elements from p are 16-byte aligned and whole vectors long.
inline bool rows_take_vectors(const void* p, int64_t ld, int cols, size_t elem) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * elem) % 16 == 0 && (cols * elem) % 16 == 0;
}

}  // namespace sgc
