// Launches over a whole list of tensors (adamw.hip, grad_norm.hip): the list is a kernel argument, every workgroup takes
// one span of consecutive elements of one tensor.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace galore {

constexpr int64_t kMaxBlocks = (int64_t)1 << 23;  // workgroups per launch: a launch has fewer than 2^32 work-items

// Tensor that workgroup `block` belongs to: begin[i] is the first workgroup of tensor i, ascending.  One load per 64
// tensors and a ballot in place of a binary search, whose steps would wait for each other.
template <int N> __device__ __forceinline__ int tensor_of_block(const int32_t (&begin)[N], int count, int block) {
  const int lane = threadIdx.x & 63;
  int found = -1;
#pragma unroll
  for (int base = 0; base < N; base += 64) {
    const int i = base + lane;
    const int b = i < count && i < N ? begin[i < N ? i : 0] : INT32_MAX;
    found += __popcll(__ballot(b <= block));
  }
  return __builtin_amdgcn_readfirstlane(found);
}

// Workgroups reach the 8 XCDs in turn: with this numbering each XCD takes runs of 512 consecutive spans, so that the
// streams of one XCD stay in few DRAM pages (AdamW, 128 threads each, 262M bf16 weights: 934 us numbered as launched, 912
// in runs; 30M fp32: 135 and 132).  Launches, and their ends, of fewer than 4096 workgroups keep their numbers.
__device__ __forceinline__ int span_of_block() {
  constexpr int kRun = 512, kXcds = 8;
  const int block = blockIdx.x, in_group = block % (kRun * kXcds), group = block - in_group;
  return group + kRun * kXcds <= (int)gridDim.x ? group + in_group % kXcds * kRun + in_group / kXcds : block;
}

// Where element o of a span lies in a matrix whose rows may be apart: row and column, from which every tensor of that shape
// finds its own offset.  o < 2^20 and cols < 2^30: the division is one of 32 bits.
struct RowWalk {
  int64_t row0;
  uint32_t col0, cols;
  __device__ __forceinline__ RowWalk(int64_t first, int32_t cols_) : cols(cols_) {
    row0 = first / cols_;
    col0 = (uint32_t)(first - row0 * cols_);
  }
  struct Place {
    int64_t row;
    uint32_t col, left;   // left: elements of the row from this one on
    // element o of a run without gaps, counted from where the run starts
    static __device__ __forceinline__ Place in_run(int o) { return Place{0, (uint32_t)o, 0x7FFFFFFFu}; }
    __device__ __forceinline__ int64_t offset(int32_t ld) const { return row * ld + col; }
  };
  __device__ __forceinline__ Place at(int o) const {
    const uint32_t c = col0 + (uint32_t)o, r = c / cols, x = c - r * cols;
    return Place{row0 + r, x, cols - x};
  }
};

// Vectors at element alignment: the hardware takes global accesses at any alignment.
typedef float list_f32x4 __attribute__((ext_vector_type(4)));
typedef float list_f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 list_bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float list_f32x8_any __attribute__((ext_vector_type(8), aligned(4)));
typedef __bf16 list_bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
template <class T, int N> struct ListVec;
template <> struct ListVec<float, 4> { typedef list_f32x4_any type; };
template <> struct ListVec<__bf16, 4> { typedef list_bf16x4_any type; };
template <> struct ListVec<float, 8> { typedef list_f32x8_any type; };
template <> struct ListVec<__bf16, 8> { typedef list_bf16x8_any type; };
template <int N> using ListF32 = float __attribute__((ext_vector_type(N)));

// CACHED: another kernel is about to read the same again; else past the caches
template <int N, bool CACHED = false, class T> __device__ __forceinline__ ListF32<N> list_load(const T* p) {
  typedef typename ListVec<T, N>::type V;
  const V* v = reinterpret_cast<const V*>(p);
  return __builtin_convertvector(CACHED ? *v : __builtin_nontemporal_load(v), ListF32<N>);
}
template <int N, class T> __device__ __forceinline__ void list_store(T* p, ListF32<N> x) {
  typedef typename ListVec<T, N>::type V;
  __builtin_nontemporal_store(__builtin_convertvector(x, V), reinterpret_cast<V*>(p));
}

// N elements from place `at` on, the first n of which the tensor has (the others count as zero): rows of `cols` elements
// may lie apart.  Past a row's end the offset grows by the gap: no further division, and no load waits for another.
template <int N, bool CACHED = false, class T>
__device__ __forceinline__ ListF32<N> row_load(const T* p, int32_t ld, int32_t cols, const RowWalk::Place& at, int n) {
  p += at.offset(ld);
  if (n >= N && at.left >= N) return list_load<N, CACHED>(p);
  ListF32<N> x = 0.f;
  int64_t skip = 0;
  uint32_t left = at.left;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (left == 0) { skip += ld - cols; left = cols; }
    if (e < n) x[e] = (float)p[e + skip];
    --left;
  }
  return x;
}
template <int N, class T>
__device__ __forceinline__ void row_store(T* p, int32_t ld, int32_t cols, const RowWalk::Place& at, int n, ListF32<N> x) {
  p += at.offset(ld);
  if (n >= N && at.left >= N) { list_store<N>(p, x); return; }
  int64_t skip = 0;
  uint32_t left = at.left;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (left == 0) { skip += ld - cols; left = cols; }
    if (e < n) p[e + skip] = (T)x[e];
    --left;
  }
}

}  // namespace galore
