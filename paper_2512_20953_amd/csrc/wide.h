// Consecutive elements of rows in bf16 or fp32 as one access, checks of alignment and indices of 32 or 64 bits, for the operators around the stages.
#pragma once
#include "common.h"
#include <type_traits>

namespace ah {

// N elements as they lie in memory: aligned to 16 bytes where they fill as many, else to themselves
template <class T, int N> struct Wide {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type at __attribute__((aligned(sizeof(T) * N < 16 ? sizeof(T) * N : 16)));
};
template <class T, int N> using wide_t = typename Wide<T, N>::type;
template <int N, class T> __device__ __forceinline__ wide_t<T, N> load_wide(const T* p) { return *(const typename Wide<T, N>::at*)p; }
template <int N, class T> __device__ __forceinline__ void store_wide(T* p, wide_t<T, N> v) { *(typename Wide<T, N>::at*)p = v; }

// Whether rows of elements of `size` bytes, `ld` elements apart from `p` on, all begin at multiples of 16 bytes
inline bool rows16(const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uint64_t)(ld * size)) & 15) == 0; }
inline bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// an index of 32 or 64 bits
__device__ __forceinline__ int64_t load_index(const void* p, size_t i, int bits) {
  return bits == 64 ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
}

}  // namespace ah
