// What kernels that read rows share: 16 bytes of one, and the division of a row's number.
#pragma once
#include <hip/hip_runtime.h>

namespace lazyev {

typedef __attribute__((ext_vector_type(4))) unsigned rows_u32x4_t;

// 16 bytes; `wide`: they lie at a multiple of 16, otherwise elements at any address of their own type.
template <typename T>
__device__ __forceinline__ rows_u32x4_t load_chunk(const T *p, bool wide) {
  if (wide) return *reinterpret_cast<const rows_u32x4_t *>(p);
  T e[16 / sizeof(T)];
#pragma unroll
  for (int x = 0; x < static_cast<int>(16 / sizeof(T)); ++x) e[x] = p[x];
  rows_u32x4_t w;
  __builtin_memcpy(&w, e, 16);
  return w;
}

// x / y for 0 <= x < 2^24, y > 0 (the rounded quotient is off by one at most).
__device__ __forceinline__ int quotient(int x, int y) {
  int q = static_cast<int>(static_cast<float>(x) * __builtin_amdgcn_rcpf(static_cast<float>(y)));
  const int r = x - q * y;
  q += r >= y ? 1 : 0;
  return q - (r < 0 ? 1 : 0);
}

}  // namespace lazyev
