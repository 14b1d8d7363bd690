// Numbers of the lanes of a wave joined, without LDS.
#pragma once
#include <hip/hip_runtime.h>

namespace lazyev {

// x of the lanes whose numbers differ in the bits kFrom .. kTo (powers of two) joined; a step of 4 takes the steps of 1 and 2 to be done.
template <int kStep>
__device__ __forceinline__ unsigned from_lane(unsigned x) {
  constexpr int kCtrl = kStep == 1 ? 0xB1 : kStep == 2 ? 0x4E : kStep == 4 ? 0x141 : 0x128;   // (quad_perm twice, row_half_mirror, row_ror by 8)
  return static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xF, 0xF, false));
}
template <int kStep, typename V, typename F>
__device__ __forceinline__ V join_step(V x, F join) {
  constexpr int kWords = sizeof(V) / 4;
  unsigned w[kWords], a[kWords], b[kWords];
  __builtin_memcpy(w, &x, sizeof(V));
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if constexpr (kStep < 16) {
      a[i] = w[i];
      b[i] = from_lane<kStep>(w[i]);
    } else {
      const auto r = kStep == 16 ? __builtin_amdgcn_permlane16_swap(w[i], w[i], false, false) : __builtin_amdgcn_permlane32_swap(w[i], w[i], false, false);
      a[i] = r[0];
      b[i] = r[1];
    }
  }
  V y, z;
  __builtin_memcpy(&y, a, sizeof(V));
  __builtin_memcpy(&z, b, sizeof(V));
  return join(y, z);
}
template <int kFrom, int kTo, typename V, typename F>
__device__ __forceinline__ V join_lanes(V x, F join) {
  x = join_step<kFrom>(x, join);
  if constexpr (kFrom < kTo) x = join_lanes<2 * kFrom, kTo>(x, join);
  return x;
}

}  // namespace lazyev
