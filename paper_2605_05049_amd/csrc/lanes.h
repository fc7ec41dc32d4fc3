// Sums and maxima over neighbouring lanes, by moves inside the rows of 16 lanes and exchanges of rows and halves.
#pragma once

#include "common.h"

namespace moe {

// v of another lane: 1, 2 and, where the lanes of a quad (of eight) hold the same, 4 and 8 further on by moves inside the rows of 16, else through LDS.
template <int STEP>
__device__ __forceinline__ int from_lane(int v) {
  if constexpr (STEP == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);         // quad_perm 1 0 3 2
  else if constexpr (STEP == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);    // quad_perm 2 3 0 1
  else if constexpr (STEP == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true);   // row_half_mirror
  else if constexpr (STEP == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true);   // row_mirror
  else {
    static_assert(STEP == 16 || STEP == 32, "a power of two below 64");
    const bool upper = (threadIdx.x & STEP) != 0;   // (rows, or halves, change places between two registers that hold the same)
    if constexpr (STEP == 16) {
      const auto r = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
      return upper ? r[0] : r[1];
    } else {
      const auto r = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
      return upper ? r[0] : r[1];
    }
  }
}
template <int STEP>
__device__ __forceinline__ float from_lane(float v) { return __int_as_float(from_lane<STEP>(__float_as_int(v))); }
template <int STEP>
__device__ __forceinline__ double from_lane(double v) { return __hiloint2double(from_lane<STEP>(__double2hiint(v)), from_lane<STEP>(__double2loint(v))); }

// Over W neighbouring lanes, for each of them.
template <int W, int STEP = 1, typename T>
__device__ __forceinline__ T lanes_sum(T v) {
  if constexpr (STEP < W) return lanes_sum<W, 2 * STEP>(v + from_lane<STEP>(v));
  else return v;
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
template <int W, int STEP = 1, typename T>
__device__ __forceinline__ T lanes_max(T v) {
  if constexpr (STEP < W) return lanes_max<W, 2 * STEP>(larger(v, from_lane<STEP>(v)));
  else return v;
}

}  // namespace moe
