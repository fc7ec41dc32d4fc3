// Microscaled 4-bit floating point (MXFP4 of the OCP Microscaling formats): blocks of 32 values along the contraction share a scale
// 2^(s - 127), s an 8-bit code (255: the block is NaN); a value is an E2M1 code, +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, times the scale.
// Even positions sit in the low nibble of a byte.
#pragma once

#include "few_rows.h"   // (wave_prefix_sum, pack8)

namespace moe {

constexpr int kMxBlock = 32;

typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x8 __attribute__((ext_vector_type(8)));

// The scale code of a block whose largest magnitude has the biased 8-bit exponent `e` (bf16 and fp32 share it): floor(log2) - 2, the
// exponent of the largest element 6 = 1.5 * 2^2, at least 2^-127; 255 for infinities and NaN.
__device__ __forceinline__ unsigned mx_scale_code(unsigned e) { return e == 255u ? 255u : e < 2u ? 0u : e - 2u; }

// Eight values of a block with scale code s -> eight codes (round to nearest even, at most 6).  The values are brought into range in fp32,
// exactly (a product with a power of two; those that fall below the range of fp32 are below 2^-100 of the smallest code), and converted at scale 1.
__device__ __forceinline__ unsigned mx_encode8(const float (&x)[8], unsigned s) {
  if (s == 255u) return 0u;
  const float inv = __uint_as_float((254u - s) << 23);   // 2^(127 - s); s <= 253
  unsigned q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[0] * inv, x[1] * inv, 1.0f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[2] * inv, x[3] * inv, 1.0f, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[4] * inv, x[5] * inv, 1.0f, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[6] * inv, x[7] * inv, 1.0f, 3);
  return q;
}

// The expert that row tile u belongs to, among tiles of TILE rows of each expert's segment; false past the last tile.  Every wavefront looks
// for itself: 64 experts at a time, one per lane, until the running sum of their tiles passes u.
struct MxSegment { int expert, lo, hi, first; };   // rows lo .. hi - 1, index of the first tile
template <int TILE>
__device__ __forceinline__ bool mx_find_expert(const int32_t* __restrict__ offsets, int E, int u, int lane, MxSegment& S) {
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = min(e0 + lane, E - 1);
    const int lo = offsets[e], hi = e0 + lane < E ? offsets[e + 1] : lo;
    const int n = (hi - lo + TILE - 1) / TILE;
    const int incl = before + wave_prefix_sum(n);
    const unsigned long long past = __ballot(incl > u);
    if (past) {
      const int l = __builtin_ctzll(past);
      S.expert = e0 + l;
      S.first = __builtin_amdgcn_readlane(incl - n, l);
      S.lo = __builtin_amdgcn_readlane(lo, l);
      S.hi = __builtin_amdgcn_readlane(hi, l);
      return true;
    }
    before = __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  return false;
}

}  // namespace moe
