// Grouped products of rows and weights in microscaled 4-bit floating point.
#pragma once

#include "mxfp4.h"

namespace moe {

enum MxKind { MX_PRODUCT = 0, MX_GATE_UP = 1 };   // bf16 y = x W; or silu(x W_gate) (x W_up), quantised
struct MxGemmArgs {
  const int32_t* offsets;   // [E + 1]
  int E, n, k;              // columns of the result, length of the contraction
  const uint8_t* x; const uint8_t* xs;      // [rows, k / 2], [rows, k / 32]
  const uint8_t* w0; const uint8_t* ws0;    // [E, n, k / 2], [E, n, k / 32]
  const uint8_t* w1; const uint8_t* ws1;    // W_up
  uint16_t* y;              // [rows, n]
  uint8_t* h; uint8_t* hs;  // [rows, n / 2], [rows, n / 32]
};
void launch_mx_gemm(const char* label, hipStream_t st, MxKind kind, const MxGemmArgs& A, long long rows);
void launch_mx_quantize(hipStream_t st, const uint16_t* x, uint8_t* q, uint8_t* scales, long long n);

}  // namespace moe
