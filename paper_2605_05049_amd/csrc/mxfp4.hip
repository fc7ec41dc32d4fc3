// Quantisation to microscaled 4-bit floating point, along rows and along columns, and the way back.
//
// All three are bound by HBM: 2 + 17/32 bytes per value.  Measured: rows 65536 x 4096, 118 us (5.8 TB/s); columns of 66 matrices of 2048 x 1408, 118 us
// (4.1 TB/s), and back, 73 us (6.6 TB/s).  A copy of 8.6 GB reaches 4.75 TB/s of both ways, a read 6.2, a fill 6.85.
#include "mxfp4.h"

namespace moe {

namespace {

constexpr int kMxChunks = 4;   // chunks of 8 values per thread

// Largest magnitude of 8 bf16, as a bit pattern (order of the patterns without sign = order of the magnitudes; NaN above infinity).
__device__ __forceinline__ unsigned abs_max8(const uint4& v) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  auto mag = [](unsigned w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
  u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(v.x), mag(v.y)), __builtin_elementwise_max(mag(v.z), mag(v.w)));
  return m.x > m.y ? m.x : m.y;
}

}  // namespace

// x [n] -> q [n / 2], scales [n / 32]: rows are a multiple of 32 long, so the blocks lie one after the other in memory whatever the row
// length.  A lane holds 8 values (one 16-byte load), four lanes a block.
__global__ __launch_bounds__(256) void mx_quantize_kernel(const uint4* __restrict__ x, uint32_t* __restrict__ q, uint8_t* __restrict__ scales,
                                                          long long n8) {
  const long long base = (long long)blockIdx.x * (256 * kMxChunks) + threadIdx.x;
  uint4 v[kMxChunks];
#pragma unroll
  for (int i = 0; i < kMxChunks; i++)
    if (base + i * 256 < n8) v[i] = x[base + i * 256];
#pragma unroll
  for (int i = 0; i < kMxChunks; i++) {
    const long long c = base + i * 256;
    if (c >= n8) break;   // (whole blocks leave together: n8 is a multiple of 4)
    unsigned m = abs_max8(v[i]);
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));   // quad_perm 1 0 3 2
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));   // quad_perm 2 3 0 1
    const unsigned s = mx_scale_code(m >> 7);
    float f[8];
    unpack8(v[i], f);
    q[c] = mx_encode8(f, s);
    if ((threadIdx.x & 3) == 0) scales[c >> 2] = (uint8_t)s;
  }
}

// w [K][C] of one matrix -> q [C][K / 2], scales [C][K / 32].  A block takes 256 k x 128 columns: a wavefront one block of 32 k of them, a lane
// two columns (a dword of each k-row, so that the largest magnitudes are packed maxima of whole dwords).  The codes meet in LDS, from where
// a column's 128 bytes are stored at once.
constexpr int kMxTK = 256, kMxTC = 128, kMxTPitch = kMxTK / 2 + 16;
__global__ __launch_bounds__(512) void mx_quantize_t_kernel(const uint16_t* __restrict__ w, uint8_t* __restrict__ q, uint8_t* __restrict__ scales,
                                                            int K, int C) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  __shared__ __attribute__((aligned(16))) char codes[kMxTC * kMxTPitch];
  __shared__ uint8_t code_scales[kMxTC][kMxTK / kMxBlock];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c0 = blockIdx.x * kMxTC, k0 = blockIdx.y * kMxTK;
  const size_t matrix = (size_t)blockIdx.z * K * C;
  const int c = min(c0 + 2 * lane, C - 2), k = k0 + wave * kMxBlock;   // (C is even)
  if (k < K) {
    const uint16_t* const src = w + matrix + (size_t)k * C + c;
    unsigned v[kMxBlock];
#pragma unroll
    for (int i = 0; i < kMxBlock; i++) v[i] = *reinterpret_cast<const unsigned*>(src + (size_t)i * C);
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < kMxBlock; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
    const unsigned s0 = mx_scale_code((unsigned)m.x >> 7), s1 = mx_scale_code((unsigned)m.y >> 7);
    unsigned q0[4], q1[4];
#pragma unroll
    for (int g = 0; g < 4; g++) {
      float lo[8], hi[8];
#pragma unroll
      for (int j = 0; j < 8; j++) { lo[j] = bf16lo(v[8 * g + j]); hi[j] = bf16hi(v[8 * g + j]); }
      q0[g] = mx_encode8(lo, s0);
      q1[g] = mx_encode8(hi, s1);
    }
    char* const dst = codes + 2 * lane * kMxTPitch + wave * 16;
    *reinterpret_cast<uint4*>(dst) = make_uint4(q0[0], q0[1], q0[2], q0[3]);
    *reinterpret_cast<uint4*>(dst + kMxTPitch) = make_uint4(q1[0], q1[1], q1[2], q1[3]);
    code_scales[2 * lane][wave] = (uint8_t)s0;
    code_scales[2 * lane + 1][wave] = (uint8_t)s1;
  }
  __syncthreads();
  const size_t col0 = (size_t)blockIdx.z * C + c0;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int item = threadIdx.x + i * 512, col = item >> 3, part = item & 7;   // 16 bytes (a block of 32 k) of a column
    if (c0 + col < C && k0 + part * kMxBlock < K) {
      *reinterpret_cast<uint4*>(q + (col0 + col) * (size_t)(K / 2) + k0 / 2 + part * 16) =
          *reinterpret_cast<const uint4*>(codes + col * kMxTPitch + part * 16);
      scales[(col0 + col) * (size_t)(K / kMxBlock) + k0 / kMxBlock + part] = code_scales[col][part];
    }
  }
}

// q [n / 2], scales [n / 32] -> x [n] bf16 (exact: a code has 2 significant bits; beyond the range of bf16 an infinity).
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t* __restrict__ q, const uint8_t* __restrict__ scales, uint4* __restrict__ x,
                                                            long long n8) {
  const long long base = (long long)blockIdx.x * (256 * kMxChunks) + threadIdx.x;
  uint32_t v[kMxChunks];
  unsigned s[kMxChunks];
#pragma unroll
  for (int i = 0; i < kMxChunks; i++)
    if (base + i * 256 < n8) { v[i] = q[base + i * 256]; s[i] = scales[(base + i * 256) >> 2]; }
#pragma unroll
  for (int i = 0; i < kMxChunks; i++) {
    if (base + i * 256 >= n8) break;
    // 2^(s - 127): at 0 half the smallest normal number; 255 is NaN
    const float scale = __uint_as_float(s[i] == 0u ? 0x00400000u : s[i] == 255u ? 0x7fc00000u : s[i] << 23);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    float f[8];
#define MOE_MX_PAIR(j) { const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[i], 1.0f, j); f[2 * j] = p.x * scale; f[2 * j + 1] = p.y * scale; }
    MOE_MX_PAIR(0) MOE_MX_PAIR(1) MOE_MX_PAIR(2) MOE_MX_PAIR(3)
#undef MOE_MX_PAIR
    x[base + i * 256] = pack8(f);
  }
}

// Argument checks shared by the three: `values` = bf16 side.
static int check_mx(const void* values, const void* q, const void* scales, int64_t rows, int cols) {
  if (rows < 0 || cols < kMxBlock || cols % kMxBlock) return MOE_ERR_SHAPE;
  if (rows > ((int64_t)1 << 36) / cols) return MOE_ERR_SHAPE;   // (a launch has fewer than 2^32 threads, of 32 values each)
  if (rows == 0) return MOE_OK;
  MOE_REQUIRE_PTR(values); MOE_REQUIRE_PTR(q); MOE_REQUIRE_PTR(scales);
  MOE_REQUIRE_ALIGNED(values); MOE_REQUIRE_ALIGNED(q); MOE_REQUIRE_ALIGNED(scales);
  return MOE_OK;
}

void launch_mx_quantize(hipStream_t st, const uint16_t* x, uint8_t* q, uint8_t* scales, long long n) {
  const long long n8 = n / 8, per = 256 * kMxChunks;
  MOE_LAUNCH("mx_quantize", st, mx_quantize_kernel, dim3((unsigned)((n8 + per - 1) / per)), dim3(256), 0, st, reinterpret_cast<const uint4*>(x),
             reinterpret_cast<uint32_t*>(q), scales, n8);
}

}  // namespace moe

extern "C" int moe_mxfp4_quantize(const uint16_t* x, int64_t rows, int cols, uint8_t* q, uint8_t* scales, void* stream) {
  using namespace moe;
  const int rc = check_mx(x, q, scales, rows, cols);
  if (rc != MOE_OK || rows == 0) return rc;
  launch_mx_quantize((hipStream_t)stream, x, q, scales, rows * cols);
  return launch_status();
}

extern "C" int moe_mxfp4_quantize_t(const uint16_t* w, int batch, int rows, int cols, uint8_t* q, uint8_t* scales, void* stream) {
  using namespace moe;
  if (batch < 0 || batch > 65535 || cols < 8 || cols % 8 || rows > 65535 * kMxTK) return MOE_ERR_SHAPE;
  const int rc = check_mx(w, q, scales, (int64_t)batch * cols, rows);
  if (rc != MOE_OK || batch == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)((cols + kMxTC - 1) / kMxTC), (unsigned)((rows + kMxTK - 1) / kMxTK), (unsigned)batch);
  if ((unsigned long long)grid.x * grid.y * grid.z >= (1ull << 23)) return MOE_ERR_SHAPE;   // (of 512 threads)
  MOE_LAUNCH("mx_quantize_t", st, mx_quantize_t_kernel, grid, dim3(512), 0, st, w, q, scales, rows, cols);
  return launch_status();
}

extern "C" int moe_mxfp4_dequantize(const uint8_t* q, const uint8_t* scales, int64_t rows, int cols, uint16_t* x, void* stream) {
  using namespace moe;
  const int rc = check_mx(x, q, scales, rows, cols);
  if (rc != MOE_OK || rows == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const long long n8 = rows * cols / 8, per = 256 * kMxChunks;
  MOE_LAUNCH("mx_dequantize", st, mx_dequantize_kernel, dim3((unsigned)((n8 + per - 1) / per)), dim3(256), 0, st,
             reinterpret_cast<const uint32_t*>(q), scales, reinterpret_cast<uint4*>(x), n8);
  return launch_status();
}
