// The norm in front of a layer, with the residual sum in front of it, and its gradients.
//
//   h = x + addend,  y = (h - mean) rstd gamma + beta,  rstd = 1 / sqrt(mean((h - mean)^2) + eps)   (RMS norm: mean taken as 0)
//   dx = rstd (g - mean(g) - xh mean(g xh)) + dx_addend,  g = dy gamma,  xh = (h - mean) rstd;   dgamma = sum dy xh,  dbeta = sum dy
//
// Bound by HBM: a row is read once into registers, where all passes over it are made (so the squares are those of the differences from the mean), and
// written once.  8 neighbouring values per lane and chunk (16 bytes).
#include "common.h"

namespace moe {

// Sum over the 64 lanes, for all of them: inside the rows of 16 lanes, then from the last lane of a row (of the first half) to the rows (the half)
// after it; lane 63 has it in the end.
__device__ __forceinline__ float wave_add(float v) {
#define MOE_ADD_STEP(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xF, false))
  MOE_ADD_STEP(0x111, 0xF); MOE_ADD_STEP(0x112, 0xF); MOE_ADD_STEP(0x114, 0xF); MOE_ADD_STEP(0x118, 0xF);   // row_shr:1, 2, 4, 8
  MOE_ADD_STEP(0x142, 0xA);   // row_bcast:15 into rows 1 and 3
  MOE_ADD_STEP(0x143, 0xC);   // row_bcast:31 into rows 2 and 3
#undef MOE_ADD_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

// Sums over the WAVES wavefronts of a row; `slot`: their LDS, used once between two barriers.
template <int WAVES>
__device__ __forceinline__ float row_add(float v, float* slot, int wave) {
  v = wave_add(v);
  if constexpr (WAVES == 1) return v;
  if (threadIdx.x % kWave == 0) slot[wave] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int i = 0; i < WAVES; i++) v += slot[i];
  return v;
}

__device__ __forceinline__ void unpack8(const uint4& r, float* v) {
  v[0] = bf16lo(r.x); v[1] = bf16hi(r.x); v[2] = bf16lo(r.y); v[3] = bf16hi(r.y);
  v[4] = bf16lo(r.z); v[5] = bf16hi(r.z); v[6] = bf16lo(r.w); v[7] = bf16hi(r.w);
}
__device__ __forceinline__ uint4 pack8(const float* v) {
  return uint4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}

struct NormFwdArgs {
  long long rows;
  int cols;
  float eps, inv_cols;
  const uint16_t* x; const uint16_t* addend; const uint16_t* gamma; const uint16_t* beta;
  uint16_t* sum; uint16_t* y; float* mean; float* rstd;
};

// A row for WAVES wavefronts, CH chunks of 8 values a lane; blocks of 4 wavefronts at least.
template <int WAVES, int CH, bool CENTRE>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * kWave) void norm_fwd_kernel(NormFwdArgs A) {
  constexpr int THREADS = WAVES * kWave, ROWS = WAVES < 4 ? 4 / WAVES : 1;
  __shared__ float slots[ROWS][2][WAVES];
  const int tid = threadIdx.x % THREADS, in_block = threadIdx.x / THREADS, wave = tid / kWave;
  long long row = (long long)blockIdx.x * ROWS + in_block;
  const bool live = row < A.rows;   // (the others take part in the barriers)
  if (!live) row = A.rows - 1;
  const size_t base = (size_t)row * A.cols;
  uint4 raw[CH];
  float total = 0.f;
#pragma unroll
  for (int c = 0; c < CH; c++) {
    const int col = 8 * (tid + c * THREADS);
    raw[c] = uint4{0, 0, 0, 0};
    if (col < A.cols) raw[c] = *reinterpret_cast<const uint4*>(A.x + base + col);
  }
  if (A.addend) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int col = 8 * (tid + c * THREADS);
      if (col < A.cols) {
        float v[8], a[8];
        unpack8(raw[c], v);
        unpack8(*reinterpret_cast<const uint4*>(A.addend + base + col), a);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += a[i];
        raw[c] = pack8(v);
      }
    }
  }
  if (CENTRE) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      float v[8];
      unpack8(raw[c], v);
#pragma unroll
      for (int i = 0; i < 8; i++) total += v[i];
    }
    total = row_add<WAVES>(total, slots[in_block][0], wave) * A.inv_cols;
  }
  float squares = 0.f;
#pragma unroll
  for (int c = 0; c < CH; c++) {
    if (8 * (tid + c * THREADS) < A.cols) {
      float v[8];
      unpack8(raw[c], v);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float d = v[i] - total;
        squares = fmaf(d, d, squares);
      }
    }
  }
  squares = row_add<WAVES>(squares, slots[in_block][1], wave);
  if (!live) return;
  const float rstd = 1.0f / sqrtf(fmaf(squares, A.inv_cols, A.eps));
  if (tid == 0) {
    if (CENTRE && A.mean) A.mean[row] = total;
    if (A.rstd) A.rstd[row] = rstd;
  }
#pragma unroll
  for (int c = 0; c < CH; c++) {
    const int col = 8 * (tid + c * THREADS);
    if (col < A.cols) {
      if (A.sum) *reinterpret_cast<uint4*>(A.sum + base + col) = raw[c];
      float v[8], f[8];
      unpack8(raw[c], v);
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = (v[i] - total) * rstd;
      if (A.gamma) {
        unpack8(*reinterpret_cast<const uint4*>(A.gamma + col), f);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] *= f[i];
      }
      if (A.beta) {
        unpack8(*reinterpret_cast<const uint4*>(A.beta + col), f);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += f[i];
      }
      *reinterpret_cast<uint4*>(A.y + base + col) = pack8(v);
    }
  }
}

struct NormBwdArgs {
  long long rows;
  int cols;
  float inv_cols;
  const uint16_t* dy; const uint16_t* h; const uint16_t* gamma; const float* mean; const float* rstd; const uint16_t* dx_addend;
  uint16_t* dx;
  float* part;   // [blocks][2][cols]: a block's sums of dy xh and of dy; null: not wanted
};

// Rows in turn for WAVES wavefronts each; a lane keeps the sums of its columns.
template <int WAVES, int CH, bool CENTRE>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * kWave) void norm_bwd_kernel(NormBwdArgs A) {
  constexpr int THREADS = WAVES * kWave, ROWS = WAVES < 4 ? 4 / WAVES : 1;
  __shared__ float slots[2][ROWS][2][WAVES];
  __shared__ float join[ROWS > 1 ? (ROWS - 1) * THREADS * 8 : 1];
  const int tid = threadIdx.x % THREADS, in_block = threadIdx.x / THREADS, wave = tid / kWave;
  float dgamma[8 * CH], dbeta[8 * CH];
#pragma unroll
  for (int i = 0; i < 8 * CH; i++) dgamma[i] = dbeta[i] = 0.f;
  const long long step = (long long)gridDim.x * ROWS;
  int turn = 0;
  for (long long first = (long long)blockIdx.x * ROWS; first < A.rows; first += step, turn ^= 1) {
    const long long row = first + in_block;
    const bool live = row < A.rows;
    const size_t base = (size_t)(live ? row : 0) * A.cols;
    const float mean = live && CENTRE ? A.mean[row] : 0.f, rstd = live ? A.rstd[row] : 0.f;
    uint4 rdy[CH], rh[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int col = 8 * (tid + c * THREADS);
      rdy[c] = rh[c] = uint4{0, 0, 0, 0};
      if (live && col < A.cols) {
        rdy[c] = *reinterpret_cast<const uint4*>(A.dy + base + col);
        rh[c] = *reinterpret_cast<const uint4*>(A.h + base + col);
      }
    }
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int col = 8 * (tid + c * THREADS);
      if (live && col < A.cols) {
        float d[8], v[8], f[8];
        unpack8(rdy[c], d);
        unpack8(rh[c], v);
        if (A.gamma) unpack8(*reinterpret_cast<const uint4*>(A.gamma + col), f);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float xh = (v[i] - mean) * rstd, g = A.gamma ? d[i] * f[i] : d[i];
          dgamma[8 * c + i] = fmaf(d[i], xh, dgamma[8 * c + i]);
          dbeta[8 * c + i] += d[i];
          sg += g;
          sgx = fmaf(g, xh, sgx);
        }
      }
    }
    if (CENTRE) sg = wave_add(sg);
    sgx = wave_add(sgx);
    if constexpr (WAVES > 1) {   // (two sets of slots in turn: one barrier a row)
      if (threadIdx.x % kWave == 0) { slots[turn][in_block][0][wave] = sg; slots[turn][in_block][1][wave] = sgx; }
      __syncthreads();
      sg = sgx = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; i++) { sg += slots[turn][in_block][0][i]; sgx += slots[turn][in_block][1][i]; }
    }
    sg = CENTRE ? sg * A.inv_cols : 0.f;
    sgx *= A.inv_cols;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int col = 8 * (tid + c * THREADS);
      if (live && col < A.cols) {
        float d[8], v[8], f[8];
        unpack8(rdy[c], d);
        unpack8(rh[c], v);
        if (A.gamma) unpack8(*reinterpret_cast<const uint4*>(A.gamma + col), f);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float xh = (v[i] - mean) * rstd, g = A.gamma ? d[i] * f[i] : d[i];
          d[i] = rstd * (g - sg - xh * sgx);
        }
        if (A.dx_addend) {
          unpack8(*reinterpret_cast<const uint4*>(A.dx_addend + base + col), f);
#pragma unroll
          for (int i = 0; i < 8; i++) d[i] += f[i];
        }
        *reinterpret_cast<uint4*>(A.dx + base + col) = pack8(d);
      }
    }
  }
  if (A.part == nullptr) return;
  float* part = A.part + (size_t)blockIdx.x * 2 * A.cols;
#pragma unroll
  for (int which = 0; which < 2; which++) {
    float* sums = which ? dbeta : dgamma;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      if constexpr (ROWS > 1) {   // the block's other rows, in order
        __syncthreads();
        if (in_block > 0)
#pragma unroll
          for (int i = 0; i < 8; i++) join[((in_block - 1) * 8 + i) * THREADS + tid] = sums[8 * c + i];
        __syncthreads();
        if (in_block == 0)
#pragma unroll
          for (int o = 0; o < ROWS - 1; o++)
#pragma unroll
            for (int i = 0; i < 8; i++) sums[8 * c + i] += join[(o * 8 + i) * THREADS + tid];
      }
      const int col = 8 * (tid + c * THREADS);
      if (in_block == 0 && col < A.cols) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          *reinterpret_cast<float4*>(part + (size_t)which * A.cols + col + i) = float4{sums[8 * c + i], sums[8 * c + i + 1], sums[8 * c + i + 2], sums[8 * c + i + 3]};
      }
    }
  }
}

// dgamma and dbeta from the blocks' sums: 64 columns a block, 16 wavefronts that take every 16th part, joined in order.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* __restrict__ part, int parts, int cols, float* __restrict__ dgamma,
                                                            float* __restrict__ dbeta, int accumulate) {
  __shared__ float join[16][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = blockIdx.x * kWave + lane;
  float* out = blockIdx.y ? dbeta : dgamma;
  if (out == nullptr) return;   // (whole blocks)
  float v = 0.f;
  if (col < cols)
    for (int p = wave; p < parts; p += 16) v += part[((size_t)p * 2 + blockIdx.y) * cols + col];
  join[wave][lane] = v;
  __syncthreads();
  if (wave != 0 || col >= cols) return;
  v = accumulate ? out[col] : 0.f;
#pragma unroll
  for (int i = 0; i < 16; i++) v += join[i][lane];
  out[col] = v;
}

static bool norm_sizes(long long rows, int cols) { return rows >= 0 && rows < (1ll << 31) && cols >= 8 && cols <= MOE_NORM_COLS_MAX && cols % 8 == 0; }
static int norm_rows_per_block(int cols) { return cols <= 512 ? 4 : cols <= 2048 ? 1 : 1; }
static int norm_bwd_blocks(long long rows, int cols) {
  const long long units = (rows + norm_rows_per_block(cols) - 1) / norm_rows_per_block(cols);
  return (int)(units < 1024 ? units : 1024);
}

}  // namespace moe

extern "C" int moe_norm_fwd(int64_t rows, int cols, int centre, float eps, const uint16_t* x, const uint16_t* addend, const uint16_t* gamma,
                            const uint16_t* beta, uint16_t* sum, uint16_t* y, float* mean, float* rstd, void* stream) {
  using namespace moe;
  if (!norm_sizes(rows, cols) || !(eps > 0.f) || eps > 3.402823466e38f) return MOE_ERR_SHAPE;
  if (rows == 0) return MOE_OK;   // (tensors without elements may be NULL)
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(y);
  MOE_REQUIRE_ALIGNED(x); MOE_REQUIRE_ALIGNED(addend); MOE_REQUIRE_ALIGNED(gamma); MOE_REQUIRE_ALIGNED(beta); MOE_REQUIRE_ALIGNED(sum);
  MOE_REQUIRE_ALIGNED(y); MOE_REQUIRE_ALIGNED(mean); MOE_REQUIRE_ALIGNED(rstd);
  hipStream_t st = (hipStream_t)stream;
  const NormFwdArgs A = {rows, cols, eps, 1.0f / cols, x, addend, gamma, beta, sum, y, mean, rstd};
#define MOE_LAUNCH_NORM(W_, CH_)                                                                                              \
  do {                                                                                                                        \
    const dim3 grid((unsigned)((rows + (W_ < 4 ? 4 / W_ : 1) - 1) / (W_ < 4 ? 4 / W_ : 1))), block(W_ < 4 ? 256 : W_ * kWave); \
    if (centre) MOE_LAUNCH("norm_fwd", st, (norm_fwd_kernel<W_, CH_, true>), grid, block, 0, st, A);                          \
    else MOE_LAUNCH("norm_fwd", st, (norm_fwd_kernel<W_, CH_, false>), grid, block, 0, st, A);                                \
  } while (0)
  if (cols <= 512) MOE_LAUNCH_NORM(1, 1);
  else if (cols <= 2048) MOE_LAUNCH_NORM(4, 1);
  else if (cols <= 4096) MOE_LAUNCH_NORM(4, 2);
  else if (cols <= 8192) MOE_LAUNCH_NORM(4, 4);
  else MOE_LAUNCH_NORM(8, 4);
#undef MOE_LAUNCH_NORM
  return launch_status();
}

extern "C" size_t moe_norm_workspace_bytes(int64_t rows, int cols) {
  using namespace moe;
  if (!norm_sizes(rows, cols)) return 0;
  return round_up((size_t)norm_bwd_blocks(rows, cols) * 2 * cols * sizeof(float) + 256, 256);
}

extern "C" int moe_norm_bwd(int64_t rows, int cols, int centre, const uint16_t* dy, const uint16_t* h, const uint16_t* gamma, const float* mean,
                            const float* rstd, const uint16_t* dx_addend, uint16_t* dx, float* dgamma, float* dbeta, int accumulate, void* ws,
                            size_t ws_bytes, void* stream) {
  using namespace moe;
  if (!norm_sizes(rows, cols)) return MOE_ERR_SHAPE;
  if (rows > 0) {   // (tensors without elements may be NULL)
    MOE_REQUIRE_PTR(dy); MOE_REQUIRE_PTR(h); MOE_REQUIRE_PTR(rstd); MOE_REQUIRE_PTR(dx);
    if (centre) MOE_REQUIRE_PTR(mean);
  }
  MOE_REQUIRE_ALIGNED(dy); MOE_REQUIRE_ALIGNED(h); MOE_REQUIRE_ALIGNED(gamma); MOE_REQUIRE_ALIGNED(mean); MOE_REQUIRE_ALIGNED(rstd);
  MOE_REQUIRE_ALIGNED(dx_addend); MOE_REQUIRE_ALIGNED(dx); MOE_REQUIRE_ALIGNED(dgamma); MOE_REQUIRE_ALIGNED(dbeta);
  const bool weights = dgamma != nullptr || dbeta != nullptr;
  if (weights) {
    MOE_REQUIRE_PTR(ws);
    if (!aligned(ws, 256)) return MOE_ERR_ALIGN;
    if (ws_bytes < moe_norm_workspace_bytes(rows, cols)) return MOE_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  const int blocks = norm_bwd_blocks(rows, cols);
  float* part = weights ? (float*)ws : nullptr;
  if (rows > 0) {
    const NormBwdArgs A = {rows, cols, 1.0f / cols, dy, h, gamma, mean, rstd, dx_addend, dx, part};
#define MOE_LAUNCH_NORM(W_, CH_)                                                                                                           \
  do {                                                                                                                                     \
    if (centre) MOE_LAUNCH("norm_bwd", st, (norm_bwd_kernel<W_, CH_, true>), dim3(blocks), dim3(W_ < 4 ? 256 : W_ * kWave), 0, st, A);     \
    else MOE_LAUNCH("norm_bwd", st, (norm_bwd_kernel<W_, CH_, false>), dim3(blocks), dim3(W_ < 4 ? 256 : W_ * kWave), 0, st, A);           \
  } while (0)
    if (cols <= 512) MOE_LAUNCH_NORM(1, 1);
    else if (cols <= 2048) MOE_LAUNCH_NORM(4, 1);
    else if (cols <= 4096) MOE_LAUNCH_NORM(4, 2);
    else if (cols <= 8192) MOE_LAUNCH_NORM(4, 4);
    else MOE_LAUNCH_NORM(8, 4);
#undef MOE_LAUNCH_NORM
  }
  if (weights)
    MOE_LAUNCH("norm_weights", st, norm_weights_kernel, dim3((cols + kWave - 1) / kWave, dbeta ? 2 : 1), dim3(1024), 0, st, part, blocks, cols, dgamma, dbeta,
               accumulate);
  return launch_status();
}
