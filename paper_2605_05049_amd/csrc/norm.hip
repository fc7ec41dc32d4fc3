// The norm in front of a layer, with the residual sum in front of it, and its gradients.
//
//   h = x + addend,  y = (h - mean) rstd gamma + beta,  rstd = 1 / sqrt(mean((h - mean)^2) + eps)   (RMS norm: mean taken as 0)
//   dx = rstd (g - mean(g) - xh mean(g xh)) + dx_addend,  g = dy gamma,  xh = (h - mean) rstd;   dgamma = sum dy xh,  dbeta = sum dy
//
// Bound by HBM: a row is read once into registers, where all passes over it are made (so the squares are those of the differences from the mean), and
// written once.  8 neighbouring values per lane and chunk (16 bytes).  Rates: 16384 x 4096, RMS norm with the residual sum, 537 MB: 92 us, 5.9 TB/s;
// gradients of 32768 x 7168 with an addend and dgamma, 1.88 GB: 335 us, 5.6 TB/s (a pass over the rows and one over the columns took 527);
// 4099 x 2056, 51 MB: 13.1 us and 3.7 for the blocks' sums.  Few rows are a launch: 1 x 4096 2.0 us, gradients of 256 x 512 3.3.
#include "lanes.h"

namespace moe {

// Sums over the THREADS lanes of a row (16, 32, 64 or several wavefronts); `slot`: LDS of a float a wavefront, used once between two barriers.
template <int THREADS>
__device__ __forceinline__ float row_add(float v, float* slot, int wave) {
  v = lanes_sum<(THREADS < kWave ? THREADS : kWave)>(v);
  if constexpr (THREADS <= kWave) return v;
  if (threadIdx.x % kWave == 0) slot[wave] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int i = 0; i < THREADS / kWave; i++) v += slot[i];
  return v;
}
// The value of the first lane for a whole wavefront (which row it works on) where a row has a wavefront and more.
template <int THREADS>
__device__ __forceinline__ int of_row(int v) {
  if constexpr (THREADS >= kWave) return __builtin_amdgcn_readfirstlane(v);
  else return v;
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

// A row for THREADS lanes, CH chunks of 8 values a lane; blocks of 4 wavefronts at least.
template <int THREADS, int CH, bool CENTRE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_fwd_kernel(NormFwdArgs A) {
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float slots[ROWS][2][THREADS < kWave ? 1 : THREADS / kWave];
  const int tid = threadIdx.x % THREADS, in_block = of_row<THREADS>(threadIdx.x / THREADS), wave = of_row<THREADS>(tid / kWave);
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
    total = row_add<THREADS>(total, slots[in_block][0], wave) * A.inv_cols;
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
  squares = row_add<THREADS>(squares, slots[in_block][1], wave);
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
  float* part;          // [row_blocks][2][cols]: a block's sums of dy xh and of dy; null: not wanted, or made by blocks of their own
  int row_blocks;       // blocks behind them make dgamma and dbeta, kNormColumns columns each
  float* dgamma; float* dbeta;
  int accumulate;
};

// dgamma and dbeta of 32 columns from dy and h themselves: the wavefronts take rows in turn, their sums are joined in order.
constexpr int kNormColumns = 32;
template <int WAVES_IN_BLOCK, bool CENTRE>
__device__ __forceinline__ void weights_of_columns(const NormBwdArgs& A, int block, float* join) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int pair = lane % 16, quarter = lane / 16, col = block * kNormColumns + 2 * pair;   // two columns a lane, four rows a wavefront
  float g0 = 0.f, g1 = 0.f, b0 = 0.f, b1 = 0.f;
  if (col < A.cols) {
#pragma unroll 8
    for (long long row = 4 * wave + quarter; row < A.rows; row += 4 * WAVES_IN_BLOCK) {
      const uint32_t d = *reinterpret_cast<const uint32_t*>(A.dy + (size_t)row * A.cols + col);
      const uint32_t h = *reinterpret_cast<const uint32_t*>(A.h + (size_t)row * A.cols + col);
      const float mean = CENTRE ? A.mean[row] : 0.f, rstd = A.rstd[row];
      g0 = fmaf(bf16lo(d), (bf16lo(h) - mean) * rstd, g0);
      g1 = fmaf(bf16hi(d), (bf16hi(h) - mean) * rstd, g1);
      b0 += bf16lo(d);
      b1 += bf16hi(d);
    }
  }
  float* mine = join + (size_t)(4 * wave + quarter) * 4 * 16 + pair;   // [row group][4][16]
  mine[0] = g0; mine[16] = g1; mine[32] = b0; mine[48] = b1;
  __syncthreads();
  const int which = threadIdx.x / kNormColumns, c = threadIdx.x % kNormColumns;   // dgamma, dbeta
  float* out = which == 0 ? A.dgamma : which == 1 ? A.dbeta : nullptr;
  if (out == nullptr || block * kNormColumns + c >= A.cols) return;
  float v = A.accumulate ? out[block * kNormColumns + c] : 0.f;
  for (int i = 0; i < 4 * WAVES_IN_BLOCK; i++) v += join[(size_t)i * 4 * 16 + (2 * which + c % 2) * 16 + c / 2];
  out[block * kNormColumns + c] = v;
}

// Rows in turn for THREADS lanes each; a lane keeps gamma and the sums of its columns, and requests the next row before it computes this one.
template <int THREADS, int CH, bool CENTRE, bool BETA>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_bwd_kernel(NormBwdArgs A) {
  constexpr int BLOCK_WAVES = THREADS < 256 ? 4 : THREADS / kWave, WAVES = THREADS < kWave ? 1 : THREADS / kWave, ROWS = BLOCK_WAVES * kWave / THREADS;
  constexpr bool AHEAD = CH <= 2;   // (registers; of 3 and 4 chunks up to 6 % slower)
  constexpr int JOIN = (ROWS - 1) * THREADS * 8, COLUMNS = 4 * BLOCK_WAVES * 4 * 16;
  __shared__ float slots[2][ROWS][2][WAVES];
  __shared__ float join[JOIN > COLUMNS ? JOIN : COLUMNS];
  if ((int)blockIdx.x >= A.row_blocks) {
    weights_of_columns<BLOCK_WAVES, CENTRE>(A, blockIdx.x - A.row_blocks, join);
    return;
  }
  const int tid = threadIdx.x % THREADS, in_block = of_row<THREADS>(threadIdx.x / THREADS), wave = of_row<THREADS>(tid / kWave);
  const bool sums = A.part != nullptr;
  float dgamma[8 * CH], dbeta[BETA ? 8 * CH : 1];
#pragma unroll
  for (int i = 0; i < 8 * CH; i++) dgamma[i] = 0.f;
#pragma unroll
  for (int i = 0; i < (BETA ? 8 * CH : 1); i++) dbeta[i] = 0.f;
  // (columns behind the last are read as the last ones and count as zeros: dy and gamma of them are 0)
  uint4 gamma[CH];
  bool in[CH];
  unsigned bytes_at[CH];
#pragma unroll
  for (int c = 0; c < CH; c++) {
    const int col = 8 * (tid + c * THREADS);
    in[c] = col < A.cols;
    bytes_at[c] = 2u * (unsigned)(in[c] ? col : A.cols - 8);
    gamma[c] = uint4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    if (A.gamma) gamma[c] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(A.gamma) + bytes_at[c]);
  }
  struct Row { uint4 dy[CH], h[CH], addend[CH]; float mean, rstd; };
  auto request = [&](long long row, Row& r) __attribute__((always_inline)) {
    const long long at = row < A.rows ? row : A.rows - 1;
    const char* dy = reinterpret_cast<const char*>(A.dy + (size_t)at * A.cols);   // (of the wavefront; a lane's offset has 32 bits)
    const char* h = reinterpret_cast<const char*>(A.h + (size_t)at * A.cols);
#pragma unroll
    for (int c = 0; c < CH; c++) {
      r.dy[c] = *reinterpret_cast<const uint4*>(dy + bytes_at[c]);
      r.h[c] = *reinterpret_cast<const uint4*>(h + bytes_at[c]);
    }
    if (A.dx_addend) {
      const char* addend = reinterpret_cast<const char*>(A.dx_addend + (size_t)at * A.cols);
#pragma unroll
      for (int c = 0; c < CH; c++) r.addend[c] = *reinterpret_cast<const uint4*>(addend + bytes_at[c]);
    }
    r.mean = CENTRE ? A.mean[at] : 0.f;
    r.rstd = A.rstd[at];
  };
  const long long step = (long long)A.row_blocks * ROWS;
  int turn = 0;
  Row cur, next;
  if constexpr (AHEAD) request((long long)blockIdx.x * ROWS + in_block, cur);
  for (long long first = (long long)blockIdx.x * ROWS; first < A.rows; first += step, turn ^= 1) {
    const long long row = first + in_block;
    const bool live = row < A.rows;
    if constexpr (AHEAD) {
      if (first + step < A.rows) request(row + step, next);
    } else {
      request(row, cur);
    }
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      if (!in[c] || !live) cur.dy[c] = uint4{0, 0, 0, 0};
      if (ROWS > 1 && !live) cur.h[c] = uint4{0, 0, 0, 0};   // (the last row's, which dx may have overwritten)
      float d[8], v[8], f[8];
      unpack8(cur.dy[c], d);
      unpack8(cur.h[c], v);
      unpack8(gamma[c], f);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float xh = (v[i] - cur.mean) * cur.rstd, g = d[i] * f[i];
        dgamma[8 * c + i] = fmaf(d[i], xh, dgamma[8 * c + i]);
        if (BETA) dbeta[8 * c + i] += d[i];
        if (CENTRE) sg += g;
        sgx = fmaf(g, xh, sgx);
      }
    }
    if (CENTRE) sg = lanes_sum<(THREADS < kWave ? THREADS : kWave)>(sg);
    sgx = lanes_sum<(THREADS < kWave ? THREADS : kWave)>(sgx);
    if constexpr (WAVES > 1) {   // (two sets of slots in turn: one barrier a row)
      if (threadIdx.x % kWave == 0) { slots[turn][in_block][0][wave] = sg; slots[turn][in_block][1][wave] = sgx; }
      __syncthreads();
      sg = sgx = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; i++) { sg += slots[turn][in_block][0][i]; sgx += slots[turn][in_block][1][i]; }
    }
    // dx = rstd (d gamma - (sg - mean rstd sgx) - h rstd sgx), kept as differences from the mean
    sg = CENTRE ? sg * A.inv_cols : 0.f;
    sgx *= A.inv_cols;
    char* dx = reinterpret_cast<char*>(A.dx + (size_t)(live ? row : 0) * A.cols);
#pragma unroll
    for (int c = 0; c < CH; c++) {
      float d[8], v[8], f[8];
      unpack8(cur.dy[c], d);
      unpack8(cur.h[c], v);
      unpack8(gamma[c], f);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float xh = (v[i] - cur.mean) * cur.rstd;
        d[i] = cur.rstd * (fmaf(d[i], f[i], -sg) - xh * sgx);
      }
      if (A.dx_addend) {
        unpack8(cur.addend[c], f);
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] += f[i];
      }
      if (in[c] && live) *reinterpret_cast<uint4*>(dx + bytes_at[c]) = pack8(d);
    }
    if constexpr (AHEAD) cur = next;
  }
  if (!sums) return;
  float* part = A.part + (size_t)blockIdx.x * 2 * A.cols;
#pragma unroll
  for (int which = 0; which < (BETA ? 2 : 1); which++) {
    float* of = which ? dbeta : dgamma;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      if constexpr (ROWS > 1) {   // the block's other rows, in order
        __syncthreads();
        if (in_block > 0)
#pragma unroll
          for (int i = 0; i < 8; i++) join[((in_block - 1) * 8 + i) * THREADS + tid] = of[8 * c + i];
        __syncthreads();
        if (in_block == 0)
#pragma unroll
          for (int o = 0; o < ROWS - 1; o++)
#pragma unroll
            for (int i = 0; i < 8; i++) of[8 * c + i] += join[(o * 8 + i) * THREADS + tid];
      }
      if (in_block == 0 && in[c]) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          *reinterpret_cast<float4*>(part + (size_t)which * A.cols + bytes_at[c] / 2 + i) = float4{of[8 * c + i], of[8 * c + i + 1], of[8 * c + i + 2], of[8 * c + i + 3]};
      }
    }
  }
}

// dgamma and dbeta from the blocks' sums: 32 columns a block, 32 groups that take every 32nd part, joined in order.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* __restrict__ part, int parts, int cols, float* __restrict__ dgamma,
                                                            float* __restrict__ dbeta, int accumulate) {
  __shared__ float join[32][33];
  const int c = threadIdx.x % 32, group = threadIdx.x / 32, col = blockIdx.x * 32 + c;
  float* out = blockIdx.y ? dbeta : dgamma;
  if (out == nullptr) return;   // (whole blocks)
  float v = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int p = group; p < parts; p += 32) v += part[((size_t)p * 2 + blockIdx.y) * cols + col];
  }
  join[group][c] = v;
  __syncthreads();
  if (group != 0 || col >= cols) return;
  v = accumulate ? out[col] : 0.f;
#pragma unroll
  for (int i = 0; i < 32; i++) v += join[i][c];
  out[col] = v;
}

constexpr long long kNormRows = 1 << 22;   // of a launch of the forward pass at most: a grid has less than 2^32 threads
static bool norm_sizes(long long rows, int cols) { return rows >= 0 && rows < (1ll << 31) && cols >= 8 && cols <= MOE_NORM_COLS_MAX && cols % 8 == 0; }
// 64 to 512 lanes, as few as have at most `chunks` chunks of 8 columns each.
static int norm_lanes_of_chunks(int cols, int chunks) {
  int lanes = 64;
  while (lanes < 512 && cols > 8 * chunks * lanes) lanes *= 2;
  return lanes;
}
// Lanes of a row in the forward pass: up to 3 chunks of 8 values a lane; with the residual sum, whose loads wait in registers, one or two.
// (67 million values, 512 .. 16384 columns: 5.8 to 6.3 TB/s, with the sum 5.1 to 6.0; half as many lanes with the sum 3 to 8 % slower, twice as many
// without it 1 to 40 %.)
static int norm_fwd_lanes(int cols, bool addend) {
  if (cols <= 128) return 16;
  if (cols <= 256) return 32;
  if (addend) return cols <= 512 ? 128 : cols <= 2048 ? 256 : 512;
  return norm_lanes_of_chunks(cols, 3);
}
// In the backward pass: as few as leave a lane at most 3 chunks of 8 values (4 from 12288 columns on), whose sums it keeps.  Blocks: two a CU of 4
// wavefronts, one of 8.  (Twice and half as many blocks, lanes: 2 to 40 % slower at 512 .. 16384 columns; 2 blocks of 8 are 6 % slower. Numbers that
// even out the blocks' rows but not those of the CUs: 10 to 60 %.)
static int norm_bwd_lanes(int cols) { return cols <= 128 ? 16 : cols <= 256 ? 32 : norm_lanes_of_chunks(cols, 3); }
static int norm_bwd_blocks(long long rows, int cols) {
  const int lanes = norm_bwd_lanes(cols), per_block = lanes < 256 ? 256 / lanes : 1;
  const long long units = (rows + per_block - 1) / per_block;
  const int most = lanes < 512 && units >= 2048 ? 512 : 256;   // (half as many for shorter batches: a block's sums are read again.  2048 x 1024 9.5 -> 8.5 us)
  return (int)(units < most ? units : most);
}
// dgamma and dbeta by blocks of their own in the launch of dx: they read dy and h again, but there is one launch, and no sums on the way.  Of one launch
// and two, us: 256 x 512 3.2, 5.7; 1024 x 1024 5.5, 7.4; 139 x 11464 6.9, 18.7; 1024 x 4096 12.2, 14.4; 2048 x 1024 12.0, 8.5; 4096 x 4096 40, 30.
static bool norm_bwd_one_launch(long long rows) { return rows <= 1024; }

}  // namespace moe

// The launch of a row's lanes for their number of chunks, of which FIRST_ to 3 occur, of 512 lanes also 4.  (A form that no size reaches is not made.)
#define MOE_LAUNCH_NORM_CHUNKS(L_, FIRST_)             \
  do {                                                 \
    const int chunks = (cols + 8 * L_ - 1) / (8 * L_); \
    if (chunks <= FIRST_) MOE_LAUNCH_NORM(L_, FIRST_); \
    else if (chunks == 2) MOE_LAUNCH_NORM(L_, 2);      \
    else if (chunks == 3) MOE_LAUNCH_NORM(L_, 3);      \
    else MOE_LAUNCH_NORM(L_, (L_ < 512 ? 3 : 4));      \
  } while (0)
#define MOE_LAUNCH_NORM_LANES(lanes, FIRST_)                    \
  do {                                                          \
    if (lanes == 16) MOE_LAUNCH_NORM(16, 1);                    \
    else if (lanes == 32) MOE_LAUNCH_NORM(32, 1);               \
    else if (lanes == 64) MOE_LAUNCH_NORM_CHUNKS(64, 1);        \
    else if (lanes == 128) MOE_LAUNCH_NORM_CHUNKS(128, FIRST_); \
    else if (lanes == 256) MOE_LAUNCH_NORM_CHUNKS(256, FIRST_); \
    else MOE_LAUNCH_NORM_CHUNKS(512, FIRST_);                   \
  } while (0)

extern "C" int moe_norm_fwd(int64_t rows, int cols, int centre, float eps, const uint16_t* x, const uint16_t* addend, const uint16_t* gamma,
                            const uint16_t* beta, uint16_t* sum, uint16_t* y, float* mean, float* rstd, void* stream) {
  using namespace moe;
  if (!norm_sizes(rows, cols) || !(eps > 0.f) || eps > 3.402823466e38f) return MOE_ERR_SHAPE;
  if (rows == 0) return MOE_OK;   // (tensors without elements may be NULL)
  MOE_REQUIRE_PTR(x); MOE_REQUIRE_PTR(y);
  MOE_REQUIRE_ALIGNED(x); MOE_REQUIRE_ALIGNED(addend); MOE_REQUIRE_ALIGNED(gamma); MOE_REQUIRE_ALIGNED(beta); MOE_REQUIRE_ALIGNED(sum);
  MOE_REQUIRE_ALIGNED(y); MOE_REQUIRE_ALIGNED(mean); MOE_REQUIRE_ALIGNED(rstd);
  hipStream_t st = (hipStream_t)stream;
#define MOE_LAUNCH_NORM(L_, CH_)                                                                     \
  do {                                                                                               \
    constexpr int per_block = L_ < 256 ? 256 / L_ : 1;                                               \
    const dim3 grid((unsigned)((rows + per_block - 1) / per_block)), block(L_ < 256 ? 256 : L_);     \
    if (centre) MOE_LAUNCH("norm_fwd", st, (norm_fwd_kernel<L_, CH_, true>), grid, block, 0, st, A); \
    else MOE_LAUNCH("norm_fwd", st, (norm_fwd_kernel<L_, CH_, false>), grid, block, 0, st, A);       \
  } while (0)
  const int lanes = norm_fwd_lanes(cols, addend != nullptr);
  const int64_t all = rows;
  for (int64_t done = 0; done < all; done += kNormRows) {
    rows = all - done < kNormRows ? all - done : kNormRows;
    const size_t at = (size_t)done * cols;
    const NormFwdArgs A = {rows, cols, eps, 1.0f / cols, x + at, addend ? addend + at : nullptr, gamma, beta, sum ? sum + at : nullptr, y + at,
                           mean ? mean + done : nullptr, rstd ? rstd + done : nullptr};
    MOE_LAUNCH_NORM_LANES(lanes, 1);
  }
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
  const bool one = rows > 0 && norm_bwd_one_launch(rows) && dx != dy && dx != h;   // (both are still read when dx is written)
  if (rows > 0) {
    const NormBwdArgs A = {rows, cols, 1.0f / cols, dy, h, gamma, mean, rstd, dx_addend, dx, one ? nullptr : part, blocks, dgamma, dbeta, accumulate};
    const dim3 grid(blocks + (one && weights ? (cols + kNormColumns - 1) / kNormColumns : 0));
#define MOE_LAUNCH_NORM_BETA(L_, CH_, C_, B_) \
  MOE_LAUNCH("norm_bwd", st, (norm_bwd_kernel<L_, CH_, C_, B_>), grid, dim3(L_ < 256 ? 256 : L_), 0, st, A)
#define MOE_LAUNCH_NORM(L_, CH_)                                    \
  do {                                                              \
    if (centre && dbeta) MOE_LAUNCH_NORM_BETA(L_, CH_, true, true); \
    else if (centre) MOE_LAUNCH_NORM_BETA(L_, CH_, true, false);    \
    else if (dbeta) MOE_LAUNCH_NORM_BETA(L_, CH_, false, true);     \
    else MOE_LAUNCH_NORM_BETA(L_, CH_, false, false);               \
  } while (0)
    const int lanes = norm_bwd_lanes(cols);
    MOE_LAUNCH_NORM_LANES(lanes, 2);
#undef MOE_LAUNCH_NORM
#undef MOE_LAUNCH_NORM_BETA
  }
  if (weights && !one)
    MOE_LAUNCH("norm_weights", st, norm_weights_kernel, dim3((cols + 31) / 32, dbeta ? 2 : 1), dim3(1024), 0, st, part, blocks, cols, dgamma, dbeta, accumulate);
  return launch_status();
}
