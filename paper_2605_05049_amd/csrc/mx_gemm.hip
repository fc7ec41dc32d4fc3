// Grouped products in microscaled 4-bit floating point (E2M1 values, a power-of-two scale per 32 along the contraction):
//     y[r, c] = sum_k x[r, k] w[e(r)][c, k]      and the SwiGLU pair  h = Q(silu(x W_gate) (x W_up)),
// on the block-scaled MFMA, which applies both scales and accumulates in fp32.  H is quantised from those sums (one rounding, to 4 bits).
//
// Operand layout of 16x16x128 (both operands alike): lane l holds row l % 16, k = 32 (l / 16) .. + 31, i.e. one block and its scale.  The weights are the A
// operand, so that a lane owns consecutive columns of a result row: with frag a's row m taken from column CPL (m / 4) + 4 a + m % 4 of the
// wavefront's columns (CPL = columns per lane), lane l ends up with columns CPL (l / 16) .. + CPL - 1 of row l % 16.
#include "mx_gemm.h"

#include <type_traits>
#include <utility>

namespace moe {

constexpr int MXR = 128;   // rows of a tile

// silu(g), for g < 0 within a relative (1.25 |g| + 6) 2^-24 (the exponential is 2^t of a rounded t = -g log2 e, by a rounded log2 e; a unit in the last place
// each for 2^t and the reciprocal, half of one for the sum and the product), for g >= 0 within 6 2^-24.  At g = -80 that is 2^-17: H keeps 4 bits, a block's
// values differ by a seventh and more, so a value's code is another one only if it lies that near to the middle between two.  Below -87, where the reciprocal is
// flushed, 0 for at most 2e-36 in magnitude.
// (A division is ten instructions, which nothing hides behind the last product of a tile: 8192 rows of 8 experts of 4096 x 14336, 907 -> 872 us in all.)
__device__ __forceinline__ float mx_silu(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// Small problems: 128 rows x 128 columns (of a pair 64 of either) per block of 4 wavefronts, each 64 x 64, the fragments from memory straight into
// registers; what it takes is the time of a few loads for each 128 k.  512 rows of 8 experts, 1024 columns, K = 512: 8.9 us.
template <int KIND>
__global__ __launch_bounds__(256) void mx_small_kernel(const MxGemmArgs A) {
  constexpr int NW = KIND == MX_GATE_UP ? 2 : 1;
  constexpr int WC = 64 / NW;          // columns of a wavefront, of either weight
  constexpr int FR = WC / 16;          // their frags
  constexpr int CPL = WC / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, q = lane >> 4;
  const int n_ct = (A.n + 2 * WC - 1) / (2 * WC);
  const int u = blockIdx.x / n_ct, ct = blockIdx.x % n_ct;
  MxSegment T;
  if (!mx_find_expert<MXR>(A.offsets, A.E, u, lane, T)) return;
  const int r0 = T.lo + (u - T.first) * MXR + (wave & 1) * 64, c0 = (ct * 2 + (wave >> 1)) * WC;
  if (r0 >= T.hi || c0 >= A.n) return;
  const int kb = A.k / kMxBlock;
  size_t xrow[4], wrow[FR];
#pragma unroll
  for (int b = 0; b < 4; b++) xrow[b] = (size_t)min(r0 + 16 * b + m, T.hi - 1) * kb;
#pragma unroll
  for (int a = 0; a < FR; a++) wrow[a] = ((size_t)T.expert * A.n + min(c0 + CPL * (m >> 2) + 4 * a + (m & 3), A.n - 1)) * kb;
  mx_f32x4 acc[NW][FR][4];
#pragma unroll
  for (int w = 0; w < NW; w++)
#pragma unroll
    for (int a = 0; a < FR; a++)
#pragma unroll
      for (int b = 0; b < 4; b++) acc[w][a][b] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
  auto frag = [&](const uint8_t* v, const uint8_t* s, size_t row, int block, mx_i32x8& f, int& scale) __attribute__((always_inline)) {
    uint4 d = make_uint4(0, 0, 0, 0);
    scale = 127;
    if (block < kb) {
      d = *reinterpret_cast<const uint4*>(v + (row + block) * 16);
      scale = s[row + block];
    }
    f = mx_i32x8{(int)d.x, (int)d.y, (int)d.z, (int)d.w, 0, 0, 0, 0};
  };
  for (int k0 = 0; k0 < kb; k0 += 4) {
    mx_i32x8 xf[4], wf[NW][FR];
    int xsc[4], wsc[NW][FR];
#pragma unroll
    for (int b = 0; b < 4; b++) frag(A.x, A.xs, xrow[b], k0 + q, xf[b], xsc[b]);
#pragma unroll
    for (int w = 0; w < NW; w++)
#pragma unroll
      for (int a = 0; a < FR; a++) frag(w ? A.w1 : A.w0, w ? A.ws1 : A.ws0, wrow[a], k0 + q, wf[w][a], wsc[w][a]);
#pragma unroll
    for (int w = 0; w < NW; w++)
#pragma unroll
      for (int a = 0; a < FR; a++)
#pragma unroll
        for (int b = 0; b < 4; b++)
          acc[w][a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[w][a], xf[b], acc[w][a][b], 4, 4, 0, wsc[w][a], 0, xsc[b]);
  }
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const int row = r0 + 16 * b + m;
    const int col = c0 + CPL * q;
    if (KIND == MX_PRODUCT) {
#pragma unroll
      for (int a = 0; a < FR; a += 2) {
        const mx_f32x4 lo = acc[0][a][b], hi = acc[0][a + 1][b];
        const float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (row < T.hi && col + 4 * a < A.n) *reinterpret_cast<uint4*>(A.y + (size_t)row * A.n + col + 4 * a) = pack8(f);
      }
    } else {
      // 32 columns of a row lie on the four lanes m, m + 16, m + 32, m + 48: one block
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float g = acc[0][i >> 2][b][i & 3], v = acc[NW - 1][i >> 2][b][i & 3];
        f[i] = mx_silu(g) * v;
      }
      unsigned e = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) e = max(e, (__float_as_uint(f[i]) >> 23) & 255u);
      e = max(e, (unsigned)__shfl_xor((int)e, 16));
      e = max(e, (unsigned)__shfl_xor((int)e, 32));
      const unsigned s = mx_scale_code(e);
      if (row < T.hi && col < A.n) {
        *reinterpret_cast<uint32_t*>(A.h + ((size_t)row * A.n + col) / 2) = mx_encode8(f, s);
        if (q == 0) A.hs[((size_t)row * A.n + col) / kMxBlock] = (uint8_t)s;
      }
    }
  }
}

// ---- large problems ----------------------------------------------------------------------------------------------------------------------
//
// 256 rows x 256 weight rows (of a pair 128 columns of W_gate and the same of W_up) per block of 4 wavefronts, one per SIMD, each 128 x 128: at
// 4 bits the matrix cores need an operand byte for every 64 multiplies, so what counts is how often a byte leaves LDS, and a wavefront's
// tile of 128 x 128 reads half of what four of 64 x 64 would.  Its 256 accumulators leave half of the registers for two sets of fragments: one
// is multiplied while the other is read.
//
// A stage is 256 k (128 bytes of a row), two of them in LDS; rows lie as in the bf16 kernels (chunk c of row r at c ^ ((r >> 1) & 7)), the
// weights' rows in the order in which the fragments take them.  The scales of a stage go through registers into LDS, turned so that one
// 8-byte read gives a lane the codes of all its fragments.  One barrier per stage, in its middle: what is read after it has landed
// before, and what has been read before it is overwritten after.
constexpr int MXT = 256;              // rows, and weight rows, of a tile
constexpr int MX_STAGE = MXT * 128;   // bytes of an operand's stage
constexpr int MX_XCDS = 8, MX_CHUNK = 32;   // consecutive tiles that go to one XCD
constexpr int MX_BAND = 8;            // row tiles walked side by side

template <int OW, int OX>
__device__ __forceinline__ mx_f32x4 mx_mfma(const int4& w, const int4& x, const mx_f32x4& acc, int ws, int xs) {
  const mx_i32x8 a = {w.x, w.y, w.z, w.w, 0, 0, 0, 0}, b = {x.x, x.y, x.z, x.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, OW, ws, OX, xs);
}
template <class F, int... I>
__device__ __forceinline__ void mx_each(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void mx_for(F&& f) { mx_each(static_cast<F&&>(f), std::make_integer_sequence<int, N>{}); }

// Frag a's row m of a wavefront's weight rows -> its column among the wavefront's 128 (64 of either of a pair): lane l's elements of frags 2 p
// and 2 p + 1 are 8 consecutive columns, 32 p + 8 (l / 16) .. + 7, and the four lanes of a row hold a block of 32.
__device__ __forceinline__ int mx_column(int a, int m) { return 32 * (a >> 1) + 8 * (m >> 2) + 4 * (a & 1) + (m & 3); }

// Block -> tile: chunks of consecutive tiles go to the XCDs in turn; an expert's tiles are walked in bands of row tiles, down the columns.
struct MxTile { int expert, r0, n_rows, c0; };
template <int COLS>
__device__ __forceinline__ bool mx_find_tile(const MxGemmArgs& A, int lane, MxTile& T) {
  const int n_ct = (A.n + COLS - 1) / COLS;
  const int within = blockIdx.x / MX_XCDS, xcd = blockIdx.x % MX_XCDS;
  const int lid = (within / MX_CHUNK * MX_XCDS + xcd) * MX_CHUNK + within % MX_CHUNK;
  MxSegment S;
  if (!mx_find_expert<MXT>(A.offsets, A.E, lid / n_ct, lane, S)) return false;
  const int e_tiles = (S.hi - S.lo + MXT - 1) / MXT;
  const int local = lid - S.first * n_ct, band = local / (MX_BAND * n_ct), in_band = local - band * MX_BAND * n_ct;
  const int b_rows = min(MX_BAND, e_tiles - band * MX_BAND);
  T.expert = S.expert;
  T.r0 = S.lo + (band * MX_BAND + in_band % b_rows) * MXT;
  T.n_rows = min(MXT, S.hi - T.r0);
  T.c0 = in_band / b_rows * COLS;
  return true;
}

template <int KIND>
__global__ __launch_bounds__(256, 1) void mx_tile_kernel(const MxGemmArgs A) {
  constexpr bool PAIR = KIND == MX_GATE_UP;
  constexpr int COLS = PAIR ? MXT / 2 : MXT;   // columns of the result per tile
  __shared__ __attribute__((aligned(1024))) char lds[2][2][MX_STAGE];   // [stage][x, w]
  __shared__ __attribute__((aligned(16))) char sc[2][2][8 * 256];      // scales: [stage][x, w][block][row group, m, frag]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int wr = wave & 1, wc = wave >> 1;

  MxTile T;
  if (!mx_find_tile<COLS>(A, lane, T)) return;
  const int r0 = T.r0, n_rows = T.n_rows, c0 = T.c0;
  const int kb = A.k / kMxBlock, nt = (kb + 7) / 8;

  auto run = [&](auto rb_c) __attribute__((always_inline)) {
    constexpr int RB = decltype(rb_c)::value;   // row frags of a wavefront: 32 RB rows in all
    constexpr int XI = RB;                      // direct loads of x per wavefront and stage (of 8 rows)
    // ---- addresses, from a base per tile and 32 bits.  Instruction i of wavefront w brings rows 8 (w XI + i) .. + 7 of x and LDS rows
    // 8 (8 w + i) .. + 7 of the weights, LDS row r being frag (r / 16) % 8, m = r % 16 of wavefront column r / 128; lane l row l / 8 of them, and
    // the chunk that belongs at position l % 8 (which depends on the parity of the instruction)
    const unsigned pitch = (unsigned)kb * 16;
    const uint8_t* const xb = A.x + (size_t)r0 * pitch;
    const size_t e_row0 = (size_t)T.expert * A.n + c0;
    const bool up = PAIR && (wave & 1);   // (wavefront w loads LDS rows 64 w .. 64 w + 63: of a pair either all gate or all up)
    const uint8_t* const wb = (up ? A.w1 : A.w0) + e_row0 * pitch;
    auto w_column = [&](int row) {   // LDS row -> column of the tile
      const int g = row >> 7, a = (row >> 4) & 7;
      return min(PAIR ? 64 * g + mx_column(a & 3, row & 15) : 128 * g + mx_column(a, row & 15), A.n - 1 - c0);
    };
    unsigned xo[XI], wo[8];
#pragma unroll
    for (int i = 0; i < XI; i++) xo[i] = (unsigned)min(8 * (wave * XI + i) + (lane >> 3), n_rows - 1) * pitch;
#pragma unroll
    for (int i = 0; i < 8; i++) wo[i] = (unsigned)w_column(8 * (wave * 8 + i) + (lane >> 3)) * pitch;
    const int chunk = (lane & 7) ^ (lane >> 4);
    auto chunk_offset = [&](int t, int instruction) __attribute__((always_inline)) {   // (blocks past the end: any bytes, their scales are zero)
      return (unsigned)min(8 * t + (chunk ^ (4 * (instruction & 1))), kb - 1) * 16u;
    };
    auto load_x = [&](int t, int i) __attribute__((always_inline)) {
      direct_load16(xb, xo[i] + chunk_offset(t, wave * XI + i), &lds[t & 1][0][(wave * XI + i) * 1024]);
    };
    auto load_w = [&](int t, int i) __attribute__((always_inline)) {
      direct_load16(wb, wo[i] + chunk_offset(t, i), &lds[t & 1][1][(wave * 8 + i) * 1024]);
    };
    // ---- scales: thread r brings those of row r and of LDS row r of the weights
    const int sr = min(tid, 32 * RB - 1);
    const uint8_t* const xsp = A.xs + (size_t)(r0 + min(sr, n_rows - 1)) * kb;
    const bool s_up = PAIR && ((tid >> 6) & 1);
    const uint8_t* const wsp = (s_up ? A.ws1 : A.ws0) + (e_row0 + w_column(tid)) * kb;
    const int xpos = (sr / (16 * RB)) * 128 + (sr & 15) * 8 + (sr % (16 * RB)) / 16;
    const int wpos = (tid >> 7) * 128 + (tid & 15) * 8 + ((tid >> 4) & 7);
    unsigned long long xsv, wsv;
    auto load_scales = [&](int t) __attribute__((always_inline)) {   // (rows of scales have any alignment; the last 8 of a row: zeros follow)
      const int o = min(8 * t, kb - 8);
      __builtin_memcpy(&xsv, xsp + o, 8);
      __builtin_memcpy(&wsv, wsp + o, 8);
    };
    auto write_scales = [&](int t) __attribute__((always_inline)) {
      const int past = 8 * (8 * t - min(8 * t, kb - 8));
      const unsigned long long x = xsv >> past, w = wsv >> past;
#pragma unroll
      for (int j = 0; j < 8; j++) {
        sc[t & 1][0][j * 256 + xpos] = (char)(x >> (8 * j));
        sc[t & 1][1][j * 256 + wpos] = (char)(w >> (8 * j));
      }
    };
    // ---- fragments
    struct Set { int4 x[RB], w[8]; int xs[2], ws[2]; } set[2];
    const unsigned frag_off = (unsigned)(m * 128 + ((q ^ ((m >> 1) & 7)) << 4));   // (half 1: chunk + 4, i.e. ^ 64)
    auto read_x = [&](Set& F, int t, int h, int b) __attribute__((always_inline)) {
      F.x[b] = *reinterpret_cast<const int4*>(&lds[t & 1][0][(wr * RB + b) * 2048 + (frag_off ^ (unsigned)(h * 64))]);
    };
    auto read_w = [&](Set& F, int t, int h, int a) __attribute__((always_inline)) {
      F.w[a] = *reinterpret_cast<const int4*>(&lds[t & 1][1][(wc * 8 + a) * 2048 + (frag_off ^ (unsigned)(h * 64))]);
    };
    auto read_s = [&](Set& F, int t, int h) __attribute__((always_inline)) {
      const int2 x = *reinterpret_cast<const int2*>(&sc[t & 1][0][(4 * h + q) * 256 + wr * 128 + m * 8]);
      const int2 w = *reinterpret_cast<const int2*>(&sc[t & 1][1][(4 * h + q) * 256 + wc * 128 + m * 8]);
      F.xs[0] = x.x; F.xs[1] = x.y; F.ws[0] = w.x; F.ws[1] = w.y;
    };
    mx_f32x4 acc[8][RB];
#pragma unroll
    for (int a = 0; a < 8; a++)
#pragma unroll
      for (int b = 0; b < RB; b++) acc[a][b] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
    // 8 groups of RB products, `between(a)` before each
    auto multiply = [&](const Set& F, auto&& between) __attribute__((always_inline)) {
      mx_for<8>([&](auto ac) __attribute__((always_inline)) {
        constexpr int a = decltype(ac)::value;
        between(a);
        __builtin_amdgcn_sched_barrier(0);
        mx_for<RB>([&](auto bc) __attribute__((always_inline)) {
          constexpr int b = decltype(bc)::value;
          acc[a][b] = mx_mfma<(a & 3), (b & 3)>(F.w[a], F.x[b], acc[a][b], F.ws[a >> 2], F.xs[b >> 2]);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto load_part = [&](int t, int a) __attribute__((always_inline)) {   // one eighth of a stage
      if (a < XI) load_x(t, a);
      load_w(t, a);
    };
#pragma unroll
    for (int a = 0; a < 8; a++) load_part(0, a);
    load_scales(0);
    write_scales(0);
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0), lgkmcnt(0)
    __syncthreads();
    if (nt > 1) {
#pragma unroll
      for (int a = 0; a < 8; a++) load_part(1, a);
      load_scales(1);
    }
    read_s(set[0], 0, 0);
#pragma unroll
    for (int b = 0; b < RB; b++) read_x(set[0], 0, 0, b);
#pragma unroll
    for (int a = 0; a < 8; a++) read_w(set[0], 0, 0, a);
    // One stage: its first half is multiplied while the second is read, the second while the next stage's first half is read and the stage
    // after that is requested.
    auto stage = [&](int t, auto more_c, auto more2_c) __attribute__((always_inline)) {
      constexpr bool MORE = decltype(more_c)::value, MORE2 = decltype(more2_c)::value;
      multiply(set[0], [&](int a) __attribute__((always_inline)) {
        if (a == 0) read_s(set[1], t, 1);
        if (a < RB) read_x(set[1], t, 1, a);
        read_w(set[1], t, 1, a);
      });
      if constexpr (MORE) {
        write_scales(t + 1);
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
      } else {
        if (kb - 8 * t <= 4) return;   // (the half has no blocks)
      }
      multiply(set[1], [&](int a) __attribute__((always_inline)) {
        if constexpr (MORE) {
          if (a == 0) read_s(set[0], t + 1, 0);
          if (a < RB) read_x(set[0], t + 1, 0, a);
          read_w(set[0], t + 1, 0, a);
        }
        if constexpr (MORE2) {
          load_part(t + 2, a);
          if (a == 7) load_scales(t + 2);
        }
      });
    };
    int t = 0;
    for (; t + 2 < nt; t++) stage(t, std::true_type{}, std::true_type{});
    if (t + 1 < nt) stage(t++, std::true_type{}, std::false_type{});
    stage(t, std::false_type{}, std::false_type{});
    // (the sums are complete here, in all lanes: left to itself the compiler moves the last products, and the reads of their operands, to the stores, past
    // the branch for the rows that there are)
#pragma unroll
    for (int a = 0; a < 8; a++)
#pragma unroll
      for (int b = 0; b < RB; b++) asm volatile("" : "+a"(acc[a][b]));
    // ---- results: acc[a][b][i] is row 16 (wr RB + b) + m, column mx_column(a, 4 q + i) of the wavefront's
#pragma unroll
    for (int b = 0; b < RB; b++) {
      const int row = 16 * (wr * RB + b) + m;
      if (row >= n_rows) continue;
      if constexpr (!PAIR) {
        uint16_t* const dst = A.y + (size_t)(r0 + row) * A.n;
#pragma unroll
        for (int p = 0; p < 4; p++) {
          const int col = c0 + wc * 128 + 32 * p + 8 * q;
          const mx_f32x4 lo = acc[2 * p][b], hi = acc[2 * p + 1][b];
          const float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          if (col < A.n) *reinterpret_cast<uint4*>(dst + col) = pack8(f);
        }
      } else {
#pragma unroll
        for (int p = 0; p < 2; p++) {
          const int col = c0 + wc * 64 + 32 * p + 8 * q;
          float f[8];
          unsigned e = 0;
#pragma unroll
          for (int i = 0; i < 8; i++) {
            const float g = acc[2 * p + (i >> 2)][b][i & 3], v = acc[4 + 2 * p + (i >> 2)][b][i & 3];
            f[i] = mx_silu(g) * v;
            e = max(e, (__float_as_uint(f[i]) >> 23) & 255u);
          }
          // (the four lanes of a row are in or out together)
          e = max(e, (unsigned)__shfl_xor((int)e, 16));
          e = max(e, (unsigned)__shfl_xor((int)e, 32));
          const unsigned s = mx_scale_code(e);
          if (col < A.n) {
            *reinterpret_cast<uint32_t*>(A.h + ((size_t)(r0 + row) * A.n + col) / 2) = mx_encode8(f, s);
            if (q == 0) A.hs[((size_t)(r0 + row) * A.n + col) / kMxBlock] = (uint8_t)s;
          }
        }
      }
    }
  };
  if (n_rows > 192) run(std::integral_constant<int, 8>{});
  else if (n_rows > 128) run(std::integral_constant<int, 6>{});
  else if (n_rows > 64) run(std::integral_constant<int, 4>{});
  else if (n_rows > 32) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 1>{});
}

// The same tile where rows of scales are whole dwords (K a multiple of 128): the scales, too, come directly into LDS, 32 bytes (1024 k) of a row at a time.
// A load's cost goes by the lines of 128 bytes that it touches (L2 -> LDS: 56 bytes a clock and CU with rows of 128 bytes, 30 with rows of 64), and
// 8 bytes of scales of each row for every stage cost as much as the stage itself: 8192 rows x 14336 x 4096,
// 322 -> 308 us (3.1 PFLOP/s; without any loads, 216).  A ring of four stages
// of 128 k, 64 bytes of a row each, was no faster than two of 256.  The products are 32x32x64: registers alone, 9.3 PFLOP/s on zeros and 6.4 on
// random codes, where 16x16x128 makes 5.5 and 5.1.
//
// In LDS the dwords of scales of row r, d of 8, are at d ^ ((r >> 3) & 7).  A batch of 1024 k comes in four parts with four stages, one batch ahead.
typedef float mx_f32x16 __attribute__((ext_vector_type(16)));
template <int BYTE>
__device__ __forceinline__ mx_f32x16 mx_mfma32(const int4& w, const int4& x, const mx_f32x16& acc, int ws, int xs) {
  const mx_i32x8 a = {w.x, w.y, w.z, w.w, 0, 0, 0, 0}, b = {x.x, x.y, x.z, x.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 4, BYTE, ws, BYTE, xs);
}
// Loads straight into LDS from a scalar base and the lane's offset; lane i's bytes land 16 i (4 i) further than `to`.
__device__ __forceinline__ unsigned long long mx_uniform(const void* p) {   // the same in all lanes: the compiler is told so
  const unsigned long long v = (unsigned long long)p;
  return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ __forceinline__ void mx_bring16(unsigned long long base, unsigned off, unsigned to) {
  to = (unsigned)__builtin_amdgcn_readfirstlane((int)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void mx_bring4(unsigned long long base, unsigned off, unsigned to) {
  to = (unsigned)__builtin_amdgcn_readfirstlane((int)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(to), "v"(off), "s"(base) : "memory");
}
template <int N>
__device__ __forceinline__ void mx_wait() {   // until at most N loads are on their way, and LDS has answered
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}

// Frag a's row m of a wavefront's weight rows -> its column among the wavefront's 128 (64 of either of a pair): a frag is a block of 32 columns, and
// lane l's 16 elements of it are its columns 16 (l / 32) .. + 15.
__device__ __forceinline__ int mx_column32(int a, int m) { return 32 * a + 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

constexpr int MX_BATCH = 2 * MXT * 32;   // bytes of a batch of scales of both operands

template <int KIND>
__global__ __launch_bounds__(256, 1) void mx_direct_kernel(const MxGemmArgs A) {
  constexpr bool PAIR = KIND == MX_GATE_UP;
  constexpr int COLS = PAIR ? MXT / 2 : MXT;   // columns of the result per tile
  __shared__ __attribute__((aligned(1024))) char lds[2][2][MX_STAGE];   // [stage][x, w]
  __shared__ __attribute__((aligned(1024))) char sc[2][2][MXT * 32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 31, q = lane >> 5;
  const int wr = wave & 1, wc = wave >> 1;
  MxTile T;
  if (!mx_find_tile<COLS>(A, lane, T)) return;
  const int kb = A.k / kMxBlock, dwords = kb / 4, nt = (kb + 7) / 8;

  auto run = [&](auto rb_c) __attribute__((always_inline)) {
    constexpr int RB = decltype(rb_c)::value;   // row frags of a wavefront: 64 RB rows in all
    constexpr int XI = 2 * RB;                  // loads of x per wavefront and stage
    // ---- addresses: a base per tile and 32 bits.  Load i of wavefront w brings rows 8 (w XI + i) .. + 7 of x and LDS rows 8 (8 w + i) .. + 7 of
    // the weights, LDS row r being frag (r / 32) % 4, m = r % 32 of wavefront column r / 128; lane l row l / 8 of them, and the chunk
    // (of scales the dword) that belongs at position l % 8.
    const unsigned pitch = (unsigned)kb * 16;
    const bool up = PAIR && (wave & 1);   // (LDS rows 64 w .. 64 w + 63: of a pair either all gate or all up)
    const size_t e_row0 = (size_t)T.expert * A.n + T.c0;
    const unsigned long long xb = mx_uniform(A.x + (size_t)T.r0 * pitch), wb = mx_uniform((up ? A.w1 : A.w0) + e_row0 * pitch);
    const unsigned long long xsb = mx_uniform(A.xs + (size_t)T.r0 * kb), wsb = mx_uniform((up ? A.ws1 : A.ws0) + e_row0 * kb);
    auto x_row = [&](int i) { return (unsigned)min(8 * (wave * XI + i) + (lane >> 3), T.n_rows - 1); };
    auto w_row = [&](int i) {
      const int row = 8 * (wave * 8 + i) + (lane >> 3), g = row >> 7, a = (row >> 5) & 3;
      return (unsigned)min(PAIR ? 64 * g + mx_column32(a & 1, row & 31) : 128 * g + mx_column32(a, row & 31), A.n - 1 - T.c0);
    };
    unsigned xo[XI], wo[8];
#pragma unroll
    for (int i = 0; i < XI; i++) xo[i] = x_row(i) * pitch;
#pragma unroll
    for (int i = 0; i < 8; i++) wo[i] = w_row(i) * pitch;
    const int chunk = (lane & 7) ^ (lane >> 4);
    const unsigned lds0 = (unsigned)(size_t)(lptr_t)&lds[0][0][0], sc0 = (unsigned)(size_t)(lptr_t)&sc[0][0][0];
    struct Part { unsigned offset[2], to; };   // of a stage: the chunk's offset by the parity of the load (blocks past the end: the last), LDS
    auto part_of = [&](int t) __attribute__((always_inline)) {
      return Part{{(unsigned)min(8 * t + chunk, kb - 1) * 16u, (unsigned)min(8 * t + (chunk ^ 4), kb - 1) * 16u}, lds0 + (t & 1) * 2 * MX_STAGE};
    };
    auto bring = [&](const Part& P, int i) __attribute__((always_inline)) {   // (load w XI + i is as odd as i: XI is even)
      if (i < XI) mx_bring16(xb, xo[i] + P.offset[i & 1], P.to + (wave * XI + i) * 1024);
      else mx_bring16(wb, wo[i - XI] + P.offset[(i - XI) & 1], P.to + MX_STAGE + (wave * 8 + i - XI) * 1024);
    };
    // two loads, v of them, of part u of batch b of x or (i) the weights; past the end of K: the last dword
    auto bring_scales = [&](int b, int u, int i, int v) __attribute__((always_inline)) {
      const int load = i ? 2 * u + v : min(2 * u + v, XI - 1), rows8 = wave * (i ? 8 : XI) + load;
      const unsigned dword = (unsigned)min(8 * b + ((lane & 7) ^ (rows8 & 7)), dwords - 1) * 4u, to = sc0 + (b & 1) * MX_BATCH + (i ? MXT * 32 : 0) + rows8 * 256;
      if (i) mx_bring4(wsb, w_row(load) * (unsigned)kb + dword, to);
      else mx_bring4(xsb, x_row(load) * (unsigned)kb + dword, to);
    };
    // ---- fragments: quarter j of a stage, 64 k
    struct Set { int4 x[RB], w[4]; } set[2];
    int raw[RB + 4], code[RB + 4];   // scales of half a stage: of the next one as they lie in memory; of this one, the lane's own in bytes 0 and 2
    const char* const f0 = &lds[0][0][0] + m * 128;
    constexpr int READS = RB + 4;
    auto read = [&](Set& F, int t, int j, int i) __attribute__((always_inline)) {
      const int at = (t & 1) * (2 * MX_STAGE) + ((2 * j + q) ^ ((m >> 1) & 7)) * 16;
      if (i < RB) F.x[i] = *reinterpret_cast<const int4*>(f0 + at + (wr * RB + i) * 4096);
      else F.w[i - RB] = *reinterpret_cast<const int4*>(f0 + at + MX_STAGE + (wc * 4 + i - RB) * 4096);
    };
    auto read_scale = [&](int t, int half, int i) __attribute__((always_inline)) {
      const int frag = i < RB ? wr * RB + i : wc * 4 + i - RB;   // (rows 32 frag + m)
      const int d = (2 * (t & 3) + half) ^ ((4 * frag + (m >> 3)) & 7);
      raw[i] = *reinterpret_cast<const int*>(&sc[0][0][0] + ((t >> 2) & 1) * MX_BATCH + (i < RB ? 0 : MXT * 32) + (32 * frag + m) * 32 + 4 * d);
    };
    mx_f32x16 acc[4][RB];
#pragma unroll
    for (int a = 0; a < 4; a++)
#pragma unroll
      for (int b = 0; b < RB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[a][b][i] = 0.f;
    // 4 RB products, `between(i)` before product i: a wavefront alone on its SIMD issues what else there is while one is under way, a little at a time.
    constexpr int PRODUCTS = 4 * RB;
    auto multiply = [&](const Set& F, auto byte_c, auto&& between) __attribute__((always_inline)) {
      mx_for<PRODUCTS>([&](auto ic) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value, a = i / RB, b = i % RB;
        between(ic);
        __builtin_amdgcn_sched_barrier(0);
        acc[a][b] = mx_mfma32<decltype(byte_c)::value>(F.w[a], F.x[b], acc[a][b], code[RB + a], code[b]);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // those of N things that come before product i
    auto share = [&](auto ic, auto nc, auto&& f) __attribute__((always_inline)) {
      mx_for<decltype(nc)::value>([&](auto kc) __attribute__((always_inline)) {
        if constexpr (decltype(kc)::value * PRODUCTS / decltype(nc)::value == decltype(ic)::value) f(decltype(kc)::value);
      });
    };
    typedef std::integral_constant<int, READS> Reads;
    typedef std::integral_constant<int, XI + 8> Loads;
    typedef std::integral_constant<int, 4> Four;
    auto shift_codes = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < READS; i++) code[i] = (int)((unsigned)raw[i] >> (8 * q));
    };
    // ---- the first two stages, the first batch and a part of the second
#pragma unroll
    for (int u = 0; u < 4; u++)
#pragma unroll
      for (int v = 0; v < 4; v++) bring_scales(0, u, v >> 1, v & 1);
    {
      const Part P = part_of(0);
#pragma unroll
      for (int i = 0; i < XI + 8; i++) bring(P, i);
    }
    mx_wait<0>();
    __syncthreads();
    if (nt > 1) {
      const Part P = part_of(1);
#pragma unroll
      for (int i = 0; i < XI + 8; i++) bring(P, i);
#pragma unroll
      for (int v = 0; v < 4; v++) bring_scales(1, 0, v >> 1, v & 1);
    }
#pragma unroll
    for (int i = 0; i < READS; i++) { read(set[0], 0, 0, i); read_scale(0, 0, i); }
    // Quarter j of stage t (not its last) while the next one, and before a half its scales, are read.
    auto quarter = [&](int t, auto jc) __attribute__((always_inline)) {
      constexpr int j = decltype(jc)::value;
      if constexpr (j != 1) shift_codes();
      multiply(set[j & 1], std::integral_constant<int, j & 1 ? 2 : 0>{}, [&](auto ic) __attribute__((always_inline)) {
        share(ic, Reads{}, [&](int i) __attribute__((always_inline)) {
          read(set[(j + 1) & 1], t, j + 1, i);
          if constexpr (j == 1) read_scale(t, 1, i);
        });
      });
    };
    // Stage t; before the barrier all of stage t + 1 has landed.  With its last quarter (MORE) stage t + 2 and a part of a batch are requested.
    auto stage = [&](int t, auto more_c) __attribute__((always_inline)) {
      constexpr bool MORE = decltype(more_c)::value;
      mx_for<3>([&](auto jc) __attribute__((always_inline)) { quarter(t, jc); });
      mx_wait<0>();
      __syncthreads();
      Part P;
      if constexpr (MORE) P = part_of(t + 2);
      multiply(set[1], std::integral_constant<int, 2>{}, [&](auto ic) __attribute__((always_inline)) {
        share(ic, Reads{}, [&](int i) __attribute__((always_inline)) { read(set[0], t + 1, 0, i); read_scale(t + 1, 0, i); });
        if constexpr (MORE) {
          share(ic, Loads{}, [&](int i) __attribute__((always_inline)) { bring(P, i); });
          share(ic, Four{}, [&](int v) __attribute__((always_inline)) { bring_scales((t + 5) >> 2, (t + 1) & 3, v >> 1, v & 1); });
        }
      });
    };
    int t = 0;
    for (; t + 2 < nt; t++) stage(t, std::true_type{});
    if (t + 1 < nt) stage(t++, std::false_type{});
    quarter(t, std::integral_constant<int, 0>{});
    quarter(t, std::integral_constant<int, 1>{});
    if (kb - 8 * t > 4) {   // (else the half has no blocks)
      quarter(t, std::integral_constant<int, 2>{});
      multiply(set[1], std::integral_constant<int, 2>{}, [&](auto) __attribute__((always_inline)) {});
    }
    // (the sums are complete here, in all lanes: left to itself the compiler moves the last products, and the reads of their operands, to the stores, past
    // the branch for the rows that there are)
#pragma unroll
    for (int a = 0; a < 4; a++)
#pragma unroll
      for (int b = 0; b < RB; b++) asm volatile("" : "+a"(acc[a][b]));
    // ---- results: acc[a][b][i] is row 32 (wr RB + b) + m, column 32 a + 16 q + i of the wavefront's
#pragma unroll
    for (int b = 0; b < RB; b++) {
      const int row = 32 * (wr * RB + b) + m;
      if (row >= T.n_rows) continue;
      const size_t out_row = (size_t)(T.r0 + row) * A.n;
      if constexpr (!PAIR) {
#pragma unroll
        for (int a = 0; a < 4; a++)
#pragma unroll
          for (int h = 0; h < 2; h++) {
            const int col = T.c0 + wc * 128 + 32 * a + 16 * q + 8 * h;
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; i++) f[i] = acc[a][b][8 * h + i];
            if (col < A.n) *reinterpret_cast<uint4*>(A.y + out_row + col) = pack8(f);
          }
      } else {
#pragma unroll
        for (int p = 0; p < 2; p++) {
          const int col = T.c0 + wc * 64 + 32 * p + 16 * q;
          float f[2][8];
          unsigned e = 0;
#pragma unroll
          for (int i = 0; i < 16; i++) {
            const float g = acc[p][b][i], h = mx_silu(g) * acc[2 + p][b][i];
            f[i >> 3][i & 7] = h;
            e = max(e, (__float_as_uint(h) >> 23) & 255u);
          }
          // (the two lanes of a row are in or out together)
          e = max(e, (unsigned)__shfl_xor((int)e, 32));
          const unsigned s = mx_scale_code(e);
          if (col < A.n) {
            *reinterpret_cast<uint2*>(A.h + (out_row + col) / 2) = make_uint2(mx_encode8(f[0], s), mx_encode8(f[1], s));
            if (q == 0) A.hs[(out_row + col) / kMxBlock] = (uint8_t)s;
          }
        }
      }
    }
  };
  if (T.n_rows > 192) run(std::integral_constant<int, 4>{});
  else if (T.n_rows > 128) run(std::integral_constant<int, 3>{});
  else if (T.n_rows > 64) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 1>{});
}

// Large tiles (8 scales of a row at once: 256 k at least) where there is work for the CUs, or where the contraction is long and most experts have
// rows; small ones elsewhere.  Measured, large to small tiles: 8 experts, 4096 columns, K = 4096, 128 rows 22 to 28 us, 1024 rows 28 to 60, 8192 rows 80 to
// 451; 64 experts, 2048 columns, K = 1408, 512 rows 23 to 22, 2048 rows (64 tiles) 25 to 26, 8192 rows 33 to 50; 8 experts, 1024 columns, K = 512, 2048 rows
// 15 to 10, 8192 rows 16 to 19; 1000 experts, 2048 columns, K = 2048, 16 rows 144 to 96 (a block has all of a CU's LDS), 1024 rows 581 to 606.
// Work is rows times columns (of a pair those of both weights), 2^22 of them: a round of small tiles.  From 512 k on a tile that its columns do not fill
// pays, too: 8 experts, 60000 rows of 96 columns, K = 512 11 to 16 us, 1920 22 to 32; 65536 rows of 192, K = 512 14 to 31, 1920 27 to 66; a pair of 64, 50000
// rows, K = 512 15 to 19, 1920 28 to 40.  With K = 256 and 320 the first and the last are 8.6 to 9.9 and 9.5 to 8.7, 13 to 11 and 15 to 11: there only whole tiles
// count, or three rounds' work of more than 128 columns (65536 rows of 192, 12 to 19 and 12 to 16).  Of 64 columns and fewer a tile is mostly empty: 131072
// rows of 64, K = 512 24 to 21, 1920 56 to 47.
static bool mx_large_tiles(MxKind kind, long long rows, int E, int n, int k) {
  const int columns = kind == MX_GATE_UP ? 2 * n : n;
  const long long work = rows * columns, round = 64ll * MXT * MXT;
  const bool fills = k >= 512 ? columns > 64 && work >= round : rows * (columns / MXT) >= 64ll * MXT || (columns > 128 && work >= 3 * round);
  return k >= 8 * kMxBlock && (fills || (k >= 2048 && rows >= E / 2));
}

template <int KIND>
static void launch_kind(const char* label, hipStream_t st, const MxGemmArgs& A, long long rows) {
  const int cols = KIND == MX_GATE_UP ? MXT / 2 : MXT, small_cols = KIND == MX_GATE_UP ? 64 : 128;
  const long long tiles = (rows / MXT + A.E) * ((A.n + cols - 1) / cols);   // (at most)
  if (mx_large_tiles((MxKind)KIND, rows, A.E, A.n, A.k)) {
    const long long round = MX_XCDS * MX_CHUNK;
    const dim3 grid((unsigned)((tiles + round - 1) / round * round));
    if (A.k % (4 * kMxBlock) == 0) MOE_LAUNCH(label, st, (mx_direct_kernel<KIND>), grid, dim3(256), 0, st, A);
    else MOE_LAUNCH(label, st, (mx_tile_kernel<KIND>), grid, dim3(256), 0, st, A);
  } else {
    MOE_LAUNCH(label, st, (mx_small_kernel<KIND>), dim3((unsigned)((rows / MXR + A.E) * ((A.n + small_cols - 1) / small_cols))), dim3(256), 0, st, A);
  }
}

void launch_mx_gemm(const char* label, hipStream_t st, MxKind kind, const MxGemmArgs& A, long long rows) {
  if (kind == MX_GATE_UP) launch_kind<MX_GATE_UP>(label, st, A, rows);
  else launch_kind<MX_PRODUCT>(label, st, A, rows);
}

}  // namespace moe

static int check_gemm(int experts, int64_t rows, int n, int k) {
  if (experts < 1 || experts > moe::kMaxExperts || rows < 0 || rows >= (1ll << 31)) return MOE_ERR_SHAPE;
  if (n < 8 || n % 8 || n > moe::kMaxWidth || k < moe::kMxBlock || k % moe::kMxBlock || k > moe::kMaxWidth) return MOE_ERR_SHAPE;
  if ((rows / moe::MXR + experts) * ((n + 127) / 128) >= (1ll << 24)) return MOE_ERR_SHAPE;   // (a launch has fewer than 2^32 threads)
  return MOE_OK;
}

extern "C" int moe_mxfp4_grouped_gemm_large_tiles(int experts, int64_t rows, int n, int k) {
  return check_gemm(experts, rows, n, k) == MOE_OK && moe::mx_large_tiles(moe::MX_PRODUCT, rows, experts, n, k);
}

extern "C" int moe_mxfp4_grouped_gemm(int experts, int64_t rows, int n, int k, const uint8_t* xq, const uint8_t* x_scales, const int32_t* offsets,
                                      const uint8_t* wq, const uint8_t* w_scales, uint16_t* y, void* stream) {
  using namespace moe;
  const int rc = check_gemm(experts, rows, n, k);
  if (rc != MOE_OK || rows == 0) return rc;
  MOE_REQUIRE_PTR(xq); MOE_REQUIRE_PTR(x_scales); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(wq); MOE_REQUIRE_PTR(w_scales); MOE_REQUIRE_PTR(y);
  MOE_REQUIRE_ALIGNED(xq); MOE_REQUIRE_ALIGNED(x_scales); MOE_REQUIRE_ALIGNED(offsets); MOE_REQUIRE_ALIGNED(wq); MOE_REQUIRE_ALIGNED(w_scales);
  MOE_REQUIRE_ALIGNED(y);
  MxGemmArgs A = {};
  A.offsets = offsets; A.E = experts; A.n = n; A.k = k;
  A.x = xq; A.xs = x_scales; A.w0 = wq; A.ws0 = w_scales; A.y = y;
  launch_mx_gemm("mx_grouped_gemm", (hipStream_t)stream, MX_PRODUCT, A, rows);
  return launch_status();
}

extern "C" size_t moe_mxfp4_workspace_bytes(const moe_shape* shape) {
  moe::Dims D;
  return moe::check_shape(shape, &D) == MOE_OK ? moe::ws_layout(D).mx_total : 0;
}

extern "C" int moe_mxfp4_grouped_ffn_fwd(const moe_shape* shape, const uint16_t* x_perm, const int32_t* offsets, const uint8_t* wq_gate,
                                         const uint8_t* s_gate, const uint8_t* wq_up, const uint8_t* s_up, const uint8_t* wq_down,
                                         const uint8_t* s_down, uint16_t* y_perm, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  Dims D;
  const int rc = check_shape(shape, &D);
  if (rc != MOE_OK) return rc;
  if ((D.N / MXR + D.Et) * (long long)(D.f / 64) >= (1ll << 24) || (D.N / MXR + D.Et) * (long long)((D.d + 127) / 128) >= (1ll << 24)) return MOE_ERR_SHAPE;
  if (D.N == 0) return MOE_OK;
  const void* const ptrs[] = {x_perm, offsets, wq_gate, s_gate, wq_up, s_up, wq_down, s_down, y_perm, ws};
  for (const void* p : ptrs) MOE_REQUIRE_PTR(p);
  for (const void* p : ptrs) MOE_REQUIRE_ALIGNED(p);
  if (!aligned(ws, 256)) return MOE_ERR_ALIGN;
  const WsLayout L = ws_layout(D);
  if (ws_bytes < L.mx_total) return MOE_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  uint8_t* const wsb = static_cast<uint8_t*>(ws);
  uint8_t* const xq = wsb + L.mx_x; uint8_t* const xs = wsb + L.mx_xs; uint8_t* const hq = wsb + L.mx_h; uint8_t* const hs = wsb + L.mx_hs;
  launch_mx_quantize(st, x_perm, xq, xs, D.N * D.d);
  MxGemmArgs A = {};
  A.offsets = offsets; A.E = D.Et; A.n = D.f; A.k = D.d;
  A.x = xq; A.xs = xs; A.w0 = wq_gate; A.ws0 = s_gate; A.w1 = wq_up; A.ws1 = s_up; A.h = hq; A.hs = hs;
  launch_mx_gemm("mx_gate_up", st, MX_GATE_UP, A, D.N);
  A.n = D.d; A.k = D.f; A.x = hq; A.xs = hs; A.w0 = wq_down; A.ws0 = s_down; A.y = y_perm;
  launch_mx_gemm("mx_down", st, MX_PRODUCT, A, D.N);
  return launch_status();
}
