// Grouped products in microscaled 4-bit floating point (E2M1 values, a power-of-two scale per 32 along the contraction):
//     y[r, c] = sum_k x[r, k] w[e(r)][c, k]      and the SwiGLU pair  h = Q(silu(x W_gate) (x W_up)),
// on the block-scaled MFMA 16x16x128, which applies both scales and accumulates in fp32.
//
// Operand layout (both operands alike): lane l holds row l % 16, k = 32 (l / 16) .. + 31, i.e. one block and its scale.  The weights are the A
// operand, so that a lane owns consecutive columns of a result row: with frag a's row m taken from column CPL (m / 4) + 4 a + m % 4 of the
// wavefront's columns (CPL = columns per lane), lane l ends up with columns CPL (l / 16) .. + CPL - 1 of row l % 16.
#include "mx_gemm.h"

namespace moe {

constexpr int MXR = 128;   // rows of a tile

template <int KIND>
__global__ __launch_bounds__(256) void mx_gemm_kernel(const MxGemmArgs A) {
  constexpr int NW = KIND == MX_GATE_UP ? 2 : 1;
  constexpr int WC = 64 / NW;          // columns of a wavefront, of either weight
  constexpr int FR = WC / 16;          // their frags
  constexpr int CPL = WC / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, q = lane >> 4;
  const int n_ct = (A.n + 2 * WC - 1) / (2 * WC);
  const int u = blockIdx.x / n_ct, ct = blockIdx.x % n_ct;
  MxTile T;
  if (!mx_find_tile<MXR>(A.offsets, A.E, u, lane, T)) return;
  const int r0 = T.lo + (wave & 1) * 64, c0 = (ct * 2 + (wave >> 1)) * WC;
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
        f[i] = g / (1.0f + __expf(-g)) * v;
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

void launch_mx_gemm(const char* label, hipStream_t st, MxKind kind, const MxGemmArgs& A, long long rows) {
  const long long row_tiles = rows / MXR + A.E;   // (at most)
  const int wc = kind == MX_GATE_UP ? 64 : 128;
  const dim3 grid((unsigned)(row_tiles * ((A.n + wc - 1) / wc)));
  if (kind == MX_GATE_UP) MOE_LAUNCH(label, st, (mx_gemm_kernel<MX_GATE_UP>), grid, dim3(256), 0, st, A);
  else MOE_LAUNCH(label, st, (mx_gemm_kernel<MX_PRODUCT>), grid, dim3(256), 0, st, A);
}

}  // namespace moe

extern "C" int moe_mxfp4_grouped_gemm(int experts, int64_t rows, int n, int k, const uint8_t* xq, const uint8_t* x_scales, const int32_t* offsets,
                                      const uint8_t* wq, const uint8_t* w_scales, uint16_t* y, void* stream) {
  using namespace moe;
  if (experts < 1 || experts > kMaxExperts || rows < 0 || rows >= (1ll << 31)) return MOE_ERR_SHAPE;
  if (n < 8 || n % 8 || n > kMaxWidth || k < kMxBlock || k % kMxBlock || k > kMaxWidth) return MOE_ERR_SHAPE;
  if ((rows / MXR + experts) * ((n + 127) / 128) >= (1ll << 24)) return MOE_ERR_SHAPE;   // (a launch has fewer than 2^32 threads)
  if (rows == 0) return MOE_OK;
  MOE_REQUIRE_PTR(xq); MOE_REQUIRE_PTR(x_scales); MOE_REQUIRE_PTR(offsets); MOE_REQUIRE_PTR(wq); MOE_REQUIRE_PTR(w_scales); MOE_REQUIRE_PTR(y);
  MOE_REQUIRE_ALIGNED(xq); MOE_REQUIRE_ALIGNED(x_scales); MOE_REQUIRE_ALIGNED(offsets); MOE_REQUIRE_ALIGNED(wq); MOE_REQUIRE_ALIGNED(w_scales);
  MOE_REQUIRE_ALIGNED(y);
  MxGemmArgs A = {};
  A.offsets = offsets; A.E = experts; A.n = n; A.k = k;
  A.x = xq; A.xs = x_scales; A.w0 = wq; A.ws0 = w_scales; A.y = y;
  launch_mx_gemm("mx_grouped_gemm", (hipStream_t)stream, MX_PRODUCT, A, rows);
  return launch_status();
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
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
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
