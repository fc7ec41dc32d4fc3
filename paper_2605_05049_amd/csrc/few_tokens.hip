// A whole MoE layer for a few tokens (at most 64): logits = x W_r^T, top-k gate, the chosen experts' SwiGLU FFNs and the weighted sum,
//     out[t] = sum_j w[t, j] (silu(x_t Wg) * (x_t Wu)) Wd     over the experts of token t,
// on weights in bf16 (W_gate, W_up [E', d, f], W_down [E', f, d]) or microscaled 4-bit floating point ([E', f, d / 2], [E', d, f / 2]).
//
// What bounds it: the weights of the experts that some token chose are read once and multiply a handful of rows, so the time is that of
// streaming them.  The rows are not permuted into buffers: an expert's tokens are columns 0 .. 15 (of up to four groups) of an MFMA whose
// other operand is the weights.  The weights go from memory straight into registers: of bf16 weights a lane holds 4 columns of 8 k-rows, and
// turns them with byte permutes into the MFMA's operand, 8 k of one column; of 4-bit weights it holds 32 k of one column (a block, one scale) and
// widens them to bf16, exactly.  The hidden activation stays in fp32 in effect: it is kept as a bf16 head and a bf16 remainder, both of
// which multiply W_down; the partial sums of W_down's parts and the experts are added in fp32, in a fixed order.
#include "mxfp4.h"
#include "route.h"

#include <type_traits>

namespace moe {

namespace {

constexpr int kFewTokens = MOE_FEW_TOKENS_MAX;
constexpr int kFewSlots = 4096;    // T * K' at most
constexpr int kFewWaves = 8;
constexpr int kFewTileCols = 64;   // columns of a block's tile (of either matrix of the pair)
constexpr int kFewPitch = kFewTileCols + 4;

// What the gate kernel leaves for the others: the experts that have tokens, in expert order, and the slots of each.
struct FewSched {
  int32_t n_live, pad[3];
  int4 live[kMaxExperts];     // expert, its first entry in slots, its slots
  int32_t slots[kFewSlots];   // t * K' + j
};

struct FewWeights { const uint8_t* w; const uint8_t* scales; };   // bf16 weights have no scales
struct FewArgs {
  int T, d, f, E, Es, k, Kp, renorm, parts;   // parts of d_ffn in the down projection
  const uint16_t* x; const uint16_t* w_router;
  float* logits; int32_t* topk_idx; float* topk_w; FewSched* sched;
  FewWeights gate, up, down;
  uint16_t* h; size_t h_lo;      // [N, f] bf16 heads, the remainders h_lo elements further
  float* partial;                // [N, parts, d]
  uint16_t* out;
};

// ---- logits and gate ---------------------------------------------------------------------------------------------------------------

// 16 experts x 16 tokens per block, K split over the wavefronts, whose sums are added in order.
__global__ __launch_bounds__(kFewWaves * kWave) void few_router_kernel(const FewArgs A) {
  __shared__ float part[kFewWaves][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
  const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  const uint16_t* const wr = A.w_router + (size_t)min(e0 + n, A.E - 1) * A.d + 8 * q;
  const uint16_t* const xr = A.x + (size_t)min(t0 + n, A.T - 1) * A.d + 8 * q;
  const int steps = A.d / 32, per = (steps + kFewWaves - 1) / kFewWaves;
  mx_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = wave * per; s < min(steps, (wave + 1) * per); s++)
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const mx_bf16x8*>(wr + s * 32), *reinterpret_cast<const mx_bf16x8*>(xr + s * 32), acc, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; i++) part[wave][n][4 * q + i] = acc[i];   // [token][expert]
  __syncthreads();
  if (threadIdx.x < 256) {
    const int t = threadIdx.x >> 4, e = threadIdx.x & 15;
    float sum = 0.f;
#pragma unroll
    for (int p = 0; p < kFewWaves; p++) sum += part[p][t][e];
    if (t0 + t < A.T && e0 + e < A.E) A.logits[(size_t)(t0 + t) * A.E + e0 + e] = sum;
  }
}

// One block: the gate of every token (unless the caller brought it), then the experts that have tokens and the slots of each.
template <int PER>
__global__ __launch_bounds__(1024) void few_gate_kernel(const FewArgs A) {
  __shared__ int count[kMaxExperts], first[kMaxExperts], live_before[kMaxExperts];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int Et = A.E + A.Es, N = A.T * A.Kp;
  if (A.w_router)
    for (int t = wave; t < A.T; t += 16)
      route_token<kWave, PER>(A.logits + (size_t)t * A.E, t, lane, A.topk_idx, A.topk_w, nullptr, A.E, A.k, A.Es, A.renorm);
  count[threadIdx.x] = 0;
  __threadfence_block();
  __syncthreads();
  auto expert_of = [&](int s) { return min(max(A.topk_idx[s], 0), Et - 1); };
  for (int s = threadIdx.x; s < N; s += 1024) atomicAdd(&count[expert_of(s)], 1);
  __syncthreads();
  if (wave == 0) {
    int slots = 0, live = 0;
    for (int e0 = 0; e0 < Et; e0 += kWave) {
      const int e = e0 + lane, c = e < Et ? count[e] : 0;
      const int incl = wave_prefix_sum(c), l_incl = wave_prefix_sum(c > 0 ? 1 : 0);
      if (e < Et) { first[e] = slots + incl - c; live_before[e] = live + l_incl - (c > 0 ? 1 : 0); }
      slots += __builtin_amdgcn_readlane(incl, kWave - 1);
      live += __builtin_amdgcn_readlane(l_incl, kWave - 1);
    }
    if (lane == 0) A.sched->n_live = live;
  }
  __syncthreads();
  if ((int)threadIdx.x < Et && count[threadIdx.x] > 0)
    A.sched->live[live_before[threadIdx.x]] = make_int4(threadIdx.x, first[threadIdx.x], count[threadIdx.x], 0);
  __syncthreads();
  // (the order of an expert's slots follows no rule and changes no result: every slot's sums are its own)
  for (int s = threadIdx.x; s < N; s += 1024) A.sched->slots[atomicAdd(&first[expert_of(s)], 1)] = s;
}

// ---- streaming products --------------------------------------------------------------------------------------------------------------

// acc[g][j] += W[k][col] X[k][token]: lane l's element i of acc[g][j] is column 16 (l / 16) + 4 i + j of the tile's 64, token 16 g + l % 16.
// Steps step0 .. step1 - 1 of 32 (bf16) or 128 k (4 bits; the last one may be cut short).  w: the expert's matrix, C columns of K values;
// x: the lane's rows (LO: and remainders x_lo elements further).
template <bool MX, int TG, bool LO>
__device__ __forceinline__ void few_multiply(mx_f32x4 (&acc)[TG][4], const FewWeights W, int expert, int K, int C, int col0,
                                             const uint16_t* const (&x)[TG], size_t x_lo, int step0, int step1, int lane) {
  const int c = lane & 15, q = lane >> 4;
  constexpr int KS = MX ? 4 : 1;   // MFMAs (of 32 k) per step and column frag
  constexpr int DEPTH = 2;
  struct Stage { uint4 w4[MX ? 4 : 1]; unsigned s[MX ? 4 : 1]; uint2 w2[MX ? 1 : 8]; } st[DEPTH];
  const int kb = K / kMxBlock;
  const uint8_t* base;
  const uint8_t* sbase = nullptr;
  size_t lane_off = 0;
  if constexpr (MX) {
    const size_t row = (size_t)expert * C + col0 + 4 * c;
    base = W.w + row * (kb * 16) + q * 16;
    sbase = W.scales + row * kb + q;
  } else {
    base = W.w + ((size_t)expert * K * C + col0) * 2;
    lane_off = ((size_t)(8 * q) * C + 4 * c) * 2;
  }
  auto load = [&](Stage& s, int step) __attribute__((always_inline)) {
    if constexpr (MX) {
      const bool in = 4 * step + q < kb;
#pragma unroll
      for (int a = 0; a < 4; a++) {
        s.w4[a] = make_uint4(0, 0, 0, 0);
        s.s[a] = 127;
        if (in) {
          s.w4[a] = *reinterpret_cast<const uint4*>(base + (size_t)a * (kb * 16) + (size_t)step * 64);
          s.s[a] = sbase[(size_t)a * kb + step * 4];
        }
      }
    } else {
      const uint8_t* const p = base + (size_t)step * 64 * C + lane_off;
#pragma unroll
      for (int i = 0; i < 8; i++) s.w2[i] = *reinterpret_cast<const uint2*>(p + (size_t)i * C * 2);
    }
  };
  auto consume = [&](const Stage& s, int step) __attribute__((always_inline)) {
    const bool in = !MX || 4 * step + q < kb;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      mx_bf16x8 w[4];
      if constexpr (MX) {
#pragma unroll
        for (int a = 0; a < 4; a++) {
          const float scale = __uint_as_float(s.s[a] == 255u ? 0x7fc00000u : s.s[a] << 23);
          const unsigned v = ks == 0 ? s.w4[a].x : ks == 1 ? s.w4[a].y : ks == 2 ? s.w4[a].z : s.w4[a].w;
          union { mx_bf16x2 p[4]; mx_bf16x8 v; } u;
          u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0);
          u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1);
          u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2);
          u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3);
          w[a] = u.v;
        }
      } else {
#pragma unroll
        for (int a = 0; a < 4; a++) {
          union { unsigned p[4]; mx_bf16x8 v; } u;
#pragma unroll
          for (int p = 0; p < 4; p++) {
            const unsigned lo = a < 2 ? s.w2[2 * p].x : s.w2[2 * p].y, hi = a < 2 ? s.w2[2 * p + 1].x : s.w2[2 * p + 1].y;
            u.p[p] = __builtin_amdgcn_perm(hi, lo, a & 1 ? 0x07060302u : 0x05040100u);
          }
          w[a] = u.v;
        }
      }
#pragma unroll
      for (int g = 0; g < TG; g++) {
        const size_t o = MX ? (size_t)step * 128 + 32 * q + 8 * ks : (size_t)step * 32 + 8 * q;
        mx_bf16x8 v = {}, v_lo = {};
        if (in) {
          v = *reinterpret_cast<const mx_bf16x8*>(x[g] + o);
          if constexpr (LO) v_lo = *reinterpret_cast<const mx_bf16x8*>(x[g] + x_lo + o);
        }
#pragma unroll
        for (int a = 0; a < 4; a++) {
          acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[a], v, acc[g][a], 0, 0, 0);
          if constexpr (LO) acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[a], v_lo, acc[g][a], 0, 0, 0);
        }
      }
    }
  };
#pragma unroll
  for (int i = 0; i < DEPTH - 1; i++)
    if (step0 + i < step1) load(st[i], step0 + i);
  for (int s = step0; s < step1; s += DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; i++) {
      if (s + i < step1) {
        if (s + i + DEPTH - 1 < step1) load(st[(i + DEPTH - 1) % DEPTH], s + i + DEPTH - 1);
        consume(st[i], s + i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}

// Runs `body` with the groups of 16 tokens that `rows` need, at most TGMAX.
template <int TGMAX, class F>
__device__ __forceinline__ void few_groups(int rows, F&& body) {
  if constexpr (TGMAX >= 4) { if (rows > 32) { body(std::integral_constant<int, 4>{}); return; } }
  if constexpr (TGMAX >= 2) { if (rows > 16) { body(std::integral_constant<int, 2>{}); return; } }
  body(std::integral_constant<int, 1>{});
}

// H = silu(x W_gate) * (x W_up) of 64 columns of one expert; wavefronts 0, 2, 4, 6 make G, the others U, each over a quarter of d.
template <bool MX, int TGMAX>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void few_gate_up_kernel(const FewArgs A) {
  __shared__ __attribute__((aligned(16))) float part[kFewWaves][16][kFewPitch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.y >= A.sched->n_live) return;
  const int4 L = A.sched->live[blockIdx.y];
  const int32_t* const slots = A.sched->slots + L.y;
  const int col0 = blockIdx.x * kFewTileCols;
  const int steps = MX ? (A.d / 32 + 3) / 4 : A.d / 32, per = (steps + 3) / 4;
  const int step0 = min(steps, (wave >> 1) * per), step1 = min(steps, step0 + per);
  for (int r0 = 0; r0 < L.z; r0 += 16 * TGMAX) {
    few_groups<TGMAX>(L.z - r0, [&](auto tg) __attribute__((always_inline)) {
      constexpr int TG = decltype(tg)::value;
      mx_f32x4 acc[TG][4];
      const uint16_t* x[TG];
#pragma unroll
      for (int g = 0; g < TG; g++) {
        x[g] = A.x + (size_t)(slots[min(r0 + 16 * g + (lane & 15), L.z - 1)] / A.Kp) * A.d;
#pragma unroll
        for (int a = 0; a < 4; a++) acc[g][a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
      }
      few_multiply<MX, TG, false>(acc, wave & 1 ? A.up : A.gate, L.x, A.d, A.f, col0, x, 0, step0, step1, lane);
#pragma unroll
      for (int g = 0; g < TG; g++) {
        __syncthreads();
        float* const dst = &part[wave][lane & 15][16 * (lane >> 4)];
#pragma unroll
        for (int i = 0; i < 4; i++) *reinterpret_cast<float4*>(dst + 4 * i) = make_float4(acc[g][0][i], acc[g][1][i], acc[g][2][i], acc[g][3][i]);
        __syncthreads();
        // 512 threads: 16 tokens x 32 pairs of columns
        const int t = threadIdx.x >> 5, c = 2 * (threadIdx.x & 31), row = r0 + 16 * g + t;
        if (row < L.z) {
          float v[2][2] = {};
#pragma unroll
          for (int w = 0; w < kFewWaves; w++) {
            const float2 p = *reinterpret_cast<const float2*>(&part[w][t][c]);
            v[w & 1][0] += p.x;
            v[w & 1][1] += p.y;
          }
          float h[2], lo[2];
#pragma unroll
          for (int i = 0; i < 2; i++) {
            h[i] = v[0][i] / (1.0f + __expf(-v[0][i])) * v[1][i];
            lo[i] = h[i] - bf16_to_f32(f32_to_bf16(h[i]));
          }
          uint16_t* const o = A.h + (size_t)slots[row] * A.f + col0 + c;
          *reinterpret_cast<uint32_t*>(o) = pack_bf16(h[0], h[1]);
          *reinterpret_cast<uint32_t*>(o + A.h_lo) = pack_bf16(lo[0], lo[1]);
        }
      }
    });
  }
}

// 64 columns of H W_down of one expert over one part of d_ffn, which the wavefronts share.
template <bool MX, int TGMAX>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void few_down_kernel(const FewArgs A) {
  __shared__ __attribute__((aligned(16))) float part[kFewWaves][16][kFewPitch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.y >= A.sched->n_live) return;
  const int4 L = A.sched->live[blockIdx.y];
  const int32_t* const slots = A.sched->slots + L.y;
  const int col0 = blockIdx.x * kFewTileCols;
  const int steps = MX ? (A.f / 32 + 3) / 4 : A.f / 32, waves = A.parts * kFewWaves, per = (steps + waves - 1) / waves;
  const int step0 = min(steps, ((int)blockIdx.z * kFewWaves + wave) * per), step1 = min(steps, step0 + per);
  for (int r0 = 0; r0 < L.z; r0 += 16 * TGMAX) {
    few_groups<TGMAX>(L.z - r0, [&](auto tg) __attribute__((always_inline)) {
      constexpr int TG = decltype(tg)::value;
      mx_f32x4 acc[TG][4];
      const uint16_t* h[TG];
#pragma unroll
      for (int g = 0; g < TG; g++) {
        h[g] = A.h + (size_t)slots[min(r0 + 16 * g + (lane & 15), L.z - 1)] * A.f;
#pragma unroll
        for (int a = 0; a < 4; a++) acc[g][a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
      }
      few_multiply<MX, TG, true>(acc, A.down, L.x, A.f, A.d, col0, h, A.h_lo, step0, step1, lane);
#pragma unroll
      for (int g = 0; g < TG; g++) {
        __syncthreads();
        float* const dst = &part[wave][lane & 15][16 * (lane >> 4)];
#pragma unroll
        for (int i = 0; i < 4; i++) *reinterpret_cast<float4*>(dst + 4 * i) = make_float4(acc[g][0][i], acc[g][1][i], acc[g][2][i], acc[g][3][i]);
        __syncthreads();
        const int t = threadIdx.x >> 5, c = 2 * (threadIdx.x & 31), row = r0 + 16 * g + t;
        if (row < L.z) {
          float2 v = make_float2(0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kFewWaves; w++) {
            const float2 p = *reinterpret_cast<const float2*>(&part[w][t][c]);
            v.x += p.x;
            v.y += p.y;
          }
          *reinterpret_cast<float2*>(A.partial + ((size_t)slots[row] * A.parts + blockIdx.z) * A.d + col0 + c) = v;
        }
      }
    });
  }
}

// out[t] = sum_j w[t, j] sum_parts partial: slots in order, fp32, one rounding.
__global__ __launch_bounds__(256) void few_combine_kernel(const FewArgs A) {
  const int i = blockIdx.x * 256 + threadIdx.x, per = A.d / 4;
  const int t = i / per, c = 4 * (i % per);
  if (t >= A.T) return;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < A.Kp; j++) {
    const int s = t * A.Kp + j;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < A.parts; p++) {
      const float4 v = *reinterpret_cast<const float4*>(A.partial + ((size_t)s * A.parts + p) * A.d + c);
      y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
    }
    const float w = A.topk_w[s];
    sum.x += w * y.x; sum.y += w * y.y; sum.z += w * y.z; sum.w += w * y.w;
  }
  *reinterpret_cast<uint2*>(A.out + (size_t)t * A.d + c) = make_uint2(pack_bf16(sum.x, sum.y), pack_bf16(sum.z, sum.w));
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

// Experts that can have tokens.
int few_live_bound(const Dims& D) { return (int)min((long long)D.E, (long long)D.T * D.k) + D.Es; }

// Parts of d_ffn in the down projection: as many as give every CU two blocks, but at least four steps of 32 k for a wavefront.
int few_parts(const Dims& D) {
  const long long blocks = (long long)(D.d / kFewTileCols) * few_live_bound(D);
  const int most = max(1, D.f / (32 * 4 * kFewWaves));
  return (int)min((long long)most, max(1ll, (512 + blocks - 1) / blocks));
}

struct FewLayout { size_t logits, sched, h, partial, total; };
FewLayout few_layout(const Dims& D) {
  FewLayout L;
  size_t o = 0;
  L.sched = o; o += round_up(sizeof(FewSched), 256);
  L.logits = o; o += round_up((size_t)D.T * D.E * sizeof(float), 256);
  L.h = o; o += round_up((size_t)D.N * D.f * 2 * sizeof(uint16_t), 256);
  L.partial = o; o += round_up((size_t)D.N * few_parts(D) * D.d * sizeof(float), 256);
  L.total = o;
  return L;
}

int check_few(const moe_shape* s, Dims* D) {
  const int rc = check_shape(s, D);
  if (rc != MOE_OK) return rc;
  if (D->T > kFewTokens || D->N > kFewSlots) return MOE_ERR_SHAPE;
  return MOE_OK;
}

template <bool MX, int TGMAX>
void few_launch_experts(hipStream_t st, const FewArgs& A, int live) {
  const dim3 block(kFewWaves * kWave);
  MOE_LAUNCH("few_gate_up", st, (few_gate_up_kernel<MX, TGMAX>), dim3(A.f / kFewTileCols, live), block, 0, st, A);
  MOE_LAUNCH("few_down", st, (few_down_kernel<MX, (MX && TGMAX > 2 ? 2 : TGMAX)>), dim3(A.d / kFewTileCols, live, A.parts), block, 0, st, A);
}

template <bool MX>
int few_forward(const moe_shape* shape, const uint16_t* x, const uint16_t* w_router, const FewWeights (&W)[3], uint16_t* out, int32_t* topk_idx,
                float* topk_w, void* ws, size_t ws_bytes, void* stream) {
  Dims D;
  const int rc = check_few(shape, &D);
  if (rc != MOE_OK || D.T == 0) return rc;
  const void* const ptrs[] = {x, W[0].w, W[1].w, W[2].w, out, topk_idx, topk_w, ws};
  for (const void* p : ptrs) MOE_REQUIRE_PTR(p);
  for (const void* p : ptrs) MOE_REQUIRE_ALIGNED(p);
  MOE_REQUIRE_ALIGNED(w_router);
  if (MX)
    for (const FewWeights& w : W) { MOE_REQUIRE_PTR(w.scales); MOE_REQUIRE_ALIGNED(w.scales); }
  if (!aligned(ws, 256)) return MOE_ERR_ALIGN;
  const FewLayout L = few_layout(D);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  uint8_t* const wsb = static_cast<uint8_t*>(ws);
  FewArgs A = {};
  A.T = D.T; A.d = D.d; A.f = D.f; A.E = D.E; A.Es = D.Es; A.k = D.k; A.Kp = D.Kp; A.renorm = D.renorm; A.parts = few_parts(D);
  A.x = x; A.w_router = w_router; A.topk_idx = topk_idx; A.topk_w = topk_w; A.out = out;
  A.gate = W[0]; A.up = W[1]; A.down = W[2];
  A.logits = reinterpret_cast<float*>(wsb + L.logits);
  A.sched = reinterpret_cast<FewSched*>(wsb + L.sched);
  A.h = reinterpret_cast<uint16_t*>(wsb + L.h);
  A.h_lo = (size_t)D.N * D.f;
  A.partial = reinterpret_cast<float*>(wsb + L.partial);
  hipStream_t st = (hipStream_t)stream;
  if (w_router)
    MOE_LAUNCH("few_router", st, few_router_kernel, dim3((D.E + 15) / 16, (D.T + 15) / 16), dim3(kFewWaves * kWave), 0, st, A);
  if (D.E <= 64) MOE_LAUNCH("few_gate", st, few_gate_kernel<1>, dim3(1), dim3(1024), 0, st, A);
  else if (D.E <= 256) MOE_LAUNCH("few_gate", st, few_gate_kernel<4>, dim3(1), dim3(1024), 0, st, A);
  else MOE_LAUNCH("few_gate", st, few_gate_kernel<16>, dim3(1), dim3(1024), 0, st, A);
  const int live = few_live_bound(D);
  if (D.T <= 16) few_launch_experts<MX, 1>(st, A, live);
  else few_launch_experts<MX, 4>(st, A, live);
  MOE_LAUNCH("few_combine", st, few_combine_kernel, dim3((unsigned)(((size_t)D.T * (D.d / 4) + 255) / 256)), dim3(256), 0, st, A);
  return launch_status();
}

}  // namespace

}  // namespace moe

extern "C" size_t moe_layer_few_workspace_bytes(const moe_shape* shape) {
  moe::Dims D;
  return moe::check_few(shape, &D) == MOE_OK ? moe::few_layout(D).total : 0;
}

extern "C" int moe_layer_few_fwd(const moe_shape* shape, const uint16_t* x, const uint16_t* w_router, const uint16_t* w_gate, const uint16_t* w_up,
                                 const uint16_t* w_down, uint16_t* out, int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes,
                                 void* stream) {
  auto bytes = [](const uint16_t* p) { return moe::FewWeights{reinterpret_cast<const uint8_t*>(p), nullptr}; };
  const moe::FewWeights W[3] = {bytes(w_gate), bytes(w_up), bytes(w_down)};
  return moe::few_forward<false>(shape, x, w_router, W, out, topk_idx, topk_w, ws, ws_bytes, stream);
}

extern "C" int moe_layer_few_mxfp4_fwd(const moe_shape* shape, const uint16_t* x, const uint16_t* w_router, const uint8_t* wq_gate,
                                       const uint8_t* s_gate, const uint8_t* wq_up, const uint8_t* s_up, const uint8_t* wq_down,
                                       const uint8_t* s_down, uint16_t* out, int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes,
                                       void* stream) {
  const moe::FewWeights W[3] = {{wq_gate, s_gate}, {wq_up, s_up}, {wq_down, s_down}};
  return moe::few_forward<true>(shape, x, w_router, W, out, topk_idx, topk_w, ws, ws_bytes, stream);
}
