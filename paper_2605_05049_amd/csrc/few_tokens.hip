// A whole MoE layer for a few tokens (at most 64): logits = x W_r^T, top-k gate, the chosen experts' SwiGLU FFNs and the weighted sum,
//     out[t] = sum_j w[t, j] (silu(x_t Wg) * (x_t Wu)) Wd     over the experts of token t,
// on weights in bf16 (W_gate, W_up [E', d, f], W_down [E', f, d]) or microscaled 4-bit floating point ([E', f, d / 2], [E', d, f / 2]).
//
// What bounds it: the weights of the experts that some token chose are read once and multiply a handful of rows, so the time is that of
// streaming them.  The rows are not permuted into buffers: an expert's tokens are columns 0 .. 15 (of one or two groups) of an MFMA whose
// other operand is the weights.  The weights go from memory straight into registers: of bf16 weights a lane holds 2 or 4 columns of 8 k-rows, and
// turns them with byte permutes into the MFMA's operand, 8 k of one column; of 4-bit weights it holds 32 k of one column (a block, one scale) and
// widens them to bf16, exactly.  The hidden activation stays in fp32 in effect: it is kept as a bf16 head and a bf16 remainder, both of
// which multiply W_down; the partial sums over K and the experts are added in fp32, in a fixed order.
//
// Launches: logits; gate (with at most 16 tokens every block of the next one makes it for itself, and the logits of a small router); G and U by columns
// and parts of d; with more than 16 tokens H; H W_down by columns and parts of d_ffn; the weighted sum.  Measured, 8 experts of 4096 x 14336, top 2:
// 1 token 119 us in bf16 (5.9 TB/s; a large read reaches 6.2) and 49 us in 4 bits (3.8 TB/s); 16 tokens 431 (6.5 TB/s) and 177 us; 64 tokens 473 and
// 224 us.
#include "mxfp4.h"
#include "route.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace moe {

namespace {

constexpr int kFewTokens = MOE_FEW_TOKENS_MAX;
constexpr int kFewSlots = 4096;       // T * K' at most
constexpr int kFewWaves = 8;          // wavefronts of a block
constexpr int kFewFusedSlots = 512, kFewFusedExperts = 256;   // at most, where every block makes the gate for itself
// Bytes of router weights at most, where it makes the logits too.  Measured, the layer with the logits made so and by a launch of their own: 8 KB (8 experts
// of 512 x 1024), 1 and 16 tokens, 16.5 and 20.0 us to 17.8 and 21.4; 28 KB (13 of 1088 x 1984) 21.7 and 43.0 to 23.0 and 44.0, in 4 bits 18.1 and 34.8 to 19.3
// and 34.8; 64 KB (32 of 1024 x 1024) 20.7 and 58 to 19.3 and 43.
constexpr size_t kFewFusedRouter = 16 * 1024;
constexpr int kFewGroup = 16;         // tokens of an MFMA
constexpr int kFewTurn = 2 * kFewGroup;   // rows at most that go through the weights together

// The experts that have tokens, in expert order (from few_gate_kernel in turns of kFewTurn slots at most), and the slots of each.
struct FewSched {
  int32_t n_live, pad[3];
  int4 live[kMaxExperts + kFewSlots / kFewTurn];   // expert, the first entry in slots, how many
  int32_t slots[kFewSlots];   // t * K' + j
};

struct FewWeights { const uint8_t* w; const uint8_t* scales; };   // bf16 weights have no scales
struct FewArgs {
  int T, d, f, E, Es, k, Kp, renorm;
  int parts, h_parts;            // of d_ffn in the down projection; of d in the other two, at most 16 tokens
  int fused_gate, fused_router;  // the gate, and the logits, are made by few_gate_up_kernel
  const uint16_t* x; const uint16_t* w_router;
  float* logits; int32_t* topk_idx; float* topk_w; FewSched* sched;
  FewWeights gate, up, down;
  uint16_t* h; size_t h_lo;      // [N, f] bf16 heads, the remainders h_lo elements further
  float* partial;                // [N, parts, d]
  float* h_partial;              // [N, h_parts, 2, f]
  uint16_t* out;
};

__device__ __forceinline__ int few_scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }   // the same in all lanes: the compiler is told so

// ---- logits and gate ---------------------------------------------------------------------------------------------------------------

// Logits of 16 experts x 16 tokens by one block: K split over the wavefronts, whose sums are added in order.
typedef float FewLogitParts[kFewWaves][16][17];
__device__ __forceinline__ void few_logits(const FewArgs& A, int e0, int t0, FewLogitParts& part, float* logits) {
  const int lane = threadIdx.x & 63, wave = few_scalar(threadIdx.x >> 6), n = lane & 15, q = lane >> 4;
  const uint16_t* const wr = A.w_router + (size_t)min(e0 + n, A.E - 1) * A.d + 8 * q;
  const uint16_t* const xr = A.x + (size_t)min(t0 + n, A.T - 1) * A.d + 8 * q;
  const int steps = A.d / 32, per = (steps + kFewWaves - 1) / kFewWaves;
  mx_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int end = min(steps, (wave + 1) * per);
  // Eight steps requested at once; past the end the last one, not multiplied.  (The guard is a scalar branch: a product ignores the lane mask.)
  for (int s0 = wave * per; s0 < end; s0 += 8) {
    mx_bf16x8 w[8], x[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const int s = min(s0 + u, end - 1);
      w[u] = *reinterpret_cast<const mx_bf16x8*>(wr + s * 32);
      x[u] = *reinterpret_cast<const mx_bf16x8*>(xr + s * 32);
    }
#pragma unroll
    for (int u = 0; u < 8; u++) asm volatile("" : "+v"(w[u]), "+v"(x[u]));   // (or the compiler moves a step's loads behind its guard)
#pragma unroll
    for (int u = 0; u < 8; u++)
      if (s0 + u < end) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[u], x[u], acc, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 4; i++) part[wave][n][4 * q + i] = acc[i];   // [token][expert]
  __syncthreads();
  if (threadIdx.x < 256) {
    const int t = threadIdx.x >> 4, e = threadIdx.x & 15;
    float sum = 0.f;
#pragma unroll
    for (int p = 0; p < kFewWaves; p++) sum += part[p][t][e];
    if (t0 + t < A.T && e0 + e < A.E) logits[(size_t)(t0 + t) * A.E + e0 + e] = sum;
  }
}
__global__ __launch_bounds__(kFewWaves * kWave) void few_router_kernel(const FewArgs A) {
  __shared__ FewLogitParts part;
  few_logits(A, blockIdx.x * 16, blockIdx.y * 16, part, A.logits);
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
      const int turns = (c + kFewTurn - 1) / kFewTurn, incl = wave_prefix_sum(c), l_incl = wave_prefix_sum(turns);
      if (e < Et) { first[e] = slots + incl - c; live_before[e] = live + l_incl - turns; }
      slots += __builtin_amdgcn_readlane(incl, kWave - 1);
      live += __builtin_amdgcn_readlane(l_incl, kWave - 1);
    }
    if (lane == 0) A.sched->n_live = live;
  }
  __syncthreads();
  if ((int)threadIdx.x < Et)
    for (int r = 0; r < count[threadIdx.x]; r += kFewTurn)
      A.sched->live[live_before[threadIdx.x] + r / kFewTurn] = make_int4(threadIdx.x, first[threadIdx.x] + r, min(kFewTurn, count[threadIdx.x] - r), 0);
  __syncthreads();
  // (the order of an expert's slots follows no rule and changes no result: every slot's sums are its own)
  for (int s = threadIdx.x; s < N; s += 1024) A.sched->slots[atomicAdd(&first[expert_of(s)], 1)] = s;
}

// ---- what a lane holds of the weights --------------------------------------------------------------------------------------------------

// FR frags of 16 columns: column FR * m + a of the tile is row m of frag a.  A step is 32 k of bf16 or 256 k of 4-bit weights (the last one may be
// cut short: past the end the rows are zero).
template <bool MX, int FR> struct FewTile;
// 4-bit weights: steps of a chunk at most; bytes of a column's scales in LDS.
constexpr int few_scale_steps(int groups) { return groups > 1 ? 4 : 8; }
constexpr int few_scale_pitch(int groups) { return 8 * few_scale_steps(groups) + 8; }

// Global memory by a scalar address: the compiler is told that it is the same in all lanes.
typedef const uint8_t __attribute__((address_space(1)))* FewBase;
__device__ __forceinline__ FewBase few_base(const uint8_t* p) {
  const unsigned long long v = (unsigned long long)p;
  return (FewBase)((unsigned long long)(unsigned)few_scalar((int)(v >> 32)) << 32 | (unsigned)few_scalar((int)v));
}
// From a scalar base and 32 bits of the lane's own (left to itself the compiler keeps a 64-bit address per lane and load, 48 registers in all).
// ONCE: nothing else of the lines is read, they need not stay in the caches (a row of 64 bf16 columns is a line of 128 bytes).  One token, 2 of 8 experts of
// 4096 x 14336 in bf16: 149 -> 134 us; of 4-bit weights, whose lines are read in halves, 50 -> 59.
template <class T, bool ONCE>
__device__ __forceinline__ T few_load(FewBase base, unsigned off) {
  asm("" : "+s"(base));
  const auto p = (const T __attribute__((address_space(1)))*)(base + off);
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int FR> struct FewTile<false, FR> {
  static constexpr int KS = 1;   // MFMAs of 32 k per step and frag
  typedef uint32_t word __attribute__((ext_vector_type(FR / 2)));   // the lane's FR columns of a k-row
  struct Stage { word w[8]; };
  FewBase base;
  unsigned lane_off;
  size_t row;
  __device__ __forceinline__ FewTile(const FewWeights& W, int expert, int K, int C, int col0, int lane) {
    base = few_base(W.w + ((size_t)expert * K * C + col0) * 2);
    row = (size_t)C * 2;
    lane_off = ((unsigned)(8 * (lane >> 4)) * (unsigned)C + FR * (lane & 15)) * 2;
  }
  __device__ __forceinline__ void load(Stage& s, int step) const {
    step = few_scalar(step);
    FewBase p = base + (size_t)step * 32 * row;   // (scalar: a load's address is this and 32 bits of the lane's own)
#pragma unroll
    for (int i = 0; i < 8; i++, p += row) s.w[i] = few_load<word, FR == 4>(p, lane_off);
  }
  struct Codes {};
  template <int GROUPS> __device__ __forceinline__ void bring_scales(char*, int, int, int) const {}
  template <int GROUPS> __device__ __forceinline__ Codes codes(const char*, int) const { return {}; }
  // frag a: 8 k of column a, from the halves of 8 words
  __device__ __forceinline__ mx_bf16x8 frag(const Stage& s, Codes, int a, int) const {
    union { unsigned p[4]; mx_bf16x8 v; } u;
#pragma unroll
    for (int p = 0; p < 4; p++) u.p[p] = __builtin_amdgcn_perm(s.w[2 * p + 1][a / 2], s.w[2 * p][a / 2], a & 1 ? 0x07060302u : 0x05040100u);
    return u.v;
  }
};

template <int FR> struct FewTile<true, FR> {
  static constexpr int KS = 8;
  typedef uint32_t quad __attribute__((ext_vector_type(4)));   // a block of 32 k
  struct Stage { quad w[2][FR]; };             // blocks q and 4 + q of the step's eight: whole lines of 128 bytes
  FewBase base, sbase;                         // of column 0
  unsigned lane_off;                           // this lane's first column, block q
  int kb, q, m;
  __device__ __forceinline__ FewTile(const FewWeights& W, int expert, int K, int C, int col0, int lane) {
    kb = K / kMxBlock;
    q = lane >> 4;
    m = lane & 15;
    const size_t row = (size_t)expert * C + col0;
    base = few_base(W.w + row * (kb * 16));
    sbase = few_base(W.scales + row * kb);
    lane_off = ((unsigned)(FR * m) * (unsigned)kb + q) * 16;
  }
  __device__ __forceinline__ void load(Stage& s, int step) const {
    step = few_scalar(step);
    const int b0 = min(8 * step, kb - 1 - q), b1 = min(8 * step + 4, kb - 1 - q);   // (a block past the end: the last one)
#pragma unroll
    for (int a = 0; a < FR; a++) {
      const FewBase p = base + (size_t)a * (kb * 16);
      s.w[0][a] = few_load<quad, false>(p, lane_off + b0 * 16);
      s.w[1][a] = few_load<quad, false>(p, lane_off + b1 * 16);
    }
  }
  // The scales of `steps` (at most few_scale_steps) steps of the wavefront's columns into LDS, 8 bytes a step; 1 past the end of K, where the rows are zero.
  // (Read by steps from memory, a line of a column's scales was fetched again for each: 4096 x 14336, 8 experts, 16 rows: 220 against 170 us.)
  template <int GROUPS>
  __device__ __forceinline__ void bring_scales(char* to, int step0, int steps, int lane) const {
    constexpr int MOST = few_scale_steps(GROUPS);
    typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(2)));   // (kb is even)
#pragma unroll
    for (int i = 0; i < 16 * FR * MOST / kWave; i++) {
      const int c = i * (kWave / MOST) + lane / MOST, st = lane % MOST, b = 8 * (step0 + st);
      if (st < steps) {
        unsigned long long v = ~0ull / 255 * 127;
        if (kb >= 8) {
          const int at = min(b, kb - 8);
          const pair w = few_load<pair, false>(sbase, (unsigned)c * (unsigned)kb + at);
          const int past = 8 * (b - at);   // bits that are of blocks before b
          const unsigned long long all = (unsigned long long)w[1] << 32 | w[0];
          v = past ? all >> past | v << (64 - past) : all;
        } else {
          for (int k = 0; k < kb; k++) v = (v & ~(255ull << (8 * k))) | (unsigned long long)few_load<uint8_t, false>(sbase, (unsigned)c * (unsigned)kb + k) << (8 * k);
        }
        *reinterpret_cast<unsigned long long*>(to + c * few_scale_pitch(GROUPS) + 8 * st) = v;
      }
    }
  }
  struct Codes { float scale[2][FR]; };   // of the stage's blocks
  template <int GROUPS>
  __device__ __forceinline__ Codes codes(const char* at, int step) const {   // step: from the chunk's first
    Codes c;
#pragma unroll
    for (int a = 0; a < FR; a++) {
      const uint2 v = *reinterpret_cast<const uint2*>(at + (FR * m + a) * few_scale_pitch(GROUPS) + 8 * step);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const unsigned code = ((h ? v.y : v.x) >> (8 * q)) & 255u;
        c.scale[h][a] = __uint_as_float(code == 255u ? 0x7fc00000u : code << 23);
      }
    }
    return c;
  }
  __device__ __forceinline__ mx_bf16x8 frag(const Stage& s, const Codes& c, int a, int ks) const {   // ks: part ks % 4 (of 8 k) of block 4 (ks / 4) + q
    const float scale = c.scale[ks >> 2][a];
    const unsigned v = s.w[ks >> 2][a][ks & 3];
    union { mx_bf16x2 p[4]; mx_bf16x8 v; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3);
    return u.v;
  }
};

// Live expert i of the schedule, in scalar registers: expert, its first entry in slots, its slots.
__device__ __forceinline__ int4 few_live(const FewArgs& A, int i) {
  const int4 v = A.sched->live[i];
  return make_int4(__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), 0);
}

constexpr int few_step(bool mx) { return mx ? 256 : 32; }
__device__ __host__ __forceinline__ int few_steps(bool mx, int K) { return (K + few_step(mx) - 1) / few_step(mx); }
// In LDS: the lane's 8 k for MFMA ks of a step, from the step's first k on, in units of 8 k.
template <bool MX>
__device__ __forceinline__ int few_piece(int q, int ks) { return MX ? 16 * (ks >> 2) + 4 * q + (ks & 3) : q; }

// h and what its bf16 head leaves: nothing where the head is an infinity (h - head would be NaN, or an infinity of the other sign) or NaN.
__device__ __forceinline__ void few_swiglu(float g, float u, float& h, float& lo) {
  h = g / (1.0f + __expf(-g)) * u;
  const float head = bf16_to_f32(f32_to_bf16(h));
  lo = fabsf(head) < __builtin_inff() ? h - head : 0.f;
}

// A lane's sums of one token, 4 FR consecutive columns.
template <int FR>
__device__ __forceinline__ void few_put(float* dst, const mx_f32x4 (&acc)[FR]) {
  typedef float vec __attribute__((ext_vector_type(FR)));
#pragma unroll
  for (int i = 0; i < 4; i++) {
    vec v;
#pragma unroll
    for (int a = 0; a < FR; a++) v[a] = acc[a][i];
    *reinterpret_cast<vec*>(dst + FR * i) = v;
  }
}

// ---- the experts' products ------------------------------------------------------------------------------------------------------------------
//
// The wavefronts of a block have columns next to each other, and the contraction is shared between blocks, whose partial sums the next launch adds.  A
// step of bf16 weights takes 32 k-rows that lie 2 C bytes apart: if each wavefront of a block goes through rows of its own, a CU has 8 times as many
// pages in use at once (reading two pairs of 4096 x 14336 alone, 5.0 against 6.1 TB/s).  A launch that goes on from the logits to the end by itself
// was slower: its wavefronts take their work from counters and wait for each other through memory, and 512 blocks that begin with an atomic each have
// their answers after 25 us.

// The gate of the call for one block, in LDS; the experts that have slots.
struct FewGate {
  int idx[kFewFusedSlots], list[kFewFusedSlots];   // the slots' experts; the slots of the expert at hand
  float weight[kFewFusedSlots];
  unsigned words[kFewFusedExperts / 32];
  int found[2];
};
// Live expert blockIdx.y of the call: its id and its slots; count = 0: there is none.  With the gate fused, every block makes it from the logits for
// itself (a launch and the wait for it cost more); block (0, 0) leaves ids and weights in memory, block (0, `last_row`) the schedule.
struct FewExpert { int id, count; const int* slots; };
template <bool FUSED>
__device__ __forceinline__ FewExpert few_expert(const FewArgs& A, FewGate& S, char* scratch, int last_row) {
  FewExpert X;
  if (!FUSED || !A.fused_gate) {
    const int n_live = A.sched->n_live;
    const bool live = (int)blockIdx.y < n_live;
    const int4 v = few_live(A, live ? n_live - 1 - blockIdx.y : 0);
    X.id = v.x;
    X.count = live ? v.z : 0;
    X.slots = A.sched->slots + v.y;
    return X;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = few_scalar(tid >> 6), N = A.T * A.Kp, Et = A.E + A.Es;
  if (tid < kFewFusedExperts / 32) S.words[tid] = 0;
  if (A.w_router) {
    const float* logits = A.logits;
    if (A.fused_router) {
      float* const own = reinterpret_cast<float*>(scratch + sizeof(FewLogitParts));
      for (int e0 = 0; e0 < A.E; e0 += 16) {
        if (e0 > 0) __syncthreads();
        few_logits(A, e0, 0, *reinterpret_cast<FewLogitParts*>(scratch), own);
      }
      __syncthreads();
      logits = own;
    }
    for (int t = wave; t < A.T; t += kFewWaves) {
      if (A.E <= kWave) route_token<kWave, 1>(logits + (size_t)t * A.E, t, lane, S.idx, S.weight, nullptr, A.E, A.k, A.Es, A.renorm);
      else route_token<kWave, 4>(logits + (size_t)t * A.E, t, lane, S.idx, S.weight, nullptr, A.E, A.k, A.Es, A.renorm);
    }
  } else {
    for (int s = tid; s < N; s += kFewWaves * kWave) S.idx[s] = min(max(A.topk_idx[s], 0), Et - 1);
  }
  __syncthreads();
  for (int s = tid; s < N; s += kFewWaves * kWave) {
    atomicOr(&S.words[S.idx[s] >> 5], 1u << (S.idx[s] & 31));
    if (blockIdx.x == 0 && blockIdx.y == 0 && A.w_router) { A.topk_idx[s] = S.idx[s]; A.topk_w[s] = S.weight[s]; }
  }
  __syncthreads();
  if (wave == 0) {
    // 4 ids per lane
    const unsigned bits = (S.words[lane >> 3] >> (4 * (lane & 7))) & 15u;
    const int n = __popc(bits), incl = wave_prefix_sum(n), total = __builtin_amdgcn_readlane(incl, kWave - 1);
    auto slots_of = [&](int e, int32_t* to) __attribute__((always_inline)) {   // the slots of expert e, in order; how many
      int count = 0;
      for (int s0 = 0; s0 < N; s0 += kWave) {
        const bool mine = s0 + lane < N && S.idx[s0 + lane] == e;
        const unsigned long long who = __ballot(mine);
        if (mine) to[count + __popcll(who & ((1ull << lane) - 1))] = s0 + lane;
        count += __popcll(who);
      }
      return count;
    };
    int expert = -1, count = 0;
    const unsigned long long past = __ballot(incl > (int)blockIdx.y);
    if (past && (int)blockIdx.y != last_row) {
      const int l = __builtin_ctzll(past);
      unsigned b = __builtin_amdgcn_readlane(bits, l);
      for (int skip = (int)blockIdx.y - __builtin_amdgcn_readlane(incl - n, l); skip > 0; skip--) b &= b - 1;
      expert = 4 * l + __builtin_ctz(b);
      count = slots_of(expert, S.list);
    }
    if (lane == 0) { S.found[0] = expert; S.found[1] = count; }
    if ((int)blockIdx.y == last_row && blockIdx.x == 0) {   // every live expert's turn
      int at = 0, i = 0;
      for (int l = 0; l < kWave; l++)
        for (unsigned b = __builtin_amdgcn_readlane(bits, l); b; b &= b - 1, i++) {
          const int e = 4 * l + __builtin_ctz(b), c = slots_of(e, A.sched->slots + at);
          if (lane == 0) A.sched->live[i] = make_int4(e, at, c, 0);
          at += c;
        }
      if (lane == 0) A.sched->n_live = total;
    }
  }
  __syncthreads();
  X.id = few_scalar(S.found[0]);
  X.count = few_scalar(S.found[1]);
  X.slots = S.list;
  return X;
}

// Rows of a product in LDS: of one turn (16 GROUPS rows of an expert at most), as many steps of k as fit.
// A block has half of a CU's LDS, 80 KB: with the gate (at most 16 tokens) or without it, and the scales.
__device__ __host__ constexpr int few_row_bytes(bool mx, int groups) { return (groups > 1 ? mx ? 66 : 79 : mx ? 54 : 72) * 1024; }
__device__ __host__ constexpr int few_scale_bytes(bool mx, int FR, int groups) { return mx ? kFewWaves * 16 * FR * few_scale_pitch(groups) : 16; }
__device__ __forceinline__ int few_row_pitch(int k) { return 2 * k + 16; }
template <bool MX, int GROUPS, bool LO>
__device__ __forceinline__ int few_chunk_steps(int n_rows) {
  const int fit = max(1, (few_row_bytes(MX, GROUPS) / ((LO ? 2 : 1) * n_rows) - 16) / (2 * few_step(MX)));
  return MX ? min(fit, few_scale_steps(GROUPS)) : fit;
}

// acc[g][a] += over `count` steps from step0 on: lane l's element i of acc[g][a] is column FR (4 (l / 16) + i) + a, row 16 g + l % 16 of `rows` (LO: with
// the remainders after all rows; rows past the last repeat it).  Between the first weights' requests and their use stands `bring`, which fills `rows`.
template <bool MX, int FR, int GROUPS, int TG, bool LO, int DEPTH, class F>
__device__ __forceinline__ void few_multiply(mx_f32x4 (&acc)[TG][FR], const FewTile<MX, FR>& W, F&& bring, const char* rows, int n_rows, int pitch, const char* scales,
                                             int step0, int count, int lane) {
  typedef FewTile<MX, FR> Tile;
  constexpr int STEP = few_step(MX);
  const int last = step0 + count - 1;
  typename Tile::Stage st[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; i++)
    if (i < count) W.load(st[i], step0 + i);
  bring();
  const char* at[TG];
#pragma unroll
  for (int g = 0; g < TG; g++) at[g] = rows + min(16 * g + (lane & 15), n_rows - 1) * pitch;
  auto consume = [&](const typename Tile::Stage& s, int i) __attribute__((always_inline)) {
    const auto codes = W.template codes<GROUPS>(scales, i);
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ks++) {
      if (ks > 0 && TG > 1) __builtin_amdgcn_sched_barrier(0);   // (or the operands of all are in registers at once)
      mx_bf16x8 v[TG], l[TG];
#pragma unroll
      for (int g = 0; g < TG; g++) {
        const char* const x = at[g] + i * (STEP * 2) + 16 * few_piece<MX>(lane >> 4, ks);
        v[g] = *reinterpret_cast<const mx_bf16x8*>(x);
        if constexpr (LO) l[g] = *reinterpret_cast<const mx_bf16x8*>(x + n_rows * pitch);
      }
#pragma unroll
      for (int a = 0; a < FR; a++) {
        const mx_bf16x8 w = W.frag(s, codes, a, ks);
#pragma unroll
        for (int g = 0; g < TG; g++) {
          acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, v[g], acc[g][a], 0, 0, 0);
          if constexpr (LO) acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, l[g], acc[g][a], 0, 0, 0);
        }
      }
    }
  };
  // (no branch in the loop: what the registers of a stage are is then fixed, and a wait is for the oldest stage alone)
  const int body = max(count - 1, 0) / DEPTH * DEPTH;
  int i = 0;
  for (; i < body; i += DEPTH) {
#pragma unroll
    for (int u = 0; u < DEPTH; u++) {
      consume(st[u], i + u);
      __builtin_amdgcn_sched_barrier(0);
      W.load(st[u], min(step0 + i + u + DEPTH, last));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int u = 0; u < DEPTH; u++) {
    if (i + u < count) {
      consume(st[u], i + u);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// Parts of K: this block's steps.
struct FewPart { int step0, steps; };
template <bool MX>
__device__ __forceinline__ FewPart few_part(int K, int part, int parts) {
  const int steps = few_steps(MX, K), per = (steps + parts - 1) / parts, step0 = min(steps, part * per);
  return {step0, min(steps, step0 + per) - step0};
}

// The sums of the rows r0 .. of an expert over one part of K, chunk by chunk.  `bring` makes sizeof(V) / 2 k of row r0 + r, from k on.
template <bool MX, int FR, int GROUPS, int TG, bool LO, int DEPTH, class V, class F>
__device__ __forceinline__ void few_turn(mx_f32x4 (&acc)[TG][FR], const FewTile<MX, FR>& W, F&& bring, char* rows, char* scales, int n_rows, int K, FewPart part,
                                         bool active, int lane) {
  constexpr int STEP = few_step(MX), THREADS = kFewWaves * kWave;
  const int fills = (part.steps - 1) / few_chunk_steps<MX, GROUPS, LO>(n_rows) + 1, per = (part.steps + fills - 1) / fills;
  const int pitch = few_row_pitch(per * STEP), pieces = per * STEP * 2 / (int)sizeof(V);
#pragma unroll
  for (int g = 0; g < TG; g++)
#pragma unroll
    for (int a = 0; a < FR; a++) acc[g][a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < part.steps; s0 += per) {
    const int step0 = part.step0 + s0, count = min(per, part.steps - s0);
    few_multiply<MX, FR, GROUPS, TG, LO, DEPTH>(acc, W, [&]() __attribute__((always_inline)) {
      __syncthreads();
      W.template bring_scales<GROUPS>(scales, step0, count, lane);
      for (int i = threadIdx.x; i < n_rows * pieces; i += THREADS) {
        const int r = i / pieces, c = i - r * pieces, k = step0 * STEP + (int)sizeof(V) / 2 * c;
        V v = {}, lo = {};   // (past the end of K)
        if (k < K) bring(r, k, v, lo);
        V* const to = reinterpret_cast<V*>(rows + r * pitch) + c;
        *to = v;
        if constexpr (LO) *reinterpret_cast<V*>(reinterpret_cast<char*>(to) + n_rows * pitch) = lo;
      }
      __syncthreads();
    }, rows, n_rows, pitch, scales, step0, active ? count : 0, lane);
  }
}

// One of `h_parts` parts of G and U of 64 FR columns of one expert: wavefronts 0, 2, 4, 6 make G, the others U, of 16 FR columns each.
template <bool MX, int FR, int GROUPS, int DEPTH>
__global__ __launch_bounds__(kFewWaves * kWave, 4) void few_gate_up_kernel(const FewArgs A) {
  constexpr int WC = 16 * FR;
  __shared__ __attribute__((aligned(16))) char rows[few_row_bytes(MX, GROUPS)];
  __shared__ __attribute__((aligned(16))) char scales[few_scale_bytes(MX, FR, GROUPS)];
  __shared__ FewGate S;
  const int lane = threadIdx.x & 63, wave = few_scalar(threadIdx.x >> 6);
  const FewExpert X = few_expert<GROUPS == 1>(A, S, rows, gridDim.y - 1);
  if (X.count == 0) return;
  const int ct = blockIdx.x / A.h_parts, part = blockIdx.x - ct * A.h_parts;
  const int col0 = ct * 4 * WC + WC * (wave >> 1);
  const bool active = col0 < A.f;   // (widths are multiples of 64: a wavefront has all its columns or none)
  const FewTile<MX, FR> W(wave & 1 ? A.up : A.gate, X.id, A.d, A.f, active ? col0 : 0, lane);
  auto turn = [&](int r0, auto tg) __attribute__((always_inline)) {
    constexpr int TG = decltype(tg)::value;
    mx_f32x4 acc[TG][FR];
    few_turn<MX, FR, GROUPS, TG, false, DEPTH, uint4>(acc, W, [&](int r, int k, uint4& v, uint4&) __attribute__((always_inline)) {
      v = *reinterpret_cast<const uint4*>(A.x + (size_t)(X.slots[r0 + r] / A.Kp) * A.d + k);
    }, rows, scales + (MX ? wave * 16 * FR * few_scale_pitch(GROUPS) : 0), min(kFewGroup * TG, X.count - r0), A.d, few_part<MX>(A.d, part, A.h_parts), active, lane);
#pragma unroll
    for (int g = 0; g < TG; g++) {
      const int row = r0 + 16 * g + (lane & 15);
      if (active && row < X.count)
        few_put(A.h_partial + (((size_t)X.slots[row] * A.h_parts + part) * 2 + (wave & 1)) * A.f + col0 + 4 * FR * (lane >> 4), acc[g]);
    }
  };
  if (GROUPS == 2 && X.count > kFewGroup) turn(0, std::integral_constant<int, GROUPS>{});
  else
    for (int r0 = 0; r0 < X.count; r0 += kFewGroup) turn(r0, std::integral_constant<int, 1>{});
}

// H = silu(G) * U of 4 columns, from the partial sums of G and U (in order): heads and remainders.
__device__ __forceinline__ void few_hidden(const FewArgs& A, int slot, int k, uint2& head, uint2& rest) {
  const float* const src = A.h_partial + (size_t)slot * A.h_parts * 2 * A.f + k;
  float4 g = make_float4(0.f, 0.f, 0.f, 0.f), u = g;
  for (int p0 = 0; p0 < A.h_parts; p0 += 4) {   // (four parts at a time: each takes the way to the L2)
    float4 pg[4], pu[4];
#pragma unroll
    for (int p = 0; p < 4; p++) {
      const float* const at = src + (size_t)min(p0 + p, A.h_parts - 1) * 2 * A.f;
      pg[p] = *reinterpret_cast<const float4*>(at);
      pu[p] = *reinterpret_cast<const float4*>(at + A.f);
    }
#pragma unroll
    for (int p = 0; p < 4; p++)
      if (p0 + p < A.h_parts) {
        g.x += pg[p].x; g.y += pg[p].y; g.z += pg[p].z; g.w += pg[p].w;
        u.x += pu[p].x; u.y += pu[p].y; u.z += pu[p].z; u.w += pu[p].w;
      }
  }
  float h[4], lo[4];
  few_swiglu(g.x, u.x, h[0], lo[0]);
  few_swiglu(g.y, u.y, h[1], lo[1]);
  few_swiglu(g.z, u.z, h[2], lo[2]);
  few_swiglu(g.w, u.w, h[3], lo[3]);
  head = make_uint2(pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]));
  rest = make_uint2(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]));
}

// H of every slot, where more than 16 tokens would have few_down_kernel's blocks make it over and over.
__global__ __launch_bounds__(256) void few_hidden_kernel(const FewArgs A) {
  const int k = 4 * (blockIdx.x * 256 + threadIdx.x);
  if (k >= A.f) return;
  uint2 head, rest;
  few_hidden(A, blockIdx.y, k, head, rest);
  uint16_t* const o = A.h + (size_t)blockIdx.y * A.f + k;
  *reinterpret_cast<uint2*>(o) = head;
  *reinterpret_cast<uint2*>(o + A.h_lo) = rest;
}

// 128 FR columns of H W_down of one expert over one of `parts` parts of d_ffn.
template <bool MX, int FR, int GROUPS, int DEPTH>
__global__ __launch_bounds__(kFewWaves * kWave, 4) void few_down_kernel(const FewArgs A) {
  constexpr int WC = 16 * FR;
  __shared__ __attribute__((aligned(16))) char rows[few_row_bytes(MX, GROUPS)];
  __shared__ __attribute__((aligned(16))) char scales[few_scale_bytes(MX, FR, GROUPS)];
  const int lane = threadIdx.x & 63, wave = few_scalar(threadIdx.x >> 6);
  const int n_live = A.sched->n_live;
  if ((int)blockIdx.y >= n_live) return;
  const int4 L = few_live(A, n_live - 1 - blockIdx.y);
  const int32_t* const slots = A.sched->slots + L.y;
  const int ct = blockIdx.x / A.parts, part = blockIdx.x - ct * A.parts;
  const int col0 = ct * 8 * WC + WC * wave;
  const bool active = col0 < A.d;
  const FewTile<MX, FR> W(A.down, L.x, A.f, A.d, active ? col0 : 0, lane);
  auto turn = [&](int r0, auto tg) __attribute__((always_inline)) {
    constexpr int TG = decltype(tg)::value;
    mx_f32x4 acc[TG][FR];
    typedef std::conditional_t<(GROUPS > 1), uint4, uint2> piece;
    few_turn<MX, FR, GROUPS, TG, true, DEPTH, piece>(acc, W, [&](int r, int k, piece& v, piece& lo) __attribute__((always_inline)) {
      const int slot = slots[r0 + r];
      if constexpr (GROUPS > 1) {
        const uint16_t* const h = A.h + (size_t)slot * A.f + k;
        v = *reinterpret_cast<const uint4*>(h);
        lo = *reinterpret_cast<const uint4*>(h + A.h_lo);
      } else {
        few_hidden(A, slot, k, v, lo);
      }
    }, rows, scales + (MX ? wave * 16 * FR * few_scale_pitch(GROUPS) : 0), min(kFewGroup * TG, L.z - r0), A.f, few_part<MX>(A.f, part, A.parts), active, lane);
#pragma unroll
    for (int g = 0; g < TG; g++) {
      const int row = r0 + 16 * g + (lane & 15);
      if (active && row < L.z) few_put(A.partial + ((size_t)slots[row] * A.parts + part) * A.d + col0 + 4 * FR * (lane >> 4), acc[g]);
    }
  };
  if (GROUPS == 2 && L.z > kFewGroup) turn(0, std::integral_constant<int, GROUPS>{});
  else
    for (int r0 = 0; r0 < L.z; r0 += kFewGroup) turn(r0, std::integral_constant<int, 1>{});
}

// out[t] = sum_j w[t, j] sum_parts partial, fp32, one rounding.  A block has 128 columns of a token; its wavefronts share the K' parts terms, each eight or more
// next to each other, and their sums are added in order (one alone takes the way to the L2 several times: 1 token, 2 x 32 terms, 9.8 against 4.5 us).
__global__ __launch_bounds__(kFewWaves * kWave) void few_combine_kernel(const FewArgs A) {
  __shared__ float2 part[kFewWaves][kWave];
  const int lane = threadIdx.x & 63, wave = few_scalar(threadIdx.x >> 6), t = blockIdx.y, c = blockIdx.x * 128 + 2 * lane;
  const int waves = blockDim.x / kWave, n = A.Kp * A.parts, per = (n + waves - 1) / waves, end = min(n, (wave + 1) * per);
  float2 sum = make_float2(0.f, 0.f);
  if (c < A.d) {
    const float* const src = A.partial + (size_t)t * n * A.d + c;
    for (int i0 = wave * per; i0 < end; i0 += 8) {   // (eight at a time)
      float2 v[8];
      float w[8];
#pragma unroll
      for (int u = 0; u < 8; u++) {
        const int i = min(i0 + u, end - 1);
        v[u] = *reinterpret_cast<const float2*>(src + (size_t)i * A.d);
        w[u] = A.topk_w[t * A.Kp + i / A.parts];
      }
#pragma unroll
      for (int u = 0; u < 8; u++)
        if (i0 + u < end) { sum.x += w[u] * v[u].x; sum.y += w[u] * v[u].y; }
    }
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || c >= A.d) return;
  for (int p = 1; p < waves; p++) { sum.x += part[p][lane].x; sum.y += part[p][lane].y; }
  *reinterpret_cast<uint32_t*>(A.out + (size_t)t * A.d + c) = pack_bf16(sum.x, sum.y);
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

// Experts that can have tokens.
int few_live_bound(const Dims& D) { return (int)std::min((long long)D.Et, D.N); }

// How a problem is cut.
struct FewPlan {
  bool turns;             // of 32 rows
  int frags;              // of a wavefront's columns
  int parts, h_parts;
};
FewPlan few_plan(const Dims& D, bool mx) {
  FewPlan P = {false, 2, 1, 1};
  if (D.N == 0) return P;   // (no token: nothing is cut, and the blocks below are a divisor)
  // experts with tokens, if the tokens choose evenly
  const double live = std::min((double)few_live_bound(D), D.Es + D.E * -expm1(D.T * log1p(-(double)D.k / (D.E + 1e-9))));
  const long long step = few_step(mx);
  auto divide = [](long long a, long long b) { return (a + b - 1) / b; };
  P.turns = D.T > kFewGroup;
  // Of bf16 weights a wavefront's 64 columns are whole lines, 32 make twice as many blocks.  Measured, 64 and 32: 8 experts of 4096 x 14336, 1 and 16
  // tokens, 118 and 431 us to 151 and 563; 66 of 2048 x 1408, 4 and 16 tokens, 90 and 171 to 104 and 187, but 1 token (23M values of a matrix
  // read) 44 to 38; 14 of 1088 x 1984, 16 tokens (30M), 55 to 48.
  P.frags = mx || live * D.d * D.f < 48e6 ? 2 : 4;
  // Parts: two blocks for each of 256 CUs, or one and a half where that is all that fits in one go, and none of fewer than `least` steps (a block's start
  // costs as much as some steps).  One part of d to three, 8 experts of 4096 x 14336, 443 blocks: 431 us to 464; 1 token, 112 blocks, one part to
  // four: 156 to 120.
  auto cut = [&](int K, int cols, int C, int at_least, int least) {
    const double blocks = live * divide(C, cols);
    const long long steps = divide(K, step), want = std::max((long long)at_least, std::max((long long)(512 / blocks), (long long)std::ceil(400 / blocks)));
    const long long parts = std::max(1ll, std::min(want, steps / least));
    return (int)divide(steps, divide(steps, parts));   // (no part without steps)
  };
  P.h_parts = cut(D.d, 64 * P.frags, D.f, 1, mx ? 2 : 8);
  P.parts = cut(D.f, 128 * P.frags, D.d, 2, mx ? 1 : 8);   // (two at least: 66 experts of 2048 x 1408, 64 tokens, 303 us to 354)
  return P;
}

struct FewLayout { size_t logits, sched, h, partial, h_partial, total; };
FewLayout few_layout(const Dims& D) {
  FewLayout L;
  const FewPlan P = few_plan(D, false), Q = few_plan(D, true);
  size_t o = 0;
  L.sched = o; o += round_up(sizeof(FewSched), 256);
  L.logits = o; o += round_up((size_t)D.T * D.E * sizeof(float), 256);
  L.h = o; o += P.turns ? round_up((size_t)D.N * D.f * 2 * sizeof(uint16_t), 256) : 0;
  L.partial = o; o += round_up((size_t)D.N * max(P.parts, Q.parts) * D.d * sizeof(float), 256);
  L.h_partial = o; o += round_up((size_t)D.N * max(P.h_parts, Q.h_parts) * 2 * D.f * sizeof(float), 256);
  L.total = o;
  return L;
}

int check_few(const moe_shape* s, Dims* D) {
  const int rc = check_shape(s, D);
  if (rc != MOE_OK) return rc;
  if (D->T > kFewTokens || D->N > kFewSlots) return MOE_ERR_SHAPE;
  return MOE_OK;
}

template <bool MX>
void few_launch_experts(hipStream_t st, const FewArgs& A, const Dims& D, const FewPlan& P) {
  const unsigned live = few_live_bound(D) + (unsigned)(D.N / kFewTurn);
  auto products = [&](auto frags) {
    constexpr int FR = decltype(frags)::value, DEEP = MX ? 2 : FR == 2 ? 4 : 3, DEPTH = MX || FR == 4 ? 2 : 4;   // (what 128 registers hold)
    const dim3 block(kFewWaves * kWave), h((D.f + 64 * FR - 1) / (64 * FR) * P.h_parts, live + (A.fused_gate ? 1 : 0)),
        d((D.d + 128 * FR - 1) / (128 * FR) * P.parts, live);
    if (P.turns) {
      MOE_LAUNCH("few_gate_up", st, (few_gate_up_kernel<MX, FR, 2, DEPTH>), h, block, 0, st, A);
      MOE_LAUNCH("few_hidden", st, few_hidden_kernel, dim3((D.f / 4 + 255) / 256, (unsigned)D.N), dim3(256), 0, st, A);
      MOE_LAUNCH("few_down", st, (few_down_kernel<MX, FR, 2, DEPTH>), d, block, 0, st, A);
    } else {
      MOE_LAUNCH("few_gate_up", st, (few_gate_up_kernel<MX, FR, 1, DEEP>), h, block, 0, st, A);
      MOE_LAUNCH("few_down", st, (few_down_kernel<MX, FR, 1, DEPTH>), d, block, 0, st, A);
    }
  };
  if constexpr (MX) products(std::integral_constant<int, 2>{});
  else if (P.frags == 4) products(std::integral_constant<int, 4>{});
  else products(std::integral_constant<int, 2>{});
  MOE_LAUNCH("few_combine", st, few_combine_kernel, dim3((D.d + 127) / 128, (unsigned)D.T),
             dim3(kWave * std::min(kFewWaves, std::max(1, D.Kp * P.parts / 8))), 0, st, A);
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
  const FewPlan P = few_plan(D, MX);
  FewArgs A = {};
  A.parts = P.parts; A.h_parts = P.h_parts;
  A.T = D.T; A.d = D.d; A.f = D.f; A.E = D.E; A.Es = D.Es; A.k = D.k; A.Kp = D.Kp; A.renorm = D.renorm;
  A.fused_gate = !P.turns && D.Et <= kFewFusedExperts && D.N <= kFewFusedSlots;
  A.fused_router = A.fused_gate && (size_t)D.E * D.d * 2 <= kFewFusedRouter;
  A.x = x; A.w_router = w_router; A.topk_idx = topk_idx; A.topk_w = topk_w; A.out = out;
  A.gate = W[0]; A.up = W[1]; A.down = W[2];
  A.logits = reinterpret_cast<float*>(wsb + L.logits);
  A.sched = reinterpret_cast<FewSched*>(wsb + L.sched);
  A.h = reinterpret_cast<uint16_t*>(wsb + L.h);
  A.h_lo = (size_t)D.N * D.f;
  A.partial = reinterpret_cast<float*>(wsb + L.partial);
  A.h_partial = reinterpret_cast<float*>(wsb + L.h_partial);
  hipStream_t st = (hipStream_t)stream;
  if (w_router && !A.fused_router)
    MOE_LAUNCH("few_router", st, few_router_kernel, dim3((D.E + 15) / 16, (D.T + 15) / 16), dim3(kFewWaves * kWave), 0, st, A);
  if (!A.fused_gate) {
    if (D.E <= 64) MOE_LAUNCH("few_gate", st, few_gate_kernel<1>, dim3(1), dim3(1024), 0, st, A);
    else if (D.E <= 256) MOE_LAUNCH("few_gate", st, few_gate_kernel<4>, dim3(1), dim3(1024), 0, st, A);
    else MOE_LAUNCH("few_gate", st, few_gate_kernel<16>, dim3(1), dim3(1024), 0, st, A);
  }
  few_launch_experts<MX>(st, A, D, P);
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
