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
constexpr int kFewSlots = 4096;       // T * K' at most
constexpr int kFewWaves = 8;          // wavefronts of a block that share a contraction
constexpr int kFewFusedSlots = 512, kFewFusedExperts = 256;   // at most, where every block makes the gate for itself
constexpr int kFewGroup = 16;         // tokens of an MFMA
constexpr int kFewBlocks = 512;       // two per CU

// The experts that have tokens, in expert order, and the slots of each.
struct FewSched {
  int32_t n_live, pad[3];
  int4 live[kMaxExperts];     // expert, its first entry in slots, its slots
  int32_t slots[kFewSlots];   // t * K' + j
};

// Cleared by the launch before the one that uses them.  Counters that many blocks use lie in lines of their own.
constexpr int kFewLists = 64;
struct FewLine { int32_t n, pad[31]; };
struct FewCounters {
  FewLine taken[2][kFewLists];    // tiles of H, tiles of W_down: taken of each list
  FewLine ready[kMaxExperts];     // per live expert: tiles of H that are there
  int32_t arrivals[1];            // per column tile of the down projection: parts that are there (d / 32 at most)
};
inline size_t few_counters_bytes(int d) { return sizeof(FewCounters) + (size_t)(d / 32) * sizeof(int32_t); }

struct FewWeights { const uint8_t* w; const uint8_t* scales; };   // bf16 weights have no scales
struct FewArgs {
  int T, d, f, E, Es, k, Kp, renorm, parts;   // parts of d_ffn in the down projection
  int fused_gate;                // the gate is made by few_layer_kernel
  const uint16_t* x; const uint16_t* w_router;
  float* logits; int32_t* topk_idx; float* topk_w; FewSched* sched;
  FewCounters* counters;
  FewWeights gate, up, down;
  uint16_t* h; size_t h_lo;      // [N, f] bf16 heads, the remainders h_lo elements further
  float* partial;                // [N, parts, d]
  uint16_t* out;
};

// ---- logits and gate ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void few_clear(const FewArgs& A) {
  int32_t* const lists = &A.counters->taken[0][0].n;
  for (int i = threadIdx.x; i < 2 * kFewLists; i += blockDim.x) lists[32 * i] = 0;
  for (int i = threadIdx.x; i < A.E + A.Es; i += blockDim.x) A.counters->ready[i].n = 0;
  for (int i = threadIdx.x; i < A.d / 32; i += blockDim.x) A.counters->arrivals[i] = 0;
}
__global__ __launch_bounds__(256) void few_clear_kernel(const FewArgs A) { few_clear(A); }

// 16 experts x 16 tokens per block, K split over the wavefronts, whose sums are added in order.
__global__ __launch_bounds__(kFewWaves * kWave) void few_router_kernel(const FewArgs A) {
  __shared__ float part[kFewWaves][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
  const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  if (blockIdx.x == 0 && blockIdx.y == 0) few_clear(A);
  const uint16_t* const wr = A.w_router + (size_t)min(e0 + n, A.E - 1) * A.d + 8 * q;
  const uint16_t* const xr = A.x + (size_t)min(t0 + n, A.T - 1) * A.d + 8 * q;
  const int steps = A.d / 32, per = (steps + kFewWaves - 1) / kFewWaves;
  mx_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int end = min(steps, (wave + 1) * per);
  for (int s0 = wave * per; s0 < end; s0 += 8) {   // (eight steps requested at once; past the end the last one, not multiplied)
    mx_bf16x8 w[8], x[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const int s = min(s0 + u, end - 1);
      w[u] = *reinterpret_cast<const mx_bf16x8*>(wr + s * 32);
      x[u] = *reinterpret_cast<const mx_bf16x8*>(xr + s * 32);
    }
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
    if (t0 + t < A.T && e0 + e < A.E) A.logits[(size_t)(t0 + t) * A.E + e0 + e] = sum;
  }
}

// One block: the gate of every token (unless the caller brought it), then the experts that have tokens and the slots of each.
template <int PER>
__global__ __launch_bounds__(1024) void few_gate_kernel(const FewArgs A) {
  __shared__ int count[kMaxExperts], first[kMaxExperts], live_before[kMaxExperts];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int Et = A.E + A.Es, N = A.T * A.Kp;
  if (!A.w_router) few_clear(A);
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

// ---- what a lane holds of the weights --------------------------------------------------------------------------------------------------

// FR frags of 16 columns: column FR * m + a of the tile is row m of frag a.  A step is 32 k of bf16 or 128 k of 4-bit weights (the last one may be
// cut short: its codes are zero past the end).
template <bool MX, int FR> struct FewTile;

// From a scalar base and 32 bits of the lane's own (left to itself the compiler keeps a 64-bit address per lane and load, 48 registers in all).
template <class T>
__device__ __forceinline__ T few_load(const uint8_t* base, unsigned off) {
  asm("" : "+s"(base));
  return *reinterpret_cast<const T*>(base + off);
}

template <int FR> struct FewTile<false, FR> {
  static constexpr int KS = 1;   // MFMAs of 32 k per step and frag
  typedef uint32_t word __attribute__((ext_vector_type(FR / 2)));   // the lane's FR columns of a k-row
  struct Stage { word w[8]; };
  const uint8_t* base;
  unsigned lane_off;
  size_t row;
  __device__ __forceinline__ FewTile(const FewWeights& W, int expert, int K, int C, int col0, int lane) {
    base = W.w + ((size_t)expert * K * C + col0) * 2;
    row = (size_t)C * 2;
    lane_off = ((unsigned)(8 * (lane >> 4)) * (unsigned)C + FR * (lane & 15)) * 2;
  }
  __device__ __forceinline__ void load(Stage& s, int step) const {
    const uint8_t* p = base + (size_t)step * 32 * row;   // (scalar: a load's address is this and 32 bits of the lane's own)
#pragma unroll
    for (int i = 0; i < 8; i++, p += row) s.w[i] = few_load<word>(p, lane_off);
  }
  __device__ __forceinline__ void end(Stage&, int) const {}
  // frag a: 8 k of column a, from the halves of 8 words
  __device__ __forceinline__ mx_bf16x8 frag(const Stage& s, int a, int) const {
    union { unsigned p[4]; mx_bf16x8 v; } u;
#pragma unroll
    for (int p = 0; p < 4; p++) u.p[p] = __builtin_amdgcn_perm(s.w[2 * p + 1][a / 2], s.w[2 * p][a / 2], a & 1 ? 0x07060302u : 0x05040100u);
    return u.v;
  }
};

template <int FR> struct FewTile<true, FR> {
  static constexpr int KS = 4;
  struct Stage { uint4 w[FR]; unsigned s[FR]; };
  const uint8_t* base; const uint8_t* sbase;   // of column 0
  unsigned lane_off, lane_soff;                // this lane's first column, block q
  int kb, q;
  __device__ __forceinline__ FewTile(const FewWeights& W, int expert, int K, int C, int col0, int lane) {
    kb = K / kMxBlock;
    q = lane >> 4;
    const size_t row = (size_t)expert * C + col0;
    base = W.w + row * (kb * 16);
    sbase = W.scales + row * kb;
    lane_soff = (unsigned)(FR * (lane & 15)) * (unsigned)kb + q;
    lane_off = lane_soff * 16;
  }
  __device__ __forceinline__ void load(Stage& s, int step) const {
    const int b = min(4 * step, kb - 1 - q);   // (a block past the end: the last one)
#pragma unroll
    for (int a = 0; a < FR; a++) {
      s.w[a] = few_load<uint4>(base + (size_t)a * (kb * 16), lane_off + b * 16);
      s.s[a] = few_load<uint8_t>(sbase + (size_t)a * kb, lane_soff + b);
    }
  }
  __device__ __forceinline__ mx_bf16x8 frag(const Stage& s, int a, int ks) const {
    const float scale = __uint_as_float(s.s[a] == 255u ? 0x7fc00000u : s.s[a] << 23);
    const unsigned v = ks == 0 ? s.w[a].x : ks == 1 ? s.w[a].y : ks == 2 ? s.w[a].z : s.w[a].w;
    union { mx_bf16x2 p[4]; mx_bf16x8 v; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3);
    return u.v;
  }
  // the last step of K: blocks past the end become zeros
  __device__ __forceinline__ void end(Stage& s, int step) const {
    if (4 * step + q >= kb) {
#pragma unroll
      for (int a = 0; a < FR; a++) { s.w[a] = make_uint4(0, 0, 0, 0); s.s[a] = 127; }
    }
  }
};

// Live expert i of the schedule, in scalar registers: expert, its first entry in slots, its slots.
__device__ __forceinline__ int4 few_live(const FewArgs& A, int i) {
  const int4 v = A.sched->live[i];
  return make_int4(__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), 0);
}

__device__ __forceinline__ int few_steps(bool mx, int K) { return mx ? (K / 32 + 3) / 4 : K / 32; }

__device__ __forceinline__ void few_swiglu(float g, float u, float& h, float& lo) {
  h = g / (1.0f + __expf(-g)) * u;
  lo = h - bf16_to_f32(f32_to_bf16(h));
}

// ---- at most 16 tokens: the wavefronts of a block share a tile's contraction ------------------------------------------------------------

// The rows of a product lie in LDS for the whole range of k that a block works on: as many rows as fit go through the weights together.
constexpr int kFewRowBytes = 64 * 1024;
constexpr int kFewRowK = 8192;   // k at most (LO: half of them): two rows fit
__device__ __forceinline__ int few_row_pitch(int k) { return 2 * k + 16; }
template <bool LO>
__device__ __forceinline__ int few_rows_at_once(int k) { return min(kFewGroup, kFewRowBytes / ((LO ? 2 : 1) * few_row_pitch(k))); }

__device__ __forceinline__ uint4 few_load_agent(const uint16_t* p) {   // 16 bytes, past this XCD's L2
  const unsigned long long* const q = reinterpret_cast<const unsigned long long*>(p);
  const unsigned long long a = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), b = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_uint4((unsigned)a, (unsigned)(a >> 32), (unsigned)b, (unsigned)(b >> 32));
}

// acc[a] += over `n_steps` steps from step0 on: lane l's element i of acc[a] is column FR (4 (l / 16) + i) + a, token l % 16 (tokens past the last
// repeat it).  row(i): element 0 of row i of X, its remainders (LO) x_lo elements further.  Wavefront `part` of PARTS takes its share of the steps;
// their weights go into registers, DEPTH - 1 steps ahead.
// Between the first requests and the rows stands `ready()`.
template <bool MX, int FR, bool LO, int DEPTH, int PARTS, class F, class G>
__device__ __forceinline__ void few_multiply(mx_f32x4 (&acc)[FR], const FewTile<MX, FR>& W, F&& row, G&& ready, size_t x_lo, int K, int n_rows,
                                             int step0, int n_steps, char* buf, int part, int tid, int lane) {
  typedef FewTile<MX, FR> Tile;
  constexpr int STEP = MX ? 128 : 32, THREADS = kFewWaves * kWave;
  const int pitch = few_row_pitch(n_steps * STEP), pieces = n_steps * STEP / 8, total = n_rows * pieces;
  const int per = (n_steps + PARTS - 1) / PARTS;
  const int first = min(n_steps, part * per), count = min(n_steps, first + per) - first, last = max(first + count - 1, 0);
  typename Tile::Stage st[DEPTH];
  // rows into LDS, zeros past the end of K; the first weights are requested while the first of them come
  struct Piece { uint4 v, w; };
  auto bring = [&](int i) __attribute__((always_inline)) {
    Piece p = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    const int r = i / pieces, k = step0 * STEP + 8 * (i - r * pieces);
    if (i < total && k < K) {
      const uint16_t* const src = row(r) + k;
      if constexpr (LO) {   // (written in this launch)
        p.v = few_load_agent(src);
        p.w = few_load_agent(src + x_lo);
      } else {
        p.v = *reinterpret_cast<const uint4*>(src);
      }
    }
    return p;
  };
  auto put = [&](int i, const Piece& p) __attribute__((always_inline)) {
    if (i >= total) return;
    const int r = i / pieces;
    char* const to = buf + r * pitch + 16 * (i - r * pieces);
    *reinterpret_cast<uint4*>(to) = p.v;
    if constexpr (LO) *reinterpret_cast<uint4*>(to + n_rows * pitch) = p.w;
  };
#pragma unroll
  for (int i = 0; i < DEPTH; i++)
    if (i < count) W.load(st[i], step0 + first + i);
  ready();
  const Piece p0 = bring(tid);
  __syncthreads();   // (what was in LDS has been read)
  put(tid, p0);
  for (int i = tid + THREADS; i < total; i += 2 * THREADS) {
    const Piece a = bring(i), b = bring(i + THREADS);
    put(i, a);
    put(i + THREADS, b);
  }
  __syncthreads();
  const char* const at = buf + min(lane & 15, n_rows - 1) * pitch + first * (STEP * 2) + (MX ? 64 : 16) * (lane >> 4);
  auto consume = [&](const typename Tile::Stage& s, int i) __attribute__((always_inline)) {
    const char* const x = at + i * (STEP * 2);
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ks++) {
      const mx_bf16x8 v = *reinterpret_cast<const mx_bf16x8*>(x + ks * 16);
      mx_bf16x8 l = v;
      if constexpr (LO) l = *reinterpret_cast<const mx_bf16x8*>(x + n_rows * pitch + ks * 16);
#pragma unroll
      for (int a = 0; a < FR; a++) {
        const mx_bf16x8 w = W.frag(s, a, ks);
        acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, v, acc[a], 0, 0, 0);
        if constexpr (LO) acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, l, acc[a], 0, 0, 0);
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
      W.load(st[u], step0 + min(first + i + u + DEPTH, last));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int u = 0; u < DEPTH; u++) {
    if (i + u < count) {
      if (i + u == count - 1) W.end(st[u], step0 + first + i + u);
      __builtin_amdgcn_sched_barrier(0);
      consume(st[u], i + u);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
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

// What blocks of one launch hand to each other (they may run on different XCDs, with an L2 each) is stored and loaded at agent scope, past those
// caches.  A block counts itself as arrived when its stores have been acknowledged.  (Ordinary stores and a device-wide fence, which writes
// the L2 back and empties it, make the down projection 3 to 8 times as long.)
__device__ __forceinline__ void few_store_agent(void* p, unsigned a, unsigned b) {
  __hip_atomic_store(static_cast<unsigned long long*>(p), (unsigned long long)b << 32 | a, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 few_load_partial(const float* p) {
  const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
// Counts this block: all that its threads have stored is then where every block sees it.  True for thread 0 of the one that completes `of`.
__device__ __forceinline__ bool few_arrive(int32_t* counter, int of) {
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wavefront's stores have been acknowledged
  __syncthreads();
  return threadIdx.x == 0 && __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
}

// The live expert `index` among the slots' experts `idx` (in LDS, N of them), its slots into `slots`; n_live: how many there are.  Ends with the
// answers in `found` ({expert, slots, n_live}), before a barrier.
__device__ __forceinline__ void few_find_live(const int* idx, int N, int index, int* slots, const unsigned* words, int* found) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x >= kWave) return;
  // 4 ids per lane
  const unsigned bits = (words[lane >> 3] >> (4 * (lane & 7))) & 15u;
  const int n = __popc(bits), incl = wave_prefix_sum(n);
  const unsigned long long past = __ballot(incl > index);
  int expert = -1, count = 0;
  if (past) {
    const int l = __builtin_ctzll(past);
    unsigned b = __builtin_amdgcn_readlane(bits, l);
    for (int skip = index - __builtin_amdgcn_readlane(incl - n, l); skip > 0; skip--) b &= b - 1;
    expert = 4 * l + __builtin_ctz(b);
    for (int s0 = 0; s0 < N; s0 += kWave) {
      const bool mine = s0 + lane < N && idx[s0 + lane] == expert;
      const unsigned long long who = __ballot(mine);
      if (mine) slots[count + __popcll(who & ((1ull << lane) - 1))] = s0 + lane;
      count += __popcll(who);
    }
  }
  if (lane == 0) { found[0] = expert; found[1] = count; found[2] = __builtin_amdgcn_readlane(incl, kWave - 1); }
}

// The whole layer from the logits on, in one launch.  Its work is a list of tiles: H = silu(x W_gate) * (x W_up) of 16 FR columns, expert after
// expert, then the parts of H W_down of 16 FR columns, expert after expert.  A block takes the next tile when it has done one, so that no CU waits at
// the end of an expert or of the first half.  The tiles are dealt to 64 lists of either kind, each with a counter (one counter for all costs 35 ns
// for every tile, one after the other); a block takes from its own list, then from those that have tiles left.  A tile of W_down waits for its
// expert's tiles of H, with its own first weights on the way, and no block comes to one before all tiles of H have been taken: by blocks that are
// running, whatever else is on the GPU, so every wait ends.  The last part of a column tile of W_down adds the parts and experts.
//
// Of the pair wavefronts 0, 2, 4, 6 make G, the others U, each over a quarter of d; of W_down each takes an eighth of its part of d_ffn.  With the
// gate fused, every block makes it from the logits for itself (a launch and the wait for it cost more).
template <bool MX, int FR, int DEPTH>
__global__ __launch_bounds__(kFewWaves * kWave, 4) void few_layer_kernel(const FewArgs A) {
  constexpr int COLS = 16 * FR, PITCH = COLS + 4, STEP = MX ? 128 : 32;
  __shared__ __attribute__((aligned(16))) union { char rows[kFewRowBytes]; float part[kFewWaves][kFewGroup][PITCH]; } lds;
  __shared__ int idx[kFewFusedSlots], list[kFewFusedSlots];
  __shared__ float weight[kFewFusedSlots];
  __shared__ unsigned words[kFewFusedExperts / 32];
  __shared__ int found[3], next, last;
  int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int N = A.T * A.Kp;
  const int list_id = blockIdx.x % kFewLists;
  auto take = [&](int kind, int l) __attribute__((always_inline)) {   // the next tile of list l
    return __hip_atomic_fetch_add(&A.counters->taken[kind][l].n, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) * kFewLists + l;
  };
  int h_ticket = 0, d_ticket = 0;   // (thread 0)
  if (tid == 0) { h_ticket = take(0, list_id); d_ticket = take(1, list_id); }
  const float* topk_w = A.topk_w;
  int n_live;
  if (A.fused_gate) {
    if (tid < kFewFusedExperts / 32) words[tid] = 0;
    if (A.w_router) {
      for (int t = wave; t < A.T; t += kFewWaves) {
        if (A.E <= kWave) route_token<kWave, 1>(A.logits + (size_t)t * A.E, t, lane, idx, weight, nullptr, A.E, A.k, A.Es, A.renorm);
        else route_token<kWave, 4>(A.logits + (size_t)t * A.E, t, lane, idx, weight, nullptr, A.E, A.k, A.Es, A.renorm);
      }
      topk_w = weight;
    } else {
      for (int s = tid; s < N; s += kFewWaves * kWave) idx[s] = min(max(A.topk_idx[s], 0), A.E + A.Es - 1);
    }
    __syncthreads();
    for (int s = tid; s < N; s += kFewWaves * kWave) {
      atomicOr(&words[idx[s] >> 5], 1u << (idx[s] & 31));
      if (blockIdx.x == 0 && A.w_router) { A.topk_idx[s] = idx[s]; A.topk_w[s] = weight[s]; }
    }
    __syncthreads();
    int n = 0;
    for (int i = 0; i < kFewFusedExperts / 32; i++) n += __popc(words[i]);
    n_live = __builtin_amdgcn_readfirstlane(n);
  } else {
    n_live = __builtin_amdgcn_readfirstlane(A.sched->n_live);
  }
  const int h_tiles = A.f / COLS, d_tiles = A.d / COLS, n_h = n_live * h_tiles, n_d = n_live * d_tiles * A.parts;
  const int h_steps = few_steps(MX, A.d), d_steps = few_steps(MX, A.f), per = (d_steps + A.parts - 1) / A.parts;
  int current = -1, expert = 0, count = 0;   // the live expert whose slots are at hand
  const int* slots = list;

  int kind = 0;
  while (true) {
    asm volatile("" : "+v"(tid), "+v"(lane));   // (nothing that a tile makes of them is kept in registers from one tile to the next)
    const bool down = kind == 1;
    const int n_tiles = down ? n_d : n_h;
    if (tid == 0) next = down ? d_ticket : h_ticket;
    __syncthreads();   // (and what the tile before has left in LDS has been read)
    int item = __builtin_amdgcn_readfirstlane(next);
    if (item >= n_tiles) {   // this list is empty: which are not?
      if (tid < kWave) {
        const int taken = __hip_atomic_load(&A.counters->taken[kind][tid].n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        unsigned long long left = __ballot((long long)taken * kFewLists + tid < n_tiles);
        if (tid == 0) {
          int got = -1;
          if (left) {
            const unsigned long long after = left & ~((2ull << list_id) - 1);   // (from the own one on, so that not all take from the same)
            got = take(kind, __builtin_ctzll(after ? after : left));
          }
          last = got;
        }
      }
      __syncthreads();
      item = __builtin_amdgcn_readfirstlane(last);
      if (item < 0) {
        if (down) break;
        kind = 1;
        continue;
      }
      if (item >= n_tiles) continue;
    } else if (tid == 0) {
      if (down) d_ticket = take(1, list_id);
      else h_ticket = take(0, list_id);
    }
    const int local = item, tiles = down ? d_tiles * A.parts : h_tiles;
    const int live = local / tiles, in_expert = local - live * tiles;
    if (live != current) {
      current = live;
      if (A.fused_gate) {
        few_find_live(idx, N, live, list, words, found);
        __syncthreads();
        expert = __builtin_amdgcn_readfirstlane(found[0]);
        count = __builtin_amdgcn_readfirstlane(found[1]);
      } else {
        const int4 v = few_live(A, live);
        expert = v.x;
        count = v.z;
        slots = A.sched->slots + v.y;
      }
    }
    if (!down) {
      const int col0 = in_expert * COLS;
      const FewTile<MX, FR> W(wave & 1 ? A.up : A.gate, expert, A.d, A.f, col0, lane);
      const int at_once = few_rows_at_once<false>(h_steps * STEP);
      for (int r0 = 0; r0 < count; r0 += at_once) {
        const int n_rows = min(at_once, count - r0);
        mx_f32x4 acc[FR];
#pragma unroll
        for (int a = 0; a < FR; a++) acc[a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
        few_multiply<MX, FR, false, DEPTH, 4>(acc, W, [&](int r) { return A.x + (size_t)(slots[r0 + r] / A.Kp) * A.d; }, [] {}, 0, A.d, n_rows, 0, h_steps,
                                              lds.rows, wave >> 1, tid, lane);
        __syncthreads();   // (the rows have been read)
        few_put(lds.part[wave][lane & 15] + FR * 4 * (lane >> 4), acc);
        __syncthreads();
        const int t = tid / (COLS / 4), c = 4 * (tid % (COLS / 4));   // four columns
        if (t < n_rows) {
          float v[2][4] = {};
#pragma unroll
          for (int w = 0; w < kFewWaves; w++) {
            const float4 p = *reinterpret_cast<const float4*>(&lds.part[w][t][c]);
            v[w & 1][0] += p.x; v[w & 1][1] += p.y; v[w & 1][2] += p.z; v[w & 1][3] += p.w;
          }
          float h[4], lo[4];
#pragma unroll
          for (int i = 0; i < 4; i++) few_swiglu(v[0][i], v[1][i], h[i], lo[i]);
          uint16_t* const o = A.h + (size_t)slots[r0 + t] * A.f + col0 + c;
          few_store_agent(o, pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]));
          few_store_agent(o + A.h_lo, pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]));
        }
      }
      few_arrive(&A.counters->ready[live].n, h_tiles);
    } else {
      const int ct = in_expert % d_tiles, part = in_expert / d_tiles, col0 = ct * COLS;
      const int step0 = min(d_steps, part * per), step1 = min(d_steps, step0 + per);
      const FewTile<MX, FR> W(A.down, expert, A.f, A.d, col0, lane);
      const int at_once = few_rows_at_once<true>(per * STEP);
      auto ready = [&]() __attribute__((always_inline)) {
        if (tid == 0)
          while (__hip_atomic_load(&A.counters->ready[live].n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < h_tiles) __builtin_amdgcn_s_sleep(8);
        __syncthreads();
      };
      for (int r0 = 0; r0 < count; r0 += at_once) {
        const int n_rows = min(at_once, count - r0);
        mx_f32x4 acc[FR];
#pragma unroll
        for (int a = 0; a < FR; a++) acc[a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
        if (step1 > step0)
          few_multiply<MX, FR, true, DEPTH, kFewWaves>(acc, W, [&](int r) { return A.h + (size_t)slots[r0 + r] * A.f; }, ready, A.h_lo, A.f, n_rows, step0,
                                                       step1 - step0, lds.rows, wave, tid, lane);
        __syncthreads();
        few_put(lds.part[wave][lane & 15] + FR * 4 * (lane >> 4), acc);
        __syncthreads();
        const int t = tid / (COLS / 2), c = 2 * (tid % (COLS / 2));
        if (t < n_rows) {
          float2 v = make_float2(0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kFewWaves; w++) {
            const float2 p = *reinterpret_cast<const float2*>(&lds.part[w][t][c]);
            v.x += p.x;
            v.y += p.y;
          }
          few_store_agent(A.partial + ((size_t)slots[r0 + t] * A.parts + part) * A.d + col0 + c, __float_as_uint(v.x), __float_as_uint(v.y));
        }
      }
      const bool complete = few_arrive(&A.counters->arrivals[ct], n_live * A.parts);
      if (tid == 0) last = complete;
      __syncthreads();
      // out[t] = sum_j w[t, j] sum_parts partial of this column tile: slots in order, parts in order, fp32, one rounding
      if (last) {
        for (int i = tid; i < A.T * (COLS / 2); i += kFewWaves * kWave) {
          const int t = i / (COLS / 2), c = col0 + 2 * (i % (COLS / 2));
          float2 sum = make_float2(0.f, 0.f), y = sum;
          const int n = A.Kp * A.parts;
          const float* const src = A.partial + (size_t)t * n * A.d + c;
          int j = 0, p = 0;
          for (int i0 = 0; i0 < n; i0 += 8) {   // (eight at a time: each takes the way to memory)
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; u++) v[u] = few_load_partial(src + (size_t)min(i0 + u, n - 1) * A.d);
#pragma unroll
            for (int u = 0; u < 8; u++) {
              if (i0 + u < n) {
                y.x += v[u].x; y.y += v[u].y;
                if (++p == A.parts) {
                  const float w = topk_w[t * A.Kp + j];
                  sum.x += w * y.x; sum.y += w * y.y;
                  y = make_float2(0.f, 0.f);
                  p = 0;
                  j++;
                }
              }
            }
          }
          *reinterpret_cast<uint32_t*>(A.out + (size_t)t * A.d + c) = pack_bf16(sum.x, sum.y);
        }
      }
    }
  }
}

// ---- 17 to 64 tokens: the wavefronts of a block share the rows ----------------------------------------------------------------------------

constexpr int kFewChunk = 128;        // k of the rows in LDS at a time
constexpr int kFewRowWaves = 4;       // wavefronts, of 64 columns each

// Until at most N of this wavefront's vector memory loads are outstanding (they come back in order).
template <int N>
__device__ __forceinline__ void few_wait_loads() {
  static_assert(N < 64, "the counter has 6 bits");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}
constexpr int few_rows_bytes(int TG) { return kFewGroup * TG * kFewChunk * 2; }   // of a buffer
constexpr int kFewRowsLds = 64 * 1024;   // all buffers: 2 (64 rows with remainders) to 4

// acc[g][a] += over the chunks c0 .. c1 - 1 of K: lane l's element i is column FR (4 (l / 16) + i) + a of the wavefront's 16 FR, token 16 g + l % 16.
// The rows go directly into a ring of buffers (LO: with the remainders after them), all but one chunks ahead: chunk c (8 k) of row r lies at position
// c ^ (r % 16), so that 16 rows' chunks lie in different banks.  src: lane l's row 4 (wave + 4 i) + l / 16 of instruction i, at the 8 k that belong
// at position l % 16.  The weights of a step go into registers, DEPTH - 1 steps ahead.
//
// What is waited for: the rows of chunk c + 1, before the barrier that ends chunk c.  They were requested NBUF - 2 chunks before, and since then this
// wavefront has requested the rows and weights of NBUF - 2 chunks; every step requests the same number (past the end the last ones again).
template <bool MX, int FR, int TG, bool LO>
__device__ __forceinline__ void few_multiply_rows(mx_f32x4 (&acc)[TG][FR], const FewTile<MX, FR>& W, const uint16_t* const (&src)[TG], size_t x_lo,
                                                  char* buf, int K, int c0, int c1, int wave, int lane) {
  typedef FewTile<MX, FR> Tile;
  constexpr int PER = MX ? 1 : kFewChunk / 32;   // steps of a chunk
  constexpr int HALF = few_rows_bytes(TG), BUF = HALF * (LO ? 2 : 1);
  constexpr int NBUF = kFewRowsLds / BUF < 4 ? kFewRowsLds / BUF : 4;
  constexpr int DEPTH = TG == 4 && LO && FR == 4 ? 2 : MX && TG == 4 ? 3 : 4;
  constexpr int ROW_LOADS = TG * (LO ? 2 : 1), WEIGHT_LOADS = MX ? 2 * FR : 8;
  constexpr int SINCE = (NBUF - 2) * (ROW_LOADS + PER * WEIGHT_LOADS);   // requests of this wavefront since those of the chunk after this one
  constexpr int NEWER = SINCE < 63 ? SINCE : 63;                         // (as many as can be waited for)
  if (c0 >= c1) return;
  const int n = lane & 15, q = lane >> 4;
  const int last_step = few_steps(MX, K) - 1, step1 = min(c1 * PER, last_step + 1);
  typename Tile::Stage st[DEPTH];
  const int k_of = 8 * ((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15));   // (the row's position mod 16 is the same in all instructions)
  auto load_rows = [&](int chunk) __attribute__((always_inline)) {   // (past the end of K: its last values; the weights there are zero or not multiplied)
    const int k = min(min(chunk, c1 - 1) * kFewChunk + k_of, K - 8);
    char* const to = buf + (unsigned)(chunk - c0) % NBUF * BUF + wave * 1024;
#pragma unroll
    for (int i = 0; i < TG; i++) {
      direct_load16(src[i] + k, to + i * 4096);
      if constexpr (LO) direct_load16(src[i] + x_lo + k, to + HALF + i * 4096);
    }
  };
  auto consume = [&](const typename Tile::Stage& s, const char* rows, int part) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ks++) {
      mx_bf16x8 f[FR];
#pragma unroll
      for (int a = 0; a < FR; a++) f[a] = W.frag(s, a, ks);
      const int c = MX ? 4 * q + ks : 4 * part + q;
#pragma unroll
      for (int g = 0; g < TG; g++) {
        const char* const at = rows + (16 * g + n) * (kFewChunk * 2) + ((c ^ n) << 4);
        const mx_bf16x8 x = *reinterpret_cast<const mx_bf16x8*>(at);
#pragma unroll
        for (int a = 0; a < FR; a++) acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[a], x, acc[g][a], 0, 0, 0);
        if constexpr (LO) {
          const mx_bf16x8 l = *reinterpret_cast<const mx_bf16x8*>(at + HALF);
#pragma unroll
          for (int a = 0; a < FR; a++) acc[g][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[a], l, acc[g][a], 0, 0, 0);
        }
      }
    }
  };
  __syncthreads();   // (the buffers may still be read)
#pragma unroll
  for (int i = 0; i < NBUF - 1; i++) load_rows(c0 + i);
  const int s_begin = c0 * PER;
#pragma unroll
  for (int i = 0; i < DEPTH - 1; i++) W.load(st[i], min(s_begin + i, last_step));
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  // (no branch in the loop: what the registers of a stage are is then fixed, and a wait is for the oldest stage alone)
  constexpr int UNROLL = MX ? DEPTH : PER;   // a multiple of DEPTH and of PER
  const int body = max(step1 - s_begin - 1, 0) / UNROLL * UNROLL;
  int s = s_begin;
  for (; s < s_begin + body; s += UNROLL) {
#pragma unroll
    for (int i = 0; i < UNROLL; i++) {
      const int chunk = s / PER + i / PER;
      if (i % PER == 0) load_rows(chunk + NBUF - 1);
      W.load(st[(i + DEPTH - 1) % DEPTH], min(s + i + DEPTH - 1, last_step));
      __builtin_amdgcn_sched_barrier(0);
      consume(st[i % DEPTH], buf + (unsigned)(chunk - c0) % NBUF * BUF, i % PER);
      __builtin_amdgcn_sched_barrier(0);
      if (i % PER == PER - 1) {
        few_wait_loads<NEWER>();
        __syncthreads();
      }
    }
  }
#pragma unroll
  for (int i = 0; i < UNROLL; i++) {
    const int chunk = s / PER + i / PER;
    if (s + i < step1) {
      if (i % PER == 0) load_rows(chunk + NBUF - 1);
      W.load(st[(i + DEPTH - 1) % DEPTH], min(s + i + DEPTH - 1, last_step));
      if (s + i == last_step) W.end(st[i % DEPTH], s + i);
      consume(st[i % DEPTH], buf + (unsigned)(chunk - c0) % NBUF * BUF, i % PER);
    }
    if (i % PER == PER - 1 && s + i + 1 < step1) {
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (nothing may land in LDS any more)
}

template <class F>
__device__ __forceinline__ void few_groups(int rows, F&& body) {
  if (rows > 32) body(std::integral_constant<int, 4>{});
  else if (rows > 16) body(std::integral_constant<int, 2>{});
  else body(std::integral_constant<int, 1>{});
}

// H of 32 FR columns of one expert: wavefront w makes G (w even) or U of columns 16 FR (w / 2) .. of them.
template <bool MX, int FR>
__global__ __launch_bounds__(kFewRowWaves * kWave, 2) void few_rows_gate_up_kernel(const FewArgs A) {
  constexpr int COLS = 16 * FR;
  __shared__ __attribute__((aligned(1024))) char buf[kFewRowsLds];
  __shared__ __attribute__((aligned(16))) float half[2][kFewGroup][COLS + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if ((int)blockIdx.y >= A.sched->n_live) return;
  const int4 L = few_live(A, blockIdx.y);
  const int32_t* const slots = A.sched->slots + L.y;
  const int col0 = blockIdx.x * 2 * COLS + COLS * (wave >> 1);
  const bool active = col0 < A.f;   // (widths are multiples of 64: a wavefront has all its columns, or none and repeats the first ones)
  const FewTile<MX, FR> W(wave & 1 ? A.up : A.gate, L.x, A.d, A.f, active ? col0 : 0, lane);
  for (int r0 = 0; r0 < L.z; r0 += 64) {
    few_groups(L.z - r0, [&](auto tg) __attribute__((always_inline)) {
      constexpr int TG = decltype(tg)::value;
      const uint16_t* src[TG];
      mx_f32x4 acc[TG][FR];
#pragma unroll
      for (int g = 0; g < TG; g++) {
        src[g] = A.x + (size_t)(slots[min(r0 + 16 * g + 4 * wave + (lane >> 4), L.z - 1)] / A.Kp) * A.d;
#pragma unroll
        for (int a = 0; a < FR; a++) acc[g][a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
      }
      few_multiply_rows<MX, FR, TG, false>(acc, W, src, 0, buf, A.d, 0, (A.d + kFewChunk - 1) / kFewChunk, wave, lane);
#pragma unroll
      for (int g = 0; g < TG; g++) {
        __syncthreads();
        float* const mine = &half[wave >> 1][lane & 15][4 * FR * (lane >> 4)];
        if (wave & 1) few_put(mine, acc[g]);
        __syncthreads();
        const int row = r0 + 16 * g + (lane & 15);
        if (!(wave & 1) && active && row < L.z) {
          uint32_t h[2 * FR], lo[2 * FR];
#pragma unroll
          for (int i = 0; i < 4; i++)
#pragma unroll
            for (int a = 0; a < FR; a += 2) {
              float v[2], l[2];
              few_swiglu(acc[g][a][i], mine[FR * i + a], v[0], l[0]);
              few_swiglu(acc[g][a + 1][i], mine[FR * i + a + 1], v[1], l[1]);
              h[(FR * i + a) / 2] = pack_bf16(v[0], v[1]);
              lo[(FR * i + a) / 2] = pack_bf16(l[0], l[1]);
            }
          uint16_t* const o = A.h + (size_t)slots[row] * A.f + col0 + 4 * FR * (lane >> 4);
#pragma unroll
          for (int i = 0; i < FR / 2; i++) {
            *reinterpret_cast<uint4*>(o + 8 * i) = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
            *reinterpret_cast<uint4*>(o + A.h_lo + 8 * i) = make_uint4(lo[4 * i], lo[4 * i + 1], lo[4 * i + 2], lo[4 * i + 3]);
          }
        }
      }
    });
  }
}

// 64 FR columns of H W_down of one expert over one part of d_ffn.
template <bool MX, int FR>
__global__ __launch_bounds__(kFewRowWaves * kWave, 2) void few_rows_down_kernel(const FewArgs A) {
  constexpr int COLS = 16 * FR;
  __shared__ __attribute__((aligned(1024))) char buf[kFewRowsLds];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if ((int)blockIdx.y >= A.sched->n_live) return;
  const int4 L = few_live(A, blockIdx.y);
  const int32_t* const slots = A.sched->slots + L.y;
  const int col0 = (blockIdx.x * kFewRowWaves + wave) * COLS;
  const bool active = col0 < A.d;
  const int chunks = (A.f + kFewChunk - 1) / kFewChunk, per = (chunks + A.parts - 1) / A.parts;
  const int chunk0 = min(chunks, (int)blockIdx.z * per), chunk1 = min(chunks, chunk0 + per);
  const FewTile<MX, FR> W(A.down, L.x, A.f, A.d, active ? col0 : 0, lane);
  for (int r0 = 0; r0 < L.z; r0 += 64) {
    few_groups(L.z - r0, [&](auto tg) __attribute__((always_inline)) {
      constexpr int TG = decltype(tg)::value;
      const uint16_t* src[TG];
      mx_f32x4 acc[TG][FR];
#pragma unroll
      for (int g = 0; g < TG; g++) {
        src[g] = A.h + (size_t)slots[min(r0 + 16 * g + 4 * wave + (lane >> 4), L.z - 1)] * A.f;
#pragma unroll
        for (int a = 0; a < FR; a++) acc[g][a] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
      }
      few_multiply_rows<MX, FR, TG, true>(acc, W, src, A.h_lo, buf, A.f, chunk0, chunk1, wave, lane);
#pragma unroll
      for (int g = 0; g < TG; g++) {
        const int row = r0 + 16 * g + (lane & 15);
        if (active && row < L.z) few_put(A.partial + ((size_t)slots[row] * A.parts + blockIdx.z) * A.d + col0 + 4 * FR * (lane >> 4), acc[g]);
      }
    });
  }
}

// The same sum as few_combine's, in a launch of its own: with many tokens too much for one block.
__global__ __launch_bounds__(256) void few_combine_kernel(const FewArgs A) {
  const int i = blockIdx.x * 256 + threadIdx.x, per = A.d / 2;
  const int t = i / per, c = 2 * (i % per);
  if (t >= A.T) return;
  float2 sum = make_float2(0.f, 0.f);
  for (int j = 0; j < A.Kp; j++) {
    const int s = t * A.Kp + j;
    const float w = A.topk_w[s];
    float2 y = make_float2(0.f, 0.f);
    for (int p = 0; p < A.parts; p++) {
      const float2 v = *reinterpret_cast<const float2*>(A.partial + ((size_t)s * A.parts + p) * A.d + c);
      y.x += v.x; y.y += v.y;
    }
    sum.x += w * y.x; sum.y += w * y.y;
  }
  *reinterpret_cast<uint32_t*>(A.out + (size_t)t * A.d + c) = pack_bf16(sum.x, sum.y);
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------

// Experts that can have tokens.
int few_live_bound(const Dims& D) { return (int)min((long long)D.E, (long long)D.T * D.k) + D.Es; }

// Whether the wavefronts of a block share the contraction (at most 16 tokens, whose rows fit LDS) or the rows.
bool few_share_k(const Dims& D) { return D.T <= kFewGroup && D.d <= kFewRowK; }

// Frags of 16 columns of a wavefront where the rows are shared: 4, or 2 where that leaves CUs without a block.
int few_rows_frags(const Dims& D, int C) { return (long long)((C + 127) / 128) * few_live_bound(D) >= 512 ? 4 : 2; }

// Columns of a tile of the down projection, and parts of d_ffn: as many as give every CU two blocks, but at least four steps (of 32 k) for
// a wavefront, and no more k in a part than fit LDS.
int few_down_cols(const Dims& D, bool mx) { return !few_share_k(D) ? 64 * few_rows_frags(D, D.d) : mx ? 32 : 64; }
int few_parts(const Dims& D, bool mx) {
  const int cols = few_down_cols(D, mx), waves = few_share_k(D) ? kFewWaves : 1;
  const long long blocks = (long long)((D.d + cols - 1) / cols) * few_live_bound(D);
  const int most = max(1, D.f / ((mx ? 128 : 32) * 4 * waves)), least = few_share_k(D) ? (D.f + kFewRowK / 2 - 1) / (kFewRowK / 2) : 1;
  return max(least, (int)min((long long)most, max(1ll, (512 + blocks - 1) / blocks)));
}

struct FewLayout { size_t logits, sched, counters, h, partial, total; };
FewLayout few_layout(const Dims& D) {
  FewLayout L;
  size_t o = 0;
  L.sched = o; o += round_up(sizeof(FewSched), 256);
  L.logits = o; o += round_up((size_t)D.T * D.E * sizeof(float), 256);
  L.counters = o; o += round_up(few_counters_bytes(D.d), 256);
  L.h = o; o += round_up((size_t)D.N * D.f * 2 * sizeof(uint16_t), 256);
  L.partial = o; o += round_up((size_t)D.N * max(few_parts(D, false), few_parts(D, true)) * D.d * sizeof(float), 256);
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
void few_launch_experts(hipStream_t st, const FewArgs& A, const Dims& D) {
  const int live = few_live_bound(D);
  if (!few_share_k(D)) {
    const dim3 block(kFewRowWaves * kWave);
    if (few_rows_frags(D, D.f) == 4) MOE_LAUNCH("few_gate_up", st, (few_rows_gate_up_kernel<MX, 4>), dim3((D.f + 127) / 128, live), block, 0, st, A);
    else MOE_LAUNCH("few_gate_up", st, (few_rows_gate_up_kernel<MX, 2>), dim3((D.f + 63) / 64, live), block, 0, st, A);
    if (few_rows_frags(D, D.d) == 4) MOE_LAUNCH("few_down", st, (few_rows_down_kernel<MX, 4>), dim3((D.d + 255) / 256, live, A.parts), block, 0, st, A);
    else MOE_LAUNCH("few_down", st, (few_rows_down_kernel<MX, 2>), dim3((D.d + 127) / 128, live, A.parts), block, 0, st, A);
    MOE_LAUNCH("few_combine", st, few_combine_kernel, dim3((unsigned)(((size_t)D.T * (D.d / 2) + 255) / 256)), dim3(256), 0, st, A);
    return;
  }
  constexpr int FR = MX ? 2 : 4;
  const int tiles = live * (D.f / (16 * FR) + D.d / (16 * FR) * A.parts);   // (at most)
  MOE_LAUNCH("few_layer", st, (few_layer_kernel<MX, FR, 3>), dim3(min(tiles, kFewBlocks)), dim3(kFewWaves * kWave), 0, st, A);
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
  A.T = D.T; A.d = D.d; A.f = D.f; A.E = D.E; A.Es = D.Es; A.k = D.k; A.Kp = D.Kp; A.renorm = D.renorm; A.parts = few_parts(D, MX);
  A.fused_gate = few_share_k(D) && D.Et <= kFewFusedExperts && D.N <= kFewFusedSlots;
  A.x = x; A.w_router = w_router; A.topk_idx = topk_idx; A.topk_w = topk_w; A.out = out;
  A.gate = W[0]; A.up = W[1]; A.down = W[2];
  A.logits = reinterpret_cast<float*>(wsb + L.logits);
  A.sched = reinterpret_cast<FewSched*>(wsb + L.sched);
  A.counters = reinterpret_cast<FewCounters*>(wsb + L.counters);
  A.h = reinterpret_cast<uint16_t*>(wsb + L.h);
  A.h_lo = (size_t)D.N * D.f;
  A.partial = reinterpret_cast<float*>(wsb + L.partial);
  hipStream_t st = (hipStream_t)stream;
  if (w_router)
    MOE_LAUNCH("few_router", st, few_router_kernel, dim3((D.E + 15) / 16, (D.T + 15) / 16), dim3(kFewWaves * kWave), 0, st, A);
  if (!w_router && A.fused_gate) MOE_LAUNCH("few_clear", st, few_clear_kernel, dim3(1), dim3(256), 0, st, A);
  if (!A.fused_gate) {
    if (D.E <= 64) MOE_LAUNCH("few_gate", st, few_gate_kernel<1>, dim3(1), dim3(1024), 0, st, A);
    else if (D.E <= 256) MOE_LAUNCH("few_gate", st, few_gate_kernel<4>, dim3(1), dim3(1024), 0, st, A);
    else MOE_LAUNCH("few_gate", st, few_gate_kernel<16>, dim3(1), dim3(1024), 0, st, A);
  }
  few_launch_experts<MX>(st, A, D);
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
