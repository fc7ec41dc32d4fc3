// Routing to experts with softmax or sigmoid scores, a bias that balances, groups of experts, and the gradient of its weights.
//
//   s = softmax(l) or 1 / (1 + exp(-l)) over the E logits of a token;  c = s + bias (without a bias: l, of which s is a monotone function)
//   a group of E / groups neighbouring experts has as score the sum of its `group_best` best c;  the groups_kept best groups stay
//   the k best c among them are chosen, ties to the lowest id;  w_j = scale s_j / sum_i s_i  or  scale s_j
//
// Decisions (which groups, which experts, in which order) are those of scores in 64 bits; the weights are fp32.
#include "lanes.h"

#include <type_traits>

namespace moe {

constexpr float kMaskedLogit = -1e30f;   // logits up to it, and NaN, are no experts to choose
constexpr float kMaxLogit = 3.402823466e38f;
constexpr int kGateFewWaves = 1024;   // up to so many wavefronts a token has more lanes than it needs
constexpr long long kGateIds = 1 << 20;   // of experts, shared ones among them, where only ids are made of these (lanes' counts over them stay in an int)
constexpr int kGateTokens = 1 << 24;   // of a launch of the forward kernels at most: a grid has less than 2^32 threads
constexpr int kGateBwdBlocks = 512;     // at most (two a CU; more, with more parts of the loss to add, 31 -> 40 us); each adds up its tokens' share of the loss

struct GateArgs {
  int T, E, k, Es, renorm;
  int sigmoid, groups, groups_kept, group_best;
  float scale;
};

__device__ __forceinline__ bool gate_masked(float l) { return !(l > kMaskedLogit); }
__device__ __forceinline__ float gate_finite(float l) { return l > kMaxLogit ? kMaxLogit : l; }   // (NaN stays)

// sigmoid(l) / sigmoid-like factor exp(top) with top = min(0, the largest logit that is looked at): scores far below zero keep their ratios.
__device__ __forceinline__ float sigmoid_over(float l, float top) { return 1.0f / (expf(top - l) + expf(top)); }

// A token's choices in 64 bits by a wavefront: any number of groups and experts, any k.  Choice j comes back on lane j % 64 in held[j / 64].  c: LDS of
// E + groups doubles; k rounds find the best one left.  Where this is the way out of the other kernel, one wavefront in some hundred takes it (of
// 65536 tokens of 256 experts 3 in 10000, most of which need less than this), alone: its time is that of one instruction after another, 5 us of a launch.
template <int PER>
__device__ __forceinline__ void choose_exactly(const float* __restrict__ row, const float* __restrict__ bias, double* c, int (&held)[PER], const GateArgs& A) {
  const int lane = threadIdx.x % kWave, E = A.E;
  constexpr double OUT = -__builtin_inf(), LAST = -1.7e308;   // not to be chosen; masked: after all others
  const bool by_logits = bias == nullptr, by_score = by_logits && A.group_best > 1;   // (a sum of logits would say nothing)
  constexpr int UN = PER < 4 ? PER : 4;
  float m = -kMaxLogit;
#pragma unroll UN
  for (int p = 0; p < PER; p++) {
    const int e = lane + p * kWave;
    const float l = gate_finite(row[min(e, E - 1)]);
    if (e < E) c[e] = gate_masked(l) ? LAST : (double)l;
    m = gate_masked(l) ? m : fmaxf(m, l);
  }
  if (!by_logits || by_score) {
    double z = 1.0;
    if (!A.sigmoid) {
      m = lanes_max<kWave>(m);
      z = 0.0;
    }
#pragma unroll UN
    for (int p = 0; p < PER; p++) {
      const int e = min(lane + p * kWave, E - 1);
      const double l = lane + p * kWave < E ? c[e] : LAST, x = exp(A.sigmoid ? -l : l - (double)m);
      const double v = A.sigmoid ? 1.0 / (1.0 + x) : x;
      if (l != LAST) {
        c[e] = v;
        z += v;
      }
    }
    const double over = A.sigmoid ? 1.0 : 1.0 / lanes_sum<kWave>(z);
#pragma unroll UN
    for (int p = 0; p < PER; p++) {
      const int e = min(lane + p * kWave, E - 1);
      double v = lane + p * kWave < E ? c[e] : LAST;
      if (v != LAST) {
        v = A.sigmoid ? v : v * over;
        if (!by_logits) v += (double)bias[e];
        c[e] = v > (double)kMaskedLogit ? v : LAST;
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (A.groups > 1) {
    const int S = E / A.groups;
    double* group_c = c + E;
    int L = kWave;   // lanes of a group: as many as there are for all of them at once, one if there are more
    while (L > 1 && L * A.groups > kWave) L >>= 1;
    const int sub = lane & (L - 1), per_turn = kWave / L, log2_L = __builtin_ctz(L);
#pragma unroll 1
    for (int g0 = 0; g0 < A.groups; g0 += per_turn) {
      const int g = g0 + (lane >> log2_L);
      double first = LAST, second = LAST;
      if (g < A.groups) {
#pragma unroll 4
        for (int i = sub; i < S; i += L) {
          const double v = c[g * S + i];
          second = fmax(second, fmin(first, v));
          first = fmax(first, v);
        }
      }
#pragma unroll 1
      for (int o = 1; o < L; o <<= 1) {
        const double f = __shfl_xor(first, o, kWave), n = __shfl_xor(second, o, kWave);
        second = fmax(fmax(second, n), fmin(first, f));
        first = fmax(first, f);
      }
      if (g < A.groups && sub == 0) group_c[g] = A.group_best > 1 && second != LAST ? first + second : first;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (int g0 = 0; g0 < A.groups; g0 += per_turn) {
      const int g = min(g0 + (lane >> log2_L), A.groups - 1);
      const double v = group_c[g];
      int better = 0;
#pragma unroll 8
      for (int o = 0; o < A.groups; o++) {
        const double u = group_c[o];
        better += u > v || (u == v && o < g);
      }
      if (better >= A.groups_kept) {
#pragma unroll 4
        for (int i = sub; i < S; i += L) c[g * S + i] = OUT;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (by_score) {   // (the scores were for the groups)
#pragma unroll 1
      for (int e = lane; e < E; e += kWave)
        if (c[e] != OUT && c[e] != LAST) c[e] = (double)gate_finite(row[e]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
#pragma unroll
  for (int p = 0; p < PER; p++) held[p] = 0;
#pragma unroll 1
  for (int j = 0; j < A.k; j++) {
    double best = OUT;
    int at = 0;   // a lane's best and its first place
#pragma unroll 4
    for (int p = 0; p < PER; p++) {
      const int e = lane + p * kWave;
      const double v = e < E ? c[e] : OUT;
      at = v > best ? e : at;
      best = fmax(best, v);
    }
    const double top = lanes_max<kWave>(best);
    // of the lanes that have it the lowest place
    const int choice = -(int)lanes_max<kWave>(best == top ? (float)-at : -2048.f);
    if (choice % kWave == lane) c[choice] = OUT;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int p = 0; p < PER; p++)
      if (lane == j % kWave && p == j / kWave) held[p] = choice;
  }
}

// Any number of groups and experts, any k: a wavefront per token.  For k over 16 and groups over 64 alone: 65536 tokens of 256 experts, top-8 of 4 of 8
// groups, took 197 us in rounds like these and take 21 us below.
template <int PER>
__global__ __launch_bounds__(256) void gate_general_kernel(const float* __restrict__ logits, const float* __restrict__ bias,
                                                           int32_t* __restrict__ topk_idx, float* __restrict__ topk_w, GateArgs A) {
  __shared__ double row_c[4][2 * PER * kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int t = blockIdx.x * 4 + wave;
  if (t >= A.T) return;   // (whole wavefronts; no barrier below)
  const int E = A.E, k = A.k, Kp = k + A.Es;
  const float* row = logits + (size_t)t * E;
  int held[PER];
  choose_exactly<PER>(row, bias, row_c[wave], held, A);
  float m = -kMaxLogit, all = 0.f;
  if (!A.sigmoid && !A.renorm) {
    float l[PER];
#pragma unroll
    for (int p = 0; p < PER; p++) {
      l[p] = lane + p * kWave < E ? gate_finite(row[lane + p * kWave]) : -__builtin_inff();
      if (!gate_masked(l[p])) m = fmaxf(m, l[p]);
    }
    m = lanes_max<kWave>(m);
#pragma unroll
    for (int p = 0; p < PER; p++)
      if (!gate_masked(l[p])) all += expf(l[p] - m);
    all = lanes_sum<kWave>(all);
  }
  // the weights: over the largest chosen logit where they are renormalised (scores far below zero keep their ratios)
  float top = -kMaxLogit, chosen[PER], w[PER], sum = 0.f;
#pragma unroll
  for (int p = 0; p < PER; p++) {
    chosen[p] = lane + p * kWave < k ? gate_finite(row[held[p]]) : -__builtin_inff();
    if (!gate_masked(chosen[p])) top = fmaxf(top, chosen[p]);
  }
  float z = 1.f;
  if (A.renorm) {
    top = lanes_max<kWave>(top);
    if (A.sigmoid) top = fminf(top, 0.f);
  } else {
    top = A.sigmoid ? 0.f : m;
    if (!A.sigmoid) z = all;
  }
#pragma unroll
  for (int p = 0; p < PER; p++) {
    w[p] = gate_masked(chosen[p]) ? 0.f : A.sigmoid ? sigmoid_over(chosen[p], top) : expf(chosen[p] - top);
    sum += w[p];
  }
  if (A.renorm) z = lanes_sum<kWave>(sum);
  const float factor = z > 0.f ? A.scale / z : 0.f;
#pragma unroll
  for (int p = 0; p < PER; p++) {
    const int j = lane + p * kWave;
    if (j < k) {
      topk_idx[(size_t)t * Kp + j] = held[p];
      topk_w[(size_t)t * Kp + j] = w[p] * factor;
    }
  }
  for (int j = lane; j < A.Es; j += kWave) {
    topk_idx[(size_t)t * Kp + k + j] = E + j;
    topk_w[(size_t)t * Kp + k + j] = 1.0f;
  }
}

// ---- k <= 16, groups <= 64: W lanes per token, each with a run of neighbouring experts of one group.
//
// A value to select by (c, or l) is a key: a double whose high word is the fp32 value and whose low word its expert, so that one comparison orders by
// value and then by the lower id, keys are never equal, and a maximum and a minimum (an instruction each) exchange two of them.  A lane sorts its
// experts' keys, K at a time, by a network and keeps the K best; two lists of K join by K maxima (of one and the other backwards) and a merging
// network, first in the lane, then lane by lane in log2 W steps, at the end of which all lanes have the token's K best.  When a list is a group's, its
// first two give the group's score, and the lists of groups that do not stay are emptied.
// The logits come in through LDS: a wavefront's tokens lie next to each other in memory whatever E is, and all its loads are under way at once.
//
// Bound by the vector instructions: 65536 tokens of 256 experts, sigmoid scores, a bias, top-8 of 4 of 8 groups: 21 us for 72 MB (HBM's share: 11),
// 933 instructions a wavefront of 8 tokens, 3 in 4 of a SIMD's cycles.  One in 15 is an exponential or a reciprocal, at a quarter of the rate; networks
// and joins are half.  Few tokens: 2.5 us for one of 64 experts, the latency of one wavefront.  16384 tokens of 128: 4.8 to 5.9 us.
// Measured and left out, on the large case: a wavefront that goes on to the next tokens with their loads under way (registers spill: 84 for 25 us); the
// order in 64 bits of all tokens' candidates, each on its token's lanes (30 for 25).
//
// fp32 orders two values right if they are further apart than twice what either may be off.  Where a choice or its order hangs on less, which adjacent
// keys, the first one left out and the groups next to the cut tell, the wavefront makes that token's choice again in 64 bits, among the experts near its k-th
// best where the groups are sure.  Tokens whose c are all equal (rows of zeros) go there every one, one after another: on the large case 178 us where all rows
// are so, 40 where one in 16 is, 22 without.

constexpr float kDeadKey = -3.0e38f;   // masked experts: after all others
constexpr float kNoKey = -3.3e38f;     // of groups that do not stay, and behind the last expert

// signs: the low word goes by the sign of the value.
__device__ __forceinline__ double make_key(float v, int e, bool signs) {
  const int bits = __float_as_int(v);
  return __hiloint2double(bits, ~e ^ (signs ? bits >> 31 : 0));
}
__device__ __forceinline__ float key_value(double key) { return __int_as_float(__double2hiint(key)); }
__device__ __forceinline__ int key_expert(double key, bool signs) { return ~(__double2loint(key) ^ (signs ? __double2hiint(key) >> 31 : 0)); }

// The instructions themselves: fmax and fmin first rewrite each operand that could be a signalling NaN, and no key is a NaN.
__device__ __forceinline__ double key_max(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double key_min(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
// The largest of `a` and the smaller ones of two pairs.
__device__ __forceinline__ float max_of_mins(float a, float b0, float b1, float c0, float c1) {
  float b, c, r;
  asm("v_min_f32 %0, %1, %2" : "=v"(b) : "v"(b0), "v"(b1));
  asm("v_min_f32 %0, %1, %2" : "=v"(c) : "v"(c0), "v"(c1));
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ void exchange(double& a, double& b) {
  const double hi = key_max(a, b);
  b = key_min(a, b);
  a = hi;
}
// Falling order (Batcher's odd-even merge sort: 19 exchanges for 8, 63 for 16).
template <int K>
__device__ __forceinline__ void sort_keys(double (&a)[K]) {
#pragma unroll
  for (int p = 1; p < K; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < K; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; i++)
          if (i + j + q < K && (i + j) / (2 * p) == (i + j + q) / (2 * p)) exchange(a[i + j], a[i + j + q]);
}
// a: the K best of a and b, both falling.
template <int K>
__device__ __forceinline__ void join_keys(double (&a)[K], const double (&b)[K]) {
#pragma unroll
  for (int i = 0; i < K; i++) a[i] = key_max(a[i], b[K - 1 - i]);
#pragma unroll
  for (int q = K / 2; q >= 1; q /= 2)
#pragma unroll
    for (int i = 0; i < K; i++)
      if (!(i & q)) exchange(a[i], a[i + q]);
}

__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

struct GatePlan {        // how a token's experts lie on its lanes
  int lanes_of_group;    // a power of two, and its logarithm
  int lanes_log2;
  int size;              // experts of a group
  int piece;             // experts of a lane at most
};
// Where the i-th float of a wavefront's logits lies in LDS: 4 floats are left free after every RUN, which keeps the lanes off each other's banks.
template <int RUN>
__device__ __forceinline__ int gate_place(int i) { return i + 4 * (int)((unsigned)i / RUN); }

// FULL: every lane has PER experts, and so a run of its own.
template <int K, int W, int PER, bool FULL>
__global__ __launch_bounds__(256, 4) void gate_kernel(const float* __restrict__ logits, const float* __restrict__ bias, int32_t* __restrict__ topk_idx,
                                                      float* __restrict__ topk_w, GateArgs A, GatePlan P) {
  static_assert(K <= W && PER % K == 0 && PER <= 32, "a choice for each of the first K lanes, a bit for each expert of a lane");
  constexpr int TOKENS = kWave / W;
  constexpr int MAX_E = W * PER < kMaxExperts ? W * PER : kMaxExperts;
  constexpr int RUN = FULL ? PER : 32;
  constexpr int ROW_FLOATS = kWave * (PER + 4) + PER;                   // (gate_place; the last lane reads on behind its run)
  constexpr int EXACT_FLOATS = 2 * (MAX_E + kWave);                     // what choose_exactly takes of them
  __shared__ __attribute__((aligned(16))) float rows[4][ROW_FLOATS > EXACT_FLOATS ? ROW_FLOATS : EXACT_FLOATS];
  __shared__ double group_scores[4][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane % W, tt = lane / W;
  const int t0 = (blockIdx.x * 4 + wave) * TOKENS, t = t0 + tt;
  const int E = A.E, k = A.k, Kp = k + A.Es;
  const bool by_logits = bias == nullptr;
  // The bias into LDS, a run for each lane of a token: read from memory by every wavefront, the few lines of it are what all of them wait for
  __shared__ __attribute__((aligned(16))) float biases[W * (PER + 4)];
  __shared__ int dead_bias;
  if (!by_logits) {
    if (threadIdx.x == 0) dead_bias = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < W * PER; i += 256) {
      const int run = i / PER, p = i % PER, of_group = run >> P.lanes_log2, from = (run & (P.lanes_of_group - 1)) * P.piece + p;
      const bool exists = of_group < A.groups && p < P.piece && from < P.size;
      const float b = exists ? bias[of_group * P.size + from] : 0.f;
      biases[run * (PER + 4) + p] = b;
      if (!(b > kMaskedLogit)) dead_bias = 1;
    }
    __syncthreads();
  }
  if (t0 >= A.T) return;   // (whole wavefronts; no barrier below)

  // the tokens' logits into LDS (t0 E is a multiple of 4 but for two tokens of odd E)
  const int n = min(TOKENS, A.T - t0) * E;
  const float* src = logits + (size_t)t0 * E;
  // (all requested before the first one is waited for)
  if (FULL && n == kWave * PER) {   // (whole wavefronts of whole lanes)
    float4 in[PER / 4];
#pragma unroll
    for (int j = 0; j < PER / 4; j++) in[j] = *reinterpret_cast<const float4*>(src + 4 * lane + 4 * kWave * j);
#pragma unroll
    for (int j = 0; j < PER / 4; j++) {
      const int at = (4 * kWave) % RUN ? gate_place<RUN>(4 * (lane + kWave * j)) : gate_place<RUN>(4 * lane) + gate_place<RUN>(4 * kWave) * j;
      *reinterpret_cast<float4*>(&rows[wave][at]) = in[j];
    }
  } else if ((TOKENS % 4 == 0 || (E * TOKENS) % 4 == 0) && n >= 4) {
    float4 in[PER / 4];
#pragma unroll
    for (int j = 0; j < PER / 4; j++) in[j] = *reinterpret_cast<const float4*>(src + min(4 * (lane + kWave * j), (n - 4) & ~3));
#pragma unroll
    for (int j = 0; j < PER / 4; j++) *reinterpret_cast<float4*>(&rows[wave][gate_place<RUN>(4 * (lane + kWave * j))]) = in[j];   // (what lies behind n is not read)
    if (lane < (n & 3)) rows[wave][gate_place<RUN>((n & ~3) + lane)] = src[(n & ~3) + lane];
  } else {
    for (int i = lane; i < n; i += kWave) rows[wave][gate_place<RUN>(i)] = src[i];
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

  const int size = P.size;
  const int group = g >> P.lanes_log2;
  const int begin = (g & (P.lanes_of_group - 1)) * P.piece;
  const int first = group * size + begin, count = group < A.groups && t < A.T ? max(0, min(P.piece, size - begin)) : 0;
  float l[PER], c[PER];
  // (of a lane without a group: the last one's; its keys are behind all others by their ids, or its group does not stay)
  if constexpr (FULL) {
    const int from = min(first, E - PER);
    const float* run = &rows[wave][gate_place<RUN>(tt * E + from)];
#pragma unroll
    for (int p = 0; p < PER; p += 4) {
      const float4 u = *reinterpret_cast<const float4*>(run + p);
      l[p] = u.x; l[p + 1] = u.y; l[p + 2] = u.z; l[p + 3] = u.w;
    }
  } else {
    const int at = tt * E + min(first, E - 1), turn = RUN - at % RUN;   // (PER <= RUN: one place at most where floats are left free)
    const float* run = &rows[wave][gate_place<RUN>(at)];
#pragma unroll
    for (int p = 0; p < PER; p++) l[p] = (p < turn ? run : run + 4)[p];
  }
  auto bias_of = [&](int p, float* b) __attribute__((always_inline)) {   // of a lane's experts p .. p + 3
    const float4 u = *reinterpret_cast<const float4*>(&biases[g * (PER + 4) + p]);
    b[0] = u.x; b[1] = u.y; b[2] = u.z; b[3] = u.w;
  };
  bool some_dead = !by_logits && dead_bias != 0;   // a key of the wavefront may be one
  const float lowest = group < A.groups ? kMaskedLogit : __builtin_inff();   // (nothing of a lane without a group counts)
  // what is selected by, in c.  (Functions are evaluated for all, then chosen from: no branch for an element.)
  float m = -kMaxLogit, inv_z = 1.f;
  if (A.sigmoid && !by_logits) {
    unsigned top_bits = 0;   // of the exponentials: infinite or NaN where one is masked (or a score too small to be told from that)
#pragma unroll
    for (int p = 0; p < PER; p += 8) {   // (eight at a time, step by step: no instruction waits for the one before it)
      float b[8], e[8];
      bias_of(p, b);
      bias_of(p + 4, b + 4);
#pragma unroll
      for (int i = 0; i < 8; i++) e[i] = fast_exp(-l[p + i]);
#pragma unroll
      for (int i = 0; i < 8; i++) top_bits = max(top_bits, __float_as_uint(e[i]));
#pragma unroll
      for (int i = 0; i < 8; i++) e[i] = __builtin_amdgcn_rcpf(1.0f + e[i]);
#pragma unroll
      for (int i = 0; i < 8; i++) c[p + i] = e[i] + b[i];
    }
    some_dead = __any(some_dead || top_bits >= 0x7f800000u);
    if (some_dead) {
      asm volatile("");   // (a branch: mostly it is not taken)
#pragma unroll
      for (int p = 0; p < PER; p++) c[p] = l[p] > kMaskedLogit && c[p] > kMaskedLogit ? c[p] : kDeadKey;
    }
  } else {
#pragma unroll
    for (int p = 0; p < PER; p++) {
      const float finite = fminf(l[p], kMaxLogit);
      l[p] = l[p] > lowest && (FULL || p < count) ? finite : -__builtin_inff();   // (and NaN)
    }
    some_dead = true;
    if (!A.sigmoid && !(by_logits && A.renorm && A.group_best == 1)) {
#pragma unroll
      for (int p = 0; p < PER; p++) m = fmaxf(m, l[p]);
      m = lanes_max<W>(m);
    }
    if (by_logits) {
#pragma unroll
      for (int p = 0; p < PER; p++) c[p] = l[p] > kMaskedLogit ? l[p] + 0.0f : kDeadKey;   // (-0 is 0)
    }
    if (!A.sigmoid && !(by_logits && A.renorm)) {
      float z = 0.f;
#pragma unroll
      for (int p = 0; p < PER; p++) z += fast_exp(l[p] - m);
      z = lanes_sum<W>(z);
      inv_z = z > 0.f ? 1.0f / z : 0.f;
      if (!by_logits) {
#pragma unroll
        for (int p = 0; p < PER; p += 4) {
          float b[4];
          bias_of(p, b);
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const float v = fmaf(fast_exp(l[p + i] - m), inv_z, b[i]);
            c[p + i] = l[p + i] > kMaskedLogit && v > kMaskedLogit ? v : kDeadKey;
          }
        }
      }
    }
  }
  if constexpr (!FULL) {
#pragma unroll
    for (int p = 0; p < PER; p++) c[p] = p < count ? c[p] : kNoKey;
  }
  // How far c may be off, in units of 2^-24.  sigmoid: the exponential's argument 1.5 |l| times s (1 - s) <= 0.23 / |l|, the exponential 2 s (1 - s), the
  // sum s, the reciprocal 2 s: under 4.  softmax, times 1 / z, which no score is above: the sum of exponentials z is off by the mean of their
  // arguments, 1.5 times under 5 of 1024, by 2 and by PER + 6 additions; its reciprocal by 2; a score by its own argument, 1.5 times 0.37, by 2 and by
  // the product: under PER + 22.  And c by a rounding.  For both of a pair, twice that.
  const float slack = by_logits ? 0.f : A.sigmoid ? 0x1p-21f : (PER + 22) * 0x1p-23f * inv_z, slack_c = 0x1p-23f;
  const bool track = !by_logits && k == K;   // (else the first one left out is in the list, or order needs no margin)
  // Up to a few lanes' experts stay: one lane may well have all choices.  With more, what a lane lets go matters in 4 (1/4)^K of the tokens,
  // which is few from K = 8 on.
  const bool track_lane = track && (K < 8 || A.groups_kept * P.lanes_of_group < 4);
  float lost = kNoKey;                       // the best that joining lists has let go
  auto let_go = [&](const double (&a)[K], const double (&b)[K]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < K; i += 2) lost = max_of_mins(lost, key_value(a[i]), key_value(b[K - 1 - i]), key_value(a[i + 1]), key_value(b[K - 2 - i]));
  };
  // Of negative values the larger low word is the smaller number.  Where c is selected by, equal values are told apart in 64 bits, but for dead ones.
  const bool signs = by_logits || some_dead;
  double best[K];
#pragma unroll
  for (int b = 0; b < PER / K; b++) {
    double more[K];
#pragma unroll
    for (int i = 0; i < K; i++) more[i] = make_key(c[b * K + i], first + b * K + i, false);
    if (signs) {
#pragma unroll
      for (int i = 0; i < K; i++) more[i] = make_key(c[b * K + i], first + b * K + i, true);
    }
    sort_keys<K>(more);
    if (b == 0) {
#pragma unroll
      for (int i = 0; i < K; i++) best[i] = more[i];
    } else {
      if (track_lane) let_go(best, more);
      join_keys<K>(best, more);
    }
  }
  float lane_last = PER > K && track && !track_lane ? key_value(best[K - 1]) : kNoKey;   // (nothing that the lane has let go is above it)
  bool unsure = false, unsure_group = false;
  unsigned long long kept_lanes = ~0ull;   // whose group stays

  auto select_groups = [&]() __attribute__((always_inline)) {
    const float a = key_value(best[0]), b = key_value(best[1]);
    float score = kDeadKey;
    if (a > kMaskedLogit) {
      score = a;
      if (A.group_best > 1) {
        const bool two = b > kMaskedLogit;
        if (!by_logits) score = two ? a + b : a;
        else if (A.sigmoid) score = __builtin_amdgcn_rcpf(1.0f + fast_exp(-a)) + (two ? __builtin_amdgcn_rcpf(1.0f + fast_exp(-b)) : 0.f);
        else score = fast_exp(a - m) + (two ? fast_exp(b - m) : 0.f);   // (over the sum that all groups share)
      }
    }
    // (a key of the score and the group: equal ones go by the group, those without living experts below all others)
    const double mark = __hiloint2double(__float_as_int(score), score < 0.f ? group : ~group);
    double* marks = group_scores[wave];
    marks[lane] = mark;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int better = 0;
#pragma unroll 4
    for (int o = 0; o < A.groups; o++) better += marks[lane - g + o * P.lanes_of_group] > mark;
    const bool exists = group < A.groups, stays = exists && better < A.groups_kept;
    if (!by_logits || A.group_best > 1) {
      const float low = -lanes_max<W>(stays ? -score : -__builtin_inff()), high = lanes_max<W>(exists && !stays ? score : -__builtin_inff());
      // Two c, off as above, and a rounding of their sum, for two groups; the c themselves may be large and cancel.  Scores without a bias: of sigmoid
      // as above, of softmax (without the shared sum, each at most 1) the argument, the exponential, the sum: under 8 in all.
      const float far = by_logits ? 0x1p-20f : 2.0f * slack + slack_c * (fabsf(low) + lanes_max<W>(a > kMaskedLogit ? fabsf(a) + (b > kMaskedLogit ? fabsf(b) : 0.f) : 0.f));
      unsure_group = unsure_group || (high > kMaskedLogit && !(low - high > far));   // (also two sums past fp32, whose difference is NaN)
    }
    const double none = make_key(kNoKey, 0, false);
#pragma unroll
    for (int i = 0; i < K; i++) best[i] = stays ? best[i] : none;
    lost = stays ? lost : kNoKey;
    lane_last = stays ? lane_last : kNoKey;
    kept_lanes = __ballot(stays);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  auto join_lanes = [&](auto step_c) __attribute__((always_inline)) {
    constexpr int STEP = decltype(step_c)::value;
    if constexpr (STEP < W) {
      if (A.groups > 1 && STEP == P.lanes_of_group) select_groups();
      double other[K];
#pragma unroll
      for (int i = 0; i < K; i++) other[i] = from_lane<STEP>(best[i]);
      if (track) {
        lost = fmaxf(lost, from_lane<STEP>(lost));
        let_go(best, other);
      }
      join_keys<K>(best, other);
    }
  };
  join_lanes(std::integral_constant<int, 1>{});
  join_lanes(std::integral_constant<int, 2>{});
  join_lanes(std::integral_constant<int, 4>{});
  join_lanes(std::integral_constant<int, 8>{});
  join_lanes(std::integral_constant<int, 16>{});
  join_lanes(std::integral_constant<int, 32>{});

  // lane g takes choice g
  double mine = best[0];
#pragma unroll
  for (int i = 1; i < K; i++) mine = g == i ? best[i] : mine;
  int choice = key_expert(mine, signs);
  if (!by_logits) {
    const float a = key_value(mine);
    const float after = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), 0x101, 0xF, 0xF, true));   // row_shl:1: the next lane's
    const float b = g == K - 1 ? lost : after;
    unsure = unsure || (g < k && b > kMaskedLogit && a - b <= slack + slack_c * fmaxf(fabsf(a), fabsf(b)));
    unsure = unsure || (lane_last > kMaskedLogit && lane_last >= key_value(best[K - 1]));
  }
  const bool live = t < A.T && g < k;
  float x = live ? rows[wave][gate_place<RUN>(tt * E + choice)] : -__builtin_inff();
  unsigned long long again = __ballot((unsure || unsure_group) && t < A.T);
  if (again) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // the k-th c, and how far below it one may be that belongs before it
    const float kth = by_logits || unsure_group ? -__builtin_inff() : __shfl(key_value(mine), lane - g + k - 1, kWave);
    const float least = kth - (slack + slack_c * (fabsf(kth) + slack));
    const unsigned long long by_groups = __ballot(unsure_group);
    unsigned long long all_again = 0;
    const auto lanes_of = [](int token) { return (W == kWave ? ~0ull : (1ull << (W & 63)) - 1) << (token * W); };
    if (!by_logits) {
      // Sure of the groups: the experts that may be among the k best are looked up again in fp32 (a run by a lane of each token), and these are put in
      // order in 64 bits, which takes a third of the time of the whole: 4096 tokens of 256 experts, one or two of which come here, 9.0 -> 6.0 us.
      int* found = reinterpret_cast<int*>(group_scores[wave]);
      const int exist = group < A.groups ? max(0, min(P.piece, size - begin)) : 0;
      do {
        const int token = __builtin_ctzll(again) / W;
        again &= ~lanes_of(token);
        const float from = __shfl(least, token * W, kWave);
        const float top = A.sigmoid ? 0.f : __shfl(m, token * W, kWave), over = A.sigmoid ? 1.f : __shfl(inv_z, token * W, kWave);
        int n = 0;
        if (!(by_groups & lanes_of(token)) && from > kMaskedLogit) {
          const bool kept = (kept_lanes >> (token * W + g)) & 1;
#pragma unroll
          for (int i = 0; i < PER / TOKENS; i++) {
            const int p = tt + TOKENS * i;
            const float lp = gate_finite(rows[wave][gate_place<RUN>(token * E + min(first + p, E - 1))]), b = biases[g * (PER + 4) + p];
            const float v = A.sigmoid ? __builtin_amdgcn_rcpf(1.0f + fast_exp(-lp)) + b : fmaf(fast_exp(lp - top), over, b);
            const bool one = kept && p < exist && lp > kMaskedLogit && v >= from;
            const unsigned long long all = __ballot(one);
            const int at = n + __popcll(all & ((1ull << lane) - 1));
            if (one && at < kWave) found[at] = first + p + (g << 10) + (p << 16);
            n += __popcll(all);
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        if (n < k || n > kWave) {   // (of a group in doubt, or very many alike)
          all_again |= lanes_of(token);
          continue;
        }
        const int it = found[min(lane, n - 1)], e = it & 1023;
        const double le = gate_finite(rows[wave][gate_place<RUN>(token * E + e)]), b = biases[((it >> 10) & 63) * (PER + 4) + (it >> 16)];
        double v;
        if (A.sigmoid) {
          v = 1.0 / (1.0 + exp(-le)) + b;
        } else {
          double z = 0.0;
#pragma unroll
          for (int i = 0; i < PER / TOKENS; i++) {
            const int p = tt + TOKENS * i;
            const float lp = gate_finite(rows[wave][gate_place<RUN>(token * E + min(first + p, E - 1))]);
            z += p < exist && lp > kMaskedLogit ? exp((double)lp - (double)top) : 0.0;
          }
          v = exp(le - (double)top) / lanes_sum<kWave>(z) + b;
        }
        int place = 0;
        for (int o = 0; o < n; o++) {
          const double u = __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), o), __builtin_amdgcn_readlane(__double2loint(v), o));
          place += u > v || (u == v && __builtin_amdgcn_readlane(e, o) < e);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < n) found[place] = e;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (tt == token && g < k) choice = found[g];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      } while (again);
      if (live) x = rows[wave][gate_place<RUN>(tt * E + choice)];
    } else {
      all_again = again;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    again = all_again;
    while (again) {   // (the logits in LDS make room)
      const int token = __builtin_ctzll(again) / W;
      int held[(MAX_E + kWave - 1) / kWave];
      choose_exactly<(MAX_E + kWave - 1) / kWave>(logits + (size_t)(t0 + token) * E, bias, reinterpret_cast<double*>(rows[wave]), held, A);
      const int found = __shfl(held[0], g, kWave);
      if (tt == token) {
        choice = found;
        if (live) x = logits[(size_t)t * E + choice];
      }
      again &= ~lanes_of(token);
    }
  }

  // the weights: over the largest chosen logit where they are renormalised (scores far below zero keep their ratios)
  x = gate_finite(x);
  const bool dead = gate_masked(x);
  float w = 0.f, factor = A.scale;
  if (A.renorm) {
    float top = lanes_max<K>(dead ? -kMaxLogit : x);
    if (A.sigmoid) top = fminf(top, 0.f);
    w = fast_exp(x - top);
    if (A.sigmoid) w = __builtin_amdgcn_rcpf(fast_exp(top - x) + fast_exp(top));
    w = dead ? 0.f : w;
    const float z = lanes_sum<K>(w);
    factor = z > 0.f ? A.scale * __builtin_amdgcn_rcpf(z) : 0.f;
  } else {
    w = A.sigmoid ? __builtin_amdgcn_rcpf(fast_exp(-x) + 1.0f) : fast_exp(x - m) * inv_z;
    w = dead ? 0.f : w;
  }
  if (live) {
    topk_idx[(size_t)t * Kp + g] = choice;
    topk_w[(size_t)t * Kp + g] = w * factor;
  }
  if (t < A.T)
    for (int j = g; j < A.Es; j += W) {
      topk_idx[(size_t)t * Kp + k + j] = E + j;
      topk_w[(size_t)t * Kp + k + j] = 1.0f;
    }
}

// Gradient of the weights and of the balance loss.  With q = s / sum s, n_e the slots of expert e, C_e = balance E n_e / (k T^2):
//   softmax  dl_m = q_m (C_m - <q, C>) [- s_m <w, dw> where not renormalised] + d_j of the slots with expert m
//   sigmoid  dl_m = (1 - s_m) (q_m (C_m - <q, C>) + d_j)
//   d_j = w_j (dw_j - <w, dw> / scale) where renormalised, else w_j dw_j
// Bound by HBM: the logits in, their gradients out (65536 tokens of 256 experts with the loss: 31 us, 4.5 TB/s; of their first form, a wavefront a token
// with selections for all cases, 111).  W lanes per token; a lane holds 4 neighbouring experts (VEC; else every W-th) in each of C chunks.
// The slots' d go to their experts through a row in LDS; a wavefront goes from tokens to tokens, the next ones' loads under way.
constexpr int kGateBwdWaves = 8;
template <int W, int C, bool VEC>
__global__ __launch_bounds__(kGateBwdWaves * kWave, 4) void gate_bwd_kernel(const float* __restrict__ dtopk_w, const float* __restrict__ logits,
                                                                            const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w,
                                                                            const int32_t* __restrict__ counts, float cost, float* __restrict__ dlogits,
                                                                            float* __restrict__ loss_part, GateArgs A) {
  constexpr int TOKENS = kWave / W, ROW = W * C * 4;   // floats of a token's row
  __shared__ __attribute__((aligned(16))) float rows[kGateBwdWaves][TOKENS * ROW];
  __shared__ float part[kGateBwdWaves];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane % W, tt = lane / W;
  const int E = A.E, k = A.k, Kp = k + A.Es;
  const bool dense = counts != nullptr || (!A.sigmoid && !A.renorm);
  const float inv_scale = 1.0f / A.scale;
  float* row = &rows[wave][tt * ROW];
  auto expert = [&](int c, int i) { return VEC ? 4 * (g + W * c) + i : g + W * (4 * c + i); };
  // C_e in LDS.  (The counts read from memory by every wavefront, their few lines would be what all of them wait for.)
  __shared__ __attribute__((aligned(16))) float costs[ROW];
  for (int e = threadIdx.x; e < ROW; e += kGateBwdWaves * kWave) costs[e] = counts && e < E ? cost * (float)counts[e] : 0.f;
  __syncthreads();
  auto four_of = [&](const float* from, int c, float (&v)[4]) __attribute__((always_inline)) {
    if (VEC) {
      const float4 u = *reinterpret_cast<const float4*>(from + 4 * (g + W * c));
      v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = from[expert(c, i)];
    }
  };
  float loss = 0.f;
  const int batches = (A.T - 1) / TOKENS + 1, step = gridDim.x * kGateBwdWaves;
  struct Batch { float l[4 * C]; int e; float w, dw; };   // what a batch of tokens reads: requested while the one before is computed
  auto request = [&](int batch, Batch& b) __attribute__((always_inline)) {
    const size_t at = (size_t)min(batch * TOKENS + tt, A.T - 1);
    const float* src = logits + at * E;
    if (dense) {
#pragma unroll
      for (int c = 0; c < C; c++) {
        if (VEC) {
          const float4 u = *reinterpret_cast<const float4*>(src + min(expert(c, 0), E - 4));
          b.l[4 * c] = u.x; b.l[4 * c + 1] = u.y; b.l[4 * c + 2] = u.z; b.l[4 * c + 3] = u.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; i++) b.l[4 * c + i] = src[min(expert(c, i), E - 1)];
        }
      }
    }
    const size_t slot = at * Kp + min(g, k - 1);
    b.e = topk_idx[slot];
    b.w = topk_w[slot];
    b.dw = dtopk_w[slot];
  };
  Batch cur, next;
  int batch = blockIdx.x * kGateBwdWaves + wave;
  constexpr bool AHEAD = VEC || C <= 2;   // (12 and 16 experts one by one take the registers: 30000 x 190 13.8 us, ahead 14.8)
  if (AHEAD && batch < batches) request(batch, cur);
  for (; batch < batches; batch += step) {
    if constexpr (AHEAD) {
      if (batch + step < batches) request(batch + step, next);
    } else {
      request(batch, cur);
    }
    const int t = batch * TOKENS + tt;
    const bool live = t < A.T;
    const size_t at = (size_t)(live ? t : A.T - 1);
    const float* src = logits + at * E;
    float (&l)[4 * C] = cur.l;
    // the slots (k of them, W at a time; one without weight, a masked expert's, counts as nothing, whatever its dw is)
    float inner = g < k && cur.w != 0.f ? cur.w * cur.dw : 0.f;
    for (int j = g + W; j < k; j += W) {
      const float w = topk_w[at * Kp + j];
      inner = w != 0.f ? fmaf(w, dtopk_w[at * Kp + j], inner) : inner;
    }
    inner = lanes_sum<W>(inner);
#pragma unroll
    for (int c = 0; c < C; c++) *reinterpret_cast<float4*>(row + 4 * (g + W * c)) = float4{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int j0 = 0; j0 < k; j0 += W) {
      const int j = j0 + g;
      int e = cur.e;
      float w = cur.w, dw = cur.dw;
      if (j0 > 0 && j < k) {
        e = topk_idx[at * Kp + j];
        w = topk_w[at * Kp + j];
        dw = dtopk_w[at * Kp + j];
      }
      const bool mine = j < k && (unsigned)e < (unsigned)E;   // (no other id has a logit)
      float d = A.renorm ? w * (dw - inner * inv_scale) : w * dw;
      d = w != 0.f ? d : 0.f;
      if (A.sigmoid && !dense && mine) {
        const float x = src[e];
        d = gate_masked(x) ? 0.f : d * __builtin_amdgcn_rcpf(1.0f + fast_exp(gate_finite(x)));
      }
      // whether an expert is named twice, which its place in the row tells: then its slots one after another
      float old = 0.f;
      bool twice = false;
      if (mine) {
        if (j0 > 0) old = row[e];
        row[e] = __int_as_float(g);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (mine) twice = __float_as_int(row[e]) != g;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const bool any = __any(twice);
      if (mine) row[e] = any ? old : old + d;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (any) {
        for (int o = 0; o < W; o++) {
          if (g == o && mine) row[e] += d;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
    float* out = dlogits + at * E;
    float s[4 * C], slope[4 * C], mean = 0.f;
    if (dense) {
      float z = 0.f, m = -kMaxLogit;
#pragma unroll
      for (int i = 0; i < 4 * C; i++) {
        const float finite = fminf(l[i], kMaxLogit);
        l[i] = expert(i / 4, i % 4) < E && l[i] > kMaskedLogit ? finite : -__builtin_inff();   // (and NaN)
        m = fmaxf(m, l[i]);
      }
      // Scores over exp(top), which keeps the ratios of those far below zero.  sigmoid: e = exp(top - l) is at least exp(top), which is at most 1.
      float top = 0.f;
      if (!A.sigmoid) top = lanes_max<W>(m);
      else if (__any(m < 0.f)) top = fminf(lanes_max<W>(m), 0.f);
      const float unit = A.sigmoid ? fast_exp(top) : 0.f;
#pragma unroll
      for (int i = 0; i < 4 * C; i++) {
        if (A.sigmoid) {
          const float e = fast_exp(top - l[i]);
          s[i] = __builtin_amdgcn_rcpf(e + unit);
          slope[i] = e < 0x1p100f ? e * s[i] : l[i] > kMaskedLogit ? 1.0f : 0.f;   // 1 - s = exp(-l) / (1 + exp(-l))
        } else {
          s[i] = fast_exp(l[i] - top);
          slope[i] = l[i] > kMaskedLogit ? 1.0f : 0.f;
        }
        z += s[i];
      }
      z = lanes_sum<W>(z);
      const float inv = z > 0.f ? 1.0f / z : 0.f;
#pragma unroll
      for (int c = 0; c < C; c++) {
        float Ce[4];
        four_of(costs, c, Ce);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          s[4 * c + i] *= inv;
          mean = fmaf(s[4 * c + i], Ce[i], mean);
        }
      }
      mean = lanes_sum<W>(mean);
      if (live && g == 0) loss += mean;
    }
    const float less = mean + (!A.sigmoid && !A.renorm ? inner : 0.f);
#pragma unroll
    for (int c = 0; c < C; c++) {
      float v[4];
      four_of(row, c, v);
      if (dense) {
        float Ce[4];
        four_of(costs, c, Ce);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = fmaf(s[4 * c + i], Ce[i] - less, v[i]) * slope[4 * c + i];
      }
      if (VEC) {
        if (live && expert(c, 0) < E) *reinterpret_cast<float4*>(out + expert(c, 0)) = float4{v[0], v[1], v[2], v[3]};
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
          if (live && expert(c, i) < E) out[expert(c, i)] = v[i];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (the next batch's zeros)
    if constexpr (AHEAD) cur = next;
  }
  if (loss_part) {
    loss = lanes_sum<kWave>(loss);
    if (lane == 0) part[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
      float sum = 0.f;
      for (int i = 0; i < kGateBwdWaves; i++) sum += part[i];
      loss_part[blockIdx.x] = sum;   // (of a block by itself: the loss)
    }
  }
}

// The sum of at most kGateBwdBlocks parts, in a fixed order (4.4 us by itself, 2 behind the kernel above: latency).
__global__ __launch_bounds__(256) void gate_loss_kernel(const float* __restrict__ loss_part, int parts, float* __restrict__ loss) {
  __shared__ double sum[256 / kWave];
  double v = 0.0;
#pragma unroll
  for (int i = 0; i < kGateBwdBlocks / 256; i++) {
    const int at = threadIdx.x + 256 * i;
    v += at < parts ? (double)loss_part[at] : 0.0;
  }
  v = lanes_sum<kWave>(v);
  if (threadIdx.x % kWave == 0) sum[threadIdx.x / kWave] = v;
  __syncthreads();
  if (threadIdx.x == 0) *loss = (float)((sum[0] + sum[1]) + (sum[2] + sum[3]));
}

// bias_e += rate where expert e has fewer slots than the mean, -= rate where it has more.
__global__ __launch_bounds__(256) void gate_bias_step_kernel(const int32_t* __restrict__ counts, int E, float rate, float* __restrict__ bias) {
  __shared__ long long sum[256];
  long long n = 0;
  for (int e = threadIdx.x; e < E; e += 256) n += counts[e];
  sum[threadIdx.x] = n;
  for (int o = 128; o > 0; o >>= 1) {
    __syncthreads();
    if (threadIdx.x < o) sum[threadIdx.x] += sum[threadIdx.x + o];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += 256) {
    const long long have = (long long)counts[e] * E;
    if (have != sum[0]) bias[e] += have < sum[0] ? rate : -rate;
  }
}

// Checks a gate against the shape, and joins the two.
static int gate_checks(const moe_shape* shape, const moe_gate* gate, Dims* D, GateArgs* A, long long max_ids = kGateIds) {
  const int rc = check_shape(shape, D, max_ids);
  if (rc != MOE_OK) return rc;
  if (!gate) return MOE_ERR_NULL;
  if (gate->scores != MOE_SCORES_SOFTMAX && gate->scores != MOE_SCORES_SIGMOID) return MOE_ERR_SHAPE;
  if (gate->groups < 1 || gate->groups > D->E || D->E % gate->groups || gate->groups_kept < 1 || gate->groups_kept > gate->groups) return MOE_ERR_SHAPE;
  const int size = D->E / gate->groups;
  if (gate->group_best < 1 || gate->group_best > 2 || gate->group_best > size || D->k > gate->groups_kept * size) return MOE_ERR_SHAPE;
  if (!(gate->scale > 0.f) || gate->scale > kMaxLogit) return MOE_ERR_SHAPE;
  *A = GateArgs{D->T, D->E, D->k, D->Es, D->renorm, gate->scores == MOE_SCORES_SIGMOID, gate->groups, gate->groups_kept,
                gate->groups > 1 ? gate->group_best : 1, gate->scale};
  return MOE_OK;
}

// W lanes per token (0: the general kernel): as few as hold its groups, and its experts 32 each; of few tokens as many as leave a lane K of them, up to a
// wavefront a SIMD: there a lane's instructions are the time.
// (Experts of a lane come in 8, 16, 24 or 32, lists in 4, 8 or 16: 65536 tokens of 192 experts in lanes of 24 17.8 us, of 32 22.2; of 128 experts, top-4,
// in lists of 4 10.5 us, of 8 11.7.)
static int gate_lanes(const GateArgs& A, GatePlan* P) {
  if (A.k > 16 || A.groups > kWave) return 0;
  int padded = 1;   // groups, filled up to a power of two
  while (padded < A.groups) padded *= 2;
  const int size = A.E / A.groups, K = A.k > 8 ? 16 : A.k > 4 ? 8 : 4;
  for (int W = K > 8 ? 16 : 8; W <= kWave; W *= 2) {
    if (padded > W) continue;
    const int lanes = W / padded, piece = (size + lanes - 1) / lanes;
    if (piece > 32) continue;
    if (piece > (K > 8 ? 16 : 8) && W < kWave && (long long)A.T * 2 * W <= kWave * kGateFewWaves) continue;
    *P = GatePlan{lanes, __builtin_ctz(lanes), size, piece};
    return W;
  }
  return 0;
}

// The form of gate_kernel, or of the general kernel (K = 0), that so many tokens run.  FULL with 64 lanes of 32 experts would be more than 1024 of these.
struct GateForm { int K, W, PER; bool full; };
static GateForm gate_form(const GateArgs& A, GatePlan* P) {
  const int W = gate_lanes(A, P), K = A.k > 8 ? 16 : A.k > 4 ? 8 : 4;
  if (!W) return {0, kWave, A.E <= 64 ? 1 : A.E <= 128 ? 2 : A.E <= 256 ? 4 : A.E <= 512 ? 8 : 16, false};
  const int per = K <= 8 && P->piece <= 8 ? 8 : P->piece <= 16 ? 16 : K <= 8 && P->piece <= 24 ? 24 : 32;
  return {K, W, per, P->piece == per && per * P->lanes_of_group * A.groups == A.E};
}

template <int K, int W, int PER>
static void launch_gate_kernel(hipStream_t st, const GateForm& F, const GateArgs& A, const GatePlan& P, const float* logits, const float* bias,
                               int32_t* topk_idx, float* topk_w) {
  constexpr int TOKENS = 4 * kWave / W;
  constexpr bool SOME_FULL = W < kWave || PER < 32;
  const dim3 grid((A.T + TOKENS - 1) / TOKENS), block(256);
  if (SOME_FULL && F.full) MOE_LAUNCH("gate", st, (gate_kernel<K, W, PER, SOME_FULL>), grid, block, 0, st, logits, bias, topk_idx, topk_w, A, P);
  else MOE_LAUNCH("gate", st, (gate_kernel<K, W, PER, false>), grid, block, 0, st, logits, bias, topk_idx, topk_w, A, P);
}
template <int K, int W>
static void launch_gate_lanes(hipStream_t st, const GateForm& F, const GateArgs& A, const GatePlan& P, const float* logits, const float* bias,
                              int32_t* topk_idx, float* topk_w) {
  constexpr int FEWEST = K <= 8 ? 8 : 16;
  if (F.PER == FEWEST) launch_gate_kernel<K, W, FEWEST>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else if (F.PER == 16) launch_gate_kernel<K, W, 16>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else if (K <= 8 && F.PER == 24) launch_gate_kernel<K, W, K <= 8 ? 24 : 32>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else launch_gate_kernel<K, W, 32>(st, F, A, P, logits, bias, topk_idx, topk_w);
}
template <int K>
static void launch_gate_lists(hipStream_t st, const GateForm& F, const GateArgs& A, const GatePlan& P, const float* logits, const float* bias,
                              int32_t* topk_idx, float* topk_w) {
  constexpr int FEWEST = K <= 8 ? 8 : 16;
  if (F.W == FEWEST) launch_gate_lanes<K, FEWEST>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else if (F.W == 16) launch_gate_lanes<K, 16>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else if (F.W == 32) launch_gate_lanes<K, 32>(st, F, A, P, logits, bias, topk_idx, topk_w);
  else launch_gate_lanes<K, 64>(st, F, A, P, logits, bias, topk_idx, topk_w);
}

static void launch_gate(hipStream_t st, const GateArgs& all, const float* logits, const float* bias, int32_t* topk_idx, float* topk_w) {
  GateArgs A = all;
  if (A.T > kGateTokens) {
    for (long long t = 0; t < all.T; t += kGateTokens) {
      A.T = (int)(all.T - t < kGateTokens ? all.T - t : kGateTokens);
      launch_gate(st, A, logits + (size_t)t * A.E, bias, topk_idx + (size_t)t * (A.k + A.Es), topk_w + (size_t)t * (A.k + A.Es));
    }
    return;
  }
  GatePlan P;
  const GateForm F = gate_form(A, &P);
  if (F.K == 4) return launch_gate_lists<4>(st, F, A, P, logits, bias, topk_idx, topk_w);
  if (F.K == 8) return launch_gate_lists<8>(st, F, A, P, logits, bias, topk_idx, topk_w);
  if (F.K == 16) return launch_gate_lists<16>(st, F, A, P, logits, bias, topk_idx, topk_w);
  const dim3 grid((A.T + 3) / 4), block(256);
#define MOE_LAUNCH_GATE(PER) MOE_LAUNCH("gate_general", st, (gate_general_kernel<PER>), grid, block, 0, st, logits, bias, topk_idx, topk_w, A)
  if (F.PER == 1) MOE_LAUNCH_GATE(1);
  else if (F.PER == 2) MOE_LAUNCH_GATE(2);
  else if (F.PER == 4) MOE_LAUNCH_GATE(4);
  else if (F.PER == 8) MOE_LAUNCH_GATE(8);
  else MOE_LAUNCH_GATE(16);
#undef MOE_LAUNCH_GATE
}

}  // namespace moe

extern "C" int moe_gate_fwd(const moe_shape* shape, const moe_gate* gate, const float* logits, const float* bias, int32_t* topk_idx,
                            float* topk_w, void* stream) {
  using namespace moe;
  Dims D;
  GateArgs A;
  const int rc = gate_checks(shape, gate, &D, &A);
  if (rc != MOE_OK) return rc;
  if (D.T == 0) return MOE_OK;   // (tensors without elements may be NULL)
  MOE_REQUIRE_PTR(logits); MOE_REQUIRE_PTR(topk_idx); MOE_REQUIRE_PTR(topk_w);
  MOE_REQUIRE_ALIGNED(logits); MOE_REQUIRE_ALIGNED(bias); MOE_REQUIRE_ALIGNED(topk_idx); MOE_REQUIRE_ALIGNED(topk_w);
  launch_gate((hipStream_t)stream, A, logits, bias, topk_idx, topk_w);
  return launch_status();
}

extern "C" int moe_gate_form(const moe_shape* shape, const moe_gate* gate, int32_t* form) {
  using namespace moe;
  Dims D;
  GateArgs A;
  const int rc = gate_checks(shape, gate, &D, &A);
  if (rc != MOE_OK) return rc;
  MOE_REQUIRE_PTR(form);
  GatePlan P;
  A.T = D.T < kGateTokens ? D.T : kGateTokens;
  const GateForm F = gate_form(A, &P);
  form[0] = F.K; form[1] = F.W; form[2] = F.PER; form[3] = F.full;
  return MOE_OK;
}

extern "C" int moe_router_gate_fwd(const moe_shape* shape, const moe_gate* gate, const uint16_t* x, const uint16_t* w_router, const float* bias,
                                   float* logits, int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  Dims D;
  GateArgs A;
  int rc = gate_checks(shape, gate, &D, &A, kMaxExperts);   // (as moe_router_fwd)
  if (rc != MOE_OK) return rc;
  if (D.T == 0) return MOE_OK;   // (tensors without elements may be NULL)
  MOE_REQUIRE_PTR(topk_idx); MOE_REQUIRE_PTR(topk_w);
  MOE_REQUIRE_ALIGNED(bias); MOE_REQUIRE_ALIGNED(topk_idx); MOE_REQUIRE_ALIGNED(topk_w);
  rc = moe_router_fwd(shape, x, w_router, logits, ws, ws_bytes, stream);
  if (rc != MOE_OK) return rc;
  launch_gate((hipStream_t)stream, A, logits, bias, topk_idx, topk_w);
  return launch_status();
}

extern "C" int moe_gate_bwd(const moe_shape* shape, const moe_gate* gate, const float* dtopk_w, const float* logits, const int32_t* topk_idx,
                            const float* topk_w, const int32_t* counts, float balance, float* dlogits, float* loss, void* ws, size_t ws_bytes,
                            void* stream) {
  using namespace moe;
  Dims D;
  GateArgs A;
  const int rc = gate_checks(shape, gate, &D, &A);
  if (rc != MOE_OK) return rc;
  if (D.T > 0) {   // (tensors without elements may be NULL)
    MOE_REQUIRE_PTR(dtopk_w); MOE_REQUIRE_PTR(logits); MOE_REQUIRE_PTR(topk_idx); MOE_REQUIRE_PTR(topk_w); MOE_REQUIRE_PTR(dlogits);
  }
  MOE_REQUIRE_ALIGNED(dtopk_w); MOE_REQUIRE_ALIGNED(logits); MOE_REQUIRE_ALIGNED(topk_idx); MOE_REQUIRE_ALIGNED(topk_w); MOE_REQUIRE_ALIGNED(dlogits);
  MOE_REQUIRE_ALIGNED(counts); MOE_REQUIRE_ALIGNED(loss);
  if (counts && !(balance >= -kMaxLogit && balance <= kMaxLogit)) return MOE_ERR_SHAPE;   // (without counts it is not read)
  // lanes of a token, and its chunks of 4 experts a lane: up to 16 experts 4 each; else up to 4 chunks, one by one 3 (of 64 lanes 4).
  // (Chunks of 3 beside 1, 2 and 4: 65536 x 160 22 -> 19.6 us, 32768 x 384 26.5 -> 23.9, 30000 x 190 20 -> 13.8.)
  const bool vec = D.E % 4 == 0;
  int W = vec && D.E <= 8 ? 2 : vec && D.E <= 16 ? 4 : 8;
  while (W < kWave && (vec ? 16 : 12) * W < D.E) W *= 2;
  const int chunks = (D.E + 4 * W - 1) / (4 * W);
  const long long units = ((long long)D.T + kGateBwdWaves * (kWave / W) - 1) / (kGateBwdWaves * (kWave / W));
  // With the loss, one or two batches of tokens a wavefront stay in one block, which then has the whole sum: a launch less.  (On the device, of 8 and of
  // 256 experts: one batch 3.0 for 4.5 us and 4.9 for 6.3, two 4.1 for 4.7 and 7.4 for 6.5, four 6.1 for 4.7 and 12.4 for 6.5; a call's own launch 3 us.)
  const bool alone = loss && D.T > 0 && units <= 2;
  const int blocks = (int)(alone ? 1 : units < kGateBwdBlocks ? units : kGateBwdBlocks);
  if (loss) {
    MOE_REQUIRE_PTR(counts); MOE_REQUIRE_PTR(ws);
    if (!aligned(ws, 256)) return MOE_ERR_ALIGN;
    if (ws_bytes < 4096) return MOE_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  if (D.T > 0) {
    const float cost = (float)((double)balance * D.E / ((double)D.k * D.T * D.T));
    float* parts = alone ? loss : loss ? (float*)ws : nullptr;
#define MOE_LAUNCH_GATE_BWD(W_, C_, VEC_)                                                                                                             \
  MOE_LAUNCH("gate_bwd", st, (gate_bwd_kernel<W_, C_, VEC_>), dim3(blocks), dim3(kGateBwdWaves * kWave), 0, st, dtopk_w, logits, topk_idx, topk_w, counts, \
             cost, dlogits, parts, A)
#define MOE_LAUNCH_GATE_BWD_EITHER(few, W_, FEW_, MANY_, VEC_) \
  do {                                                         \
    if (few) MOE_LAUNCH_GATE_BWD(W_, FEW_, VEC_);              \
    else MOE_LAUNCH_GATE_BWD(W_, MANY_, VEC_);                 \
  } while (0)
    if (vec) {
      if (W == 2) MOE_LAUNCH_GATE_BWD(2, 1, true);
      else if (W == 4) MOE_LAUNCH_GATE_BWD(4, 1, true);
      else if (W == 8 && chunks <= 2) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 1, 8, 1, 2, true);
      else if (W == 8) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 3, 8, 3, 4, true);
      else if (W == 16) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 3, 16, 3, 4, true);
      else if (W == 32) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 3, 32, 3, 4, true);
      else MOE_LAUNCH_GATE_BWD_EITHER(chunks == 3, 64, 3, 4, true);
    } else {
      if (chunks == 1) MOE_LAUNCH_GATE_BWD(8, 1, false);
      else if (W == 8) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 2, 8, 2, 3, false);
      else if (W == 16) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 2, 16, 2, 3, false);
      else if (W == 32) MOE_LAUNCH_GATE_BWD_EITHER(chunks == 2, 32, 2, 3, false);
      else if (chunks == 4) MOE_LAUNCH_GATE_BWD(64, 4, false);
      else MOE_LAUNCH_GATE_BWD_EITHER(chunks == 2, 64, 2, 3, false);
    }
#undef MOE_LAUNCH_GATE_BWD_EITHER
#undef MOE_LAUNCH_GATE_BWD
  }
  if (loss && !alone) MOE_LAUNCH("gate_loss", st, gate_loss_kernel, dim3(1), dim3(256), 0, st, (const float*)ws, blocks, loss);
  return launch_status();
}

extern "C" int moe_gate_bias_step(const moe_shape* shape, const int32_t* counts, float rate, float* bias, void* stream) {
  using namespace moe;
  Dims D;
  const int rc = check_shape(shape, &D, kGateIds);
  if (rc != MOE_OK) return rc;
  MOE_REQUIRE_PTR(counts); MOE_REQUIRE_PTR(bias);
  MOE_REQUIRE_ALIGNED(counts); MOE_REQUIRE_ALIGNED(bias);
  if (!(rate >= 0.f && rate <= kMaxLogit)) return MOE_ERR_SHAPE;
  if (D.T == 0) return MOE_OK;
  MOE_LAUNCH("gate_bias_step", (hipStream_t)stream, gate_bias_step_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, counts, D.E, rate, bias);
  return launch_status();
}
