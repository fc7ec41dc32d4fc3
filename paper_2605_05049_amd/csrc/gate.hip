// Routing to experts with softmax or sigmoid scores, a bias that balances, groups of experts, and the gradient of its weights.
//
//   s = softmax(l) or 1 / (1 + exp(-l)) over the E logits of a token;  c = s + bias (without a bias: l, of which s is a monotone function)
//   a group of E / groups neighbouring experts has as score the sum of its `group_best` best c;  the groups_kept best groups stay
//   the k best c among them are chosen, ties to the lowest id;  w_j = scale s_j / sum_i s_i  or  scale s_j
//
// Decisions (which groups, which experts, in which order) are those of scores in 64 bits; the weights are fp32.
#include "common.h"

namespace moe {

constexpr float kMaskedLogit = -1e30f;   // logits up to it, and NaN, are no experts to choose
constexpr float kMaxLogit = 3.402823466e38f;
constexpr int kGateBwdBlocks = 4096;      // at most; each adds up its tokens' share of the loss

struct GateArgs {
  int T, E, k, Es, renorm;
  int sigmoid, groups, groups_kept, group_best;
  float scale;
};

__device__ __forceinline__ bool gate_masked(float l) { return !(l > kMaskedLogit); }
__device__ __forceinline__ float gate_finite(float l) { return l > kMaxLogit ? kMaxLogit : l; }   // (NaN stays)

template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, W);
  return v;
}
template <int W>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, W));
  return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// sigmoid(l) / sigmoid-like factor exp(top) with top = min(0, the largest logit that is looked at): scores far below zero keep their ratios.
__device__ __forceinline__ float sigmoid_over(float l, float top) { return 1.0f / (expf(top - l) + expf(top)); }

// Any number of groups and experts, any k: a wavefront per token, lane g holds experts g, g + 64, ..., everything in 64 bits.  k rounds of finding
// the best one left.
template <int PER>
__global__ __launch_bounds__(256) void gate_general_kernel(const float* __restrict__ logits, const float* __restrict__ bias,
                                                           int32_t* __restrict__ topk_idx, float* __restrict__ topk_w, GateArgs A) {
  __shared__ double row_c[4][PER * kWave];    // c of every expert, for the groups' scores
  __shared__ double group_c[4][PER * kWave];  // the groups' scores
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int t = blockIdx.x * 4 + wave;
  if (t >= A.T) return;   // (whole wavefronts; no barrier below)
  const int E = A.E, k = A.k, Kp = k + A.Es;
  const double NEG = -__builtin_inf();
  const float* row = logits + (size_t)t * E;
  float l[PER];
  float m = -kMaxLogit;
#pragma unroll
  for (int p = 0; p < PER; p++) {
    const int e = lane + p * kWave;
    l[p] = e < E ? gate_finite(row[e]) : -__builtin_inff();
    if (!gate_masked(l[p])) m = fmaxf(m, l[p]);
  }
  m = lanes_max<kWave>(m);
  const bool by_logits = bias == nullptr, need_scores = !by_logits || A.group_best > 1 || (!A.sigmoid && !A.renorm);
  double s[PER];
#pragma unroll
  for (int p = 0; p < PER; p++) s[p] = 0.0;
  if (need_scores) {
    double z = 0.0;
#pragma unroll
    for (int p = 0; p < PER; p++)
      if (!gate_masked(l[p])) {
        s[p] = A.sigmoid ? 1.0 / (1.0 + exp(-(double)l[p])) : exp((double)l[p] - (double)m);
        z += s[p];
      }
    if (!A.sigmoid) {
      z = wave_sum_f64(z);
#pragma unroll
      for (int p = 0; p < PER; p++)
        if (!gate_masked(l[p])) s[p] /= z;
    }
  }
  double c[PER];
  bool taken[PER];
#pragma unroll
  for (int p = 0; p < PER; p++) {
    const int e = lane + p * kWave;
    taken[p] = e >= E;
    c[p] = NEG;
    if (e < E && !gate_masked(l[p])) {
      const double b = by_logits ? (double)l[p] : s[p] + (double)bias[e];
      c[p] = b == b ? b : NEG;
    }
  }
  if (A.groups > 1) {
    const int S = E / A.groups;
    const bool by_score = by_logits && A.group_best > 1;   // (a sum of logits would say nothing)
#pragma unroll
    for (int p = 0; p < PER; p++)
      if (lane + p * kWave < E) row_c[wave][lane + p * kWave] = by_score && c[p] != NEG ? s[p] : c[p];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int g = lane; g < A.groups; g += kWave) {
      double first = NEG, second = NEG;
      for (int i = 0; i < S; i++) {
        const double v = row_c[wave][g * S + i];
        second = fmax(second, fmin(first, v));
        first = fmax(first, v);
      }
      group_c[wave][g] = A.group_best > 1 && second != NEG ? first + second : first;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int p = 0; p < PER; p++) {
      const int e = lane + p * kWave;
      if (e < E) {
        const int g = e / S;
        const double v = group_c[wave][g];
        int better = 0;
        for (int o = 0; o < A.groups; o++) {
          const double u = group_c[wave][o];
          better += u > v || (u == v && o < g);
        }
        if (better >= A.groups_kept) taken[p] = true;
      }
    }
  }
  // selection j stays on lane j % 64, slot j / 64, until all are known
  int held[PER];
#pragma unroll
  for (int p = 0; p < PER; p++) held[p] = 0;
  for (int j = 0; j < k; j++) {
    double bv = NEG;
    int bi = 0x7fffffff;
#pragma unroll
    for (int p = 0; p < PER; p++)
      if (!taken[p] && (c[p] > bv || (c[p] == bv && lane + p * kWave < bi))) { bv = c[p]; bi = lane + p * kWave; }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
      const double ov = __shfl_xor(bv, o, kWave);
      const int oi = __shfl_xor(bi, o, kWave);
      if (ov > bv || (ov == bv && oi < bi)) { bv = ov; bi = oi; }
    }
#pragma unroll
    for (int p = 0; p < PER; p++) {
      if (lane + p * kWave == bi) taken[p] = true;
      if (lane == j % kWave && p == j / kWave) held[p] = bi;
    }
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
    if (!A.sigmoid) {
      z = 0.f;
#pragma unroll
      for (int p = 0; p < PER; p++)
        if (!gate_masked(l[p])) z += expf(l[p] - m);
      z = lanes_sum<kWave>(z);
    }
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

// Gradient of the weights and of the balance loss.  A wavefront per token, lane g holds experts g, g + 64, ...; with q = s / sum s, n_e the slots
// of expert e, C_e = balance E n_e / (k T^2):
//   softmax  dl_m = q_m (C_m - <q, C>) [- s_m <w, dw> where not renormalised] + d_j of the slots with expert m
//   sigmoid  dl_m = (1 - s_m) (q_m (C_m - <q, C>) + d_j)
//   d_j = w_j (dw_j - <w, dw> / scale) where renormalised, else w_j dw_j
template <int PER>
__global__ __launch_bounds__(256) void gate_bwd_kernel(const float* __restrict__ dtopk_w, const float* __restrict__ logits,
                                                       const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w,
                                                       const int32_t* __restrict__ counts, float cost, float* __restrict__ dlogits,
                                                       float* __restrict__ loss_part, GateArgs A) {
  __shared__ float part[4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int E = A.E, k = A.k, Kp = k + A.Es;
  const bool dense = counts != nullptr || (!A.sigmoid && !A.renorm);
  float loss = 0.f;
  for (int t = blockIdx.x * 4 + wave; t < A.T; t += gridDim.x * 4) {
    const float* dw = dtopk_w + (size_t)t * Kp;
    const float* w = topk_w + (size_t)t * Kp;
    const int32_t* idx = topk_idx + (size_t)t * Kp;
    const float* row = logits + (size_t)t * E;
    float inner = 0.f;
    for (int j = lane; j < k; j += kWave) inner += w[j] * dw[j];
    inner = lanes_sum<kWave>(inner);
    float v[PER], slope[PER];
#pragma unroll
    for (int p = 0; p < PER; p++) { v[p] = 0.f; slope[p] = 1.f; }
    if (dense || A.sigmoid) {
      float l[PER], s[PER], m = -kMaxLogit, z = 0.f, mean = 0.f;
#pragma unroll
      for (int p = 0; p < PER; p++) {
        const int e = lane + p * kWave;
        l[p] = e < E ? gate_finite(row[e]) : -__builtin_inff();
        if (!gate_masked(l[p])) m = fmaxf(m, l[p]);
      }
      m = lanes_max<kWave>(m);
      const float top = A.sigmoid ? fminf(m, 0.f) : m;   // (scores over exp(top))
#pragma unroll
      for (int p = 0; p < PER; p++) {
        s[p] = gate_masked(l[p]) ? 0.f : A.sigmoid ? sigmoid_over(l[p], top) : expf(l[p] - top);
        if (A.sigmoid) slope[p] = gate_masked(l[p]) ? 0.f : 1.0f / (1.0f + expf(l[p]));
        z += s[p];
      }
      if (dense) {
        z = lanes_sum<kWave>(z);
        const float inv = z > 0.f ? 1.0f / z : 0.f;
        float C[PER];
#pragma unroll
        for (int p = 0; p < PER; p++) {
          const int e = lane + p * kWave;
          C[p] = counts && e < E ? cost * (float)counts[e] : 0.f;
          s[p] *= inv;
          mean += s[p] * C[p];
        }
        mean = lanes_sum<kWave>(mean);
        loss += mean;
#pragma unroll
        for (int p = 0; p < PER; p++) {
          v[p] = s[p] * (C[p] - mean);
          if (!A.sigmoid && !A.renorm) v[p] -= s[p] * inner;
        }
      }
    }
    for (int j = 0; j < k; j++) {
      const int e = idx[j];
      const float d = A.renorm ? w[j] * (dw[j] - inner / A.scale) : w[j] * dw[j];
#pragma unroll
      for (int p = 0; p < PER; p++)
        if (e == lane + p * kWave) v[p] += d;
    }
#pragma unroll
    for (int p = 0; p < PER; p++) {
      const int e = lane + p * kWave;
      if (e < E) dlogits[(size_t)t * E + e] = v[p] * slope[p];
    }
  }
  if (loss_part) {
    if (lane == 0) part[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0) loss_part[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
  }
}

// The sum of the blocks' parts, in a fixed order.
__global__ __launch_bounds__(256) void gate_loss_kernel(const float* __restrict__ loss_part, int parts, float* __restrict__ loss) {
  __shared__ double sum[256];
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) v += (double)loss_part[i];
  sum[threadIdx.x] = v;
  for (int o = 128; o > 0; o >>= 1) {
    __syncthreads();
    if (threadIdx.x < o) sum[threadIdx.x] += sum[threadIdx.x + o];
  }
  if (threadIdx.x == 0) *loss = (float)sum[0];
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
static int gate_checks(const moe_shape* shape, const moe_gate* gate, Dims* D, GateArgs* A) {
  const int rc = check_shape(shape, D);
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

static void launch_gate(hipStream_t st, const GateArgs& A, const float* logits, const float* bias, int32_t* topk_idx, float* topk_w) {
  const dim3 grid((A.T + 3) / 4), block(256);
#define MOE_LAUNCH_GATE(PER) MOE_LAUNCH("gate_general", st, (gate_general_kernel<PER>), grid, block, 0, st, logits, bias, topk_idx, topk_w, A)
  if (A.E <= 64) MOE_LAUNCH_GATE(1);
  else if (A.E <= 128) MOE_LAUNCH_GATE(2);
  else if (A.E <= 256) MOE_LAUNCH_GATE(4);
  else if (A.E <= 512) MOE_LAUNCH_GATE(8);
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

extern "C" int moe_router_gate_fwd(const moe_shape* shape, const moe_gate* gate, const uint16_t* x, const uint16_t* w_router, const float* bias,
                                   float* logits, int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  Dims D;
  GateArgs A;
  int rc = gate_checks(shape, gate, &D, &A);
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
  if (!(balance >= -kMaxLogit && balance <= kMaxLogit)) return MOE_ERR_SHAPE;
  const int blocks = D.T < 4 * kGateBwdBlocks ? (D.T + 3) / 4 : kGateBwdBlocks;
  if (loss) {
    MOE_REQUIRE_PTR(counts); MOE_REQUIRE_PTR(ws);
    if (!aligned(ws, 256)) return MOE_ERR_ALIGN;
    if (ws_bytes < (size_t)kGateBwdBlocks * sizeof(float)) return MOE_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  if (D.T > 0) {
    const float cost = (float)((double)balance * D.E / ((double)D.k * D.T * D.T));
    float* parts = loss ? (float*)ws : nullptr;
#define MOE_LAUNCH_GATE_BWD(PER) \
  MOE_LAUNCH("gate_bwd", st, (gate_bwd_kernel<PER>), dim3(blocks), dim3(256), 0, st, dtopk_w, logits, topk_idx, topk_w, counts, cost, dlogits, parts, A)
    if (D.E <= 64) MOE_LAUNCH_GATE_BWD(1);
    else if (D.E <= 128) MOE_LAUNCH_GATE_BWD(2);
    else if (D.E <= 256) MOE_LAUNCH_GATE_BWD(4);
    else if (D.E <= 512) MOE_LAUNCH_GATE_BWD(8);
    else MOE_LAUNCH_GATE_BWD(16);
#undef MOE_LAUNCH_GATE_BWD
  }
  if (loss) MOE_LAUNCH("gate_loss", st, gate_loss_kernel, dim3(1), dim3(256), 0, st, (const float*)ws, blocks, loss);
  return launch_status();
}

extern "C" int moe_gate_bias_step(const moe_shape* shape, const int32_t* counts, float rate, float* bias, void* stream) {
  using namespace moe;
  Dims D;
  const int rc = check_shape(shape, &D);
  if (rc != MOE_OK) return rc;
  MOE_REQUIRE_PTR(counts); MOE_REQUIRE_PTR(bias);
  MOE_REQUIRE_ALIGNED(counts); MOE_REQUIRE_ALIGNED(bias);
  if (!(rate >= 0.f && rate <= kMaxLogit)) return MOE_ERR_SHAPE;
  if (D.T == 0) return MOE_OK;
  MOE_LAUNCH("gate_bias_step", (hipStream_t)stream, gate_bias_step_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, counts, D.E, rate, bias);
  return launch_status();
}
