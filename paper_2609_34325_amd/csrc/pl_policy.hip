// The clipped policy loss of ordered Plackett-Luce draws and its gradient with
// respect to the removal scores.  DORA (arXiv 2609.34325): App. A.3, Eq.
// (app-actor-pl) (the ordered log-probability of a selection) and App. D
// (clipped updates of the selector).
//
// Draws i_0 .. i_{k-1} of an image with visual scores s:
//   S_t = sum of exp(s_j) over the tokens left before draw t
//   logp = sum_t s_{i_t} - log S_t
//   d logp / d s_j = [j drawn] - exp(s_j) sum_{t <= tau_j} 1 / S_t
// with tau_j the draw that takes j, or k - 1 for a token never drawn.  Both
// sums are scans along the drawing order: the S_t from the back (the tokens
// left at the end are one term), the sums of 1 / S_t from the front.  Terms
// and sums are pairs v 2^e with 64-bit v, joined at the larger e by shifting
// exponents: a score far below the largest, drawn late, neither vanishes nor
// divides zero by zero, and no exp is taken inside the scans.  64 bits because
// logp sums up to 2047 logarithms of running sums and the loss takes exp of
// its difference to the old one.
//
// One workgroup per image; launch and barrier latency bound (an image is a few
// KB).  Loss terms per image go to the workspace and are added by a second
// launch in a fixed order.
#include "dora_internal.h"
#include "policy_terms.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSlots = DORA_MAX_ROW_TOKENS;
constexpr double kNever = -1e300;  // exponent of no term
constexpr double kLog2E = 1.4426950408889634, kLn2 = 0.6931471805599453;

struct PLPolicyParams {
  const float* s;
  const int32_t* order;
  const int32_t* cu_order;
  const int32_t* cu_in;
  int64_t total_in;
  const float* old;
  const float* ref;
  const float* adv;
  const float* weight;
  int32_t B, N;
  PolicyCoef coef;
  float* grad;
  float* logp;
  double* parts;
  int32_t* status;
};

// v 2^e, e a whole number (64 bits hold one for every fp32 score).
struct Scaled {
  double v, e;
};
__device__ __forceinline__ double shifted(Scaled x, double e) {
  return ldexp(x.v, static_cast<int>(fmax(x.e - e, -4000.0)));
}
__device__ __forceinline__ Scaled operator+(Scaled x, Scaled y) {
  const double e = fmax(x.e, y.e);
  return {shifted(x, e) + shifted(y, e), e};
}
__device__ __forceinline__ Scaled exp_of(float x) {
  const double y = x * kLog2E, e = floor(y);
  return {exp2(y - e), e};
}
__device__ __forceinline__ Scaled shfl_down(Scaled x, int d) { return {__shfl_down(x.v, d), __shfl_down(x.e, d)}; }
__device__ __forceinline__ Scaled shfl_up(Scaled x, int d) { return {__shfl_up(x.v, d), __shfl_up(x.e, d)}; }

// Sum of the values of the threads after (before, if FRONT) this one.
template <bool FRONT>
__device__ Scaled scan_others(Scaled own, Scaled* s_red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Scaled incl = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Scaled y = FRONT ? shfl_up(incl, d) : shfl_down(incl, d);
    if (FRONT ? lane >= d : lane + d < 64) incl = incl + y;
  }
  Scaled excl = FRONT ? shfl_up(incl, 1) : shfl_down(incl, 1);
  if (lane == (FRONT ? 0 : 63)) excl = {0.0, kNever};
  __syncthreads();
  if (lane == (FRONT ? 63 : 0)) s_red[wave] = incl;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w)
    if (FRONT ? w < wave : w > wave) excl = excl + s_red[w];
  return excl;
}

__global__ __launch_bounds__(kThreads) void pl_policy_kernel(PLPolicyParams p) {
  __shared__ float s_x[kSlots];       // visual scores by position - 1
  __shared__ int s_rank[kSlots];      // draw that takes the position, -1: none
  __shared__ Scaled s_exp[kSlots];    // exp of the scores
  __shared__ Scaled s_front[kSlots];  // sum over the draws up to and with t of 1 / S
  __shared__ Scaled s_red[kWaves];
  __shared__ double s_sum[kWaves];
  __shared__ int s_bad;
  const int b = blockIdx.x, tid = threadIdx.x;

  int64_t off;
  int n;
  bool seg_ok = true;
  if (p.cu_in) {
    const int lo = p.cu_in[b], hi = p.cu_in[b + 1];
    off = lo;
    n = hi - lo;
    seg_ok = lo >= 0 && hi > lo && n <= p.N && hi <= p.total_in && (b > 0 || lo == 0);
  } else {
    off = static_cast<int64_t>(b) * p.N;
    n = p.N;
  }
  const int nv = seg_ok ? n - 1 : 0;
  const float w = p.weight ? p.weight[b] : 1.0f;
  const int o0 = p.cu_order[b], o1 = p.cu_order[b + 1], oend = p.cu_order[p.B];
  const int k = (o0 >= 0 && o1 >= o0 && o1 <= oend && p.cu_order[0] == 0) ? o1 - o0 : -1;
  const bool on = seg_ok && w != 0.0f;
  bool ok = on && k >= 0 && k <= nv;

  if (tid == 0) s_bad = 0;
  for (int j = tid; j < nv; j += kThreads) {
    const float x = p.s[off + j + 1];
    s_x[j] = x;
    s_exp[j] = exp_of(x);
    s_rank[j] = -1;
  }
  __syncthreads();
  if (ok) {
    for (int t = tid; t < k; t += kThreads) {
      const int pos = p.order[o0 + t];
      if (pos < 1 || pos > nv || atomicCAS(&s_rank[pos - 1], -1, t) != -1) s_bad = 1;
    }
  }
  __syncthreads();
  ok = ok && s_bad == 0;
  if (!ok) {
    for (int j = tid; seg_ok && j < n; j += kThreads) p.grad[off + j] = 0.0f;
    if (tid < kPolicyTerms) p.parts[static_cast<int64_t>(b) * kPolicyTerms + tid] = 0.0;
    if (tid == 0) {
      p.logp[b] = seg_ok && w == 0.0f ? 0.0f : __builtin_nanf("");
      if (!seg_ok) atomicOr(p.status, DORA_DEV_CU_IN);
      else if (w != 0.0f) atomicOr(p.status, DORA_DEV_KEEP_RANGE);
    }
    return;
  }

  // The tokens left at the end: one term after the last draw.
  Scaled left{0.0, kNever};
  for (int j = tid; j < nv; j += kThreads)
    if (s_rank[j] < 0) left = left + s_exp[j];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) left = left + Scaled{__shfl_xor(left.v, d), __shfl_xor(left.e, d)};
  if ((tid & 63) == 0) s_red[tid >> 6] = left;
  __syncthreads();
  left = s_red[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) left = left + s_red[i];
  __syncthreads();  // s_red is used again

  // S from the back.  Thread i scans the draws [i c, (i + 1) c); the last one adds what is left.
  const int c = (k + kThreads - 1) / kThreads, first = min(k, tid * c), last = min(k, first + c);
  Scaled own = tid == kThreads - 1 ? left : Scaled{0.0, kNever};
  for (int t = last - 1; t >= first; --t) own = own + s_exp[p.order[o0 + t] - 1];
  Scaled run = scan_others<false>(own, s_red);
  if (tid == kThreads - 1) run = left;
  double lp = 0.0;
  own = {0.0, kNever};
  for (int t = last - 1; t >= first; --t) {
    const int pos = p.order[o0 + t] - 1;
    run = run + s_exp[pos];
    lp += s_x[pos] - (log(run.v) + run.e * kLn2);
    const Scaled inv{1.0 / run.v, -run.e};
    s_front[t] = inv;
    own = own + inv;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) lp += __shfl_xor(lp, d);
  if ((tid & 63) == 0) s_sum[tid >> 6] = lp;

  // Sums of 1 / S from the front (the scan's barriers cover s_sum too).
  run = scan_others<true>(own, s_red);
  for (int t = first; t < last; ++t) {
    run = run + s_front[t];
    s_front[t] = run;
  }
  __syncthreads();
  lp = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) lp += s_sum[i];

  PolicyTerms terms{};
  const double slope = policy_decision(lp, 0.0, p.old[b], p.adv[b], w, p.ref != nullptr,
                                       p.ref ? p.ref[b] : 0.0f, p.coef, terms);
  if (tid == 0) {
    p.logp[b] = static_cast<float>(lp);
#pragma unroll
    for (int i = 0; i < kPolicyTerms; ++i) p.parts[static_cast<int64_t>(b) * kPolicyTerms + i] = terms.v[i];
    p.grad[off] = 0.0f;  // CLS is never drawn
  }
  for (int j = tid; j < nv; j += kThreads) {
    float g = 0.0f;
    if (k > 0) {
      const int r = s_rank[j];
      const Scaled f = s_front[r < 0 ? k - 1 : r], e = s_exp[j];
      g = static_cast<float>(slope * ((r < 0 ? 0.0 : 1.0) - shifted({e.v * f.v, e.e + f.e}, 0.0)));
    }
    p.grad[off + j + 1] = g;
  }
}

}  // namespace
}  // namespace dora

extern "C" size_t dora_pl_policy_workspace_size(int32_t B) {
  using namespace dora;
  if (B < 1 || B > kPlanMaxB) return 0;
  return policy_parts_bytes(B);
}

extern "C" int dora_pl_policy_loss(const float* scores, const int32_t* order, const int32_t* cu_order,
                                   const int32_t* cu_in, int64_t total_in, const float* old_logprob,
                                   const float* ref_logprob, const float* advantage, const float* weight, int32_t B,
                                   int32_t N, float clip_low, float clip_high, float kl_coef, float* dscores,
                                   float* logprob_out, float* stats_out, void* workspace, size_t workspace_bytes,
                                   int32_t* dev_status, void* stream) {
  using namespace dora;
  if (!scores || !order || !cu_order || !old_logprob || !advantage || !dscores || !logprob_out || !stats_out ||
      !dev_status)
    return DORA_ERR_NULL;
  if (B < 1 || B > kPlanMaxB || N < 1 || N > DORA_MAX_ROW_TOKENS) return DORA_ERR_SHAPE;
  if (cu_in && (total_in < 0 || total_in > 0x7FFFFFFF)) return DORA_ERR_SHAPE;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f) || !(kl_coef - kl_coef == 0.0f))
    return DORA_ERR_SHAPE;
  if (kl_coef != 0.0f && !ref_logprob) return DORA_ERR_NULL;
  const uintptr_t sa = reinterpret_cast<uintptr_t>(scores), ga = reinterpret_cast<uintptr_t>(dscores);
  const uintptr_t len = static_cast<uintptr_t>(cu_in ? total_in : static_cast<int64_t>(B) * N) * sizeof(float);
  if (sa != ga && sa < ga + len && ga < sa + len) return DORA_ERR_OVERLAP;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u ||
      workspace_bytes < dora_pl_policy_workspace_size(B))
    return DORA_ERR_WORKSPACE;
  PLPolicyParams p{scores, order, cu_order, cu_in, total_in, old_logprob, ref_logprob, advantage, weight, B, N,
                   PolicyCoef{clip_low, clip_high, kl_coef, 0.0f}, dscores, logprob_out,
                   static_cast<double*>(workspace), dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(pl_policy_kernel, dim3(B), dim3(kThreads), 0, st, p);
  launch_policy_finish(p.parts, B, stats_out, st);
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
