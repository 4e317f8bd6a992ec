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
// left at the end are one term), the sums of 1 / S_t from the front.  64 bits,
// because logp sums up to 2047 logarithms of running sums and the loss takes
// exp of its difference to the old one.  Terms are relative to the image's
// largest score while all are within 2^900 of it, else pairs v 2^e, joined at
// the larger e by shifting exponents: a score however far below, drawn late,
// neither vanishes nor divides zero by zero.  A score of -inf is a token that
// counts for nothing in either form.
//
// One workgroup per image; launch, memory and barrier latency bound (an image
// is a few KB): 256 x 577 tokens 7.4 us, 48 x 2048 11.8, 8192 x 257 29.
// Shared memory is sized by N, so that several images share a compute unit.
// Loss terms per image go to the workspace and are added by a second launch in
// a fixed order.
#include "dora_internal.h"
#include "policy_terms.h"

namespace dora {
namespace {

constexpr double kLog2E = 1.4426950408889634, kLn2 = 0.6931471805599453;

struct PLPolicyParams {
  const float* s;
  const int32_t* order;
  const int32_t* cu_order;
  int64_t cap;  // entries of the order
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
  float* stats;
  int32_t* status;
};

// exp(x - top), where every score is within 2^900 of the largest, top.
struct Plain {
  double v;
  __device__ static Plain zero() { return {0.0}; }
  __device__ static Plain exp_of(float x, double top) { return {exp2((x - top) * kLog2E)}; }
  __device__ Plain operator+(Plain o) const { return {v + o.v}; }
  __device__ Plain inverse() const { return {1.0 / v}; }
  // log of exp(x) over this sum.
  __device__ double share_of(float x, double top) const { return (x - top) - log(v); }
  __device__ double times(Plain o) const { return v * o.v; }
};

// v 2^e, e a whole number (64 bits hold one for every fp32 score).
struct Scaled {
  double v, e;
  __device__ static Scaled zero() { return {0.0, -1e300}; }
  // Rounded before anything is taken from it: the rest that a fused step would
  // keep is 1e22 for the lowest score (a mask), and differs between 0 and that
  // for what is equal.
  __device__ static double log2_of(float x) {
#pragma clang fp contract(off)
    return x * kLog2E;
  }
  __device__ static Scaled exp_of(float x, double) {
    if (x == -__builtin_inff()) return zero();
    const double y = log2_of(x), e = floor(y);
    return {exp2(y - e), e};
  }
  __device__ double at(double to) const { return ldexp(v, static_cast<int>(fmax(e - to, -4000.0))); }
  __device__ Scaled operator+(Scaled o) const {
    const double to = fmax(e, o.e);
    return {at(to) + o.at(to), to};
  }
  __device__ Scaled inverse() const { return {1.0 / v, -e}; }
  __device__ double share_of(float x, double) const { return (log2_of(x) - e) * kLn2 - log(v); }
  __device__ double times(Scaled o) const { return Scaled{v * o.v, e + o.e}.at(0.0); }
  __device__ Scaled down(int d) const { return {__shfl_down(v, d), __shfl_down(e, d)}; }
  __device__ Scaled up(int d) const { return {__shfl_up(v, d), __shfl_up(e, d)}; }
};

// Shared memory: what depends on N, 24 bytes a token.
struct Tokens {
  char* scan;     // 16 bytes a token: Scaled sums of 1 / S by draw; or Plain, and exp by position behind them
  float* x;       // visual scores by position - 1
  int16_t* rank;  // draw that takes the position, -1: none
  int16_t* draw;  // position - 1 of each draw
};
constexpr int kTokenBytes = 24;

// Sum of the values of the wave's lanes after (before, if FRONT) this one; the
// wave's whole sum goes to *total.  All lanes active.
template <bool FRONT>
__device__ __forceinline__ Scaled scan_lanes(Scaled own, Scaled* total) {
  const int lane = threadIdx.x & 63;
  Scaled incl = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Scaled y = FRONT ? incl.up(d) : incl.down(d);
    if (FRONT ? lane >= d : lane + d < 64) incl = incl + y;
  }
  total->v = __shfl(incl.v, FRONT ? 63 : 0);
  total->e = __shfl(incl.e, FRONT ? 63 : 0);
  const Scaled excl = FRONT ? incl.up(1) : incl.down(1);
  return lane == (FRONT ? 0 : 63) ? Scaled::zero() : excl;
}

// The value of the lane CTRL (a DPP shift inside a row of 16 lanes) points to, 0 past the row.
template <int CTRL>
__device__ __forceinline__ double row_shift(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                          __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// The same without shared memory: shifts inside rows of 16 lanes, and the rows'
// sums as scalars.
template <bool FRONT>
__device__ __forceinline__ Plain scan_lanes(Plain own, Plain* total) {
  constexpr int kShift = FRONT ? 0x110 : 0x100;  // row_shr, row_shl
  double v = own.v;
  v += row_shift<kShift + 1>(v);
  v += row_shift<kShift + 2>(v);
  v += row_shift<kShift + 4>(v);
  v += row_shift<kShift + 8>(v);
  constexpr int kEnd = FRONT ? 15 : 0;
  const int row = (threadIdx.x & 63) >> 4;
  const double r0 = lane_value(v, kEnd), r1 = lane_value(v, kEnd + 16), r2 = lane_value(v, kEnd + 32),
               r3 = lane_value(v, kEnd + 48);
  double others;
  if (FRONT) others = row == 0 ? 0.0 : (row == 1 ? r0 : (row == 2 ? r0 + r1 : r0 + r1 + r2));
  else others = row == 3 ? 0.0 : (row == 2 ? r3 : (row == 1 ? r3 + r2 : r3 + r2 + r1));
  total->v = (r0 + r1) + (r2 + r3);
  return {others + row_shift<kShift + 1>(v)};
}

// The image's log-probability; its sums of 1 / S by draw are left in `front`.
// Called by the whole workgroup, scores and draws being there and the ranks
// all -1; *bad is set where a position is drawn twice (what comes out then is
// of no use, but all of it stays in bounds).
template <int kThreads, class T>
__device__ __forceinline__ double scan_draws(const Tokens& s, int nv, int k, double top, T* front, int* bad) {
  constexpr int kWaves = kThreads / 64;
  constexpr bool kStored = sizeof(T) == sizeof(Plain);  // exp is looked up, not formed again
  __shared__ T s_left[kWaves], s_back[kWaves], s_front[kWaves];
  __shared__ double s_sum[kWaves];
  const int tid = threadIdx.x, wave = tid >> 6;
  T* const exps = front + nv;  // Plain only
  for (int t = tid; t < k; t += kThreads) s.rank[s.draw[t]] = static_cast<int16_t>(t);
  if constexpr (kStored)
    for (int j = tid; j < nv; j += kThreads) exps[j] = T::exp_of(s.x[j], top);
  __syncthreads();
  auto exp_at = [&](int pos) {
    if constexpr (kStored) return exps[pos];
    else return T::exp_of(s.x[pos], top);
  };
  T left = T::zero();  // the tokens never drawn
  for (int j = tid; j < nv; j += kThreads)
    if (s.rank[j] < 0) left = left + exp_at(j);
  T sum;
  scan_lanes<false>(left, &sum);
  if ((tid & 63) == 0) s_left[wave] = sum;
  // S from the back.  Thread i scans the draws [i c, (i + 1) c).
  const int c = (k + kThreads - 1) / kThreads, first = min(k, tid * c), last = min(k, first + c);
  T own = T::zero();
  for (int t = last - 1; t >= first; --t) {
    const int pos = s.draw[t];
    if (s.rank[pos] != t) *bad = 1;
    own = own + exp_at(pos);
  }
  T run = scan_lanes<false>(own, &sum);
  if ((tid & 63) == 0) s_back[wave] = sum;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    run = run + s_left[w];
    if (w > wave) run = run + s_back[w];
  }
  double lp = 0.0;
  own = T::zero();
  for (int t = last - 1; t >= first; --t) {
    const int pos = s.draw[t];
    run = run + exp_at(pos);
    lp += run.share_of(s.x[pos], top);
    front[t] = run.inverse();
    own = own + front[t];
  }
  Plain part;
  scan_lanes<false>(Plain{lp}, &part);
  run = scan_lanes<true>(own, &sum);
  if ((tid & 63) == 0) {
    s_sum[wave] = part.v;
    s_front[wave] = sum;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w)
    if (w < wave) run = run + s_front[w];
  for (int t = first; t < last; ++t) {
    run = run + front[t];
    front[t] = run;
  }
  lp = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) lp += s_sum[w];
  __syncthreads();
  return lp;
}

// d loss / d s of the visual tokens.
template <int kThreads, class T>
__device__ __forceinline__ void put_gradient(const Tokens& s, const T* front, int nv, int k, double top, double slope,
                                             float* grad) {
  for (int j = threadIdx.x; j < nv; j += kThreads) {
    float g = 0.0f;
    if (k > 0) {
      const int r = s.rank[j];
      T e;
      if constexpr (sizeof(T) == sizeof(Plain)) e = front[nv + j];
      else e = T::exp_of(s.x[j], top);
      g = static_cast<float>(slope * ((r < 0 ? 0.0 : 1.0) - e.times(front[r < 0 ? k - 1 : r])));
    }
    grad[j] = g;
  }
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void pl_policy_kernel(PLPolicyParams p) {
  constexpr int kWaves = kThreads / 64;
  extern __shared__ double s_tokens[];
  __shared__ float s_max[kWaves], s_min[kWaves];
  __shared__ int s_bad;
  const int b = blockIdx.x, tid = threadIdx.x;
  // Everything that says where the image lies is loaded side by side.
  const int lo = p.cu_in ? p.cu_in[b] : 0, hi = p.cu_in ? p.cu_in[b + 1] : 0;
  const int o0 = p.cu_order[b], o1 = p.cu_order[b + 1], oend = p.cu_order[p.B], ofirst = p.cu_order[0];
  const float w = p.weight ? p.weight[b] : 1.0f, old = p.old[b], adv = p.adv[b], refp = p.ref ? p.ref[b] : 0.0f;
  const int64_t off = p.cu_in ? lo : static_cast<int64_t>(b) * p.N;
  const int n = p.cu_in ? hi - lo : p.N;
  const bool seg_ok = !p.cu_in || (lo >= 0 && hi > lo && n <= p.N && hi <= p.total_in && (b > 0 || lo == 0));
  const int nv = seg_ok ? n - 1 : 0;
  const int k = (o0 >= 0 && o1 >= o0 && o1 <= oend && o1 <= p.cap && ofirst == 0) ? o1 - o0 : -1;
  bool ok = seg_ok && w != 0.0f && k >= 0 && k <= nv;

  char* const at = reinterpret_cast<char*>(s_tokens);
  const Tokens s{at, reinterpret_cast<float*>(at + 16 * p.N), reinterpret_cast<int16_t*>(at + 20 * p.N),
                 reinterpret_cast<int16_t*>(at + 22 * p.N)};
  double lp = 0.0, ref = 0.0;  // ref: the largest score
  bool plain = true;
  if (ok) {
    float top = -__builtin_inff(), low = __builtin_inff();
    if (tid == 0) s_bad = 0;
    bool bad = false;
    for (int t = tid; t < nv; t += kThreads) {  // scores and draws (no more of them) side by side
      const float x = p.s[off + t + 1];
      const int pos = t < k ? p.order[o0 + t] - 1 : 0;
      s.x[t] = x;
      s.rank[t] = -1;
      s.draw[t] = static_cast<int16_t>(min(max(pos, 0), nv - 1));
      bad = bad || pos < 0 || pos >= nv;
      top = fmaxf(top, x);
      low = fminf(low, x == -__builtin_inff() ? low : x);  // exp of it is 0 in either form
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      top = fmaxf(top, __shfl_xor(top, d));
      low = fminf(low, __shfl_xor(low, d));
    }
    if ((tid & 63) == 0) {
      s_max[tid >> 6] = top;
      s_min[tid >> 6] = low;
    }
    __syncthreads();
    if (bad) s_bad = 1;
    top = s_max[0];
    low = s_min[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) {
      top = fmaxf(top, s_max[i]);
      low = fminf(low, s_min[i]);
    }
    ref = nv > 0 ? top : 0.0;
    plain = (static_cast<double>(top) - low) * kLog2E < 900.0;  // also for no token: -inf
    lp = plain ? scan_draws<kThreads>(s, nv, k, ref, reinterpret_cast<Plain*>(s.scan), &s_bad)
               : scan_draws<kThreads>(s, nv, k, ref, reinterpret_cast<Scaled*>(s.scan), &s_bad);
    ok = s_bad == 0;
  }
  if (!ok) {
    for (int j = tid; seg_ok && j < n; j += kThreads) p.grad[off + j] = 0.0f;
    if (tid < kPolicyTerms) {
      if (gridDim.x == 1) p.stats[tid] = 0.0f;
      else p.parts[static_cast<int64_t>(b) * kPolicyTerms + tid] = 0.0;
    }
    if (tid == 0) {
      p.logp[b] = seg_ok && w == 0.0f ? 0.0f : __builtin_nanf("");
      if (!seg_ok) atomicOr(p.status, DORA_DEV_CU_IN);
      else if (w != 0.0f) atomicOr(p.status, DORA_DEV_KEEP_RANGE);
    }
    return;
  }
  PolicyTerms terms{};
  const double slope = policy_decision(lp, 0.0, old, adv, w, p.ref != nullptr, refp, p.coef, terms);
  if (tid == 0) {
    p.logp[b] = static_cast<float>(lp);
#pragma unroll
    for (int i = 0; i < kPolicyTerms; ++i) {
      if (gridDim.x == 1) p.stats[i] = static_cast<float>(terms.v[i]);  // there is nothing to add to it
      else p.parts[static_cast<int64_t>(b) * kPolicyTerms + i] = terms.v[i];
    }
    p.grad[off] = 0.0f;  // CLS is never drawn
  }
  float* const grad = p.grad + off + 1;
  if (plain) put_gradient<kThreads>(s, reinterpret_cast<const Plain*>(s.scan), nv, k, ref, slope, grad);
  else put_gradient<kThreads>(s, reinterpret_cast<const Scaled*>(s.scan), nv, k, ref, slope, grad);
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
  return dora_pl_policy_loss_cap(scores, order, cu_order, 0x7FFFFFFF, cu_in, total_in, old_logprob, ref_logprob,
                                 advantage, weight, B, N, clip_low, clip_high, kl_coef, dscores, logprob_out, stats_out,
                                 workspace, workspace_bytes, dev_status, stream);
}

extern "C" int dora_pl_policy_loss_cap(const float* scores, const int32_t* order, const int32_t* cu_order, int64_t cap,
                                       const int32_t* cu_in, int64_t total_in, const float* old_logprob,
                                       const float* ref_logprob, const float* advantage, const float* weight, int32_t B,
                                       int32_t N, float clip_low, float clip_high, float kl_coef, float* dscores,
                                       float* logprob_out, float* stats_out, void* workspace, size_t workspace_bytes,
                                       int32_t* dev_status, void* stream) {
  using namespace dora;
  if (!scores || (!order && cap != 0) || !cu_order || !old_logprob || !advantage || !dscores || !logprob_out || !stats_out ||
      !dev_status)
    return DORA_ERR_NULL;
  if (B < 1 || B > kPlanMaxB || N < 1 || N > DORA_MAX_ROW_TOKENS) return DORA_ERR_SHAPE;
  if (cu_in && (total_in < 0 || total_in > 0x7FFFFFFF)) return DORA_ERR_SHAPE;
  if (cap < 0) return DORA_ERR_CAPACITY;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f) || !(kl_coef - kl_coef == 0.0f))
    return DORA_ERR_SHAPE;
  if (kl_coef != 0.0f && !ref_logprob) return DORA_ERR_NULL;
  const uintptr_t sa = reinterpret_cast<uintptr_t>(scores), ga = reinterpret_cast<uintptr_t>(dscores);
  const uintptr_t len = static_cast<uintptr_t>(cu_in ? total_in : static_cast<int64_t>(B) * N) * sizeof(float);
  if (sa != ga && sa < ga + len && ga < sa + len) return DORA_ERR_OVERLAP;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u ||
      workspace_bytes < dora_pl_policy_workspace_size(B))
    return DORA_ERR_WORKSPACE;
  // A list of no stated length counts as its first entry.
  const size_t vec = static_cast<size_t>(B) * 4, ends = vec + 4, list = cap < 0x7FFFFFFF ? cap * sizeof(int32_t) : 4;
  const Extent lp_out(logprob_out, vec), sums(stats_out, kPolicyTerms * 4), ws(workspace, dora_pl_policy_workspace_size(B)),
      flag(dev_status, 4), grad(dscores, len), s_in(scores, len), draws(order, list), cuo(cu_order, ends), cu(cu_in, ends),
      old(old_logprob, vec), ref(ref_logprob, vec), adv(advantage, vec), w(weight, vec);
  if (outputs_clash({sums, ws, flag, grad}, {draws, cuo, cu, old, ref, adv, w, lp_out}, {}) ||
      outputs_clash({sums, ws, flag}, {s_in}, {}) ||
      outputs_clash({lp_out}, {s_in, draws, cuo, cu}, {old, ref, adv, w}))
    return DORA_ERR_OVERLAP;
  PLPolicyParams p{scores, order, cu_order, cap, cu_in, total_in, old_logprob, ref_logprob, advantage, weight, B, N,
                   PolicyCoef{clip_low, clip_high, kl_coef, 0.0f}, dscores, logprob_out,
                   static_cast<double*>(workspace), stats_out, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  // Wide workgroups shorten a long row's way through the scans, narrow ones
  // repeat less (every wave takes the loss's exp and log) where the images fill
  // the GPU.  64 / 128 / 256 threads, us a pass: 8192 x 257 tokens 30 / 34 / 45,
  // 512 x 257 9.6 / 9.4 / 9.2, 8192 x 577 52 / 46 / 55, 512 x 577 13.4 / 11.3 / 9.9,
  // 2048 x 1200 47 / 34 / 27, 2048 x 65 9.6 / 10.8 / 14.4.
  const bool many = B > 1024;
  const int threads = N <= 128 || (N <= 320 && many) ? 64 : (N <= 320 || (N <= 800 && many) ? 128 : 256);
  const size_t lds = static_cast<size_t>(N) * kTokenBytes;
  if (threads == 64) hipLaunchKernelGGL(pl_policy_kernel<64>, dim3(B), dim3(64), lds, st, p);
  else if (threads == 128) hipLaunchKernelGGL(pl_policy_kernel<128>, dim3(B), dim3(128), lds, st, p);
  else hipLaunchKernelGGL(pl_policy_kernel<256>, dim3(B), dim3(256), lds, st, p);
  if (B > 1) launch_policy_finish(p.parts, B, stats_out, st);
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
