// The clipped policy loss of one decision, shared by the losses on logits and
// on ordered Plackett-Luce draws, and the sum of the decisions' terms.
//
//   r = exp(logp - old),  gain = min(r A, clip(r, 1 - low, 1 + high) A)
//   kl = exp(ref - logp) - (ref - logp) - 1     (0 without a reference)
//   loss = w (-gain + kl_coef kl - entropy_coef H)
//   slope = w (-r A where the clip does not bind + kl_coef (1 - exp(ref - logp)))
//
// slope is d loss / d logp without the entropy's share.  One decision is a few
// dozen operations beside the thousands of its row, so they are done in 64
// bits: kl is the small difference of numbers near one, and a ratio's side of
// the clip's border does not hang on an fp32 rounding.
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "dora.h"

namespace dora {

struct PolicyCoef {
  float clip_low, clip_high, kl, entropy;
};

// Sums over decisions, in the order of stats_out.
constexpr int kPolicyTerms = 6;
struct PolicyTerms {
  double v[kPolicyTerms];  // loss, gain, kl, entropy, clipped, weight: each times w
};

__device__ __forceinline__ double policy_decision(double logp, double entropy, float old, float adv, float w,
                                                  bool with_ref, float ref, const PolicyCoef& c, PolicyTerms& sum) {
  const double r = exp(logp - static_cast<double>(old)), a = adv, wd = w;
  const double lo = 1.0 - static_cast<double>(c.clip_low), hi = 1.0 + static_cast<double>(c.clip_high);
  const double held = (r < lo ? lo : (r > hi ? hi : r)) * a, open = r * a;
  const bool clipped = held < open;
  const double gain = clipped ? held : open;
  double slope = clipped ? 0.0 : -open, kl = 0.0;
  if (with_ref) {
    const double d = static_cast<double>(ref) - logp, up = expm1(d);
    kl = up - d;
    if (c.kl != 0.0f) slope -= c.kl * up;  // an infinite distance counts for nothing at coefficient 0
  }
  sum.v[0] += wd * ((c.kl != 0.0f ? c.kl * kl : 0.0) - gain - (c.entropy != 0.0f ? c.entropy * entropy : 0.0));
  sum.v[1] += wd * gain;
  sum.v[2] += wd * kl;
  sum.v[3] += wd * entropy;
  sum.v[4] += clipped ? wd : 0.0;
  sum.v[5] += wd;
  return wd * slope;
}

// stats_out from n sets of sums, added in a fixed order: by one workgroup, or
// past kFinishDirect sets first by up to kFinishGroups workgroups into the room
// behind them (one workgroup: 32 sets 1.8 us, 1024 4.1 to 4.7, 8192 14; more threads
// or loads in flight made no difference to a pass over long rows).
constexpr int kFinishDirect = 8192, kFinishGroups = 256;
inline size_t policy_parts_bytes(int32_t n) {
  const size_t sets = static_cast<size_t>(n) + (n > kFinishDirect ? kFinishGroups : 0);
  return (sets * sizeof(PolicyTerms) + 255) & ~size_t(255);
}
void launch_policy_finish(double* parts, int32_t n, float* stats, hipStream_t stream);

// Memory of a call's tensor (none at address 0 or without elements).
struct Extent {
  uintptr_t at;
  size_t bytes;
  Extent(const void* p, size_t n) : at(reinterpret_cast<uintptr_t>(p)), bytes(n) {}
  bool meets(Extent o) const {
    return at && o.at && bytes && o.bytes && at < o.at + o.bytes && o.at < at + bytes;
  }
};
// Outputs that share memory with another output or with an input.  `own` are
// inputs whose place an output may take as a whole: a row reads its entry of
// them before it writes its own.
inline bool outputs_clash(std::initializer_list<Extent> out, std::initializer_list<Extent> in,
                          std::initializer_list<Extent> own) {
  for (const Extent* o = out.begin(); o != out.end(); ++o) {
    for (const Extent* q = out.begin(); q != o; ++q)
      if (o->meets(*q)) return true;
    for (const Extent& i : in)
      if (o->meets(i)) return true;
    for (const Extent& i : own)
      if (o->meets(i) && (o->at != i.at || o->bytes != i.bytes)) return true;
  }
  return false;
}

}  // namespace dora
