// What stands between two branches of a transformer block (dora_residual_norm),
// and its gradients:
//   u = a or norm(a),  h = x + gate scale u,  y = norm(h)
//   norm(z) = zhat gamma + beta,  zhat = (z - mean) r,  r = 1 / sqrt(var + eps)
//             (rms: mean 0 and var the mean square)
//   backward of norm, with g = dz gamma:  r (g - mean(g) - zhat mean(g zhat))
//             (rms: without mean(g)),  dgamma = sum dz zhat,  dbeta = sum dz
//
// HBM bound: each row is read once into registers, by 16 lanes to a workgroup of
// 512 that hold one to four 16-byte pieces of each tensor a lane; means come
// from the registers (the variance from the deviations, in a second pass over
// them).  Workgroups go over rows and keep the parameters, and in the backward
// pass the parameters' gradients, in registers; those meet in LDS and in
// memory, in a fixed order.
//
// Gradients of 50432 rows of 768, bf16, with layer scale and dropped branches: 110
// us, 4.2 TB/s; of 35295 rows of 1024, fp32, with a norm after the branch: 170 us,
// 5.1 TB/s; the sums' launch 5 (a large copy runs at 4.9).  16 rows of 4096: 6 us,
// a launch and one chain of loads.
#include <math.h>

#include <algorithm>

#include "dora_internal.h"
#include "lanes.h"
#include "rows.h"

namespace dora {
namespace {

constexpr int kMaxC = 8192;
constexpr int kParams = 5;  // dgamma, dbeta, dscale, dpost_gamma, dpost_beta
constexpr int kFinishCols = 16, kFinishThreads = 512;

struct NormArgs {
  RowView x, a, h, y;            // backward: x is h
  RowView dy, dh, dx, da;
  int64_t T;
  int32_t C, rms;
  float eps;
  const float* gamma;
  const float* beta;
  const float* scale;
  const float* gate;
  const float* post_gamma;
  const float* post_beta;
  float* dgate;
  float* part;  // [workgroups][kParams][C]
  int32_t grads;  // some parameter's gradient is wanted
};

template <class E>
struct Vec {
  static constexpr int kE = 16 / sizeof(E);
  float v[kE];
  __device__ __forceinline__ void unpack(u32x4 w) {
    if (sizeof(E) == 4) {
#pragma unroll
      for (int i = 0; i < kE; ++i) v[i] = __builtin_bit_cast(float, static_cast<uint32_t>(w[i]));
    } else {
#pragma unroll
      for (int i = 0; i < kE; ++i)
        v[i] = __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xFFFF0000u : static_cast<uint32_t>(w[i / 2]) << 16);
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    E e[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) e[i] = static_cast<E>(v[i]);
    u32x4 w;
    __builtin_memcpy(&w, e, 16);
    *reinterpret_cast<u32x4*>(p) = w;
  }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = x;
  }
};

// Sums over the L lanes of a row, N at a time; every lane gets them.
template <int L, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* lds) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    s[n] = sum16(s[n]);
    if (L > 16) s[n] = add32(add16(s[n]));
  }
  if (L > 64) {  // the row is the workgroup
    constexpr int kWaves = L / 64;
    __syncthreads();  // the last sums have been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) lds[n * kWaves + (threadIdx.x >> 6)] = s[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s[n] += lds[n * kWaves + w];
    }
  }
}

// A row's pieces as they lie in memory, 0 past its end: asked for one row ahead.
template <int L, int NP>
struct Raw {
  u32x4 w[NP];
  __device__ __forceinline__ void load(const RowView& v, int64_t t, int lane, int pieces) {
    if (!v.at) return;
    const char* row = v.at + t * v.row;
#pragma unroll
    for (int j = 0; j < NP; ++j)
      w[j] = lane + j * L < pieces ? *reinterpret_cast<const u32x4*>(row + static_cast<uint32_t>(lane + j * L) * 16u)
                                   : u32x4{0u, 0u, 0u, 0u};
  }
};

// A row's pieces in the lanes' registers.
template <class E, int L, int NP>
struct Row {
  static constexpr int kE = Vec<E>::kE;
  Vec<E> p[NP];
  __device__ __forceinline__ void unpack(const Raw<L, NP>& raw) {
#pragma unroll
    for (int j = 0; j < NP; ++j) p[j].unpack(raw.w[j]);
  }
  __device__ __forceinline__ void store(char* row, int lane, int pieces) const {
#pragma unroll
    for (int j = 0; j < NP; ++j)
      if (lane + j * L < pieces) p[j].store(row + static_cast<uint32_t>(lane + j * L) * 16u);
  }
  // A parameter's values at the lane's columns, x where there is none; 0 past the row's end, which makes what
  // is multiplied by it 0 there.
  __device__ __forceinline__ void param(const float* q, float x, int lane, int pieces) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      p[j].fill(lane + j * L < pieces ? x : 0.f);
      if (q && lane + j * L < pieces) {
        // a 32-bit offset from the parameter's address: one register for all of them
        const char* at = reinterpret_cast<const char*>(q) + static_cast<uint32_t>((lane + j * L) * kE) * 4u;
#pragma unroll
        for (int i = 0; i < kE; ++i) p[j].v[i] = reinterpret_cast<const float*>(at)[i];
      }
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int i = 0; i < kE; ++i) f(p[j].v[i], j, i);
  }
};

// A parameter at the lane's columns: in registers where a lane has at most eight
// elements of a row, else read again for each row (from the L2; the registers of
// the widest rows, five sums and four tensors beside, would spill).
template <class E, int L, int NP>
struct Param {
  static constexpr bool kHeld = NP * Vec<E>::kE <= 8;
  const float* q;
  float none;
  Row<E, L, NP> held;
  __device__ __forceinline__ Param(const float* p, float x, int lane, int pieces) : q(p), none(x) {
    if constexpr (kHeld) held.param(q, none, lane, pieces);
  }
  __device__ __forceinline__ Row<E, L, NP> row(int lane, int pieces) const {
    if constexpr (kHeld) return held;
    asm volatile("" : "+v"(lane));  // addresses are formed here, not kept in registers for every row
    Row<E, L, NP> r;
    r.param(q, none, lane, pieces);
    return r;
  }
};

// The row normed in place, without its parameters; returns r.
template <class E, int L, int NP>
__device__ __forceinline__ float to_hat(Row<E, L, NP>& z, const NormArgs& a, int lane, int pieces, float* lds) {
  const float n = 1.f / a.C;
  float s[1] = {0.f};
  if (!a.rms) {
    z.each([&](float& v, int, int) { s[0] += v; });
    row_sum<L>(s, lds);
    const float mean = s[0] * n;
#pragma unroll
    for (int j = 0; j < NP; ++j)
      if (lane + j * L < pieces)
#pragma unroll
        for (int i = 0; i < Vec<E>::kE; ++i) z.p[j].v[i] -= mean;
    s[0] = 0.f;
  }
  z.each([&](float& v, int, int) { s[0] = __builtin_fmaf(v, v, s[0]); });
  row_sum<L>(s, lds);
  const float r = 1.f / __builtin_sqrtf(s[0] * n + a.eps);
  z.each([&](float& v, int, int) { v *= r; });
  return r;
}

// g -> r (g - mean(g) - hat mean(g hat)).
template <class E, int L, int NP>
__device__ __forceinline__ void hat_grad(Row<E, L, NP>& g, Row<E, L, NP>& hat, float r, const NormArgs& a, float* lds) {
  float s[2] = {0.f, 0.f};
  g.each([&](float& v, int j, int i) {
    s[0] += v;
    s[1] = __builtin_fmaf(v, hat.p[j].v[i], s[1]);
  });
  row_sum<L>(s, lds);
  const float m = a.rms ? 0.f : s[0] / a.C, c = s[1] / a.C;
  g.each([&](float& v, int j, int i) { v = r * (v - m - hat.p[j].v[i] * c); });
}

template <int L>
constexpr int threads_of() {
  return L > 256 ? L : 256;
}

template <class E, int L, int NP, bool POST>
__global__ __launch_bounds__(threads_of<L>()) void residual_norm_kernel(NormArgs a) {
  constexpr int kGroups = threads_of<L>() / L, kE = Vec<E>::kE;
  typedef Row<E, L, NP> R;
  typedef Param<E, L, NP> P;
  __shared__ float lds[L > 64 ? L / 64 : 1];
  const int lane = threadIdx.x % L, group = threadIdx.x / L, pieces = a.C / kE;
  const P gamma(a.gamma, 1.f, lane, pieces), beta(a.beta, 0.f, lane, pieces), scale(a.scale, 1.f, lane, pieces),
      pg(POST ? a.post_gamma : nullptr, 1.f, lane, pieces), pb(POST ? a.post_beta : nullptr, 0.f, lane, pieces);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + group;
  Raw<L, NP> rx, ra;
  const auto ask = [&](int64_t row) {
    rx.load(a.x, row, lane, pieces);
    ra.load(a.a, row, lane, pieces);
  };
  if (t < a.T) ask(t);
  // A row of many lanes is its workgroup's alone: its barriers are reached by all of them.
  for (; t < a.T; t += step) {
    R h, u;
    h.unpack(rx);
    if (a.a.at) u.unpack(ra);
    if (t + step < a.T) ask(t + step);
    if (a.a.at) {
      const float gate = a.gate ? a.gate[t] : 1.f;
      if (POST) {
        to_hat(u, a, lane, pieces, lds);
        const R w = pg.row(lane, pieces), w0 = pb.row(lane, pieces);
        u.each([&](float& v, int j, int i) { v = __builtin_fmaf(v, w.p[j].v[i], w0.p[j].v[i]); });
      }
      const R w = scale.row(lane, pieces);
      if (gate != 0.f) h.each([&](float& v, int j, int i) { v = __builtin_fmaf(u.p[j].v[i] * w.p[j].v[i], gate, v); });
    }
    if (a.h.at) h.store(a.h.at + t * a.h.row, lane, pieces);
    to_hat(h, a, lane, pieces, lds);
    const R w = gamma.row(lane, pieces), w0 = beta.row(lane, pieces);
    h.each([&](float& v, int j, int i) { v = __builtin_fmaf(v, w.p[j].v[i], w0.p[j].v[i]); });
    h.store(a.y.at + t * a.y.row, lane, pieces);
  }
}

template <class E, int L, int NP, bool POST>
__global__ __launch_bounds__(threads_of<L>()) void residual_norm_grad_kernel(NormArgs a) {
  constexpr int kThreads = threads_of<L>(), kGroups = kThreads / L, kE = Vec<E>::kE;
  typedef Row<E, L, NP> R;
  typedef Param<E, L, NP> P;
  __shared__ float lds[L > 64 ? 2 * L / 64 : 1];
  __shared__ float meet[kGroups > 1 ? kGroups * L * NP * kE : 1];
  const int lane = threadIdx.x % L, group = threadIdx.x / L, pieces = a.C / kE;
  const P gamma(a.gamma, 1.f, lane, pieces), scale(a.scale, 1.f, lane, pieces),
      pg(POST ? a.post_gamma : nullptr, 1.f, lane, pieces), pb(POST ? a.post_beta : nullptr, 0.f, lane, pieces);
  // The branch's sums of the widest lanes stand in LDS, a slot for each lane: with them the registers spill.
  constexpr bool kLdsSums = POST && NP * kE > 8;
  constexpr int kSums = kLdsSums ? 2 : POST ? 5 : 3;
  __shared__ float lds_sums[kLdsSums ? (5 - kSums) * NP * kE * kThreads : 1];
  const auto slot = [&](int n, int j, int i) -> float& {
    return lds_sums[((n - kSums) * NP * kE + j * kE + i) * kThreads + threadIdx.x];
  };
  R sum[kSums];
#pragma unroll
  for (int n = 0; n < kSums; ++n) sum[n].param(nullptr, 0.f, lane, pieces);
  if constexpr (kLdsSums)
    for (int n = 0; n < (5 - kSums) * NP * kE; ++n) lds_sums[n * kThreads + threadIdx.x] = 0.f;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  int64_t t = static_cast<int64_t>(blockIdx.x) * kGroups + group;
  Raw<L, NP> ry, rdh, rh, ra;
  const auto ask = [&](int64_t row) {
    if (a.dy.at) rh.load(a.x, row, lane, pieces);
    ry.load(a.dy, row, lane, pieces);
    rdh.load(a.dh, row, lane, pieces);
    ra.load(a.a, row, lane, pieces);
  };
  constexpr bool kAhead = NP <= 2;  // one row ahead, where the registers hold two
  if (kAhead && t < a.T) ask(t);
  for (; t < a.T; t += step) {
    Raw<L, NP> cy = ry, cdh = rdh, ch = rh, ca = ra;
    if (kAhead && t + step < a.T) ask(t + step);
    if (!kAhead && a.dy.at) {
      ch.load(a.x, t, lane, pieces);
      cy.load(a.dy, t, lane, pieces);
    }
    R g, u;
    if (a.dy.at) {
      R hat;
      hat.unpack(ch);
      g.unpack(cy);
      const float r = to_hat(hat, a, lane, pieces, lds);
      const R w = gamma.row(lane, pieces);
      g.each([&](float& v, int j, int i) {
        sum[0].p[j].v[i] = __builtin_fmaf(v, hat.p[j].v[i], sum[0].p[j].v[i]);
        sum[1].p[j].v[i] += v;
        v *= w.p[j].v[i];
      });
      hat_grad(g, hat, r, a, lds);
    } else {
      g.param(nullptr, 0.f, lane, pieces);
    }
    if (a.dh.at) {
      R dh;
      if (!kAhead) cdh.load(a.dh, t, lane, pieces);
      dh.unpack(cdh);
      g.each([&](float& v, int j, int i) { v += dh.p[j].v[i]; });
    }
    if (!kAhead) ca.load(a.a, t, lane, pieces);  // before dx, which may take its place
    g.store(a.dx.at + t * a.dx.row, lane, pieces);
    if (!a.a.at) continue;
    const float gate = a.gate ? a.gate[t] : 1.f;
    u.unpack(ca);
    R ahat;
    float ar = 0.f;
    if constexpr (POST) {
      ahat = u;
      ar = to_hat(ahat, a, lane, pieces, lds);
      const R w = pg.row(lane, pieces), w0 = pb.row(lane, pieces);
      u.each([&](float& v, int j, int i) { v = __builtin_fmaf(ahat.p[j].v[i], w.p[j].v[i], w0.p[j].v[i]); });
    }
    // u turns into the branch's gradient; a dropped row's branch counts for nothing, whatever it holds.
    const R sc = scale.row(lane, pieces);
    float s[1] = {0.f};
    u.each([&](float& v, int j, int i) {
      const float d = g.p[j].v[i], gated = gate != 0.f ? d * gate : 0.f;
      s[0] = __builtin_fmaf(d, v * sc.p[j].v[i], s[0]);
      if (gate != 0.f) {
        if constexpr (kLdsSums) slot(2, j, i) = __builtin_fmaf(gated, v, slot(2, j, i));
        else sum[2].p[j].v[i] = __builtin_fmaf(gated, v, sum[2].p[j].v[i]);
      }
      v = gated * sc.p[j].v[i];
    });
    if (a.dgate) {
      row_sum<L>(s, lds);
      if (lane == 0) a.dgate[t] = s[0];
    }
    if constexpr (POST) {
      const R w = pg.row(lane, pieces);
      if (gate != 0.f)
        u.each([&](float& v, int j, int i) {
          if constexpr (kLdsSums) {
            slot(3, j, i) = __builtin_fmaf(v, ahat.p[j].v[i], slot(3, j, i));
            slot(4, j, i) += v;
          } else {
            sum[3].p[j].v[i] = __builtin_fmaf(v, ahat.p[j].v[i], sum[3].p[j].v[i]);
            sum[4].p[j].v[i] += v;
          }
          v *= w.p[j].v[i];
        });
      hat_grad(u, ahat, ar, a, lds);
      if (gate == 0.f) u.param(nullptr, 0.f, lane, pieces);
    }
    if (a.da.at) u.store(a.da.at + t * a.da.row, lane, pieces);
  }
  if (!a.grads) return;
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * kParams * a.C;
#pragma unroll
  for (int n = 0; n < (POST ? 5 : 3); ++n) {
    R all;
    if (n < kSums) all = sum[n < kSums ? n : 0];
    else all.each([&](float& v, int j, int i) { v = slot(n, j, i); });
    if (kGroups > 1) {
      constexpr int kCols = L * NP * kE;
      __syncthreads();
      all.each([&](float& v, int j, int i) { meet[group * kCols + (lane + j * L) * kE + i] = v; });
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int x = 0; x < kGroups; ++x) s += meet[x * kCols + c];
        part[n * a.C + c] = s;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NP; ++j)
        if (lane + j * L < pieces)
#pragma unroll
          for (int i = 0; i < kE; ++i) part[n * a.C + (lane + j * L) * kE + i] = all.p[j].v[i];
    }
  }
}

struct FinishArgs {
  const float* part;
  float* out[kParams];
  int32_t parts, C;
};

// The workgroups' sums added in 64 bits: 16 columns of one parameter a workgroup, 32 parts side by side, eight
// loads of each on their way at a time.
__global__ __launch_bounds__(kFinishThreads) void norm_finish_kernel(FinishArgs f) {
  constexpr int kRows = kFinishThreads / kFinishCols;
  __shared__ double meet[kRows][kFinishCols];
  float* const out = f.out[blockIdx.y];
  if (!out) return;
  const int col = blockIdx.x * kFinishCols + threadIdx.x % kFinishCols, row = threadIdx.x / kFinishCols;
  double s = 0.0;
  if (col < f.C)
    for (int p = row; p < f.parts; p += 8 * kRows) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t at = static_cast<int64_t>(min(p + i * kRows, f.parts - 1)) * kParams + blockIdx.y;
        x[i] = f.part[at * f.C + col];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += p + i * kRows < f.parts ? x[i] : 0.f;
    }
  meet[row][threadIdx.x % kFinishCols] = s;
  __syncthreads();
  if (row == 0 && col < f.C) {
    s = 0.0;
    for (int i = 0; i < kRows; ++i) s += meet[i][threadIdx.x];
    out[col] = static_cast<float>(s);
  }
}

int lanes_of(int pieces) { return pieces <= 32 ? 16 : pieces <= 128 ? 64 : pieces <= 512 ? 256 : 512; }

// Workgroups of a launch: what the GPU holds a few times over, each with rows to spare.
int64_t groups_of(int64_t T, int32_t C, int dtype, int64_t most) {
  const int pieces = C * elem_bytes(dtype) / 16, L = lanes_of(pieces), rows = L >= 256 ? 1 : 256 / L;
  const bool wide = L == 512 || (dtype == DORA_BF16 && pieces > L);  // 16 elements a lane: half as many fit
  return std::min((T + rows - 1) / rows, wide ? most / 2 : most);
}
constexpr int64_t kForwardGroups = 2048, kBackwardGroups = 1024;

// f(element, lanes of a row, pieces a lane)
template <class F>
void with_shape(int dtype, int C, F f) {
  const auto lanes = [&](auto e) {
    const int pieces = C * static_cast<int>(sizeof(e)) / 16, L = lanes_of(pieces);
    const auto per = [&](auto l) {
      if (pieces <= decltype(l)::value) f(e, l, std::integral_constant<int, 1>{});
      else f(e, l, std::integral_constant<int, 2>{});
    };
    if (L == 16) per(std::integral_constant<int, 16>{});
    else if (L == 64) per(std::integral_constant<int, 64>{});
    else if (L == 256) per(std::integral_constant<int, 256>{});
    else if (sizeof(e) == 2 || pieces <= 1024) f(e, std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    else if constexpr (sizeof(e) == 4) f(e, std::integral_constant<int, 512>{}, std::integral_constant<int, 4>{});
  };
  if (dtype == DORA_BF16) lanes(__bf16{});
  else lanes(float{});
}

bool good_width(int64_t C, int elem) { return C >= 1 && C <= kMaxC && C * elem % 16 == 0; }

// A matrix of the call like `like` (or of its own size).
int check_matrix(const dora_rows* t, const dora_rows* like) {
  if (!t) return DORA_OK;
  const int rc = check_rows(t, 16);
  if (rc != DORA_OK) return rc;
  if (t->heads != 1 || t->rows != like->rows || t->dim != like->dim) return DORA_ERR_SHAPE;
  return t->dtype == like->dtype ? DORA_OK : DORA_ERR_DTYPE;
}

Extent vec(const float* p, int64_t n) { return Extent(p, static_cast<size_t>(n) * sizeof(float)); }

}  // namespace
}  // namespace dora

extern "C" int dora_residual_norm(const dora_rows* x, const dora_rows* a, const float* gamma, const float* beta,
                                  const float* scale, const float* gate, const float* post_gamma,
                                  const float* post_beta, int32_t kind, float eps, const dora_rows* h_out,
                                  const dora_rows* y_out, void* stream) {
  using namespace dora;
  if (!x || !y_out || !gamma || (a && !h_out)) return DORA_ERR_NULL;
  for (const dora_rows* t : {x, a, h_out, y_out}) {
    const int rc = check_matrix(t, x);
    if (rc != DORA_OK) return rc;
  }
  if (!good_width(x->dim, elem_bytes(x->dtype)) || (kind != DORA_NORM_LAYER && kind != DORA_NORM_RMS) || !(eps >= 0.f))
    return DORA_ERR_SHAPE;
  if ((!a && (scale || gate || post_gamma || post_beta)) || (post_beta && !post_gamma)) return DORA_ERR_UNSUPPORTED;
  const int64_t T = x->rows;
  const int32_t C = x->dim;
  if (rows_clash({h_out, y_out}, {}, {x, a}, {},
                 {vec(gamma, C), vec(beta, C), vec(scale, C), vec(gate, T), vec(post_gamma, C), vec(post_beta, C)}))
    return DORA_ERR_OVERLAP;
  if (T == 0) return DORA_OK;
  NormArgs n{};
  n.x = row_view(x), n.a = row_view(a), n.h = row_view(h_out), n.y = row_view(y_out);
  n.T = T, n.C = C, n.rms = kind == DORA_NORM_RMS, n.eps = eps;
  n.gamma = gamma, n.beta = beta, n.scale = scale, n.gate = gate, n.post_gamma = post_gamma, n.post_beta = post_beta;
  const dim3 grid(static_cast<uint32_t>(groups_of(T, C, x->dtype, kForwardGroups)));
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_shape(x->dtype, C, [&](auto e, auto l, auto np) {
    typedef decltype(e) E;
    constexpr int L = decltype(l)::value, NP = decltype(np)::value;
    if (post_gamma) hipLaunchKernelGGL((residual_norm_kernel<E, L, NP, true>), grid, dim3(threads_of<L>()), 0, st, n);
    else hipLaunchKernelGGL((residual_norm_kernel<E, L, NP, false>), grid, dim3(threads_of<L>()), 0, st, n);
  });
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}

extern "C" size_t dora_residual_norm_workspace_size(int64_t T, int32_t C) {
  using namespace dora;
  if (T < 0 || T > 0x7FFFFFFF || C < 1 || C > kMaxC) return 0;
  const int64_t groups = std::max(groups_of(T, C, DORA_BF16, kBackwardGroups), groups_of(T, C, DORA_F32, kBackwardGroups));
  return (static_cast<size_t>(std::max<int64_t>(groups, 1)) * kParams * C * sizeof(float) + 255) & ~size_t(255);
}

extern "C" int dora_residual_norm_backward(const dora_rows* dy, const dora_rows* dh, const dora_rows* h,
                                           const dora_rows* a, const float* gamma, const float* scale,
                                           const float* gate, const float* post_gamma, const float* post_beta,
                                           int32_t kind, float eps, const dora_rows* dx, const dora_rows* da,
                                           float* dgamma, float* dbeta, float* dscale, float* dgate,
                                           float* dpost_gamma, float* dpost_beta, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace dora;
  if (!h || !dx || !gamma || (!dy && !dh)) return DORA_ERR_NULL;
  for (const dora_rows* t : {h, dy, dh, a, dx, da}) {
    const int rc = check_matrix(t, h);
    if (rc != DORA_OK) return rc;
  }
  if (!good_width(h->dim, elem_bytes(h->dtype)) || (kind != DORA_NORM_LAYER && kind != DORA_NORM_RMS) || !(eps >= 0.f))
    return DORA_ERR_SHAPE;
  if ((!a && (da || scale || gate || post_gamma || post_beta)) || (post_beta && !post_gamma) || (dscale && !scale) ||
      (dgate && !gate) || (dpost_gamma && !post_gamma) || (dpost_beta && !post_gamma))
    return DORA_ERR_UNSUPPORTED;
  const int64_t T = h->rows;
  const int32_t C = h->dim;
  const size_t need = dora_residual_norm_workspace_size(T, C);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < need) return DORA_ERR_WORKSPACE;
  if (rows_clash({dx, da}, {}, {dy, dh, h, a},
                 {vec(dgamma, C), vec(dbeta, C), vec(dscale, C), vec(dgate, T), vec(dpost_gamma, C), vec(dpost_beta, C),
                  Extent(workspace, need)},
                 {vec(gamma, C), vec(scale, C), vec(gate, T), vec(post_gamma, C), vec(post_beta, C)}))
    return DORA_ERR_OVERLAP;
  NormArgs n{};
  n.x = row_view(h), n.dy = row_view(dy), n.dh = row_view(dh), n.a = row_view(a);
  n.dx = row_view(dx), n.da = row_view(da);
  n.T = T, n.C = C, n.rms = kind == DORA_NORM_RMS, n.eps = eps;
  n.gamma = gamma, n.scale = scale, n.gate = gate, n.post_gamma = post_gamma, n.post_beta = post_beta;
  n.dgate = dgate;
  n.part = static_cast<float*>(workspace);
  n.grads = dgamma || dbeta || dscale || dpost_gamma || dpost_beta;
  const int64_t groups = groups_of(T, C, h->dtype, kBackwardGroups);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (T > 0)
    with_shape(h->dtype, C, [&](auto e, auto l, auto np) {
      typedef decltype(e) E;
      constexpr int L = decltype(l)::value, NP = decltype(np)::value;
      const dim3 grid(static_cast<uint32_t>(groups)), block(threads_of<L>());
      if (post_gamma) hipLaunchKernelGGL((residual_norm_grad_kernel<E, L, NP, true>), grid, block, 0, st, n);
      else hipLaunchKernelGGL((residual_norm_grad_kernel<E, L, NP, false>), grid, block, 0, st, n);
    });
  if (n.grads) {
    const FinishArgs f{n.part, {dgamma, dbeta, dscale, dpost_gamma, dpost_beta}, static_cast<int32_t>(groups), C};
    hipLaunchKernelGGL(norm_finish_kernel, dim3((C + kFinishCols - 1) / kFinishCols, kParams), dim3(kFinishThreads), 0, st,
                       f);
  }
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
