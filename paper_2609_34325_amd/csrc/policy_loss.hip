// Log-probabilities of chosen actions and the clipped policy loss with its
// gradient, from logits.  DORA (arXiv 2609.34325): Sec. 3.2 "Sampling and
// deployment" and App. A.3 (the gate and the budget are categorical choices,
// the budget masked to the legal ones, a prefix of the grid); App. D (clipped
// policy updates).  The same loss trains any head that chooses one of V
// actions per row, up to the vocabulary of a language model.
//
// Row t with logits x_j, 0 <= j < n (n legal actions), action a:
//   s = sum exp(x_j - m), logp = x_a - m - log s            (any m near max x)
//   H = log s - sum exp(x_j - m)(x_j - m) / s
//   d loss / d x_j = slope ([j = a] - p_j) + entropy_coef w p_j (log p_j + H)
// with slope = d loss / d logp (policy_terms.h).
//
// One pass over a row keeps a running (reference, sum, entropy sum) per lane,
// merged over the lanes.  The row's pieces stay packed in registers until its
// gradient is written, so the large cases read and write each byte once and are
// HBM bound: 8192 x 131072 bf16 797 us (5.4 TB/s), 8192 x 50304 288 (5.7), 1024
// x 32000 fp32 46; log-probabilities alone 4096 x 50257 bf16 54 us (5.7 TB/s).
// Per bf16 element 16 vector instructions, two of them exponentials that take
// four issue slots: 22 of the 31 slots that its four bytes leave at 5 TB/s.
// Sums are fp32, the row's own figures 64 bits, a gradient is rounded once, to
// its type.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "dora_internal.h"
#include "policy_terms.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxSplit = 64;  // workgroups a row
// A launch has fewer than 2^32 threads; rows of more than kThreads are long, and
// as many as this of them take more memory than there is.
static_assert(int64_t{DORA_MAX_DECISIONS} * kThreads < int64_t{1} << 32, "threads of a launch");
constexpr float kLog2E = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr float kFarDown = -30000.0f;  // exp2 of it is 0, and 0 times it is 0

struct RowParams {
  const char* logits;
  int64_t ld;  // elements between rows
  const int32_t* actions;
  const int32_t* legal;
  const float* old;
  const float* ref;
  const float* adv;
  const float* weight;
  int32_t T, V;
  PolicyCoef coef;
  char* grad;
  int64_t ld_grad;
  float* logp_out;
  float* entropy_out;
  double* parts;  // [workgroups][kPolicyTerms]
  float4* split_stats;  // split rows: [T][split] of (m, s, h, the action's logit)
  int32_t split;        // workgroups a row
  float* stats;
  int32_t* status;
};

// 16 bytes of a row.  Rows start wherever their leading dimension puts them,
// so pieces are loaded and stored at the element's alignment; the hardware
// takes unaligned 16-byte accesses and splits those that cross a cache line.
template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
  static constexpr int kPer = 8;
  static constexpr int kBytes = 2;
  typedef u32x4 __attribute__((aligned(2))) Vec;
  __device__ static float get(const char* p) {
    return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p)) << 16);
  }
  __device__ static void put(char* p, float v) { *reinterpret_cast<__bf16*>(p) = static_cast<__bf16>(v); }
  __device__ static void unpack(u32x4 v, float (&f)[kPer]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
  __device__ static u32x4 pack(const float (&f)[kPer]) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < kPer; ++i) b[i] = static_cast<__bf16>(f[i]);
    return __builtin_bit_cast(u32x4, b);
  }
};
template <>
struct Elem<false> {
  static constexpr int kPer = 4;
  static constexpr int kBytes = 4;
  typedef u32x4 __attribute__((aligned(4))) Vec;
  __device__ static float get(const char* p) { return *reinterpret_cast<const float*>(p); }
  __device__ static void put(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
  __device__ static void unpack(u32x4 v, float (&f)[kPer]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  __device__ static u32x4 pack(const float (&f)[kPer]) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
    return v;
  }
};

// PASSING: data that is not to stay in the caches (read or written once).
template <bool BF16, bool PASSING = false>
__device__ __forceinline__ u32x4 load_piece(const char* p) {
  const auto* from = reinterpret_cast<const typename Elem<BF16>::Vec*>(p);
  return PASSING ? __builtin_nontemporal_load(from) : *from;
}
template <bool BF16, bool PASSING = false>
__device__ __forceinline__ void store_piece(char* p, u32x4 v) {
  auto* to = reinterpret_cast<typename Elem<BF16>::Vec*>(p);
  if (PASSING) __builtin_nontemporal_store(v, to);
  else *to = v;
}

// A row's exponentials are 2^d with d = x c1 - e, c1 = log2(e) rounded and e
// the whole number next to m c1 for a reference m: one fused step whose only
// error is its own rounding, and another m scales the older sums by a power of
// two, exactly.  The shift in natural units is then e / c1 (in 64 bits): terms
// near the largest, which make up the sums, all carry c1's rounding alike.
// Past 1e9 two different floats lie at least 64 apart, so any factor tells
// them from each other (a million of 2^-64 are nothing beside 1), and m c1
// would leave a large rest or overflow: there d = x - m (a row whose open
// logits all hold the type's lowest value is uniform).
constexpr float kVast = 1.0e9f;
struct Shift {
  float c1, e;
  __device__ explicit Shift(float m) {
    const bool vast = fabsf(m) > kVast;
    c1 = vast ? 1.0f : kLog2E;
    e = vast ? m : rintf(m * kLog2E);
  }
  __device__ float operator()(float x) const { return fmaf(x, c1, -e); }
  __device__ double natural() const { return static_cast<double>(e) / static_cast<double>(c1); }
};

// Running softmax statistics: s = sum 2^d, h = sum 2^d d at reference m.  m is
// an element that was seen, or the lowest float; s = 0 where nothing but -inf
// was.  fmaxf passes over NaN, so m never is one; a NaN logit reaches s and h.
struct Stat {
  float m, s, h;
  __device__ static Stat none() { return {-FLT_MAX, 0.0f, 0.0f}; }
  __device__ void raise(float to) {
    const bool vast = fabsf(m) > kVast || fabsf(to) > kVast;
    const float step = vast ? m - to : rintf(m * kLog2E) - rintf(to * kLog2E);
    const float delta = fmaxf(step, kFarDown);
    const float f = __builtin_amdgcn_exp2f(delta);
    h = f * fmaf(s, delta, h);
    s *= f;
    m = to;
  }
  __device__ void merge(Stat o) {
    const float to = fmaxf(m, o.m);
    raise(to);
    o.raise(to);
    s += o.s;
    h += o.h;
  }
};

// The statistics while a thread takes its pieces.  The reference is raised
// only past 2^kRaise of it: seldom after the first piece.  (h grows with the
// distance to the reference, and the entropy is a difference with it.)
constexpr float kRaise = 10.0f;
struct Taker {
  Stat st = Stat::none();
  Shift sh{-FLT_MAX};
  template <int N>
  __device__ void take(const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    if (sh(top) > kRaise) {
      st.raise(top);
      sh = Shift(top);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = sh(x[i]), e = __builtin_amdgcn_exp2f(d);
      st.s += e;
      st.h = fmaf(e, fmaxf(d, kFarDown), st.h);
    }
  }
};

template <bool BF16>
__device__ __forceinline__ void take_one(Taker& tk, const char* row, int j) {
  const float x[1] = {Elem<BF16>::get(row + static_cast<int64_t>(j) * Elem<BF16>::kBytes)};
  tk.take(x);
}

// Open elements of row t (0: padding or a bad row), its weight and action (0
// for such a row).  The three are loaded side by side.
__device__ __forceinline__ int open_row(const RowParams& p, int64_t t, float& w, int& a) {
  w = p.weight ? p.weight[t] : 1.0f;
  const int n = p.legal ? p.legal[t] : p.V, act = p.actions[t];
  const bool good = w != 0.0f && n >= 1 && n <= p.V && act >= 0 && act < n;
  a = good ? act : 0;
  return good ? n : 0;
}

// A value of the lanes of a group of G (all active) folded by op, to every
// lane: inside 16 lanes by DPP, then by row swaps; no trip through shared memory.
template <int G, class Op>
__device__ __forceinline__ float fold_lanes(float v, Op op) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  if constexpr (G >= 2) v = op(v, dpp(v, std::integral_constant<int, 0xB1>()));    // quad_perm 1,0,3,2
  if constexpr (G >= 4) v = op(v, dpp(v, std::integral_constant<int, 0x4E>()));    // quad_perm 2,3,0,1
  if constexpr (G >= 8) v = op(v, dpp(v, std::integral_constant<int, 0x141>()));   // row_half_mirror
  if constexpr (G >= 16) v = op(v, dpp(v, std::integral_constant<int, 0x140>()));  // row_mirror
  if constexpr (G >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  if constexpr (G >= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  return v;
}

// Merged over groups of G lanes; every lane gets the same triple.
template <int G>
__device__ __forceinline__ Stat merge_lanes(Stat a) {
  a.raise(fold_lanes<G>(a.m, [](float x, float y) { return fmaxf(x, y); }));
  const auto add = [](float x, float y) { return x + y; };
  a.s = fold_lanes<G>(a.s, add);
  a.h = fold_lanes<G>(a.h, add);
  return a;
}

// What a row's gradient needs: element j gets 2^d (base + k1 d), d from the
// shift of m, and slope more at the action; n open elements (0: none).
struct RowSlope {
  float m, base, k1, slope;
  int n, action;
};

// A row cut at the 16-byte boundaries of memory (of the gradient's, where
// there is one): `head` elements, `all` pieces, fewer elements than a piece.
// The first `open` pieces are all open, the next may be in part.
template <bool BF16>
struct RowCut {
  static constexpr int E = Elem<BF16>::kPer, kBytes = Elem<BF16>::kBytes;
  int head, open, all, n, V;
  __device__ RowCut(const char* at, int n_, int V_) : n(n_), V(V_) {
    head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(at) & 15)) & 15) / kBytes);
    all = (V - head) / E;
    open = max(n - head, 0) / E;
  }
  __device__ int64_t byte(int piece) const { return static_cast<int64_t>(piece) * 16 + head * kBytes; }
  // The element outside the pieces that is the lane's, V or more: none.
  __device__ int edge(int lane) const {
    return lane < 8 ? (lane < head ? lane : V) : (lane < 16 ? head + all * E + lane - 8 : V);
  }
  // Its element of the piece that is open in part; n or more: none.
  __device__ int part(int lane) const { return lane < E && open < all ? head + open * E + lane : n; }
  __device__ int closed() const { return open + (part(0) < n ? 1 : 0); }  // the first piece with nothing open
};

// The gradient's elements from the logits'.  ENT: with an entropy term.
template <bool BF16, bool ENT>
struct Slope {
  using X = Elem<BF16>;
  Shift sh;
  RowSlope rs;
  int at_piece, at_element;
  __device__ Slope(const RowSlope& r, int head) : sh(r.m), rs(r) {
    at_piece = (r.action - head) >> (BF16 ? 3 : 2);
    at_element = (r.action - head) & (X::kPer - 1);
  }
  __device__ float open(float x) const {
    const float d = sh(x), e = __builtin_amdgcn_exp2f(d);
    return ENT ? e * fmaf(rs.k1, fmaxf(d, kFarDown), rs.base) : e * rs.base;
  }
  __device__ u32x4 piece(u32x4 v, int i) const {
    float x[X::kPer];
    X::unpack(v, x);
#pragma unroll
    for (int e = 0; e < X::kPer; ++e) x[e] = open(x[e]);
    if (i == at_piece)
#pragma unroll
      for (int e = 0; e < X::kPer; ++e) x[e] += e == at_element ? rs.slope : 0.0f;
    return X::pack(x);
  }
  // Element j < V of the row.
  __device__ void one(const char* row, char* out, int j) const {
    float g = 0.0f;
    if (j < rs.n) g = open(X::get(row + static_cast<int64_t>(j) * X::kBytes)) + (j == rs.action ? rs.slope : 0.0f);
    X::put(out + static_cast<int64_t>(j) * X::kBytes, g);
  }
};

// What closing a row takes, beside its statistics.
struct RowIn {
  float w, xa;
  int n, a;
};
// Its constants of the loss.
struct RowLoss {
  float old, adv, ref;
};
template <bool GRAD>
__device__ __forceinline__ RowLoss row_loss(const RowParams& p, int64_t t) {
  if constexpr (GRAD) return {p.old[t], p.adv[t], p.ref ? p.ref[t] : 0.0f};
  return {};
}

// The row's own figures; WRITES: to the outputs, and its terms are added to sum.
template <bool GRAD, bool WRITES>
__device__ __forceinline__ RowSlope close_row(const RowParams& p, int64_t t, RowIn in, RowLoss lc, Stat st,
                                              PolicyTerms* sum) {
  double logp = 0.0, entropy = 0.0;
  RowSlope rs{st.m, 0.0f, 0.0f, 0.0f, 0, in.a};
  if (in.n > 0 && st.s != 0.0f) {  // 0: nothing open
    const double s = st.s, logs = log(s);
    logp = static_cast<double>(in.xa) - Shift(st.m).natural() - logs;
    entropy = logs - static_cast<double>(st.h) / s * kLn2;
    if constexpr (GRAD) {
      PolicyTerms unused{};
      const double slope =
          policy_decision(logp, entropy, lc.old, lc.adv, in.w, p.ref != nullptr, lc.ref, p.coef, WRITES ? *sum : unused);
      const double c = static_cast<double>(p.coef.entropy) * in.w;
      rs.n = in.n;
      rs.slope = static_cast<float>(slope);
      rs.base = static_cast<float>(((p.coef.entropy != 0.0f ? c * (entropy - logs) : 0.0) - slope) / s);
      rs.k1 = p.coef.entropy != 0.0f ? static_cast<float>(c * kLn2 / s) : 0.0f;
    }
  } else if (in.w != 0.0f) {
    logp = entropy = __builtin_nan("");
    if (WRITES) atomicOr(p.status, DORA_DEV_ACTION);
  }
  if (WRITES) {
    p.logp_out[t] = static_cast<float>(logp);
    if (p.entropy_out) p.entropy_out[t] = static_cast<float>(entropy);
  }
  return rs;
}

// Threads of a workgroup for rows of L threads.
constexpr int group_threads(int L) { return L >= 256 ? L : (L == 64 ? 512 : 256); }

// L threads a row.  Each holds its first NV pieces (thread i: pieces i, i + L,
// ...) in registers from the statistics to the gradient and the next NS in
// shared memory, so that a row of up to L (NV + NS) pieces is read once; what
// is past them is read again.  Shared memory only extends the longest rows
// (2048 x 131072 fp32 505 -> 456 us); taking registers off shorter ones for a
// third workgroup a compute unit made them slower (2048 x 50257 bf16 83 -> 89).
template <bool BF16, int L, int NV, int NS, int WG, bool GRAD, bool ENT>
__global__ __launch_bounds__(WG, 4) void policy_rows_kernel(RowParams p) {
  using X = Elem<BF16>;
  constexpr int kRows = WG / L, kWaves = L / 64;
  constexpr bool kPark = GRAD && NV > 4;
  // Past the caches, us a pass without and with: stores of 1024 x 32000 fp32
  // 54.6, 48.8, of 8192 x 4096 bf16 36.7, 30.5; rows of 1024 threads are better
  // off through them (8192 x 131072 bf16 800, 811).  Loads as well only for 256
  // threads a row (8192 x 32768 bf16 227, 204; for 64 and 512 30.5, 33.2 and
  // 48.8, 50.7).
  constexpr bool kPassStores = L <= 512, kPassLoads = GRAD && L == 256;
  __shared__ Stat s_stat[L > 64 ? kWaves : kRows];
  __shared__ RowIn s_in[kRows];
  __shared__ RowSlope s_slope[kRows];
  __shared__ u32x4 s_held[kPark ? NV * 64 : 1];
  __shared__ u32x4 s_stash[NS > 0 ? NS * L : 1];
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows, t = min(t0 + group, static_cast<int64_t>(p.T) - 1);
  const bool mine = t0 + group < p.T;  // a group past the last row goes along with it, and writes nothing
  const char* row = p.logits + t * p.ld * X::kBytes;
  char* out = GRAD ? p.grad + t * p.ld_grad * X::kBytes : nullptr;
  // For the row that this thread may close.
  const RowLoss lc = row_loss<GRAD>(p, min(t0 + static_cast<int>(threadIdx.x) % kRows, static_cast<int64_t>(p.T) - 1));
  Taker tk;
  u32x4 held[NV];
  // Loads are unconditional (a piece past the last one is the last one again),
  // so that they are counted and waited for one by one.
  auto load = [&](const RowCut<BF16>& cut, int last) {
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = load_piece<BF16, kPassLoads>(row + cut.byte(min(lane + i * L, last)));
    asm volatile("" ::: "memory");
  };
  RowIn in;
  if constexpr (L <= 64) {
    // Short rows are loaded beside what says whether they count, long ones
    // after it.
    const RowCut<BF16> whole(GRAD ? out : row, p.V, p.V);
    if (whole.all > 0) load(whole, whole.all - 1);
  }
  in.n = open_row(p, t, in.w, in.a);
  const RowCut<BF16> cut(GRAD ? out : row, in.n, p.V);
  // The action's logit, ahead of a long row's pieces: waiting for it is not waiting for them.
  in.xa = X::get(row + static_cast<int64_t>(in.a) * X::kBytes);
  if (L > 64 && cut.open > 0) load(cut, cut.open - 1);  // the same for all threads of a row
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (lane + i * L < cut.open) {
      float x[X::kPer];
      X::unpack(held[i], x);
      tk.take(x);
    }
  }
  if constexpr (NS > 0) {
    constexpr int kFlight = 2;
#pragma unroll
    for (int b = 0; b < NS; b += kFlight) {
      u32x4 v[kFlight];
      if (NV * L + b * L < cut.open) {
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
          v[k] = load_piece<BF16, kPassLoads>(row + cut.byte(min(lane + (NV + b + k) * L, cut.open - 1)));
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
          if (b + k < NS && lane + (NV + b + k) * L < cut.open) {
            s_stash[(b + k) * L + lane] = v[k];
            float x[X::kPer];
            X::unpack(v[k], x);
            tk.take(x);
          }
        }
      }
    }
  }
  for (int i = lane + (NV + NS) * L; i < cut.open; i += L) {
    float x[X::kPer];
    X::unpack(load_piece<BF16>(row + cut.byte(i)), x);
    tk.take(x);
  }
  if (cut.edge(lane) < in.n) take_one<BF16>(tk, row, cut.edge(lane));
  if (cut.part(lane) < in.n) take_one<BF16>(tk, row, cut.part(lane));

  // The first wave closes the workgroup's rows, a lane a row (all its lanes the
  // one row of a wide group): 64-bit exp and log by all waves would cost as
  // much as the rows' own exponentials.
  const Stat st = merge_lanes<(L < 64 ? L : 64)>(tk.st);
  if (lane == 0) s_in[group] = in;
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) s_stat[threadIdx.x >> 6] = st;
  } else {
    if (lane == 0) s_stat[group] = st;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    // Its pieces wait in shared memory meanwhile: the registers of the 64-bit
    // functions would come on top of them, for every wave.
    if constexpr (kPark) {
#pragma unroll
      for (int i = 0; i < NV; ++i) s_held[i * 64 + threadIdx.x] = held[i];
      asm volatile("" ::: "memory");
    }
    PolicyTerms sum{};
    if constexpr (L > 64) {
      const Stat all = merge_lanes<kWaves>(s_stat[threadIdx.x % kWaves]);
      if (threadIdx.x == 0) s_slope[0] = close_row<GRAD, true>(p, t0, s_in[0], lc, all, &sum);
    } else {
      const int r = threadIdx.x;
      if (r < kRows && t0 + r < p.T) s_slope[r] = close_row<GRAD, true>(p, t0 + r, s_in[r], lc, s_stat[r], &sum);
#pragma unroll
      for (int k = 0; GRAD && k < kPolicyTerms; ++k)
#pragma unroll
        for (int off = kRows / 2; off > 0; off >>= 1) sum.v[k] += __shfl_xor(sum.v[k], off);
    }
    if constexpr (GRAD) {
      if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < kPolicyTerms; ++k) {
          if (gridDim.x == 1) p.stats[k] = static_cast<float>(sum.v[k]);  // there is nothing to add to it
          else p.parts[static_cast<int64_t>(blockIdx.x) * kPolicyTerms + k] = sum.v[k];
        }
      }
    }
    if constexpr (kPark) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < NV; ++i) held[i] = s_held[i * 64 + threadIdx.x];
    }
  }
  if constexpr (GRAD) {
    __syncthreads();
    if (!mine) return;
    const RowSlope rs = s_slope[group];
    // A row that was found bad after all has nothing open.
    const RowCut<BF16> cut(out, rs.n, p.V);
    const Slope<BF16, ENT> slope(rs, cut.head);
    // Opaque to the compiler, which would otherwise keep the pieces unpacked
    // (twice the registers) from the statistics on.
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(held[i]));
    auto put = [&](u32x4 v, int i) { store_piece<BF16, kPassStores>(out + cut.byte(i), slope.piece(v, i)); };
    for (int i = lane + (NV + NS) * L; i < cut.open; i += L) put(load_piece<BF16>(row + cut.byte(i)), i);
    if constexpr (NS > 0)
#pragma unroll
      for (int k = 0; k < NS; ++k)
        if (lane + (NV + k) * L < cut.open) put(s_stash[k * L + lane], lane + (NV + k) * L);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (lane + i * L < cut.open) put(held[i], lane + i * L);
    for (int i = cut.closed() + lane; i < cut.all; i += L) store_piece<BF16, kPassStores>(out + cut.byte(i), u32x4{});
    if (lane < X::kPer && cut.part(0) < rs.n)
      slope.one(row, out, cut.head + cut.open * X::kPer + lane);
    if (cut.edge(lane) < p.V) slope.one(row, out, cut.edge(lane));
  }
}

// Statistics of the open pieces [lo, hi) of a row and, if `ends`, of the open
// elements outside the pieces that are open.  Four pieces in flight a thread.
template <bool BF16, bool PASSING>
__device__ __forceinline__ Stat range_stats(const char* row, const RowCut<BF16>& cut, int lo, int hi, bool ends) {
  using X = Elem<BF16>;
  constexpr int kFlight = 4;
  const int tid = threadIdx.x;
  Taker tk;
  for (int i = lo + tid; i < hi; i += kFlight * kThreads) {
    u32x4 v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) v[k] = load_piece<BF16, PASSING>(row + cut.byte(min(i + k * kThreads, hi - 1)));
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (i + k * kThreads < hi) {
        float x[X::kPer];
        X::unpack(v[k], x);
        tk.take(x);
      }
    }
  }
  if (ends && cut.edge(tid) < cut.n) take_one<BF16>(tk, row, cut.edge(tid));
  if (ends && cut.part(tid) < cut.n) take_one<BF16>(tk, row, cut.part(tid));
  return tk.st;
}

// A workgroup's share of a row's pieces, split over p.split.
__device__ __forceinline__ int2 share_of(const RowParams& p, int chunk, int all) {
  const int each = (all + p.split - 1) / p.split;
  return make_int2(min(all, chunk * each), min(all, (chunk + 1) * each));
}

// Statistics of long rows, p.split workgroups a row.  One a row: it closes the
// row (log-probability only), and the logits pass the caches by (4096 x 50257
// bf16 54 us; through them 62).  Several: each leaves its triple for the next
// launch, with the action's logit (which a gradient over the logits would
// overwrite).
template <bool BF16, bool SPLIT>
__global__ __launch_bounds__(kThreads) void policy_stats_kernel(RowParams p) {
  using X = Elem<BF16>;
  __shared__ Stat s_red[kThreads / 64];
  const int64_t t = blockIdx.x / p.split;
  const int chunk = blockIdx.x % p.split;
  RowIn in;
  in.n = open_row(p, t, in.w, in.a);
  const char* row = p.logits + t * p.ld * X::kBytes;
  const RowCut<BF16> cut(p.grad ? p.grad + t * p.ld_grad * X::kBytes : row, in.n, p.V);
  const int2 c = share_of(p, chunk, cut.all);
  Stat st = merge_lanes<64>(range_stats<BF16, !SPLIT>(row, cut, min(c.x, cut.open), min(c.y, cut.open), chunk == 0));
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = st;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  st = merge_lanes<kThreads / 64>(s_red[threadIdx.x % (kThreads / 64)]);
  in.xa = X::get(row + static_cast<int64_t>(in.a) * X::kBytes);
  if (threadIdx.x > 0) return;
  if (SPLIT) p.split_stats[blockIdx.x] = make_float4(st.m, st.s, st.h, in.xa);
  else close_row<false, true>(p, t, in, RowLoss{}, st, nullptr);
}

// Row t closed from its workgroups' triples by a group of G lanes.
template <bool GRAD, bool WRITES, int G>
__device__ __forceinline__ RowSlope close_split_row(const RowParams& p, int64_t t, PolicyTerms* sum) {
  constexpr int kEach = kMaxSplit / G;
  const int lane = threadIdx.x % G;
  const float4* from = p.split_stats + t * p.split;
  float4 v[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) v[k] = from[min(lane + k * G, p.split - 1)];
  RowIn in;
  in.n = open_row(p, t, in.w, in.a);
  const RowLoss lc = row_loss<GRAD>(p, t);
  in.xa = v[0].w;
  Stat st = Stat::none();
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    if (lane + k * G < p.split) st.merge(Stat{v[k].x, v[k].y, v[k].z});
  st = merge_lanes<G>(st);
  RowSlope rs{};
  if (lane == 0) rs = close_row<GRAD, WRITES>(p, t, in, lc, st, sum);
  return rs;  // the first lane's
}

// Log-probabilities of split rows.
__global__ __launch_bounds__(kThreads) void policy_close_kernel(RowParams p) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kThreads / 8) + threadIdx.x / 8;
  if (t < p.T) close_split_row<false, true, 8>(p, t, nullptr);
}

// Gradient of split rows: each workgroup closes its row for itself and writes
// its share.  One workgroup more, the last, closes all rows for the outputs
// and sums.
template <bool BF16, bool ENT>
__global__ __launch_bounds__(kThreads, 3) void policy_split_grad_kernel(RowParams p) {
  using X = Elem<BF16>;
  __shared__ RowSlope s_slope;
  __shared__ PolicyTerms s_terms[kThreads / 8];
  const int64_t t = blockIdx.x / p.split;
  const int tid = threadIdx.x;
  if (t == p.T) {
    PolicyTerms sum{};
    for (int64_t r = tid / 8; r < p.T; r += kThreads / 8) close_split_row<true, true, 8>(p, r, &sum);
    if (tid % 8 == 0) s_terms[tid / 8] = sum;
    __syncthreads();
    if (tid < kPolicyTerms) {
      double v = 0.0;
      for (int i = 0; i < kThreads / 8; ++i) v += s_terms[i].v[tid];
      p.stats[tid] = static_cast<float>(v);
    }
    return;
  }
  if (tid < 64) {
    const RowSlope rs = close_split_row<true, false, 64>(p, t, nullptr);
    if (tid == 0) s_slope = rs;
  }
  __syncthreads();
  const RowSlope rs = s_slope;
  const char* row = p.logits + t * p.ld * X::kBytes;
  char* out = p.grad + t * p.ld_grad * X::kBytes;
  const RowCut<BF16> cut(out, rs.n, p.V);
  const Slope<BF16, ENT> slope(rs, cut.head);
  const int chunk = blockIdx.x % p.split;
  const int2 c = share_of(p, chunk, cut.all);
  for (int i = c.x + tid; i < min(c.y, cut.open); i += kThreads)
    store_piece<BF16>(out + cut.byte(i), slope.piece(load_piece<BF16>(row + cut.byte(i)), i));
  for (int i = max(c.x, cut.closed()) + tid; i < c.y; i += kThreads) store_piece<BF16>(out + cut.byte(i), u32x4{});
  if (c.x <= cut.open && cut.open < c.y && cut.part(0) < rs.n && tid < X::kPer)
    slope.one(row, out, cut.head + cut.open * X::kPer + tid);
  if (chunk == 0 && cut.edge(tid) < p.V) slope.one(row, out, cut.edge(tid));
}

// Sums of the terms of workgroups [blockIdx per_group, + per_group) of n, to
// out[blockIdx] or, rounded, to stats.  Thread i adds term i % 6 of every 64th
// set, eight sets in flight; then 8 x 8 sums a term meet in order.
constexpr int kFinishSets = 64, kFinishThreads = kFinishSets * kPolicyTerms;
__global__ __launch_bounds__(kFinishThreads) void policy_finish_kernel(const double* parts, int32_t n, int32_t per_group,
                                                                       double* out, float* stats) {
  constexpr int kFlight = 8;
  __shared__ double s_sum[kFinishThreads];
  const int tid = threadIdx.x;
  const int64_t lo = static_cast<int64_t>(blockIdx.x) * per_group, hi = min(static_cast<int64_t>(n), lo + per_group);
  double sum = 0.0;
  for (int64_t i = lo + tid / kPolicyTerms; i < hi; i += kFlight * kFinishSets) {
    double v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      v[k] = parts[min(i + k * kFinishSets, hi - 1) * kPolicyTerms + tid % kPolicyTerms];
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < kFlight; ++k) sum += i + k * kFinishSets < hi ? v[k] : 0.0;
  }
  s_sum[tid] = sum;
  __syncthreads();
  if (tid < 8 * kPolicyTerms) {
    sum = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += s_sum[tid + k * 8 * kPolicyTerms];
  }
  __syncthreads();
  if (tid < 8 * kPolicyTerms) s_sum[tid] = sum;
  __syncthreads();
  if (tid < kPolicyTerms) {
    sum = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += s_sum[tid + k * kPolicyTerms];
    if (stats) stats[tid] = static_cast<float>(sum);
    else out[static_cast<int64_t>(blockIdx.x) * kPolicyTerms + tid] = sum;
  }
}

template <bool BF16, bool GRAD, bool ENT, int L, int NV, int NS = 0>
void launch_shape(const RowParams& p, hipStream_t st) {
  constexpr int kWG = group_threads(L), kRows = kWG / L;
  const int groups = (p.T + kRows - 1) / kRows;
  // A batch of short rows that one wide workgroup holds needs no second launch
  // for its sums (64 x 96 fp32 8.6 -> 5.8 us, 16 x 1000 8.4 -> 6.6).
  if constexpr (GRAD && L <= 64) {
    if (groups > 1 && p.T <= 1024 / L) {
      hipLaunchKernelGGL((policy_rows_kernel<BF16, L, NV, NS, 1024, GRAD, ENT>), dim3(1), dim3(1024), 0, st, p);
      return;
    }
  }
  hipLaunchKernelGGL((policy_rows_kernel<BF16, L, NV, NS, kWG, GRAD, ENT>), dim3(groups), dim3(kWG), 0, st, p);
  if (GRAD && groups > 1) launch_policy_finish(p.parts, groups, p.stats, st);
}

// Workgroups a row, for long rows that are few: as many as bring about
// kSplitGroups of them, each with at least two pieces a thread.  It pays where
// a row is long against the batch; the loss closes all rows in one workgroup
// besides.  us a pass split and not, bf16: loss of 8 x 131072 8.3, 20.2, 128 x
// 131072 23.0, 24.9, 64 x 32768 9.9, 11.9, but 192 x 131072 34.9, 27.7, 128 x
// 32768 14.3, 11.9, 64 x 10000 9.3, 8.8; log-probabilities of 8 x 131072 7.9, 20.4,
// 256 x 131072 18.2, 22.4, but 8 x 32768 8.0, 7.1.
constexpr int kSplitGroups = 512;
int split_of(bool grad, int32_t T, int pieces) {
  if (grad ? T > 128 || pieces / 64 < T : T > 256 || pieces <= 4096) return 1;
  return std::max(1, std::min({kSplitGroups / T, pieces / (2 * kThreads), kMaxSplit}));
}

// The fewest threads a row that hold it in 16 pieces each (8 where rows share
// a workgroup), and the fewest pieces, of those there are kernels for: a piece
// too many is registers that another row could use (2048 x 50257 bf16, 13 of
// 16 pieces in use 114 us, of 13 106).
template <bool BF16, bool GRAD, bool ENT>
void launch_rows(RowParams p, hipStream_t st) {
  const int pieces = (p.V + Elem<BF16>::kPer - 1) / Elem<BF16>::kPer;
  if (pieces <= 16) return launch_shape<BF16, GRAD, ENT, 16, 1>(p, st);
  if (pieces <= 32) return launch_shape<BF16, GRAD, ENT, 16, 2>(p, st);
  if (pieces <= 64) return launch_shape<BF16, GRAD, ENT, 16, 4>(p, st);
  if (pieces <= 256) return launch_shape<BF16, GRAD, ENT, 64, 4>(p, st);
  if (pieces <= 512) return launch_shape<BF16, GRAD, ENT, 64, 8>(p, st);
  p.split = p.split_stats ? split_of(GRAD, p.T, pieces) : 1;
  if (p.split > 1 || !GRAD) {
    const dim3 groups(static_cast<uint32_t>(p.T) * p.split);
    if (p.split > 1) hipLaunchKernelGGL((policy_stats_kernel<BF16, true>), groups, dim3(kThreads), 0, st, p);
    else hipLaunchKernelGGL((policy_stats_kernel<BF16, false>), groups, dim3(kThreads), 0, st, p);
    if constexpr (GRAD)
      hipLaunchKernelGGL((policy_split_grad_kernel<BF16, ENT>), dim3(p.T * p.split + 1), dim3(kThreads), 0, st, p);
    else if (p.split > 1)
      hipLaunchKernelGGL(policy_close_kernel, dim3((p.T * 8 + kThreads - 1) / kThreads), dim3(kThreads), 0, st, p);
    return;
  }
  if constexpr (GRAD) {
    const int L = pieces <= 256 * 16 ? 256 : (pieces <= 512 * 16 ? 512 : 1024), each = (pieces + L - 1) / L;
    if (L == 256) {
      if (each <= 4) launch_shape<BF16, GRAD, ENT, 256, 4>(p, st);
      else if (each <= 8) launch_shape<BF16, GRAD, ENT, 256, 8>(p, st);
      else if (each <= 12) launch_shape<BF16, GRAD, ENT, 256, 12>(p, st);
      else launch_shape<BF16, GRAD, ENT, 256, 16>(p, st);
    } else if (L == 512) {
      if (each <= 10) launch_shape<BF16, GRAD, ENT, 512, 10>(p, st);
      else if (each <= 12) launch_shape<BF16, GRAD, ENT, 512, 12>(p, st);
      else if (each <= 14) launch_shape<BF16, GRAD, ENT, 512, 14>(p, st);
      else launch_shape<BF16, GRAD, ENT, 512, 16>(p, st);
    } else {
      if (each <= 10) launch_shape<BF16, GRAD, ENT, 1024, 10>(p, st);
      else if (each <= 12) launch_shape<BF16, GRAD, ENT, 1024, 12>(p, st);
      else if (each <= 14) launch_shape<BF16, GRAD, ENT, 1024, 14>(p, st);
      else if (each <= 16) launch_shape<BF16, GRAD, ENT, 1024, 16>(p, st);
      else launch_shape<BF16, GRAD, ENT, 1024, 16, 8>(p, st);
    }
  }
}

// Sets of sums that the workgroups of T rows of V elements write (of the
// element type that has fewer rows a workgroup).
int32_t row_groups(int32_t T, int32_t V) {
  const int pieces = (V + 3) / 4;
  const int rows = pieces <= 64 ? group_threads(16) / 16 : (pieces <= 512 ? group_threads(64) / 64 : 1);
  return (T + rows - 1) / rows;
}

int check_rows(const void* logits, int64_t ld, const int32_t* actions, int32_t T, int32_t V, dora_dtype dtype,
               const int32_t* dev_status) {
  if (!logits || !actions || !dev_status) return DORA_ERR_NULL;
  if (dtype != DORA_BF16 && dtype != DORA_F32) return DORA_ERR_DTYPE;
  if (T < 1 || T > DORA_MAX_DECISIONS || V < 1 || V > DORA_MAX_ACTIONS || ld < V || ld > (int64_t{1} << 32))
    return DORA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == DORA_BF16 ? 2 : 4)) return DORA_ERR_ALIGN;
  return DORA_OK;
}

// Rows of V elements every ld at base against rows every ld_o at other: apart,
// the same rows, or rows in the gaps of the others.
bool rows_clash(uintptr_t base, int64_t ld, uintptr_t other, int64_t ld_o, int32_t T, int32_t V, int elt) {
  const uintptr_t len = (static_cast<uintptr_t>(T - 1) * ld + V) * elt;
  const uintptr_t len_o = (static_cast<uintptr_t>(T - 1) * ld_o + V) * elt;
  if (base + len <= other || other + len_o <= base) return false;
  if (ld != ld_o) return true;
  if (base == other) return false;
  const uintptr_t off = (other > base ? other - base : base - other) % (static_cast<uintptr_t>(ld) * elt);
  const uintptr_t row = static_cast<uintptr_t>(V) * elt;
  return off < row || off + row > static_cast<uintptr_t>(ld) * elt;
}

// Rows of V elements every ld at base against vectors, which may stand in the
// gaps between the rows.
bool rows_meet(const void* base, int64_t ld, int32_t T, int32_t V, int elt, std::initializer_list<Extent> vectors) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(base), pitch = static_cast<uintptr_t>(ld) * elt;
  const uintptr_t row = static_cast<uintptr_t>(V) * elt, end = lo + (T - 1) * pitch + row;
  for (const Extent& v : vectors) {
    if (!v.at || v.at >= end || v.at + v.bytes <= lo) continue;
    // The last row that starts at or before the vector does, and the one after it.
    const uintptr_t start = v.at > lo ? lo + (v.at - lo) / pitch * pitch : lo;
    if (v.at < start + row || v.at + v.bytes > start + pitch) return true;
  }
  return false;
}

}  // namespace

void launch_policy_finish(double* parts, int32_t n, float* stats, hipStream_t stream) {
  if (n > kFinishDirect) {
    const int32_t each = (n + kFinishGroups - 1) / kFinishGroups, groups = (n + each - 1) / each;
    double* mid = parts + static_cast<int64_t>(n) * kPolicyTerms;
    hipLaunchKernelGGL(policy_finish_kernel, dim3(groups), dim3(kFinishThreads), 0, stream, parts, n, each, mid, nullptr);
    parts = mid;
    n = groups;
  }
  hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(kFinishThreads), 0, stream, parts, n, n, nullptr, stats);
}

}  // namespace dora

extern "C" size_t dora_policy_workspace_size(int32_t T, int32_t V) {
  using namespace dora;
  if (T < 1 || T > DORA_MAX_DECISIONS || V < 1 || V > DORA_MAX_ACTIONS) return 0;
  // Either the sums' sets or the split rows' triples; the type with more pieces a row splits further.
  const int most = std::max(split_of(true, T, (V + 3) / 4), split_of(false, T, (V + 3) / 4));
  const size_t split = static_cast<size_t>(T) * most * sizeof(float4);
  return std::max(policy_parts_bytes(row_groups(T, V)), (split + 255) & ~size_t(255));
}

extern "C" int dora_action_logprob(const void* logits, int64_t ld, const int32_t* actions, const int32_t* legal,
                                   const float* weight, int32_t T, int32_t V, dora_dtype dtype, float* logprob_out,
                                   float* entropy_out, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                   void* stream) {
  using namespace dora;
  const int rc = check_rows(logits, ld, actions, T, V, dtype, dev_status);
  if (rc != DORA_OK) return rc;
  if (!logprob_out) return DORA_ERR_NULL;
  if (workspace &&
      (reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < dora_policy_workspace_size(T, V)))
    return DORA_ERR_WORKSPACE;
  const size_t vec = static_cast<size_t>(T) * 4;
  const Extent lp_out(logprob_out, vec), ent_out(entropy_out, vec), ws(workspace, dora_policy_workspace_size(T, V)),
      flag(dev_status, 4);
  if (outputs_clash({lp_out, ent_out, ws, flag}, {Extent(actions, vec), Extent(legal, vec)}, {Extent(weight, vec)}) ||
      rows_meet(logits, ld, T, V, dtype == DORA_BF16 ? 2 : 4, {lp_out, ent_out, ws, flag}))
    return DORA_ERR_OVERLAP;
  RowParams p{};
  p.logits = static_cast<const char*>(logits);
  p.ld = ld;
  p.actions = actions;
  p.legal = legal;
  p.weight = weight;
  p.T = T;
  p.V = V;
  p.logp_out = logprob_out;
  p.entropy_out = entropy_out;
  p.split_stats = static_cast<float4*>(workspace);
  p.split = 1;
  p.status = dev_status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == DORA_BF16) launch_rows<true, false, false>(p, st);
  else launch_rows<false, false, false>(p, st);
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}

extern "C" int dora_policy_loss(const void* logits, int64_t ld, const int32_t* actions, const int32_t* legal,
                                const float* old_logprob, const float* ref_logprob, const float* advantage,
                                const float* weight, int32_t T, int32_t V, dora_dtype dtype, float clip_low,
                                float clip_high, float kl_coef, float entropy_coef, void* dlogits, int64_t ld_grad,
                                float* logprob_out, float* stats_out, void* workspace, size_t workspace_bytes,
                                int32_t* dev_status, void* stream) {
  using namespace dora;
  const int rc = check_rows(logits, ld, actions, T, V, dtype, dev_status);
  if (rc != DORA_OK) return rc;
  if (!old_logprob || !advantage || !dlogits || !logprob_out || !stats_out) return DORA_ERR_NULL;
  if (ld_grad < V || ld_grad > (int64_t{1} << 32)) return DORA_ERR_SHAPE;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f)) return DORA_ERR_SHAPE;
  if (!(kl_coef - kl_coef == 0.0f && entropy_coef - entropy_coef == 0.0f)) return DORA_ERR_SHAPE;
  if (kl_coef != 0.0f && !ref_logprob) return DORA_ERR_NULL;
  const int elt = dtype == DORA_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(dlogits) % elt) return DORA_ERR_ALIGN;
  if (rows_clash(reinterpret_cast<uintptr_t>(logits), ld, reinterpret_cast<uintptr_t>(dlogits), ld_grad, T, V, elt))
    return DORA_ERR_OVERLAP;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u ||
      workspace_bytes < dora_policy_workspace_size(T, V))
    return DORA_ERR_WORKSPACE;
  const size_t vec = static_cast<size_t>(T) * 4;
  const Extent lp_out(logprob_out, vec), sums(stats_out, kPolicyTerms * 4), ws(workspace, dora_policy_workspace_size(T, V)),
      flag(dev_status, 4), act(actions, vec), open(legal, vec), old(old_logprob, vec), ref(ref_logprob, vec),
      adv(advantage, vec), w(weight, vec);
  if (outputs_clash({sums, ws, flag}, {act, open, old, ref, adv, w, lp_out}, {}) ||
      outputs_clash({lp_out}, {act, open}, {old, ref, adv, w}) ||
      rows_meet(logits, ld, T, V, elt, {lp_out, sums, ws, flag}) ||
      rows_meet(dlogits, ld_grad, T, V, elt, {lp_out, sums, ws, flag, act, open, old, ref, adv, w}))
    return DORA_ERR_OVERLAP;
  // Split rows are closed by several workgroups, of which one writes the log-probability: not in a constant's place.
  const bool in_place = lp_out.meets(old) || lp_out.meets(ref) || lp_out.meets(adv) || lp_out.meets(w);
  RowParams p{static_cast<const char*>(logits), ld, actions, legal, old_logprob, ref_logprob, advantage, weight, T, V,
              PolicyCoef{clip_low, clip_high, kl_coef, entropy_coef}, static_cast<char*>(dlogits), ld_grad,
              logprob_out, nullptr, static_cast<double*>(workspace), in_place ? nullptr : static_cast<float4*>(workspace), 1,
              stats_out, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool ent = entropy_coef != 0.0f;
  if (dtype == DORA_BF16) ent ? launch_rows<true, true, true>(p, st) : launch_rows<true, true, false>(p, st);
  else ent ? launch_rows<false, true, true>(p, st) : launch_rows<false, true, false>(p, st);
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
