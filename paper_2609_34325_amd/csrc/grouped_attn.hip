// Attention over packed sequences with grouped heads, forward and backward: the
// training and language-model form of varlen_attn.hip (own boundaries for
// queries and keys, causal or full, 32/64/128-wide heads, bf16 or fp32).
//
// The G = H / Hk heads that read one key head are stacked: sequence b and key
// head hk make one problem of nq G rows (row r = query r / G of head hk G + r %
// G) against nk keys, with limit(r) = the keys that row r sees, nk or, causal,
// r / G + 1 + nk - nq.  Keys and values are then read once for the G heads, dk
// and dv are sums over rows like any other, and one query of many heads fills a
// tile.  With c = softmax_scale log2(e):
//   s = c q k^T,  m = max s,  p = 2^(s - m),  l = sum p
//   out = p v / l,  lse = (m + log2 l) ln 2
// in one pass over the keys, m, l and the products' sums in fp32.  Backward,
// P = 2^(s - lse log2 e), delta = rowsum(dout out):
//   grad_q   a tile of rows over the keys:  dS = P (dout v^T - delta), dq += dS k
//   grad_kv  a tile of keys over the rows:  dv += P^T dout, dk += dS^T q
// Each forms P and dS for itself (seven products in place of five, eight for bf16
// heads of 128), so that no sum goes through memory and results do not depend on
// timing.  Eight packed sequences of up to 8192, 30497 rows, 32 query and 8 key
// heads of 128, bf16, causal: forward 1.25 ms, grad_q 1.6, grad_kv 2.9 to 3.3; 650 to
// 700 TFLOP/s of seven products, 930 to 1000 of the ten that are formed, where a large
// library product reaches 1254 on the same card.  Sums of dq by atomics would save
// three of the ten, and depend on timing.
//
// Kernels of 64 rows (16 a wave) take every type and width; those of 128 rows (32
// a wave) longer sequences of bf16 heads of 64 and 128.
//
// Tiles of sequences are found without a plan: tile t of all belongs to the last
// b with floor(cu[b] G / tile) + b <= t.  That leaves each sequence at least its
// tiles' numbers, and at most total / tile + B numbers in all, which the host
// knows; every wave looks its sequence up with ballots over 64 boundaries.  Up to
// 64 sequences, whose boundaries one wave holds, are numbered by length (by_length).
#include <math.h>

#include <algorithm>

#include "dora_internal.h"
#include "grouped_attn_split.h"
#include "lanes.h"
#include "rows.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttnArgs {
  RowView q, k, v, out, dout, dq, dk, dv;
  const int32_t* cu_q;
  const int32_t* cu_k;
  int32_t B, H, Hk, G;
  uint32_t g_mul, g_shift;  // r / G = mulhi(r, g_mul) >> g_shift for r < 2^31, G > 1
  int64_t total_q, total_k;
  int32_t max_q, max_k, causal;
  float scale, c2;  // softmax_scale, softmax_scale * log2(e)
  float* lse;
  float2* stat;  // of a row: log2 of its sum of exponentials, delta
  float* part;       // split sums
  float2* part_ml;   // of a row's part: m and l
  int32_t part_rows;  // rows of a part
  int32_t splits;     // parts of a tile's keys (forward) or of a tile's rows (grad_kv)
  int32_t chunk;      // or: keys of a part, every sequence one tile of rows
  int32_t step;       // rows of whole queries in 64 (grad_kv_wide)
  int32_t blocks;
  int32_t mixed, ranked;  // the order of tiles: tile_number, by_length
  int32_t* status;
};

__device__ __forceinline__ int div_group(const AttnArgs& a, int r) {
  return a.G == 1 ? r : static_cast<int>(__umulhi(static_cast<uint32_t>(r), a.g_mul) >> a.g_shift);
}

// First tile number of sequence b, which begins at `boundary`.
__device__ __forceinline__ int64_t first_tile(int boundary, int b, int mul, int tile) {
  return static_cast<int64_t>(max(boundary, 0)) * mul / tile + b;
}

// Tile number of workgroup i of n (without heads): i, or (a.mixed) in another order, sixteen at a time, each sixteen turned
// one further than the last.  Numbers that hold no tile (a sequence of exactly one tile has one such beside it) recur at a
// fixed distance, and workgroups go to dies and shader engines by their number: in plain order the tiles that exist meet on
// half of the GPU (512 sequences of 64 rows, 8 heads of 64, bf16: 73 us in place of 51; 256 of 128 in the wide kernel 71 in
// place of 48).  Long sequences have few such numbers, and their tiles share keys in the L2 in plain order (5670 us in place
// of 6000 for forward and backward over eight of up to 8192).
__device__ __forceinline__ int tile_number(const AttnArgs& a, int i) {
  const int n = a.blocks / a.Hk, lo = i & ~15;
  return a.mixed && lo + 16 <= n ? lo | ((i + (i >> 4)) & 15) : i;
}

// The last b with first(b) <= t; every lane of the wave calls it.
template <class F>
__device__ __forceinline__ int last_at_most(int B, int64_t t, F first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 1) {
    const int stride = (n + 63) >> 6, at = lane * stride;
    const uint64_t hit = __ballot(at < n && first(lo + at) <= t);
    const int step = hit ? (63 - __builtin_clzll(hit)) * stride : 0;
    lo += step;
    n = min(stride, n - step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

struct Seq {
  int q0, nq, k0, nk;
};

__device__ __forceinline__ bool good_boundaries(const AttnArgs& a, int q0, int q1, int k0, int k1) {
  return q0 >= 0 && q1 >= q0 && q1 <= a.total_q && k0 >= 0 && k1 >= k0 && k1 <= a.total_k && q1 - q0 <= a.max_q &&
         k1 - k0 <= a.max_k;
}

// Sequence b; nothing of it where its boundaries are no good.
__device__ __forceinline__ bool sequence(const AttnArgs& a, int b, Seq* s) {
  const int q0 = a.cu_q[b], q1 = a.cu_q[b + 1], k0 = a.cu_k[b], k1 = a.cu_k[b + 1];
  if (!good_boundaries(a, q0, q1, k0, k1)) return false;
  *s = Seq{q0, q1 - q0, k0, k1 - k0};
  return true;
}

// The last sequence b with first(boundary, b) <= t, boundary = cu_q[b] (QUERIES) or cu_k[b]; false where its boundaries
// are no good.  Every lane of the wave calls it.  Fewer than 64 sequences take one trip to memory, each lane holding a
// boundary of both lists (a trip on cold lines is 1 to 2 us, of a small call's 10).
template <bool QUERIES, class F>
__device__ __forceinline__ bool locate(const AttnArgs& a, int64_t t, F first, int* found, Seq* s) {
  if (a.B >= 64) {
    const int32_t* cu = QUERIES ? a.cu_q : a.cu_k;
    *found = last_at_most(a.B, t, [&](int b) { return first(cu[b], b); });
    return sequence(a, *found, s);
  }
  const int lane = threadIdx.x & 63, at = min(lane, a.B);
  const int q = a.cu_q[at], k = a.cu_k[at];
  const uint64_t hit = __ballot(lane < a.B && first(QUERIES ? q : k, lane) <= t);
  const int b = hit ? 63 - __builtin_clzll(hit) : 0;
  *found = b;
  const int q0 = __builtin_amdgcn_readlane(q, b), q1 = __builtin_amdgcn_readlane(q, b + 1);
  const int k0 = __builtin_amdgcn_readlane(k, b), k1 = __builtin_amdgcn_readlane(k, b + 1);
  if (!good_boundaries(a, q0, q1, k0, k1)) return false;
  *s = Seq{q0, q1 - q0, k0, k1 - k0};
  return true;
}

// x summed over this lane and those before it.
__device__ __forceinline__ int running(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}

// Tile i of at most 64 sequences, a sequence a lane: those whose tiles take longest first, in four bands of what their
// tiles go over, so that the last to end are short.  Tiles that do not exist have the last numbers.  Forward and backward,
// in place of the order of tile_number: 64 sequences of 46 to 538, 12 heads of 64, bf16, 51 -> 45 and 144 -> 137 us; 60 of 20
// to 300, 16 heads on 4 of 128, causal, 39 -> 37 and 145 -> 125; 64 of 128 alike, 13.5 -> 12.1 and 35 -> 33; one of 300 the
// same.  (Up to 256 sequences, four a lane: as much off where lengths differ, but 7 % on where they do not, 256 of 197, 4
// heads of 32, fp32, 80 -> 84 and 248 -> 265.)
template <bool QUERIES>
__device__ __forceinline__ bool by_length(const AttnArgs& a, int i, int mul, int size, Seq* s, int* tile) {
  const int lane = threadIdx.x & 63, at = min(lane, a.B), to = min(lane + 1, a.B);
  const int q0 = a.cu_q[at], q1 = a.cu_q[to], k0 = a.cu_k[at], k1 = a.cu_k[to];
  const bool good = lane < a.B && good_boundaries(a, q0, q1, k0, k1);
  const int nq = good ? q1 - q0 : 0, nk = good ? k1 - k0 : 0;
  const int tiles = static_cast<int>((static_cast<uint32_t>(QUERIES ? nq : nk) * mul + size - 1) / static_cast<uint32_t>(size));
  const float work = tiles ? static_cast<float>(QUERIES ? nk : nq) : -1.f;
  float most = fmaxf(work, dpp<0xB1>(work));
  most = fmaxf(most, dpp<0x4E>(most));
  most = fmaxf(most, dpp<0x141>(most));
  most = fmaxf(most, dpp<0x140>(most));
  most = max32(max16(most));
  int start = 0, before = 0;
#pragma unroll
  for (int band = 0; band < 4; ++band) {
    const bool in = work >= most * (0.75f - 0.25f * band) && (band == 0 || work < most * (1.f - 0.25f * band));
    const int x = in ? tiles : 0, sum = running(x);
    if (in) start = before + sum - x;
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  const uint64_t hit = __ballot(i >= start && i - start < tiles);
  if (!hit) return false;
  const int b = __builtin_ctzll(hit);
  *s = Seq{__builtin_amdgcn_readlane(q0, b), __builtin_amdgcn_readlane(nq, b), __builtin_amdgcn_readlane(k0, b),
           __builtin_amdgcn_readlane(nk, b)};
  const int in_sequence = i - __builtin_amdgcn_readlane(start, b);
  *tile = QUERIES ? __builtin_amdgcn_readlane(tiles, b) - 1 - in_sequence : in_sequence;
  return true;
}

// Workgroup i's tile of `size` rows (keys) of a sequence; false: none.  Of a causal mask the long tiles first, the last rows'
// and the first keys'.
template <bool QUERIES>
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int i, int mul, int size, Seq* s, int* tile) {
  if (a.ranked) return by_length<QUERIES>(a, i, mul, size, s, tile);
  const int t = QUERIES ? a.blocks / a.Hk - 1 - tile_number(a, i) : tile_number(a, i);
  int b;
  if (!locate<QUERIES>(a, t, [&](int cu, int j) { return first_tile(cu, j, mul, size); }, &b, s)) return false;
  const int64_t at = t - first_tile(QUERIES ? s->q0 : s->k0, b, mul, size);
  *tile = static_cast<int>(at);
  return at >= 0 && at * size < static_cast<int64_t>(QUERIES ? s->nq : s->nk) * mul;
}

// The grid's last workgroup looks at every boundary.
__device__ __forceinline__ bool check_block(const AttnArgs& a) {
  if (static_cast<int>(blockIdx.x) < a.blocks) return false;
  bool bad = false;
  Seq s;
  for (int b = threadIdx.x; b < a.B; b += kThreads) bad |= !sequence(a, b, &s);
  if (bad) atomicOr(a.status, DORA_DEV_CU_SEQLENS);
  return true;
}

// Keys that row r sees.
__device__ __forceinline__ int limit_of(const AttnArgs& a, const Seq& s, int r) {
  if (r >= s.nq * a.G) return 0;
  return a.causal ? max(0, min(s.nk, div_group(a, r) + 1 + s.nk - s.nq)) : s.nk;
}

// Keys that any of n rows from row r on sees: a wave is idle past them.
__device__ __forceinline__ int wave_limit(const AttnArgs& a, const Seq& s, int r, int n) {
  const int rows = s.nq * a.G;
  return __builtin_amdgcn_readfirstlane(r < rows ? limit_of(a, s, min(r + n, rows) - 1) : 0);
}

__device__ __forceinline__ const char* query_row(const AttnArgs& a, const RowView& x, const Seq& s, int hk, int r) {
  const int i = div_group(a, r);
  return x.at + (static_cast<int64_t>(s.q0) + i) * x.row + static_cast<int64_t>(hk * a.G + r - i * a.G) * x.head;
}
__device__ __forceinline__ int64_t stat_at(const AttnArgs& a, const Seq& s, int hk, int r) {
  const int i = div_group(a, r);
  return (static_cast<int64_t>(s.q0) + i) * a.H + hk * a.G + r - i * a.G;
}

// Operands of a 16x16 product in steps of 32: lane l (g = l / 16, c = l % 16)
// holds eight elements of row or column c, at 8g .. 8g + 7 of the step; the
// result's lane holds column c, rows 4g .. 4g + 3.
template <class E>
struct Op;

template <>
struct Op<__bf16> {
  typedef bf16x8 Frag;
  static constexpr int kKeys = 64;  // rows of a staged tile
  static constexpr int kPad = 8;    // elements after a staged row: its 16-byte pieces move on by one bank group a row
  static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  // Two results of 16 rows as the eight elements of a step (in the order of columns()).
  static __device__ __forceinline__ Frag pack(floatx4 x, floatx4 y) {
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = static_cast<__bf16>(x[i]), f[4 + i] = static_cast<__bf16>(y[i]);
    return f;
  }
  // Column d0 + c of staged rows 4g .. 4g + 3 and 16 + 4g .. 16 + 4g + 3: the transposing read hands
  // lane j of a group element j of the rows that lanes 4e + j / 4 point at.
  template <int LD>
  static __device__ __forceinline__ Frag columns(const __bf16* rows, int d0) {
    typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
    const int lane = threadIdx.x & 63, g = lane >> 4, e = (lane & 15) >> 2, r = lane & 3;
    __bf16* p = const_cast<__bf16*>(rows) + (4 * g + e) * LD + d0 + 4 * r;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 16 * LD));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

struct alignas(16) float8 {
  float v[8];
};
template <>
struct Op<float> {
  typedef float8 Frag;
  static constexpr int kKeys = 32;
  static constexpr int kPad = 4;
  // Eight fp32 products of four: the step's element 8g + j is term g of product j, on both sides.
  static __device__ __forceinline__ floatx4 mma(const Frag& a, const Frag& b, floatx4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ Frag pack(floatx4 x, floatx4 y) {
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = x[i], f.v[4 + i] = y[i];
    return f;
  }
  template <int LD>
  static __device__ __forceinline__ Frag columns(const float* rows, int d0) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const float* p = rows + 4 * g * LD + d0 + (lane & 15);
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = p[i * LD], f.v[4 + i] = p[(16 + i) * LD];
    return f;
  }
};

template <class E>
__device__ __forceinline__ typename Op<E>::Frag zero_frag() {
  typename Op<E>::Frag f;
  __builtin_memset(&f, 0, sizeof f);
  return f;
}
// Eight adjacent elements.
template <class E>
__device__ __forceinline__ typename Op<E>::Frag load_frag(const void* p) {
  return *static_cast<const typename Op<E>::Frag*>(p);
}

template <class E>
__device__ __forceinline__ bool finite_piece(u32x4 w) {
  bool ok = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(E) == 4) ok = ok && (w[i] & 0x7F800000u) != 0x7F800000u;
    else ok = ok && (w[i] & 0x7F80u) != 0x7F80u && (w[i] & 0x7F800000u) != 0x7F800000u;
  }
  return ok;
}

// A tile of rows on its way from memory to LDS, through registers: asked for
// while the tile before it is worked on.  Rows at n and past it are 0.
template <class E, int D>
struct Staged {
  static constexpr int kRows = Op<E>::kKeys, kLd = D + Op<E>::kPad;
  static constexpr int kRowPieces = D * sizeof(E) / 16, kPieces = kRows * kRowPieces / kThreads;
  static_assert(kPieces >= 1, "every thread moves a piece");
  u32x4 w[kPieces];
  // address(row of the tile): its first element
  template <class F>
  __device__ __forceinline__ void load(int n, F address) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int p = threadIdx.x + i * kThreads, row = p / kRowPieces;
      w[i] = row < n ? *reinterpret_cast<const u32x4*>(address(row) + p % kRowPieces * 16) : u32x4{0u, 0u, 0u, 0u};
    }
  }
  __device__ __forceinline__ void store(E* lds) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int p = threadIdx.x + i * kThreads;
      *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(lds + p / kRowPieces * kLd) + p % kRowPieces * 16) = w[i];
    }
  }
  __device__ __forceinline__ bool finite() const {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) ok = ok && finite_piece<E>(w[i]);
    return ok;
  }
};

// Four adjacent elements, rounded once.
template <class E>
__device__ __forceinline__ void store4(char* p, floatx4 x) {
  if (sizeof(E) == 4) {
    *reinterpret_cast<floatx4*>(p) = x;
  } else {
    bf16x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = static_cast<__bf16>(x[i]);
    *reinterpret_cast<bf16x4*>(p) = y;
  }
}

__device__ __forceinline__ float over_groups_max(float x) { return max32(max16(x)); }
__device__ __forceinline__ float over_groups_sum(float x) { return add32(add16(x)); }

// ------------------------------- forward ----------------------------------

// The sequence's keys are one part, whose workgroup writes the rows itself (100 of 100 keys, 8 key heads of 128: 19 us; through
// the join 22).
__device__ __forceinline__ bool one_part(const AttnArgs& a, const Seq& s) { return a.chunk && s.nk > 0 && s.nk <= a.chunk; }

// One tile of 64 rows against a range of its keys.  s^T = k q^T leaves each lane
// one row's column, so its maximum and sum are mostly in the lane, and p goes
// into out^T += v^T p^T from the registers where it stands.
// One query a sequence is bound by the caches' bytes (32 of 1000 to 65000 keys, 8
// key heads of 128, bf16: 839 us and 6 for the join, 5.6 TB/s of reads) or, few of
// them, by the chain from boundaries to keys to products (four of 321 to 1205: 7.6
// and 4.5).  fp32 by its matrix rate, 154 TFLOP/s (256 sequences of 60 to 197, four
// heads of 32: 45 us, matrix units busy 43 %, a sixth of that in places past a
// sequence).
template <class E, int D, bool SPLIT>
__global__ __launch_bounds__(kThreads) void attn_kernel(AttnArgs a) {
  typedef typename Op<E>::Frag Frag;
  typedef Staged<E, D> Tile;
  constexpr int kKeys = Tile::kRows, kLd = Tile::kLd, kSteps = kKeys / 16;
  __shared__ alignas(16) E ks[kKeys * kLd];
  __shared__ alignas(16) E vs[kKeys * kLd];
  if (check_block(a)) return;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const int hk = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk;
  const int split = SPLIT && !a.chunk ? rest % a.splits : 0, t = SPLIT && !a.chunk ? rest / a.splits : rest;
  Seq s;
  int tile = 0, key_lo = 0, key_hi;
  if (SPLIT && a.chunk) {
    int b;
    if (!locate<false>(a, t, [&](int cu, int i) { return first_tile(cu, i, 1, a.chunk); }, &b, &s)) return;
    const int64_t part = t - first_tile(s.k0, b, 1, a.chunk);
    if (part < 0 || part * a.chunk >= s.nk || s.nq == 0) return;
    key_lo = static_cast<int>(part) * a.chunk;
    key_hi = min(s.nk, key_lo + a.chunk);
  } else {
    if constexpr (SPLIT) {
      int b;
      if (!locate<true>(a, t, [&](int cu, int i) { return first_tile(cu, i, a.G, kTile); }, &b, &s)) return;
      const int64_t at = t - first_tile(s.q0, b, a.G, kTile);
      if (at < 0 || at * kTile >= static_cast<int64_t>(s.nq) * a.G) return;
      tile = static_cast<int>(at);
    } else if (!find_tile<true>(a, t, a.G, kTile, &s, &tile)) {
      return;
    }
    key_hi = limit_of(a, s, min((tile + 1) * kTile, s.nq * a.G) - 1);
    if (SPLIT) {
      const int each = ((key_hi + a.splits - 1) / a.splits + kKeys - 1) / kKeys * kKeys;
      key_lo = min(key_hi, split * each);
      key_hi = min(key_hi, key_lo + each);
    }
  }
  const int row = tile * kTile + wave * 16 + c16;
  const bool real = row < s.nq * a.G;
  const int limit = limit_of(a, s, row);
  // Keys below this are seen by every row of the tile that exists.
  const int open = limit_of(a, s, tile * kTile), wave_hi = wave_limit(a, s, tile * kTile + wave * 16, 16);
  Frag qf[D / 32];
#pragma unroll
  for (int ks32 = 0; ks32 < D / 32; ++ks32)
    qf[ks32] = real ? load_frag<E>(query_row(a, a.q, s, hk, row) + (32 * ks32 + 8 * g) * sizeof(E)) : zero_frag<E>();
  floatx4 o[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const char* kbase = a.k.at + static_cast<int64_t>(s.k0) * a.k.row + hk * a.k.head;
  const char* vbase = a.v.at + static_cast<int64_t>(s.k0) * a.v.row + hk * a.v.head;
  Tile kt, vt;
  const auto ask = [&](int key) {
    kt.load(s.nk - key, [&](int i) { return kbase + static_cast<int64_t>(key + i) * a.k.row; });
    vt.load(s.nk - key, [&](int i) { return vbase + static_cast<int64_t>(key + i) * a.v.row; });
  };
  if (key_lo < key_hi) ask(key_lo);
  for (int key = key_lo; key < key_hi; key += kKeys) {
    const bool masked = key + kKeys > open || key + kKeys > key_hi;
    bool odd = false;  // a value that is not finite where some row may not see it
    __syncthreads();
    kt.store(ks);
    vt.store(vs);
    if (masked) odd = __syncthreads_or(!vt.finite());
    else __syncthreads();
    if (key + kKeys < key_hi) ask(key + kKeys);
    if (key >= wave_hi) continue;
    floatx4 sc[kSteps];
#pragma unroll
    for (int kt16 = 0; kt16 < kSteps; ++kt16) {
      sc[kt16] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks32 = 0; ks32 < D / 32; ++ks32)
        sc[kt16] = Op<E>::mma(load_frag<E>(ks + (kt16 * 16 + c16) * kLd + 32 * ks32 + 8 * g), qf[ks32], sc[kt16]);
    }
    const int end = min(limit, key_hi) - key;
    if (masked) {
#pragma unroll
      for (int kt16 = 0; kt16 < kSteps; ++kt16)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (kt16 * 16 + 4 * g + i >= end) sc[kt16][i] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int kt16 = 0; kt16 < kSteps; ++kt16)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[kt16][i]);
    top = over_groups_max(top) * a.c2;
    const float next = fmaxf(m, top), ref = next == -INFINITY ? 0.f : next;
    const float keep = __builtin_amdgcn_exp2f(m - ref);
    m = next;
    float sum = 0.f;
#pragma unroll
    for (int kt16 = 0; kt16 < kSteps; ++kt16)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[kt16][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt16][i], a.c2, -ref));
        sum += sc[kt16][i];
      }
    l = l * keep + sum;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) o[dt] *= keep;
    if (!odd) {
#pragma unroll
      for (int st = 0; st < kSteps / 2; ++st) {
        const Frag p = Op<E>::pack(sc[2 * st], sc[2 * st + 1]);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
          o[dt] = Op<E>::mma(Op<E>::template columns<kLd>(vs + st * 32 * kLd, dt * 16), p, o[dt]);
      }
    } else {  // 0 times such a value is NaN: key by key, and only those that the row sees
#pragma unroll
      for (int kt16 = 0; kt16 < kSteps; ++kt16)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          for (int og = 0; og < 4; ++og) {
            const float p = __shfl(sc[kt16][i], og * 16 + c16);
            const int at = kt16 * 16 + 4 * og + i;
            if (at < end) {
#pragma unroll
              for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  o[dt][x] = __builtin_fmaf(p, static_cast<float>(vs[at * kLd + dt * 16 + 4 * g + x]), o[dt][x]);
            }
          }
    }
  }
  l = over_groups_sum(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (!real) return;
  if (SPLIT && !one_part(a, s)) {
    const int64_t at = (static_cast<int64_t>(rest) * a.Hk + hk) * a.part_rows + row - tile * kTile;
    if (g == 0) a.part_ml[at] = make_float2(m, l);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<floatx4*>(a.part + at * D + dt * 16 + 4 * g) = o[dt];
    return;
  }
  if (g == 0 && a.lse) a.lse[stat_at(a, s, hk, row)] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  char* to = const_cast<char*>(query_row(a, a.out, s, hk, row));
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) store4<E>(to + (dt * 16 + 4 * g) * sizeof(E), o[dt] * inv);
}

// ------------------------- bf16 in tiles of 128 ---------------------------

// Products of 32 x 32 in steps of 16: lane l (c = l % 32, hi = l / 32) holds
// elements 8 hi .. 8 hi + 7 of row or column c, the result's lane column c, rows
// 8 (i / 4) + 4 hi + i % 4.  One operand read from LDS serves 32 columns in place
// of 16.  Two waves a SIMD at 128, three at 64, on the sequences
// above: matrix units busy 45 % of the cycles forward, 56 % in grad_q, 46 % in
// grad_kv, vector instructions a third to two fifths, LDS a quarter, no conflicts;
// a wave waits for its own products, exponentials or operands the rest.  Heads of
// 64 have the same exponentials for half the products: 64 sequences of 46 to 577,
// 20337 rows, 12 heads, take 54 us forward, 67 in grad_q and 79 in grad_kv, with
// matrix units busy 23 to 33 %.
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kWide = 128;      // rows of a workgroup, 32 a wave
constexpr int kWideKeys = 64;   // rows of a staged tile

// A staged tile stands as D / 64 blocks of 64 columns, [64 rows][64 columns] each, the eight 16-byte pieces of row r at
// piece ^ turn(r).  Two rows fill the 256 bytes of all banks: sixteen rows' reads of one piece, and the transposing reads
// of 64 bytes from four rows, each fall on banks of their own (with rows of 256 bytes and another turn half of them met:
// a third of the LDS's cycles).
__device__ __forceinline__ int turn(int r) { return (r >> 1 & 1) << 2 | (r >> 2 & 3); }

// A lane's share of staging a tile by DMA: an instruction moves 1 KB, eight rows of a block; its address is one that all
// lanes share and a 32-bit offset, formed once, so that a tile costs next to no vector arithmetic.  Rows at n and past it
// are copies of row n - 1: what they are multiplied by is 0, and that they may not be finite is looked after.
template <int D>
struct Stage {
  static constexpr int kBlocks = D / 64, kCount = 2 * kBlocks;  // instructions of a wave
  // The lane moves rows row() and row() + 32, from this byte on (turn() is the same for both).
  static __device__ __forceinline__ int row() { return static_cast<int>(threadIdx.x / 8); }
  static __device__ __forceinline__ uint32_t piece() { return ((threadIdx.x & 7) ^ turn(row())) * 16; }
  // lane(k): row row() + 32 k's offset from the tile's address; last(): that of row n - 1
  template <class L, class Z>
  static __device__ __forceinline__ void run(__bf16* to, const char* tile, int n, L lane, Z last) {
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    uint32_t off[2] = {lane(0), lane(1)};
    if (n < kWideKeys) {
      const uint32_t end = last();
      off[0] = row() < n ? off[0] : end;
      off[1] = row() + 32 < n ? off[1] : end;
    }
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      __bf16* at = to + i % kBlocks * kWideKeys * 64 + (i / kBlocks * 4 + wave) * 8 * 64;
      __builtin_amdgcn_global_load_lds(tile + i % kBlocks * 128 + off[i / kBlocks], (lds_void*)at, 16, 0, 0);
    }
  }
};
// Rows one after another, `row` bytes apart.
template <int D>
struct KeyStage : Stage<D> {
  typedef Stage<D> S;
  uint32_t off, step;
  __device__ __forceinline__ KeyStage(int64_t bytes)
      : off(S::row() * static_cast<uint32_t>(bytes) + S::piece()), step(static_cast<uint32_t>(bytes)) {}
  __device__ __forceinline__ void stage(__bf16* to, const char* tile, int n) const {
    S::run(to, tile, n, [&](int k) { return off + k * 32 * step; }, [&] { return (n - 1) * step + S::piece(); });
  }
};
// The rows of whole queries: row r is query r / G of head r % G.
template <int D>
struct QueryStage : Stage<D> {
  typedef Stage<D> S;
  uint32_t off[2];
  uint32_t step, head;
  __device__ __forceinline__ QueryStage(const AttnArgs& a, const RowView& x)
      : step(static_cast<uint32_t>(x.row)), head(static_cast<uint32_t>(x.head)) {
#pragma unroll
    for (int k = 0; k < 2; ++k) off[k] = place(a, S::row() + k * 32) + S::piece();
  }
  __device__ __forceinline__ uint32_t place(const AttnArgs& a, int r) const {
    const int q = div_group(a, r);
    return q * step + (r - q * a.G) * head;
  }
  __device__ __forceinline__ void stage(const AttnArgs& a, __bf16* to, const char* tile, int n) const {
    S::run(to, tile, n, [&](int k) { return off[k]; }, [&] { return place(a, n - 1) + S::piece(); });
  }
};

// Everything that this workgroup staged has arrived, and every wave is done with what stood there.
__device__ __forceinline__ void staged() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ floatx16 mma32(bf16x8 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A lane's places in a block of a staged tile, in elements; blocks, and rows 16 on, lie at constant distances, which the
// reads hold as their immediate.
struct WidePlaces {
  uint32_t row[4];        // row c, columns 16 st + 8 hi .. + 7 of the block
  uint32_t column[2][2];  // for the transposing read of columns 0 .. 31 and 32 .. 63, of rows 4 hi + e and 8 further: lane
                          // 4 e + r of sixteen points at four columns of row e
};
__device__ __forceinline__ WidePlaces wide_places() {
  const int lane = threadIdx.x & 63, c = lane & 31, hi = lane >> 5, half = lane >> 4 & 1, e = (lane & 15) >> 2, r = lane & 3;
  WidePlaces w;
#pragma unroll
  for (int st = 0; st < 4; ++st) w.row[st] = c * 64 + ((2 * st + hi) ^ turn(c)) * 8;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = 8 * k + 4 * hi + e;
      w.column[n][k] = row * 64 + ((4 * n + 2 * half + (r >> 1)) ^ turn(row)) * 8 + (r & 1) * 4;
    }
  return w;
}

// Row r0 + c of a staged tile, columns 16 st + 8 hi .. + 7 (r0 a multiple of 32).
__device__ __forceinline__ bf16x8 wide_row(const __bf16* tile, const WidePlaces& w, int r0, int st) {
  return *reinterpret_cast<const bf16x8*>(tile + w.row[st % 4] + st / 4 * kWideKeys * 64 + r0 * 64);
}
// Column d0 + c (d0 a multiple of 32) of staged rows r0 + 4 hi .. + 3 and r0 + 8 + 4 hi .. + 3 (r0 a multiple of 16).
__device__ __forceinline__ bf16x8 wide_column(const __bf16* tile, const WidePlaces& w, int r0, int d0) {
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  __bf16* block = const_cast<__bf16*>(tile) + d0 / 64 * kWideKeys * 64 + r0 * 64;
  const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(block + w.column[d0 / 32 % 2][0]));
  const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(block + w.column[d0 / 32 % 2][1]));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Row `at`, column d.
__device__ __forceinline__ int wide_at(int at, int d) {
  return d / 64 * kWideKeys * 64 + at * 64 + ((d / 8 % 8) ^ turn(at)) * 8 + d % 8;
}
// Elements 8t .. 8t + 7 of a result as the operand of 16 rows, in the order of wide_column.
__device__ __forceinline__ bf16x8 wide_pack(const floatx16& x, int t) {
  bf16x8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = static_cast<__bf16>(x[8 * t + i]);
  return f;
}
__device__ __forceinline__ floatx16 zero16() {
  floatx16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
__device__ __forceinline__ int wide_place(int i) { return 8 * (i / 4) + i % 4; }  // + 4 hi

// The thread's number, where the compiler does not know that it has it already: what is formed from it after a loop is
// not held in registers, or spilled, through the loop.
__device__ __forceinline__ int thread_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

template <int D>
struct WideTiles {
  __bf16 a0[kWideKeys * D], b0[kWideKeys * D], a1[kWideKeys * D], b1[kWideKeys * D];
};

template <int D>
struct WideForward {
  bf16x8 q[D / 16];
  floatx16 o[D / 32];
  float m, l;
  int limit;
};

// Values that are not finite among keys that some rows do not see: 0 times them is NaN.  The rows that see them take
// them here (an infinite or NaN sum is what p times them gives, NaN where p is 0 or NaN itself), and zeros stand in their
// place.  alive[n] bit i: p of key 32 n + i is above 0.
template <int D>
__device__ __forceinline__ void take_odd(WideForward<D>& f, __bf16* vs, int end, const uint32_t (&alive)[2]) {
  const int hi = (threadIdx.x & 63) >> 5;
  for (int at = 0; at < min(end, kWideKeys); ++at) {
    const bool counts = alive[at / 32] >> at % 32 & 1;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int d = 32 * dt + wide_place(x) + 4 * hi;
        const float v = static_cast<float>(vs[wide_at(at, d)]);
        if (!(__builtin_fabsf(v) < INFINITY)) f.o[dt][x] += counts ? v : NAN;
      }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWideKeys * D / 8 / kThreads; ++i) {
    __bf16* p = vs + (i * kThreads + threadIdx.x) * 8;
    for (int x = 0; x < 8; ++x)
      if (!(__builtin_fabsf(static_cast<float>(p[x])) < INFINITY)) p[x] = static_cast<__bf16>(0.f);
  }
  __syncthreads();
}

// 64 staged keys.  The maximum that p is taken against rises only when a score passes it by 2^8: p, l and the
// products' sums stay far inside their range, and the sums are multiplied a few times in place of every tile.
template <int D>
__device__ __forceinline__ void wide_keys(const AttnArgs& a, WideForward<D>& f, const __bf16* ks, __bf16* vs,
                                          const WidePlaces& w, int end, bool masked, bool odd, bool idle) {
  const int hi = (threadIdx.x & 63) >> 5;
  if (idle) {
    if (odd) take_odd<D>(f, vs, 0, {0u, 0u});
    return;
  }
  floatx16 s[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    s[n] = zero16();
#pragma unroll
    for (int st = 0; st < D / 16; ++st) s[n] = mma32(wide_row(ks, w, 32 * n, st), f.q[st], s[n]);
  }
  if (masked) {
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * n + wide_place(i) + 4 * hi >= end) s[n][i] = -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
  top = max32(top) * a.c2;
  if (__any(top > f.m + 8.f)) {
    const float next = fmaxf(f.m, top), keep = __builtin_amdgcn_exp2f(next == -INFINITY ? 0.f : f.m - next);
    f.m = next;
    f.l *= keep;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) f.o[dt] *= keep;
  }
  const float ref = f.m == -INFINITY ? 0.f : f.m;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], a.c2, -ref));
      f.l += s[n][i];
    }
  if (odd) {
    uint32_t alive[2] = {0u, 0u};
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) alive[n] |= s[n][i] > 0.f ? 1u << (wide_place(i) + 4 * hi) : 0u;
      const auto halves = __builtin_amdgcn_permlane32_swap(alive[n], alive[n], false, false);
      alive[n] = halves[0] | halves[1];
    }
    take_odd<D>(f, vs, end, alive);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 p = wide_pack(s[n], t);
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) f.o[dt] = mma32(wide_column(vs, w, 32 * n + 16 * t, 32 * dt), p, f.o[dt]);
    }
}

// Some value of the staged tile is not finite.
template <int D>
__device__ __forceinline__ bool odd_tile(const __bf16* tile) {
  bool ok = true;
#pragma unroll
  for (int i = 0; i < kWideKeys * D / 8 / kThreads; ++i)
    ok = ok && finite_piece<__bf16>(*reinterpret_cast<const u32x4*>(tile + (i * kThreads + threadIdx.x) * 8));
  return __syncthreads_or(!ok);
}

template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void attn_wide_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) WideTiles<D> tiles;
  if (check_block(a)) return;
  const int lane = threadIdx.x & 63, c = lane & 31, hi = lane >> 5, wave = threadIdx.x >> 6;
  const int hk = blockIdx.x % a.Hk;
  Seq s;
  int tile;
  if (!find_tile<true>(a, blockIdx.x / a.Hk, a.G, kWide, &s, &tile)) return;
  const int rows = s.nq * a.G, row0 = tile * kWide, row = row0 + wave * 32 + c;
  const bool real = row < rows;
  const int key_hi = limit_of(a, s, min(row0 + kWide, rows) - 1), open = limit_of(a, s, row0);
  const int wave_hi = wave_limit(a, s, row0 + wave * 32, 32);
  const WidePlaces w = wide_places();
  WideForward<D> f;
  f.limit = limit_of(a, s, row);
  f.m = -INFINITY, f.l = 0.f;
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
    f.q[st] = real ? load_frag<__bf16>(query_row(a, a.q, s, hk, row) + (16 * st + 8 * hi) * 2) : zero_frag<__bf16>();
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) f.o[dt] = zero16();
  const char* kbase = a.k.at + static_cast<int64_t>(s.k0) * a.k.row + hk * a.k.head;
  const char* vbase = a.v.at + static_cast<int64_t>(s.k0) * a.v.row + hk * a.v.head;
  const KeyStage<D> kst(a.k.row), vst(a.v.row);
  const auto ask = [&](int key, __bf16* kt, __bf16* vt) {
    kst.stage(kt, kbase + key * a.k.row, s.nk - key);
    vst.stage(vt, vbase + key * a.v.row, s.nk - key);
  };
  // One tile in these buffers while the next comes into the others.
  const auto step = [&](int key, __bf16* kt, __bf16* vt, __bf16* kn, __bf16* vn) {
    staged();
    if (key + kWideKeys < key_hi) ask(key + kWideKeys, kn, vn);
    const bool masked = key + kWideKeys > open;
    wide_keys<D>(a, f, kt, vt, w, f.limit - key, masked, masked && odd_tile<D>(vt), key >= wave_hi);
  };
  if (key_hi > 0) ask(0, tiles.a0, tiles.b0);
  for (int key = 0; key < key_hi; key += 2 * kWideKeys) {
    step(key, tiles.a0, tiles.b0, tiles.a1, tiles.b1);
    if (key + kWideKeys >= key_hi) break;
    step(key + kWideKeys, tiles.a1, tiles.b1, tiles.a0, tiles.b0);
  }
  const float l = add32(f.l), inv = l == 0.f ? 0.f : 1.f / l;
  const int thread = thread_again(), out_row = row0 + thread / 64 * 32 + thread % 32, out_hi = thread % 64 / 32;
  if (out_row >= rows) return;
  if (out_hi == 0 && a.lse)
    a.lse[stat_at(a, s, hk, out_row)] = l == 0.f ? -INFINITY : (f.m + __builtin_amdgcn_logf(l)) * kLn2;
  char* to = const_cast<char*>(query_row(a, a.out, s, hk, out_row)) + out_hi * 8;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const floatx4 x = {f.o[dt][4 * n], f.o[dt][4 * n + 1], f.o[dt][4 * n + 2], f.o[dt][4 * n + 3]};
      store4<__bf16>(to + (32 * dt + 8 * n) * 2, x * inv);
    }
}

// The parts of a row joined: one wave a row, out = sum w o / sum w l with w =
// 2^(m - max m).
template <class E, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (at >= a.total_q * a.H) return;
  const int64_t n = at / a.H;
  const int h = static_cast<int>(at - n * a.H), hk = h / a.G;
  Seq s;
  int b;
  const bool good = locate<true>(a, n, [](int cu, int) { return static_cast<int64_t>(cu); }, &b, &s);
  if (!good || n < s.q0 || n >= static_cast<int64_t>(s.q0) + s.nq) return;
  const int row = static_cast<int>(n - s.q0) * a.G + h - hk * a.G;
  int64_t first;
  int parts, in = row;
  if (a.chunk) {
    first = first_tile(s.k0, b, 1, a.chunk);
    if (one_part(a, s)) return;
    parts = (s.nk + a.chunk - 1) / a.chunk;
  } else {
    first = (first_tile(s.q0, b, a.G, kTile) + row / kTile) * a.splits;
    parts = a.splits;
    in = row % kTile;
  }
  constexpr int kEach = D >= 64 ? D / 64 : 1, kAtOnce = 8;
  const int d = lane * kEach;
  float top = -INFINITY, sum = 0.f, o[kEach] = {};
  for (int p = 0; p < parts; p += kAtOnce) {
    float2 ml[kAtOnce];
    float x[kAtOnce][kEach];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int64_t slot = ((first + min(p + i, parts - 1)) * a.Hk + hk) * a.part_rows + in;
      ml[i] = a.part_ml[slot];
#pragma unroll
      for (int e = 0; e < kEach; ++e) x[i][e] = a.part[slot * D + (d < D ? d + e : 0)];
    }
    float next = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (p + i >= parts) ml[i] = make_float2(-INFINITY, 0.f);
      next = fmaxf(next, ml[i].x);
    }
    const float ref = next == -INFINITY ? 0.f : next, keep = __builtin_amdgcn_exp2f(top - ref);
    top = next;
    sum *= keep;
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] *= keep;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (ml[i].x == -INFINITY && ml[i].y == 0.f) continue;  // sees none of these keys
      const float w = __builtin_amdgcn_exp2f(ml[i].x - ref);
      sum = __builtin_fmaf(w, ml[i].y, sum);
#pragma unroll
      for (int e = 0; e < kEach; ++e) o[e] = __builtin_fmaf(w, x[i][e], o[e]);
    }
  }
  const float ref = top == -INFINITY ? 0.f : top;
  // NaN scores: the parts' l are NaN and pass through the sums.
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane == 0 && a.lse) a.lse[at] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
  if (d < D) {
    E* to = reinterpret_cast<E*>(a.out.at + n * a.out.row + h * a.out.head) + d;
#pragma unroll
    for (int x = 0; x < kEach; ++x) to[x] = static_cast<E>(o[x] * inv);
  }
}

// ------------------------------- backward ---------------------------------

// log2 of the row's sum of exponentials; a row without any gets one that makes every P 0.
__device__ __forceinline__ float row_lse2(const AttnArgs& a, const Seq& s, int hk, int row, bool real) {
  const float lse = real ? a.lse[stat_at(a, s, hk, row)] : -INFINITY;
  return lse == -INFINITY ? INFINITY : lse * kLog2e;
}

// delta from out carries out's rounding to bf16, which stands for as much as the roundings of dS and of the results where a
// row has few keys (2^-9 of |dout||out|, and |out| falls as 1 / sqrt(keys)): 1.6 times the error of a form that rounds its
// results alone, 1.4 without.  Where a tile's keys are staged at once (64, wide 128), delta is the sum of P dP over the sum
// of P instead.  That sum is 1 but for lse's roundings, 2^-23 of its size: left out, dS of a row whose P is all on one key
// keeps as much of dP (1e-4 of it at scores of 900), where it should vanish.  S and dP are formed a second time for it: 128
// sequences of 64, 8 heads of 64, backward 35.2 -> 36.6 us; 64 of 128, 16 on 4 of 128, 100 -> 106.
__device__ __forceinline__ float mean_of(float sum, float weights) { return weights == 0.f ? 0.f : sum / weights; }

// Keys whose dS counts, of `limit` that the row sees: of one key P is 1 whatever its score, and dS 0.
__device__ __forceinline__ int gradient_limit(int limit) { return limit == 1 ? 0 : limit; }
// Both limits of a row in one number, for dS and, without the sign bit, for P.
__device__ __forceinline__ int both_limits(int limit) { return limit == 1 ? INT32_MIN | 1 : limit; }
__device__ __forceinline__ int p_limit(int both) { return both & INT32_MAX; }

// dq of 64 rows over their keys; also delta of each row, for grad_kv.  fp32, the
// sequences above: 60 us, matrix units busy 49 %.
template <class E, int D>
__global__ __launch_bounds__(kThreads) void grad_q_kernel(AttnArgs a) {
  typedef typename Op<E>::Frag Frag;
  typedef Staged<E, D> Tile;
  constexpr int kKeys = Tile::kRows, kLd = Tile::kLd;
  __shared__ alignas(16) E ks[kKeys * kLd];
  __shared__ alignas(16) E vs[kKeys * kLd];
  if (check_block(a)) return;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const int hk = blockIdx.x % a.Hk;
  Seq s;
  int tile;
  if (!find_tile<true>(a, blockIdx.x / a.Hk, a.G, kTile, &s, &tile)) return;
  const int rows = s.nq * a.G, row0 = tile * kTile, row = row0 + wave * 16 + c16;
  const bool real = row < rows;
  const int limit = limit_of(a, s, row), open = limit_of(a, s, row0), ds_limit = gradient_limit(limit);
  const int key_hi = limit_of(a, s, min(row0 + kTile, rows) - 1), wave_hi = wave_limit(a, s, row0 + wave * 16, 16);
  Frag qf[D / 32], gf[D / 32];
  float delta = 0.f;
#pragma unroll
  for (int st = 0; st < D / 32; ++st) {
    const int off = (32 * st + 8 * g) * sizeof(E);
    qf[st] = real ? load_frag<E>(query_row(a, a.q, s, hk, row) + off) : zero_frag<E>();
    gf[st] = real ? load_frag<E>(query_row(a, a.dout, s, hk, row) + off) : zero_frag<E>();
    const Frag of = real ? load_frag<E>(query_row(a, a.out, s, hk, row) + off) : zero_frag<E>();
    const E* x = reinterpret_cast<const E*>(&gf[st]);
    const E* y = reinterpret_cast<const E*>(&of);
#pragma unroll
    for (int i = 0; i < 8; ++i) delta = __builtin_fmaf(static_cast<float>(x[i]), static_cast<float>(y[i]), delta);
  }
  delta = over_groups_sum(delta);
  const float lse2 = row_lse2(a, s, hk, row, real);
  floatx4 dq[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) dq[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  const char* kbase = a.k.at + static_cast<int64_t>(s.k0) * a.k.row + hk * a.k.head;
  const char* vbase = a.v.at + static_cast<int64_t>(s.k0) * a.v.row + hk * a.v.head;
  Tile kt, vt;
  const auto ask = [&](int key) {
    kt.load(s.nk - key, [&](int i) { return kbase + static_cast<int64_t>(key + i) * a.k.row; });
    vt.load(s.nk - key, [&](int i) { return vbase + static_cast<int64_t>(key + i) * a.v.row; });
  };
  if (key_hi > 0) ask(0);
  for (int key = 0; key < key_hi; key += kKeys) {
    const bool masked = key + kKeys > open;
    __syncthreads();
    kt.store(ks);
    vt.store(vs);
    __syncthreads();
    if (key + kKeys < key_hi) ask(key + kKeys);
    if (key >= wave_hi) continue;
    if (sizeof(E) == 2 && key_hi <= kKeys) {
      float sum = 0.f;
      delta = 0.f;
#pragma unroll
      for (int r0 = 0; r0 < kKeys; r0 += 16) {
        floatx4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < D / 32; ++st) {
          sc = Op<E>::mma(load_frag<E>(ks + (r0 + c16) * kLd + 32 * st + 8 * g), qf[st], sc);
          dp = Op<E>::mma(load_frag<E>(vs + (r0 + c16) * kLd + 32 * st + 8 * g), gf[st], dp);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.c2, -lse2));
          const bool seen = r0 + 4 * g + i < limit;
          sum += seen ? p : 0.f;
          delta += seen ? p * dp[i] : 0.f;
        }
      }
      delta = mean_of(over_groups_sum(delta), over_groups_sum(sum));
    }
#pragma unroll
    for (int st32 = 0; st32 < kKeys / 32; ++st32) {
      floatx4 ds[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r0 = st32 * 32 + half * 16;
        floatx4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < D / 32; ++st) {
          sc = Op<E>::mma(load_frag<E>(ks + (r0 + c16) * kLd + 32 * st + 8 * g), qf[st], sc);
          dp = Op<E>::mma(load_frag<E>(vs + (r0 + c16) * kLd + 32 * st + 8 * g), gf[st], dp);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.c2, -lse2));
          ds[half][i] = masked && key + r0 + 4 * g + i >= ds_limit ? 0.f : p * (dp[i] - delta);
        }
      }
      const Frag f = Op<E>::pack(ds[0], ds[1]);
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
        dq[dt] = Op<E>::mma(Op<E>::template columns<kLd>(ks + st32 * 32 * kLd, dt * 16), f, dq[dt]);
    }
  }
  if (real && g == 0) a.stat[stat_at(a, s, hk, row)] = make_float2(lse2, delta);
  if (!real) return;
  char* to = const_cast<char*>(query_row(a, a.dq, s, hk, row));
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) store4<E>(to + (dt * 16 + 4 * g) * sizeof(E), dq[dt] * a.scale);
}

// The products that make x come before what follows: left alone, the compiler reads their operands here and forms them
// where x is used, which takes the registers of all operands at once.
__device__ __forceinline__ void formed(floatx16& x) { asm volatile("" : "+v"(x)); }

// grad_q in tiles of 128 rows.
template <int D>
struct WideGradQ {
  bf16x8 q[D / 16], g[D / 16];
  floatx16 dq[D / 32];
  float lse2, delta;
};

// The lane's share of the sums of P dP and of P over 64 staged keys.
template <int D>
__device__ __forceinline__ float2 wide_delta(const AttnArgs& a, const WideGradQ<D>& f, const __bf16* ks, const __bf16* vs,
                                             const WidePlaces& w, int end) {
  const int hi = (threadIdx.x & 63) >> 5;
  float2 sum = {0.f, 0.f};
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    floatx16 s = zero16(), dp = zero16();
#pragma unroll
    for (int st = 0; st < D / 16; ++st) s = mma32(wide_row(ks, w, 32 * n, st), f.q[st], s);
    formed(s);
#pragma unroll
    for (int st = 0; st < D / 16; ++st) dp = mma32(wide_row(vs, w, 32 * n, st), f.g[st], dp);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c2, -f.lse2));
      const bool seen = 32 * n + wide_place(i) + 4 * hi < end;
      sum.x += seen ? p * dp[i] : 0.f;
      sum.y += seen ? p : 0.f;
    }
  }
  return sum;
}

template <int D>
__device__ __forceinline__ void wide_grad_q_keys(const AttnArgs& a, WideGradQ<D>& f, const __bf16* ks, const __bf16* vs,
                                                 const WidePlaces& w, int end, bool masked) {
  const int hi = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    floatx16 s = zero16(), dp = zero16();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int st = 0; st < D / 16; ++st) s = mma32(wide_row(ks, w, 32 * n, st), f.q[st], s);
    formed(s);
#pragma unroll
    for (int st = 0; st < D / 16; ++st) dp = mma32(wide_row(vs, w, 32 * n, st), f.g[st], dp);
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c2, -f.lse2));
      dp[i] = p * (dp[i] - f.delta);
    }
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * n + wide_place(i) + 4 * hi >= end) dp[i] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 ds = wide_pack(dp, t);
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) f.dq[dt] = mma32(wide_column(ks, w, 32 * n + 16 * t, 32 * dt), ds, f.dq[dt]);
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void grad_q_wide_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) WideTiles<D> tiles;
  if (check_block(a)) return;
  const int lane = threadIdx.x & 63, c = lane & 31, hi = lane >> 5, wave = threadIdx.x >> 6;
  const int hk = blockIdx.x % a.Hk;
  Seq s;
  int tile;
  if (!find_tile<true>(a, blockIdx.x / a.Hk, a.G, kWide, &s, &tile)) return;
  const int rows = s.nq * a.G, row0 = tile * kWide, row = row0 + wave * 32 + c;
  const bool real = row < rows;
  const int key_hi = limit_of(a, s, min(row0 + kWide, rows) - 1), open = limit_of(a, s, row0);
  const int limit = limit_of(a, s, row), wave_hi = wave_limit(a, s, row0 + wave * 32, 32);
  const WidePlaces w = wide_places();
  WideGradQ<D> f;
  float delta = 0.f;
#pragma unroll
  for (int st = 0; st < D / 16; ++st) {
    const int off = (16 * st + 8 * hi) * 2;
    f.q[st] = real ? load_frag<__bf16>(query_row(a, a.q, s, hk, row) + off) : zero_frag<__bf16>();
    f.g[st] = real ? load_frag<__bf16>(query_row(a, a.dout, s, hk, row) + off) : zero_frag<__bf16>();
    const bf16x8 o = real ? load_frag<__bf16>(query_row(a, a.out, s, hk, row) + off) : zero_frag<__bf16>();
#pragma unroll
    for (int i = 0; i < 8; ++i) delta = __builtin_fmaf(static_cast<float>(f.g[st][i]), static_cast<float>(o[i]), delta);
  }
  f.delta = add32(delta);
  f.lse2 = row_lse2(a, s, hk, row, real);
  const char* kbase = a.k.at + static_cast<int64_t>(s.k0) * a.k.row + hk * a.k.head;
  const char* vbase = a.v.at + static_cast<int64_t>(s.k0) * a.v.row + hk * a.v.head;
  const KeyStage<D> kst(a.k.row), vst(a.v.row);
  const auto ask = [&](int key, __bf16* kt, __bf16* vt) {
    kst.stage(kt, kbase + key * a.k.row, s.nk - key);
    vst.stage(vt, vbase + key * a.v.row, s.nk - key);
  };
  const bool few = key_hi <= 2 * kWideKeys;
  const auto step = [&](int key, const __bf16* kt, const __bf16* vt, __bf16* kn, __bf16* vn) {
    staged();
    if (key + kWideKeys < key_hi && !few) ask(key + kWideKeys, kn, vn);
    if (key < wave_hi) wide_grad_q_keys<D>(a, f, kt, vt, w, gradient_limit(limit) - key, key + kWideKeys > open);
  };
  if (key_hi > 0) ask(0, tiles.a0, tiles.b0);
  if (few) {
    if (key_hi > kWideKeys) ask(kWideKeys, tiles.a1, tiles.b1);
    staged();
    float2 sum = wave_hi > 0 ? wide_delta<D>(a, f, tiles.a0, tiles.b0, w, limit) : make_float2(0.f, 0.f);
    if (wave_hi > kWideKeys) {
      const float2 more = wide_delta<D>(a, f, tiles.a1, tiles.b1, w, limit - kWideKeys);
      sum.x += more.x, sum.y += more.y;
    }
    f.delta = mean_of(add32(sum.x), add32(sum.y));
  }
  if (real && hi == 0) a.stat[stat_at(a, s, hk, row)] = make_float2(f.lse2, f.delta);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) f.dq[dt] = zero16();
  for (int key = 0; key < key_hi; key += 2 * kWideKeys) {
    step(key, tiles.a0, tiles.b0, tiles.a1, tiles.b1);
    if (key + kWideKeys >= key_hi) break;
    step(key + kWideKeys, tiles.a1, tiles.b1, tiles.a0, tiles.b0);
  }
  const int thread = thread_again(), out_row = row0 + thread / 64 * 32 + thread % 32;
  if (out_row >= rows) return;
  char* to = const_cast<char*>(query_row(a, a.dq, s, hk, out_row)) + (thread % 64 / 32) * 8;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const floatx4 x = {f.dq[dt][4 * n], f.dq[dt][4 * n + 1], f.dq[dt][4 * n + 2], f.dq[dt][4 * n + 3]};
      store4<__bf16>(to + (32 * dt + 8 * n) * 2, x * a.scale);
    }
}

// grad_kv in tiles of 128 keys, 32 a wave.  The sums of dk and dv of 128-wide heads, the keys' and the values' operands
// take 192 of the 256 registers that two waves a SIMD leave, too many beside the scores: there, half of the workgroups form
// dv and half dk, each with its own scores (five products in place of four: 3.0 ms on the sequences above; all four at one
// wave a SIMD 4.7).
enum Part { kBoth, kDv, kDk };

template <int D, Part PART>
struct WideGradKv {
  bf16x8 k[D / 16], v[PART == kDv ? 1 : D / 16];
  floatx16 dk[PART == kDv ? 1 : D / 32], dv[PART == kDk ? 1 : D / 32];
};

template <int D>
struct WideKvLds {
  struct Stats {
    float lse2[kWideKeys], delta[kWideKeys];
    int limit[kWideKeys];
  } stats[2];  // in front: their reads' offsets fit the instructions
  __attribute__((aligned(1024))) __bf16 q0[kWideKeys * D], g0[kWideKeys * D], q1[kWideKeys * D], g1[kWideKeys * D];
};

template <int D, Part PART>
__device__ __forceinline__ void wide_grad_kv_rows(const AttnArgs& a, WideGradKv<D, PART>& f, const __bf16* qs,
                                                  const __bf16* gs, const WidePlaces& w,
                                                  const typename WideKvLds<D>::Stats& stats, int key, bool masked) {
  const int hi = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    floatx16 s = zero16(), dp = zero16();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int st = 0; st < D / 16; ++st) {
      s = mma32(wide_row(qs, w, 32 * n, st), f.k[st], s);
      if (D == 128 && st == 3) __builtin_amdgcn_sched_barrier(0);
    }
    formed(s);
    if constexpr (PART != kDv) {
#pragma unroll
      for (int st = 0; st < D / 16; ++st) {
        dp = mma32(wide_row(gs, w, 32 * n, st), f.v[st], dp);
        if (D == 128 && st == 3) __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 32 * n + 8 * j + 4 * hi;
      const floatx4 l4 = *reinterpret_cast<const floatx4*>(stats.lse2 + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * j + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * j + i], a.c2, -l4[i]));
      if constexpr (PART != kDv) {
        const floatx4 d4 = *reinterpret_cast<const floatx4*>(stats.delta + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) dp[4 * j + i] = s[4 * j + i] * (dp[4 * j + i] - d4[i]);
      }
    }
    if (masked) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int4 m4 = *reinterpret_cast<const int4*>(stats.limit + 32 * n + 8 * j + 4 * hi);
        const int lim[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (PART != kDk && key >= p_limit(lim[i])) s[4 * j + i] = 0.f;
          if (PART != kDv && key >= lim[i]) dp[4 * j + i] = 0.f;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (PART != kDk) {
        const bf16x8 p = wide_pack(s, t);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) f.dv[dt] = mma32(wide_column(gs, w, 32 * n + 16 * t, 32 * dt), p, f.dv[dt]);
      }
      if constexpr (PART != kDv) {
        const bf16x8 ds = wide_pack(dp, t);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) f.dk[dt] = mma32(wide_column(qs, w, 32 * n + 16 * t, 32 * dt), ds, f.dk[dt]);
        if (D == 128) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}

template <int D, bool SPLIT, Part PART>
__device__ __forceinline__ void grad_kv_wide(const AttnArgs& a, int block, WideKvLds<D>& lds) {
  const int step_rows = a.step;
  const int lane = threadIdx.x & 63, c = lane & 31, hi = lane >> 5, wave = threadIdx.x >> 6;
  const int hk = block % a.Hk, rest = block / a.Hk;
  const int split = SPLIT ? rest % a.splits : 0, t = SPLIT ? rest / a.splits : rest;
  Seq s;
  int tile;
  if (!find_tile<false>(a, t, 1, kWide, &s, &tile)) return;
  const int key0 = tile * kWide, key = key0 + wave * 32 + c;
  const int wave_key = __builtin_amdgcn_readfirstlane(key0 + wave * 32);
  const bool real = key < s.nk;
  const int rows = s.nq * a.G;
  int row_lo = a.causal ? min(rows, max(0, key0 - s.nk + s.nq) * a.G) : 0, row_hi = rows;
  // Rows from here on see every key of the tile that exists, and more than one.
  const int open = s.nk == 1 ? rows : a.causal ? max(0, min(key0 + kWide, s.nk) - 1 - s.nk + s.nq) * a.G : 0;
  if (SPLIT) {
    const int each = ((rows - row_lo + a.splits - 1) / a.splits + step_rows - 1) / step_rows * step_rows;
    row_lo = min(rows, row_lo + split * each);
    row_hi = min(rows, row_lo + each);
  }
  const char* kbase = a.k.at + (static_cast<int64_t>(s.k0) + key0) * a.k.row + hk * a.k.head;
  const char* vbase = a.v.at + (static_cast<int64_t>(s.k0) + key0) * a.v.row + hk * a.v.head;
  const WidePlaces w = wide_places();
  WideGradKv<D, PART> f;
#pragma unroll
  for (int st = 0; st < D / 16; ++st) {
    const int64_t own = wave * 32 + c;
    const int off = (16 * st + 8 * hi) * 2;
    f.k[st] = real ? load_frag<__bf16>(kbase + own * a.k.row + off) : zero_frag<__bf16>();
    if constexpr (PART != kDv) f.v[st] = real ? load_frag<__bf16>(vbase + own * a.v.row + off) : zero_frag<__bf16>();
  }
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    if constexpr (PART != kDv) f.dk[dt] = zero16();
    if constexpr (PART != kDk) f.dv[dt] = zero16();
  }
  // A tile's rows are whole queries, a.step of them from row_lo on, a multiple of G.  (16 sequences of 2048, 12 heads of 64
  // that share 4, causal: backward 513 us with 63 rows a tile, 658 in the kernel of 64 keys; 20 of 577 of 128 191 and 240.)
  const QueryStage<D> qst(a, a.q), gst(a, a.dout);
  const char* qbase = a.q.at + s.q0 * a.q.row + hk * a.G * a.q.head;
  const char* gbase = a.dout.at + s.q0 * a.dout.row + hk * a.G * a.dout.head;
  const auto ask = [&](int r, __bf16* qt, __bf16* gt) {
    const int64_t n = div_group(a, r);
    qst.stage(a, qt, qbase + n * a.q.row, min(row_hi - r, step_rows));
    gst.stage(a, gt, gbase + n * a.dout.row, min(row_hi - r, step_rows));
  };
  // The rows' statistics go through a register, one tile ahead of their LDS; thread t < 64 moves row t's.
  const float2* const stats = a.stat + static_cast<int64_t>(s.q0) * a.H + hk * a.G;
  const auto ask_stat = [&](int r) {
    if (threadIdx.x >= kWideKeys) return make_float2(0.f, 0.f);
    const int n = div_group(a, r), t = thread_again(), query = div_group(a, t);
    const uint32_t off = min(query, s.nq - 1 - n) * a.H + t - query * a.G;
    return (stats + static_cast<int64_t>(n) * a.H)[off];
  };
  const auto put_stat = [&](int r, float2 stat, typename WideKvLds<D>::Stats& x) {
    if (threadIdx.x >= kWideKeys) return;
    const int query = div_group(a, r) + div_group(a, thread_again());
    const bool here = static_cast<int>(threadIdx.x) < min(row_hi - r, step_rows);
    x.lse2[threadIdx.x] = here ? stat.x : INFINITY;
    x.delta[threadIdx.x] = here ? stat.y : 0.f;
    x.limit[threadIdx.x] = !here ? 0 : both_limits(a.causal ? max(0, min(s.nk, query + 1 + s.nk - s.nq)) : s.nk);
  };
  const auto step = [&](int r, const __bf16* qt, const __bf16* gt, const typename WideKvLds<D>::Stats& here, __bf16* qn,
                        __bf16* gn, typename WideKvLds<D>::Stats& next) {
    staged();
    const bool more = r > row_lo;
    float2 stat;
    if (more) {
      stat = ask_stat(r - step_rows);
      ask(r - step_rows, qn, gn);
    }
    if (wave_key < wave_limit(a, s, r, step_rows))
      wide_grad_kv_rows<D, PART>(a, f, qt, gt, w, here, key, r < open || r + kWideKeys > row_hi || step_rows < kWideKeys);
    if (more) put_stat(r - step_rows, stat, next);
  };
  // From the last rows back: every tile of keys begins with the same rows, and the tiles at work share them in the L2
  // (each from its own first rows on: 4050 us in place of 3610).
  const int last = row_lo + max(row_hi - row_lo - 1, 0) / step_rows * step_rows;
  if (row_lo < row_hi) {
    const float2 stat = ask_stat(last);
    ask(last, lds.q0, lds.g0);
    put_stat(last, stat, lds.stats[0]);
    for (int r = last; r >= row_lo; r -= 2 * step_rows) {
      step(r, lds.q0, lds.g0, lds.stats[0], lds.q1, lds.g1, lds.stats[1]);
      if (r == row_lo) break;
      step(r - step_rows, lds.q1, lds.g1, lds.stats[1], lds.q0, lds.g0, lds.stats[0]);
    }
  }
  const int thread = thread_again(), out_key = key0 + thread / 64 * 32 + thread % 32, hi4 = thread % 64 / 32 * 4;
  if (out_key >= s.nk) return;
  const int64_t at = static_cast<int64_t>(s.k0) + out_key;
  float* part = SPLIT ? a.part + ((split * a.Hk + hk) * a.total_k + at) * 2 * D + hi4 : nullptr;
  char* kto = a.dk.at + at * a.dk.row + hk * a.dk.head + hi4 * 2;
  char* vto = a.dv.at + at * a.dv.row + hk * a.dv.head + hi4 * 2;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int d = 32 * dt + 8 * n;
      if constexpr (PART != kDv) {
        const floatx4 x = {f.dk[dt][4 * n], f.dk[dt][4 * n + 1], f.dk[dt][4 * n + 2], f.dk[dt][4 * n + 3]};
        if (SPLIT) *reinterpret_cast<floatx4*>(part + d) = x;
        else store4<__bf16>(kto + d * 2, x * a.scale);
      }
      if constexpr (PART != kDk) {
        const floatx4 y = {f.dv[dt][4 * n], f.dv[dt][4 * n + 1], f.dv[dt][4 * n + 2], f.dv[dt][4 * n + 3]};
        if (SPLIT) *reinterpret_cast<floatx4*>(part + D + d) = y;
        else store4<__bf16>(vto + d * 2, y);
      }
    }
}

template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void grad_kv_wide_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) WideKvLds<D> lds;
  if constexpr (D == 64) {
    grad_kv_wide<D, SPLIT, kBoth>(a, blockIdx.x, lds);
  } else {
    const int hk = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk, block = rest / 2 * a.Hk + hk;
    if (rest % 2) grad_kv_wide<D, SPLIT, kDv>(a, block, lds);
    else grad_kv_wide<D, SPLIT, kDk>(a, block, lds);
  }
}

// dk and dv of 64 keys over the rows that see them.  fp32, the sequences above: 77
// us, matrix units busy 53 %.  (fp32 tiles of 32 rows a wave: 53, 71 and 92 us for
// the three kernels in place of 45, 60 and 77.)
template <class E, int D, bool SPLIT>
__global__ __launch_bounds__(kThreads) void grad_kv_kernel(AttnArgs a) {
  typedef typename Op<E>::Frag Frag;
  typedef Staged<E, D> Tile;
  constexpr int kRows = Tile::kRows, kLd = Tile::kLd;
  __shared__ alignas(16) E qs[kRows * kLd];
  __shared__ alignas(16) E gs[kRows * kLd];
  __shared__ floatx4 lse_s[kRows / 4], delta_s[kRows / 4];
  __shared__ int4 limit_s[kRows / 4];
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const int hk = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk;
  const int split = SPLIT ? rest % a.splits : 0, t = SPLIT ? rest / a.splits : rest;
  Seq s;
  int tile;
  if (!find_tile<false>(a, t, 1, kTile, &s, &tile)) return;
  const int key0 = tile * kTile, key = key0 + wave * 16 + c16;
  const int wave_key = __builtin_amdgcn_readfirstlane(key0 + wave * 16);
  const bool real = key < s.nk;
  const int rows = s.nq * a.G;
  // The first row that sees a key of the tile.
  int row_lo = a.causal ? min(rows, max(0, key0 - s.nk + s.nq) * a.G) : 0, row_hi = rows;
  if (SPLIT) {
    const int each = ((rows - row_lo + a.splits - 1) / a.splits + kRows - 1) / kRows * kRows;
    row_lo = min(rows, row_lo + split * each);
    row_hi = min(rows, row_lo + each);
  }
  // Rows before this one see at most one key, where that key is the tile's first.
  const int one_key = key0 > 0 ? 0 : s.nk == 1 ? rows : a.causal ? max(0, s.nq - s.nk + 1) * a.G : 0;
  const char* krow = a.k.at + (static_cast<int64_t>(s.k0) + key) * a.k.row + hk * a.k.head;
  const char* vrow = a.v.at + (static_cast<int64_t>(s.k0) + key) * a.v.row + hk * a.v.head;
  Frag kf[D / 32], vf[D / 32];
#pragma unroll
  for (int st = 0; st < D / 32; ++st) {
    const int off = (32 * st + 8 * g) * sizeof(E);
    kf[st] = real ? load_frag<E>(krow + off) : zero_frag<E>();
    vf[st] = real ? load_frag<E>(vrow + off) : zero_frag<E>();
  }
  floatx4 dk[D / 16], dv[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) dk[dt] = dv[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  Tile qt, gt;
  float2 stat = {};
  int limit = 0;
  const auto ask = [&](int r) {
    qt.load(row_hi - r, [&](int i) { return query_row(a, a.q, s, hk, r + i); });
    gt.load(row_hi - r, [&](int i) { return query_row(a, a.dout, s, hk, r + i); });
    if (threadIdx.x < kRows) {
      const int row = r + threadIdx.x;
      const bool here = row < row_hi;
      stat = here ? a.stat[stat_at(a, s, hk, row)] : make_float2(INFINITY, 0.f);
      limit = here ? limit_of(a, s, row) : 0;
    }
  };
  if (row_lo < row_hi) ask(row_lo);
  for (int r = row_lo; r < row_hi; r += kRows) {
    __syncthreads();
    qt.store(qs);
    gt.store(gs);
    if (threadIdx.x < kRows) {
      reinterpret_cast<float*>(lse_s)[threadIdx.x] = stat.x;
      reinterpret_cast<float*>(delta_s)[threadIdx.x] = stat.y;
      reinterpret_cast<int*>(limit_s)[threadIdx.x] = limit;
    }
    __syncthreads();
    if (r + kRows < row_hi) ask(r + kRows);
    if (wave_key >= wave_limit(a, s, r, kRows)) continue;
#pragma unroll
    for (int st32 = 0; st32 < kRows / 32; ++st32) {
      floatx4 p[2], ds[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r0 = st32 * 32 + half * 16;
        floatx4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < D / 32; ++st) {
          sc = Op<E>::mma(load_frag<E>(qs + (r0 + c16) * kLd + 32 * st + 8 * g), kf[st], sc);
          dp = Op<E>::mma(load_frag<E>(gs + (r0 + c16) * kLd + 32 * st + 8 * g), vf[st], dp);
        }
        const floatx4 l4 = lse_s[r0 / 4 + g], d4 = delta_s[r0 / 4 + g];
        const int4 m4 = limit_s[r0 / 4 + g];
        const int lim[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = key < lim[i];
          p[half][i] = seen ? __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.c2, -l4[i])) : 0.f;
          ds[half][i] = seen ? p[half][i] * (dp[i] - d4[i]) : 0.f;
        }
        if (r < one_key) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (lim[i] == 1) ds[half][i] = 0.f;
        }
      }
      const Frag pf = Op<E>::pack(p[0], p[1]), df = Op<E>::pack(ds[0], ds[1]);
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        dv[dt] = Op<E>::mma(Op<E>::template columns<kLd>(gs + st32 * 32 * kLd, dt * 16), pf, dv[dt]);
        dk[dt] = Op<E>::mma(Op<E>::template columns<kLd>(qs + st32 * 32 * kLd, dt * 16), df, dk[dt]);
      }
    }
  }
  if (!real) return;
  const int64_t at = static_cast<int64_t>(s.k0) + key;
  if (SPLIT) {
    float* to = a.part + ((split * a.Hk + hk) * a.total_k + at) * 2 * D;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      *reinterpret_cast<floatx4*>(to + dt * 16 + 4 * g) = dk[dt];
      *reinterpret_cast<floatx4*>(to + D + dt * 16 + 4 * g) = dv[dt];
    }
    return;
  }
  char* kto = a.dk.at + at * a.dk.row + hk * a.dk.head;
  char* vto = a.dv.at + at * a.dv.row + hk * a.dv.head;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    store4<E>(kto + (dt * 16 + 4 * g) * sizeof(E), dk[dt] * a.scale);
    store4<E>(vto + (dt * 16 + 4 * g) * sizeof(E), dv[dt]);
  }
}

// The parts of dk and dv added in their order: four elements a thread.
template <class E, int D>
__global__ __launch_bounds__(kThreads) void join_kv_kernel(AttnArgs a) {
  constexpr int kQuads = 2 * D / 4, kKeysHere = kThreads / kQuads;
  const int64_t at = static_cast<int64_t>(blockIdx.x / a.Hk) * kKeysHere + threadIdx.x / kQuads;
  const int hk = blockIdx.x % a.Hk, d = threadIdx.x % kQuads * 4;
  const bool here = at < a.total_k;
  const int64_t key = here ? at : a.total_k - 1;
  // Each wave holds one key at D 128, else several: the search is for the wave, so each of them in turn.
  constexpr int kPerWave = 64 / kQuads > 1 ? 64 / kQuads : 1;
  bool mine = false;
  for (int i = 0; i < kPerWave; ++i) {
    const int64_t n = __shfl(static_cast<int>(key), i * (64 / kPerWave));
    const int b = last_at_most(a.B, n, [&](int j) { return static_cast<int64_t>(a.cu_k[j]); });
    Seq s;
    const bool in = sequence(a, b, &s) && n >= s.k0 && n < static_cast<int64_t>(s.k0) + s.nk;
    if ((threadIdx.x & 63) / (64 / kPerWave) == i) mine = in;
  }
  if (!here || !mine) return;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < a.splits; ++p)
    sum += *reinterpret_cast<const floatx4*>(a.part + ((p * a.Hk + hk) * a.total_k + at) * 2 * D + d);
  if (d < D) store4<E>(a.dk.at + at * a.dk.row + hk * a.dk.head + d * sizeof(E), sum * a.scale);
  else store4<E>(a.dv.at + at * a.dv.row + hk * a.dv.head + (d - D) * sizeof(E), sum);
}

// --------------------------------- host -----------------------------------

// The kernels of 128 rows or keys: where the bytes from a staged tile's first row to its last fit the 32-bit offsets, and
// from this many rows (keys) a sequence on, by the average.  Both sides in us, 8 heads, as many sequences as fill the GPU:
//   forward   64 rows of 64 50.6 narrow, 52.5 wide; 65 rows 74, 61; 64 rows of 128 80.7, 83.2; 65 rows 133, 102
//   backward  160 rows of 64 186, 188; 200 rows 142, 129; 64 rows of 128 271, 275; 65 rows 451, 324
constexpr int64_t kWideRows = kTile, kWideGradRows64 = 176;
bool near(const RowView& x, int64_t rows, int64_t heads) { return x.row * rows + x.head * heads < (int64_t{1} << 31); }
bool use_wide(const Sizes& z, int dtype, const AttnArgs& a, bool grad) {
  return dtype == DORA_BF16 && z.D >= 64 && near(a.k, 128, 0) && near(a.v, 128, 0) &&
         z.total_q * a.G / z.B > (grad && z.D == 64 ? kWideGradRows64 : kWideRows);
}
bool use_wide_kv(const Sizes& z, int dtype, const AttnArgs& a) {
  return dtype == DORA_BF16 && z.D >= 64 && a.step >= 48 && near(a.q, 64, a.G) && near(a.dout, 64, a.G) &&
         z.total_k / z.B > (z.D == 64 ? kWideGradRows64 : kWideRows);
}

bool same_sizes(const dora_rows* s, const dora_rows* t) {
  return s->rows == t->rows && s->heads == t->heads && s->dim == t->dim && s->dtype == t->dtype;
}

// Everything but the outputs and the workspace; fills the kernels' arguments.
int check_attn(const dora_rows* q, const dora_rows* k, const dora_rows* v, const int32_t* cu_q, const int32_t* cu_k,
               int32_t B, int32_t max_q, int32_t causal, float softmax_scale, int32_t* dev_status, Sizes* z,
               AttnArgs* a) {
  if (!q || !k || !v || !cu_q || !cu_k || !dev_status) return DORA_ERR_NULL;
  for (const dora_rows* t : {q, k, v}) {
    const int rc = check_rows(t, 16);
    if (rc != DORA_OK) return rc;
  }
  if (q->dtype != k->dtype) return DORA_ERR_DTYPE;
  if (!same_sizes(k, v) || k->dim != q->dim) return DORA_ERR_SHAPE;
  *z = Sizes{B, q->heads, k->heads, q->dim, max_q, q->rows, k->rows};
  if (!good_sizes(*z) || !(softmax_scale < INFINITY)) return DORA_ERR_SHAPE;
  *a = AttnArgs{};
  a->q = row_view(q), a->k = row_view(k), a->v = row_view(v);
  a->cu_q = cu_q, a->cu_k = cu_k;
  a->B = B, a->H = z->H, a->Hk = z->Hk, a->G = z->H / z->Hk;
  int bits = 0;
  while ((1 << bits) < a->G) ++bits;
  // mul = ceil(2^(31 + bits) / G) < 2^32: r mul / 2^(31 + bits) lies less than 1 / G above r / G for r < 2^31
  a->g_mul = bits ? static_cast<uint32_t>(((uint64_t{1} << (31 + bits)) + a->G - 1) / a->G) : 0;
  a->g_shift = bits ? bits - 1 : 0;
  a->total_q = z->total_q, a->total_k = z->total_k;
  a->max_q = max_q, a->max_k = 0x7FFFFFFF, a->causal = causal != 0;
  a->scale = softmax_scale > 0.f ? softmax_scale : static_cast<float>(1.0 / std::sqrt(static_cast<double>(z->D)));
  a->c2 = a->scale * kLog2e;
  a->step = kWideKeys / a->G * a->G;
  a->ranked = B <= 64;
  a->status = dev_status;
  return DORA_OK;
}

bool too_small(const void* ws, size_t bytes, size_t need) {
  return !ws || reinterpret_cast<uintptr_t>(ws) & 255u || bytes < need;
}

constexpr int64_t kMaxBlocks = (int64_t{1} << 32) / kThreads - 2;  // threads of a launch in 32 bits

// The launch for an element type and a head width: f(E{}, integral_constant D).
template <class F>
void with_type(int dtype, int D, F f) {
  const auto width = [&](auto e) {
    if (D == 32) f(e, std::integral_constant<int, 32>{});
    else if (D == 64) f(e, std::integral_constant<int, 64>{});
    else f(e, std::integral_constant<int, 128>{});
  };
  if (dtype == DORA_BF16) width(__bf16{});
  else width(float{});
}

}  // namespace
}  // namespace dora

extern "C" size_t dora_grouped_attn_workspace_size(int32_t B, int32_t H, int32_t Hk, int32_t D, int32_t max_q,
                                                   int64_t total_q, int64_t total_k) {
  const dora::Sizes z{B, H, Hk, D, max_q, total_q, total_k};
  return dora::good_sizes(z) ? dora::forward_bytes(z) : 0;
}

extern "C" size_t dora_grouped_attn_backward_workspace_size(int32_t B, int32_t H, int32_t Hk, int32_t D, int32_t max_q,
                                                            int64_t total_q, int64_t total_k) {
  const dora::Sizes z{B, H, Hk, D, max_q, total_q, total_k};
  return dora::good_sizes(z) ? dora::backward_bytes(z) : 0;
}

extern "C" int dora_grouped_attn(const dora_rows* q, const dora_rows* k, const dora_rows* v, const int32_t* cu_q,
                                 const int32_t* cu_k, int32_t B, int32_t max_q, int32_t max_k, int32_t causal,
                                 float softmax_scale, const dora_rows* out, float* lse_out, void* workspace, size_t workspace_bytes,
                                 int32_t* dev_status, void* stream) {
  using namespace dora;
  if (!out) return DORA_ERR_NULL;
  Sizes z;
  AttnArgs a;
  int rc = check_attn(q, k, v, cu_q, cu_k, B, max_q, causal, softmax_scale, dev_status, &z, &a);
  if (rc == DORA_OK) rc = check_rows(out, 16);
  if (rc != DORA_OK) return rc;
  if (!same_sizes(out, q) || max_k < 0) return DORA_ERR_SHAPE;
  if (max_k > 0) a.max_k = max_k;
  if (too_small(workspace, workspace_bytes, forward_bytes(z))) return DORA_ERR_WORKSPACE;
  const size_t cu_bytes = (static_cast<size_t>(B) + 1) * sizeof(int32_t);
  if (rows_clash({out}, {q, k, v}, {},
                 {{lse_out, static_cast<size_t>(z.total_q) * z.H * sizeof(float)},
                  {workspace, forward_bytes(z)},
                  {dev_status, sizeof(int32_t)}},
                 {{cu_q, cu_bytes}, {cu_k, cu_bytes}}))
    return DORA_ERR_OVERLAP;
  if (z.total_q == 0) return DORA_OK;
  const Split p = forward_split(z, max_k);
  const bool split = p.splits > 1 || p.chunk;
  const bool wide = !split && use_wide(z, q->dtype, a, false);
  const int64_t blocks = (wide ? tiles(z.total_q * a.G, B, kWide) : p.blocks) * z.Hk, join = (z.total_q * z.H + kThreads / 64 - 1) / (kThreads / 64);
  if (blocks > kMaxBlocks || (split && join > kMaxBlocks)) return DORA_ERR_UNSUPPORTED;
  a.out = row_view(out);
  a.lse = lse_out;
  // 16-byte rows first
  a.part = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part + p.blocks * z.Hk * p.part_rows * z.D);
  a.splits = p.splits, a.chunk = p.chunk, a.part_rows = p.part_rows;
  a.blocks = static_cast<int32_t>(blocks);
  a.mixed = !split && mix_tiles(z.total_q * a.G, B, wide ? kWide : kTile);
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(q->dtype, z.D, [&](auto e, auto d) {
    typedef decltype(e) E;
    constexpr int D = decltype(d)::value;
    if (split) {
      hipLaunchKernelGGL((attn_kernel<E, D, true>), dim3(a.blocks + 1), dim3(kThreads), 0, st, a);
      hipLaunchKernelGGL((join_kernel<E, D>), dim3(static_cast<uint32_t>(join)), dim3(kThreads), 0, st, a);
    } else if constexpr (sizeof(E) == 2 && D >= 64) {
      if (wide) hipLaunchKernelGGL((attn_wide_kernel<D>), dim3(a.blocks + 1), dim3(kThreads), 0, st, a);
      else hipLaunchKernelGGL((attn_kernel<E, D, false>), dim3(a.blocks + 1), dim3(kThreads), 0, st, a);
    } else {
      hipLaunchKernelGGL((attn_kernel<E, D, false>), dim3(a.blocks + 1), dim3(kThreads), 0, st, a);
    }
  });
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}

extern "C" int dora_grouped_attn_backward(const dora_rows* dout, const dora_rows* q, const dora_rows* k,
                                          const dora_rows* v, const dora_rows* out, const float* lse,
                                          const int32_t* cu_q, const int32_t* cu_k, int32_t B, int32_t max_q,
                                          int32_t causal, float softmax_scale, const dora_rows* dq,
                                          const dora_rows* dk, const dora_rows* dv, void* workspace,
                                          size_t workspace_bytes, int32_t* dev_status, void* stream) {
  using namespace dora;
  if (!q || !dout || !out || (!lse && q->rows > 0) || !dq || !dk || !dv) return DORA_ERR_NULL;
  Sizes z;
  AttnArgs a;
  int rc = check_attn(q, k, v, cu_q, cu_k, B, max_q, causal, softmax_scale, dev_status, &z, &a);
  for (const dora_rows* t : {dout, out, dq, dk, dv})
    if (rc == DORA_OK) rc = check_rows(t, 16);
  if (rc != DORA_OK) return rc;
  if (!same_sizes(dout, q) || !same_sizes(out, q) || !same_sizes(dq, q) || !same_sizes(dk, k) || !same_sizes(dv, k))
    return DORA_ERR_SHAPE;
  if (too_small(workspace, workspace_bytes, backward_bytes(z))) return DORA_ERR_WORKSPACE;
  const size_t cu_bytes = (static_cast<size_t>(B) + 1) * sizeof(int32_t);
  if (rows_clash({dq, dk, dv}, {q, k, v, out, dout}, {},
                 {{workspace, backward_bytes(z)}, {dev_status, sizeof(int32_t)}},
                 {{cu_q, cu_bytes}, {cu_k, cu_bytes}, {lse, static_cast<size_t>(z.total_q) * z.H * sizeof(float)}}))
    return DORA_ERR_OVERLAP;
  a.dout = row_view(dout);
  const bool wide_q = use_wide(z, q->dtype, a, true), wide_kv = use_wide_kv(z, q->dtype, a);
  const int64_t q_blocks = tiles(z.total_q * a.G, B, wide_q ? kWide : kTile) * z.Hk;
  const int32_t splits = backward_splits(z);
  const int64_t kv_blocks = tiles(z.total_k, B, wide_kv ? kWide : kTile) * z.Hk * splits * (wide_kv && z.D == 128 ? 2 : 1);
  const int keys_here = kThreads / (2 * z.D / 4);
  const int64_t join = (z.total_k + keys_here - 1) / keys_here * z.Hk;
  if (q_blocks > kMaxBlocks || kv_blocks > kMaxBlocks || join > kMaxBlocks) return DORA_ERR_UNSUPPORTED;
  a.out = row_view(out);
  a.dq = row_view(dq), a.dk = row_view(dk), a.dv = row_view(dv);
  a.lse = const_cast<float*>(lse);
  a.stat = static_cast<float2*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + stat_bytes(z));
  a.splits = splits;
  a.blocks = static_cast<int32_t>(q_blocks);
  a.mixed = mix_tiles(z.total_q * a.G, B, wide_q ? kWide : kTile);
  AttnArgs kv = a;
  kv.blocks = static_cast<int32_t>(tiles(z.total_k, B, wide_kv ? kWide : kTile) * z.Hk * splits);
  kv.mixed = splits == 1 && mix_tiles(z.total_k, B, wide_kv ? kWide : kTile);
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(q->dtype, z.D, [&](auto e, auto d) {
    typedef decltype(e) E;
    constexpr int D = decltype(d)::value;
    const dim3 gq(a.blocks + 1), gkv(static_cast<uint32_t>(kv_blocks)), block(kThreads);
    bool launched_q = false, launched_kv = z.total_k == 0;
    if constexpr (sizeof(E) == 2 && D >= 64) {
      if (wide_q) hipLaunchKernelGGL((grad_q_wide_kernel<D>), gq, block, 0, st, a);
      if (wide_kv && !launched_kv) {
        if (!wide_q) hipLaunchKernelGGL((grad_q_kernel<E, D>), gq, block, 0, st, a);
        launched_q = launched_kv = true;
        if (splits > 1) hipLaunchKernelGGL((grad_kv_wide_kernel<D, true>), gkv, block, 0, st, kv);
        else hipLaunchKernelGGL((grad_kv_wide_kernel<D, false>), gkv, block, 0, st, kv);
      }
      launched_q = launched_q || wide_q;
    }
    if (!launched_q) hipLaunchKernelGGL((grad_q_kernel<E, D>), gq, block, 0, st, a);
    if (!launched_kv) {
      if (splits > 1) hipLaunchKernelGGL((grad_kv_kernel<E, D, true>), gkv, block, 0, st, kv);
      else hipLaunchKernelGGL((grad_kv_kernel<E, D, false>), gkv, block, 0, st, kv);
    }
    if (splits > 1 && z.total_k > 0)
      hipLaunchKernelGGL((join_kv_kernel<E, D>), dim3(static_cast<uint32_t>(join)), block, 0, st, a);
  });
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
