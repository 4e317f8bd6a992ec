// Global norm of many gradient tensors, and clipping by it.  DORA (arXiv
// 2609.34325), App. D: the actor's gradients are clipped at a global norm.
//
//   norm = sqrt(sum over tensors and elements of g^2)
//   c = min(1, max_norm / (norm + eps)),  out = c g
//
// HBM bound: one read for the norm, one read and one write to scale.  The
// tensors' addresses go in by kernel argument, as many as 4 KB hold; tensors
// are cut into chunks, and a workgroup takes every gridDim-th chunk, four
// 16-byte pieces in flight a thread.  Squares are added in 64 bits: no fp32
// gradient overflows them, and the sum does not hang on the split.  Workgroups
// write their sums to the workspace; every workgroup of a scaling launch adds
// them all in the same order.  304M fp32 elements in 296 tensors, out of place:
// norm 237 us (5.1 TB/s), scaling 493 (4.9 TB/s); 22M bf16 in 152: 11 and 15.
#include <algorithm>
#include <cstdlib>

#include "dora_internal.h"
#include "policy_terms.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr int kFlight = 4;                       // pieces in flight a thread
// Elements of a chunk: what makes about 2048 of them, one a workgroup, within
// these bounds.  (22M bf16 elements: 2048 chunks 27.5 us, 4096 29.9.)
constexpr int kMinChunk = 2048, kMaxChunk = 32768, kManyChunks = 2048;
constexpr int kMaxGroups = 2048;                 // workgroups of a pass, the share of each launch rounded up
constexpr int kMaxSpans = 1 << 16;
// Up to these bytes both passes give a chunk to the same workgroup, whose die
// may still hold it; past them the norm's pass takes the list from its end, so
// that the scaling begins with what the caches still hold.  us a pass the same
// way and from the end: 21 MB 14.6, 15.5, 44 MB 27.1, 27.7, 1.2 GB 750.9, 747.8.
constexpr int64_t kWhole = int64_t{64} << 20;
constexpr int64_t kPart = int64_t{1} << 30;      // longer tensors go in as several
constexpr int64_t kMaxTotal = int64_t{1} << 40;  // elements of a call
constexpr uint32_t kBF16 = 1u << 31;

// Tensors of one launch, in at most 4 KB of arguments.
template <int N, bool OUT>
struct SpanBlock {
  static constexpr int kSpans = N;
  const char* in[N];
  char* out[OUT ? N : 1];
  uint32_t numel[N];  // | kBF16
  int32_t first[N];   // chunks before the tensor, in this launch
  int32_t n, chunks, chunk;
};
typedef SpanBlock<248, false> InBlock;   // read, or scaled in place
typedef SpanBlock<160, true> PairBlock;
static_assert(sizeof(InBlock) + 64 <= 4096 && sizeof(PairBlock) + 64 <= 4096, "kernel arguments");

// A chunk's tensor and elements.  BACK: the tensor's chunks from its end.
struct Chunk {
  int span;
  int64_t lo, hi;
  bool bf16;
};
// The tensor is the last that starts at or before the chunk: the lanes compare
// with all of them at once (a search by halves would wait for memory eight times).
template <bool BACK, class B>
__device__ __forceinline__ Chunk find_chunk(const B& b, int chunk) {
  const int lane = threadIdx.x & 63;
  int before = 0;
#pragma unroll
  for (int i = 0; i < B::kSpans; i += 64) {
    const int j = i + lane;
    before += __popcll(__ballot(j < b.n && b.first[min(j, B::kSpans - 1)] <= chunk));
  }
  const int t = __builtin_amdgcn_readfirstlane(before - 1);
  const uint32_t code = b.numel[t];
  const int numel = static_cast<int>(code & ~kBF16), place = chunk - b.first[t];
  const int64_t lo = static_cast<int64_t>(BACK ? (numel - 1) / b.chunk - place : place) * b.chunk;
  return {t, lo, min(static_cast<int64_t>(numel), lo + b.chunk), (code & kBF16) != 0};
}

// Pieces of 16 bytes at the element's alignment: the hardware takes unaligned
// ones, so that views into a flat buffer run like tensors of their own.
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
  static constexpr int E = 8, kBytes = 2;
  __device__ static float get(const char* p) {
    return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p)) << 16);
  }
  __device__ static void put(char* p, float v) { *reinterpret_cast<__bf16*>(p) = static_cast<__bf16>(v); }
  __device__ static float part(u32x4 v, int i) {
    return __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
  }
  __device__ static u32x4 pack(const float (&f)[E]) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < E; ++i) b[i] = static_cast<__bf16>(f[i]);
    return __builtin_bit_cast(u32x4, b);
  }
};
template <>
struct Piece<false> {
  static constexpr int E = 4, kBytes = 4;
  __device__ static float get(const char* p) { return *reinterpret_cast<const float*>(p); }
  __device__ static void put(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
  __device__ static float part(u32x4 v, int i) { return __uint_as_float(v[i]); }
  __device__ static u32x4 pack(const float (&f)[E]) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};

// kFlight pieces of a thread, from piece `first` on.  Loaded unconditionally,
// from clamped places: counted loads, waited for one by one.  whole > 0.
struct Batch {
  typedef u32x4 __attribute__((aligned(2))) Vec;
  u32x4 v[kFlight];
  __device__ void load(const char* p, int first, int whole) {
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      v[k] = *reinterpret_cast<const Vec*>(p + static_cast<int64_t>(min(first + k * kThreads, whole - 1)) * 16);
    asm volatile("" ::: "memory");
  }
  template <class Each>
  __device__ void each(int first, int whole, Each f) const {
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (first + k * kThreads < whole) f(v[k], first + k * kThreads);
  }
};

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s_red[kThreads / 64];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) t += s_red[w];
  return t;
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const char* p, int n) {
  using P = Piece<BF16>;
  const int whole = n / P::E;
  double s = 0.0;
  for (int i = threadIdx.x; i < whole; i += kFlight * kThreads) {
    Batch b;
    b.load(p, i, whole);
    b.each(i, whole, [&](u32x4 v, int) {
#pragma unroll
      for (int e = 0; e < P::E; ++e) {
        const double g = P::part(v, e);
        s = fma(g, g, s);
      }
    });
  }
  const int j = whole * P::E + threadIdx.x;
  if (j < n) {
    const double g = P::get(p + static_cast<int64_t>(j) * P::kBytes);
    s = fma(g, g, s);
  }
  return s;
}

template <bool BACK>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(InBlock b, double* parts) {
  double s = 0.0;
  for (int c = blockIdx.x; c < b.chunks; c += gridDim.x) {
    const Chunk k = find_chunk<BACK>(b, c);
    const char* p = b.in[k.span] + k.lo * (k.bf16 ? 2 : 4);
    const int n = static_cast<int>(k.hi - k.lo);
    s += k.bf16 ? chunk_squares<true>(p, n) : chunk_squares<false>(p, n);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// Every workgroup that asks gets the same value.
__device__ __forceinline__ double norm_of(const double* parts, int32_t n) {
  constexpr int kAtOnce = kMaxGroups / kThreads;
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kAtOnce * kThreads) {
    double v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) v[k] = parts[min(i + k * kThreads, n - 1)];
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) s += i + k * kThreads < n ? v[k] : 0.0;
  }
  return sqrt(block_sum(s));
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* parts, int32_t n, float* norm) {
  const double v = norm_of(parts, n);
  if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

// The factor as a product: a small one (gradients near fp32's limit) would
// itself be subnormal in fp32 and short of bits, or 0.  Results that are not
// subnormal have a factor of at least 2^-254, so c is not subnormal there.
struct Factor {
  float pre, c;
  __device__ explicit Factor(double f) {
    pre = f >= 0x1p-64 ? 1.0f : (f >= 0x1p-128 ? 0x1p-64f : 0x1p-128f);
    c = static_cast<float>(f / pre);
  }
  __device__ float operator*(float g) const { return g * pre * c; }
  __device__ bool keeps() const { return pre == 1.0f && c == 1.0f; }
};

// The chunk's n elements scaled, the thread's first pieces being there.
template <bool BF16>
__device__ __forceinline__ void chunk_scale(const char* in, char* out, int n, Batch b, Factor f) {
  using P = Piece<BF16>;
  const int whole = n / P::E;
  for (int i = threadIdx.x; i < whole;) {
    b.each(i, whole, [&](u32x4 v, int at) {
      float x[P::E];
#pragma unroll
      for (int e = 0; e < P::E; ++e) x[e] = f * P::part(v, e);
      *reinterpret_cast<Batch::Vec*>(out + static_cast<int64_t>(at) * 16) = P::pack(x);
    });
    i += kFlight * kThreads;
    if (i < whole) b.load(in, i, whole);
  }
  const int j = whole * P::E + threadIdx.x;
  if (j < n) P::put(out + static_cast<int64_t>(j) * P::kBytes, f * P::get(in + static_cast<int64_t>(j) * P::kBytes));
}

// PairBlock: out of place; InBlock: in place.  Every workgroup has a chunk;
// its first pieces are on their way while the norm is added up.
template <class B>
__global__ __launch_bounds__(kThreads, 6) void grad_scale_kernel(B b, const double* parts, int32_t n, float max_norm,
                                                              float eps, float* norm_out) {
  constexpr bool kInPlace = sizeof(b.out) == sizeof(char*);
  Factor f(1.0);
  for (int i = blockIdx.x; i < b.chunks; i += gridDim.x) {
    const Chunk k = find_chunk<false>(b, i);
    const int len = static_cast<int>(k.hi - k.lo), size = k.bf16 ? 2 : 4;
    const char* in = b.in[k.span] + k.lo * size;
    char* out = kInPlace ? const_cast<char*>(in) : b.out[k.span] + k.lo * size;
    Batch first;
    if (len * size >= 16) first.load(in, threadIdx.x, len * size / 16);
    if (i == blockIdx.x) {
      const double norm = norm_of(parts, n);
      if (norm_out && i == 0 && threadIdx.x == 0) *norm_out = static_cast<float>(norm);
      const double ratio = norm == 0.0 || max_norm == __builtin_inff()
                               ? 1.0
                               : static_cast<double>(max_norm) / (norm + static_cast<double>(eps));
      f = Factor(ratio >= 1.0 ? 1.0 : ratio);  // NaN stays
      if (kInPlace && f.keeps()) return;
    }
    if (f.keeps() && in == out) continue;
    if (k.bf16) chunk_scale<true>(in, out, len, first, f);
    else chunk_scale<false>(in, out, len, first, f);
  }
}

struct Range {
  uintptr_t lo, hi;
  int32_t span;
  bool written;
};

int64_t span_bytes(const dora_span& s) { return s.numel * (s.dtype == DORA_BF16 ? 2 : 4); }

// Each output apart from every other tensor but its own input.
bool ranges_clash(const dora_span* grads, const dora_span* out, int32_t n, Range* r) {
  int64_t m = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (grads[i].numel == 0) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(grads[i].data), len = span_bytes(grads[i]);
    const uintptr_t o = out ? reinterpret_cast<uintptr_t>(out[i].data) : a;
    r[m++] = Range{o, o + len, i, true};
    if (a != o) r[m++] = Range{a, a + len, i, false};
  }
  std::sort(r, r + m, [](const Range& x, const Range& y) { return x.lo < y.lo; });
  uintptr_t read_end = 0, write_end = 0;
  for (int64_t i = 0; i < m; ++i) {
    if (r[i].lo < write_end || (r[i].written && r[i].lo < read_end)) return true;
    uintptr_t& end = r[i].written ? write_end : read_end;
    end = std::max(end, r[i].hi);
  }
  return false;
}

int check_spans(const dora_span* s, int32_t n) {
  for (int32_t i = 0; i < n; ++i) {
    if (s[i].dtype != DORA_BF16 && s[i].dtype != DORA_F32) return DORA_ERR_DTYPE;
    if (s[i].numel < 0 || s[i].numel > (int64_t{1} << 40)) return DORA_ERR_SHAPE;
    if (s[i].numel > 0 && !s[i].data) return DORA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(s[i].data) % (s[i].dtype == DORA_BF16 ? 2 : 4)) return DORA_ERR_ALIGN;
  }
  return DORA_OK;
}

// How far a pass over the list has come: tensors, and elements of the next one.
struct Place {
  int32_t spans;
  int64_t elements;
};

// The next launch's tensors, empty ones left out; BACK: from the list's end.
template <bool BACK, class B>
void fill_block(const dora_span* grads, const dora_span* out, int32_t n, Place& at, int chunk, B* b) {
  b->n = b->chunks = 0;
  b->chunk = chunk;
  while (at.spans < n && b->n < B::kSpans) {
    const int32_t s = BACK ? n - 1 - at.spans : at.spans;
    const dora_span& g = grads[s];
    const int64_t len = std::min(g.numel - at.elements, kPart);
    if (len > 0) {
      const int i = b->n++;
      const int64_t byte = (BACK ? g.numel - at.elements - len : at.elements) * (g.dtype == DORA_BF16 ? 2 : 4);
      b->in[i] = static_cast<const char*>(g.data) + byte;
      if (sizeof(b->out) > sizeof(char*)) b->out[i] = static_cast<char*>(out[s].data) + byte;
      b->numel[i] = static_cast<uint32_t>(len) | (g.dtype == DORA_BF16 ? kBF16 : 0u);
      b->first[i] = b->chunks;
      b->chunks += static_cast<int32_t>((len + chunk - 1) / chunk);
      at.elements += len;
    }
    if (at.elements >= g.numel) at = {at.spans + 1, 0};
  }
}

// A launch's share of the pass's workgroups.
int launch_groups(int32_t chunks, int64_t all) {
  const int64_t share = (static_cast<int64_t>(chunks) * kMaxGroups + all - 1) / all;
  return static_cast<int>(std::min<int64_t>(chunks, share));
}

}  // namespace
}  // namespace dora

extern "C" size_t dora_grad_clip_workspace_size(int32_t n) {
  using namespace dora;
  if (n < 1 || n > kMaxSpans) return 0;
  // One sum a workgroup: kMaxGroups, and at most one more a launch.  A launch holds 248 tensors, or parts of
  // longer ones, of which kMaxTotal elements make 1024 more.
  const size_t launches = (static_cast<size_t>(n) + kMaxTotal / kPart) / InBlock::kSpans + 1;
  return ((kMaxGroups + launches) * sizeof(double) + 255) & ~size_t(255);
}

extern "C" int dora_grad_clip(const dora_span* grads, const dora_span* out, int32_t n, float max_norm, float eps,
                              float* norm_out, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace dora;
  if (!grads || !norm_out) return DORA_ERR_NULL;
  if (n < 1 || n > kMaxSpans || !(max_norm >= 0.0f) || !(eps >= 0.0f)) return DORA_ERR_SHAPE;
  int rc = check_spans(grads, n);
  if (rc != DORA_OK) return rc;
  const bool scale = out || max_norm != __builtin_inff();  // in place, no limit leaves nothing to write
  if (out) {
    rc = check_spans(out, n);
    if (rc != DORA_OK) return rc;
    for (int32_t i = 0; i < n; ++i)
      if (out[i].numel != grads[i].numel || out[i].dtype != grads[i].dtype) return DORA_ERR_SHAPE;
  }
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < dora_grad_clip_workspace_size(n))
    return DORA_ERR_WORKSPACE;
  const Extent norm_at(norm_out, sizeof(float)), ws(workspace, dora_grad_clip_workspace_size(n));
  bool shared = norm_at.meets(ws);
  for (const dora_span* s : {grads, out})
    for (int32_t i = 0; s && i < n; ++i) {
      const Extent t(s[i].data, span_bytes(s[i]));
      shared = shared || t.meets(norm_at) || t.meets(ws);
    }
  if (shared) return DORA_ERR_OVERLAP;
  if (scale) {
    Range* r = static_cast<Range*>(std::malloc(sizeof(Range) * 2 * static_cast<size_t>(n)));
    if (!r) return DORA_ERR_CAPACITY;
    const bool clash = ranges_clash(grads, out, n, r);
    std::free(r);
    if (clash) return DORA_ERR_OVERLAP;
  }
  double* parts = static_cast<double*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  int64_t total = 0, bytes = 0, all = 0;
  for (int32_t i = 0; i < n; ++i) {
    total += grads[i].numel;
    bytes += span_bytes(grads[i]);
  }
  const bool back = bytes > kWhole;
  if (total > kMaxTotal) return DORA_ERR_SHAPE;
  const int chunk = static_cast<int>(std::min<int64_t>(
      kMaxChunk, std::max<int64_t>(1, (total + kManyChunks * kMinChunk - 1) / (kManyChunks * kMinChunk)) * kMinChunk));
  for (int32_t i = 0; i < n; ++i) all += (grads[i].numel + chunk - 1) / chunk;
  int32_t used = 0;
  InBlock b;
  for (Place at{0, 0}; at.spans < n;) {
    if (back) fill_block<true>(grads, nullptr, n, at, chunk, &b);
    else fill_block<false>(grads, nullptr, n, at, chunk, &b);
    if (b.n == 0) continue;
    const int groups = launch_groups(b.chunks, all);
    if (back) hipLaunchKernelGGL(grad_squares_kernel<true>, dim3(groups), dim3(kThreads), 0, st, b, parts + used);
    else hipLaunchKernelGGL(grad_squares_kernel<false>, dim3(groups), dim3(kThreads), 0, st, b, parts + used);
    used += groups;
  }
  if (!scale || used == 0) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, parts, used, norm_out);
  } else {
    float* norm = norm_out;  // written by the first launch
    PairBlock pair;
    for (Place at{0, 0}; at.spans < n;) {
      if (out) {
        fill_block<false>(grads, out, n, at, chunk, &pair);
        if (pair.n == 0) continue;
        hipLaunchKernelGGL(grad_scale_kernel<PairBlock>, dim3(launch_groups(pair.chunks, all)), dim3(kThreads), 0, st,
                           pair, parts, used, max_norm, eps, norm);
      } else {
        fill_block<false>(grads, out, n, at, chunk, &b);
        if (b.n == 0) continue;
        hipLaunchKernelGGL(grad_scale_kernel<InBlock>, dim3(launch_groups(b.chunks, all)), dim3(kThreads), 0, st, b,
                           parts, used, max_norm, eps, norm);
      }
      norm = nullptr;
    }
  }
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
