// Global norm of many gradient tensors, and clipping by it.  DORA (arXiv
// 2609.34325), App. D: the actor's gradients are clipped at a global norm.
//
//   norm = sqrt(sum over tensors and elements of g^2)
//   c = min(1, max_norm / (norm + eps)),  out = c g
//
// HBM bound: one read for the norm, one read and write to scale (what the
// caches still hold of the first read is not read again).  The tensors'
// addresses go in by kernel argument, kSpans at a launch; a chunk of
// kChunk elements belongs to one tensor, and a workgroup takes every
// gridDim-th chunk.  Squares are added in 64 bits: no fp32 gradient overflows
// them, and the sum does not hang on the split.  Workgroups write their sums
// to the workspace; every workgroup of the scaling launch adds them all in
// the same order.
#include <algorithm>
#include <cstdlib>

#include "dora_internal.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr int kSpans = 96;         // tensors per launch: the argument block stays under 4 KB
constexpr int kChunk = 16384;      // elements
constexpr int kMaxGroups = 1024;   // workgroups of a launch
constexpr int kMaxSpans = 1 << 16;

struct SpanBlock {
  const char* in[kSpans];
  char* out[kSpans];
  int64_t numel[kSpans];
  int64_t first[kSpans];  // chunks before the tensor, in this launch
  uint64_t bf16[(kSpans + 63) / 64];
  int64_t chunks;
  int32_t n;
};
static_assert(sizeof(SpanBlock) + 64 <= 4096, "kernel arguments");

__device__ __forceinline__ int find_span(const SpanBlock& b, int64_t chunk) {
  int lo = 0, hi = b.n - 1;  // the last tensor that starts at or before the chunk
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (b.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

template <bool BF16>
__device__ __forceinline__ float element(const char* p, int64_t i) {
  if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[i]) << 16);
  else return reinterpret_cast<const float*>(p)[i];
}

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
__device__ __forceinline__ double chunk_squares(const char* p, int64_t lo, int64_t hi) {
  double s = 0.0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const double g = element<BF16>(p, i);
    s += g * g;
  }
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_squares_kernel(SpanBlock b, double* parts) {
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < b.chunks; c += gridDim.x) {
    const int t = find_span(b, c);
    const int64_t lo = (c - b.first[t]) * kChunk, hi = min(b.numel[t], lo + kChunk);
    s += (b.bf16[t / 64] >> (t % 64)) & 1 ? chunk_squares<true>(b.in[t], lo, hi)
                                          : chunk_squares<false>(b.in[t], lo, hi);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* parts, int32_t n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += parts[i];
  return sqrt(block_sum(s));
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* parts, int32_t n, float* norm) {
  const double v = norm_of(parts, n);
  if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

// The factor as a product: a factor below 2^-64 (gradients near fp32's limit)
// would itself be subnormal in fp32 and short of bits.
struct Factor {
  float pre, c;
  __device__ explicit Factor(double f) {
    const bool tiny = f < 0x1p-64;
    pre = tiny ? 0x1p-64f : 1.0f;
    c = static_cast<float>(tiny ? f * 0x1p64 : f);
  }
  __device__ float operator*(float g) const { return g * pre * c; }
};

template <bool BF16>
__device__ __forceinline__ void chunk_scale(const char* in, char* out, int64_t lo, int64_t hi, Factor f) {
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const float g = f * element<BF16>(in, i);
    if constexpr (BF16) reinterpret_cast<__bf16*>(out)[i] = static_cast<__bf16>(g);
    else reinterpret_cast<float*>(out)[i] = g;
  }
}

__global__ __launch_bounds__(kThreads) void grad_scale_kernel(SpanBlock b, const double* parts, int32_t n,
                                                              float max_norm, float eps, float* norm_out) {
  const double norm = norm_of(parts, n);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = static_cast<float>(norm);
  const double ratio = norm == 0.0 ? 1.0 : static_cast<double>(max_norm) / (norm + static_cast<double>(eps));
  const Factor f(ratio >= 1.0 ? 1.0 : ratio);  // NaN stays
  for (int64_t i = blockIdx.x; i < b.chunks; i += gridDim.x) {
    const int t = find_span(b, i);
    if (f.pre * f.c == 1.0f && b.in[t] == b.out[t]) continue;  // in place and nothing to clip
    const int64_t lo = (i - b.first[t]) * kChunk, hi = min(b.numel[t], lo + kChunk);
    if ((b.bf16[t / 64] >> (t % 64)) & 1) chunk_scale<true>(b.in[t], b.out[t], lo, hi, f);
    else chunk_scale<false>(b.in[t], b.out[t], lo, hi, f);
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

// The next launch's tensors from span `at` on, empty ones left out; returns
// the span after them.
int32_t fill_block(const dora_span* grads, const dora_span* out, int32_t n, int32_t at, SpanBlock* b) {
  *b = SpanBlock{};
  for (; at < n && b->n < kSpans; ++at) {
    if (grads[at].numel == 0) continue;
    const int i = b->n++;
    b->in[i] = static_cast<const char*>(grads[at].data);
    b->out[i] = static_cast<char*>(out ? out[at].data : grads[at].data);
    b->numel[i] = grads[at].numel;
    b->first[i] = b->chunks;
    if (grads[at].dtype == DORA_BF16) b->bf16[i / 64] |= uint64_t{1} << (i % 64);
    b->chunks += (grads[at].numel + kChunk - 1) / kChunk;
  }
  return at;
}

int block_groups(const SpanBlock& b) { return static_cast<int>(std::min<int64_t>(b.chunks, kMaxGroups)); }

}  // namespace
}  // namespace dora

extern "C" size_t dora_grad_clip_workspace_size(int32_t n) {
  using namespace dora;
  if (n < 1 || n > kMaxSpans) return 0;
  return static_cast<size_t>((n + kSpans - 1) / kSpans) * kMaxGroups * sizeof(double);
}

extern "C" int dora_grad_clip(const dora_span* grads, const dora_span* out, int32_t n, float max_norm, float eps,
                              float* norm_out, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace dora;
  if (!grads || !norm_out) return DORA_ERR_NULL;
  if (n < 1 || n > kMaxSpans || !(max_norm >= 0.0f) || !(eps >= 0.0f)) return DORA_ERR_SHAPE;
  int rc = check_spans(grads, n);
  if (rc != DORA_OK) return rc;
  const bool scale = max_norm != __builtin_inff();
  if (out && scale) {
    rc = check_spans(out, n);
    if (rc != DORA_OK) return rc;
    for (int32_t i = 0; i < n; ++i)
      if (out[i].numel != grads[i].numel || out[i].dtype != grads[i].dtype) return DORA_ERR_SHAPE;
  }
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < dora_grad_clip_workspace_size(n))
    return DORA_ERR_WORKSPACE;
  if (scale) {
    Range* r = static_cast<Range*>(std::malloc(sizeof(Range) * 2 * static_cast<size_t>(n)));
    if (!r) return DORA_ERR_CAPACITY;
    const bool clash = ranges_clash(grads, out, n, r);
    std::free(r);
    if (clash) return DORA_ERR_OVERLAP;
  }
  double* parts = static_cast<double*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  int32_t used = 0;
  SpanBlock b;
  for (int32_t at = 0; at < n;) {
    at = fill_block(grads, out, n, at, &b);
    const int groups = block_groups(b);
    if (groups == 0) continue;
    hipLaunchKernelGGL(grad_squares_kernel, dim3(groups), dim3(kThreads), 0, st, b, parts + used);
    used += groups;
  }
  bool norm_written = false;
  for (int32_t at = 0; scale && at < n;) {
    at = fill_block(grads, out, n, at, &b);
    const int groups = block_groups(b);
    if (groups == 0) continue;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(groups), dim3(kThreads), 0, st, b, parts, used, max_norm, eps,
                       norm_written ? nullptr : norm_out);
    norm_written = true;
  }
  if (!norm_written) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, parts, used, norm_out);
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
