// Rotary positions of packed query and key heads (dora_rope): pair i of a head
// turned by the angle t = position * freq[i],
//   u' = scale (u cos t - v sin t),  v' = scale (u sin t + v cos t)
//
// HBM bound: each element is read and written once.  A workgroup forms the
// cosines and sines of its rows once, in LDS, for all heads (the angle in 64
// bits, as a fraction of a turn, so that the fp32 sine and cosine see at most
// half a turn however far the position), while its first elements are already
// on their way.  A thread's unit is the two 16-byte pieces that hold its pairs'
// ends, or, with adjacent pairs, one piece.
//
// 32749 rows of 40 heads of 128, half of each turned, bf16: 119 us, 5.6 TB/s; 35295
// of 24 heads of 64, fp32: 84 us, 5.2 TB/s (a large copy runs at 4.9); 16 rows: 6 us,
// a launch and one chain of loads.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dora_internal.h"
#include "rows.h"

namespace dora {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 4;           // units a thread
constexpr int kTable = 2048;        // pairs of a workgroup's rows
constexpr int kMaxDim = 1024;

struct RopeArgs {
  RowView q, k, q_out, k_out;
  int32_t H, heads;  // heads of q; of q and k
  int64_t rows;
  int32_t D, R, axes;
  int32_t units;      // units of a head
  int32_t per_group;  // rows of a workgroup
  int32_t chunks;     // workgroups that share a group's rows
  const int32_t* pos;
  const double* freq;
  float sign, scale;
};

// VEC: pieces of 16 bytes; else single pairs and elements.
template <class E, bool ADJACENT, bool VEC>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  constexpr int kE = VEC ? 16 / sizeof(E) : 1;
  typedef std::conditional_t<VEC, u32x4, E> Piece;
  __shared__ float2 turn[kTable];
  const int half = a.R / 2;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x / a.chunks) * a.per_group;
  const int rows = static_cast<int>(min(static_cast<int64_t>(a.per_group), a.rows - row0));
  const int row_units = a.heads * a.units, total = rows * row_units;
  // Units of a head: its turned pieces first (with pairs half a head apart, two pieces a unit), then its copied ones.
  const int turned = ADJACENT ? (VEC ? a.R / kE : half) : half / kE;
  const char* from[kUnits];
  char* to[kUnits];
  int64_t second[kUnits];  // bytes to the pair's other end; 0: none
  int at[kUnits];          // first pair in the table; -1: copied; -2: nothing
  Piece x[kUnits], y[kUnits];
#pragma unroll
  for (int n = 0; n < kUnits; ++n) {
    const int id = (static_cast<int>(blockIdx.x % a.chunks) * kUnits + n) * kThreads + threadIdx.x;
    at[n] = -2;
    second[n] = 0;
    if (id >= total) continue;
    const int row = id / row_units, in_row = id - row * row_units, h = in_row / a.units, u = in_row - h * a.units;
    const bool is_q = h < a.H;
    const RowView in = is_q ? a.q : a.k, out = is_q ? a.q_out : a.k_out;
    const int64_t hh = is_q ? h : h - a.H, r = row0 + row;
    int elem, pair;
    if (u < turned) {
      elem = ADJACENT && !VEC ? 2 * u : u * kE;
      pair = ADJACENT ? elem / 2 : elem;
      second[n] = ADJACENT ? (VEC ? 0 : sizeof(E)) : static_cast<int64_t>(half) * sizeof(E);
      at[n] = row * half + pair;
    } else {
      elem = a.R + (u - turned) * kE;
      at[n] = -1;
    }
    from[n] = in.at + r * in.row + hh * in.head + elem * static_cast<int64_t>(sizeof(E));
    to[n] = out.at + r * out.row + hh * out.head + elem * static_cast<int64_t>(sizeof(E));
    x[n] = *reinterpret_cast<const Piece*>(from[n]);
    if (second[n]) y[n] = *reinterpret_cast<const Piece*>(from[n] + second[n]);
  }
  const int per_axis = half / a.axes;
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int row = i / half, pair = i - row * half;
    const double turns =
        static_cast<double>(a.pos[(row0 + row) * a.axes + pair / per_axis]) * a.freq[pair] * 0.15915494309189534561;
    float sn, cs;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &cs);
    turn[i] = make_float2(cs * a.scale, sn * a.sign * a.scale);
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kUnits; ++n) {
    if (at[n] == -2) continue;
    if (at[n] >= 0) {
      E* xe = reinterpret_cast<E*>(&x[n]);
      E* ye = reinterpret_cast<E*>(&y[n]);
      if (ADJACENT && VEC) {
#pragma unroll
        for (int i = 0; i < kE / 2; ++i) {
          const float2 t = turn[at[n] + i];
          const float u = static_cast<float>(xe[2 * i]), v = static_cast<float>(xe[2 * i + 1]);
          xe[2 * i] = static_cast<E>(__builtin_fmaf(u, t.x, -v * t.y));
          xe[2 * i + 1] = static_cast<E>(__builtin_fmaf(u, t.y, v * t.x));
        }
      } else {
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          const float2 t = turn[at[n] + i];
          const float u = static_cast<float>(xe[i]), v = static_cast<float>(ye[i]);
          xe[i] = static_cast<E>(__builtin_fmaf(u, t.x, -v * t.y));
          ye[i] = static_cast<E>(__builtin_fmaf(u, t.y, v * t.x));
        }
        *reinterpret_cast<Piece*>(to[n] + second[n]) = y[n];
      }
    }
    *reinterpret_cast<Piece*>(to[n]) = x[n];
  }
}

bool same_but_heads(const dora_rows* s, const dora_rows* t) {
  return s->rows == t->rows && s->dim == t->dim && s->dtype == t->dtype;
}

}  // namespace
}  // namespace dora

extern "C" int dora_rope(const dora_rows* q, const dora_rows* k, const int32_t* positions, int32_t axes,
                         const double* freq, int32_t R, int32_t interleaved, int32_t inverse, float scale,
                         const dora_rows* q_out, const dora_rows* k_out, void* stream) {
  using namespace dora;
  if (!q || !q_out || !freq || (k && !k_out)) return DORA_ERR_NULL;
  const dora_rows* in[2] = {q, k};
  const dora_rows* out[2] = {q_out, k ? k_out : nullptr};
  const int e = elem_bytes(q->dtype);
  bool pieces = true;  // of 16 bytes
  for (int i = 0; i < 2; ++i)
    for (const dora_rows* t : {in[i], out[i]})
      if (t) {
        const int rc = check_rows(t, e);
        if (rc != DORA_OK) return rc;
        pieces = pieces && check_rows(t, 16) == DORA_OK;
      }
  for (int i = 0; i < 2; ++i)
    if (in[i] && (!same_but_heads(in[i], q) || !same_but_heads(out[i], q) || in[i]->heads != out[i]->heads))
      return DORA_ERR_SHAPE;
  const int64_t heads = static_cast<int64_t>(q->heads) + (k ? k->heads : 0);
  if (axes < 1 || axes > 4 || R < 2 || R > q->dim || R % (2 * axes) || q->dim > kMaxDim || heads > 65535)
    return DORA_ERR_SHAPE;
  if (q->rows == 0) return DORA_OK;
  if (!positions) return DORA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(freq) % 8) return DORA_ERR_ALIGN;
  const Extent pos(positions, static_cast<size_t>(q->rows) * axes * sizeof(int32_t)),
      angles(freq, static_cast<size_t>(R / 2) * sizeof(double));
  for (int i = 0; i < 2; ++i)
    if (in[i] && (rows_clash({out[i]}, {in[1 - i]}, {in[i]}, {}, {pos, angles}) || rows_meet(out[i], out[1 - i])))
      return DORA_ERR_OVERLAP;
  const int n = 16 / e;
  pieces = pieces && q->dim % n == 0 && (interleaved ? R % n == 0 : R / 2 % n == 0);
  RopeArgs a{row_view(q), row_view(k), row_view(q_out), row_view(out[1]), q->heads, static_cast<int32_t>(heads), q->rows,
             q->dim, R, axes, 0, 1, 1, positions, freq, inverse ? -1.f : 1.f, scale};
  const int copied = q->dim - R;
  a.units = pieces ? (interleaved ? R : R / 2) / n + copied / n : R / 2 + copied;
  const int64_t row_units = static_cast<int64_t>(a.units) * heads, room = kThreads * kUnits;
  a.per_group = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(room / row_units, kTable / (R / 2))));
  a.chunks = static_cast<int32_t>((a.per_group * row_units + room - 1) / room);
  const int64_t blocks = (q->rows + a.per_group - 1) / a.per_group * a.chunks;
  if (blocks > (int64_t{1} << 32) / kThreads - 1) return DORA_ERR_UNSUPPORTED;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  };
  if (q->dtype == DORA_BF16) {
    if (interleaved) pieces ? launch(rope_kernel<__bf16, true, true>) : launch(rope_kernel<__bf16, true, false>);
    else pieces ? launch(rope_kernel<__bf16, false, true>) : launch(rope_kernel<__bf16, false, false>);
  } else {
    if (interleaved) pieces ? launch(rope_kernel<float, true, true>) : launch(rope_kernel<float, true, false>);
    else pieces ? launch(rope_kernel<float, false, true>) : launch(rope_kernel<float, false, false>);
  }
  return hipGetLastError() == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}
