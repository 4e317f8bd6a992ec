// Descriptions of packed rows (dora_rows) as the kernels take them, and which of
// them share memory.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dora.h"
#include "policy_terms.h"

namespace dora {

inline int elem_bytes(int dtype) { return dtype == DORA_BF16 ? 2 : 4; }

// Address of the first element and strides in bytes.
struct RowView {
  char* at;
  int64_t row, head;
};

inline RowView row_view(const dora_rows* t) {
  if (!t) return RowView{nullptr, 0, 0};
  const int64_t e = elem_bytes(t->dtype);
  return RowView{static_cast<char*>(t->data), t->row_stride * e, t->head_stride * e};
}

// A description that can be read: sizes, strides (0 allowed, negative not) and
// alignment to `align` bytes of the address and of every stride in use.
inline int check_rows(const dora_rows* t, int align) {
  if (t->dtype != DORA_BF16 && t->dtype != DORA_F32) return DORA_ERR_DTYPE;
  if (t->rows < 0 || t->rows > 0x7FFFFFFF || t->heads < 1 || t->dim < 1 || t->row_stride < 0 || t->head_stride < 0)
    return DORA_ERR_SHAPE;
  // far below 2^63 bytes from the first element to the last
  if (t->row_stride > (int64_t{1} << 40) || t->head_stride > (int64_t{1} << 40) ||
      t->rows * static_cast<double>(t->row_stride) + t->heads * static_cast<double>(t->head_stride) > 1e15)
    return DORA_ERR_SHAPE;
  if (t->rows == 0) return DORA_OK;
  if (!t->data) return DORA_ERR_NULL;
  const int64_t e = elem_bytes(t->dtype);
  if (reinterpret_cast<uintptr_t>(t->data) % align || (t->rows > 1 && t->row_stride * e % align) ||
      (t->heads > 1 && t->head_stride * e % align))
    return DORA_ERR_ALIGN;
  return DORA_OK;
}

// As an outer run of blocks `step` bytes apart, each an inner run of `pieces`
// pieces of `len` bytes, `gap` bytes apart; adjacent pieces are one.
struct Blocks {
  uintptr_t at;
  int64_t n, step, pieces, gap, len;
  int64_t block_bytes() const { return (pieces - 1) * gap + len; }
  int64_t bytes() const { return (n - 1) * step + block_bytes(); }
};

inline Blocks blocks_of(const dora_rows* t) {
  const int64_t e = elem_bytes(t->dtype);
  Blocks b{reinterpret_cast<uintptr_t>(t->data), t->rows, t->row_stride * e, t->heads, t->head_stride * e, t->dim * e};
  if (b.n > 1 && b.pieces > 1 && b.gap > b.step) {
    const Blocks o = b;
    b.n = o.pieces, b.step = o.gap, b.pieces = o.n, b.gap = o.step;
  }
  if (b.pieces > 1 && b.gap == b.len) b.len *= b.pieces, b.pieces = 1;
  if (b.pieces == 1) b.gap = 0;
  if (b.n == 1) b.step = 0;
  return b;
}

// An output's elements lie apart from each other.
inline bool meets_itself(const dora_rows* t) {
  if (!t || t->rows == 0) return false;
  const Blocks b = blocks_of(t);
  return (b.pieces > 1 && b.gap < b.len) || (b.n > 1 && b.step < b.block_bytes());
}

// The same memory with what is read again and again (strides of 0) once.
inline Blocks blocks_read(const dora_rows* t) {
  Blocks b = blocks_of(t);
  if (b.step == 0) b.n = 1;
  if (b.gap == 0) b.pieces = 1;
  return b;
}

// Some x = p gap, 0 <= p < n, lies in (lo, hi).
inline bool step_between(int64_t n, int64_t gap, int64_t lo, int64_t hi) {
  if (hi <= 0 || lo >= (n - 1) * gap || hi - lo < 2) return false;
  if (lo < 0) return true;  // x = 0
  return gap > 0 && (lo / gap + 1) * gap < hi;
}

// Two tensors share memory.  Tensors whose rows and heads lie between each other's
// (slices of one product) need one and the same distance between the outer of the
// two to be told apart; with different ones they count as sharing.
inline bool rows_meet(const dora_rows* s, const dora_rows* t) {
  if (!s || !t || s->rows == 0 || t->rows == 0) return false;
  Blocks a = blocks_read(s), b = blocks_read(t);
  if (!Extent(reinterpret_cast<void*>(a.at), static_cast<size_t>(a.bytes()))
           .meets(Extent(reinterpret_cast<void*>(b.at), static_cast<size_t>(b.bytes()))))
    return false;
  // Blocks of one piece each are the pieces of one block as well.
  if (a.step != b.step && a.pieces == 1 && (b.pieces > 1 || a.n >= b.n)) a = Blocks{a.at, 1, 0, a.n, a.step, a.len};
  else if (a.step != b.step && b.pieces == 1) b = Blocks{b.at, 1, 0, b.n, b.step, b.len};
  if (a.n == 1) a.step = b.step;
  if (b.n == 1) b.step = a.step;
  if (a.n == 1 && b.n == 1) a.step = b.step = a.block_bytes() + b.block_bytes();
  if (a.step != b.step) return true;
  if (a.pieces == 1) a.gap = b.gap;
  if (b.pieces == 1) b.gap = a.gap;
  // Block r of b begins at shift + (r - q) step from block q of a.
  const int64_t shift = static_cast<int64_t>(b.at - a.at);
  int64_t lo = (-b.block_bytes() - shift) / a.step - 1, hi = (a.block_bytes() - shift) / a.step + 1;
  if (lo < -(a.n - 1)) lo = -(a.n - 1);
  if (hi > b.n - 1) hi = b.n - 1;
  const bool alike = a.gap == b.gap;  // then only the difference of two pieces' numbers counts
  if ((hi - lo + 1) * (alike ? 1 : a.pieces) > 4096) return true;
  for (int64_t k = lo; k <= hi; ++k) {
    const int64_t d = shift + k * a.step;  // b's block, from the start of a's
    if (alike) {
      // piece q of b meets piece p of a where -b.len < d + (q - p) gap < a.len
      const int64_t first = d - (a.pieces - 1) * a.gap;
      if (step_between(a.pieces + b.pieces - 1, a.gap, -b.len - first, a.len - first)) return true;
      continue;
    }
    for (int64_t p = 0; p < a.pieces; ++p)
      if (step_between(b.pieces, b.gap, p * a.gap - d - b.len, p * a.gap - d + a.len)) return true;
  }
  return false;
}

inline bool rows_meet(const dora_rows* s, Extent o) {
  if (!s || s->rows == 0 || !o.at || !o.bytes) return false;
  const Blocks a = blocks_read(s);
  if (!Extent(reinterpret_cast<void*>(a.at), static_cast<size_t>(a.bytes())).meets(o)) return false;
  // The vector against each run of the blocks that it could touch.
  const int64_t from = static_cast<int64_t>(o.at - a.at), to = from + static_cast<int64_t>(o.bytes);
  int64_t lo = a.n > 1 ? (from - a.block_bytes()) / a.step - 1 : 0, hi = a.n > 1 ? to / a.step + 1 : 0;
  if (lo < 0) lo = 0;
  if (hi > a.n - 1) hi = a.n - 1;
  if (hi - lo > 4096) return true;  // a vector that long holds whole blocks
  for (int64_t k = lo; k <= hi; ++k)
    if (step_between(a.pieces, a.gap, from - a.len - k * a.step, to - k * a.step)) return true;
  return false;
}

inline bool same_rows(const dora_rows* s, const dora_rows* t) {
  return s && t && s->data == t->data && s->rows == t->rows && s->heads == t->heads && s->dim == t->dim &&
         s->dtype == t->dtype && (s->rows <= 1 || s->row_stride == t->row_stride) &&
         (s->heads <= 1 || s->head_stride == t->head_stride);
}

// Outputs share memory with each other, with an input or with a vector; an
// output may be an input of `own` as a whole.
inline bool rows_clash(std::initializer_list<const dora_rows*> out, std::initializer_list<const dora_rows*> in,
                       std::initializer_list<const dora_rows*> own, std::initializer_list<Extent> out_vectors,
                       std::initializer_list<Extent> in_vectors) {
  for (auto o = out.begin(); o != out.end(); ++o) {
    if (meets_itself(*o)) return true;
    for (auto q = out.begin(); q != o; ++q)
      if (rows_meet(*o, *q)) return true;
    for (const dora_rows* i : in)
      if (rows_meet(*o, i)) return true;
    for (const dora_rows* i : own)
      if (!same_rows(*o, i) && rows_meet(*o, i)) return true;
    for (const Extent& v : out_vectors)
      if (rows_meet(*o, v)) return true;
    for (const Extent& v : in_vectors)
      if (rows_meet(*o, v)) return true;
  }
  for (const Extent& v : out_vectors) {
    for (const dora_rows* i : in)
      if (rows_meet(i, v)) return true;
    for (const dora_rows* i : own)
      if (rows_meet(i, v)) return true;
  }
  return outputs_clash(out_vectors, in_vectors, {});
}

}  // namespace dora
