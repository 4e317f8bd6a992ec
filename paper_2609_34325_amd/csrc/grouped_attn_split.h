// Grouped attention on the host: sizes that are taken, how many workgroups there
// are, how keys are split, and the workspace that any call of these sizes needs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "dora.h"

namespace dora {
namespace {

constexpr int kTile = 64;  // rows (keys in grad_kv) of a workgroup, 16 a wave

struct Sizes {
  int32_t B, H, Hk, D, max_q;
  int64_t total_q, total_k;
};

constexpr int64_t kMaxRows = 0x7FFF0000;  // a tile's steps past the last row stay in 32 bits
inline bool good_sizes(const Sizes& z) {
  return z.B >= 1 && z.B <= DORA_MAX_SEQUENCES && z.H >= 1 && z.H <= 256 && z.Hk >= 1 && z.H % z.Hk == 0 &&
         (z.D == 32 || z.D == 64 || z.D == 128) && z.max_q >= 0 && z.total_q >= 0 && z.total_k >= 0 &&
         z.total_k <= kMaxRows && z.total_q <= kMaxRows && z.total_q * (z.H / z.Hk) <= kMaxRows;
}

inline int64_t tiles(int64_t total, int32_t B, int64_t tile) { return total / tile + B; }
// Sequences of about one to four tiles: the numbers that hold none are many (tile_number).
inline int32_t mix_tiles(int64_t total, int32_t B, int64_t tile) { return total / tile >= B / 2 && total / tile < int64_t{4} * B; }

// Workgroups of 64 rows that the GPU holds at a time, about.
constexpr int kFill = 512;

// How the forward pass splits its keys.
struct Split {
  int32_t splits, chunk, part_rows;
  int64_t blocks;  // without heads
};
// max_k: the longest sequence's keys; 0: not known; -1: as if it were long (for the workspace, which serves any).
inline Split forward_split(const Sizes& z, int32_t max_k) {
  const int32_t G = z.H / z.Hk;
  const int64_t rows = static_cast<int64_t>(std::min<int64_t>(z.max_q, z.total_q)) * G;
  const int64_t n = tiles(z.total_q * G, z.B, kTile);
  if (rows <= kTile && z.total_k > 0) {
    // Every sequence is one tile: parts of the same number of keys, as many as fill the GPU once, 128 keys or more and at
    // most 32 a sequence, by the average.  A part's 64 keys take 1.3 us one after another, the parts' join 4 to 5: whole
    // sequences where the longest is short, 64 of 400 keys and 8 key heads of 128 25 us whole and 35 split, one of 512 12.5
    // in two parts and 10 in four.  Where the longest is not known, any one may have all the keys: whole only where those are few
    // tiles.  (One list of 60000 among 500 of one key, 8 key heads of 128: 1268 us whole, 86 in parts; 100 of 100 keys 17 and
    // 19; 64 of 120, 12 of 64, 7.4 and 12.8, the call's own launches: a caller who knows the longest has them whole.)
    const int64_t keys = z.total_k / z.B, want = std::max(z.total_k * z.Hk / kFill, keys / 32);
    const int64_t chunk = std::min<int64_t>(4096, std::max<int64_t>(128, (want + 63) / 64 * 64));
    const bool whole = max_k > 0 ? max_k <= std::max<int64_t>(chunk, 256) : max_k == 0 && z.total_k <= 1024;
    // The workspace is sized for these parts: whole sequences are not cut again below, where a part keeps kTile rows.
    if (whole) return Split{1, 0, kTile, n};
    return Split{1, static_cast<int32_t>(chunk), static_cast<int32_t>(rows), tiles(z.total_k, z.B, chunk)};
  }
  const int64_t keys = z.total_k / z.B;
  int32_t splits = 1;
  while (splits < 16 && n * z.Hk * splits < kFill && keys / (splits * 2) >= 512) splits *= 2;
  return Split{splits, 0, kTile, n * splits};
}

inline int32_t backward_splits(const Sizes& z) {
  const int64_t n = tiles(z.total_k, z.B, kTile) * z.Hk, rows = z.total_q / z.B * (z.H / z.Hk);
  int32_t splits = 1;
  while (splits < 16 && n * splits < kFill && rows / (splits * 2) >= 512) splits *= 2;
  return splits;
}

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

inline size_t forward_bytes(const Sizes& z) {
  const Split p = forward_split(z, -1);
  if (p.splits == 1 && !p.chunk) return 256;
  // 0 is for sizes out of range: no queries have parts of no rows
  return std::max<size_t>(256, round256(static_cast<size_t>(p.blocks) * z.Hk * p.part_rows * (z.D + 2) * sizeof(float)));
}
inline size_t stat_bytes(const Sizes& z) { return round256(static_cast<size_t>(z.total_q) * z.H * sizeof(float2)); }
inline size_t backward_bytes(const Sizes& z) {
  const int32_t splits = backward_splits(z);
  return stat_bytes(z) + 256 +
         (splits == 1 ? 0 : round256(static_cast<size_t>(splits) * z.Hk * z.total_k * 2 * z.D * sizeof(float)));
}

}  // namespace
}  // namespace dora
