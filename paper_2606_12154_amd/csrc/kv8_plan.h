// How the calls on an 8-bit cache (k_kv8.hip, k_kv8_select.hip) are cut up.  Host code
// that needs sizes alone, so that it builds and is tested without a GPU.
#pragma once

#include "kv4_plan.h"

namespace hh {

// The attention over all keys is cut up as the one over a 4-bit cache: a step of
// either takes the same products and exponentials.
typedef Kv4Plan Kv8Plan;
inline Kv8Plan kv8_plan(const Kv4Sizes& z) { return kv4_plan(z); }

// The attention over listed blocks: a workgroup has 16 columns of one row (the
// group's query heads), its waves take the list's pairs of blocks in turn.
struct Kv8ListPlan {
  int waves, splits;
  int tiles;          // workgroups a row and kv head
  bool packed;        // two blocks side by side in one tile
  int64_t threads;    // of a sequence's larger grid
  size_t workspace;   // bytes
};
inline Kv8ListPlan kv8_list_plan(const Kv4Sizes& z, int n) {
  Kv8ListPlan p;
  const int group = z.hq / z.hkv, pairs = (n + 1) / 2;
  const int64_t outputs = (int64_t)z.n_rows * z.hq;
  p.tiles = (group + 15) / 16;
  p.packed = group <= 8;
  const int64_t items = (int64_t)z.n_rows * z.hkv * p.tiles;
  p.waves = 4;
  p.splits = 1;
  while (items * p.splits < 512 && pairs / (2 * p.splits) >= 2 * p.waves && p.splits < kMaxSplits &&
         split_bytes(2 * p.splits, outputs) <= kKv4Workspace)
    p.splits *= 2;
  p.threads = z.hq >= 1 << 25 || (int64_t)z.max_rows * group > INT32_MAX - 1024
                  ? INT64_MAX
                  : (int64_t)z.max_rows * p.tiles * z.hkv * p.splits * 64 * p.waves;
  if (p.splits > 1) p.threads = std::max(p.threads, (int64_t)z.max_rows * z.hq * 256);
  p.workspace = p.splits > 1 ? split_bytes(p.splits, outputs) : 0;
  return p;
}

// Selection: `lanes` threads have a (row, kv head), `keys` scores each in registers.
constexpr int kMaxSelectPages = 1 << 16;
struct Kv8SelectPlan {
  int lanes, keys;
  int64_t threads;   // of a sequence's grid
  size_t workspace;  // bytes
};
inline Kv8SelectPlan kv8_select_plan(const Kv4Sizes& z) {
  Kv8SelectPlan p;
  const int64_t items = (int64_t)z.n_rows * z.hkv;
  p.lanes = z.pages > 4096 || items <= 512 ? 1024 : z.pages > 1024 || items <= 2048 ? 256 : 64;
  const int each = (z.pages + p.lanes - 1) / p.lanes;
  p.keys = each <= 4 ? 4 : each <= 16 ? 16 : 64;
  p.threads = (int64_t)z.max_rows * z.hkv * p.lanes;
  p.workspace = 0;
  return p;
}

}  // namespace hh
