// How the calls on an 8-bit cache (k_kv8.hip, k_kv8_select.hip) are cut up.  Host code
// that needs sizes alone, so that it builds and is tested without a GPU.
#pragma once

#include "kv4_plan.h"

namespace hh {

// The attention over all keys is cut up as the one over a 4-bit cache: what that one's
// times choose is within 3% of the best here too (12 sizes, one to 64 splits; us: 8,192 prompt rows
// four tiles 493, two 548, one 705; 1,200 two 24.9, four 27.1; 32 tokens at 4,000 eight waves and
// no split 27.2, two splits 31.4, four waves 34.0; one at 131,072 64 splits 30.0, 32 29.3).
typedef Kv4Plan Kv8Plan;
inline Kv8Plan kv8_plan(const Kv4Sizes& z) { return kv4_plan(z); }

// The attention over listed blocks: a workgroup has 16 columns of one row (the
// group's query heads), its waves take the list's pairs of blocks in turn.
struct Kv8ListPlan {
  int waves, splits;
  int tiles;          // workgroups a row and kv head
  int64_t threads;    // of a sequence's larger grid
  size_t workspace;   // bytes
};
// Waves of a workgroup and splits of a list over workgroups: those of the least time by
// what was measured, in ns (eight sizes, 32 and 64 query heads on 8, with one to eight waves and
// splits; the choices cost 2% on average against the best ones, 7% at most).  A step
// takes a wave alone on its SIMD 500 ns and 100 more for each neighbour, and the SIMD 455 of
// its own; a wave's start and end 730 of them.  So (us) 4,000 rows of 32 blocks take one
// wave (163; two 188, four 232, eight 371), 200 such rows one (16.7; two 17.3, eight 24.9), 32
// of 64 eight (10.3; one 19.6), and one of 128 eight waves and splits (8.0; no split 9.5).
struct Kv8ListCut {
  int waves, splits;
};
inline Kv8ListCut kv8_list_cut(int64_t items, int pairs, int64_t outputs) {
  Kv8ListCut best{};
  double best_ns = 0;
  for (int w = 1; w <= 8; w *= 2)
    for (int s = 1; s <= std::min(kMaxSplits, pairs) && (s == 1 || split_bytes(s, outputs) <= kKv4Workspace); s += s < 8 ? 1 : 4) {
      const int steps = ((pairs + s - 1) / s + w - 1) / w;
      const double load = (double)items * s * w / 1024, held = std::min(4.0, std::max(1.0, round_up(load)));
      double ns = std::max(3700 + steps * (500 + 100 * (held - 1)), 2500 + load * (730 + 455 * steps));
      if (s > 1) ns += 3340 + 0.093 * (double)outputs * s;
      if (best.waves == 0 || ns < best_ns) {
        best = Kv8ListCut{w, s};
        best_ns = ns;
      }
    }
  return best;
}
inline Kv8ListPlan kv8_list_plan(const Kv4Sizes& z, int n) {
  Kv8ListPlan p;
  const int group = z.hq / z.hkv;
  const int64_t outputs = (int64_t)z.n_rows * z.hq;
  p.tiles = (group + 15) / 16;
  const Kv8ListCut c = kv8_list_cut((int64_t)z.n_rows * z.hkv * p.tiles, (n + 1) / 2, outputs);
  p.waves = c.waves;
  p.splits = c.splits;
  p.threads = z.hq >= 1 << 25 || (int64_t)z.max_rows * group > INT32_MAX - 1024
                  ? INT64_MAX
                  : (int64_t)z.max_rows * p.tiles * z.hkv * p.splits * 64 * p.waves;
  if (p.splits > 1) p.threads = std::max(p.threads, (int64_t)z.max_rows * z.hq * 256);
  p.workspace = p.splits > 1 ? split_bytes(p.splits, outputs) : 0;
  return p;
}

// Selection: a workgroup has `rows` rows and one kv head.  A wave of it searches a row, with
// up to `keys` scores a lane, or (team) all of them search one: rows of more than 2,048 blocks.
// Measured, us:
//   rows of a workgroup, which share what they read: 4,000 rows of 437 blocks 16 rows 44, 8 54;
//   1,200 of 1,770 8 rows 62 (66 KiB of scores), 16 74, 4 92;
//   its waves: 4,000 rows 8 waves 44, 4 48, 16 56; 32 of 1,400 blocks 19 with any of them;
//   a launch of its own for the scores, which has workgroups enough where rows are few: one
//   row of 8,192 blocks 19.6, without 55; 8 of 2,600 21.7 and 35; but 32 of 3,500 50 and 33.6
//   (33.6 in most runs, 45 to 47 in others of the same code, for a reason not known);
//   waves of a team: 8,192 blocks 4 waves 19.6, 8 20.0, 16 26.7.
// All of this goes by the table's width, as if rows had that many blocks: the 4,000 rows of 437 take
// 73 us behind a table of 1,024 columns, 114 behind 2,048 and 458 behind 8,192; the 32 rows 22.
constexpr int kMaxSelectPages = 1 << 15;  // a row's scores fit LDS
struct Kv8SelectPlan {
  int rows, waves, keys;
  bool team;
  int chunks;        // of 256 blocks that score a row in a launch of their own; 0: one launch
  size_t lds;        // bytes of the scores
  int64_t threads;   // of a sequence's larger grid
  size_t workspace;  // bytes
};
// The most that a call asks for: 33 scores of each thread, of a team of 1,024 or of 8 waves.
constexpr size_t kMostTeamLds = (size_t)33 * 1024 * sizeof(unsigned), kMostRowsLds = (size_t)33 * 512 * sizeof(unsigned);
inline int kv8_score_pitch(int pages) { return (pages + 15) / 16 * 16; }
inline Kv8SelectPlan kv8_select_plan(const Kv4Sizes& z) {
  Kv8SelectPlan p;
  const int64_t items = (int64_t)z.n_rows * z.hkv;
  p.team = z.pages > 2048;
  p.rows = p.team ? 1 : std::min(z.max_rows, z.pages > 512 ? 8 : 16);
  p.waves = p.team ? (z.pages > 8192 ? 16 : 4) : 8;
  p.chunks = p.team && items <= 128 ? (z.pages + 255) / 256 : 0;
  const int most = p.team ? 64 * p.waves : 64, each = ((z.pages + most - 1) / most) | 1;
  p.keys = !p.team && each <= 9 ? 9 : !p.team && each <= 17 ? 17 : 33;
  p.lds = (size_t)p.rows * each * most * sizeof(unsigned);
  p.threads = ((int64_t)z.max_rows + p.rows - 1) / p.rows * z.hkv * std::max(64 * p.waves, 256 * p.chunks);
  p.workspace = p.chunks > 0 ? (size_t)items * kv8_score_pitch(z.pages) * sizeof(unsigned) : 0;
  return p;
}

}  // namespace hh
