// How the attention over a 4-bit cache (k_kv4.hip) is cut up.  Host code that
// needs sizes alone, so that it builds and is tested without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace hh {

constexpr int kMaxSplits = 64;
// Waves that a SIMD holds, by their registers.
constexpr int waves_fit(int nq) { return nq == 1 ? 4 : nq == 2 ? 3 : 2; }
// Workspace of s splits: 64 dimensions, base and sum of weights each.
inline size_t split_bytes(int s, int64_t outputs) { return (size_t)s * (size_t)outputs * (64 + 2) * sizeof(float); }
// Split outputs: as many splits as fit.  (300 rows of 32 heads over 8,192 pages would take
// ten splits, 25 MB, without a bound; where rows are many, there are workgroups enough.)
constexpr size_t kKv4Workspace = (size_t)16 << 20;

struct Kv4Sizes {
  int n_seqs, n_rows, max_rows;  // as in Kv4Rows
  int hq, hkv;
  int pages;  // a bound of the pages that a sequence holds
};

struct Kv4Plan {
  int nq;      // 16-column tiles of a workgroup
  bool packed; // two pages side by side in one tile
  int waves;   // of a workgroup
  int tiles;   // column tiles (workgroups) a sequence and kv head
  int splits;  // key splits over workgroups
  int64_t threads;   // of a sequence's larger grid
  size_t workspace;  // bytes
};

// Column tiles and waves of a workgroup and key splits over workgroups: those of
// the least time by what was measured, in ns (48 sizes, 32 query heads on 8, queries of
// one and of two terms; the choices cost 1.4% on average against the best ones, 16% at
// most).  A step (two pages) takes a wave that is alone on
// its SIMD 610 ns with one column tile, 700 with two and 1,250 with four, and 205, 285
// and 390 more for each neighbour there, of which there are up to three, two and one.
// What comes before and after is 3.5, 5.2 and 6.4 us, and 0.7, 0.25 and 0.4 more for each
// neighbour; the join 3 us, and its reads.  So (fp32, us) 8,192 prompt rows take four tiles
// (518; two 573, one 752), 1,200 two (23.8; four 25.7, one 28.9), 300 one (7.4; two 8.0, four
// 10.5), 8 sequences of 64 rows behind 1,000 positions two (22.8; one 25.2, four 26.7).
// One token at 700 positions is not split; at 3,000 it takes splits of four waves
// (8.0; one of eight waves 13.3), at 32,768 32 splits of eight (11.2; of four 11.4); 32
// tokens at 1,500 take eight waves (11.4; four 13.2), 128 at 1,000 four (20.2; eight 22.3),
// 100 at 300 four (10.9; eight 13.5).  Eight waves are for sequences of one tile.
struct Kv4Cut {
  int nq, waves, splits;
};
// Sizes here are far below 2^63.
inline double round_up(double x) {
  const double y = (double)(int64_t)x;
  return y < x ? y + 1 : y;
}
inline Kv4Cut kv4_cut(const Kv4Sizes& z) {
  struct Cost {
    int nq;
    double alone, more, ends, near;
  };
  constexpr Cost kCosts[] = {{1, 610, 205, 3500, 680}, {2, 700, 285, 5200, 250}, {4, 1250, 390, 6400, 400}};
  const int group = z.hq / z.hkv, pages = z.pages;
  const int64_t cols = (int64_t)z.max_rows * group, outputs = (int64_t)z.n_rows * z.hq;
  const double mean_cols = (double)z.n_rows * group / z.n_seqs;
  const int pairs = std::max(1, (pages + 1) / 2), most = std::max(1, std::min(kMaxSplits, pairs / 4));
  // Pairs that a tile attends to on average: a causal prompt's see half.
  const double mean_pairs = std::max(pages - z.max_rows / 32.0, pages / 2.0) / 2;
  const double even = 4 * mean_pairs / std::max(pages, 1) - 1;  // 1: all tiles alike, 0: from none to all
  Kv4Cut best{};
  double best_ns = 0;
  for (const Cost& c : kCosts) {
    if (c.nq > 1 && cols <= 8 * c.nq) break;  // half of its columns would be none
    const double seqs = (double)z.n_seqs * z.hkv * std::max(1.0, round_up(mean_cols / (16 * c.nq)));
    const int fit = waves_fit(c.nq);
    for (int w = 4; w <= (cols <= 16 ? 8 : 4); w += 4) {
      // (Every number up to 16, then less dense: this runs at each call.)
      for (int s = 1; s <= most && (s == 1 || split_bytes(s, outputs) <= kKv4Workspace); s += s < 16 ? 1 : s < 32 ? 2 : 4) {
        const int per = (pairs + s - 1) / s, steps = (per + w - 1) / w;
        const double here = std::max(1.0, seqs * s / 256);          // workgroups a CU gets
        const double load = here * w / 4, held = std::min<double>(fit, round_up(load));  // waves a SIMD, and at once
        const double busy = std::min<double>(fit, std::max(1.0, round_up(load * std::min(w, per) / w)));  // with keys
        auto step = [&](double waves) { return c.alone + c.more * (waves - 1); };
        // A wave's steps are the longest one's at least.  More waves than fit come in
        // turns, which end together where all have as many keys, and even out in a prompt.
        double each = load > held ? step(held) * load / held : step(busy);
        if (load > fit) {
          const double turns = (double)(int64_t)(round_up(here) * w / 4 / fit), rest = round_up(here) * w / 4 - turns * fit;
          each += even * std::max(0.0, turns * step(fit) + (rest > 0 ? step(rest) : 0) - each);
        }
        double ns = c.ends + c.near * (held - 1) + 0.75 * c.ends * std::max(0.0, load / fit - 1) +
                    std::max(step(busy) * steps, each * std::max(1.0, mean_pairs / s / w));
        if (w > 4 && load <= fit) ns -= s == 1 ? 650 : 200;  // (their waves start and end together)
        if (s > 1) ns += 3000 + 0.12 * (double)outputs * s;
        if (best.nq == 0 || ns < best_ns) {
          best = Kv4Cut{c.nq, w, s};
          best_ns = ns;
        }
      }
    }
  }
  return best;
}

inline Kv4Plan kv4_plan(const Kv4Sizes& z) {
  Kv4Plan p;
  const Kv4Cut c = kv4_cut(z);
  const int64_t cols = (int64_t)z.max_rows * (z.hq / z.hkv), outputs = (int64_t)z.n_rows * z.hq;
  p.nq = c.nq;
  p.waves = c.waves;
  p.splits = c.splits;
  p.packed = cols <= 8;
  const int64_t tiles = (cols + 16 * p.nq - 1) / (16 * p.nq);
  p.tiles = (int)std::min<int64_t>(tiles, INT32_MAX);
  // (Columns, and the elements of a row, are counted in 32 bits.)
  p.threads = cols > INT32_MAX - 1024 || z.hq >= 1 << 25 ? INT64_MAX : tiles * z.hkv * p.splits * 64 * p.waves;
  if (p.splits > 1) p.threads = std::max(p.threads, (int64_t)z.max_rows * z.hq * 256);
  p.workspace = p.splits > 1 ? split_bytes(p.splits, outputs) : 0;
  return p;
}

}  // namespace hh
