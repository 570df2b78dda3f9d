// Prints how the attention over a 4-bit cache is cut up, for lines of
// "n_seqs n_rows max_rows heads kv_heads pages": column tiles, pages side by side, waves, splits.
#include <cstdio>

#include "kv4_plan.h"

int main() {
  hh::Kv4Sizes z;
  while (std::scanf("%d %d %d %d %d %d", &z.n_seqs, &z.n_rows, &z.max_rows, &z.hq, &z.hkv, &z.pages) == 6) {
    const hh::Kv4Plan p = hh::kv4_plan(z);
    std::printf("%d %d %d %d\n", p.nq, p.nq == 1 && p.packed ? 1 : 0, p.waves, p.splits);
  }
}
