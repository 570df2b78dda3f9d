// Prints how calls on an 8-bit cache are cut up, for lines of
// "l n_seqs n_rows max_rows heads kv_heads pages blocks": waves, splits, tiles, workspace, threads of the
// attention over listed blocks; and
// "s n_seqs n_rows max_rows heads kv_heads pages 0": rows, waves, scores a thread, team, chunks, LDS bytes,
// workspace, threads of a selection.
#include <cstdio>

#include "kv8_plan.h"

int main() {
  hh::Kv4Sizes z;
  char what;
  int n;
  while (std::scanf(" %c %d %d %d %d %d %d %d", &what, &z.n_seqs, &z.n_rows, &z.max_rows, &z.hq, &z.hkv, &z.pages, &n) == 8) {
    if (what == 'l') {
      const hh::Kv8ListPlan p = hh::kv8_list_plan(z, n);
      std::printf("%d %d %d %zu %lld\n", p.waves, p.splits, p.tiles, p.workspace, (long long)p.threads);
    } else {
      const hh::Kv8SelectPlan p = hh::kv8_select_plan(z);
      std::printf("%d %d %d %d %d %zu %zu %lld\n", p.rows, p.waves, p.keys, (int)p.team, p.chunks, p.lds, p.workspace,
                  (long long)p.threads);
    }
  }
}
