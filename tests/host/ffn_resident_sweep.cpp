// Workgroups of the feed-forward block's tiles that a CU holds at once: the
// number that the launch choices are made with against a count from the sizes of
// a workgroup's LDS. Tiles over grouped rows have the list of the groups there too.
#include <stdio.h>

#include "../../paper_2609_21137_amd/csrc/cardan_ffn_plan.h"

using namespace cardan;

int main() {
  long failures = 0, fewer = 0;
  for (int E = 0; E <= 1024; ++E)
    for (int t = 0; t < kFfnTileCount; ++t) {
      const FfnTile& T = kFfnTiles[t];
      const long bytes = (long)T.stages * (T.bm + T.bn) * 64 * 2 + 12 * E, waves = T.wm * T.wn;
      long fit = 0;
      while ((fit + 1) * bytes <= 160 * 1024 && (fit + 1) * waves <= 8) ++fit;
      if (fit < 1 || fit != ffn_resident(T, ffn_list_bytes(E))) {
        ++failures;
        printf("E=%d tile %d: %ld fit, counted %d\n", E, t, fit, ffn_resident(T, ffn_list_bytes(E)));
      }
      fewer += E > 0 && fit < ffn_resident(T, 0);
    }
  // the products whose rows are grouped have the list, the others not
  for (int kind = K_UP; kind <= K_DWD; ++kind)
    for (bool grouped : {false, true}) {
      const FfnProduct p = ffn_product((FfnKind)kind, 64, 8, 2048, 768, true, grouped);
      const bool rows = kind != K_DWI && kind != K_DWD;
      if (p.list != (grouped && rows ? 96u : 0u)) {
        ++failures;
        printf("kind %d grouped %d: list of %zu bytes\n", kind, grouped, p.list);
      }
    }
  printf("%ld failures, %ld tiles with fewer workgroups beside a list\n", failures, fewer);
  return failures || !fewer;
}
