// Checks the feed-forward block's launch choices over many shapes: every part
// of a split product has a step of the sum and a place in the workspace.
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "../../paper_2609_21137_amd/csrc/cardan_ffn_plan.h"

using namespace cardan;

int main(int argc, char** argv) {
  std::mt19937 rng(7);
  auto log_uniform = [&](double lo, double hi) {
    return (int64_t)(lo * pow(hi / lo, std::uniform_real_distribution<double>(0, 1)(rng)));
  };
  const int n = argc > 1 ? atoi(argv[1]) : 1000;
  long failures = 0, splits = 0, tails = 0;
  for (int i = 0; i < n; ++i) {
    const int N = i % 50 == 0 ? 0 : (int)log_uniform(1, 4.0e6);
    const int E = i % 2 ? 1 : (int)log_uniform(1, 1024);
    const int H = 64 * (int)log_uniform(1, 512), I = 32 * (int)log_uniform(1, 1024);
    for (int kind = K_UP; kind <= K_DWD; ++kind)
      for (bool gated : {false, true})
        for (bool grouped : {false, true}) {
          if (E > 1 && !grouped) continue;
          const FfnProduct p = ffn_product((FfnKind)kind, N, E, H, I, gated, grouped);
          for (int cus : {304, 256, 1}) {
            const FfnChoice c = choose_ffn(p, cus);
            bool ok = c.tile >= 0 && c.tile < kFfnTileCount && c.split >= 1 && c.split <= kMaxSplit;
            if (ok && c.split > 1) {
              const FfnTile& T = kFfnTiles[c.tile];
              const int64_t most = ffn_tiles(p, T), rest = most - c.full;
              ok = !(p.grad && grouped) && c.split <= p.steps && rest > 0 && c.full >= 0 && (p.known || c.full == 0);
              ok = ok && (size_t)rest * c.split * T.bm * T.bn * 4 <= ffn_partial_bytes(N, H, I, gated);
              ++splits;
              tails += c.full > 0;
            }
            // a workspace for more rows holds a call over fewer
            ok = ok && ffn_partial_bytes(N, H, I, gated) <= ffn_partial_bytes(N + 1, H, I, gated);
            if (!ok && ++failures < 20)
              printf("N=%d E=%d H=%d I=%d kind=%d gated=%d: tile %d split %d full %ld\n", N, E, H, I, kind, gated, c.tile,
                     c.split, (long)c.full);
          }
        }
  }
  // quotients at and around multiples of the divisor, up to the largest dividend
  for (int i = 0; i < 20 * n; ++i) {
    const int64_t d = i < 300 ? i + 1 : log_uniform(1, 1.0e9);
    const Divisor D(d);
    const int64_t most = 0x7fffffff / d;
    for (int64_t q : {(int64_t)0, most, most / 2, log_uniform(1, (double)most + 1.5) - 1})
      for (int64_t off : {-1, 0, 1}) {
        const int64_t v = q * d + off;
        if (v < 0 || v > 0x7fffffff) continue;
        if (D.quotient((int)v) != v / d && ++failures < 20) printf("%ld / %ld\n", (long)v, (long)d);
        if (d < 8 && v * d < 0x100000000ll && small_quotient((int)v, inverse_of((uint32_t)d)) != v / d && ++failures < 20)
          printf("small %ld / %ld\n", (long)v, (long)d);
      }
  }
  printf("%ld split products, %ld of them in a last round, %ld failures\n", splits, tails, failures);
  return failures != 0 || splits == 0 || tails == 0;
}
