// Launch planning of the feed-forward block (host only): the tile of a product
// and the number of parts that its sum is split into.
#ifndef CARDAN_FFN_PLAN_H
#define CARDAN_FFN_PLAN_H

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace cardan {

#ifdef __HIPCC__
#define CARDAN_HD __host__ __device__
#else
#define CARDAN_HD
#endif

// Division of 0 <= n < 2^31 by a constant of the launch: with l = ceil(log2 d)
// and m = floor(2^(31 + l) / d) + 1, n m / 2^(31 + l) exceeds n / d by less than
// 1 / d. (The compiler's division takes two dozen vector instructions.)
struct Divisor {
  uint32_t d, m, shift;
  Divisor() = default;
  explicit Divisor(int64_t by) : d((uint32_t)by), m(0), shift(0) {
    int l = 0;
    while (((int64_t)1 << l) < by) ++l;
    if (l > 0) {
      m = (uint32_t)((((uint64_t)1 << (31 + l)) / d) + 1);
      shift = l - 1;
    }
  }
  CARDAN_HD int quotient(int n) const { return d == 1 ? n : (int)((uint32_t)((uint64_t)(uint32_t)n * m >> 32) >> shift); }
};

// Division of n by a small d of the kernel, n d < 2^32: inv = ceil(2^32 / d), 0 for 1.
CARDAN_HD inline uint32_t inverse_of(uint32_t d) { return d > 1 ? 0xffffffffu / d + 1 : 0; }
CARDAN_HD inline int small_quotient(int n, uint32_t inv) {
  return inv ? (int)((uint64_t)(uint32_t)n * inv >> 32) : n;
}

// The products of the block. "rows" are the rows of a group (tokens).
enum FfnKind {
  K_UP = 0,    // [rows, H] x [H, I] (gate and up): activation -> h, and g, u where kept
  K_DOWN = 1,  // [rows, I] x [I, H] -> y
  K_DH = 2,    // [rows, H] x Wd^T -> dh, turned into dg, du
  K_DX = 3,    // dg Wg^T + du Wu^T -> dx
  K_DWI = 4,   // x^T dg and x^T du: the sum runs over the group's rows
  K_DWD = 5    // h^T dy, likewise
};

// The tiles of a product's last round, or all of them where they are few, are
// split over the sum into at most kMaxSplit parts, whose float32 partial
// outputs take at most this many bytes for N rows or fewer.
constexpr int kMaxSplit = 32;
constexpr size_t kPartialMax = (size_t)64 << 20;
inline size_t ffn_partial_bytes(int32_t N, int32_t H, int32_t I, bool gated) {
  const auto up = [](int64_t v) { return (size_t)((v + 255) / 256 * 256); };
  const size_t wide = std::max(up(H), up((gated ? 2 : 1) * (int64_t)I));
  return std::min(kPartialMax, (size_t)kMaxSplit * 4 * std::max(up(N) * wide, (gated ? 2 : 1) * up(H) * up(I)));
}

// Tiles (output rows x columns), their waves and stages of LDS, and the time of
// one step of 64 of the sum, measured with every CU busy: with as many workgroups
// on a CU as fit, and with one, where that differs. y = h Wd of 8192 rows, 4096 x
// 11008, runs at 1.32, 1.18, 0.89, 1.05, 0.69 and 0.36 PFLOP/s; over the four row
// products two tiles of 32 x 128 on a CU take 0.47 to 0.71 us a step and one alone
// 0.25 to 0.32, of 64 x 128 0.65 to 0.81 and 0.30 to 0.42.
struct FfnTile {
  int bm, bn, wm, wn, stages;
  double step_us, alone_us;
};
constexpr FfnTile kFfnTiles[] = {{256, 256, 2, 4, 2, 1.60, 1.60}, {128, 256, 2, 4, 3, 0.98, 0.98}, {64, 256, 1, 8, 3, 0.62, 0.62},
                                 {128, 128, 2, 2, 2, 1.06, 1.06}, {64, 128, 1, 4, 3, 0.78, 0.35}, {32, 128, 1, 4, 4, 0.61, 0.27}};
constexpr int kFfnTileCount = sizeof kFfnTiles / sizeof kFfnTiles[0];

// LDS of a workgroup, with the list of the row groups (of E > 0 of them) behind
// the stages, and the workgroups that a CU holds at once.
constexpr size_t kLdsBytes = 160 * 1024;
inline size_t ffn_list_bytes(int32_t E) { return (size_t)E * 12; }
inline size_t ffn_lds(const FfnTile& t, size_t list) { return (size_t)t.stages * (t.bm + t.bn) * 128 + list; }
inline int ffn_resident(const FfnTile& t, size_t list) {
  return (int)std::min<size_t>(kLdsBytes / ffn_lds(t, list), 8 / (t.wm * t.wn));
}

constexpr double kUnitUs = 3.8;         // a unit's setup and epilogue ...
constexpr double kUnitAreaUs = 4.0;     // ... plus this for 256 x 256 outputs
constexpr double kJoinUs = 3.5;         // a joining kernel
constexpr double kStreamBytesUs = 4.5e6;  // bytes per us that weights stream at

// One product: `rows` output rows in `groups` groups (weight gradients: the
// rows of one gradient, times `mats` matrices), `cols` columns, a sum of
// `steps` steps, `weight_bytes` read or written once whatever the tile.
struct FfnProduct {
  int64_t rows, groups, mats;
  int cols;
  bool dual;   // two products side by side in a tile (gate and up)
  bool grad;   // a weight gradient: every group has `rows` rows of its own
  bool known;  // the number of tiles is known on the host
  size_t list; // bytes of LDS that the list of the row groups takes
  int64_t steps;
  int max_split;
  size_t partial_bytes;
  double weight_bytes;
};

inline FfnProduct ffn_product(FfnKind kind, int32_t N, int32_t E, int32_t H, int32_t I, bool gated, bool grouped) {
  const bool grad = kind == K_DWI || kind == K_DWD;
  const bool over_h = kind == K_UP || kind == K_DH;  // the sum runs over H
  const int64_t active = std::max(1, std::min(E, N));
  FfnProduct p;
  p.dual = kind == K_UP && gated;
  p.grad = grad;
  p.known = grad || !grouped;
  p.list = p.known ? 0 : ffn_list_bytes(E);
  p.cols = over_h || kind == K_DWI ? I : H;
  p.groups = grad ? E : active;
  p.rows = kind == K_DWI ? H : kind == K_DWD ? I : N;
  p.mats = kind == K_DWI && gated ? 2 : 1;
  p.steps = grad ? (N / active + 63) / 64 : ((over_h ? H : I) + 63) / 64 * (kind == K_DX && gated ? 2 : 1);
  p.weight_bytes = (double)p.groups * H * I * 2 * (p.dual || p.mats == 2 || (kind == K_DX && gated) ? 2 : 1);
  p.partial_bytes = ffn_partial_bytes(N, H, I, gated);
  // every part has a step (the groups' rows, and so a gradient's steps, are not known here)
  p.max_split = grad && grouped ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(p.steps, kMaxSplit));
  return p;
}

// Tiles of a product, at most (groups end inside tiles).
inline int64_t ffn_tiles(const FfnProduct& p, const FfnTile& t) {
  const int bc = p.dual ? t.bn / 2 : t.bn;
  const int64_t cols = (p.cols + bc - 1) / bc, own = (p.rows + t.bm - 1) / t.bm;
  return cols * (p.grad ? own * p.groups * p.mats : p.known ? own : p.rows / t.bm + p.groups);
}

struct FfnChoice {
  int tile;
  int split;     // parts of each split tile; 1: none is split
  int64_t full;  // tiles before the split ones
};

// The tile and split of least estimated time: rounds of tiles over the chip's
// slots, each as long as its steps, against the time that the weights take to
// stream. The tiles of a last round that does not fill the slots are split
// (where their number is known; else all are, or none), which adds the joining
// kernel and the partial sums' bytes. Groups end inside tiles: half a tile of
// each is counted as lost.
inline FfnChoice choose_ffn(const FfnProduct& p, int cus) {
  FfnChoice best = {0, 1, 0};
  double best_us = 1e30;
  for (int t = 0; t < kFfnTileCount; ++t) {
    const FfnTile& T = kFfnTiles[t];
    const int bc = p.dual ? T.bn / 2 : T.bn;
    const int resident = ffn_resident(T, p.list);
    const double step_us = resident > 1 ? T.step_us : T.alone_us;
    const int64_t most = ffn_tiles(p, T), slots = (int64_t)cus * resident;
    const int64_t tiles = p.known ? most
                                  : (int64_t)(std::max((double)std::min(p.groups, p.rows), (double)p.rows / T.bm + 0.5 * p.groups) *
                                              ((p.cols + bc - 1) / bc));
    const double unit_us = kUnitUs + kUnitAreaUs * T.bm * T.bn / 65536.0;
    const double stream_us = p.weight_bytes / kStreamBytesUs;
    for (int s = 1; s <= p.max_split; s = s < 8 ? s + 1 : s * 2) {
      const int64_t full = s == 1 || !p.known ? 0 : tiles / slots * slots;
      const double bytes = (double)(most - full) * s * T.bm * T.bn * 4.0;
      if (s > 1 && (most == full || bytes > (double)p.partial_bytes)) continue;
      const int64_t rest = tiles - full;
      const double rounds = (double)(full / slots), last = (double)((rest * s + slots - 1) / slots);
      const double work = rounds * (step_us * (double)p.steps + unit_us) +
                          last * (step_us * (double)((p.steps + s - 1) / s) + unit_us);
      const double join = s == 1 ? 0.0 : kJoinUs + (double)rest * s * T.bm * T.bn * 4.0 / 4.0e6;
      const double us = std::max(work, stream_us) + 0.1 * std::min(work, stream_us) + join;
      if (us < best_us) {
        best_us = us;
        best = {t, s, full};
      }
    }
  }
  return best;
}

// Whether a forward pass takes the kernels for few rows: one launch a product,
// no join, but 2.5 TB/s of weights and less (one row, 2048 x 1408: 2.5 in the
// first product, 1.0 in the second) against the tiles' 4.8.
inline bool few_rows(int32_t N, int32_t H, int32_t I, bool grouped) {
  return !grouped && N <= 64 && (int64_t)H * I * ((N + 15) / 16) <= (6 << 20);
}

// Workgroups that share a column group's sum in such a pass over at most 16
// rows: as many as the chip's CUs allow, up to 8, and at least a step for every
// wave. Each of the second product's workgroups adds the parts of all of h and
// holds it in LDS. (One row through 2048 x 1408: the two products take 4.7 and
// 5.7 us with four parts, 9.4 and 5.8 without.)
inline int few_split(int32_t N, int32_t H, int32_t I, int cus) {
  if (N > 16 || (int64_t)N * I > 32768) return 1;
  int s = 1;
  while (s < 8 && (I + 31) / 32 * (2 * s) <= cus && H / 32 >= 16 * 2 * s) s *= 2;
  return s;
}

}  // namespace cardan

#endif  // CARDAN_FFN_PLAN_H
