// Routing of many rows: scores of E experts, the top k of each row, their
// weights, the rows' places in an array grouped by expert, and the gradient of
// the logits.
//
// Per row with logits z: score s_e = softmax(z)_e or sigmoid(z_e); the
// selection goes by v_e = s_e + bias_e in float64 where there is a bias, else by
// z_e, whose order is the scores'. Groups of E / G consecutive experts count by
// their best v, or by the sum of their best two (of scores); the top_k largest v
// of the kept groups, descending, ties to the lower index. weight_j = scale s_j, over the sum of the kept s if
// renormalised.
//
// A row is spread over LPR lanes of one wave, EPL consecutive experts a lane,
// so that the lowest lane with the largest value holds the lowest index. Bound
// by vector instructions and latency, not by memory: 65536 rows of 128 float32
// logits take 16 us, of which 8 are the read of 34 MB and the launch (4.2 TB/s);
// a wave's pass over 8 rows is about 660 vector instructions. With a bias and
// groups (8191 x 256) 14 us, 19 to 20 where there are a few rows whose groups
// float32 does not tell apart: their wave's float64 scores end the kernel. The places
// are a second launch of 6 to 9 us, most of it the length of its barriers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_rows.h"

namespace cardan {
namespace {

constexpr int kMostK = 32;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ double widen(double v) { return v; }
__device__ __forceinline__ void narrow(uint16_t& o, float v) { o = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void narrow(float& o, float v) { o = v; }
__device__ __forceinline__ void narrow(double& o, double v) { o = v; }

// Wide type of a logit's arithmetic: float, or double for float64 logits.
template <class L> struct Wide { typedef float type; };
template <> struct Wide<double> { typedef double type; };

template <int CTRL>
__device__ __forceinline__ int lane_move(int v) {
  return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __int_as_float(lane_move<CTRL>(__float_as_int(v)));
}
template <int CTRL>
__device__ __forceinline__ double lane_move(double v) {
  return __hiloint2double(lane_move<CTRL>(__double2hiint(v)), lane_move<CTRL>(__double2loint(v)));
}

// Reduction over the LPR lanes of a row; every lane gets the result, formed in
// the same order.
template <int LPR, class V, class F>
__device__ __forceinline__ V over_row(V v, F f) {
  v = f(v, lane_move<0xB1>(v));   // lane ^ 1
  v = f(v, lane_move<0x4E>(v));   // lane ^ 2
  v = f(v, lane_move<0x141>(v));  // the other half of 8
  if constexpr (LPR >= 16) v = f(v, lane_move<0x140>(v));  // the other half of 16
  if constexpr (LPR >= 32) v = f(v, __shfl_xor(v, 16));
  if constexpr (LPR == 64) v = f(v, __shfl_xor(v, 32));
  return v;
}
template <int LPR, class V>
__device__ __forceinline__ V row_max(V v) {
  return over_row<LPR>(v, [](V a, V b) { return a > b ? a : b; });
}
template <int LPR, class V>
__device__ __forceinline__ V row_sum(V v) {
  return over_row<LPR>(v, [](V a, V b) { return a + b; });
}
// The lanes of this lane's row whose flag is set, from bit 0.
template <int LPR>
__device__ __forceinline__ uint64_t row_ballot(bool f, int lane) {
  const uint64_t all = __ballot(f);
  return LPR == 64 ? all : all >> (lane & ~(LPR - 1)) & ((1ull << (LPR & 63)) - 1);
}

// Orders a wave's LDS accesses: its lanes read what others of them wrote.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// EPL consecutive values of a row from expert `e0` on; -infinity past the last.
template <int EPL, class L, class V>
__device__ __forceinline__ void load_row(const L* row, int e0, int E, bool wide, V (&z)[EPL]) {
  constexpr int kBytes = EPL * (int)sizeof(L), kPart = kBytes < 16 ? kBytes : 16, kEach = kPart / (int)sizeof(L);
  if (wide) {
#pragma unroll
    for (int i = 0; i < EPL; i += kEach) {
      struct alignas(kPart) Part { L v[kEach]; } p;
      if (e0 + i < E) p = *reinterpret_cast<const Part*>(row + e0 + i);
#pragma unroll
      for (int q = 0; q < kEach; ++q) z[i + q] = e0 + i < E ? (V)widen(p.v[q]) : (V)-INFINITY;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) z[i] = e0 + i < E ? (V)widen(row[e0 + i]) : (V)-INFINITY;
  }
}

template <int EPL, class L, class T>
__device__ __forceinline__ void store_row(L* row, int e0, int E, bool wide, const T* z) {
  constexpr int kBytes = EPL * (int)sizeof(L), kPart = kBytes < 16 ? kBytes : 16, kEach = kPart / (int)sizeof(L);
  if (wide) {
#pragma unroll
    for (int i = 0; i < EPL; i += kEach) {
      struct alignas(kPart) Part { L v[kEach]; } p;
#pragma unroll
      for (int q = 0; q < kEach; ++q) narrow(p.v[q], z[i + q]);
      if (e0 + i < E) *reinterpret_cast<Part*>(row + e0 + i) = p;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      L v;
      narrow(v, z[i]);
      if (e0 + i < E) row[e0 + i] = v;
    }
  }
}

template <class T> __device__ __forceinline__ T exp_of(T v);
template <> __device__ __forceinline__ float exp_of(float v) { return expf(v); }
template <> __device__ __forceinline__ double exp_of(double v) { return exp(v); }

// A logit as float32; a float64 one below float32's range is one all the same.
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(double v) {
  const float f = (float)v;
  return f == -INFINITY && v != -INFINITY ? -3.402823466e38f : f;
}

template <int EPL, class V>
__device__ __forceinline__ V local_max(const V (&v)[EPL]) {
  V m = v[0];
#pragma unroll
  for (int i = 1; i < EPL; ++i) m = v[i] > m ? v[i] : m;
  return m;
}

// Exponentials of a row's sum and of float32 scores: exp2 of one product is off
// by |v| 2^-24 of the result, as the difference v to the row's top is itself.
__device__ __forceinline__ float quick_exp(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896340736f); }
__device__ __forceinline__ double quick_exp(double v) { return exp(v); }

// Descending order of N = 4, 8 or 16 keys (odd-even merge).
template <int N>
__device__ __forceinline__ void sort_keys(uint32_t (&v)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j <= N - 1 - k; j += 2 * k)
#pragma unroll
        for (int i = 0; i <= (k - 1 < N - j - k - 1 ? k - 1 : N - j - k - 1); ++i)
          if ((i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const uint32_t a = v[i + j], b = v[i + j + k];
            v[i + j] = a > b ? a : b;
            v[i + j + k] = a > b ? b : a;
          }
}

// Order of float32 values as unsigned numbers; -infinity is below kNone, also
// with other low bits.
constexpr uint32_t kNone = 0x00800000u;
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v + 0.0f);  // (-0 is 0)
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// A row's part of LDS: the candidates' experts and keys, with groups their
// values and whether they are kept, and an area for one thing after another:
// staged values of the groups, the lanes' sorted keys, the values of the
// candidates or of all experts, the weights.
constexpr int kSpare = 2;  // candidates behind the selection
constexpr int kGroupBytes = 64 * (8 + 4);
struct RowLds {
  int* e;
  uint32_t* key;
  unsigned char *group, *area;
  __device__ __forceinline__ RowLds(unsigned char* lds, const RouteArgs& A) {
    e = reinterpret_cast<int*>(lds);
    key = reinterpret_cast<uint32_t*>(e + A.slots);
    group = lds + A.slots * 8;
    area = group + (A.groups > 1 ? kGroupBytes : 0);
  }
};
// A lane's sorted keys, apart from the next lane's by an odd number of 16 bytes.
template <int EPL>
constexpr int kListStep = EPL % 8 ? EPL : EPL + 4;
template <class V, int LPR, int EPL>
int row_bytes(const RouteArgs& A) {
  const int list = LPR * kListStep<EPL> * 4, values = LPR * EPL * (int)sizeof(V), more = A.slots * 8;
  return A.slots * 8 + (A.groups > 1 ? kGroupBytes : 0) + std::max(std::max(list, values), more);
}

// value[g], g < groups (LDS): which are kept. near(kept, x, g) for this lane's
// groups that are there.
template <int LPR, class V, class F>
__device__ __forceinline__ void rank_groups(const RouteArgs& A, int at, const V* value, int* keep, F near) {
  for (int grp = at; grp < A.groups; grp += LPR) {
    const V x = value[grp];
    int before = 0;
    for (int h = 0; h < A.groups; ++h) {
      const V o = value[h];
      before += o > x || (o == x && h < grp);
    }
    const bool there = x != (V)-INFINITY, in = there && before < A.top_groups;
    keep[grp] = in;
    if (there) near(in, x, grp);
  }
}
// What a group counts by from all[E] (LDS), as put(g, best, second best or 0):
// 2^group_split lanes a group (237 rows of 180 experts in two groups: 11.5 us,
// with one lane a group 17.8; 56 of 504 in four: 14.2 and 23.0).
template <int LPR, class V, class F>
__device__ __forceinline__ void value_groups(const RouteArgs& A, int at, const V* all, F put) {
  const int lg = A.group_split, sub = at & ((1 << lg) - 1);
  for (int first = 0; first < A.groups; first += LPR >> lg) {
    const int grp = first + (at >> lg);
    V b1 = (V)-INFINITY, b2 = (V)-INFINITY;
    if (grp < A.groups) {
#pragma unroll 4
      for (int i = sub; i < A.each; i += 1 << lg) {
        const V x = all[grp * A.each + i], lo = x < b1 ? x : b1;
        b1 = x > b1 ? x : b1;
        b2 = lo > b2 ? lo : b2;
      }
    }
    const auto join = [&](V o1, V o2) {
      const V lo = o1 < b1 ? o1 : b1, hi = o2 > b2 ? o2 : b2;
      b1 = o1 > b1 ? o1 : b1;
      b2 = lo > hi ? lo : hi;
    };
    if (lg > 0) join(lane_move<0xB1>(b1), lane_move<0xB1>(b2));
    if (lg > 1) join(lane_move<0x4E>(b1), lane_move<0x4E>(b2));
    if (lg > 2) join(lane_move<0x141>(b1), lane_move<0x141>(b2));
    if (lg > 3) join(lane_move<0x140>(b1), lane_move<0x140>(b2));
    if (sub == 0 && grp < A.groups) put(grp, b1, A.best == 2 && b2 != (V)-INFINITY ? b2 : (V)0);
  }
}

// The values that define the selection, logits or float64 scores with their
// bias, -infinity for NaN and what is not there, into all[E] (X.area).
template <class L, class V, int LPR, int EPL>
__device__ __forceinline__ void exact_values(const RouteArgs& A, bool scores, int at, const L* row, const RowLds& X) {
  const int lo = at * EPL;
  V* all = reinterpret_cast<V*>(X.area);
  V x[EPL], top = (V)-INFINITY, sum = 0;
  load_row<EPL>(row, lo, A.E, A.wide, x);
  if (sizeof(V) == 8 && scores) {
    if (!A.sigmoid) {
      top = row_max<LPR>(local_max(x));
      if (top == (V)-INFINITY) top = 0;
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) all[lo + i] = A.sigmoid ? -x[i] : x[i] - top;
    // (loops of few exponentials: the code of all of them at once would push the rest out of the caches)
#pragma unroll 4
    for (int i = 0; i < EPL; ++i) {
      const V e = exp_of(all[lo + i]);
      all[lo + i] = A.sigmoid ? (V)1 / ((V)1 + e) : e;
      sum += e;
    }
    sum = A.sigmoid ? (V)1 : row_sum<LPR>(sum);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const V s = all[lo + i] / sum + (A.bias && lo + i < A.E ? (V)A.bias[lo + i] : (V)0);
      all[lo + i] = x[i] == (V)-INFINITY || s != s ? (V)-INFINITY : s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) all[lo + i] = x[i] == x[i] ? x[i] : (V)-INFINITY;
  }
  wave_sync();
}

// Experts outside the kept groups leave the selection, by float32 values v
// whose scores are at most `margin` / 4 off; by the exact ones where that does
// not decide. A group's value is off by margin / 2 for its scores, by 2^-24 |v|
// for each of its best two (the bias was added to them) and 2^-24 of the sum;
// the end of that interval is rounded once more. All of these are relative to
// the sizes of the two, whose sum may be small where they cancel: 3 2^-24 of
// |best| + |second| and a little, each group's own.
template <class L, class V, int LPR, int EPL>
__device__ __forceinline__ void keep_groups(float (&v)[EPL], const RouteArgs& A, int at, const L* row, float margin,
                                            const RowLds& X) {
  float *value = reinterpret_cast<float*>(X.group), *off = value + 64;  // (exact values take the place of both)
  int* keep = reinterpret_cast<int*>(X.group + 64 * 8);
  const auto put = [&](int grp, float best, float second) {
    // (a group that is there stays above -infinity, also where float32 has no such sum)
    value[grp] = best == -INFINITY ? best : fmaxf(best + second, -3.402823466e38f);
    off[grp] = 0.5f * margin + (fabsf(best) + fabsf(second)) * 0x1.9p-23f;
  };
  const int lg = A.group_lanes;  // log2 of a group's lanes where it is made of whole ones, else -1
  if (lg >= 0) {
    float b1 = -INFINITY, b2 = -INFINITY;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      b2 = fmaxf(b2, fminf(b1, v[i]));
      b1 = fmaxf(b1, v[i]);
    }
    const auto join = [&](float o1, float o2) {
      b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
      b1 = fmaxf(b1, o1);
    };
    if (lg > 0) join(lane_move<0xB1>(b1), lane_move<0xB1>(b2));
    if (lg > 1) join(lane_move<0x4E>(b1), lane_move<0x4E>(b2));
    if (lg > 2) join(lane_move<0x141>(b1), lane_move<0x141>(b2));
    if (lg > 3) join(lane_move<0x140>(b1), lane_move<0x140>(b2));
    if ((at & ((1 << lg) - 1)) == 0 && at >> lg < A.groups) put(at >> lg, b1, A.best == 2 && b2 != -INFINITY ? b2 : 0.f);
  } else {
    float* all = reinterpret_cast<float*>(X.area);
#pragma unroll
    for (int i = 0; i < EPL; ++i) all[at * EPL + i] = v[i];
    wave_sync();
    value_groups<LPR>(A, at, all, put);
  }
  wave_sync();
  // the least that a kept group may be, the most that another one may be
  float least = INFINITY, most = -INFINITY;
  rank_groups<LPR>(A, at, value, keep, [&](bool in, float x, int grp) {
    const float o = off[grp];
    const float end = o < INFINITY ? (in ? x - o : x + o) : in ? -INFINITY : INFINITY;
    if (in) least = fminf(least, end);
    else most = fmaxf(most, end);
  });
  wave_sync();
  if (margin != 0.f) {
    least = -row_max<LPR>(-least);
    most = row_max<LPR>(most);
    if (!(most == -INFINITY || least > most)) {
      V* exact = reinterpret_cast<V*>(X.group);
      exact_values<L, V, LPR, EPL>(A, A.by_score, at, row, X);
      value_groups<LPR>(A, at, reinterpret_cast<V*>(X.area), [&](int grp, V best, V second) { exact[grp] = best + second; });
      wave_sync();
      rank_groups<LPR>(A, at, exact, keep, [](bool, V, int) {});
      wave_sync();
    }
  }
  if (lg >= 0) {
    const bool in = at >> lg < A.groups && keep[at >> lg];
#pragma unroll
    for (int i = 0; i < EPL; ++i) v[i] = in ? v[i] : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) v[i] = at * EPL + i < A.E && keep[A.by_each.quotient(at * EPL + i)] ? v[i] : -INFINITY;
  }
}

// The experts of a row in 32-bit keys: the upper bits of the value's order,
// below them the expert's place (LOGITS: of the row, so that all keys differ;
// else of the lane). The lanes' keys are sorted, each step takes the largest
// of the lanes' first ones: the selection and two behind it. Where neighbours
// among these are closer than what the keys tell apart (the bits cut off, and
// `margin` for values that are themselves rounded), all candidates are put in
// the order of their exact values; false if the last of them is that close to
// the selection's last, so that others may be, too. (A lane's keys come out of
// LDS one by one: shifted in registers they took a third of the kernel's
// instructions.)
template <class L, int LPR, int EPL, bool LOGITS, class F>
__device__ __forceinline__ bool select_keys(const float (&v)[EPL], const RouteArgs& A, int lane, const L* row, float margin,
                                            const RowLds& X, F ahead) {
  constexpr uint32_t kMask = (LOGITS ? LPR * EPL : EPL) - 1;
  const int at = lane & (LPR - 1);
  uint32_t key[EPL], low = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    if constexpr (LOGITS) low |= __float_as_uint(v[i]);
    key[i] = (ordered(v[i]) & ~kMask) | (kMask - (LOGITS ? at * EPL + i : i));
  }
  ahead();
  // logits whose low bits are all zero (bf16 ones) lose nothing in the keys
  bool whole = LOGITS && sizeof(L) == 2;
  if constexpr (LOGITS && sizeof(L) == 4) whole = row_ballot<LPR>((low & kMask) != 0, lane) == 0;
  sort_keys(key);
  // The keys behind the first one wait in LDS until the lane has had that. (All
  // lanes' keys are at least 64, those of what is not there among them: the
  // zero behind a lane's last one never is the largest.)
  uint32_t* list = reinterpret_cast<uint32_t*>(X.area) + at * kListStep<EPL>;
#pragma unroll
  for (int i = 0; i < EPL; i += 4)
    *reinterpret_cast<u32x4*>(list + i) = u32x4{key[i + 1], key[i + 2], key[i + 3], i + 4 < EPL ? key[i + 4 < EPL ? i + 4 : 0] : 0u};
  uint32_t head = key[0];
  const int total = LOGITS && sizeof(L) == 2 ? A.k : A.k + kSpare;
  for (int j = 0; j < total; ++j) {
    const uint32_t mine = LOGITS ? head : head & ~kMask;
    const uint32_t m = over_row<LPR>(mine, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    bool win = mine == m;
    if constexpr (!LOGITS) win = at == __ffsll((unsigned long long)row_ballot<LPR>(win, lane)) - 1;
    if (win) {
      X.key[j] = head;
      if constexpr (!LOGITS) X.e[j] = at;
      head = *list++;
    }
  }
  wave_sync();
  for (int j = at; j < total; j += LPR) {
    const uint32_t m = X.key[j];
    X.e[j] = m < kNone ? -1 : (LOGITS ? 0 : X.e[j] * EPL) + (int)(kMask - (m & kMask));
    X.key[j] = m & ~kMask;
  }
  wave_sync();
  if (whole) return true;
  const auto near = [&](uint32_t a, uint32_t b) {  // a >= b
    if (b < kNone) return false;
    if constexpr (LOGITS) return a == b;
    const float hi = from_ordered(a), lo = from_ordered(b);
    return !(hi - lo > margin + fabsf(lo) * (0x1p-22f * (float)(kMask + 1)) + 0x1p-120f);
  };
  bool close = false;
  for (int j = at; j < A.k; j += LPR) close |= near(X.key[j], X.key[j + 1]);
  if (row_ballot<LPR>(close, lane) == 0) return true;
  if (near(X.key[A.k - 1], X.key[total - 1])) return false;
  // the candidates' ranks: by logit and expert, or by float64 score and expert
  if constexpr (LOGITS) {
    uint64_t* value = reinterpret_cast<uint64_t*>(X.area);
    for (int j = at; j < total; j += LPR) {
      const int e = X.e[j];
      value[j] = e < 0 ? (uint64_t)(total - j) : (uint64_t)ordered((float)widen(row[e])) << 32 | (uint32_t)~e;
    }
    wave_sync();
    for (int j = at; j < total; j += LPR) {
      const uint64_t x = value[j];
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < total; ++i) before += value[i] > x;
      X.key[before] = (uint32_t)X.e[j];
    }
  } else {
    double *value = reinterpret_cast<double*>(X.area), top = 0, sum = 1;
    const bool scores = sizeof(L) < 8 || A.bias != nullptr;  // (float64 logits are rounded in v, too)
    if (scores && !A.sigmoid) {
      double z[EPL];
      load_row<EPL>(row, at * EPL, A.E, A.wide, z);
      top = row_max<LPR>(local_max(z));
#pragma unroll
      for (int i = 0; i < EPL; ++i) value[at * EPL + i] = z[i] - top;
      sum = 0;
#pragma unroll 4
      for (int i = 0; i < EPL; ++i) sum += exp_of(value[at * EPL + i]);
      sum = row_sum<LPR>(sum);
      wave_sync();
    }
    for (int j = at; j < total; j += LPR) {
      const int e = X.e[j];
      double x = e >= 0 ? (double)widen(row[e]) : -INFINITY;
      if (scores && e >= 0) {
        const double y = exp_of(A.sigmoid ? -x : x - top);
        x = (A.sigmoid ? 1.0 / (1.0 + y) : y / sum) + (A.bias ? (double)A.bias[e] : 0.0);
      }
      value[j] = x;
    }
    wave_sync();
    for (int j = at; j < total; j += LPR) {
      const double x = value[j];
      const int e = X.e[j];
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < total; ++i) before += value[i] > x || (value[i] == x && (X.e[i] < e || (X.e[i] == e && i < j)));
      X.key[before] = (uint32_t)e;
    }
  }
  wave_sync();
  for (int j = at; j < A.k; j += LPR) X.e[j] = (int)X.key[j];
  wave_sync();
  return true;
}

// The selection in the exact values, for rows that neither keys nor their
// candidates decide (several equal or nearly equal values at its end): loops
// over LDS, as it is rare. V is float for float32 logits alone.
template <class L, class V, int LPR, int EPL>
__device__ __forceinline__ void select_values(const RouteArgs& A, int lane, const L* row, const RowLds& X) {
  const int at = lane & (LPR - 1), lo = at * EPL, hi = lo + EPL < A.E ? lo + EPL : A.E;
  V* all = reinterpret_cast<V*>(X.area);
  exact_values<L, V, LPR, EPL>(A, A.bias != nullptr, at, row, X);
  if (A.groups > 1) {
    const int* keep = reinterpret_cast<const int*>(X.group + 64 * 8);
    for (int e = lo; e < hi; ++e)
      if (!keep[A.by_each.quotient(e)]) all[e] = (V)-INFINITY;
  }
  V last = (V)INFINITY;
  int last_e = -1;
  for (int j = 0; j < A.k; ++j) {
    V best = (V)-INFINITY;
    int be = -1;
#pragma unroll 4
    for (int e = lo; e < hi; ++e) {
      const V x = all[e];
      const bool left = x < last || (x == last && e > last_e);
      if (left && x > best) {
        best = x;
        be = e;
      }
    }
    last = row_max<LPR>(best);
    const int first = __ffsll((unsigned long long)row_ballot<LPR>(best == last, lane)) - 1;
    last_e = __shfl(be, (lane & ~(LPR - 1)) + first);
    if (at == first) X.e[j] = be;
  }
  wave_sync();
}

// The selection and the weights of row n, whose logits are z; X.e receives the
// experts. ahead() is called once z is used up: it fetches the next row's.
template <class L, class V, int LPR, int EPL, class F>
__device__ __forceinline__ void route_row(const RouteArgs& A, int n, int lane, const RowLds& X,
                                          const typename Wide<L>::type (&z)[EPL], F ahead) {
  typedef typename Wide<L>::type T;
  const int at = lane & (LPR - 1), e0 = at * EPL;
  const L* row = static_cast<const L*>(A.logits) + (int64_t)n * A.ld;
  // (float32 values: logits; float64 values of narrower logits: scores)
  const bool by_score = sizeof(V) == 8 && (sizeof(L) < 8 || A.by_score);
  T top = 0, sum = 1;
  bool bad = false;
  {
    float v[EPL];
    {
      if (!A.sigmoid && (by_score || !A.renorm)) {
        // the largest logit (0 if there is none) and the exponentials' sum relative to it
        top = row_max<LPR>(local_max(z));
        if (top == (T)-INFINITY) top = 0;
        sum = 0;
#pragma unroll
        for (int i = 0; i < EPL; ++i) sum += quick_exp(z[i] - top);
        sum = row_sum<LPR>(sum);
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) v[i] = to_float(z[i]);
      if (by_score) {
        // float32 scores: a sigmoid s is off by at most s (1 - s) (|z| + 2) 2^-24 for the exponential (below
        // 3/4 2^-24) and 3 2^-24 for sum and reciprocal, so two of them by less than 2^-21; a softmax, whose
        // largest is 1 / sum, by 2^-18 of that (the mean distance from the top that the sum weighs is below ln 1024)
        if (A.sigmoid) {
#pragma unroll
          for (int i = 0; i < EPL; ++i)
            v[i] = v[i] == -INFINITY ? v[i] : __builtin_amdgcn_rcpf(1.0f + quick_exp(-v[i]));
        } else {
          const float share = 1.0f / (float)sum;
#pragma unroll
          for (int i = 0; i < EPL; ++i) v[i] = v[i] == -INFINITY ? v[i] : quick_exp((float)(z[i] - top)) * share;
        }
        if (A.bias) {
#pragma unroll
          for (int i = 0; i < EPL; ++i) {  // (no bias makes an expert be there)
            const float b = e0 + i < A.E ? A.bias[e0 + i] : 0.f;
            v[i] = v[i] == -INFINITY ? v[i] : v[i] + b;
          }
        }
      }
    }
    float any = 0;  // NaN where a value is (or infinities of either sign are)
#pragma unroll
    for (int i = 0; i < EPL; ++i) any += v[i];
    if (row_ballot<LPR>(any != any, lane) != 0) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        bad |= v[i] != v[i];
        v[i] = v[i] != v[i] ? -INFINITY : v[i];
      }
      bad = row_ballot<LPR>(bad, lane) != 0;
    }
    const float least = sizeof(T) == 8 ? 0x1p-100f : 0.f;  // (float64 logits are rounded, too)
    const float margin = !by_score ? least : A.sigmoid ? 0x1p-21f : 0x1p-17f / (float)sum + 0x1p-22f;
    if (A.groups > 1) keep_groups<L, V, LPR>(v, A, at, row, 2.f * margin, X);
    bool decided;
    if (by_score && !A.bias) {  // scores were for the groups alone
#pragma unroll
      for (int i = 0; i < EPL; ++i) v[i] = v[i] == -INFINITY ? v[i] : to_float(z[i]);
    }
    if (sizeof(V) == 4 || (sizeof(L) < 8 && !A.bias)) decided = select_keys<L, LPR, EPL, sizeof(L) < 8>(v, A, lane, row, least, X, ahead);
    else decided = select_keys<L, LPR, EPL, false>(v, A, lane, row, A.bias ? margin : least, X, ahead);
    if (!decided) select_values<L, V, LPR, EPL>(A, lane, row, X);
  }

  // the weights, a selection a lane
  T* part = reinterpret_cast<T*>(X.area);
  T most = (T)-INFINITY, total = 0;
  for (int j = at; j < A.k; j += LPR) {
    const int e = X.e[j];
    const T x = e >= 0 ? (T)widen(row[e]) : (T)-INFINITY;
    part[j] = x;
    most = x > most ? x : most;
  }
  if (A.renorm) most = row_max<LPR>(most);
  for (int j = at; j < A.k; j += LPR) {
    const T x = part[j];
    T w;
    if (!A.sigmoid) {
      w = exp_of(x - (A.renorm ? most : top));
    } else {
      // all of them below 1/2: relative to exp(most), so that none is lost
      const bool low = A.renorm && most < 0;
      w = (low ? exp_of(x - most) : (T)1) / ((T)1 + exp_of(low ? x : -x));
    }
    w = x == (T)-INFINITY ? (T)0 : w;
    part[j] = w;
    total += w;
  }
  if (A.renorm) total = row_sum<LPR>(total);
  else total = A.sigmoid ? (T)1 : sum;
  const T share = (T)A.scale / total;
  for (int j = at; j < A.k; j += LPR) {
    const int e = X.e[j];
    A.idx[(int64_t)n * A.k + j] = e;
    A.weight[(int64_t)n * A.k + j] = bad ? NAN : e < 0 ? 0.f : (float)(part[j] * share);
  }
}

// Exclusive sums of count[E] in place (LDS) by all NT threads, the total in count[E].
template <int NT>
__device__ __forceinline__ void scan_experts(int* count, int E, int* part) {
  constexpr int EPT = (1024 + NT - 1) / NT, NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int c[EPT], sum = 0;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int e = tid * EPT + i;
    c[i] = sum;
    sum += e < E ? count[e] : 0;
  }
  int up = sum;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int o = __shfl_up(up, s);
    if (lane >= s) up += o;
  }
  if (lane == 63) part[wave] = up;
  __syncthreads();
  int before = up - sum;
#pragma unroll
  for (int w = 0; w < NW; ++w) before += w < wave ? part[w] : 0;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int e = tid * EPT + i;
    if (e < E) count[e] = before + c[i];
  }
  if (tid == NT - 1) count[E] = before + sum;
  __syncthreads();
}

// A wave's run of a block's n slots, 64 at a time; the experts of the first few
// are read ahead of everything else.
template <int NT>
struct Slots {
  static constexpr int NW = NT / 64, AHEAD = 4;
  int n, lane, begin, end;  // chunks of 64
  int ahead[AHEAD];
  template <class F>
  __device__ __forceinline__ Slots(int count, F slot) : n(count) {
    lane = threadIdx.x & 63;
    const int wave = threadIdx.x >> 6, chunks = (n + 63) / 64, per = (chunks + NW - 1) / NW;
    begin = wave * per;
    end = std::min(chunks, begin + per);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) ahead[q] = begin + q < end && (begin + q) * 64 + lane < n ? slot((begin + q) * 64 + lane) : -1;
  }
  // f(i, e): slot i (may be past the last) has expert e, -1 where there is none
  template <class F, class G>
  __device__ __forceinline__ void each(F slot, G f) const {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
      if (begin + q < end) f((begin + q) * 64 + lane, ahead[q]);
    for (int c = begin + AHEAD; c < end; ++c) {
      const int i = c * 64 + lane;
      f(i, i < n ? slot(i) : -1);
    }
  }
};

// Places of a wave's slots in their order: next[wave][E] (LDS) holds where its
// first slot of every expert goes.
template <int NT, class F>
__device__ __forceinline__ void place_slots(const Slots<NT>& S, int E, int* next, F slot, int32_t* place) {
  const int lane = S.lane;
  int* mine = next + (threadIdx.x >> 6) * E;
  S.each(slot, [&](int i, int e) {
    // the lanes with the same expert
    uint64_t same = __ballot(e >= 0);
    for (int bit = 0; (E - 1) >> bit; ++bit) {
      const uint64_t set = __ballot(e >> bit & 1);
      same &= e >> bit & 1 ? set : ~set;
    }
    int at = -1;
    if (e >= 0) {
      const int before = __popcll(same & ((1ull << lane) - 1));
      const int first = __ffsll((unsigned long long)same) - 1;
      int start = 0;
      if (lane == first) start = atomicAdd(&mine[e], __popcll(same));
      at = __shfl(start, first) + before;
    }
    if (i < S.n) place[i] = at;
  });
}

// next[wave][E]: how many of a wave's slots every expert has. next is zero.
template <int NT, class F>
__device__ __forceinline__ void count_slots(const Slots<NT>& S, int E, int* next, F slot) {
  int* mine = next + (threadIdx.x >> 6) * E;
  S.each(slot, [&](int, int e) {
    if (e >= 0) atomicAdd(&mine[e], 1);
  });
  __syncthreads();
}
// ... and from that where a wave's first slot of every expert goes: behind those
// of the block's earlier waves, the first of which goes to base[e].
template <int NT>
__device__ __forceinline__ void start_slots(int E, int* next, const int* base) {
  constexpr int NW = NT / 64;
  for (int e = threadIdx.x; e < E; e += NT) {
    int at = base[e], c[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) c[w] = next[w * E + e];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      next[w * E + e] = at;
      at += c[w];
    }
  }
  __syncthreads();
}

// Rows of a block, their experts' counts, and where ONE workgroup does all of
// the call also the places.
template <class L, class V, int LPR, int EPL, int NT, bool ONE>
__global__ __launch_bounds__(NT) void k_route_rows(const RouteArgs A) {
  constexpr int ROWS = NT / LPR;  // rows at a time
  extern __shared__ __align__(16) unsigned char lds[];
  int* sel = reinterpret_cast<int*>(lds + ROWS * A.row_lds);  // ONE: [N][k]
  int* count = sel + (ONE ? A.N * A.k : 0);                   // [E + 1], ONE: then [NT / 64][E]
  const int tid = threadIdx.x, lane = tid & 63, r = tid / LPR;
  unsigned char* own = lds + r * A.row_lds;
  const RowLds X(own, A);
  if (!ONE && A.place) {
    for (int i = tid; i < A.E; i += NT) count[i] = 0;
    __syncthreads();
  }
  const int first = ONE ? 0 : blockIdx.x * A.block_rows;
  const int last = ONE ? A.N : (int)std::min<int64_t>(A.N, (int64_t)first + A.block_rows);
  // a row's logits are on their way while the one before is worked on
  typedef typename Wide<L>::type T;
  const auto load = [&](int n, T (&z)[EPL]) {
    if (n < last) load_row<EPL>(static_cast<const L*>(A.logits) + (int64_t)n * A.ld, (lane & (LPR - 1)) * EPL, A.E, A.wide, z);
  };
  T z[EPL];
  load(first + r, z);
  for (int n = first + r; n < last; n += ROWS) {
    route_row<L, V, LPR, EPL>(A, n, lane, X, z, [&] { load(n + ROWS, z); });
    if (ONE || A.place)
      for (int j = lane & (LPR - 1); j < A.k; j += LPR) {
        const int e = X.e[j];
        if (ONE) sel[n * A.k + j] = e;
        else if (e >= 0) atomicAdd(&count[e], 1);
      }
    wave_sync();
  }
  if (!A.place) return;
  __syncthreads();
  if constexpr (ONE) {
    int *next = count + A.E + 1, *part = next + NT / 64 * A.E;
    const int n = A.N * A.k;
    const auto slot = [&](int i) { return sel[i]; };
    const Slots<NT> S(n, slot);
    for (int i = tid; i < NT / 64 * A.E; i += NT) next[i] = 0;
    __syncthreads();
    count_slots<NT>(S, A.E, next, slot);
    for (int e = tid; e < A.E; e += NT) {
      int c = 0;
      for (int w = 0; w < NT / 64; ++w) c += next[w * A.E + e];
      count[e] = c;
    }
    __syncthreads();
    scan_experts<NT>(count, A.E, part);
    for (int e = tid; e <= A.E; e += NT) A.offsets[e] = count[e];
    start_slots<NT>(A.E, next, count);
    place_slots<NT>(S, A.E, next, slot, A.place);
  } else {
    for (int i = tid; i < A.E; i += NT) A.count[(int64_t)blockIdx.x * count_row(A.E) + i] = (uint16_t)count[i];
  }
}

constexpr int kPlaceThreads = 1024;

// Places of a block's slots: after the slots of the experts before, of the same
// expert in the blocks before, and of the waves before. Every workgroup sums
// the blocks' counts by itself; a launch of its own for that took 5 us, this
// takes one or two with the 256 blocks of large calls (past 2^23 rows there are
// more blocks, and every one sums all of them).
__global__ __launch_bounds__(kPlaceThreads) void k_route_place(const RouteArgs A) {
  constexpr int NT = kPlaceThreads;
  extern __shared__ __align__(16) unsigned char lds[];
  int* count = reinterpret_cast<int*>(lds);  // [E + 1], then those of the blocks before [E]
  int *before = count + A.E + 1, *next = before + A.E, *part = next + NT / 64 * A.E;
  const int tid = threadIdx.x, b = blockIdx.x;
  const int64_t first = (int64_t)b * A.block_rows * A.k;
  const int n = (int)std::min((int64_t)A.block_rows * A.k, (int64_t)A.N * A.k - first);
  const int32_t* idx = A.idx + first;
  const auto slot = [&](int i) { return idx[i]; };
  const Slots<NT> S(n, slot);
  for (int e = tid; e < (2 + NT / 64) * A.E + 1; e += NT) count[e] = 0;  // (before and next behind it)
  __syncthreads();
  // a thread eight experts and a slice of the blocks
  const int cols = (A.E + 7) / 8, width = cols > 64 ? 128 : cols > 32 ? 64 : cols > 16 ? 32 : cols > 8 ? 16 : 8;
  if (const int col = tid % width; col < cols) {
    uint32_t total[8] = {}, sum[8] = {};
#pragma unroll 8
    for (int c = tid / width; c < A.blocks; c += NT / width) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(A.count + (int64_t)c * count_row(A.E) + col * 8);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const uint32_t x = v[q >> 1] >> 16 * (q & 1) & 0xffffu;
        total[q] += x;
        sum[q] += c < b ? x : 0u;
      }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (col * 8 + q < A.E) {
        atomicAdd(&count[col * 8 + q], (int)total[q]);
        atomicAdd(&before[col * 8 + q], (int)sum[q]);
      }
  }
  count_slots<NT>(S, A.E, next, slot);
  scan_experts<NT>(count, A.E, part);
  if (b == 0)
    for (int e = tid; e <= A.E; e += NT) A.offsets[e] = count[e];
  __syncthreads();
  for (int e = tid; e < A.E; e += NT) count[e] += before[e];
  __syncthreads();
  start_slots<NT>(A.E, next, count);
  place_slots<NT>(S, A.E, next, slot, A.place + first);
}

// Without rows: no expert has any.
__global__ void k_route_none(int32_t* offsets, int E) {
  for (int e = threadIdx.x; e <= E; e += blockDim.x) offsets[e] = 0;
}

// Gradient of the logits. With w the weights without scale and d the weights'
// gradient times scale:
//   renormalised: dz_j = w_j (d_j - sum_i w_i d_i), sigmoid: times (1 - s_j);
//   sigmoid: dz_j = s_j (1 - s_j) d_j;
//   softmax: dz_e = s_e (d_e [e selected] - sum_i s_i d_i) for every expert.
// A row's gradient is put together in LDS and stored in whole accesses. Bound
// by the write of the rows and the reads of the chosen logits, which fetch
// most of their lines: 65536 x 128 float32 in 13 us (5.2 TB/s of 67 MB).
template <class L, int LPR, int EPL>
__global__ __launch_bounds__(256) void k_route_backward(const RouteArgs A) {
  typedef typename Wide<L>::type T;
  constexpr int NT = 256, ROWS = NT / LPR;
  extern __shared__ __align__(16) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, at = lane & (LPR - 1), r = tid / LPR, e0 = at * EPL;
  T* grad = reinterpret_cast<T*>(lds) + r * (LPR * EPL);  // this row's gradient
  for (int64_t n = (int64_t)blockIdx.x * ROWS + r; n < A.N; n += (int64_t)gridDim.x * ROWS) {
    const L* row = static_cast<const L*>(A.logits) + n * A.ld;
    L* out = static_cast<L*>(A.dlogits) + n * A.dld;
    constexpr int JPL = kMostK / LPR > 0 ? kMostK / LPR : 1;
    int e[JPL];
    T z[JPL], d[JPL], w[JPL], most = (T)-INFINITY;
#pragma unroll
    for (int q = 0; q < JPL; ++q) {
      const int j = q * LPR + at;
      e[q] = -1;
      z[q] = (T)-INFINITY;
      d[q] = 0;
      if (q * LPR >= A.k) continue;
      e[q] = j < A.k ? A.idx[n * A.k + j] : -1;
      if (e[q] >= A.E) e[q] = -1;
      z[q] = e[q] >= 0 ? (T)widen(row[e[q]]) : (T)-INFINITY;
      d[q] = e[q] >= 0 ? (T)A.dweight[n * A.k + j] * (T)A.scale : (T)0;
      most = z[q] > most ? z[q] : most;
    }
    T base[EPL];
    const bool whole = !A.sigmoid && !A.renorm;
    T top = 0, sum = 1;
    if (whole) {
      load_row<EPL>(row, e0, A.E, A.wide, base);
      T b = (T)-INFINITY;
#pragma unroll
      for (int i = 0; i < EPL; ++i) b = base[i] > b ? base[i] : b;
      top = row_max<LPR>(b);
      if (top == (T)-INFINITY) top = 0;
      sum = 0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        base[i] = exp_of(base[i] - top);
        sum += base[i];
      }
      sum = row_sum<LPR>(sum);
    } else if (A.renorm) {
      most = row_max<LPR>(most);
    }
    T total = 0, dot = 0;
    T lift[JPL];  // 1 - s_j
#pragma unroll
    for (int q = 0; q < JPL; ++q) {
      w[q] = 0;
      lift[q] = 1;
      if (e[q] < 0) continue;
      if (!A.sigmoid) {
        w[q] = whole ? exp_of(z[q] - top) / sum : exp_of(z[q] - most);
      } else {
        lift[q] = (T)1 / ((T)1 + exp_of(z[q]));
        w[q] = A.renorm && most < 0 ? exp_of(z[q] - most) * lift[q] : (T)1 / ((T)1 + exp_of(-z[q]));
      }
      total += w[q];
    }
    if (A.renorm) {
      total = row_sum<LPR>(total);
#pragma unroll
      for (int q = 0; q < JPL; ++q)
        if (e[q] >= 0) w[q] /= total;
    }
#pragma unroll
    for (int q = 0; q < JPL; ++q) dot += w[q] * d[q];
    if (A.renorm || whole) dot = row_sum<LPR>(dot);
#pragma unroll
    for (int i = 0; i < EPL; ++i) grad[e0 + i] = whole && sum != 0 ? -(base[i] / sum) * dot : (T)0;
    wave_sync();
#pragma unroll
    for (int q = 0; q < JPL; ++q)
      if (e[q] >= 0) {
        if (A.renorm) grad[e[q]] = w[q] * lift[q] * (d[q] - dot);
        else if (A.sigmoid) grad[e[q]] = w[q] * lift[q] * d[q];
        else grad[e[q]] = w[q] * (d[q] - dot);
      }
    wave_sync();
    store_row<EPL>(out, e0, A.E, A.wide, grad + e0);
    wave_sync();
  }
}

// Threads of a workgroup: 256 while the blocks of so many rows are no more than
// kRouteBlocks, else as many as its registers and LDS allow, so that large
// calls fill the chip with few blocks.
template <class L, class V, int LPR, int EPL, int NT>
hipError_t run_blocks(RouteArgs& A, hipStream_t s) {
  constexpr int ROWS = NT / LPR;
  const int64_t per = ((int64_t)A.N + kRouteBlocks - 1) / kRouteBlocks;
  A.block_rows = (int32_t)std::min<int64_t>(kBlockRows, std::max<int64_t>(ROWS, (per + ROWS - 1) / ROWS * ROWS));
  A.blocks = (int32_t)(((int64_t)A.N + A.block_rows - 1) / A.block_rows);
  const size_t lds = (size_t)ROWS * A.row_lds + 4 * ((size_t)A.E + 1);
  k_route_rows<L, V, LPR, EPL, NT, false><<<dim3((unsigned)A.blocks), dim3(NT), lds, s>>>(A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !A.place) return e;
  constexpr int kWaves = kPlaceThreads / 64;
  const size_t lds2 = 4 * ((size_t)A.E + 1 + A.E + kWaves * A.E + kWaves);
  k_route_place<<<dim3((unsigned)A.blocks), dim3(kPlaceThreads), lds2, s>>>(A);
  return hipGetLastError();
}

template <class L, class V, int LPR, int EPL, bool ONE>
hipError_t run_rows(const RouteArgs& given, hipStream_t s) {
  RouteArgs A = given;
  A.slots = (A.k + kSpare + 1) / 2 * 2;
  A.row_lds = row_bytes<V, LPR, EPL>(A);
  A.by_each = Divisor(A.each);
  A.group_lanes = -1;
  for (int lg = 0; 1 << lg <= 16; ++lg)
    if (A.each == EPL << lg) A.group_lanes = lg;
  A.group_split = 0;
  while (A.group_split < 4 && A.groups << (A.group_split + 1) <= LPR) ++A.group_split;
  if constexpr (ONE) {
    constexpr int NT = EPL <= 8 && LPR == 16 ? 512 : 256, ROWS = NT / LPR;  // (their LDS is below 160 KiB)
    const size_t lds = (size_t)ROWS * A.row_lds + 4 * ((size_t)A.N * A.k + A.E + 1 + NT / 64 * A.E + NT / 64);
    k_route_rows<L, V, LPR, EPL, NT, true><<<dim3(1), dim3(NT), lds, s>>>(A);
    return hipGetLastError();
  } else {
    if (A.N <= kRouteBlocks * (256 / LPR)) return run_blocks<L, V, LPR, EPL, 256>(A, s);
    if constexpr (LPR == 8 && sizeof(V) == 4) {
      if (A.groups == 1) return run_blocks<L, V, LPR, EPL, 1024>(A, s);  // (with groups' values: up to 210 KiB of LDS)
    }
    return run_blocks<L, V, LPR, EPL, 512>(A, s);
  }
}

// Lanes of a row: 8 or 16 of up to 16 experts each, so that a reduction takes
// three or four steps and serves 8 or 4 rows of a wave (128 experts with 16
// lanes of 8: 20.3 us for 65536 rows, with 8 of 16: 16.2); a few rows, whose
// latency counts, have more lanes.
template <class L, class V>
hipError_t run_width(const RouteArgs& A, hipStream_t s) {
  if (A.N <= route_small(A.E)) {
    if (A.E <= 64) return run_rows<L, V, 16, 4, true>(A, s);
    if (A.E <= 128) return run_rows<L, V, 16, 8, true>(A, s);
    if (A.E <= 256) return run_rows<L, V, 16, 16, true>(A, s);
    if (A.E <= 512) return run_rows<L, V, 64, 8, true>(A, s);
    return run_rows<L, V, 64, 16, true>(A, s);
  }
  if (A.E <= 64) return run_rows<L, V, 8, 8, false>(A, s);
  if (A.E <= 128) return run_rows<L, V, 8, 16, false>(A, s);
  if (A.E <= 256) return run_rows<L, V, 16, 16, false>(A, s);
  if (A.E <= 512) return run_rows<L, V, 32, 16, false>(A, s);
  return run_rows<L, V, 64, 16, false>(A, s);
}

template <class L, int LPR, int EPL>
hipError_t run_back(const RouteArgs& A, hipStream_t s) {
  constexpr int ROWS = 256 / LPR;
  const size_t lds = (size_t)ROWS * LPR * EPL * sizeof(typename Wide<L>::type);
  const int64_t blocks = std::min<int64_t>(((int64_t)A.N + ROWS - 1) / ROWS, 1 << 16);
  k_route_backward<L, LPR, EPL><<<dim3((unsigned)blocks), dim3(256), lds, s>>>(A);
  return hipGetLastError();
}

template <class L>
hipError_t back_width(const RouteArgs& A, hipStream_t s) {
  if (A.E <= 64) return run_back<L, 16, 4>(A, s);
  if (A.E <= 128) return run_back<L, 16, 8>(A, s);
  if (A.E <= 256) return run_back<L, 16, 16>(A, s);
  if (A.E <= 512) return run_back<L, 64, 8>(A, s);
  return run_back<L, 64, 16>(A, s);
}

}  // namespace

hipError_t launch_route(const RouteArgs& A, hipStream_t s) {
  if (A.N == 0) {
    if (A.offsets) k_route_none<<<dim3(1), dim3(256), 0, s>>>(A.offsets, A.E);
    return hipGetLastError();
  }
  if (A.type == LOGIT_F64) return run_width<double, double>(A, s);
  if (A.type == LOGIT_F32) return A.by_score ? run_width<float, double>(A, s) : run_width<float, float>(A, s);
  return A.by_score ? run_width<uint16_t, double>(A, s) : run_width<uint16_t, float>(A, s);
}

hipError_t launch_route_backward(const RouteArgs& A, hipStream_t s) {
  if (A.type == LOGIT_F64) return back_width<double>(A, s);
  if (A.type == LOGIT_F32) return back_width<float>(A, s);
  return back_width<uint16_t>(A, s);
}

}  // namespace cardan
