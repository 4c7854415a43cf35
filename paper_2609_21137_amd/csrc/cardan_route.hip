// Routing of many rows: scores of E experts, the top k of each row, their
// weights, the rows' places in an array grouped by expert, and the gradient of
// the logits.
//
// Per row with logits z: score s_e = softmax(z)_e or sigmoid(z_e); the
// selection goes by v_e = s_e + bias_e in float64 where there is a bias or a
// group counts by its best two, else by z_e, whose order is the scores'.
// Groups of E / G consecutive experts count by their best v, or by the sum of
// their best two; the top_k largest v of the kept groups, descending, ties to
// the lower index. weight_j = scale s_j, over the sum of the kept s if
// renormalised.
//
// A row is spread over LPR lanes of one wave, EPL consecutive experts a lane,
// so that the lowest lane with the largest value holds the lowest index.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_rows.h"

namespace cardan {
namespace {

constexpr int kMostK = 32;

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
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
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
  v = f(v, lane_move<0x140>(v));  // the other half of 16
  if constexpr (LPR == 64) {
    v = f(v, __shfl_xor(v, 16));
    v = f(v, __shfl_xor(v, 32));
  }
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

// The largest of a lane's values and its removal.
template <int EPL, class V>
__device__ __forceinline__ V local_max(const V (&v)[EPL]) {
  V m = v[0];
#pragma unroll
  for (int i = 1; i < EPL; ++i) m = v[i] > m ? v[i] : m;
  return m;
}

// Selects the experts of one row into sel[k] (LDS of this row), -1 where none
// is left; v is used up.
template <int LPR, int EPL, class V>
__device__ __forceinline__ void select_top(V (&v)[EPL], int k, int lane, int* sel) {
  const int at = lane & (LPR - 1);
  V b = local_max(v);
  for (int j = 0; j < k; ++j) {
    const V m = row_max<LPR>(b);
    const uint64_t have = row_ballot<LPR>(b == m, lane);
    if (at == __ffsll((unsigned long long)have) - 1) {
      int hit = 0;
      bool found = false;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const bool here = !found && v[i] == b;
        hit = here ? i : hit;
        v[i] = here ? (V)-INFINITY : v[i];
        found |= here;
      }
      sel[j] = m == (V)-INFINITY ? -1 : at * EPL + hit;
      b = local_max(v);
    }
  }
}

// Experts outside the kept groups leave the selection. `all` [E] and `of`
// [groups] are LDS of this row.
template <int LPR, int EPL, class V>
__device__ __forceinline__ void keep_groups(V (&v)[EPL], const RouteArgs& A, int lane, V* all) {
  const int at = lane & (LPR - 1);
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (at * EPL + i < A.E) all[at * EPL + i] = v[i];
  wave_sync();
  constexpr int GPL = 64 / LPR;  // groups a lane: at most 64 in all
  V g[GPL];
#pragma unroll
  for (int q = 0; q < GPL; ++q) {
    const int grp = at * GPL + q;
    V b1 = (V)-INFINITY, b2 = (V)-INFINITY;
    if (grp < A.groups)
      for (int i = 0; i < A.each; ++i) {
        const V x = all[grp * A.each + i], lo = x < b1 ? x : b1;
        b1 = x > b1 ? x : b1;
        b2 = lo > b2 ? lo : b2;
      }
    g[q] = A.best == 2 && b2 != (V)-INFINITY ? b1 + b2 : b1;
  }
  wave_sync();
  uint64_t kept = 0;
  V b = local_max(g);
  for (int j = 0; j < A.top_groups; ++j) {
    const V m = row_max<LPR>(b);
    const uint64_t have = row_ballot<LPR>(b == m, lane);
    const int first = __ffsll((unsigned long long)have) - 1;
    int hit = 0;
    if (at == first) {
      bool found = false;
#pragma unroll
      for (int q = 0; q < GPL; ++q) {
        const bool here = !found && g[q] == b;
        hit = here ? q : hit;
        g[q] = here ? (V)-INFINITY : g[q];
        found |= here;
      }
      b = local_max(g);
    }
    hit = __shfl(hit, (lane & ~(LPR - 1)) + first);
    if (m != (V)-INFINITY) kept |= 1ull << (first * GPL + hit);
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = at * EPL + i;
    if (e < A.E && !(kept >> (e / A.each) & 1)) v[i] = (V)-INFINITY;
  }
}

// The selection and the weights of row n; sel[k] (LDS of this row) receives the experts.
template <class L, class V, int LPR, int EPL>
__device__ __forceinline__ void route_row(const RouteArgs& A, int n, int lane, int* sel, V* all) {
  typedef typename Wide<L>::type T;
  const int at = lane & (LPR - 1), e0 = at * EPL;
  const L* row = static_cast<const L*>(A.logits) + (int64_t)n * A.ld;
  V v[EPL];
  load_row<EPL>(row, e0, A.E, A.wide, v);
  // largest logit and sum of the softmax over all experts, where they are needed
  V top = 0, sum = 1;
  const bool whole = !A.sigmoid && (A.by_score || !A.renorm);
  if (whole) {
    V b = (V)-INFINITY;
#pragma unroll
    for (int i = 0; i < EPL; ++i) b = v[i] > b ? v[i] : b;
    top = row_max<LPR>(b);
    if (top == (V)-INFINITY) top = 0;
    sum = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) sum += exp_of(v[i] - top);
    sum = row_sum<LPR>(sum);
  }
  bool bad = false;
  if (A.by_score) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = e0 + i;
      if (v[i] == (V)-INFINITY) continue;
      V s;
      if (A.sigmoid) s = (V)1 / ((V)1 + exp_of(-v[i]));
      else s = exp_of(v[i] - top) / sum;
      v[i] = s + (A.bias ? (V)A.bias[e] : (V)0);
    }
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (v[i] != v[i]) {
      bad = true;
      v[i] = (V)-INFINITY;
    }
  bad = row_ballot<LPR>(bad, lane) != 0;
  if (A.groups > 1) keep_groups<LPR, EPL>(v, A, lane, all);
  select_top<LPR, EPL>(v, A.k, lane, sel);
  wave_sync();

  // the weights, a selection or two a lane
  constexpr int JPL = kMostK / LPR > 0 ? kMostK / LPR : 1;
  T z[JPL], w[JPL];
  int e[JPL];
  T most = (T)-INFINITY;
#pragma unroll
  for (int q = 0; q < JPL; ++q) {
    const int j = q * LPR + at;
    e[q] = -1;
    z[q] = (T)-INFINITY;
    if (q * LPR >= A.k) continue;
    e[q] = j < A.k ? sel[j] : -1;
    if (e[q] >= 0) z[q] = (T)widen(row[e[q]]);
    most = z[q] > most ? z[q] : most;
  }
  if (A.renorm) most = row_max<LPR>(most);
  T total = 0;
#pragma unroll
  for (int q = 0; q < JPL; ++q) {
    w[q] = 0;
    if (e[q] < 0) continue;
    if (!A.sigmoid) {
      w[q] = A.renorm ? exp_of(z[q] - most) : exp_of(z[q] - (T)top) / (T)sum;
    } else if (A.renorm && most < 0) {
      // all of them below 1/2: relative to exp(most), so that none is lost
      w[q] = exp_of(z[q] - most) / ((T)1 + exp_of(z[q]));
    } else {
      w[q] = (T)1 / ((T)1 + exp_of(-z[q]));
    }
    total += w[q];
  }
  if (A.renorm) total = row_sum<LPR>(total);
#pragma unroll
  for (int q = 0; q < JPL; ++q) {
    const int j = q * LPR + at;
    if (j >= A.k) continue;
    T r = A.renorm && e[q] >= 0 ? w[q] / total : w[q];
    r *= (T)A.scale;
    A.idx[(int64_t)n * A.k + j] = e[q];
    A.weight[(int64_t)n * A.k + j] = bad ? NAN : (float)r;
  }
}

// Exclusive sums of count[E] in place (LDS), all NT threads; returns nothing,
// total behind the last (count[E]).
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

// Places of n slots whose experts `slot(i)` gives, in their order: next[wave][E]
// (LDS) holds where a wave's first slot of every expert goes.
template <int NT, class F>
__device__ __forceinline__ void place_slots(int n, int E, int* next, F slot, int32_t* place) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int NW = NT / 64;
  const int chunks = (n + 63) / 64, per = (chunks + NW - 1) / NW;
  int* mine = next + wave * E;
  for (int c = wave * per; c < std::min(chunks, (wave + 1) * per); ++c) {
    const int i = c * 64 + lane;
    const int e = i < n ? slot(i) : -1;
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
    if (i < n) place[i] = at;
  }
}

// next[wave][E] from where the block's slots of every expert start (base[E])
// and the slots of the waves before.
template <int NT, class F>
__device__ __forceinline__ void count_slots(int n, int E, int* next, F slot) {
  constexpr int NW = NT / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < NW * E; i += NT) next[i] = 0;
  __syncthreads();
  const int chunks = (n + 63) / 64, per = (chunks + NW - 1) / NW;
  for (int c = wave * per; c < std::min(chunks, (wave + 1) * per); ++c) {
    const int i = c * 64 + lane;
    const int e = i < n ? slot(i) : -1;
    if (e >= 0) atomicAdd(&next[wave * E + e], 1);
  }
  __syncthreads();
}
template <int NT>
__device__ __forceinline__ void start_slots(int E, int* next, const int* base) {
  for (int e = threadIdx.x; e < E; e += NT) {
    int at = base[e];
    for (int w = 0; w < NT / 64; ++w) {
      const int c = next[w * E + e];
      next[w * E + e] = at;
      at += c;
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
  V* all = reinterpret_cast<V*>(lds);                                      // [ROWS][E] with groups
  int* sel = reinterpret_cast<int*>(all + (A.groups > 1 ? ROWS * A.E : 0));  // [ROWS][k], all rows if ONE
  int* count = sel + (ONE ? std::max(A.N, ROWS) : ROWS) * A.k;             // [E + 1], ONE: then [NT / 64][E]
  const int tid = threadIdx.x, lane = tid & 63, r = tid / LPR;
  if (!ONE && A.place) {
    for (int i = tid; i < A.E; i += NT) count[i] = 0;
    __syncthreads();
  }
  const int first = ONE ? 0 : blockIdx.x * A.block_rows;
  const int last = ONE ? A.N : (int)std::min<int64_t>(A.N, (int64_t)first + A.block_rows);
  for (int n = first + r; n < last; n += ROWS) {
    int* mine = sel + (ONE ? n : r) * A.k;
    route_row<L, V, LPR, EPL>(A, n, lane, mine, all + (A.groups > 1 ? r * A.E : 0));
    if (!ONE && A.place)
      for (int j = lane & (LPR - 1); j < A.k; j += LPR)
        if (mine[j] >= 0) atomicAdd(&count[mine[j]], 1);
    wave_sync();
  }
  if (!A.place) return;
  __syncthreads();
  if constexpr (ONE) {
    int *next = count + A.E + 1, *part = next + NT / 64 * A.E;
    const int n = A.N * A.k;
    const auto slot = [&](int i) { return sel[i]; };
    count_slots<NT>(n, A.E, next, slot);
    for (int e = tid; e < A.E; e += NT) {
      int c = 0;
      for (int w = 0; w < NT / 64; ++w) c += next[w * A.E + e];
      count[e] = c;
    }
    __syncthreads();
    scan_experts<NT>(count, A.E, part);
    for (int e = tid; e <= A.E; e += NT) A.offsets[e] = count[e];
    start_slots<NT>(A.E, next, count);
    place_slots<NT>(n, A.E, next, slot, A.place);
  } else {
    for (int i = tid; i < A.E; i += NT) A.count[(int64_t)blockIdx.x * A.E + i] = count[i];
  }
}

// Counts of the blocks -> sums over the blocks before, and totals behind them:
// a workgroup 16 experts, a thread up to 16 blocks of one, in registers. (With
// a lane an expert and a wave 64 blocks, read twice, 24 us at 1024 blocks.)
__global__ __launch_bounds__(1024) void k_route_scan(const RouteArgs A) {
  constexpr int PER = kRouteBlocks / 64;
  __shared__ int part[16][65];
  const int tid = threadIdx.x, col = tid & 15, slice = tid >> 4, e = blockIdx.x * 16 + col;
  const int per = (A.blocks + 63) / 64, lo = slice * per;
  int c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) c[i] = i < per && lo + i < A.blocks && e < A.E ? A.count[(int64_t)(lo + i) * A.E + e] : 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += c[i];
  part[col][slice] = sum;
  __syncthreads();
  {
    const int lane = tid & 63, wave = tid >> 6;  // a wave an expert, a lane a slice
    const int own = part[wave][lane];
    int up = own;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(up, s);
      if (lane >= s) up += o;
    }
    part[wave][lane] = up - own;
    if (lane == 63 && blockIdx.x * 16 + wave < (unsigned)A.E)
      A.count[(int64_t)A.blocks * A.E + blockIdx.x * 16 + wave] = up;
  }
  __syncthreads();
  int at = part[col][slice];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i < per && lo + i < A.blocks && e < A.E) A.count[(int64_t)(lo + i) * A.E + e] = at;
    at += c[i];
  }
}

__global__ __launch_bounds__(256) void k_route_place(const RouteArgs A) {
  constexpr int NT = 256;
  extern __shared__ __align__(16) unsigned char lds[];
  int* count = reinterpret_cast<int*>(lds);  // [E + 1]
  int *next = count + A.E + 1, *part = next + NT / 64 * A.E;
  const int tid = threadIdx.x, b = blockIdx.x;
  const int64_t first = (int64_t)b * A.block_rows * A.k;
  const int n = (int)std::min((int64_t)A.block_rows * A.k, (int64_t)A.N * A.k - first);
  const int32_t* idx = A.idx + first;
  const auto slot = [&](int i) { return idx[i]; };
  for (int e = tid; e < A.E; e += NT) count[e] = A.count[(int64_t)A.blocks * A.E + e];
  count_slots<NT>(n, A.E, next, slot);
  scan_experts<NT>(count, A.E, part);
  if (b == 0)
    for (int e = tid; e <= A.E; e += NT) A.offsets[e] = count[e];
  __syncthreads();
  for (int e = tid; e < A.E; e += NT) count[e] += A.count[(int64_t)b * A.E + e];
  __syncthreads();
  start_slots<NT>(A.E, next, count);
  place_slots<NT>(n, A.E, next, slot, A.place + first);
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

template <class L, class V, int LPR, int EPL>
hipError_t run_rows(const RouteArgs& A, hipStream_t s) {
  if (A.N <= kRouteSmall) {
    constexpr int NT = 512, ROWS = NT / LPR;
    const size_t lds = (A.groups > 1 ? (size_t)ROWS * A.E * sizeof(V) : 0) + 4 * ((size_t)std::max(A.N, ROWS) * A.k +
                       A.E + 1 + NT / 64 * A.E + NT / 64);
    k_route_rows<L, V, LPR, EPL, NT, true><<<dim3(1), dim3(NT), lds, s>>>(A);
    return hipGetLastError();
  }
  constexpr int NT = 256, ROWS = NT / LPR;
  const size_t lds = (A.groups > 1 ? (size_t)ROWS * A.E * sizeof(V) : 0) + 4 * ((size_t)ROWS * A.k + A.E + 1);
  k_route_rows<L, V, LPR, EPL, NT, false><<<dim3((unsigned)A.blocks), dim3(NT), lds, s>>>(A);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !A.place) return e;
  k_route_scan<<<dim3((unsigned)((A.E + 15) / 16)), dim3(1024), 0, s>>>(A);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const size_t lds2 = 4 * ((size_t)A.E + 1 + 4 * A.E + 4);
  k_route_place<<<dim3((unsigned)A.blocks), dim3(256), lds2, s>>>(A);
  return hipGetLastError();
}

template <class L, class V>
hipError_t run_width(const RouteArgs& A, hipStream_t s) {
  if (A.E <= 64) return run_rows<L, V, 16, 4>(A, s);
  if (A.E <= 128) return run_rows<L, V, 16, 8>(A, s);
  if (A.E <= 256) return run_rows<L, V, 16, 16>(A, s);
  if (A.E <= 512) return run_rows<L, V, 64, 8>(A, s);
  return run_rows<L, V, 64, 16>(A, s);
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

// Lanes of a row: its experts stay in at most 16 registers a lane. Rows of a
// block: a whole number of passes of its 256 threads.
void plan_route(RouteArgs* A) {
  const int rows = A->E <= 256 ? 16 : 4;  // of 256 threads at a time
  const int64_t per = ((int64_t)A->N + kRouteBlocks - 1) / kRouteBlocks;
  A->block_rows = (int32_t)std::max<int64_t>(rows, (per + rows - 1) / rows * rows);
  A->blocks = (int32_t)(((int64_t)A->N + A->block_rows - 1) / A->block_rows);
}

hipError_t launch_route(const RouteArgs& A, hipStream_t s) {
  if (A.N == 0) {
    if (A.offsets) k_route_none<<<dim3(1), dim3(256), 0, s>>>(A.offsets, A.E);
    return hipGetLastError();
  }
  RouteArgs B = A;
  plan_route(&B);
  if (A.type == LOGIT_F64) return run_width<double, double>(B, s);
  if (A.type == LOGIT_F32) return A.by_score ? run_width<float, double>(B, s) : run_width<float, float>(B, s);
  return A.by_score ? run_width<uint16_t, double>(B, s) : run_width<uint16_t, float>(B, s);
}

hipError_t launch_route_backward(const RouteArgs& A, hipStream_t s) {
  if (A.type == LOGIT_F64) return back_width<double>(A, s);
  if (A.type == LOGIT_F32) return back_width<float>(A, s);
  return back_width<uint16_t>(A, s);
}

}  // namespace cardan
