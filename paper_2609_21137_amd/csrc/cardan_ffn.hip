// Feed-forward block of dense bf16 weights, forward and backward, for one
// matrix set or for the row groups of E experts.
//
//   h = silu(x Wg) * (x Wu)   (or max(x Wu, 0)^2),   y = h Wd
//   dh = dy Wd^T, dg = dh u s(1 + g(1 - s)), du = dh g s,  s = 1 / (1 + e^-g)
//   dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  dWd = h^T dy
//
// Every product runs on v_mfma_f32_16x16x32_bf16 with float32 accumulators. g
// and u are kept in float32, so that h, dg and du, which enter the second
// products in bf16, are rounded once (pack4() below): half a step, 2^-8, of their
// values. Outputs are then off by 2.3e-3 of their norm, two roundings' root of
// squares, where one that is rounded at the end alone is off by 1.7e-3. More bits
// of h, dg and du would be a second product of their low halves: six of a training
// step's nine products twice.
//
// Measured at 8192 rows, 4096 x 11008: gate/up 1.15 PFLOP/s (0.9 GB of kept
// projections and h beside it), down 1.38, dh 0.99 (1.1 GB in its epilogues),
// dx 1.34, weight gradients 1.33; MFMA busy 63 to 75 % of the cycles (52 % in dh).
// 6144 rows of 128 experts, 2688 x 1856: weights at 5 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_ffn.h"

namespace cardan {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#define LDS __attribute__((address_space(3)))

constexpr uint32_t kOob = 0x80000000u;     // an offset past every resource

struct TileGrid {
  Divisor band;       // tiles of a band of row tiles (below: place())
  Divisor group;      // tiles of one group's gradients
  int32_t band_log;   // log2 of a band's row tiles
  int32_t col_tiles;  // tiles along the output's columns
  int32_t row_tiles;  // along its rows (weight gradients; others count their groups' rows)
  int32_t full;       // tiles before the split ones
  int32_t split;      // parts of each split tile; 1: none is split
};

__device__ __forceinline__ u32x4 make_rsrc(const void* base, int bytes) {
  const uint32_t n = bytes < 0 ? 0u : (uint32_t)bytes;
  const uint64_t b = reinterpret_cast<uintptr_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)b),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) & 0xffffu,
               (uint32_t)__builtin_amdgcn_readfirstlane((int)n), 0x00020000u};
}

// 64 lanes x 16 bytes from the resource at `voff` to 1024 bytes of LDS at
// `lds`. Written as asm because the compiler, which cannot tell the stages of
// LDS apart, waits for every such load before the next transposing read; the
// wait that is needed is wait_loads(). It has no output register. (M0 holds
// the LDS address and must be a wait state old.) It writes LDS and M0: no other
// memory access moves across it, which the counts of wait_loads() rely on. The
// compiler takes M0 for reserved and warns that it is not kept, as it need not be.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(u32x4 rs, uint32_t lds, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rs)
               : "m0", "memory");
}
#pragma clang diagnostic pop

// float32 -> bf16, nearest even (NaN stays NaN)
__device__ __forceinline__ uint32_t bf16_bits(float f) {
  const __bf16 b = (__bf16)f;
  return (uint32_t)__builtin_bit_cast(unsigned short, b);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
__device__ __forceinline__ uint2 pack4(f32x4 v) { return make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])); }

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows [lo, hi) of group e. Offsets outside [0, N] or out of order are cut to
// a range inside the tensors.
__device__ __forceinline__ void group_rows(const FfnArgs& A, int e, int& lo, int& hi) {
  if (!A.off) {
    lo = 0;
    hi = A.N;
    return;
  }
  lo = clampi(A.off[e], 0, A.N);
  hi = clampi(A.off[e + 1], lo, A.N);
}

// The groups' row tiles, counted group by group: cum[e] tiles up to and with
// group e, and each group's rows. Built in LDS by the first wave; returns the
// number of tiles.
__device__ __forceinline__ int count_tiles(const FfnArgs& A, int BM, int* cum) {
  if (!A.off) return (A.N + BM - 1) / BM;
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int before = 0, past = 0;
    for (int e0 = 0; e0 < A.E; e0 += 64) {
      int lo = 0, hi = 0;
      if (e0 + lane < A.E) group_rows(A, e0 + lane, lo, hi);
      // a group begins where those before it have ended, whatever the offsets
      int top = hi;
      for (int s = 1; s < 64; s <<= 1) {
        const int v = __shfl_up(top, s);
        top = lane >= s && v > top ? v : top;
      }
      const int ended = __shfl_up(top, 1);
      if (lane > 0 && ended > lo) lo = ended;
      if (past > lo) lo = past;
      if (lo > hi) hi = lo;
      past = max(past, __builtin_amdgcn_readlane(top, 63));
      int c = (hi - lo + BM - 1) / BM;
      for (int s = 1; s < 64; s <<= 1) {
        const int v = __shfl_up(c, s);
        c += lane >= s ? v : 0;
      }
      c += before;
      if (e0 + lane < A.E) {
        cum[e0 + lane] = c;
        cum[A.E + 2 * (e0 + lane)] = lo;
        cum[A.E + 2 * (e0 + lane) + 1] = hi;
      }
      before = __builtin_amdgcn_readlane(c, 63);
    }
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(cum[A.E - 1]);
}

// Group, first row and end of rows of row tile t (0 <= t < count_tiles()).
__device__ __forceinline__ void locate(const FfnArgs& A, int BM, const int* cum, int t, int& e, int& row, int& end) {
  if (!A.off) {
    e = 0;
    row = t * BM;
    end = A.N;
    return;
  }
  const int lane = threadIdx.x & 63;
  for (int e0 = 0;; e0 += 64) {
    const unsigned long long past = __ballot(e0 + lane < A.E && cum[e0 + lane] > t);
    if (past == 0 && e0 + 64 < A.E) continue;
    e = e0 + (past ? __ffsll((long long)past) - 1 : 0);
    break;
  }
  const int before = e ? __builtin_amdgcn_readfirstlane(cum[e - 1]) : 0;
  row = __builtin_amdgcn_readfirstlane(cum[A.E + 2 * e]) + (t - before) * BM;
  end = __builtin_amdgcn_readfirstlane(cum[A.E + 2 * e + 1]);
}

// One operand of a tile product: R rows (of the output's row or column axis)
// by 64 steps of the sum, 128 R bytes of LDS per stage, filled by loads that
// go to LDS directly. A wave's load writes 1024 consecutive bytes of LDS, so
// the order within a tile is made by which address each lane reads from.
//
// TR = false: memory has the sum along its rows. LDS [R][64], 16-byte chunk c
// of row r at place c ^ (r & 7): the 16 rows of an operand read land in
// different banks.
// TR = true: memory has the sum down its columns. LDS [64][R], 32-byte pair p
// of row k at place p ^ swz(k). A transposing read takes one pair of four rows
// in each 16 lanes, and 32 lanes are served at a time: rows k..k+3 and
// k+8..k+11, which the places spread over the 64 banks.
template <int R, bool TR, int NW>
struct Operand {
  static constexpr int kLoads = R / 8 / NW;     // loads of one wave per stage
  static constexpr int kRow = TR ? R * 2 : 128;  // bytes of an LDS row
  static constexpr int kPairs = TR ? (R / 16 < 8 ? R / 16 : 8) : 1;
  static_assert(R % (8 * NW) == 0, "whole loads");

  static __device__ __forceinline__ int swz(int k) {
    return kPairs == 8 ? (k & 3) | (k >> 1 & 4) : kPairs == 4 ? (k >> 1 & 1) | (k >> 2 & 2) : k >> 3 & 1;
  }

  uint32_t voff[kLoads];
  bool tail;  // this lane's chunk lies past the last step's end (TR = false)

  __device__ __forceinline__ void init(int wave, int ld, int ksum) {
    const int l = threadIdx.x & 63;
    if constexpr (TR) {
      constexpr int per = 1024 / kRow;  // LDS rows of one load
      const int k = l / (kRow / 16), c = l % (kRow / 16);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int kk = (j * NW + wave) * per + k;
        const int src = (((c >> 1) ^ swz(kk)) << 1) | (c & 1);
        voff[j] = (uint32_t)(kk * ld * 2 + src * 16);
      }
      tail = false;
    } else {
      const int r = l >> 3, c = (l & 7) ^ r;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) voff[j] = (uint32_t)(((j * NW + wave) * 8 + r) * ld * 2 + c * 16);
      tail = (ksum & 63) != 0 && c * 8 >= (ksum & 63);
    }
  }

  // load j of this wave; `last`: the step is the sum's last
  __device__ __forceinline__ void issue(u32x4 rs, uint32_t lds, int wave, bool last, int j) const {
    load_to_lds(rs, lds + (j * NW + wave) * 1024, voff[j] | (last && tail ? kOob : 0u));
  }

  // byte of the first operand read of the 16-row block that starts at row r0
  static __device__ __forceinline__ int base(int r0) {
    const int l = threadIdx.x & 63;
    if constexpr (TR) {
      const int k = (l >> 4) * 8 + ((l & 15) >> 2);
      return k * kRow + ((r0 >> 4) ^ swz(k)) * 32 + (l & 3) * 8;
    } else {
      return (r0 + (l & 15)) * 128 + ((l >> 4) ^ (l & 7)) * 16;
    }
  }
  // operand of step half kk (32 of 64) and block f after the one of `b`
  static __device__ __forceinline__ bf16x8 read(const char* lds, int b, int f, int kk) {
    if constexpr (TR) {
      const int at = (b ^ (f << 5)) + kk * 32 * kRow;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4*)(lds + at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4*)(lds + at + 4 * kRow));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(const bf16x8*)(lds + ((b ^ (kk << 6)) + f * 2048));
    }
  }
};

// s(g) = 1 / (1 + e^-g) by the reciprocal instruction (1 ulp; the division's
// dozen instructions were a third of an epilogue's). e^-g overflows to infinity
// for g < -88 and gives 0.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * g));
}

// Waits until at most N loads of this wave are in flight and all of its LDS
// reads have returned, then for the workgroup's other waves.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "vmcnt");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0070);  // vmcnt(N), lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// max(u, 0) that keeps a NaN (fmaxf returns its other operand).
__device__ __forceinline__ float relu(float u) { return u < 0.f ? 0.f : u; }

// Activation of four projections; g is not used by up-only experts.
template <bool RELU2>
__device__ __forceinline__ f32x4 activate(f32x4 g, f32x4 u) {
  f32x4 h;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (RELU2) {
      const float p = relu(u[q]);
      h[q] = p * p;
    } else {
      h[q] = g[q] * sigmoid(g[q]) * u[q];
    }
  }
  return h;
}

// Gradients of four projections from that of h.
template <bool RELU2>
__device__ __forceinline__ void activate_grad(f32x4 dh, f32x4 g, f32x4 u, f32x4& dg, f32x4& du) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (RELU2) {
      du[q] = dh[q] * 2.f * relu(u[q]);
    } else {
      const float s = sigmoid(g[q]);
      dg[q] = dh[q] * u[q] * s * (1.f + g[q] * (1.f - s));
      du[q] = dh[q] * g[q] * s;
    }
  }
}

// The bf16 values of two neighbouring 16x16 blocks, four of a lane in each, as
// eight consecutive columns a lane: the odd 16-lane groups' part of the first
// block changes places with the even groups' part of the second. The lane's
// columns begin at pair_col().
__device__ __forceinline__ u32x4 pair_up(uint2 a, uint2 b) {
  const auto x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
__device__ __forceinline__ int pair_col() {
  const int grp = (threadIdx.x & 63) >> 4;
  return (grp & 1) * 16 + (grp >> 1) * 8;
}

// Two 64-byte pieces of a row, a and b (four lanes' 16 bytes each, in 16
// rows): lanes 8..15 of a row group's a change places with lanes 0..7's b, so
// that one store covers whole 128-byte lines of eight rows. Lane (lane & 15)
// stores `s0` to row (lane & 7), `s1` to row (lane & 7) + 8, at the first
// piece's columns for lanes 0..7 and the second's for 8..15.
__device__ __forceinline__ void lines_of(u32x4 a, u32x4 b, u32x4& s0, u32x4& s1) {
  const bool high = threadIdx.x & 8;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t give = high ? a[q] : b[q];
    const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x128, 0xF, 0xF, false);  // row_ror:8
    s0[q] = high ? got : a[q];
    s1[q] = high ? b[q] : got;
  }
}

template <bool NT>
__device__ __forceinline__ void put16(void* p, u32x4 v) {
  if constexpr (NT) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

// Whole lines of rows r8 and r8 + 8 (those below `end`), pieces a and b.
template <bool NT>
__device__ __forceinline__ void put_lines(char* p, int64_t row_bytes, int r8, int end, u32x4 a, u32x4 b) {
  u32x4 s0, s1;
  lines_of(a, b, s0, s1);
  if (r8 < end) put16<NT>(p, s0);
  if (r8 + 8 < end) put16<NT>(p + 8 * row_bytes, s1);
}

// A tile's outputs: group, first row and end of rows, first column, and which
// of dWg (0) and dWu (1).
struct Place {
  int e, row, end, n0, mat;
};

// Tiles are numbered band by band of 2^band_log row tiles, all columns of a
// band with the rows fastest: a run of neighbours shares its operands in the
// XCD's L2. `rows` row tiles (of a group's gradient); the last band may be
// lower: `inv` is inverse_of() its height.
__device__ __forceinline__ uint32_t last_band(const TileGrid& G, int rows) {
  const uint32_t low = (uint32_t)rows & ((1u << G.band_log) - 1);
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)inverse_of(low));
}

template <int KIND, bool RELU2, int BM, int BN>
__device__ __forceinline__ Place place(const FfnArgs& A, const TileGrid& G, const int* cum, int rows, uint32_t inv, int id) {
  constexpr int kMats = KIND == K_DWI && !RELU2 ? 2 : 1, BC = KIND == K_UP && !RELU2 ? BN / 2 : BN;
  constexpr bool kDW = KIND == K_DWI || KIND == K_DWD;
  Place P;
  P.e = 0;
  P.mat = 1;
  if constexpr (kDW) {
    P.e = G.group.quotient(id);
    id -= P.e * (int)G.group.d;
    if (kMats == 2) {
      P.mat = id & 1;
      id >>= 1;
    }
  }
  const int band = G.band.quotient(id), in = id - band * (int)G.band.d, left = rows - (band << G.band_log);
  int row, col;
  if (left >> G.band_log) {
    col = in >> G.band_log;
    row = in & ((1 << G.band_log) - 1);
  } else {
    col = small_quotient(in, inv);
    row = in - col * left;
  }
  row += band << G.band_log;
  P.n0 = col * BC;
  if constexpr (kDW) {
    P.row = row * BM;
    P.end = KIND == K_DWI ? A.H : A.I;
  } else {
    locate(A, BM, cum, row, P.e, P.row, P.end);
  }
  return P;
}

// The epilogue of one row of 16x16 blocks: output rows row16 .. row16 + 15,
// columns from wcol. Lane -> output row (lane & 15), columns (lane >> 4) * 4 + 0..3
// of a block. `in`: the projections that K_DH needs, of fetch().
template <int KIND, bool RELU2, int NF>
struct Emit {
  static constexpr bool kDual = KIND == K_UP && !RELU2, kDW = KIND == K_DWI || KIND == K_DWD;
  static constexpr int NC = kDual ? NF / 2 : NF;  // 16-column blocks of the output
  static constexpr int kIn = KIND == K_DH ? NC : 1, kGu = KIND == K_DH && !RELU2 ? 2 : 1;

  static __device__ __forceinline__ void fetch(const FfnArgs& A, const Place& P, int row16, int wcol, int nout, f32x4 (&in)[kIn][kGu]) {
    if constexpr (KIND == K_DH) {
      const int lane = threadIdx.x & 63, r = min(row16 + (lane & 15), P.end - 1);
      const int64_t rb = (int64_t)r * nout + (lane >> 4) * 4;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = wcol + j * 16 < nout ? wcol + j * 16 : wcol;
        in[j][0] = __builtin_nontemporal_load((const f32x4*)(A.u + rb + c));
        if constexpr (!RELU2) in[j][1] = __builtin_nontemporal_load((const f32x4*)(A.g + rb + c));
      }
    }
  }

  static __device__ __forceinline__ void put(const FfnArgs& A, const Place& P, int row16, int wcol, int nout, const f32x4 (&acc)[NF], const f32x4 (&in)[kIn][kGu]) {
    const int lane = threadIdx.x & 63, q4 = (lane >> 4) * 4;
    uint16_t* o0 = KIND == K_UP ? A.h : KIND == K_DH ? A.du : KIND == K_DOWN ? A.y : KIND == K_DX ? A.dx
                 : (KIND == K_DWD ? A.dWd : P.mat ? A.dWu : A.dWg) + (int64_t)P.e * A.H * A.I;
    uint2 v0[NC], v1[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      if constexpr (KIND == K_UP) {
        v0[j] = pack4(activate<RELU2>(acc[j], acc[kDual ? j + NC : j]));
      } else if constexpr (KIND == K_DH) {
        f32x4 dg, du;
        activate_grad<RELU2>(acc[j], in[j][kGu - 1], in[j][0], dg, du);
        v0[j] = pack4(du);
        if constexpr (!RELU2) v1[j] = pack4(dg);
      } else {
        v0[j] = pack4(acc[j]);
      }
    }
    const int r = row16 + (lane & 15), r8 = row16 + (lane & 7), high = lane >> 3 & 1;
    const int64_t rb = (int64_t)r * nout, rb8 = (int64_t)r8 * nout;
    const auto bits = [](f32x4 v) { return __builtin_bit_cast(u32x4, v); };
    if constexpr (KIND == K_UP && NC % 2 == 0) {  // kept projections: pieces are blocks of 16 float32
      if (A.u) {
#pragma unroll
        for (int j = 0; j < NC; j += 2) {
          if (wcol + j * 16 >= nout) continue;
          const int64_t at = rb8 + wcol + j * 16 + high * 16 + q4;
          constexpr int U = kDual ? NC : 0;
          if constexpr (!RELU2) put_lines<true>((char*)(A.g + at), (int64_t)nout * 4, r8, P.end, bits(acc[j]), bits(acc[j + 1]));
          put_lines<true>((char*)(A.u + at), (int64_t)nout * 4, r8, P.end, bits(acc[U + j]), bits(acc[U + j + 1]));
        }
      }
    } else if constexpr (KIND == K_UP) {
      static_assert(NC == 1, "blocks come in pairs or alone");
      if (r < P.end && A.u && wcol < nout) {
        if constexpr (!RELU2) *(f32x4*)(A.g + rb + wcol + q4) = acc[0];
        *(f32x4*)(A.u + rb + wcol + q4) = acc[kDual ? NC : 0];
      }
    }
    if constexpr (NC % 2 == 0) {  // pieces are pairs of bf16 blocks, two where both lie inside
#pragma unroll
      for (int j = 0; j < NC; j += 2) {
        const int c = wcol + j * 16;
        if (c >= nout) continue;
        if constexpr (NC % 4 == 0) {
          if (j % 4 == 2 && c < nout) continue;  // stored with the pair before it
          if (c + 32 < nout) {
            const int64_t at = rb8 + c + high * 32 + pair_col();
            put_lines<kDW>((char*)(o0 + at), (int64_t)nout * 2, r8, P.end, pair_up(v0[j], v0[j + 1]), pair_up(v0[j + 2], v0[j + 3]));
            if constexpr (KIND == K_DH && !RELU2)
              put_lines<false>((char*)(A.dg + at), (int64_t)nout * 2, r8, P.end, pair_up(v1[j], v1[j + 1]), pair_up(v1[j + 2], v1[j + 3]));
            continue;
          }
        }
        const u32x4 a = pair_up(v0[j], v0[j + 1]);
        if (r < P.end) put16<false>(o0 + rb + c + pair_col(), a);
        if constexpr (KIND == K_DH && !RELU2) {
          const u32x4 b = pair_up(v1[j], v1[j + 1]);
          if (r < P.end) put16<false>(A.dg + rb + c + pair_col(), b);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = wcol + j * 16;
        if (c >= nout || r >= P.end) continue;
        *(uint2*)(o0 + rb + c + q4) = v0[j];
        if constexpr (KIND == K_DH && !RELU2) *(uint2*)(A.dg + rb + c + q4) = v1[j];
      }
    }
  }
};

// Output tiles [BM x BN] of one product. WM x WN waves; a wave holds
// (BM / WM) x (BN / WN) outputs as 16x16 blocks whose columns are the output's
// rows, so a lane has four consecutive columns of one row.
//
// Workgroups take units (a tile, or a part of a split tile's sum) in turn. Loads run NS steps of
// 64 ahead of the products, through the end of a unit into the next one, so
// only a workgroup's first unit waits for memory and an epilogue's stores and
// reads overlap the next unit's loads. A unit that is one of several parts
// writes its float32 partial output, in the order of the accumulators, and
// k_ffn_join adds the parts in order.
template <int KIND, bool RELU2, int BM, int BN, int WM, int WN, int NS>
__device__ __forceinline__ void run_units(const FfnArgs& A, const TileGrid& G, int block, int grid) {
  constexpr int NW = WM * WN;
  constexpr bool kDW = KIND == K_DWI || KIND == K_DWD;
  constexpr bool kAT = kDW, kBT = kDW || KIND == K_UP || KIND == K_DOWN;
  constexpr bool kDual = KIND == K_UP && !RELU2;  // gate and up columns side by side in the tile
  constexpr int kPh = KIND == K_DX && !RELU2 ? 2 : 1;
  constexpr int kMats = KIND == K_DWI && !RELU2 ? 2 : 1;  // dWg, dWu
  constexpr int BC = kDual ? BN / 2 : BN;         // output columns of a tile
  constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int kStage = (BM + BN) * 128;
  typedef Operand<BM, kAT, NW> OpA;
  typedef Operand<BC, kBT, NW> OpB;
  extern __shared__ __align__(1024) char smem[];
  int* cum = reinterpret_cast<int*>(smem + NS * kStage);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave / WN, wn = wave % WN;
  const int H = A.H, I = A.I;
  const int nout = KIND == K_UP || KIND == K_DH || KIND == K_DWI ? I : H;
  const int mout = KIND == K_DWI ? H : I;             // rows of a weight gradient
  const int ksum = KIND == K_UP || KIND == K_DH ? H : I;  // (row products)
  const int lda = kDW ? mout : ksum, ldb = kBT ? nout : ksum;
  const int64_t astep = kAT ? (int64_t)64 * lda * 2 : 128, bstep = kBT ? (int64_t)64 * ldb * 2 : 128;

  // units of this workgroup: workgroups go round robin over the 8 XCDs; an XCD
  // takes runs of neighbouring tiles, which share operands in its L2
  const int rows = kDW ? G.row_tiles : count_tiles(A, BM, cum);  // row tiles
  const uint32_t inv = last_band(G, rows);
  const int tiles = rows * G.col_tiles * (kDW ? kMats * A.E : 1), full = G.split > 1 ? G.full : tiles;
  const int rest = tiles - full, units = full + rest * G.split;
  const int per = grid >> 3;
  const int stride = grid, first = (block & 7) * per + (block >> 3);

  // Where the loads of a unit are: the next step's operands, the bytes that
  // they may read (a resource ends with its operand: what lies past it is
  // zero), and the steps. Operands with the sum along memory rows have `na` (nb)
  // bytes from there to the end of the tile's last row; those with the sum down
  // the columns have `rows` memory rows left.
  struct Unit {
    const char *a, *b, *a1, *b1;
    int na, nb, na0, nb0, rows;
    int k, kend, kt1;  // next step, end, and steps of a phase
  };
  auto where = [&](int u, int& slot, int& part, int& parts) {
    int id = u;
    slot = -1;
    part = 0;
    parts = 1;
    if (u >= full) {
      slot = u - full;
      part = slot / rest;
      parts = G.split;
      id = full + slot - part * rest;
    }
    return place<KIND, RELU2, BM, BN>(A, G, cum, rows, inv, id);
  };
  auto setup = [&](int u, Unit& U) {
    int slot, part, parts;
    const Place p = where(u, slot, part, parts);
    if constexpr (kDW) {
      // (a scalar load: a vector load's wait would be one for the stores of the
      // unit before, too)
      int lo = 0, hi = A.N;
      if (A.off) {
        const auto* off = (const __attribute__((address_space(4))) int32_t*)A.off;
        lo = clampi(off[p.e], 0, A.N);
        hi = clampi(off[p.e + 1], lo, A.N);
      }
      U.rows = hi - lo;
      U.a = (const char*)((KIND == K_DWD ? A.h : A.x) + (int64_t)lo * lda + p.row);
      U.b = (const char*)((KIND == K_DWD ? A.dy : p.mat ? A.du : A.dg) + (int64_t)lo * ldb + p.n0);
      U.na0 = p.row * 2;  // (bytes of a memory row before the tile)
      U.nb0 = p.n0 * 2;
      U.kt1 = U.rows > 0 ? (U.rows + 63) >> 6 : 1;  // a group without rows: one step of zeros
    } else {
      const int64_t ar = (int64_t)p.row * lda;
      const int64_t w = (int64_t)p.e * H * I + (kBT ? p.n0 : (int64_t)p.n0 * ldb);
      U.a = (const char*)((KIND == K_UP ? A.x : KIND == K_DOWN ? A.h : KIND == K_DH ? A.dy : kPh == 2 ? A.dg : A.du) + ar);
      U.b = (const char*)((KIND == K_UP || KIND == K_DX ? (RELU2 ? A.Wu : A.Wg) : A.Wd) + w);
      U.na0 = min(p.end - p.row, BM) * lda * 2;
      U.nb0 = kBT ? p.n0 * 2 : min(nout - p.n0, BN) * ldb * 2;
      if constexpr (kPh == 2) U.a1 = (const char*)(A.du + ar);
      if constexpr (kPh == 2 || kDual) U.b1 = (const char*)(A.Wu + w);
      U.rows = ksum;
      U.kt1 = (ksum + 63) >> 6;
    }
    const int64_t all = (int64_t)U.kt1 * kPh;
    U.k = (int)(all * part / parts);
    U.kend = (int)(all * (part + 1) / parts);
    // to the first step
    const bool second = kPh == 2 && U.k >= U.kt1;
    const int k = second ? U.k - U.kt1 : U.k;
    if (second) {
      U.a = U.a1;
      U.b = U.b1;
    }
    U.a += k * astep;
    U.b += k * bstep;
    if constexpr (kDual) U.b1 += k * bstep;
    U.na = U.na0 - k * 128;
    U.nb = U.nb0 - k * 128;
    U.rows -= k * 64;
  };

  OpA opa;
  OpB opb;
  opa.init(wave, lda, kDW ? 0 : ksum);
  opb.init(wave, ldb, kDW ? 0 : ksum);
  const int abase = OpA::base(wm * (BM / WM));
  const int bbase = OpB::base(wn * (BC / WN));
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS char*)smem;

  // The loads: one step of the unit P into a stage. step_ahead() forms the
  // resources of the next step, fill() issues the wave's load q of it. Past the
  // last unit empty resources are loaded, so that every wave always has the
  // same number of loads in flight.
  int pu = first;
  Unit P;
  if (pu < units) setup(pu, P);
  constexpr int kLoads = OpA::kLoads + OpB::kLoads * (kDual ? 2 : 1);
  u32x4 ra, rb, rb1;
  bool last = false;
  auto step_ahead = [&]() {
    const bool some = pu < units;
    const int mem = P.rows < 64 ? P.rows : 64;  // memory rows of this step
    last = P.k == P.kt1 - 1 || P.k == P.kt1 * kPh - 1;
    ra = make_rsrc(P.a, !some ? 0 : kAT ? mem * lda * 2 - P.na0 : P.na);
    rb = make_rsrc(P.b, !some ? 0 : kBT ? mem * ldb * 2 - P.nb0 : P.nb);
    if constexpr (kDual) rb1 = make_rsrc(P.b1, !some ? 0 : mem * ldb * 2 - P.nb0);
    if (!some) return;
    ++P.k;
    P.a += astep;
    P.b += bstep;
    if constexpr (kDual) P.b1 += bstep;
    P.na -= 128;
    P.nb -= 128;
    P.rows -= 64;
    if (kPh == 2 && P.k == P.kt1) {
      P.a = P.a1;
      P.b = P.b1;
      P.na = P.na0;
      P.nb = P.nb0;
    }
    if (P.k == P.kend) {
      pu += stride;
      if (pu < units) setup(pu, P);
    }
  };
  auto fill = [&](int stage, int q) {
    const uint32_t buf = lds0 + stage * kStage;
    if (q < OpA::kLoads) opa.issue(ra, buf, wave, last, q);
    else if (q < OpA::kLoads + OpB::kLoads) opb.issue(rb, buf + BM * 128, wave, last, q - OpA::kLoads);
    else opb.issue(rb1, buf + (BM + BC) * 128, wave, last, q - OpA::kLoads - OpB::kLoads);
  };

  bf16x8 a0f[MF], b0f[NF], a1f[MF], b1f[NF];  // operands of the two halves of a step
  auto read1 = [&](int st, int kk, bf16x8(&a)[MF], bf16x8(&b)[NF], int q) {
    const char* la = smem + st * kStage;
    const char* lb = la + BM * 128;
    if (q >= NF) a[q - NF] = OpA::read(la, abase, q - NF, kk);
    else if constexpr (kDual) b[q] = OpB::read(lb + (q < NF / 2 ? 0 : BC * 128), bbase, q % (NF / 2), kk);
    else b[q] = OpB::read(lb, bbase, q, kk);
  };
  f32x4 acc[MF][NF];
  // Half a step: its products row by row, and between them the operand reads
  // of the next half (all issued in the first three quarters, so that they have
  // returned at its end) and, in the second half, the loads of a step ahead.
  auto half = [&](bf16x8(&a)[MF], bf16x8(&b)[NF], int st, int kk, bf16x8(&an)[MF], bf16x8(&bn)[NF], bool loads, int to) {
    constexpr int kR = MF + NF, kQ = MF > 2 ? MF - 1 : MF;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      if (loads)
#pragma unroll
        for (int q = kLoads * i / MF; q < kLoads * (i + 1) / MF; ++q) fill(to, q);
      if (i < kQ)
#pragma unroll
        for (int q = kR * i / kQ; q < kR * (i + 1) / kQ; ++q) read1(st, kk, an, bn, q);
#pragma unroll
      for (int j = 0; j < NF; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  typedef Emit<KIND, RELU2, NF> Out;
  auto epilogue = [&](const Place& C, int slot, int wrow, int wcol) {
    if (slot >= 0) {
      float* p = A.part + ((int64_t)slot * NW + wave) * (MF * NF * 256) + lane * 4;
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) *(f32x4*)(p + (i * NF + j) * 256) = acc[i][j];
      return;
    }
    // what a block row needs is read one block row ahead
    f32x4 in[2][Out::kIn][Out::kGu];
    Out::fetch(A, C, wrow, wcol, nout, in[0]);
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      if (wrow + i * 16 >= C.end) break;
      if (i + 1 < MF) Out::fetch(A, C, wrow + i * 16 + 16, wcol, nout, in[(i + 1) & 1]);
      Out::put(A, C, wrow + i * 16, wcol, nout, acc[i], in[i & 1]);
    }
  };

  if (first >= units) return;
#pragma unroll
  for (int st = 0; st < NS; ++st) {
    step_ahead();
#pragma unroll
    for (int q = 0; q < kLoads; ++q) fill(st, q);
  }
  step_ahead();
  wait_loads<(NS - 1) * kLoads>();
  auto read_first = [&](int st) {
#pragma unroll
    for (int q = 0; q < MF + NF; ++q) read1(st, 0, a0f, b0f, q);
  };
  read_first(0);
  // Stores of an epilogue whose outputs all lie inside (at least: kept
  // projections and partial sums are more). Memory operations complete in the
  // order they were issued, and the loads of a unit's second step are older
  // than the stores of the unit before: the wait for them need not wait for
  // those stores.
  constexpr int kOutBlocks = kDual ? NF / 2 : NF;
  constexpr int kStores = MF * (kOutBlocks > 1 ? kOutBlocks / 2 : 1) * (KIND == K_DH && !RELU2 ? 2 : 1);
  constexpr int kBehind = (NS - 2) * kLoads;
  constexpr int kBehindStores = kBehind + kStores < 63 ? kBehind + kStores : 63;
  bool stored = false;
  int stage = 0;
  for (int u = first; u < units; u += stride) {
    int slot, part, parts;
    const Place C = where(u, slot, part, parts);
    int steps;  // of this unit
    {
      int kt1 = (ksum + 63) >> 6;
      if constexpr (kDW) {
        int lo = 0, hi = A.N;
        if (A.off) {
          const auto* off = (const __attribute__((address_space(4))) int32_t*)A.off;
          lo = clampi(off[C.e], 0, A.N);
          hi = clampi(off[C.e + 1], lo, A.N);
        }
        kt1 = hi > lo ? (hi - lo + 63) >> 6 : 1;
      }
      const int64_t all = (int64_t)kt1 * kPh;
      steps = (int)(all * (part + 1) / parts) - (int)(all * part / parts);
    }
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wrow = C.row + wm * (BM / WM), wcol = C.n0 + wn * (BC / WN);
    if (wrow < C.end && wcol < nout) {
      for (int kt = 0; kt < steps; ++kt) {
        half(a0f, b0f, stage, 1, a1f, b1f, false, 0);
        // the next step has landed, and this step's stage has been read by every wave
        if (kDW && stored) wait_loads<kBehindStores>();
        else wait_loads<kBehind>();
        stored = false;
        const int next = stage == NS - 1 ? 0 : stage + 1;
        half(a1f, b1f, next, 0, a0f, b0f, true, stage);
        stage = next;
        step_ahead();
      }
    } else {  // a wave whose outputs lie past the end only loads
      stored = false;
      for (int kt = 0; kt < steps; ++kt) {
        wait_loads<kBehind>();
#pragma unroll
        for (int q = 0; q < kLoads; ++q) fill(stage, q);
        stage = stage == NS - 1 ? 0 : stage + 1;
        step_ahead();
      }
      read_first(stage);
      continue;
    }

    epilogue(C, slot, wrow, wcol);
    stored = wrow + BM / WM <= C.end && wcol + BC / WN <= nout;
    read_first(stage);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): no load to LDS outlives the workgroup
}

template <int KIND, bool RELU2, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_ffn(const FfnArgs A, const TileGrid G) {
  run_units<KIND, RELU2, BM, BN, WM, WN, NS>(A, G, blockIdx.x, gridDim.x);
}

// The three products behind dg and du in one launch, for the smallest problems,
// whose launches are most of their time (33 rows, 256 x 128: a training step 44.6
// -> 36.6 us; this kernel 5.7):
// `at` workgroups for the first, up to at[1] for the second.
struct GradGrids {
  TileGrid g[3];
  int at[3];
};
template <bool RELU2, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_ffn_grads(const FfnArgs A, const GradGrids S) {
  const int b = blockIdx.x;
  if (b < S.at[0]) run_units<K_DX, RELU2, BM, BN, WM, WN, NS>(A, S.g[0], b, S.at[0]);
  else if (b < S.at[1]) run_units<K_DWI, RELU2, BM, BN, WM, WN, NS>(A, S.g[1], b - S.at[0], S.at[1] - S.at[0]);
  else run_units<K_DWD, RELU2, BM, BN, WM, WN, NS>(A, S.g[2], b - S.at[1], S.at[2] - S.at[1]);
}

// Sums of the parts of split tiles, in order, and their epilogue: a workgroup
// per tile and row of blocks, with the waves of the tile. Bound by latency (16 rows,
// 14336 -> 4096, eight parts: 4.8 us) or by the parts' bytes (1000 rows, 11008 -> 4096:
// 12 us). Joining in a launch of its own keeps the order of the sum and any waiting
// between workgroups out.
template <int KIND, bool RELU2, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_ffn_join(const FfnArgs A, const TileGrid G) {
  constexpr bool kDW = KIND == K_DWI || KIND == K_DWD;
  constexpr int NW = WM * WN, MF = BM / WM / 16, NF = BN / WN / 16, BC = KIND == K_UP && !RELU2 ? BN / 2 : BN;
  extern __shared__ __align__(16) int cum_[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int nout = KIND == K_UP || KIND == K_DH || KIND == K_DWI ? A.I : A.H;
  const int rows = kDW ? G.row_tiles : count_tiles(A, BM, cum_);
  const int rest = rows * G.col_tiles * (kDW ? (KIND == K_DWI && !RELU2 ? 2 : 1) * A.E : 1) - G.full, tile = blockIdx.x, i = blockIdx.y;
  if (tile >= rest) return;
  const Place P = place<KIND, RELU2, BM, BN>(A, G, cum_, rows, last_band(G, rows), G.full + tile);
  const int row16 = P.row + wave / WN * (BM / WM) + i * 16, wcol = P.n0 + wave % WN * (BC / WN);
  if (row16 >= P.end || wcol >= nout) return;
  typedef Emit<KIND, RELU2, NF> Out;
  f32x4 in[Out::kIn][Out::kGu];
  Out::fetch(A, P, row16, wcol, nout, in);
  const float* p = A.part + ((int64_t)tile * NW + wave) * (MF * NF * 256) + i * NF * 256 + lane * 4;
  const int64_t step = (int64_t)rest * NW * MF * NF * 256;
  f32x4 acc[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < G.split; s0 += 4) {  // four parts' loads at once; a part past the end is read as the last
    f32x4 v[4][NF];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < NF; ++j) v[k][j] = *(const f32x4*)(p + step * (s0 + k < G.split ? s0 + k : G.split - 1) + j * 256);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (s0 + k >= G.split) break;
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[j] += v[k][j];
    }
  }
  Out::put(A, P, row16, wcol, nout, acc, in);
}

// Grid of a product: its tiles, the number of workgroups and their LDS.
struct Launch {
  TileGrid G;
  int64_t units, rest;
  int grid;
  size_t list, lds;  // of the groups' list, and of all
};

template <int KIND, bool RELU2, int TILE>
Launch plan(const FfnArgs& A, const FfnProduct& p, const FfnChoice& c, int cus) {
  constexpr FfnTile T = kFfnTiles[TILE];
  constexpr int BM = T.bm, BN = T.bn;
  constexpr bool kDW = KIND == K_DWI || KIND == K_DWD;
  constexpr int BC = KIND == K_UP && !RELU2 ? BN / 2 : BN;
  Launch L;
  L.G.col_tiles = (p.cols + BC - 1) / BC;
  L.G.row_tiles = kDW ? (int)((p.rows + BM - 1) / BM) : 0;
  // 8 row tiles (4 of both gradients): 12 tiles of operands for 32 products. Against
  // bands of one row tile, dW of gate/up and of down, us: 48 experts of 2688 x 1856,
  // sums of 1 step 257 and 134 -> 235 and 131, of 8 steps 631 and 325 -> 570 and 330;
  // 64 of 2048 x 1024, 8 steps 342 and 170 -> 339 and 169; 4096 x 11008, 128 steps
  // 1175 and 624 -> 1076 and 584. Only one group of few rows is slower (33 rows of
  // 4096 x 11008: 42 -> 45).
  L.G.band_log = p.mats == 2 ? 2 : 3;
  L.G.band = Divisor((int64_t)L.G.col_tiles << L.G.band_log);
  L.G.group = Divisor(std::max<int64_t>(1, (int64_t)L.G.row_tiles * L.G.col_tiles * p.mats));
  // at most this many tiles (groups end inside tiles); the kernel counts them
  const int64_t tiles = ffn_tiles(p, T);
  L.rest = c.split > 1 ? tiles - c.full : 0;
  L.units = tiles + L.rest * (c.split - 1);
  L.G.full = (int)c.full;
  L.G.split = c.split;
  L.list = p.list;
  L.lds = ffn_lds(T, L.list);
  const int64_t most = (int64_t)cus * ffn_resident(T, L.list);
  L.grid = (int)((std::min(L.units, most) + 7) / 8 * 8);
  return L;
}

template <int KIND, bool RELU2, int TILE>
hipError_t run(const FfnArgs& A, const FfnProduct& p, const FfnChoice& c, int cus, hipStream_t s) {
  constexpr FfnTile T = kFfnTiles[TILE];
  constexpr int kThreads = 64 * T.wm * T.wn;
  const Launch L = plan<KIND, RELU2, TILE>(A, p, c, cus);
  if (L.units == 0) return hipSuccess;
  if (L.units > 0x40000000) return hipErrorInvalidValue;
  k_ffn<KIND, RELU2, T.bm, T.bn, T.wm, T.wn, T.stages><<<dim3(L.grid), dim3(kThreads), L.lds, s>>>(A, L.G);
  hipError_t e = hipGetLastError();
  if (L.rest == 0 || e != hipSuccess) return e;
  k_ffn_join<KIND, RELU2, T.bm, T.bn, T.wm, T.wn><<<dim3((unsigned)L.rest, T.bm / T.wm / 16), dim3(kThreads), L.list, s>>>(A, L.G);
  return hipGetLastError();
}

template <int KIND, bool RELU2>
hipError_t run_kind(const FfnArgs& A, int cus, hipStream_t s) {
  const FfnProduct p = ffn_product((FfnKind)KIND, A.N, A.E, A.H, A.I, !RELU2, A.off != nullptr);
  const FfnChoice c = choose_ffn(p, cus);
  switch (c.tile) {
    case 0: return run<KIND, RELU2, 0>(A, p, c, cus, s);
    case 1: return run<KIND, RELU2, 1>(A, p, c, cus, s);
    case 2: return run<KIND, RELU2, 2>(A, p, c, cus, s);
    case 3: return run<KIND, RELU2, 3>(A, p, c, cus, s);
    case 4: return run<KIND, RELU2, 4>(A, p, c, cus, s);
    default: return run<KIND, RELU2, 5>(A, p, c, cus, s);
  }
}

// dx and the weights' gradients. Where all three products take the smallest
// tile unsplit they share a launch, which is most of such a call's time.
template <bool RELU2>
hipError_t run_grads(const FfnArgs& A, int cus, hipStream_t s) {
  const FfnKind kinds[3] = {K_DX, K_DWI, K_DWD};
  FfnProduct p[3];
  FfnChoice c[3];
  bool one = A.N > 0 && A.dx && A.dWu && A.dWd;
  for (int i = 0; i < 3; ++i) {
    p[i] = ffn_product(kinds[i], A.N, A.E, A.H, A.I, !RELU2, A.off != nullptr);
    c[i] = choose_ffn(p[i], cus);
    one = one && c[i].tile == kFfnTileCount - 1 && c[i].split == 1;
  }
  if (one) {
    constexpr int kLast = kFfnTileCount - 1;
    constexpr FfnTile T = kFfnTiles[kLast];
    const Launch L[3] = {plan<K_DX, RELU2, kLast>(A, p[0], c[0], cus), plan<K_DWI, RELU2, kLast>(A, p[1], c[1], cus),
                         plan<K_DWD, RELU2, kLast>(A, p[2], c[2], cus)};
    GradGrids S;
    int at = 0;
    for (int i = 0; i < 3; ++i) {
      if (L[i].units > 0x40000000) return hipErrorInvalidValue;
      S.g[i] = L[i].G;
      S.at[i] = at += L[i].grid;
    }
    k_ffn_grads<RELU2, T.bm, T.bn, T.wm, T.wn, T.stages><<<dim3(at), dim3(64 * T.wm * T.wn), L[0].lds, s>>>(A, S);
    return hipGetLastError();
  }
  hipError_t e = A.N > 0 && A.dx ? run_kind<K_DX, RELU2>(A, cus, s) : hipSuccess;
  if (e == hipSuccess && A.dWu) e = run_kind<K_DWI, RELU2>(A, cus, s);
  if (e == hipSuccess && A.dWd) e = run_kind<K_DWD, RELU2>(A, cus, s);
  return e;
}

template <int KIND>
hipError_t run_act(const FfnArgs& A, int cus, hipStream_t s) {
  return A.relu2 ? run_kind<KIND, true>(A, cus, s) : run_kind<KIND, false>(A, cus, s);
}

// ---------------------------------------------------------------------------
// Few rows through one small matrix set: the latency of two launches is most
// of the time (one row, 2048 x 1408: 4.7 and 5.7 us; a call through the tiles took
// 23 us where one through these kernels took 15). The weights go from memory to the matrix operands without LDS.
// A workgroup has 32 output columns (of both projections for gated experts),
// its NW waves take the sum's steps of 32 in turn. A lane reads two neighbouring
// columns of eight rows of a step, and byte permutations turn them into two
// operands of eight sum elements of one column; x comes as 16-byte row pieces.
// The waves' partial outputs are added in order through LDS.
// ---------------------------------------------------------------------------
//
// Where the groups of columns are fewer than the CUs, gridDim.y workgroups of
// the first product share a group's sum (PART) and leave their partial
// projections; each of the second product's workgroups adds them, in order,
// and forms h in LDS: no launch in between.
template <int KIND, bool RELU2, int MB, int NW, bool PART>
__global__ __launch_bounds__(64 * NW, NW / 4) void k_ffn_few(const FfnArgs A, int split) {
  constexpr bool kDual = KIND == K_UP && !RELU2;
  constexpr int CW = 2;  // neighbouring columns of a lane
  constexpr int NM = kDual ? 2 : 1, kCols = 16 * CW, kPad = kCols + CW;
  constexpr int kAhead = 2;  // steps of a wave whose loads are in flight
  __shared__ float red[NW][NM][16 * kPad];
  extern __shared__ __align__(16) uint16_t hidden[];  // [N][I] (second product, PART)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n16 = lane & 15, kg = lane >> 4;
  const int nout = KIND == K_UP ? A.I : A.H, ksum = KIND == K_UP ? A.H : A.I;
  // neighbouring columns, which may share memory lines, go to one XCD
  const int groups = (nout + kCols - 1) / kCols, per = (gridDim.x + 7) >> 3;
  const int grp = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (grp >= groups) return;
  const int c0 = grp * kCols;
  const int all = ksum >> 5, y = blockIdx.y;
  const int beg = KIND == K_UP && PART ? all * y / split : 0, steps = KIND == K_UP && PART ? all * (y + 1) / split : all;

  const auto res = [](const void* p, uint32_t n) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)n, 0x00020000);
  };
  const uint32_t wbytes = (uint32_t)((size_t)ksum * nout * 2);
  const auto rw0 = res(KIND == K_UP ? (RELU2 ? A.Wu : A.Wg) : A.Wd, wbytes);
  const auto rw1 = res(A.Wu, wbytes);
  const auto rx = res(KIND == K_UP ? A.x : A.h, (uint32_t)((size_t)A.N * ksum * 2));
  const int col = c0 + n16 * CW;
  const uint32_t wv = col < nout ? (uint32_t)((kg * 8 * nout + col) * 2) : kOob;
  uint32_t xv[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) xv[b] = b * 16 + n16 < A.N ? (uint32_t)(((b * 16 + n16) * ksum + kg * 8) * 2) : kOob;

  uint32_t wb[kAhead][NM][8];
  u32x4 xb[kAhead][MB];
  auto load = [&](int slot, int st) {
    if (st >= steps) return;
    const uint32_t wo = (uint32_t)st * 32u * (uint32_t)nout * 2u;
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int m = 0; m < NM; ++m)
        wb[slot][m][r] = __builtin_amdgcn_raw_buffer_load_b32(m ? rw1 : rw0, (wv + (uint32_t)r * nout * 2) | (wv & kOob), wo, 0);
    if constexpr (!(KIND == K_DOWN && PART)) {
#pragma unroll
      for (int b = 0; b < MB; ++b) xb[slot][b] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, xv[b], st * 64, 0));
    }
  };
  f32x4 acc[NM][CW][MB];
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int c = 0; c < CW; ++c)
#pragma unroll
      for (int b = 0; b < MB; ++b) acc[m][c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int a = 0; a < kAhead; ++a) load(a, beg + wave + a * NW);
  if constexpr (KIND == K_DOWN && PART) {
    // h of all rows from the parts of its projections, while the weights are on their way
    constexpr int P = RELU2 ? 1 : 2;
    const int plane = A.N * ksum;
    for (int at = threadIdx.x * 4; at < plane; at += 64 * NW * 4) {
      f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = g;
      const float* p = A.part + at;
#pragma unroll 4
      for (int k = 0; k < split; ++k) {
        if constexpr (!RELU2) g += *(const f32x4*)p;
        u += *(const f32x4*)(p + (P - 1) * plane);
        p += P * plane;
      }
      *(uint2*)(hidden + at) = pack4(activate<RELU2>(g, u));
    }
    __syncthreads();
  }
  for (int st0 = beg + wave; st0 < steps; st0 += kAhead * NW) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      if (st0 + a * NW >= steps) break;
      if constexpr (KIND == K_DOWN && PART)  // rows past the last one are the last one's: not stored
        xb[a][0] = *(const u32x4*)(hidden + (n16 < A.N ? n16 : A.N - 1) * ksum + (st0 + a * NW) * 32 + kg * 8);
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int c = 0; c < CW; ++c) {
          u32x4 w;
#pragma unroll
          for (int d = 0; d < 4; ++d)
            w[d] = __builtin_amdgcn_perm(wb[a][m][2 * d + 1], wb[a][m][2 * d], c ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int b = 0; b < MB; ++b)
            acc[m][c][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, xb[a][b]), acc[m][c][b], 0, 0, 0);
        }
      load(a, st0 + (kAhead + a) * NW);
    }
  }

  // lane -> row (lane & 15) of a block of 16, columns kg * 4 CW + i CW + c
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (b * 16 >= A.N) break;
    if (b) __syncthreads();
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < CW; ++c) red[wave][m][n16 * kPad + kg * 4 * CW + i * CW + c] = acc[m][c][b][i];
    __syncthreads();
    for (int o = threadIdx.x; o < 16 * kCols; o += 64 * NW) {
      const int r = o / kCols, c = o % kCols, row = b * 16 + r;
      if (row >= A.N || c0 + c >= nout) continue;
      float s[NM];
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        s[m] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s[m] += red[w][m][r * kPad + c];
      }
      const int64_t at = (int64_t)row * nout + c0 + c;
      if constexpr (KIND == K_UP && PART) {
#pragma unroll
        for (int m = 0; m < NM; ++m) A.part[(int64_t)(y * NM + m) * A.N * nout + at] = s[m];
      } else if constexpr (KIND == K_UP) {
        const f32x4 g = {s[0], 0.f, 0.f, 0.f}, u = {s[NM - 1], 0.f, 0.f, 0.f};
        A.h[at] = (uint16_t)bf16_bits(activate<RELU2>(g, u)[0]);
        if (A.u) {
          if constexpr (!RELU2) A.g[at] = s[0];
          A.u[at] = s[NM - 1];
        }
      } else {
        A.y[at] = (uint16_t)bf16_bits(s[0]);
      }
    }
  }
}

template <bool RELU2, int MB, int NW, bool PART>
hipError_t run_few(const FfnArgs& A, int split, hipStream_t s) {
  const int up = (A.I + 31) / 32, down = (A.H + 31) / 32;
  k_ffn_few<K_UP, RELU2, MB, NW, PART><<<dim3((unsigned)((up + 7) / 8 * 8), split), dim3(64 * NW), 0, s>>>(A, split);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // without parts the activation is in h, and both kinds of experts are alike
  const size_t hidden = PART ? (size_t)A.N * A.I * 2 : 0;
  k_ffn_few<K_DOWN, RELU2 && PART, MB, NW, PART><<<dim3((unsigned)((down + 7) / 8 * 8)), dim3(64 * NW), hidden, s>>>(A, split);
  return hipGetLastError();
}

template <bool RELU2>
hipError_t run_few_act(const FfnArgs& A, int cus, hipStream_t s) {
  const int split = A.u ? 1 : few_split(A.N, A.H, A.I, cus);
  if (split > 1) return run_few<RELU2, 1, 16, true>(A, split, s);
  if (A.N <= 16) return run_few<RELU2, 1, 16, false>(A, 1, s);
  return A.N <= 32 ? run_few<RELU2, 2, 8, false>(A, 1, s) : run_few<RELU2, 4, 8, false>(A, 1, s);
}

hipError_t device_cus(int* cus) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  return e != hipSuccess ? e : hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
}

}  // namespace

hipError_t launch_ffn_forward(const FfnArgs& A, hipStream_t s) {
  int cus = 0;
  hipError_t e = device_cus(&cus);
  if (few_rows(A.N, A.H, A.I, A.off != nullptr)) {
    if (e == hipSuccess) e = A.relu2 ? run_few_act<true>(A, cus, s) : run_few_act<false>(A, cus, s);
    return e;
  }
  if (e == hipSuccess) e = run_act<K_UP>(A, cus, s);
  if (e == hipSuccess) e = run_act<K_DOWN>(A, cus, s);
  return e;
}

hipError_t launch_ffn_backward(const FfnArgs& A, hipStream_t s) {
  int cus = 0;
  hipError_t e = device_cus(&cus);
  if (e == hipSuccess && A.N > 0 && (A.dx || A.dWu)) e = run_act<K_DH>(A, cus, s);
  if (e == hipSuccess) e = A.relu2 ? run_grads<true>(A, cus, s) : run_grads<false>(A, cus, s);
  return e;
}

}  // namespace cardan
