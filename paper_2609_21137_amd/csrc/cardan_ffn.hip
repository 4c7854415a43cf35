// Feed-forward block of dense bf16 weights, forward and backward, for one
// matrix set or for the row groups of E experts.
//
//   h = silu(x Wg) * (x Wu)   (or max(x Wu, 0)^2),   y = h Wd
//   dh = dy Wd^T, dg = dh u s(1 + g(1 - s)), du = dh g s,  s = 1 / (1 + e^-g)
//   dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  dWd = h^T dy
//
// Every product runs on v_mfma_f32_16x16x32_bf16 with float32 accumulators.
#include <hip/hip_runtime.h>

#include "cardan_ffn.h"

namespace cardan {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
#define LDS __attribute__((address_space(3)))

constexpr uint32_t kOob = 0x80000000u;     // an offset past every resource
constexpr uint32_t kSpan = 0x7fffff00u;    // largest resource

// The products of the block. "rows" are the rows of a group (tokens).
enum Kind {
  K_UP = 0,    // [rows, H] x [H, I] (gate and up): activation -> h, and g, u where kept
  K_DOWN = 1,  // [rows, I] x [I, H] -> y
  K_DH = 2,    // [rows, H] x Wd^T -> dh, turned into dg, du
  K_DX = 3,    // dg Wg^T + du Wu^T -> dx
  K_DW = 4     // x^T dg, x^T du, h^T dy: the sum runs over the group's rows
};

__device__ __forceinline__ rsrc_t make_rsrc(const void* base, int64_t bytes) {
  const uint32_t n = bytes <= 0 ? 0u : bytes > (int64_t)kSpan ? kSpan : (uint32_t)bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)n, 0x00020000);
}

// float32 -> bf16, nearest even (NaN stays NaN)
__device__ __forceinline__ uint32_t bf16_bits(float f) {
  const __bf16 b = (__bf16)f;
  return (uint32_t)__builtin_bit_cast(unsigned short, b);
}
__device__ __forceinline__ uint2 pack4(f32x4 v) {
  return make_uint2(bf16_bits(v[0]) | bf16_bits(v[1]) << 16, bf16_bits(v[2]) | bf16_bits(v[3]) << 16);
}

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

// Group and first row of row tile t, tiles of BM rows counted group by group.
template <int BM>
__device__ __forceinline__ bool locate(const FfnArgs& A, int t, int& e, int& row, int& end) {
  if (!A.off) {
    e = 0;
    row = t * BM;
    end = A.N;
    return row < A.N;
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < A.E; e0 += 64) {
    int lo = 0, hi = 0;
    if (e0 + lane < A.E) group_rows(A, e0 + lane, lo, hi);
    const int tiles = (hi - lo + BM - 1) / BM;
    int cum = tiles;
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(cum, s);
      cum += lane >= s ? v : 0;
    }
    const unsigned long long past = __ballot(before + cum > t);
    if (past) {
      const int src = __ffsll((long long)past) - 1;
      e = e0 + src;
      const int first = __builtin_amdgcn_readlane(lo, src);
      end = __builtin_amdgcn_readlane(hi, src);
      row = first + (t - before - (__builtin_amdgcn_readlane(cum, src) - __builtin_amdgcn_readlane(tiles, src))) * BM;
      return true;
    }
    before += __builtin_amdgcn_readlane(cum, 63);
  }
  return false;
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
// of row k at place p ^ (k & 7): a transposing read takes four rows of a pair.
template <int R, bool TR, int NW>
struct Operand {
  static constexpr int kLoads = R / 8 / NW;     // loads of one wave per stage
  static constexpr int kRow = TR ? R * 2 : 128;  // bytes of an LDS row
  static constexpr int kPairs = TR ? (R / 16 < 8 ? R / 16 : 8) : 1;
  static_assert(R % (8 * NW) == 0, "whole loads");

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
        const int src = (((c >> 1) ^ (kk & (kPairs - 1))) << 1) | (c & 1);
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

  __device__ __forceinline__ void issue(rsrc_t rs, char* lds, int wave, bool last) const {
    const uint32_t drop = last && tail ? kOob : 0u;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS void*)(lds + (j * NW + wave) * 1024), 16,
                                               (int)(voff[j] | drop), 0, 0, 0);
  }

  // byte of the first operand read of the 16-row block that starts at row r0
  static __device__ __forceinline__ int base(int r0) {
    const int l = threadIdx.x & 63;
    if constexpr (TR) {
      const int a = (l & 15) >> 2, k = (l >> 4) * 8 + a;
      return k * kRow + ((r0 >> 4) ^ (a & (kPairs - 1))) * 32 + (l & 3) * 8;
    } else {
      return (r0 + (l & 15)) * 128 + ((l >> 4) ^ (l & 7)) * 16;
    }
  }
  // operand of step half kk (32 of 64) and block f after the one of `b`
  static __device__ __forceinline__ bf16x8 read(const char* lds, int b, int f, int kk) {
    if constexpr (TR) {
      const int at = (b ^ (f << 5)) + kk * 32 * kRow;
      const int at4 = (kPairs > 4 ? at ^ 128 : at) + 4 * kRow;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4*)(lds + at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS s16x4*)(lds + at4));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *(const bf16x8*)(lds + ((b ^ (kk << 6)) + f * 2048));
    }
  }
};

// s(g) = 1 / (1 + e^-g); e^-g overflows to infinity for g < -88 and gives 0
__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + __expf(-g)); }

// Output tile [BM x BN] of one product. WM x WN waves; a wave holds
// (BM / WM) x (BN / WN) outputs as 16x16 blocks whose columns are the output's
// rows, so a lane has four consecutive columns of one row.
template <int KIND, bool RELU2, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_ffn(const FfnArgs A) {
  constexpr int NW = WM * WN;
  constexpr bool kAT = KIND == K_DW, kBT = KIND == K_UP || KIND == K_DOWN || KIND == K_DW;
  constexpr bool kDual = KIND == K_UP && !RELU2;  // gate and up columns side by side in the tile
  constexpr int kPh = KIND == K_DX && !RELU2 ? 2 : 1;
  constexpr int BC = kDual ? BN / 2 : BN;         // output columns of a tile
  constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int kStage = (BM + BN) * 128;
  typedef Operand<BM, kAT, NW> OpA;
  typedef Operand<BC, kBT, NW> OpB;
  extern __shared__ __align__(1024) char smem[];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int H = A.H, I = A.I;

  // workgroups go round robin over the 8 XCDs: give each XCD a run of tiles
  const int total = gridDim.x;
  int id = blockIdx.x;
  {
    const int per = total >> 3, whole = per << 3;
    if (id < whole) id = (id & 7) * per + (id >> 3);
  }

  int e, row = 0, end = 0, n0, m0 = 0;
  const uint16_t *a0, *a1 = nullptr, *b0, *b1 = nullptr;
  uint16_t* out = nullptr;
  int lda, ldb, nout, ksum, mout = 0;
  int64_t abytes, bbytes;  // from a0 / b0 to the end of the operand
  if constexpr (KIND == K_DW) {
    // tiles of dWg, dWu ([H][I]) and dWd ([I][H]) of one group after another
    const int th = (H + BM - 1) / BM, ti = (I + BN - 1) / BN;
    const int ti2 = (I + BM - 1) / BM, th2 = (H + BN - 1) / BN;
    const int n_in = A.dWu ? th * ti * (RELU2 ? 1 : 2) : 0, n_dn = A.dWd ? ti2 * th2 : 0;
    e = id / (n_in + n_dn);
    int t = id - e * (n_in + n_dn);
    int lo, hi;
    group_rows(A, e, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    ksum = hi - lo;
    const bool down = t >= n_in;
    bool gate = false;
    if (down) t -= n_in;
    else if (!RELU2) {
      gate = t & 1;
      t >>= 1;
    }
    mout = down ? I : H;
    nout = down ? H : I;
    const int tn = down ? th2 : ti;
    m0 = t / tn * BM;
    n0 = t % tn * BN;
    lda = mout;
    ldb = nout;
    a0 = (down ? A.h : A.x) + (int64_t)lo * lda + m0;
    b0 = (down ? A.dy : gate ? A.dg : A.du) + (int64_t)lo * ldb + n0;
    abytes = ((int64_t)ksum * lda - m0) * 2;
    bbytes = ((int64_t)ksum * ldb - n0) * 2;
    out = (down ? A.dWd : gate ? A.dWg : A.dWu) + (int64_t)e * H * I;
  } else {
    nout = KIND == K_UP || KIND == K_DH ? I : H;
    ksum = KIND == K_UP || KIND == K_DH ? H : I;
    const int tn = (nout + BC - 1) / BC, tm = total / tn;
    // 8 row tiles by all column tiles at a time: a run of neighbours shares
    // its operands in the XCD's L2
    const int band = id / (8 * tn), in = id - band * 8 * tn;
    const int rows8 = tm - band * 8 < 8 ? tm - band * 8 : 8;
    const int t = band * 8 + in % rows8;
    n0 = in / rows8 * BC;
    if (!locate<BM>(A, t, e, row, end)) return;
    row = __builtin_amdgcn_readfirstlane(row);
    lda = ksum;
    abytes = (int64_t)(end - row) * lda * 2;
    const int64_t w = (int64_t)e * H * I, ar = (int64_t)row * lda;
    a0 = (KIND == K_UP ? A.x : KIND == K_DOWN ? A.h : KIND == K_DH ? A.dy : kPh == 2 ? A.dg : A.du) + ar;
    const uint16_t* wt = KIND == K_UP || KIND == K_DX ? (RELU2 ? A.Wu : A.Wg) : A.Wd;
    if constexpr (kBT) {  // weights [ksum][nout]
      ldb = nout;
      b0 = wt + w + n0;
      bbytes = ((int64_t)ksum * ldb - n0) * 2;
    } else {              // weights [nout][ksum]
      ldb = ksum;
      b0 = wt + w + (int64_t)n0 * ldb;
      bbytes = (int64_t)(nout - n0) * ldb * 2;
    }
    if constexpr (kDual) b1 = A.Wu + (b0 - A.Wg);
    if constexpr (kPh == 2) {
      a1 = A.du + ar;
      b1 = A.Wu + (b0 - A.Wg);
    }
  }

  OpA opa;
  OpB opb;
  opa.init(wave, lda, ksum);
  opb.init(wave, ldb, ksum);
  const int wm = wave / WN, wn = wave % WN;
  const int abase = OpA::base(wm * (BM / WM));
  const int bbase = OpB::base(wn * (BC / WN));

  f32x4 acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int kt1 = (ksum + 63) >> 6, kts = kt1 * kPh;
  const int64_t astep = kAT ? (int64_t)64 * lda * 2 : 128, bstep = kBT ? (int64_t)64 * ldb * 2 : 128;
  auto issue = [&](int kt) {
    char* buf = smem + (kt & 1) * kStage;
    const int ph = kPh == 2 && kt >= kt1, k = kt - (ph ? kt1 : 0);
    const bool last = k == kt1 - 1;
    const int64_t ao = k * astep, bo = k * bstep;
    opa.issue(make_rsrc((const char*)(ph ? a1 : a0) + ao, abytes - ao), buf, wave, last);
    opb.issue(make_rsrc((const char*)(ph ? b1 : b0) + bo, bbytes - bo), buf + BM * 128, wave, last);
    if constexpr (kDual)
      opb.issue(make_rsrc((const char*)b1 + bo, bbytes - bo), buf + (BM + BC) * 128, wave, last);
  };
  if (kts > 0) issue(0);
  for (int kt = 0; kt < kts; ++kt) {
    __syncthreads();  // stage kt has landed, and no wave reads the other stage any more
    if (kt + 1 < kts) issue(kt + 1);
    const char* la = smem + (kt & 1) * kStage;
    const char* lb = la + BM * 128;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 a[MF], b[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        if constexpr (kDual)
          b[j] = OpB::read(lb + (j < NF / 2 ? 0 : BC * 128), bbase, j % (NF / 2), kk);
        else
          b[j] = OpB::read(lb, bbase, j, kk);
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) a[i] = OpA::read(la, abase, i, kk);
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
    }
  }

  // epilogue: lane -> output row (lane & 15) of a block, columns (lane >> 4) * 4 + 0..3
  const int rmax = KIND == K_DW ? mout : end;
  const int r0 = (KIND == K_DW ? m0 : row) + wm * (BM / WM) + (lane & 15);
  const int c0 = n0 + wn * (BC / WN) + (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int r = r0 + i * 16;
    if (r >= rmax) continue;
    const int64_t rb = (int64_t)r * nout;
    if constexpr (KIND == K_UP) {
      constexpr int NC = kDual ? NF / 2 : NF;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = c0 + j * 16;
        if (c >= nout) continue;
        f32x4 h;
        const f32x4 u = acc[i][kDual ? j + NC : j];
        if constexpr (RELU2) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float p = fmaxf(u[q], 0.f);
            h[q] = p * p;
          }
        } else {
          const f32x4 g = acc[i][j];
#pragma unroll
          for (int q = 0; q < 4; ++q) h[q] = g[q] * sigmoid(g[q]) * u[q];
          if (A.g) *(f32x4*)(A.g + rb + c) = g;
        }
        if (A.u) *(f32x4*)(A.u + rb + c) = u;
        *(uint2*)(A.h + rb + c) = pack4(h);
      }
    } else if constexpr (KIND == K_DH) {
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int c = c0 + j * 16;
        if (c >= nout) continue;
        const f32x4 dh = acc[i][j], u = *(const f32x4*)(A.u + rb + c);
        f32x4 du;
        if constexpr (RELU2) {
#pragma unroll
          for (int q = 0; q < 4; ++q) du[q] = dh[q] * 2.f * fmaxf(u[q], 0.f);
        } else {
          const f32x4 g = *(const f32x4*)(A.g + rb + c);
          f32x4 dg;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float s = sigmoid(g[q]);
            dg[q] = dh[q] * u[q] * s * (1.f + g[q] * (1.f - s));
            du[q] = dh[q] * g[q] * s;
          }
          *(uint2*)(A.dg + rb + c) = pack4(dg);
        }
        *(uint2*)(A.du + rb + c) = pack4(du);
      }
    } else {
      uint16_t* o = KIND == K_DW ? out : KIND == K_DOWN ? A.y : A.dx;
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int c = c0 + j * 16;
        if (c < nout) *(uint2*)(o + rb + c) = pack4(acc[i][j]);
      }
    }
  }
}

template <int KIND, bool RELU2, int BM, int BN, int WM, int WN>
hipError_t run(const FfnArgs& A, hipStream_t s) {
  constexpr bool kDual = KIND == K_UP && !RELU2;
  constexpr int BC = kDual ? BN / 2 : BN;
  constexpr size_t lds = (size_t)2 * (BM + BN) * 128;
  int64_t grid;
  if (KIND == K_DW) {
    const int64_t th = (A.H + BM - 1) / BM, ti = (A.I + BN - 1) / BN, ti2 = (A.I + BM - 1) / BM, th2 = (A.H + BN - 1) / BN;
    grid = A.E * ((A.dWu ? th * ti * (RELU2 ? 1 : 2) : 0) + (A.dWd ? ti2 * th2 : 0));
  } else {
    const int nout = KIND == K_UP || KIND == K_DH ? A.I : A.H;
    const int64_t tm = A.off ? A.N / BM + (A.E < A.N ? A.E : A.N) : (A.N + BM - 1) / BM;
    grid = tm * ((nout + BC - 1) / BC);
  }
  if (grid == 0) return hipSuccess;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  k_ffn<KIND, RELU2, BM, BN, WM, WN><<<dim3((unsigned)grid), dim3(64 * WM * WN), lds, s>>>(A);
  return hipGetLastError();
}

template <int KIND>
hipError_t run_kind(const FfnArgs& A, hipStream_t s) {
  return A.relu2 ? run<KIND, true, 256, 256, 2, 4>(A, s) : run<KIND, false, 256, 256, 2, 4>(A, s);
}

}  // namespace

hipError_t launch_ffn_forward(const FfnArgs& A, hipStream_t s) {
  hipError_t e = run_kind<K_UP>(A, s);
  return e != hipSuccess ? e : run_kind<K_DOWN>(A, s);
}

hipError_t launch_ffn_backward(const FfnArgs& A, hipStream_t s) {
  hipError_t e = run_kind<K_DH>(A, s);
  if (e == hipSuccess && A.dx) e = run_kind<K_DX>(A, s);
  if (e == hipSuccess && (A.dWu || A.dWd)) e = run_kind<K_DW>(A, s);
  return e;
}

}  // namespace cardan
