// Rows of tokens to their experts' rows and back, with the gradients:
//   dispatch: xe[place[n][j]] = x[n]
//   combine:  y[n] = sum_j w[n][j] ye[place[n][j]], in the order of j
//   backward: dye[place[n][j]] = w[n][j] dy[n], dw[n][j] = <dy[n], ye[place[n][j]]>
// (the gradient of dispatch is combine without weights). Bound by the rows' bytes:
// 8192 x 8 rows of 2048 copied in 52 us (5.8 TB/s), combined in 60 (5.0), combine's
// gradients in 114 (5.0); counters show the floor's bytes and no others. A
// thread takes eight values of a row and goes through its k rows, so that a
// token's row is read once and its sum stays in registers; the gradients take a
// wave a row, whose inner products need no other one.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_rows.h"

namespace cardan {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A thread handles eight values at once. WIDE: every row starts on 16 bytes and
// has a multiple of eight; else accesses of 16 bytes start on any value, and a
// row's last values come one by one (3000 x 6 rows through all four calls: 105
// us at 2001 values, 96 at 2000).
constexpr int kVec = 8;
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));
template <bool WIDE> struct At { typedef u32x4_at2 bf16; typedef f32x4_at4 f32; };
template <> struct At<true> { typedef u32x4 bf16; typedef f32x4 f32; };

__device__ __forceinline__ void unpack(u32x4 v, float (&f)[kVec]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = __uint_as_float(v[q] << 16);
    f[2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack(const float (&f)[kVec]) {
  u32x4 v;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    v[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * q], f[2 * q + 1]}, bf16x2));
  return v;
}

// The values at position `at` of a row of bf16 or float32, zeros past its end.
// PAST: past the caches.
template <bool WIDE, bool F32, bool PAST = false>
__device__ __forceinline__ void load_row(const void* base, int64_t row, int H, int at, float (&f)[kVec]) {
  if constexpr (F32) {
    const float* p = static_cast<const float*>(base) + row * H + at;
    if (WIDE || at + kVec <= H) {
      typedef typename At<WIDE>::f32 V;
      const f32x4 a = *reinterpret_cast<const V*>(p), b = *reinterpret_cast<const V*>(p + 4);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f[q] = a[q];
        f[4 + q] = b[q];
      }
    } else {
#pragma unroll
      for (int q = 0; q < kVec; ++q) f[q] = at + q < H ? p[q] : 0.f;
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(base) + row * H + at;
    if (WIDE || at + kVec <= H) {
      typedef typename At<WIDE>::bf16 V;
      if constexpr (PAST) unpack(__builtin_nontemporal_load(reinterpret_cast<const V*>(p)), f);
      else unpack(*reinterpret_cast<const V*>(p), f);
    } else {
#pragma unroll
      for (int q = 0; q < kVec; ++q) f[q] = at + q < H ? __uint_as_float((uint32_t)p[q] << 16) : 0.f;
    }
  }
}
template <bool WIDE, bool F32, bool PAST = false>
__device__ __forceinline__ void store_row(void* base, int64_t row, int H, int at, const float (&f)[kVec]) {
  if constexpr (F32) {
    float* p = static_cast<float*>(base) + row * H + at;
    if (WIDE || at + kVec <= H) {
      typedef typename At<WIDE>::f32 V;
      *reinterpret_cast<V*>(p) = f32x4{f[0], f[1], f[2], f[3]};
      *reinterpret_cast<V*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
    } else {
#pragma unroll
      for (int q = 0; q < kVec; ++q)
        if (at + q < H) p[q] = f[q];
    }
  } else {
    uint16_t* p = static_cast<uint16_t*>(base) + row * H + at;
    if (WIDE || at + kVec <= H) {
      typedef typename At<WIDE>::bf16 V;
      if constexpr (PAST) __builtin_nontemporal_store(pack(f), reinterpret_cast<V*>(p));
      else *reinterpret_cast<V*>(p) = pack(f);
    } else {
#pragma unroll
      for (int q = 0; q < kVec; ++q)
        if (at + q < H) p[q] = __builtin_bit_cast(uint16_t, (__bf16)f[q]);
    }
  }
}

constexpr int kThreads = 256;
// A grouped array that the last-level cache (256 MB) does not keep is read and
// written past the caches, which leaves them to the tokens' rows: 65536 x 2048
// copied, combined and both gradients 286 us (about 50 more through the caches;
// combine 60 instead of 80). A smaller one, just written, is still there: 12282 x 2816
// combined in 14.6 us, past the caches 20.2. The array's size decides, also where a
// call touches few of its rows: 2000 x 8 of 65536 rows of 2048 copied in 13.5 us and
// combined in 15.6, through the caches 12.2 and 12.5; 16 x 8 of them no slower.
constexpr int64_t kPastBytes = (int64_t)192 << 20;

// The rows of a workgroup's threads. NT > 0: blockIdx.x is a run of a row's
// values, blockIdx.y rows, strided. NT == 0: rows of less than half a workgroup's
// values one behind the other (15138 x 2 rows of 92: copied in 5.1 us, combined in
// 4.9, with a workgroup a row 14.0 and 13.8). f(n, position).
template <int NT, class F>
__device__ __forceinline__ void each_row(const RowsArgs& A, F f) {
  if constexpr (NT > 0) {
    const int at = (blockIdx.x * NT + threadIdx.x) * kVec;
    if (at >= A.H) return;
    for (int64_t n = blockIdx.y; n < A.N; n += gridDim.y) f(n, at);
  } else {
    const int vecs = (A.H + kVec - 1) / kVec, rows = kThreads / vecs;
    const int r = threadIdx.x / vecs, at = (threadIdx.x - r * vecs) * kVec;
    if (r >= rows) return;
    for (int64_t n = (int64_t)blockIdx.x * rows + r; n < A.N; n += (int64_t)gridDim.x * rows) f(n, at);
  }
}

template <bool WIDE, bool PAST, int NT>
__global__ __launch_bounds__(NT ? NT : kThreads) void k_dispatch(const RowsArgs A) {
  typedef typename At<WIDE>::bf16 V;
  each_row<NT>(A, [&](int64_t n, int at) {
    const uint16_t* from = A.x + n * A.H + at;
    if (WIDE || at + kVec <= A.H) {
      const u32x4 v = *reinterpret_cast<const V*>(from);
      for (int j = 0; j < A.k; ++j) {
        const int p = A.place[n * A.k + j];
        if ((uint32_t)p >= (uint32_t)A.M) continue;
        V* to = reinterpret_cast<V*>(A.xe + (int64_t)p * A.H + at);
        if constexpr (PAST) __builtin_nontemporal_store(v, to);
        else *to = v;
      }
    } else {
      for (int j = 0; j < A.k; ++j) {
        const int p = A.place[n * A.k + j];
        if ((uint32_t)p >= (uint32_t)A.M) continue;
        for (int q = 0; at + q < A.H; ++q) A.xe[(int64_t)p * A.H + at + q] = from[q];
      }
    }
  });
}

template <bool WIDE, bool F32, bool PAST, int NT>
__global__ __launch_bounds__(NT ? NT : kThreads) void k_combine(const RowsArgs A) {
  each_row<NT>(A, [&](int64_t n, int at) {
    float sum[kVec];
#pragma unroll
    for (int q = 0; q < kVec; ++q) sum[q] = 0.f;
#pragma unroll 4
    for (int j = 0; j < A.k; ++j) {
      const int p = A.place[n * A.k + j];
      if ((uint32_t)p >= (uint32_t)A.M) continue;
      const float w = A.weight ? A.weight[n * A.k + j] : 1.0f;
      float f[kVec];
      load_row<WIDE, false, PAST>(A.ye, p, A.H, at, f);
#pragma unroll
      for (int q = 0; q < kVec; ++q) sum[q] = fmaf(w, f[q], sum[q]);
    }
    store_row<WIDE, F32>(A.y, n, A.H, at, sum);
  });
}

// A wave a row: the products of the row of dy with its k rows are summed over
// the wave's lanes, each in one order. A lane keeps up to KEEP runs of eight
// values of dy's row (read again for every one of the k rows, they came from
// memory: 509 MB instead of 302 for 65536 x 2048; 18000 x 2001 39 us, now 30).
// KEEP == 0: a wave a row and place, for few rows (2 x 7 rows of 6215: 9.4 us, with a wave a row 44.8).
template <bool WIDE, bool F32, bool PAST, int KEEP>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const RowsArgs A) {
  const int lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)gridDim.x * (kThreads / 64);
  const int64_t items = KEEP ? A.N : (int64_t)A.N * A.k;
  for (int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); item < items; item += waves) {
    const int64_t n = KEEP ? item : item / A.k;
    const int j0 = KEEP ? 0 : (int)(item - n * A.k), j1 = KEEP ? A.k : j0 + 1;
    float kept[KEEP ? KEEP : 1][kVec];
#pragma unroll
    for (int c = 0; c < KEEP; ++c) {
      const int at = (c * 64 + lane) * kVec;
      if (at < A.H) load_row<WIDE, F32>(A.dy, n, A.H, at, kept[c]);
    }
    for (int j = j0; j < j1; ++j) {
      const int p = A.place[n * A.k + j];
      float dot = 0.f;
      if ((uint32_t)p < (uint32_t)A.M) {
        const float w = A.weight ? A.weight[n * A.k + j] : 1.0f;
        const auto both = [&](int at, const float (&d)[kVec]) {
          if (A.dweight) {
            float f[kVec];
            load_row<WIDE, false, PAST>(A.ye, p, A.H, at, f);
#pragma unroll
            for (int q = 0; q < kVec; ++q) dot = fmaf(d[q], f[q], dot);
          }
          if (A.dye) {
            float g[kVec];
#pragma unroll
            for (int q = 0; q < kVec; ++q) g[q] = d[q] * w;
            store_row<WIDE, false, PAST>(A.dye, p, A.H, at, g);
          }
        };
#pragma unroll
        for (int c = 0; c < KEEP; ++c) {
          const int at = (c * 64 + lane) * kVec;
          if (at < A.H) both(at, kept[c]);
        }
#pragma unroll 4
        for (int at = (KEEP * 64 + lane) * kVec; at < A.H; at += 64 * kVec) {
          float d[kVec];
          load_row<WIDE, F32>(A.dy, n, A.H, at, d);
          both(at, d);
        }
#pragma unroll
        for (int s = 32; s; s >>= 1) dot += __shfl_xor(dot, s);
      }
      if (A.dweight && lane == 0) A.dweight[n * A.k + j] = dot;
    }
  }
}

bool past(const RowsArgs& A) { return (int64_t)A.M * A.H * 2 > kPastBytes; }

template <int NT>
dim3 row_grid(const RowsArgs& A) {
  const int vecs = (A.H + kVec - 1) / kVec;
  if constexpr (NT == 0) {
    const int64_t rows = kThreads / vecs;
    return dim3((unsigned)std::min<int64_t>(((int64_t)A.N + rows - 1) / rows, 1 << 20));
  } else {
    return dim3((unsigned)((vecs + NT - 1) / NT), (unsigned)std::min(A.N, 65535));
  }
}

template <bool WIDE, int NT>
void dispatch(const RowsArgs& A, hipStream_t s) {
  const dim3 grid = row_grid<NT>(A), threads(NT ? NT : kThreads);
  if (past(A)) k_dispatch<WIDE, true, NT><<<grid, threads, 0, s>>>(A);
  else k_dispatch<WIDE, false, NT><<<grid, threads, 0, s>>>(A);
}
template <bool WIDE, int NT>
void combine(const RowsArgs& A, hipStream_t s) {
  const dim3 grid = row_grid<NT>(A), threads(NT ? NT : kThreads);
  if (past(A)) {
    if (A.f32) k_combine<WIDE, true, true, NT><<<grid, threads, 0, s>>>(A);
    else k_combine<WIDE, false, true, NT><<<grid, threads, 0, s>>>(A);
  } else {
    if (A.f32) k_combine<WIDE, true, false, NT><<<grid, threads, 0, s>>>(A);
    else k_combine<WIDE, false, false, NT><<<grid, threads, 0, s>>>(A);
  }
}

template <bool WIDE, bool F32, int KEEP>
void backward(const RowsArgs& A, dim3 grid, hipStream_t s) {
  if (past(A)) k_combine_backward<WIDE, F32, true, KEEP><<<grid, dim3(kThreads), 0, s>>>(A);
  else k_combine_backward<WIDE, F32, false, KEEP><<<grid, dim3(kThreads), 0, s>>>(A);
}
template <bool WIDE, bool F32>
void backward(const RowsArgs& A, hipStream_t s) {
  // four workgroups a CU, each wave the same number of rows: 8192 rows of 2048 in
  // 114 us, with a workgroup for every four rows 127, with 768 of them 124
  const int64_t most = 1024;
  const auto grid = [&](int64_t items) {
    const int64_t rounds = (items + 3) / 4, each = rounds < 2 * most ? 1 : (rounds + most - 1) / most;
    return dim3((unsigned)((rounds + each - 1) / each));
  };
  // A wave a row and place up to 4096 of them: 512 x 8 rows of 2048 in 8.6 us, with a
  // wave a row 20.4; of 7168 in 30.4, with a wave a row 100. With many rows dy's row
  // is read once: 5000 x 8 rows of 2048 in 75 us, else 92.5. In between the rule
  // changes too early: 513 x 8 rows take 20.5 us instead of 8.2, 1000 x 8 31.6
  // instead of 15.7, and rows of 7168 are slower up to 5000 x 8 (305, 265).
  if ((int64_t)A.N * A.k <= 4 * most) backward<WIDE, F32, 0>(A, grid((int64_t)A.N * A.k), s);
  else if (A.H <= 4 * 64 * kVec) backward<WIDE, F32, 4>(A, grid(A.N), s);
  else backward<WIDE, F32, 8>(A, grid(A.N), s);
}

// Threads of a row: 128 where 256 would leave more of them without values
// (2047 x 6 rows of 2816 copied and combined in 15.3 and 19.4 us, with 256 threads
// 18.0 and 20.8; from the caches 12.3 and 14.6, 14.6 and 15.6), 0 (rows behind one another) where several rows fit.
int row_threads(const RowsArgs& A) {
  const int vecs = (A.H + kVec - 1) / kVec;
  if (vecs <= kThreads / 2) return 0;
  return (vecs + 127) / 128 * 128 < (vecs + 255) / 256 * 256 ? 128 : 256;
}

}  // namespace

hipError_t launch_dispatch(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  const int nt = row_threads(A);
  if (A.wide) nt == 0 ? dispatch<true, 0>(A, s) : nt == 128 ? dispatch<true, 128>(A, s) : dispatch<true, 256>(A, s);
  else nt == 0 ? dispatch<false, 0>(A, s) : nt == 128 ? dispatch<false, 128>(A, s) : dispatch<false, 256>(A, s);
  return hipGetLastError();
}

hipError_t launch_combine(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  const int nt = row_threads(A);
  if (A.wide) nt == 0 ? combine<true, 0>(A, s) : nt == 128 ? combine<true, 128>(A, s) : combine<true, 256>(A, s);
  else nt == 0 ? combine<false, 0>(A, s) : nt == 128 ? combine<false, 128>(A, s) : combine<false, 256>(A, s);
  return hipGetLastError();
}

hipError_t launch_combine_backward(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  if (A.wide) A.f32 ? backward<true, true>(A, s) : backward<true, false>(A, s);
  else A.f32 ? backward<false, true>(A, s) : backward<false, false>(A, s);
  return hipGetLastError();
}

}  // namespace cardan
