// Rows of tokens to their experts' rows and back, with the gradients:
//   dispatch: xe[place[n][j]] = x[n]
//   combine:  y[n] = sum_j w[n][j] ye[place[n][j]], in the order of j
//   backward: dye[place[n][j]] = w[n][j] dy[n], dw[n][j] = <dy[n], ye[place[n][j]]>
// (the gradient of dispatch is combine without weights).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_rows.h"

namespace cardan {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Values that a thread handles at once: 8 in 16 bytes where all rows start on
// 16 bytes, else single ones.
template <int NV> struct Vec;
template <> struct Vec<8> {
  typedef u32x4 type;
  static __device__ __forceinline__ void unpack(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[2 * q] = __uint_as_float(v[q] << 16);
      f[2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * q], f[2 * q + 1]}, bf16x2));
    return v;
  }
};
template <> struct Vec<1> {
  typedef uint16_t type;
  static __device__ __forceinline__ void unpack(uint16_t v, float (&f)[1]) { f[0] = __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ uint16_t pack(const float (&f)[1]) { return __builtin_bit_cast(uint16_t, (__bf16)f[0]); }
};

// NV values at position `at` of a row of bf16 or float32. PAST: past the caches.
template <int NV, bool F32, bool PAST = false>
__device__ __forceinline__ void load_row(const void* base, int64_t row, int H, int at, float (&f)[NV]) {
  if constexpr (F32) {
    const float* p = static_cast<const float*>(base) + row * H + at;
    if constexpr (NV == 8) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f[q] = a[q];
        f[4 + q] = b[q];
      }
    } else {
      f[0] = *p;
    }
  } else {
    typedef Vec<NV> X;
    const typename X::type* p = reinterpret_cast<const typename X::type*>(static_cast<const uint16_t*>(base) + row * H + at);
    if constexpr (PAST) X::unpack(__builtin_nontemporal_load(p), f);
    else X::unpack(*p, f);
  }
}
template <int NV, bool F32, bool PAST = false>
__device__ __forceinline__ void store_row(void* base, int64_t row, int H, int at, const float (&f)[NV]) {
  if constexpr (F32) {
    float* p = static_cast<float*>(base) + row * H + at;
    if constexpr (NV == 8) {
      *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
      *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
    } else {
      *p = f[0];
    }
  } else {
    typedef Vec<NV> X;
    typename X::type* p = reinterpret_cast<typename X::type*>(static_cast<uint16_t*>(base) + row * H + at);
    if constexpr (PAST) __builtin_nontemporal_store(X::pack(f), p);
    else *p = X::pack(f);
  }
}

constexpr int kThreads = 256;
// A grouped array that the last-level cache (256 MB) does not keep is read and
// written past the caches, which leaves them to the tokens' rows: 65536 x 2048
// copied, combined and both gradients 295 us (347 through the caches; combine
// 60 instead of 80). A smaller one, just written, is still there: 12282 x 2816
// combined in 15.5 us, past the caches 20.8.
constexpr int64_t kPastBytes = (int64_t)192 << 20;

// blockIdx.x: a run of a row's values, blockIdx.y: rows, strided.
template <int NV, bool PAST, int NT>
__global__ __launch_bounds__(NT) void k_dispatch(const RowsArgs A) {
  typedef typename Vec<NV>::type V;
  const int at = (blockIdx.x * NT + threadIdx.x) * NV;
  if (at >= A.H) return;
  for (int64_t n = blockIdx.y; n < A.N; n += gridDim.y) {
    const V v = *reinterpret_cast<const V*>(A.x + n * A.H + at);
    for (int j = 0; j < A.k; ++j) {
      const int p = A.place[n * A.k + j];
      if ((uint32_t)p >= (uint32_t)A.M) continue;
      V* to = reinterpret_cast<V*>(A.xe + (int64_t)p * A.H + at);
      if constexpr (PAST) __builtin_nontemporal_store(v, to);
      else *to = v;
    }
  }
}

template <int NV, bool F32, bool PAST, int NT>
__global__ __launch_bounds__(NT) void k_combine(const RowsArgs A) {
  const int at = (blockIdx.x * NT + threadIdx.x) * NV;
  if (at >= A.H) return;
  for (int64_t n = blockIdx.y; n < A.N; n += gridDim.y) {
    float sum[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) sum[q] = 0.f;
#pragma unroll 4
    for (int j = 0; j < A.k; ++j) {
      const int p = A.place[n * A.k + j];
      if ((uint32_t)p >= (uint32_t)A.M) continue;
      const float w = A.weight ? A.weight[n * A.k + j] : 1.0f;
      float f[NV];
      load_row<NV, false, PAST>(A.ye, p, A.H, at, f);
#pragma unroll
      for (int q = 0; q < NV; ++q) sum[q] = fmaf(w, f[q], sum[q]);
    }
    store_row<NV, F32>(A.y, n, A.H, at, sum);
  }
}

// A wave a row: the products of the row of dy with its k rows are summed over
// the wave's lanes, each in one order.
template <int NV, bool F32, bool PAST>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const RowsArgs A) {
  const int lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)gridDim.x * (kThreads / 64);
  for (int64_t n = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); n < A.N; n += waves) {
    for (int j = 0; j < A.k; ++j) {
      const int p = A.place[n * A.k + j];
      float dot = 0.f;
      if ((uint32_t)p < (uint32_t)A.M) {
        const float w = A.weight ? A.weight[n * A.k + j] : 1.0f;
        for (int at = lane * NV; at < A.H; at += 64 * NV) {
          float d[NV];
          load_row<NV, F32>(A.dy, n, A.H, at, d);
          if (A.dweight) {
            float f[NV];
            load_row<NV, false, PAST>(A.ye, p, A.H, at, f);
#pragma unroll
            for (int q = 0; q < NV; ++q) dot = fmaf(d[q], f[q], dot);
          }
          if (A.dye) {
#pragma unroll
            for (int q = 0; q < NV; ++q) d[q] *= w;
            store_row<NV, false, PAST>(A.dye, p, A.H, at, d);
          }
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
dim3 row_grid(const RowsArgs& A, int nv) {
  return dim3((unsigned)(((int64_t)A.H + nv * NT - 1) / (nv * NT)), (unsigned)std::min(A.N, 65535));
}

template <int NV, int NT>
void dispatch(const RowsArgs& A, hipStream_t s) {
  const dim3 grid = row_grid<NT>(A, NV);
  if (past(A)) k_dispatch<NV, true, NT><<<grid, dim3(NT), 0, s>>>(A);
  else k_dispatch<NV, false, NT><<<grid, dim3(NT), 0, s>>>(A);
}
template <int NV, int NT>
void combine(const RowsArgs& A, hipStream_t s) {
  const dim3 grid = row_grid<NT>(A, NV);
  if (past(A)) {
    if (A.f32) k_combine<NV, true, true, NT><<<grid, dim3(NT), 0, s>>>(A);
    else k_combine<NV, false, true, NT><<<grid, dim3(NT), 0, s>>>(A);
  } else {
    if (A.f32) k_combine<NV, true, false, NT><<<grid, dim3(NT), 0, s>>>(A);
    else k_combine<NV, false, false, NT><<<grid, dim3(NT), 0, s>>>(A);
  }
}

template <int NV, bool F32>
void backward(const RowsArgs& A, dim3 grid, hipStream_t s) {
  if (past(A)) k_combine_backward<NV, F32, true><<<grid, dim3(kThreads), 0, s>>>(A);
  else k_combine_backward<NV, F32, false><<<grid, dim3(kThreads), 0, s>>>(A);
}

// Threads of a workgroup: 128 where 256 would leave more of them without values
// (rows of 2816: 14.3 and 12.4 us for 2047 x 6, with 256 threads 15.5 and 14.5).
bool narrow(const RowsArgs& A) {
  const int vecs = A.H / 8;
  return (vecs + 127) / 128 * 128 < (vecs + 255) / 256 * 256;
}

}  // namespace

hipError_t launch_dispatch(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  if (!A.wide) dispatch<1, 256>(A, s);
  else narrow(A) ? dispatch<8, 128>(A, s) : dispatch<8, 256>(A, s);
  return hipGetLastError();
}

hipError_t launch_combine(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  if (!A.wide) combine<1, 256>(A, s);
  else narrow(A) ? combine<8, 128>(A, s) : combine<8, 256>(A, s);
  return hipGetLastError();
}

hipError_t launch_combine_backward(const RowsArgs& A, hipStream_t s) {
  if (A.N == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>(((int64_t)A.N + 3) / 4, 1 << 16));
  if (!A.wide) A.f32 ? backward<1, true>(A, grid, s) : backward<1, false>(A, grid, s);
  else A.f32 ? backward<8, true>(A, grid, s) : backward<8, false>(A, grid, s);
  return hipGetLastError();
}

}  // namespace cardan
