// Distillation loss of student logits against a teacher's kept top logits,
// with its gradient.
//
// Per row with student logits s over V entries, temperature T, and the
// teacher's logits t_j at entries i_j:
//   p = softmax_j(t_j / T),  q = softmax(s / T),  r = softmax(s)
//   kd = T^2 sum_j p_j (log p_j - log q_{i_j}),  ce = -log r_label
//   d/ds [w (kd + c ce)] = w T (q - sum_j p_j 1_{i_j}) + w c (r - 1_label)
//
// Bound by the logits' read and the gradient's write: 8192 x 128256 bf16 in
// 922 us (4.6 TB/s of those bytes; T = 2, 896 at T = 1 and 1005 at others, with two
// exponentials a value), 1500 x 151936 float32 in 391 us (4.7).
#include <hip/hip_runtime.h>

#include "cardan_ffn.h"

namespace cardan {
namespace {

constexpr int kMaxTeacher = 1024, kTable = 2048;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));  // rows may start on any value
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How many softmaxes of a row are needed and how they are formed.
enum Mode {
  ONE = 0,     // one temperature: T, or T = 1 for both losses
  SQUARE = 1,  // T = 2 and 1: exp(s) = exp(s / 2)^2, one exponential serves both
  TWO = 2      // T and 1
};

// logits of one type: single values, and 16-byte vectors of kVec
template <bool F32>
struct Logits {
  static constexpr int kSize = F32 ? 4 : 2, kVec = 16 / kSize;
  static constexpr uint32_t kNone = F32 ? 0xff800000u : 0xff80ff80u;  // -infinity
  static __device__ __forceinline__ float get(const void* row, int64_t i) {
    if constexpr (F32) return static_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[i] << 16);
  }
  static __device__ __forceinline__ void put(void* row, int64_t i, float v) {
    if constexpr (F32) static_cast<float*>(row)[i] = v;
    else static_cast<uint16_t*>(row)[i] = __builtin_bit_cast(unsigned short, (__bf16)v);
  }
  static __device__ __forceinline__ void unpack(u32x4 v, float (&z)[kVec]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (F32) z[q] = __uint_as_float(v[q]);
      else {
        z[2 * q] = __uint_as_float(v[q] << 16);
        z[2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u);
      }
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&z)[kVec]) {
    u32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (F32) v[q] = __float_as_uint(z[q]);
      else v[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){z[2 * q], z[2 * q + 1]}, bf16x2));
    }
    return v;
  }
};

// Running maximum m and sums of exp at both temperatures relative to it. The
// maximum starts at the lowest finite value, so rows and parts that hold
// nothing but -infinity give sums of zero and no NaN. Differences are formed
// before they are scaled: z c - m c in one instruction would be infinity less
// infinity in a row of the lowest value.
template <int MODE>
struct Stat {
  float m = kLowest, st = 0.f, s1 = 0.f;
  __device__ __forceinline__ void raise(float n, float ct) {  // to the maximum n >= m
    const float a = __builtin_amdgcn_exp2f((m - n) * ct);
    st *= a;
    if constexpr (MODE == SQUARE) s1 *= a * a;
    if constexpr (MODE == TWO) s1 *= __builtin_amdgcn_exp2f((m - n) * kLog2e);
    m = n;
  }
  __device__ __forceinline__ void join(Stat o, float ct) {
    const float n = fmaxf(m, o.m);
    raise(n, ct);
    o.raise(n, ct);
    st += o.st;
    s1 += o.s1;
  }
  template <int NV>
  __device__ __forceinline__ void add(const float (&z)[NV], float ct) {
    float mx = z[0];
#pragma unroll
    for (int q = 1; q < NV; ++q) mx = fmaxf(mx, z[q]);
    if (mx > m) raise(mx, ct);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const float d = z[q] - m, e = __builtin_amdgcn_exp2f(d * ct);
      st += e;
      if constexpr (MODE == SQUARE) s1 = fmaf(e, e, s1);
      if constexpr (MODE == TWO) s1 += __builtin_amdgcn_exp2f(d * kLog2e);
    }
  }
};

// a value that every lane has, in a scalar register
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v)));
}

// One workgroup per row; each thread keeps KEEP vectors of the row in
// registers, so that a row of up to NT * KEEP * 16 bytes is read once. What
// lies past them is read again for the gradient, last vectors first (those
// are still in the caches).
template <bool F32, int MODE, int NT, int KEEP>
__global__ __launch_bounds__(NT) void k_distill(const DistillArgs A, int first) {
  typedef Logits<F32> L;
  constexpr int NV = L::kVec, NW = NT / 64;
  __shared__ float part[3][NW];    // a wave's maximum and sums
  __shared__ float tmax_w[NW], tsum_w[NW];
  __shared__ double kd_w[NW];
  __shared__ int tid_[kMaxTeacher];
  __shared__ float tp[kMaxTeacher];
  __shared__ int table[kTable];
  __shared__ int flags[3];         // some entry, an entry named twice, the label is an entry
  const int n = first + blockIdx.x, tid = threadIdx.x, wave = tid >> 6, V = A.V, K = A.K;
  const char* row = static_cast<const char*>(A.logits) + (int64_t)n * A.ld * L::kSize;
  char* grow = A.dlogits ? static_cast<char*>(A.dlogits) + (int64_t)n * A.dld * L::kSize : nullptr;
  const float invT = 1.0f / A.temperature, ct = kLog2e * invT;

  // the vectors of the row that start on 16 bytes, and the values before and
  // after them (fewer than 16, one a thread)
  const int lead = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / L::kSize;
  const int head = lead < V ? lead : V, nvec = (V - head) / NV, tail0 = head + nvec * NV;
  const u32x4* vec = reinterpret_cast<const u32x4*>(row + (int64_t)head * L::kSize);
  u32x4 keep[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int at = i * NT + tid;
    keep[i] = at < nvec ? vec[at] : u32x4{L::kNone, L::kNone, L::kNone, L::kNone};
  }
  const bool odd = tid < head + (V - tail0);
  const int odd_at = tid < head ? tid : tail0 + (tid - head);
  const float odd_z = odd ? L::get(row, odd_at) : -INFINITY;

  // the teacher's entries, while the row is on its way
  const int label = A.labels ? A.labels[n] : -1;
  const bool has_label = label >= 0 && label < V;
  const float zlab = has_label ? L::get(row, label) : 0.f;
  for (int i = tid; i < kTable; i += NT) table[i] = -1;
  if (tid < 3) flags[tid] = 0;
  constexpr int JT = (kMaxTeacher + NT - 1) / NT;  // entries of a thread
  int id[JT];
  float t[JT], z[JT];
  float tmax = kLowest;
#pragma unroll
  for (int q = 0; q < JT; ++q) {
    const int j = q * NT + tid;
    id[q] = j < K ? A.ids[(int64_t)n * K + j] : -1;
    if (id[q] >= V) id[q] = -1;
    t[q] = id[q] >= 0 ? A.teacher[(int64_t)n * K + j] : -INFINITY;
    z[q] = id[q] >= 0 ? L::get(row, id[q]) : 0.f;
    if (t[q] == -INFINITY) id[q] = -1;  // of probability zero: no entry, also where all are
    tmax = fmaxf(tmax, t[q]);
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) tmax = fmaxf(tmax, __shfl_xor(tmax, s));
  if ((tid & 63) == 0) tmax_w[wave] = tmax;
  __syncthreads();
  tmax = tmax_w[tid & (NW - 1)];
#pragma unroll
  for (int s = NW / 2; s; s >>= 1) tmax = fmaxf(tmax, __shfl_xor(tmax, s));
  tmax = uniform(tmax);
  float tsum = 0.f;
#pragma unroll
  for (int q = 0; q < JT; ++q) {
    if (q * NT >= K) break;
    if (id[q] >= 0) {
      tsum += t[q] = __expf((t[q] - tmax) * invT);
      flags[0] = 1;
      if (id[q] == label) flags[2] = 1;
      // an open hash table finds out whether an entry is named twice
      uint32_t at = (uint32_t)id[q] * 2654435761u >> 21;
      for (;;) {
        const int was = atomicCAS(&table[at], -1, id[q]);
        if (was == id[q]) flags[1] = 1;
        if (was == -1 || was == id[q]) break;
        at = (at + 1) & (kTable - 1);
      }
    }
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) tsum += __shfl_xor(tsum, s);
  if ((tid & 63) == 0) tsum_w[wave] = tsum;

  // the row's maximum and sums
  Stat<MODE> S;
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    float v[NV];
    L::unpack(keep[i], v);
    S.add(v, ct);
  }
  for (int at = KEEP * NT + tid; at < nvec; at += NT) {
    float v[NV];
    L::unpack(vec[at], v);
    S.add(v, ct);
  }
  // the registers hold the stored values, not what the sums made of them
#pragma unroll
  for (int i = 0; i < KEEP; ++i) asm volatile("" : "+v"(keep[i]));
  const float odd_v[1] = {odd_z};
  S.add(odd_v, ct);
#pragma unroll
  for (int s = 32; s; s >>= 1) {
    Stat<MODE> o;
    o.m = __shfl_xor(S.m, s);
    o.st = __shfl_xor(S.st, s);
    if constexpr (MODE != ONE) o.s1 = __shfl_xor(S.s1, s);
    S.join(o, ct);
  }
  if ((tid & 63) == 0) {
    part[0][wave] = S.m;
    part[1][wave] = S.st;
    part[2][wave] = S.s1;
  }
  __syncthreads();
  S.m = part[0][tid & (NW - 1)];
  S.st = part[1][tid & (NW - 1)];
  S.s1 = part[2][tid & (NW - 1)];
  tsum = tsum_w[tid & (NW - 1)];
#pragma unroll
  for (int s = NW / 2; s; s >>= 1) {
    Stat<MODE> o;
    o.m = __shfl_xor(S.m, s);
    o.st = __shfl_xor(S.st, s);
    if constexpr (MODE != ONE) o.s1 = __shfl_xor(S.s1, s);
    S.join(o, ct);
    tsum += __shfl_xor(tsum, s);
  }
  tsum = uniform(tsum);
  const float m = uniform(S.m), st = uniform(S.st), s1 = MODE == ONE ? st : uniform(S.s1);
  const bool some = __builtin_amdgcn_readfirstlane(flags[0]), twice = __builtin_amdgcn_readfirstlane(flags[1]);
  const bool label_in = __builtin_amdgcn_readfirstlane(flags[2]);

  // the losses, from differences to the maxima in float64
  if (wave * 64 < K) {
    double kd = 0.0;
    const double dT = 1.0 / (double)A.temperature;
    const double logs = some ? log((double)st) - log((double)tsum) : 0.0;
#pragma unroll
    for (int q = 0; q < JT; ++q) {
      const int j = q * NT + tid;
      if (q * NT >= K) break;
      const float p = id[q] >= 0 ? t[q] / tsum : 0.f;
      if (p != 0.f) {  // (a NaN goes on into the loss)
        const double tt = (double)A.teacher[(int64_t)n * K + j] - tmax;
        kd += (double)p * ((tt - ((double)z[q] - m)) * dT + logs);
      }
      t[q] = p;
      if (twice && j < K) {
        tid_[j] = id[q];
        tp[j] = p;
      }
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) kd += __shfl_xor(kd, s);
    if ((tid & 63) == 0) kd_w[wave] = kd;
  }

  // a row with neither entries nor a label gets zeros, whatever its logits are
  const bool none = !some && !has_label;
  const float w = A.weight ? A.weight[n] : 1.0f;
  const float a = some ? w * A.temperature : 0.f, b = has_label ? w * A.ce_weight : 0.f;
  const float ait = uniform(some ? a / st : 0.f), bi1 = uniform(has_label ? b / s1 : 0.f);
  auto grad = [&](float x) {
    const float d = x - m, e = __builtin_amdgcn_exp2f(d * ct);
    if constexpr (MODE == ONE) return (ait + bi1) * e;
    if constexpr (MODE == SQUARE) return e * fmaf(bi1, e, ait);
    return fmaf(bi1, __builtin_amdgcn_exp2f(d * kLog2e), ait * e);
  };
  if (grow && none) {
    for (int i = tid; i < V; i += NT) L::put(grow, i, 0.f);
  } else if (grow) {
    // the gradient is not read again here: its stores do not stay in the caches
    auto store = [&](int at, u32x4 v) {
      float x[NV];
      L::unpack(v, x);
#pragma unroll
      for (int q = 0; q < NV; ++q) x[q] = grad(x[q]);
      __builtin_nontemporal_store(L::pack(x), (u32x4_at2*)(grow + ((int64_t)head + (int64_t)at * NV) * L::kSize));
    };
    if (nvec > KEEP * NT) {
      const int last = KEEP * NT + (nvec - 1 - KEEP * NT) / NT * NT;
      for (int at = last + tid; at >= KEEP * NT; at -= NT)
        if (at < nvec) store(at, vec[at]);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      if (i * NT + tid < nvec) store(i * NT + tid, keep[i]);
    if (odd) L::put(grow, odd_at, grad(odd_z));
    // the entries of the teacher and the label are written again, once
    // rounded, after the dense values have been stored
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  }
  __syncthreads();
  if (tid == 0) {
    double kd = 0.0;
    for (int i = 0; i < NW && i * 64 < K; ++i) kd += kd_w[i];
    A.loss[2 * (int64_t)n] = some ? (float)(kd * A.temperature * A.temperature) : 0.f;
    A.loss[2 * (int64_t)n + 1] = has_label ? (float)(log((double)s1) - ((double)zlab - m)) : 0.f;
  }
  if (!grow || none) return;
#pragma unroll
  for (int q = 0; q < JT; ++q) {
    if (q * NT >= K) break;
    const int j = q * NT + tid;
    if (id[q] < 0) continue;
    float sub = t[q];
    if (twice) {  // the first that names an entry writes it, with all of its probabilities
      bool first = true;
      sub = 0.f;
      for (int i = 0; i < K; ++i)
        if (tid_[i] == id[q]) {
          first &= i >= j;
          sub += tp[i];
        }
      if (!first) continue;
    }
    float g = grad(z[q]) - a * sub;
    if (id[q] == label) g -= b;
    L::put(grow, id[q], g);
  }
  if (tid == 0 && has_label && !label_in) L::put(grow, label, grad(zlab) - b);
}

template <bool F32, int MODE, int NT, int KEEP>
hipError_t run(const DistillArgs& A, hipStream_t s) {
  constexpr int kMost = 1 << 21;  // rows of a launch: its threads are counted in 32 bits
  hipError_t e = hipSuccess;
  for (int first = 0; first < A.N && e == hipSuccess; first += kMost) {
    const int rows = A.N - first < kMost ? A.N - first : kMost;
    k_distill<F32, MODE, NT, KEEP><<<dim3((unsigned)rows), dim3(NT), 0, s>>>(A, first);
    e = hipGetLastError();
  }
  return e;
}

// A row's vectors are spread over as few threads as keep it in registers, so
// that several rows share a CU; 16 vectors a thread fit beside the kernel's
// other registers. bf16 rows of more than 128 KiB keep half: two rows a CU,
// one of which computes while the other loads or stores, beat the second read
// of the rest (8192 x 128256: 922 us, all of one row in 1024 threads' registers
// 1058); float32 rows, with half the exponentials a byte, keep 256 KiB (1500 x
// 151936: 391 us against 443).
template <bool F32, int MODE>
hipError_t run_rows(const DistillArgs& A, hipStream_t s) {
  const int64_t vecs = ((int64_t)A.V * (F32 ? 4 : 2) + 15) / 16;
  if (vecs <= 256) return run<F32, MODE, 256, 1>(A, s);
  if (vecs <= 256 * 4) return run<F32, MODE, 256, 4>(A, s);
  if (vecs <= 512 * 4) return run<F32, MODE, 512, 4>(A, s);
  if (vecs <= 512 * 8) return run<F32, MODE, 512, 8>(A, s);
  if (vecs <= 512 * 12) return run<F32, MODE, 512, 12>(A, s);
  if (vecs <= 512 * 16) return run<F32, MODE, 512, 16>(A, s);
  if constexpr (!F32) return run<F32, MODE, 512, 16>(A, s);
  if (vecs <= 1024 * 12) return run<F32, MODE, 1024, 12>(A, s);
  return run<F32, MODE, 1024, 16>(A, s);
}

template <bool F32>
hipError_t run_mode(const DistillArgs& A, hipStream_t s) {
  if (!A.labels || A.temperature == 1.0f) return run_rows<F32, ONE>(A, s);
  return A.temperature == 2.0f ? run_rows<F32, SQUARE>(A, s) : run_rows<F32, TWO>(A, s);
}

}  // namespace

hipError_t launch_distill(const DistillArgs& A, hipStream_t s) {
  return A.f32 ? run_mode<true>(A, s) : run_mode<false>(A, s);
}

}  // namespace cardan
