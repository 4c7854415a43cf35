// Distillation loss of student logits against a teacher's kept top logits,
// with its gradient.
//
// Per row with student logits s over V entries, temperature T, and the
// teacher's logits t_j at entries i_j:
//   p = softmax_j(t_j / T),  q = softmax(s / T),  r = softmax(s)
//   kd = T^2 sum_j p_j (log p_j - log q_{i_j}),  ce = -log r_label
//   d/ds [w (kd + c ce)] = w T (q - sum_j p_j 1_{i_j}) + w c (r - 1_label)
#include <hip/hip_runtime.h>

#include "cardan_ffn.h"

namespace cardan {
namespace {

constexpr int kMaxTeacher = 1024;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_bits(float f) {
  const __bf16 b = (__bf16)f;
  return (uint32_t)__builtin_bit_cast(unsigned short, b);
}

// logits of one type: single values, and 16-byte vectors of kVec
template <bool F32>
struct Logits {
  static constexpr int kSize = F32 ? 4 : 2, kVec = 16 / kSize;
  static __device__ __forceinline__ float get(const void* row, int64_t i) {
    if constexpr (F32) return static_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[i] << 16);
  }
  static __device__ __forceinline__ void put(void* row, int64_t i, float v) {
    if constexpr (F32) static_cast<float*>(row)[i] = v;
    else static_cast<uint16_t*>(row)[i] = (uint16_t)bf16_bits(v);
  }
  static __device__ __forceinline__ void unpack(u32x4 v, float (&z)[kVec]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (F32) z[q] = __uint_as_float(v[q]);
      else {
        z[2 * q] = bf_lo(v[q]);
        z[2 * q + 1] = bf_hi(v[q]);
      }
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&z)[kVec]) {
    u32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (F32) v[q] = __float_as_uint(z[q]);
      else v[q] = bf16_bits(z[2 * q]) | bf16_bits(z[2 * q + 1]) << 16;
    }
    return v;
  }
};

// Running maximum m and sums of exp at both temperatures relative to it. The
// maximum starts at the lowest finite value, so rows and parts that hold
// nothing but -infinity give sums of zero and no NaN.
template <bool TWO>
struct Stat {
  float m = kLowest, st = 0.f, s1 = 0.f;
  __device__ __forceinline__ void join(float om, float ost, float os1, float ct) {
    const float n = fmaxf(m, om);
    const float a = exp2f((m - n) * ct), b = exp2f((om - n) * ct);
    st = st * a + ost * b;
    if constexpr (TWO) s1 = s1 * exp2f((m - n) * kLog2e) + os1 * exp2f((om - n) * kLog2e);
    m = n;
  }
  template <int NV>
  __device__ __forceinline__ void add(const float (&z)[NV], float ct) {
    float mx = z[0];
#pragma unroll
    for (int q = 1; q < NV; ++q) mx = fmaxf(mx, z[q]);
    if (mx > m) {
      st *= exp2f((m - mx) * ct);
      if constexpr (TWO) s1 *= exp2f((m - mx) * kLog2e);
      m = mx;
    }
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const float d = z[q] - m;
      st += __builtin_amdgcn_exp2f(d * ct);
      if constexpr (TWO) s1 += __builtin_amdgcn_exp2f(d * kLog2e);
    }
  }
};

template <int NT>
__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int s = 32; s; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int i = 1; i < NT / 64; ++i) v = fmaxf(v, red[i]);
  return v;
}
template <int NT>
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int i = 1; i < NT / 64; ++i) v += red[i];
  return v;
}

// One workgroup per row. TWO: the row's softmax is needed at T and at 1.
template <bool F32, bool TWO, int NT>
__global__ __launch_bounds__(NT) void k_distill(const DistillArgs A) {
  typedef Logits<F32> L;
  constexpr int NV = L::kVec;
  __shared__ double red[NT / 64];
  __shared__ float redm[NT / 64], redt[NT / 64], red1[NT / 64];
  __shared__ int tid_[kMaxTeacher + 1];
  __shared__ float tp[kMaxTeacher + 1], tz[kMaxTeacher + 1];
  const int n = blockIdx.x, tid = threadIdx.x, V = A.V, K = A.K;
  const char* row = static_cast<const char*>(A.logits) + (int64_t)n * A.ld * L::kSize;
  char* grow = A.dlogits ? static_cast<char*>(A.dlogits) + (int64_t)n * A.dld * L::kSize : nullptr;
  const float invT = 1.0f / A.temperature, ct = kLog2e * invT;

  // the teacher's distribution over its entries
  float tmax = kLowest;
  int some = 0;
  for (int j = tid; j < K; j += NT) {
    const int id = A.ids[(int64_t)n * K + j];
    const bool ok = id >= 0 && id < V;
    const float t = ok ? A.teacher[(int64_t)n * K + j] : -INFINITY;
    tid_[j] = ok ? id : -1;
    tp[j] = t;
    tz[j] = ok ? L::get(row, id) : 0.f;
    some |= ok;
    tmax = fmaxf(tmax, t);
  }
  const int label = A.labels ? A.labels[n] : -1;
  const bool has_label = label >= 0 && label < V;
  const float zlab = has_label ? L::get(row, label) : 0.f;
  some = __syncthreads_or(some);
  tmax = block_max<NT>(tmax, redm);
  double tsum = 0.0;
  for (int j = tid; j < K; j += NT) {
    const float ex = tid_[j] >= 0 ? __expf((tp[j] - tmax) * invT) : 0.f;
    tsum += ex;
  }
  tsum = block_sum<NT>(tsum, red);

  const float w = A.weight ? A.weight[n] : 1.0f;
  if (!some && !has_label) {  // nothing to learn from this row
    if (tid == 0) {
      A.loss[2 * (int64_t)n] = 0.f;
      A.loss[2 * (int64_t)n + 1] = 0.f;
    }
    if (grow)
      for (int64_t i = tid; i < V; i += NT) L::put(grow, i, 0.f);
    return;
  }

  // the vectors of the row that start on 16 bytes, and the values before and after them
  const int lead = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / L::kSize;
  const int head = lead < V ? lead : V, nvec = (V - head) / NV, tail0 = head + nvec * NV;
  const u32x4* vec = reinterpret_cast<const u32x4*>(row + (int64_t)head * L::kSize);

  Stat<TWO> S;
  for (int i = tid; i < nvec; i += NT) {
    float z[NV];
    L::unpack(vec[i], z);
    S.add(z, ct);
  }
  for (int i = tid; i < head + (V - tail0); i += NT) {
    const float z[1] = {L::get(row, i < head ? i : tail0 + (i - head))};
    S.add(z, ct);
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) S.join(__shfl_xor(S.m, s), __shfl_xor(S.st, s), __shfl_xor(S.s1, s), ct);
  __syncthreads();
  if ((tid & 63) == 0) {
    redm[tid >> 6] = S.m;
    redt[tid >> 6] = S.st;
    red1[tid >> 6] = S.s1;
  }
  __syncthreads();
  S = Stat<TWO>();
  for (int i = 0; i < NT / 64; ++i) S.join(redm[i], redt[i], red1[i], ct);
  const float m = S.m, st = S.st, s1 = TWO ? S.s1 : S.st;

  // losses: differences to the maximum, in float64 (K terms a row)
  const double dT = 1.0 / (double)A.temperature;
  const double logst = log((double)st), logtt = log(tsum);
  double kd = 0.0;
  for (int j = tid; j < K; j += NT) {
    float p = 0.f;
    if (tid_[j] >= 0) {
      const double lp = ((double)tp[j] - tmax) * dT - logtt;
      p = (float)exp(lp);
      if (p > 0.f) kd += (double)p * (lp - (((double)tz[j] - m) * dT - logst));
    }
    tp[j] = p;
  }
  kd = block_sum<NT>(kd, red);
  if (tid == 0) {
    A.loss[2 * (int64_t)n] = some ? (float)(kd * A.temperature * A.temperature) : 0.f;
    A.loss[2 * (int64_t)n + 1] = has_label ? (float)(log((double)s1) - ((double)zlab - m)) : 0.f;
  }
  if (!grow) return;

  const float a = some ? w * A.temperature : 0.f, b = has_label ? w * A.ce_weight : 0.f;
  const float ait = a / st, bi1 = b / s1;
  auto grad = [&](float z) {
    const float d = z - m;
    if constexpr (TWO) return ait * __builtin_amdgcn_exp2f(d * ct) + bi1 * __builtin_amdgcn_exp2f(d * kLog2e);
    else return (ait + bi1) * __builtin_amdgcn_exp2f(d * ct);
  };
  for (int i = tid; i < nvec; i += NT) {
    float z[NV];
    L::unpack(vec[i], z);
#pragma unroll
    for (int q = 0; q < NV; ++q) z[q] = grad(z[q]);
    const u32x4 o = L::pack(z);
    __builtin_memcpy(grow + ((int64_t)head + (int64_t)i * NV) * L::kSize, &o, 16);
  }
  for (int i = tid; i < head + (V - tail0); i += NT) {
    const int at = i < head ? i : tail0 + (i - head);
    L::put(grow, at, grad(L::get(row, at)));
  }
  // the entries of the teacher and the label: written again, once rounded, by
  // the first that names an entry, after the dense values have been stored
  if (tid == 0) tid_[K] = has_label ? label : -1;
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  for (int j = tid; j <= K; j += NT) {
    const int id = tid_[j];
    if (id < 0) continue;
    bool first = true;
    float sub = 0.f;
    for (int i = 0; i < K; ++i) {
      if (tid_[i] != id) continue;
      if (i < j) first = false;
      sub += tp[i];
    }
    if (!first) continue;
    const float z = j < K ? tz[j] : zlab;
    float g = grad(z) - a * sub;
    if (tid_[K] == id) g -= b;
    L::put(grow, id, g);
  }
}

template <bool F32, bool TWO>
hipError_t run(const DistillArgs& A, hipStream_t s) {
  k_distill<F32, TWO, 512><<<dim3((unsigned)A.N), dim3(512), 0, s>>>(A);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const DistillArgs& A, hipStream_t s) {
  const bool two = A.labels && A.temperature != 1.0f;
  if (A.f32) return two ? run<true, true>(A, s) : run<true, false>(A, s);
  return two ? run<false, true>(A, s) : run<false, false>(A, s);
}

}  // namespace cardan
