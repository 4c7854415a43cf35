// AdamW over many tensors, moments in float32 or in 8 bits.
//
// Per value with gradient g (times grad_scale), t the step:
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - lr decay p - (lr / (1 - b1^t)) m / (sqrt(v / (1 - b2^t)) + eps)
// 8-bit moments: m as e4m3, v as e5m2, times one float32 scale for each 256
// consecutive values (largest size over the type's largest value). A step
// changes v by a thousandth, an e5m2 step is up to a quarter: rounded to
// nearest, v would stand still. Both roundings are dithered instead: up where
// the fraction of a step and a 16-bit number u give (u + 1/2) / 2^16 +
// fraction >= 1, u from a mix of the value's place in its tensor and the step,
// so each is right in the mean and a call's result depends on its arguments
// alone. bf16 weights are rounded the same way (an update is often below half
// a step of them).
//
// Bound by memory: 38 M float32 weights with float32 moments in 202 us (5.3
// TB/s), 403 M with bf16 gradients, bf16 copies and 8-bit moments in 1200 us (5.4;
// a large copy reaches 4.8). A lane holds eight values, half a wave a block, so
// that a scale is five steps over lanes and no LDS; the update has no fused
// products, so that it is the same number wherever it is computed.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cardan_rows.h"

namespace cardan {
namespace {

constexpr int kThreads = 256, kEach = 8;           // values of a lane at once: half a wave holds a block
constexpr int kPass = 64 * kEach;                  // values of a wave at once
constexpr int kWork = kThreads / 64 * kPass;        // values of a workgroup: one pass (two 4 % slower, four 6 %)
static_assert(kWork == kAdamwWork, "the host counts workgroups");

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// tensors start on their own elements' size
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at1 __attribute__((aligned(1)));

struct Floats {
  float v[kEach];
};

__device__ __forceinline__ Floats load_f32(const float* p) {
  const u32x4 a = *reinterpret_cast<const u32x4_at4*>(p), b = *reinterpret_cast<const u32x4_at4*>(p + 4);
  Floats f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f.v[q] = __uint_as_float(a[q]);
    f.v[4 + q] = __uint_as_float(b[q]);
  }
  return f;
}
__device__ __forceinline__ void store_f32(float* p, const Floats& f) {
  u32x4 a, b;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    a[q] = __float_as_uint(f.v[q]);
    b[q] = __float_as_uint(f.v[4 + q]);
  }
  *reinterpret_cast<u32x4_at4*>(p) = a;
  *reinterpret_cast<u32x4_at4*>(p + 4) = b;
}
__device__ __forceinline__ Floats load_bf16(const uint16_t* p) {
  const u32x4 a = *reinterpret_cast<const u32x4_at2*>(p);
  Floats f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f.v[2 * q] = __uint_as_float(a[q] << 16);
    f.v[2 * q + 1] = __uint_as_float(a[q] & 0xffff0000u);
  }
  return f;
}
__device__ __forceinline__ void store_bf16(uint16_t* p, const uint32_t (&h)[kEach]) {
  u32x4 a;
#pragma unroll
  for (int q = 0; q < 4; ++q) a[q] = h[2 * q] | h[2 * q + 1] << 16;
  *reinterpret_cast<u32x4_at2*>(p) = a;
}
__device__ __forceinline__ uint32_t nearest_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// A 32-bit number for place i of a tensor at step t: multiplications by odd
// constants (bits of the golden ratio and of the roots of 2 and 3) and folds.
__device__ __forceinline__ uint32_t mixed(int64_t i, uint32_t t) {
  uint32_t h = (uint32_t)i * 0x9E3779B9u + t * 0x6A09E667u + (uint32_t)(i >> 32) * 0xBB67AE85u;
  h ^= h >> 16;
  h *= 0x6A09E667u;
  h ^= h >> 15;
  h *= 0xBB67AE85u;
  return h ^ h >> 16;
}

// |x| up to the type's largest value as a code of M mantissa bits: scaled by
// 2^SHIFT its float32 exponent field is the type's, also for subnormal codes,
// and the float32 mantissa bits below the code's are the fraction of a step.
template <int M, int SHIFT, uint32_t TOP>
__device__ __forceinline__ uint32_t code_of(float x, uint32_t u) {
  constexpr int kLow = 23 - M;
  const uint32_t bits = __float_as_uint(x * __uint_as_float((uint32_t)(127 + SHIFT) << 23));
  const uint32_t code = (bits + (u << (kLow - 16)) + (1u << (kLow - 17))) >> kLow;
  return code < TOP ? code : TOP;
}

// The largest of the 32 lanes that hold a block, as bits of a size >= 0: NaN
// is above infinity and infinity above all others.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  auto most = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0xB1, 0xf, 0xf, false));
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x4E, 0xf, 0xf, false));
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x141, 0xf, 0xf, false));
  v = most(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x140, 0xf, 0xf, false));
  return most(v, (uint32_t)__shfl_xor((int)v, 16));
}

__device__ __forceinline__ float scale_of(uint32_t most, float inv_top) {
  const float a = __uint_as_float(most);
  const float s = a * inv_top;
  // (subnormal scales would have no reciprocal)
  return a == 0.f ? 0.f : s < 0x1p-126f ? 0x1p-126f : s;
}

template <bool PBF, bool GBF, bool S8>
__global__ __launch_bounds__(kThreads) void k_adamw(const AdamwArgs A) {
#pragma clang fp contract(off)
  // the tensor of this workgroup
  int lo = 0, hi = A.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (A.first[mid] <= (int)blockIdx.x) lo = mid;
    else hi = mid;
  }
  const AdamwTensor& T = A.t[lo];
  const int64_t n = T.n, start = (int64_t)((int)blockIdx.x - A.first[lo]) * kWork;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  uint32_t t = (uint32_t)A.step;
  float lr_decay = A.lr_decay, lr_c1 = A.lr_c1, inv_c2 = A.inv_c2;
  if (A.step_device || A.lr_device) {
    double c1 = 1.0, c2 = 1.0;
    if (A.step_device) {
      const int s = A.step_device[0];
      t = s > 1 ? (uint32_t)s : 1u;
    }
    double x1 = A.beta1, x2 = A.beta2;
    for (uint32_t b = t; b; b >>= 1) {
      if (b & 1) {
        c1 *= x1;
        c2 *= x2;
      }
      x1 *= x1;
      x2 *= x2;
    }
    const double lr = A.lr_device ? (double)A.lr_device[0] : A.lr;
    lr_decay = (float)(lr * A.decay);
    lr_c1 = (float)(lr / (1.0 - c1));
    inv_c2 = (float)(1.0 / (1.0 - c2));
  }
  const float gs = A.grad_scale ? A.grad_scale[0] : 1.0f;

  const int64_t at = start + wave * kPass + lane * kEach;
  const int64_t left = n - at;
  const int have = left >= kEach ? kEach : left > 0 ? (int)left : 0;
  const bool full = have == kEach;
  Floats p, g, m, v;
#pragma unroll
  for (int q = 0; q < kEach; ++q) p.v[q] = g.v[q] = m.v[q] = v.v[q] = 0.f;
  float ms = 0.f, vs = 0.f;
  uint8_t* m8 = static_cast<uint8_t*>(T.m);
  uint8_t* v8 = static_cast<uint8_t*>(T.v);
  const int64_t block = at / kAdamwBlock;
  if (full) {
    p = PBF ? load_bf16(static_cast<const uint16_t*>(T.p) + at) : load_f32(static_cast<const float*>(T.p) + at);
    g = GBF ? load_bf16(static_cast<const uint16_t*>(T.g) + at) : load_f32(static_cast<const float*>(T.g) + at);
    if constexpr (!S8) {
      m = load_f32(static_cast<const float*>(T.m) + at);
      v = load_f32(static_cast<const float*>(T.v) + at);
    }
  } else {
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      if (q >= have) break;
      p.v[q] = PBF ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(T.p)[at + q] << 16)
                   : static_cast<const float*>(T.p)[at + q];
      g.v[q] = GBF ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(T.g)[at + q] << 16)
                   : static_cast<const float*>(T.g)[at + q];
      if constexpr (!S8) {
        m.v[q] = static_cast<const float*>(T.m)[at + q];
        v.v[q] = static_cast<const float*>(T.v)[at + q];
      }
    }
  }
  if constexpr (S8) {
    u32x2 mc = {0, 0}, vc = {0, 0};
    if (full) {
      mc = *reinterpret_cast<const u32x2_at1*>(m8 + at);
      vc = *reinterpret_cast<const u32x2_at1*>(v8 + at);
    } else {
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        if (q >= have) break;
        mc[q >> 2] |= (uint32_t)m8[at + q] << 8 * (q & 3);
        vc[q >> 2] |= (uint32_t)v8[at + q] << 8 * (q & 3);
      }
    }
    if (have > 0) {
      ms = T.ms[block];
      vs = T.vs[block];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x2 a = q & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(mc[q >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(mc[q >> 1], false);
      const f32x2 b = q & 1 ? __builtin_amdgcn_cvt_pk_f32_bf8(vc[q >> 1], true) : __builtin_amdgcn_cvt_pk_f32_bf8(vc[q >> 1], false);
      m.v[2 * q] = a[0] * ms;
      m.v[2 * q + 1] = a[1] * ms;
      v.v[2 * q] = b[0] * vs;
      v.v[2 * q + 1] = b[1] * vs;
    }
  }
  uint32_t mtop = 0, vtop = 0;
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const float x = g.v[q] * gs;
    m.v[q] = m.v[q] * A.b1 + x * A.a1;
    v.v[q] = v.v[q] * A.b2 + x * x * A.a2;
    p.v[q] = p.v[q] - p.v[q] * lr_decay - (m.v[q] * lr_c1) / (sqrtf(v.v[q] * inv_c2) + A.eps);
    if constexpr (S8) {
      if (q < have) {
        const uint32_t a = __float_as_uint(m.v[q]) & 0x7fffffffu, b = __float_as_uint(v.v[q]) & 0x7fffffffu;
        mtop = a > mtop ? a : mtop;
        vtop = b > vtop ? b : vtop;
      }
    }
  }
  uint32_t h[kEach];
  if constexpr (S8 || PBF) {
#pragma unroll
    for (int q = 0; q < kEach; ++q) h[q] = mixed(at + q, t);
  }
  if constexpr (S8) {
    const float new_ms = scale_of(block_max(mtop), 1.0f / 448.0f), new_vs = scale_of(block_max(vtop), 1.0f / 57344.0f);
    const float mi = new_ms > 0.f ? 1.0f / new_ms : new_ms, vi = new_vs > 0.f ? 1.0f / new_vs : new_vs;
    u32x2 mc = {0, 0}, vc = {0, 0};
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const uint32_t sign = __float_as_uint(m.v[q]) >> 24 & 0x80u;
      mc[q >> 2] |= (code_of<3, -120, 0x7e>(fabsf(m.v[q]) * mi, h[q] & 0xffffu) | sign) << 8 * (q & 3);
      vc[q >> 2] |= code_of<2, -112, 0x7b>(v.v[q] * vi, h[q] >> 16) << 8 * (q & 3);
    }
    if (full) {
      *reinterpret_cast<u32x2_at1*>(m8 + at) = mc;
      *reinterpret_cast<u32x2_at1*>(v8 + at) = vc;
    } else {
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        if (q >= have) break;
        m8[at + q] = (uint8_t)(mc[q >> 2] >> 8 * (q & 3));
        v8[at + q] = (uint8_t)(vc[q >> 2] >> 8 * (q & 3));
      }
    }
    if (have > 0 && at % kAdamwBlock == 0) {
      T.ms[block] = new_ms;
      T.vs[block] = new_vs;
    }
  } else if (full) {
    store_f32(static_cast<float*>(T.m) + at, m);
    store_f32(static_cast<float*>(T.v) + at, v);
  } else {
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      if (q >= have) break;
      static_cast<float*>(T.m)[at + q] = m.v[q];
      static_cast<float*>(T.v)[at + q] = v.v[q];
    }
  }
  if constexpr (PBF) {
    uint32_t b[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      uint32_t u = h[q] * 0x9E3779B9u;
      u = (u ^ u >> 16) & 0xffffu;
      const uint32_t bits = __float_as_uint(p.v[q]);
      // (a sum past the largest value is infinity; infinity and NaN stay what they are)
      b[q] = (bits & 0x7f800000u) == 0x7f800000u ? nearest_bf16(p.v[q]) : (bits + u) >> 16;
    }
    if (full) store_bf16(static_cast<uint16_t*>(T.p) + at, b);
    else
#pragma unroll
      for (int q = 0; q < kEach; ++q)
        if (q < have) static_cast<uint16_t*>(T.p)[at + q] = (uint16_t)b[q];
  } else {
    if (full) store_f32(static_cast<float*>(T.p) + at, p);
    else
#pragma unroll
      for (int q = 0; q < kEach; ++q)
        if (q < have) static_cast<float*>(T.p)[at + q] = p.v[q];
    if (T.copy) {
      uint32_t b[kEach];
#pragma unroll
      for (int q = 0; q < kEach; ++q) b[q] = nearest_bf16(p.v[q]);
      if (full) store_bf16(T.copy + at, b);
      else
#pragma unroll
        for (int q = 0; q < kEach; ++q)
          if (q < have) T.copy[at + q] = (uint16_t)b[q];
    }
  }
}

template <bool PBF, bool GBF>
void run(const AdamwArgs& A, bool s8, dim3 grid, hipStream_t s) {
  if (s8) k_adamw<PBF, GBF, true><<<grid, dim3(kThreads), 0, s>>>(A);
  else k_adamw<PBF, GBF, false><<<grid, dim3(kThreads), 0, s>>>(A);
}

}  // namespace

// Tensors of one launch; first[] is filled in here.
hipError_t launch_adamw(const AdamwArgs& given, bool pbf, bool gbf, bool s8, hipStream_t s) {
  AdamwArgs A = given;
  int64_t blocks = 0;
  for (int i = 0; i < A.count; ++i) {
    A.first[i] = (int32_t)blocks;
    blocks += (A.t[i].n + kWork - 1) / kWork;
  }
  A.first[A.count] = (int32_t)blocks;
  if (blocks == 0) return hipSuccess;
  const dim3 grid((unsigned)blocks);
  if (pbf) gbf ? run<true, true>(A, s8, grid, s) : run<true, false>(A, s8, grid, s);
  else gbf ? run<false, true>(A, s8, grid, s) : run<false, false>(A, s8, grid, s);
  return hipGetLastError();
}

}  // namespace cardan
