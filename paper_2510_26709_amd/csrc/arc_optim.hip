// Gradient norms and AdamW over many tensors (the formulas and the states'
// layout are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arc_device.h"
#include "arc_train.h"

namespace arc {
namespace {

constexpr int kThreads = 256;
constexpr int kLane = 8;  // consecutive elements of a thread: 16 lanes hold a block of scales
static_assert(kOptimChunk % (kThreads * kLane) == 0, "whole passes of a workgroup");

// Eight elements at any element alignment (the hardware's 16-byte accesses
// need none).
struct __attribute__((packed, aligned(2))) Halves8 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) Words4 {
  float w[4];
};

__device__ __forceinline__ void load8(const void* base, int32_t bf16, int64_t at, int64_t count,
                                      float (&x)[kLane]) {
  if (at + kLane <= count) {
    if (bf16) {
      const Halves8 h = *reinterpret_cast<const Halves8*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[2 * k] = bf16_lo(h.w[k]);
        x[2 * k + 1] = bf16_hi(h.w[k]);
      }
    } else {
      const Words4* p = reinterpret_cast<const Words4*>(static_cast<const float*>(base) + at);
      const Words4 a = p[0], b = p[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = a.w[k];
        x[4 + k] = b.w[k];
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kLane; ++k) {
    x[k] = 0.f;
    if (at + k < count)
      x[k] = bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[at + k] << 16)
                  : static_cast<const float*>(base)[at + k];
  }
}

__device__ __forceinline__ uint32_t bf16_nearest(float x) {
  const uint32_t b = __float_as_uint(x);
  return x != x ? 0x7FC0u : (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ void store8_bf16(uint16_t* base, int64_t at, int64_t count,
                                            const uint32_t (&h)[kLane]) {
  if (at + kLane <= count) {
    Halves8 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w.w[k] = h[2 * k] | (h[2 * k + 1] << 16);
    *reinterpret_cast<Halves8*>(base + at) = w;
    return;
  }
#pragma unroll
  for (int k = 0; k < kLane; ++k)
    if (at + k < count) base[at + k] = (uint16_t)h[k];
}

__device__ __forceinline__ void store8_f32(float* base, int64_t at, int64_t count,
                                           const float (&x)[kLane]) {
  if (at + kLane <= count) {
    Words4* p = reinterpret_cast<Words4*>(base + at);
    p[0] = Words4{{x[0], x[1], x[2], x[3]}};
    p[1] = Words4{{x[4], x[5], x[6], x[7]}};
    return;
  }
#pragma unroll
  for (int k = 0; k < kLane; ++k)
    if (at + k < count) base[at + k] = x[k];
}

// 32 random bits of a state's element: its index and the step's key through a
// bijection of 32-bit words (two multiplications, three folds), with the high
// half of the key in between.
__device__ __forceinline__ uint32_t random_bits(uint32_t z, uint32_t key_high) {
  z = (z ^ (z >> 16)) * 0x7FEB352Du;
  z ^= key_high;
  z = (z ^ (z >> 15)) * 0x846CA68Bu;
  return z ^ (z >> 16);
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Four e4m3 values of a word, exactly.
__device__ __forceinline__ void from_f8(uint32_t w, float* x) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo.x;
  x[1] = lo.y;
  x[2] = hi.x;
  x[3] = hi.y;
}

__device__ __forceinline__ uint32_t to_f8(const float* x) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  return (uint32_t)w;
}

// |x| < 256 to a value of e4m3, up with the chance of what is cut off; draw: 20
// random bits.  Normal values lose the 20 low bits of their mantissa, those
// below 2^-6 what is left of a multiple of 2^-9.
__device__ __forceinline__ float round_f8(float x, uint32_t draw) {
  const float normal = __uint_as_float((__float_as_uint(x) + draw) & 0xFFF00000u);
  const float small = floorf(x * 512.f + (float)draw * 0x1p-20f) * 0x1p-9f;
  return x < 0x1p-6f ? small : normal;
}

// Largest of the 16 lanes that hold a block (magnitudes as words, so that a
// NaN is the largest).
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) {
    const uint32_t o = __shfl_xor(v, off);
    v = o > v ? o : v;
  }
  return v;
}

// Exponent field of a block's scale, from the words of its largest magnitude.
__device__ __forceinline__ uint32_t scale_exponent(uint32_t most) {
  const uint32_t e = most >> 23;
  return e > 8 ? e - 7 : 1;
}

template <bool F8>
__global__ void __launch_bounds__(kThreads)
adamw_kernel(OptimBatch b, OptimPointers p, AdamArgs a) {
  const float factor = a.factor ? *a.factor : 1.f;
  if (!(fabsf(factor) < INFINITY)) return;
  const int32_t chunk = b.first_chunk + blockIdx.x;
  const int32_t i = b.chunk_tensor[chunk];
  const OptimTensor t = b.tensors[i];
  const int32_t at_batch = i - b.first;
  const void* grad = p.grad[at_batch];
  void* param = p.param[at_batch];
  uint16_t* copy = p.copy[at_batch];
  const float lr = a.lr * t.lr_scale;
  const float keep = 1.f - lr * t.weight_decay;
  const float step = lr * a.inv_c1;
  const int64_t padded = (t.count + kStateBlock - 1) / kStateBlock * kStateBlock;
#pragma unroll
  for (int u = 0; u < kOptimChunk / (kThreads * kLane); ++u) {
    const int64_t e = (int64_t)(chunk - t.first_chunk) * kOptimChunk +
                      (u * kThreads + (int)threadIdx.x) * kLane;
    if (e >= padded) continue;  // a block's 16 lanes alike
    const int64_t s = t.state + e;
    float g[kLane], x[kLane], m[kLane], v[kLane];
    load8(grad, t.grad_bf16, e, t.count, g);
    load8(param, t.param_bf16, e, t.count, x);
    if constexpr (F8) {
      const uint2 mw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.m) + s);
      const uint2 vw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.v) + s);
      const float ms = a.m_scale[s / kStateBlock], vs = a.v_scale[s / kStateBlock];
      from_f8(mw.x, m);
      from_f8(mw.y, m + 4);
      from_f8(vw.x, v);
      from_f8(vw.y, v + 4);
#pragma unroll
      for (int k = 0; k < kLane; ++k) {
        m[k] *= ms;
        v[k] *= vs;
        v[k] *= v[k];
      }
    } else {
      load8(a.m, 0, s, INT64_MAX, m);
      load8(a.v, 0, s, INT64_MAX, v);
    }
    float root[kLane];
#pragma unroll
    for (int k = 0; k < kLane; ++k) {
      const float gk = g[k] * factor;
      m[k] = a.beta1 * m[k] + a.one_minus_beta1 * gk;
      v[k] = a.beta2 * v[k] + a.one_minus_beta2 * (gk * gk);
      if (e + k >= t.count) m[k] = v[k] = 0.f;
      root[k] = sqrtf(v[k]);
      x[k] = x[k] * keep - step * (m[k] / (root[k] * a.inv_root_c2 + a.eps));
    }
    uint32_t r[kLane];
    if (F8 || a.stochastic) {
      const uint32_t z = (uint32_t)s + a.key_low + (uint32_t)((uint64_t)s >> 32) * 0x9E3779B9u;
#pragma unroll
      for (int k = 0; k < kLane; ++k) r[k] = random_bits(z + k, a.key_high);
    }
    if constexpr (F8) {
      uint32_t most_m = 0, most_v = 0;
#pragma unroll
      for (int k = 0; k < kLane; ++k) {
        most_m = max(most_m, __float_as_uint(m[k]) & 0x7FFFFFFFu);
        most_v = max(most_v, __float_as_uint(root[k]));
      }
      const uint32_t em = scale_exponent(block_max(most_m));
      const uint32_t ev = scale_exponent(block_max(most_v));
      const float im = __uint_as_float((254u - em) << 23), iv = __uint_as_float((254u - ev) << 23);
      float qm[kLane], qv[kLane];
#pragma unroll
      for (int k = 0; k < kLane; ++k) {
        qm[k] = copysignf(round_f8(fabsf(m[k]) * im, r[k] & 0xFFFFFu), m[k]);
        qv[k] = round_f8(root[k] * iv, r[k] >> 12);
        if (qv[k] == 0.f && root[k] > 0.f) qv[k] = 0x1p-9f;
      }
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + s) =
          make_uint2(to_f8(qm), to_f8(qm + 4));
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + s) =
          make_uint2(to_f8(qv), to_f8(qv + 4));
      if (threadIdx.x % 16 == 0) {
        a.m_scale[s / kStateBlock] = __uint_as_float(em << 23);
        a.v_scale[s / kStateBlock] = __uint_as_float(ev << 23);
      }
    } else {
      store8_f32(static_cast<float*>(a.m), s, INT64_MAX, m);
      store8_f32(static_cast<float*>(a.v), s, INT64_MAX, v);
    }
    uint32_t h[kLane];
    if (t.param_bf16) {
#pragma unroll
      for (int k = 0; k < kLane; ++k) {
        h[k] = bf16_nearest(x[k]);
        if (a.stochastic && fabsf(x[k]) < INFINITY)
          h[k] = (__float_as_uint(x[k]) + (r[k] & 0xFFFFu)) >> 16;
      }
      store8_bf16(static_cast<uint16_t*>(param), e, t.count, h);
    } else {
      store8_f32(static_cast<float*>(param), e, t.count, x);
#pragma unroll
      for (int k = 0; k < kLane; ++k) h[k] = bf16_nearest(x[k]);
    }
    if (copy) store8_bf16(copy, e, t.count, h);
  }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// The sum over a workgroup of 256, on every thread of its first wave.
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double part[kThreads / kWave];
  v = wave_sum_f64(v);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ void __launch_bounds__(kThreads)
norm_chunk_kernel(OptimBatch b, OptimPointers p, double* __restrict__ partial) {
  const int32_t chunk = b.first_chunk + blockIdx.x;
  const int32_t i = b.chunk_tensor[chunk];
  const OptimTensor t = b.tensors[i];
  const void* grad = p.grad[i - b.first];
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < kOptimChunk / (kThreads * kLane); ++u) {
    const int64_t e = (int64_t)(chunk - t.first_chunk) * kOptimChunk +
                      (u * kThreads + (int)threadIdx.x) * kLane;
    float g[kLane];
    load8(grad, t.grad_bf16, e, t.count, g);
#pragma unroll
    for (int k = 0; k < kLane; ++k) sum = fma((double)g[k], (double)g[k], sum);
  }
  sum = group_sum(sum);
  if (threadIdx.x == 0) partial[chunk] = sum;
}

__global__ void __launch_bounds__(kThreads)
norm_tensor_kernel(const OptimTensor* __restrict__ tensors, const double* __restrict__ partial,
                   double* __restrict__ squares, float scale, float* __restrict__ norms) {
  const OptimTensor t = tensors[blockIdx.x];
  const int64_t chunks = (t.count + kOptimChunk - 1) / kOptimChunk;
  double sum = 0.0;
  for (int64_t c = threadIdx.x; c < chunks; c += kThreads) sum += partial[t.first_chunk + c];
  sum = group_sum(sum);
  if (threadIdx.x == 0) {
    squares[blockIdx.x] = sum;
    if (norms) norms[blockIdx.x] = (float)((double)scale * sqrt(sum));
  }
}

__global__ void __launch_bounds__(kThreads)
norm_total_kernel(const double* __restrict__ squares, int32_t num, float scale, float max_norm,
                  float* __restrict__ total) {
  double sum = 0.0;
  for (int32_t i = threadIdx.x; i < num; i += kThreads) sum += squares[i];
  sum = group_sum(sum);
  if (threadIdx.x == 0) {
    const double norm = (double)scale * sqrt(sum);
    const float out = (float)norm;
    double factor = scale;
    if (norm > (double)max_norm) factor *= (double)max_norm / norm;
    total[0] = out;
    total[1] = out < INFINITY ? (float)factor : NAN;
  }
}

}  // namespace

hipError_t launch_adamw(bool f8, const OptimBatch& b, const OptimPointers& p, const AdamArgs& a,
                        hipStream_t stream) {
  hipLaunchKernelGGL(f8 ? adamw_kernel<true> : adamw_kernel<false>, dim3((unsigned)b.chunks),
                     dim3(kThreads), 0, stream, b, p, a);
  return hipGetLastError();
}

hipError_t launch_norm_chunks(const OptimBatch& b, const OptimPointers& p, double* partial,
                              hipStream_t stream) {
  hipLaunchKernelGGL(norm_chunk_kernel, dim3((unsigned)b.chunks), dim3(kThreads), 0, stream, b, p,
                     partial);
  return hipGetLastError();
}

hipError_t launch_norm_tensors(const OptimTensor* tensors, int32_t num, const double* partial,
                               double* squares, float scale, float* norms, hipStream_t stream) {
  hipLaunchKernelGGL(norm_tensor_kernel, dim3((unsigned)num), dim3(kThreads), 0, stream, tensors,
                     partial, squares, scale, norms);
  return hipGetLastError();
}

hipError_t launch_norm_total(const double* squares, int32_t num, float scale, float max_norm,
                             float* total, hipStream_t stream) {
  hipLaunchKernelGGL(norm_total_kernel, dim3(1), dim3(kThreads), 0, stream, squares, num, scale,
                     max_norm, total);
  return hipGetLastError();
}

}  // namespace arc
