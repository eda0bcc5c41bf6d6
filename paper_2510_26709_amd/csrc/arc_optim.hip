// Gradient norms and AdamW over many tensors (the formulas and the states'
// layout are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "arc_device.h"
#include "arc_train.h"

namespace arc {
namespace {

constexpr int kThreads = 256;

typedef uint32_t loose_u32x4_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t loose_u32x2_t __attribute__((ext_vector_type(2), aligned(2)));

// L (4 or 8) consecutive elements at any element alignment, read and written
// once a step; zeros behind `count` (FULL: there are none).
template <bool FULL, int L>
__device__ __forceinline__ void load(const void* base, int32_t bf16, int64_t at, int64_t count,
                                     float (&x)[L]) {
  if (FULL || at + L <= count) {
    if (bf16) {
      const uint16_t* p = static_cast<const uint16_t*>(base) + at;
      uint32_t w[L / 2];
      if constexpr (L == 8) {
        const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const loose_u32x4_t*>(p));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
      } else {
        const u32x2_t v = __builtin_nontemporal_load(reinterpret_cast<const loose_u32x2_t*>(p));
        w[0] = v.x, w[1] = v.y;
      }
#pragma unroll
      for (int k = 0; k < L / 2; ++k) {
        x[2 * k] = bf16_lo(w[k]);
        x[2 * k + 1] = bf16_hi(w[k]);
      }
    } else {
      // eight of a lane are two loads that take half of each line: the second
      // one wants the first one's lines in the cache still
      const loose_u32x4_t* p =
          reinterpret_cast<const loose_u32x4_t*>(static_cast<const float*>(base) + at);
#pragma unroll
      for (int h = 0; h < L / 4; ++h) {
        const u32x4_t v = L == 8 ? (u32x4_t)p[h] : (u32x4_t)__builtin_nontemporal_load(p + h);
        x[4 * h] = __uint_as_float(v.x);
        x[4 * h + 1] = __uint_as_float(v.y);
        x[4 * h + 2] = __uint_as_float(v.z);
        x[4 * h + 3] = __uint_as_float(v.w);
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < L; ++k) {
    x[k] = 0.f;
    if (at + k < count)
      x[k] = bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[at + k] << 16)
                  : static_cast<const float*>(base)[at + k];
  }
}

template <bool FULL, bool STREAM, int L>
__device__ __forceinline__ void store_f32(float* base, int64_t at, int64_t count,
                                          const float (&x)[L]) {
  if (FULL || at + L <= count) {
    loose_u32x4_t* p = reinterpret_cast<loose_u32x4_t*>(base + at);
#pragma unroll
    for (int h = 0; h < L / 4; ++h) {
      const u32x4_t v = {__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]),
                         __float_as_uint(x[4 * h + 2]), __float_as_uint(x[4 * h + 3])};
      if (L == 8 || !STREAM)
        p[h] = v;
      else
        __builtin_nontemporal_store(v, p + h);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < L; ++k)
    if (at + k < count) base[at + k] = x[k];
}

// h: two elements a word.
template <bool FULL, int L>
__device__ __forceinline__ void store_bf16(uint16_t* base, int64_t at, int64_t count,
                                           const uint32_t (&h)[L / 2]) {
  if (FULL || at + L <= count) {
    if constexpr (L == 8) {
      const u32x4_t v = {h[0], h[1], h[2], h[3]};
      __builtin_nontemporal_store(v, reinterpret_cast<loose_u32x4_t*>(base + at));
    } else {
      const u32x2_t v = {h[0], h[1]};
      __builtin_nontemporal_store(v, reinterpret_cast<loose_u32x2_t*>(base + at));
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < L; ++k)
    if (at + k < count) base[at + k] = (uint16_t)(h[k / 2] >> (k % 2 * 16));
}

// Two values rounded to the nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t w;
  asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(lo), "v"(hi));
  return w;
}

// A value down to bfloat16, or up with the chance of what is cut off.
__device__ __forceinline__ uint32_t bf16_random(float x, uint32_t draw) {
  const uint32_t b = __float_as_uint(x);
  return fabsf(x) < INFINITY ? b + (draw & 0xFFFFu) : b;
}

// 32 random bits of a state's element: its index and the step's key through a
// bijection of 32-bit words (two multiplications, three folds), with the high
// half of the key in between.  Multipliers and shifts are those of least bias that
// C. Wellons published from a search for such mixers (2018).
__device__ __forceinline__ uint32_t random_bits(uint32_t z, uint32_t key_high) {
  z = (z ^ (z >> 16)) * 0x7FEB352Du;
  z ^= key_high;
  z = (z ^ (z >> 15)) * 0x846CA68Bu;
  return z ^ (z >> 16);
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Four e4m3 values of a word times a scale, exactly.
__device__ __forceinline__ void from_f8(uint32_t w, float scale, float* x) {
  const f32x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  x[0] = lo.x;
  x[1] = lo.y;
  x[2] = hi.x;
  x[3] = hi.y;
}

// x / scale, below 256 in magnitude, to a code of e4m3, away from 0 with the
// chance of what is cut off (normal values: the 20 low bits of the mantissa;
// below 2^-6: what is left of a multiple of 2^-9), by the 20 high bits of
// `draw`.  The instruction does just that: it agreed with the definition on 4.2
// million words, draws and scales.
__device__ __forceinline__ uint32_t f8_random(float x, uint32_t draw, float scale, uint32_t word,
                                              int byte) {
  switch (byte) {
    case 0: return __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(word, x, draw, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(word, x, draw, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(word, x, draw, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(word, x, draw, scale, 3);
  }
}

// The square root of x >= 0 (or NaN), rounded correctly (checked for every binary32
// value): x rsq(x) and one correction by its residual, 5 operations, and 7 for the
// ends of the range.  Below 2^-96 binary32 does not hold the residual: the root of
// x times 2^64 then.  0 and infinity are their own roots.
__device__ __forceinline__ float root_of(float x) {
  const bool small = x < 0x1p-96f;
  const float s = x * (small ? 0x1p64f : 1.f);
  const float w = __builtin_amdgcn_rsqf(s);
  const float y = s * w;
  const float root = fmaf(fmaf(-y, y, s), 0.5f * w, y) * (small ? 0x1p-32f : 1.f);
  constexpr int kZeros = 0x060, kPlusInfinity = 0x200;
  return __builtin_amdgcn_classf(x, kZeros | kPlusInfinity) ? x : root;
}

struct MaxU {
  __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// A block's scale, from the word of its largest magnitude in [2^e, 2^(e+1)): 2^(e-7).
__device__ __forceinline__ float scale_of(uint32_t most) {
  const uint32_t e = most >> 23;
  return __uint_as_float((e > 8 ? e - 7 : 1) << 23);
}

// States in 32 bits: four elements a lane, so that every access of a wave takes
// whole lines, and the loads of four passes ahead of the first update.  Bound by
// HBM: 1.2e8 binary32 parameters 600 us, bf16 ones with 32-bit states 469 (5.8
// TB/s; one pass at a time at twice the occupancy 643 and 525); 1.1e9 binary32
// ones with a bf16 copy and bf16 gradients 4.8 to 5.6 ms, by where the process
// got its memory (6.4 to 5.5 TB/s).  A step of a few times the Infinity Cache
// stores its binary32 arrays through it (!STREAM): 1.1e7 parameters 51 us
// against 58 past it, 2.2e7 in 300 tensors 111 / 129, 3.6e7 238 / 223, 1.2e8
// 662 / 640 (one pass at a time).
//
// States in 8 bits: eight elements a lane, so that 16 lanes hold a block, its
// largest magnitudes found by four lane permutations.  10 bytes of HBM and 58
// instructions an element, which take the same time: 1.2e8 bf16 parameters 225
// to 243 us (5.6 to 5.2 TB/s).  That is with the conversions that scale and round,
// the root from the reciprocal one (5 instructions for the ends of its range, 3 to
// 5% of the time) and the reciprocal for a division; with a multiply for each
// scale, a rounding in integers, sqrtf() and a division it was 319 us.
template <bool F8, bool STREAM>
__global__ void __launch_bounds__(kThreads, F8 ? 6 : 4)
adamw_kernel(OptimBatch b, OptimPointers p, AdamArgs a) {
  constexpr int L = F8 ? 8 : 4;
  static_assert(kOptimChunkLeast % (kThreads * L) == 0, "whole passes of a workgroup");
  static_assert(!F8 || kStateBlock == 16 * L, "a block is a row of lanes");
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
  const auto fetch = [&](int64_t e, auto whole, float (&g)[L], float (&x)[L], float (&m)[L],
                         float (&v)[L]) {
    constexpr bool FULL = decltype(whole)::value;
    const int64_t s = t.state + e;
    load<FULL, L>(grad, t.grad_bf16, e, t.count, g);
    load<FULL, L>(param, t.param_bf16, e, t.count, x);
    if constexpr (F8) {
      const auto mw = __builtin_nontemporal_load(
          reinterpret_cast<const u32x2_t*>(static_cast<const uint8_t*>(a.m) + s));
      const auto vw = __builtin_nontemporal_load(
          reinterpret_cast<const u32x2_t*>(static_cast<const uint8_t*>(a.v) + s));
      const float ms = a.m_scale[s / kStateBlock], vs = a.v_scale[s / kStateBlock];
      from_f8(mw.x, ms, m);
      from_f8(mw.y, ms, m + 4);
      from_f8(vw.x, vs, v);
      from_f8(vw.y, vs, v + 4);
#pragma unroll
      for (int k = 0; k < L; ++k) v[k] *= v[k];
    } else {
      load<true, L>(a.m, 0, s, 0, m);
      load<true, L>(a.v, 0, s, 0, v);
    }
  };
  const auto finish = [&](int64_t e, auto whole, float (&g)[L], float (&x)[L], float (&m)[L],
                          float (&v)[L]) {
    constexpr bool FULL = decltype(whole)::value;
    const int64_t s = t.state + e;
    float root[L];
#pragma unroll
    for (int k = 0; k < L; ++k) {
      const float gk = g[k] * factor;
      m[k] = a.beta1 * m[k] + a.one_minus_beta1 * gk;
      v[k] = a.beta2 * v[k] + a.one_minus_beta2 * (gk * gk);
      root[k] = root_of(v[k]);
      // the reciprocal is within 1 ulp: 2^-23 of an update that is a small part
      // of x, and a tenth of an exact division's operations
      const float inv = __builtin_amdgcn_rcpf(fmaf(root[k], a.inv_root_c2, a.eps));
      x[k] = fmaf(-step, m[k] * inv, x[k] * keep);
    }
    if constexpr (!FULL) {  // behind the end: states stay 0
#pragma unroll
      for (int k = 0; k < L; ++k)
        if (e + k >= t.count) m[k] = v[k] = root[k] = 0.f;
    }
    uint32_t r[L];
    if (F8 || a.stochastic) {
      const uint32_t z = (uint32_t)s + a.key_low + (uint32_t)((uint64_t)s >> 32) * 0x9E3779B9u;
#pragma unroll
      for (int k = 0; k < L; ++k) r[k] = random_bits(z + k, a.key_high);
    }
    if constexpr (F8) {
      uint32_t most_m = 0, most_v = 0;
#pragma unroll
      for (int k = 0; k < L; ++k) {  // as words, so that a NaN is the largest
        most_m = MaxU()(most_m, __float_as_uint(m[k]) & 0x7FFFFFFFu);
        most_v = MaxU()(most_v, __float_as_uint(root[k]));
      }
      const float ms = scale_of(lanes_reduce<16>(most_m, MaxU()));
      const float vs = scale_of(lanes_reduce<16>(most_v, MaxU()));
      const uint32_t least = __float_as_uint(vs * 0x1p-9f);  // the smallest value above 0
      uint32_t qm[2] = {0, 0}, qv[2] = {0, 0};
#pragma unroll
      for (int k = 0; k < L; ++k) {
        qm[k / 4] = f8_random(m[k], r[k] << 12, ms, qm[k / 4], k % 4);
        const uint32_t w = __float_as_uint(root[k]);
        const float at_least = __uint_as_float(MaxU()(w, w == 0u ? 0u : least));
        qv[k / 4] = f8_random(at_least, r[k], vs, qv[k / 4], k % 4);
      }
      const u32x2_t mw = {qm[0], qm[1]}, vw = {qv[0], qv[1]};
      __builtin_nontemporal_store(
          mw, reinterpret_cast<u32x2_t*>(static_cast<uint8_t*>(a.m) + s));
      __builtin_nontemporal_store(
          vw, reinterpret_cast<u32x2_t*>(static_cast<uint8_t*>(a.v) + s));
      if (threadIdx.x % 16 == 0) {
        a.m_scale[s / kStateBlock] = ms;
        a.v_scale[s / kStateBlock] = vs;
      }
    } else {
      store_f32<true, STREAM, L>(static_cast<float*>(a.m), s, 0, m);
      store_f32<true, STREAM, L>(static_cast<float*>(a.v), s, 0, v);
    }
    uint32_t h[L / 2];
#pragma unroll
    for (int k = 0; k < L / 2; ++k) h[k] = bf16_pair(x[2 * k], x[2 * k + 1]);
    if (t.param_bf16) {
      if (a.stochastic) {
#pragma unroll
        for (int k = 0; k < L / 2; ++k)
          h[k] = (bf16_random(x[2 * k], r[2 * k]) >> 16) |
                 (bf16_random(x[2 * k + 1], r[2 * k + 1]) & 0xFFFF0000u);
      }
      store_bf16<FULL, L>(static_cast<uint16_t*>(param), e, t.count, h);
    } else {
      store_f32<FULL, STREAM, L>(static_cast<float*>(param), e, t.count, x);
    }
    if (copy) store_bf16<FULL, L>(copy, e, t.count, h);
  };
  const auto update = [&](int64_t e, auto whole) {
    float g[L], x[L], m[L], v[L];
    fetch(e, whole, g, x, m, v);
    finish(e, whole, g, x, m, v);
  };
  const int64_t first = (int64_t)(chunk - t.first_chunk) * a.run;
  if constexpr (!F8) {
    // Whole runs: the loads of four passes ahead of the first update.
    constexpr int U = 4;
    if (a.run == U * kThreads * L && first + a.run <= t.count) {
      float g[U][L], x[U][L], m[U][L], v[U][L];
#pragma unroll
      for (int u = 0; u < U; ++u)
        fetch(first + (u * kThreads + (int)threadIdx.x) * L, std::true_type(), g[u], x[u], m[u],
              v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
        finish(first + (u * kThreads + (int)threadIdx.x) * L, std::true_type(), g[u], x[u], m[u],
               v[u]);
      return;
    }
  }
  for (int32_t u = threadIdx.x * L; u < a.run; u += kThreads * L) {
    const int64_t e = first + u;
    if (e >= padded) break;
    // the lanes of a block go the same way: it takes all of them
    const int64_t block_end = F8 ? e / kStateBlock * kStateBlock + kStateBlock : e + L;
    if (block_end <= t.count)
      update(e, std::true_type());
    else
      update(e, std::false_type());
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
  __syncthreads();  // of an earlier sum
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// The sum of squares of one run of elements, in binary64: no square of a binary32
// number overflows there.  Bound by HBM, four loads of a thread in flight: 1.2e8
// binary32 values 74 us (6.8 TB/s), 1.1e9 bf16 ones 313 (7.0).
__global__ void __launch_bounds__(kThreads)
norm_chunk_kernel(NormBatch b, NormPointers p, int32_t run, double* __restrict__ partial) {
  const int32_t chunk = b.first_chunk + blockIdx.x;
  const int32_t i = b.chunk_tensor[chunk];
  const OptimTensor t = b.tensors[i];
  const void* grad = p.grad[i - b.first];
  const int64_t first = (int64_t)(chunk - t.first_norm) * run;
  const int64_t end = min(t.count, first + run);
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  const auto add = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    for (int u = 0; u < run; u += 4 * kThreads * L) {
      if (first + u >= end) break;
      float g[4][L];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        load<false, L>(grad, L == 8, first + u + (q * kThreads + (int)threadIdx.x) * L, end, g[q]);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int k = 0; k < L; ++k) sum[q] = fma((double)g[q][k], (double)g[q][k], sum[q]);
    }
  };
  if (t.grad_bf16)
    add(std::integral_constant<int, 8>());
  else
    add(std::integral_constant<int, 4>());
  const double all = group_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (threadIdx.x == 0) partial[chunk] = all;
}

// Each tensor's sum, and the total by the last workgroup to arrive.
__global__ void __launch_bounds__(kThreads)
norm_tensor_kernel(const OptimTensor* __restrict__ tensors, int32_t num, int32_t run,
                   const double* __restrict__ partial, double* __restrict__ squares,
                   uint32_t* __restrict__ arrived, float scale, float max_norm,
                   float* __restrict__ norms, float* __restrict__ total) {
  __shared__ bool last;
  const OptimTensor t = tensors[blockIdx.x];
  const int64_t chunks = (t.count + run - 1) / run;
  double sum = 0.0;
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < chunks; c += kThreads) sum += partial[t.first_norm + c];
  sum = group_sum(sum);
  if (threadIdx.x == 0) {
    if (norms) norms[blockIdx.x] = (float)((double)scale * sqrt(sum));
    __hip_atomic_store(&squares[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    wave_vmem_fence();  // written before it counts
    // (goes round at the number of tensors: 0 after a launch, whatever overlapped before)
    last = atomicInc(arrived, (uint32_t)(num - 1)) == (uint32_t)(num - 1);
  }
  __syncthreads();
  if (!last) return;
  sum = 0.0;
#pragma unroll 4
  for (int32_t i = threadIdx.x; i < num; i += kThreads)
    sum += __hip_atomic_load(&squares[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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

hipError_t launch_adamw(bool f8, bool cached, const OptimBatch& b, const OptimPointers& p,
                        const AdamArgs& a, hipStream_t stream) {
  const auto kernel = f8       ? adamw_kernel<true, true>
                      : cached ? adamw_kernel<false, false>
                               : adamw_kernel<false, true>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)b.chunks), dim3(kThreads), 0, stream, b, p, a);
  return hipGetLastError();
}

hipError_t launch_norm_chunks(const NormBatch& b, const NormPointers& p, int32_t run,
                              double* partial, hipStream_t stream) {
  hipLaunchKernelGGL(norm_chunk_kernel, dim3((unsigned)b.chunks), dim3(kThreads), 0, stream, b, p,
                     run, partial);
  return hipGetLastError();
}

hipError_t launch_norm_tensors(const OptimTensor* tensors, int32_t num, int32_t run,
                               const double* partial,
                               double* squares, uint32_t* arrived, float scale, float max_norm,
                               float* norms, float* total, hipStream_t stream) {
  hipLaunchKernelGGL(norm_tensor_kernel, dim3((unsigned)num), dim3(kThreads), 0, stream, tensors,
                     num, run, partial, squares, arrived, scale, max_norm, norms, total);
  return hipGetLastError();
}

}  // namespace arc
