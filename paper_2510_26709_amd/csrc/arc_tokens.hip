// Token log probabilities: for each row of logits the normaliser, the log
// probability of the given token, the entropy and the top alternatives, and
// their gradient (the formulas are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arc_device.h"
#include "arc_train.h"

namespace arc {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

template <bool BF16>
__device__ __forceinline__ float logit(const void* row, int64_t j) {
  if constexpr (BF16)
    return __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[j] << 16);
  return static_cast<const float*>(row)[j];
}

template <bool BF16>
__device__ __forceinline__ const void* row_at(const void* base, int64_t element) {
  return static_cast<const char*>(base) + element * (BF16 ? 2 : 4);
}

// Softmax statistics of part of a row relative to its largest value `most`:
// total = sum exp(z - most), spread = sum exp(z - most) (z - most).
struct Stats {
  float most, total, spread;
};

__device__ __forceinline__ Stats join(Stats a, Stats b) {
  const float most = fmaxf(a.most, b.most);
  if (most == -INFINITY)  // nothing, or NaN, on both sides
    return {most, a.total + b.total, a.spread + b.spread};
  const float da = a.most - most, db = b.most - most;
  const float ea = expf(da), eb = expf(db);
  // a side without weight adds nothing, however far away (0 * infinity); NaN
  // goes by way of the total
  const float sa = ea > 0.f ? ea * (a.spread + da * a.total) : 0.f;
  const float sb = eb > 0.f ? eb * (b.spread + db * b.total) : 0.f;
  return {most, ea * a.total + eb * b.total, sa + sb};
}

// A larger key is a larger logit, or the same logit of a lower token.
__device__ __forceinline__ uint64_t rank_key(float x, int64_t j) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  const uint32_t up = b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  return ((uint64_t)up << 32) | (0xFFFFFFFFu - (uint32_t)j);
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads)
token_score_kernel(TokenArgs a, TokenScores out) {
  __shared__ Stats part[kWaves];
  __shared__ uint64_t best[kWaves];
  const int64_t i = blockIdx.x, V = a.vocab;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const void* row = row_at<BF16>(a.logits, i * a.stride);
  Stats s{-INFINITY, 0.f, 0.f};
  for (int64_t j = threadIdx.x; j < V; j += kThreads) {
    const float z = logit<BF16>(row, j) * a.scale;
    if (z == -INFINITY) continue;
    s = join(s, {z, z != z ? z : 1.f, 0.f});
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1)
    s = join(s, {__shfl_xor(s.most, off), __shfl_xor(s.total, off), __shfl_xor(s.spread, off)});
  if (lane == 0) part[wave] = s;
  __syncthreads();
  s = part[0];
  for (int w = 1; w < kWaves; ++w) s = join(s, part[w]);
  const bool empty = s.total == 0.f;
  const float log_total = logf(s.total);
  const float lse = empty ? -INFINITY : s.most + log_total;
  if (threadIdx.x == 0) {
    if (out.lse) out.lse[i] = lse;
    if (out.entropy) out.entropy[i] = empty ? 0.f : log_total - s.spread / s.total;
    if (out.logp) {
      const int64_t y = a.targets[i];
      float lp = 0.f;
      if (y >= V)
        lp = NAN;
      else if (y >= 0)
        lp = empty ? -INFINITY : (logit<BF16>(row, y) * a.scale - s.most) - log_total;
      out.logp[i] = lp;
    }
  }
  if (!out.top_ids) return;
  const bool none = lse != lse;
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t key = 0;
    if (!none)
      for (int64_t j = threadIdx.x; j < V; j += kThreads) {
        const uint64_t q = rank_key(logit<BF16>(row, j), j);
        if (q < last && q > key) key = q;
      }
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const uint64_t q = __shfl_xor((unsigned long long)key, off);
      key = q > key ? q : key;
    }
    __syncthreads();
    if (lane == 0) best[wave] = key;
    __syncthreads();
    key = best[0];
    for (int w = 1; w < kWaves; ++w) key = best[w] > key ? best[w] : key;
    last = key;
    if (threadIdx.x == 0) {
      const int64_t j = 0xFFFFFFFFu - (uint32_t)key;
      out.top_ids[i * a.top + k] = none ? -1 : (int32_t)j;
      out.top_logp[i * a.top + k] =
          none ? NAN : empty ? -INFINITY : (logit<BF16>(row, j) * a.scale - s.most) - log_total;
    }
  }
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads)
token_grad_kernel(TokenArgs a, TokenGrad g) {
  const int64_t i = blockIdx.x, V = a.vocab;
  const void* row = row_at<BF16>(a.logits, i * a.stride);
  void* to = const_cast<void*>(row_at<BF16>(g.grad, i * g.stride));
  const int64_t y = a.targets && g.d_logp ? a.targets[i] : -1;
  const float dl = g.d_logp && y >= 0 ? g.d_logp[i] : 0.f;
  const float dh = g.d_entropy ? g.d_entropy[i] : 0.f;
  const float dz = g.d_lse ? g.d_lse[i] : 0.f;
  const float lse = g.lse[i], H = g.d_entropy ? g.entropy[i] : 0.f;
  const bool zero = (dl == 0.f && dh == 0.f && dz == 0.f) || lse == -INFINITY;
  for (int64_t j = threadIdx.x; j < V; j += kThreads) {
    float d = 0.f;
    if (!zero) {
      const float lp = logit<BF16>(row, j) * a.scale - lse;
      const float p = expf(lp);
      d = p * (dz - dl);
      if (p != 0.f) d -= dh * (p * (lp + H));
      if (j == y) d += dl;
      d *= a.scale;
    }
    if constexpr (BF16) {
      const uint32_t b = __float_as_uint(d);
      static_cast<uint16_t*>(to)[j] =
          d != d ? 0x7FC0 : (uint16_t)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
    } else {
      static_cast<float*>(to)[j] = d;
    }
  }
}

}  // namespace

hipError_t launch_token_score(const TokenArgs& a, const TokenScores& out, hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(a.bf16 ? token_score_kernel<true> : token_score_kernel<false>,
                     dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a, out);
  return hipGetLastError();
}

hipError_t launch_token_grad(const TokenArgs& a, const TokenGrad& g, hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(a.bf16 ? token_grad_kernel<true> : token_grad_kernel<false>,
                     dim3((unsigned)a.rows), dim3(kThreads), 0, stream, a, g);
  return hipGetLastError();
}

}  // namespace arc
