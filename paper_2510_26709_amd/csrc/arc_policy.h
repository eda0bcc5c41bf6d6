// One token's policy loss on the device: for the kernels that hold rows of logits
// (arc_tokens.hip) and the one that has their log probabilities (arc_objective.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arc_device.h"
#include "arc_objective.h"

namespace arc {

struct PolicyTerm {
  float loss, ratio, kl;      // of the token, not weighted
  float d_logp, d_entropy;    // weighted
  float weight;
  bool clipped;
};

struct ExpBeyond {
  float one, line;  // e^x - 1, e^x - 1 - x
};

// Without the differences that cancel them near 0: up to |x| = 1 by e^x's series (what is
// left out is 2^-27 of the value), where the plain difference of binary32 numbers would
// lose two bits and, further in, all.
__device__ __forceinline__ ExpBeyond exp_beyond(float x) {
  if (!(fabsf(x) < 1.f)) {
    const float e = expf(x);
    return {e - 1.f, e == INFINITY ? INFINITY : e - 1.f - x};
  }
  float s = 1.f / 39916800.f;
  s = fmaf(s, x, 1.f / 3628800.f);
  s = fmaf(s, x, 1.f / 362880.f);
  s = fmaf(s, x, 1.f / 40320.f);
  s = fmaf(s, x, 1.f / 5040.f);
  s = fmaf(s, x, 1.f / 720.f);
  s = fmaf(s, x, 1.f / 120.f);
  s = fmaf(s, x, 1.f / 24.f);
  s = fmaf(s, x, 1.f / 6.f);
  s = fmaf(s, x, 0.5f);
  s = s * x * x;
  return {x + s, s};
}

// What a token's terms are made of.
struct PolicyToken {
  float old_logp, ref_logp, advantage, weight;
};

__device__ __forceinline__ PolicyToken policy_token(const PolicyArgs& p, int64_t i) {
  return {p.old_logp ? p.old_logp[i] : 0.f, p.ref_logp ? p.ref_logp[i] : 0.f, p.advantages[i],
          p.weights ? p.weights[i] : 1.f};
}

// A token's terms; `given`: it has a token of its own.  What a token without one
// holds, and what one of weight 0 does to sums and gradients, is left out by
// selection, not by a product, so that no infinity or NaN there gets through.
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& p, const PolicyToken& of,
                                                  bool given, float logp, float H) {
  PolicyTerm t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, false};
  if (!given) return t;
  const float A = of.advantage;
  t.weight = of.weight * p.scale;
  t.ratio = p.old_logp ? expf(logp - of.old_logp) : logp != logp ? logp : 1.f;
  const float held = fminf(fmaxf(t.ratio, p.low), p.high) * A;
  float gain = t.ratio * A;
  t.clipped = gain > held;  // (a ratio that is NaN is not, and stays one)
  if (t.clipped) gain = held;
  if (p.dual != 0.f && A < 0.f && gain < p.dual * A) {
    gain = p.dual * A;
    t.clipped = true;
  }
  float d = t.clipped ? 0.f : -t.ratio * A;
  t.loss = -gain;
  if (p.ref_logp) {
    const ExpBeyond grown = exp_beyond(of.ref_logp - logp);
    t.kl = grown.line;
    if (p.kl != 0.f) {
      t.loss = fmaf(p.kl, t.kl, t.loss);
      d = fmaf(-p.kl, grown.one, d);
    }
  }
  if (p.entropy != 0.f) t.loss = fmaf(-p.entropy, H, t.loss);
  if (t.weight != 0.f) {
    t.d_logp = t.weight * d;
    t.d_entropy = -p.entropy * t.weight;
  }
  return t;
}

// A token's part of the totals.
__device__ __forceinline__ void add_term(const PolicyTerm& t, float H,
                                         double (&sums)[kPolicyTotals]) {
  if (t.weight == 0.f) return;
  const double w = t.weight;
  sums[0] += w * t.loss;
  sums[1] += w * t.ratio;
  sums[2] += w * t.kl;
  sums[3] += w * H;
  sums[4] += t.clipped ? w : 0.0;
}

// Sums of K values over a workgroup of W threads, on every thread, in a fixed order.
template <int W, int K>
__device__ __forceinline__ void group_sums(double (&v)[K]) {
  __shared__ double part[K][W / kWave];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v[k] += __shfl_xor(v[k], off);
  __syncthreads();  // of an earlier sum
  if (threadIdx.x % kWave == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) part[k][threadIdx.x / kWave] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = part[k][0];
#pragma unroll
    for (int w = 1; w < W / kWave; ++w) v[k] += part[k][w];
  }
}

// The values of workgroup `group` of `groups`, the same on all its threads, to
// `totals`: alone at once, otherwise by the last one to arrive, in the order of the
// groups.  They are written through to where every compute unit sees them, and
// read from there.
template <int W, int K>
__device__ __forceinline__ void add_groups(double (&v)[K], uint32_t group, uint32_t groups,
                                           ObjectiveScratch* scratch, float* totals) {
  __shared__ bool last;
  if (groups > 1) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        __hip_atomic_store(&scratch->totals[group][k], v[k], __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
      wave_vmem_fence();  // written before it counts
      last = atomicInc(&scratch->arrived[groups], groups - 1) == groups - 1;
    }
    __syncthreads();
    if (!last) return;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.0;
#pragma unroll 4
    for (uint32_t g = threadIdx.x; g < groups; g += W)
#pragma unroll
      for (int k = 0; k < K; ++k)
        v[k] += __hip_atomic_load(&scratch->totals[g][k], __ATOMIC_RELAXED,
                                  __HIP_MEMORY_SCOPE_AGENT);
    group_sums<W, K>(v);
  }
  if (threadIdx.x == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) totals[k] = (float)v[k];
}

// One row's terms; true on the whole first wave of the last row to come, whose turn
// it is to add_rows().  For that wave alone.
__device__ __forceinline__ bool write_row(const PolicyRowTerms& out, int64_t i,
                                          const PolicyTerm& t, float H) {
  uint32_t before = 0;
  if (threadIdx.x == 0) {
    double v[kPolicyTotals] = {};
    add_term(t, H, v);
#pragma unroll
    for (int k = 0; k < kPolicyTotals; ++k)
      __hip_atomic_store(&out.scratch->totals[i][k], v[k], __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    wave_vmem_fence();  // written before it counts
    before = atomicInc(&out.scratch->arrived[out.rows], out.rows - 1);
    if (out.loss) out.loss[i] = t.loss;
    if (out.ratio) out.ratio[i] = t.ratio;
    if (out.kl) out.kl[i] = t.kl;
  }
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)before) == out.rows - 1;
}

__device__ __forceinline__ void add_rows(const PolicyRowTerms& out) {
  double v[kPolicyTotals] = {};
#pragma unroll 2
  for (uint32_t i = threadIdx.x; i < out.rows; i += kWave)
#pragma unroll
    for (int k = 0; k < kPolicyTotals; ++k)
      v[k] += __hip_atomic_load(&out.scratch->totals[i][k], __ATOMIC_RELAXED,
                                __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
  for (int k = 0; k < kPolicyTotals; ++k) {
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v[k] += __shfl_xor(v[k], off);
    if (threadIdx.x == 0) out.totals[k] = (float)v[k];
  }
}

}  // namespace arc
