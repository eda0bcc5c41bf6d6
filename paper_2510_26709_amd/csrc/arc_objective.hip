// The clipped policy loss and the preference loss of token log probabilities
// (the formulas are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "arc_device.h"
#include "arc_objective.h"
#include "arc_policy.h"

namespace arc {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Sums of K values over a workgroup, on every thread, in a fixed order.
template <int K>
__device__ __forceinline__ void group_sums(double (&v)[K]) {
  __shared__ double part[K][kThreads / kWave];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum_f64(v[k]);
  __syncthreads();  // of an earlier sum
  if (threadIdx.x % kWave == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) part[k][threadIdx.x / kWave] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = (part[k][0] + part[k][1]) + (part[k][2] + part[k][3]);
}

// Every workgroup's sums to `totals`: alone at once, otherwise by the last one to
// arrive, in the order of the workgroups.  Parts are written through to where
// every compute unit sees them, and read from there.
template <int K>
__device__ __forceinline__ void add_groups(double (&v)[K], ObjectiveScratch* scratch,
                                           float* totals) {
  __shared__ bool last;
  group_sums<K>(v);
  const uint32_t groups = gridDim.x;
  if (groups > 1) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        __hip_atomic_store(&scratch->totals[blockIdx.x][k], v[k], __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
      wave_vmem_fence();  // written before it counts
      last = __hip_atomic_fetch_add(&scratch->arrived, 1u, __ATOMIC_RELAXED,
                                    __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
      if (last)
        __hip_atomic_store(&scratch->arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.0;
    for (uint32_t g = threadIdx.x; g < groups; g += kThreads)
#pragma unroll
      for (int k = 0; k < K; ++k)
        v[k] += __hip_atomic_load(&scratch->totals[g][k], __ATOMIC_RELAXED,
                                  __HIP_MEMORY_SCOPE_AGENT);
    group_sums<K>(v);
  }
  if (threadIdx.x == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) totals[k] = (float)v[k];
}

// One token a thread and pass: every array is read and written in whole lines.
__global__ void __launch_bounds__(kThreads)
policy_kernel(PolicyArgs p, PolicyRows r, PolicyOutputs out, ObjectiveScratch* scratch) {
  double sums[kPolicyTotals] = {};
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < r.rows;
       i += (int64_t)gridDim.x * kThreads) {
    const bool given = r.targets[i] >= 0;
    const float H = r.entropy ? r.entropy[i] : 0.f;
    const PolicyTerm t = policy_term(p, i, given, r.logp[i], H);
    if (out.loss) out.loss[i] = t.loss;
    if (out.ratio) out.ratio[i] = t.ratio;
    if (out.kl) out.kl[i] = t.kl;
    if (out.d_logp) out.d_logp[i] = t.d_logp;
    if (out.d_entropy) out.d_entropy[i] = t.d_entropy;
    if (t.weight != 0.f) {
      const double w = t.weight;
      sums[0] += w * t.loss;
      sums[1] += w * t.ratio;
      sums[2] += w * t.kl;
      sums[3] += w * H;
      sums[4] += t.clipped ? w : 0.0;
    }
  }
  add_groups<kPolicyTotals>(sums, scratch, out.totals);
}

// ---------------------------------------------------------------- preference

struct Sequence {
  int64_t first, last;  // inside the rows, whatever the offsets hold
};

__device__ __forceinline__ Sequence sequence(const PreferenceArgs& a, int64_t s) {
  const int64_t first = min(max(a.offsets[s], (int64_t)0), a.rows);
  return {first, min(max(a.offsets[s + 1], first), a.rows)};
}

// The sum of logp - ref of the given tokens among [first, last), and their count.
__device__ __forceinline__ void sum_tokens(const PreferenceArgs& a, int64_t first, int64_t last,
                                           double (&v)[2]) {
  constexpr int U = 4;  // passes whose loads are in flight together
  for (int64_t i = first + threadIdx.x; i < last; i += U * kThreads) {
    int64_t y[U];
    float lp[U], ref[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = i + u * kThreads;
      y[u] = at < last ? a.targets[at] : -1;
      lp[u] = at < last ? a.logp[at] : 0.f;
      ref[u] = a.ref_logp && at < last ? a.ref_logp[at] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (y[u] >= 0) {
        v[0] += (double)lp[u] - (double)ref[u];
        v[1] += 1.0;
      }
  }
}

struct PairTerm {
  double loss, reward[2], d[2];  // d: by each token of the two sequences
  double weight;
};

__device__ __forceinline__ PairTerm pair_term(const PreferenceArgs& a, int64_t pair,
                                              const double (&sum)[2], const double (&count)[2]) {
  PairTerm t;
  const double beta = a.beta;
  double share[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    share[k] = a.average ? beta / (count[k] > 1.0 ? count[k] : 1.0) : beta;
    t.reward[k] = sum[k] * share[k];
  }
  const double z = t.reward[0] - t.reward[1] - (double)a.margin;
  double dz;
  if (a.kind == 0) {
    const double e = a.smoothing, s = exp(-fabs(z));  // sigmoid(-|z|) = s / (1 + s)
    const double soft = log1p(s), under = s / (1.0 + s), over = 1.0 / (1.0 + s);
    t.loss = soft + (1.0 - e) * fmax(-z, 0.0) + e * fmax(z, 0.0);
    if (z != z) t.loss = z;
    dz = e * (z >= 0.0 ? over : under) - (1.0 - e) * (z >= 0.0 ? under : over);
    if (z != z) dz = z;
  } else if (a.kind == 1) {
    t.loss = z >= 1.0 ? 0.0 : 1.0 - z;
    dz = z >= 1.0 ? 0.0 : z < 1.0 ? -1.0 : z;
  } else {
    const double off = (z - 0.5) / beta;
    t.loss = off * off;
    dz = 2.0 * off / beta;
  }
  t.weight = (a.weights ? (double)a.weights[pair] : 1.0) * (double)a.scale;
  t.d[0] = t.weight != 0.0 ? t.weight * dz * share[0] : 0.0;
  t.d[1] = t.weight != 0.0 ? -t.weight * dz * share[1] : 0.0;
  return t;
}

__device__ __forceinline__ void write_pair(const PreferenceArgs& a, const PreferenceOutputs& out,
                                           int64_t pair, const PairTerm& t) {
  if (out.loss) out.loss[pair] = (float)t.loss;
  if (out.rewards) {
    out.rewards[pair] = (float)t.reward[0];
    out.rewards[a.pairs + pair] = (float)t.reward[1];
  }
}

__device__ __forceinline__ void add_pair(const PairTerm& t, double (&totals)[kPreferenceTotals]) {
  if (t.weight == 0.0) return;
  totals[0] += t.weight * t.loss;
  totals[1] += t.weight * (t.reward[0] - t.reward[1]);
  totals[2] += t.reward[0] > t.reward[1] ? t.weight : 0.0;
}

__device__ __forceinline__ void write_tokens(const PreferenceArgs& a, float* d_logp, int64_t first,
                                             int64_t last, float d) {
  for (int64_t i = first + threadIdx.x; i < last; i += kThreads)
    d_logp[i] = a.targets[i] < 0 ? 0.f : d;
}

// Rows before the first sequence and behind the last one have no gradient.
__device__ __forceinline__ void clear_outside(const PreferenceArgs& a, float* d_logp) {
  const int64_t head = a.pairs > 0 ? min(max(a.offsets[0], (int64_t)0), a.rows) : 0;
  const int64_t tail =
      a.pairs > 0 ? min(max(a.offsets[2 * a.pairs], (int64_t)0), a.rows) : 0;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = at; i < head; i += step) d_logp[i] = 0.f;
  for (int64_t i = tail + at; i < a.rows; i += step) d_logp[i] = 0.f;
}

// A workgroup takes whole pairs: both sums, then both gradients.
__global__ void __launch_bounds__(kThreads)
preference_kernel(PreferenceArgs a, PreferenceOutputs out, ObjectiveScratch* scratch) {
  double totals[kPreferenceTotals] = {};
  for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    const Sequence seq[2] = {sequence(a, pair), sequence(a, a.pairs + pair)};
    double v[2][2] = {};
    sum_tokens(a, seq[0].first, seq[0].last, v[0]);
    sum_tokens(a, seq[1].first, seq[1].last, v[1]);
    double all[4] = {v[0][0], v[0][1], v[1][0], v[1][1]};
    group_sums<4>(all);
    const PairTerm t = pair_term(a, pair, {all[0], all[2]}, {all[1], all[3]});
    if (threadIdx.x == 0) {
      write_pair(a, out, pair, t);
      add_pair(t, totals);
    }
    if (out.d_logp) {
      write_tokens(a, out.d_logp, seq[0].first, seq[0].last, (float)t.d[0]);
      write_tokens(a, out.d_logp, seq[1].first, seq[1].last, (float)t.d[1]);
    }
  }
  if (out.d_logp) clear_outside(a, out.d_logp);
  add_groups<kPreferenceTotals>(totals, scratch, out.totals);
}

// Few pairs of long sequences: `parts` workgroups for each sequence, one launch
// for the sums and one for the gradients.
__device__ __forceinline__ Sequence part_of(const Sequence& s, int32_t part, int32_t parts) {
  const int64_t run = ((s.last - s.first + parts - 1) / parts + kThreads - 1) / kThreads * kThreads;
  const int64_t first = min(s.first + part * run, s.last);
  return {first, min(first + run, s.last)};
}

__global__ void __launch_bounds__(kThreads)
sequence_sum_kernel(PreferenceArgs a, int32_t parts, ObjectiveScratch* scratch) {
  const Sequence s = part_of(sequence(a, blockIdx.x / parts), blockIdx.x % parts, parts);
  double v[2] = {};
  sum_tokens(a, s.first, s.last, v);
  group_sums<2>(v);
  if (threadIdx.x == 0) {
    scratch->sum[blockIdx.x] = v[0];
    scratch->count[blockIdx.x] = (int64_t)v[1];
  }
}

__global__ void __launch_bounds__(kThreads)
pair_grad_kernel(PreferenceArgs a, int32_t parts, PreferenceOutputs out,
                 ObjectiveScratch* scratch) {
  const int64_t number = blockIdx.x / parts;
  const int32_t part = blockIdx.x % parts;
  const int64_t pair = number < a.pairs ? number : number - a.pairs;
  double v[4] = {};
  for (int32_t q = threadIdx.x; q < parts; q += kThreads)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t at = (pair + k * a.pairs) * parts + q;
      v[2 * k] += scratch->sum[at];
      v[2 * k + 1] += (double)scratch->count[at];
    }
  group_sums<4>(v);
  const PairTerm t = pair_term(a, pair, {v[0], v[2]}, {v[1], v[3]});
  double totals[kPreferenceTotals] = {};
  if (part == 0 && number < a.pairs && threadIdx.x == 0) {
    write_pair(a, out, pair, t);
    add_pair(t, totals);
  }
  if (out.d_logp) {
    const Sequence s = part_of(sequence(a, number), part, parts);
    write_tokens(a, out.d_logp, s.first, s.last, (float)(number < a.pairs ? t.d[0] : t.d[1]));
    clear_outside(a, out.d_logp);
  }
  add_groups<kPreferenceTotals>(totals, scratch, out.totals);
}

}  // namespace

hipError_t launch_policy_terms(const PolicyArgs& p, const PolicyRows& r, const PolicyOutputs& out,
                               ObjectiveScratch* scratch, hipStream_t stream) {
  const int64_t groups = std::max<int64_t>(
      1, std::min<int64_t>(kTotalsGroups, (r.rows + kThreads - 1) / kThreads));
  hipLaunchKernelGGL(policy_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, p, r, out,
                     scratch);
  return hipGetLastError();
}

hipError_t launch_preference(const PreferenceArgs& a, const PreferenceOutputs& out,
                             ObjectiveScratch* scratch, hipStream_t stream) {
  // Parts of a sequence of at least 2048 tokens on average, where there are few.
  constexpr int64_t kPartTokens = 2048;
  const int64_t most = a.pairs > 0 ? kTotalsGroups / (2 * a.pairs) : 0;
  const int64_t parts =
      a.pairs > 0 ? std::min<int64_t>(most, a.rows / (2 * a.pairs) / kPartTokens) : 0;
  if (parts > 1) {
    const auto grid = dim3((unsigned)(2 * a.pairs * parts));
    hipLaunchKernelGGL(sequence_sum_kernel, grid, dim3(kThreads), 0, stream, a, (int32_t)parts,
                       scratch);
    hipLaunchKernelGGL(pair_grad_kernel, grid, dim3(kThreads), 0, stream, a, (int32_t)parts, out,
                       scratch);
    return hipGetLastError();
  }
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(kTotalsGroups, a.pairs));
  hipLaunchKernelGGL(preference_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a, out,
                     scratch);
  return hipGetLastError();
}

}  // namespace arc
