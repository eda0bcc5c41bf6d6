// The clipped policy loss and the preference loss of token log probabilities
// (the formulas are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "arc_device.h"
#include "arc_objective.h"
#include "arc_policy.h"

namespace arc {
namespace {

constexpr int kThreads = 256;

typedef float loose_f4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef int64_t loose_i2_t __attribute__((ext_vector_type(2), aligned(8)));

// Four numbers from i on, of which `left` are there (FULL: all); `none` for an array
// that is not there.
template <bool FULL>
__device__ __forceinline__ void load_four(const float* p, int64_t i, int64_t left, float none,
                                          float (&x)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = none;
  if (!p) return;
  if (FULL) {
    const loose_f4_t v = __builtin_nontemporal_load(reinterpret_cast<const loose_f4_t*>(p + i));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) x[k] = p[i + k];
  }
}

template <bool FULL>
__device__ __forceinline__ void store_four(float* p, int64_t i, int64_t left,
                                           const float (&x)[4]) {
  if (!p) return;
  if (FULL) {
    const loose_f4_t v = {x[0], x[1], x[2], x[3]};
    __builtin_nontemporal_store(v, reinterpret_cast<loose_f4_t*>(p + i));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) p[i + k] = x[k];
  }
}

// Four tokens a thread and pass, every array in 16 bytes a lane.  With a reference, old
// log probabilities and weights 28 bytes of a token are read and 16 written: 4,000,003
// take 38.5 us, 4.6 TB/s, as much as a copy of 256 MB reaches (4.7).  Single words a lane
// took 62 us; twice as many workgroups 46, for the totals of each; the next pass's loads
// ahead 41.  Up to some thousand tokens it is a launch's latency, 4 us.
__global__ void __launch_bounds__(kThreads)
policy_kernel(PolicyArgs p, PolicyRows r, PolicyOutputs out, ObjectiveScratch* scratch) {
  double sums[kPolicyTotals] = {};
  const auto four = [&](int64_t i, auto whole) {
    constexpr bool FULL = decltype(whole)::value;
    const int64_t left = r.rows - i;
    float lp[4], H[4], old[4], ref[4], A[4], w[4];
    bool given[4];
    if constexpr (FULL) {
      const auto* y = reinterpret_cast<const loose_i2_t*>(r.targets + i);
      const loose_i2_t y0 = __builtin_nontemporal_load(y), y1 = __builtin_nontemporal_load(y + 1);
      given[0] = y0[0] >= 0, given[1] = y0[1] >= 0, given[2] = y1[0] >= 0, given[3] = y1[1] >= 0;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) given[k] = k < left && r.targets[i + k] >= 0;
    }
    load_four<FULL>(r.logp, i, left, 0.f, lp);
    load_four<FULL>(r.entropy, i, left, 0.f, H);
    load_four<FULL>(p.old_logp, i, left, 0.f, old);
    load_four<FULL>(p.ref_logp, i, left, 0.f, ref);
    load_four<FULL>(p.advantages, i, left, 0.f, A);
    load_four<FULL>(p.weights, i, left, 1.f, w);
    float loss[4], ratio[4], kl[4], d_logp[4], d_entropy[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const PolicyTerm t = policy_term(p, {old[k], ref[k], A[k], w[k]}, given[k], lp[k], H[k]);
      add_term(t, H[k], sums);
      loss[k] = t.loss, ratio[k] = t.ratio, kl[k] = t.kl;
      d_logp[k] = t.d_logp, d_entropy[k] = t.d_entropy;
    }
    store_four<FULL>(out.loss, i, left, loss);
    store_four<FULL>(out.ratio, i, left, ratio);
    store_four<FULL>(out.kl, i, left, kl);
    store_four<FULL>(out.d_logp, i, left, d_logp);
    store_four<FULL>(out.d_entropy, i, left, d_entropy);
  };
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4; i < r.rows;
       i += (int64_t)gridDim.x * kThreads * 4) {
    if (i + 4 <= r.rows)
      four(i, std::true_type());
    else
      four(i, std::false_type());
  }
  group_sums<kThreads, kPolicyTotals>(sums);
  add_groups<kThreads, kPolicyTotals>(sums, blockIdx.x, gridDim.x, scratch, out.totals);
}

// ---------------------------------------------------------------- preference

struct Sequence {
  int64_t first, last;  // inside the rows, whatever the offsets hold
};

__device__ __forceinline__ Sequence sequence(const PreferenceArgs& a, int64_t s) {
  const int64_t first = min(max(a.offsets[s], (int64_t)0), a.rows);
  return {first, min(max(a.offsets[s + 1], first), a.rows)};
}

// The sums of logp - ref of the given tokens of N runs, and their counts: v[2 n],
// v[2 n + 1].  The loads of all runs' first passes are in flight together.
template <int N>
__device__ __forceinline__ void sum_tokens(const PreferenceArgs& a, const Sequence (&run)[N],
                                           double (&v)[2 * N]) {
  constexpr int U = 4;
  int64_t longest = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) longest = max(longest, run[n].last - run[n].first);
  for (int64_t i = threadIdx.x; i < longest; i += U * kThreads) {
    int64_t y[N][U];
    float lp[N][U], ref[N][U];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = run[n].first + i + u * kThreads;
        const bool there = at < run[n].last;
        y[n][u] = there ? a.targets[at] : -1;
        lp[n][u] = there ? a.logp[at] : 0.f;
        ref[n][u] = there && a.ref_logp ? a.ref_logp[at] : 0.f;
      }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (y[n][u] >= 0) {
          v[2 * n] += (double)lp[n][u] - (double)ref[n][u];
          v[2 * n + 1] += 1.0;
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
    // -log sigmoid(-|z|) is |z| more than that of |z|.  Without smoothing the loss at z =
    // infinity (a rejected answer with a masked token) is 0, and not 0 times infinity.
    const double far = z >= 0.0 ? e : 1.0 - e;
    t.loss = far != 0.0 ? soft + far * fabs(z) : soft;
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

// A workgroup takes whole pairs: both sums, then both gradients (16 bytes of a token read,
// 4 written).  Bound by latency: the offsets, the tokens of both sequences at once, the
// sums over the workgroup, and the targets once more take 5 us, 16 pairs of up to 700
// tokens 7.7.
__global__ void __launch_bounds__(kThreads)
preference_kernel(PreferenceArgs a, PreferenceOutputs out, ObjectiveScratch* scratch) {
  double totals[kPreferenceTotals] = {};
  for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    const Sequence seq[2] = {sequence(a, pair), sequence(a, a.pairs + pair)};
    double v[4] = {};
    sum_tokens(a, seq, v);
    group_sums<kThreads, 4>(v);
    const PairTerm t = pair_term(a, pair, {v[0], v[2]}, {v[1], v[3]});
    if (threadIdx.x == 0) write_pair(a, out, pair, t);
    add_pair(t, totals);
    if (out.d_logp) {
      write_tokens(a, out.d_logp, seq[0].first, seq[0].last, (float)t.d[0]);
      write_tokens(a, out.d_logp, seq[1].first, seq[1].last, (float)t.d[1]);
    }
  }
  if (out.d_logp) clear_outside(a, out.d_logp);
  add_groups<kThreads, kPreferenceTotals>(totals, blockIdx.x, gridDim.x, scratch, out.totals);
}

// Few pairs of long sequences: `parts` workgroups for each sequence, one launch
// for the sums and one for the gradients, as a gradient needs both sequences' sums: 4 us
// each at least, 504,741 tokens 4.5 and 6.2 (600,000 by one workgroup 1390).
__device__ __forceinline__ Sequence part_of(const Sequence& s, int32_t part, int32_t parts) {
  const int64_t run = ((s.last - s.first + parts - 1) / parts + kThreads - 1) / kThreads * kThreads;
  const int64_t first = min(s.first + part * run, s.last);
  return {first, min(first + run, s.last)};
}

__global__ void __launch_bounds__(kThreads)
sequence_sum_kernel(PreferenceArgs a, int32_t parts, ObjectiveScratch* scratch) {
  const Sequence run[1] = {part_of(sequence(a, blockIdx.x / parts), blockIdx.x % parts, parts)};
  double v[2] = {};
  sum_tokens(a, run, v);
  group_sums<kThreads, 2>(v);
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
  group_sums<kThreads, 4>(v);
  const PairTerm t = pair_term(a, pair, {v[0], v[2]}, {v[1], v[3]});
  if (out.d_logp) {
    const Sequence s = part_of(sequence(a, number), part, parts);
    write_tokens(a, out.d_logp, s.first, s.last, (float)(number < a.pairs ? t.d[0] : t.d[1]));
    clear_outside(a, out.d_logp);
  }
  if (part != 0 || number >= a.pairs) return;
  if (threadIdx.x == 0) write_pair(a, out, pair, t);
  double totals[kPreferenceTotals] = {};
  add_pair(t, totals);
  add_groups<kThreads, kPreferenceTotals>(totals, (uint32_t)pair, (uint32_t)a.pairs, scratch,
                                          out.totals);
}

}  // namespace

hipError_t launch_policy_terms(const PolicyArgs& p, const PolicyRows& r, const PolicyOutputs& out,
                               ObjectiveScratch* scratch, hipStream_t stream) {
  const int64_t groups = std::max<int64_t>(
      1, std::min<int64_t>(kTotalsGroups, (r.rows + 4 * kThreads - 1) / (4 * kThreads)));
  hipLaunchKernelGGL(policy_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, p, r, out,
                     scratch);
  return hipGetLastError();
}

hipError_t launch_preference(const PreferenceArgs& a, const PreferenceOutputs& out,
                             ObjectiveScratch* scratch, hipStream_t stream) {
  // Sequences of more than 1280 tokens on average are taken in parts of 256 or more, by two
  // launches.  us in one launch and in two, pairs x tokens of a sequence: 1 x 600 5.5 / 7.1,
  // 16 x 700 7.7 / 9.1, 1 x 1500 7.8 / 7.4, 64 x 3000 13.8 / 11.7, 1 x 6000 18.5 / 7.6, 16 x
  // 6000 21.2 / 10.8, 200 x 6000 35.8 / 22.2; two launches with parts of 1024 or more, 1 x
  // 6000 8.7, of 2048 11.2.  Every workgroup of the second one reads the sums of all its
  // pair's parts: 1 x 100,000 in 128 parts 8.5, in 390 10.3; 1 x 300,000 in 128 11.1, 256
  // 10.3, 512 11.9; 1 x 1,000,000 33, 21 and 17.7.  A batch whose average is short is taken
  // in pairs, however long one is: 300,000 tokens among 300 pairs of 100 511 us.
  constexpr int64_t kLong = 1280, kPartTokens = 256, kParts = 128, kManyTokens = 1024;
  const int64_t average = a.pairs > 0 ? a.rows / (2 * a.pairs) : 0;
  const int64_t parts = average > kLong
                            ? std::min({kTotalsGroups / (2 * a.pairs), average / kPartTokens,
                                        std::max(kParts, average / kManyTokens)})
                            : 1;
  if (parts > 1) {
    const auto grid = dim3((unsigned)(2 * a.pairs * parts));
    hipLaunchKernelGGL(sequence_sum_kernel, grid, dim3(kThreads), 0, stream, a, (int32_t)parts,
                       scratch);
    hipLaunchKernelGGL(pair_grad_kernel, grid, dim3(kThreads), 0, stream, a, (int32_t)parts, out,
                       scratch);
    return hipGetLastError();
  }
  // (Without pairs there are rows to clear, 8 a thread.)
  const int64_t groups = std::max<int64_t>(
      1, std::min<int64_t>(kTotalsGroups, a.pairs > 0 ? a.pairs : a.rows / (8 * kThreads)));
  hipLaunchKernelGGL(preference_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a, out,
                     scratch);
  return hipGetLastError();
}

}  // namespace arc
