// Token log probabilities: for each row of logits the normaliser, the log
// probability of the given token, the entropy and the top alternatives, and
// their gradient (the formulas are in libarctopk.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "arc_device.h"
#include "arc_objective.h"
#include "arc_policy.h"
#include "arc_train.h"

namespace arc {
namespace {

constexpr int kMaxTop = 32;                  // ARC_MAX_TOP
constexpr int64_t kRowsPerLaunch = 1 << 20;  // threads of a launch stay below 2^32

// Few rows are split into pieces of 2048 chunks, a batch of loads for each of
// 512 threads: at most 16 of them, whose alternatives fit the joining
// workgroup's list, and as many as fill the card.  One row of 32,000 bf16 without
// / with 5 alternatives 4.7 / 8.0 us (pieces of 1024: 4.4 / 7.9), 24 of 50,257
// binary32 with 20 12.1 (15.2), 100 of 50,257 bf16 with 5 11.9 (12.6).
constexpr int kSplitThreads = 512;
constexpr int64_t kPieceChunks = 4 * kSplitThreads, kMostPieces = 16, kSplitParts = 1024;

// Chunks of a row up to which workgroups of 64, 256 and 512 threads take it
// (above: 1024).  The same with and without alternatives, so that a row's sums
// have the same bits.  us at 64 / 256 / 512 / 1024 threads, 5e8 bytes of rows of
// bf16, without and with 20 alternatives: 600 chunks 86 / 108 / 176 / 287 and 129 /
// 199 / 423 / 796, 1200 83 / 85 / 107 / 183 and 131 / 135 / 225 / 458, 2400 82 / 80 /
// 86 / 115 and 128 / 101 / 143 / 251, 3300 87 / 82 / 79 / 99 and 133 / 100 / 122 /
// 196, 6000 94 / 82 / 79 / 86 and 144 / 99 / 96 / 142, 10,000 89 / 84 / 82 / 82 and
// 140 / 103 / 96 / 115, 16,000 86 / 82 / 81 / 79 and 141 / 100 / 95 / 97, 25,000 122 /
// 85 / 81 / 79 and 180 / 101 / 97 / 94.  From 3300 to 5500 the larger workgroup gains
// 1 to 4% without alternatives and loses with 20 of them, 20% falling to 4% (with 5,
// 8192 rows of 4000 chunks 100 / 99).  Between 512 and 1024 the two kinds together are even near 16,000: 12,600
// bf16 81 / 79 and 97 / 103, binary32 78 / 76 and 93 / 92; 17,500 83 / 81 and 96 / 100,
// 80 / 77 and 91 / 92; 19,000 83 / 83 and 100 / 100, 80 / 78 and 96 / 93.
constexpr int64_t kRow64 = 1200, kRow256 = 3300, kRow512 = 16000;

// ---------------------------------------------------------------------------
// A row is read in chunks of 16 bytes a lane, from its first whole word on (a
// row of bfloat16 may begin between words: its 16-byte loads would then reach
// 5.5 TB/s instead of 6.5), and single elements at its ends.
// ---------------------------------------------------------------------------
template <bool BF16>
constexpr int kChunk = BF16 ? 8 : 4;

struct __attribute__((packed, aligned(4))) Words16 {
  uint32_t w[4];
};

typedef uint32_t loose_u32x4_t __attribute__((ext_vector_type(4), aligned(2)));

// Of what is read once.
__device__ __forceinline__ Words16 stream_load16(const Words16* p) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const loose_u32x4_t*>(p));
  return Words16{{v.x, v.y, v.z, v.w}};
}

template <bool BF16>
__device__ __forceinline__ void unpack(const Words16& r, float (&x)[kChunk<BF16>]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (BF16) {
      x[2 * k] = bf16_lo(r.w[k]);
      x[2 * k + 1] = bf16_hi(r.w[k]);
    } else {
      x[k] = __uint_as_float(r.w[k]);
    }
  }
}

// Words that the compiler has to keep as they are: it would hold on to what it
// unpacked from them otherwise, twice the registers.
__device__ __forceinline__ void keep_packed(Words16& r) {
  asm volatile("" : "+v"(r.w[0]), "+v"(r.w[1]), "+v"(r.w[2]), "+v"(r.w[3]));
}

template <bool BF16>
__device__ __forceinline__ float element(const void* row, int64_t j) {
  if constexpr (BF16)
    return __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[j] << 16);
  return static_cast<const float*>(row)[j];
}

template <bool BF16>
__device__ __forceinline__ const void* row_at(const void* base, int64_t element) {
  return static_cast<const char*>(base) + element * (BF16 ? 2 : 4);
}

// Where a row's chunks lie: `head` single elements (0 or 1), `chunks` chunks,
// `tail` single elements.
template <bool BF16>
struct RowShape {
  int32_t head, chunks, tail;
  __device__ RowShape(const void* row, int32_t V) {
    head = BF16 ? (int32_t)((reinterpret_cast<uintptr_t>(row) >> 1) & 1) : 0;
    chunks = (V - head) / kChunk<BF16>;
    tail = (V - head) % kChunk<BF16>;
  }
  // Single element e of head + tail.
  __device__ int32_t edge(int32_t e, int32_t V) const {
    return e < head ? e : V - tail + (e - head);
  }
  __device__ const Words16* body(const void* row) const {
    return reinterpret_cast<const Words16*>(row_at<BF16>(row, head));
  }
};

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Softmax statistics of part of a row relative to a logit `most`, in powers of
// two: total = sum 2^t, spread = sum 2^t t for t = c x - R, c = scale log2(e).
// `most` is the part's largest logit, or less by no more than 16 in t: a sum of
// binary32 numbers does not care, and needs no scaling of what it holds
// whenever a larger logit comes.  R is c most rounded, and t one fma: R need not
// be the exact product, as what it lacks (`rest`, exactly known) is the same for
// all of the part, and is made up for where parts are joined.
//
// Far from zero (|R| >= 2^30) neighbouring logits are 2^6 apart in t and more,
// so that only those equal to the largest count: it is `most`, they are taken as
// 0 and all others as -infinity, with R = 0 (far_logit()).
struct Stats {
  float most, total, spread;
};

struct Reference {
  float R, rest;
  bool far;
};

__device__ __forceinline__ Reference reference(float most, float c) {
  const float p = most == -INFINITY ? 0.f : most * c;  // nothing above -infinity: from 0
  if (!(fabsf(p) < 0x1p30f)) return {0.f, 0.f, true};
  return {p, most == -INFINITY ? 0.f : fmaf(most, c, -p), false};
}

// NaN stays NaN, and an infinite `most` becomes one.
__device__ __forceinline__ float far_logit(float x, float most) {
  return x < most ? -INFINITY : x - most;
}

__device__ __forceinline__ float exponent(float x, float most, const Reference& r, float c) {
  return r.far ? (x - most) * c : fmaf(x, c, -r.R);
}

// t below this adds nothing to a spread, and 0 * infinity would.
constexpr float kFarBelow = -300.f;

constexpr float kMostAbove = 16.f;  // of a t

// s relative to `most` (not below s.most) instead.
__device__ __forceinline__ Stats moved(const Stats& s, float most, const Reference& to, float c) {
  if (s.most == -INFINITY) return {most, s.total, 0.f};  // total: 0, or a NaN to keep
  const float t = (s.most - most) * c - reference(s.most, c).rest + to.rest;
  const float e = __builtin_amdgcn_exp2f(t);
  return {most, e * s.total, e * (s.spread + fmaxf(t, kFarBelow) * s.total)};
}

struct MaxF {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct SumF {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct MaxKey {
  __device__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; }
};

// What a workgroup found out about its piece of a row, for the workgroup that
// joins the pieces.
struct TokenPart {
  float most, total, spread, pad;
  uint64_t top[kMaxTop];  // keys in falling order, 0 where the piece has no more
};

// Parts are written through to where every compute unit sees them and read
// from there.  A fence for the whole device writes back all that its XCD's
// cache holds instead, of every workgroup: 1024 of them took 250 us.
template <typename T>
__device__ __forceinline__ void share_store(T* p, T v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T share_load(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Alternatives.  Every thread keeps the largest logit of each run of its chunks
// (at most kRuns runs).  The threads form 64 groups, and the k-th largest of
// the groups' largest logits is a bound `tau` that at least k elements reach.
// Only runs whose largest one reaches it are read once more (from the cache),
// by the whole workgroup; in a row of noise they are about 64 log(64 / (64 -
// k)).  What reaches tau there, some dozens, is ordered by counting.
template <int W>
constexpr int kRuns = W == 64 ? 4 : 8;
template <int W>
constexpr int kListed = W == 64 ? 256 : 512;
template <int W>
constexpr int kCandidates = W == 64 ? 256 : 512;
template <int W>
struct TopShared {
  float group[64];
  float run_most[kRuns<W>][W];
  int32_t listed, found;
  int32_t list[kListed<W>];
  uint64_t best[16];
  uint64_t found_keys[kCandidates<W>];  // 0 behind the last
};

// The order of logits as unsigned words, and back.
__device__ __forceinline__ uint32_t order_word(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float word_logit(uint32_t w) {
  return __uint_as_float(w ^ ((w >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// A larger key is a larger logit, or the same logit of a lower token.
__device__ __forceinline__ uint64_t rank_key(float x, int32_t j) {
  return ((uint64_t)order_word(x) << 32) | (0xFFFFFFFFu - (uint32_t)j);
}
__device__ __forceinline__ int32_t key_token(uint64_t key) {
  return (int32_t)(0xFFFFFFFFu - (uint32_t)key);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  return word_logit((uint32_t)(key >> 32));
}

// A bound that at least k of the wave's 64 values reach (or all that are above
// -infinity), and k + 3 at most where that can be: bits of the k-th largest from
// the top, counting.
__device__ __forceinline__ float kth_bound(float v, int32_t k) {
  const uint32_t key = order_word(v);
  uint32_t bound = 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    const int32_t n = __popcll(__ballot(key >= (bound | bit)));
    if (n >= k) bound |= bit;
    if (n >= k && n <= k + 3) break;
  }
  // not -infinity, which is masked, but what is next to it
  return fmaxf(word_logit(bound < 0x00800000u ? 0x00800000u : bound), -FLT_MAX);
}

template <bool BF16, int W>
struct Scorer {
  static constexpr int C = kChunk<BF16>;
  static constexpr int U = 4;  // chunks of a thread in flight
  static constexpr int kWaves = W / kWave;
  static constexpr int kLanes = W / 64;  // of a group

  // Statistics of a thread's share of chunks [first, end); with TOP, the largest
  // logit of each run of `run_batches` batches of U chunks, and their number
  // (chunks may then be read again, and should stay in the cache).
  template <bool TOP>
  static __device__ __forceinline__ Stats share(const Words16* body, int32_t first, int32_t end,
                                                float c, int32_t run_batches,
                                                float (*run_most)[W], int32_t* runs,
                                                float* largest) {
    Stats s{-INFINITY, 0.f, 0.f};
    Reference ref{0.f, 0.f, false};
    float limit = -INFINITY;  // logits up to which `most` serves
    const float above = kMostAbove / c;
    float run = -INFINITY, top = -INFINITY;
    int32_t batch = 0, done = 0;
    // ALL: every thread has all U chunks.  The others, at the end, would cost
    // as much arithmetic as chunks that are there, if they were not left out.
    const auto take = [&](int32_t k, auto all) {
      constexpr bool ALL = decltype(all)::value;
      Words16 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t low = BF16 ? 0xFF80FF80u : 0xFF800000u;  // -infinity
        if (!ALL) raw[u] = Words16{{low, low, low, low}};
        if (ALL || k + u * W < end)
          raw[u] = TOP ? body[k + u * W] : stream_load16(body + k + u * W);
      }
      float x[U][C];
      float here = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        unpack<BF16>(raw[u], x[u]);
#pragma unroll
        for (int q = 0; q < C; ++q) here = fmaxf(here, x[u][q]);
      }
      if constexpr (TOP) {
        run = fmaxf(run, here);
        top = fmaxf(top, here);
        if (++batch == run_batches) {
          run_most[done++][threadIdx.x] = run;
          run = -INFINITY;
          batch = 0;
        }
      }
      if (here > limit) {
        ref = reference(here, c);
        s = moved(s, here, ref, c);
        limit = ref.far ? here : here + above;
      }
      if (ref.far) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int q = 0; q < C; ++q) x[u][q] = far_logit(x[u][q], s.most);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!ALL && k + u * W >= end) break;
#pragma unroll
        for (int q = 0; q < C; ++q) {
          const float t = fmaf(x[u][q], c, -ref.R);
          const float e = __builtin_amdgcn_exp2f(t);
          s.total += e;
          s.spread = fmaf(e, fmaxf(t, kFarBelow), s.spread);
        }
      }
    };
    int32_t k = first + threadIdx.x;
    const int32_t whole = (end - first) / (W * U);
    for (int32_t q = 0; q < whole; ++q, k += W * U) take(k, std::true_type());
    if (k < end) take(k, std::false_type());
    if constexpr (TOP) {
      if (batch > 0) run_most[done++][threadIdx.x] = run;
      *runs = done;
      *largest = top;
    }
    return s;
  }

  static __device__ __forceinline__ void add_edge(float x, float c, Stats* s) {
    const float most = fmaxf(s->most, x);
    const Reference ref = reference(most, c);
    *s = moved(*s, most, ref, c);
    const float t = exponent(x, most, ref, c), e = __builtin_amdgcn_exp2f(t);
    s->total += e;
    s->spread = fmaf(e, fmaxf(t, kFarBelow), s->spread);
  }

  // Over the workgroup, on every thread.
  static __device__ __forceinline__ float all_max(float v, float* part) {
    v = lanes_reduce<64>(v, MaxF());
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = fmaxf(v, part[w]);
    return v;
  }

  // The keys found are ordered by counting, and the first k written.
  template <typename Write>
  static __device__ __forceinline__ void order(const TopShared<W>& sh, int32_t n, int32_t k,
                                               const Write& write) {
    for (int32_t i = threadIdx.x; i < n; i += W) {
      const uint64_t key = sh.found_keys[i];
      int32_t rank = 0;
      for (int32_t q = 0; q < n; q += 8) {  // eight reads at a time; behind the n keys are 0s
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += sh.found_keys[q + u] > key;
      }
      if (rank < k) write(rank, key);
    }
  }
};

// A row's results from its statistics.
struct RowResult {
  float most, scale, c, log_total;
  Reference ref;
  bool empty, none;
  __device__ float logp(float x) const {
    const float t = exponent(x, most, ref, c);
    // the lowest values' t can be beyond the type where their z is not
    const float z = t > -0x1p31f ? t * kLn2 : (x - most) * scale;
    return none ? NAN : empty ? -INFINITY : z - log_total;
  }
};

__device__ __forceinline__ RowResult finish_row(const TokenArgs& a, const TokenScores& out,
                                                int64_t i, const Stats& s, int64_t y, float xy) {
  RowResult r;
  r.most = s.most;
  r.scale = a.scale;
  r.c = a.scale * kLog2e;
  r.ref = reference(s.most, r.c);
  r.empty = s.total == 0.f;
  r.log_total = logf(s.total);
  const float lse = r.empty ? -INFINITY : s.most * a.scale + (r.log_total - r.ref.rest * kLn2);
  r.none = lse != lse;
  if (threadIdx.x == 0) {
    if (out.lse) out.lse[i] = lse;
    if (out.entropy) out.entropy[i] = r.empty ? 0.f : r.log_total - s.spread * kLn2 / s.total;
    if (out.sums) {
      out.sums[2 * i] = s.most;
      out.sums[2 * i + 1] = s.total;
    }
    if (out.logp) out.logp[i] = y < 0 ? 0.f : y >= a.vocab ? NAN : r.logp(xy);
  }
  return r;
}

template <bool BF16, int W, bool TOP>
__global__ void __launch_bounds__(W, 8)
token_score_kernel(TokenArgs a, TokenScores out, int32_t pieces, int32_t piece_chunks,
                   TokenPart* __restrict__ parts, uint32_t* __restrict__ arrived) {
  using S = Scorer<BF16, W>;
  __shared__ float part_most[S::kWaves];
  __shared__ float part_sum[2][S::kWaves];
  __shared__ float given;
  __shared__ int32_t last;
  __shared__ TopShared<W> sh;
  const int64_t i = pieces == 1 ? blockIdx.x : blockIdx.x / pieces;
  const int32_t piece = pieces == 1 ? 0 : blockIdx.x % pieces;
  const int32_t V = (int32_t)a.vocab, k = TOP ? a.top : 0;
  const float c = a.scale * kLog2e;
  const void* row = row_at<BF16>(a.logits, i * a.stride);
  const RowShape<BF16> shape(row, V);
  const Words16* body = shape.body(row);
  const int32_t first = piece * piece_chunks;
  const int32_t end = min(shape.chunks, first + piece_chunks);
  const bool edges = piece == pieces - 1;  // single elements are the last piece's
  const int64_t y = out.logp ? a.targets[i] : -1;
  if (threadIdx.x == W - 1) given = y >= 0 && y < V ? element<BF16>(row, y) : 0.f;

  // Batches of a run, so that a thread has kRuns at most.
  constexpr int32_t kMost = kRuns<W> * W * S::U;
  const int32_t run_batches = max(1, (end - first + kMost - 1) / kMost);
  int32_t runs = 0;
  float largest = -INFINITY;  // of the thread's logits
  Stats s = S::template share<TOP>(body, first, end, c, run_batches, sh.run_most, &runs, &largest);
  if (edges && (int)threadIdx.x < shape.head + shape.tail) {
    const float x = element<BF16>(row, shape.edge(threadIdx.x, V));
    S::add_edge(x, c, &s);
    largest = fmaxf(largest, x);
  }
  if constexpr (TOP) {
    const float g = lanes_reduce<S::kLanes>(largest, MaxF());
    if (threadIdx.x % S::kLanes == 0) sh.group[threadIdx.x / S::kLanes] = g;
    if (threadIdx.x == 0) sh.listed = sh.found = 0;
#pragma unroll
    for (int q = 0; q < kCandidates<W>; q += W)
      if (q + (int)threadIdx.x < kCandidates<W>) sh.found_keys[q + threadIdx.x] = 0;
  }
  const float most = S::all_max(s.most, part_most);
  s = moved(s, most, reference(most, c), c);
  s.total = lanes_reduce<64>(s.total, SumF());
  s.spread = lanes_reduce<64>(s.spread, SumF());
  if (threadIdx.x % kWave == 0) {
    part_sum[0][threadIdx.x / kWave] = s.total;
    part_sum[1][threadIdx.x / kWave] = s.spread;
  }
  float tau = 0.f;
  if constexpr (TOP) {
    tau = kth_bound(sh.group[threadIdx.x % kWave], k);
    for (int32_t r = 0; r < runs; ++r)
      if (sh.run_most[r][threadIdx.x] >= tau) {
        const int32_t n = atomicAdd(&sh.listed, 1);
        if (n < kListed<W>) sh.list[n] = r * W + threadIdx.x;
      }
  }
  __syncthreads();
  s = {most, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < S::kWaves; ++w) {
    s.total += part_sum[0][w];
    s.spread += part_sum[1][w];
  }
  if constexpr (TOP) {
    const int32_t of_run = run_batches * S::U;  // chunks of a run, at most
    const int32_t items = sh.listed <= kListed<W> ? sh.listed * of_run : 0;
    const auto found = [&](float x, int32_t j) {
      if (x >= tau) {
        const int32_t n = atomicAdd(&sh.found, 1);
        if (n < kCandidates<W>) sh.found_keys[n] = rank_key(x, j);
      }
    };
    for (int32_t q = threadIdx.x; q < items; q += W) {
      const int32_t of = sh.list[q / of_run], r = of / W;
      const int32_t chunk = first + of % W + (r * of_run + q % of_run) * W;
      if (chunk >= end) continue;
      float x[S::C];
      unpack<BF16>(body[chunk], x);
#pragma unroll
      for (int e = 0; e < S::C; ++e) found(x[e], shape.head + chunk * S::C + e);
    }
    if (edges && (int)threadIdx.x < shape.head + shape.tail) {
      const int32_t j = shape.edge(threadIdx.x, V);
      found(element<BF16>(row, j), j);
    }
    __syncthreads();
  }
  int32_t n = TOP ? sh.found : 0;
  bool one_by_one = false;
  if constexpr (TOP) {
    // Tokens of the piece but for the single elements, in order; one at a time,
    // so that this rare way leaves the common one its registers.  No step goes past
    // the last token: the longest row's is 2^31 - 2.
    const int32_t begin = shape.head + first * S::C, stop = shape.head + end * S::C;
    const auto each = [&](int32_t from, int32_t to, const auto& look) {
      if ((int32_t)threadIdx.x >= to - from) return;
#pragma unroll 1
      for (int32_t j = from + threadIdx.x;; j += W) {
        look(element<BF16>(row, j), j);
        if (to - j <= W) break;
      }
    };
    const auto each_edge = [&](const auto& look) {
      if (edges && (int)threadIdx.x < shape.head + shape.tail) {
        const int32_t j = shape.edge(threadIdx.x, V);
        look(element<BF16>(row, j), j);
      }
    };
    const auto add = [&](float x, int32_t j) {
      const int32_t at = atomicAdd(&sh.found, 1);
      if (at < kCandidates<W>) sh.found_keys[at] = rank_key(x, j);
    };
    if (n > kCandidates<W> || sh.listed > kListed<W>) {
      // Too many for the lists: as a rule equal ones (a mask of the type's lowest
      // value, logits of a head of zeros).  What is above tau, then as many of
      // those at tau as are wanted, from the first token on.
      __syncthreads();
      for (int q = threadIdx.x; q < kCandidates<W>; q += W) sh.found_keys[q] = 0;
      if (threadIdx.x == 0) sh.found = 0;
      __syncthreads();
      const auto above = [&](float x, int32_t j) {
        if (x > tau) add(x, j);
      };
      each(begin, stop, above);
      each_edge(above);
      __syncthreads();
      n = sh.found;
      __syncthreads();  // the same n on every wave, before more is found
      // few threads' chunks hold the largest: the keys one after the other
      one_by_one = n > kCandidates<W> / 2;
      if (n < k) {
        const auto at_tau = [&](float x, int32_t j) {
          if (x == tau) add(x, j);
        };
        constexpr int32_t kSome = kCandidates<W> / 2 - 8;  // half the list, with the single ones
        each_edge(at_tau);
        for (int32_t from = begin, to; from < stop; from = to) {
          to = from + min(kSome, stop - from);
          each(from, to, at_tau);
          __syncthreads();
          n = sh.found;
          __syncthreads();
          if (n >= k + 8) break;  // the single ones may be behind those still to come
        }
        __syncthreads();
        n = sh.found;
      }
    } else if (n < k) {
      // Fewer than k that are not masked (tau is above -infinity): among the
      // piece's first k tokens are as many masked ones as are wanted.
      __syncthreads();
      const auto masked = [&](float x, int32_t j) {
        if (x == -INFINITY) add(x, j);
      };
      each(begin, min(stop, begin + k), masked);
      each_edge(masked);
      __syncthreads();
      n = sh.found;
    }
    if (one_by_one) {  // each key the largest below the one before
      uint64_t before = ~0ull;
      for (int32_t r = 0; r < k; ++r) {
        uint64_t key = 0;
        const auto look = [&](float x, int32_t j) {
          const uint64_t q = rank_key(x, j);
          if (q < before && q > key) key = q;
        };
        each(begin, stop, look);
        each_edge(look);
        key = lanes_reduce<64>(key, MaxKey());
        __syncthreads();
        if (threadIdx.x % kWave == 0) sh.best[threadIdx.x / kWave] = key;
        __syncthreads();
        key = sh.best[0];
        for (int w = 1; w < S::kWaves; ++w) key = MaxKey()(key, sh.best[w]);
        if (threadIdx.x == 0) sh.found_keys[r] = key;
        before = key;
      }
      n = k;
      __syncthreads();
      if ((int)threadIdx.x >= k && threadIdx.x < 40) sh.found_keys[threadIdx.x] = 0;
      __syncthreads();
    }
  }

  if (pieces == 1) {
    const RowResult r = finish_row(a, out, i, s, y, given);
    if (!k) return;
    const auto write = [&](int32_t rank, uint64_t key) {
      out.top_ids[i * k + rank] = r.none ? -1 : key_token(key);
      out.top_logp[i * k + rank] = r.logp(key_logit(key));
    };
    if (r.none) {
      if ((int)threadIdx.x < k) write(threadIdx.x, 0);
    } else {
      S::order(sh, n, k, write);
    }
    return;
  }

  TokenPart* part = parts + blockIdx.x;
  if (threadIdx.x == 0) {
    share_store(&part->most, s.most);
    share_store(&part->total, s.total);
    share_store(&part->spread, s.spread);
  }
  if (k) {
    const auto write = [&](int32_t rank, uint64_t key) { share_store(&part->top[rank], key); };
    if ((int)threadIdx.x >= n && (int)threadIdx.x < k) write(threadIdx.x, 0);
    S::order(sh, n, k, write);
  }
  // The last workgroup of a row to arrive joins the pieces: every wave's part
  // has been written before the barrier, and the count goes up behind it.
  wave_vmem_fence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const auto most_before = (uint32_t)(pieces - 1);
    last = atomicInc(&arrived[i], most_before) == most_before;  // and 0 for the next call
  }
  __syncthreads();
  if (!last) return;
  const TokenPart* of = parts + i * pieces;
  // A lane of each wave takes a piece (there are fewer), in the same order.
  const int32_t lane = threadIdx.x % kWave;
  s = {-INFINITY, 0.f, 0.f};
  if (lane < pieces)
    s = {share_load(&of[lane].most), share_load(&of[lane].total), share_load(&of[lane].spread)};
  const float pm = lanes_reduce<64>(s.most, MaxF());
  s = moved(s, pm, reference(pm, c), c);
  s = {pm, lanes_reduce<64>(s.total, SumF()), lanes_reduce<64>(s.spread, SumF())};
  const RowResult r = finish_row(a, out, i, s, y, given);
  if (!k) return;
  // Each piece's k-th key is a bound for the row's.
  uint64_t least = lane < pieces ? share_load(&of[lane].top[k - 1]) : 0;
  least = lanes_reduce<64>(least, MaxKey());
  if (threadIdx.x == 0) sh.found = 0;
  for (int q = threadIdx.x; q < kCandidates<W>; q += W) sh.found_keys[q] = 0;
  __syncthreads();
  static_assert(kMostPieces * kMaxTop <= kCandidates<kSplitThreads>, "room for all");
  for (int32_t q = threadIdx.x; q < pieces * k; q += W) {
    const uint64_t key = share_load(&of[q / k].top[q % k]);
    if (key != 0 && key >= least) sh.found_keys[atomicAdd(&sh.found, 1)] = key;
  }
  __syncthreads();
  const auto write = [&](int32_t rank, uint64_t key) {
    out.top_ids[i * k + rank] = r.none ? -1 : key_token(key);
    out.top_logp[i * k + rank] = r.logp(key_logit(key));
  };
  if (r.none) {
    if ((int)threadIdx.x < k) write(threadIdx.x, 0);
  } else {
    S::order(sh, sh.found, k, write);
  }
}

// ---------------------------------------------------------------------------
// Gradients.  With lp = log p of an element, dx = p (A + B lp) for the row's
// A = scale (dz - dl - dh H) and B = -scale dh, and scale dl more at the token.
// ---------------------------------------------------------------------------
struct GradRow {
  float A, B, given;
  int32_t y;  // -1: none
  bool zero;
};

__device__ __forceinline__ GradRow grad_row(const TokenArgs& a, int64_t y, float dl, float dh,
                                            float dz, float H, bool empty) {
  GradRow r;
  r.A = a.scale * (dz - dl - (dh != 0.f ? dh * H : 0.f));
  r.B = -a.scale * dh;
  r.given = a.scale * dl;
  r.zero = (dl == 0.f && dh == 0.f && dz == 0.f) || empty;
  r.y = y < a.vocab && !r.zero ? (int32_t)y : -1;
  return r;
}

__device__ __forceinline__ GradRow grad_row(const TokenArgs& a, const TokenGrad& g, int64_t i,
                                            float H, bool empty) {
  const int64_t y = g.d_logp ? a.targets[i] : -1;
  return grad_row(a, y, y >= 0 ? g.d_logp[i] : 0.f, g.d_entropy ? g.d_entropy[i] : 0.f,
                  g.d_lse ? g.d_lse[i] : 0.f, H, empty);
}

// Natural logarithms of p below this have p = 0, and 0 * infinity is none.
constexpr float kNoWeight = -150.f;

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t w;
  asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(lo), "v"(hi));
  return w;
}

// 16 bytes at any element alignment (the rows of a gradient need not lie as
// those of the logits do), read again by later launches at the earliest.
__device__ __forceinline__ void stream_store16(void* p, const uint32_t (&w)[4]) {
  const u32x4_t v = {w[0], w[1], w[2], w[3]};
  __builtin_nontemporal_store(v, reinterpret_cast<loose_u32x4_t*>(p));
}

template <bool BF16>
__device__ __forceinline__ Words16 pack(const float (&d)[kChunk<BF16>]) {
  Words16 w;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    w.w[k] = BF16 ? bf16_pair(d[BF16 ? 2 * k : 0], d[BF16 ? 2 * k + 1 : 0])
                  : __float_as_uint(d[k]);
  return w;
}

template <bool BF16>
__device__ __forceinline__ void store_chunk(void* row, int32_t j, const float (&d)[kChunk<BF16>]) {
  stream_store16(static_cast<char*>(row) + (int64_t)j * (BF16 ? 2 : 4), pack<BF16>(d).w);
}

template <bool BF16>
__device__ __forceinline__ void store_element(void* row, int32_t j, float d) {
  if constexpr (BF16)
    static_cast<uint16_t*>(row)[j] = (uint16_t)bf16_pair(d, d);
  else
    static_cast<float*>(row)[j] = d;
}

constexpr int kGradThreads = 128;
constexpr int kGradChunks = 2;  // of a thread, in flight

// dx = s (dl ([j = y] - p) + dz p - dh p (log p + H)) with p = exp(s x - lse): one
// exponential and a product with A + B log p an element, A and B the row's.  One
// workgroup for each run of kGradThreads * kGradChunks chunks of a row, so that
// few rows fill the card too.  Bound by HBM: 2048 rows of 32,000 binary32 80 us
// (6.6 TB/s; 14 instructions an element).  us with one, two and four chunks of 256
// threads, and with two of 512 and of 128: those 81 / 82 / 87, 88 / 80; 20,000 rows
// of 1001 bf16 24 / 25 / 25, 36 / 21; 8192 of 50,257 bf16 269 / 270 / 283, 270 /
// 275.  SUMS: from the row's sums, as token_loss_kernel does.
template <bool BF16, bool SUMS>
__global__ void __launch_bounds__(kGradThreads)
token_grad_kernel(TokenArgs a, TokenGrad g, int32_t tiles) {
  constexpr int C = kChunk<BF16>;
  const int64_t i = blockIdx.x / tiles;
  const int32_t tile = blockIdx.x % tiles, V = (int32_t)a.vocab;
  const void* row = row_at<BF16>(a.logits, i * a.stride);
  void* to = const_cast<void*>(row_at<BF16>(g.grad, i * g.stride));
  const RowShape<BF16> shape(row, V);
  const Words16* body = shape.body(row);
  const float most = SUMS ? g.sums[2 * i] : 0.f, total = SUMS ? g.sums[2 * i + 1] : 1.f;
  const float lse = SUMS ? 0.f : g.lse[i];
  const bool empty = SUMS ? total == 0.f : lse == -INFINITY;
  const GradRow r = grad_row(a, g, i, g.d_entropy ? g.entropy[i] : 0.f, empty);
  const float c = a.scale * kLog2e;
  const Reference ref = reference(most, c);
  const float B2 = r.B * kLn2 / total, A2 = r.A / total - B2 * (logf(total) * kLog2e);
  const auto one = [&](float x) {
    if (r.zero) return 0.f;
    if constexpr (SUMS) {
      const float t = fmaf(ref.far ? far_logit(x, most) : x, c, -ref.R);
      return __builtin_amdgcn_exp2f(t) * fmaf(B2, fmaxf(t, kFarBelow), A2);
    }
    const float lp = fmaf(x, a.scale, -lse);
    return __builtin_amdgcn_exp2f(lp * kLog2e) * fmaf(r.B, fmaxf(lp, kNoWeight), r.A);
  };
  Words16 raw[kGradChunks];
  const int32_t k0 = tile * (kGradThreads * kGradChunks) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kGradChunks; ++u) {
    raw[u] = Words16{{0, 0, 0, 0}};
    const int32_t k = k0 + u * kGradThreads;
    if (k < shape.chunks && !r.zero) raw[u] = stream_load16(body + k);
  }
#pragma unroll
  for (int u = 0; u < kGradChunks; ++u) {
    const int32_t k = k0 + u * kGradThreads;
    if (k >= shape.chunks) break;
    const int32_t j = shape.head + k * C;
    float x[C];
    unpack<BF16>(raw[u], x);
#pragma unroll
    for (int q = 0; q < C; ++q) x[q] = one(x[q]);
    if (r.y >= j && r.y < j + C) {
#pragma unroll
      for (int q = 0; q < C; ++q)
        if (r.y == j + q) x[q] += r.given;
    }
    store_chunk<BF16>(to, j, x);
  }
  if (tile == tiles - 1 && (int)threadIdx.x < shape.head + shape.tail) {
    const int32_t j = shape.edge(threadIdx.x, V);
    float d = r.zero ? 0.f : one(element<BF16>(row, j));
    if (j == r.y) d += r.given;
    store_element<BF16>(to, j, d);
  }
}

// Scores and gradient in one pass: a workgroup holds a whole row, N chunks a
// thread, in its registers as it lies in memory, so that HBM moves each logit
// once in and its gradient once out.  dx = 2^t (A' + B' t) from the exponent
// relative to the row's reference, A' and B' divided by the row's sum.  8192 rows of
// 32,000 binary32 361 us (5.8 TB/s): HBM.  4096 of 50,257 bf16 159 us (5.2 TB/s): two
// workgroups a compute unit that read, add and write more or less in step (three
// of its 19 instructions an element left out made no difference).  kPolicy: the
// upstream gradients come from the row's own logp and entropy (policy_term()): 8192 x
// 32,000 358 us, 512 x 50,257 bf16 24 (23 without), and a launch of 4 us behind it for the
// terms and totals.  kPolicyWithTerms makes those as well, for few rows.
enum LossKind { kGivenGradients, kPolicy, kPolicyWithTerms };

template <bool BF16, int W, int N, LossKind KIND>
__global__ void __launch_bounds__(W, N <= 8 ? 8 : 4)
token_loss_kernel(TokenArgs a, TokenScores out, TokenGrad g, PolicyArgs p, PolicyRowTerms rows) {
  using S = Scorer<BF16, W>;
  constexpr int C = S::C;
  __shared__ float part_most[S::kWaves];
  __shared__ float part_sum[2][S::kWaves];
  const int64_t i = blockIdx.x;
  const int32_t V = (int32_t)a.vocab;
  const float c = a.scale * kLog2e;
  const void* row = row_at<BF16>(a.logits, i * a.stride);
  void* to = const_cast<void*>(row_at<BF16>(g.grad, i * g.stride));
  const RowShape<BF16> shape(row, V);
  const Words16* body = shape.body(row);
  constexpr uint32_t low = BF16 ? 0xFF80FF80u : 0xFF800000u;  // -infinity
  Words16 raw[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    raw[n] = Words16{{low, low, low, low}};
    const int32_t k = n * W + threadIdx.x;
    if (k < shape.chunks) raw[n] = stream_load16(body + k);
  }
  const bool edge = (int)threadIdx.x < shape.head + shape.tail;
  const int32_t edge_j = edge ? shape.edge(threadIdx.x, V) : 0;
  const float edge_logit = edge ? element<BF16>(row, edge_j) : -INFINITY;
  const int64_t y = a.targets ? a.targets[i] : -1;
  const float given = y >= 0 && y < V ? element<BF16>(row, y) : 0.f;
  float most = edge_logit;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float x[C];
    unpack<BF16>(raw[n], x);
#pragma unroll
    for (int q = 0; q < C; ++q) most = fmaxf(most, x[q]);
  }
  most = S::all_max(most, part_most);
  const Reference ref = reference(most, c);
  float edge_x = edge_logit;
  if (ref.far) {  // the whole row alike
    edge_x = far_logit(edge_x, most);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      keep_packed(raw[n]);
      float x[C];
      unpack<BF16>(raw[n], x);
#pragma unroll
      for (int q = 0; q < C; ++q) x[q] = far_logit(x[q], most);
      raw[n] = pack<BF16>(x);
    }
  }
  Stats s{most, 0.f, 0.f};
  const auto add = [&](float x) {
    const float t = fmaf(x, c, -ref.R);
    const float e = __builtin_amdgcn_exp2f(t);
    s.total += e;
    s.spread = fmaf(e, fmaxf(t, kFarBelow), s.spread);
  };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * W + (int)threadIdx.x >= shape.chunks) break;
    float x[C];
    if constexpr (BF16) keep_packed(raw[n]);
    unpack<BF16>(raw[n], x);
#pragma unroll
    for (int q = 0; q < C; ++q) add(x[q]);
    __builtin_amdgcn_sched_barrier(0);  // one chunk's values at a time in registers
  }
  add(edge_x);
  s.total = lanes_reduce<64>(s.total, SumF());
  s.spread = lanes_reduce<64>(s.spread, SumF());
  if (threadIdx.x % kWave == 0) {
    part_sum[0][threadIdx.x / kWave] = s.total;
    part_sum[1][threadIdx.x / kWave] = s.spread;
  }
  __syncthreads();
  s.total = s.spread = 0.f;
#pragma unroll
  for (int w = 0; w < S::kWaves; ++w) {
    s.total += part_sum[0][w];
    s.spread += part_sum[1][w];
  }
  const RowResult res = finish_row(a, out, i, s, y, given);
  const float H = res.empty ? 0.f : res.log_total - s.spread * kLn2 / s.total;
  GradRow r;
  bool last = false;
  if constexpr (KIND != kGivenGradients) {
    const float logp = y >= a.vocab ? NAN : res.logp(given);
    const PolicyTerm t = policy_term(p, policy_token(p, i), y >= 0, logp, H);
    r = grad_row(a, y, t.d_logp, t.d_entropy, 0.f, H, res.empty);
    if constexpr (KIND == kPolicyWithTerms)
      if (threadIdx.x < kWave) last = write_row(rows, i, t, H);
  } else {
    r = grad_row(a, g, i, H, res.empty);
  }
  // p (A + B log p) with p = 2^t / total: 2^t (A' + B' t).  (t less the logarithm
  // of the total would be rounded as R is, however large.)
  const float B = r.B * kLn2 / s.total;
  const float A = r.A / s.total - B * (res.log_total * kLog2e);
  // A row's gradient is zero, or p A, or p (A + B log p): 1, 9.5 or 11.5 operations an
  // element beside the unpacking, and the row's whole workgroup does one of them.
  const auto emit = [&](const auto& one) {
    int32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));  // chunk numbers are made anew, not kept in registers
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int32_t k = n * W + thread;
      if (k < shape.chunks) {
        const int32_t j = shape.head + k * C;
        float x[C];
        if constexpr (BF16) keep_packed(raw[n]);
        unpack<BF16>(raw[n], x);
#pragma unroll
        for (int q = 0; q < C; ++q) x[q] = one(x[q]);
        if (r.y >= j && r.y < j + C) {
#pragma unroll
          for (int q = 0; q < C; ++q)
            if (r.y == j + q) x[q] += r.given;
        }
        store_chunk<BF16>(to, j, x);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (edge) store_element<BF16>(to, edge_j, one(edge_x) + (edge_j == r.y ? r.given : 0.f));
  };
  const auto power = [&](float x) { return fmaf(x, c, -ref.R); };
  if (r.zero) {
    emit([](float) { return 0.f; });
  } else if (r.B == 0.f) {
    emit([&](float x) { return __builtin_amdgcn_exp2f(power(x)) * A; });
  } else {
    emit([&](float x) {
      const float t = power(x);
      return __builtin_amdgcn_exp2f(t) * fmaf(B, fmaxf(t, kFarBelow), A);
    });
  }
  if constexpr (KIND == kPolicyWithTerms)
    if (last) add_rows(rows);
}

}  // namespace

// Rows in two pieces or more, at most.
constexpr int64_t kSplitRows = kSplitParts / 2;

// Parts, and for each number of pieces the rows' counts of those that have arrived, which go
// round at that number: 0 between launches, whatever launches overlapped before.
size_t token_workspace_bytes() {
  return (size_t)kSplitParts * sizeof(TokenPart) +
         (size_t)(kMostPieces + 1) * kSplitRows * sizeof(uint32_t);
}

// Pieces of a row of that many chunks, for few rows.
static int32_t row_pieces(int64_t rows, int64_t chunks) {
  const int64_t p = (chunks + kPieceChunks - 1) / kPieceChunks;
  return static_cast<int32_t>(
      std::max<int64_t>(std::min<int64_t>({p, kMostPieces, kSplitParts / rows}), 1));
}

// Calls launch(args, outputs, gradient) for runs of at most kRowsPerLaunch rows.
template <typename Launch>
static void each_rows(const TokenArgs& a, const TokenScores& out, const TokenGrad& g,
                      int64_t most, const Launch& launch) {
  const int64_t bytes = a.bf16 ? 2 : 4;
  for (int64_t lo = 0; lo < a.rows; lo += most) {
    TokenArgs b = a;
    TokenScores o = out;
    TokenGrad h = g;
    b.rows = a.rows - lo < most ? a.rows - lo : most;
    b.logits = static_cast<const char*>(a.logits) + lo * a.stride * bytes;
    if (b.targets) b.targets += lo;
    for (float** p : {&o.logp, &o.entropy, &o.lse})
      if (*p) *p += lo;
    if (o.top_ids) {
      o.top_ids += lo * a.top;
      o.top_logp += lo * a.top;
    }
    if (o.sums) o.sums += 2 * lo;
    if (h.sums) h.sums += 2 * lo;
    for (const float** p : {&h.lse, &h.entropy, &h.d_logp, &h.d_entropy, &h.d_lse})
      if (*p) *p += lo;
    h.grad = static_cast<char*>(g.grad) + lo * g.stride * bytes;
    launch(b, o, h);
  }
}

template <int W>
static void launch_score(const TokenArgs& a, const TokenScores& o, int32_t pieces, int64_t chunks,
                         void* workspace, hipStream_t stream) {
  const auto piece_chunks = static_cast<int32_t>((chunks + pieces - 1) / pieces);
  auto* parts = static_cast<TokenPart*>(workspace);
  auto* arrived = reinterpret_cast<uint32_t*>(parts + kSplitParts) + pieces * kSplitRows;
  const auto kernel =
      o.top_ids && a.top > 0
          ? (a.bf16 ? token_score_kernel<true, W, true> : token_score_kernel<false, W, true>)
          : (a.bf16 ? token_score_kernel<true, W, false> : token_score_kernel<false, W, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.rows * pieces)), dim3(W), 0, stream, a, o, pieces,
                     piece_chunks, parts, arrived);
}

hipError_t launch_token_score(const TokenArgs& a, const TokenScores& out, void* workspace,
                              hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  const int64_t chunks = a.vocab / (a.bf16 ? 8 : 4);
  const int32_t pieces = row_pieces(a.rows, chunks);
  each_rows(a, out, {}, kRowsPerLaunch, [&](const TokenArgs& b, const TokenScores& o,
                                            const TokenGrad&) {
    if (pieces > 1)
      launch_score<kSplitThreads>(b, o, pieces, chunks, workspace, stream);
    else if (chunks <= kRow64)
      launch_score<64>(b, o, 1, chunks, workspace, stream);
    else if (chunks <= kRow256)
      launch_score<256>(b, o, 1, chunks, workspace, stream);
    else if (chunks <= kRow512)
      launch_score<512>(b, o, 1, chunks, workspace, stream);
    else
      launch_score<1024>(b, o, 1, chunks, workspace, stream);
  });
  return hipGetLastError();
}

hipError_t launch_token_grad(const TokenArgs& a, const TokenGrad& g, hipStream_t stream) {
  if (a.rows <= 0) return hipSuccess;
  const int64_t chunks = a.vocab / (a.bf16 ? 8 : 4);
  const int32_t tiles = (int32_t)((chunks + kGradThreads * kGradChunks - 1) /
                                  (kGradThreads * kGradChunks));
  const int32_t least_one = tiles > 0 ? tiles : 1;
  const int64_t most = (int64_t{1} << 23) / least_one > 0 ? (int64_t{1} << 23) / least_one : 1;
  each_rows(a, {}, g, most, [&](const TokenArgs& b, const TokenScores&, const TokenGrad& h) {
    hipLaunchKernelGGL(h.sums ? (a.bf16 ? token_grad_kernel<true, true>
                                        : token_grad_kernel<false, true>)
                              : (a.bf16 ? token_grad_kernel<true, false>
                                        : token_grad_kernel<false, false>),
                       dim3((unsigned)(b.rows * least_one)), dim3(kGradThreads), 0, stream, b, h,
                       least_one);
  });
  return hipGetLastError();
}

template <LossKind KIND>
using Kind = std::integral_constant<LossKind, KIND>;

bool launch_token_loss(const TokenArgs& a, const TokenScores& out, const TokenGrad& g,
                       hipStream_t stream, hipError_t* e, const PolicyArgs* policy,
                       const PolicyRowTerms* terms) {
  *e = hipSuccess;
  if (a.rows <= 0) return true;
  const int64_t chunks = a.vocab / (a.bf16 ? 8 : 4);
  // Few rows leave most of the card idle this way.  Two launches split them
  // instead, and read them twice; one row of 128,256 bf16 18.8 against 7.7 us, 16
  // of 50,257 10.6 / 9.3 (binary32 11.0 / 9.5), 64 of 90,000 binary32 17.9 / 19.9,
  // 64 of 128,256 bf16 25.6 / 16.1, 128 26.4 / 24.9, 256 32.8 / 40.3.
  if (chunks > 5000 && a.rows <= (chunks > 12288 && a.bf16 ? 128 : 32)) return false;
  bool found = true;
  PolicyArgs p = policy ? *policy : PolicyArgs{};
  const PolicyRowTerms t = terms ? *terms : PolicyRowTerms{};
  each_rows(a, out, g, kRowsPerLaunch, [&](const TokenArgs& b, const TokenScores& o,
                                           const TokenGrad& h) {
  // The smallest that holds the row.  us with a variant and with the next larger, 2.5e8
  // bytes of rows, bf16 and binary32: (64, 8) 125 chunks 130 / 258 and 91 / 203, 500
  // 101 / 112 and 93 / 87; (256, 5) 600 104 / 163 and 82 / 110, 1250 91 / 112 and 92 /
  // 87; (512, 8) 2500 97 / 111 and 88 / 93, 4000 96 / 104 and 89 / 86; (1024, 8) 5000
  // 100 / 120 and 86 / 87, 8190 107 / 115 and 96 / 96; (512, 24) 9000 111 / 138 and 92 /
  // 98, 12,288 107 / 128 and 94 / 98.  Binary32 rows that just fit one of the first
  // three would be 3 to 6% faster in the next; the rule is the same for both types.
#define ARC_LOSS(WW, NN)                                                                        \
  if (chunks <= (WW) * (NN)) {                                                                  \
    const auto kernel = [&](auto kind) {                                                        \
      return a.bf16 ? token_loss_kernel<true, WW, NN, decltype(kind)::value>                    \
                    : token_loss_kernel<false, WW, NN, decltype(kind)::value>;                  \
    };                                                                                          \
    hipLaunchKernelGGL(t.rows > 0 ? kernel(Kind<kPolicyWithTerms>())                            \
                       : policy   ? kernel(Kind<kPolicy>())                                     \
                                  : kernel(Kind<kGivenGradients>()),                            \
                       dim3((unsigned)b.rows), dim3(WW), 0, stream, b, o, h, p, t);             \
  } else
    ARC_LOSS(64, 8)
    ARC_LOSS(256, 5)
    ARC_LOSS(512, 8)
    ARC_LOSS(1024, 8)
    ARC_LOSS(512, 24)
    ARC_LOSS(1024, 24)
    found = false;
#undef ARC_LOSS
    for (const float** q : {&p.old_logp, &p.ref_logp, &p.advantages, &p.weights})
      if (*q) *q += b.rows;
  });
  *e = hipGetLastError();
  return found;
}

}  // namespace arc
