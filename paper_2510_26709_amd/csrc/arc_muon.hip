
// Matrices orthogonalised by Newton-Schulz products, and the optimizer step made
// of them (the formulas are in libarctopk.h).
//
// X is held as pairs of binary16 numbers (arc_muon.h), 22 bits in all, and a
// product of two takes three matrix instructions, hi hi + hi lo + lo hi, summed in
// binary32: what is left out (lo lo) is 2^-24 of a term, so that the result is as
// exact as a binary32 product's, at a third of binary16's rate, which is three
// times what binary32 matrix instructions reach (132 to 153 TFLOP/s).  Rounded once
// to binary16 or bfloat16 instead, X is off by 1e-3 and 1e-2 after five steps, since
// small singular values grow 3.4 times in each and errors in their directions with
// them.
//
// All three products of a step have rows on both sides that lie along the sum:
// X X' from X, A A' (A is symmetric), and P X from P and the transpose of X.  So X
// is kept both ways, and every product writes what the next ones read.  Only half
// the tiles of a symmetric result are made; each is written twice.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "arc_device.h"
#include "arc_muon.h"

namespace arc {
namespace {

constexpr int kThreads = 256;
constexpr int kLineBytes = 4 * kPairLine;

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bool skipped(const MuonArgs& a) {
  return a.factor && !(fabsf(*a.factor) < INFINITY);
}

template <bool BF16>
__device__ __forceinline__ float load_one(const void* p, int64_t at) {
  if constexpr (BF16)
    return __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[at] << 16);
  return static_cast<const float*>(p)[at];
}

// Calls f(std::true_type()) or f(std::false_type()).
template <typename F>
__device__ __forceinline__ void choose(bool which, const F& f) {
  if (which)
    f(std::true_type());
  else
    f(std::false_type());
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t w;
  asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(lo), "v"(hi));
  return w;
}

typedef uint32_t loose_u32x4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t loose_u32x2_t __attribute__((ext_vector_type(2), aligned(2)));

// Four numbers from element `at` on, at any element alignment, of which `left` are
// there (FULL: all of them).  The type is a template's argument: a branch around each
// load would wait for it before the next.
template <bool BF16, bool FULL>
__device__ __forceinline__ void load_four(const void* p, int64_t at, int32_t left,
                                          float (&x)[4]) {
  if (FULL || left >= 4) {
    if constexpr (BF16) {
      const u32x2_t w =
          *reinterpret_cast<const loose_u32x2_t*>(static_cast<const uint16_t*>(p) + at);
      x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
    } else {
      const u32x4_t w = *reinterpret_cast<const loose_u32x4_t*>(static_cast<const float*>(p) + at);
      x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y);
      x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = k < left ? load_one<BF16>(p, at + k) : 0.f;
}

template <bool BF16, bool FULL>
__device__ __forceinline__ void store_four(void* p, int64_t at, int32_t left,
                                           const float (&x)[4]) {
  const u32x2_t h = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
  if (FULL || left >= 4) {
    if constexpr (BF16)
      *reinterpret_cast<loose_u32x2_t*>(static_cast<uint16_t*>(p) + at) = h;
    else
      *reinterpret_cast<loose_u32x4_t*>(static_cast<float*>(p) + at) =
          u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                  __float_as_uint(x[3])};
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k >= left) break;
    if constexpr (BF16)
      static_cast<uint16_t*>(p)[at + k] = (uint16_t)((k < 2 ? h.x : h.y) >> (k % 2 * 16));
    else
      static_cast<float*>(p)[at + k] = x[k];
  }
}

// hi in the low half, lo in the high one, of a number times kPairScale.
__device__ __forceinline__ uint32_t pair_of(float scaled) {
  const _Float16 hi = (_Float16)scaled;
  const _Float16 lo = (_Float16)(scaled - (float)hi);
  return (uint32_t)__builtin_bit_cast(uint16_t, hi) |
         ((uint32_t)__builtin_bit_cast(uint16_t, lo) << 16);
}

// What is orthogonalised, from a gradient times the factor and the new momentum.
__device__ __forceinline__ float direction(const MuonArgs& a, float g, float m) {
  return a.m == nullptr ? g : a.nesterov ? fmaf(a.momentum, m, g) : m;
}

// ---------------------------------------------------------------- momenta

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

__device__ __forceinline__ double group_sum(double v) {
  __shared__ double part[kThreads / kWave];
  v = wave_sum_f64(v);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ void __launch_bounds__(kThreads)
muon_momentum_kernel(MuonArgs a, MuonPointers p, const int32_t* __restrict__ run_matrix,
                     int64_t first_run) {
  if (skipped(a)) return;
  const int64_t run = first_run + blockIdx.x;
  const int32_t i = run_matrix[run];
  const MuonMatrix& t = a.matrices[i];
  const void* grad = p.grad[i - a.first];
  const float factor = a.factor ? *a.factor : 1.f;
  const int64_t count = (int64_t)t.rows * t.cols;
  const int64_t first = (run - t.first_run) * kMuonRun;
  float* m = a.m ? a.m + t.state : nullptr;
  double sum = 0.0;
  const auto passes = [&](auto bf16, auto whole, auto kept) {
    constexpr bool BF16 = decltype(bf16)::value, FULL = decltype(whole)::value;
    constexpr bool KEPT = decltype(kept)::value;
    constexpr int U = 4;  // passes whose loads are in flight together
    for (int u = 0; u < kMuonRun; u += U * 4 * kThreads) {
      if (!FULL && first + u >= count) break;
      float g[U][4], v[U][4];
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int64_t e = first + u + (q * kThreads + (int)threadIdx.x) * 4;
        const int32_t left = FULL ? 4 : (int32_t)max(min(count - e, (int64_t)4), (int64_t)0);
        load_four<BF16, FULL>(grad, e, left, g[q]);
        if constexpr (KEPT) load_four<false, FULL>(m, e, left, v[q]);
      }
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int64_t e = first + u + (q * kThreads + (int)threadIdx.x) * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          g[q][k] *= factor;
          if constexpr (KEPT) v[q][k] = a.momentum * v[q][k] + g[q][k];
          const double d = direction(a, g[q][k], KEPT ? v[q][k] : 0.f);
          sum = fma(d, d, sum);  // (behind the end: zeros)
        }
        if constexpr (KEPT)
          store_four<false, FULL>(
              m, e, FULL ? 4 : (int32_t)max(min(count - e, (int64_t)4), (int64_t)0), v[q]);
      }
    }
  };
  choose(t.grad_bf16, [&](auto bf16) {
    choose(first + kMuonRun <= count, [&](auto whole) {
      choose(m != nullptr, [&](auto kept) { passes(bf16, whole, kept); });
    });
  });
  sum = group_sum(sum);
  if (threadIdx.x == 0) a.sums[run] = sum;
}

// ---------------------------------------------------------------- pairs

// Eight numbers of a row, `at` the first one's place in it: four threads that follow
// one another write 64 bytes together, twice.  (16 numbers a thread take twice the
// requests, which the L2 has to take beside those of the tiles that are read.)
__device__ __forceinline__ void store_8(char* row, int32_t at, const uint32_t (&v)[8]) {
  char* line = row + (int64_t)(at / kPairLine) * kLineBytes + at % kPairLine * 2;
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    hi[k] = (v[2 * k] & 0xFFFFu) | (v[2 * k + 1] << 16);
    lo[k] = (v[2 * k] >> 16) | (v[2 * k + 1] & 0xFFFF0000u);
  }
  *reinterpret_cast<u32x4_t*>(line) = u32x4_t{hi[0], hi[1], hi[2], hi[3]};
  *reinterpret_cast<u32x4_t*>(line + 2 * kPairLine) = u32x4_t{lo[0], lo[1], lo[2], lo[3]};
}

__global__ void __launch_bounds__(kThreads)
muon_split_kernel(MuonArgs a, MuonPointers p, const MuonTile* __restrict__ tiles) {
  constexpr int S = kSplitTile;
  __shared__ uint32_t tile[S][S + 2];  // as the caller's matrix lies
  if (skipped(a)) return;
  const MuonTile at = tiles[blockIdx.x];
  const MuonMatrix& t = a.matrices[at.matrix];
  const void* grad = p.grad[at.matrix - a.first];
  const float factor = a.factor ? *a.factor : 1.f;
  double squares = 0.0;  // every workgroup adds the runs' sums in the same order
#pragma unroll 4
  for (int32_t r = threadIdx.x; r < t.runs; r += kThreads) squares += a.sums[t.first_run + r];
  squares = group_sum(squares);
  const double inverse = squares == 0.0 ? 0.0 : (double)kPairScale / sqrt(squares);
  const float* m = a.m ? a.m + t.state : nullptr;
  const int32_t r0 = (t.tall ? at.j : at.i) * S, c0 = (t.tall ? at.i : at.j) * S;
  const auto fill = [&](auto bf16, auto kept, auto whole) {
    constexpr bool BF16 = decltype(bf16)::value, KEPT = decltype(kept)::value;
    constexpr bool FULL = decltype(whole)::value;
    constexpr int U = S * S / 4 / kThreads, kDown = kThreads / (S / 4);
    const int32_t c = c0 + (int)threadIdx.x % (S / 4) * 4, left = t.cols - c;
    const int32_t r = r0 + (int)threadIdx.x / (S / 4);
    float g[U][4], v[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int k = 0; k < 4; ++k) g[u][k] = v[u][k] = 0.f;
      if (!FULL && r + u * kDown >= t.rows) continue;
      const int64_t e = (int64_t)(r + u * kDown) * t.cols + c;
      load_four<BF16, FULL>(grad, e, left, g[u]);
      if constexpr (KEPT) load_four<false, FULL>(m, e, left, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        tile[r - r0 + u * kDown][c - c0 + k] =
            pair_of((float)((double)direction(a, g[u][k] * factor, v[u][k]) * inverse));
  };
  choose(t.grad_bf16, [&](auto bf16) {
    choose(m != nullptr, [&](auto kept) {
      choose(r0 + S <= t.rows && c0 + S <= t.cols, [&](auto whole) { fill(bf16, kept, whole); });
    });
  });
  __syncthreads();
  char* x = a.workspace + array_at(at.base, at.mp, at.np, kMuonX) + at.i * S * pair_pitch(at.np);
  char* xt = a.workspace + array_at(at.base, at.mp, at.np, kMuonXt) + at.j * S * pair_pitch(at.mp);
  char *along = t.tall ? xt : x, *across = t.tall ? x : xt;
  const int64_t along_pitch = pair_pitch(t.tall ? at.mp : at.np);
  const int64_t across_pitch = pair_pitch(t.tall ? at.np : at.mp);
#pragma unroll
  for (int u = threadIdx.x; u < S * S / 8; u += kThreads) {
    uint32_t v[8];
    const int line = u / (S / 8), part = u % (S / 8) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = tile[line][part + k];
    store_8(along + line * along_pitch, c0 + part, v);
    const int column = u / 4 % S, run = u / (4 * S) * 32 + u % 4 * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = tile[run + k][column];
    store_8(across + column * across_pitch, r0 + run, v);
  }
}

// ---------------------------------------------------------------- products

// 16 bytes a lane to the wave's LDS at dst + 16 * lane, without a register in
// between; counts as a vector memory load.
__device__ __forceinline__ void load_lds(buffer_rsrc r, uint32_t lane_at, uint32_t at, char* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)dst, 16,
                                           (int)lane_at, (int)at, 0, 0);
}

// The loads of all but the last `N` of this wave have arrived, its reads of LDS
// are done, and so are those of the whole workgroup.
template <int N>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Waves of a tile, lines of its sum in LDS (one is multiplied while the others
// arrive; as many as leave kGroups workgroups room on a compute unit), workgroups that
// the registers are shared by.  Four waves in all: each then holds 64 x 64, 32 x 32 or
// 16 x 16 of a result.
template <int SIDE>
struct Shape;
template <>
struct Shape<32> {
  static constexpr int kWavesI = 2, kWavesJ = 2, kStages = 4, kGroups = 4;
};
template <>
struct Shape<64> {
  static constexpr int kWavesI = 2, kWavesJ = 2, kStages = 3, kGroups = 3;
};
template <>
struct Shape<128> {
  static constexpr int kWavesI = 2, kWavesJ = 2, kStages = 2, kGroups = 2;
};
template <int SIDE>
constexpr int kProductThreads = Shape<SIDE>::kWavesI * Shape<SIDE>::kWavesJ* kWave;
// Results go through LDS, rows two words apart from each other: 16 columns of four
// runs of eight rows then lie in 64 different banks.
template <int SIDE>
constexpr int kSlabPitch = SIDE + 2;
template <int SIDE>
constexpr int kProductLds =
    std::max(Shape<SIDE>::kStages * 2 * SIDE * kLineBytes, SIDE* kSlabPitch<SIDE> * 4);

// The numbers of eight pairs of a row, in units of 1 / kPairScale.
__device__ __forceinline__ void load_8(const char* row, int32_t at, float (&x)[8]) {
  const char* line = row + (int64_t)(at / kPairLine) * kLineBytes + at % kPairLine * 2;
  const half8_t hi = *reinterpret_cast<const half8_t*>(line);
  const half8_t lo = *reinterpret_cast<const half8_t*>(line + 2 * kPairLine);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = (float)hi[k] + (float)lo[k];
}

// Adds a tile's parts in their order, in the last workgroup to arrive; false: this is
// not the last.  Parts are written through to where every compute unit sees them,
// and read from there.
template <int SIDE, int TI, int TJ>
__device__ __forceinline__ bool join_parts(const MuonArgs& a, const MuonTile& at,
                                           f32x4_t (&acc)[TI][TJ]) {
  __shared__ bool last;
  constexpr int kThread = kProductThreads<SIDE>;
  constexpr int kDevice = 16;  // the sc1 bit
  constexpr uint32_t kBytes = SIDE * SIDE * 4u;
  float* first = a.parts + (int64_t)at.place * SIDE * SIDE;
  const buffer_rsrc mine = make_buffer(first + (int64_t)at.part * SIDE * SIDE, kBytes);
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, acc[i][j]), mine,
                                             (int)threadIdx.x * 16, (i * TJ + j) * kThread * 16,
                                             kDevice);
  wave_vmem_fence();  // written before it counts
  __syncthreads();
  if (threadIdx.x == 0) {
    last = __hip_atomic_fetch_add(&a.arrived[at.place], 1u, __ATOMIC_RELAXED,
                                  __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(at.parts - 1);
    if (last)
      __hip_atomic_store(&a.arrived[at.place], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return false;
  for (int32_t q = 0; q < at.parts; ++q) {
    const buffer_rsrc of = make_buffer(first + (int64_t)q * SIDE * SIDE, kBytes);
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const f32x4_t v = __builtin_bit_cast(
            f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                         of, (int)threadIdx.x * 16, (i * TJ + j) * kThread * 16, kDevice));
        acc[i][j] = q == 0 ? v : acc[i][j] + v;
      }
  }
  return true;
}

struct NoPointers {};
template <MuonKind WHAT>
using PointersOf = std::conditional_t<WHAT == kMuonLast, MuonPointers, NoPointers>;

// A tile of L R', both [rows][sum] in pairs.  The sum is taken a line (32 numbers)
// at a time, staged in LDS: row r's 16-byte pieces lie at piece ^ (r / 2 % 8), so
// that 16 rows' pieces, which are read together, lie in different banks.
//
// Bound by the matrix units at the clock that the card's power leaves them (1.7 GHz of
// 2.4; of a matrix of zeros the same products take 0.7 of the time): 4096^3 in 323 to
// 360 us, 1140 to 1280 TFLOP/s of binary16 products, where the library's plain binary16
// product runs at 1390; small contexts are bound by latency, 4 us a launch with tiles
// of 32 and 5 to 6 with tiles of 64 (five steps of a few vectors 63 and 73 us).  Hence 16 x 16 x 32 instructions, which read and write each binary32 sum once
// for 32 terms: with 32 x 32 x 16 (16 terms) a 4096 x 4096 took 3.96 ms against 3.61.
// Within 1% either way, timed in turn: the next line's pairs read while one is
// multiplied, wave priorities, rows an odd number of lines apart; 1 to 4% slower: no
// products above the diagonal of symmetric tiles; tiles of 256 x 256 by eight waves
// were even at sums of 4096 and slower at others, as nothing hides a workgroup's ends.
// A tile's end (results through LDS, 64 bytes of a line together) is 13% of the time
// with sums of 2048, a third with 640.
template <int SIDE, MuonKind WHAT>
__global__ void __launch_bounds__(kProductThreads<SIDE>, Shape<SIDE>::kGroups)
muon_product_kernel(MuonArgs a, PointersOf<WHAT> p, MuonProduct s,
                    const MuonTile* __restrict__ tiles) {
  using Sh = Shape<SIDE>;
  constexpr int kWaves = Sh::kWavesI * Sh::kWavesJ, kStages = Sh::kStages;
  constexpr int TI = SIDE / Sh::kWavesI / 16, TJ = SIDE / Sh::kWavesJ / 16;
  constexpr int kStage = 2 * SIDE * kLineBytes;
  constexpr int kLoads = kStage / 1024 / kWaves;  // of a wave and stage
  extern __shared__ __attribute__((aligned(256))) char lds[];
  const MuonTile at = tiles[blockIdx.x];
  const MuonMatrix& t = a.matrices[at.matrix];  // (read by kMuonLast alone)
  const auto array = [&](int32_t which) {
    return a.workspace + array_at(at.base, at.mp, at.np, which);
  };
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wi = wave / Sh::kWavesJ, wj = wave % Sh::kWavesJ;
  const bool swap = WHAT == kMuonLast && t.tall;  // lanes go along the parameter's rows
  const int32_t ti = swap ? at.j : at.i, tj = swap ? at.i : at.j;
  const char* left = array(swap ? s.right : s.left);
  const char* right = array(swap ? s.left : s.right);
  const int32_t sum = WHAT == kMuonGram ? at.np : at.mp;
  const uint32_t pitch = (uint32_t)pair_pitch(sum);
  left += (int64_t)ti * SIDE * pitch;
  right += (int64_t)tj * SIDE * pitch;
  const buffer_rsrc from[2] = {make_buffer(left, SIDE * pitch), make_buffer(right, SIDE * pitch)};
  uint32_t lane_at[2];  // in even and odd pieces of 8 rows
#pragma unroll
  for (int q = 0; q < 2; ++q)
    lane_at[q] = (uint32_t)(lane / 8) * pitch + (uint32_t)((lane % 8) ^ (4 * q + lane / 16)) * 16u;
  static_assert(kLoads % 2 == 0, "a wave's first piece is an even one");
  const auto stage = [&](int32_t line) {
    char* to = lds + line % kStages * kStage;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int piece = wave * kLoads + q;  // of 8 rows; the first half are left's
      const int rows = piece % (SIDE / 8) * 8;
      load_lds(from[piece / (SIDE / 8)], lane_at[q % 2],
               (uint32_t)rows * pitch + (uint32_t)(at.first + line) * kLineBytes,
               to + piece * 1024);
    }
  };
  f32x4_t acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
  const int32_t lines = at.lines;
#pragma unroll
  for (int q = 0; q < kStages - 1; ++q)
    if (q < lines) stage(q);
  const int row = lane % 16, quarter = lane / 16;
  for (int32_t line = 0; line < lines; ++line) {
    if (line + kStages - 2 < lines)
      arrived<(kStages - 2) * kLoads>();
    else
      arrived<0>();
    if (line + kStages - 1 < lines) stage(line + kStages - 1);
    const char* base = lds + line % kStages * kStage;
    const char* l = base + (wi * TI * 16 + row) * kLineBytes;
    const char* r = base + (SIDE + wj * TJ * 16 + row) * kLineBytes;
    half8_t lh[TI], ll[TI], rh[TJ], rl[TJ];
    const int hi = (quarter ^ (row / 2)) * 16, lo = hi ^ 64;
#pragma unroll
    for (int j = 0; j < TJ; ++j) {
      rh[j] = *reinterpret_cast<const half8_t*>(r + j * 16 * kLineBytes + hi);
      rl[j] = *reinterpret_cast<const half8_t*>(r + j * 16 * kLineBytes + lo);
    }
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      lh[i] = *reinterpret_cast<const half8_t*>(l + i * 16 * kLineBytes + hi);
      ll[i] = *reinterpret_cast<const half8_t*>(l + i * 16 * kLineBytes + lo);
    }
    __builtin_amdgcn_sched_barrier(0);  // all reads ahead of the products
    const auto multiply = [&](const half8_t(&x)[TI], const half8_t(&y)[TJ]) {
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[i], y[j], acc[i][j], 0, 0, 0);
    };
    multiply(lh, rl);
    multiply(lh, rh);
    multiply(ll, rh);
  }
  if (at.parts > 1 && !join_parts<SIDE>(a, at, acc)) return;
  // Lane l holds column l % 16 of a 16 x 16 tile, element k in row 4 (l / 16) + k.
  constexpr int kThread = kWaves * kWave, kPitch = kSlabPitch<SIDE>;
  float* slab = reinterpret_cast<float*>(lds);
  const int32_t r0 = ti * SIDE, c0 = tj * SIDE;
  const auto to_slab = [&] {
    __syncthreads();  // the stages are read
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          slab[((wi * TI + i) * 16 + 4 * quarter + k) * kPitch + (wj * TJ + j) * 16 + row] =
              acc[i][j][k];
    __syncthreads();
  };
  if constexpr (WHAT == kMuonLast) {
    // A thread has all its loads in flight together, and whole lines are read and
    // written.
    if (skipped(a)) return;
    constexpr int kAcross = SIDE / 4, kDown = kThread / kAcross, kPasses = SIDE / kDown;
    const int32_t q = at.matrix - a.first;
    const float step = a.lr * t.lr_scale;
    const float keep = 1.f - step * t.weight_decay;
    void* param = p.param[q];
    uint16_t* copy = p.copy[q];
    const int32_t down = (int)threadIdx.x / kAcross, across = (int)threadIdx.x % kAcross * 4;
    const int32_t left = t.cols - c0 - across;
    const int32_t r = r0 + down;
    const int64_t e0 = (int64_t)r * t.cols + c0 + across;
    const auto passes = [&](auto bf16, auto whole) {
      constexpr bool BF16 = decltype(bf16)::value, FULL = decltype(whole)::value;
      float x[kPasses][4];
      if (a.update)
#pragma unroll
        for (int q = 0; q < kPasses; ++q)
          if (FULL || r + q * kDown < t.rows)
            load_four<BF16, FULL>(param, e0 + (int64_t)q * kDown * t.cols, left, x[q]);
      to_slab();
#pragma unroll
      for (int q = 0; q < kPasses; ++q) {
        if (!FULL && r + q * kDown >= t.rows) continue;
        const float* of = slab + (q * kDown + down) * kPitch + across;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = of[k] * s.scale;
          if (a.update) v[k] = fmaf(-step, v[k], x[q][k] * keep);
        }
        const int64_t e = e0 + (int64_t)q * kDown * t.cols;
        store_four<BF16, FULL>(param, e, left, v);
        if (copy) store_four<true, FULL>(copy, e, left, v);
      }
    };
    choose(t.param_bf16, [&](auto bf16) {
      choose(r0 + SIDE <= t.rows && c0 + SIDE <= t.cols,
             [&](auto whole) { passes(bf16, whole); });
    });
  } else {
    char* to = array(s.out);
    char* turned = array(s.turned);
    const int64_t to_pitch = pair_pitch(WHAT == kMuonApply ? at.np : at.mp);
    const int64_t turned_pitch = pair_pitch(at.mp);
    const bool mirror = WHAT == kMuonApply || ti != tj;
    to_slab();
    // Rows as they are, eight numbers a thread and pass; the pairs take the numbers'
    // places.
    constexpr int kRuns = SIDE / 8;
#pragma unroll 4
    for (int u = threadIdx.x; u < SIDE * kRuns; u += kThread) {
      const int r = u / kRuns, c = u % kRuns * 8;
      float* of = slab + r * kPitch + c;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = of[k] * s.scale;
      if constexpr (WHAT == kMuonStep) {
        float square[8];
        load_8(array(s.left) + (r0 + r) * to_pitch, c0 + c, square);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] = fmaf(s.c, x[k], s.b * square[k]);
          if (r0 + r == c0 + c + k) x[k] += s.a * kPairScale;
        }
      }
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = pair_of(x[k]);
      store_8(to + (r0 + r) * to_pitch, c0 + c, v);
      if (mirror)
#pragma unroll
        for (int k = 0; k < 8; ++k) of[k] = __uint_as_float(v[k]);
    }
    if (!mirror) return;
    __syncthreads();
    // And transposed, four threads to a line.
#pragma unroll 4
    for (int u = threadIdx.x; u < SIDE * kRuns; u += kThread) {
      const int c = u / 4 % SIDE, r = u / (4 * SIDE) * 32 + u % 4 * 8;
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(slab[(r + k) * kPitch + c]);
      store_8(turned + (c0 + c) * turned_pitch, r0 + r, v);
    }
  }
}

template <int SIDE, MuonKind WHAT>
void launch_tiles(const MuonArgs& a, const PointersOf<WHAT>& p, const MuonProduct& s,
                  const MuonTile* tiles, int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL((muon_product_kernel<SIDE, WHAT>), dim3((unsigned)count),
                     dim3(kProductThreads<SIDE>), kProductLds<SIDE>, stream, a, p, s, tiles);
}

template <int SIDE>
hipError_t launch_product(MuonKind kind, const MuonArgs& a, const MuonPointers& p,
                          const MuonProduct& s, const MuonTile* tiles, int64_t count,
                          hipStream_t stream) {
  switch (kind) {
    case kMuonGram: launch_tiles<SIDE, kMuonGram>(a, {}, s, tiles, count, stream); break;
    case kMuonStep: launch_tiles<SIDE, kMuonStep>(a, {}, s, tiles, count, stream); break;
    case kMuonHalf: launch_tiles<SIDE, kMuonHalf>(a, {}, s, tiles, count, stream); break;
    case kMuonApply: launch_tiles<SIDE, kMuonApply>(a, {}, s, tiles, count, stream); break;
    case kMuonLast: launch_tiles<SIDE, kMuonLast>(a, p, s, tiles, count, stream); break;
  }
  return hipGetLastError();
}

template <int SIDE>
hipError_t reserve_lds() {
  for (const void* kernel : {reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonGram>),
                             reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonStep>),
                             reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonHalf>),
                             reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonApply>),
                             reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonLast>)}) {
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             kProductLds<SIDE>);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t prepare_muon_products() {
  hipError_t e = reserve_lds<32>();
  if (e == hipSuccess) e = reserve_lds<64>();
  if (e == hipSuccess) e = reserve_lds<128>();
  return e;
}

hipError_t launch_muon_momentum(const MuonArgs& a, const MuonPointers& p, const int32_t* run_matrix,
                                int64_t first_run, int64_t runs, hipStream_t stream) {
  hipLaunchKernelGGL(muon_momentum_kernel, dim3((unsigned)runs), dim3(kThreads), 0, stream, a, p,
                     run_matrix, first_run);
  return hipGetLastError();
}

hipError_t launch_muon_split(const MuonArgs& a, const MuonPointers& p, const MuonTile* tiles,
                             int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL(muon_split_kernel, dim3((unsigned)count), dim3(kThreads), 0, stream, a, p,
                     tiles);
  return hipGetLastError();
}

hipError_t launch_muon_product(MuonKind kind, int32_t side, const MuonArgs& a,
                               const MuonPointers& p, const MuonProduct& s,
                               const MuonTile* tiles, int64_t count, hipStream_t stream) {
  return side == 32   ? launch_product<32>(kind, a, p, s, tiles, count, stream)
         : side == 64 ? launch_product<64>(kind, a, p, s, tiles, count, stream)
                      : launch_product<128>(kind, a, p, s, tiles, count, stream);
}

}  // namespace arc
