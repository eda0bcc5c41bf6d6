
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

// The same for the N numbers that a lane holds of a row.
template <bool BF16, bool FULL, int N>
__device__ __forceinline__ void load_some(const void* p, int64_t at, int32_t left,
                                          float (&x)[N]) {
  if constexpr (N == 4) {
    load_four<BF16, FULL>(p, at, left, x);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = FULL || k < left ? load_one<BF16>(p, at + k) : 0.f;
  }
}

template <bool BF16, bool FULL, int N>
__device__ __forceinline__ void store_some(void* p, int64_t at, int32_t left,
                                           const float (&x)[N]) {
  if constexpr (N == 4) {
    store_four<BF16, FULL>(p, at, left, x);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (!FULL && k >= left) break;
      if constexpr (BF16)
        static_cast<uint16_t*>(p)[at + k] = (uint16_t)bf16_pair(x[k], 0.f);
      else
        static_cast<float*>(p)[at + k] = x[k];
    }
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

// The new momenta and the squares of U, a workgroup for each 8192 elements of a matrix
// (their sums are added in order by whoever needs the norm).  HBM: 1.76e8 elements with
// bf16 gradients (10 bytes) 299 us, 5.9 TB/s; 5.9e7 in binary32 (12) 119, 6.0.
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

// X and its transpose in pairs, a workgroup for each 64 x 64 of a matrix.  The norm has to
// be known first, so that U is read, and made of the momentum, a second time; every
// workgroup adds all the runs' sums of its matrix, which grows with the square of the size
// (4096 x 4096 31 us, 128,256 x 4096 4.4 ms, of which 3.3 for that).  Else HBM, more
// than half of it writes: 1.76e8 elements with bf16 gradients (6 bytes read, 8 written)
// 494 us, 5.0 TB/s; 5.9e7 in binary32 (8, 8) 183, 5.2.
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
template <int SIDE>
constexpr int kProductLds = std::max(Shape<SIDE>::kStages * 2 * SIDE * kLineBytes, SIDE* SIDE * 4);

// N numbers that lie side by side in a row, `at` the first one's place: the hi and lo
// halves of their pairs.
template <int N>
struct Halves {
  static_assert(N == 1 || N == 2 || N == 4, "a lane's columns");
  using Word = std::conditional_t<N == 1, uint16_t, std::conditional_t<N == 2, uint32_t, u32x2_t>>;
  Word hi, lo;
  static __device__ __forceinline__ int64_t place(int32_t at) {
    return (int64_t)(at / kPairLine) * kLineBytes + at % kPairLine * 2;
  }
  __device__ __forceinline__ void load(const char* row, int32_t at) {
    hi = *reinterpret_cast<const Word*>(row + place(at));
    lo = *reinterpret_cast<const Word*>(row + place(at) + 2 * kPairLine);
  }
  __device__ __forceinline__ void store(char* row, int32_t at) const {
    *reinterpret_cast<Word*>(row + place(at)) = hi;
    *reinterpret_cast<Word*>(row + place(at) + 2 * kPairLine) = lo;
  }
  // In units of 1 / kPairScale.
  __device__ __forceinline__ float number(int k) const {
    return (float)half(hi, k) + (float)half(lo, k);
  }
  __device__ __forceinline__ void set(const uint32_t (&pair)[N]) {
    if constexpr (N == 1) {
      hi = (uint16_t)pair[0], lo = (uint16_t)(pair[0] >> 16);
    } else if constexpr (N == 2) {
      hi = low(pair[0], pair[1]), lo = high(pair[0], pair[1]);
    } else {
      hi = Word{low(pair[0], pair[1]), low(pair[2], pair[3])};
      lo = Word{high(pair[0], pair[1]), high(pair[2], pair[3])};
    }
  }

 private:
  static __device__ __forceinline__ _Float16 half(const Word& w, int k) {
    uint32_t v;
    if constexpr (N == 4)
      v = k < 2 ? w.x : w.y;
    else
      v = w;
    return __builtin_bit_cast(_Float16, (uint16_t)(v >> (k % 2 * 16)));
  }
  static __device__ __forceinline__ uint32_t low(uint32_t a, uint32_t b) {
    return (a & 0xFFFFu) | (b << 16);
  }
  static __device__ __forceinline__ uint32_t high(uint32_t a, uint32_t b) {
    return (a >> 16) | (b & 0xFFFF0000u);
  }
};

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
    const auto most_before = (uint32_t)(at.parts - 1);
    last = atomicInc(&a.arrived[at.place], most_before) == most_before;
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
// X X' is summed in blocks of as many lines as there are blocks, or nearly, each added to
// those before it: what a chain of additions is off by grows with its length, and steps in
// runs let the error of X X' grow (runs_of()).  Its diagonal is off by 1.6 * 2^-24, of 2048
// numbers to 65,536, where one chain had 2.3 to 5.8; X X' of 4096^3 takes 190 us, not 185.
//
// Large sums are bound by the matrix units at the clock that the card's power leaves them
// (1.6 GHz of 2.4; of zeros the same products take 0.8 of the time): P X of 4096^3 in 317
// us, 1300 TFLOP/s of binary16 products, where the library's plain binary16 product runs
// at 1390.  With short sums the ends count: 48 matrices of width 640 take P X in 282 us,
// of which 179 are the sums (1260 TFLOP/s) and 90 the writing of X both ways (472
// MB, 5.2 TB/s), one after the other though two workgroups share a compute unit; starting
// them apart, priorities and fewer stores in flight made no difference.  Small contexts
// are bound by latency, 4 us a launch with tiles of 32 and 5 to 6 with tiles of 64 (five
// steps of a few vectors 63 and 73 us).
//
// Hence 16 x 16 x 32 instructions, which read and write each binary32 sum once for 32
// terms: with 32 x 32 x 16 (16 terms) a 4096 x 4096 took 3.96 ms against 3.61.  Within 1%
// either way, timed in turn: the next line's pairs read while one is multiplied, wave
// priorities, rows an odd number of lines apart; 1 to 4% slower: no products above the
// diagonal of symmetric tiles; tiles of 256 x 256 by eight waves were even at sums of 4096
// and slower at others, as nothing hides a workgroup's ends.  Results go from registers to
// their rows, 64 bytes of a line together, and only the transposed copy through LDS: a
// 4096 x 4096 3470 us against 3540 with both through it.
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
  // The right side's rows are staged in the order 0, TJ, 2 TJ, .. 15 TJ, 1, TJ + 1, .. of
  // each 16 TJ, so that a lane's columns of the result follow one another.
  static_assert(kWaves % 2 == 0 && kLoads % 2 == 0, "a wave has one side, an even piece first");
  const bool of_right = wave >= kWaves / 2;
  const uint32_t apart = pitch * (of_right ? TJ : 1);
  uint32_t lane_at[2];  // in even and odd pieces of 8 rows
#pragma unroll
  for (int q = 0; q < 2; ++q)
    lane_at[q] = (uint32_t)(lane / 8) * apart + (uint32_t)((lane % 8) ^ (4 * q + lane / 16)) * 16u;
  const buffer_rsrc from = make_buffer(of_right ? right : left, SIDE * pitch);
  const auto stage = [&](int32_t line) {
    char* to = lds + line % kStages * kStage + wave * kLoads * 1024;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int piece = (of_right ? wave - kWaves / 2 : wave) * kLoads + q;
      const int first = of_right ? piece / (2 * TJ) * 16 * TJ + piece % 2 * 8 * TJ + piece / 2 % TJ
                                 : piece * 8;
      load_lds(from, lane_at[q % 2],
               (uint32_t)first * pitch + (uint32_t)(at.first + line) * kLineBytes, to + q * 1024);
    }
  };
  f32x4_t acc[TI][TJ], sums[TI][TJ];  // sums: kMuonGram's, of blocks that are done
  const auto each = [&](const auto& f) {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) f(acc[i][j], sums[i][j]);
  };
  each([](f32x4_t& x, f32x4_t& done) { x = done = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
  const int32_t lines = at.lines;
  int32_t block = 8;  // lines, a power of two
  while (block * block < lines) block *= 2;
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
    if constexpr (WHAT == kMuonGram)
      if ((line & (block - 1)) == block - 1)
        each([](f32x4_t& x, f32x4_t& done) { done += x, x = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
  }
  if constexpr (WHAT == kMuonGram) each([](f32x4_t& x, f32x4_t& done) { x += done; });
  if (at.parts > 1 && !join_parts<SIDE>(a, at, acc)) return;
  // Lane l holds columns TJ (l % 16) + j of its wave's result and rows 16 i + 4 (l / 16)
  // + k: TJ numbers that follow one another in a row, 16 lanes' together whole lines.
  const int32_t r0 = ti * SIDE + wi * TI * 16 + 4 * quarter;
  const int32_t c0 = tj * SIDE + wj * TJ * 16 + row * TJ;
  if constexpr (WHAT == kMuonLast) {
    if (skipped(a)) return;
    const int32_t q = at.matrix - a.first;
    const float step = a.lr * t.lr_scale;
    const float keep = 1.f - step * t.weight_decay;
    void* param = p.param[q];
    uint16_t* copy = p.copy[q];
    const int32_t left = t.cols - c0;
    const auto rows = [&](auto bf16, auto whole) {
      constexpr bool BF16 = decltype(bf16)::value, FULL = decltype(whole)::value;
      float x[TI][4][TJ];  // all loads are in flight together
      if (a.update)
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (FULL || r0 + 16 * i + k < t.rows)
              load_some<BF16, FULL>(param, (int64_t)(r0 + 16 * i + k) * t.cols + c0, left, x[i][k]);
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (!FULL && r0 + 16 * i + k >= t.rows) continue;
          float v[TJ];
#pragma unroll
          for (int j = 0; j < TJ; ++j) {
            v[j] = acc[i][j][k] * s.scale;
            if (a.update) v[j] = fmaf(-step, v[j], x[i][k][j] * keep);
          }
          const int64_t e = (int64_t)(r0 + 16 * i + k) * t.cols + c0;
          store_some<BF16, FULL>(param, e, left, v);
          if (copy) store_some<true, FULL>(copy, e, left, v);
        }
    };
    choose(t.param_bf16, [&](auto bf16) {
      choose((ti + 1) * SIDE <= t.rows && (tj + 1) * SIDE <= t.cols,
             [&](auto whole) { rows(bf16, whole); });
    });
  } else {
    const int64_t out_pitch = pair_pitch(WHAT == kMuonApply ? at.np : at.mp);
    char* out = array(s.out) + r0 * out_pitch;
    uint32_t pair[TI][TJ][4];
    Halves<TJ> square[TI][4];  // of X X', for a step's polynomial of it
    if constexpr (WHAT == kMuonStep)
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          square[i][k].load(array(s.left) + (r0 + 16 * i + k) * out_pitch, c0);
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t side_by_side[TJ];
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          float x = acc[i][j][k] * s.scale;
          if constexpr (WHAT == kMuonStep) {
            x = fmaf(s.c, x, s.b * square[i][k].number(j));
            if (r0 + 16 * i + k == c0 + j) x += s.a * kPairScale;
          }
          side_by_side[j] = pair[i][j][k] = pair_of(x);
        }
        Halves<TJ> h;
        h.set(side_by_side);
        h.store(out + (16 * i + k) * out_pitch, c0);
      }
    if (WHAT != kMuonApply && ti == tj) return;
    // And transposed, through LDS: a column's rows follow one another there, in pieces of
    // four, which 16 lanes write and read from different banks.
    u32x4_t* slab = reinterpret_cast<u32x4_t*>(lds);
    constexpr int kPieces = SIDE / 4, kTurn = TJ > 2 ? TJ : 2, kTurns = kPieces < 16 ? kPieces : 16;
    const auto place = [=](int32_t column, int32_t piece) {
      return column * kPieces + (piece ^ (column / kTurn % kTurns));
    };
    __syncthreads();  // the stages are read
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        slab[place((wj * 16 + row) * TJ + j, (wi * TI + i) * 4 + quarter)] =
            u32x4_t{pair[i][j][0], pair[i][j][1], pair[i][j][2], pair[i][j][3]};
    __syncthreads();
    const int64_t turned_pitch = pair_pitch(at.mp);
    char* turned = array(s.turned) + tj * SIDE * turned_pitch;
    constexpr int kThread = kWaves * kWave;
#pragma unroll 4
    for (int u = threadIdx.x; u < SIDE * SIDE / 8; u += kThread) {  // four threads to a line
      const int n = u / 4 % SIDE, r = u / (4 * SIDE) * 32 + u % 4 * 8;
      const int column = n % 32 * TJ + n / 32;
      const u32x4_t x = slab[place(column, r / 4)], y = slab[place(column, r / 4 + 1)];
      const uint32_t v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      store_8(turned + column * turned_pitch, ti * SIDE + r, v);
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
