// Matrices orthogonalised by Newton-Schulz products, and the optimizer step made
// of them (the formulas are in libarctopk.h).
//
// X is held as pairs of binary16 numbers (arc_muon.h), 22 bits in all, and a
// product of two takes three matrix instructions, hi hi + hi lo + lo hi, summed in
// binary32: what is left out (lo lo) is 2^-22 of a term, so that the result is as
// exact as a binary32 product's, at a third of binary16's rate, which is four
// times binary32's.  Rounded once to binary16 or bfloat16 instead, X is off by 1e-3
// and 1e-2 after five steps, since small singular values grow 3.4 times in each
// and errors in their directions with them.
//
// All three products of a step have rows on both sides that lie along the sum:
// X X' from X, A A' (A is symmetric), and P X from P and the transpose of X.  So X
// is kept both ways, and every product writes what the next ones read.  Only half
// the tiles of a symmetric result are made; each is written twice.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "arc_device.h"
#include "arc_muon.h"

namespace arc {
namespace {

constexpr int kThreads = 256;
constexpr int kLineBytes = 4 * kPairLine;

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ bool skipped(const MuonArgs& a) {
  return a.factor && !(fabsf(*a.factor) < INFINITY);
}

__device__ __forceinline__ float load_one(const void* p, int32_t bf16, int64_t at) {
  return bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[at] << 16)
              : static_cast<const float*>(p)[at];
}

__device__ __forceinline__ uint32_t bf16_bits(float x) {
  uint32_t w;
  asm("v_cvt_pk_bf16_f32 %0, %1, %1" : "=v"(w) : "v"(x));
  return w & 0xFFFFu;
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
  const int32_t bf16 = t.grad_bf16;
  const float factor = a.factor ? *a.factor : 1.f;
  const int64_t count = (int64_t)t.rows * t.cols;
  const int64_t first = (run - t.first_run) * kMuonRun;
  float* m = a.m ? a.m + t.state : nullptr;
  double sum = 0.0;
#pragma unroll 4
  for (int u = threadIdx.x; u < kMuonRun; u += kThreads) {
    const int64_t e = first + u;
    if (e >= count) break;
    const float g = load_one(grad, bf16, e) * factor;
    float v = 0.f;
    if (m) {
      v = a.momentum * m[e] + g;
      m[e] = v;
    }
    const double d = direction(a, g, v);
    sum = fma(d, d, sum);
  }
  sum = group_sum(sum);
  if (threadIdx.x == 0) a.sums[run] = sum;
}

__global__ void __launch_bounds__(kThreads) muon_norm_kernel(MuonArgs a) {
  const int32_t i = a.first + blockIdx.x;
  const MuonMatrix& t = a.matrices[i];
  double sum = 0.0;
#pragma unroll 4
  for (int32_t r = threadIdx.x; r < t.runs; r += kThreads) sum += a.sums[t.first_run + r];
  sum = group_sum(sum);
  if (threadIdx.x == 0) a.inverse[i] = sum == 0.0 ? 0.0 : (double)kPairScale / sqrt(sum);
}

// ---------------------------------------------------------------- pairs

// 16 numbers of a row: `at` is their first one's place in the row.
__device__ __forceinline__ void store_16(char* row, int32_t at, const uint32_t (&v)[16]) {
  char* line = row + (int64_t)(at / kPairLine) * kLineBytes + at % kPairLine * 2;
  uint32_t hi[8], lo[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    hi[k] = (v[2 * k] & 0xFFFFu) | (v[2 * k + 1] << 16);
    lo[k] = (v[2 * k] >> 16) | (v[2 * k + 1] & 0xFFFF0000u);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    *reinterpret_cast<u32x4_t*>(line + 16 * h) =
        u32x4_t{hi[4 * h], hi[4 * h + 1], hi[4 * h + 2], hi[4 * h + 3]};
    *reinterpret_cast<u32x4_t*>(line + 2 * kPairLine + 16 * h) =
        u32x4_t{lo[4 * h], lo[4 * h + 1], lo[4 * h + 2], lo[4 * h + 3]};
  }
}

__global__ void __launch_bounds__(kThreads)
muon_split_kernel(MuonArgs a, MuonPointers p, const MuonTile* __restrict__ tiles) {
  constexpr int S = kSplitTile;
  __shared__ uint32_t tile[S][S + 1];  // as the caller's matrix lies
  if (skipped(a)) return;
  const MuonTile at = tiles[blockIdx.x];
  const MuonMatrix& t = a.matrices[at.matrix];
  const void* grad = p.grad[at.matrix - a.first];
  const int32_t bf16 = t.grad_bf16;
  const float factor = a.factor ? *a.factor : 1.f;
  const double inverse = a.inverse[at.matrix];
  const float* m = a.m ? a.m + t.state : nullptr;
  const int32_t r0 = (t.tall ? at.j : at.i) * S, c0 = (t.tall ? at.i : at.j) * S;
#pragma unroll 4
  for (int u = threadIdx.x; u < S * S; u += kThreads) {
    const int32_t r = r0 + u / S, c = c0 + u % S;
    uint32_t v = 0;
    if (r < t.rows && c < t.cols) {
      const int64_t e = (int64_t)r * t.cols + c;
      const float d = direction(a, load_one(grad, bf16, e) * factor, m ? m[e] : 0.f);
      v = pair_of((float)((double)d * inverse));
    }
    tile[u / S][u % S] = v;
  }
  __syncthreads();
  const int line = threadIdx.x / 4, part = threadIdx.x % 4 * 16;
  uint32_t along[16], across[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    along[k] = tile[line][part + k];
    across[k] = tile[part + k][line];
  }
  char* x = a.workspace + t.x + (int64_t)(at.i * S + line) * t.np * 4;
  char* xt = a.workspace + t.xt[0] + (int64_t)(at.j * S + line) * t.mp * 4;
  if (t.tall) {
    store_16(x, at.j * S + part, across);
    store_16(xt, at.i * S + part, along);
  } else {
    store_16(x, at.j * S + part, along);
    store_16(xt, at.i * S + part, across);
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

template <int SIDE>
struct Shape;
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
constexpr int kProductLds = Shape<SIDE>::kStages * 2 * SIDE* kLineBytes;

struct NoPointers {};
template <MuonProduct WHAT>
using PointersOf = std::conditional_t<WHAT == kMuonLast, MuonPointers, NoPointers>;

// A tile of L R', both [rows][sum] in pairs.  The sum is taken a line (32 numbers)
// at a time, staged in LDS: row r's 16-byte pieces lie at piece ^ (r % 8), so that
// the eight rows that are read together lie in different banks.
template <int SIDE, MuonProduct WHAT>
__global__ void __launch_bounds__(kProductThreads<SIDE>, Shape<SIDE>::kGroups)
muon_product_kernel(MuonArgs a, PointersOf<WHAT> p, MuonStep s,
                    const MuonTile* __restrict__ tiles) {
  using Sh = Shape<SIDE>;
  constexpr int kWaves = Sh::kWavesI * Sh::kWavesJ, kStages = Sh::kStages;
  constexpr int TI = SIDE / Sh::kWavesI / 32, TJ = SIDE / Sh::kWavesJ / 32;
  constexpr int kStage = 2 * SIDE * kLineBytes;
  constexpr int kLoads = kStage / 1024 / kWaves;  // of a wave and stage
  extern __shared__ char lds[];
  if (skipped(a)) return;
  const MuonTile at = tiles[blockIdx.x];
  const MuonMatrix& t = a.matrices[at.matrix];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wi = wave / Sh::kWavesJ, wj = wave % Sh::kWavesJ;
  const bool swap = WHAT == kMuonLast && t.tall;  // lanes go along the parameter's rows
  const int32_t ti = swap ? at.j : at.i, tj = swap ? at.i : at.j;
  const char* xt = a.workspace + t.xt[s.from];
  const char* poly = a.workspace + t.poly;
  const char *left, *right;
  int32_t sum;
  if constexpr (WHAT == kMuonGram) {
    left = right = a.workspace + t.x;
    sum = t.np;
  } else if constexpr (WHAT == kMuonPoly) {
    left = right = a.workspace + t.gram;
    sum = t.mp;
  } else {
    left = swap ? xt : poly;
    right = swap ? poly : xt;
    sum = t.mp;
  }
  const uint32_t pitch = (uint32_t)sum * 4u;
  left += (int64_t)ti * SIDE * pitch;
  right += (int64_t)tj * SIDE * pitch;
  const buffer_rsrc from[2] = {make_buffer(left, SIDE * pitch), make_buffer(right, SIDE * pitch)};
  const uint32_t lane_at = (uint32_t)(lane / 8) * pitch + (uint32_t)((lane % 8) ^ (lane / 8)) * 16u;
  const auto stage = [&](int32_t line) {
    char* to = lds + line % kStages * kStage;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int piece = wave * kLoads + q;  // of 8 rows; the first half are left's
      const int rows = piece % (SIDE / 8) * 8;
      load_lds(from[piece / (SIDE / 8)], lane_at,
               (uint32_t)rows * pitch + (uint32_t)line * kLineBytes, to + piece * 1024);
    }
  };
  f32x16_t acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
  const int32_t lines = sum / kPairLine;
#pragma unroll
  for (int q = 0; q < kStages - 1; ++q)
    if (q < lines) stage(q);
  const int row = lane % 32, half = lane / 32;
  for (int32_t line = 0; line < lines; ++line) {
    if (line + kStages - 2 < lines)
      arrived<(kStages - 2) * kLoads>();
    else
      arrived<0>();
    if (line + kStages - 1 < lines) stage(line + kStages - 1);
    const char* base = lds + line % kStages * kStage;
    const char* l = base + (wi * TI * 32 + row) * kLineBytes;
    const char* r = base + (SIDE + wj * TJ * 32 + row) * kLineBytes;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      half8_t lh[TI], ll[TI], rh[TJ], rl[TJ];
      const int hi = ((2 * k + half) ^ (row % 8)) * 16, lo = ((4 + 2 * k + half) ^ (row % 8)) * 16;
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        lh[i] = *reinterpret_cast<const half8_t*>(l + i * 32 * kLineBytes + hi);
        ll[i] = *reinterpret_cast<const half8_t*>(l + i * 32 * kLineBytes + lo);
      }
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        rh[j] = *reinterpret_cast<const half8_t*>(r + j * 32 * kLineBytes + hi);
        rl[j] = *reinterpret_cast<const half8_t*>(r + j * 32 * kLineBytes + lo);
      }
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rl[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll[i], rh[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rh[j], acc[i][j], 0, 0, 0);
    }
  }
  // Lane l holds column l % 32 of a 32 x 32 tile, element k in row 8 (k / 4) +
  // 4 (l / 32) + k % 4; all in units of kPairScale^-2.
  if constexpr (WHAT == kMuonLast) {
    const int32_t q = at.matrix - a.first;
    const float step = a.lr * t.lr_scale;
    const float keep = 1.f - step * t.weight_decay;
    void* param = p.param[q];
    uint16_t* copy = p.copy[q];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int32_t r = ti * SIDE + (wi * TI + i) * 32 + 8 * (k / 4) + 4 * half + k % 4;
          const int32_t c = tj * SIDE + (wj * TJ + j) * 32 + row;
          if (r >= t.rows || c >= t.cols) continue;
          const int64_t e = (int64_t)r * t.cols + c;
          float v = acc[i][j][k] * (1.f / (kPairScale * kPairScale));
          if (a.update) v = fmaf(-step, v, load_one(param, t.param_bf16, e) * keep);
          const uint32_t b = bf16_bits(v);
          if (t.param_bf16)
            static_cast<uint16_t*>(param)[e] = (uint16_t)b;
          else
            static_cast<float*>(param)[e] = v;
          if (copy) copy[e] = (uint16_t)b;
        }
  } else {
    __syncthreads();  // the stages are read; each wave takes a part of them for itself
    constexpr int kPitch = 33;
    static_assert(kWaves * 32 * kPitch * 4 <= kProductLds<SIDE>, "room to turn a tile");
    uint32_t* turn = reinterpret_cast<uint32_t*>(lds) + wave * 32 * kPitch;
    char* to = a.workspace + (WHAT == kMuonGram ? t.gram : WHAT == kMuonPoly ? t.poly : t.x);
    char* turned = a.workspace + (WHAT == kMuonGram   ? t.gram
                                  : WHAT == kMuonPoly ? t.poly
                                                      : t.xt[1 - s.from]);
    const int64_t to_pitch = (int64_t)(WHAT == kMuonApply ? t.np : t.mp) * 4;
    const int64_t turned_pitch = (int64_t)t.mp * 4;
    const bool mirror = WHAT == kMuonApply || ti != tj;
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const int32_t r0 = ti * SIDE + (wi * TI + i) * 32, c0 = tj * SIDE + (wj * TJ + j) * 32;
        uint32_t v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          float x = acc[i][j][k] * (1.f / kPairScale);
          const int32_t r = r0 + 8 * (k / 4) + 4 * half + k % 4;
          if constexpr (WHAT == kMuonPoly) {
            const char* g = a.workspace + t.gram + (int64_t)r * to_pitch +
                            (int64_t)(c0 / kPairLine) * kLineBytes + row * 2;
            const float gram = (float)*reinterpret_cast<const _Float16*>(g) +
                               (float)*reinterpret_cast<const _Float16*>(g + 2 * kPairLine);
            x = fmaf(s.c, x, s.b * gram) + (r == c0 + row ? s.a * kPairScale : 0.f);
          }
          v[k] = pair_of(x);
        }
        // rows as they are: turned in LDS, 16 numbers a lane
#pragma unroll
        for (int k = 0; k < 16; ++k) turn[(8 * (k / 4) + 4 * half + k % 4) * kPitch + row] = v[k];
        wave_lds_fence();
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = turn[lane / 2 * kPitch + lane % 2 * 16 + k];
        store_16(to + (r0 + lane / 2) * to_pitch, c0 + lane % 2 * 16, w);
        wave_lds_fence();
        // and transposed: four numbers of a lane follow one another
        if (mirror) {
          char* line = turned + (int64_t)(c0 + row) * turned_pitch +
                       (int64_t)(r0 / kPairLine) * kLineBytes;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const u32x2_t hi = {(v[4 * q] & 0xFFFFu) | (v[4 * q + 1] << 16),
                                (v[4 * q + 2] & 0xFFFFu) | (v[4 * q + 3] << 16)};
            const u32x2_t lo = {(v[4 * q] >> 16) | (v[4 * q + 1] & 0xFFFF0000u),
                                (v[4 * q + 2] >> 16) | (v[4 * q + 3] & 0xFFFF0000u)};
            *reinterpret_cast<u32x2_t*>(line + (8 * q + 4 * half) * 2) = hi;
            *reinterpret_cast<u32x2_t*>(line + 2 * kPairLine + (8 * q + 4 * half) * 2) = lo;
          }
        }
      }
  }
}

template <int SIDE, MuonProduct WHAT>
void launch_tiles(const MuonArgs& a, const PointersOf<WHAT>& p, const MuonStep& s,
                  const MuonTile* tiles, int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL((muon_product_kernel<SIDE, WHAT>), dim3((unsigned)count),
                     dim3(kProductThreads<SIDE>), kProductLds<SIDE>, stream, a, p, s, tiles);
}

template <int SIDE>
hipError_t launch_product(MuonProduct what, const MuonArgs& a, const MuonPointers* p,
                          const MuonStep& s, const MuonTile* tiles, int64_t count,
                          hipStream_t stream) {
  if (what == kMuonGram)
    launch_tiles<SIDE, kMuonGram>(a, {}, s, tiles, count, stream);
  else if (what == kMuonPoly)
    launch_tiles<SIDE, kMuonPoly>(a, {}, s, tiles, count, stream);
  else if (what == kMuonApply)
    launch_tiles<SIDE, kMuonApply>(a, {}, s, tiles, count, stream);
  else
    launch_tiles<SIDE, kMuonLast>(a, *p, s, tiles, count, stream);
  return hipGetLastError();
}

template <int SIDE>
hipError_t reserve_lds() {
  for (const void* kernel : {reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonGram>),
                             reinterpret_cast<const void*>(muon_product_kernel<SIDE, kMuonPoly>),
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
  const hipError_t e = reserve_lds<64>();
  return e != hipSuccess ? e : reserve_lds<128>();
}

hipError_t launch_muon_momentum(const MuonArgs& a, const MuonPointers& p, const int32_t* run_matrix,
                                int64_t first_run, int64_t runs, hipStream_t stream) {
  hipLaunchKernelGGL(muon_momentum_kernel, dim3((unsigned)runs), dim3(kThreads), 0, stream, a, p,
                     run_matrix, first_run);
  return hipGetLastError();
}

hipError_t launch_muon_norms(const MuonArgs& a, int32_t count, hipStream_t stream) {
  hipLaunchKernelGGL(muon_norm_kernel, dim3((unsigned)count), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_muon_split(const MuonArgs& a, const MuonPointers& p, const MuonTile* tiles,
                             int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL(muon_split_kernel, dim3((unsigned)count), dim3(kThreads), 0, stream, a, p,
                     tiles);
  return hipGetLastError();
}

hipError_t launch_muon_product(MuonProduct what, int32_t side, const MuonArgs& a,
                               const MuonPointers* p, const MuonStep& s, const MuonTile* tiles,
                               int64_t count, hipStream_t stream) {
  return side == 64 ? launch_product<64>(what, a, p, s, tiles, count, stream)
                    : launch_product<128>(what, a, p, s, tiles, count, stream);
}

}  // namespace arc
