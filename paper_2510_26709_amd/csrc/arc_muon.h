// Internal declarations of the matrix optimizer: momenta orthogonalised by
// Newton-Schulz products (arc_muon.hip), and its host side (arc_muon.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace arc {

// Binary32 numbers inside the products are pairs of binary16: hi = x 2^13 rounded,
// lo = what hi lacks, rounded.  2^13, because no entry of a matrix here is larger
// than 2^2.9 (the host checks the coefficients for it) and binary16 ends at 2^16.
constexpr float kPairScale = 8192.f;
constexpr int kPairLine = 32;  // numbers of a row whose pairs lie in one line: 32 hi, 32 lo

constexpr int kMuonRun = 8192;  // elements of a matrix whose squares one workgroup sums
constexpr int kSplitTile = 64;  // sides of what one workgroup splits into pairs
constexpr int kMuonBatch = 160; // matrices of a launch (their pointers are arguments)

// What lies there: X, its transpose (in turn), X X' and what follows from it, all in
// pairs: the polynomial of a step, the product of those of some steps (in turn) and
// a product of two of these on the way.
enum MuonArray {
  kMuonX, kMuonXt, kMuonXt2, kMuonSquare, kMuonPoly, kMuonWay, kMuonAll, kMuonAll2
};

// A matrix, seen from its shorter side: X is m x n, m <= n, or its transpose.
struct MuonMatrix {
  int64_t state;                        // first element of its momentum
  int64_t base;                         // of its pairs in the workspace, bytes
  int64_t first_run;                    // its runs' sums
  int32_t rows, cols;                   // as the caller has it
  int32_t m, n, mp, np;                 // sides, and those of the workspace
  int32_t tall;                         // X is its transpose
  int32_t param_bf16, grad_bf16;
  float weight_decay, lr_scale;
  int32_t runs;
};

// One workgroup's part of a launch: a tile, or with parts > 1 the terms of its sum
// in `lines` lines from `first` on, which the last workgroup of the tile to arrive
// adds to those of the others, at `place` and after it in the list of parts.
struct MuonTile {
  int32_t matrix;
  int32_t i, j;
  int32_t first, lines;
  int32_t part, parts, place;
  int64_t base;    // its matrix's, here too: one load less ahead of the first product
  int32_t mp, np;
};

// Bytes from one row of n numbers to the next.
__host__ __device__ inline int64_t pair_pitch(int32_t n) { return int64_t{4} * n; }

// Where an array of a matrix lies.
__host__ __device__ inline int64_t array_at(int64_t base, int32_t mp, int32_t np, int32_t array) {
  const int64_t x = pair_pitch(np) * mp, xt = pair_pitch(mp) * np, square = pair_pitch(mp) * mp;
  if (array == kMuonX) return base;
  if (array < kMuonSquare) return base + x + (array - kMuonXt) * xt;
  return base + x + 2 * xt + (array - kMuonSquare) * square;
}
constexpr int32_t kMuonArrays = kMuonAll2 + 1;

struct MuonPointers {
  const void* grad[kMuonBatch];
  void* param[kMuonBatch];
  uint16_t* copy[kMuonBatch];
};

struct MuonArgs {
  const MuonMatrix* matrices;  // all of them
  int32_t first;               // matrix of the first pointers
  const float* factor;         // NULL: 1
  float* m;                    // momenta; NULL: the gradients themselves are taken
  float momentum, lr;
  int32_t nesterov, update;    // update: parameters; otherwise they are overwritten
  char* workspace;
  float* parts;                // of tiles whose sums are split, side * side each
  uint32_t* arrived;           // of each place, which go round at its number of parts
  double* sums;                // of the runs' squares
};

// kMuonGram: X X'.  kMuonStep: a + b A + c A A of A = X X'.  kMuonHalf: a product of
// two such, which commute, so that it is symmetric too.  kMuonApply: one of them times
// X, and kMuonLast the same with the parameters' update at its end.
enum MuonKind { kMuonGram, kMuonStep, kMuonHalf, kMuonApply, kMuonLast };

struct MuonProduct {
  int32_t left, right, out, turned;  // MuonArray; turned: the transpose's place
  float scale;                       // of the result in pairs, from the sums of pairs
  float a, b, c;                     // kMuonStep
};

// The momenta, and the squares of what is orthogonalised.
hipError_t launch_muon_momentum(const MuonArgs& a, const MuonPointers& p, const int32_t* run_matrix,
                                int64_t first_run, int64_t runs, hipStream_t stream);
// X and its transpose in pairs, of norm 1.
hipError_t launch_muon_split(const MuonArgs& a, const MuonPointers& p, const MuonTile* tiles,
                             int64_t count, hipStream_t stream);
// Products of square tiles of `side`.
hipError_t launch_muon_product(MuonKind kind, int32_t side, const MuonArgs& a,
                               const MuonPointers& p, const MuonProduct& s,
                               const MuonTile* tiles, int64_t count, hipStream_t stream);
hipError_t prepare_muon_products();

}  // namespace arc
