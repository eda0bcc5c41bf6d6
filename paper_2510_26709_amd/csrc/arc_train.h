// Internal declarations of the training operators: token log probabilities
// (arc_tokens.hip), gradient norms and AdamW (arc_optim.hip), and their host
// side (arc_train.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace arc {

// ---------------------------------------------------------------- tokens

struct TokenArgs {
  const void* logits = nullptr;
  const int64_t* targets = nullptr;
  int64_t rows = 0, stride = 0, vocab = 0;
  float scale = 1.f;
  int32_t bf16 = 0, top = 0;
};

struct TokenScores {
  float *logp = nullptr, *entropy = nullptr, *lse = nullptr;
  int32_t* top_ids = nullptr;
  float* top_logp = nullptr;
  float* sums = nullptr;  // for a gradient that follows: each row's largest logit and its total
};

struct TokenGrad {
  const float *lse = nullptr, *entropy = nullptr;
  const float *d_logp = nullptr, *d_entropy = nullptr, *d_lse = nullptr;
  void* grad = nullptr;
  int64_t stride = 0;
  const float* sums = nullptr;  // TokenScores' instead of lse: not rounded at its size
};

// Bytes that launch_token_score's workspace needs, zeroed before its first use;
// it leaves the part that has to be zero so.
size_t token_workspace_bytes();
hipError_t launch_token_score(const TokenArgs& a, const TokenScores& out, void* workspace,
                              hipStream_t stream);
// Both in one pass, where a workgroup can hold a row (false: it cannot, and
// nothing was launched); g's lse and entropy are not read.
bool launch_token_loss(const TokenArgs& a, const TokenScores& out, const TokenGrad& g,
                       hipStream_t stream, hipError_t* e);
hipError_t launch_token_grad(const TokenArgs& a, const TokenGrad& g, hipStream_t stream);

// ---------------------------------------------------------------- optimizer

// Elements of a tensor that one workgroup updates, and that one sums the squares
// of: fewer where there are few in all.
constexpr int kOptimChunkLeast = 2048, kOptimChunkMost = 4096, kNormChunkLeast = 4096;
constexpr int kNormChunkMost = 32768;
constexpr int kStateBlock = 128;  // ARC_STATE_BLOCK

// A tensor's place in the states and its constants.
struct OptimTensor {
  int64_t count;
  int64_t state;       // first element of its states
  float weight_decay, lr_scale;
  int32_t first_chunk, first_norm;  // its runs of elements
  int32_t param_bf16, grad_bf16;
};

// Pointers travel in the kernel's arguments (4 KB of them at most), so that a
// call neither copies tables to the device nor waits for an earlier copy.
constexpr int kOptimBatch = 160;
struct OptimPointers {
  const void* grad[kOptimBatch];
  void* param[kOptimBatch];
  uint16_t* copy[kOptimBatch];
};

struct AdamArgs {
  float lr, beta1, beta2, one_minus_beta1, one_minus_beta2, eps;
  float inv_c1, inv_root_c2;
  uint32_t key_low, key_high;  // of this step's random bits
  int32_t stochastic;
  int32_t run;  // elements of a workgroup
  const float* factor;
  void *m, *v;
  float *m_scale, *v_scale;
};

// The chunks [first_chunk, first_chunk + chunks) of tensors first .. of a batch.
struct OptimBatch {
  const OptimTensor* tensors;     // all tensors
  const int32_t* chunk_tensor;    // tensor of each chunk
  int32_t first, first_chunk, chunks;
};

// cached: binary32 arrays are stored through the caches, not past them.
hipError_t launch_adamw(bool f8, bool cached, const OptimBatch& b, const OptimPointers& p,
                        const AdamArgs& a, hipStream_t stream);
constexpr int kNormBatch = 480;
struct NormPointers {
  const void* grad[kNormBatch];
};
typedef OptimBatch NormBatch;

hipError_t launch_norm_chunks(const NormBatch& b, const NormPointers& p, int32_t run,
                              double* partial, hipStream_t stream);
// Each tensor's norm and the total; `arrived` is 0 before and after.
hipError_t launch_norm_tensors(const OptimTensor* tensors, int32_t num, int32_t run,
                               const double* partial,
                               double* squares, uint32_t* arrived, float scale, float max_norm,
                               float* norms, float* total, hipStream_t stream);

}  // namespace arc
