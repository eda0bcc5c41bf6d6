// Drives the host side of the training operators (arc_train.cpp) where it needs
// no device: refusals, the planning of valid configurations (which then fail at
// the first HIP call and release what they built, or succeed on a machine with
// a device), and the NULL contexts.  Built with AddressSanitizer on the host
// code; prints "ok" when every check holds.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <string>
#include <vector>

#include "arc_context.h"

namespace arc {
static std::string why;
arc_status fail(arc_status s, const std::string& w) {
  why = w;
  return s;
}
arc_status fail_hip(hipError_t e, const char* where) {
  why = std::string(where) + ": " + hipGetErrorString(e);
  return e == hipErrorOutOfMemory ? ARC_ERR_NOMEM : ARC_ERR_DEVICE;
}
}  // namespace arc

static int failures = 0;
#define CHECK(cond)                                                                        \
  do {                                                                                     \
    if (!(cond)) {                                                                         \
      std::fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #cond, arc::why.c_str());       \
      ++failures;                                                                          \
    }                                                                                      \
  } while (0)

static bool refused(arc_status s) { return s == ARC_ERR_INVALID && !arc::why.empty(); }

static void plan(const std::vector<arc_optim_tensor>& tensors, int32_t state) {
  arc_optim_config cfg{tensors.data(), static_cast<int32_t>(tensors.size()), state, 0, 0, 7};
  arc_optim* opt = nullptr;
  const arc_status st = arc_optim_create(&cfg, nullptr, &opt);
  if (st == ARC_OK) {
    int64_t at = 0;
    for (size_t i = 0; i < tensors.size(); ++i) {
      CHECK(arc_optim_state_offset(opt, static_cast<int32_t>(i)) == at);
      at += (tensors[i].count + ARC_STATE_BLOCK - 1) / ARC_STATE_BLOCK * ARC_STATE_BLOCK;
    }
    CHECK(arc_optim_state_elems(opt) == at);
    CHECK(arc_optim_state_offset(opt, static_cast<int32_t>(tensors.size())) == -1);
    CHECK(refused(arc_optim_norm(opt, nullptr, 1.f, 1.f, nullptr, nullptr)));
    CHECK(arc_optim_destroy(opt) == ARC_OK);
  } else {
    CHECK(st == ARC_ERR_DEVICE && opt == nullptr);
  }
}

int main() {
  const float inf = INFINITY, nan = NAN;
  plan({{5, 0, 1, 0.1f, 1.f}}, ARC_STATE_F32);
  plan({{0, 0, 0, 0.f, 1.f}, {0, 1, 1, 0.f, 1.f}}, ARC_STATE_F8);
  plan({{int64_t{1} << 33, 1, 1, 0.f, 1.f}, {1, 0, 0, 0.f, 1.f}}, ARC_STATE_F8);
  uint64_t x = 12345;
  for (int round = 0; round < 50; ++round) {
    std::vector<arc_optim_tensor> t;
    for (int i = 0; i < 1 + round * 9; ++i) {
      x = x * 6364136223846793005ull + 1442695040888963407ull;
      t.push_back({static_cast<int64_t>((x >> 40) % (round % 2 ? 300 : 3000000)),
                   static_cast<int32_t>((x >> 33) % 2), static_cast<int32_t>((x >> 34) % 2), 0.1f,
                   1.f});
    }
    plan(t, round % 2);
  }
  arc_optim_tensor one{5, 0, 0, 0.f, 1.f};
  for (const arc_optim_tensor& bad :
       {arc_optim_tensor{-1, 0, 0, 0.f, 1.f}, arc_optim_tensor{(int64_t{1} << 42) + 1, 0, 0, 0.f, 1.f},
        arc_optim_tensor{5, 2, 0, 0.f, 1.f}, arc_optim_tensor{5, 0, -1, 0.f, 1.f},
        arc_optim_tensor{5, 0, 0, nan, 1.f}, arc_optim_tensor{5, 0, 0, 0.f, inf}}) {
    arc_optim_config cfg{&bad, 1, 0, 0, 0, 0};
    arc_optim* opt = reinterpret_cast<arc_optim*>(1);
    CHECK(refused(arc_optim_create(&cfg, nullptr, &opt)) && opt == nullptr);
  }
  for (const arc_optim_config& bad :
       {arc_optim_config{nullptr, 1, 0, 0, 0, 0}, arc_optim_config{&one, 0, 0, 0, 0, 0},
        arc_optim_config{&one, 1, 2, 0, 0, 0}, arc_optim_config{&one, 1, 0, 2, 0, 0},
        arc_optim_config{&one, 1, 0, 0, 1, 0}}) {
    arc_optim* opt = nullptr;
    CHECK(refused(arc_optim_create(&bad, nullptr, &opt)) && opt == nullptr);
  }
  for (const arc_tokens_config& bad :
       {arc_tokens_config{0, 1, 0, 0, 1.f, 0}, arc_tokens_config{10, 0, 0, 0, 1.f, 0},
        arc_tokens_config{10, 1, 2, 0, 1.f, 0}, arc_tokens_config{10, 1, 0, 11, 1.f, 0},
        arc_tokens_config{100, 1, 0, 33, 1.f, 0}, arc_tokens_config{10, 1, 0, 0, 0.f, 0},
        arc_tokens_config{10, 1, 0, 0, nan, 0}, arc_tokens_config{10, 1, 0, 0, 1e30f, 0},
        arc_tokens_config{10, 1, 0, 0, 1.f, 1}}) {
    arc_tokens* tok = reinterpret_cast<arc_tokens*>(1);
    CHECK(refused(arc_tokens_create(&bad, nullptr, &tok)) && tok == nullptr);
  }
  for (int i = 0; i < 3; ++i) {
    const arc_tokens_config good{50257, 16, i % 2, 5, 1.f, 0};
    arc_tokens* tok = nullptr;
    const arc_status st = arc_tokens_create(&good, nullptr, &tok);
    if (st == ARC_OK) {
      float f[4];
      CHECK(refused(arc_tokens_score(tok, 17, f, 50257, nullptr, nullptr, nullptr, f, nullptr,
                                     nullptr)));
      CHECK(refused(arc_tokens_score(tok, 1, f, 50256, nullptr, nullptr, nullptr, f, nullptr,
                                     nullptr)));
      CHECK(refused(arc_tokens_score(tok, 1, f, INT64_MAX, nullptr, nullptr, nullptr, f, nullptr,
                                     nullptr)));
      CHECK(arc_tokens_destroy(tok) == ARC_OK);
    } else {
      CHECK((st == ARC_ERR_DEVICE || st == ARC_ERR_NOMEM) && tok == nullptr);
    }
  }
  CHECK(refused(arc_tokens_create(nullptr, nullptr, nullptr)));
  CHECK(refused(arc_optim_create(nullptr, nullptr, nullptr)));
  CHECK(arc_tokens_destroy(nullptr) == ARC_OK && arc_optim_destroy(nullptr) == ARC_OK);
  if (failures) return 1;
  std::printf("ok\n");
  return 0;
}
