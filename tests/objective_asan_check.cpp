// Drives the host side of the training objectives and of the matrix optimizer
// (arc_objective.cpp, arc_muon.cpp) where it needs no device: refusals with a token
// context made by hand, the tables of many lists of matrices (every tile of every
// product once, sums whole, nothing in the workspace shared), and the launches of a
// pass followed with numbers in the place of matrices.  Built with AddressSanitizer
// on the host code; prints "ok" when every check holds.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <map>
#include <set>
#include <string>
#include <tuple>
#include <vector>

#include "arc_muon.cpp"

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
      if (++failures > 20) return;                                                         \
    }                                                                                      \
  } while (0)

static bool refused(arc_status s) { return s == ARC_ERR_INVALID && !arc::why.empty(); }

// ---------------------------------------------------------------- plans

static void check_list(const arc_muon& c, const arc::MuonGroup& g,
                       const arc::MuonGroup::Range& range, int32_t whole_of, int what) {
  const int32_t side = range.side;
  CHECK((what == 0 ? side == arc::kSplitTile : side == 32 || side == 64 || side == 128) &&
        side <= whole_of);
  std::map<std::tuple<int32_t, int32_t, int32_t>, std::vector<arc::MuonTile>> seen;
  CHECK(range.at >= 0 && range.at + range.count <= static_cast<int64_t>(c.tiles.size()));
  for (int64_t k = range.at; k < range.at + range.count; ++k) {
    const arc::MuonTile& t = c.tiles[static_cast<size_t>(k)];
    CHECK(t.matrix >= g.first && t.matrix < g.first + g.count);
    const arc::MuonMatrix& m = c.matrices[static_cast<size_t>(t.matrix)];
    CHECK(t.base == m.base && t.mp == m.mp && t.np == m.np);
    seen[{t.matrix, t.i, t.j}].push_back(t);
  }
  size_t expected = 0;
  std::set<int32_t> places;
  for (int32_t i = g.first; i < g.first + g.count; ++i) {
    const arc::MuonMatrix& m = c.matrices[static_cast<size_t>(i)];
    if (m.m == 0) continue;
    const int32_t rows = m.mp / side, cols = what == 0 || what == 3 ? m.np / side : rows;
    const int32_t lines = what == 0 ? 0 : (what == 1 ? m.np : m.mp) / arc::kPairLine;
    for (int32_t a = 0; a < rows; ++a)
      for (int32_t b = 0; b < cols; ++b) {
        if ((what == 1 || what == 2) && b > a) continue;
        ++expected;
        auto at = seen.find({i, a, b});
        CHECK(at != seen.end());
        if (at == seen.end()) continue;
        std::vector<bool> taken(static_cast<size_t>(lines));
        std::set<int32_t> parts;
        for (const arc::MuonTile& t : at->second) {
          CHECK(t.parts == static_cast<int32_t>(at->second.size()));
          CHECK(t.part >= 0 && t.part < t.parts && parts.insert(t.part).second);
          CHECK(t.place == at->second[0].place);
          CHECK(what == 0 || t.lines > 0);
          for (int32_t q = t.first; q < t.first + t.lines; ++q) {
            CHECK(q >= 0 && q < lines && !taken[static_cast<size_t>(q)]);
            taken[static_cast<size_t>(q)] = true;
          }
          if (t.parts > 1) {
            CHECK(t.place + t.part < c.parts && places.insert(t.place + t.part).second);
            CHECK(int64_t{t.place + t.part + 1} * side * side <= c.part_elems);
          }
        }
        for (const bool x : taken) CHECK(x);
      }
  }
  CHECK(expected == seen.size());
}

static void check_plan(const std::vector<arc_muon_matrix>& list) {
  const arc_muon_config cfg{list.data(), nullptr, static_cast<int32_t>(list.size()), 5, 0};
  CHECK(check_muon(&cfg) == ARC_OK);
  for (const int32_t whole_of : {64, 128}) {
    arc_muon c;
    const Times times = plan_muon(&cfg, whole_of, &c);
    CHECK(std::isfinite(times.gram + times.half + times.whole));
    CHECK(c.matrices.size() == list.size());
    int64_t state = 0, runs = 0;
    int32_t next = 0;
    for (const arc::MuonGroup& g : c.groups) {
      CHECK(g.first == next && g.count >= 1 && g.count <= arc::kMuonBatch);
      next += g.count;
      CHECK(g.first_run == runs);
      int64_t end = 0;
      for (int32_t i = g.first; i < g.first + g.count; ++i) {
        const arc::MuonMatrix& m = c.matrices[static_cast<size_t>(i)];
        const int64_t count = int64_t{m.rows} * m.cols;
        CHECK(m.state == state && m.first_run == runs);
        state += (count + 127) / 128 * 128;
        runs += m.runs;
        CHECK(int64_t{m.runs} * arc::kMuonRun >= count);
        if (count == 0) continue;
        CHECK(m.mp % whole_of == 0 && m.np % whole_of == 0 && m.mp >= m.m && m.np >= m.n);
        CHECK(m.base >= end && m.base % 256 == 0);
        // the arrays of a matrix, one after the other
        for (int32_t k = 0; k < arc::kMuonArrays; ++k) {
          const int64_t bytes = k == arc::kMuonX ? arc::pair_pitch(m.np) * m.mp
                                : k < arc::kMuonSquare ? arc::pair_pitch(m.mp) * m.np
                                                       : arc::pair_pitch(m.mp) * m.mp;
          CHECK(arc::array_at(m.base, m.mp, m.np, k + 1) -
                    arc::array_at(m.base, m.mp, m.np, k) == bytes);
        }
        end = arc::array_at(m.base, m.mp, m.np, arc::kMuonArrays);
        CHECK(end <= c.workspace_bytes);
      }
      CHECK(g.runs == runs - g.first_run);
      check_list(c, g, g.split, whole_of, 0);
      check_list(c, g, g.gram, whole_of, 1);
      check_list(c, g, g.half, whole_of, 2);
      check_list(c, g, g.whole, whole_of, 3);
    }
    CHECK(next == static_cast<int32_t>(list.size()) && c.state_elems == state);
    CHECK(static_cast<int64_t>(c.run_matrix.size()) == runs);
  }
  const std::vector<int64_t> order = launch_order(1000 + 37 * static_cast<int64_t>(list.size()));
  std::set<int64_t> all(order.begin(), order.end());
  CHECK(all.size() == order.size() && *all.begin() == 0 &&
        *all.rbegin() == static_cast<int64_t>(order.size()) - 1);
}

// ---------------------------------------------------------------- launches

// A pass with a number s in the place of X, as a 1 x 1 matrix: what the launches make
// of it, in the units that the kernels hold it in.
static void check_sequence(const std::vector<float>& q, int32_t together) {
  const std::vector<double> bounds = polynomial_bounds(q);
  CHECK(!bounds.empty());
  const std::vector<arc::MuonLaunch> launches = sequence(q, bounds, together);
  for (double s = 0.0; s <= 1.0; s += 1.0 / 64) {
    double held[arc::kMuonArrays] = {};
    held[arc::kMuonX] = held[arc::kMuonXt] = s * arc::kPairScale;
    double got = NAN, want = s;
    for (size_t k = 0; k < q.size(); k += 3)
      want = want * (q[k] + q[k + 1] * want * want + q[k + 2] * want * want * want * want);
    for (const arc::MuonLaunch& l : launches) {
      const arc::MuonProduct& p = l.product;
      double x = held[p.left] * held[p.right] * p.scale;
      if (l.kind == arc::kMuonStep) {
        CHECK(p.left == p.right);
        x = p.c * x + p.b * held[p.left] + p.a * arc::kPairScale;
      }
      if (l.kind == arc::kMuonLast) {
        got = x;
        continue;
      }
      CHECK(std::fabs(x) < 65504.0);  // binary16's end
      // nothing is written that the same launch still reads
      CHECK(p.out != p.left && p.out != p.right && p.turned != p.left && p.turned != p.right);
      if (l.kind != arc::kMuonApply) CHECK(p.out == p.turned);
      held[p.out] = held[p.turned] = x;
    }
    CHECK(std::fabs(got - want) <= 1e-5 * (1.0 + std::fabs(want)));
  }
}

// ---------------------------------------------------------------- objectives

static void check_objectives() {
  arc_tokens c;
  c.vocab = 10;
  c.max_rows = 8;
  float f[100];
  int64_t y[20] = {};
  const arc_policy_config p{0.2f, 0.2f, 0.f, 0.f, 0.f, 1.f};
  const arc_preference_config q{0, 0, 0.1f, 0.f, 0.f, 1.f};
  const auto policy = [&](const arc_policy_config* cfg, int64_t rows, const void* x, int64_t stride,
                          const int64_t* t, const float* ref, const float* A, float* totals,
                          void* grad, int64_t to) {
    return arc_tokens_policy(&c, cfg, rows, x, stride, t, nullptr, ref, A, nullptr, nullptr,
                             nullptr, nullptr, nullptr, nullptr, nullptr, totals, grad, to);
  };
  CHECK(refused(policy(nullptr, 1, f, 10, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 9, f, 10, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, -1, f, 10, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, 9, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, INT64_MAX, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, nullptr, 10, y, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, 10, nullptr, nullptr, f, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, nullptr, f + 50, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 20, nullptr, f + 60, 10)));
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 20, f + 50, nullptr, 10)));
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 20, f + 50, f + 60, 9)));
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 20, f + 5, f + 60, 10)));   // totals on logits
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 20, f + 62, f + 60, 10)));  // and on the gradient
  CHECK(refused(policy(&p, 1, f, 10, y, nullptr, f + 65, f + 50, f + 60, 10)));  // gradient on inputs
  for (const arc_policy_config& bad :
       {arc_policy_config{-1.f, 0.f, 0.f, 0.f, 0.f, 1.f}, {NAN, 0.f, 0.f, 0.f, 0.f, 1.f},
        {0.f, NAN, 0.f, 0.f, 0.f, 1.f}, {0.f, 0.f, .5f, 0.f, 0.f, 1.f},
        {0.f, 0.f, 0.f, 1.f, 0.f, 1.f}, {0.f, 0.f, 0.f, -1.f, 0.f, 1.f},
        {0.f, 0.f, 0.f, 0.f, INFINITY, 1.f}, {0.f, 0.f, 0.f, 0.f, 0.f, NAN}})
    CHECK(refused(policy(&bad, 1, f, 10, y, nullptr, f + 20, f + 50, f + 60, 10)));
  const auto pairs = [&](const arc_preference_config* cfg, int64_t rows, const float* lp,
                         const int64_t* t, int64_t n, const int64_t* o, float* loss, float* totals,
                         float* d) {
    return arc_tokens_preference_terms(&c, cfg, rows, lp, t, n, o, nullptr, nullptr, loss, nullptr,
                                       totals, d);
  };
  CHECK(refused(pairs(nullptr, 4, f, y, 1, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 9, f, y, 1, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, nullptr, y, 1, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, nullptr, 1, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, 1, nullptr, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, -1, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, int64_t{1} << 31, y + 10, f + 40, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, 1, y + 10, f + 40, nullptr, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, 1, y + 10, f + 2, f + 50, f + 60)));
  CHECK(refused(pairs(&q, 4, f, y, 1, y + 10, f + 61, f + 50, f + 60)));
  for (const arc_preference_config& bad :
       {arc_preference_config{3, 0, .1f, 0.f, 0.f, 1.f}, {0, 2, .1f, 0.f, 0.f, 1.f},
        {0, 0, 0.f, 0.f, 0.f, 1.f}, {0, 0, .1f, NAN, 0.f, 1.f}, {0, 0, .1f, 0.f, .6f, 1.f},
        {1, 0, .1f, 0.f, .1f, 1.f}, {0, 0, .1f, 0.f, 0.f, INFINITY}})
    CHECK(refused(pairs(&bad, 4, f, y, 1, y + 10, f + 40, f + 50, f + 60)));
}

static void check_all() {
  uint64_t x = 99;
  const auto draw = [&](uint64_t n) {
    x = x * 6364136223846793005ull + 1442695040888963407ull;
    return static_cast<int64_t>((x >> 33) % n);
  };
  const auto one = [](int64_t r, int64_t c) { return arc_muon_matrix{r, c, 0, 1, 0.1f, 1.f}; };
  check_plan({one(1, 1)});
  check_plan({one(0, 5), one(5, 0)});
  check_plan({one(257, 1001)});
  check_plan({one(4096, 4096)});
  check_plan({one(64, 4608), one(512, 4608), one(512, 4608), one(3, 0), one(64, 27)});
  check_plan(std::vector<arc_muon_matrix>(400, one(33, 65)));
  check_plan(std::vector<arc_muon_matrix>(9, one(4096, 11008)));  // more than one group
  check_plan({one(16, 1 << 21), one(1 << 21, 1)});
  for (int round = 0; round < 40; ++round) {
    std::vector<arc_muon_matrix> list;
    for (int64_t i = 0, n = 1 + draw(60); i < n; ++i)
      list.push_back(one(draw(round % 2 ? 200 : 1500), draw(round % 3 ? 200 : 3000)));
    check_plan(list);
  }
  const std::vector<float> quintic = {3.4445f, -4.7750f, 2.0315f};
  for (int steps = 1; steps <= 9; ++steps) {
    std::vector<float> q, cubic, mixed;
    for (int k = 0; k < steps; ++k) {
      q.insert(q.end(), quintic.begin(), quintic.end());
      for (const float v : {1.5f, -0.5f, 0.f}) cubic.push_back(v);
      for (const float v : k % 2 ? std::vector<float>{1.875f, -1.25f, 0.375f} : quintic)
        mixed.push_back(v);
    }
    for (int32_t together = 1; together <= 3; ++together) {
      check_sequence(q, together);
      check_sequence(cubic, together);
      check_sequence(mixed, together);
      check_sequence({7.7f, -20.f, 14.f}, together);
    }
  }
  // the largest values of polynomials, against a fine grid
  for (int round = 0; round < 200; ++round) {
    const double a = static_cast<double>(draw(2000)) / 100 - 10,
                 b = static_cast<double>(draw(2000)) / 100 - 10,
                 c = round % 4 ? static_cast<double>(draw(2000)) / 100 - 10 : 0.0;
    for (const bool odd : {false, true}) {
      double most = 0.0;
      for (int k = 0; k <= 20000; ++k) {
        const double s = 1.3 * k / 20000, v = a + b * s + c * s * s;
        most = std::fmax(most, std::fabs(odd ? std::sqrt(s) * v : v));
      }
      const double found = largest(a, b, c, 1.3, odd);
      CHECK(found >= most - 1e-12 && found <= most + 1e-4 * (1 + most));
    }
  }
  check_objectives();
  for (const std::vector<arc_muon_matrix>& list :
       {std::vector<arc_muon_matrix>{one(5, 7)}, std::vector<arc_muon_matrix>(30, one(300, 200))}) {
    const arc_muon_config cfg{list.data(), nullptr, static_cast<int32_t>(list.size()), 5, 0};
    arc_muon* opt = nullptr;
    const arc_status st = arc_muon_create(&cfg, nullptr, &opt);
    if (st == ARC_OK) {
      CHECK(refused(arc_muon_orthogonalize(opt, nullptr, nullptr)));
      CHECK(arc_muon_destroy(opt) == ARC_OK);
    } else {
      CHECK((st == ARC_ERR_DEVICE || st == ARC_ERR_NOMEM) && opt == nullptr);
    }
  }
}

int main() {
  check_all();
  if (failures) return 1;
  std::printf("ok\n");
  return 0;
}
