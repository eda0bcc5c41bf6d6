// Host side of the matrix optimizer: argument checks, the plan of a context (its
// matrices in groups that share a workspace, and each group's tiles) and the
// enqueue on its stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>
#include <utility>
#include <vector>

#include "arc_context.h"
#include "arc_muon.h"
#include "arc_train_host.h"

namespace arc {

// Matrices that go through the launches together.
struct MuonGroup {
  int32_t first = 0, count = 0;
  int64_t first_run = 0, runs = 0;
  struct Range {  // their tiles in the context's list, and those tiles' sides
    int64_t at = 0, count = 0;
    int32_t side = kSplitTile;
    int64_t counts = 0;  // where their counts of parts begin
  };
  Range split, gram, half, whole;
};

struct MuonLaunch {
  MuonKind kind;
  MuonProduct product;
};

}  // namespace arc

struct arc_muon {
  std::vector<arc::MuonMatrix> matrices;
  std::vector<arc::MuonGroup> groups;
  std::vector<arc::MuonTile> tiles;
  std::vector<int32_t> run_matrix;
  // The products of a pass, for each way to make it: step by step, or the steps'
  // polynomials multiplied first.
  std::vector<arc::MuonLaunch> plain, grouped;
  bool group = false;     // the second one takes less time
  bool any_f32 = false;   // a parameter is binary32
  int64_t state_elems = 0, workspace_bytes = 0;
  int64_t parts = 0, part_elems = 0;  // most of one launch
  int64_t counts = 0;                 // of all ranges
  hipStream_t stream = nullptr;
  int device = 0;
  arc::MuonMatrix* matrices_dev = nullptr;
  arc::MuonTile* tiles_dev = nullptr;
  int32_t* run_matrix_dev = nullptr;
  double* sums_dev = nullptr;
  char* workspace = nullptr;
  float* parts_dev = nullptr;
  uint32_t* arrived_dev = nullptr;

  void release() {
    (void)hipStreamSynchronize(stream);
    for (void* p : {static_cast<void*>(matrices_dev), static_cast<void*>(tiles_dev),
                    static_cast<void*>(run_matrix_dev), static_cast<void*>(sums_dev),
                    static_cast<void*>(workspace),
                    static_cast<void*>(parts_dev), static_cast<void*>(arrived_dev)})
      if (p) (void)hipFree(p);
  }
};

namespace {

using arc::device_copy;
using arc::fail;
using arc::finite;
using arc::OnDevice;
using arc::overlap;

constexpr int64_t kMaxShort = int64_t{1} << 15, kMaxLong = int64_t{1} << 21;
constexpr int64_t kMaxMatrix = int64_t{1} << 34, kMaxElements = int64_t{1} << 42;
constexpr int32_t kMaxSteps = 64;
constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
// What a group's pairs may take: enough matrices to fill the card many times over.
constexpr int64_t kGroupBytes = int64_t{4} << 30;
// Steps whose polynomials are multiplied before X is: then X X' and P X, the products
// that grow with the longer side, are made once for a run of steps and not in each, for
// three more products of the shorter side with each step that joins one (five steps of m x n
// numbers: 15 m^2 n + 5 m^3 multiplications step by step, 9 m^2 n + 11 m^3 in runs of two,
// one and two, 6 m^2 n + 14 m^3 in runs of two and three).
//
// An error of A = X X' is taken from step to step within a run, and in the directions of
// small singular values it grows as A does there, with the square of the polynomial (12
// times for the usual one), where step by step A is made anew from X.  What O is off by, of
// its norm, and how many times step by step or binary32 products, the larger: matrices of
// 4 to 640 rows, one to half of whose singular values are the strong ones, runs of three and
// two 4e-5 to 2e-4, up to 90 times; of two and three 7e-5, 14 times; of two, one and two
// 1e-5, 1.7 times (step by step 1e-5 too, of matrices whose others are 0.003).  So runs of
// two where a parameter is binary32, and runs of two and three where all are bfloat16,
// whose rounding is off by 1.7e-3.  O itself in binary32 is made step by step.
constexpr int32_t kTogetherF32 = 2, kTogetherBf16 = 3;
// What errors may grow in a run, and in a last run of three, before which as small singular
// values have grown as much.
constexpr double kRunGrows = 12.0, kLastRunGrows = 144.0;

int64_t up_to(int64_t v, int64_t of) { return (v + of - 1) / of * of; }

// The largest |a + b s + c s^2| for s in [0, top].
double largest(double a, double b, double c, double top, bool odd) {
  // odd: of x (a + b x^2 + c x^4), x = sqrt(s), whose derivative is a + 3 b s + 5 c s^2
  const auto at = [&](double s) {
    const double v = a + b * s + c * s * s;
    return std::fabs(odd ? std::sqrt(s) * v : v);
  };
  double most = std::max(at(0.0), at(top));
  const double q = odd ? 5.0 * c : 0.0, h = odd ? 3.0 * b : 2.0 * c, k = odd ? a : b;
  const auto turn = [&](double s) {
    if (s > 0.0 && s < top) most = std::max(most, at(s));
  };
  if (q != 0.0) {
    const double d = h * h - 4.0 * q * k;
    if (d >= 0.0) {
      turn((-h + std::sqrt(d)) / (2.0 * q));
      turn((-h - std::sqrt(d)) / (2.0 * q));
    }
  } else if (h != 0.0) {
    turn(-k / h);
  }
  return most;
}

// The largest entries of each step's polynomial; empty where an entry of X, X X' or
// of one of those leaves the pairs' range.  Entries are at most the largest singular
// value, which starts at 1.
std::vector<double> polynomial_bounds(const std::vector<float>& coefficients) {
  constexpr double kMost = 7.75;  // 2^13 times it is below binary16's end
  double top = 1.001;             // rounding
  std::vector<double> bounds;
  for (size_t k = 0; k < coefficients.size(); k += 3) {
    const double a = coefficients[k], b = coefficients[k + 1], c = coefficients[k + 2];
    bounds.push_back(largest(a, b, c, top * top, false));
    if (top * top > kMost || bounds.back() > kMost) return {};
    top = largest(a, b, c, top * top, true) * 1.001;
  }
  return bounds;  // the last X is not held in pairs
}

// How many steps each run takes, at most `together` (1 to 3).  Of an odd number in pairs the
// lone one comes second (in a model of the roundings, of five steps at most 3.3 times what
// step by step or binary32 is off by; with it last 3.5, and first 7.3).
std::vector<int32_t> runs_of(const std::vector<double>& bounds, int32_t together) {
  std::vector<int32_t> runs;
  const size_t steps = bounds.size();
  const auto grown = [&](size_t from, size_t to) {  // what errors of A grow in these steps
    double most = 1.0;
    for (size_t k = from; k < to; ++k) most *= bounds[k] * bounds[k];
    return most;
  };
  size_t end = steps;
  if (together > 2 && steps > 4 && grown(steps - 3, steps - 1) <= kLastRunGrows &&
      grown(steps - 3, steps - 1) <= grown(0, steps - 3))
    end -= 3;
  for (size_t k = 0; k < end;) {
    const bool alone = k + 1 == end || (end % 2 == 1 && runs.size() == 1);
    const bool pair = together > 1 && !alone && grown(k, k + 1) <= kRunGrows;
    runs.push_back(pair ? 2 : 1);
    k += pair ? 2 : 1;
  }
  if (end < steps) runs.push_back(3);
  return runs;
}

// The launches of a pass in which runs of at most `together` steps have their polynomials
// multiplied before X is.
std::vector<arc::MuonLaunch> sequence(const std::vector<float>& coefficients,
                                      const std::vector<double>& bounds, int32_t together) {
  using namespace arc;
  constexpr float kUnit = 1.f / kPairScale;
  std::vector<MuonLaunch> out;
  const auto steps = static_cast<int32_t>(bounds.size());
  int32_t xt = kMuonXt, k = 0;
  for (const int32_t count : runs_of(bounds, together)) {
    out.push_back({kMuonGram, {kMuonX, kMuonX, kMuonSquare, kMuonSquare, kUnit, 0, 0, 0}});
    int32_t all = kMuonPoly;
    float all_scale = kPairScale;
    double bound = 1.0;
    for (int32_t q = 0; q < count; ++q, ++k) {
      const float a = coefficients[3 * k], b = coefficients[3 * k + 1],
                  c = coefficients[3 * k + 2];
      bound *= bounds[k];
      out.push_back({kMuonStep, {kMuonSquare, kMuonSquare, kMuonPoly, kMuonPoly, kUnit, a, b, c}});
      if (count > 1 && q == 0) {
        out.back().product.out = out.back().product.turned = kMuonAll;
        all = kMuonAll;
      }
      const int32_t poly = out.back().product.out;
      if (q > 0) {
        float scale = kPairScale;
        while (scale * bound > 6e4) scale *= 0.5f;
        const int32_t next = all == kMuonAll ? kMuonAll2 : kMuonAll;
        // sums are in units of 1 / (kPairScale all_scale)
        out.push_back({kMuonHalf,
                       {poly, all, next, next, scale / (kPairScale * all_scale), 0, 0, 0}});
        all = next;
        all_scale = scale;
      }
      if (q + 1 < count) {
        out.push_back({kMuonHalf, {poly, kMuonSquare, kMuonWay, kMuonWay, kUnit, 0, 0, 0}});
        out.push_back({kMuonHalf, {poly, kMuonWay, kMuonSquare, kMuonSquare, kUnit, 0, 0, 0}});
      }
    }
    const int32_t next = xt == kMuonXt ? kMuonXt2 : kMuonXt;
    if (k < steps)
      out.push_back({kMuonApply, {all, xt, kMuonX, next, 1.f / all_scale, 0, 0, 0}});
    else
      out.push_back({kMuonLast, {all, xt, kMuonX, next, 1.f / (kPairScale * all_scale), 0, 0, 0}});
    xt = next;
  }
  return out;
}

arc_status check_muon(const arc_muon_config* cfg) {
  if (cfg == nullptr) return fail(ARC_ERR_INVALID, "cfg is NULL");
  if (cfg->matrices == nullptr) return fail(ARC_ERR_INVALID, "matrices is NULL");
  if (cfg->num_matrices < 1 || cfg->num_matrices > (1 << 20))
    return fail(ARC_ERR_INVALID, "num_matrices must be in 1..2^20");
  if (cfg->steps < 1 || cfg->steps > kMaxSteps)
    return fail(ARC_ERR_INVALID, "steps must be in 1..64");
  if (cfg->reserved != 0) return fail(ARC_ERR_INVALID, "reserved must be 0");
  if (cfg->coefficients != nullptr)
    for (int32_t k = 0; k < 3 * cfg->steps; ++k)
      if (!finite(cfg->coefficients[k]))
        return fail(ARC_ERR_INVALID, "coefficients must be finite");
  int64_t left = kMaxElements;
  for (int32_t i = 0; i < cfg->num_matrices; ++i) {
    const arc_muon_matrix& t = cfg->matrices[i];
    if (t.rows < 0 || t.cols < 0 || std::min(t.rows, t.cols) > kMaxShort ||
        std::max(t.rows, t.cols) > kMaxLong || t.rows * t.cols > kMaxMatrix ||
        t.rows * t.cols > left)
      return fail(ARC_ERR_INVALID,
                  "sides must be >= 0, the shorter one 2^15 at most and the longer one 2^21, "
                  "2^34 elements a matrix and 2^42 in all");
    left -= t.rows * t.cols;
    for (int32_t dt : {t.param_dtype, t.grad_dtype})
      if (dt != ARC_DTYPE_F32 && dt != ARC_DTYPE_BF16)
        return fail(ARC_ERR_INVALID, "dtypes must be ARC_DTYPE_F32 or ARC_DTYPE_BF16");
    if (!(t.weight_decay >= 0.f) || !finite(t.weight_decay) || !finite(t.lr_scale))
      return fail(ARC_ERR_INVALID, "weight_decay must be >= 0 and finite, lr_scale finite");
  }
  return ARC_OK;
}

// Which element of a list each workgroup takes: they go to the eight XCDs in turn,
// and runs of neighbours to the same one, whose L2 then holds what they share: runs of
// 32, and shorter ones towards the end, so that every XCD gets as many.
std::vector<int64_t> launch_order(int64_t count) {
  constexpr int64_t kXcds = 8;
  std::vector<int64_t> order(static_cast<size_t>(count));
  int64_t from = 0;
  for (int64_t run = 32; run > 0; run /= 2)
    for (; count - from >= kXcds * run; from += kXcds * run)
      for (int64_t b = 0; b < kXcds * run; ++b)
        order[static_cast<size_t>(from + b)] = from + b % kXcds * run + b / kXcds;
  for (; from < count; ++from) order[static_cast<size_t>(from)] = from;
  return order;
}

// Tiles of a grid of rows x cols (only those on and below the diagonal), in blocks
// of 4 x 8 neighbours.
template <typename Add>
void each_tile(int32_t rows, int32_t cols, bool half, const Add& add) {
  for (int32_t i0 = 0; i0 < rows; i0 += 4)
    for (int32_t j0 = 0; j0 < cols; j0 += 8)
      for (int32_t i = i0; i < std::min(rows, i0 + 4); ++i)
        for (int32_t j = j0; j < std::min(cols, j0 + 8); ++j)
          if (!half || j <= i) add(i, j);
}

// What a launch is expected to take, in us, by which tiles' sums are split and the
// tiles' side and the way through the steps are chosen.  Measured: a line of a tile's
// sum on a compute unit that is full, and in a workgroup that has it for itself; a
// result written; a part written (and read once more by the workgroup that adds them);
// a launch.  us with tiles of 32, 64 and 128, the better of step by step and in runs:
// 24 vectors and small matrices 82, 81 and 138, 257 x 1001 100, 127 and 259, a ResNet-18's
// convolutions 485, 411 and 502, three layers of width 384 280, 243 and 324, of width 576
// 717, 539 and 681, 48 matrices of width 640 4023, 2772 and 2376, a 4096 x 4096 in bfloat16
// 7752, 4437 and 3524.  Step by step and in runs: the convolutions 495 and 411, width 576
// 633 and 539, width 640 2911 and 2376, 4096 x 4096 3524 and 3713.  Each product has a side
// of its own: the convolutions then take 398.  Of 51 drawn cases (in runs of three and two)
// what is chosen was within 3% of the best of the six in 48, and within 16% in all.  Split
// sums: X X' of a ResNet-18's convolutions (sums of 4608 in few tiles) 40 us against 103.
// The plan takes the host 1.4 ms for 257 x 1001, 15 for a 4096 x 4096, 3 to 5 for the
// convolutions and the 48 matrices, 91 for 224 of an 8-billion-weight model.
struct Rates {
  int32_t side;
  double line, alone, result, part;
};
constexpr Rates kRates[] = {{128, 0.66, 0.90, 6.7, 3.2},
                            {64, 0.24, 0.32, 1.7, 0.8},
                            {32, 0.10, 0.16, 0.5, 0.3}};
constexpr double kLaunch = 5.0;
constexpr int64_t kUnits = 256;
// Tiles of 128, most of them full, that fill the card so often that smaller ones are not
// looked at.
constexpr int64_t kPlenty = 16 * 2 * kUnits;

// The parts of each of `lines`, which descend, from number `from` on `parts` of them;
// and the time that the busiest compute unit then needs.
double launch_time(const Rates& r, const std::vector<int32_t>& lines, size_t from, int32_t parts) {
  std::vector<double> queue;  // a heap, the least busy first
  queue.assign(static_cast<size_t>(kUnits), 0.0);
  double longest = 0.0;
  const auto add = [&](double time, double least) {
    std::pop_heap(queue.begin(), queue.end(), std::greater<>());
    queue.back() += time;
    std::push_heap(queue.begin(), queue.end(), std::greater<>());
    longest = std::max(longest, least);
  };
  for (size_t k = 0; k < lines.size(); ++k) {
    const int32_t p = k < from ? 1 : std::min(parts, lines[k]);
    const int32_t each = (lines[k] + p - 1) / p;
    const double end = p == 1 ? r.result : r.part;
    for (int32_t q = 0; q < p; ++q) add(each * r.line + end, each * r.alone + end);
    if (p > 1) add(r.result + p * r.part, each * r.alone + r.result + (p + 1) * r.part);
  }
  return kLaunch + std::max(longest, *std::max_element(queue.begin(), queue.end()));
}

// Turns a product's tiles (their sums `lines` long, descending) into workgroups, and
// adds the time that they are expected to take.  Sums are split where tiles are few,
// or where the last ones would leave most of the card idle.
double plan_product(const Rates& r, std::vector<arc::MuonTile>* tiles, int64_t* parts_of_launch) {
  constexpr size_t kMany = 4096;  // a split gains little then
  double work = 0.0;
  std::vector<int32_t> lines;
  for (const arc::MuonTile& t : *tiles) {
    lines.push_back(t.lines);
    work += t.lines * r.line + r.result;
  }
  if (tiles->size() > kMany) return kLaunch + work / kUnits;
  double best = launch_time(r, lines, lines.size(), 1);
  if (best < 1.1 * (kLaunch + work / kUnits)) return best;  // nearly even as it is
  size_t from = lines.size();
  int32_t parts = 1;
  const size_t rounds = lines.size() / kUnits * kUnits;
  for (const int32_t p : {2, 3, 4, 6, 8, 12, 16})
    for (const size_t f : {size_t{0}, rounds}) {
      if (f == lines.size()) continue;
      const double t = launch_time(r, lines, f, p);
      if (t < 0.95 * best) best = t, from = f, parts = p;
    }
  std::vector<arc::MuonTile> out;
  int32_t place = 0;
  for (size_t k = 0; k < tiles->size(); ++k) {
    arc::MuonTile t = (*tiles)[k];
    const int32_t p = k < from ? 1 : std::min(parts, t.lines);
    const int32_t each = (t.lines + p - 1) / p, all = t.lines;
    t.parts = (all + each - 1) / each;
    t.place = place;
    if (t.parts > 1) place += t.parts;
    for (t.part = 0; t.part < t.parts; ++t.part) {
      t.first = t.part * each;
      t.lines = std::min(each, all - t.first);
      out.push_back(t);
    }
  }
  *parts_of_launch = std::max<int64_t>(*parts_of_launch, place);
  tiles->swap(out);
  return best;
}

// What the products of a context's matrices are expected to take, once each.
struct Times {
  double gram = 0.0, half = 0.0, whole = 0.0;
  double of(const std::vector<arc::MuonLaunch>& launches) const {
    double t = 0.0;
    for (const arc::MuonLaunch& l : launches)
      t += l.kind == arc::kMuonGram ? gram
           : l.kind == arc::kMuonStep || l.kind == arc::kMuonHalf ? half
                                                                  : whole;
    return t;
  }
};

// The tables of a checked configuration whose matrices' sides are rounded up to
// multiples of `whole_of` (may throw std::bad_alloc).
Times plan_muon(const arc_muon_config* cfg, int32_t whole_of, arc_muon* c) {
  Times times;
  arc::MuonGroup g;
  int64_t bytes = 0, runs = 0;
  // A product's tiles of a side: of m x n or m x m (half of them) results.
  const auto tiles_of = [&](int32_t side, bool whole, bool long_sum) {
    std::vector<arc::MuonTile> list;
    for (int32_t i = g.first; i < g.first + g.count; ++i) {
      const arc::MuonMatrix& t = c->matrices[static_cast<size_t>(i)];
      if (t.m == 0) continue;
      const int32_t lines = (long_sum ? t.np : t.mp) / arc::kPairLine;
      each_tile(t.mp / side, (whole ? t.np : t.mp) / side, !whole, [&](int32_t a, int32_t b) {
        list.push_back({i, a, b, 0, lines, 0, 1, 0, t.base, t.mp, t.np});
      });
    }
    return list;
  };
  const auto take = [&](const std::vector<arc::MuonTile>& from, arc::MuonGroup::Range* range) {
    range->at = static_cast<int64_t>(c->tiles.size());
    range->count = static_cast<int64_t>(from.size());
    for (const int64_t k : launch_order(range->count))
      c->tiles.push_back(from[static_cast<size_t>(k)]);
  };
  // The tiles that are expected to take the least time.
  const auto product = [&](bool whole, bool long_sum, arc::MuonGroup::Range* range) {
    std::vector<arc::MuonTile> best;
    double least = INFINITY;
    int64_t parts = 0;
    for (const Rates& r : kRates) {
      if (r.side > whole_of) continue;
      std::vector<arc::MuonTile> tiles = tiles_of(r.side, whole, long_sum);
      const auto count = static_cast<int64_t>(tiles.size());
      // the longest sums first, so that short ones fill the end
      std::stable_sort(tiles.begin(), tiles.end(),
                       [](const arc::MuonTile& x, const arc::MuonTile& y) {
                         return x.lines > y.lines;
                       });
      int64_t places = 0;
      const double t = plan_product(r, &tiles, &places);
      if (t < least) {
        least = t;
        parts = places;
        range->side = r.side;
        best.swap(tiles);
      }
      if (count > kPlenty) break;
    }
    // (A count is of the same number of parts in every launch, and goes round at it.)
    range->counts = c->counts;
    c->counts += parts;
    c->parts = std::max(c->parts, parts);
    c->part_elems = std::max(c->part_elems, parts * range->side * range->side);
    take(best, range);
    return least;
  };
  const auto finish = [&] {
    if (g.count == 0) return;
    std::vector<arc::MuonTile> split = tiles_of(arc::kSplitTile, true, false);
    for (arc::MuonTile& t : split) t.lines = 0;
    take(split, &g.split);
    times.gram += product(false, true, &g.gram);
    times.half += product(false, false, &g.half);
    times.whole += product(true, false, &g.whole);
    g.runs = runs - g.first_run;
    c->groups.push_back(g);
    c->workspace_bytes = std::max(c->workspace_bytes, bytes);
  };
  for (int32_t i = 0; i < cfg->num_matrices; ++i) {
    const arc_muon_matrix& in = cfg->matrices[i];
    arc::MuonMatrix t{};
    const int64_t count = in.rows * in.cols;
    t.rows = static_cast<int32_t>(in.rows);
    t.cols = static_cast<int32_t>(in.cols);
    t.tall = in.rows > in.cols;
    t.m = std::min(t.rows, t.cols);
    t.n = std::max(t.rows, t.cols);
    t.mp = static_cast<int32_t>(up_to(t.m, whole_of));
    t.np = static_cast<int32_t>(count > 0 ? up_to(t.n, whole_of) : 0);
    t.param_bf16 = in.param_dtype == ARC_DTYPE_BF16;
    t.grad_bf16 = in.grad_dtype == ARC_DTYPE_BF16;
    t.weight_decay = in.weight_decay;
    t.lr_scale = in.lr_scale;
    t.state = c->state_elems;
    c->state_elems += up_to(count, ARC_STATE_BLOCK);
    const int64_t need =
        count > 0 ? arc::array_at(0, t.mp, t.np, arc::kMuonArrays) : 0;
    if (g.count == arc::kMuonBatch || (g.count > 0 && bytes + need > kGroupBytes)) {
      finish();
      g = arc::MuonGroup{};
      g.first = i;
      g.first_run = runs;
      bytes = 0;
    }
    ++g.count;
    t.first_run = runs;
    t.runs = static_cast<int32_t>((count + arc::kMuonRun - 1) / arc::kMuonRun);
    runs += t.runs;
    c->run_matrix.insert(c->run_matrix.end(), static_cast<size_t>(t.runs), i);
    t.base = bytes;
    bytes += need;
    if (count > 0 && !t.param_bf16) c->any_f32 = true;
    c->matrices.push_back(t);
  }
  finish();
  return times;
}

// The plan, and the way to go through the steps, whose products are expected to take
// the least time.
arc_muon plan_best(const arc_muon_config* cfg, const std::vector<float>& coefficients,
                   const std::vector<double>& bounds) {
  const auto plain = sequence(coefficients, bounds, 1);
  bool any_f32 = false;
  for (int32_t i = 0; i < cfg->num_matrices; ++i)
    any_f32 = any_f32 || cfg->matrices[i].param_dtype == ARC_DTYPE_F32;
  const auto grouped = sequence(coefficients, bounds, any_f32 ? kTogetherF32 : kTogetherBf16);
  arc_muon best;
  double least = INFINITY;
  int64_t tiles = 0, full = 0;  // of 128
  for (int32_t i = 0; i < cfg->num_matrices; ++i) {
    const arc_muon_matrix& t = cfg->matrices[i];
    tiles += up_to(t.rows, 128) / 128 * (up_to(t.cols, 128) / 128);
    full += t.rows * t.cols / (128 * 128);
  }
  const bool plenty = full > kPlenty && full > tiles / 4 * 3;
  for (const int32_t whole_of : {128, arc::kSplitTile}) {
    if (whole_of < 128 && plenty) continue;
    arc_muon c;
    const Times times = plan_muon(cfg, whole_of, &c);
    const double one = times.of(plain), other = times.of(grouped);
    c.group = other < 0.97 * one;
    if (std::min(one, other) < least) {
      least = std::min(one, other);
      best = std::move(c);
    }
  }
  best.plain = plain;
  best.grouped = grouped;
  return best;
}

arc_status check_pointers(const arc_muon* c, const void* const* p, const char* what) {
  if (p == nullptr) return fail(ARC_ERR_INVALID, std::string(what) + " is NULL");
  for (size_t i = 0; i < c->matrices.size(); ++i)
    if (p[i] == nullptr && c->matrices[i].m > 0)
      return fail(ARC_ERR_INVALID, std::string(what) + " holds a NULL");
  return ARC_OK;
}

// One pass over all groups.
arc_status enqueue(const arc_muon* c, arc::MuonArgs a, void* const* params,
                   const void* const* grads, void* const* copies) {
  a.matrices = c->matrices_dev;
  a.workspace = c->workspace;
  a.sums = c->sums_dev;
  a.parts = c->parts_dev;
  const OnDevice here(c->device);
  const auto& launches = c->group && (a.update || !c->any_f32) ? c->grouped : c->plain;
  for (const arc::MuonGroup& g : c->groups) {
    if (g.split.count == 0) continue;
    a.first = g.first;
    arc::MuonPointers p;
    for (int32_t i = 0; i < g.count; ++i) {
      p.grad[i] = grads[g.first + i];
      p.param[i] = params[g.first + i];
      p.copy[i] = copies ? static_cast<uint16_t*>(copies[g.first + i]) : nullptr;
    }
    ARC_HIP(arc::launch_muon_momentum(a, p, c->run_matrix_dev, g.first_run, g.runs, c->stream),
            "momentum launch");
    ARC_HIP(arc::launch_muon_split(a, p, c->tiles_dev + g.split.at, g.split.count, c->stream),
            "split launch");
    for (const arc::MuonLaunch& l : launches) {
      const auto& range = l.kind == arc::kMuonGram ? g.gram
                          : l.kind == arc::kMuonStep || l.kind == arc::kMuonHalf ? g.half
                                                                                 : g.whole;
      a.arrived = c->arrived_dev + range.counts;
      ARC_HIP(arc::launch_muon_product(l.kind, range.side, a, p, l.product, c->tiles_dev + range.at,
                                       range.count, c->stream),
              "product launch");
    }
  }
  return ARC_OK;
}

}  // namespace

extern "C" {

arc_status arc_muon_create(const arc_muon_config* cfg, void* hip_stream, arc_muon** out) {
  if (out == nullptr) return fail(ARC_ERR_INVALID, "out is NULL");
  *out = nullptr;
  arc_status st = check_muon(cfg);
  if (st != ARC_OK) return st;
  arc_muon* c = nullptr;
  try {
    std::vector<float> coefficients;
    for (int32_t k = 0; k < 3 * cfg->steps; ++k)
      coefficients.push_back(cfg->coefficients ? cfg->coefficients[k] : kQuintic[k % 3]);
    const std::vector<double> bounds = polynomial_bounds(coefficients);
    if (bounds.empty())
      return fail(ARC_ERR_INVALID,
                  "coefficients: singular values in 0..1 have to stay below 2.7, and the "
                  "polynomials below 7.7");
    c = new arc_muon(plan_best(cfg, coefficients, bounds));
  } catch (const std::exception&) {
    delete c;
    return fail(ARC_ERR_NOMEM, "host allocation failed");
  }
  c->stream = static_cast<hipStream_t>(hip_stream);
  const auto bail = [&](arc_status s) {
    c->release();
    delete c;
    return s;
  };
  hipError_t e = hipGetDevice(&c->device);
  if (e != hipSuccess) return bail(arc::fail_hip(e, "hipGetDevice"));
  if ((st = device_copy(&c->matrices_dev, c->matrices, "matrix tables")) != ARC_OK ||
      (st = device_copy(&c->tiles_dev, c->tiles, "matrix tables")) != ARC_OK ||
      (st = device_copy(&c->run_matrix_dev, c->run_matrix, "matrix tables")) != ARC_OK)
    return bail(st);
  const auto room = [&](auto** p, size_t bytes) {
    if (e != hipSuccess) return;
    e = hipMalloc(reinterpret_cast<void**>(p), std::max<size_t>(bytes, 16));
    if (e != hipSuccess) *p = nullptr;
  };
  room(&c->sums_dev, c->run_matrix.size() * sizeof(double));
  room(&c->workspace, static_cast<size_t>(c->workspace_bytes));
  room(&c->parts_dev, static_cast<size_t>(c->part_elems) * sizeof(float));
  room(&c->arrived_dev, static_cast<size_t>(c->counts) * sizeof(uint32_t));
  if (e == hipSuccess && c->counts > 0)
    e = hipMemset(c->arrived_dev, 0, static_cast<size_t>(c->counts) * sizeof(uint32_t));
  if (e == hipSuccess) e = arc::prepare_muon_products();
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return bail(arc::fail_hip(e, "matrix workspace"));
  }
  c->tiles = {};  // on the device from here on
  c->run_matrix = {};
  *out = c;
  return ARC_OK;
}

int64_t arc_muon_state_elems(const arc_muon* c) { return c ? c->state_elems : -1; }

int64_t arc_muon_state_offset(const arc_muon* c, int32_t i) {
  if (c == nullptr || i < 0 || static_cast<size_t>(i) >= c->matrices.size()) return -1;
  return c->matrices[static_cast<size_t>(i)].state;
}

arc_status arc_muon_orthogonalize(arc_muon* c, const void* const* in, void* const* out) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  arc_status st;
  if ((st = check_pointers(c, in, "in")) != ARC_OK ||
      (st = check_pointers(c, out, "out")) != ARC_OK)
    return st;
  return enqueue(c, arc::MuonArgs{}, out, in, nullptr);
}

arc_status arc_muon_step(arc_muon* c, const arc_muon_step_config* sc, void* const* params,
                         const void* const* grads, void* const* copies, const float* factor,
                         float* m) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  if (sc == nullptr) return fail(ARC_ERR_INVALID, "config is NULL");
  if (!finite(sc->lr)) return fail(ARC_ERR_INVALID, "lr must be finite");
  if (!(sc->momentum >= 0.f && sc->momentum < 1.f))
    return fail(ARC_ERR_INVALID, "momentum must be in [0, 1)");
  if (sc->nesterov != 0 && sc->nesterov != 1)
    return fail(ARC_ERR_INVALID, "nesterov must be 0 or 1");
  if (sc->reserved != 0) return fail(ARC_ERR_INVALID, "reserved must be 0");
  arc_status st;
  if ((st = check_pointers(c, params, "params")) != ARC_OK ||
      (st = check_pointers(c, grads, "grads")) != ARC_OK)
    return st;
  if (c->state_elems > 0 && m == nullptr) return fail(ARC_ERR_INVALID, "m is NULL");
  if (reinterpret_cast<uintptr_t>(m) % 16)
    return fail(ARC_ERR_INVALID, "m must be 16-byte aligned");
  if (overlap({m, c->state_elems * 4}, {factor, 4}))
    return fail(ARC_ERR_INVALID, "m and factor must not overlap");
  arc::MuonArgs a{};
  a.factor = factor;
  a.m = m;
  a.momentum = sc->momentum;
  a.lr = sc->lr;
  a.nesterov = sc->nesterov;
  a.update = 1;
  return enqueue(c, a, params, grads, copies);
}

arc_status arc_muon_destroy(arc_muon* c) {
  if (c == nullptr) return ARC_OK;
  c->release();
  delete c;
  return ARC_OK;
}

}  // extern "C"
