// Plans of the matrix optimizer (arc_muon.cpp): a count of arrived parts belongs to
// tiles of one list and one number of parts, so that it is 0 after any launches, however
// they overlapped.  Prints "ok" and how many counts were looked at.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <map>
#include <string>
#include <utility>
#include <vector>

#include "arc_muon.cpp"

namespace arc {
arc_status fail(arc_status s, const std::string&) { return s; }
arc_status fail_hip(hipError_t, const char*) { return ARC_ERR_DEVICE; }
}  // namespace arc

static int wrong = 0;
static size_t looked_at = 0;

static void check(const std::vector<arc_muon_matrix>& list) {
  const arc_muon_config cfg{list.data(), nullptr, static_cast<int32_t>(list.size()), 5, 0};
  for (const int32_t whole_of : {64, 128}) {
    arc_muon c;
    plan_muon(&cfg, whole_of, &c);
    std::map<int64_t, std::pair<const arc::MuonGroup::Range*, int32_t>> of;
    for (const arc::MuonGroup& g : c.groups)
      for (const arc::MuonGroup::Range* r : {&g.gram, &g.half, &g.whole})
        for (int64_t k = r->at; k < r->at + r->count; ++k) {
          const arc::MuonTile& t = c.tiles[static_cast<size_t>(k)];
          if (t.parts < 2) continue;
          const int64_t at = r->counts + t.place;
          const auto seen = of.emplace(at, std::make_pair(r, t.parts)).first->second;
          if (at < 0 || at >= c.counts || seen.first != r || seen.second != t.parts) ++wrong;
        }
    looked_at += of.size();
  }
}

int main() {
  const auto list = [](std::vector<std::pair<int64_t, int64_t>> sides) {
    std::vector<arc_muon_matrix> out;
    for (const auto& s : sides) out.push_back({s.first, s.second, 0, 0, 0.f, 1.f});
    return out;
  };
  check(list({{257, 1001}}));
  check(list({{64, 4096}, {33, 31}, {768, 2304}, {0, 9}, {1500, 700}}));
  check(list(std::vector<std::pair<int64_t, int64_t>>(170, {33, 4000})));
  check(list({{4096, 4096}, {1, 70001}}));
  check(list(std::vector<std::pair<int64_t, int64_t>>(20, {512, 4608})));
  std::printf("%zu counts, %d wrong\n", looked_at, wrong);
  if (wrong == 0 && looked_at > 0) std::printf("ok\n");
  return wrong != 0;
}
