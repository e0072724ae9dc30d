// Plans of windows with sinks where a launch is full or a record is: parts of the long items are as short as they were
// meant to be or as the number of parts allows, and a query tile whose sinks and window need more ranges than a record
// holds walks from its document's start.  Built with g++ (no GPU code), with the sanitizers, by tests/test_window_split.py.
#include <algorithm>
#include <cstdio>
#include <numeric>
#include <random>
#include <vector>

#include "plan.h"

using namespace hydra;

namespace {
std::mt19937_64 rng(5);
int64_t uni(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (trial %d)\n", #x, trial); return 1; } } while (0)

int64_t tiles_of(const int32_t* u) {
  int64_t t = 0;
  for (int r = 0; r < u[3]; ++r) t += (u[6 + 3 * r] + KV_QTILE_ROWS - 1) / KV_QTILE_ROWS;
  return t;
}
}  // namespace

int main() {
  int64_t split = 0, capped = 0;
  for (int trial = 0; trial < 200; ++trial) {
    const int heads[] = {1, 8, 16, 24, 64, 3, 12}, H = heads[trial % 7];
    std::vector<int32_t> cu{0};
    for (int d = int(uni(1, 3)); d > 0; --d) cu.push_back(cu.back() + int32_t(uni(1, trial % 5 ? 30000 : 200000)));
    hydra_problem_t p{};
    p.n_heads = H;
    p.d_qk = 192;
    p.d_v = 128;
    p.cu_seqlens = cu.data();
    p.n_docs = int32_t(cu.size()) - 1;
    p.q.n_segs = p.kv.n_segs = 1;
    p.q.len[0] = p.kv.len[0] = cu.back();
    hydra_scores_t sc{};
    sc.window = int32_t(uni(1, 6000));
    sc.sinks = int32_t(uni(1, 300));
    Problem pr;
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK);
    std::vector<int32_t> items, records;
    plan_items(pr, 1, &items);
    launch_units(pr, 1, items, {}, &records);
    const int64_t n = int64_t(records.size()) / kUnitInts;
    if (n * H < kSplitBelow) continue;  // a launch that is not full is split to fill it
    std::vector<int64_t> tiles;
    for (int64_t i = 0; i < n; ++i) tiles.push_back(tiles_of(&records[size_t(i) * kUnitInts]));
    UnitList l;
    split_units(pr, Kernel::kDkdv, records, H, &l);
    int64_t longest = 0;
    for (size_t i = 0; i < l.units.size(); i += kUnitInts)
      longest = std::max(longest, l.units[i + REC_T1] < 0 ? tiles_of(&l.units[i]) : int64_t(l.units[i + REC_T1] - l.units[i + REC_T0]));
    if (l.units.empty()) longest = *std::max_element(tiles.begin(), tiles.end());
    // what runs beside an item, in tiles: its head's items over 32 CUs, or all heads' over 256 (an item costs two more)
    const double all = double(std::accumulate(tiles.begin(), tiles.end(), int64_t(0))) + 2.0 * double(n);
    const int64_t bound = std::max<int64_t>(8, int64_t(H % 8 == 0 ? all / 32 : all * H / 256));
    auto parts_at = [&](int64_t most) {
      int64_t parts = 0;
      for (int64_t t : tiles)
        if (t > most) parts += (t + most - 1) / most;
      return parts * H;
    };
    split += !l.units.empty();
    if (longest <= bound) continue;
    // longer only where that many parts are too many, and then by no more than a step of a quarter
    CHECK(parts_at(bound) > max_parts(pr));
    int64_t fits = bound;
    while (parts_at(fits) > max_parts(pr)) ++fits;
    CHECK(longest <= fits + (fits + 3) / 4);
    ++capped;
  }
  std::printf("%lld split, %lld of them by the number of parts\n", (long long)split, (long long)capped);
  if (split < 20 || capped < 1) return 1;

  const int trial = -1;
  std::vector<int32_t> cu{0, 5000};
  hydra_problem_t p{};
  p.n_heads = 2;
  p.d_qk = 192;
  p.d_v = 128;
  p.cu_seqlens = cu.data();
  p.n_docs = 1;
  p.q.n_segs = 1;
  p.q.start[0] = 4000;
  p.q.len[0] = 256;
  const int32_t segs[4][2] = {{0, 100}, {150, 100}, {300, 3200}, {3600, 700}};
  p.kv.n_segs = 4;
  for (int s = 0; s < 4; ++s) {
    p.kv.start[s] = segs[s][0];
    p.kv.len[s] = segs[s][1];
  }
  hydra_scores_t sc{};
  sc.window = 1000;
  for (int sinks : {100, 350}) {  // sinks of one segment, of three
    sc.sinks = sinks;
    Problem pr;
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK);
    std::vector<int32_t> items;
    plan_items(pr, 0, &items);
    CHECK(items.size() == kItemInts);
    int64_t keys = 0;
    for (int r = 0; r < items[3]; ++r) keys += items[6 + 3 * size_t(r)];
    // the sinks, and from position 3001 to 3500 and 3600 to 4255; or everything up to there
    CHECK(items[3] == (sinks == 100 ? 3 : 4) && keys == (sinks == 100 ? 100 + 499 + 656 : 100 + 100 + 3200 + 656));
  }
  return 0;
}
