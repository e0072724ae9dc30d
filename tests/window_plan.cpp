// Plans of problems with a sliding window and sinks, against the definition of what a row sees: every visible pair lies
// in the ranges of its query item and of its key item, ranges do not overlap, the stored dS of every block that the dQ
// kernel reads was stored, at the place where it reads it and once, and the visible pairs are counted.  Built with g++
// (no GPU code), with the sanitizers, by tests/test_window_host.py.
#include <algorithm>
#include <cstdio>
#include <random>
#include <set>
#include <vector>

#include "plan.h"

using namespace hydra;

namespace {
std::mt19937_64 rng(11);
int64_t uni(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (trial %d)\n", #x, trial); return 1; } } while (0)
}  // namespace

int main() {
  int64_t pairs_seen = 0, two_ranges = 0, merged = 0, blocks = 0;
  for (int trial = 0; trial < 600; ++trial) {
    const int n_docs = int(uni(1, 8));
    std::vector<int32_t> cu(size_t(n_docs) + 1, 0);
    for (int d = 0; d < n_docs; ++d)
      cu[size_t(d) + 1] = cu[size_t(d)] + int32_t(uni(0, 4) == 0 ? uni(0, 3) : uni(0, trial % 3 ? 260 : 1500));
    hydra_problem_t p{};
    p.n_heads = 2;
    p.d_qk = 192;
    p.d_v = 128;
    p.cu_seqlens = cu.data();
    p.n_docs = n_docs;
    const int grain = trial % 2 ? 32 : 1;
    for (hydra_chunk_t* c : {&p.q, &p.kv}) {
      c->n_segs = int32_t(uni(1, 4));
      int64_t at = 0;
      for (int s = 0; s < c->n_segs; ++s) {
        const int64_t a = uni(at, cu.back()) / grain * grain, b = uni(a, cu.back()) / grain * grain;
        c->start[s] = int32_t(std::max(a, at));
        c->len[s] = int32_t(std::max<int64_t>(0, b - c->start[s]));
        at = c->start[s] + c->len[s];
      }
    }
    hydra_scores_t sc{};
    sc.window = int32_t(uni(0, 9) == 0 ? 0x7fffffff : uni(1, trial % 3 ? 200 : 900));
    sc.sinks = int32_t(uni(0, 2) == 0 ? 0 : uni(0, 9) == 0 ? 0x7fffffff : uni(0, 3) == 0 ? uni(100, 400) : uni(1, 8));
    Problem pr, bad;
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK && pr.scored && pr.window == sc.window);
    hydra_scores_t wrong = sc;
    wrong.window = 0;
    wrong.sinks = 1;
    CHECK(check_problem(&p, &wrong, &bad) == HYDRA_ERR_INVALID);
    wrong = sc;
    std::vector<int32_t> prefix(static_cast<size_t>(n_docs), 0);
    wrong.prefix_len = prefix.data();
    CHECK(check_problem(&p, &wrong, &bad) == HYDRA_ERR_INVALID);
    wrong = sc;
    (trial % 2 ? wrong.window : wrong.sinks) = -1;
    CHECK(check_problem(&p, &wrong, &bad) == HYDRA_ERR_INVALID);

    std::vector<int32_t> pos[2];
    for (int side = 0; side < 2; ++side) {
      const hydra_chunk_t& c = side == 0 ? p.q : p.kv;
      for (int s = 0; s < c.n_segs; ++s)
        for (int32_t i = 0; i < c.len[s]; ++i) pos[side].push_back(c.start[s] + i);
    }
    auto doc = [&](int32_t x) { return int(std::upper_bound(cu.begin(), cu.end(), x) - cu.begin()) - 1; };
    auto sees = [&](int32_t q, int32_t k) {
      return k <= q && doc(q) == doc(k) && (int64_t(q) - k < sc.window || int64_t(k) - cu[size_t(doc(k))] < sc.sinks);
    };
    int64_t pairs = 0;
    for (int32_t q : pos[0])
      for (int32_t k : pos[1]) pairs += k <= q && sees(q, k);
    CHECK(pairs == visible_pairs(pr));
    pairs_seen += pairs;

    std::vector<int32_t> items[2];
    for (int side = 0; side < 2; ++side) {
      plan_items(pr, side, &items[side]);
      for (size_t i = 0; i < items[side].size(); i += kItemInts) {
        const int32_t* it = &items[side][i];
        std::vector<char> in(pos[1 - side].size(), 0);
        for (int r = 0; r < it[3]; ++r)
          for (int32_t x = it[4 + 3 * r]; x < it[4 + 3 * r] + it[6 + 3 * r]; ++x) {
            CHECK(x >= 0 && x < int32_t(in.size()) && !in[size_t(x)]);
            CHECK(pos[1 - side][size_t(x)] == it[5 + 3 * r] + x - it[4 + 3 * r]);
            in[size_t(x)] = 1;
          }
        if (side == 0 && it[3] > 1 && it[5] + it[6] < it[8]) ++two_ranges;
        for (int32_t x = it[0]; x < it[0] + it[2]; ++x)
          for (size_t y = 0; y < in.size(); ++y)
            if (!in[y]) CHECK(!(side == 0 ? sees(pos[0][size_t(x)], pos[1][y]) : sees(pos[0][y], pos[1][size_t(x)])));
        if (side == 0 && it[3] > 0 && pos[0][size_t(it[0])] - it[5] > 2 * int64_t(sc.window) + 600) ++merged;
      }
    }
    if (!ds_path_applies(pr)) continue;
    // the dQ kernel's walk: halves of key items, each read once, where the dK/dV kernel stored them
    std::vector<int32_t> kbase, kmap32, krec;
    const int64_t slots = ds_tables(pr, items[1], &kbase, &kmap32, &krec);
    for (size_t i = 0; i < items[0].size(); i += kItemInts) {
      const int32_t* it = &items[0][i];
      std::set<std::pair<int, int>> halves;
      for (int r = 0; r < it[3]; ++r) {
        int j = kmap32[size_t(it[4 + 3 * r]) / 32];
        for (int32_t x = it[4 + 3 * r], end = x + it[6 + 3 * r]; x < end;) {
          if (x >= krec[size_t(j) * kItemInts] + krec[size_t(j) * kItemInts + 1]) ++j;
          const int32_t* rec = &krec[size_t(j) * kItemInts];
          CHECK(x >= rec[0] && x < rec[0] + rec[1]);
          const int half = (x - rec[0]) >> 6;
          CHECK(halves.insert({j, half}).second);
          const int32_t k0 = rec[0] + 64 * half, kn = std::min(64, rec[1] - 64 * half);
          for (int32_t q0 = it[0]; q0 < it[0] + it[2]; q0 += 32) {
            bool any = false;
            for (int32_t q = q0; q < q0 + 32 && !any; ++q)
              for (int32_t k = k0; k < k0 + kn && !any; ++k) any = sees(pos[0][size_t(q)], pos[1][size_t(k)]);
            int found = 0;
            int32_t slot = rec[3];
            for (int q = 0; q < rec[2]; slot += (rec[5 + 2 * q] + KV_QTILE_ROWS - 1) / KV_QTILE_ROWS, ++q)
              if (q0 >= rec[4 + 2 * q] && q0 < rec[4 + 2 * q] + rec[5 + 2 * q]) {
                ++found;
                CHECK((q0 - rec[4 + 2 * q]) % 32 == 0 && slot + (q0 - rec[4 + 2 * q]) / KV_QTILE_ROWS < slots);
              }
            CHECK(found <= 1 && (found == 1 || !any));
            blocks += any;
          }
          x = k0 + 64;
        }
      }
    }
  }
  // launches of many items, one of which all queries see: its parts cover its tiles, the lists fit their place, and no part
  // is longer than what a head's items take on an eighth of the CUs
  int64_t split = 0;
  for (int trial = 0; trial < 60; ++trial) {
    const int heads[] = {1, 8, 16, 24, 64, 3};
    std::vector<int32_t> cu{0};
    for (int d = int(uni(1, 3)); d > 0; --d) cu.push_back(cu.back() + int32_t(uni(1, trial % 5 ? 30000 : 200000)));
    hydra_problem_t p{};
    p.n_heads = heads[trial % 6];
    p.d_qk = 192;
    p.d_v = 128;
    p.cu_seqlens = cu.data();
    p.n_docs = int32_t(cu.size()) - 1;
    p.q.n_segs = p.kv.n_segs = 1;
    p.q.len[0] = p.kv.len[0] = cu.back();
    hydra_scores_t sc{};
    sc.window = int32_t(uni(1, 6000));
    sc.sinks = int32_t(uni(0, 3) * uni(1, 100));
    Problem pr;
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK);
    const WsLayout w = ws_layout(pr);
    for (PlanFor call : {PlanFor::kForward, PlanFor::kBackward, PlanFor::kStoredDs}) {
      PlanImage img;
      plan_image(pr, w, call, true, &img);
      CHECK(img.off + img.bytes.size() <= w.d_off);
    }
    std::vector<int32_t> items, records;
    plan_items(pr, 1, &items);
    launch_units(pr, 1, items, {}, &records);
    UnitList l;
    split_units(pr, Kernel::kDkdv, records, pr.Hkv, &l);
    CHECK(l.parts * pr.Hkv <= max_parts(pr) && (sc.sinks > 0) == (max_parts(pr) > MAX_PARTS));
    const bool many = int64_t(records.size()) / kUnitInts * pr.Hkv >= kSplitBelow;
    if (many && sc.sinks == 0) CHECK(l.units.empty());
    if (l.units.empty()) continue;
    split += many;
    std::vector<int64_t> covered(size_t(l.parts), 0);
    for (size_t m = 0; m < l.merges.size(); m += kMergeInts) {
      int64_t tiles = 0, next = 0;
      for (size_t i = 0; i < records.size(); i += kUnitInts)
        if (records[i] == l.merges[m])
          for (int r = 0; r < records[i + 3]; ++r) tiles += (records[i + 6 + 3 * size_t(r)] + KV_QTILE_ROWS - 1) / KV_QTILE_ROWS;
      for (int32_t part = l.merges[m + 2]; part < l.merges[m + 2] + l.merges[m + 3]; ++part)
        for (size_t u = 0; u < l.units.size(); u += kUnitInts)
          if (l.units[u + REC_PART] == part) {
            CHECK(l.units[u] == l.merges[m] && l.units[u + REC_T0] == next && l.units[u + REC_T1] > next);
            next = l.units[u + REC_T1];
            ++covered[size_t(part)];
          }
      CHECK(next == tiles);
    }
    for (int64_t c : covered) CHECK(c == 1);
  }
  if (split < 5) return 1;
  std::printf("%lld pairs, %lld items of two ranges, %lld merged, %lld blocks\n", (long long)pairs_seen, (long long)two_ranges,
              (long long)merged, (long long)blocks);
  return two_ranges > 50 && blocks > 1000 ? 0 : 1;
}
