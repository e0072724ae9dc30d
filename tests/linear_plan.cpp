// Plans of the linear attention: every row of every sequence lies in one item, items of a cut sequence are in order, in
// slots of their own one after another, with lengths that the scan may take as equal, and the workspace holds what the
// calls write.  Built with g++ (no GPU code), with the sanitizers, by tests/test_linear_host.py.
#include <cstdio>
#include <random>
#include <vector>

#include "linear_plan.h"

using namespace hydra;

namespace {
std::mt19937_64 rng(3);
int64_t uni(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (trial %d)\n", #x, trial); return 1; } } while (0)
}  // namespace

int main() {
  int64_t cut = 0, refused = 0;
  for (int trial = 0; trial < 2000; ++trial) {
    std::vector<int32_t> cu{0};
    for (int s = int(uni(1, 12)); s > 0; --s) cu.push_back(cu.back() + int32_t(uni(0, 3) ? uni(0, 900) : uni(0, 40000)));
    hydra_linear_t p{};
    const int dks[] = {64, 128, 192}, dvs[] = {64, 128}, heads[] = {1, 3, 8, 16, 64};
    p.n_heads = heads[uni(0, 4)];
    p.n_kv_heads = uni(0, 1) ? 0 : 1;
    p.d_k = dks[uni(0, 2)];
    p.d_v = dvs[uni(0, 1)];
    p.cu_seqlens = cu.data();
    p.n_seqs = int32_t(cu.size()) - 1;
    LinearProblem pr;
    CHECK(check_linear(&p, &pr) == HYDRA_OK && pr.rows == cu.back());
    LinearPlan plans[2];
    linear_plan(pr, LinearFor::kForward, &plans[0]);
    linear_plan(pr, LinearFor::kBackward, &plans[1]);
    const LinearLayout w = linear_layout(pr, plans[0], plans[1]);
    CHECK(w.slots_off <= w.dk_off && w.dk_off <= w.dv_off && w.dv_off <= w.total && w.total > 0);
    const uint64_t state = uint64_t(pr.H) * uint64_t(pr.dk) * uint64_t(pr.dv) * 4;
    for (int i = 0; i < 2; ++i) {
      const LinearPlan& plan = plans[i];
      CHECK(w.items_off[i] + plan.items.size() * 4 <= w.scans_off[i] && w.scans_off[i] + plan.scans.size() * 4 <= w.slots_off);
      CHECK(w.slots_off + uint64_t(plan.n_split) * state * (i == 0 ? 1 : 3) <= w.dk_off);
      CHECK(plan.items.size() == size_t(plan.n_items) * LIN_INTS && plan.scans.size() == size_t(plan.n_scans) * 2);
      std::vector<int> seen(size_t(cu.back()), 0), sequences(size_t(p.n_seqs), 0);
      for (int k = 0; k < plan.n_items; ++k) {
        const int32_t* it = &plan.items[size_t(k) * LIN_INTS];
        CHECK(it[LIN_SEQ] >= 0 && it[LIN_SEQ] < p.n_seqs && it[LIN_ROWS] <= plan.seg);
        CHECK(it[LIN_ROW0] >= cu[size_t(it[LIN_SEQ])] && it[LIN_ROW0] + it[LIN_ROWS] <= cu[size_t(it[LIN_SEQ]) + 1]);
        CHECK(it[LIN_FIRST] == (it[LIN_ROW0] == cu[size_t(it[LIN_SEQ])]));
        CHECK(it[LIN_LAST] == (it[LIN_ROW0] + it[LIN_ROWS] == cu[size_t(it[LIN_SEQ]) + 1]));
        CHECK((it[LIN_SLOT] >= 0) == (k < plan.n_split) && (it[LIN_SLOT] < 0 || it[LIN_SLOT] == k));
        CHECK((it[LIN_SLOT] < 0) == (it[LIN_FIRST] && it[LIN_LAST]));
        if (it[LIN_SLOT] >= 0 && !it[LIN_LAST]) {
          const int32_t* next = it + LIN_INTS;
          CHECK(it[LIN_ROWS] == plan.seg && next[LIN_SEQ] == it[LIN_SEQ] && next[LIN_ROW0] == it[LIN_ROW0] + it[LIN_ROWS]);
        }
        sequences[size_t(it[LIN_SEQ])] += it[LIN_FIRST];
        for (int32_t r = 0; r < it[LIN_ROWS]; ++r) ++seen[size_t(it[LIN_ROW0] + r)];
      }
      for (int n : seen) CHECK(n == 1);
      for (int n : sequences) CHECK(n == 1);  // those without rows too: their states are copied
      int at = 0;
      for (int s = 0; s < plan.n_scans; ++s) {
        CHECK(plan.scans[size_t(s) * 2] == at && plan.scans[size_t(s) * 2 + 1] >= 2);
        at += plan.scans[size_t(s) * 2 + 1];
      }
      CHECK(at == plan.n_split);
      cut += plan.n_split;
    }
    hydra_linear_t bad = p;
    std::vector<int32_t> other = cu;
    int want = HYDRA_ERR_INVALID;
    switch (trial % 11) {
      case 0: bad.n_heads = uni(0, 1) ? 0 : 4097; break;
      case 1: bad.n_kv_heads = p.n_heads + 1; break;
      case 2: bad.d_k = 96; want = HYDRA_ERR_UNSUPPORTED; break;
      case 3: bad.d_v = 192; want = HYDRA_ERR_UNSUPPORTED; break;
      case 4: bad.n_seqs = 0; break;
      case 5: bad.cu_seqlens = nullptr; break;
      case 6: other[0] = 1; bad.cu_seqlens = other.data(); break;
      case 7: other.back() = -1; bad.cu_seqlens = other.data(); break;
      case 8: bad.q_tok_stride = p.n_heads * p.d_k - 8; break;
      case 9: bad.v_tok_stride = p.n_heads * p.d_v + 4; break;
      case 10: bad.scale = 1.0f / 0.0f; break;
    }
    LinearProblem x;
    CHECK(check_linear(&bad, &x) == want);
    ++refused;
  }
  std::printf("%lld items of cut sequences, %lld refusals\n", (long long)cut, (long long)refused);
  return cut > 1000 ? 0 : 1;
}
