// Plans of problems with prefixes: what the stored-dS backward relies on.  Every 32-row block of queries that
// sees a key finds the block of the key item's dS slots that holds its rows, at the place the kernels
// compute it; slots of different items do not overlap; the images of the forward's upload and of the
// complete plan agree; and without any modification the plan is the plain problem's.  Built with g++
// (no GPU code), with the sanitizers, by tests/test_scores_host.py.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "plan.h"

using namespace hydra;

namespace {
std::mt19937_64 rng(5);
int64_t uni(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (trial %d)\n", #x, trial); return 1; } } while (0)
}  // namespace

int main() {
  int64_t blocks = 0, refused = 0;
  for (int trial = 0; trial < 400; ++trial) {
    const int n_docs = int(uni(1, 14));
    std::vector<int32_t> cu(size_t(n_docs) + 1, 0), prefix(static_cast<size_t>(n_docs));
    for (int d = 0; d < n_docs; ++d) {
      const int32_t len = int32_t(uni(0, 5) == 0 ? uni(0, 3) : uni(0, trial % 3 ? 200 : 900));
      cu[size_t(d) + 1] = cu[size_t(d)] + len;
      const int64_t how = uni(0, 3);
      prefix[size_t(d)] = int32_t(how == 0 ? 0 : how == 1 ? len : uni(0, len));
    }
    hydra_problem_t p{};
    p.n_heads = 2;
    p.d_qk = 192;
    p.d_v = 128;
    p.cu_seqlens = cu.data();
    p.n_docs = n_docs;
    for (hydra_chunk_t* c : {&p.q, &p.kv}) {
      c->n_segs = int32_t(uni(1, 4));
      int64_t at = 0;  // segments of one chunk do not overlap: a row then has one place
      for (int s = 0; s < c->n_segs; ++s) {
        const int64_t a = uni(at, cu.back()) / 32 * 32, b = uni(a, cu.back()) / 32 * 32;
        c->start[s] = int32_t(std::max(a, at));
        c->len[s] = int32_t(std::max<int64_t>(0, b - c->start[s]));
        at = c->start[s] + c->len[s];
      }
    }
    hydra_scores_t sc{};
    Problem pr, plain;
    CHECK(check_problem(&p, &plain) == HYDRA_OK);
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK && !pr.scored && pr.pe.empty());  // nothing on
    sc.prefix_len = prefix.data();
    CHECK(check_problem(&p, &sc, &pr) == HYDRA_OK && pr.scored);
    // refusals
    const int64_t d = uni(0, n_docs - 1);
    const int32_t old = prefix[size_t(d)];
    prefix[size_t(d)] = uni(0, 1) ? -1 : cu[size_t(d) + 1] - cu[size_t(d)] + 1;
    Problem bad;
    CHECK(check_problem(&p, &sc, &bad) == HYDRA_ERR_INVALID);
    prefix[size_t(d)] = old;
    ++refused;

    const WsLayout w = ws_layout(pr);
    CHECK(w.total >= ws_layout(plain).total);
    PlanImage all, fwd;
    plan_image(pr, w, PlanFor::kStoredDs, true, &all);
    plan_image(pr, w, PlanFor::kForward, true, &fwd);
    CHECK(all.off + all.bytes.size() <= w.d_off);
    CHECK(std::equal(fwd.bytes.begin(), fwd.bytes.end(), all.bytes.begin() + int64_t(fwd.off - all.off)));
    const int32_t* at = reinterpret_cast<const int32_t*>(all.bytes.data() + (w.cu_off - all.off));
    CHECK(std::equal(pr.cu.begin(), pr.cu.end(), at) && std::equal(pr.pe.begin(), pr.pe.end(), at + pr.cu.size()));
    if (!ds_path_applies(pr)) continue;

    std::vector<int32_t> kitems, kbase, kmap32, krec;
    plan_items(pr, 1, &kitems);
    const int64_t slots = ds_tables(pr, kitems, &kbase, &kmap32, &krec);
    std::vector<int32_t> qpos, kpos;
    for (int s = 0; s < p.q.n_segs; ++s)
      for (int32_t i = 0; i < p.q.len[s]; ++i) qpos.push_back(p.q.start[s] + i);
    for (int s = 0; s < p.kv.n_segs; ++s)
      for (int32_t i = 0; i < p.kv.len[s]; ++i) kpos.push_back(p.kv.start[s] + i);
    auto doc = [&](int32_t x) { return int(std::upper_bound(cu.begin(), cu.end(), x) - cu.begin()) - 1; };
    auto sees = [&](int32_t q, int32_t k) {
      const int dq = doc(q);
      return dq == doc(k) && (k <= q || k < pr.pe[size_t(dq)]);
    };
    std::vector<int> used(size_t(slots), -1);
    for (size_t j = 0; j < krec.size() / kItemInts; ++j) {
      const int32_t* rec = &krec[j * kItemInts];
      int32_t slot = rec[3];
      for (int r = 0; r < rec[2]; ++r)
        for (int32_t t = 0; t < (rec[5 + 2 * r] + KV_QTILE_ROWS - 1) / KV_QTILE_ROWS; ++t) {
          CHECK(slot < slots && used[size_t(slot)] < 0);
          used[size_t(slot++)] = int(j);
        }
      // the 32-row blocks of queries, as the dQ kernel's waves hold them: from their segment's start on
      int32_t row0 = 0;
      for (int s = 0; s < p.q.n_segs; ++s) {
        for (int32_t b = 0; b < p.q.len[s]; b += 32) {
          const int32_t qrow = row0 + b;
          bool any = false;
          for (int32_t i = qrow; i < qrow + 32 && !any; ++i)
            for (int32_t k = rec[0]; k < rec[0] + rec[1] && !any; ++k) any = sees(qpos[size_t(i)], kpos[size_t(k)]);
          if (!any) continue;
          ++blocks;
          int found = 0;
          for (int r = 0; r < rec[2]; ++r)
            if (qrow >= rec[4 + 2 * r] && qrow < rec[4 + 2 * r] + rec[5 + 2 * r]) {
              ++found;
              CHECK((qrow - rec[4 + 2 * r]) % 32 == 0);
              // every row of the block that sees a key lies in the range
              for (int32_t i = qrow; i < qrow + 32; ++i)
                for (int32_t k = rec[0]; k < rec[0] + rec[1]; ++k)
                  if (sees(qpos[size_t(i)], kpos[size_t(k)])) CHECK(i < rec[4 + 2 * r] + rec[5 + 2 * r]);
            }
          CHECK(found == 1);
        }
        row0 += p.q.len[s];
      }
    }
  }
  std::printf("%lld blocks, %lld refusals\n", (long long)blocks, (long long)refused);
  return blocks > 1000 ? 0 : 1;
}
