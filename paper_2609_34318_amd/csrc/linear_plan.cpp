// Host-side argument checks and work planning of the linear attention.
#include "linear_plan.h"

#include <algorithm>
#include <cmath>

namespace hydra {

namespace {
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Workgroups that a walk is cut into: two run on each of 256 CUs.  The three walks of the backward make 1.5 times as
// many of half the number, and its states and their scan cost more.  16K rows x 16 heads of 128 x 128: forward 143 us in
// 512 items, 164 in 336, 154 in 256 (one run); backward (another run) 251 in 512, 250 in 384, 228 in 256, 223 in 170 and 128.
// The backward takes 256 because of ten shapes of 2K to 64K rows it is within 8% of the best number on nine: 512 is 10 to
// 29% slower than it on six; 170 is 7% faster on 4K rows x 32 heads and 2 to 5% on three others, but 19% slower on 32K x 16 of
// 64 x 64, 5% on 16K x 16 of 128 x 64, and 28% on eight documents of 1000 rows x 16 (138 us; 108 in 256, and 79 in 128,
// which leaves them whole).
constexpr int64_t kLinearGroups[2] = {512, 256};
// The fewest rows of an item of a cut sequence (2K rows in four documents x 8 heads of 64 x 64: forward 26 us, 33 with 256).
constexpr int64_t kLinearMinRows = 128;
}  // namespace

int check_linear(const hydra_linear_t* p, LinearProblem* out) {
  if (!p || !out) return HYDRA_ERR_INVALID;
  if (p->n_heads <= 0 || p->n_heads > 4096) return HYDRA_ERR_INVALID;
  const int hkv = p->n_kv_heads == 0 ? p->n_heads : p->n_kv_heads;
  if (hkv < 0 || hkv > p->n_heads || p->n_heads % hkv != 0) return HYDRA_ERR_INVALID;
  if (p->d_k <= 0 || p->d_v <= 0) return HYDRA_ERR_INVALID;
  if ((p->d_k != 64 && p->d_k != 128 && p->d_k != 192) || (p->d_v != 64 && p->d_v != 128)) return HYDRA_ERR_UNSUPPORTED;
  if (!std::isfinite(p->scale)) return HYDRA_ERR_INVALID;
  if (!p->cu_seqlens || p->n_seqs < 1 || p->cu_seqlens[0] != 0) return HYDRA_ERR_INVALID;
  for (int64_t s = 0; s < p->n_seqs; ++s)
    if (p->cu_seqlens[s + 1] < p->cu_seqlens[s]) return HYDRA_ERR_INVALID;
  const int64_t rows = p->cu_seqlens[p->n_seqs];
  if (rows > (int64_t(1) << 30)) return HYDRA_ERR_INVALID;
  auto stride = [&](int32_t s, int64_t dense, int* dst) {
    if (s == 0) s = int32_t(dense);
    if (s < dense || s % 8 != 0 || s >= (1 << 22)) return false;
    *dst = s;
    return rows * s < (int64_t(1) << 40);
  };
  if (!stride(p->q_tok_stride, int64_t(p->n_heads) * p->d_k, &out->q_s) ||
      !stride(p->k_tok_stride, int64_t(hkv) * p->d_k, &out->k_s) ||
      !stride(p->v_tok_stride, int64_t(hkv) * p->d_v, &out->v_s))
    return HYDRA_ERR_INVALID;
  out->H = p->n_heads;
  out->Hkv = hkv;
  out->dk = p->d_k;
  out->dv = p->d_v;
  out->scale = p->scale > 0.f ? p->scale : 1.0f / std::sqrt(float(p->d_k));
  out->cu.assign(p->cu_seqlens, p->cu_seqlens + size_t(p->n_seqs) + 1);
  out->rows = rows;
  // one workgroup per item and head, of three walks in the backward, in a dispatch of fewer than 2^32 lanes
  const int64_t most = (rows * out->H + kLinearMinRows - 1) / kLinearMinRows + int64_t(p->n_seqs) * out->H;
  if (most >= (int64_t(1) << 21)) {  // what the bound without the plan does not say
    LinearPlan plan;
    for (LinearFor call : {LinearFor::kForward, LinearFor::kBackward}) {
      linear_plan(*out, call, &plan);
      if (int64_t(plan.n_items) * out->H >= (int64_t(1) << 21)) return HYDRA_ERR_INVALID;
    }
  }
  return HYDRA_OK;
}

void linear_plan(const LinearProblem& pr, LinearFor call, LinearPlan* out) {
  *out = LinearPlan{};
  const int64_t groups = kLinearGroups[int(call)], even = (pr.rows * pr.H + groups - 1) / groups;
  out->seg = int(std::max(kLinearMinRows, (even + 63) / 64 * 64));
  const int n_seqs = int(pr.cu.size()) - 1;
  std::vector<std::pair<int32_t, int>> whole;  // rows, sequence
  auto add = [&](int64_t row0, int64_t rows, int seq, bool first, bool last, int slot) {
    const int32_t it[LIN_INTS] = {int32_t(row0), int32_t(rows), seq, first, last, slot, 0, 0};
    out->items.insert(out->items.end(), it, it + LIN_INTS);
    ++out->n_items;
  };
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t n = int64_t(pr.cu[size_t(s) + 1]) - pr.cu[size_t(s)], parts = (n + out->seg - 1) / out->seg;
    if (parts <= 1) {
      whole.push_back({int32_t(n), s});
      continue;
    }
    out->scans.push_back(out->n_split);
    out->scans.push_back(int32_t(parts));
    for (int64_t j = 0; j < parts; ++j)
      add(pr.cu[size_t(s)] + j * out->seg, std::min<int64_t>(out->seg, n - j * out->seg), s, j == 0, j + 1 == parts, out->n_split++);
  }
  out->n_scans = int(out->scans.size() / 2);
  std::stable_sort(whole.begin(), whole.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
  for (const auto& w : whole) add(pr.cu[size_t(w.second)], w.first, w.second, true, true, -1);
}

LinearLayout linear_layout(const LinearProblem& pr, const LinearPlan& fwd, const LinearPlan& bwd) {
  LinearLayout w{};
  size_t off = 0;
  auto take = [&](uint64_t bytes) {
    const size_t at = off;
    off = align_up(off + size_t(bytes), 256);
    return at;
  };
  for (int i = 0; i < 2; ++i) {
    const LinearPlan& plan = i == 0 ? fwd : bwd;
    w.items_off[i] = take(plan.items.size() * sizeof(int32_t));
    w.scans_off[i] = take(plan.scans.size() * sizeof(int32_t));
  }
  const uint64_t slots = uint64_t(std::max(fwd.n_split, 3 * bwd.n_split));
  w.slots_off = take(slots * uint64_t(pr.H) * uint64_t(pr.dk) * uint64_t(pr.dv) * 4);
  const uint64_t heads = pr.Hkv < pr.H ? uint64_t(pr.rows) * uint64_t(pr.H) : 0;
  w.dk_off = take(heads * uint64_t(pr.dk) * 4);
  w.dv_off = take(heads * uint64_t(pr.dv) * 4);
  w.total = std::max<size_t>(off, 256);
  return w;
}

}  // namespace hydra
