// Host-side argument checks and work planning of the linear attention (no HIP calls).
#pragma once
#include <cstddef>
#include <cstdint>
#include <vector>

#include "hydra_linear.h"

namespace hydra {

// A work item: consecutive rows of one sequence, which one workgroup per head walks in chunks.
enum LinearItem {
  LIN_ROW0 = 0,
  LIN_ROWS,
  LIN_SEQ,
  LIN_FIRST,  // 1: the sequence's first rows
  LIN_LAST,
  LIN_SLOT,   // of a sequence of several items, where the state lies that it starts from; else -1
  LIN_INTS = 8
};

// Checked and normalised view of a hydra_linear_t.
struct LinearProblem {
  int H = 0, Hkv = 0, dk = 0, dv = 0;
  float scale = 0.f;
  std::vector<int32_t> cu;
  int64_t rows = 0;
  int q_s = 0, k_s = 0, v_s = 0;  // token-row strides in elements
};
int check_linear(const hydra_linear_t* p, LinearProblem* out);

// The forward and the backward cut long sequences at different lengths.
enum class LinearFor { kForward, kBackward };
// The items, those of sequences of several items first (n_split of them, each sequence's in order and in slots one
// after another), the others by length; and of every such sequence {first slot, items}.
struct LinearPlan {
  int seg = 0;  // rows of an item but a sequence's last
  int n_items = 0, n_split = 0, n_scans = 0;
  std::vector<int32_t> items, scans;
};
void linear_plan(const LinearProblem& pr, LinearFor call, LinearPlan* out);

// Byte offsets of the workspace regions: the plans of both, the states of the walks of either (one of the forward, three
// of the backward), and for grouped heads dk and dv of every query head in 32 bits.
struct LinearLayout {
  size_t items_off[2], scans_off[2], slots_off, dk_off, dv_off, total;
};
LinearLayout linear_layout(const LinearProblem& pr, const LinearPlan& fwd, const LinearPlan& bwd);

}  // namespace hydra
