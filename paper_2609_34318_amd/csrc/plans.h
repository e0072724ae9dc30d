// Which plan each workspace holds, as far as this library uploaded it (abi.cpp): planned calls launch on the plan in
// the workspace and refuse one that was made for another problem.  Keys of different kinds of plans differ in their
// first number.
#pragma once
#include <cstdint>
#include <vector>

namespace hydra {
void plans_record(const void* ws, std::vector<int64_t>&& key);
bool plans_hold(const void* ws, const std::vector<int64_t>& key);
}  // namespace hydra
