// Tree steps, bf16 tensors over packed rings: see tree_group.hpp.
#include "tree_group.hpp"

namespace rattn {

void tree_step_bf16_packed(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  if (td.D == 64) pick_tree<bf16_t, fp8_t, 64>(td, t, pl, st);
  else pick_tree<bf16_t, fp8_t, 128>(td, t, pl, st);
}

}  // namespace rattn
