// Tree steps, fp32 tensors and rings: see tree_group.hpp.
#include "tree_group.hpp"

namespace rattn {

void tree_step_f32(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  if (td.D == 64) pick_tree<float, float, 64>(td, t, pl, st);
  else pick_tree<float, float, 128>(td, t, pl, st);
}

}  // namespace rattn
