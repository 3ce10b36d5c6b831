// Tree steps of many rows, bf16 tensors: see tree_tiles.hpp.
#include "tree_tiles.hpp"

namespace rattn {

void tree_step_tiles(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  if (t.k_scale) {
    if (td.D == 64) pick_tree_tile<fp8_t, 64>(td, t, pl, st);
    else pick_tree_tile<fp8_t, 128>(td, t, pl, st);
  } else {
    if (td.D == 64) pick_tree_tile<bf16_t, 64>(td, t, pl, st);
    else pick_tree_tile<bf16_t, 128>(td, t, pl, st);
  }
}

}  // namespace rattn
