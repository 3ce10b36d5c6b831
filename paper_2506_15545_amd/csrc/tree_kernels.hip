// Tree steps: the choice of kernels, and those of bf16 tensors and rings (tree_group.hpp; the other types are compiled apart).
#include "tree_group.hpp"

namespace rattn {

void tree_step_f32(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st);
void tree_step_f32_packed(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st);
void tree_step_bf16_packed(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st);

void tree_step_tiles(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st);

void tree_step(const TreeDims& td, int dtype, const TreeTensors& t, hipStream_t st) {
  const bool packed = t.k_scale != nullptr;
  const TreePlan pl = tree_plan(td, dtype, packed);
  ProfScope ps(pl.tiles ? "tree_tile_kernel" : "tree_kernel", st);
  if (pl.tiles) tree_step_tiles(td, t, pl, st);
  else if (dtype == 0) (packed ? tree_step_f32_packed : tree_step_f32)(td, t, pl, st);
  else if (packed) tree_step_bf16_packed(td, t, pl, st);
  else if (td.D == 64) pick_tree<bf16_t, bf16_t, 64>(td, t, pl, st);
  else pick_tree<bf16_t, bf16_t, 128>(td, t, pl, st);
}

}  // namespace rattn
