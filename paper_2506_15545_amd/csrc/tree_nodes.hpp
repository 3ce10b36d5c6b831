// Trees of drafted tokens: what a wave knows of one, node i in lane i.
#pragma once
#include "common.hpp"

namespace rattn {

constexpr int TREE_MAX_NODES = 64;   // a node's ancestors are one 64-bit mask, and a wave has a lane for each

__device__ __forceinline__ unsigned long long shfl64(unsigned long long x, int lane) {
  const unsigned lo = __shfl((unsigned)x, lane), hi = __shfl((unsigned)(x >> 32), lane);
  return (unsigned long long)hi << 32 | lo;
}

struct TreeNodes {
  unsigned long long anc;    // this node and its ancestors
  unsigned long long left;   // those of them that are W or more tokens back
  __device__ __forceinline__ int depth() const { return __popcll(anc) - 1; }
};
// parent: of node `lane` (anything for lanes without one).  A parent that is no earlier node counts as the sequence's last token
// (-1).  Called by whole waves.  Six rounds that double the distance: `jump` is the ancestor 2^r back, `far` the one W back.
__device__ __forceinline__ TreeNodes tree_nodes(int parent, int W, int lane) {
  int jump = parent < 0 || parent >= lane ? -1 : parent;
  int far = W < TREE_MAX_NODES ? lane : -1;
  TreeNodes t;
  t.anc = 1ull << lane;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    const unsigned long long up = shfl64(t.anc, max(jump, 0));
    if (jump >= 0) t.anc |= up;
    if (W >> r & 1) {   // (uniform)
      const int f = __shfl(jump, max(far, 0));
      far = far >= 0 ? f : -1;
    }
    const int j = __shfl(jump, max(jump, 0));
    jump = jump >= 0 ? j : -1;
  }
  const unsigned long long l = shfl64(t.anc, max(far, 0));
  t.left = far >= 0 ? l : 0;
  return t;
}

}  // namespace rattn
