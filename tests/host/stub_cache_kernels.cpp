// Stand-ins for the launchers behind csrc/cache_api.hip (see stub_kernels.cpp): they record the call and touch no memory.
#include "kernels.hpp"

namespace rattn {

extern int g_stub_launches;
int g_split = 0;   // work-groups that the last call's plan shares a pair's keys among

void ring_pack(int, long long, const void*, const void*, void*, void*, void*, void*, hipStream_t) { ++g_stub_launches; }
void ring_unpack(int, long long, const void*, const void*, const void*, const void*, void*, void*, hipStream_t) { ++g_stub_launches; }
void decode_step_packed(const DecodeDims& dd, int, const void*, const void*, const void*, const int32_t*, void*, void*, void*, void*,
                        float*, const float*, const float*, void*, hipStream_t) {
  g_split = dd.workspace ? decode_split(dd, 1).n : 1;
  ++g_stub_launches;
}
void tree_step(const TreeDims& td, int dtype, const TreeTensors& t, hipStream_t) {
  g_split = td.workspace ? tree_plan(td, dtype, t.k_scale != nullptr).nsplit : 1;
  ++g_stub_launches;
}
void tree_commit(const TreeDims&, int, const TreeTensors&, const int32_t*, hipStream_t) { ++g_stub_launches; }

}  // namespace rattn
