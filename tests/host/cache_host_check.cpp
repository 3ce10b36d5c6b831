// Drives the host layer of packed rings and trees (csrc/cache_api.hip, csrc/plan.hip) built for the CPU with stub launchers:
// validation, plans and workspace sizes from the smallest to extreme shapes.  Pointers are fake and never dereferenced.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "kernels.hpp"
#include "rattn.h"

namespace rattn { extern int g_stub_launches; extern int g_split; }

static int failures = 0;
#define CHECK(cond)                                                                  \
  do {                                                                               \
    if (!(cond)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)
static bool launched(rattn_status st) { return st == RATTN_OK || st == RATTN_ERR_HIP; }   // (no device on a CPU machine)

int main() {
  void* x = (void*)(uintptr_t)0x7f0000001000ull;
  const int32_t* ix = (const int32_t*)x;
  float* fx = (float*)x;
  const int shapes[][5] = {{1, 1, 1, 64, 1},       {1, 16, 4, 128, 512},   {128, 32, 8, 128, 512}, {65535, 1, 1, 128, 9},
                           {1, 65535, 65535, 64, 3}, {1, 4, 1, 128, 1 << 30}, {7, 320, 1, 64, 1000}, {3, 65535, 1, 128, 70000},
                           {1, 4, 1, 64, 0x7fffffff}, {24, 40, 8, 128, 2048}, {400, 8, 2, 64, 300}, {2, 8, 2, 128, 320}, {3, 8, 2, 128, 4096},
                           {16, 20, 4, 64, 1500}};
  for (auto& s : shapes)
    for (int dtype = 0; dtype < 2; ++dtype)
      for (int nodes : {1, 2, 3, 16, 17, 33, 63, 64})
        for (int packed = 0; packed < 2; ++packed) {
          rattn_tree_params t = {s[0], s[1], s[2], s[3], s[4], dtype, nodes, 0.1f, 1e-6f, 0};
          size_t bytes = 1;
          const rattn_status st = rattn_tree_workspace_bytes(&t, packed, &bytes);
          if (st == RATTN_ERR_UNSUPPORTED) continue;
          CHECK(st == RATTN_OK);
          rattn::TreeDims td;
          td.N = s[0]; td.M = nodes; td.Hq = s[1]; td.Hkv = s[2]; td.D = s[3]; td.W = s[4]; td.G = s[1] / s[2];
          const rattn::TreePlan pl = rattn::tree_plan(td, dtype, packed);
          const int rows = nodes * td.G, per = pl.NW / pl.KG * 16 * pl.CT;
          CHECK(pl.CT >= 1 && pl.KG >= 1 && pl.NW % pl.KG == 0 && pl.nsplit >= 1 && pl.nsplit <= 128);
          CHECK((long long)pl.blocks * per >= rows && (long long)(pl.blocks - 1) * per < rows);
          CHECK(pl.nsplit == 1 || (pl.KG == 8 && pl.NW == 8));   // the forms in which work-groups share keys
          // a launch's grid, and a ticket and the partial sums for every work-group
          const long long grid = ((long long)td.N * td.Hkv + 7) / 8 * 8 * pl.blocks * pl.nsplit;
          CHECK(grid < (1ll << 31));
          const size_t cells = (size_t)td.N * td.Hkv * pl.blocks;
          CHECK(pl.bytes == bytes);
          CHECK(pl.nsplit == 1 ? bytes == 0 : pl.part_off >= 8 * cells && bytes == pl.part_off + cells * pl.nsplit * per * (2 * td.D + 4) * 4);
          const int before = rattn::g_stub_launches;
          void* scale = packed ? x : nullptr;
          CHECK(launched(rattn_tree_step(&t, x, x, x, ix, nullptr, ix, x, scale, x, scale, fx, nullptr, nullptr, x, bytes ? x : nullptr, bytes, nullptr)));
          CHECK(rattn::g_split == pl.nsplit);
          CHECK(launched(rattn_tree_step(&t, x, x, x, ix, ix, ix, x, scale, x, scale, fx, nullptr, nullptr, x, nullptr, 0, nullptr)));
          CHECK(rattn::g_split == 1);
          CHECK(launched(rattn_tree_commit(&t, x, x, ix, ix, ix, x, scale, x, scale, fx, nullptr)));
          CHECK(rattn::g_stub_launches == before + 3);
          if (bytes) {
            CHECK(rattn_tree_step(&t, x, x, x, ix, nullptr, ix, x, scale, x, scale, fx, nullptr, nullptr, x, x, bytes - 1, nullptr) == RATTN_ERR_WORKSPACE);
            CHECK(rattn::g_stub_launches == before + 3 && strlen(rattn_last_error()) > 0);
          }
          CHECK(rattn_tree_step(&t, x, x, x, ix, nullptr, ix, x, x, x, nullptr, fx, nullptr, nullptr, x, nullptr, 0, nullptr) == RATTN_ERR_INVALID_ARG);
          CHECK(rattn_tree_commit(&t, x, x, ix, ix, ix, x, nullptr, x, x, fx, nullptr) == RATTN_ERR_INVALID_ARG);
        }
  for (auto& s : shapes) {
    rattn_decode_params p = {s[0], s[1], s[2], s[3], s[4], 1, 0.1f, 1e-6f, 0};
    size_t bytes = 1;
    CHECK(rattn_decode_packed_workspace_bytes(&p, &bytes) == RATTN_OK);
    CHECK(launched(rattn_ring_pack(&p, x, x, x, x, x, x, nullptr)) && launched(rattn_ring_unpack(&p, x, x, x, x, x, x, nullptr)));
    CHECK(launched(rattn_decode_step_packed(&p, x, x, x, ix, x, x, x, x, fx, nullptr, nullptr, x, bytes ? x : nullptr, bytes, nullptr)));
    CHECK((rattn::g_split > 1) == (bytes > 0));
  }
  if (failures == 0) printf("ALL OK\n");
  return failures != 0;
}
