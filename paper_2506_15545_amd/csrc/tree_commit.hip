// The accepted path of a tree of drafted tokens enters the cache (Sec. 2.1: the window cache; Sec. 2.2 and Eq. 4: the lagged
// state): with L tokens on the path behind position p, tokens p - W .. p - W + L - 1 leave the window and are folded into the
// state, S += sum phi(k)^T v, and the path's last min(L, W) keys and values go to the slots (p + d) mod W, which are those that the
// leaving tokens had.  Where L > W the first of the path leave at once.
// One work-group per (sequence, KV head): the leaving rows as phi(k) and v in LDS, then the slots are free; a thread holds 4 x 4
// tiles of the state, requested before anything else, and adds the L outer products in the order of the tokens, in fp32 fused
// multiply-adds (L of them per entry of the state, which decode steps would have added one by one in the same order).  Over packed
// rings the tokens that leave at once (L > W) are folded in as given, where decode steps would have stored them in 8 bits first.
// Bound: HBM, the state once in and once out.  128 sequences of 8 KV heads, D = 128, paths of up to 6 tokens, packed rings of 512 slots:
// 19 us, 7 TB/s (a part of the state from the last-level cache); one sequence of 4 KV heads 4.4 us, a launch and three trips to memory.
#include "packed.hpp"
#include "ring_set.hpp"
#include "tree_nodes.hpp"

namespace rattn {

namespace {

template <typename IO, typename RT, int D, int NT>
__global__ __launch_bounds__(NT) void tree_commit_kernel(const IO* __restrict__ k, const IO* __restrict__ v,
                                                         const int32_t* __restrict__ parent, const int32_t* __restrict__ accepted,
                                                         const int32_t* __restrict__ pos, RT* __restrict__ k_ring,
                                                         RT* __restrict__ v_ring, float* __restrict__ state, int Hkv, int M, int W,
                                                         int phi, RingScales<RT> scales) {
  constexpr bool PACKED = sizeof(RT) == 1;
  constexpr int EPL = D / 64, SB = scale_bytes(D), NW = NT / 64, TILES = D * D / 16 / NT;
  extern __shared__ __align__(16) float lds[];   // phi(k) [L][D], v [L][D] of the leaving tokens
  const int g = blockIdx.x, n = blockIdx.y, lane = lane_id(), w = wave_id();
  const int acc = accepted[n], p = pos[n];
  if (acc < 0 || acc >= M || p < 0) return;
  const TreeNodes t = tree_nodes(lane < M ? parent[(size_t)n * M + lane] : -1, W, lane);
  const unsigned long long path = shfl64(t.anc, acc);   // parents come first: bits in the order of depth
  const int L = __popcll(path);
  const int first = max(0, W - p), E = L - first;   // leaving: j = first .. L - 1, token p - W + j
  const size_t pair = (size_t)n * Hkv + g;
  RT *kr = k_ring + pair * W * D, *vr = v_ring + pair * W * D;
  uint8_t* krs = PACKED ? scales.k + pair * W * SB : nullptr;
  uint8_t* vrs = PACKED ? scales.v + pair * W * SB : nullptr;
  auto drafted = [&](const IO* x, int node) { return x + (((size_t)n * M + node) * Hkv + g) * D; };
  auto node_at = [&](int depth) {   // the path's node at a depth: lane `depth`-th set bit
    const unsigned long long below = path & ((1ull << lane) - 1);
    const unsigned long long hit = __ballot((path >> lane & 1) && __popcll(below) == depth);
    return (int)__builtin_ctzll(hit);
  };
  // state tiles: 4 rows from f0, features d0 .. d0 + 3
  float* S = state + pair * D * D;
  const int d0 = (threadIdx.x % (D / 4)) * 4, f0 = (threadIdx.x / (D / 4)) * 4;
  constexpr int FSTEP = NT / (D / 4) * 4;
  f32x4_t s[TILES][4];
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      s[i][r] = E > 0 && p > W ? *reinterpret_cast<const f32x4_t*>(S + (size_t)(f0 + FSTEP * i + r) * D + d0) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  float *kf = lds, *vf = lds + (size_t)max(E, 0) * D;
  const int slot0 = p % W;
  for (int e = w; e < E; e += NW) {
    const int j = first + e;
    float x[EPL], y[EPL], f[EPL];
    if (j < W) {
      const int slot = j < W - slot0 ? slot0 + j : j - (W - slot0);
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        x[i] = ring_value(kr, krs, (size_t)slot * D + lane + 64 * i);
        y[i] = ring_value(vr, vrs, (size_t)slot * D + lane + 64 * i);
      }
    } else {
      const int node = node_at(j - W);
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        x[i] = io_traits<IO>::ld(drafted(k, node) + lane + 64 * i);
        y[i] = io_traits<IO>::ld(drafted(v, node) + lane + 64 * i);
      }
    }
    feature_row<EPL>(x, f, phi);
#pragma unroll
    for (int i = 0; i < EPL; ++i) { kf[e * D + lane + 64 * i] = f[i]; vf[e * D + lane + 64 * i] = y[i]; }
  }
  __syncthreads();   // the leaving rows are out of their slots
  for (int d = max(0, L - W) + w; d < L; d += NW) {
    const int node = node_at(d), slot = (int)(((long long)p + d) % W);
    const IO *kd = drafted(k, node), *vd = drafted(v, node);
    if constexpr (PACKED) {
      float x[EPL], y[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) { x[i] = io_traits<IO>::ld(kd + lane + 64 * i); y[i] = io_traits<IO>::ld(vd + lane + 64 * i); }
      pack_row<EPL>(x, reinterpret_cast<uint8_t*>(kr) + (size_t)slot * D, krs + (size_t)slot * SB, lane);
      pack_row<EPL>(y, reinterpret_cast<uint8_t*>(vr) + (size_t)slot * D, vrs + (size_t)slot * SB, lane);
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        kr[(size_t)slot * D + lane + 64 * i] = kd[lane + 64 * i];
        vr[(size_t)slot * D + lane + 64 * i] = vd[lane + 64 * i];
      }
    }
  }
  if (E <= 0) return;   // nothing leaves: the state stays as it is
  for (int e = 0; e < E; ++e) {
    const f32x4_t y = *reinterpret_cast<const f32x4_t*>(vf + e * D + d0);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(kf + e * D + f0 + FSTEP * i);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[i][r][c] = __builtin_fmaf(x[r], y[c], s[i][r][c]);
    }
  }
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) *reinterpret_cast<f32x4_t*>(S + (size_t)(f0 + FSTEP * i + r) * D + d0) = s[i][r];
}

template <typename IO, typename RT, int D>
void launch_commit(const TreeDims& td, const TreeTensors& t, const int32_t* accepted, hipStream_t st) {
  constexpr int NT = 256;
  const size_t bytes = (size_t)2 * td.M * D * 4;
  static const bool attr = hipFuncSetAttribute(reinterpret_cast<const void*>(tree_commit_kernel<IO, RT, D, NT>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, 2 * TREE_MAX_NODES * D * 4) == hipSuccess;
  (void)attr;
  tree_commit_kernel<IO, RT, D, NT><<<dim3(td.Hkv, td.N), NT, bytes, st>>>(
      (const IO*)t.k, (const IO*)t.v, t.parent, accepted, t.pos, (RT*)t.k_ring, (RT*)t.v_ring, (float*)t.state, td.Hkv, td.M, td.W,
      td.phi, RingScales<RT>((uint8_t*)t.k_scale, (uint8_t*)t.v_scale));
}

}  // namespace

void tree_commit(const TreeDims& td, int dtype, const TreeTensors& t, const int32_t* accepted, hipStream_t st) {
  ProfScope ps("tree_commit_kernel", st);
#define RATTN_COMMIT(IO)                                                          \
  do {                                                                            \
    if (t.k_scale) {                                                              \
      if (td.D == 64) launch_commit<IO, fp8_t, 64>(td, t, accepted, st);          \
      else launch_commit<IO, fp8_t, 128>(td, t, accepted, st);                    \
    } else {                                                                      \
      if (td.D == 64) launch_commit<IO, IO, 64>(td, t, accepted, st);             \
      else launch_commit<IO, IO, 128>(td, t, accepted, st);                       \
    }                                                                             \
  } while (0)
  if (dtype == 0) RATTN_COMMIT(float); else RATTN_COMMIT(bf16_t);
#undef RATTN_COMMIT
}

}  // namespace rattn
