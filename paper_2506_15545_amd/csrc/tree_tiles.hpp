// Tree steps of many rows (bf16; see tree_group.hpp for the mathematics): the keys come through LDS, where the waves of a work-group
// share them, each for 32 rows of its own.
//
// Few rows are bound by what a CU takes in; with many every wave would fetch the same ring again (192 pairs, W = 2048, 230 rows each:
// 2 GB through L1 at 64 bytes a cycle and CU), so here a tile of 64 keys is fetched once for a work-group's 128 rows.  The formulation is the
// layer forward's: S^T = K Q^T and O^T += V^T P^T with 32 x 32 tiles, a lane owns one row, and the accumulator registers of P^T are the
// second product's operand.  Nothing meets across waves: a wave has its rows' whole sums.  After the keys the same buffers hold
// phi(k) of the keys that leave, then the state, both as two bf16 terms.
// 24 sequences of 61 nodes, 40 query and 8 KV heads, D = 128, W = 2048 (half of the rings not full): 95 us, 380 TFLOP/s; fetching their
// own keys the waves take 164.  Bound by the way of a wave through its tiles (products, masks and exponentials, products): the
// work-groups with full rings, less than half of all, are about one for each CU, and the rest waits for them.  Over the whole launch
// the matrix units are busy for 29 % of it, the vector units for 38 %, LDS for 12 %.
#pragma once
#include "tree_group.hpp"

namespace rattn {

namespace {

constexpr int TILE_KEYS = 64;
constexpr int TILE_WAVES = TREE_TILE_WAVES, TILE_THREADS = 64 * TILE_WAVES;
// two buffers of a K and a V tile, and the gains of up to TILE_GAINS query heads of a KV head (more are read from memory): fetched
// with the rest of the inputs, where the end of a work-group waited for them (13 k of 196 k cycles)
constexpr int TILE_GAINS = 8;
// More work-groups than run at once (two on each of 256 CUs) take the sequences with the longest rings first: one that starts when
// others end is a short one.  (24 sequences of 100 to 4000 tokens, 8 KV heads, 305 rows, W = 2048, when a work-group took less:
// 96 us in order, 91 so; then the longest work-groups are what the rest waits for.)  A wave orders as many sequences as it has lanes:
// more than 64 come in the caller's order (72 of these 331 us, 297 where the caller has them in order of length).
constexpr unsigned TILE_AT_ONCE = 512;
template <int D> constexpr size_t tree_tile_lds() { return 4 * (size_t)TileGeom<D>::KT + 2 * TILE_GAINS * D * 4; }

// 16 bytes of a tile: chunk c (8 features) of row r
template <int D> __device__ __forceinline__ unsigned char* tile_chunk(unsigned char* tile, int r, int c) {
  return tile + r * TileGeom<D>::ROWB + ((c ^ swz<D>(r)) << 4);
}
// lds_row, lds_trp and lds_trn (mfma.hpp) of tiles whose address is known to lie in LDS: which of two buffers it is changes from
// tile to tile, and through a general pointer the compiler would ask where it points
typedef __attribute__((address_space(3))) unsigned char lds_byte;
// A wave's share of a tile (blocks blk0 .. blk0 + NBLK - 1 of 1024 bytes) straight from memory: whole tiles of rows that lie one
// behind the other (which `dl` is for) from a scalar base; of others the rows from nrows on are read as row nrows - 1
template <int D, int NBLK>
__device__ __forceinline__ void tile_fetch(const uint16_t* rows, size_t stride, int nrows, lds_byte* tile, int blk0, const DmaLane<D>& dl, int lane) {
  typedef TileGeom<D> G;
  if (nrows >= 64 && stride == D) {
#pragma unroll
    for (int i = 0; i < NBLK; ++i)
      dma16s(rows + (size_t)(blk0 + i) * G::RPB * stride, dl.off[i % G::NV], (unsigned)(size_t)(tile + (blk0 + i) * 1024));
  } else {
#pragma unroll
    for (int i = 0; i < NBLK; ++i) {
      const int r = (blk0 + i) * G::RPB + lane / G::CH, c = (lane % G::CH) ^ swz<D>(r);
      dma16(rows + (size_t)min(r, nrows - 1) * stride + c * 8, (unsigned)(size_t)(tile + (blk0 + i) * 1024));
    }
  }
}
template <int D> __device__ __forceinline__ bf16x8_t tile_row(const lds_byte* tile, const LaneOff<D>& lo, int R0, int c2) {
  return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8_t*>(tile + lo.row[c2] + R0 * TileGeom<D>::ROWB);
}
__device__ __forceinline__ bf16x8_t tile_tr2(const lds_byte* pa, const lds_byte* pb) {
  union { struct { s16x4_t lo, hi; } s; bf16x8_t v; } u;
  u.s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(pa));
  u.s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(pb));
  return u.v;
}
template <int D> __device__ __forceinline__ bf16x8_t tile_trp(const lds_byte* tile, const LaneOff<D>& lo, int K0, int ct) {
  return tile_tr2(tile + lo.trp[ct][0] + K0 * TileGeom<D>::ROWB, tile + lo.trp[ct][1] + K0 * TileGeom<D>::ROWB);
}
template <int D> __device__ __forceinline__ bf16x8_t tile_trn(const lds_byte* tile, const LaneOffN<D>& lo, int K0, int ct) {
  return tile_tr2(tile + lo.trn[ct][0] + K0 * TileGeom<D>::ROWB, tile + lo.trn[ct][1] + K0 * TileGeom<D>::ROWB);
}
template <int LANES> __device__ __forceinline__ float lanes_max(float x) {
  x = fmaxf(x, dpp_get<0xB1>(x));
  x = fmaxf(x, dpp_get<0x4E>(x));
  x = fmaxf(x, dpp_get<0x141>(x));
  return LANES == 16 ? fmaxf(x, dpp_get<0x140>(x)) : x;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
  x += dpp_get<0xB1>(x);
  x += dpp_get<0x4E>(x);
  x += dpp_get<0x141>(x);
  return LANES == 16 ? x + dpp_get<0x140>(x) : x;
}
__device__ __forceinline__ unsigned pack2(float x, float y) {
  typedef float pair_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector(pair_t{x, y}, bf16x2_t));
}
__device__ __forceinline__ void split2(float (&x)[8], bf16x8_t& hi, bf16x8_t& lo) {   // (see TreeMath::two_terms)
  float t[8];
  hi = pack_bf16x8(x);
  unpack_bf16x8(hi, t);
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = x[i] - t[i];
  lo = pack_bf16x8(t);
}

// SOFT: the softmax map.  (Left to run time, the choice cut every piece of phi out of the products around it.)
template <typename RT, int D, bool SOFT>
__global__ __launch_bounds__(TILE_THREADS, 2) void tree_tile_kernel(TreeArgs<bf16_t, RT> a) {
  constexpr bool PACKED = sizeof(RT) == 1;
  typedef TileGeom<D> TG;
  constexpr int KT = TG::KT, CH = TG::CH, SB = scale_bytes(D), NCT = D / 32, NC2 = D / 16;
  extern __shared__ __align__(16) unsigned char smem[];   // [2][K, V][64 rows]
  const int lane = lane_id(), w = wave_id(), r32 = lane & 31, hl = lane >> 5;
  const int W = a.W, G = a.G, M = a.M, Hkv = a.Hkv, rows_wg = 32 * TILE_WAVES;
  int block;
  const unsigned pairs = a.N * Hkv;
  unsigned pair = tree_pair(blockIdx.x, pairs, a.blocks, block);
  if (pair >= pairs) return;
  const int g = pair % Hkv;
  int n = pair / Hkv;
  if (a.N <= 64 && gridDim.x > TILE_AT_ONCE) {
    const int held = lane < a.N ? min(a.pos[lane], W) : -1;
    int before = 0;
    for (int i = 0; i < a.N; ++i) {
      const int other = __builtin_amdgcn_readlane(held, i);
      before += other > held || (other == held && i < lane);
    }
    n = (int)__builtin_ctzll(__ballot(lane < a.N && before == n));
    pair = (unsigned)n * Hkv + g;
  }
  const int p = a.pos[n], cnt = a.count ? min(a.count[n], M) : M;
  const int row0 = block * rows_wg, nrows = cnt * G;
  if (row0 >= nrows || p < 0) return;
  const int slot0 = p % W, nvalid = min(p, W);
  const RT *kr = a.k_ring + (size_t)pair * W * D, *vr = a.v_ring + (size_t)pair * W * D;
  const uint8_t* krs = PACKED ? a.ks + (size_t)pair * W * SB : nullptr;
  const uint8_t* vrs = PACKED ? a.vs + (size_t)pair * W * SB : nullptr;
  const bf16_t *kn = a.k + ((size_t)n * M * Hkv + g) * D, *vn = a.v + ((size_t)n * M * Hkv + g) * D;
  const size_t nstride = (size_t)Hkv * D;
  auto age = [&](int slot) { const int j = slot - slot0; return j + (j >> 31 & W); };

  // ---- this wave's rows: lane r32 has row r32's operand, features 16 c2 + 8 hl ..+7.  A negative scale goes to q's signs, so
  // that the largest score is that of the largest product
  const int up = lane < M ? a.parent[(size_t)n * M + lane] : -1;
  const int row = min(row0 + 32 * w + r32, nrows - 1), node_of = row / G;
  const bool live = row0 + 32 * w < nrows;   // (of the wave: the last work-group of a pair may have rows for some of its waves only)
  bf16x8_t q[NC2];
  {
    const bf16_t* qp = a.q + (((size_t)n * M + node_of) * a.Hq + g * G + row % G) * D + 8 * hl;
#pragma unroll
    for (int c2 = 0; c2 < NC2; ++c2) q[c2] = *reinterpret_cast<const bf16x8_t*>(qp + 16 * c2);
  }
  const float sc = __builtin_fabsf(a.scale) * LOG2E;
  const unsigned flip = a.scale < 0.f ? 0x80008000u : 0u;

  // ---- tiles: 64 ring slots each (the pairs start at different ones), then 64 drafted keys
  const int nring = (nvalid + TILE_KEYS - 1) / TILE_KEYS, ntile = nring + 1;
  const int rot = (int)(pair % (unsigned)max(nring, 1));
  auto ring_base = [&](int t) { const int s = t + rot; return (s < nring ? s : s - nring) * TILE_KEYS; };
  constexpr int PK = TILE_KEYS * CH / 2;          // packed: 16-byte pieces of codes in a tile
  constexpr int PT = PACKED ? (PK + TILE_THREADS - 1) / TILE_THREADS : 1;
  u32x4_t codes[PT];
  uint8_t code_scale[PT];
  // requests tile t for `buf`: rows behind the last one are read as that one (their weight is 0).  The codes of a packed ring pass
  // through registers, the keys' while the tile before has its first products and the values' while it has its second ones
  lds_byte* const lds = (lds_byte*)smem;
  const DmaLane<D> dma_lane = make_dma_lane<D>(lane, D);
  auto request_codes = [&](int t, const RT* ring, const uint8_t* scales) {
    if constexpr (PACKED) {
      const int base = ring_base(t), last = nvalid - 1 - base;
      const uint8_t *rc = reinterpret_cast<const uint8_t*>(ring) + (size_t)base * D, *rs = scales + (size_t)base * SB;   // (scalar)
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        const int x = threadIdx.x + i * TILE_THREADS;
        if (x < PK) {
          const unsigned r = min(x / (CH / 2), last), c = x % (CH / 2);
          codes[i] = *reinterpret_cast<const u32x4_t*>(rc + (r * D + 16 * c));
          code_scale[i] = rs[r * SB + c / 2];
        }
      }
    }
  };
  auto deliver_codes = [&](unsigned char* tile) {
    if constexpr (PACKED) {
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        const int x = threadIdx.x + i * TILE_THREADS;
        if (x < PK) {
          const int r = x / (CH / 2), c = x % (CH / 2);
          const float f = scale_of(code_scale[i]);
          uint32_t t8[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) unpack_bf16x4(codes[i][j], f, t8[2 * j], t8[2 * j + 1]);
          *reinterpret_cast<u32x4_t*>(tile_chunk<D>(tile, r, 2 * c)) = u32x4_t{t8[0], t8[1], t8[2], t8[3]};
          *reinterpret_cast<u32x4_t*>(tile_chunk<D>(tile, r, 2 * c + 1)) = u32x4_t{t8[4], t8[5], t8[6], t8[7]};
        }
      }
    }
  };
  auto request = [&](int t, int buf) {
    const bool nodes = t >= nring;
    if (PACKED && !nodes) {
      request_codes(t, kr, krs);
    } else {
      const uint16_t* ks_ = nodes ? kn : reinterpret_cast<const uint16_t*>(kr) + (size_t)ring_base(t) * D;
      const uint16_t* vs_ = nodes ? vn : reinterpret_cast<const uint16_t*>(vr) + (size_t)ring_base(t) * D;
      const size_t stride = nodes ? nstride : D;
      const int have = nodes ? cnt : nvalid - ring_base(t);
      constexpr int NBLK = TG::NB / TILE_WAVES;
      static_assert(NBLK % TG::NV == 0, "a wave's blocks start where the swizzle does");
      tile_fetch<D, NBLK>(ks_, stride, have, lds + buf * 2 * KT, NBLK * w, dma_lane, lane);
      tile_fetch<D, NBLK>(vs_, stride, have, lds + buf * 2 * KT + KT, NBLK * w, dma_lane, lane);
    }
  };
  // half way: packed keys are in `buf`, the values requested.  At the end: the tile is in `buf`, for this thread's part
  auto half_way = [&](int t, int buf) {
    if (PACKED && t < nring) {
      deliver_codes(smem + buf * 2 * KT);
      request_codes(t, vr, vrs);
    }
  };
  auto deliver = [&](int t, int buf) {
    if (PACKED && t < nring) deliver_codes(smem + buf * 2 * KT + KT);
    else wait_vmem();
  };
  float* glds = reinterpret_cast<float*>(smem + 4 * KT);   // [2][G][D]
  const bool staged = G <= TILE_GAINS;
  constexpr int NG = TILE_GAINS * D / TILE_THREADS;
  float gain[2][NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int e = threadIdx.x + i * TILE_THREADS;
    gain[0][i] = gain[1][i] = 0.f;
    if (staged && e < G * D) {
      if (a.gs) gain[0][i] = a.gs[g * G * D + e];
      if (a.gr) gain[1][i] = a.gr[g * G * D + e];
    }
  }
  request(0, 0);
  const TreeNodes node = tree_nodes(up, W, lane);
  const unsigned long long anc = shfl64(node.anc, node_of), left = shfl64(node.left, node_of);
  const int depth = __popcll(anc) - 1;
  int dmax = depth;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) dmax = max(dmax, __shfl_xor(dmax, s));
  dmax = __builtin_amdgcn_readfirstlane(dmax);
  int dall = lane < cnt ? node.depth() : 0;   // of the sequence's nodes: all waves agree on it
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) dall = max(dall, __shfl_xor(dall, s));
  dall = __builtin_amdgcn_readfirstlane(dall);
  // maximum and sum of phi(q), while the first tile is on its way
  float fm = 0.f, fz = 1.f;
  if (SOFT && p >= W - dall) {
    float x[8], s = 0.f;
    fm = -INFINITY;
#pragma unroll
    for (int c2 = 0; c2 < NC2; ++c2) {
      unpack_bf16x8(q[c2], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) fm = fmaxf(fm, x[i]);
    }
    fm = half_max(fm);
#pragma unroll
    for (int c2 = 0; c2 < NC2; ++c2) {
      unpack_bf16x8(q[c2], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += fast_exp2((x[i] - fm) * LOG2E);
    }
    fz = 1.f / half_sum(s);
  }
#pragma unroll
  for (int c2 = 0; c2 < NC2; ++c2) q[c2] = __builtin_bit_cast(bf16x8_t, __builtin_bit_cast(u32x4_t, q[c2]) ^ flip);

  // ---- softmax branch
  const LaneOff<D> lo = make_lane_off<D>(lane);
  f32x16_t acc[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[ct][i] = 0.f;
  float m = -1.0e30f, l = 0.f, lsum[4] = {0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  half_way(0, 0);
  deliver(0, 0);
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int e = threadIdx.x + i * TILE_THREADS;
    if (staged && e < G * D) { glds[e] = gain[0][i]; glds[G * D + e] = gain[1][i]; }
  }
  __syncthreads();
#pragma unroll 1
  for (int t = 0; t < ntile; ++t) {
    if (t + 1 < ntile) request(t + 1, buf ^ 1);
    const lds_byte *K = lds + buf * 2 * KT, *V = K + KT;
    const bool nodes = t >= nring;
    const int base = nodes ? 0 : ring_base(t);
    if (live) {
      // both halves of the tile together: one maximum, and the products of either fill the other's waits
      f32x16_t s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
#pragma unroll
      for (int c2 = 0; c2 < NC2; ++c2)
#pragma unroll
        for (int h = 0; h < 2; ++h) s[h] = mfma32(tile_row<D>(K, lo, 32 * h, c2), q[c2], s[h]);
      // operand reads four products ahead (left to itself the compiler waits for every read right in front of its product)
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < 2 * NC2; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      if constexpr (PACKED) { if (t + 1 < ntile) half_way(t + 1, buf ^ 1); }
      if (nodes) {
        const unsigned long long see = (anc & ~left) >> (4 * hl);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[h][i] = (unsigned)(see >> (32 * h)) >> (8 * (i / 4) + i % 4) & 1 ? s[h][i] : -INFINITY;
      } else {
        const int youngest = base < slot0 && slot0 < base + TILE_KEYS ? 0 : age(base);
        if (base + TILE_KEYS > nvalid || youngest <= dmax) {   // wave-uniform
          const int s0 = opaque(base + 4 * hl);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int slot = s0 + 32 * h + 8 * (i / 4) + i % 4;
              s[h][i] = (slot < nvalid) & (age(slot) > depth) ? s[h][i] : -INFINITY;
            }
        }
      }
      float mx = fmaxf(s[0][15], s[1][15]);
#pragma unroll
      for (int i = 0; i < 15; ++i) mx = max3(mx, s[0][i], s[1][i]);
      mx = half_max(mx) * sc;
      if (__any(mx > m + 8.f)) {   // (a running maximum stays while no score is far above it)
        const float top = fmaxf(m, mx), alpha = fast_exp2(m - top);
        m = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) lsum[i] *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) acc[ct] *= alpha;
      }
      // The second products in explicit order: operands are read three ahead, and the next eight keys' probabilities are formed
      // between the products of the eight before (all of a half's ahead of its products: 99 -> 95 us).  Of the two waves of a SIMD the
      // one that is here goes first, so that the other's first products fill what it leaves (101 -> 95; the first products preferred
      // as well 97).
      // Two bf16 terms for the probabilities, as in the direct kernel, so that a sequence's result does not get worse in a larger
      // batch: with one the output is off by 2.1e-3 of its norm, with two by the 1.66e-3 of its own rounding (81 | 95 us).
      __builtin_amdgcn_s_setprio(1);
      constexpr int AHEAD = 3;   // operands that are read ahead
      bf16x8_t v[AHEAD];
      u32x4_t ph[2], pl[2];
      auto read = [&](int x) { v[x % AHEAD] = tile_trp<D>(V, lo, 16 * (x / NCT), x % NCT); };
      auto pair_of = [&](int g, int j) {   // keys 2j and 2j + 1 of the g-th eight of this lane's row
        float p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          p[i] = fast_exp2(__builtin_fmaf(s[g / 2][8 * (g % 2) + 2 * j + i], sc, -m));
          lsum[2 * (j & 1) + i] += p[i];
        }
        const unsigned hi = (unsigned)opaque((int)pack2(p[0], p[1]));   // (else the compiler rounds each alone once more)
        ph[g % 2][j] = hi;
        pl[g % 2][j] = pack2(p[0] - __uint_as_float(hi << 16), p[1] - __uint_as_float(hi & 0xffff0000u));
      };
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) read(x);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) pair_of(0, j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < 4 * NCT; ++x) {
        const int g = x / NCT, ct = x % NCT;
        acc[ct] = mfma32(v[x % AHEAD], __builtin_bit_cast(bf16x8_t, pl[g % 2]), acc[ct]);
        acc[ct] = mfma32(v[x % AHEAD], __builtin_bit_cast(bf16x8_t, ph[g % 2]), acc[ct]);
        if (x + AHEAD < 4 * NCT) read(x + AHEAD);
        if (g < 3) {
#pragma unroll
          for (int j = 4 / NCT * ct; j < 4 / NCT * (ct + 1); ++j) pair_of(g + 1, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    if (PACKED && !live && t + 1 < ntile) half_way(t + 1, buf ^ 1);
    if (t + 1 < ntile) deliver(t + 1, buf ^ 1);
    __syncthreads();
    buf ^= 1;
  }
  l = half_sum((lsum[0] + lsum[1]) + (lsum[2] + lsum[3]));

  // ---- linear branch.  phi(q) is formed a piece at a time
  f32x16_t acr[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) acr[ct][i] = 0.f;
  if (p >= W - dall) {
#pragma unroll
    for (int c2 = 0; c2 < NC2; ++c2) q[c2] = __builtin_bit_cast(bf16x8_t, __builtin_bit_cast(u32x4_t, q[c2]) ^ flip);
    const float least = a.phi == PHI_RELU ? 0.f : -INFINITY;   // of the other two maps' values
    auto feature = [&](int c2, bf16x8_t& hi, bf16x8_t& lw) {
      float x[8];
      u32x4_t raw = __builtin_bit_cast(u32x4_t, q[c2]);   // (not what a loop would keep of all pieces in registers)
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = (unsigned)opaque((int)raw[i]);
      unpack_bf16x8(__builtin_bit_cast(bf16x8_t, raw), x);
      if constexpr (SOFT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fast_exp2((x[i] - fm) * LOG2E) * fz;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaxf(x[i], least);
      }
      split2(x, hi, lw);
    };
    // keys that leave, 32 at a time: ring tokens by age 0 .. min(dall, W - 1), then (paths longer than the window) drafted ones
    const int nage = min(dall + 1, W), sets = (nage + 31) / 32, all = sets + (dall >= W ? (cnt + 31) / 32 : 0);
    unsigned char *Fh = smem, *Fl = smem + KT / 2, *Vt = smem + KT;
#pragma unroll 1
    for (int x = 0; x < all; ++x) {
      // a thread has eight features of a row
      for (int e = threadIdx.x; e < 32 * CH; e += TILE_THREADS) {
        const int r = e / CH, c = e % CH, t = 32 * x + r;
        u32x4_t kb = {0, 0, 0, 0}, vb = {0, 0, 0, 0};
        if (x < sets) {
          if (t < nage && t >= W - p) {
            const size_t slot = t < W - slot0 ? slot0 + t : t - (W - slot0);
            if constexpr (PACKED) {
              const u32x2_t k8 = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint8_t*>(kr) + slot * D + 8 * c);
              const u32x2_t v8 = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint8_t*>(vr) + slot * D + 8 * c);
              const float fk = scale_of(krs[slot * SB + c / 4]), fv = scale_of(vrs[slot * SB + c / 4]);
              uint32_t y[8];
              unpack_bf16x4(k8[0], fk, y[0], y[1]);
              unpack_bf16x4(k8[1], fk, y[2], y[3]);
              unpack_bf16x4(v8[0], fv, y[4], y[5]);
              unpack_bf16x4(v8[1], fv, y[6], y[7]);
              kb = u32x4_t{y[0], y[1], y[2], y[3]};
              vb = u32x4_t{y[4], y[5], y[6], y[7]};
            } else {
              kb = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const uint16_t*>(kr) + slot * D + 8 * c);
              vb = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const uint16_t*>(vr) + slot * D + 8 * c);
            }
          }
        } else if (t - 32 * sets < cnt) {
          kb = *reinterpret_cast<const u32x4_t*>(kn + (size_t)(t - 32 * sets) * nstride + 8 * c);
          vb = *reinterpret_cast<const u32x4_t*>(vn + (size_t)(t - 32 * sets) * nstride + 8 * c);
        }
        float f[8];
        unpack_bf16x8(__builtin_bit_cast(bf16x8_t, kb), f);
        if constexpr (SOFT) {
          float mx = f[0], s = 0.f;
#pragma unroll
          for (int i = 1; i < 8; ++i) mx = fmaxf(mx, f[i]);
          mx = lanes_max<CH>(mx);
#pragma unroll
          for (int i = 0; i < 8; ++i) { f[i] = fast_exp2((f[i] - mx) * LOG2E); s += f[i]; }
          s = 1.f / lanes_sum<CH>(s);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= s;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = fmaxf(f[i], least);
        }
        bf16x8_t hi, lw;
        split2(f, hi, lw);
        *reinterpret_cast<bf16x8_t*>(tile_chunk<D>(Fh, r, c)) = hi;
        *reinterpret_cast<bf16x8_t*>(tile_chunk<D>(Fl, r, c)) = lw;
        *reinterpret_cast<u32x4_t*>(tile_chunk<D>(Vt, r, c)) = vb;
      }
      __syncthreads();
      if (live) {
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        bf16x8_t hi, lw, kh = tile_row<D>(lds, lo, 0, 0), kl = tile_row<D>(lds + KT / 2, lo, 0, 0);
        feature(0, hi, lw);
#pragma unroll
        for (int c2 = 0; c2 < NC2; ++c2) {   // the next piece of phi(q), and of phi(k), behind this one's products
          s = mfma32(kl, hi, s);
          s = mfma32(kh, lw, s);
          s = mfma32(kh, hi, s);
          if (c2 + 1 < NC2) {
            kh = tile_row<D>(lds, lo, 0, c2 + 1);
            kl = tile_row<D>(lds + KT / 2, lo, 0, c2 + 1);
            feature(c2 + 1, hi, lw);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        // which of the 32 keys this lane's row has left behind, from bit 4 hl on
        auto below = [](int k) { return k <= 0 ? 0u : k >= 32 ? ~0u : (1u << k) - 1; };
        unsigned see = x < sets ? below(min(depth, W - 1) + 1 - 32 * x) & ~below(W - p - 32 * x) : (unsigned)(left >> (32 * (x - sets)));
        see >>= 4 * hl;
        float y[16], z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = see >> (8 * (i / 4) + i % 4) & 1 ? s[i] : 0.f;
        bf16x8_t ph[2] = {pack_bf16x8(y), pack_bf16x8(y + 8)}, pl[2];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          unpack_bf16x8(ph[kk], z + 8 * kk);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[8 * kk + i] = y[8 * kk + i] - z[8 * kk + i];
          pl[kk] = pack_bf16x8(z + 8 * kk);
        }
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            const bf16x8_t v = tile_trp<D>(lds + KT, lo, 16 * kk, ct);
            acr[ct] = mfma32(v, pl[kk], acr[ct]);
            acr[ct] = mfma32(v, ph[kk], acr[ct]);
          }
      }
      __syncthreads();
    }
    // the state as two terms [feature][value]
    if (p > W) {
      unsigned char *Sh = smem, *Sl = smem + D * TG::ROWB;
      const float* S = a.state + (size_t)pair * D * D;
      constexpr int NE = D * CH / TILE_THREADS, BATCH = NE < 4 ? NE : 4;
#pragma unroll 1
      for (int e0 = threadIdx.x; e0 < D * CH; e0 += BATCH * TILE_THREADS) {
        f32x4_t u[BATCH][2];   // (the batch is requested before any of it is worked on)
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
#pragma unroll
          for (int k = 0; k < 2; ++k) u[b][k] = *reinterpret_cast<const f32x4_t*>(S + (size_t)(e0 + b * TILE_THREADS) * 8 + 4 * k);
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
          const int e = e0 + b * TILE_THREADS, r = e / CH, c = e % CH;
          float x[8] = {u[b][0][0], u[b][0][1], u[b][0][2], u[b][0][3], u[b][1][0], u[b][1][1], u[b][1][2], u[b][1][3]};
          bf16x8_t hi, lw;
          split2(x, hi, lw);
          *reinterpret_cast<bf16x8_t*>(tile_chunk<D>(Sh, r, c)) = hi;
          *reinterpret_cast<bf16x8_t*>(tile_chunk<D>(Sl, r, c)) = lw;
        }
      }
      __syncthreads();
      if (live) {
        const LaneOffN<D> ln = make_lane_off_n<D>(lane);
        bf16x8_t hi, lw;
        feature(0, hi, lw);
#pragma unroll
        for (int c2 = 0; c2 < NC2; ++c2) {   // operands, the next piece of phi(q), products
          bf16x8_t sh[NCT], sl[NCT];
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) {
            sh[ct] = tile_trn<D>(lds, ln, 16 * c2, ct);
            sl[ct] = tile_trn<D>(lds + D * TG::ROWB, ln, 16 * c2, ct);
          }
          const bf16x8_t h0 = hi, l0 = lw;
          if (c2 + 1 < NC2) feature(c2 + 1, hi, lw);
#pragma unroll
          for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) acr[ct] = mfma32(k == 0 ? sl[ct] : sh[ct], k == 1 ? l0 : h0, acr[ct]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  const bool mine = row0 + 32 * w + r32 < nrows;
  if (!live) return;
  // ---- combination (Sec. 3.2)
  const float inv = 1.f / l;
  float s1 = 0.f, s2 = 0.f, z = inv * 0.f;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      acc[ct][i] *= inv;
      s1 += acc[ct][i] * acc[ct][i];
      s2 += acr[ct][i] * acr[ct][i];
      z += acc[ct][i] * 0.f + acr[ct][i] * 0.f;
    }
  s1 = half_sum(s1);
  s2 = half_sum(s2);
  z = half_sum(z);
  const bool bad = mine && !(z == 0.f);
  if (mine && !bad) {
    const float r1 = rsqrtf(s1 / D + a.eps), r2 = rsqrtf(s2 / D + a.eps);
    const int head = g * G + row % G;
    bf16_t* o = a.o + (((size_t)n * M + node_of) * a.Hq + head) * D + 4 * hl;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) { acc[ct] *= r1; acr[ct] *= r2; }
    auto gains = [&](const float* gp, f32x16_t (&x)[NCT]) {
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          f32x4_t y;
          __builtin_memcpy(&y, gp + 32 * ct + 8 * b, 16);   // (aligned like a float)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[ct][4 * b + i] *= y[i];
        }
    };
    const int hd = (row % G) * D + 4 * hl;
    if (a.gs) { if (staged) gains(glds + hd, acc); else gains(a.gs + g * G * D + hd, acc); }
    if (a.gr) { if (staged) gains(glds + G * D + hd, acr); else gains(a.gr + g * G * D + hd, acr); }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        store4(o + 32 * ct + 8 * b, f32x4_t{acc[ct][4 * b] + acr[ct][4 * b], acc[ct][4 * b + 1] + acr[ct][4 * b + 1],
                                            acc[ct][4 * b + 2] + acr[ct][4 * b + 2], acc[ct][4 * b + 3] + acr[ct][4 * b + 3]});
  }
  unsigned long long again = __ballot(bad && hl == 0);
  while (again) {
    const int from = __builtin_ctzll(again);
    again &= again - 1;
    const int r = __shfl(row, from), i = r / G;
    tree_row_again<bf16_t, RT, D>(a, n, g, r, shfl64(node.anc, i), shfl64(node.left, i), lane);
  }
}

template <typename RT, int D, bool SOFT>
void launch_tree_tile(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  const size_t bytes = tree_tile_lds<D>();
  static const bool attr = hipFuncSetAttribute(reinterpret_cast<const void*>(tree_tile_kernel<RT, D, SOFT>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
  (void)attr;
  tree_tile_kernel<RT, D, SOFT><<<(unsigned)tree_grid(td, pl), TILE_THREADS, bytes, st>>>(tree_args<bf16_t, RT>(td, t, pl));
}
template <typename RT, int D>
void pick_tree_tile(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  if (td.phi == PHI_SOFTMAX) launch_tree_tile<RT, D, true>(td, t, pl, st);
  else launch_tree_tile<RT, D, false>(td, t, pl, st);
}

}  // namespace

}  // namespace rattn
