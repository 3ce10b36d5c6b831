// Shape planning shared by the C ABI and the kernel launchers: which shapes the matrix-core kernels take, how many
// chunk states a call needs and how large its scratch areas are.  Host arithmetic only (nothing here touches a
// device), so this file is also part of the CPU build of the host layer that runs under the sanitizers.
#include "kernels.hpp"

namespace rattn {

// dm: the dimensions the kernels would see, i.e. with the sequence length rounded up to whole tiles
bool fast_fwd_supported(const LayerDims& dm, int dtype) {
  if (dtype != 1 || dm.T % 128 != 0) return false;
  if (!(dm.scale > 0.f)) return false;
  // Windows below 8 keys stay on the general path: their softmax rows are close to one-hot, so the backward's
  // dS = P (dP - delta) is a near-cancellation (exact for W = 1) that bf16 operands turn into rounding noise
  // above the gradient tolerance (measured: worst element 4 % of RMS at W = 2, 3 % at W = 4, 2.5 % from W = 8 on)
  if (dm.W < 8) return false;
  return true;
}

int generic_chunk(const LayerDims& dm, int Tp) {
  const long long groups = (long long)((dm.T + 15) / 16) * dm.Hq * dm.B;
  return Tp > 64 && Tp <= (groups <= 256 ? 320 : groups <= 512 ? 224 : 128) ? Tp : 64;
}

FastFwdPlan fast_fwd_plan(const LayerDims& dm) {
  FastFwdPlan p;
  const int wt = dm.W >= dm.T ? dm.T : dm.W;
  p.W = (wt + 63) / 64 * 64;
  p.gap = p.W - wt;
  p.base = p.W % 128;
  p.nstf = dm.T / 128 - (p.W + 127) / 128;
  if (p.nstf < 0) p.nstf = 0;
  // chunk-local products of `ckeys` keys each (128 unless the caller asks for `chunk` = 64); with 128 and states at the 64
  // alignment the first product covers the 64 keys in front of state 0
  p.ckeys = dm.chunk_req == 64 ? 64 : 128;
  p.nchunks = p.nstf > 0 ? (p.nstf - 1) * (128 / p.ckeys) + (p.base > 0 ? 1 : 0) : 0;
  p.u_bytes = (size_t)dm.B * dm.Hkv * p.nchunks * dm.D * dm.D * 4;
  p.state_bytes = (size_t)dm.B * dm.Hkv * p.nstf * dm.D * dm.D * 2;
  return p;
}

ChunkPlan chunk_plan(const LayerDims& dm, int P, int R, int Tc) {
  ChunkPlan c = {0, 0, 0, 0, 0, 0};
  const FastFwdPlan pl = fast_fwd_plan(dm);
  const long long bg = (long long)dm.B * dm.Hkv;
  c.end = P + Tc - dm.W;
  // Every call whose forward reads states that hold a key shares its products; with a carried state every call does.  (One
  // sequence of one KV head, 128 new tokens, ring of 128: separate launches 30.1 us, shared 26.2.)
  if (pl.nstf <= 0 || R + Tc <= dm.W) return c;
  c.head = pl.base > 0 ? 1 : 0;
  // (the last state is in front of the last row that leaves the window: at least one product follows it)
  const int rest = c.end - 64 * c.head, n = (rest + 127) / 128;
  // Products of 64 rows where those of 128 leave half of the chip idle, as long as the scan's chain stays short: 32/8 heads,
  // W = 512, products of 64 | 128 rows: 700 tokens 41.2 | 41.9 us, 1024 41.4 | 42.7, 1500 50.6 | 52.3, two sequences of 1500
  // 74.9 | 71.9; 16/2 heads, 2048 tokens (16 products of 128 rows in a chain) 41.8 | 40.8.
  c.ckeys = dm.chunk_req == 64 || (n <= 12 && n * bg <= 128) ? 64 : 128;
  c.nprod = c.head + (rest + c.ckeys - 1) / c.ckeys;
  // Chains of 64 keys as in the prefill export, of 128 where that has more tiles than two work-groups per CU (export_plan): another
  // 64 registers and additions, 4 x 2048 tokens after 2048, 8 KV heads 134.6 -> 137.8 us
  c.piece = (R + Tc - dm.W + 63) / 64 * bg > 512 ? c.ckeys : 64;
  c.u_bytes = (size_t)bg * c.nprod * dm.D * dm.D * 4;
  return c;
}

FastBwdPlan fast_bwd_plan(const LayerDims& dm) {
  FastBwdPlan p;
  p.fwd = fast_fwd_plan(dm);
  const int Tp = dm.T - p.fwd.W;
  p.nk = Tp > 0 ? (Tp + 127) / 128 : 0;
  // reverse-time chunk products: query rows t' in [128, Tp) in pieces of ckeys
  p.nrchunks = Tp > 128 ? (Tp - 128 + p.fwd.ckeys - 1) / p.fwd.ckeys : 0;
  // A work-group visits the query heads of its product in turn; where there are few products the heads are split over two
  // or four work-groups, as long as those fit on the chip together (two per CU).  2 x 1000 tokens, 4 KV heads of 4 query
  // heads: 24 -> 96 work-groups, 19 -> 8.5 us.  Every further product is written, and read again in the scan's one chain of
  // additions per element.  So a doubling must take at least as many keys (heads x keys of a product) off the longest
  // work-group as it adds products, and eight times the products that it adds to a chain.  Backward at D = 128, one | two |
  // four work-groups: 64 products of 4 heads in chains of 8 96.6 | 90.2 | 89.7 us, of 16 97.1 | 91.2 | 92.4; 96 products of
  // 4 heads 102.6 | 97.7 | 99.3; 128 of 2 heads 82.5 | 81.1, of 3 98.6 | 98.8, of 8 in chains of 8 228.7 | 216.6 | 215.0, of
  // 32 224.8 | 215.4 | 217.1; 192 of 2 heads 88.7 | 89.6, of 3 124.9 | 127.0; 256 of 4 heads 228.6 | 226.5 | 243.7.
  const long long chains = (long long)dm.Hkv * dm.B;
  auto longest = [&](int s) { return (long long)((dm.G + s - 1) / s) * p.fwd.ckeys; };   // keys
  p.rsplit = 1;
  for (int s = 1; s < 4 && 2 * s <= dm.G && chains * p.nrchunks * 2 * s <= 512; s *= 2) {
    const long long added = (long long)p.nrchunks * s, fewer = longest(s) - longest(2 * s);
    if (chains * added > fewer || 8 * added > fewer) break;
    p.rsplit = 2 * s;
  }
  const int heads = (dm.G + p.rsplit - 1) / p.rsplit;
  p.rsplit = (dm.G + heads - 1) / heads;   // 5, 6 or 9 heads: the fourth work-group would have none
  const int nrev = p.nrchunks * p.rsplit, nch = p.fwd.nchunks > nrev ? p.fwd.nchunks : nrev;
  p.u_bytes = (size_t)dm.B * dm.Hkv * (nch > 0 ? nch : 0) * dm.D * dm.D * 4;
  p.rstate_bytes = (size_t)dm.B * dm.Hkv * p.nk * dm.D * dm.D * 2;
  p.RB = 4 * (dm.T / 128) * dm.B;  // one gain-gradient partial per wave of the dq kernel
  // The dk/dv kernel holds one work-group per CU (two at D = 64), which visits the G query heads of its key tile in turn.  With few key
  // tiles the heads are split over several work-groups (partial sums in fp32, added in order): the split with the fewest
  // head visits on the busiest CU, where a work-group costs about half a visit on top of its own.
  const long long tiles = (long long)(dm.T / 128) * dm.Hkv * dm.B, slots = dm.D == 64 ? 512 : 256;
  p.nsplit = 1;
  double best = 0.0;
  for (int s = 1; s <= dm.G; ++s) {
    const int hps = (dm.G + s - 1) / s, used = (dm.G + hps - 1) / hps;
    if (used != s) continue;   // the same heads per work-group with fewer of them
    const double cost = (double)((tiles * s + slots - 1) / slots) * (hps + 0.5) + (s > 1 ? 0.5 : 0.0);
    if (s == 1 || cost < best) { best = cost; p.nsplit = s; }
  }
  p.dkv_part_bytes = p.nsplit > 1 ? (size_t)2 * p.nsplit * dm.B * dm.T * dm.Hkv * dm.D * 4 : 0;
  return p;
}

DecodeSplit decode_split(const DecodeDims& dd, int esize) {
  // A work-group of eight waves for every 64 KB of rings, up to 128 of them in all: more are bound by what the memory delivers.
  // Captured steps in us, one work-group per pair (16 waves) | as split, bf16, D = 128, full rings:
  //   4 pairs, W = 512 11.1 | 9.0;  1024 14.5 | 9.5;  2048 23.4 | 10.8;  4096 41.0 | 12.1;  16, 512 11.2 | 9.3;  2048 23.6 | 11.7
  //   32, 512 10.9 | 9.5;  2048 24.7 | 13.4;  64, 512 12.1 | 11.4;  1024 16.1 | 14.3;  2048 25.7 | 19.6;  4096 44.2 | 29.5
  //   D = 64, 4 pairs, W = 1024 9.6 | 7.8;  4096 25.2 | 9.4;  fp32, 4 pairs, W = 512 17.9 | 10.6;  16 pairs, 4096 91.7 | 21.5
  // Rings that are not full, 100 tokens 7.3 | 6.9 (4 pairs), 7.5 | 7.1 (64);  380, one work-group of eight waves, 9.4 | 8.7, 9.5 | 9.0;
  // slower by up to 3 % remain D = 64, 4 pairs, 550 - 768 tokens 7.6 | 7.8 and fp32, 100 tokens 9.0 | 9.3.
  // How many were compared eagerly, when the host took 8 of each step and 9.5 with a workspace (now 3.6 and 3.9); one | 2 | 4 | 8 | 16:
  //   4 pairs, W = 512 12.0 | 10.7 | 9.5 | 9.5 | 10.3;  W = 2048 25.0 | 18.6 | 13.4 | 11.5 | 11.5;  W = 4096 42.8 | 29.0 | 18.6 | 13.7 | 12.7
  //   16 pairs, W = 1024 15.9 | 13.4 | 11.0 | 11.0 | 12.4;  64, W = 512 14.3 | 13.3 | 13.4 | 15.1 | 26.5
  //   128 pairs, W = 512 16.1 | 16.8 | 17.4;  W = 2048 38.1 | 34.1 | 34.2 | 39.4 (not taken: rings with 100 - 400 tokens
  //   10.7 | 11.6);  192, W = 2048 35.5 | 39.2 | 39.6
  //   32 pairs, D = 64, W = 512 7.8 | 9.9;  4 pairs, fp32, W = 512 18.5 | 15.4 | 12.6 | 11.2 | 11.8
  // Packed rings (work to unpack for each byte): 32 KB each, four or more, up to 256 of them, or 512 of 128 KB.  One | as split, bf16,
  // D = 128: 4 pairs, W = 512 12.2 | 9.8;  1024 15.5 | 10.5;  2048 22.3 | 11.8;  4096 35.3 | 13.1;  32, 512 13.2 | 11.1;  2048 24.1 |
  // 15.0;  64, 512 13.4 | 12.2;  2048 24.7 | 16.2;  128, 2048 26.0 | 22.7.  Two are as slow as one (12.2 | 11.8, 24.1 | 24.2); not
  // taken: 128 pairs, W = 512 14.5 | 15.0;  192, 2048 32.9 | 34.8.  D = 64, 64 pairs, W = 2048 14.5 | 11.7;  512 8.2 | 9.0 (not taken)
  DecodeSplit s = {1, dd.W, 0, 0};
  const long long pairs = (long long)dd.N * dd.Hkv, ring = 2ll * dd.W * dd.D * esize;
  const bool packed = esize == 1;
  const int share = packed ? 32 << 10 : 64 << 10, least = packed ? 4 : 2, most = packed ? ring >= 512 << 10 && pairs > 64 ? 512 : 256 : 128;
  if (dd.G > 16 || ring < 4 * share) return s;
  s.n = DEC_MAX_SPLIT;
  while (s.n > 1 && (ring / s.n < share || pairs * s.n > most)) s.n /= 2;
  if (s.n < least) { s.n = 1; return s; }
  s.rows = (int)(share * (long long)dd.W / ring);
  s.part_off = ((size_t)pairs * 8 + 255) / 256 * 256;
  s.bytes = s.part_off + (size_t)pairs * s.n * dd.G * (2 * dd.D + 4) * 4;
  return s;
}

ExportPlan export_plan(const LayerDims& dm) {
  ExportPlan pl;
  pl.Tp = dm.T > dm.W ? dm.T - dm.W : 0;
  // Segments of 64-key tiles, enough of them for two work-groups on every CU: more only add partial states to write
  // and read back (each as large as 128 keys and values of a bf16 head)
  const int tiles = (pl.Tp + 63) / 64, most = 512 / (dm.B * dm.Hkv) > 1 ? 512 / (dm.B * dm.Hkv) : 1;
  const int per = (tiles + most - 1) / most;
  pl.seg_len = 64 * per;
  pl.nseg = per > 0 ? (tiles + per - 1) / per : 0;
  pl.partial_bytes = (size_t)dm.B * dm.Hkv * pl.nseg * dm.D * dm.D * sizeof(float);
  return pl;
}

TreePlan tree_plan(const TreeDims& td, int dtype, bool packed) {
  TreePlan p = {1, 8, 8, 1, 1, 6, 0, 0, 0};
  const int rows = td.M * td.G, keys = dtype == 0 ? 16 : 32, pieces = td.D / keys + 1;
  const int sets = (int)((td.W + (keys - 1ll)) / keys) + (td.M + keys - 1) / keys;
  const long long pairs = (long long)td.N * td.Hkv;
  // Keys through LDS where waves that fetch them themselves would be more than the chip holds at once (work-groups of 64 rows, one per
  // CU).  us, direct | tiles, bf16, full rings, D = 128, W = 512 and 2048: 96 pairs of 128 rows 25.5 | 37.5, 56.9 | 75.8; of 256
  // 48.3 | 41.7, 108 | 80; 128 of 128 rows 26.0 | 37.8, 58.9 | 76.7; 136 of 128 44.4 | 38.1, 106 | 77; 192 of 96 45.3 | 38.5, 107 |
  // 77; 64 of 256 28.6 | 40.0, 55.1 | 78.8; of 512 51.9 | 44.5, 106 | 83.  D = 64: 64 of 256 17.6 | 26.8, 35.1 | 54.5; of 512 31.4 |
  // 28.9, 67.6 | 57.7 (packed: 17.7 | 29.6, 39.2 | 69.4; of 512 31.3 | 31.7, 72.8 | 71.0).  Packed rings of D = 128, which they unpack
  // on the way (at the cost of registers), from twice as many on: 192 of 128 44.9 | 47.3, 105 | 110; 256 of 128 48.7 | 49.6, 106 | 112;
  // 320 of 128 65.1 | 62.7, 152 | 128; 96 of 256 46.8 | 47.1, 102 | 107; 128 of 512 91.9 | 65.7, 209 | 138
  if (dtype == 1 && rows > 64 && pairs * ((rows + 63) / 64) > (packed && td.D == 128 ? 512 : 256)) {
    p.tiles = 1;
    p.CT = 2;
    p.KG = 1;
    p.NW = TREE_TILE_WAVES;
    p.blocks = ((rows + 31) / 32 + p.NW - 1) / p.NW;
    return p;
  }
  // Rows of a work-group: 16, so that there are many work-groups for the few; 32 or 64 (which read the ring less often) where those of
  // 16 or 32 would be more than the CUs, or with long rings, which work-groups share, half as many.
  // us, bf16, D = 128, W = 64, 512, 2048:        64 (32)           32                16
  //   4 pairs of 48 rows                  15.2  18.3  21.7  13.1  15.9  19.5  10.4  12.8  15.8
  //   32 of 128                           17.0  23.6  28.0  14.5  17.3  24.9  11.5  14.4  28.2
  //   64 of 48                            16.3  21.2  26.2  14.0  17.1  24.9  11.6  14.1  28.5
  //   64 of 128                           17.4  22.6  38.7  14.9  17.8  31.7  20.4  25.2  51.3
  //   128 of 128                          18.7  25.7  59.5  27.4  33.0  65.2
  //   128 of 24                                             13.8  17.5  34.7  11.4  15.3  36.2
  //   fp32, 64 of 48 (32 | 16 rows)                         17.1  27.4  73.7  14.8  26.2  62.7
  //   128 of 48                                             18.0  40.1   132  25.9  48.0   122
  const long long by16 = pairs * ((rows + 15) / 16), by32 = pairs * ((rows + 31) / 32);
  if (dtype == 0) {
    p.KG = rows <= 16 || by16 <= 256 ? 8 : 4;
  } else if (rows > 16 && by16 * (sets >= 40 ? 2 : 1) > 256) {
    p.CT = 2;
    p.KG = rows <= 32 || by32 <= 256 ? 8 : 4;
  }
  // Four waves where there is too little for eight: bf16, D = 128, eight | four, 4 pairs of 16 rows, W = 64 10.2 | 10.2, 256 12.2 | 10.8,
  // 512 12.9 | 12.8; of 32 rows 13.3 | 13.5, 15.9 | 14.1, 16.3 | 16.4; 256 pairs of 16 rows 12.6 | 12.5, 16.9 | 14.3, 19.2 | 18.9;
  // packed, of 32 rows 15.8 | 15.7, 17.0 | 15.8, 17.9 | 19.3
  // More pairs than CUs (two such work-groups on one), of 24 rows, W = 64, 512, 1024: 288 25.1 | 17.6, 33.2 | 27.9, 50.9 | 48.5; 512 26.8 |
  // 18.8, 41.7 | 37.9, 64.0 | 68.6; 768, W = 1024 93.5 | 105; packed, 512 26.9 | 19.0, 33.4 | 27.9, 48.6 | 47.2; D = 64 16.9 | 12.5,
  // 22.2 | 18.2, 34.3 | 33.1
  const int group = 16 * p.CT;
  if (dtype == 1 && p.KG == 8 && (pairs > 256 ? sets <= 24 : sets > 4 && sets <= 12)) p.KG = p.NW = 4;
  const int per = p.NW / p.KG * group;
  p.blocks = (rows + per - 1) / per;
  const long long groups = pairs * p.blocks;
  // waves by what either branch has to do: a piece of the state counts two sets of keys (bf16, D = 128, W = 512, 1 | 2 | 3 | 4 of eight
  // waves for it: 8 pairs of 16 rows 15.0 | 14.0 | 13.1 | 13.3, 128 of 24 20.9 | 20.1 | 18.7 | 19.2; W = 2048, 8 of 24 16.9 | 16.8 |
  // 16.9 | 19.2)
  int kl = (p.KG * 4 * pieces + sets + 2 * pieces) / (2 * (sets + 2 * pieces));
  if (kl < 1) kl = 1;
  if (kl > p.KG / 2) kl = p.KG / 2;
  p.KW = p.KG - kl;
  // Work-groups that share a pair's keys, up to 256 in all, by how many sets of keys each wave has: joining them costs 2 to 4 us,
  // for two as much as for four.  1 | 2 | 4 | 8, D = 128, bf16:
  //   4 pairs of 16 rows, W = 512 12.9 | 12.9 | 13.1 | 12.9;  1024 16.2 | 14.8 | 13.6 | 14.1;  2048 25.1 | 18.0 | 15.4 | 14.4;  4096
  //   44.8 | 27.7 | 18.8 | 15.6;  of 64 rows, W = 256 17.1 | 18.9 | 17.6 | 19.1;  512 20.3 | 20.9 | 18.9 | 20.3;  4096 86 | 51 | 33 | 25
  //   64 pairs of 32 rows, W = 512 17.5 | 18.3 | 18.3 | 28.5;  1024 20.4 | 21.1 | 19.4 | 31.0;  4096 60 | 43 | 37 | 43
  //   128 pairs of 32 rows, W = 1024 21.4 | 23.2 | 30.5;  2048 38.2 | 35.8 | 41.6;  of 64, 512 24.5 | 26.4 | 35.4;  1024 33.2 | 28.5 | 41.1
  //   fp32, 4 pairs of 16 rows, W = 512 24.3 | 18.6 | 14.7 | 15.8;  2048 57.6 | 35.6 | 24.1 | 18.7;  128, 512 26.4 | 22.2 | 28.6
  p.nsplit = p.NW == 4 ? 1 : sets >= 18 * p.KW ? 8 : sets >= 5 * p.KW ? 4 : 1;
  if (groups * p.nsplit > 256 && p.nsplit == 8) p.nsplit = 4;
  if (groups * p.nsplit > 256) p.nsplit = groups * 2 <= 256 && sets >= 6 * p.KW ? 2 : 1;
  if (p.nsplit > 1) {
    p.part_off = ((size_t)groups * 8 + 255) / 256 * 256;
    p.bytes = p.part_off + (size_t)groups * p.nsplit * per * (2 * td.D + 4) * 4;
  }
  return p;
}

}  // namespace rattn
