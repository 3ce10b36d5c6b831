// The layer for a tree of drafted tokens behind each sequence: rings and state are read and stay as they are, so that any path of
// the tree can still be accepted (tree_commit.hip).
//
// Node i at depth d (position p + d) sees, besides itself and its ancestors, the ring tokens of its window.  With j the age of a
// ring token (token p - W + j; j = 0 is the next to leave), those are the ones with j > d; the ones with j <= d have left the
// window by then, without being in the state:
//     x^s = softmax over {ring tokens, j > d} and {ancestors and itself, less than W back} of scale q.k, times v     (Sec. 2.1)
//     x^r = phi(q) S + sum of (phi(q).phi(k)) v over {ring tokens, j <= d} and {ancestors W or more back}            (Eq. 4)
//     o   = RMS_s(x^s) + RMS_r(x^r)                                                                                 (Sec. 3.2)
//
// A row is a query head of a node; the rows of a (sequence, KV head) share its ring, state and drafted keys.  Both branches are
// computed transposed, as in the decode step: S^T = K Q^T and O^T += V^T P^T with 16 x 16 tiles whose columns are rows, K and V
// straight from memory in operand layout, and the probabilities already in the registers that the second product wants.  The
// state is a "V" of D rows, whose "probabilities" are phi(q).
// A wave has CT tiles of 16 rows and a share of the keys (of the ring sets, then of the sets of drafted keys); the KG waves that
// share the rows meet in LDS, where 16 lanes take a row.  Several work-groups with the same keys lie side by side on one XCD.
#pragma once
#include "packed.hpp"
#include "ring_set.hpp"
#include "tree_nodes.hpp"

namespace rattn {

namespace {

// ---- bf16: sets of 32 keys, 16x16x32 tiles.  Operand piece j of a lane holds features feature<PERM>(j, q4) ..+7 of a row; with
// packed rings in the order in which a lane's 16 bytes of codes come.
template <bool PERM> __device__ __forceinline__ constexpr int piece_feature(int j, int q4) {
  return PERM ? 64 * (j >> 1) + 16 * q4 + 8 * (j & 1) : 32 * j + 8 * q4;
}

template <typename IO, int D, bool PERM, int CT> struct TreeMath;

template <int D, bool PERM, int CT> struct TreeMath<bf16_t, D, PERM, CT> {
  static constexpr int KEYS = 32, EV = D / 16, NT = 2, J = D / 32;
  static constexpr int PTERMS = 2;
  typedef uint32_t vrow_t __attribute__((ext_vector_type(EV / 2)));
  struct Row { bf16x8_t op[J]; };            // a column's operand: a query row
  struct Feat { bf16x8_t hi[J], lo[J]; };    // phi of one, as two terms
  struct Weights { bf16x8_t t[PTERMS]; };    // probabilities of a set's keys, one column tile
  static __device__ __forceinline__ float to_log(float scale) { return scale * LOG2E; }
  static __device__ __forceinline__ float pexp(float x) { return fast_exp2(x); }
  static constexpr float LAZY = 8.f;

  static __device__ __forceinline__ void load_row(Row& r, const bf16_t* x, int q4) {
#pragma unroll
    for (int j = 0; j < J; ++j) r.op[j] = *reinterpret_cast<const bf16x8_t*>(x + piece_feature<PERM>(j, q4));
  }
  // phi, a piece at a time: with all of a row's exponentials at once the registers of the other operands do not hold
  struct Stats { float m, z; };   // of a row: this lane's pieces and those of the lanes of the same r16
  static __device__ __forceinline__ Stats stats_of(const Row& r, int phi) {
    Stats t = {0.f, 1.f};
    if (phi == PHI_SOFTMAX) {
      float x[8];
      t.m = -INFINITY;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        unpack_bf16x8(r.op[j], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) t.m = fmaxf(t.m, x[i]);
      }
      t.m = rows_max(t.m);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        unpack_bf16x8(r.op[j], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += fast_exp2((x[i] - t.m) * LOG2E);
      }
      t.z = 1.f / rows_sum(s);
    }
    return t;
  }
  static __device__ __forceinline__ void phi_piece(const Row& r, int j, Stats t, float (&x)[8], int phi) {
    unpack_bf16x8(r.op[j], x);
    if (phi == PHI_SOFTMAX) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fast_exp2((x[i] - t.m) * LOG2E) * t.z;
    } else if (phi == PHI_RELU) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaxf(x[i], 0.f);
    }
  }
  static __device__ __forceinline__ void two_terms(float (&x)[8], bf16x8_t& hi, bf16x8_t& lo) {
    float t[8];
    hi = pack_bf16x8(x);
    unpack_bf16x8(hi, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = x[i] - t[i];
    lo = pack_bf16x8(t);
  }
  // (phi and products of it pass through the tiles as two terms of 8 bits, with the product of the two second terms left out:
  // 2^-16 of a value, far below the rounding of the output to bf16)
  static __device__ __forceinline__ void feat_of(const Row& r, Feat& o, int phi) {
    const Stats t = stats_of(r, phi);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float x[8];
      phi_piece(r, j, t, x, phi);
      two_terms(x, o.hi[j], o.lo[j]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // a set of rows in the tensors' type: keys at `stride` bytes
  struct Plain {
    Row k[2];
    vrow_t v[8];
    __device__ __forceinline__ void load_k(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(stride * r16 + 2 * piece_feature<PERM>(0, q4));
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int j = 0; j < J; ++j)
          k[c].op[j] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rows, off + 2 * piece_feature<PERM>(j, 0), 16 * stride * c, 0));
    }
    __device__ __forceinline__ void load_v(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(4 * stride * q4 + 2 * EV * r16);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int row = (u < 4 ? 0 : 16) + (u & 3);
        if constexpr (EV == 8) v[u] = __builtin_bit_cast(vrow_t, __builtin_amdgcn_raw_buffer_load_b128(rows, off, stride * row, 0));
        else v[u] = __builtin_bit_cast(vrow_t, __builtin_amdgcn_raw_buffer_load_b64(rows, off, stride * row, 0));
      }
    }
    __device__ __forceinline__ void key_row(int c, Row& r) const { r = k[c]; }
    __device__ __forceinline__ void scores(const Row (&q)[CT], f32x4_t (&s)[CT][NT]) const {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int c = 0; c < 2; ++c) s[ct][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int c = 0; c < 2; ++c) s[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c].op[j], q[ct].op[j], s[ct][c], 0, 0, 0);
    }
    __device__ __forceinline__ void accumulate(const Weights (&p)[CT], f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
        u32x4_t a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(v[2 * i + 1][e >> 1], v[2 * i][e >> 1], sel);
        add_products(__builtin_bit_cast(bf16x8_t, a), p, acc, e);
      }
    }
  };
  static __device__ __forceinline__ void add_products(bf16x8_t a, const Weights (&p)[CT], f32x4_t (&acc)[CT][EV], int e) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int term = PTERMS - 1; term >= 0; --term)
        acc[ct][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[ct].t[term], acc[ct][e], 0, 0, 0);
  }
  // a set of packed rows
  struct Packed {
    RingSet<bf16_t, fp8_t, D, false> s;
    __device__ __forceinline__ void load_k(rsrc_t rows, rsrc_t scales, int r16, int q4) { s.load_k(rows, scales, r16, q4); }
    __device__ __forceinline__ void load_v(rsrc_t rows, rsrc_t scales, int r16, int q4) { s.load_v(rows, scales, r16, q4); }
    __device__ __forceinline__ void key_row(int c, Row& r) const {
#pragma unroll
      for (int j = 0; j < D / 64; ++j) s.operands(c, j, r.op[2 * j], r.op[2 * j + 1]);
    }
    __device__ __forceinline__ void scores(const Row (&q)[CT], f32x4_t (&o)[CT][NT]) const {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int c = 0; c < 2; ++c) o[ct][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          bf16x8_t a[2];
          s.operands(c, j, a[0], a[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[h], q[ct].op[2 * j + h], o[ct][c], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void accumulate(const Weights (&p)[CT], f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int i = 0; i < EV / 4; ++i) {
        u32x2_t rows[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          uint32_t lo, hi;
          unpack_bf16x4(s.v[u][i], scale_of(s.vs[u]), lo, hi);
          rows[u] = u32x2_t{lo, hi};
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
          u32x4_t a;
#pragma unroll
          for (int h = 0; h < 4; ++h) a[h] = __builtin_amdgcn_perm(rows[2 * h + 1][e >> 1], rows[2 * h][e >> 1], sel);
          add_products(__builtin_bit_cast(bf16x8_t, a), p, acc, 4 * i + e);
        }
      }
    }
  };
  // probabilities (or weights of the linear branch) of a set's keys as the second product's operand
  static __device__ __forceinline__ void weights(const f32x4_t (&s)[NT], Weights& w) {
    float r[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
#pragma unroll
    for (int k = 0; k < PTERMS; ++k) {
      float t[8];
      w.t[k] = pack_bf16x8(r);
      unpack_bf16x8(w.t[k], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] -= t[i];
    }
  }
  // phi(k).phi(q) of keys 16c ..+15 of a set
  static __device__ __forceinline__ void feature_scores(const Row& k, const Feat (&q)[CT], f32x4_t (&s)[CT][NT], int c, int phi) {
    const Stats t = stats_of(k, phi);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s[ct][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float x[8];
      bf16x8_t hi, lo;
      phi_piece(k, j, t, x, phi);
      two_terms(x, hi, lo);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        s[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q[ct].hi[j], s[ct][c], 0, 0, 0);
        s[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[ct].lo[j], s[ct][c], 0, 0, 0);
        s[ct][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[ct].hi[j], s[ct][c], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // piece j of the features: acc += S^T phi(q)^T over state rows piece_feature(j, q4) ..+7 of each lane group
  struct State {
    f32x4_t v[8][EV / 4];
    __device__ __forceinline__ void load(const float* S, int j, int r16, int q4) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int i = 0; i < EV / 4; ++i)
          v[u][i] = *reinterpret_cast<const f32x4_t*>(S + (size_t)(piece_feature<PERM>(j, q4) + u) * D + EV * r16 + 4 * i);
    }
    __device__ __forceinline__ void accumulate(const Feat (&q)[CT], int j, f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        float x[8];
        bf16x8_t hi, lo;
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = v[u][e >> 2][e & 3];
        __builtin_amdgcn_sched_barrier(0);
        two_terms(x, hi, lo);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          acc[ct][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q[ct].hi[j], acc[ct][e], 0, 0, 0);
          acc[ct][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[ct].lo[j], acc[ct][e], 0, 0, 0);
          acc[ct][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[ct].hi[j], acc[ct][e], 0, 0, 0);
        }
      }
    }
  };
  static __device__ __forceinline__ int feature0(int e4, int i, int q4) { return EV * (4 * q4 + i) + 4 * e4; }
};

// ---- fp32: sets of 16 keys, 16x16x4 tiles (exact products, fp32 sums); packed rows become fp32 values
template <int D, bool PERM, int CT> struct TreeMath<float, D, PERM, CT> {
  static constexpr int KEYS = 16, EV = D / 16, NT = 1, J = D / 16;
  struct Row { f32x4_t op[J]; };   // features 16j + 4 q4 ..+3
  typedef Row Feat;
  struct Weights { f32x4_t t; };
  static __device__ __forceinline__ f32x4_t mfma(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ float to_log(float scale) { return scale; }
  static __device__ __forceinline__ float pexp(float x) { return expf(x); }
  static constexpr float LAZY = 5.f;

  static __device__ __forceinline__ void load_row(Row& r, const float* x, int q4) {
#pragma unroll
    for (int j = 0; j < J; ++j) r.op[j] = *reinterpret_cast<const f32x4_t*>(x + 16 * j + 4 * q4);
  }
  static __device__ __forceinline__ void feat_of(const Row& r, Feat& o, int phi) {
    if (phi == PHI_SOFTMAX) {
      float m = -INFINITY, s = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, r.op[j][i]);
      m = rows_max(m);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) { o.op[j][i] = expf(r.op[j][i] - m); s += o.op[j][i]; }
      s = 1.f / rows_sum(s);
#pragma unroll
      for (int j = 0; j < J; ++j) o.op[j] *= s;
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o.op[j][i] = phi == PHI_RELU ? fmaxf(r.op[j][i], 0.f) : r.op[j][i];
    }
  }
  struct Base {
    Row k;
    f32x4_t v[4][D / 64];   // features 64 hf + 4 r16 ..+3 of keys 4 q4 + i
    __device__ __forceinline__ void key_row(int, Row& r) const { r = k; }
    // (short chains and a tree of sums, as in the decode step: the rounding of the logits grows with the chain)
    static __device__ __forceinline__ f32x4_t dots(const Row& a, const Row& b) {
      f32x4_t t[J];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        f32x4_t u[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e & 1] = mfma(a.op[j][e], b.op[j][e], u[e & 1]);
        t[j] = u[0] + u[1];
      }
#pragma unroll
      for (int n = J / 2; n > 0; n >>= 1)
#pragma unroll
        for (int j = 0; j < n; ++j) t[j] += t[j + n];
      return t[0];
    }
    __device__ __forceinline__ void scores(const Row (&q)[CT], f32x4_t (&s)[CT][NT]) const {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) s[ct][0] = dots(k, q[ct]);
    }
    __device__ __forceinline__ void accumulate(const Weights (&p)[CT], f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) acc[ct][4 * hf + e] = mfma(v[i][hf][e], p[ct].t[i], acc[ct][4 * hf + e]);
    }
  };
  struct Plain : Base {
    __device__ __forceinline__ void load_k(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(stride * r16 + 16 * q4);
#pragma unroll
      for (int j = 0; j < J; ++j) this->k.op[j] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, off + 64 * j, 0, 0));
    }
    __device__ __forceinline__ void load_v(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(4 * stride * q4 + 16 * r16);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
          this->v[i][hf] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, off + 256 * hf, stride * i, 0));
    }
  };
  struct Packed : Base {
    __device__ __forceinline__ void load_k(rsrc_t rows, rsrc_t scales, int r16, int q4) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t c = __builtin_amdgcn_raw_buffer_load_b32(rows, D * r16 + 4 * q4 + 16 * j, 0, 0);
        const uint8_t s = __builtin_amdgcn_raw_buffer_load_b8(scales, scale_bytes(D) * r16 + (j >> 1), 0, 0);
        this->k.op[j] = unpack_f32x4(c, scale_of(s));
      }
    }
    __device__ __forceinline__ void load_v(rsrc_t rows, rsrc_t scales, int r16, int q4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf) {
          const uint32_t c = __builtin_amdgcn_raw_buffer_load_b32(rows, D * (4 * q4 + i) + 4 * r16 + 64 * hf, 0, 0);
          const uint8_t s = __builtin_amdgcn_raw_buffer_load_b8(scales, scale_bytes(D) * (4 * q4 + i) + 2 * hf + (r16 >> 3), 0, 0);
          this->v[i][hf] = unpack_f32x4(c, scale_of(s));
        }
    }
  };
  static __device__ __forceinline__ void weights(const f32x4_t (&s)[NT], Weights& w) { w.t = s[0]; }
  static __device__ __forceinline__ void feature_scores(const Row& k, const Feat (&q)[CT], f32x4_t (&s)[CT][NT], int, int phi) {
    Feat f;
    feat_of(k, f, phi);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s[ct][0] = Base::dots(f, q[ct]);
  }
  struct State {
    f32x4_t v[4][D / 64];
    __device__ __forceinline__ void load(const float* S, int j, int r16, int q4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf) v[i][hf] = *reinterpret_cast<const f32x4_t*>(S + (size_t)(16 * j + 4 * q4 + i) * D + 64 * hf + 4 * r16);
    }
    __device__ __forceinline__ void accumulate(const Feat (&q)[CT], int j, f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) acc[ct][4 * hf + e] = mfma(v[i][hf][e], q[ct].op[j][i], acc[ct][4 * hf + e]);
    }
  };
  static __device__ __forceinline__ int feature0(int e4, int i, int q4) { return 64 * e4 + 4 * (4 * q4 + i); }
};

template <typename IO, typename RT> struct TreeArgs {
  const IO *q, *k, *v;
  const int32_t *parent, *count, *pos;
  const RT *k_ring, *v_ring;
  const float *state, *gs, *gr;
  IO* o;
  int N, M, Hq, Hkv, W, G, blocks, phi;
  float scale, eps;
  const uint8_t *ks, *vs;
};

constexpr size_t tree_lds_bytes(int D, int CT, int NW) { return (size_t)NW * 16 * CT * ((D + 4) + 2) * 4; }

// A row whose sums hold something that is no finite number, by a whole wave, key by key: only the keys that the row sees are
// touched.  (The tiles multiply the others by 0, which is not 0 for an infinite or NaN feature.)
template <typename IO, typename RT, int D>
__device__ void tree_row_again(const TreeArgs<IO, RT>& a, int n, int g, int row, unsigned long long anc, unsigned long long left, int lane) {
  constexpr int EPL = D / 64, SB = scale_bytes(D);
  const int W = a.W, p = a.pos[n], slot0 = p % W, node = row / a.G, h = g * a.G + row % a.G;
  const int depth = __popcll(anc) - 1;
  const size_t pair = (size_t)n * a.Hkv + g;
  const RT *kr = a.k_ring + pair * W * D, *vr = a.v_ring + pair * W * D;
  const uint8_t* krs = sizeof(RT) == 1 ? a.ks + pair * W * SB : nullptr;
  const uint8_t* vrs = sizeof(RT) == 1 ? a.vs + pair * W * SB : nullptr;
  const size_t q0 = (((size_t)n * a.M + node) * a.Hq + h) * D;
  float q[EPL], f[EPL], xs[EPL], xr[EPL], k[EPL], kf[EPL], v[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) { q[e] = io_traits<IO>::ld(a.q + q0 + lane + 64 * e); xs[e] = xr[e] = 0.f; }
  feature_row<EPL>(q, f, a.phi);
  // key t: ring tokens by age, then nodes; calls see(in the window or not) with the row in k, v
  auto each = [&](auto&& see) {
    for (int t = max(0, W - p); t < W + a.M; ++t) {
      bool in;
      if (t < W) {
        in = t > depth;
        const int slot = slot0 + t < W ? slot0 + t : slot0 + t - W;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          k[e] = ring_value(kr, krs, (size_t)slot * D + lane + 64 * e);
          v[e] = ring_value(vr, vrs, (size_t)slot * D + lane + 64 * e);
        }
      } else {
        if (!(anc >> (t - W) & 1)) continue;
        in = !(left >> (t - W) & 1);
        const size_t i = (((size_t)n * a.M + t - W) * a.Hkv + g) * D + lane;
#pragma unroll
        for (int e = 0; e < EPL; ++e) { k[e] = io_traits<IO>::ld(a.k + i + 64 * e); v[e] = io_traits<IO>::ld(a.v + i + 64 * e); }
      }
      see(in);
    }
  };
  auto dot = [&](const float (&x)[EPL], const float (&y)[EPL]) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) s += x[e] * y[e];
    return wave_sum(s);
  };
  float m = -INFINITY, l = 0.f;
  each([&](bool in) { if (in) m = fmaxf(m, dot(q, k) * a.scale); });
  each([&](bool in) {
    if (in) {
      const float w = expf(dot(q, k) * a.scale - m);
      l += w;
#pragma unroll
      for (int e = 0; e < EPL; ++e) xs[e] += w * v[e];
    } else {
      feature_row<EPL>(k, kf, a.phi);
      const float w = dot(f, kf);
#pragma unroll
      for (int e = 0; e < EPL; ++e) xr[e] += w * v[e];
    }
  });
  if (p > W) {
    const float* S = a.state + pair * D * D;
#pragma unroll
    for (int e = 0; e < EPL; ++e)
      for (int r = 0; r < 64; ++r) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f[e]), r));
#pragma unroll
        for (int i = 0; i < EPL; ++i) xr[i] += w * S[(size_t)(64 * e + r) * D + lane + 64 * i];
      }
  }
  float s1 = 0.f, s2 = 0.f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) { xs[e] /= l; s1 += xs[e] * xs[e]; s2 += xr[e] * xr[e]; }
  const float r1 = rsqrtf(wave_sum(s1) / D + a.eps), r2 = rsqrtf(wave_sum(s2) / D + a.eps);
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    const int d = lane + 64 * e;
    const float g1 = a.gs ? a.gs[h * D + d] : 1.f, g2 = a.gr ? a.gr[h * D + d] : 1.f;
    io_traits<IO>::st(a.o + q0 + d, g1 * xs[e] * r1 + g2 * xr[e] * r2);
  }
}

template <typename IO> __device__ __forceinline__ void store4(IO* p, f32x4_t x) {
  if constexpr (sizeof(IO) == 4) *reinterpret_cast<f32x4_t*>(p) = x;
  else *reinterpret_cast<bf16x4_t*>(p) = __builtin_convertvector(x, bf16x4_t);
}

// A row's results from its sums, by 16 lanes (lane r16 has features 64 h + 4 r16 ..+3): the two RMS norms and their sum
// (Sec. 3.2); false where something is no finite number, and nothing is stored.
template <typename IO, typename RT, int D>
__device__ __forceinline__ bool tree_row_out(const TreeArgs<IO, RT>& a, int n, int g, int row, int r16, f32x4_t (&xs)[D / 64],
                                             const f32x4_t (&xr)[D / 64], float den, bool mine) {
  constexpr int NH = D / 64;
  const float inv = 1.f / den;
  float s1 = 0.f, s2 = 0.f, z = inv * 0.f;
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xs[h][i] *= inv;
      s1 += xs[h][i] * xs[h][i];
      s2 += xr[h][i] * xr[h][i];
      z += xs[h][i] * 0.f + xr[h][i] * 0.f;
    }
  s1 = sum16(s1);
  s2 = sum16(s2);
  z = sum16(z);
  if (!mine) return true;
  if (!(z == 0.f)) return false;
  const float r1 = rsqrtf(s1 / D + a.eps), r2 = rsqrtf(s2 / D + a.eps);
  const int head = g * a.G + row % a.G;
  IO* o = a.o + (((size_t)n * a.M + row / a.G) * a.Hq + head) * D;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    const int d = 64 * h + 4 * r16;
    f32x4_t y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float g1 = a.gs ? a.gs[head * D + d + i] : 1.f, g2 = a.gr ? a.gr[head * D + d + i] : 1.f;
      y[i] = g1 * xs[h][i] * r1 + g2 * xr[h][i] * r2;
    }
    store4(o + d, y);
  }
  return true;
}

// Few rows.  Of the KG waves that share a group's rows the first KW have the softmax branch (ring sets, then sets of drafted keys),
// the others the linear one (pieces of the state, then the keys that leave): each holds one set of accumulators, both branches'
// loads are under way at once, and all meet in LDS once.
template <typename IO, typename RT, int D, int CT, int KG, int NW, bool SPLIT>
__global__ __launch_bounds__(NW * 64, 2) void tree_kernel(TreeArgs<IO, RT> a, int KW, std::conditional_t<SPLIT, SplitArgs, NoSplit> split) {
  constexpr bool PACKED = sizeof(RT) == 1;
  typedef TreeMath<IO, D, PACKED, CT> Math;
  typedef std::conditional_t<PACKED, typename Math::Packed, typename Math::Plain> RingRows;
  typedef typename Math::Plain NodeRows;
  constexpr int KEYS = Math::KEYS, NT = Math::NT, EV = Math::EV, SB = scale_bytes(D);
  constexpr int RG = NW / KG, ROWS = RG * 16 * CT, LD = D + 4;
  constexpr int NH = D / 64, TURNS = (ROWS + 4 * NW - 1) / (4 * NW);   // rows per 16 lanes in the end
  extern __shared__ __align__(16) float lds[];
  float* part = lds;                          // [NW][16 CT][LD]
  float* ml = part + NW * 16 * CT * LD;       // [NW][16 CT][2]
  const int lane = lane_id(), w = wave_id(), r16 = lane & 15, q4 = lane >> 4;
  const int W = a.W, G = a.G, M = a.M, Hkv = a.Hkv;
  // Eight pairs at a time, the blocks of each eight apart: those that read the same ring sit on one XCD, at the same time
  const unsigned pairs = a.N * Hkv, per = (pairs + 7) / 8 * 8 * a.blocks;
  const int sp = SPLIT ? blockIdx.x / per : 0;
  const unsigned id = SPLIT ? blockIdx.x % per : blockIdx.x;
  const unsigned pair = id / (8 * a.blocks) * 8 + id % 8;
  const int block = id / 8 % a.blocks;
  if (pair >= pairs) return;
  const int g = pair % Hkv, n = pair / Hkv;
  const int p = a.pos[n], cnt = a.count ? min(a.count[n], M) : M;
  const int row0 = block * ROWS, nrows = cnt * G;
  if (row0 >= nrows || p < 0) return;
  const int rg = w % RG, kg = w / RG;
  const int nsplit = SPLIT ? split.n : 1;
  const int slot0 = p % W, nvalid = min(p, W);
  const RT *kr = a.k_ring + (size_t)pair * W * D, *vr = a.v_ring + (size_t)pair * W * D;
  const uint8_t* krs = PACKED ? a.ks + (size_t)pair * W * SB : nullptr;
  const uint8_t* vrs = PACKED ? a.vs + (size_t)pair * W * SB : nullptr;
  const IO *kn = a.k + ((size_t)n * M * Hkv + g) * D, *vn = a.v + ((size_t)n * M * Hkv + g) * D;
  const int nstride = Hkv * D * (int)sizeof(IO);
  const int nring = (nvalid + KEYS - 1) / KEYS, nset = nring + (cnt + KEYS - 1) / KEYS;
  const int32_t* parent = a.parent + (size_t)n * M;
  const int up = lane < M ? parent[lane] : -1;

  RingRows ring;
  auto load_ring_k = [&](int base, int rows) {   // `rows` of them exist
    rows = min(rows, KEYS);
    const rsrc_t r = make_rsrc(kr + (size_t)base * D, (unsigned)(rows * D * (int)sizeof(RT)));
    if constexpr (PACKED) ring.load_k(r, make_rsrc(krs + (size_t)base * SB, (unsigned)(rows * SB)), r16, q4);
    else ring.load_k(r, D * (int)sizeof(RT), r16, q4);
  };
  auto load_ring_v = [&](int base, int rows) {
    rows = min(rows, KEYS);
    const rsrc_t r = make_rsrc(vr + (size_t)base * D, (unsigned)(rows * D * (int)sizeof(RT)));
    if constexpr (PACKED) ring.load_v(r, make_rsrc(vrs + (size_t)base * SB, (unsigned)(rows * SB)), r16, q4);
    else ring.load_v(r, D * (int)sizeof(RT), r16, q4);
  };
  auto node_rsrc = [&](const IO* x, int base) {   // nodes base .. M-1 of this sequence (of the last one only its D features)
    return make_rsrc(x + (size_t)base * Hkv * D, (unsigned)((M - 1 - base) * nstride + D * (int)sizeof(IO)));
  };
  // age of the token in a slot
  auto age = [&](int slot) { return slot - slot0 + (slot < slot0 ? W : 0); };

  // ---- this wave's rows
  typename Math::Row q[CT];
  int node_of[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int row = min(row0 + (rg * CT + ct) * 16 + r16, nrows - 1);
    node_of[ct] = row / G;
    Math::load_row(q[ct], a.q + (((size_t)n * M + node_of[ct]) * a.Hq + g * G + row % G) * D, q4);
  }
  int depth[CT], dmax = 0;
  auto depths = [&](const TreeNodes& t) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      depth[ct] = __shfl(t.depth(), node_of[ct]);
      dmax = max(dmax, depth[ct]);
    }
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) dmax = max(dmax, __shfl_xor(dmax, s));
    dmax = __builtin_amdgcn_readfirstlane(dmax);
  };
  f32x4_t acc[CT][EV];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int e = 0; e < EV; ++e) acc[ct][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (kg < KW) {
    // ---- softmax branch
    const int w0 = kg * nsplit + sp, nw = KW * nsplit;
    // a set's first row; the pairs start at different sets, which spreads the simultaneous requests over the memory channels
    const int rot = (int)(pair % (unsigned)max(nring, 1));
    auto ring_base = [&](int it) { const int s = it + rot; return (s < nring ? s : s - nring) * KEYS; };
    if (w0 < nring) {
      load_ring_k(ring_base(w0), nvalid - ring_base(w0));
      load_ring_v(ring_base(w0), nvalid - ring_base(w0));
    }
    const TreeNodes node = tree_nodes(up, W, lane);
    depths(node);
    const float sc = Math::to_log(a.scale);
    float m[CT], l[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) { m[ct] = -1.0e30f; l[ct] = 0.f; }
    // scaled scores of a set, masked with -inf, into weights; a running maximum stays while no score is far above it
    auto softmax_step = [&](f32x4_t (&s)[CT][NT], typename Math::Weights (&pw)[CT]) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float mx = -INFINITY;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[ct][c][i]);
        mx = rows_max(mx);
        if (__any(mx > m[ct] + Math::LAZY)) {
          const float top = fmaxf(m[ct], mx), alpha = Math::pexp(m[ct] - top);
          m[ct] = top;
          l[ct] *= alpha;
#pragma unroll
          for (int e = 0; e < EV; ++e) acc[ct][e] *= alpha;
        }
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) { s[ct][c][i] = Math::pexp(s[ct][c][i] - m[ct]); l[ct] += s[ct][c][i]; }
        Math::weights(s[ct], pw[ct]);
      }
    };
    int it = w0;
    while (it < nring) {
      const int base = ring_base(it);
      it += nw;
      const int next = it < nring ? ring_base(it) : 0;
      f32x4_t s[CT][NT];
      ring.scores(q, s);
      if (it < nring) load_ring_k(next, nvalid - next);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int c = 0; c < NT; ++c) s[ct][c] *= sc;
      // ages in the set start at its first slot's, or at 0 where slot0 is inside
      const int youngest = base < slot0 && slot0 < base + KEYS ? 0 : age(base);
      if (base + KEYS > nvalid || youngest <= dmax) {   // wave-uniform
        const int s0 = opaque(base + 4 * q4);
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int slot = s0 + 16 * c + i, j = slot < nvalid ? age(slot) : -1;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][c][i] = j > depth[ct] ? s[ct][c][i] : -INFINITY;
          }
      }
      typename Math::Weights pw[CT];
      softmax_step(s, pw);
      ring.accumulate(pw, acc);
      if (it < nring) load_ring_v(next, nvalid - next);
    }
    // drafted keys
    for (; it < nset; it += nw) {
      const int base = (it - nring) * KEYS;
      NodeRows rows;
      rows.load_k(node_rsrc(kn, base), nstride, r16, q4);
      rows.load_v(node_rsrc(vn, base), nstride, r16, q4);
      f32x4_t s[CT][NT];
      rows.scores(q, s);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const unsigned see = (unsigned)(shfl64(node.anc & ~node.left, node_of[ct]) >> (base + 4 * q4));
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[ct][c][i] = see >> (16 * c + i) & 1 ? s[ct][c][i] * sc : -INFINITY;
      }
      typename Math::Weights pw[CT];
      softmax_step(s, pw);
      rows.accumulate(pw, acc);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      l[ct] = rows_sum(l[ct]);
      if (q4 == 0) {
        ml[((w * CT + ct) * 16 + r16) * 2] = m[ct];
        ml[((w * CT + ct) * 16 + r16) * 2 + 1] = l[ct];
      }
    }
  } else {
    // ---- linear branch
    const int w0 = (kg - KW) * nsplit + sp, nw = (KG - KW) * nsplit;
    typename Math::Feat f[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) Math::feat_of(q[ct], f[ct], a.phi);
    if (p > W) {
      const float* S = a.state + (size_t)pair * D * D;
#pragma unroll
      for (int j = 0; j < Math::J; ++j)
        if (j % nw == w0) {
          typename Math::State st;
          st.load(S, j, r16, q4);
          st.accumulate(f, j, acc);
        }
    }
    const TreeNodes node = tree_nodes(up, W, lane);
    depths(node);
    // ring tokens that leave: slots slot0 .., then 0 ..; then drafted ones, where a path is longer than the window.  Of the waves the
    // last come first (the first ones may have a piece of the state more)
    const bool any = p + dmax >= W;
    const int nleave = any ? min(dmax + 1, W) : 0, len0 = min(nleave, W - slot0), sets0 = (len0 + KEYS - 1) / KEYS;
    const int sets = sets0 + (nleave - len0 + KEYS - 1) / KEYS, nodes = any && dmax >= W ? (cnt + KEYS - 1) / KEYS : 0;
    for (int x = nw - 1 - w0; x < sets + nodes; x += nw) {
      f32x4_t s[CT][NT];
      typename Math::Weights pw[CT];
      if (x < sets) {
        const int base = x < sets0 ? slot0 + x * KEYS : (x - sets0) * KEYS;
        const int rows = min(KEYS, min(x < sets0 ? slot0 + len0 : nleave - len0, nvalid) - base);
        if (rows <= 0) continue;   // (a ring that is not full: those slots hold nothing yet)
        load_ring_k(base, rows);
        load_ring_v(base, rows);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          typename Math::Row kx;
          ring.key_row(c, kx);
          Math::feature_scores(kx, f, s, c, a.phi);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 16 * c + 4 * q4 + i, j = r < rows ? age(base + r) : W;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][c][i] = j <= depth[ct] && j < W ? s[ct][c][i] : 0.f;
          }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) Math::weights(s[ct], pw[ct]);
        ring.accumulate(pw, acc);
      } else {
        const int base = (x - sets) * KEYS;
        NodeRows rows;
        rows.load_k(node_rsrc(kn, base), nstride, r16, q4);
        rows.load_v(node_rsrc(vn, base), nstride, r16, q4);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          typename Math::Row kx;
          rows.key_row(c, kx);
          Math::feature_scores(kx, f, s, c, a.phi);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const unsigned see = (unsigned)(shfl64(node.left, node_of[ct]) >> (base + 4 * q4));
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[ct][c][i] = see >> (16 * c + i) & 1 ? s[ct][c][i] : 0.f;
          Math::weights(s[ct], pw[ct]);
        }
        rows.accumulate(pw, acc);
      }
    }
  }
  // ---- the waves meet: partial sums in LDS, a row at a time
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int e4 = 0; e4 < EV / 4; ++e4)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(part + ((w * CT + ct) * 16 + r16) * LD + Math::feature0(e4, i, q4)) =
            f32x4_t{acc[ct][4 * e4][i], acc[ct][4 * e4 + 1][i], acc[ct][4 * e4 + 2][i], acc[ct][4 * e4 + 3][i]};
  __syncthreads();
  // 16 lanes take a row: row t of the work-group is row t % (16 CT) of the waves kg * RG + t / (16 CT)
  const int group = w * 4 + q4;
  auto turn_row = [&](int turn) { return turn * 4 * NW + group; };
  auto slice = [&](int t, int k) { return (k * RG + t / (16 * CT)) * 16 * CT + t % (16 * CT); };
  f32x4_t xs[TURNS][NH], xr[TURNS][NH];
  float top[TURNS], den[TURNS];
#pragma unroll
  for (int turn = 0; turn < TURNS; ++turn) {
    const int t = min(turn_row(turn), ROWS - 1);
    top[turn] = -1.0e30f;
    den[turn] = 0.f;
#pragma unroll
    for (int h = 0; h < NH; ++h) xs[turn][h] = xr[turn][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KG; ++k)
      if (k < KW) top[turn] = fmaxf(top[turn], ml[slice(t, k) * 2]);
#pragma unroll
    for (int k = 0; k < KG; ++k) {
      f32x4_t x[NH];
#pragma unroll
      for (int h = 0; h < NH; ++h) x[h] = *reinterpret_cast<const f32x4_t*>(part + slice(t, k) * LD + 64 * h + 4 * r16);
      if (k < KW) {
        const float f = Math::pexp(ml[slice(t, k) * 2] - top[turn]);
        den[turn] = __builtin_fmaf(f, ml[slice(t, k) * 2 + 1], den[turn]);
#pragma unroll
        for (int h = 0; h < NH; ++h) xs[turn][h] += f * x[h];
      } else {
#pragma unroll
        for (int h = 0; h < NH; ++h) xr[turn][h] += x[h];
      }
    }
  }
  // ---- SPLIT: the sums of all work-groups of these rows, by the one that arrives last (see SplitArgs)
  if constexpr (SPLIT) {
    constexpr int LINE = SplitArgs::row(D);
    const size_t cell = (size_t)pair * a.blocks + block;
    float* all = split.part + cell * split.n * ROWS * LINE;
    const rsrc_t mem = make_rsrc(all, (unsigned)(split.n * ROWS * LINE * 4));
#pragma unroll
    for (int turn = 0; turn < TURNS; ++turn) {
      const int t = turn_row(turn);
      if (t < ROWS && row0 + t < nrows) {
        const int at = (sp * ROWS + t) * LINE * 4;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          put_shared16(mem, xs[turn][h], at + 256 * h + 16 * r16);
          put_shared16(mem, xr[turn][h], at + 4 * D + 256 * h + 16 * r16);
        }
        if (r16 == 0) put_shared16(mem, f32x4_t{top[turn], den[turn], 0.f, 0.f}, at + 8 * D);
      }
    }
    if (!arrive_last(split.ticket + cell, split.nonce, nsplit)) return;
    constexpr int AT_ONCE = 4;
#pragma unroll
    for (int turn = 0; turn < TURNS; ++turn) {
      const int t = turn_row(turn);
      if (t >= ROWS || row0 + t >= nrows) continue;
      top[turn] = -1.0e30f;
      den[turn] = 0.f;
#pragma unroll
      for (int h = 0; h < NH; ++h) xs[turn][h] = xr[turn][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int k0 = 0; k0 < nsplit; k0 += AT_ONCE) {
        f32x4_t x[AT_ONCE][NH], y[AT_ONCE][NH], ml4[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
          const int at = (min(k0 + k, nsplit - 1) * ROWS + t) * LINE * 4;
          ml4[k] = get_shared16(mem, at + 8 * D);
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            x[k][h] = get_shared16(mem, at + 256 * h + 16 * r16);
            y[k][h] = get_shared16(mem, at + 4 * D + 256 * h + 16 * r16);
          }
        }
        float to = top[turn];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) to = fmaxf(to, ml4[k][0]);
        const float keep = Math::pexp(top[turn] - to);
        top[turn] = to;
        den[turn] *= keep;
#pragma unroll
        for (int h = 0; h < NH; ++h) xs[turn][h] *= keep;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
          if (k0 + k < nsplit) {
            const float f = Math::pexp(ml4[k][0] - to);
            den[turn] += f * ml4[k][1];
#pragma unroll
            for (int h = 0; h < NH; ++h) { xs[turn][h] += f * x[k][h]; xr[turn][h] += y[k][h]; }
          }
      }
    }
  }
  unsigned again = 0;   // turns whose row has something that is no finite number
#pragma unroll
  for (int turn = 0; turn < TURNS; ++turn) {
    const int t = turn_row(turn);
    if (!tree_row_out<IO, RT, D>(a, n, g, row0 + t, r16, xs[turn], xr[turn], den[turn], t < ROWS && row0 + t < nrows)) again |= 1u << turn;
  }
  if (!__any(again != 0)) return;
  const TreeNodes node = tree_nodes(up, W, lane);
  for (int turn = 0; turn < TURNS; ++turn) {
    unsigned long long todo = __ballot((again >> turn & 1) && r16 == 0);
    while (todo) {
      const int from = __builtin_ctzll(todo);
      todo &= todo - 1;
      const int row = __shfl(row0 + turn_row(turn), from), i = row / G;
      tree_row_again<IO, RT, D>(a, n, g, row, shfl64(node.anc, i), shfl64(node.left, i), lane);
    }
  }
}

template <typename IO, typename RT, int D, int CT, int KG, int NW, bool SPLIT>
void launch_tree(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  const size_t bytes = tree_lds_bytes(D, CT, NW);
  static const bool attr = hipFuncSetAttribute(reinterpret_cast<const void*>(tree_kernel<IO, RT, D, CT, KG, NW, SPLIT>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
  (void)attr;
  const TreeArgs<IO, RT> a = {(const IO*)t.q, (const IO*)t.k, (const IO*)t.v, t.parent, t.count, t.pos, (const RT*)t.k_ring,
                              (const RT*)t.v_ring, (const float*)t.state, t.gs, t.gr, (IO*)t.o, td.N, td.M, td.Hq, td.Hkv, td.W,
                              td.G, pl.blocks, td.phi, td.scale, td.eps, (const uint8_t*)t.k_scale, (const uint8_t*)t.v_scale};
  std::conditional_t<SPLIT, SplitArgs, NoSplit> split;
  if constexpr (SPLIT)
    split = {(float*)((char*)td.workspace + pl.part_off), (unsigned long long*)td.workspace, td.nonce, pl.nsplit, 0};
  const long long grid = ((long long)td.N * td.Hkv + 7) / 8 * 8 * pl.blocks * (SPLIT ? pl.nsplit : 1);
  tree_kernel<IO, RT, D, CT, KG, NW, SPLIT><<<(unsigned)grid, NW * 64, bytes, st>>>(a, pl.KW, split);
}

template <typename IO, typename RT, int D>
void pick_tree(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
#define RATTN_TREE(CT_, KG_, NW_)                                                                   \
  if (pl.CT == CT_ && pl.KG == KG_ && pl.NW == NW_) {                                               \
    if (td.workspace && pl.nsplit > 1) launch_tree<IO, RT, D, CT_, KG_, NW_, true>(td, t, pl, st);  \
    else launch_tree<IO, RT, D, CT_, KG_, NW_, false>(td, t, pl, st);                               \
    return;                                                                                         \
  }
  RATTN_TREE(1, 8, 8)
  RATTN_TREE(1, 4, 4)
  RATTN_TREE(1, 4, 8)
  if constexpr (sizeof(IO) == 2) {
    RATTN_TREE(2, 8, 8)
    RATTN_TREE(2, 4, 4)
    RATTN_TREE(2, 4, 8)
  }
#undef RATTN_TREE
}

}  // namespace

}  // namespace rattn
