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
// Few sequences are bound by the way of one work-group through its inputs (12 nodes behind one sequence, 16 query and 4 KV heads, D = 128,
// W = 512: 12 us, of which 3 are the launch and the walk of the tree, 3 the meeting and the rows' end), many by memory and by
// what a CU takes in (64 sequences of 6 nodes, 32 query and 8 KV heads, packed rings of 512 slots: 25.6 us, 4.2 TB/s).
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
  struct Weights { bf16x8_t t[PTERMS]; };    // probabilities of a set's keys, one column tile
  static __device__ __forceinline__ float to_log(float scale) { return scale * LOG2E; }
  static __device__ __forceinline__ float pexp(float x) { return fast_exp2(x); }
  static constexpr float LAZY = 8.f;

  static __device__ __forceinline__ void load_row(Row& r, const bf16_t* x, int q4) {
#pragma unroll
    for (int j = 0; j < J; ++j) r.op[j] = *reinterpret_cast<const bf16x8_t*>(x + piece_feature<PERM>(j, q4));
  }
  // phi, a piece at a time: with all of a row's exponentials at once the registers of the other operands do not hold.
  // (Of a row: this lane's pieces and those of the lanes of the same r16.)
  struct Stats { float m, z; };
  static __device__ __forceinline__ Stats softmax_stats(const Row& r) {
    float x[8], m = -INFINITY, s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      unpack_bf16x8(r.op[j], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, x[i]);
    }
    m = rows_max(m);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      unpack_bf16x8(r.op[j], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += fast_exp2((x[i] - m) * LOG2E);
    }
    return {m, 1.f / rows_sum(s)};
  }
  // calls use(j, hi, lo) with piece j of phi(r) as two terms; the other maps' values are bf16 ones, which one term holds
  template <typename F> static __device__ __forceinline__ void each_piece(const Row& r, int phi, F&& use) {
    if (phi == PHI_SOFTMAX) {
      const Stats t = softmax_stats(r);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float x[8];
        bf16x8_t hi, lo;
        unpack_bf16x8(r.op[j], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fast_exp2((x[i] - t.m) * LOG2E) * t.z;
        two_terms(x, hi, lo);
        use(j, hi, lo);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        bf16x8_t hi = r.op[j];
        if (phi == PHI_RELU) {
          float x[8];
          unpack_bf16x8(hi, x);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = fmaxf(x[i], 0.f);
          hi = pack_bf16x8(x);
        }
        use(j, hi, __builtin_bit_cast(bf16x8_t, u32x4_t{0, 0, 0, 0}));
      }
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
  // phi(q) of a wave's rows, in its own part of LDS: two terms of every piece, [piece][row tile][term][lane].  (phi and products of
  // it pass through the tiles as two terms of 8 bits, with the product of the two second terms left out: 2^-16 of a value, far
  // below the rounding of the output to bf16.)
  static constexpr int FEAT_BYTES = J * CT * 2 * 1024;
  static __device__ __forceinline__ void put_feat(const Row& r, unsigned char* lds, int ct, int lane, int phi) {
    each_piece(r, phi, [&](int j, bf16x8_t hi, bf16x8_t lo) {
      *reinterpret_cast<bf16x8_t*>(lds + ((j * CT + ct) * 2) * 1024 + 16 * lane) = hi;
      *reinterpret_cast<bf16x8_t*>(lds + ((j * CT + ct) * 2 + 1) * 1024 + 16 * lane) = lo;
    });
  }
  struct Piece { bf16x8_t hi[CT], lo[CT]; };
  static __device__ __forceinline__ void get_feat(Piece& f, const unsigned char* lds, int j, int lane) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      f.hi[ct] = *reinterpret_cast<const bf16x8_t*>(lds + ((j * CT + ct) * 2) * 1024 + 16 * lane);
      f.lo[ct] = *reinterpret_cast<const bf16x8_t*>(lds + ((j * CT + ct) * 2 + 1) * 1024 + 16 * lane);
    }
  }

  // a set of rows in the tensors' type: keys at `stride` bytes.  (The rows' offsets are part of each lane's, which is what a resource's
  // size is compared with: rows behind the last one read as zero)
  struct Plain {
    Row k[2];
    vrow_t v[8];
    __device__ __forceinline__ void load_k(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(stride * r16 + 2 * piece_feature<PERM>(0, q4));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int offc = off + 16 * stride * c;
#pragma unroll
        for (int j = 0; j < J; ++j)
          k[c].op[j] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rows, offc + 2 * piece_feature<PERM>(j, 0), 0, 0));
      }
    }
    __device__ __forceinline__ void load_v(rsrc_t rows, int stride, int r16, int q4) {
      const int off = opaque(4 * stride * q4 + 2 * EV * r16);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int offu = off + stride * ((u < 4 ? 0 : 16) + (u & 3));
        if constexpr (EV == 8) v[u] = __builtin_bit_cast(vrow_t, __builtin_amdgcn_raw_buffer_load_b128(rows, offu, 0, 0));
        else v[u] = __builtin_bit_cast(vrow_t, __builtin_amdgcn_raw_buffer_load_b64(rows, offu, 0, 0));
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
  // phi(k).phi(q) of 16 keys
  static __device__ __forceinline__ void feature_scores(const Row& k, const unsigned char* lds, f32x4_t (&s)[CT], int lane, int phi) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s[ct] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    each_piece(k, phi, [&](int j, bf16x8_t hi, bf16x8_t lo) {
      Piece f;
      get_feat(f, lds, j, lane);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        s[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, f.hi[ct], s[ct], 0, 0, 0);
        s[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, f.lo[ct], s[ct], 0, 0, 0);
        s[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, f.hi[ct], s[ct], 0, 0, 0);
      }
    });
  }
  // piece j of the features: acc += S^T phi(q)^T over state rows piece_feature(j, q4) ..+7 of each lane group, four of a lane's
  // EV value features at a time
  struct State {
    static constexpr int PARTS = EV / 4;
    f32x4_t v[PARTS][8];
    __device__ __forceinline__ void load(const float* S, int j, int part, int r16, int q4) {
      const float* s = S + (size_t)piece_feature<PERM>(j, q4) * D + EV * r16 + 4 * part;
#pragma unroll
      for (int u = 0; u < 8; ++u) v[part][u] = *reinterpret_cast<const f32x4_t*>(s + u * D);
    }
    __device__ __forceinline__ void accumulate(const Piece& f, int part, f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x[8];
        bf16x8_t hi, lo;
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = v[part][u][e];
        two_terms(x, hi, lo);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          f32x4_t& a = acc[ct][4 * part + e];
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, f.hi[ct], a, 0, 0, 0);
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, f.lo[ct], a, 0, 0, 0);
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, f.hi[ct], a, 0, 0, 0);
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
  struct Weights { f32x4_t t; };
  static __device__ __forceinline__ f32x4_t mfma(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ float to_log(float scale) { return scale; }
  static __device__ __forceinline__ float pexp(float x) { return expf(x); }
  static constexpr float LAZY = 5.f;

  static __device__ __forceinline__ void load_row(Row& r, const float* x, int q4) {
#pragma unroll
    for (int j = 0; j < J; ++j) r.op[j] = *reinterpret_cast<const f32x4_t*>(x + 16 * j + 4 * q4);
  }
  static __device__ __forceinline__ void feat_of(const Row& r, Row& o, int phi) {
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
  static constexpr int FEAT_BYTES = J * CT * 1024;
  static __device__ __forceinline__ void put_feat(const Row& r, unsigned char* lds, int ct, int lane, int phi) {
    Row f;
    feat_of(r, f, phi);
#pragma unroll
    for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4_t*>(lds + (j * CT + ct) * 1024 + 16 * lane) = f.op[j];
  }
  struct Piece { f32x4_t x[CT]; };
  static __device__ __forceinline__ void get_feat(Piece& f, const unsigned char* lds, int j, int lane) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) f.x[ct] = *reinterpret_cast<const f32x4_t*>(lds + (j * CT + ct) * 1024 + 16 * lane);
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
          this->v[i][hf] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, off + stride * i + 256 * hf, 0, 0));
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
  static __device__ __forceinline__ void feature_scores(const Row& k, const unsigned char* lds, f32x4_t (&s)[CT], int lane, int phi) {
    Row f, q;
    feat_of(k, f, phi);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int j = 0; j < J; ++j) q.op[j] = *reinterpret_cast<const f32x4_t*>(lds + (j * CT + ct) * 1024 + 16 * lane);
      s[ct] = Base::dots(f, q);
    }
  }
  struct State {
    static constexpr int PARTS = D / 64;
    f32x4_t v[PARTS][4];
    __device__ __forceinline__ void load(const float* S, int j, int part, int r16, int q4) {
      const float* s = S + (size_t)(16 * j + 4 * q4) * D + 64 * part + 4 * r16;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[part][i] = *reinterpret_cast<const f32x4_t*>(s + i * D);
    }
    __device__ __forceinline__ void accumulate(const Piece& f, int part, f32x4_t (&acc)[CT][EV]) const {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) acc[ct][4 * part + e] = mfma(v[part][i][e], f.x[ct][i], acc[ct][4 * part + e]);
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

// Which (sequence, KV head) pair and which of its `blocks` work-group `id` has: eight pairs at a time, the blocks of each eight apart, so
// that those that read the same ring sit on one XCD, at the same time; fewer than eight pairs are spread over all XCDs (4 pairs of 256
// rows, W = 2048, 256 work-groups: 25.5 us on four XCDs, 16.4)
__device__ __forceinline__ unsigned tree_pair(unsigned id, unsigned pairs, unsigned blocks, int& block) {
  const unsigned side = pairs < 8 ? pairs : 8;
  block = id / side % blocks;
  return id / (side * blocks) * side + id % side;
}
inline long long tree_grid(const TreeDims& td, const TreePlan& pl) {
  const long long pairs = (long long)td.N * td.Hkv, side = pairs < 8 ? pairs : 8;
  return (pairs + side - 1) / side * side * pl.blocks;
}

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
        const int slot = t < W - slot0 ? slot0 + t : t - (W - slot0);
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
    f32x4_t g1 = {1.f, 1.f, 1.f, 1.f}, g2 = g1;
    if (a.gs) __builtin_memcpy(&g1, a.gs + head * D + d, 16);   // (gains need no more than a float's alignment)
    if (a.gr) __builtin_memcpy(&g2, a.gr + head * D + d, 16);
    store4(o + d, g1 * xs[h] * r1 + g2 * xr[h] * r2);
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
  const unsigned pairs = a.N * Hkv, per = SPLIT ? gridDim.x / split.n : gridDim.x;
  const int sp = SPLIT ? blockIdx.x / per : 0;
  int block;
  const unsigned pair = tree_pair(SPLIT ? blockIdx.x % per : blockIdx.x, pairs, a.blocks, block);
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
  auto node_rsrc = [&](const IO* x, int base) {   // nodes base .. cnt-1 of this sequence (of the last one only its D features)
    return make_rsrc(x + (size_t)base * Hkv * D, (unsigned)((cnt - 1 - base) * nstride + D * (int)sizeof(IO)));
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
    auto mask_ring = [&](f32x4_t (&s)[CT][NT], int base) {
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
    };
    auto mask_nodes = [&](f32x4_t (&s)[CT][NT], int base) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const unsigned see = (unsigned)(shfl64(node.anc & ~node.left, node_of[ct]) >> (base + 4 * q4));
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[ct][c][i] = see >> (16 * c + i) & 1 ? s[ct][c][i] : -INFINITY;
      }
    };
    // sets of ring keys (of rings in the tensors' type also of drafted keys, which come last)
    const int nloop = PACKED ? nring : nset;
    auto load_k = [&](int it) {
      if constexpr (!PACKED) {
        const bool r = it < nring;
        const int base = r ? ring_base(it) : (it - nring) * KEYS;
        ring.load_k(r ? make_rsrc(kr + (size_t)base * D, (unsigned)(min(KEYS, nvalid - base) * D * (int)sizeof(RT))) : node_rsrc(kn, base),
                    r ? D * (int)sizeof(RT) : nstride, r16, q4);
      } else load_ring_k(ring_base(it), nvalid - ring_base(it));
    };
    auto load_v = [&](int it) {
      if constexpr (!PACKED) {
        const bool r = it < nring;
        const int base = r ? ring_base(it) : (it - nring) * KEYS;
        ring.load_v(r ? make_rsrc(vr + (size_t)base * D, (unsigned)(min(KEYS, nvalid - base) * D * (int)sizeof(RT))) : node_rsrc(vn, base),
                    r ? D * (int)sizeof(RT) : nstride, r16, q4);
      } else load_ring_v(ring_base(it), nvalid - ring_base(it));
    };
    int it = w0;
    if (PACKED || it < nring) {
      // (requested in front of the tree's walk, above)
    } else if (it < nloop) { load_k(it); load_v(it); }
#pragma unroll 1
    while (it < nloop) {
      const int now = it;
      it += nw;
      f32x4_t s[CT][NT];
      ring.scores(q, s);
      if (it < nloop) load_k(it);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int c = 0; c < NT; ++c) s[ct][c] *= sc;
      if (PACKED || now < nring) mask_ring(s, ring_base(now)); else mask_nodes(s, (now - nring) * KEYS);
      typename Math::Weights pw[CT];
      softmax_step(s, pw);
      ring.accumulate(pw, acc);
      if (it < nloop) load_v(it);
    }
    if constexpr (PACKED) {
#pragma unroll 1
      for (; it < nset; it += nw) {
        const int base = (it - nring) * KEYS;
        NodeRows rows;
        rows.load_k(node_rsrc(kn, base), nstride, r16, q4);
        rows.load_v(node_rsrc(vn, base), nstride, r16, q4);
        f32x4_t s[CT][NT];
        rows.scores(q, s);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int c = 0; c < NT; ++c) s[ct][c] *= sc;
        mask_nodes(s, base);
        typename Math::Weights pw[CT];
        softmax_step(s, pw);
        rows.accumulate(pw, acc);
      }
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
    unsigned char* feats = reinterpret_cast<unsigned char*>(part + w * CT * 16 * LD);   // (free until the waves meet)
    static_assert(Math::FEAT_BYTES <= CT * 16 * LD * 4, "features of a wave's rows");
    const TreeNodes node = tree_nodes(up, W, lane);
    depths(node);
    // Keys that leave: ring tokens in slots slot0 .., then 0 ..; then drafted ones, where a path is longer than the window.  Of the
    // waves the last come first (the first ones may have a piece of the state more)
    const bool any = p >= W - dmax;
    const int nleave = any ? min(dmax + 1, W) : 0, len0 = min(nleave, W - slot0), sets0 = (len0 + KEYS - 1) / KEYS;
    const int sets = sets0 + (nleave - len0 + KEYS - 1) / KEYS, nodes = any && dmax >= W ? (cnt + KEYS - 1) / KEYS : 0;
    auto leave_base = [&](int x) { return x < sets0 ? slot0 + x * KEYS : (x - sets0) * KEYS; };
    auto leave_rows = [&](int x) {   // (a ring that is not full: the first of those slots hold nothing yet)
      return min(KEYS, min(x < sets0 ? slot0 + len0 : nleave - len0, nvalid) - leave_base(x));
    };
    auto load_leaving = [&](int x) {
      if (x < sets && leave_rows(x) > 0) {
        load_ring_k(leave_base(x), leave_rows(x));
        load_ring_v(leave_base(x), leave_rows(x));
      }
    };
    int x = nw - 1 - w0;
    load_leaving(x);
    if (any) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) Math::put_feat(q[ct], feats, ct, lane, a.phi);
    }
#pragma unroll 1
    for (; x < sets; x += nw) {
      const int base = leave_base(x), rows = leave_rows(x);
      if (rows > 0) {
        f32x4_t s[CT][NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          typename Math::Row kx;
          ring.key_row(c, kx);
          f32x4_t t[CT];
          Math::feature_scores(kx, feats, t, lane, a.phi);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 16 * c + 4 * q4 + i, j = r < rows ? age(base + r) : W;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][c][i] = j <= depth[ct] && j < W ? t[ct][i] : 0.f;
          }
        }
        typename Math::Weights pw[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) Math::weights(s[ct], pw[ct]);
        ring.accumulate(pw, acc);
      }
      load_leaving(x + nw);
    }
#pragma unroll 1
    for (; x < sets + nodes; x += nw) {
      const int base = (x - sets) * KEYS;
      NodeRows rows;
      rows.load_k(node_rsrc(kn, base), nstride, r16, q4);
      rows.load_v(node_rsrc(vn, base), nstride, r16, q4);
      f32x4_t s[CT][NT];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        typename Math::Row kx;
        rows.key_row(c, kx);
        f32x4_t t[CT];
        Math::feature_scores(kx, feats, t, lane, a.phi);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const unsigned see = (unsigned)(shfl64(node.left, node_of[ct]) >> (base + 4 * q4));
#pragma unroll
          for (int i = 0; i < 4; ++i) s[ct][c][i] = see >> (16 * c + i) & 1 ? t[ct][i] : 0.f;
        }
      }
      typename Math::Weights pw[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) Math::weights(s[ct], pw[ct]);
      rows.accumulate(pw, acc);
    }
    // pieces of the state, each part of the next one under way when this one's products are done
    if (p > W && w0 < Math::J) {
      const float* S = a.state + (size_t)pair * D * D;
      typename Math::State st;
#pragma unroll
      for (int h = 0; h < Math::State::PARTS; ++h) st.load(S, w0, h, r16, q4);
      for (int j = w0; j < Math::J; j += nw) {
        typename Math::Piece f;
        Math::get_feat(f, feats, j, lane);
#pragma unroll
        for (int h = 0; h < Math::State::PARTS; ++h) {
          st.accumulate(f, h, acc);
          if (j + nw < Math::J) st.load(S, j + nw, h, r16, q4);
        }
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
  f32x4_t xs[NH], xr[NH];
  float top, den;
  auto add_up = [&](int turn) {
    const int t = min(turn_row(turn), ROWS - 1);
    top = -1.0e30f;
    den = 0.f;
#pragma unroll
    for (int h = 0; h < NH; ++h) xs[h] = xr[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // (a factor for either branch: what is no finite number in one of them is looked at again in both anyway)
    float mk[KG], lk[KG];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
      mk[k] = ml[slice(t, k) * 2];
      lk[k] = ml[slice(t, k) * 2 + 1];
      top = fmaxf(top, k < KW ? mk[k] : top);
    }
#pragma unroll
    for (int k = 0; k < KG; ++k) {
      const float f = k < KW ? Math::pexp(mk[k] - top) : 0.f, add = k < KW ? 0.f : 1.f;
      den += k < KW ? f * lk[k] : 0.f;
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(part + slice(t, k) * LD + 64 * h + 4 * r16);
        xs[h] += f * x;
        xr[h] += add * x;
      }
    }
  };
  unsigned again = 0;   // turns whose row has something that is no finite number
  auto out = [&](int turn) {
    const int t = turn_row(turn);
    if (!tree_row_out<IO, RT, D>(a, n, g, row0 + t, r16, xs, xr, den, t < ROWS && row0 + t < nrows)) again |= 1u << turn;
  };
  if constexpr (!SPLIT) {
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) { add_up(turn); out(turn); }
  } else {
    // the sums of all work-groups of these rows, by the one that arrives last (see SplitArgs)
    constexpr int LINE = SplitArgs::row(D), AT_ONCE = 4;
    const size_t cell = (size_t)pair * a.blocks + block;
    const rsrc_t mem = make_rsrc(split.part + cell * split.n * ROWS * LINE, (unsigned)(split.n * ROWS * LINE * 4));
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
      const int t = turn_row(turn), at = (sp * ROWS + t) * LINE * 4;
      add_up(turn);
      if (t >= ROWS || row0 + t >= nrows) continue;
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        put_shared16(mem, xs[h], at + 256 * h + 16 * r16);
        put_shared16(mem, xr[h], at + 4 * D + 256 * h + 16 * r16);
      }
      if (r16 == 0) put_shared16(mem, f32x4_t{top, den, 0.f, 0.f}, at + 8 * D);
    }
    if (!arrive_last(split.ticket + cell, split.nonce, nsplit)) return;
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
      const int t = turn_row(turn);
      top = -1.0e30f;
      den = 0.f;
#pragma unroll
      for (int h = 0; h < NH; ++h) xs[h] = xr[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (t < ROWS && row0 + t < nrows)
#pragma unroll 1
        for (int k0 = 0; k0 < nsplit; k0 += AT_ONCE) {
          f32x4_t x[AT_ONCE][NH], y[AT_ONCE][NH], md[AT_ONCE];
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k) {
            const int at = (min(k0 + k, nsplit - 1) * ROWS + t) * LINE * 4;
            md[k] = get_shared16(mem, at + 8 * D);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              x[k][h] = get_shared16(mem, at + 256 * h + 16 * r16);
              y[k][h] = get_shared16(mem, at + 4 * D + 256 * h + 16 * r16);
            }
          }
          float to = top;
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k) to = fmaxf(to, md[k][0]);
          const float keep = Math::pexp(top - to);
          top = to;
          den *= keep;
#pragma unroll
          for (int h = 0; h < NH; ++h) xs[h] *= keep;
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k)
            if (k0 + k < nsplit) {
              const float f = Math::pexp(md[k][0] - to);
              den += f * md[k][1];
#pragma unroll
              for (int h = 0; h < NH; ++h) { xs[h] += f * x[k][h]; xr[h] += y[k][h]; }
            }
        }
      out(turn);
    }
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

template <typename IO, typename RT> TreeArgs<IO, RT> tree_args(const TreeDims& td, const TreeTensors& t, const TreePlan& pl) {
  return {(const IO*)t.q, (const IO*)t.k, (const IO*)t.v, t.parent, t.count, t.pos, (const RT*)t.k_ring, (const RT*)t.v_ring,
          (const float*)t.state, t.gs, t.gr, (IO*)t.o, td.N, td.M, td.Hq, td.Hkv, td.W, td.G, pl.blocks, td.phi, td.scale, td.eps,
          (const uint8_t*)t.k_scale, (const uint8_t*)t.v_scale};
}

template <typename IO, typename RT, int D, int CT, int KG, int NW, bool SPLIT>
void launch_tree(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
  const size_t bytes = tree_lds_bytes(D, CT, NW);
  static const bool attr = hipFuncSetAttribute(reinterpret_cast<const void*>(tree_kernel<IO, RT, D, CT, KG, NW, SPLIT>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
  (void)attr;
  const TreeArgs<IO, RT> a = tree_args<IO, RT>(td, t, pl);
  std::conditional_t<SPLIT, SplitArgs, NoSplit> split;
  if constexpr (SPLIT)
    split = {(float*)((char*)td.workspace + pl.part_off), (unsigned long long*)td.workspace, td.nonce, pl.nsplit, 0};
  const long long grid = tree_grid(td, pl) * (SPLIT ? pl.nsplit : 1);
  tree_kernel<IO, RT, D, CT, KG, NW, SPLIT><<<(unsigned)grid, NW * 64, bytes, st>>>(a, pl.KW, split);
}

template <typename IO, typename RT, int D>
void pick_tree(const TreeDims& td, const TreeTensors& t, const TreePlan& pl, hipStream_t st) {
#define RATTN_TREE(CT_, KG_, NW_)                                                                   \
  if (pl.CT == CT_ && pl.KG == KG_ && pl.NW == NW_) {                                               \
    if constexpr (KG_ == 8) {   /* (the others have too many work-groups to share keys) */          \
      if (td.workspace && pl.nsplit > 1) {                                                          \
        launch_tree<IO, RT, D, CT_, KG_, NW_, true>(td, t, pl, st);                                 \
        return;                                                                                     \
      }                                                                                             \
    }                                                                                               \
    launch_tree<IO, RT, D, CT_, KG_, NW_, false>(td, t, pl, st);                                    \
    return;                                                                                         \
  }
  RATTN_TREE(1, 8, 8)
  if constexpr (sizeof(IO) == 4) {
    RATTN_TREE(1, 4, 8)
  } else {
    RATTN_TREE(1, 4, 4)
    RATTN_TREE(2, 8, 8)
    RATTN_TREE(2, 4, 4)
    RATTN_TREE(2, 4, 8)
  }
#undef RATTN_TREE
}

}  // namespace

}  // namespace rattn
