// What the kernels that read a layer's rings share: memory behind buffer resources, sets of ring rows as operands of the matrix
// cores (rings in the type of the tensors, or packed), and the meeting of work-groups that share a ring.
#pragma once
#include "common.hpp"
#include "kernels.hpp"
#include "mfma.hpp"
#include "packed.hpp"
#include <type_traits>

namespace rattn {

namespace {

__device__ __forceinline__ f32x4_t mfma16_f32(float a, float b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Memory behind a buffer resource: accesses past its `bytes` touch nothing (reads return zero), so the last set of a ring
// needs no per-row address selection, and a lane's address is one 32-bit offset.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t make_rsrc(const void* base, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// Keeps the compiler from reasoning about a per-lane value: offsets built from it stay one register plus an immediate,
// and what is computed from it inside a loop is not hoisted out of it into registers.
__device__ __forceinline__ int opaque(int x) { asm volatile("" : "+v"(x)); return x; }
// ONCE: marked non-temporal
template <typename V, bool ONCE = false> __device__ __forceinline__ V buf_load(rsrc_t r, int off) {
  if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, ONCE ? 2 : 0));
  else return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, ONCE ? 2 : 0));
}
__device__ __forceinline__ void buf_store(rsrc_t r, f32x4_t v, int off) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, off, 0, 0);
}

// A set of ring rows as one wave holds it (lane = 16*q4 + r16), for the two window contractions on 16 x 16 matrix-core
// tiles whose columns are the query heads of the group:
//   S^T[key][head] = K Q^T : A rows are keys, read straight from the ring in operand layout (lane = key row r16, a
//       16-byte piece of its features per lane group q4; the feature order of the contraction is free as long as the q
//       operand follows it).  The result has key 16c + 4*q4 + i of head r16 in register i of tile c.
//   O^T[d][head] = V^T P^T : the probabilities stay in the registers the first product left them in; as a B operand
//       they pin which keys contraction slot (q4, .) stands for, and lane group q4 loads the V rows of exactly those
//       keys, lane r16 taking the r16-th piece (EV features) of each row.
// bf16: 32 keys, 16x16x32 tiles; fp32: 16 keys, 16x16x4 tiles (exact fp32 products and sums).
template <typename IO, typename RT, int D, bool ONCE> struct RingSet;

// x as three bf16 terms of 8 bits, together exact; x is left with what they leave
__device__ __forceinline__ void three_terms(float (&x)[8], bf16x8_t (&term)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float t[8];
    term[k] = pack_bf16x8(x);
    unpack_bf16x8(term[k], t);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= t[i];  // exact
  }
}
// The fp32 probabilities pass through the bf16 tiles as three terms of 8 bits whose products share one accumulator, which is
// as good as fp32 products with the bf16 values (one term: 1.12 - 1.16 times the error of the output against fp64,
// which is mostly the output's own rounding).  The extra products hide behind the rings: 24 x 8 KV heads, W = 2048, 39.9 us
// either way, packed 25.5 against 25.2 with two terms; one sequence, where they are part of the chain, 11.2 us against 10.8.
__device__ __forceinline__ void prob_terms(const f32x4_t (&p)[2], bf16x8_t (&pop)[3]) {
  float r[8] = {p[0][0], p[0][1], p[0][2], p[0][3], p[1][0], p[1][1], p[1][2], p[1][3]};
  three_terms(r, pop);
}
// acc[e] += V^T P^T for feature EV*r16 + e of each lane's piece; two rows are interleaved per dword with v_perm_b32
template <int EV, typename ROW>
__device__ __forceinline__ void accumulate_bf16(const ROW (&v)[8], const bf16x8_t (&pop)[3], f32x4_t* acc) {
#pragma unroll
  for (int e = 0; e < EV; ++e) {
    const int j = e >> 1;
    const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
    u32x4_t a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(v[2 * i + 1][j], v[2 * i][j], sel);
#pragma unroll
    for (int term = 2; term >= 0; --term)
      acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), pop[term], acc[e], 0, 0, 0);
  }
}

template <int D, bool ONCE> struct RingSet<bf16_t, bf16_t, D, ONCE> {
  static constexpr int KEYS = 32, EV = D / 16;
  static constexpr bool K_AHEAD = false;
  typedef uint32_t vrow_t __attribute__((ext_vector_type(EV / 2)));
  bf16x8_t k[2][D / 32];
  vrow_t v[8];
  __device__ __forceinline__ void load_k(rsrc_t rows, int r16, int q4) {
    const int off = opaque(2 * D * r16 + 16 * q4);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int offc = c ? opaque(off + 32 * D) : off;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) k[c][j] = buf_load<bf16x8_t, ONCE>(rows, offc + 64 * j);
    }
  }
  __device__ __forceinline__ void load_v(rsrc_t rows, int r16, int q4) {
    const int off = opaque(8 * D * q4 + 2 * EV * r16), off1 = opaque(off + 32 * D);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = buf_load<vrow_t, ONCE>(rows, (u < 4 ? off : off1) + 2 * D * (u & 3));
  }
  // q: this lane's head in LDS
  __device__ __forceinline__ void scores(const bf16_t* q, int q4, f32x4_t (&s)[2]) const {
    s[0] = s[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const bf16x8_t op = *reinterpret_cast<const bf16x8_t*>(q + 32 * j + 8 * q4);
#pragma unroll
      for (int c = 0; c < 2; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c][j], op, s[c], 0, 0, 0);
    }
  }
  static __device__ __forceinline__ float pexp(float x, float m) { return fast_exp2(x - m); }
  __device__ __forceinline__ void accumulate(const f32x4_t (&p)[2], f32x4_t (&acc)[EV]) const {
    bf16x8_t pop[3];
    prob_terms(p, pop);
    accumulate_bf16<EV>(v, pop, acc);
  }
  // feature held by element (e, i) of a lane's accumulators
  static __device__ __forceinline__ int feature0(int e4, int i, int q4) { return EV * (4 * q4 + i) + 4 * e4; }
};

template <int D, bool ONCE> struct RingSet<float, float, D, ONCE> {
  static constexpr int KEYS = 16, EV = D / 16;
  static constexpr bool K_AHEAD = true;
  f32x4_t k[D / 16];
  f32x4_t v[4][D / 64];
  __device__ __forceinline__ void load_k(rsrc_t rows, int r16, int q4) {
    const int off = opaque(4 * D * r16 + 16 * q4);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) k[j] = buf_load<f32x4_t, ONCE>(rows, off + 64 * j);
  }
  __device__ __forceinline__ void load_v(rsrc_t rows, int r16, int q4) {
    const int off = opaque(16 * D * q4 + 16 * r16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int hf = 0; hf < D / 64; ++hf) v[i][hf] = buf_load<f32x4_t, ONCE>(rows, off + 4 * D * i + 256 * hf);
  }
  // Short chains of products and a tree of sums: the rounding of the logits grows with the chain.  With all features in two
  // chains it was 2.1 times that of the sums of partial sums per lane before (error of o at logits of std 4: 5.5e-7, 2.7e-7).
  __device__ __forceinline__ void scores(const float* q, int q4, f32x4_t (&s)[1]) const {
    f32x4_t t[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const f32x4_t op = *reinterpret_cast<const f32x4_t*>(q + 16 * j + 4 * q4);
      f32x4_t u[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e & 1] = mfma16_f32(k[j][e], op[e], u[e & 1]);
      t[j] = u[0] + u[1];
    }
#pragma unroll
    for (int n = D / 32; n > 0; n >>= 1)
#pragma unroll
      for (int j = 0; j < n; ++j) t[j] += t[j + n];
    s[0] = t[0];
  }
  static __device__ __forceinline__ float pexp(float x, float m) { return expf(x - m); }
  __device__ __forceinline__ void accumulate(const f32x4_t (&p)[1], f32x4_t (&acc)[EV]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int hf = 0; hf < D / 64; ++hf)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[4 * hf + e] = mfma16_f32(v[i][hf][e], p[0][i], acc[4 * hf + e]);
  }
  static __device__ __forceinline__ int feature0(int e4, int i, int q4) { return 64 * e4 + 4 * (4 * q4 + i); }
};

// Packed rings: 32 keys, whose values the tiles take as bf16, exactly; the scale is applied by the conversion.  A lane's 16 bytes
// of a K row are 16 features, two operand pieces (q follows).  fp32 q goes through the bf16 tiles as three terms of 8 bits, like
// the probabilities: exact products again.  Scales come one by one from their own bytes, so that rows behind the last one read
// as zero whatever the ring's length and alignment.
template <typename IO, int D, bool ONCE> struct RingSet<IO, fp8_t, D, ONCE> {
  static constexpr int KEYS = 32, EV = D / 16;
  static constexpr bool K_AHEAD = true;
  u32x4_t k[2][D / 64];
  uint32_t v[8][EV / 4];
  uint8_t ks[2][D / 64], vs[8];
  __device__ __forceinline__ void load_k(rsrc_t rows, rsrc_t scales, int r16, int q4) {
    const int off = opaque(D * r16 + 16 * q4), soff = opaque(scale_bytes(D) * r16 + (q4 >> 1));
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) k[c][j] = buf_load<u32x4_t, ONCE>(rows, off + 16 * D * c + 64 * j);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        ks[c][j] = __builtin_amdgcn_raw_buffer_load_b8(scales, soff + 16 * scale_bytes(D) * c + 2 * j, 0, 0);
  }
  __device__ __forceinline__ void load_v(rsrc_t rows, rsrc_t scales, int r16, int q4) {
    const int off = opaque(4 * D * q4 + EV * r16), soff = opaque(4 * scale_bytes(D) * q4 + EV * r16 / 32);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int row = (u < 4 ? 0 : 16) + (u & 3);
      if constexpr (EV == 8) {
        const u32x2_t x = buf_load<u32x2_t, ONCE>(rows, off + D * row);
        v[u][0] = x[0];
        v[u][1] = x[1];
      } else {
        v[u][0] = __builtin_amdgcn_raw_buffer_load_b32(rows, off + D * row, 0, ONCE ? 2 : 0);
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      vs[u] = __builtin_amdgcn_raw_buffer_load_b8(scales, soff + scale_bytes(D) * ((u < 4 ? 0 : 16) + (u & 3)), 0, 0);
  }
  // operand pieces 2j, 2j + 1 of rows 16c + r16: features 64j + 16 q4 + 0 .. 7 and + 8 .. 15
  __device__ __forceinline__ void operands(int c, int j, bf16x8_t& a, bf16x8_t& b) const {
    const float f = scale_of(ks[c][j]);
    u32x4_t x, y;
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack_bf16x4(k[c][j][i], f, t[2 * i], t[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = t[i]; y[i] = t[4 + i]; }
    a = __builtin_bit_cast(bf16x8_t, x);
    b = __builtin_bit_cast(bf16x8_t, y);
  }
  __device__ __forceinline__ void scores(const IO* q, int q4, f32x4_t (&s)[2]) const {
    s[0] = s[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      bf16x8_t a[2][2];
      operands(0, j, a[0][0], a[0][1]);
      operands(1, j, a[1][0], a[1][1]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const IO* piece = q + 64 * j + 16 * q4 + 8 * h;
        if constexpr (sizeof(IO) == 2) {
          const bf16x8_t op = *reinterpret_cast<const bf16x8_t*>(piece);
#pragma unroll
          for (int c = 0; c < 2; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c][h], op, s[c], 0, 0, 0);
        } else {
          const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(piece), hi = *reinterpret_cast<const f32x4_t*>(piece + 4);
          float r[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          bf16x8_t op[3];
          three_terms(r, op);
#pragma unroll
          for (int c = 0; c < 2; ++c) {   // (a sum of its own for every piece: rounding grows with the length of a chain)
            f32x4_t t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int term = 2; term >= 0; --term) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c][h], op[term], t, 0, 0, 0);
            s[c] += t;
          }
        }
      }
    }
  }
  static __device__ __forceinline__ float pexp(float x, float m) { return sizeof(IO) == 2 ? fast_exp2(x - m) : expf(x - m); }
  __device__ __forceinline__ void accumulate(const f32x4_t (&p)[2], f32x4_t (&acc)[EV]) const {
    bf16x8_t pop[3];
    prob_terms(p, pop);
#pragma unroll
    for (int i = 0; i < EV / 4; ++i) {   // four features of each piece at a time: the unpacked rows are all of V's otherwise
      u32x2_t rows[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        uint32_t lo, hi;
        unpack_bf16x4(v[u][i], scale_of(vs[u]), lo, hi);
        rows[u] = u32x2_t{lo, hi};
      }
      accumulate_bf16<4>(rows, pop, acc + 4 * i);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  static __device__ __forceinline__ int feature0(int e4, int i, int q4) { return EV * (4 * q4 + i) + 4 * e4; }
};

// scales of packed rings; rings in the type of the tensors have none
template <typename RT> struct RingScales {
  static constexpr uint8_t *k = nullptr, *v = nullptr;
  RingScales(uint8_t*, uint8_t*) {}
};
template <> struct RingScales<fp8_t> {
  uint8_t *k, *v;
  RingScales(uint8_t* ks, uint8_t* vs) : k(ks), v(vs) {}
};
// element i of a ring as a number
template <typename RT> __device__ __forceinline__ float ring_value(const RT* ring, const uint8_t* scales, size_t i) {
  if constexpr (sizeof(RT) == 1) return unpack_one(ring[i].b, scales[i >> 5]);
  else return io_traits<RT>::ld(ring + i);
}

// Where few (sequence, kv head) pairs have long rings, several work-groups share each (decode_split, with times): a CU takes in
// some 59 bytes a nanosecond, a hundredth of what the memory delivers.  Every work-group leaves the partial
// results of its share of ring and state rows in the workspace; the one that arrives last adds them up in order (no matter who
// that is), forms the output and puts the new token into its slot, from which everyone has taken the evicted one by then.
// Nobody waits for anybody.
// Arrivals are counted in a ticket per pair, nonce | count.  The workspace is not initialised: a ticket whose upper 56 bits are
// not this call's nonce counts as zero, and the last arrival clears it, so that a captured launch finds none of its own
// when it is replayed.  (A ticket that holds the nonce by accident, one in 2^56, is the one case that goes wrong.)
struct SplitArgs {
  float* part;                   // [pair][work-group][head][row]: window sums, state sums, maximum, sum of exponentials
  unsigned long long* ticket;    // [pair]
  unsigned long long nonce;      // low 8 bits zero
  int n, rows;                   // work-groups per pair, 2 .. DEC_MAX_SPLIT, and ring rows for each before there is another
  static constexpr __host__ __device__ int row(int D) { return 2 * D + 4; }
};
struct NoSplit {
  static constexpr float* part = nullptr;
  static constexpr unsigned long long *ticket = nullptr, nonce = 0;
  static constexpr int n = 1, rows = 1;
};
// Stores and loads of agent scope meet in memory, past the caches of an XCD.  So the order of a wave's own accesses is all
// that an arrival needs: its stores are complete (vmcnt) before its work-group is counted, and the last one's loads are issued
// after it was.  A release and an acquire of agent scope instead write back and drop the XCD's whole L2 for every
// work-group: 12.0 -> 22.8 us at 16 work-groups for each of 4 pairs, 24 -> 83 at 4 for 256, where this way takes 18.2 and 30.4.
__device__ __forceinline__ void put_shared(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get_shared(const float* p) { return __hip_atomic_load(const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// 16 bytes in one access (bit 4: agent scope)
__device__ __forceinline__ void put_shared16(rsrc_t r, f32x4_t v, int off) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, off, 0, 16);
}
__device__ __forceinline__ f32x4_t get_shared16(rsrc_t r, int off) {
  return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 16));
}
// Called by the whole work-group after its put_shared; true in the one that arrives last, whose get_shared then see everyone's
__device__ __forceinline__ bool arrive_last(unsigned long long* ticket, unsigned long long nonce, int n) {
  __shared__ int last;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  wait_vmem();  // this wave's stores are in memory
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __syncthreads();
  if (threadIdx.x == 0) {
    // A cleared ticket gets the nonce from whoever comes first, and one more arrival is counted, in one trip to memory
    unsigned long long old = 0, now;
    __hip_atomic_compare_exchange_strong(ticket, &old, nonce, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    now = __hip_atomic_fetch_add(ticket, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    // Added to something else: counted again by exchange (which fails only because another of the n arrivals came in between,
    // n rounds at most for each of its two kinds)
    if ((now & ~255ull) != nonce) {
      old = now;
      do now = (old & ~255ull) == nonce ? old + 1 : nonce + 1;
      while (!__hip_atomic_compare_exchange_strong(ticket, &old, now, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    }
    last = (int)(now & 255) == n;
    if (last) __hip_atomic_store(ticket, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return last != 0;
}

}  // namespace

}  // namespace rattn
