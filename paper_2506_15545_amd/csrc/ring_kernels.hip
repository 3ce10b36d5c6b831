// Rings between the type of the tensors and 8 bits (packed.hpp): what a program does with the rings that a prompt left before
// it decodes over packed ones, and with packed ones before it continues a prompt.
// Bound: HBM.  A thread has eight features, so that loads and stores of a wave are whole runs of memory, and a block's four
// threads meet in registers.  Both rings of 128 sequences of 8 KV heads, D = 128, W = 512, bf16: packed in 71 us, 5.7 TB/s (a large copy
// reaches 5.0); unpacked, 24 sequences, W = 2048, 54 us, 5.7 TB/s; one sequence of 4 KV heads 3.6 us, a launch.
#include "kernels.hpp"
#include "packed.hpp"

namespace rattn {

namespace {

// eight features of a row
template <typename IO> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4_t v;
  __device__ __forceinline__ void get(float (&x)[8]) const { unpack_bf16x8(__builtin_bit_cast(bf16x8_t, v), x); }
  // bf16 holds a packed value exactly
  __device__ __forceinline__ void set(u32x2_t codes, float f) {
    uint32_t a, b, c, d;
    unpack_bf16x4(codes[0], f, a, b);
    unpack_bf16x4(codes[1], f, c, d);
    v = u32x4_t{a, b, c, d};
  }
};
template <> struct Eight<float> {
  f32x4_t v[2];
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i >> 2][i & 3];
  }
  __device__ __forceinline__ void set(u32x2_t codes, float f) {
    v[0] = unpack_f32x4(codes[0], f);
    v[1] = unpack_f32x4(codes[1], f);
  }
};

constexpr int CONV_STEPS = 4;   // pieces of eight features in flight per thread

// n pieces of eight features in each of the two rings; work-groups alternate between runs of CONV_STEPS * 256 pieces
template <typename IO>
__global__ __launch_bounds__(256) void ring_pack_kernel(const Eight<IO>* __restrict__ k, const Eight<IO>* __restrict__ v,
                                                        u32x2_t* __restrict__ kc, uint8_t* __restrict__ ks,
                                                        u32x2_t* __restrict__ vc, uint8_t* __restrict__ vs, long long n) {
  const Eight<IO>* src = blockIdx.y ? v : k;
  u32x2_t* codes = blockIdx.y ? vc : kc;
  uint8_t* scales = blockIdx.y ? vs : ks;
  const long long first = (long long)blockIdx.x * (CONV_STEPS * 256) + threadIdx.x;
  Eight<IO> in[CONV_STEPS];
#pragma unroll
  for (int j = 0; j < CONV_STEPS; ++j)
    if (first + 256 * j < n) in[j] = src[first + 256 * j];
#pragma unroll
  for (int j = 0; j < CONV_STEPS; ++j) {
    const long long i = first + 256 * j;
    if (i >= n) break;   // (a row's pieces are a multiple of four: the threads of a block stay together)
    float x[8];
    in[j].get(x);
    float a = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a = fmaxf(a, finite_abs(x[e]));
    a = fmaxf(a, dpp_get<0xB1>(a));
    a = fmaxf(a, dpp_get<0x4E>(a));
    const uint32_t s = scale_byte(a);
    const float inv = inverse_factor(s);
    int lo = two_codes<false>(x[0], x[1], inv, 0), hi = two_codes<false>(x[4], x[5], inv, 0);
    lo = two_codes<true>(x[2], x[3], inv, lo);
    hi = two_codes<true>(x[6], x[7], inv, hi);
    codes[i] = u32x2_t{(unsigned)lo, (unsigned)hi};
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)s;
  }
}

template <typename IO>
__global__ __launch_bounds__(256) void ring_unpack_kernel(const u32x2_t* __restrict__ kc, const uint8_t* __restrict__ ks,
                                                          const u32x2_t* __restrict__ vc, const uint8_t* __restrict__ vs,
                                                          Eight<IO>* __restrict__ k, Eight<IO>* __restrict__ v, long long n) {
  const u32x2_t* codes = blockIdx.y ? vc : kc;
  const uint8_t* scales = blockIdx.y ? vs : ks;
  Eight<IO>* dst = blockIdx.y ? v : k;
  const long long first = (long long)blockIdx.x * (CONV_STEPS * 256) + threadIdx.x;
  u32x2_t c[CONV_STEPS];
  uint32_t s[CONV_STEPS];
#pragma unroll
  for (int j = 0; j < CONV_STEPS; ++j) {
    const long long i = first + 256 * j;
    if (i < n) { c[j] = codes[i]; s[j] = scales[i >> 2]; }
  }
#pragma unroll
  for (int j = 0; j < CONV_STEPS; ++j) {
    const long long i = first + 256 * j;
    if (i >= n) break;
    Eight<IO> out;
    out.set(c[j], scale_of(s[j]));
    dst[i] = out;
  }
}

}  // namespace

void ring_pack(int dtype, long long elements, const void* k, const void* v, void* kc, void* ks, void* vc, void* vs, hipStream_t st) {
  ProfScope ps("ring_pack_kernel", st);
  const long long n = elements / 8;
  const dim3 grid((unsigned)((n + CONV_STEPS * 256 - 1) / (CONV_STEPS * 256)), 2);
#define RATTN_PACK(IO)                                                                                                     \
  ring_pack_kernel<IO><<<grid, 256, 0, st>>>((const Eight<IO>*)k, (const Eight<IO>*)v, (u32x2_t*)kc, (uint8_t*)ks, (u32x2_t*)vc, \
                                             (uint8_t*)vs, n)
  if (dtype == 0) RATTN_PACK(float); else RATTN_PACK(bf16_t);
#undef RATTN_PACK
}

void ring_unpack(int dtype, long long elements, const void* kc, const void* ks, const void* vc, const void* vs, void* k, void* v,
                 hipStream_t st) {
  ProfScope ps("ring_unpack_kernel", st);
  const long long n = elements / 8;
  const dim3 grid((unsigned)((n + CONV_STEPS * 256 - 1) / (CONV_STEPS * 256)), 2);
#define RATTN_UNPACK(IO)                                                                                                   \
  ring_unpack_kernel<IO><<<grid, 256, 0, st>>>((const u32x2_t*)kc, (const uint8_t*)ks, (const u32x2_t*)vc, (const uint8_t*)vs, \
                                               (Eight<IO>*)k, (Eight<IO>*)v, n)
  if (dtype == 0) RATTN_UNPACK(float); else RATTN_UNPACK(bf16_t);
#undef RATTN_UNPACK
}

}  // namespace rattn
