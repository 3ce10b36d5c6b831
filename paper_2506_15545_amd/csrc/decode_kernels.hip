// Decode step of the RAttention layer over rings in the type of the tensors: see decode_group.hpp.
#include "decode_group.hpp"

namespace rattn {

void decode_step(const DecodeDims& dd, int dtype, const void* q, const void* k_new, const void* v_new,
                 const int32_t* pos, void* k_ring, void* v_ring, float* state, const float* gs, const float* gr,
                 void* o, hipStream_t st) {
  ProfScope ps("decode_kernel", st);
  const DecodeTensors t = {q, k_new, v_new, pos, k_ring, v_ring, state, gs, gr, o, nullptr, nullptr};
#define RATTN_DECODE(IO, DD)                            \
  do {                                                  \
    if (dd.G <= DEC_HB) pick_decode<IO, IO, DD, false>(dd, t, st);  \
    else pick_decode<IO, IO, DD, true>(dd, t, st);          \
  } while (0)
  if (dtype == 0) {
    if (dd.D == 64) RATTN_DECODE(float, 64); else RATTN_DECODE(float, 128);
  } else {
    if (dd.D == 64) RATTN_DECODE(bf16_t, 64); else RATTN_DECODE(bf16_t, 128);
  }
#undef RATTN_DECODE
}

}  // namespace rattn
