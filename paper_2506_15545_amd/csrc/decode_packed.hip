// Decode step over packed rings (packed.hpp): see decode_group.hpp.
#include "decode_group.hpp"

namespace rattn {

void decode_step_packed(const DecodeDims& dd, int dtype, const void* q, const void* k_new, const void* v_new, const int32_t* pos,
                        void* k_ring, void* k_scale, void* v_ring, void* v_scale, float* state, const float* gs, const float* gr,
                        void* o, hipStream_t st) {
  ProfScope ps("decode_packed_kernel", st);
  const DecodeTensors t = {q, k_new, v_new, pos, k_ring, v_ring, state, gs, gr, o, (uint8_t*)k_scale, (uint8_t*)v_scale};
#define RATTN_DECODE(IO, DD)                                          \
  do {                                                                \
    if (dd.G <= DEC_HB) pick_decode<IO, fp8_t, DD, false>(dd, t, st); \
    else pick_decode<IO, fp8_t, DD, true>(dd, t, st);                 \
  } while (0)
  if (dtype == 0) {
    if (dd.D == 64) RATTN_DECODE(float, 64); else RATTN_DECODE(float, 128);
  } else {
    if (dd.D == 64) RATTN_DECODE(bf16_t, 64); else RATTN_DECODE(bf16_t, 128);
  }
#undef RATTN_DECODE
}

}  // namespace rattn
