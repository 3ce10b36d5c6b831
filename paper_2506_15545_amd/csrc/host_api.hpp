// What the C entry points share (api.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rattn.h"

namespace rattn {

// `s`, with the detail that rattn_last_error returns
rattn_status fail(rattn_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
rattn_status check_launch(const char* what);
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// the parameters of a decode step, checked
rattn_status decode_dims(const rattn_decode_params* p, DecodeDims* dd);
unsigned long long decode_nonce();

}  // namespace rattn
