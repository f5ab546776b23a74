// The handle of a rotary table, shared by the calls that take one.
#pragma once

#include "../../include/ravel_decode.h"
#include "decode.h"

struct ravel_rotary_ctx {
  ravel::RotaryTable table{};
  int device = 0, num_sms = 0;
};

namespace ravel {
// f_i / (2 pi) modulo 1 in units of 2^-64
unsigned long long rotary_turns(const ravel_rotary_config& c, int i);
}
