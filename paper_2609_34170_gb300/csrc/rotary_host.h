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

// Whether rows of `width` values, n for each of `batch` robots, may share memory: then they are not written, since
// threads would overwrite each other's results (in place: turn a row twice).
inline bool rows_overlap(int batch, int n, long long width, long long robot_stride, long long token_stride) {
  if ((n > 1 && token_stride < width) || (batch > 1 && robot_stride < width)) return true;
  if (n < 2 || batch < 2) return false;
  const bool inside = token_stride <= robot_stride;   // a robot's tokens lie between its start and the next one's
  const long long near = inside ? token_stride : robot_stride, far = inside ? robot_stride : token_stride;
  return (far - width) / near < (inside ? n : batch) - 1;
}
}  // namespace ravel
