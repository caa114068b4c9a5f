// Rotary positions as host and kernels share them.
#pragma once
#include <stdint.h>

namespace arckv {

struct RotaryRows {
  const void *x;
  void *y;
  int64_t x_token, x_head, y_token, y_head;   // in elements
};

struct Rotary {
  RotaryRows r[2];
  int heads[2];              // of the second: 0 where there is none
  int N, half;               // tokens, pairs
  int neighbours;
  float sign, factor;        // -1 turns back
  const int32_t *positions;  // or null
  const double *freq;
  uint32_t by_heads;         // 2^16 / heads, rounded up
};

}  // namespace arckv
