// The 8-bit cache as host and kernels share it.
#pragma once
#include <stdint.h>

namespace arckv {

constexpr int kQBlock = 64;         // tokens that share a scale

// The cache arrays of a call (device pointers) and their geometry.
struct QCache {
  uint8_t *K, *V;        // codes [P][rows][128]
  float *Ks, *Vs;        // scales [P][nblk]
  uint8_t *bounds;       // smallest and largest key code per channel [P][nblk][2][128], or null
  int P, rows, nblk;
};

}  // namespace arckv
