// The 4-bit cache as host and kernels share it.
#pragma once
#include <stdint.h>

namespace arckv {

constexpr int kNRow = 64;           // bytes of a row's codes
constexpr int kNGroup = 32;         // channels that share a scale

// The cache arrays of a call (device pointers) and their geometry.
struct NCache {
  uint8_t *K, *V;        // codes [P][rows][64]
  uint32_t *Ks, *Vs;     // scales [P][rows], a byte per group
  int P, rows;
};

}  // namespace arckv
