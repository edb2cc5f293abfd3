// Rotary positions: the plan's table and the launch interface (internal).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cqsa.h"

namespace cqsa {

constexpr int kMaxPairs = 128;  // d = 256

// Turns a position of every pair, in units of 2^-64 turns (whole turns
// dropped), and the pair's axis.
struct RotaryTable {
  uint64_t turn[kMaxPairs];
  uint8_t axis[kMaxPairs];
};

struct RotaryArgs {
  struct Tensor {
    const void* x;
    void* y;
    int64_t x_b, x_l, x_h, y_b, y_l, y_h;  // strides in elements
  } t[2];
  const int32_t* pos;  // [n_axes, rows]
  int64_t rows;        // B * L
  int64_t row0;        // first row of this launch
  uint32_t n;          // threads of this launch with work
  uint32_t L;
  uint32_t H0, H;      // heads of the first tensor, of both
  uint32_t chunks;     // threads' chunks (two vectors of 16 bytes) of a head that are turned
  uint32_t units;      // and, out of place, those that are copied
  uint32_t parts;      // threads that share a row's heads
  uint32_t pairs;      // n: pairs that are turned
  int32_t inverse;
  RotaryTable tab;
};

constexpr int kRotaryBatch = 8;  // heads that a thread reads at a time

hipError_t launch_rotary(cqsa_dtype dt, bool adjacent, const RotaryArgs& a, hipStream_t s);

}  // namespace cqsa

struct cqsa_rotary_s {
  cqsa_rotary_opts opts;
  int32_t n;  // pairs
  cqsa::RotaryTable tab;
};
