// Launch parameters of the 4-bit matrix kernels (host and device).
#pragma once

#include <stdint.h>

#include "../host/kparams.h"

namespace fluid {

// A matrix in 4 bits: words of a tile of 16 rows and 128 channels, then pairs.
struct W4Arg {
  const uint8_t* words;
  const uint8_t* pairs;
};

struct W4Params {
  W4Arg w, gate;       // gate: matmul only, words NULL for none
  int32_t n, k;        // rows and channels
  int32_t group;
  int32_t tiles, blocks;  // of 16 rows, of 128 channels
  const void* x;       // rows of the product, or the matrix to pack
  const void* add;     // NULL: none
  void* out;           // of the product, or the matrix read
  int64_t xs, as, os;  // their rows' strides in elements
  int32_t m;           // rows of x
  // few rows
  int32_t wide;   // two tiles to a workgroup
  int32_t waves;  // wavefronts that share a tile's channels
  // more
  int32_t splits;  // runs of blocks that workgroups of their own take; 0: few rows
  int32_t run;     // blocks of a run
  float* ws;       // splits > 1: [run][matrix][row][output] sums
};

}  // namespace fluid
