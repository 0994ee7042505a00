// Which document a token is in (also run by a CPU test).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xhc {

// The last i in 0 .. n with starts[i] <= t, where starts (ascending, n + 1 of
// them) begin at or in front of t; 0 where they do not.
__host__ __device__ inline int last_start(const int32_t* starts, int n, int t) {
  int a = 0, b = n;
  while (a < b) {
    const int c = b - (b - a) / 2;          // (the middle, upwards: a + b may pass 31 bits)
    if (starts[c] <= t) a = c; else b = c - 1;
  }
  return a;
}

}  // namespace xhc
