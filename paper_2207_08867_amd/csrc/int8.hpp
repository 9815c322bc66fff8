// int8.hpp -- what the kernels on 8-bit tensors share.
//
// An 8-bit tensor of rows of n elements: codes [rows][P] signed bytes from -127 to 127, P the next
// multiple of 128 at or above n, zeros past n; scales [rows] binary32.  Element i of a row stands for
// code_i scale.  The padding spares the products a tail of the reduction and aligns every row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mcf {

inline __host__ __device__ int64_t int8_pitch(int64_t n) { return (n + 127) / 128 * 128; }

// The integer nearest 127 p / m, ties to even, of the binary64 quotient fl(fl(127 p) / m); inv = 1 / m.
// Multiplying by inv is off by a few units in the last place, which decides nothing but next to a tie: there
// the quotient itself is taken.
__device__ inline int int8_code(double p, double m, double inv) {
  const double t = 127.0 * p, q = t * inv;
  double k = rint(q);
  if (fabs(q - k) > 0.5 - 1e-9) k = rint(t / m);
  return (int)k;
}

}  // namespace mcf
