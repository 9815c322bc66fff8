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

// A row's largest magnitude m and what its codes need; s.inv = 0 where they are all zero.
struct Int8Row {
  double m, inv;  // inv = 1 / m
  float scale;
  bool near;      // m from 2^-60 to 2^100: binary32 quotients do but next to a tie
};
__device__ inline Int8Row int8_row(double m, double r) {
  Int8Row s;
  s.scale = (float)(m * r / 127.0);
  const bool fine = isfinite(s.scale);
  if (!fine) s.scale = NAN;
  s.m = m;
  s.inv = fine && m > 0.0 ? 1.0 / m : 0.0;
  s.near = s.inv != 0.0 && m >= 0x1p-60 && m <= 0x1p100;
  return s;
}

// The codes of eight numbers p of a row with s.near, by p fl(127 / m): its nearest integer comes out of an addition of
// 1.5 2^23, whose unit in the last place is 1.  The product is within 2^-16 of the quotient; where it is that near
// to a tie (a few of a thousand bfloat16 numbers have the largest one's significand, and are ties) the sign of
// 254 |p| - (2 k + 1) m decides, whose terms are exact in binary64: p and m have 24 bits.
__device__ inline uint64_t int8_codes8(const float p[8], const Int8Row &s) {
  constexpr float MAGIC = 12582912.0f, NEAR = 0.5f - 0x1p-15f;
  const float inv = (float)(127.0 * s.inv);
  uint32_t k[8];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = fmaf(p[i], inv, MAGIC);
    k[i] = __builtin_bit_cast(uint32_t, q);
    off = fmaxf(off, fabsf(fmaf(p[i], inv, MAGIC - q)));
  }
  if (off >= NEAR) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = fabsf(p[i]) * inv, whole = floorf(q);
      if (fabsf(q - whole - 0.5f) > 0.5f - NEAR) continue;
      const double over = fma(254.0, fabs((double)p[i]), -(double)(2.0f * whole + 1.0f) * s.m);
      const int up = over > 0.0 || (over == 0.0 && ((int)whole & 1)), size = (int)whole + up;
      k[i] = (uint32_t)(p[i] < 0.0f ? -size : size);
    }
  }
  const uint32_t a01 = __builtin_amdgcn_perm(k[1], k[0], 0x0c0c0400), a23 = __builtin_amdgcn_perm(k[3], k[2], 0x04000c0c);
  const uint32_t a45 = __builtin_amdgcn_perm(k[5], k[4], 0x0c0c0400), a67 = __builtin_amdgcn_perm(k[7], k[6], 0x04000c0c);
  return (uint64_t)(a45 | a67) << 32 | (a01 | a23);
}

// The codes of eight numbers of any row.
template <typename P>
__device__ inline uint64_t int8_codes8_any(const P p[8], const Int8Row &s) {
  uint64_t w = 0;
  if (s.inv == 0.0) return w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w |= (uint64_t)(int8_code((double)p[i], s.m, s.inv) & 255) << (8 * i);
  return w;
}

// |v| as an integer: in the order of magnitudes, infinities and then NaN above them.
__device__ inline uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

}  // namespace mcf
