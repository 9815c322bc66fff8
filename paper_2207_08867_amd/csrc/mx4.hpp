// mx4.hpp -- what the kernels on microscaled 4-bit (MXFP4) tensors share: the element
// conversions of gfx950, 8-element loads and stores of plain tensors, and the splitting of
// wider formats into bfloat16 pieces.
//
// A block is 32 elements along a row.  An element is E2M1 (sign, 2 exponent bits, 1 mantissa
// bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), the block's scale E8M0 (byte s stands for 2^(s - 127), 255
// for NaN).  Four blocks form a group of 128 elements: 64 bytes of codes (element 2i in the low
// half of byte i) and one 32-bit word of scales.  Codes are [nc][rows][64 G] bytes, scales
// [nc][G][rows] words, G = ceil(n / 128): the words of neighbouring rows lie side by side, as the
// product kernels read them, and the zero padding of a row's last group spares them a K tail.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mcf {

constexpr int MX_GROUP = 128;
inline __host__ __device__ int64_t mx_groups(int64_t n) { return (n + MX_GROUP - 1) / MX_GROUP; }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef double f64x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <bool B>
struct Flag {
  static constexpr bool value = B;
};

// Eight elements of a plain tensor.  The address is aligned to the element only: rows of odd
// length start anywhere, and gfx950 loads 16 bytes from any address.
template <typename T>
struct Raw8 {
  T v[8];
};

template <typename T>
__device__ inline Raw8<T> load8(const T *p) {
  Raw8<T> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}

// Eight elements from p, of which those at or past `left` are read as zero.
template <typename T>
__device__ inline Raw8<T> load8_tail(const T *p, int64_t left) {
  if (left >= 8) return load8(p);
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = i < left ? p[i] : (T)0.0f;
  return r;
}

// Eight elements from column col of a row of n >= 8, as many as are left of it last and then others in front of them;
// load8_settle moves those down, where `left` are wanted, and fills up.  Apart, so that a wavefront's loads all go out
// before the first of them is looked at: a second form of a load, or a move right behind it, makes the wavefront wait
// there (a 4096 x 4096 bfloat16 norm 41 us, 27 so).
template <typename T>
__device__ inline Raw8<T> load8_clamped(const T *row, int64_t col, int64_t n) {
  // rows have at most 2^30 elements: a 32-bit offset to the row's start
  const uint32_t at = (uint32_t)(col < n - 8 ? col : n - 8) * (uint32_t)sizeof(T);
  return load8(reinterpret_cast<const T *>(reinterpret_cast<const char *>(row) + at));
}
template <typename T>
__device__ inline void load8_settle(Raw8<T> &r, int64_t left, T fill) {
  if (!__any(left < 8)) return;  // a scalar branch: nothing of what follows elsewhere
  constexpr int W = sizeof(r) / 4;
  // whole words, so that 16-bit elements stay packed
  uint32_t w[W], f;
  __builtin_memcpy(w, &r, sizeof(r));
  if constexpr (sizeof(T) == 2)
    f = (uint32_t)__builtin_bit_cast(uint16_t, fill) * 0x10001u;
  else
    f = __builtin_bit_cast(uint32_t, fill);
  const uint32_t over = left >= 8 ? 0u : (left > 0 ? (uint32_t)(8 - left) : 8u);
#pragma unroll
  for (int b = W; b; b >>= 1) {  // words
    const bool go = over & (uint32_t)(b * 8 / W);
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = go ? (i + b < W ? w[i + b] : f) : w[i];
  }
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = over & 1 ? __builtin_amdgcn_alignbit(i + 1 < W ? w[i + 1] : f, w[i], 16) : w[i];
  }
  __builtin_memcpy(&r, w, sizeof(r));
}
// Both.  EVEN: n is a multiple of 8 and col < n.
template <bool EVEN, typename T>
__device__ inline Raw8<T> load8_row(const T *row, int64_t col, int64_t n, T fill) {
  if constexpr (EVEN) return load8(row + col);
  Raw8<T> r = load8_clamped(row, col, n);
  load8_settle(r, n - col, fill);
  return r;
}

template <typename T>
__device__ inline void store8_tail(T *p, const Raw8<T> &r, int64_t left) {
  if (left >= 8) {
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = r.v[i];
  }
}

// Held elements as another value, so that the compiler works out again what follows from them (wider forms of 16-bit
// ones, say) instead of holding it.
template <typename T>
__device__ inline Raw8<T> renewed(const Raw8<T> &r) {
  u32x4 u[sizeof(T) / 2];
  __builtin_memcpy(&u, &r, sizeof(u));
  if constexpr (sizeof(T) == 2)
    asm volatile("" : "+v"(u[0]));
  else
    asm volatile("" : "+v"(u[0]), "+v"(u[1]));
  Raw8<T> o;
  __builtin_memcpy(&o, &u, sizeof(u));
  return o;
}

// Eight E2M1 codes (one word) of a block as bfloat16 values.  scale: the binary32 number whose
// exponent field is the block's scale byte (byte << 23; the conversion reads that field alone, 0
// standing for 2^-127 and 255 for NaN).  Exact but for a value past bfloat16's range (inf).
__device__ inline bf16x8 mx_bf16(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  bf16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  return r;
}

// The same as binary16; exact where the scale is between 2^-23 and 2^13.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ inline f16x8 mx_f16(uint32_t w, float scale) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
  f16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  return r;
}

__device__ inline void mx_f32(uint32_t w, float scale, float v[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

__device__ inline float mx_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// The number of bfloat16 pieces that hold a value of T exactly (8 significant bits each; the
// last of a binary32 value below 2^-100 may lose bits under bfloat16's smallest number).
template <typename T>
constexpr int mx_pieces() {
  return sizeof(T) == 4 ? 3 : (__is_same(T, __bf16) ? 1 : 2);
}

// v = p[0] + p[1] + ..., each piece the leading 8 bits of what is left, of v's sign, its bfloat16 bits in
// the upper half of p[i].  T: the format v comes from.  The median of the remainder, 0 and v is the
// remainder of a finite v; of an infinity the remainder is NaN, which a median ignores, and the
// later pieces are 0 or the infinity again: its products are those of one 16-bit number.
template <typename T, int P>
__device__ inline void mx_cut(float v, uint32_t p[P]) {
  // a NaN of the lower half's bits alone would turn into an infinity
  float r = sizeof(T) == 4 ? __builtin_canonicalizef(v) : v;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    p[i] = __builtin_bit_cast(uint32_t, r);
    if (i + 1 < P) r = __builtin_amdgcn_fmed3f(r - __builtin_bit_cast(float, p[i] & 0xffff0000u), 0.0f, r);
  }
}

// Eight values into P registers of eight pieces.
template <typename T, int P>
__device__ inline void mx_cut8(const Raw8<T> &x, bf16x8 f[P]) {
  if constexpr (P == 1) {
    f[0] = __builtin_bit_cast(bf16x8, x);
  } else {
    u32x4 w[P];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      uint32_t p[P], q[P];
      mx_cut<T, P>((float)x.v[i], p);
      mx_cut<T, P>((float)x.v[i + 1], q);
#pragma unroll
      for (int k = 0; k < P; ++k) w[k][i / 2] = __builtin_amdgcn_perm(q[k], p[k], 0x07060302);
    }
#pragma unroll
    for (int k = 0; k < P; ++k) f[k] = __builtin_bit_cast(bf16x8, w[k]);
  }
}

// The same of binary32 with each piece what is left rounded to bfloat16, which makes the later ones
// smaller: at most 2^-8 and 2^-17 of v's power of two.  For products that leave pairs of pieces out.  A
// value that would round past bfloat16's largest number is cut off instead; an infinity's later pieces
// are 0.
__device__ inline void mx_round3(float v, __bf16 p[3]) {
  p[0] = (__bf16)v;
  const uint32_t u = __builtin_bit_cast(uint32_t, v), a = u & 0x7fffffffu;
  if (a >= 0x7f7f8000u && a < 0x7f800000u) p[0] = __builtin_bit_cast(__bf16, (uint16_t)(u >> 16));
  const float r = a == 0x7f800000u ? 0.0f : v - (float)p[0];
  p[1] = (__bf16)r;
  p[2] = (__bf16)(r - (float)p[1]);
}

// What lanes of a wavefront wrote to LDS is there for its other lanes.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace mcf
