// wave.hpp -- sums and maxima over the 64 lanes of a wavefront, in registers.
//
// Steps inside a row of 16 lanes are DPP moves, the last two exchange rows (v_permlane16_swap and
// v_permlane32_swap of a register with itself give both sides of a pair to all lanes).  Both lanes of a
// pair combine the same two values with an operation that commutes, so all lanes end with the same bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mcf {

template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ inline float dpp(float v) {
  return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v)));
}
template <int CTRL>
__device__ inline uint64_t dpp(uint64_t v) {
  return (uint64_t)dpp<CTRL>((uint32_t)(v >> 32)) << 32 | dpp<CTRL>((uint32_t)v);
}
template <int CTRL>
__device__ inline double dpp(double v) {
  return __builtin_bit_cast(double, dpp<CTRL>(__builtin_bit_cast(uint64_t, v)));
}

// v of the lower and the upper row (ROW 16) or half (ROW 32) of a pair, in both.
template <typename T>
struct Pair {
  T lo, hi;
};
template <int ROW>
__device__ inline Pair<uint32_t> swap_rows(uint32_t v) {
  if constexpr (ROW == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {r[0], r[1]};
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {r[0], r[1]};
  }
}
template <int ROW>
__device__ inline Pair<float> swap_rows(float v) {
  const Pair<uint32_t> r = swap_rows<ROW>(__builtin_bit_cast(uint32_t, v));
  return {__builtin_bit_cast(float, r.lo), __builtin_bit_cast(float, r.hi)};
}
template <int ROW>
__device__ inline Pair<uint64_t> swap_rows(uint64_t v) {
  const Pair<uint32_t> h = swap_rows<ROW>((uint32_t)(v >> 32)), l = swap_rows<ROW>((uint32_t)v);
  return {(uint64_t)h.lo << 32 | l.lo, (uint64_t)h.hi << 32 | l.hi};
}
template <int ROW>
__device__ inline Pair<double> swap_rows(double v) {
  const Pair<uint64_t> r = swap_rows<ROW>(__builtin_bit_cast(uint64_t, v));
  return {__builtin_bit_cast(double, r.lo), __builtin_bit_cast(double, r.hi)};
}

// Over N neighbouring lanes, a power of two up to 64.
template <int N, typename T, typename Op>
__device__ inline T lanes_join(T v, Op op) {
  if constexpr (N > 1) v = op(v, dpp<0xb1>(v));    // lane ^ 1
  if constexpr (N > 2) v = op(v, dpp<0x4e>(v));    // lane ^ 2
  if constexpr (N > 4) v = op(v, dpp<0x141>(v));   // 7 - lane of 8: the other quad
  if constexpr (N > 8) v = op(v, dpp<0x140>(v));   // 15 - lane of 16: the other eight
  if constexpr (N > 16) {
    const Pair<T> r = swap_rows<16>(v);
    v = op(r.lo, r.hi);
  }
  if constexpr (N > 32) {
    const Pair<T> r = swap_rows<32>(v);
    v = op(r.lo, r.hi);
  }
  return v;
}
template <int N = 64, typename T>
__device__ inline T lanes_sum(T v) {
  return lanes_join<N>(v, [](T a, T b) { return a + b; });
}
template <int N = 64>
__device__ inline float lanes_max(float v) {
  return lanes_join<N>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int N = 64>
__device__ inline double lanes_max(double v) {
  return lanes_join<N>(v, [](double a, double b) { return fmax(a, b); });
}
template <int N = 64>
__device__ inline uint32_t lanes_max(uint32_t v) {
  return lanes_join<N>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int N = 64>
__device__ inline uint64_t lanes_max(uint64_t v) {
  return lanes_join<N>(v, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}

}  // namespace mcf
