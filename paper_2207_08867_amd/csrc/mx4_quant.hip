// mx4_quant.hip -- quantisation into MXFP4 components and reading back.
//
// Quantisation of a block v_0 .. v_31: X = max(floor(log2 max|v_i|) - 2, -127), the element i
// is v_i 2^-X rounded to nearest E2M1, ties to even, at most 6; what is left, v_i minus the
// number the element stands for, is the next component's input.  The remainder is exact in
// binary32: it is a multiple of v_i's last place and no larger than v_i, or within 2^(X-2) of
// zero.  Both directions stream: 2 to 4 bytes read and 17/32 of a byte written per element and
// component (or back), so HBM bounds them (8192 x 8192 bfloat16: 28 us, 6.1 TB/s, and back 35 us, 4.9
// TB/s; binary32 45 us, 6.7 TB/s, and back 86 us, 3.6 TB/s: its 32 bytes a lane go out in two halves).  A lane takes 8 elements and four lanes a block; the block's maximum is two DPP steps
// inside a quad.
#include <type_traits>

#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace mcf {
namespace {

template <int CTRL>
__device__ inline uint32_t quad_max(uint32_t m) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true);
  return o > m ? o : m;
}

// The largest value of a quad of lanes.
__device__ inline uint32_t block_max(uint32_t m) { return quad_max<0x4e>(quad_max<0xb1>(m)); }

struct QuantArgs {
  const void *x;
  uint8_t *codes, *scales;
  int64_t rows, n, groups, across;  // workgroups side by side along a row
  int64_t first;                    // the launch's first workgroup
  int nc, shift;
};

__device__ inline uint32_t pack8(const float v[8], float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

// d as binary32 with its inexactness kept in the last bit (rounding to odd), so that a later
// rounding to E2M1 equals one rounding of d.
__device__ inline float round_odd(double d) {
  const float f = (float)d;
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  const double back = (double)f;
  if (back == d || !(u & 0x7f800000u)) return f;  // exact, or far below every rounding boundary
  const uint32_t cut = (fabs(back) > fabs(d) ? u - 1 : u) | 1u;
  return __builtin_bit_cast(float, cut);
}

// A workgroup covers 16 groups of 16 lanes: 1 << tile_shift rows of 16 >> tile_shift groups each.  Short
// rows take 16 rows of one group, so that no lane lies past a row's end and the scales of 16
// neighbouring rows fall into one line; long rows 4 x 4, which reads longer runs.  Measured (us,
// quantising and reading back), 100000 x 100 binary16: 7.3 and 10.3 as 16 rows, 22 and 18 as 4, 38
// and 35 as one; 4099 x 4097 binary16 in two planes and components: 21.1 and 15.6, 18.7 and 15.4, 18.8
// and 15.4; 8192 x 8192 bfloat16: 27 to 29 (6.2 TB/s) and 35 to 37 (4.6 TB/s and more) in all of them.
int tile_shift(int64_t groups) { return groups >= 16 ? 2 : 4; }

__device__ inline int64_t divide(int64_t a, int64_t b) {
  return (a | b) <= 0xffffffffll ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

struct BlockAt {
  int64_t row, group;
  int in;  // the lane's piece of the group, 0 .. 15
};

__device__ inline void put(const QuantArgs &a, const BlockAt &b, int c, uint32_t word, uint32_t byte) {
  uint8_t *codes = a.codes + ((int64_t)c * a.rows + b.row) * (a.groups * 64) + b.group * 64 + b.in * 4;
  *reinterpret_cast<uint32_t *>(codes) = word;
  if ((b.in & 3) == 0) a.scales[(((int64_t)c * a.groups + b.group) * a.rows + b.row) * 4 + (b.in >> 2)] = (uint8_t)byte;
}

// Components of binary32 values.  A block with an infinity or NaN gets the scale 255 (NaN) and
// zero codes in every component.
__device__ inline void quantize32(const QuantArgs &a, const BlockAt &b, float v[8]) {
  for (int c = 0; c < a.nc; ++c) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
      m = u > m ? u : m;
    }
    const uint32_t e = block_max(m) >> 23;
    const uint32_t byte = e == 255 ? 255 : (e > 2 ? e - 2 : 0);
    const float scale = mx_scale(byte == 255 ? 127 : byte);
    const uint32_t word = byte == 255 ? 0 : pack8(v, scale);
    put(a, b, c, word, byte);
    if (c + 1 < a.nc && byte != 255) {
      float q[8];
      mx_f32(word, scale, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= q[i];
    }
  }
}

// The same from binary64 values, for sums of planes that binary32 does not hold.
__device__ inline void quantize64(const QuantArgs &a, const BlockAt &b, double v[8]) {
  for (int c = 0; c < a.nc; ++c) {
    uint32_t m = 0;  // the largest biased binary64 exponent
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t e = (uint32_t)(__builtin_bit_cast(uint64_t, v[i]) >> 52) & 0x7ffu;
      m = e > m ? e : m;
    }
    m = block_max(m);
    const int X = (int)m - 1023 - 2;
    const uint32_t byte = m == 0x7ff ? 255 : (X < -127 ? 0 : (X > 127 ? 254 : X + 127));
    const int E = (int)byte - 127;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = round_odd(ldexp(v[i], -E));
    const uint32_t word = byte == 255 ? 0 : pack8(y, 1.0f);
    put(a, b, c, word, byte);
    if (c + 1 < a.nc && byte != 255) {
      float q[8];
      mx_f32(word, 1.0f, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= ldexp((double)q[i], E);
    }
  }
}

template <typename T, int NIN>
__global__ __launch_bounds__(256) void mx_quant_kernel(QuantArgs a) {
  BlockAt b;
  const int64_t id = a.first + blockIdx.x, tile = divide(id, a.across);
  const int g = threadIdx.x >> 4;
  b.in = (int)(threadIdx.x & 15);
  b.row = (tile << a.shift) + (g >> (4 - a.shift));
  b.group = ((id - tile * a.across) << (4 - a.shift)) + (g & ((16 >> a.shift) - 1));
  if (b.row >= a.rows || b.group >= a.groups) return;  // whole quads leave together
  const int64_t col = b.group * MX_GROUP + b.in * 8;
  const T *x = reinterpret_cast<const T *>(a.x) + b.row * a.n + col;
  float v[8];
  if constexpr (NIN == 1) {
    const Raw8<T> r = load8_tail(x, a.n - col);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)r.v[i];
    quantize32(a, b, v);
  } else {
    // the planes' sum, the last plane first, with the error of every addition (Two-Sum): where
    // all errors are zero the binary32 sum is exact
    Raw8<T> r[NIN];
#pragma unroll
    for (int p = 0; p < NIN; ++p) r[p] = load8_tail(x + p * a.rows * a.n, a.n - col);
    bool exact = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s = (float)r[NIN - 1].v[i];
#pragma unroll
      for (int p = NIN - 2; p >= 0; --p) {
        const float y = (float)r[p].v[i], t = y + s, z = t - y;
        exact = exact && ((y - (t - z)) + (s - z)) == 0.0f;
        s = t;
      }
      v[i] = s;
    }
    if (__all(exact)) {
      quantize32(a, b, v);
    } else {
      // binary16 and bfloat16 planes of one value sum exactly in 53 bits; binary32 planes that
      // span more round there
      double d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = (double)(float)r[NIN - 1].v[i];
#pragma unroll
        for (int p = NIN - 2; p >= 0; --p) d[i] += (double)(float)r[p].v[i];
      }
      quantize64(a, b, d);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void mx_dequant_kernel(const uint8_t *codes, const uint8_t *scales, T *out, int nc,
                                                         int64_t rows, int64_t n, int64_t groups, int64_t across,
                                                         int shift, int64_t first) {
  const int64_t id = first + blockIdx.x, tile = divide(id, across);
  const int g = threadIdx.x >> 4, in = (int)(threadIdx.x & 15);
  const int64_t row = (tile << shift) + (g >> (4 - shift));
  const int64_t group = ((id - tile * across) << (4 - shift)) + (g & ((16 >> shift) - 1));
  const int64_t col = group * MX_GROUP + in * 8;
  if (row >= rows || col >= n) return;
  float v[8] = {};
  for (int c = nc - 1; c >= 0; --c) {  // the smallest component first
    const int64_t plane = (int64_t)c * rows;
    const uint32_t word = *reinterpret_cast<const uint32_t *>(codes + (plane + row) * (groups * 64) + group * 64 + in * 4);
    const uint32_t byte = scales[((int64_t)c * groups * rows + group * rows + row) * 4 + (in >> 2)];
    float q[8];
    mx_f32(word, mx_scale(byte), q);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c == nc - 1 ? q[i] : v[i] + q[i];
  }
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = (T)v[i];
  store8_tail(out + row * n + col, r, n - col);
}

// Workgroups along a row, and in all.
int64_t tiles_across(int64_t groups) { return (groups + (16 >> tile_shift(groups)) - 1) >> (4 - tile_shift(groups)); }
int64_t tiles(int64_t rows, int64_t groups) {
  const int s = tile_shift(groups);
  return ((rows + (1 << s) - 1) >> s) * tiles_across(groups);
}
// launch(first, workgroups) over all of them.
template <typename F>
hipError_t in_launches(int64_t all, F launch) {
  for (int64_t first = 0; first < all; first += LAUNCH_MAX)
    launch(first, dim3((unsigned)(all - first < LAUNCH_MAX ? all - first : LAUNCH_MAX)));
  return hipGetLastError();
}

template <typename T>
hipError_t quantize(int nc_in, QuantArgs a, hipStream_t stream) {
  return in_launches(tiles(a.rows, a.groups), [&](int64_t first, dim3 grid) {
    a.first = first;
    switch (nc_in) {
      case 1: mx_quant_kernel<T, 1><<<grid, 256, 0, stream>>>(a); break;
      case 2: mx_quant_kernel<T, 2><<<grid, 256, 0, stream>>>(a); break;
      case 3: mx_quant_kernel<T, 3><<<grid, 256, 0, stream>>>(a); break;
      default: mx_quant_kernel<T, 4><<<grid, 256, 0, stream>>>(a); break;
    }
  });
}

}  // namespace

hipError_t launch_mx4_quantize(int dtype, int nc_in, int nc, int64_t rows, int64_t n, const void *x, void *codes,
                               void *scales, hipStream_t stream) {
  QuantArgs a = {};
  a.x = x;
  a.codes = (uint8_t *)codes;
  a.scales = (uint8_t *)scales;
  a.rows = rows;
  a.n = n;
  a.groups = mx_groups(n);
  a.across = tiles_across(a.groups);
  a.shift = tile_shift(a.groups);
  a.nc = nc;
  if (dtype == LM_F16) return quantize<_Float16>(nc_in, a, stream);
  if (dtype == LM_BF16) return quantize<__bf16>(nc_in, a, stream);
  return quantize<float>(nc_in, a, stream);
}

hipError_t launch_mx4_dequantize(int dtype, int nc, int64_t rows, int64_t n, const void *codes, const void *scales,
                                 void *out, hipStream_t stream) {
  const int64_t groups = mx_groups(n);
  const int64_t across = tiles_across(groups);
  const int shift = tile_shift(groups);
  const uint8_t *c = (const uint8_t *)codes, *s = (const uint8_t *)scales;
  const auto go = [&](auto *o) {
    using T = std::remove_pointer_t<decltype(o)>;
    return in_launches(tiles(rows, groups), [&](int64_t first, dim3 grid) {
      mx_dequant_kernel<T><<<grid, 256, 0, stream>>>(c, s, o, nc, rows, n, groups, across, shift, first);
    });
  };
  if (dtype == LM_F16) return go((_Float16 *)out);
  if (dtype == LM_BF16) return go((__bf16 *)out);
  return go((float *)out);
}

}  // namespace mcf
