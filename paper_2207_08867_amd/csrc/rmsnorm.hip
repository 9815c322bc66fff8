// rmsnorm.hip -- root-mean-square norm of a residual stream, with the addition of a layer's output to
// the stream, into a plain tensor or an 8-bit one; its gradients; 8-bit quantisation and reading back.
//
// The stream h is plain or an MC value.  s = the planes' sum, the last one first, plus x, in binary64; the
// new stream is s split by successive rounding (through binary32) into nc planes, v their sum.  With
//   r = 1 / sqrt(sum v^2 / n + eps)
// the plain output is y = v w r.  The 8-bit one is, with p = v w and m = max |p| over the row,
//   code = rint(127 p / m),  scale = r m / 127:
// r cancels out of the codes, which so are a fixed function of the input.  Quantisation is the same with
// p = v, r = 1.  Everything between loads and roundings is binary64: sums of squares of bfloat16 and
// binary32 numbers pass binary32's range.
//
// Gradients, given dy and the gradient g that reaches the new stream from later layers:
//   dh = g + r (w dy - v r^2 sum(v w dy) / n),   dw = sum over rows of dy v r.
// r is computed again: v is read in any case.
#include <math.h>

#include "int8.hpp"
#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace mcf {
namespace {

struct NormArgs {
  const void *h, *x, *w;  // [nc][rows][n]; [rows][n] or null; [n] or null
  void *h_out, *y;        // [nc][rows][n] with x; [rows][n] of the plain output
  uint64_t *codes;        // [rows][pitch / 8] of the 8-bit one
  float *scales;          // [rows]
  int64_t rows, n, plane, pitch;
  int64_t first;          // the launch's first row
  double eps;
  int nc;
};

// Sum and maximum over the NT threads of a row, in a fixed order; every thread gets both.
struct SumMax {
  double sum, max;
};
template <int NT>
__device__ inline SumMax row_join(SumMax v, SumMax *lds) {
#pragma unroll
  for (int d = 1; d < (NT < 64 ? NT : 64); d <<= 1) {
    v.sum += __shfl_xor(v.sum, d);
    v.max = fmax(v.max, __shfl_xor(v.max, d));
  }
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
      v.sum += lds[w].sum;
      v.max = fmax(v.max, lds[w].max);
    }
  }
  return v;
}

// Eight elements from column col as binary64; zeros past the row.
template <typename T>
__device__ inline void wide8(const T *p, int64_t left, double v[8]) {
  const Raw8<T> r = load8_tail(p, left);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (double)(float)r.v[i];
}

// The planes' sum, the last one first.
template <typename T>
__device__ inline void planes8(const T *p, int64_t plane, int nc, int64_t left, double v[8]) {
  wide8(p + (nc - 1) * plane, left, v);
  for (int c = nc - 2; c >= 0; --c) {
    double u[8];
    wide8(p + c * plane, left, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += u[i];
  }
}

// v, eight values of the stream from column col of a row; with x the new stream is written.
template <typename T, bool ONE>
__device__ inline void stream8(const NormArgs &a, int64_t at, int64_t left, double v[8]) {
  const int nc = ONE ? 1 : a.nc;
  planes8(reinterpret_cast<const T *>(a.h) + at, a.plane, nc, left, v);
  if (!a.x) return;
  double u[8];
  wide8(reinterpret_cast<const T *>(a.x) + at, left, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += u[i];
  T *out = reinterpret_cast<T *>(a.h_out) + at;
  double total[8];
  Raw8<T> part[ONE ? 1 : 4];
#pragma unroll
  for (int c = 0; c < (ONE ? 1 : 4); ++c) {
    if (c >= nc) break;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T q = (T)(float)v[i];
      part[c].v[i] = q;
      // nothing is left of a value past the format's range
      v[i] = fabsf((float)q) == INFINITY ? 0.0 : v[i] - (double)(float)q;
    }
    store8_tail(out + c * a.plane, part[c], left);
  }
#pragma unroll
  for (int c = (ONE ? 1 : 4) - 1; c >= 0; --c) {
    if (c >= nc) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) total[i] = c == nc - 1 ? (double)(float)part[c].v[i] : total[i] + (double)(float)part[c].v[i];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = total[i];
}

// p = v w.
template <typename T>
__device__ inline void weigh8(const NormArgs &a, int64_t col, int64_t left, double v[8]) {
  if (!a.w) return;
  double u[8];
  wide8(reinterpret_cast<const T *>(a.w) + col, left, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= u[i];
}

// A row's scale; codes are zero where it is not finite.
struct Scale {
  double m, inv;
  float scale;
};
__device__ inline Scale row_scale(double m, double r) {
  Scale s;
  s.scale = (float)(m * r / 127.0);
  const bool fine = isfinite(s.scale);
  if (!fine) s.scale = NAN;
  s.m = m;
  s.inv = fine && m > 0.0 ? 1.0 / m : 0.0;
  return s;
}
__device__ inline uint64_t codes8(const double p[8], const Scale &s) {
  uint32_t lo = 0, hi = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo |= (uint32_t)((s.inv != 0.0 ? int8_code(p[i], s.m, s.inv) : 0) & 255) << (8 * i);
    hi |= (uint32_t)((s.inv != 0.0 ? int8_code(p[i + 4], s.m, s.inv) : 0) & 255) << (8 * i);
  }
  return (uint64_t)hi << 32 | lo;
}

// NT threads a row, CH pieces of 8 elements a thread, which stay in registers between the sums and the
// output; CH = 0: any length, read again.  The row's threads are one wavefront's lanes or a whole
// workgroup.  NORM false: quantisation alone.
template <typename T, bool ONE, int NT, int CH, bool NORM, bool INT8>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_kernel(NormArgs a) {
  constexpr int BLOCK = NT < 256 ? 256 : NT, HOLD = CH > 0 ? CH : 1;
  __shared__ SumMax lds[BLOCK / 64];
  const int64_t row = a.first + (int64_t)blockIdx.x * (BLOCK / NT) + threadIdx.x / NT;
  if (NT <= 64 && row >= a.rows) return;
  const int t = threadIdx.x % NT;
  const int64_t at = row * a.n, width = INT8 ? a.pitch : a.n;
  double v[HOLD][8];
  SumMax s = {0.0, 0.0};
  bool nan = false;
  // a piece's part in the sums; INT8: it becomes p
  const auto count = [&](double *p, int64_t col) {
    if (NORM)
#pragma unroll
      for (int i = 0; i < 8; ++i) s.sum += p[i] * p[i];
    if (NORM) weigh8<T>(a, col, a.n - col, p);
    if (INT8)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s.max = fmax(s.max, fabs(p[i]));
        nan = nan || p[i] != p[i];
      }
  };
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = (int64_t)(c * NT + t) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = 0.0;
      if (col < a.n) {
        stream8<T, ONE>(a, at + col, a.n - col, v[c]);
        count(v[c], col);
      }
    }
  } else {
    for (int64_t col = t * 8; col < a.n; col += NT * 8) {
      stream8<T, ONE>(a, at + col, a.n - col, v[0]);
      count(v[0], col);
    }
  }
  if (INT8 && nan) s.max = INFINITY;
  s = row_join<NT>(s, lds);
  const double r = NORM ? 1.0 / sqrt(s.sum / (double)a.n + a.eps) : 1.0;
  Scale sc;
  if constexpr (INT8) {
    sc = row_scale(s.max, r);
    if (t == 0) a.scales[row] = sc.scale;
  }
  const auto out = [&](const double *p, int64_t col) {
    if constexpr (INT8) {
      a.codes[(row * a.pitch + col) >> 3] = codes8(p, sc);
    } else {
      Raw8<T> o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)(p[i] * r);
      store8_tail(reinterpret_cast<T *>(a.y) + at + col, o, a.n - col);
    }
  };
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = (int64_t)(c * NT + t) * 8;
      if (col < width) out(v[c], col);
    }
  } else {
    // the thread's own columns again: of the new stream, which it wrote, where there is one
    const T *h = reinterpret_cast<const T *>(a.x ? a.h_out : a.h) + at;
    for (int64_t col = t * 8; col < width; col += NT * 8) {
      planes8(h + col, a.plane, ONE ? 1 : a.nc, a.n - col, v[0]);
      if (NORM && col < a.n) weigh8<T>(a, col, a.n - col, v[0]);
      out(v[0], col);
    }
  }
}

template <typename T, bool ONE, bool NORM, bool INT8>
hipError_t run_norm(NormArgs a, hipStream_t stream) {
  const auto go = [&](auto kernel, int nt) {
    const int per = nt < 256 ? 256 / nt : 1, block = nt < 256 ? 256 : nt;
    for (a.first = 0; a.first < a.rows; a.first += LAUNCH_MAX * per) {
      const int64_t left = a.rows - a.first, groups = (left + per - 1) / per;
      kernel<<<(unsigned)(groups < LAUNCH_MAX ? groups : LAUNCH_MAX), block, 0, stream>>>(a);
    }
    return hipGetLastError();
  };
  const int64_t width = INT8 ? a.pitch : a.n;
  if (width <= 128) return go(norm_kernel<T, ONE, 16, 1, NORM, INT8>, 16);
  if (width <= 512) return go(norm_kernel<T, ONE, 64, 1, NORM, INT8>, 64);
  if (width <= 2048) return go(norm_kernel<T, ONE, 256, 1, NORM, INT8>, 256);
  if (width <= 4096) return go(norm_kernel<T, ONE, 512, 1, NORM, INT8>, 512);
  if (width <= 8192) return go(norm_kernel<T, ONE, 1024, 1, NORM, INT8>, 1024);
  if (width <= 16384) return go(norm_kernel<T, ONE, 1024, 2, NORM, INT8>, 1024);
  return go(norm_kernel<T, ONE, 1024, 0, NORM, INT8>, 1024);
}

// code scale, eight elements a thread.
template <typename T>
__global__ __launch_bounds__(256) void int8_read_kernel(const uint64_t *codes, const float *scales, T *out, int64_t rows,
                                                        int64_t n, int64_t across, int64_t first) {
  const int64_t id = (first + blockIdx.x) * 256 + threadIdx.x;
  if (id >= rows * across) return;
  const int64_t row = id <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)across) : id / across;
  const int64_t col = (id - row * across) * 8;
  const uint64_t w = codes[row * (int8_pitch(n) >> 3) + (col >> 3)];
  const float s = scales[row];
  Raw8<T> o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o.v[i] = (T)((float)(int8_t)(w >> (8 * i)) * s);
  store8_tail(out + row * n + col, o, n - col);
}

template <typename T>
hipError_t read_back(int64_t rows, int64_t n, const void *codes, const void *scales, void *out, hipStream_t stream) {
  const int64_t across = (n + 7) / 8, groups = (rows * across + 255) / 256;
  for (int64_t first = 0; first < groups; first += LAUNCH_MAX)
    int8_read_kernel<T><<<(unsigned)(groups - first < LAUNCH_MAX ? groups - first : LAUNCH_MAX), 256, 0, stream>>>(
        (const uint64_t *)codes, (const float *)scales, (T *)out, rows, n, across, first);
  return hipGetLastError();
}

// --- gradients -------------------------------------------------------------------------

struct NormBwdArgs {
  const void *h, *w, *dy, *g;  // [nc][rows][n]; [n] or null; [rows][n]; [rows][n] or null
  void *dh, *dw;               // [rows][n] or null; [n] or null
  float *partial;              // [groups][n], with dw
  int64_t rows, n, plane;
  double eps;
  int nc, groups;
};

template <int NT>
__device__ inline f64x2 row_sum2(f64x2 v, f64x2 *lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    v[0] += __shfl_xor(v[0], d);
    v[1] += __shfl_xor(v[1], d);
  }
  if constexpr (NT > 64) {
    __syncthreads();  // the row before has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v += lds[w];
  }
  return v;
}

// A workgroup takes rows blockIdx.x, blockIdx.x + groups, ...; a thread the same columns of each, of which
// it keeps dw's sums.
template <typename T, bool ONE, int NT, int CH>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(NormBwdArgs a) {
  __shared__ f64x2 lds[NT / 64];
  const int nc = ONE ? 1 : a.nc;
  double dw[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.0;
  for (int64_t row = blockIdx.x; row < a.rows; row += a.groups) {
    const int64_t at = row * a.n;
    double v[CH][8], d[CH][8], w[CH][8];
    f64x2 s = {0.0, 0.0};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = (c * NT + (int)threadIdx.x) * 8, left = a.n - col;
      if (left <= 0) break;
      planes8(reinterpret_cast<const T *>(a.h) + at + col, a.plane, nc, left, v[c]);
      wide8(reinterpret_cast<const T *>(a.dy) + at + col, left, d[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[c][i] = 1.0;
      if (a.w) wide8(reinterpret_cast<const T *>(a.w) + col, left, w[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] += v[c][i] * v[c][i];
        s[1] += v[c][i] * (w[c][i] * d[c][i]);
      }
    }
    s = row_sum2<NT>(s, lds);
    const double r = 1.0 / sqrt(s[0] / (double)a.n + a.eps), k = s[1] / (double)a.n * r * r;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = (c * NT + (int)threadIdx.x) * 8, left = a.n - col;
      if (left <= 0) break;
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[c][i] += d[c][i] * (v[c][i] * r);
      if (!a.dh) continue;
      double g[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
      if (a.g) wide8(reinterpret_cast<const T *>(a.g) + at + col, left, g);
      Raw8<T> o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)(g[i] + r * (w[c][i] * d[c][i] - v[c][i] * k));
      store8_tail(reinterpret_cast<T *>(a.dh) + at + col, o, left);
    }
  }
  if (!a.dw) return;
  float *p = a.partial + (int64_t)blockIdx.x * a.n;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t col = (c * NT + (int)threadIdx.x) * 8 + i;
      if (col < a.n) p[col] = (float)dw[c][i];
    }
}

// Rows of any length, read twice; dw by the kernel below.  r and k of each row go to partial.
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(NormBwdArgs a) {
  __shared__ f64x2 lds[16];
  for (int64_t row = blockIdx.x; row < a.rows; row += a.groups) {
    const int64_t at = row * a.n;
    f64x2 s = {0.0, 0.0};
    const auto piece = [&](int64_t col, double v[8], double d[8], double p[8]) {
      planes8(reinterpret_cast<const T *>(a.h) + at + col, a.plane, a.nc, a.n - col, v);
      wide8(reinterpret_cast<const T *>(a.dy) + at + col, a.n - col, d);
      double w[8] = {1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0};
      if (a.w) wide8(reinterpret_cast<const T *>(a.w) + col, a.n - col, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = w[i] * d[i];
    };
    double v[8], d[8], p[8];
    for (int64_t col = threadIdx.x * 8; col < a.n; col += 8192) {
      piece(col, v, d, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] += v[i] * v[i];
        s[1] += v[i] * p[i];
      }
    }
    s = row_sum2<1024>(s, lds);
    const double r = 1.0 / sqrt(s[0] / (double)a.n + a.eps), k = s[1] / (double)a.n * r * r;
    if (a.dw && threadIdx.x == 0) reinterpret_cast<double *>(a.partial)[row] = r;
    if (!a.dh) continue;
    for (int64_t col = threadIdx.x * 8; col < a.n; col += 8192) {
      piece(col, v, d, p);
      double g[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
      if (a.g) wide8(reinterpret_cast<const T *>(a.g) + at + col, a.n - col, g);
      Raw8<T> o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)(g[i] + r * (p[i] - v[i] * k));
      store8_tail(reinterpret_cast<T *>(a.dh) + at + col, o, a.n - col);
    }
  }
}

// dw of long rows: a thread 8 columns of every row, in order.
template <typename T>
__global__ __launch_bounds__(64) void norm_bwd_long_dw_kernel(NormBwdArgs a) {
  const int64_t col = ((int64_t)blockIdx.x * 64 + threadIdx.x) * 8;
  if (col >= a.n) return;
  double sum[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
#pragma unroll 2
  for (int64_t row = 0; row < a.rows; ++row) {
    double v[8], d[8];
    planes8(reinterpret_cast<const T *>(a.h) + row * a.n + col, a.plane, a.nc, a.n - col, v);
    wide8(reinterpret_cast<const T *>(a.dy) + row * a.n + col, a.n - col, d);
    const double r = reinterpret_cast<const double *>(a.partial)[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += d[i] * (v[i] * r);
  }
  Raw8<T> o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)sum[i];
  store8_tail(reinterpret_cast<T *>(a.dw) + col, o, a.n - col);
}

// The workgroups' sums: 64 columns by 16 parts of the workgroups, each in order, then the parts.
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_sum_kernel(NormBwdArgs a) {
  __shared__ double part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  const int from = a.groups * wave / 16, to = a.groups * (wave + 1) / 16;
  double s = 0.0;
  if (col < a.n)
#pragma unroll 8
    for (int g = from; g < to; ++g) s += (double)a.partial[(int64_t)g * a.n + col];
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || col >= a.n) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) s += part[w][lane];
  reinterpret_cast<T *>(a.dw)[col] = (T)(float)s;
}

constexpr int64_t BWD_LONG = 16384;  // the longest row that stays in registers

int bwd_groups(int64_t rows) { return (int)(rows < 512 ? rows : 512); }

template <typename T>
hipError_t run_bwd(const NormBwdArgs &a, hipStream_t stream) {
  const unsigned grid = (unsigned)a.groups;
  if (a.n > BWD_LONG) {
    if (grid) norm_bwd_long_kernel<T><<<grid, 1024, 0, stream>>>(a);
    if (a.dw) norm_bwd_long_dw_kernel<T><<<(unsigned)((a.n + 511) / 512), 64, 0, stream>>>(a);
    return hipGetLastError();
  }
  const auto go = [&](auto one) {
    constexpr bool ONE = decltype(one)::value;
    if (grid == 0) return;  // dw is zero
    if (a.n <= 512)
      norm_bwd_kernel<T, ONE, 64, 1><<<grid, 64, 0, stream>>>(a);
    else if (a.n <= 2048)
      norm_bwd_kernel<T, ONE, 256, 1><<<grid, 256, 0, stream>>>(a);
    else if (a.n <= 4096)
      norm_bwd_kernel<T, ONE, 512, 1><<<grid, 512, 0, stream>>>(a);
    else if (a.n <= 8192)
      norm_bwd_kernel<T, ONE, 1024, 1><<<grid, 1024, 0, stream>>>(a);
    else
      norm_bwd_kernel<T, ONE, 1024, 2><<<grid, 1024, 0, stream>>>(a);
  };
  if (a.nc == 1)
    go(Flag<true>());
  else
    go(Flag<false>());
  if (a.dw) norm_bwd_sum_kernel<T><<<(unsigned)((a.n + 63) / 64), 1024, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w,
                          double eps, void *h_out, void *y, void *codes, void *scales, bool norm, hipStream_t stream) {
  NormArgs a = {};
  a.h = h;
  a.x = x;
  a.w = w;
  a.h_out = h_out;
  a.y = y;
  a.codes = (uint64_t *)codes;
  a.scales = (float *)scales;
  a.rows = rows;
  a.n = n;
  a.plane = rows * n;
  a.pitch = int8_pitch(n);
  a.eps = eps;
  a.nc = nc;
  const auto go = [&](auto zero) {
    using T = decltype(zero);
    if (nc == 1) {
      if (!norm) return run_norm<T, true, false, true>(a, stream);
      return codes ? run_norm<T, true, true, true>(a, stream) : run_norm<T, true, true, false>(a, stream);
    }
    if (!norm) return run_norm<T, false, false, true>(a, stream);
    return codes ? run_norm<T, false, true, true>(a, stream) : run_norm<T, false, true, false>(a, stream);
  };
  if (dtype == LM_F16) return go((_Float16)0.0f);
  if (dtype == LM_BF16) return go((__bf16)0.0f);
  return go(0.0f);
}

hipError_t launch_int8_dequantize(int dtype, int64_t rows, int64_t n, const void *codes, const void *scales, void *out,
                                  hipStream_t stream) {
  if (dtype == LM_F16) return read_back<_Float16>(rows, n, codes, scales, out, stream);
  if (dtype == LM_BF16) return read_back<__bf16>(rows, n, codes, scales, out, stream);
  return read_back<float>(rows, n, codes, scales, out, stream);
}

int64_t rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t n) {
  return n > BWD_LONG ? rows * 8 : bwd_groups(rows) * n * 4;
}

hipError_t launch_rmsnorm_bwd(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *w, const void *dy,
                              const void *g, double eps, void *dh, void *dw, void *ws, hipStream_t stream) {
  NormBwdArgs a = {};
  a.h = h;
  a.w = w;
  a.dy = dy;
  a.g = g;
  a.dh = dh;
  a.dw = dw;
  a.partial = (float *)ws;
  a.rows = rows;
  a.n = n;
  a.plane = rows * n;
  a.eps = eps;
  a.nc = nc;
  a.groups = bwd_groups(rows);
  if (dtype == LM_F16) return run_bwd<_Float16>(a, stream);
  if (dtype == LM_BF16) return run_bwd<__bf16>(a, stream);
  return run_bwd<float>(a, stream);
}

}  // namespace mcf
