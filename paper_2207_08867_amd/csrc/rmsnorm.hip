// rmsnorm.hip -- root-mean-square norm of a residual stream, with the addition of a layer's output to
// the stream, into a plain tensor or an 8-bit one; its gradients; 8-bit quantisation and reading back.
//
// The stream h is plain or an MC value.  s = the planes' sum, the last one first, plus x, in binary64; the
// new stream is s split by successive rounding (through binary32) into nc planes, v their sum.  With
//   r = 1 / sqrt(sum v^2 / n + eps)
// the plain output is y = v w r.  The 8-bit one is, with p = v w and m = max |p| over the row,
//   code = rint(127 p / m),  scale = r m / 127:
// r cancels out of the codes, which so are a fixed function of the input.  Quantisation is the same with
// p = v, r = 1.  Everything between loads and roundings is binary64 (sums of squares of bfloat16 and
// binary32 numbers pass binary32's range) but where norm16_kernel says otherwise.
//
// Gradients, given dy and the gradient g that reaches the new stream from later layers:
//   dh = g + r (w dy - v r^2 sum(v w dy) / n),   dw = sum over rows of dy v r.
// r is computed again: v is read in any case.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "int8.hpp"
#include "mcf_internal.hpp"
#include "mx4.hpp"
#include "wave.hpp"

namespace mcf {
namespace {

struct NormArgs {
  const void *h, *x, *w;  // [nc][rows][n]; [rows][n] or null; [n] or null
  void *h_out, *y;        // [nc][rows][n] with x; [rows][n] of the plain output
  uint64_t *codes;        // [rows][pitch / 8] of the 8-bit one
  float *scales;          // [rows]
  int64_t rows, n, plane, pitch;
  int64_t first;          // the launch's first row
  double eps, inv_n;
  int nc;
};

// 1 / sqrt(x): the hardware's estimate and two Newton steps, each of which squares its error of 2^-26 or
// less; IEEE's results at zero and infinity.
__device__ inline double inverse_root(double x) {
  double y = __builtin_amdgcn_rsq(x);
  if (!(x > 0.0 && x < INFINITY)) return y;
  const double half = 0.5 * x;
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(y, fma(-half * y, y, 0.5), y);
  return y;
}

// Sum and maximum over the NT threads of a row, in a fixed order; every thread gets both.
template <typename M>
struct SumMax {
  double sum;
  M max;
};
template <int NT, typename M>
__device__ inline SumMax<M> row_join(SumMax<M> v, SumMax<M> *lds) {
  v.sum = lanes_sum<(NT < 64 ? NT : 64)>(v.sum);
  v.max = lanes_max<(NT < 64 ? NT : 64)>(v.max);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[threadIdx.x % (NT / 64)];
    v.sum = lanes_sum<NT / 64>(v.sum);
    v.max = lanes_max<NT / 64>(v.max);
  }
  return v;
}

// How a row's pieces of 8 elements end: n is a multiple of 8, at least 8, or less.
enum End { END_EVEN = 0, END_ODD = 1, END_SHORT = 2 };
inline End end_of(int64_t n) { return n % 8 == 0 ? END_EVEN : (n >= 8 ? END_ODD : END_SHORT); }

// Eight elements from column col of a row of n as binary64; zeros past its end.
template <End E, typename T>
__device__ inline void wide8(const T *row, int64_t col, int64_t n, double v[8]) {
  Raw8<T> r;
  if constexpr (E == END_SHORT)
    r = load8_tail(row + col, n - col);
  else
    r = load8_row<E == END_EVEN>(row, col, n, (T)0.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (double)(float)r.v[i];
}

// The planes' sum, the last one first.
template <End E, typename T>
__device__ inline void planes8(const T *row, int64_t plane, int nc, int64_t col, int64_t n, double v[8]) {
  wide8<E>(row + (nc - 1) * plane, col, n, v);
  for (int c = nc - 2; c >= 0; --c) {
    double u[8];
    wide8<E>(row + c * plane, col, n, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += u[i];
  }
}

// v, eight values of the stream from column col of a row; with x the new stream is written.
template <typename T, bool ONE, End E>
__device__ inline void stream8(const NormArgs &a, int64_t at, int64_t col, double v[8]) {
  const int nc = ONE ? 1 : a.nc;
  planes8<E>(reinterpret_cast<const T *>(a.h) + at, a.plane, nc, col, a.n, v);
  if (!a.x) return;
  double u[8];
  wide8<E>(reinterpret_cast<const T *>(a.x) + at, col, a.n, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += u[i];
  T *out = reinterpret_cast<T *>(a.h_out) + at + col;
  const int64_t left = E == END_EVEN ? 8 : a.n - col;
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
    for (int i = 0; i < 8; ++i) {
      const double q = (double)(float)part[c].v[i];
      total[i] = c == nc - 1 ? q : total[i] + q;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = total[i];
}

// p = v w.
template <End E, typename T>
__device__ inline void weigh8(const NormArgs &a, int64_t col, double v[8]) {
  if (!a.w) return;
  double u[8];
  wide8<E>(reinterpret_cast<const T *>(a.w), col, a.n, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= u[i];
}

// NT threads a row, CH pieces of 8 elements a thread, which stay in registers between the sums and the
// output; CH = 0: any length, read again.  The row's threads are one wavefront's lanes or a whole
// workgroup.  NORM false: quantisation alone.  HBM bounds binary32 rows (4096 x 4096, norm with x 50 us, 5.4 TB/s, into
// 8 bits 45 us, 4.9), binary64 arithmetic MC ones in part (two binary16 planes 46 and 49 us, 4.4 and 3.8 TB/s).
template <typename T, bool ONE, int NT, int CH, bool NORM, bool INT8, End E>
__global__ __launch_bounds__(NT <= 64 ? 256 : NT) void norm_kernel(NormArgs a) {
  constexpr int BLOCK = NT <= 64 ? 256 : NT, HOLD = CH > 0 ? CH : 1;
  __shared__ SumMax<double> lds[BLOCK / 64];
  const int64_t row = a.first + (int64_t)blockIdx.x * (BLOCK / NT) + threadIdx.x / NT;
  if (NT <= 64 && row >= a.rows) return;
  const int t = threadIdx.x % NT;
  const int64_t at = row * a.n, width = INT8 ? a.pitch : a.n;
  double v[HOLD][8];
  SumMax<double> s = {0.0, 0.0};
  bool nan = false;
  // a piece's part in the sums; INT8: it becomes p
  const auto count = [&](double *p, int64_t col) {
    if (NORM)
#pragma unroll
      for (int i = 0; i < 8; ++i) s.sum += p[i] * p[i];
    if (NORM) weigh8<E, T>(a, col, p);
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
        stream8<T, ONE, E>(a, at, col, v[c]);
        count(v[c], col);
      }
    }
  } else {
    for (int64_t col = t * 8; col < a.n; col += NT * 8) {
      stream8<T, ONE, E>(a, at, col, v[0]);
      count(v[0], col);
    }
  }
  if (INT8 && nan) s.max = INFINITY;
  s = row_join<NT>(s, lds);
  const double r = NORM ? inverse_root(s.sum * a.inv_n + a.eps) : 1.0;
  Int8Row sc;
  if constexpr (INT8) {
    sc = int8_row(s.max, r);
    if (t == 0) a.scales[row] = sc.scale;
  }
  const auto out = [&](const double *p, int64_t col) {
    if constexpr (INT8) {
      a.codes[(row * a.pitch + col) >> 3] = int8_codes8_any(p, sc);
    } else {
      Raw8<T> o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)(p[i] * r);
      store8_tail(reinterpret_cast<T *>(a.y) + at + col, o, E == END_EVEN ? 8 : a.n - col);
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
#pragma unroll
      for (int i = 0; i < 8; ++i) v[0][i] = 0.0;
      if (col < a.n) {
        planes8<E>(h, a.plane, ONE ? 1 : a.nc, col, a.n, v[0]);
        if (NORM) weigh8<E, T>(a, col, v[0]);
      }
      out(v[0], col);
    }
  }
}

// The same of plain 16-bit rows, with binary32 between the loads and the roundings where that is exact or enough: v
// and, in its range, p = v w are exact there, and their squares are summed in binary64.  Rows whose m lies near the
// ends of binary32's range, and outputs past it or whose r is far from one, take the binary64 forms; a p below binary32's
// normal numbers is off by 2^-150, which r <= 2^10 leaves below 2^-140.  All of a row's loads go out before
// the first is looked at, eight wavefronts a SIMD.  HBM bounds it: 8192 x 4096 bfloat16 with x 50 us, 5.4 TB/s, into 8
// bits 49 us, 4.8, quantisation alone 23 us, 4.3 (binary64 between loads and roundings: 4096 x 4096 into 8 bits 45 us,
// 29 so).
template <typename T, int NT, int CH, bool NORM, bool INT8, bool EVEN, int OCC>
__global__ __launch_bounds__(NT <= 64 ? 256 : NT, OCC) void norm16_kernel(NormArgs a) {
  constexpr int BLOCK = NT <= 64 ? 256 : NT;
  __shared__ SumMax<uint32_t> lds[BLOCK / 64];
  __shared__ SumMax<double> lds_wide[BLOCK / 64];
  const int64_t row = a.first + (int64_t)blockIdx.x * (BLOCK / NT) + threadIdx.x / NT;
  if (NT <= 64 && row >= a.rows) return;
  const int t = threadIdx.x % NT;
  const int64_t at = row * a.n;
  const int n = (int)a.n, width = INT8 ? (int)a.pitch : n;
  const T *h = reinterpret_cast<const T *>(a.h) + at, *x = reinterpret_cast<const T *>(a.x) + at;
  const T *w = reinterpret_cast<const T *>(a.w);
  const auto column = [&](int c) { return (c * NT + t) * 8; };
  Raw8<T> hr[CH], xr[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = column(c), left = n - col;
#pragma unroll
    for (int i = 0; i < 8; ++i) hr[c].v[i] = (T)0.0f;
    if (EVEN && left <= 0) continue;
    hr[c] = EVEN ? load8(h + col) : load8_clamped(h, col, n);
    if (a.x) xr[c] = EVEN ? load8(x + col) : load8_clamped(x, col, n);
  }
  if constexpr (!EVEN) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      load8_settle(hr[c], n - column(c), (T)0.0f);
      if (a.x) load8_settle(xr[c], n - column(c), (T)0.0f);
    }
  }
  // p of a piece; the weight is read again, from the first-level cache as a rule
  const auto weighed = [&](int c, float p[8]) {
    Raw8<T> u;
    const bool weight = NORM && w && column(c) < n;
    if (weight) u = load8_row<EVEN>(w, column(c), n, (T)0.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = weight ? (float)hr[c].v[i] * (float)u.v[i] : (float)hr[c].v[i];
  };
  SumMax<uint32_t> s = {0.0, 0};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = column(c), left = n - col;
    if (left <= 0) continue;
    if (a.x) {
#pragma unroll
      for (int i = 0; i < 8; ++i) hr[c].v[i] = (T)((float)hr[c].v[i] + (float)xr[c].v[i]);
      store8_tail(reinterpret_cast<T *>(a.h_out) + at + col, hr[c], EVEN ? 8 : left);
    }
    if (NORM)
#pragma unroll
      for (int i = 0; i < 8; ++i) s.sum = fma((double)(float)hr[c].v[i], (double)(float)hr[c].v[i], s.sum);
    if constexpr (INT8) {
      float p[8];
      weighed(c, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t u = magnitude(p[i]);
        s.max = u > s.max ? u : s.max;
      }
    }
  }
  s = row_join<NT>(s, lds);
  const double r = NORM ? inverse_root(s.sum * a.inv_n + a.eps) : 1.0;
  // p of an element in binary64, read again, one by one: rare, and so without registers of its own
  const T *again = a.x ? reinterpret_cast<const T *>(a.h_out) + at : h;
  const auto wide = [&](int col) {
    const double v = (double)(float)again[col];
    return NORM && w ? v * (double)(float)w[col] : v;
  };
  if constexpr (INT8) {
    // 2^-60 to 2^100; outside of it p may not be exact
    const bool fast = s.max >= 0x21800000u && s.max <= 0x71800000u;
    double m = (double)__builtin_bit_cast(float, s.max);
    if (!fast) {
      SumMax<double> d = {0.0, 0.0};
#pragma unroll 1
      for (int c = 0; c < CH; ++c)
#pragma unroll 1
        for (int col = column(c); col < column(c) + 8 && col < n; ++col) {
          const double v = wide(col);
          d.max = fmax(d.max, v == v ? fabs(v) : INFINITY);
        }
      m = row_join<NT>(d, lds_wide).max;
    }
    const Int8Row sc = int8_row(m, r);
    if (t == 0) a.scales[row] = sc.scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = column(c);
      if (col >= width) break;
      uint64_t codes;
      if (fast && sc.near) {
        float p[8];
        weighed(c, p);
        codes = int8_codes8(p, sc);
      } else {
        codes = 0;
#pragma unroll 1
        for (int i = 0; i < 8 && col + i < n && sc.inv != 0.0; ++i)
          codes |= (uint64_t)(int8_code(wide(col + i), sc.m, sc.inv) & 255) << (8 * i);
      }
      a.codes[(row * a.pitch + col) >> 3] = codes;
    }
  } else {
    const float r32 = (float)r;
    const bool fast = r >= 0x1p-100 && r <= 0x1p10;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = column(c);
      if (col >= n) break;
      Raw8<T> o;
      T *to = reinterpret_cast<T *>(a.y) + at + col;
      float big = 0.0f, p[8];
      weighed(c, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = p[i] * r32;
        big = y <= FLT_MAX && y >= -FLT_MAX ? big : INFINITY;
        o.v[i] = (T)y;
      }
      if (fast && big == 0.0f) {
        store8_tail(to, o, EVEN ? 8 : n - col);
      } else {
#pragma unroll 1
        for (int i = 0; i < 8 && col + i < n; ++i) to[i] = (T)(float)(wide(col + i) * r);
      }
    }
  }
}

// Threads and pieces of 8 elements by the row's length and the types alone, so that a row's result is the same alone
// and among others.  Two pieces: half the wavefronts to join and twice the loads on their way; one: less to wait for in a
// row alone.  One and two pieces (us, in a graph, with x into 8 bits unless said):
//   bfloat16, 16 x 4096 3.8 and 4.5; 8192 x 1024 14.2 and 14.7, without 8 bits 13.1 and 12.3; 4096 x 4099 45 and 41;
//     4096 x 4096 28.5 and 29.3, quantisation alone 17.7 and 13.5; four pieces 45 and 16.6
//   two binary16 planes, 4096 x 4096 59 and 49, 16 x 4096 5.2 and 6.0; three, 8192 x 1024 49 and 33
//   binary32, 4096 x 4096 45 and 46, without 8 bits 49 and 53, quantisation alone 25 and 17.
template <typename T, bool ONE, bool NORM, bool INT8>
hipError_t run_norm(NormArgs a, hipStream_t stream) {
  const auto go = [&](auto kernel, int nt) {
    const int per = nt <= 64 ? 256 / nt : 1, block = nt <= 64 ? 256 : nt;
    for (a.first = 0; a.first < a.rows; a.first += LAUNCH_MAX * per) {
      const int64_t left = a.rows - a.first, groups = (left + per - 1) / per;
      kernel<<<(unsigned)(groups < LAUNCH_MAX ? groups : LAUNCH_MAX), block, 0, stream>>>(a);
    }
    return hipGetLastError();
  };
  const int64_t width = INT8 ? a.pitch : a.n;
  const auto pick = [&](auto end) {
    constexpr End E = decltype(end)::value;
    constexpr bool PLAIN16 = ONE && sizeof(T) == 2 && E != END_SHORT;
#define ROW(NT, CH) \
  if constexpr (PLAIN16) return go(norm16_kernel<T, NT, CH, NORM, INT8, E == END_EVEN, 8>, NT); \
  else return go(norm_kernel<T, ONE, NT, CH, NORM, INT8, E>, NT)
    if constexpr (E == END_SHORT) {
      return go(norm_kernel<T, ONE, 16, 1, NORM, INT8, E>, 16);
    } else {
      if (width <= 128) { ROW(16, 1); }
      if (width <= 256) { ROW(32, 1); }
      if (width <= 512) { ROW(64, 1); }
      if constexpr (ONE && sizeof(T) == 4 && NORM) {
        if (width <= 2048) { ROW(256, 1); }
        if (width <= 4096) { ROW(512, 1); }
        if (width <= 8192) { ROW(1024, 1); }
      } else {
        if (width <= 1024) { ROW(64, 2); }
        if (width <= 2048) { ROW(128, 2); }
        if (width <= 4096) { ROW(256, 2); }
        if (width <= 8192) { ROW(512, 2); }
      }
      if (width <= 16384) { ROW(1024, 2); }
      return go(norm_kernel<T, ONE, 1024, 0, NORM, INT8, E>, 1024);
    }
#undef ROW
  };
  switch (end_of(a.n)) {
    case END_EVEN: return pick(std::integral_constant<End, END_EVEN>());
    case END_ODD: return pick(std::integral_constant<End, END_ODD>());
    default: return pick(std::integral_constant<End, END_SHORT>());
  }
}

// code scale, a thread READ pieces of 8 elements, 256 pieces apart.  HBM bounds it: 4096 x 8192 to bfloat16 20 to 21
// us, 4.8 TB/s, where a large copy reaches 5.1.  Two, four and eight pieces a thread: 27.6, 28.7, 29.7; codes that the
// norm has just written, still in a cache, take the same within 1% either way.  (Written without the arrays 25 us.)
constexpr int READ = 1;
template <typename T>
__global__ __launch_bounds__(256) void int8_read_kernel(const uint64_t *codes, const float *scales, T *out, int64_t rows,
                                                        int64_t n, int64_t across, int64_t first) {
  const int64_t total = rows * across, pitch = int8_pitch(n) >> 3;
  int64_t row[READ], col[READ];
  uint64_t w[READ];
  float s[READ];
#pragma unroll
  for (int k = 0; k < READ; ++k) {
    int64_t id = (first + blockIdx.x) * (256 * READ) + k * 256 + threadIdx.x;
    if (id >= total) id = total - 1;  // again
    row[k] = id <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)across) : id / across;
    col[k] = id - row[k] * across;
    w[k] = codes[row[k] * pitch + col[k]];
    s[k] = scales[row[k]];
  }
#pragma unroll
  for (int k = 0; k < READ; ++k) {
    Raw8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (T)((float)(int8_t)(w[k] >> (8 * i)) * s[k]);
    store8_tail(out + row[k] * n + col[k] * 8, o, n - col[k] * 8);
  }
}

template <typename T>
hipError_t read_back(int64_t rows, int64_t n, const void *codes, const void *scales, void *out, hipStream_t stream) {
  const int64_t across = (n + 7) / 8, groups = (rows * across + 256 * READ - 1) / (256 * READ);
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
  double *r;                   // [rows], of long rows
  int64_t rows, n, plane;
  int64_t first;  // the first 64 columns of a launch of the sum
  double eps, inv_n;
  int nc, groups;
};

// Two sums over the NT threads of a row.  lds: room for a row, another one for the next.
template <int NT>
__device__ inline f64x2 row_sum2(f64x2 v, f64x2 *lds) {
  v[0] = lanes_sum<(NT < 64 ? NT : 64)>(v[0]);
  v[1] = lanes_sum<(NT < 64 ? NT : 64)>(v[1]);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[threadIdx.x % (NT / 64)];
    v[0] = lanes_sum<NT / 64>(v[0]);
    v[1] = lanes_sum<NT / 64>(v[1]);
  }
  return v;
}

// What a thread asks for of a row, ahead of the row before.
template <typename T, bool ONE, int CH>
struct BwdRow {
  Raw8<T> h[ONE ? CH : 1], dy[CH], g[CH];
};

// A workgroup takes every groups-th SLOTS rows; a thread the same columns of each, of which it keeps dw's sums.  While a
// row is worked on the next one is on its way.  E, NT, CH as above.
//
// HBM and binary64 arithmetic bound it alike: 8192 x 4096 bfloat16 with g 60 us and 5 us for the sum over workgroups,
// 4.0 TB/s; 43 vector instructions an element, 60% of the cycles; binary32 4096 x 4096
// 56 us, 4.8 TB/s.  Without the next row's loads ahead 95 us, 67 so.  Two pieces a thread, rows past 8192 elements, hold
// 20 to 56 registers too many and keep them in 52 to 168 bytes of scratch memory a lane, plain 16-bit rows of whole
// pieces apart: 2048 x 16384 bfloat16 73 us (no scratch), binary32 147, 3.7 TB/s, two planes of either 109 and 188
// without g, 2048 x 12001 97 and 148.
template <typename T, bool ONE, int NT, int CH, End E>
__global__ __launch_bounds__(NT <= 64 ? 256 : NT, 4) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int BLOCK = NT <= 64 ? 256 : NT, SLOTS = BLOCK / NT;
  constexpr bool AHEAD = ONE && E != END_SHORT && CH == 1;
  __shared__ f64x2 lds[2][BLOCK / 64];
  __shared__ double joined[SLOTS > 1 ? BLOCK : 1][8];
  const int t = threadIdx.x % NT, n = (int)a.n;
  const auto column = [&](int c) { return (c * NT + t) * 8; };
  const auto load = [&](int64_t row, BwdRow<T, ONE, CH> &b) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = column(c);
      if (col >= n) break;
      const int64_t at = row * a.n;
      const auto one = [&](const void *p) {
        if constexpr (E == END_SHORT)
          return load8_tail(reinterpret_cast<const T *>(p) + at + col, (int64_t)(n - col));
        else
          return load8_row<E == END_EVEN>(reinterpret_cast<const T *>(p) + at, col, n, (T)0.0f);
      };
      if constexpr (ONE) b.h[c] = one(a.h);
      b.dy[c] = one(a.dy);
      if (a.g && a.dh) b.g[c] = one(a.g);
    }
  };
  double dw[CH][8];
  Raw8<T> weight[CH];
  BwdRow<T, ONE, CH> next;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.0, weight[c].v[i] = (T)1.0f, next.g[c].v[i] = (T)0.0f;
    if (a.w && column(c) < n) {
      if constexpr (E == END_SHORT)
        weight[c] = load8_tail(reinterpret_cast<const T *>(a.w) + column(c), (int64_t)(n - column(c)));
      else
        weight[c] = load8_row<E == END_EVEN>(reinterpret_cast<const T *>(a.w), column(c), n, (T)0.0f);
    }
  }
  const int64_t step = (int64_t)a.groups * SLOTS;
  int64_t row = (int64_t)blockIdx.x * SLOTS + threadIdx.x / NT;
  if (AHEAD && row < a.rows) load(row, next);
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    BwdRow<T, ONE, CH> b = next;
    if constexpr (AHEAD) {
      if (row + step < a.rows) load(row + step, next);
    } else {
      load(row, b);
    }
    // f(i, v, dy, w dy) of a piece's elements, in binary64, where all products here are exact but for those with r; the
    // fences keep the wide forms of few elements at a time in registers
    double sum[ONE ? 1 : CH][8];
    const auto each = [&](int c, auto f) {
      Raw8<T> hr = {};
      const Raw8<T> dr = renewed(b.dy[c]), wr = renewed(weight[c]);
      if constexpr (ONE) hr = renewed(b.h[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);
        const double d = (double)(float)dr.v[i], w = (double)(float)wr.v[i];
        if constexpr (ONE)
          f(i, (double)(float)hr.v[i], d, w * d);
        else
          f(i, sum[c][i], d, w * d);
      }
    };
    f64x2 s = {0.0, 0.0};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = column(c);
      if (col >= n) break;
      if constexpr (!ONE) planes8<E>(reinterpret_cast<const T *>(a.h) + row * a.n, a.plane, a.nc, col, a.n, sum[c]);
      each(c, [&](int, double v, double, double q) {
        s[0] = fma(v, v, s[0]);
        s[1] = fma(v, q, s[1]);
      });
    }
    s = row_sum2<NT>(s, lds[turn]);
    const double r = inverse_root(s[0] * a.inv_n + a.eps), k = s[1] * a.inv_n * r * r;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = column(c);
      if (col >= n) break;
      Raw8<T> o = {};
      each(c, [&](int i, double v, double d, double q) {
        dw[c][i] = fma(d, v * r, dw[c][i]);
        const double e = fma(-v, k, q) * r;
        o.v[i] = (T)(float)(e + (double)(float)b.g[c].v[i]);
      });
      if (!a.dh) continue;
      store8_tail(reinterpret_cast<T *>(a.dh) + row * a.n + col, o, E == END_EVEN ? 8 : n - col);
    }
  }
  if (!a.dw) return;
  float *p = a.partial + (int64_t)blockIdx.x * a.n;
  if constexpr (SLOTS > 1) {
    // the rows side by side, in order
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) joined[threadIdx.x][i] = dw[c][i];
      __syncthreads();
      for (int e = threadIdx.x; e < NT * 8; e += BLOCK) {
        const int col = c * NT * 8 + e;
        if (col >= n) break;
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) sum += joined[k * NT + e / 8][e % 8];
        p[col] = (float)sum;
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (column(c) + i < n) p[column(c) + i] = (float)dw[c][i];
  }
}

// Rows that do not stay in registers, read twice; dw by the kernel below, which takes r from here.
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(NormBwdArgs a) {
  __shared__ f64x2 lds[2][16];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += a.groups, turn ^= 1) {
    const int64_t at = row * a.n;
    f64x2 s = {0.0, 0.0};
    const auto piece = [&](int64_t col, double v[8], double d[8], double p[8]) {
      planes8<END_ODD>(reinterpret_cast<const T *>(a.h) + at, a.plane, a.nc, col, a.n, v);
      wide8<END_ODD>(reinterpret_cast<const T *>(a.dy) + at, col, a.n, d);
      double w[8] = {1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0};
      if (a.w) wide8<END_ODD>(reinterpret_cast<const T *>(a.w), col, a.n, w);
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
    s = row_sum2<1024>(s, lds[turn]);
    const double r = inverse_root(s[0] * a.inv_n + a.eps), k = s[1] * a.inv_n * r * r;
    if (a.dw && threadIdx.x == 0) a.r[row] = r;
    if (!a.dh) continue;
    for (int64_t col = threadIdx.x * 8; col < a.n; col += 8192) {
      piece(col, v, d, p);
      double g[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
      if (a.g) wide8<END_ODD>(reinterpret_cast<const T *>(a.g) + at, col, a.n, g);
      Raw8<T> o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.v[i] = (T)(float)(g[i] + r * (p[i] - v[i] * k));
      store8_tail(reinterpret_cast<T *>(a.dh) + at + col, o, a.n - col);
    }
  }
}

// dw of long rows: a thread 8 columns of every groups-th row, in order.
template <typename T>
__global__ __launch_bounds__(256) void norm_bwd_long_dw_kernel(NormBwdArgs a) {
  const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= a.n) return;
  double sum[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
  for (int64_t row = blockIdx.y; row < a.rows; row += a.groups) {
    double v[8], d[8];
    planes8<END_ODD>(reinterpret_cast<const T *>(a.h) + row * a.n, a.plane, a.nc, col, a.n, v);
    wide8<END_ODD>(reinterpret_cast<const T *>(a.dy) + row * a.n, col, a.n, d);
    const double r = a.r[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = fma(d[i], v[i] * r, sum[i]);
  }
  float *p = a.partial + (int64_t)blockIdx.y * a.n;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col + i < a.n) p[col + i] = (float)sum[i];
}

// The workgroups' sums: 64 columns by 16 parts of the workgroups, each in order, then the parts.  Rows past 2^27
// elements take several launches.
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_sum_kernel(NormBwdArgs a) {
  __shared__ double part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (a.first + blockIdx.x) * 64 + lane;
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

// Workgroups: as many as are resident, since a row's loads go out ahead of the row before: one a CU of rows that
// take 1024 threads, two of 512, four of 256, eight of 128 (16-bit rows: 32263 x 520 62 us, with 256 threads 75; binary32
// 71 and 67); four where a workgroup has several rows.  With twice (half) as many (us; 4096 x 4096 bfloat16, with g)
// 46 (49) in place of 40, 8192 x 1024 32 (33) in place of 26, 4096 x 8192 78 in place of 69.  Of rows that do not stay
// in registers, parts of the rows for dw.
int bwd_groups(int dtype, int64_t rows, int64_t n) {
  if (n > BWD_LONG) return (int)(rows < 64 ? rows : 64);
  const int64_t slots = n <= 128 ? 16 : (n <= 256 ? 8 : (n <= 512 ? 4 : 1));
  const bool narrow = dtype != LM_F32 && n > 512 && n <= 1024;
  const int64_t most = narrow ? 2048 : (n <= 2048 ? 1024 : (n <= 4096 ? 512 : 256));
  const int64_t wanted = (rows + slots - 1) / slots;
  return (int)(wanted < most ? wanted : most);
}

template <typename T>
hipError_t run_bwd(NormBwdArgs a, hipStream_t stream) {
  const unsigned grid = (unsigned)a.groups;
  if (a.n > BWD_LONG) {
    if (grid) {
      NormBwdArgs b = a;
      b.groups = (int)(a.rows < 1024 ? a.rows : 1024);
      norm_bwd_long_kernel<T><<<(unsigned)b.groups, 1024, 0, stream>>>(b);
      if (a.dw) norm_bwd_long_dw_kernel<T><<<dim3((unsigned)((a.n + 2047) / 2048), grid), 256, 0, stream>>>(a);
    }
  } else if (grid) {
    const auto go = [&](auto one, auto end) {
      constexpr bool ONE = decltype(one)::value;
      constexpr End E = decltype(end)::value;
#define ROW(NT, CH) return norm_bwd_kernel<T, ONE, NT, CH, E><<<grid, NT <= 64 ? 256 : NT, 0, stream>>>(a)
      if (E == END_SHORT || a.n <= 128) ROW(16, 1);
      if constexpr (E != END_SHORT) {
        if (a.n <= 256) ROW(32, 1);
        if (a.n <= 512) ROW(64, 1);
        if constexpr (sizeof(T) == 2)
          if (a.n <= 1024) ROW(128, 1);
        if (a.n <= 2048) ROW(256, 1);
        if (a.n <= 4096) ROW(512, 1);
        if (a.n <= 8192) ROW(1024, 1);
        ROW(1024, 2);
      }
#undef ROW
    };
    const auto pick = [&](auto end) { a.nc == 1 ? go(Flag<true>(), end) : go(Flag<false>(), end); };
    switch (end_of(a.n)) {
      case END_EVEN: pick(std::integral_constant<End, END_EVEN>()); break;
      case END_ODD: pick(std::integral_constant<End, END_ODD>()); break;
      default: pick(std::integral_constant<End, END_SHORT>());
    }
  }
  if (!a.dw) return hipGetLastError();
  const int64_t all = (a.n + 63) / 64;
  for (; a.first < all; a.first += LAUNCH_MAX)
    norm_bwd_sum_kernel<T><<<(unsigned)(all - a.first < LAUNCH_MAX ? all - a.first : LAUNCH_MAX), 1024, 0, stream>>>(a);
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
  a.inv_n = n > 0 ? 1.0 / (double)n : 0.0;
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

int64_t rmsnorm_bwd_workspace_bytes(int dtype, int64_t rows, int64_t n) {
  return bwd_groups(dtype, rows, n) * n * 4 + (n > BWD_LONG ? rows * 8 + 8 : 0);
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
  a.inv_n = n > 0 ? 1.0 / (double)n : 0.0;
  a.nc = nc;
  a.groups = bwd_groups(dtype, rows, n);
  a.r = (double *)((char *)ws + (a.groups * n * 4 + 7) / 8 * 8);
  if (dtype == LM_F16) return run_bwd<_Float16>(a, stream);
  if (dtype == LM_BF16) return run_bwd<__bf16>(a, stream);
  return run_bwd<float>(a, stream);
}

}  // namespace mcf
