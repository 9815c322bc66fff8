// distill.hip -- the distillation loss from a teacher's top logits, and its gradient.
//
// A row has student logits z_j, j < V (plain, or an MC value whose planes are summed in
// binary32, the last plane first) and up to k teacher entries (id_i, t_i).  With temperature T
//   p = softmax over the row's used entries of t_i / T,   q = softmax over the row of z_j / T,
//   loss = T^2 sum_i p_i (log p_i - log q_{id_i}),
//   dz_j = g T (q_j - sum of the p_i with id_i = j).
// An entry whose id lies outside [0, V) is unused; a row with no used entry (or none with
// p > 0) has loss 0 and gradient 0.  One pass over the row keeps the running maximum m and
// s = sum exp((z_j - m) / T); the gradient is a second pass, in the fused call over registers.
// The row is read once and the gradient written once, so HBM bounds it: 4096 rows of 32768 bfloat16
// logits take 111 us (4.8 TB/s) for both, 50 us (5.4 TB/s) for the loss alone.  Where both are asked for
// and the row does not stay in registers it is read twice: 1024 rows of 131072 binary32 logits 312 us (3.4
// TB/s), 4096 of 32768 in two binary16 planes 275 us (2.9 TB/s).
//
// The row's sums are binary32.  m starts at the lowest finite number, so that a masked logit (-inf)
// is exp(-inf) = 0 with no test, also in front of the first finite one; a row of nothing but
// -inf has s = 0 and q = 0.
#include <float.h>
#include <math.h>

#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace mcf {
namespace {

struct DistillArgs {
  const void *z, *t;
  const int32_t *ids;
  const float *g, *stats_in;
  float *loss, *stats;
  void *dz;
  f32x2 *partial;  // [rows][chunks]
  int64_t rows, plane;
  int64_t first;  // the launch's first row, where a workgroup takes one
  int vocab, k, nc, chunks;
  float temperature, c_hi, c_lo;  // c_hi + c_lo = log2(e) / T
};

constexpr int CHUNK = 4096;  // elements of a row a workgroup takes where a row has several

// exp((z - m) / T).  The second term of the factor keeps the argument's error at one rounding
// where the result is binary32; it is positive, so that a difference of -inf stays -inf.
template <typename T>
__device__ inline float expz(const DistillArgs &a, float d) {
  if constexpr (sizeof(T) == 4) return __builtin_amdgcn_exp2f(fmaf(d, a.c_hi, d * a.c_lo));
  return __builtin_amdgcn_exp2f(d * a.c_hi);
}

struct MaxSum {
  float m, s;
};

template <typename T>
__device__ inline MaxSum join(const DistillArgs &a, MaxSum x, MaxSum y) {
  MaxSum r;
  r.m = fmaxf(x.m, y.m);
  r.s = x.s * expz<T>(a, x.m - r.m) + y.s * expz<T>(a, y.m - r.m);
  return r;
}

template <typename T>
__device__ inline void add8(const DistillArgs &a, MaxSum &r, const float v[8]) {
  float m = r.m;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, v[i]);
  float s = r.s * expz<T>(a, r.m - m);
#pragma unroll
  for (int i = 0; i < 8; ++i) s += expz<T>(a, v[i] - m);
  r.m = m;
  r.s = s;
}

// Eight logits from column col of a row; those past the row are -inf.
template <typename T, bool ONE>
__device__ inline void logits8(const DistillArgs &a, const T *z, int64_t col, float v[8]) {
  const int64_t left = a.vocab - col;
  if (ONE) {
    const Raw8<T> r = load8_tail(z + col, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)r.v[i] : -INFINITY;
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  for (int p = a.nc - 1; p >= 0; --p) {
    const Raw8<T> r = load8_tail(z + p * a.plane + col, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p == a.nc - 1 ? (float)r.v[i] : v[i] + (float)r.v[i];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= left) v[i] = -INFINITY;
}

template <typename T, bool ONE>
__device__ inline float logit(const DistillArgs &a, const T *z, int64_t col) {
  if (ONE) return (float)z[col];
  float v = (float)z[(a.nc - 1) * a.plane + col];
  for (int p = a.nc - 2; p >= 0; --p) v += (float)z[p * a.plane + col];
  return v;
}

// Joins over the workgroup in a fixed order; every thread gets the result.
template <typename T, int NT>
__device__ inline MaxSum block_join(const DistillArgs &a, MaxSum r, MaxSum *lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    MaxSum o;
    o.m = __shfl_xor(r.m, d);
    o.s = __shfl_xor(r.s, d);
    // both sides join in the lower lane's order, so the lanes agree
    r = (threadIdx.x & d) ? join<T>(a, o, r) : join<T>(a, r, o);
  }
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r;
  __syncthreads();
  r = lds[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) r = join<T>(a, r, lds[w]);
  return r;
}

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// A row's teacher entries, worked out by the first wavefront while the row is on its way:
// e = exp((t - top) / T), 0 where unused; all = the sum of the e of every entry with this id; the
// teacher's softmax is p = e / sum.  The k entries' sums and the loss are binary64: they are few, the
// divergence is a small difference of large logarithms, and where a mask of the type's lowest value
// meets a teacher's entry the terms come up to binary32's largest number.
template <int NT>
struct Shared {
  MaxSum join[NT / 64];
  double sum;  // of the used entries' e; 0: none counts
  float top;   // the largest used t
};
// The entries' arrays, 16 k bytes of LDS.
extern __shared__ float entry_space[];
#define ENTRIES                                                       \
  [[maybe_unused]] int *const eid = (int *)entry_space;               \
  [[maybe_unused]] float *const ee = entry_space + a.k;               \
  [[maybe_unused]] float *const eall = ee + a.k, *const ez = eall + a.k

// The sum of the e of the entries with this id, in the entries' order.
__device__ inline float same_id(const DistillArgs &a, int id) {
  ENTRIES;
  float all = 0.0f;
  int j = 0;
  for (; j + 8 <= a.k; j += 8) {
    int other[8];
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = eid[j + i], e[i] = ee[j + i];
#pragma unroll
    for (int i = 0; i < 8; ++i) all += other[i] == id ? e[i] : 0.0f;
  }
  for (; j < a.k; ++j) all += eid[j] == id ? ee[j] : 0.0f;
  return all;
}

// The first entry of a lane, loaded ahead of the row so that it does not wait for it.
template <typename T>
struct First {
  int id;
  T t;
};
template <typename T>
__device__ inline First<T> first_entry(const DistillArgs &a, int64_t row) {
  First<T> f = {-1, (T)0.0f};
  if ((int)threadIdx.x < a.k && threadIdx.x < 64) {
    f.id = a.ids[row * a.k + threadIdx.x];
    f.t = reinterpret_cast<const T *>(a.t)[row * a.k + threadIdx.x];
  }
  return f;
}

template <typename T, bool ONE, int NT>
__device__ inline void teacher(const DistillArgs &a, int64_t row, const T *z, const First<T> &f, Shared<NT> &sh) {
  ENTRIES;
  if (threadIdx.x < 64) {
    float top = -FLT_MAX;
    for (int i = threadIdx.x; i < a.k; i += 64) {
      const int id = i < 64 ? f.id : a.ids[row * a.k + i];
      const T t = i < 64 ? f.t : reinterpret_cast<const T *>(a.t)[row * a.k + i];
      const bool used = id >= 0 && id < a.vocab;
      const float v = used ? (float)t : -INFINITY;
      eid[i] = used ? id : -1;
      ee[i] = v;
      top = fmaxf(top, v);
    }
    top = wave_max(top);
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.k; i += 64) {
      const float e = expz<float>(a, ee[i] - top);
      ee[i] = e;
      sum += (double)e;
    }
    sum = wave_sum(sum);
    if (threadIdx.x == 0) sh.top = top, sh.sum = sum;
  }
  // the logits at the entries and the sums of equal ids: up to 64 entries by the one wavefront that
  // wrote them, more by all
  if (a.k > 64)
    __syncthreads();
  else
    wave_sync();
  const int n = a.k > 64 ? NT : 64;
  if ((int)threadIdx.x < n)
    for (int i = threadIdx.x; i < a.k; i += n) {
      const int id = eid[i];
      ez[i] = id >= 0 ? logit<T, ONE>(a, z, id) : 0.0f;
      eall[i] = same_id(a, id);
    }
  // read by others only behind block_join's barrier
}

// The row's loss, by the first wavefront.
template <typename T, int NT>
__device__ inline void row_loss(const DistillArgs &a, int64_t row, const MaxSum &st, const Shared<NT> &sh) {
  const T *t = reinterpret_cast<const T *>(a.t) + row * a.k;
  ENTRIES;
  const double log_s = (double)logf(st.s), log_sum = (double)logf((float)sh.sum);
  const double inv = sh.sum == 0.0 ? 0.0 : 1.0 / sh.sum, inv_t = 1.0 / (double)a.temperature;
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.k; i += 64) {
    const double p = (double)ee[i] * inv;
    if (p == 0.0) continue;
    if (eid[i] < 0) {  // the entries' sum is not a number: so is the loss
      sum += p;
      continue;
    }
    const float zi = ez[i];
    // binary64: below a temperature of 1 the logarithm of q at a mask of the type's lowest value passes
    // binary32's range, where the loss, T^2 times it, need not
    const double log_p = ((double)(float)t[i] - (double)sh.top) * inv_t - log_sum;
    const double log_q = zi == -INFINITY ? -INFINITY : ((double)zi - (double)st.m) * inv_t - log_s;
    sum += p * (log_p - log_q);
  }
  sum = wave_sum(sum);
  if (threadIdx.x == 0) a.loss[row] = (float)((double)a.temperature * (double)a.temperature * sum);
}

// The gradient at the teacher's entries of columns [lo, hi): written over what the pass over the row
// left there.
template <typename T, int NT>
__device__ inline void entries(const DistillArgs &a, T *dz, const MaxSum &st, float inv_s, float inv_p, float coef, int lo,
                               int hi) {
  ENTRIES;
  for (int i = threadIdx.x; i < a.k; i += NT) {
    const int id = eid[i];
    if (id < lo || id >= hi) continue;
    const float q = expz<T>(a, ez[i] - st.m) * inv_s;
    dz[id] = (T)(coef * (q - eall[i] * inv_p));
  }
}

template <typename T>
__device__ inline Raw8<T> grad8(const DistillArgs &a, const float v[8], float m, float f) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = (T)(expz<T>(a, v[i] - m) * f);
  return r;
}

template <typename T>
__device__ inline Raw8<T> zero8() {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = (T)0.0f;
  return r;
}

// The kept elements as a new value, so that the compiler converts 16-bit ones again in the next
// pass instead of holding them in 32 bits.
template <typename T>
__device__ inline void renew(Raw8<T> &r) {
  if constexpr (sizeof(T) == 2) {
    u32x4 u = __builtin_bit_cast(u32x4, r);
    asm("" : "+v"(u));
    r = __builtin_bit_cast(Raw8<T>, u);
  }
}

// One workgroup a row.  CH > 0: the row, of 8 elements or more, fits CH pieces of 8 elements a
// thread and is kept in registers between the sum and the gradient; CH = 0: it is read again.  A
// piece past the row's last whole one is the row's last eight elements, of which those that belong to
// its neighbour do not count in the sum and get the same gradient twice.  With given (m, s) the
// gradient alone.  OCC: wavefronts a SIMD, bought with registers: rows' phases overlap.
template <typename T, bool ONE, int NT, int CH, bool GRAD, int OCC>
__global__ __launch_bounds__(NT, OCC) void distill_row_kernel(DistillArgs a) {
  constexpr int FLY = ONE ? 4 : 2;  // pieces in flight where the row is read again
  __shared__ Shared<NT> sh;
  const int64_t row = a.first + blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  MaxSum st = {-FLT_MAX, 0.0f};
  Raw8<T> keep[CH > 0 ? CH : 1];
  const auto column = [&](int c) { return (c * NT + (int)threadIdx.x) * 8; };
  const auto begin = [&](int c) { return column(c) < a.vocab - 8 ? column(c) : a.vocab - 8; };
  const First<T> first = first_entry<T>(a, row);
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (column(c) < a.vocab) keep[c] = load8(z + begin(c));
  }
  teacher<T, ONE, NT>(a, row, z, first, sh);
  if (a.stats_in) {
    st.m = a.stats_in[2 * row], st.s = a.stats_in[2 * row + 1];
    __syncthreads();
  } else {
    if constexpr (CH > 0) {
      // the thread's maximum first (a neighbour's elements do no harm there), then its sum
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (column(c) < a.vocab) {
#pragma unroll
          for (int i = 0; i < 8; ++i) st.m = fmaxf(st.m, (float)keep[c].v[i]);
        }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        renew(keep[c]);
        if ((c + 1) * NT * 8 <= a.vocab) {
#pragma unroll
          for (int i = 0; i < 8; ++i) st.s += expz<T>(a, (float)keep[c].v[i] - st.m);
        } else if (column(c) < a.vocab) {
          const int skip = column(c) - begin(c);
#pragma unroll
          for (int i = 0; i < 8; ++i) st.s += i < skip ? 0.0f : expz<T>(a, (float)keep[c].v[i] - st.m);
        }
      }
    } else {
      for (int64_t col = threadIdx.x * 8; col < a.vocab; col += NT * 8 * FLY) {
        float v[FLY][8];
#pragma unroll
        for (int u = 0; u < FLY; ++u) logits8<T, ONE>(a, z, col + u * NT * 8, v[u]);
#pragma unroll
        for (int u = 0; u < FLY; ++u) add8<T>(a, st, v[u]);
      }
    }
    st = block_join<T, NT>(a, st, sh.join);
  }
  if constexpr (GRAD) {
    T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
    const float coef = (a.g ? a.g[row] : 1.0f) * a.temperature;
    const float inv_s = st.s == 0.0f ? 0.0f : 1.0f / st.s;
    if (sh.sum == 0.0) {  // no entry counts
      for (int64_t col = threadIdx.x * 8; col < a.vocab; col += NT * 8) store8_tail(dz + col, zero8<T>(), a.vocab - col);
    } else {
      if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
          if (column(c) < a.vocab) {
            renew(keep[c]);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)keep[c].v[i];
            const Raw8<T> r = grad8<T>(a, v, st.m, coef * inv_s);
            __builtin_memcpy(dz + begin(c), &r, sizeof(r));
          }
      } else {
        for (int64_t col = threadIdx.x * 8; col < a.vocab; col += NT * 8 * FLY) {
          float v[FLY][8];
#pragma unroll
          for (int u = 0; u < FLY; ++u) logits8<T, ONE>(a, z, col + u * NT * 8, v[u]);
#pragma unroll
          for (int u = 0; u < FLY; ++u) {
            const int64_t at = col + u * NT * 8;
            store8_tail(dz + at, grad8<T>(a, v[u], st.m, coef * inv_s), a.vocab - at);
          }
        }
      }
      __syncthreads();  // the pass's stores come before the entries'
      entries<T, NT>(a, dz, st, inv_s, (float)(1.0 / sh.sum), coef, 0, a.vocab);
    }
  }
  if (threadIdx.x < 64) {
    if (a.loss) row_loss<T, NT>(a, row, st, sh);
    if (a.stats && threadIdx.x == 0) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.s;
  }
}

// Rows over several workgroups: the (m, s) of one chunk.
template <typename T, bool ONE>
__global__ __launch_bounds__(256) void distill_partial_kernel(DistillArgs a) {
  __shared__ MaxSum lds[4];
  const int64_t row = blockIdx.y, lo = (int64_t)blockIdx.x * CHUNK;
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  MaxSum st = {-FLT_MAX, 0.0f};
#pragma unroll
  for (int c = 0; c < CHUNK / 2048; ++c) {
    float v[8];
    logits8<T, ONE>(a, z, lo + c * 2048 + threadIdx.x * 8, v);
    add8<T>(a, st, v);
  }
  st = block_join<T, 256>(a, st, lds);
  if (threadIdx.x == 0) a.partial[row * a.chunks + blockIdx.x] = {st.m, st.s};
}

// The rest of a row over several workgroups: the chunks' (m, s), or the given ones, joined by
// every workgroup in the same order; the first one writes the loss and (m, s); GRAD: each
// writes its chunk of the gradient.
template <typename T, bool ONE, bool GRAD>
__global__ __launch_bounds__(256) void distill_finish_kernel(DistillArgs a) {
  __shared__ Shared<256> sh;
  const int64_t row = blockIdx.y;
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  MaxSum st = {-FLT_MAX, 0.0f};
  teacher<T, ONE, 256>(a, row, z, first_entry<T>(a, row), sh);
  if (a.stats_in) {
    st.m = a.stats_in[2 * row], st.s = a.stats_in[2 * row + 1];
    __syncthreads();
  } else {
    for (int c = threadIdx.x; c < a.chunks; c += 256) {
      const f32x2 p = a.partial[row * a.chunks + c];
      st = join<T>(a, st, MaxSum{p[0], p[1]});
    }
    st = block_join<T, 256>(a, st, sh.join);
  }
  if constexpr (GRAD) {
    T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
    const float coef = (a.g ? a.g[row] : 1.0f) * a.temperature;
    const float inv_s = st.s == 0.0f ? 0.0f : 1.0f / st.s;
    const bool none = sh.sum == 0.0;
    const int64_t lo = (int64_t)blockIdx.x * CHUNK;
#pragma unroll
    for (int c = 0; c < CHUNK / 2048; ++c) {
      const int64_t col = lo + c * 2048 + threadIdx.x * 8;
      Raw8<T> r = zero8<T>();
      if (!none) {
        float v[8];
        logits8<T, ONE>(a, z, col, v);
        r = grad8<T>(a, v, st.m, coef * inv_s);
      }
      store8_tail(dz + col, r, a.vocab - col);
    }
    if (!none) {
      __syncthreads();
      const int64_t hi = lo + CHUNK < a.vocab ? lo + CHUNK : a.vocab;
      entries<T, 256>(a, dz, st, inv_s, (float)(1.0 / sh.sum), coef, (int)lo, (int)hi);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    if (a.loss) row_loss<T, 256>(a, row, st, sh);
    if (a.stats && threadIdx.x == 0) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.s;
  }
}

// Few rows of a long vocabulary go to several workgroups a row; else one workgroup a row.  Loss and
// gradient by one and by several (us, launches in a graph): 131072 bfloat16 logits, 1 row 17.8 and 8.5, 64
// 20.7 and 17.2, 128 23.1 and 28.2, 255 28.6 and 47.2; of binary32 30.1 and 8.5, 36.2 and 23.2, 40.5 and
// 39.6, 65.7 and 67.4; 32768 bfloat16, 1 row 7.9 and 8.4, 255 10.8 and 16.9; 16384, 16 rows 6.6 and 8.7.
// Several pay at 131072 logits up to about 100 rows; at the shorter rows that the rule gives them they
// lose 0.5 to 6 us, a launch and a second read of the row.
bool several(int64_t rows, int64_t vocab) { return rows < 256 && vocab > 2 * CHUNK; }

// One workgroup a row, `count` rows from a.first.  The row in registers where it fits 64 of them a
// thread, read again where it does not (MC logits, rows below one piece, long rows).  Loss and gradient
// of bfloat16 rows (us, launches in a graph; threads x pieces, the rule's first): 32768 rows of 1000, 64 x 2
// 40, 256 x 1 74, read again 150; 8192 of 4096, 256 x 2 30, 64 x 8 26 (binary32: 46 and 70), 512 x 1 44, read
// again 51; 8192 of 8192, 256 x 4 46, 512 x 2 55, read again 67; 4096 of 32768, 512 x 8 110, 1024 x 4 105, read
// again 162; 2048 of 65536, 1024 x 8 107, read again 168.
template <typename T, bool ONE, bool GRAD>
void run_rows(const DistillArgs &a, int64_t count, hipStream_t stream) {
  const dim3 grid((unsigned)count);
#define ROW(NT, CH, OCC) distill_row_kernel<T, ONE, NT, CH, GRAD, OCC><<<grid, NT, 16 * a.k, stream>>>(a)
  if constexpr (ONE) {
    constexpr bool SHORT = sizeof(T) == 2;
    if (a.vocab >= 8) {
      if (a.vocab <= 512) return ROW(64, 1, 8);
      if (a.vocab <= 1024) return ROW(64, 2, 8);
      if (a.vocab <= 2048) return ROW(64, 4, 8);
      if (a.vocab <= 4096) return ROW(256, 2, 8);
      if (a.vocab <= 8192) return ROW(256, 4, SHORT ? 8 : 6);
      if (a.vocab <= 16384) return ROW(512, 4, SHORT ? 8 : 6);
      if (a.vocab <= 32768) return ROW(512, 8, SHORT ? 8 : 4);
      if (a.vocab <= 65536) return ROW(1024, 8, 4);
      if constexpr (SHORT)
        if (a.vocab <= 131072) return ROW(1024, 16, 4);
    }
  }
  if (a.vocab <= 2048)
    ROW(64, 0, 4);
  else if (a.vocab <= 32768)
    ROW(256, 0, 4);
  else
    ROW(1024, 0, 4);
#undef ROW
}

template <typename T, bool ONE, bool GRAD>
hipError_t run(DistillArgs a, hipStream_t stream) {
  if (several(a.rows, a.vocab)) {
    const dim3 grid((unsigned)a.chunks, (unsigned)a.rows);
    if (!a.stats_in) distill_partial_kernel<T, ONE><<<grid, 256, 0, stream>>>(a);
    distill_finish_kernel<T, ONE, GRAD><<<GRAD ? grid : dim3(1, (unsigned)a.rows), 256, 16 * a.k, stream>>>(a);
    return hipGetLastError();
  }
  for (a.first = 0; a.first < a.rows; a.first += LAUNCH_MAX)
    run_rows<T, ONE, GRAD>(a, a.rows - a.first < LAUNCH_MAX ? a.rows - a.first : LAUNCH_MAX, stream);
  return hipGetLastError();
}

}  // namespace

int64_t distill_workspace_bytes(int64_t rows, int64_t vocab) {
  return several(rows, vocab) ? rows * ((vocab + CHUNK - 1) / CHUNK) * (int64_t)sizeof(f32x2) : 0;
}

hipError_t launch_distill(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                          const void *t, double temperature, const void *stats_in, const void *g, void *ws, void *loss,
                          void *stats, void *dz, hipStream_t stream) {
  DistillArgs a = {};
  a.z = z;
  a.t = t;
  a.ids = (const int32_t *)ids;
  a.g = (const float *)g;
  a.stats_in = (const float *)stats_in;
  a.loss = (float *)loss;
  a.stats = (float *)stats;
  a.dz = dz;
  a.partial = (f32x2 *)ws;
  a.rows = rows;
  a.plane = rows * vocab;
  a.vocab = (int)vocab;
  a.k = (int)k;
  a.nc = nc;
  a.chunks = (int)((vocab + CHUNK - 1) / CHUNK);
  a.temperature = (float)temperature;
  const double c = 1.4426950408889634 / (double)a.temperature;
  a.c_hi = (float)c;
  if ((double)a.c_hi > c) a.c_hi = nextafterf(a.c_hi, 0.0f);
  a.c_lo = fmaxf((float)(c - (double)a.c_hi), FLT_MIN);
  const auto go = [&](auto zero) {
    using T = decltype(zero);
    if (nc == 1) return dz ? run<T, true, true>(a, stream) : run<T, true, false>(a, stream);
    return dz ? run<T, false, true>(a, stream) : run<T, false, false>(a, stream);
  };
  if (dtype == LM_F16) return go((_Float16)0.0f);
  if (dtype == LM_BF16) return go((__bf16)0.0f);
  return go(0.0f);
}

}  // namespace mcf
