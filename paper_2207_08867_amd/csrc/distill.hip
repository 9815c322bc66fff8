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
// The row is read once and the gradient written once, so HBM bounds it.
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

// Joins over the workgroup in a fixed order; every thread gets the result.  `lds`: NT / 64 slots.
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
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r;
    __syncthreads();
    r = lds[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = join<T>(a, r, lds[w]);
  }
  return r;
}

__device__ inline float combine(float a, float b) { return fmaxf(a, b); }
__device__ inline double combine(double a, double b) { return a + b; }

// The maximum of binary32 values, the sum of binary64 ones.
template <int NT, typename V>
__device__ inline V block_reduce(V v, V *lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = combine(v, __shfl_xor(v, d));
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = combine(v, lds[w]);
  }
  return v;
}

template <int NT>
struct Shared {
  MaxSum join[NT / 64];
  float top[NT / 64];
  double sum[NT / 64];
  int id[1024];
  float e[1024];
};

struct Teacher {
  float top;    // the largest used t
  double sum;   // of the used entries' exp((t - top) / T)
  float inv;    // 1 / sum; 0: no entry counts
};

// The teacher's softmax: p = e / sum; e and id of every entry into LDS (e = 0, id = -1 where
// unused).  The k entries' sums and the loss are binary64: they are few, the divergence is a
// small difference of large logarithms, and where a mask of the type's lowest value meets a
// teacher's entry the terms come up to binary32's largest number.
template <typename T, int NT>
__device__ inline Teacher teacher(const DistillArgs &a, int64_t row, Shared<NT> &sh) {
  const T *t = reinterpret_cast<const T *>(a.t) + row * a.k;
  const int32_t *ids = a.ids + row * a.k;
  float top = -FLT_MAX;
  for (int i = threadIdx.x; i < a.k; i += NT) {
    const int id = ids[i];
    const bool used = id >= 0 && id < a.vocab;
    const float v = used ? (float)t[i] : -INFINITY;
    sh.id[i] = used ? id : -1;
    sh.e[i] = v;
    top = fmaxf(top, v);
  }
  top = block_reduce<NT>(top, sh.top);
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.k; i += NT) {
    const float e = expz<float>(a, sh.e[i] - top);
    sh.e[i] = e;
    sum += (double)e;
  }
  __syncthreads();
  Teacher r;
  r.top = top;
  r.sum = block_reduce<NT>(sum, sh.sum);
  r.inv = r.sum == 0.0 ? 0.0f : (float)(1.0 / r.sum);  // a NaN stays one
  return r;
}

template <typename T, bool ONE, int NT>
__device__ inline float row_loss(const DistillArgs &a, int64_t row, const T *z, const Teacher &te, const MaxSum &st,
                                 Shared<NT> &sh) {
  const T *t = reinterpret_cast<const T *>(a.t) + row * a.k;
  const float log_s = logf(st.s), log_sum = logf((float)te.sum);
  const double inv = te.sum == 0.0 ? 0.0 : 1.0 / te.sum;
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.k; i += NT) {
    const double p = (double)sh.e[i] * inv;
    if (p == 0.0) continue;
    const int id = sh.id[i];
    if (id < 0) {  // the entries' sum is not a number: so is the loss
      sum += p;
      continue;
    }
    const float zi = logit<T, ONE>(a, z, id);
    const float log_p = ((float)t[i] - te.top) / a.temperature - log_sum;
    const float log_q = zi == -INFINITY ? -INFINITY : (zi - st.m) / a.temperature - log_s;
    sum += p * ((double)log_p - (double)log_q);
  }
  sum = block_reduce<NT>(sum, sh.sum);
  return (float)((double)a.temperature * (double)a.temperature * sum);
}

// The teacher's entries of columns [lo, hi): written over what the pass over the row left there.
template <typename T, bool ONE, int NT>
__device__ inline void entries(const DistillArgs &a, const T *z, T *dz, const MaxSum &st, float inv_s, float inv_p,
                               float coef, int lo, int hi, const Shared<NT> &sh) {
  for (int i = threadIdx.x; i < a.k; i += NT) {
    const int id = sh.id[i];
    if (id < lo || id >= hi) continue;
    float p = 0.0f;  // every entry of this id, in the entries' order
    for (int j = 0; j < a.k; ++j) p += sh.id[j] == id ? sh.e[j] : 0.0f;
    const float q = expz<T>(a, logit<T, ONE>(a, z, id) - st.m) * inv_s;
    dz[id] = (T)(coef * (q - p * inv_p));
  }
}

template <typename T>
__device__ inline void grad8(const DistillArgs &a, const float v[8], T *dz, int64_t col, float m, float f) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = (T)(expz<T>(a, v[i] - m) * f);
  store8_tail(dz + col, r, a.vocab - col);
}

template <typename T>
__device__ inline void zero8(const DistillArgs &a, T *dz, int64_t col) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = (T)0.0f;
  store8_tail(dz + col, r, a.vocab - col);
}

// One workgroup a row.  CH > 0: the row fits CH pieces of 8 elements a thread and is kept in
// registers for the gradient; CH = 0: it is read again.
template <typename T, bool ONE, int NT, int CH, bool GRAD>
__global__ __launch_bounds__(NT) void distill_row_kernel(DistillArgs a) {
  __shared__ Shared<NT> sh;
  const int64_t row = blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  MaxSum st = {-FLT_MAX, 0.0f};
  Raw8<T> keep[CH > 0 ? CH : 1];
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t col = ((int64_t)c * NT + threadIdx.x) * 8, left = a.vocab - col;
      keep[c] = load8_tail(z + col, left);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= left) keep[c].v[i] = (T)-INFINITY;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)keep[c].v[i];
      add8<T>(a, st, v);
    }
  } else {
    for (int64_t col = threadIdx.x * 8; col < a.vocab; col += NT * 8) {
      float v[8];
      logits8<T, ONE>(a, z, col, v);
      add8<T>(a, st, v);
    }
  }
  st = block_join<T, NT>(a, st, sh.join);
  const Teacher te = teacher<T, NT>(a, row, sh);
  const float loss = row_loss<T, ONE, NT>(a, row, z, te, st, sh);
  if (threadIdx.x == 0) {
    if (a.loss) a.loss[row] = loss;
    if (a.stats) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.s;
  }
  if constexpr (GRAD) {
    T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
    const float coef = (a.g ? a.g[row] : 1.0f) * a.temperature;
    const float inv_s = st.s == 0.0f ? 0.0f : 1.0f / st.s;
    const bool none = te.inv == 0.0f;
    if constexpr (CH > 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int64_t col = ((int64_t)c * NT + threadIdx.x) * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)keep[c].v[i];
        if (none)
          zero8(a, dz, col);
        else
          grad8<T>(a, v, dz, col, st.m, coef * inv_s);
      }
    } else {
      for (int64_t col = threadIdx.x * 8; col < a.vocab; col += NT * 8) {
        if (none) {
          zero8(a, dz, col);
          continue;
        }
        float v[8];
        logits8<T, ONE>(a, z, col, v);
        grad8<T>(a, v, dz, col, st.m, coef * inv_s);
      }
    }
    if (none) return;
    __syncthreads();  // the pass's stores come before the entries'
    entries<T, ONE, NT>(a, z, dz, st, inv_s, te.inv, coef, 0, a.vocab, sh);
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
  if (a.stats_in) {
    st.m = a.stats_in[2 * row], st.s = a.stats_in[2 * row + 1];
  } else {
    for (int c = threadIdx.x; c < a.chunks; c += 256) {
      const f32x2 p = a.partial[row * a.chunks + c];
      st = join<T>(a, st, MaxSum{p[0], p[1]});
    }
    st = block_join<T, 256>(a, st, sh.join);
  }
  const Teacher te = teacher<T, 256>(a, row, sh);
  if (blockIdx.x == 0) {
    if (a.loss) {
      const float loss = row_loss<T, ONE, 256>(a, row, z, te, st, sh);
      if (threadIdx.x == 0) a.loss[row] = loss;
    }
    if (a.stats && threadIdx.x == 0) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.s;
  }
  if constexpr (GRAD) {
    T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
    const float coef = (a.g ? a.g[row] : 1.0f) * a.temperature;
    const float inv_s = st.s == 0.0f ? 0.0f : 1.0f / st.s;
    const bool none = te.inv == 0.0f;
    const int64_t lo = (int64_t)blockIdx.x * CHUNK;
    for (int c = 0; c < CHUNK / 2048; ++c) {
      const int64_t col = lo + c * 2048 + threadIdx.x * 8;
      if (none) {
        zero8(a, dz, col);
      } else {
        float v[8];
        logits8<T, ONE>(a, z, col, v);
        grad8<T>(a, v, dz, col, st.m, coef * inv_s);
      }
    }
    if (none) return;
    __syncthreads();
    const int64_t hi = lo + CHUNK < a.vocab ? lo + CHUNK : a.vocab;
    entries<T, ONE, 256>(a, z, dz, st, inv_s, te.inv, coef, (int)lo, (int)hi, sh);
  }
}

// Few rows of a long vocabulary go to several workgroups a row; else one workgroup a row.
bool several(int64_t rows, int64_t vocab) { return rows < 256 && vocab > 2 * CHUNK; }

template <typename T, bool ONE, bool GRAD>
hipError_t forward(const DistillArgs &a, hipStream_t stream) {
  if (several(a.rows, a.vocab)) {
    const dim3 grid((unsigned)a.chunks, (unsigned)a.rows);
    distill_partial_kernel<T, ONE><<<grid, 256, 0, stream>>>(a);
    distill_finish_kernel<T, ONE, GRAD><<<GRAD ? grid : dim3(1, (unsigned)a.rows), 256, 0, stream>>>(a);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)a.rows);
  if (a.vocab <= 512)
    distill_row_kernel<T, ONE, 64, ONE ? 1 : 0, GRAD><<<grid, 64, 0, stream>>>(a);
  else if (a.vocab <= 8192)
    distill_row_kernel<T, ONE, 256, ONE ? 4 : 0, GRAD><<<grid, 256, 0, stream>>>(a);
  else if (a.vocab <= 32768)
    distill_row_kernel<T, ONE, 512, ONE ? 8 : 0, GRAD><<<grid, 512, 0, stream>>>(a);
  else
    distill_row_kernel<T, ONE, 1024, 0, GRAD><<<grid, 1024, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, bool ONE>
hipError_t backward(const DistillArgs &a, hipStream_t stream) {
  // the grid's second dimension holds 65535 rows a launch
  DistillArgs b = a;
  for (int64_t r = 0; r < a.rows; r += 65535) {
    b.rows = a.rows - r < 65535 ? a.rows - r : 65535;
    b.z = (const T *)a.z + r * a.vocab;
    b.dz = (T *)a.dz + r * a.vocab;
    b.t = (const T *)a.t + r * a.k;
    b.ids = a.ids + r * a.k;
    b.stats_in = a.stats_in + 2 * r;
    b.g = a.g ? a.g + r : nullptr;
    distill_finish_kernel<T, ONE, true>
        <<<dim3((unsigned)a.chunks, (unsigned)b.rows), 256, 0, stream>>>(b);
  }
  return hipGetLastError();
}

template <typename T, bool ONE>
hipError_t run(const DistillArgs &a, hipStream_t stream) {
  if (a.stats_in) return backward<T, ONE>(a, stream);
  return a.dz ? forward<T, ONE, true>(a, stream) : forward<T, ONE, false>(a, stream);
}

}  // namespace

int64_t distill_workspace_bytes(int64_t rows, int64_t vocab) {
  return several(rows, vocab) ? rows * ((vocab + CHUNK - 1) / CHUNK) * (int64_t)sizeof(f32x2) : 0;
}

hipError_t launch_distill(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                          const void *t, double temperature, const void *stats_in, const void *g, void *ws, void *loss,
                          void *stats, void *dz, hipStream_t stream) {
  DistillArgs a;
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
  if (dtype == LM_F16) return nc == 1 ? run<_Float16, true>(a, stream) : run<_Float16, false>(a, stream);
  if (dtype == LM_BF16) return nc == 1 ? run<__bf16, true>(a, stream) : run<__bf16, false>(a, stream);
  return nc == 1 ? run<float, true>(a, stream) : run<float, false>(a, stream);
}

}  // namespace mcf
