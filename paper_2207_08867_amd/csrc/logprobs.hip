// logprobs.hip -- log probabilities of given tokens, with the entropy and the most likely alternatives of
// every row of logits, and their gradient.
//
// A row has logits z_j, j < V (plain, or an MC value whose planes are summed in binary32, the last plane
// first).  With m the largest logit, d_j = m - z_j and s = sum exp(-d_j / T) over all but one logit equal to m,
//   L = log(1 + s),  log q_j = -d_j / T - L,  B = sum d_j exp(-d_j / T) / (T (1 + s)),  entropy H = L + B.
// The largest logit is kept apart so that L, and with it the log probability of a token the model is
// sure of, holds its relative accuracy; L and B are sums of numbers that are not negative.  The
// alternatives are the first k logits in the order (z descending, j ascending).
// The gradient, given g_i with respect to the log probability of token id_i and h with respect to H:
//   dz_j = (sum of the g_i with id_i = j - q_j (sum of all g_i + h (log q_j + H))) / T.
//
// Sums are binary32, in an order that depends on the sizes alone.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace mcf {
namespace {

// What a part of a row contributes: its largest logit, at least -FLT_MAX; s as above, or -1 where the
// part has no logit above -inf; a = sum d exp(-d / T).
struct Part {
  float m, s, a;
};

struct LogpArgs {
  const void *z;
  const int32_t *ids;
  float *logp, *entropy, *top_logp, *stats_out;
  int32_t *top_ids;
  Part *parts;     // [rows][chunks], where a row is several workgroups'
  uint64_t *keys;  // [rows][chunks][top]
  const float *stats, *g, *gh;
  void *dz;
  int64_t rows, plane;
  int64_t first;  // the launch's first row
  int vocab, given, top, nc, chunks;
  float temperature, inv_t, c_hi, c_lo;  // c_hi + c_lo = log2(e) / T
};

// exp(-d / T), d >= 0.  The factor's second term keeps the argument's error at one rounding; both are
// positive, so that an infinite d gives 0.
__device__ inline float expd(const LogpArgs &a, float d) {
  return __builtin_amdgcn_exp2f(-fmaf(d, a.c_hi, d * a.c_lo));
}

__device__ inline Part join(const LogpArgs &a, const Part &x, const Part &y) {
  const bool first = x.m >= y.m;
  const Part &hi = first ? x : y, &lo = first ? y : x;
  if (lo.s == -1.0f) return hi.s == -1.0f ? lo : hi;
  if (hi.s == -1.0f) return lo;
  const float d = hi.m - lo.m, f = expd(a, d), n = 1.0f + lo.s;
  return Part{hi.m, hi.s + n * f, hi.a + (lo.a + (f == 0.0f ? 0.0f : d) * n) * f};
}

// A logit's place in the order as one number: larger means earlier; 0 stands for none.
__device__ inline uint64_t key_of(float v, uint32_t j) {
  if (!(v > -INFINITY)) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);  // -0 is +0
  return (uint64_t)(u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (uint32_t)~j;
}
__device__ inline float key_value(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, u ^ ((int32_t)u < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ inline int32_t key_index(uint64_t k) { return (int32_t)~(uint32_t)k; }

__device__ inline uint64_t max64(uint64_t x, uint64_t y) { return x > y ? x : y; }
__device__ inline uint64_t shfl64(uint64_t v, int d) { return (uint64_t)__shfl_xor((unsigned long long)v, d); }

constexpr int GROUPS = 256;  // of the threads, for the alternatives; above LOGP_TOP
constexpr int KEEP = 1024;   // candidates

struct Select {
  uint64_t group[GROUPS];
  uint64_t kept[KEEP];
  uint64_t bound;
  int rank[GROUPS];
  int n;
};

// The k largest of the workgroup's keys, which are all different (but for 0).  each(f) calls f on every key of
// the thread, own is its largest.  The k-th largest of 256 groups' largest keys bounds the k-th largest
// key from below; the keys at or above it, k and a few more as a rule, are ranked by counting.
// out(r, key) takes the r-th largest, 0 where there is none.
template <int NT, typename Each, typename Out>
__device__ inline void select_top(Select &sh, int k, uint64_t own, Each each, Out out) {
  constexpr int PER = NT / GROUPS;
  static_assert(PER >= 1 && NT % GROUPS == 0 && GROUPS > LOGP_TOP, "a group has whole threads");
  const int t = threadIdx.x;
  uint64_t big = own;
#pragma unroll
  for (int d = 1; d < PER; d <<= 1) big = max64(big, shfl64(big, d));
  if (t % PER == 0) sh.group[t / PER] = big, sh.rank[t / PER] = 0;
  if (t == 0) sh.bound = 1, sh.n = 0;
  __syncthreads();
  {
    const uint64_t mine = sh.group[t % GROUPS];
    const int from = t / GROUPS * (GROUPS / PER);
    int above = 0;
#pragma unroll 16
    for (int j = 0; j < GROUPS / PER; ++j) above += sh.group[from + j] > mine;
    atomicAdd(&sh.rank[t % GROUPS], above);
  }
  __syncthreads();
  if (t < GROUPS && sh.rank[t] == k - 1 && sh.group[t] != 0) sh.bound = sh.group[t];
  __syncthreads();
  const uint64_t bound = sh.bound;
  if (own >= bound)
    each([&](uint64_t key) {
      if (key >= bound) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < KEEP) sh.kept[at] = key;
      }
    });
  __syncthreads();
  const int n = sh.n;
  if (n <= KEEP) {
    for (int i = t; i < n; i += NT) {
      const uint64_t mine = sh.kept[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += sh.kept[j] > mine;
      if (above < k) out(above, mine);
    }
    for (int r = n + t; r < k; r += NT) out(r, (uint64_t)0);
    return;
  }
  // rows whose order follows the threads': one by one
  uint64_t last = ~(uint64_t)0;
  for (int r = 0; r < k; ++r) {
    uint64_t best = 0;
    if (own < last) best = own;
    else
      each([&](uint64_t key) {
        if (key < last) best = max64(best, key);
      });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) best = max64(best, shfl64(best, d));
    __syncthreads();
    if ((t & 63) == 0) sh.group[t >> 6] = best;
    __syncthreads();
    best = sh.group[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) best = max64(best, sh.group[w]);
    if (t == 0) out(r, best);
    last = best;
  }
}

template <typename T, bool ONE>
__device__ inline float logit(const LogpArgs &a, const T *z, int64_t j) {
  if (ONE) return (float)z[j];
  float v = (float)z[(a.nc - 1) * a.plane + j];
  for (int p = a.nc - 2; p >= 0; --p) v += (float)z[p * a.plane + j];
  return v;
}

// Eight logits from column col of a row, as they are held: plain ones in their format.  Past the row
// they are -inf.
template <typename T, bool ONE>
__device__ inline Raw8<std::conditional_t<ONE, T, float>> logits8(const LogpArgs &a, const T *z, int64_t col) {
  using H = std::conditional_t<ONE, T, float>;
  const int64_t left = a.vocab - col;
  Raw8<H> r;
  if constexpr (ONE) {
    r = load8_tail(z + col, left);
  } else {
    for (int p = a.nc - 1; p >= 0; --p) {
      const Raw8<T> u = load8_tail(z + p * a.plane + col, left);
#pragma unroll
      for (int i = 0; i < 8; ++i) r.v[i] = p == a.nc - 1 ? (float)u.v[i] : r.v[i] + (float)u.v[i];
    }
  }
  if (left < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= left) r.v[i] = (H)-INFINITY;
  }
  return r;
}

// The numbers of a row from its part; every thread has them.
struct Row {
  float m, L, B;
  bool bad, none;
};
__device__ inline Row row_of(const LogpArgs &a, const Part &p) {
  Row r;
  r.none = p.s == -1.0f;
  r.bad = !(p.s < INFINITY) || p.m == INFINITY;
  r.m = r.bad ? NAN : (r.none ? -INFINITY : p.m);
  r.L = r.bad ? NAN : (r.none ? 0.0f : log1pf(p.s));
  r.B = r.bad ? NAN : (r.none ? 0.0f : p.a * a.inv_t / (1.0f + p.s));
  return r;
}
__device__ inline float log_prob(const LogpArgs &a, const Row &r, float z) {
  if (r.none) return -INFINITY;
  // binary64: the difference of a largest and a lowest number passes binary32's range, where its quotient
  // by the temperature need not
  return (float)(((double)z - (double)r.m) / (double)a.temperature - (double)r.L);
}

// A row's outputs but for the alternatives.
template <typename T, bool ONE, int NT>
__device__ inline void finish(const LogpArgs &a, int64_t row, const Row &r, const T *z) {
  for (int i = threadIdx.x; i < a.given; i += NT) {
    const int id = a.ids[row * a.given + i];
    a.logp[row * a.given + i] = id >= 0 && id < a.vocab ? log_prob(a, r, logit<T, ONE>(a, z, id)) : 0.0f;
  }
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[row] = r.L + r.B;
    if (a.stats_out) {
      a.stats_out[3 * row] = r.m;
      a.stats_out[3 * row + 1] = r.L;
      a.stats_out[3 * row + 2] = r.B;
    }
  }
}
__device__ inline void put_top(const LogpArgs &a, int64_t row, const Row &r, int i, uint64_t key) {
  const bool some = key != 0 && !r.bad;
  a.top_ids[row * a.top + i] = some ? key_index(key) : -1;
  a.top_logp[row * a.top + i] = some ? log_prob(a, r, key_value(key)) : (r.bad ? NAN : -INFINITY);
}

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ inline float wave_add(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// A chunk of NT CH pieces of 8 logits of a row, in registers; SPLIT: of several, which the kernel below joins.
template <typename T, bool ONE, int NT, int CH, bool TOP, bool SPLIT>
__global__ __launch_bounds__(NT) void logp_kernel(LogpArgs a) {
  using H = std::conditional_t<ONE, T, float>;
  constexpr int W = NT / 64;
  __shared__ float mx[W];
  __shared__ Part sums[W];
  __shared__ std::conditional_t<TOP, Select, int> sel;
  const int64_t row = SPLIT ? a.first + blockIdx.x / a.chunks : a.first + blockIdx.x;
  const int chunk = SPLIT ? blockIdx.x % a.chunks : 0, lo = chunk * (NT * CH * 8);
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  Raw8<H> v[CH];
  float own = -FLT_MAX;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = lo + (int64_t)(c * NT + (int)threadIdx.x) * 8;
    if (col < a.vocab) {
      v[c] = logits8<T, ONE>(a, z, col);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c].v[i] = (H)-INFINITY;
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) own = fmaxf(own, (float)v[c].v[i]);
  float m = wave_max(own);
  if ((threadIdx.x & 63) == 0) mx[threadIdx.x >> 6] = m;
  __syncthreads();
  m = mx[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, mx[w]);
  float s = 0.0f, d1 = 0.0f, equal = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = m - (float)v[c].v[i], e = expd(a, d);
      s += e;
      d1 += e * fminf(d, FLT_MAX);
    }
  if (own == m) {
    // a thread with a largest logit sums the others alone
    s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = (float)v[c].v[i];
        equal += x == m ? 1.0f : 0.0f;
        s += x == m ? 0.0f : expd(a, m - x);
      }
  }
  s = wave_add(s);
  d1 = wave_add(d1);
  equal = wave_add(equal);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = Part{equal, s, d1};
  __syncthreads();
  equal = sums[0].m, s = sums[0].s, d1 = sums[0].a;
#pragma unroll
  for (int w = 1; w < W; ++w) equal += sums[w].m, s += sums[w].s, d1 += sums[w].a;
  // no largest logit: nothing but -inf, or NaN, which s then is
  const Part part = {m, m == INFINITY ? NAN : (s + (equal - 1.0f)), d1};
  Row r;
  if constexpr (!SPLIT) {
    r = row_of(a, part);
    finish<T, ONE, NT>(a, row, r, z);
  } else if (threadIdx.x == 0) {
    a.parts[row * a.chunks + chunk] = part;
  }
  if constexpr (TOP) {
    const auto each = [&](auto f) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) f(key_of((float)v[c].v[i], lo + (c * NT + threadIdx.x) * 8 + i));
    };
    // the thread's first logit equal to its largest
    uint32_t at = 0;
#pragma unroll
    for (int c = CH - 1; c >= 0; --c)
#pragma unroll
      for (int i = 7; i >= 0; --i) at = (float)v[c].v[i] == own ? (c * NT * 8 + i) : at;
    uint64_t mine = key_of(own, lo + threadIdx.x * 8 + at);
    if (own == -FLT_MAX) {  // perhaps of no logit
      mine = 0;
      each([&](uint64_t key) { mine = max64(mine, key); });
    }
    select_top<NT>(sel, a.top, mine, each, [&](int i, uint64_t key) {
      if constexpr (SPLIT)
        a.keys[(row * a.chunks + chunk) * a.top + i] = key;
      else
        put_top(a, row, r, i, key);
    });
  }
}

// The chunks of a row.
template <typename T, bool ONE, bool TOP>
__global__ __launch_bounds__(256) void logp_join_kernel(LogpArgs a) {
  __shared__ Part sums[4];
  __shared__ std::conditional_t<TOP, Select, int> sel;
  const int64_t row = a.first + blockIdx.x;
  Part p = {-FLT_MAX, -1.0f, 0.0f};
  for (int c = threadIdx.x; c < a.chunks; c += 256) p = join(a, p, a.parts[row * a.chunks + c]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Part o = {__shfl_xor(p.m, d), __shfl_xor(p.s, d), __shfl_xor(p.a, d)};
    // both sides join in the lower lane's order, so the lanes agree
    p = (threadIdx.x & d) ? join(a, o, p) : join(a, p, o);
  }
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = p;
  __syncthreads();
  p = sums[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) p = join(a, p, sums[w]);
  const Row r = row_of(a, p);
  finish<T, ONE, 256>(a, row, r, reinterpret_cast<const T *>(a.z) + row * a.vocab);
  if constexpr (TOP) {
    const int64_t n = (int64_t)a.chunks * a.top;
    const uint64_t *keys = a.keys + row * n;
    const auto each = [&](auto f) {
      for (int64_t i = threadIdx.x; i < n; i += 256) f(keys[i]);
    };
    uint64_t mine = 0;
    each([&](uint64_t key) { mine = max64(mine, key); });
    select_top<256>(sel, a.top, mine, each, [&](int i, uint64_t key) { put_top(a, row, r, i, key); });
  }
}

// Chunks of a row: one while it fits, 32768 logits; rows of few, 4096 each.
constexpr int FEW = 4096, LONG = 32768;
int chunk_of(int64_t rows, int64_t vocab) {
  if (rows < 256 && vocab > 2 * FEW) return FEW;
  return vocab > LONG ? LONG : 0;
}

template <typename T, bool ONE, bool TOP>
hipError_t run_fwd(LogpArgs a, hipStream_t stream) {
  const int chunk = chunk_of(a.rows, a.vocab);
  const int64_t most = LAUNCH_MAX / a.chunks > 0 ? LAUNCH_MAX / a.chunks : 1;
  for (a.first = 0; a.first < a.rows; a.first += most) {
    const int64_t rows = a.rows - a.first < most ? a.rows - a.first : most;
    const unsigned grid = (unsigned)(rows * a.chunks);
#define ROW(NT, CH, SPLIT) logp_kernel<T, ONE, NT, CH, TOP, SPLIT><<<grid, NT, 0, stream>>>(a)
    if (chunk == FEW)
      ROW(256, 2, true);
    else if (chunk == LONG)
      ROW(512, 8, true);
    else if (a.vocab <= 2048)
      ROW(256, 1, false);
    else if (a.vocab <= 4096)
      ROW(256, 2, false);
    else if (a.vocab <= 8192)
      ROW(256, 4, false);
    else if (a.vocab <= 16384)
      ROW(512, 4, false);
    else
      ROW(512, 8, false);
#undef ROW
    if (chunk) logp_join_kernel<T, ONE, TOP><<<(unsigned)rows, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

// --- the gradient ----------------------------------------------------------------------

// The given tokens' ids and gradients, 8 bytes of LDS each.
extern __shared__ float given_space[];

// A workgroup takes 8 CH NT logits of a row.
template <typename T, bool ONE, int NT, int CH>
__global__ __launch_bounds__(NT) void logp_bwd_kernel(LogpArgs a) {
  int *const id = (int *)given_space;
  float *const g = given_space + a.given;
  const int64_t row = a.first + blockIdx.x / a.chunks;
  const int lo = (int)(blockIdx.x % a.chunks) * (NT * CH * 8);
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
  Raw8<std::conditional_t<ONE, T, float>> v[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = lo + (int64_t)(c * NT + (int)threadIdx.x) * 8;
    if (col < a.vocab) v[c] = logits8<T, ONE>(a, z, col);
  }
  for (int i = threadIdx.x; i < a.given; i += NT) {
    const int j = a.ids[row * a.given + i];
    const bool used = j >= 0 && j < a.vocab;
    id[i] = used ? j : -1;
    g[i] = used ? (a.g ? a.g[row * a.given + i] : 1.0f) : 0.0f;
  }
  const float m = a.stats[3 * row], L = a.stats[3 * row + 1], B = a.stats[3 * row + 2];
  const float gh = a.gh ? a.gh[row] : 0.0f;
  __syncthreads();
  float all = 0.0f;
  for (int i = 0; i < a.given; ++i) all += g[i];
  const bool none = m == -INFINITY;
  const float inv_s = expf(-L) * a.inv_t;
  const auto grad = [&](float x) {
    const float d = m - x, q = expd(a, d) * inv_s;
    return q == 0.0f ? 0.0f : -q * (all + gh * (B - d * a.inv_t));
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = lo + (int64_t)(c * NT + (int)threadIdx.x) * 8;
    if (col >= a.vocab) break;
    Raw8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = none ? (T)0.0f : (T)grad((float)v[c].v[i]);
    store8_tail(dz + col, o, a.vocab - col);
  }
  if (none) return;
  __syncthreads();  // the pass's stores come before the tokens'
  const int hi = lo + NT * CH * 8;
  for (int i = threadIdx.x; i < a.given; i += NT) {
    const int j = id[i];
    if (j < lo || j >= hi) continue;
    // equal ids write the same sum
    float sum = 0.0f;
    for (int k = 0; k < a.given; ++k) sum += id[k] == j ? g[k] : 0.0f;
    dz[j] = (T)(sum * a.inv_t + grad(logit<T, ONE>(a, z, j)));
  }
}

template <typename T, bool ONE>
hipError_t run_bwd(LogpArgs a, hipStream_t stream) {
  const bool small = a.vocab <= 512;
  const int per = small ? 512 : 8192;
  a.chunks = (a.vocab + per - 1) / per;
  const int64_t most = LAUNCH_MAX / a.chunks > 0 ? LAUNCH_MAX / a.chunks : 1;
  for (a.first = 0; a.first < a.rows; a.first += most) {
    const int64_t rows = a.rows - a.first < most ? a.rows - a.first : most;
    const unsigned grid = (unsigned)(rows * a.chunks);
    if (small)
      logp_bwd_kernel<T, ONE, 64, 1><<<grid, 64, 8 * a.given, stream>>>(a);
    else
      logp_bwd_kernel<T, ONE, 256, 4><<<grid, 256, 8 * a.given, stream>>>(a);
  }
  return hipGetLastError();
}

LogpArgs args_of(int nc, int64_t rows, int64_t vocab, int64_t given, const void *z, const void *ids, double temperature) {
  LogpArgs a = {};
  a.z = z;
  a.ids = (const int32_t *)ids;
  a.rows = rows;
  a.plane = rows * vocab;
  a.vocab = (int)vocab;
  a.given = (int)given;
  a.nc = nc;
  a.temperature = (float)temperature;
  a.inv_t = 1.0f / a.temperature;
  const double c = 1.4426950408889634 / (double)a.temperature;
  a.c_hi = (float)c;
  if ((double)a.c_hi > c) a.c_hi = nextafterf(a.c_hi, 0.0f);
  a.c_lo = fmaxf((float)(c - (double)a.c_hi), FLT_MIN);
  return a;
}

int64_t parts_bytes(int64_t parts) { return (parts * (int64_t)sizeof(Part) + 15) / 16 * 16; }

}  // namespace

int64_t logprobs_workspace_bytes(int64_t rows, int64_t vocab, int64_t top) {
  const int chunk = chunk_of(rows, vocab);
  if (!chunk) return 0;
  const int64_t parts = rows * ((vocab + chunk - 1) / chunk);
  return parts_bytes(parts) + parts * top * 8;
}

hipError_t launch_logprobs_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, int64_t top, const void *z,
                               const void *ids, double temperature, void *ws, void *logp, void *entropy, void *top_ids,
                               void *top_logp, void *stats, hipStream_t stream) {
  LogpArgs a = args_of(nc, rows, vocab, given, z, ids, temperature);
  const int chunk = chunk_of(rows, vocab);
  a.chunks = chunk ? (int)((vocab + chunk - 1) / chunk) : 1;
  a.top = (int)top;
  a.parts = (Part *)ws;
  a.keys = (uint64_t *)((char *)ws + parts_bytes(rows * a.chunks));
  a.logp = (float *)logp;
  a.entropy = (float *)entropy;
  a.top_ids = (int32_t *)top_ids;
  a.top_logp = (float *)top_logp;
  a.stats_out = (float *)stats;
  const auto go = [&](auto zero) {
    using T = decltype(zero);
    if (nc == 1) return top > 0 ? run_fwd<T, true, true>(a, stream) : run_fwd<T, true, false>(a, stream);
    return top > 0 ? run_fwd<T, false, true>(a, stream) : run_fwd<T, false, false>(a, stream);
  };
  if (dtype == LM_F16) return go((_Float16)0.0f);
  if (dtype == LM_BF16) return go((__bf16)0.0f);
  return go(0.0f);
}

hipError_t launch_logprobs_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, const void *z,
                               const void *ids, double temperature, const void *stats, const void *g,
                               const void *g_entropy, void *dz, hipStream_t stream) {
  LogpArgs a = args_of(nc, rows, vocab, given, z, ids, temperature);
  a.stats = (const float *)stats;
  a.g = (const float *)g;
  a.gh = (const float *)g_entropy;
  a.dz = dz;
  const auto go = [&](auto zero) {
    using T = decltype(zero);
    return nc == 1 ? run_bwd<T, true>(a, stream) : run_bwd<T, false>(a, stream);
  };
  if (dtype == LM_F16) return go((_Float16)0.0f);
  if (dtype == LM_BF16) return go((__bf16)0.0f);
  return go(0.0f);
}

}  // namespace mcf
