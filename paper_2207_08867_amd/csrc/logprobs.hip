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
// Sums are binary32, in an order that depends on the sizes (rows and vocabulary) alone.  From a temperature of 2^64 up
// differences are taken of logits times 2^-64, with T 2^-64 in T's place, so that neither a difference of the format's
// whole range nor a row's sum of them passes binary32's range; what that rounds away is below 2^-126 of T.  The kernels
// of MC logits alone do so, and take plain rows then too, of one plane: in the others it cost bfloat16 rows 1 to 2% of
// a call.
//
// A row is read once, and the gradient reads it again and writes as much, so HBM bounds the large calls: 4096 rows of
// 32768 bfloat16 logits (268 MB) 54 to 61 us, 4.4 to 5.0 TB/s, the gradient 108 us, 5.0 TB/s; binary32 97 and 195 us,
// 5.5 TB/s.  The alternatives are found where the row is held: 66 us with 20, 73 with 64, 123 with 128.
// Calls of few rows are launches and waits: one row of 131071 binary32 logits 7.4 us, 13.8 with 20 alternatives.  Two
// planes: 2048 rows of 32768 binary16 70 us, 90 with 20 alternatives, the gradient 89, 4.5 TB/s; of binary32 98, 117
// and 150.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "mcf_internal.hpp"
#include "mx4.hpp"
#include "wave.hpp"

namespace mcf {
namespace {

// What a part of a row contributes: its largest logit, at least -FLT_MAX; s as above, or -1 where the
// part has no logit above -inf; a = sum d exp(-d / T), of scaled differences.
struct Part {
  float m, s, a;
};

struct LogpArgs {
  const void *z;
  const int32_t *ids;
  float *logp, *entropy, *top_logp, *stats_out;
  int32_t *top_ids;
  Part *parts;     // [rows][chunks], where a row is several workgroups'
  uint64_t *keys;  // [rows][top][chunks]: the chunks' largest keys first, which so fall to different threads
  const float *stats, *g, *gh;
  void *dz;
  int64_t rows, plane;
  int64_t first;  // the launch's first row
  int vocab, given, top, nc, chunks;
  float temperature, scale;  // T; what differences are scaled by, 1 or 2^-64
  float inv_t, c_hi, c_lo;   // 1 / (T scale); c_hi + c_lo = log2(e) / (T scale)
};

// The scaled difference of a larger logit m, given as `scaled`, and a smaller one; the scale is a power of two, so that
// it is rounded once.  ONE: the scale is 1.
template <bool ONE>
__device__ inline float scaled(const LogpArgs &a, float v) {
  return ONE ? v : v * a.scale;
}
template <bool ONE>
__device__ inline float below(const LogpArgs &a, float m_scaled, float z) {
  return ONE ? m_scaled - z : fmaf(-a.scale, z, m_scaled);
}

// exp(-d / T) of a scaled d >= 0.  The factor's second term keeps the argument's error at one rounding; both are
// positive, so that an infinite d gives 0.
__device__ inline float expd(const LogpArgs &a, float d) {
  return __builtin_amdgcn_exp2f(-fmaf(d, a.c_hi, d * a.c_lo));
}

template <bool ONE>
__device__ inline Part join(const LogpArgs &a, const Part &x, const Part &y) {
  // member by member: a reference to one or the other would put both into memory
  const bool first = x.m >= y.m;
  const Part hi = {first ? x.m : y.m, first ? x.s : y.s, first ? x.a : y.a};
  const Part lo = {first ? y.m : x.m, first ? y.s : x.s, first ? y.a : x.a};
  if (lo.s == -1.0f) return hi.s == -1.0f ? lo : hi;
  if (hi.s == -1.0f) return lo;
  const float d = below<ONE>(a, scaled<ONE>(a, hi.m), lo.m), f = expd(a, d), n = 1.0f + lo.s;
  return Part{hi.m, hi.s + n * f, hi.a + (lo.a + (f == 0.0f ? 0.0f : d) * n) * f};
}

// Logits in the order of integers, and back.
__device__ inline uint32_t ordered(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);  // -0 is +0
  return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ inline float ordered_value(uint32_t u) {
  return __builtin_bit_cast(float, u ^ ((int32_t)u < 0 ? 0x80000000u : 0xffffffffu));
}
// A logit's place in the order of the alternatives as one number: larger means earlier; 0 stands for none.
__device__ inline uint64_t key_of(float v, uint32_t j) { return (uint64_t)ordered(v) << 32 | (uint32_t)~j; }
__device__ inline float key_value(uint64_t k) { return ordered_value((uint32_t)(k >> 32)); }
__device__ inline int32_t key_index(uint64_t k) { return (int32_t)~(uint32_t)k; }

constexpr int GROUPS = 256;  // of the threads, for the alternatives; above LOGP_TOP
constexpr int KEEP = 1024;   // candidates
constexpr int RANKS = 256;   // candidates that are ranked, above LOGP_TOP + LOGP_TOP / 8

struct Select {
  union {
    uint64_t group[GROUPS];      // of keys
    uint32_t logit[2 * GROUPS];  // the threads' largest logits, of which threads GROUPS apart are a group
    int rank[RANKS];  // once the groups are done with
  };
  uint64_t kept[KEEP];
  uint64_t bound;
  int n, slots, wave[16];
};

// The largest b of the form "some leading bits, then zeros" that at least k numbers reach, 0 where fewer
// are there.  count(b) tells how many reach b.  It ends as soon as the numbers that reach b are few.
template <typename U, typename Count>
__device__ inline U bound_of(int k, int few, Count count) {
  U b = 0;
#pragma unroll 1
  for (U bit = (U)1 << (8 * sizeof(U) - 1); bit; bit >>= 1) {
    const int n = count(b | bit);
    if (n < k) continue;
    b |= bit;
    if (n <= few) break;
  }
  return b;
}

// The same of the 256 groups' numbers, in sh.group or sh.logit, by one wavefront, for all.
template <int NT, typename U>
__device__ inline U bound_of_groups(Select &sh, int k) {
  __syncthreads();
  if (threadIdx.x < 64) {
    U g[GROUPS / 64];
#pragma unroll
    for (int i = 0; i < GROUPS / 64; ++i) {
      const int at = threadIdx.x + 64 * i;
      if constexpr (sizeof(U) == 8) {
        g[i] = sh.group[at];
      } else {
        g[i] = sh.logit[at];
        if (NT > GROUPS) g[i] = sh.logit[at + GROUPS] > g[i] ? sh.logit[at + GROUPS] : g[i];
      }
    }
    const U b = bound_of<U>(k, k + k / 8, [&](U b) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < GROUPS / 64; ++i) n += __popcll(__ballot(g[i] >= b));
      return n;
    });
    if (threadIdx.x == 0) sh.bound = b, sh.n = 0, sh.slots = 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < RANKS; i += NT) sh.rank[i] = 0;
  return (U)sh.bound;
}

// The sum of the workgroup's wavefronts' numbers.
template <int NT>
__device__ inline int waves_sum(Select &sh, int n) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) n += sh.wave[w];
  return n;
}

// out(r, key) takes the r-th largest of the n <= KEEP kept keys, r < k, and 0 where there is none: ranks by
// counting, each wavefront a part of the comparisons.  They grow with n^2, so that many keys are cut down to little
// more than k first (1000 candidates for 128 places, 8192 rows: 905 us ranked as they are, 91 us so).
template <int NT, typename Out>
__device__ inline void rank_kept(Select &sh, int k, int n, Out out) {
  static_assert(RANKS >= LOGP_TOP + LOGP_TOP / 8 && KEEP % NT == 0, "what is cut down is ranked");
  constexpr int W = NT / 64, PER = KEEP / NT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (n > RANKS) {
    uint64_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = (int)threadIdx.x + i * NT < n ? sh.kept[threadIdx.x + i * NT] : 0;
    const uint64_t bound = bound_of<uint64_t>(k, k + k / 8, [&](uint64_t b) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) c += __popcll(__ballot(key[i] >= b));
      return waves_sum<NT>(sh, c);
    });
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (key[i] >= bound) sh.kept[atomicAdd(&sh.n, 1)] = key[i];
    __syncthreads();
    n = sh.n;
  }
  const int from = n * wave / W, to = n * (wave + 1) / W;
  for (int i = lane; i < n; i += 64) {
    const uint64_t mine = sh.kept[i];
    int above = 0;
#pragma unroll 4
    for (int j = from; j < to; ++j) above += sh.kept[j] > mine;
    atomicAdd(&sh.rank[i], above);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT)
    if (sh.rank[i] < k) out(sh.rank[i], sh.kept[i]);
  for (int r = n + (int)threadIdx.x; r < k; r += NT) out(r, (uint64_t)0);
}

// The first keys of a thread, held in registers.
struct Held {
  static constexpr int N = 4;
  uint64_t key[N];
};

// The k largest of a list of keys, which are all different (but for 0): by a bound that at least k of 256
// groups' largest keys reach, which so bounds the k-th largest key from below.  More than KEEP keys at or
// above it: the same bisection over all keys.
template <int NT, typename Out>
__device__ inline void select_keys(Select &sh, int k, const uint64_t *keys, int64_t n, const Held &held, Out out) {
  static_assert(NT == GROUPS, "a group is a thread's keys");
  const auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < Held::N; ++i) f(held.key[i]);  // 0 past the list
    for (int64_t i = threadIdx.x + Held::N * NT; i < n; i += NT) f(keys[i]);
  };
  uint64_t own = 0;
  each([&](uint64_t key) { own = key > own ? key : own; });
  sh.group[threadIdx.x] = own;
  uint64_t bound = bound_of_groups<NT, uint64_t>(sh, k);
  int kept;
  for (int pass = 0;; ++pass) {
    if (bound == 0) bound = 1;
    if (own >= bound)
      each([&](uint64_t key) {
        if (key < bound) return;
        const int at = atomicAdd(&sh.n, 1);
        if (at < KEEP) sh.kept[at] = key;
      });
    __syncthreads();
    kept = sh.n;
    if (kept <= KEEP || pass == 1) break;
    bound = bound_of<uint64_t>(k, KEEP, [&](uint64_t b) {
      uint32_t c = 0;
      each([&](uint64_t key) { c += key >= b; });
      return waves_sum<NT>(sh, (int)lanes_sum(c));
    });
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
  }
  rank_kept<NT>(sh, k, kept, out);
}

template <typename T, bool ONE>
__device__ inline float logit(const LogpArgs &a, const T *z, int64_t j) {
  if (ONE) return (float)z[j];
  float v = (float)z[(a.nc - 1) * a.plane + j];
  for (int p = a.nc - 2; p >= 0; --p) v += (float)z[p * a.plane + j];
  return v;
}

// CH pieces of 8 logits of a row, piece c from column lo + 8 (c NT + t) of thread t, as they are held: plain ones in
// their format.  Past the row they are -inf.
template <typename T, bool ONE, int NT, int CH>
__device__ inline void logits(const LogpArgs &a, const T *z, int lo, Raw8<std::conditional_t<ONE, T, float>> (&v)[CH]) {
  using H = std::conditional_t<ONE, T, float>;
  const auto column = [&](int c) { return lo + (c * NT + (int)threadIdx.x) * 8; };
  const bool tiny = CH == 1 && a.vocab < 8;  // which takes the smallest kernels
  const auto plane = [&](const T *p, int c) {
    if (!tiny) return load8_clamped(p, column(c), a.vocab);
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = column(c) + i < a.vocab ? p[column(c) + i] : (T)-INFINITY;
    return r;
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (ONE) {
      v[c] = plane(z, c);
    } else {
      for (int p = a.nc - 1; p >= 0; --p) {
        const Raw8<T> u = plane(z + p * a.plane, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c].v[i] = p == a.nc - 1 ? (float)u.v[i] : v[c].v[i] + (float)u.v[i];
      }
    }
  }
  if (tiny) return;
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (lo + (c + 1) * (NT * 8) > a.vocab) load8_settle(v[c], (int64_t)(a.vocab - column(c)), (H)-INFINITY);
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
  const float d = z - r.m;
  if (d != -INFINITY) return d / a.temperature - r.L;
  // the difference of a largest and a lowest number passes binary32's range, where its quotient by the
  // temperature need not
  return (float)(((double)z - (double)r.m) / (double)a.temperature - (double)r.L);
}

// A row's outputs but for the alternatives, by NT threads of which this is the t-th; the given tokens from `from` on.
template <typename T, bool ONE, int NT>
__device__ inline void finish(const LogpArgs &a, int64_t row, const Row &r, const T *z, int from, int t) {
  for (int i = from + t; i < a.given; i += NT) {
    const int id = a.ids[row * a.given + i];
    a.logp[row * a.given + i] = id >= 0 && id < a.vocab ? log_prob(a, r, logit<T, ONE>(a, z, id)) : 0.0f;
  }
  if (t == 0) {
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

// Threads whose logits go through LDS, 16 bytes a plain 16-bit piece.
constexpr int POOL = 152;
template <int CH, typename H>
struct Pool {
  Raw8<H> piece[POOL][CH];
  uint16_t owner[POOL];
};

// The k largest of the workgroup's logits by (logit, index), those of -inf apart, where they are held: v, and the
// thread's largest, own; first: the index of thread 0's first.  A bound that at least k of 256
// groups' largest logits reach bounds the k-th largest logit from below.  The threads with a logit that reaches it, k
// and a few more as a rule, hand theirs to the workgroup, which looks through them and ranks those that reach it.  Where
// they are more than the pool takes, for about 100 alternatives and up, each reads its logits again and looks through
// them by itself.  again(c) reads the thread's piece c once more.
template <int NT, int CH, typename H, typename Again, typename Out>
__device__ inline void select_logits(Select &sh, Pool<CH, H> &pool, int k, const Raw8<H> (&v)[CH], float own,
                                     uint32_t first, Again again, Out out) {
  static_assert((NT == GROUPS || NT == 2 * GROUPS) && GROUPS > LOGP_TOP, "a group has one or two threads");
  sh.logit[threadIdx.x] = ordered(own);
  const uint32_t b = bound_of_groups<NT, uint32_t>(sh, k);
  const uint32_t lowest = ordered(-FLT_MAX);
  float bound = ordered_value(b < lowest ? lowest : b);
  if (own >= bound) {
    const int at = atomicAdd(&sh.slots, 1);
    if (at < POOL) {
      pool.owner[at] = (uint16_t)threadIdx.x;
#pragma unroll
      for (int c = 0; c < CH; ++c) pool.piece[at][c] = v[c];
    }
  }
  const auto keep = [&](const Raw8<H> &u, uint32_t j) {
    uint32_t mask = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) mask |= (float)u.v[e] >= bound ? 1u << e : 0u;
    if (mask == 0) return;
    int at = atomicAdd(&sh.n, __popc(mask));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (mask >> e & 1) {
        if (at < KEEP) sh.kept[at] = key_of((float)u.v[e], j + e);
        ++at;
      }
  };
  __syncthreads();
  const int slots = sh.slots;
  if (slots <= POOL) {
    for (int i = threadIdx.x; i < slots * CH; i += NT)
      keep(pool.piece[0][i], first + (i % CH * NT + pool.owner[i / CH]) * 8);
  } else if (own >= bound) {
#pragma unroll 1
    for (int c = 0; c < CH; ++c) keep(again(c), first + (c * NT + threadIdx.x) * 8);
  }
  __syncthreads();
  int n = sh.n;
  if (n > KEEP) {
    // Many equal logits at the bound, or a row whose order follows the threads'.  The k-th largest logit is the bound if
    // fewer than k are larger, as a rule where many are equal, or comes of a bisection over all of them; then the
    // larger ones, fewer than k, and the first of those equal to it.  The row is read again, up to 36 times, so
    // that it need not stay in registers behind the rest.
    const uint32_t mine0 = first + threadIdx.x * 8;
    const auto count = [&](auto test) {
      int n = 0;
#pragma unroll 1
      for (int c = 0; c < CH; ++c) {
        const Raw8<H> u = again(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) n += __popcll(__ballot(test((float)u.v[i])));
      }
      return n;
    };
    if (waves_sum<NT>(sh, count([&](float x) { return x > bound; })) >= k) {
      const uint32_t e = bound_of<uint32_t>(k, k, [&](uint32_t b) {
        const float least = ordered_value(b < lowest ? lowest : b);
        return waves_sum<NT>(sh, count([&](float x) { return x >= least; }));
      });
      bound = ordered_value(e < lowest ? lowest : e);
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
#pragma unroll 1
    for (int c = 0; c < CH; ++c) {
      const Raw8<H> u = again(c);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((float)u.v[i] > bound) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < KEEP) sh.kept[at] = key_of((float)u.v[i], mine0 + c * NT * 8 + i);
        }
    }
    __syncthreads();
    n = sh.n;
    if (n < k) {
      int need = k - n;
#pragma unroll 1
      for (int c = 0; c < CH; ++c) {
        const Raw8<H> u = again(c);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) mine += (float)u.v[i] == bound;
        // the equal ones of the lanes before this one, and of the wavefronts before this one
        int before = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int o = __shfl_up(before, d);
          before += (int)(threadIdx.x & 63) >= d ? o : 0;
        }
        const int all = waves_sum<NT>(sh, __shfl(before, 63));
        before -= mine;
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += sh.wave[w];
        uint32_t j = mine0 + c * NT * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i, ++j)
          if ((float)u.v[i] == bound && before < need) sh.kept[k - need + before++] = key_of(bound, j);
        need -= all;
        if (need <= 0) break;
      }
      n = k - (need > 0 ? need : 0);
      __syncthreads();
    }
  }
  rank_kept<NT>(sh, k, n, out);
}

// A value that all lanes have, in a scalar register: the scaled one takes the vector register (80 in place of 81 of MC
// rows in eight pieces, which is a workgroup more on a CU: 2048 x 32000 of two binary16 planes 72 us, 76 without).
__device__ inline float scalar(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// A chunk of NT CH pieces of 8 logits of a row, in registers; SPLIT: of several, which the kernel below joins.
// 16-bit logits stay in their format, so that four workgroups of 512 threads and 32768 logits share a CU and some
// load while others sum or select; in binary32 they are half as many.
//
// What bounds it: vector instructions beside HBM (4096 x 32768 bfloat16, 56 us: 13 a logit, 84% of the cycles; with
// alternatives 86%), for short rows and many alternatives the selection's barriers.
// Earlier forms (4096 x 32768 bfloat16, us): logits held in binary32 164, the workgroup's maximum before any sum 77,
// now 54 to 61; with 64 alternatives, each thread looking through its own logits 100, now 73.
template <typename T, bool ONE, int NT, int CH, bool TOP, bool SPLIT, int OCC>
__global__ __launch_bounds__(NT, OCC) void logp_kernel(LogpArgs a) {
  using H = std::conditional_t<ONE, T, float>;
  constexpr int W = NT / 64;
  __shared__ Part sums[W];
  __shared__ std::conditional_t<TOP, Row, int> result;
  __shared__ std::conditional_t<TOP, Pool<CH, H>, int> pool;
  __shared__ std::conditional_t<TOP, Select, int> sel;
  const int64_t row = SPLIT ? a.first + blockIdx.x / a.chunks : a.first + blockIdx.x;
  const int chunk = SPLIT ? blockIdx.x % a.chunks : 0, lo = chunk * (NT * CH * 8);
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  // the first given tokens, each wavefront's lane one: asked for ahead of the row
  const int lane = threadIdx.x & 63;
  int id = -1;
  if (!SPLIT && lane < a.given) id = a.ids[row * a.given + lane];
  Raw8<H> v[CH];
  logits<T, ONE, NT>(a, z, lo, v);
  float given = 0.0f;
  if (id >= 0 && id < a.vocab) given = logit<T, ONE>(a, z, id);
  float own = -INFINITY;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) own = fmaxf(own, (float)v[c].v[i]);
  // Each wavefront's sums relative to its own largest logit, so that it works on its logits while the others'
  // are on their way.
  const float top = lanes_max(fmaxf(own, -FLT_MAX)), mw = ONE ? top : scalar(top), mws = scaled<ONE>(a, mw);
  float s = 0.0f, d1 = 0.0f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const Raw8<H> u = renewed(v[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = below<ONE>(a, mws, (float)u.v[i]), e = expd(a, d);
      s += e;
      d1 = fmaf(e, fminf(d, FLT_MAX), d1);
    }
    // here, or the compiler keeps d and e of every element for a later sum
    asm volatile("" : "+v"(s), "+v"(d1));
  }
  const float sw = lanes_sum(s), aw = lanes_sum(d1);
  if (lane == 0) sums[threadIdx.x >> 6] = Part{mw, sw, aw};
  __syncthreads();
  float m = sums[0].m;
  int first = 0;
#pragma unroll
  for (int w = 1; w < W; ++w)
    if (sums[w].m > m) m = sums[w].m, first = w;
  // The first wavefront with the row's largest logit finishes.  It sums its others alone; one more largest logit
  // elsewhere makes the sum 1 or more, which then needs no such care.
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) == __builtin_amdgcn_readfirstlane(first)) {
    const float ms = scaled<ONE>(a, m);
    float equal = 0.0f;
    s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const Raw8<H> u = renewed(v[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = (float)u.v[i];
        equal += x == m ? 1.0f : 0.0f;
        s += x == m ? 0.0f : expd(a, below<ONE>(a, ms, x));
      }
      asm volatile("" : "+v"(s), "+v"(equal));
    }
    s = lanes_sum(s);
    equal = lanes_sum(equal);
    Part part = {m, s, aw};
    // no largest logit: nothing but -inf, or NaN, which s then is
    float more = equal - 1.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const Part x = sums[w];
      const float d = below<ONE>(a, ms, x.m), f = w == first ? 0.0f : expd(a, d);
      part.s += w == first ? 0.0f : x.s * f;
      part.a += w == first ? 0.0f : (x.a + (f == 0.0f ? 0.0f : d) * x.s) * f;
    }
    part.s += more;
    if (m == INFINITY) part.s = NAN;
    if constexpr (SPLIT) {
      if (lane == 0) a.parts[row * a.chunks + chunk] = part;
    } else {
      const Row r = row_of(a, part);
      if constexpr (TOP)
        if (lane == 0) result = r;
      if (lane < a.given) a.logp[row * a.given + lane] = id >= 0 && id < a.vocab ? log_prob(a, r, given) : 0.0f;
      finish<T, ONE, 64>(a, row, r, z, 64, lane);
    }
  }
  if constexpr (TOP) {
    const auto again = [&](int c) {
      Raw8<H> u[1];
      logits<T, ONE, NT>(a, z, lo + c * NT * 8, u);
      return u[0];
    };
    select_logits<NT, CH>(sel, pool, a.top, v, own, lo, again, [&](int i, uint64_t key) {
      if constexpr (SPLIT)
        a.keys[(row * a.top + i) * a.chunks + chunk] = key;
      else
        put_top(a, row, result, i, key);
    });
  }
}

// The chunks of a row.
template <typename T, bool ONE, bool TOP>
__global__ __launch_bounds__(256) void logp_join_kernel(LogpArgs a) {
  __shared__ Part sums[4];
  __shared__ std::conditional_t<TOP, Select, int> sel;
  const int64_t row = a.first + blockIdx.x;
  // what has to wait for nothing is asked for first
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  const int64_t n = (int64_t)a.chunks * a.top;
  const uint64_t *keys = a.keys + row * n;
  Held held = {};
  if constexpr (TOP)
#pragma unroll
    for (int i = 0; i < Held::N; ++i)
      if (threadIdx.x + i * 256 < n) held.key[i] = keys[threadIdx.x + i * 256];
  int id = -1;
  if ((int)threadIdx.x < a.given) id = a.ids[row * a.given + threadIdx.x];
  Part p = {-FLT_MAX, -1.0f, 0.0f};
  for (int c = threadIdx.x; c < a.chunks; c += 256) p = join<ONE>(a, p, a.parts[row * a.chunks + c]);
  float given = 0.0f;
  if (id >= 0 && id < a.vocab) given = logit<T, ONE>(a, z, id);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Part o = {__shfl_xor(p.m, d), __shfl_xor(p.s, d), __shfl_xor(p.a, d)};
    // both sides join in the lower lane's order, so the lanes agree
    const bool upper = threadIdx.x & d;
    p = join<ONE>(a, Part{upper ? o.m : p.m, upper ? o.s : p.s, upper ? o.a : p.a},
             Part{upper ? p.m : o.m, upper ? p.s : o.s, upper ? p.a : o.a});
  }
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = p;
  __syncthreads();
  p = sums[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) p = join<ONE>(a, p, sums[w]);
  const Row r = row_of(a, p);
  if ((int)threadIdx.x < a.given)
    a.logp[row * a.given + threadIdx.x] = id >= 0 && id < a.vocab ? log_prob(a, r, given) : 0.0f;
  finish<T, ONE, 256>(a, row, r, z, 256, threadIdx.x);
  if constexpr (TOP)
    select_keys<256>(sel, a.top, keys, n, held, [&](int i, uint64_t key) { put_top(a, row, r, i, key); });
}

// How a row is cut into chunks of `pieces` pieces of 8 logits for each of the threads.  A row is one workgroup's while
// it fits 8 pieces of 512 threads, else it is cut into chunks alike, or, where there would be few of them, of 4096
// logits.  The pieces follow the length, as lanes past a row's end cost as much as others (8184 x 8200 binary32 with 64
// alternatives in three pieces 97 us, in four 141).  One workgroup and chunks of 4096 (us, in a graph): 1 x 32000 with
// 20 alternatives 12.0 and 15.3, 128 x 32768 8.1 and 11.0; chunks of 32768 and of 4096: 1 x 131072 11.5 and 9.0, 64 x
// 131072 the same within 3%.
constexpr int MANY = 128;
struct Cut {
  int threads, pieces, chunks;
};
Cut cut_of(int64_t rows, int64_t vocab) {
  const auto up = [](int64_t n, int64_t d) { return (int)((n + d - 1) / d); };
  if (vocab > 32768 && rows * up(vocab, 32768) < MANY) return {256, 2, up(vocab, 4096)};
  if (vocab <= 8192) return {256, up(vocab, 2048), 1};
  const int chunks = up(vocab, 32768);
  return {512, up(up(vocab, chunks), 4096), chunks};
}

template <typename T, bool ONE, bool TOP>
hipError_t run_fwd(LogpArgs a, const Cut &cut, hipStream_t stream) {
  const int64_t most = LAUNCH_MAX / a.chunks > 0 ? LAUNCH_MAX / a.chunks : 1;
  for (a.first = 0; a.first < a.rows; a.first += most) {
    const int64_t rows = a.rows - a.first < most ? a.rows - a.first : most;
    const unsigned grid = (unsigned)(rows * a.chunks);
    constexpr bool SHORT = ONE && sizeof(T) == 2;
#define ROW(NT, CH, SPLIT, OCC) logp_kernel<T, ONE, NT, CH, TOP, SPLIT, OCC><<<grid, NT, 0, stream>>>(a)
    if (a.chunks > 1) {
      if (cut.threads == 256)
        ROW(256, 2, true, 8);
      else if (cut.pieces == 5)
        ROW(512, 5, true, SHORT ? 8 : 4);
      else if (cut.pieces == 6)
        ROW(512, 6, true, SHORT ? 8 : 4);
      else if (cut.pieces == 7)
        ROW(512, 7, true, SHORT ? 8 : 4);
      else
        ROW(512, 8, true, SHORT ? 8 : 4);
      logp_join_kernel<T, ONE, TOP><<<(unsigned)rows, 256, 0, stream>>>(a);
    } else if (cut.threads == 256) {
      if (cut.pieces == 1)
        ROW(256, 1, false, 8);
      else if (cut.pieces == 2)
        ROW(256, 2, false, 8);
      else if (cut.pieces == 3)
        ROW(256, 3, false, SHORT ? 8 : 6);
      else
        ROW(256, 4, false, SHORT ? 8 : (TOP ? 5 : 6));
    } else if (cut.pieces == 3) {
      ROW(512, 3, false, SHORT ? 8 : 6);
    } else if (cut.pieces == 4) {
      ROW(512, 4, false, SHORT ? 8 : 6);
    } else if (cut.pieces == 5) {
      ROW(512, 5, false, SHORT ? 8 : 4);
    } else if (cut.pieces == 6) {
      ROW(512, 6, false, SHORT ? 8 : 4);
    } else if (cut.pieces == 7) {
      ROW(512, 7, false, SHORT ? 8 : 4);
    } else {
      ROW(512, 8, false, SHORT ? 8 : 4);
    }
#undef ROW
  }
  return hipGetLastError();
}

// --- the gradient ----------------------------------------------------------------------

// The given tokens' ids and gradients, 8 bytes of LDS each.
struct Given {
  int id;
  float g;
};
extern __shared__ Given given_space[];

// A workgroup takes 8 CH NT logits of a row.  FEW: few given tokens, for which every piece of 8 logits looks;
// else they are written over what the pass left there.  HBM bounds it: 4096 x 32768 bfloat16 108 us, 5.0 TB/s, where a
// large copy reaches 5.1; from a few dozen tokens a row on, their search for equal ids, each through all: with 8 tokens
// 111 us, 64 122, 256 211, 1024 2170 (8192 x 1000 17, 23, 99, 1128).
template <typename T, bool ONE, int NT, int CH, bool FEW>
__global__ __launch_bounds__(NT) void logp_bwd_kernel(LogpArgs a) {
  Given *const given = given_space;
  const int64_t row = a.first + blockIdx.x / a.chunks;
  const int lo = (int)(blockIdx.x % a.chunks) * (NT * CH * 8);
  const T *z = reinterpret_cast<const T *>(a.z) + row * a.vocab;
  T *dz = reinterpret_cast<T *>(a.dz) + row * a.vocab;
  for (int i = threadIdx.x; i < a.given; i += NT) {
    const int j = a.ids[row * a.given + i];
    const bool used = j >= 0 && j < a.vocab;
    given[i] = Given{used ? j : -1, used ? (a.g ? a.g[row * a.given + i] : 1.0f) : 0.0f};
  }
  const float m = a.stats[3 * row], L = a.stats[3 * row + 1], B = a.stats[3 * row + 2];
  const float gh = a.gh ? a.gh[row] : 0.0f;
  Raw8<std::conditional_t<ONE, T, float>> v[CH];
  logits<T, ONE, NT>(a, z, lo, v);
  const bool whole = lo + NT * CH * 8 <= a.vocab;
  if constexpr (NT > 64)
    __syncthreads();
  else
    wave_sync();
  float all = 0.0f;
  for (int i = 0; i < a.given; ++i) all += given[i].g;
  const bool none = m == -INFINITY;
  // 1 / T goes to the weights below a temperature of 2^64 and to the upstream gradients from there up: neither
  // then passes binary32's range before the result does
  float inv_s = expf(-L);
  float slope = gh;
  if (ONE || a.scale == 1.0f)
    inv_s *= a.inv_t;
  else
    all = scaled<ONE>(a, all * a.inv_t), slope = scaled<ONE>(a, gh * a.inv_t);
  const float ms = scaled<ONE>(a, m);
  const auto grad = [&](float x) {
    const float d = below<ONE>(a, ms, x), q = expd(a, d) * inv_s;
    return q == 0.0f ? 0.0f : -q * (all + slope * (B - d * a.inv_t));
  };
  // The gradient at a given token j with logit x; equal ids add up.  A row is sure of one token at most: there it is
  // G_j (1 - q_j) - q_j (the others' sum) in place of G_j - q_j (all of them), and 1 - q_j comes from log q_j, which
  // keeps its relative accuracy.
  const auto token = [&](int j, float x) {
    const float d = below<ONE>(a, ms, x), e = d * a.inv_t, q = expd(a, d) * expf(-L);
    const bool sure = q > 0.5f;
    float own = 0.0f, others = 0.0f;
    if (__any(sure))
      for (int k = 0; k < a.given; ++k) {
        const Given t = given[k];
        own += t.id == j ? t.g : 0.0f;
        others += t.id == j ? 0.0f : t.g;
      }
    else
      for (int k = 0; k < a.given; ++k) own += given[k].id == j ? given[k].g : 0.0f;
    if (sure) return scaled<ONE>(a, (own * -expm1f(-e - L) - q * (others + gh * (B - e))) * a.inv_t);
    return grad(x) + scaled<ONE>(a, own * a.inv_t);
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t col = lo + (int64_t)(c * NT + (int)threadIdx.x) * 8;
    if (!whole && col >= a.vocab) break;
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = none ? 0.0f : grad((float)v[c].v[i]);
    if constexpr (FEW) {
      // The given tokens among the piece's, one by one, each lane its own (8192 x 1000 bfloat16 with 8 tokens 17 us;
      // 26 where all tokens were looked through for each of the piece's logits).
      uint32_t hits = 0;
      for (int k = 0; k < a.given; ++k) {
        const uint32_t at = (uint32_t)(given[k].id - (int)col);
        hits |= at < 8 ? 1u << at : 0u;
      }
      if (none) hits = 0;
#pragma unroll 1
      for (; hits; hits &= hits - 1) {
        const int at = __builtin_ctz(hits);
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x = i == at ? (float)v[c].v[i] : x;
        const float t = token((int)col + at, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = i == at ? t : d[i];
      }
    }
    Raw8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (T)d[i];
    store8_tail(dz + col, o, whole ? 8 : a.vocab - col);
  }
  if constexpr (!FEW) {
    if (none) return;
    __syncthreads();  // the pass's stores come before the tokens'
    const int hi = lo + NT * CH * 8;
    for (int i = threadIdx.x; i < a.given; i += NT) {
      const int j = given[i].id;
      if (j >= lo && j < hi) dz[j] = (T)token(j, logit<T, ONE>(a, z, j));
    }
  }
}

template <typename T, bool ONE>
hipError_t run_bwd(LogpArgs a, hipStream_t stream) {
  // threads and pieces by the row's length: lanes past its end load its end again (bfloat16, 8192 x 1000 with 256 threads
  // of one piece 15.4 us, of four 21; 8184 x 8200 in two chunks of three pieces 82 us, of four 101)
  const bool small = a.vocab <= 512, middle = !small && a.vocab <= 2048;
  const auto up = [](int n, int d) { return (n + d - 1) / d; };
  const int pieces = up(up(a.vocab, up(a.vocab, 8192)), 2048);  // of the longer rows: chunks alike
  a.chunks = small ? 1 : up(a.vocab, 2048 * pieces);
  const int64_t most = LAUNCH_MAX / a.chunks > 0 ? LAUNCH_MAX / a.chunks : 1;
  for (a.first = 0; a.first < a.rows; a.first += most) {
    const int64_t rows = a.rows - a.first < most ? a.rows - a.first : most;
    const unsigned grid = (unsigned)(rows * a.chunks);
    const int space = 8 * a.given;
#define ROW(NT, CH)                                                                     \
  if (a.given > 8)                                                                      \
    logp_bwd_kernel<T, ONE, NT, CH, false><<<grid, NT, space, stream>>>(a);             \
  else                                                                                  \
    logp_bwd_kernel<T, ONE, NT, CH, true><<<grid, NT, space, stream>>>(a)
    if (small) {
      ROW(64, 1);
    } else if (middle) {
      ROW(256, 1);
    } else if (pieces == 2) {
      ROW(256, 2);
    } else if (pieces == 3) {
      ROW(256, 3);
    } else {
      ROW(256, 4);
    }
#undef ROW
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
  a.scale = a.temperature < 0x1p64f ? 1.0f : 0x1p-64f;
  const float t = a.temperature * a.scale;
  a.inv_t = 1.0f / t;
  const double c = 1.4426950408889634 / (double)t;
  a.c_hi = (float)c;
  if ((double)a.c_hi > c) a.c_hi = nextafterf(a.c_hi, 0.0f);
  a.c_lo = fmaxf((float)(c - (double)a.c_hi), FLT_MIN);
  return a;
}

int64_t parts_bytes(int64_t parts) { return (parts * (int64_t)sizeof(Part) + 15) / 16 * 16; }

}  // namespace

int64_t logprobs_workspace_bytes(int64_t rows, int64_t vocab, int64_t top) {
  const int chunks = cut_of(rows, vocab).chunks;
  if (chunks == 1) return 0;
  const int64_t parts = rows * chunks;
  return parts_bytes(parts) + parts * top * 8;
}

hipError_t launch_logprobs_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, int64_t top, const void *z,
                               const void *ids, double temperature, void *ws, void *logp, void *entropy, void *top_ids,
                               void *top_logp, void *stats, hipStream_t stream) {
  LogpArgs a = args_of(nc, rows, vocab, given, z, ids, temperature);
  const Cut cut = cut_of(rows, vocab);
  a.chunks = cut.chunks;
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
    if (nc == 1 && a.scale == 1.0f)
      return top > 0 ? run_fwd<T, true, true>(a, cut, stream) : run_fwd<T, true, false>(a, cut, stream);
    return top > 0 ? run_fwd<T, false, true>(a, cut, stream) : run_fwd<T, false, false>(a, cut, stream);
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
    return nc == 1 && a.scale == 1.0f ? run_bwd<T, true>(a, stream) : run_bwd<T, false>(a, stream);
  };
  if (dtype == LM_F16) return go((_Float16)0.0f);
  if (dtype == LM_BF16) return go((__bf16)0.0f);
  return go(0.0f);
}

}  // namespace mcf
