// int8_matmul.hip -- products of 8-bit tensors: C = A B^T, each row of A and of B with a scale of its own
// (a token's, an output channel's), and the linear layer of a plain input, quantised on the way.
//
// The sums of the integers' products are exact in 32 bits: 127^2 K stays below 2^31 for the K that the
// calls take.  An output is (sum sa) sb + bias in binary32, rounded once to its format, so it does not depend on
// the tile, the slices or the number of rows.
#include "int8.hpp"
#include "mcf_internal.hpp"
#include "mx4_gemm.hpp"
#include "wave.hpp"

namespace mcf {
namespace {

struct Int8Args {
  const char *a, *b;      // codes [M][P], [N][P]
  const float *sa, *sb;   // [M], [N]
  const void *bias;       // [N] or null
  void *y;                // [M][N]
  int64_t M, N, P;
};

// Four sums of row m from column n on, as outputs.
template <typename T>
__device__ inline void store4(const Int8Args &a, int64_t m, int64_t n, i32x4 v, float sa) {
  T *y = reinterpret_cast<T *>(a.y) + m * a.N;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= a.N) continue;
    float f = (float)v[i] * sa * a.sb[n + i];
    if (a.bias) f += (float)reinterpret_cast<const T *>(a.bias)[n + i];
    y[n + i] = (T)f;
  }
}

// Up to 16 MT rows of A.  A workgroup owns 16 rows of B and its NW wavefronts share the reduction by groups
// of 128 bytes, two 16 x 16 x 64 products each; their sums are joined through LDS.  B is read once, straight into
// registers, U groups a wavefront asked for together, which are 4096 elements of a row (2048 past 16 rows of A); what
// those leave of a row goes a group at a time, each waited for.  What bounds the small sizes is the latency of a launch
// and of those loads (8 rows by 4096 x 1024, 2048, 4096, 5120 and 8192: 4.2, 5.0, 6.8, 7.2 and 10.4 us, 2.4 TB/s at
// 4096), the large ones the memory (one row by 32768 x 4096: 26.5 us, 5.1 TB/s).  4, 8 and 16 wavefronts with 2 to 8
// groups ahead measured the same within 5%.
template <typename T, int MT, int NW, int U>
__global__ __launch_bounds__(64 * NW) void int8_thin_kernel(Int8Args a) {
  __shared__ i32x4 part[NW][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const char *b = a.b + (n0 + r < a.N ? n0 + r : a.N - 1) * a.P + g * 16;
  const char *x[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t] = a.a + (16 * t + r < a.M ? 16 * t + r : a.M - 1) * a.P + g * 16;
  i32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
  const int groups = (int)(a.P / 128);
  const auto run = [&](int s0, auto count) {
    constexpr int C = decltype(count)::value;
    i32x4 bv[C][2], av[MT][C][2];
#pragma unroll
    for (int u = 0; u < C; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) bv[u][h] = *reinterpret_cast<const i32x4 *>(b + (s0 + u * NW) * 128 + h * 64);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int u = 0; u < C; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) av[t][u][h] = *reinterpret_cast<const i32x4 *>(x[t] + (s0 + u * NW) * 128 + h * 64);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int u = 0; u < C; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bv[u][h], av[t][u][h], acc[t], 0, 0, 0);
  };
  int s = wave;
  for (; s + (U - 1) * NW < groups; s += U * NW) run(s, std::integral_constant<int, U>());
  for (; s < groups; s += NW) run(s, std::integral_constant<int, 1>());
#pragma unroll
  for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < MT; t += NW) {
    i32x4 v = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += part[w][t][lane];
    // lane (r, g): row r of A, rows 4 g .. 4 g + 3 of B
    const int64_t m = 16 * t + r;
    if (m >= a.M) continue;
    store4<T>(a, m, n0 + 4 * g, v, a.sa[m]);
  }
}

// One or two rows of a plain x quantised on the way: the wavefronts ask for their first U groups of B, then all quantise
// x (every workgroup the same) into LDS, from which the products take it.
constexpr int TOKEN_BYTES = 32768;
template <typename T, int NW, int U>
__global__ __launch_bounds__(64 * NW) void int8_token_kernel(Int8Args a, const T *x, int64_t K) {
  extern __shared__ __attribute__((aligned(16))) char codes[];  // [M][P + 16]
  __shared__ uint32_t big[2][NW];
  __shared__ float scale[2];
  __shared__ i32x4 part[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const char *b = a.b + (n0 + r < a.N ? n0 + r : a.N - 1) * a.P + g * 16;
  const int groups = (int)(a.P / 128), M = (int)a.M, P = (int)a.P, ld = P + 16, k = (int)K;
  i32x4 bv[U][2];
  const auto ask = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int s = s0 + u * NW < groups ? s0 + u * NW : groups - 1;
        bv[u][h] = *reinterpret_cast<const i32x4 *>(b + (int64_t)s * 128 + h * 64);
      }
  };
  ask(wave);
  const auto piece = [&](int row, int col, float p[8]) {
    const Raw8<T> u = load8_tail(x + (int64_t)row * K + col, K - col);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (float)u.v[i];
  };
  // the first piece of the first row stays
  float first[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int row = 0; row < M; ++row) {
    uint32_t m = 0;
    for (int col = threadIdx.x * 8; col < k; col += 64 * NW * 8) {
      float p[8];
      piece(row, col, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t u = magnitude(p[i]);
        m = u > m ? u : m;
        if (row == 0 && col < 64 * NW * 8) first[i] = p[i];
      }
    }
    m = lanes_max(m);
    if (lane == 0) big[row][wave] = m;
  }
  __syncthreads();
  for (int row = 0; row < M; ++row) {
    const uint32_t m = lanes_max<NW>(big[row][lane % NW]);
    const Int8Row s = int8_row((double)__builtin_bit_cast(float, m), 1.0);
    if (threadIdx.x == 0) scale[row] = s.scale;
    for (int col = threadIdx.x * 8; col < P; col += 64 * NW * 8) {
      float p[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if (row == 0 && col < 64 * NW * 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = first[i];
      } else if (col < k) {
        piece(row, col, p);
      }
      *reinterpret_cast<uint64_t *>(codes + row * ld + col) = s.near ? int8_codes8(p, s) : int8_codes8_any(p, s);
    }
  }
  __syncthreads();
  i32x4 acc = {0, 0, 0, 0};
  const char *xc = codes + (r < M ? r : 0) * ld + g * 16;
  for (int s0 = wave; s0 < groups; s0 += U * NW) {
    if (s0 != wave) ask(s0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u * NW < groups)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              bv[u][h], *reinterpret_cast<const i32x4 *>(xc + (s0 + u * NW) * 128 + h * 64), acc, 0, 0, 0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || r >= M) return;
#pragma unroll
  for (int w = 1; w < NW; ++w) acc += part[w][lane];
  store4<T>(a, r, n0 + 4 * g, acc, scale[r]);
}

// Few rows read B straight into registers; tiles read it through LDS and do not read A again for every 16 rows of B,
// which costs more the larger B is.  Straight and by tiles (us, launches in a graph; rows of A, B): 4, 14336 x 4096 14.6
// and 19.6, 32768 x 4096 28.2 and 34.5; 8, 8192 x 4096 9.9 and 11.5, 14336 x 4096 16.3 and 13.8, 4096 x 16384 18.1 and
// 16.0, 24576 x 4096 24.3 and 29.2, 32768 x 4096 30.8 and 33.6, 131072 x 1024 31.4 and 37.4 (straight loses at 56 to 64
// MiB alone); 16, 4096 x 4096 7.5 and 10.3, 8192 x 4096 11.1 and 11.8, 14336 x 4096 18.2 and 14.1; 32, 4096 x 4096
// 9.6 and 11.3, 8192 x 4096 15.0 and 12.1, 32768 x 4096 55.9 and 33.7.
bool thin(int64_t M, int64_t N, int64_t P) {
  const int64_t mib = N * P >> 20;
  return M <= 8 || (M <= 16 && mib < 48) || (M <= 32 && mib < 24);
}

template <typename T>
hipError_t run(const Int8Args &a, void *ws, hipStream_t stream) {
  if (thin(a.M, a.N, a.P)) {
    const unsigned grid = (unsigned)((a.N + 15) / 16);
    if (a.M <= 16)
      int8_thin_kernel<T, 1, 8, 4><<<grid, 512, 0, stream>>>(a);
    else
      int8_thin_kernel<T, 2, 8, 2><<<grid, 512, 0, stream>>>(a);
    return hipGetLastError();
  }
  GemmArgs g = {};
  g.a = a.a;
  g.b = a.b;
  g.a_ld = g.b_ld = a.P;
  g.sa = a.sa;
  g.sb = a.sb;
  g.c = a.y;
  g.bias = a.bias;
  g.partial = (float *)ws;
  g.M = a.M;
  g.N = a.N;
  g.steps = (int)(a.P / 128);
  gemm_pair(g, 0, 0);
  return gemm<GEMM_I8, T>(g, stream);
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// One launch, in which every workgroup quantises x, in place of two.  Past two workgroups a CU, 8192 outputs, their
// quantisations follow one another; they pay where each has 64 KiB of weights or more to read beside it.  One launch
// and two (us, in a graph, bfloat16; in -> out), one row: 4096 -> 4096 7.4 and 9.8, 1024 -> 8192 7.2 and 7.2, 1024 ->
// 16384 12.6 and 9.4, 1024 -> 131072 85 and 29, 4096 -> 16384 16.0 and 17.6, 4096 -> 32768 29.7 and 31.1, 4096 -> 65536
// 53.8 and 53.0, 32768 -> 1024 26.6 and 30.5; two rows: 1024 -> 4096 6.7 and 6.8, 1024 -> 8192 8.9 and 7.2, 4096 ->
// 8192 11.8 and 12.7, 4096 -> 16384 19.5 and 17.9, 4096 -> 32768 38.2 and 30.9; four rows 4096 -> 4096 11.2 and 10.5.
bool token(int64_t batch, int64_t in, int64_t out) {
  if (batch > 2 || in == 0 || batch * int8_pitch(in) > TOKEN_BYTES) return false;
  return out <= (in < 4096 ? 8192 / batch : (batch == 1 ? 32768 : 8192));
}

template <typename T>
hipError_t run_token(const Int8Args &a, const void *x, int64_t K, hipStream_t stream) {
  int8_token_kernel<T, 8, 4><<<(unsigned)((a.N + 15) / 16), 512, a.M * (a.P + 16), stream>>>(a, (const T *)x, K);
  return hipGetLastError();
}

}  // namespace

int64_t int8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  return thin(M, N, int8_pitch(K)) ? 0 : gemm_partial_bytes(M, N, int8_pitch(K) / 128);
}

hipError_t launch_int8_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales,
                              const void *b_codes, const void *b_scales, const void *bias, void *ws, void *C,
                              hipStream_t stream) {
  Int8Args a = {};
  a.a = (const char *)a_codes;
  a.b = (const char *)b_codes;
  a.sa = (const float *)a_scales;
  a.sb = (const float *)b_scales;
  a.bias = bias;
  a.y = C;
  a.M = M;
  a.N = N;
  a.P = int8_pitch(K);
  if (dtype == LM_F16) return run<_Float16>(a, ws, stream);
  if (dtype == LM_BF16) return run<__bf16>(a, ws, stream);
  return run<float>(a, ws, stream);
}

// x in 8 bits: codes, then scales, then the product's partial sums.
int64_t int8_linear_workspace_bytes(int64_t batch, int64_t in, int64_t out) {
  if (token(batch, in, out)) return 0;
  return batch * int8_pitch(in) + up16(4 * batch) + int8_matmul_workspace_bytes(batch, out, in);
}

hipError_t launch_int8_linear(int dtype, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                              const void *scales, const void *bias, void *ws, void *y, hipStream_t stream) {
  if (token(batch, in, out)) {
    Int8Args a = {};
    a.b = (const char *)codes;
    a.sb = (const float *)scales;
    a.bias = bias;
    a.y = y;
    a.M = batch;
    a.N = out;
    a.P = int8_pitch(in);
    if (dtype == LM_F16) return run_token<_Float16>(a, x, in, stream);
    if (dtype == LM_BF16) return run_token<__bf16>(a, x, in, stream);
    return run_token<float>(a, x, in, stream);
  }
  char *const xc = (char *)ws, *const xs = xc + batch * int8_pitch(in), *const rest = xs + up16(4 * batch);
  const hipError_t e =
      launch_rmsnorm(dtype, 1, batch, in, x, nullptr, nullptr, 0.0, nullptr, nullptr, xc, xs, false, stream);
  if (e != hipSuccess) return e;
  return launch_int8_matmul(dtype, batch, out, in, xc, xs, codes, scales, bias, rest, y, stream);
}

}  // namespace mcf
