// int8_matmul.hip -- products of 8-bit tensors: C = A B^T, each row of A and of B with a scale of its own
// (a token's, an output channel's), and the linear layer of a plain input, quantised on the way.
//
// The sums of the integers' products are exact in 32 bits: 127^2 K stays below 2^31 for the K that the
// calls take.  An output is (sum sa) sb + bias in binary32, rounded once to its format, so it does not depend on
// the tile, the slices or the number of rows.
#include "int8.hpp"
#include "mcf_internal.hpp"
#include "mx4_gemm.hpp"

namespace mcf {
namespace {

struct Int8Args {
  const char *a, *b;      // codes [M][P], [N][P]
  const float *sa, *sb;   // [M], [N]
  const void *bias;       // [N] or null
  void *y;                // [M][N]
  int64_t M, N, P;
};

// Up to 16 MT rows of A.  A workgroup owns 16 rows of B and its NW wavefronts share the reduction by groups
// of 128 bytes; their sums are joined through LDS.  A lane holds 32 bytes of a row, the operands of two 16 x 16
// x 64 products (the order of the reduction is the same on both sides).  B is read once, straight into
// registers.
template <typename T, int MT, int NW, int U>
__global__ __launch_bounds__(64 * NW) void int8_thin_kernel(Int8Args a) {
  __shared__ i32x4 part[NW][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const char *b = a.b + (n0 + r < a.N ? n0 + r : a.N - 1) * a.P + g * 32;
  const char *x[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t] = a.a + (16 * t + r < a.M ? 16 * t + r : a.M - 1) * a.P + g * 32;
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
      for (int h = 0; h < 2; ++h) bv[u][h] = *reinterpret_cast<const i32x4 *>(b + (s0 + u * NW) * 128 + h * 16);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int u = 0; u < C; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) av[t][u][h] = *reinterpret_cast<const i32x4 *>(x[t] + (s0 + u * NW) * 128 + h * 16);
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
    const float sa = a.sa[m];
    T *y = reinterpret_cast<T *>(a.y) + m * a.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t n = n0 + 4 * g + i;
      if (n >= a.N) continue;
      float f = (float)v[i] * sa * a.sb[n];
      if (a.bias) f += (float)reinterpret_cast<const T *>(a.bias)[n];
      y[n] = (T)f;
    }
  }
}

constexpr int64_t THIN = 32;  // rows up to which B is read straight into registers

template <typename T>
hipError_t run(const Int8Args &a, void *ws, hipStream_t stream) {
  if (a.M <= THIN) {
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

}  // namespace

int64_t int8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  return M <= THIN ? 0 : gemm_partial_bytes(M, N, int8_pitch(K) / 128);
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
  return batch * int8_pitch(in) + up16(4 * batch) + int8_matmul_workspace_bytes(batch, out, in);
}

hipError_t launch_int8_linear(int dtype, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                              const void *scales, const void *bias, void *ws, void *y, hipStream_t stream) {
  char *const xc = (char *)ws, *const xs = xc + batch * int8_pitch(in), *const rest = xs + up16(4 * batch);
  const hipError_t e = launch_rmsnorm(dtype, 1, batch, in, x, nullptr, nullptr, 0.0, nullptr, nullptr, xc, xs, false, stream);
  if (e != hipSuccess) return e;
  return launch_int8_matmul(dtype, batch, out, in, xc, xs, codes, scales, bias, rest, y, stream);
}

}  // namespace mcf
