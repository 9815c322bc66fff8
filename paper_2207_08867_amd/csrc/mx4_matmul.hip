// mx4_matmul.hip -- products with an MXFP4 weight: C = A B^T of two MXFP4 tensors, and the linear
// layer y = x W^T + b of a plain x.
//
// With nc components an MXFP4 tensor is the sum of nc tensors, so a product is the sum of the
// component products; all of them go into one binary32 accumulator.  The numbers of the blocks
// are exact in bfloat16, and a binary16 (binary32) input is the exact sum of two (three) bfloat16
// pieces, so every product of elements is exact and the only roundings are the accumulator's and
// the result's.
#include "mcf_internal.hpp"
#include "mx4.hpp"
#include "mx4_gemm.hpp"

namespace mcf {
namespace {

struct ThinArgs {
  const void *x;             // plain [M][K], or codes [x_nc][M][64 G]
  const uint32_t *x_scales;  // [x_nc][G][M]
  const uint8_t *w;          // [w_nc][N][64 G]
  const uint32_t *w_scales;  // [w_nc][G][N]
  const void *bias;          // [N] or null
  void *y;                   // [M][N]
  int64_t M, N, K, G;
  int x_nc, w_nc;
};

// Few rows of x.  A workgroup owns 16 rows of the weight and 16 MT rows of x, and its NW
// wavefronts share the reduction, group by group; their sums are joined through LDS in the
// wavefronts' order.  A group is 128 long: lane (r, g) of the wavefront holds block g of weight row
// r, 16 bytes of codes, which is the operand of one 16 x 16 x 128 scaled product, or of four
// 16 x 16 x 32 bfloat16 products that take the reduction in the order that lays block g's eight
// numbers j before lane group g.  The weight is read once and straight into registers; U groups
// are in flight per wavefront.
template <typename T, bool PACKED, int MT, int NW, int U>
__global__ __launch_bounds__(64 * NW) void mx_thin_kernel(ThinArgs a) {
  constexpr int P = PACKED ? 1 : mx_pieces<T>();
  __shared__ f32x4 part[NW][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
  const int64_t wrow = n0 + r < a.N ? n0 + r : a.N - 1;
  int64_t xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xrow[t] = m0 + 16 * t + r < a.M ? m0 + 16 * t + r : a.M - 1;
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int cw = 0; cw < a.w_nc; ++cw) {
    const uint8_t *w = a.w + ((int64_t)cw * a.N + wrow) * (a.G * 64) + g * 16;
    const uint32_t *ws = a.w_scales + (int64_t)cw * a.G * a.N + wrow;
    for (int cx = 0; cx < a.x_nc; ++cx) {
      for (int64_t s0 = wave; s0 < a.G; s0 += NW * U) {
        u32x4 code[U];
        uint32_t scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t s = s0 + u * NW;
          code[u] = u32x4{0, 0, 0, 0};
          scale[u] = 0;
          if (s < a.G) {
            code[u] = *reinterpret_cast<const u32x4 *>(w + s * 64);
            scale[u] = (ws[s * a.N] >> (8 * g)) & 255u;
          }
        }
        if constexpr (PACKED) {
          const uint8_t *x = reinterpret_cast<const uint8_t *>(a.x);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            u32x4 xc[U];
            uint32_t xs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int64_t s = s0 + u * NW;
              xc[u] = u32x4{0, 0, 0, 0};
              xs[u] = 0;
              if (s < a.G) {
                xc[u] = *reinterpret_cast<const u32x4 *>(x + ((int64_t)cx * a.M + xrow[t]) * (a.G * 64) + s * 64 + g * 16);
                xs[u] = (a.x_scales[((int64_t)cx * a.G + s) * a.M + xrow[t]] >> (8 * g)) & 255u;
              }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              i32x8 av = {}, bv = {};
#pragma unroll
              for (int i = 0; i < 4; ++i) av[i] = (int)code[u][i], bv[i] = (int)xc[u][i];
              acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc[t], 4, 4, 0, (int)scale[u], 0,
                                                                        (int)xs[u]);
            }
          }
        } else {
          const T *x = reinterpret_cast<const T *>(a.x);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int64_t k = (s0 + u * NW) * 128 + g * 32;
            const float sc = mx_scale(scale[u]);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              Raw8<T> xr[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) xr[j] = load8_tail(x + xrow[t] * a.K + k + j * 8, a.K - (k + j * 8));
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const bf16x8 wf = mx_bf16(code[u][j], sc);
                if constexpr (P == 1) {
                  acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, __builtin_bit_cast(bf16x8, xr[j]), acc[t], 0, 0, 0);
                } else {
                  bf16x8 xf[P];
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    __bf16 q[P];
                    mx_split<P>((float)xr[j].v[i], q);
#pragma unroll
                    for (int p = 0; p < P; ++p) xf[p][i] = q[p];
                  }
#pragma unroll
                  for (int p = 0; p < P; ++p) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[p], acc[t], 0, 0, 0);
                }
              }
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < MT; t += NW) {
    f32x4 v = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += part[w][t][lane];
    // lane (r, g): row r of x, weight rows 4 g .. 4 g + 3
    const int64_t m = m0 + 16 * t + r;
    if (m >= a.M) continue;
    T *y = reinterpret_cast<T *>(a.y) + m * a.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t n = n0 + 4 * g + i;
      if (n < a.N) y[n] = (T)(a.bias ? v[i] + (float)reinterpret_cast<const T *>(a.bias)[n] : v[i]);
    }
  }
}

template <typename T, bool PACKED, int MT>
hipError_t thin_mt(const ThinArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  if (a.G <= 8)
    mx_thin_kernel<T, PACKED, MT, 4, 2><<<grid, 256, 0, stream>>>(a);
  else
    mx_thin_kernel<T, PACKED, MT, 8, 2><<<grid, 512, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, bool PACKED>
hipError_t thin(const ThinArgs &a, hipStream_t stream) {
  if (a.M <= 16) return thin_mt<T, PACKED, 1>(a, stream);
  return thin_mt<T, PACKED, 4>(a, stream);
}

template <bool PACKED>
hipError_t thin_any(int dtype, const ThinArgs &a, hipStream_t stream) {
  if (dtype == LM_F16) return thin<_Float16, PACKED>(a, stream);
  if (dtype == LM_BF16) return thin<__bf16, PACKED>(a, stream);
  return thin<float, PACKED>(a, stream);
}

}  // namespace

// Up to THIN rows of x the weight is read straight into registers; above, tiles go through LDS.
constexpr int64_t THIN = 64;

namespace {

int pieces_of(int dtype) { return dtype == LM_F32 ? 3 : (dtype == LM_F16 ? 2 : 1); }

// A bfloat16 x whose rows are whole groups at 16-byte addresses is multiplied where it lies; any
// other is staged as bfloat16 pieces of padded rows.
bool in_place(int dtype, int64_t in, const void *x) {
  return dtype == LM_BF16 && in % MX_GROUP == 0 && (uintptr_t)x % 16 == 0;
}

int64_t stage_bytes(int dtype, int64_t batch, int64_t in) {
  return pieces_of(dtype) * batch * mx_groups(in) * MX_GROUP * 2;
}

template <typename T>
hipError_t mix_gemm(GemmArgs &g, int dtype, const void *x, int64_t in, void *ws, hipStream_t stream) {
  const int64_t ld = g.groups * MX_GROUP;
  g.a = (const char *)x;
  if (!in_place(dtype, in, x)) {
    mx_stage_kernel<T><<<(unsigned)((g.M * (ld / 8) + 255) / 256), 256, 0, stream>>>((const T *)x, (uint16_t *)ws, g.M,
                                                                                     in, ld);
    g.a = (const char *)ws;
    g.partial = (float *)((char *)ws + stage_bytes(dtype, g.M, in));
  }
  g.a_ld = ld * 2;
  g.a_plane = g.M * g.a_ld;
  return gemm<GEMM_MIX, T>(g, stream);
}

void set_pairs(GemmArgs &g, int na, int nb) {
  for (int j = 0; j < nb; ++j)
    for (int i = 0; i < na; ++i) gemm_pair(g, i, j);
}

}  // namespace

int64_t mx4_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int a_nc, int b_nc) {
  if (M <= THIN) return 0;
  return gemm_partial_bytes(M, N, (mx_groups(K) + 1) / 2 * a_nc * b_nc);
}

hipError_t launch_mx4_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales,
                             int a_nc, const void *b_codes, const void *b_scales, int b_nc, void *ws, void *C,
                             hipStream_t stream) {
  const int64_t G = mx_groups(K);
  if (M <= THIN) {
    ThinArgs a = {a_codes, (const uint32_t *)a_scales, (const uint8_t *)b_codes, (const uint32_t *)b_scales, nullptr, C,
                  M, N, K, G, a_nc, b_nc};
    return thin_any<true>(dtype, a, stream);
  }
  GemmArgs g = {};
  g.a = (const char *)a_codes;
  g.b = (const char *)b_codes;
  g.a_ld = g.b_ld = G * 64;
  g.a_plane = M * g.a_ld;
  g.b_plane = N * g.b_ld;
  g.as = (const uint32_t *)a_scales;
  g.bs = (const uint32_t *)b_scales;
  g.groups = G;
  g.c = C;
  g.partial = (float *)ws;
  g.M = M;
  g.N = N;
  g.steps = (int)((G + 1) / 2);
  set_pairs(g, a_nc, b_nc);
  if (dtype == LM_F16) return gemm<GEMM_FP4, _Float16>(g, stream);
  if (dtype == LM_BF16) return gemm<GEMM_FP4, __bf16>(g, stream);
  return gemm<GEMM_FP4, float>(g, stream);
}

int64_t mx4_linear_workspace_bytes(int dtype, int nc, int64_t batch, int64_t in, int64_t out) {
  if (batch <= THIN) return 0;
  return stage_bytes(dtype, batch, in) + gemm_partial_bytes(batch, out, mx_groups(in) * 2 * nc * pieces_of(dtype));
}

hipError_t launch_mx4_linear(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x,
                             const void *codes, const void *scales, const void *bias, void *ws, void *y,
                             hipStream_t stream) {
  const int64_t G = mx_groups(in);
  if (batch <= THIN) {
    ThinArgs a = {x, nullptr, (const uint8_t *)codes, (const uint32_t *)scales, bias, y, batch, out, in, G, 1, nc};
    return thin_any<false>(dtype, a, stream);
  }
  GemmArgs g = {};
  g.b = (const char *)codes;
  g.b_ld = G * 64;
  g.b_plane = out * g.b_ld;
  g.bs = (const uint32_t *)scales;
  g.groups = G;
  g.c = y;
  g.bias = bias;
  g.partial = (float *)ws;
  g.M = batch;
  g.N = out;
  g.steps = (int)(G * 2);
  set_pairs(g, pieces_of(dtype), nc);
  if (dtype == LM_F16) return mix_gemm<_Float16>(g, dtype, x, in, ws, stream);
  if (dtype == LM_BF16) return mix_gemm<__bf16>(g, dtype, x, in, ws, stream);
  return mix_gemm<float>(g, dtype, x, in, ws, stream);
}

}  // namespace mcf
