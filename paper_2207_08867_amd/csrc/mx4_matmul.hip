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

template <int N>
struct Count {
  static constexpr int value = N;
};

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

// The 32 elements of a plain x that lane group g needs of a group of 128, as loaded.
template <typename T>
struct XRow {
  Raw8<T> v[4];
};

// acc += W x over one group: lane (r, g) holds codes of block g of weight row r and the elements of
// that block of x row r, and takes the reduction in the order that lays the blocks' eight numbers j
// side by side.
template <typename T>
__device__ inline f32x4 thin_group(f32x4 acc, u32x4 code, float scale, const XRow<T> &x) {
  constexpr int P = mx_pieces<T>();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x8 wf = mx_bf16(code[j], scale);
    bf16x8 xf[P];
    mx_cut8<T, P>(x.v[j], xf);
#pragma unroll
    for (int p = 0; p < P; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[p], acc, 0, 0, 0);
  }
  return acc;
}

__device__ inline f32x4 thin_group(f32x4 acc, u32x4 code, uint32_t scale, u32x4 x, uint32_t x_scale) {
  i32x8 av = {}, bv = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) av[i] = (int)code[i], bv[i] = (int)x[i];
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 4, 0, (int)scale, 0, (int)x_scale);
}

// Few rows of x.  A workgroup owns 16 rows of the weight and 16 MT rows of x, and its NW
// wavefronts share the reduction, group by group; their sums are joined through LDS in the
// wavefronts' order.  A lane's 16 bytes of codes, one block, are the operand of one 16 x 16 x 128
// scaled product, or of four 16 x 16 x 32 bfloat16 products.  The weight is read once, straight
// into registers.  What bounds it is the latency of its loads: U groups of a wavefront are asked for
// before the first is used, so with 4096 columns (NW = 8, U = 4) the whole weight is in flight (8 rows
// by 4096 x 4096, both MXFP4: 4.8 us, 1.9 TB/s).
template <typename T, bool PACKED, int MT, int NW, int U>
__global__ __launch_bounds__(64 * NW) void mx_thin_kernel(ThinArgs a) {
  __shared__ f32x4 part[NW][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
  const int64_t wrow = n0 + r < a.N ? n0 + r : a.N - 1;
  int64_t xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xrow[t] = m0 + 16 * t + r < a.M ? m0 + 16 * t + r : a.M - 1;
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t whole = PACKED ? a.G : a.K / MX_GROUP;  // groups that need no tail check

  for (int cw = 0; cw < a.w_nc; ++cw) {
    const uint8_t *w = a.w + ((int64_t)cw * a.N + wrow) * (a.G * 64) + g * 16;
    const uint32_t *ws = a.w_scales + (int64_t)cw * a.G * a.N + wrow;
    const auto codes_at = [&](int64_t s) { return *reinterpret_cast<const u32x4 *>(w + s * 64); };
    const auto scale_at = [&](int64_t s) { return (ws[s * a.N] >> (8 * g)) & 255u; };
    if constexpr (PACKED) {
      for (int cx = 0; cx < a.x_nc; ++cx) {
        const uint8_t *x = reinterpret_cast<const uint8_t *>(a.x) + (int64_t)cx * a.M * (a.G * 64) + g * 16;
        const uint32_t *xs = a.x_scales + (int64_t)cx * a.G * a.M;
        const auto run = [&](int64_t s0, auto count) {
          constexpr int C = decltype(count)::value;
          u32x4 code[C], xc[MT][C];
          uint32_t scale[C], sc[MT][C];
#pragma unroll
          for (int u = 0; u < C; ++u) code[u] = codes_at(s0 + u * NW), scale[u] = scale_at(s0 + u * NW);
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < C; ++u) {
              xc[t][u] = *reinterpret_cast<const u32x4 *>(x + xrow[t] * (a.G * 64) + (s0 + u * NW) * 64);
              sc[t][u] = (xs[(s0 + u * NW) * a.M + xrow[t]] >> (8 * g)) & 255u;
            }
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < C; ++u) acc[t] = thin_group(acc[t], code[u], scale[u], xc[t][u], sc[t][u]);
        };
        int64_t s = wave;
        for (; s + (U - 1) * NW < whole; s += U * NW) run(s, Count<U>());
        for (; s < whole; s += NW) run(s, Count<1>());
      }
    } else {
      const T *x = reinterpret_cast<const T *>(a.x) + g * 32;
      const auto run = [&](int64_t s0, auto count) {
        constexpr int C = decltype(count)::value;
        u32x4 code[C];
        uint32_t scale[C];
#pragma unroll
        for (int u = 0; u < C; ++u) code[u] = codes_at(s0 + u * NW), scale[u] = scale_at(s0 + u * NW);
        XRow<T> xr[C];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
#pragma unroll
          for (int u = 0; u < C; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) xr[u].v[j] = load8(x + xrow[t] * a.K + (s0 + u * NW) * MX_GROUP + j * 8);
#pragma unroll
          for (int u = 0; u < C; ++u) acc[t] = thin_group<T>(acc[t], code[u], mx_scale(scale[u]), xr[u]);
        }
      };
      int64_t s = wave;
      for (; s + (U - 1) * NW < whole; s += U * NW) run(s, Count<U>());
      for (; s < whole; s += NW) run(s, Count<1>());
      if (s < a.G) {  // the ragged last group: zeros past the row
        const u32x4 code = codes_at(s);
        const float scale = mx_scale(scale_at(s));
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          XRow<T> xr;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t k = s * MX_GROUP + j * 8;
            xr.v[j] = load8_tail(x + xrow[t] * a.K + k, a.K - k - g * 32);
          }
          acc[t] = thin_group<T>(acc[t], code, scale, xr);
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

// One to XT rows of a binary16 or binary32 x.  As above, but the pieces of x are made once: a lane
// splits 8 elements of each row, of the four groups that its wavefront holds, and the wavefront
// reads them back from LDS as operands.  Splitting in the operands' layout instead repeats it in all
// 16 lanes of a block, most of them for rows that x does not have.  What bounds it is the latency of
// its loads: 184 to 240 VGPRs leave one workgroup of eight wavefronts a CU, with nothing in flight
// while it joins and leaves.  Measured, this kernel and the one above (us, launches in a graph):
// 4096 x 4096, one row of binary16 3.8 and 5.6, of binary32 4.3 and 8.0; 32768 x 4096 23.4 (3.0 TB/s)
// and 28.4, 26.2 and 41.7.  Four rows: 5.3 and 5.7, 6.5 and 8.4; 33.7 and 29.9, 43.8 and 46.1;
// 1024 x 1024 4.5 and 3.4, 5.2 and 4.1.  (Eight rows of binary16 by the same kernel: 6.8, 6.1 by the
// one above.)
template <typename T, int XT, int NW>
__global__ __launch_bounds__(64 * NW) void mx_token_kernel(ThinArgs a) {
  constexpr int P = mx_pieces<T>(), U = 4;
  __shared__ bf16x8 pieces[NW][XT][P][U][16];  // [piece of 8 elements] of a group
  __shared__ f32x4 part[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t wrow = n0 + r < a.N ? n0 + r : a.N - 1;
  const int rows = (int)a.M, xr = r < rows ? r : 0;
  const T *x = reinterpret_cast<const T *>(a.x);
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t s0 = wave; s0 < a.G; s0 += NW * U) {
    // this lane's 8 elements: piece r of group g of the four
    const int64_t k = (s0 + g * NW) * MX_GROUP + r * 8;
    Raw8<T> raw[XT];
#pragma unroll
    for (int t = 0; t < XT; ++t) raw[t] = load8_tail(x + (t < rows ? t : 0) * a.K + k, a.K - k);
    for (int cw = 0; cw < a.w_nc; ++cw) {
      const uint8_t *w = a.w + ((int64_t)cw * a.N + wrow) * (a.G * 64) + g * 16;
      const uint32_t *ws = a.w_scales + (int64_t)cw * a.G * a.N + wrow;
      u32x4 code[U];
      uint32_t scale[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t s = s0 + u * NW < a.G ? s0 + u * NW : a.G - 1;  // past the end: x is zero there
        code[u] = *reinterpret_cast<const u32x4 *>(w + s * 64);
        scale[u] = (ws[s * a.N] >> (8 * g)) & 255u;
      }
      if (cw == 0) {
#pragma unroll
        for (int t = 0; t < XT; ++t) {
          bf16x8 f[P];
          mx_cut8<T, P>(raw[t], f);
#pragma unroll
          for (int p = 0; p < P; ++p) pieces[wave][t][p][g][r] = f[p];
        }
        wave_sync();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = s0 + u * NW < a.G;
        const float sc = mx_scale(in ? scale[u] : 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 wf = mx_bf16(code[u][j], sc);
#pragma unroll
          for (int p = 0; p < P; ++p)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, pieces[wave][XT == 1 ? 0 : xr][p][u][g * 4 + j], acc, 0, 0, 0);
        }
      }
    }
    wave_sync();  // the pieces are read before the next ones are written
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave > 0 || r >= rows) return;
  f32x4 v = part[0][lane];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += part[w][lane];
  T *y = reinterpret_cast<T *>(a.y) + r * a.N;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t n = n0 + 4 * g + i;
    if (n < a.N) y[n] = (T)(a.bias ? v[i] + (float)reinterpret_cast<const T *>(a.bias)[n] : v[i]);
  }
}

template <typename T, bool PACKED, int MT>
hipError_t thin_mt(const ThinArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  // about four groups a wavefront.  One row of binary16 by 4096 weight rows with 2, 4 and 8 wavefronts
  // (us): 512 columns 3.2, 3.4, 3.4; 2048 4.0, 3.2, 3.9; 4096 5.9, 4.1, 3.8; MXFP4 and bfloat16 rows differ
  // less, by 0.1 to 1
  constexpr int U = MT == 1 ? (sizeof(T) == 4 && !PACKED ? 2 : 4) : 2;
  if (a.G <= 4)
    mx_thin_kernel<T, PACKED, MT, 2, U><<<grid, 128, 0, stream>>>(a);
  else if (a.G <= 16)
    mx_thin_kernel<T, PACKED, MT, 4, U><<<grid, 256, 0, stream>>>(a);
  else
    mx_thin_kernel<T, PACKED, MT, 8, U><<<grid, 512, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int XT>
hipError_t token(const ThinArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.N + 15) / 16));
  if (a.G <= 4)
    mx_token_kernel<T, XT, 2><<<grid, 128, 0, stream>>>(a);
  else if (a.G <= 16)
    mx_token_kernel<T, XT, 4><<<grid, 256, 0, stream>>>(a);
  else
    mx_token_kernel<T, XT, 8><<<grid, 512, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, bool PACKED>
hipError_t thin(const ThinArgs &a, hipStream_t stream) {
  if constexpr (!PACKED && mx_pieces<T>() > 1) {
    if (a.M == 1) return token<T, 1>(a, stream);
    if (a.M <= 4) return token<T, 4>(a, stream);
    return thin_mt<T, PACKED, 1>(a, stream);
  } else {
    if (a.M <= 16) return thin_mt<T, PACKED, 1>(a, stream);
    if constexpr (!PACKED) return thin_mt<T, PACKED, 2>(a, stream);
    else return a.M <= 32 ? thin_mt<T, PACKED, 2>(a, stream) : thin_mt<T, PACKED, 4>(a, stream);
  }
}

template <bool PACKED>
hipError_t thin_any(int dtype, const ThinArgs &a, hipStream_t stream) {
  if (dtype == LM_F16) return thin<_Float16, PACKED>(a, stream);
  if (dtype == LM_BF16) return thin<__bf16, PACKED>(a, stream);
  return thin<float, PACKED>(a, stream);
}

}  // namespace

// Up to so many rows of x the weight is read straight into registers; above, tiles go through LDS.
// Registers and tiles (us, launches in a graph), K = 4096:
//   MXFP4     4096 weight rows: 64 rows of x 7.6 and 9.6, 96 11.7 and 11.5; 14336: 16 10.4 and 11.8, 64 26.3
//             and 11.9
//   bfloat16  4096: 32 10.5 and 12.0, 48 16.0 and 13.3; 14336: 16 20.8 and 22.4, 32 36.0 and 22.8
//   binary16  4096: 16 7.4 and 14.7, 48 16.8 and 17.2; 14336: 16 22.2 and 26.8, 24 32.6 and 27.1
//   binary32  4096: 16 12.4 and 20.8, 24 20.4 and 21.8; 14336: 16 42.7 and 54.5, 24 61.7 and 48.7
// and 1024 x 1024 is faster by registers past 96 rows in every format (4.1 to 7.9 and 5.6 to 11.5).  So
// where they cross depends on the weight's size too, which the rule leaves out: the first two limits
// are those of 4096 x 4096 weights, the other two hold for larger ones as well.
constexpr int64_t THIN_PACKED = 64;
int64_t thin_rows(int dtype) { return dtype == LM_BF16 ? 32 : 16; }

namespace {

// MIXH's pass over B's scales [nc][groups][N] and codes [nc][N][64 groups]: the largest scale of
// each row (NaN blocks aside), and for 64 rows whether a block with a number in it lies more than 36
// binades below its row's.  A workgroup takes 64 rows, its 16
// wavefronts a part of the groups each.
__global__ __launch_bounds__(1024) void mx_top_kernel(const uint32_t *scales, const uint8_t *codes, uint8_t *top,
                                                            uint8_t *wide, int nc, int64_t groups, int64_t N) {
  __shared__ int part[16][64];
  __shared__ int far[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 64 + lane, n = row < N ? row : N - 1;
  const int64_t total = nc * groups, from = total * wave / 16, to = total * (wave + 1) / 16;
  int m = 0;
#pragma unroll 4
  for (int64_t i = from; i < to; ++i) {
    const uint32_t w = scales[i * N + n];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int s = (int)(w >> (8 * b)) & 255;
      m = s != 255 && s > m ? s : m;
    }
  }
  part[wave][lane] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) m = part[w][lane] > m ? part[w][lane] : m;
  bool out = false;
  for (int64_t i = from; i < to; ++i) {
    const uint32_t w = scales[i * N + n];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if ((int)((w >> (8 * b)) & 255u) >= m - 36) continue;
      // component i / groups, group i mod groups
      const u32x4 c = *reinterpret_cast<const u32x4 *>(codes + ((i / groups) * N + n) * (groups * 64) + (i % groups) * 64 + b * 16);
      out = out || (((c[0] | c[1]) | (c[2] | c[3])) & 0x77777777u) != 0;
    }
  }
  const bool any = __any(out);
  if (lane == 0) far[wave] = any;
  __syncthreads();
  if (wave == 0) {
    if (row < N) top[row] = (uint8_t)m;
    const bool all = __any(lane < 16 && far[lane & 15] != 0);
    if (lane == 0) wide[blockIdx.x] = all;
  }
}

// Staged planes of a plain x: bfloat16 pieces of binary32, the 16-bit formats as they are.
int planes_of(int dtype) { return dtype == LM_F32 ? 3 : 1; }

// A 16-bit x whose rows are whole groups at 16-byte addresses is multiplied where it lies; any other
// is staged in padded rows.
bool in_place(int dtype, int64_t in, const void *x) {
  return dtype != LM_F32 && in % MX_GROUP == 0 && (uintptr_t)x % 16 == 0;
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }
int64_t stage_bytes(int dtype, int64_t batch, int64_t in) {
  return planes_of(dtype) * batch * mx_groups(in) * MX_GROUP * 2;
}
// The rows' largest scales and the flags of 64 rows each.
int64_t top_bytes(int dtype, int64_t out) { return dtype == LM_F16 ? up16(out) + up16((out + 63) / 64) : 0; }

template <typename T>
hipError_t mix_gemm(GemmArgs &g, int dtype, int nc, const void *x, int64_t in, char *ws, hipStream_t stream) {
  constexpr bool HALF = __is_same(T, _Float16);
  const int64_t ld = g.groups * MX_GROUP;
  g.a = (const char *)x;
  if (!in_place(dtype, in, x)) {
    const int64_t all = (g.M * (ld / 8) + 255) / 256;
    for (int64_t first = 0; first < all; first += LAUNCH_MAX)
      mx_stage_kernel<T><<<(unsigned)(all - first < LAUNCH_MAX ? all - first : LAUNCH_MAX), 256, 0, stream>>>(
          (const T *)x, (uint16_t *)ws, g.M, in, ld, first);
    g.a = ws;
  }
  ws += stage_bytes(dtype, g.M, in);
  if constexpr (HALF) {
    g.top = (const uint8_t *)ws;
    g.wide = g.top + up16(g.N);
    mx_top_kernel<<<(unsigned)((g.N + 63) / 64), 1024, 0, stream>>>(g.bs, (const uint8_t *)g.b, (uint8_t *)g.top,
                                                                  (uint8_t *)g.wide, nc, g.groups, g.N);
    ws += top_bytes(dtype, g.N);
  }
  g.partial = (float *)ws;
  g.a_ld = ld * 2;
  g.a_plane = g.M * g.a_ld;
  return gemm<HALF ? GEMM_MIXH : GEMM_MIX, T>(g, stream);
}

void set_pairs(GemmArgs &g, int na, int nb) {
  for (int j = 0; j < nb; ++j)
    for (int i = 0; i < na; ++i) gemm_pair(g, i, j);
}

}  // namespace

int64_t mx4_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int a_nc, int b_nc) {
  if (M <= THIN_PACKED) return 0;
  return gemm_partial_bytes(M, N, (mx_groups(K) + 1) / 2 * a_nc * b_nc);
}

hipError_t launch_mx4_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales,
                             int a_nc, const void *b_codes, const void *b_scales, int b_nc, void *ws, void *C,
                             hipStream_t stream) {
  const int64_t G = mx_groups(K);
  if (M <= THIN_PACKED) {
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
  if (batch <= thin_rows(dtype)) return 0;
  return stage_bytes(dtype, batch, in) + top_bytes(dtype, out) +
         gemm_partial_bytes(batch, out, mx_groups(in) * 2 * nc * planes_of(dtype));
}

hipError_t launch_mx4_linear(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x,
                             const void *codes, const void *scales, const void *bias, void *ws, void *y,
                             hipStream_t stream) {
  const int64_t G = mx_groups(in);
  if (batch <= thin_rows(dtype)) {
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
  g.M = batch;
  g.N = out;
  g.steps = (int)(G * 2);
  set_pairs(g, planes_of(dtype), nc);
  if (dtype == LM_F16) return mix_gemm<_Float16>(g, dtype, nc, x, in, (char *)ws, stream);
  if (dtype == LM_BF16) return mix_gemm<__bf16>(g, dtype, nc, x, in, (char *)ws, stream);
  return mix_gemm<float>(g, dtype, nc, x, in, (char *)ws, stream);
}

}  // namespace mcf
