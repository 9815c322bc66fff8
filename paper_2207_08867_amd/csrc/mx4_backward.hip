// mx4_backward.hip -- the gradients of the linear layer y = x W^T + b with an MXFP4 weight:
//   dX = dY W,  dW = dY^T x (the gradient of the numbers that W stands for),  db = column sums of dY.
//
// Both products reduce over an index that is not the fastest one of their operands, so the
// operands are first staged: rows of the reduction, padded with zeros to whole groups of 128, as
// 16-bit pieces whose sums are the values exactly (bfloat16; binary16 for dW of binary16 tensors,
// which is one piece).  W is staged as its components' numbers, exact in bfloat16.  Then both are
// products A B^T of staged tensors, summed over pairs of pieces in binary32.
#include "mcf_internal.hpp"
#include "mx4.hpp"
#include "mx4_gemm.hpp"

namespace mcf {
namespace {

// Sums over a workgroup's 32 groups of lanes of 64 columns, 8 a lane.
__device__ inline void join_columns(const float part[8], float (*f)[64], float *sums, int64_t cols) {
#pragma unroll
  for (int k = 0; k < 8; ++k) f[threadIdx.x >> 3][(threadIdx.x & 7) * 8 + k] = part[k];
  __syncthreads();
  if (threadIdx.x < 64 && threadIdx.x < cols) {
    float s = 0.0f;
    for (int i = 0; i < 32; ++i) s += f[i][threadIdx.x];
    sums[threadIdx.x] = s;
  }
}

// src [rows][cols] -> dst [P][cols][ld], the transpose, zeros from rows to ld (a multiple of 128).
// A workgroup turns 128 rows x 64 columns through LDS: a wavefront reads 8 rows of 64 columns in one
// instruction (16-bit formats) and writes 16 bytes a lane, 8 rows of one column.  SUM: the columns'
// sums of the 128 rows go to sums [tiles of rows][cols], for db.
template <typename T, bool HALF, bool SUM>
__global__ __launch_bounds__(256) void mx_stage_t_kernel(const T *src, uint16_t *dst, float *sums, int64_t rows,
                                                         int64_t cols, int64_t ld) {
  using S = Pieces<T, HALF>;
  // [row][column]: 66 halfwords a row, so the rows of one column lie in different banks
  __shared__ uint16_t tile[S::P][128][66];
  const int64_t c0 = (int64_t)blockIdx.x * 64, r0 = (int64_t)blockIdx.y * 128;
  float part[8] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
    Raw8<T> v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v.v[k] = (T)0.0f;
    if (r0 + r < rows) v = load8_tail(src + (r0 + r) * cols + c0 + c, cols - c0 - c);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint16_t p[S::P];
      S::of(v.v[k], p);
#pragma unroll
      for (int q = 0; q < S::P; ++q) tile[q][r][c + k] = p[q];
      if constexpr (SUM) part[k] += (float)v.v[k];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 16 + (threadIdx.x >> 4), r = (threadIdx.x & 15) * 8;
    if (c0 + c < cols) {
#pragma unroll
      for (int q = 0; q < S::P; ++q) {
        uint16_t out[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) out[k] = tile[q][r + k][c];
        __builtin_memcpy(dst + ((int64_t)q * cols + c0 + c) * ld + r0 + r, out, 16);
      }
    }
  }
  if constexpr (SUM) {
    __syncthreads();
    join_columns(part, reinterpret_cast<float(*)[64]>(tile), sums + blockIdx.y * cols + c0, cols - c0);
  }
}

// The numbers of an MXFP4 weight [nc][out][in], transposed: dst [nc][in][ld], ld >= out.
__global__ __launch_bounds__(256) void mx_unpack_t_kernel(const uint8_t *codes, const uint32_t *scales, uint16_t *dst,
                                                          int64_t out, int64_t in, int64_t groups, int64_t ld) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[128][72];  // [element][row], rows 16 bytes aligned
  const int64_t grp = blockIdx.x, r0 = (int64_t)blockIdx.y * 64, c = blockIdx.z;
  for (int i = threadIdx.x; i < 1024; i += 256) {  // 64 rows x 16 pieces of 8 elements
    const int r = i >> 4, piece = i & 15;
    uint32_t word = 0, byte = 0;
    if (r0 + r < out) {
      word = *reinterpret_cast<const uint32_t *>(codes + (c * out + r0 + r) * (groups * 64) + grp * 64 + piece * 4);
      byte = (scales[(c * groups + grp) * out + r0 + r] >> (8 * (piece >> 2))) & 255u;
    }
    const bf16x8 v = mx_bf16(word, mx_scale(byte));
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[piece * 8 + k][r] = __builtin_bit_cast(uint16_t, (__bf16)v[k]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 128 * 8; i += 256) {
    const int k = i >> 3, r = (i & 7) * 8;
    if (grp * 128 + k < in)
      *reinterpret_cast<u32x4 *>(dst + (c * in + grp * 128 + k) * ld + r0 + r) = *reinterpret_cast<const u32x4 *>(&tile[k][r]);
  }
}

// The pairs (i, j) of pieces with i + j < `below`.
void set_pairs(GemmArgs &a, int na, int nb, int below) {
  for (int i = 0; i < na; ++i)
    for (int j = 0; j < nb; ++j)
      if (i + j < below) gemm_pair(a, i, j);
}

// C [M][N] from staged a [na][M][ld] and b [nb][N][ld], pairs i + j < below.
template <typename T, bool HALF>
hipError_t staged(const uint16_t *a, int na, const uint16_t *b, int nb, int64_t M, int64_t N, int64_t ld, int below,
                  void *c, void *partial, hipStream_t stream) {
  GemmArgs g = {};
  g.a = (const char *)a;
  g.b = (const char *)b;
  g.a_plane = M * ld * 2;
  g.b_plane = N * ld * 2;
  g.a_ld = g.b_ld = ld * 2;
  g.c = c;
  g.partial = (float *)partial;
  g.M = M;
  g.N = N;
  g.steps = (int)(ld / 64);
  set_pairs(g, na, nb, below);
  return gemm<HALF ? GEMM_F16 : GEMM_BF16, T>(g, stream);
}

// Those sums alone, in the same order.
template <typename T>
__global__ __launch_bounds__(256) void mx_colsum_kernel(const T *dy, float *sums, int64_t rows, int64_t cols) {
  __shared__ float f[32][64];
  const int64_t c0 = (int64_t)blockIdx.x * 64, r0 = (int64_t)blockIdx.y * 128;
  float part[8] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
    Raw8<T> v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v.v[k] = (T)0.0f;
    if (r0 + r < rows) v = load8_tail(dy + (r0 + r) * cols + c0 + c, cols - c0 - c);
#pragma unroll
    for (int k = 0; k < 8; ++k) part[k] += (float)v.v[k];
  }
  join_columns(part, f, sums + blockIdx.y * cols + c0, cols - c0);
}

// db from the tiles' sums: a workgroup takes 64 columns, its wavefronts a quarter of the tiles each.
template <typename T>
__global__ __launch_bounds__(256) void mx_db_kernel(const float *sums, T *db, int64_t tiles, int64_t cols) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  const int64_t from = tiles * wave / 4, to = tiles * (wave + 1) / 4;
  float s = 0.0f;
  if (col < cols)
    for (int64_t i = from; i < to; ++i) s += sums[i * cols + col];
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < cols) db[col] = (T)((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]));
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Workspace: dX needs dY [P][T][Op] and W^T [nc][I][Op]; dW needs dY^T [P'][O][Tp] and x^T
// [P'][I][Tp], Op and Tp whole groups; both share one area, used one after the other.
struct Plan {
  int p, pw;        // pieces of a plain element: for dX, for dW
  int64_t op, tp;   // padded reductions
  int64_t dy, wt, dyt, xt;  // bytes of the staged operands
  int64_t partx, partw;     // of the products' partial sums
  int64_t sums;             // of the column sums' parts
};

Plan plan(int dtype, int nc, int64_t T, int64_t I, int64_t O) {
  Plan s;
  s.p = dtype == LM_F32 ? 3 : (dtype == LM_F16 ? 2 : 1);
  s.pw = dtype == LM_F32 ? 3 : 1;
  s.op = up(O, MX_GROUP);
  s.tp = up(T, MX_GROUP);
  s.dy = up(s.p * T * s.op * 2, 256);
  s.wt = up(nc * I * s.op * 2, 256);
  s.dyt = up(s.pw * O * s.tp * 2, 256);
  s.xt = up(s.pw * I * s.tp * 2, 256);
  s.partx = gemm_partial_bytes(T, I, s.op / 64 * s.p * nc);
  s.sums = up((T + 127) / 128 * O * 4, 256);
  s.partw = gemm_partial_bytes(O, I, s.tp / 64 * (s.pw == 3 ? 6 : 1));
  return s;
}

template <typename T, bool HALF>
hipError_t backward(int nc, int64_t rows, int64_t in, int64_t out, const T *x, const uint8_t *codes,
                    const uint32_t *scales, const T *dY, T *dX, T *dW, T *db, const Plan &s, char *ws,
                    hipStream_t stream) {
  const auto blocks = [](int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); };
  // the column sums' parts come first in the workspace and stay; the products' staged operands
  // follow, one product's after the other's
  float *sums = (float *)ws;
  if (db) ws += s.sums;
  if (dX) {
    uint16_t *dy = (uint16_t *)ws, *wt = (uint16_t *)(ws + s.dy);
    if (out > 0) {  // else a reduction of nothing: zeros
      mx_stage_kernel<T><<<blocks(rows * s.op / 8, 256), 256, 0, stream>>>(dY, dy, rows, out, s.op);
      mx_unpack_t_kernel<<<dim3((unsigned)mx_groups(in), blocks(s.op, 64), (unsigned)nc), 256, 0, stream>>>(
          codes, scales, wt, out, in, mx_groups(in), s.op);
    }
    const hipError_t e = staged<T, false>(dy, s.p, wt, nc, rows, in, s.op, s.p + nc, dX, ws + s.dy + s.wt, stream);
    if (e != hipSuccess) return e;
  }
  if (dW) {
    uint16_t *dyt = (uint16_t *)ws, *xt = (uint16_t *)(ws + s.dyt);
    if (rows > 0) {
      const dim3 grid(blocks(out, 64), blocks(s.tp, 128));
      if (db)
        mx_stage_t_kernel<T, HALF, true><<<grid, 256, 0, stream>>>(dY, dyt, sums, rows, out, s.tp);
      else
        mx_stage_t_kernel<T, HALF, false><<<grid, 256, 0, stream>>>(dY, dyt, nullptr, rows, out, s.tp);
      mx_stage_t_kernel<T, HALF, false>
          <<<dim3(blocks(in, 64), blocks(s.tp, 128)), 256, 0, stream>>>(x, xt, nullptr, rows, in, s.tp);
    }
    // of two values in three pieces the pairs past i + j = 2 are left out: each is within 2^-26 of
    // |dY||x|, less than one rounding of the sum
    const hipError_t e = staged<T, HALF>(dyt, s.pw, xt, s.pw, out, in, s.tp, 3, dW, ws + s.dyt + s.xt, stream);
    if (e != hipSuccess) return e;
  }
  if (db) {
    const int64_t tiles = s.tp / 128;
    if (!dW && tiles > 0)
      mx_colsum_kernel<T><<<dim3(blocks(out, 64), (unsigned)tiles), 256, 0, stream>>>(dY, sums, rows, out);
    mx_db_kernel<T><<<blocks(out, 64), 256, 0, stream>>>(sums, db, tiles, out);
  }
  return hipGetLastError();
}

}  // namespace

int64_t mx4_linear_bwd_workspace_bytes(int dtype, int nc, int64_t batch, int64_t in, int64_t out, int dx, int dw,
                                       int db) {
  const Plan s = plan(dtype, nc, batch, in, out);
  const int64_t a = dx ? s.dy + s.wt + s.partx : 0, b = dw ? s.dyt + s.xt + s.partw : 0;
  return (a > b ? a : b) + (db ? s.sums : 0);
}

hipError_t launch_mx4_linear_bwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x,
                                 const void *codes, const void *scales, const void *dY, void *dX, void *dW, void *db,
                                 void *ws, hipStream_t stream) {
  const Plan s = plan(dtype, nc, batch, in, out);
  const uint8_t *c = (const uint8_t *)codes;
  const uint32_t *sc = (const uint32_t *)scales;
  if (dtype == LM_F16)
    return backward<_Float16, true>(nc, batch, in, out, (const _Float16 *)x, c, sc, (const _Float16 *)dY,
                                    (_Float16 *)dX, (_Float16 *)dW, (_Float16 *)db, s, (char *)ws, stream);
  if (dtype == LM_BF16)
    return backward<__bf16, false>(nc, batch, in, out, (const __bf16 *)x, c, sc, (const __bf16 *)dY, (__bf16 *)dX,
                                   (__bf16 *)dW, (__bf16 *)db, s, (char *)ws, stream);
  return backward<float, false>(nc, batch, in, out, (const float *)x, c, sc, (const float *)dY, (float *)dX,
                                (float *)dW, (float *)db, s, (char *)ws, stream);
}

}  // namespace mcf
