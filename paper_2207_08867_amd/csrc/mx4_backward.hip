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

// src [rows][cols] -> dst [P][cols][ld], the transpose, zeros from rows to ld (a multiple of 64).
template <typename T, bool HALF>
__global__ __launch_bounds__(256) void mx_stage_t_kernel(const T *src, uint16_t *dst, int64_t rows, int64_t cols,
                                                         int64_t ld) {
  using S = Pieces<T, HALF>;
  __shared__ uint16_t tile[S::P][64][66];
  const int64_t c0 = (int64_t)blockIdx.x * 64, r0 = (int64_t)blockIdx.y * 64;
  for (int i = threadIdx.x; i < 4096; i += 256) {
    const int r = i >> 6, c = i & 63;
    const bool in = r0 + r < rows && c0 + c < cols;
    uint16_t p[S::P];
    S::of(in ? src[(r0 + r) * cols + c0 + c] : (T)0.0f, p);
#pragma unroll
    for (int k = 0; k < S::P; ++k) tile[k][c][r] = p[k];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 4096; i += 256) {
    const int c = i >> 6, r = i & 63;
    if (c0 + c >= cols || r0 + r >= ld) continue;
#pragma unroll
    for (int k = 0; k < S::P; ++k) dst[((int64_t)k * cols + c0 + c) * ld + r0 + r] = tile[k][c][r];
  }
}

// The numbers of an MXFP4 weight [nc][out][in], transposed: dst [nc][in][ld], ld >= out.
__global__ __launch_bounds__(256) void mx_unpack_t_kernel(const uint8_t *codes, const uint32_t *scales, uint16_t *dst,
                                                          int64_t out, int64_t in, int64_t groups, int64_t ld) {
  __shared__ uint16_t tile[128][66];
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
  for (int i = threadIdx.x; i < 128 * 64; i += 256) {
    const int k = i >> 6, r = i & 63;
    if (grp * 128 + k < in && r0 + r < ld) dst[(c * in + grp * 128 + k) * ld + r0 + r] = tile[k][r];
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

// db: a workgroup sums 64 columns, its four wavefronts every fourth row.
template <typename T>
__global__ __launch_bounds__(256) void mx_colsum_kernel(const T *dy, T *db, int64_t rows, int64_t cols) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (col < cols)
    for (int64_t r = wave; r < rows; r += 4) s += (float)dy[r * cols + col];
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
  s.partw = gemm_partial_bytes(O, I, s.tp / 64 * (s.pw == 3 ? 6 : 1));
  return s;
}

template <typename T, bool HALF>
hipError_t backward(int nc, int64_t rows, int64_t in, int64_t out, const T *x, const uint8_t *codes,
                    const uint32_t *scales, const T *dY, T *dX, T *dW, T *db, const Plan &s, char *ws,
                    hipStream_t stream) {
  const auto blocks = [](int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); };
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
      mx_stage_t_kernel<T, HALF><<<dim3(blocks(out, 64), blocks(s.tp, 64)), 256, 0, stream>>>(dY, dyt, rows, out, s.tp);
      mx_stage_t_kernel<T, HALF><<<dim3(blocks(in, 64), blocks(s.tp, 64)), 256, 0, stream>>>(x, xt, rows, in, s.tp);
    }
    // of two values in three pieces the pairs past i + j = 2 are left out: each is within 2^-26 of
    // |dY||x|, less than one rounding of the sum
    const hipError_t e = staged<T, HALF>(dyt, s.pw, xt, s.pw, out, in, s.tp, 3, dW, ws + s.dyt + s.xt, stream);
    if (e != hipSuccess) return e;
  }
  if (db) mx_colsum_kernel<T><<<blocks(out, 64), 256, 0, stream>>>(dY, db, rows, out);
  return hipGetLastError();
}

}  // namespace

int64_t mx4_linear_bwd_workspace_bytes(int dtype, int nc, int64_t batch, int64_t in, int64_t out, int dx, int dw,
                                       int db) {
  const Plan s = plan(dtype, nc, batch, in, out);
  const int64_t a = dx ? s.dy + s.wt + s.partx : 0, b = dw ? s.dyt + s.xt + s.partw : 0;
  return a > b ? a : b;
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
