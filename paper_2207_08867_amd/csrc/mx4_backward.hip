// mx4_backward.hip -- the gradients of the linear layer y = x W^T + b with an MXFP4 weight:
//   dX = dY W,  dW = dY^T x (the gradient of the numbers that W stands for),  db = column sums of dY.
//
// Both products reduce over an index that is not the fastest one of their operands, so the
// operands are first staged: rows of the reduction, padded with zeros to whole groups of 128, as
// 16-bit pieces whose sums are the values exactly (bfloat16; binary16 for dW of binary16 tensors,
// which is one piece).  W is staged as its components' numbers, exact in bfloat16.  Then both are
// products A B^T of staged tensors, summed over pairs of pieces in binary32.  They go out in one launch
// where the time model finds that faster.
//
// Measured (MI355X, 4096 x 1024 -> 1024, binary16, one component): 48 us in all; staging 12.4, both
// products 34 (the matrix instructions of three bfloat16-sized products take 18 at the rate of a large
// one), the sum of dW's slices 4.9, db 3.9.  bfloat16 41, binary32 124 (nine products of pieces, three for
// dX and six for dW).  4096 x 4096 -> 4096: 359, 254 and 998 us.
#include "mcf_internal.hpp"
#include "mx4.hpp"
#include "mx4_gemm.hpp"

namespace mcf {
namespace {

// What is staged for the two products, all of it in one launch: workgroups [0, n_dy) take tiles of dY,
// the next n_x tiles of x, the last n_w tiles of W.
struct StageArgs {
  const void *dY, *x;            // [T][O], [T][I]
  const uint8_t *codes;          // W, [nc][O][64 groups] and its scales
  const uint32_t *scales;
  uint16_t *dy, *dyt, *xt, *wt;  // [P][T][op], [P'][O][tp], [P'][I][tp], [nc][I][op]; dy or dyt may be null
  float *sums;                   // [tp / 128][O] column sums of dY's tiles, or null
  void *db;                      // with a single row of tiles their sums are db itself
  int64_t T, O, I, op, tp, groups, n_dy, n_x;
};

constexpr int TILE_ROW = 66;  // halfwords: the rows of one column lie in different banks

// A tile of 128 rows x 64 columns of src [rows][cols]: its pieces as they lie to plain [P][rows][pld]
// (zeros up to pld), transposed to dst [P'][cols][ld] (zeros up to ld), its columns' sums to sums
// [tiles of rows][cols].  A wavefront reads 8 rows of 64 columns in one instruction (16-bit
// formats) and writes 16 bytes a lane, 8 rows of one column.
template <typename T, bool HALF>
__device__ inline void stage_tile(const T *src, uint16_t *plain, uint16_t *dst, float *sums, T *whole, int64_t rows,
                                  int64_t cols, int64_t pld, int64_t ld, int64_t row_tile, int64_t col_tile, char *lds) {
  constexpr int P = mx_pieces<T>(), PW = HALF ? 1 : P;
  uint16_t(*tile)[128][TILE_ROW] = reinterpret_cast<uint16_t(*)[128][TILE_ROW]>(lds);
  const int64_t c0 = col_tile * 64, r0 = row_tile * 128;
  float part[8] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
    Raw8<T> v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v.v[k] = (T)0.0f;
    if (r0 + r < rows) v = load8_tail(src + (r0 + r) * cols + c0 + c, cols - c0 - c);
    bf16x8 f[P];
    if constexpr (P == 3) {  // dW leaves pairs of pieces out; dX takes the same ones
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        __bf16 p[3];
        mx_round3(v.v[k], p);
#pragma unroll
        for (int q = 0; q < 3; ++q) f[q][k] = p[q];
      }
    } else {
      mx_cut8<T, P>(v, f);
    }
    if (plain && r0 + r < rows) {
#pragma unroll
      for (int q = 0; q < P; ++q)
        *reinterpret_cast<bf16x8 *>(plain + ((int64_t)q * rows + r0 + r) * pld + c0 + c) = f[q];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (P == 3) {
#pragma unroll
        for (int q = 0; q < 3; ++q) tile[q][r][c + k] = __builtin_bit_cast(uint16_t, (__bf16)f[q][k]);
      } else {
        tile[0][r][c + k] = __builtin_bit_cast(uint16_t, v.v[k]);
      }
      part[k] += (float)v.v[k];
    }
  }
  __syncthreads();
  if (dst) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = i * 16 + (threadIdx.x >> 4), r = (threadIdx.x & 15) * 8;
      if (c0 + c < cols) {
#pragma unroll
        for (int q = 0; q < PW; ++q) {
          uint16_t out[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) out[k] = tile[q][r + k][c];
          __builtin_memcpy(dst + ((int64_t)q * cols + c0 + c) * ld + r0 + r, out, 16);
        }
      }
    }
  }
  if (sums || whole) {
    __syncthreads();
    float(*f)[64] = reinterpret_cast<float(*)[64]>(lds);  // 32 groups of lanes, 64 columns
#pragma unroll
    for (int k = 0; k < 8; ++k) f[threadIdx.x >> 3][(threadIdx.x & 7) * 8 + k] = part[k];
    __syncthreads();
    if (threadIdx.x < 64 && c0 + threadIdx.x < cols) {
      float t = 0.0f;
      for (int i = 0; i < 32; ++i) t += f[i][threadIdx.x];
      if (whole)
        whole[c0 + threadIdx.x] = (T)t;
      else
        sums[row_tile * cols + c0 + threadIdx.x] = t;
    }
  }
}

// The numbers of one group of 128 columns of 64 rows of W, transposed into wt [nc][in][op].
__device__ inline void unpack_tile(const StageArgs &a, int64_t grp, int64_t row_tile, int64_t c, char *lds) {
  uint16_t(*tile)[72] = reinterpret_cast<uint16_t(*)[72]>(lds);  // [element][row], rows 16 bytes aligned
  const int64_t r0 = row_tile * 64;
  for (int i = threadIdx.x; i < 1024; i += 256) {  // 64 rows x 16 pieces of 8 elements
    const int r = i >> 4, piece = i & 15;
    uint32_t word = 0, byte = 0;
    if (r0 + r < a.O) {
      word = *reinterpret_cast<const uint32_t *>(a.codes + (c * a.O + r0 + r) * (a.groups * 64) + grp * 64 + piece * 4);
      byte = (a.scales[(c * a.groups + grp) * a.O + r0 + r] >> (8 * (piece >> 2))) & 255u;
    }
    const bf16x8 v = mx_bf16(word, mx_scale(byte));
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[piece * 8 + k][r] = __builtin_bit_cast(uint16_t, (__bf16)v[k]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 128 * 8; i += 256) {
    const int k = i >> 3, r = (i & 7) * 8;
    if (grp * 128 + k < a.I)
      *reinterpret_cast<u32x4 *>(a.wt + (c * a.I + grp * 128 + k) * a.op + r0 + r) =
          *reinterpret_cast<const u32x4 *>(&tile[k][r]);
  }
}

template <typename T, bool HALF>
__global__ __launch_bounds__(256) void mx_stage_all_kernel(StageArgs a) {
  constexpr int BYTES = (HALF ? 1 : mx_pieces<T>()) * 128 * TILE_ROW * 2;
  __shared__ __attribute__((aligned(16))) char lds[BYTES > 128 * 144 ? BYTES : 128 * 144];
  int64_t id = blockIdx.x;
  if (id < a.n_dy) {
    const int64_t across = a.op / 64;
    stage_tile<T, HALF>(reinterpret_cast<const T *>(a.dY), a.dy, a.dyt, a.sums, reinterpret_cast<T *>(a.db), a.T, a.O,
                        a.op, a.tp, id / across, id % across, lds);
  } else if (id < a.n_dy + a.n_x) {
    id -= a.n_dy;
    const int64_t across = (a.I + 63) / 64;
    stage_tile<T, HALF>(reinterpret_cast<const T *>(a.x), nullptr, a.xt, nullptr, nullptr, a.T, a.I, 0, a.tp, id / across,
                        id % across, lds);
  } else {
    id -= a.n_dy + a.n_x;
    const int64_t grp = id % a.groups, row_tile = id / a.groups % (a.op / 64);
    unpack_tile(a, grp, row_tile, id / (a.groups * (a.op / 64)), lds);
  }
}

// The pairs (i, j) of pieces with i + j < `below`.
void set_pairs(GemmArgs &a, int na, int nb, int below) {
  for (int i = 0; i < na; ++i)
    for (int j = 0; j < nb; ++j)
      if (i + j < below) gemm_pair(a, i, j);
}

// C [M][N] from staged a [na][M][ld] and b [nb][N][ld], pairs i + j < below.
GemmArgs staged(const uint16_t *a, int na, const uint16_t *b, int nb, int64_t M, int64_t N, int64_t ld, int below, void *c,
                void *partial) {
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
  return g;
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
// [P'][I][Tp], Op and Tp whole groups; db the column sums of dY's tiles.
struct Plan {
  int p, pw;                // pieces of a plain element: for dX, for dW
  int64_t op, tp;           // padded reductions
  int64_t dy, wt, dyt, xt;  // bytes of the staged operands
  int64_t partx, partw;     // of the products' partial sums
  int64_t sums;             // of the column sums
  // dX and dW in one launch where two.tile is not 0; planx and planw their tiles and slices, those of the
  // call for every gradient also where one alone is asked for, so that its bits are the same
  GemmTwoPlan two;
  GemmPlan planx, planw;
};

Plan plan(int dtype, int nc, int64_t T, int64_t I, int64_t O, bool dx, bool dw, bool db) {
  Plan s;
  s.p = dtype == LM_F32 ? 3 : (dtype == LM_F16 ? 2 : 1);
  s.pw = dtype == LM_F32 ? 3 : 1;
  s.op = up(O, MX_GROUP);
  s.tp = up(T, MX_GROUP);
  s.dy = dx ? up(s.p * T * s.op * 2, 256) : 0;
  s.wt = dx ? up(nc * I * s.op * 2, 256) : 0;
  const int64_t steps_x = s.op / 64 * s.p * nc, steps_w = s.tp / 64 * (s.pw == 3 ? 6 : 1);
  s.two = gemm_two_plan(T, I, steps_x, O, I, steps_w);
  s.planx = s.two.tile ? GemmPlan{s.two.tile, s.two.slices1} : gemm_plan(T, I, steps_x);
  s.planw = s.two.tile ? GemmPlan{s.two.tile, s.two.slices2} : gemm_plan(O, I, steps_w);
  s.partx = dx ? up(gemm_slices_bytes(T, I, s.planx.slices), 256) : 0;
  s.dyt = dw ? up(s.pw * O * s.tp * 2, 256) : 0;
  s.xt = dw ? up(s.pw * I * s.tp * 2, 256) : 0;
  s.partw = dw ? up(gemm_slices_bytes(O, I, s.planw.slices), 256) : 0;
  s.sums = db ? up(s.tp / 128 * O * 4, 256) : 0;
  return s;
}

template <typename T, bool HALF>
hipError_t backward(int nc, int64_t rows, int64_t in, int64_t out, const T *x, const uint8_t *codes,
                    const uint32_t *scales, const T *dY, T *dX, T *dW, T *db, const Plan &s, char *ws,
                    hipStream_t stream) {
  const auto take = [&](int64_t bytes) {
    char *p = ws;
    ws += bytes;
    return p;
  };
  StageArgs a = {};
  a.dY = dY;
  a.x = x;
  a.codes = codes;
  a.scales = scales;
  a.T = rows;
  a.O = out;
  a.I = in;
  a.op = s.op;
  a.tp = s.tp;
  a.groups = mx_groups(in);
  uint16_t *dy = (uint16_t *)take(s.dy), *wt = (uint16_t *)take(s.wt);
  char *partx = take(s.partx);
  uint16_t *dyt = (uint16_t *)take(s.dyt), *xt = (uint16_t *)take(s.xt);
  char *partw = take(s.partw);
  float *sums = (float *)take(s.sums);
  const int64_t row_tiles = s.tp / 128;
  int64_t n_w = 0;
  if (rows > 0 && out > 0) {
    a.n_dy = row_tiles * (s.op / 64);
    if (dX) {
      a.dy = dy;
      a.wt = wt;
      n_w = a.groups * (s.op / 64) * nc;
    }
    if (dW) {
      a.dyt = dyt;
      a.xt = xt;
      a.n_x = row_tiles * ((in + 63) / 64);
    }
    if (db) {
      a.sums = sums;
      if (row_tiles == 1) a.db = db;
    }
    mx_stage_all_kernel<T, HALF><<<(unsigned)(a.n_dy + a.n_x + n_w), 256, 0, stream>>>(a);
  }
  // Reductions of nothing give zeros.  Of two values in three pieces the pairs past i + j = 2 are
  // left out of dW, a third of its products: (1, 2) and (2, 1) are at most 2^-25 of |dY||x| each, all
  // three just above 2^-24, as much as one rounding of a product to binary32.
  GemmArgs gx = staged(dy, s.p, wt, nc, rows, in, s.op, s.p + nc, dX, partx);
  GemmArgs gw = staged(dyt, s.pw, xt, s.pw, out, in, s.tp, 3, dW, partw);
  constexpr GemmKind KW = HALF ? GEMM_F16 : GEMM_BF16;
  hipError_t e = hipSuccess;
  if (dX && dW && s.two.tile) {
    e = gemm_two<GEMM_BF16, KW, T>(gx, gw, s.two, stream);
  } else {
    if (dX) e = gemm<GEMM_BF16, T>(gx, s.planx, stream);
    if (dW && e == hipSuccess) e = gemm<KW, T>(gw, s.planw, stream);
  }
  if (e != hipSuccess) return e;
  if (db && row_tiles != 1) mx_db_kernel<T><<<(unsigned)((out + 63) / 64), 256, 0, stream>>>(sums, db, row_tiles, out);
  return hipGetLastError();
}

}  // namespace

int64_t mx4_linear_bwd_workspace_bytes(int dtype, int nc, int64_t batch, int64_t in, int64_t out, int dx, int dw,
                                       int db) {
  const Plan s = plan(dtype, nc, batch, in, out, dx, dw, db);
  return s.dy + s.wt + s.partx + s.dyt + s.xt + s.partw + s.sums;
}

hipError_t launch_mx4_linear_bwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x,
                                 const void *codes, const void *scales, const void *dY, void *dX, void *dW, void *db,
                                 void *ws, hipStream_t stream) {
  const Plan s = plan(dtype, nc, batch, in, out, dX != nullptr, dW != nullptr, db != nullptr);
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
