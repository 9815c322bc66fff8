// abi_mx4.cpp -- the extern "C" entry points on MXFP4 tensors and of the distillation loss:
// argument validation, aliasing rules and dispatch to the kernel launchers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/mcf.h"
#include "mcf_internal.hpp"
#include "mx4.hpp"

namespace {

constexpr int MAX_NC = 4;

int64_t elem_size(int dtype) { return dtype == MCF_F32 ? 4 : 2; }

bool overlap(const void *a, int64_t abytes, const void *b, int64_t bbytes) {
  if (!a || !b || abytes <= 0 || bbytes <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

// a * b stays below 2^50, so byte counts and offsets never overflow int64; a, b >= 0.
bool elems_fit(int64_t a, int64_t b) { return b == 0 || a <= ((int64_t)1 << 50) / b; }

int hip_status(hipError_t e) { return e == hipSuccess ? MCF_OK : MCF_E_HIP; }

bool plain_format(int dtype) { return dtype == MCF_F16 || dtype == MCF_BF16 || dtype == MCF_F32; }

bool nc_ok(int nc) { return nc >= 1 && nc <= MAX_NC; }

int64_t codes_bytes(int nc, int64_t rows, int64_t n) { return nc * rows * mcf::mx_groups(n) * 64; }
int64_t scales_bytes(int nc, int64_t rows, int64_t n) { return nc * rows * mcf::mx_groups(n) * 4; }

// rows x n of an MXFP4 tensor: a workgroup takes 16 groups, of 4 or 16 rows; they are numbered with
// 31 bits.
int tensor_check(int64_t rows, int64_t n) {
  if (rows < 0 || n < 0 || rows > ((int64_t)1 << 40) || n > ((int64_t)1 << 40)) return MCF_E_SHAPE;
  const int64_t g = mcf::mx_groups(n);
  if (g >= ((int64_t)1 << 31) || (g > 0 && (rows + 15) / 16 >= ((int64_t)1 << 31) / g)) return MCF_E_SHAPE;
  return MCF_OK;
}

int matmul_check(int dtype, int64_t M, int64_t N, int64_t K, int a_nc, int b_nc) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(a_nc) || !nc_ok(b_nc)) return MCF_E_NC;
  if (M < 0 || N < 0 || K < 0) return MCF_E_SHAPE;
  if (M > ((int64_t)1 << 20) || N > ((int64_t)1 << 24) || K > ((int64_t)1 << 22)) return MCF_E_SHAPE;
  return MCF_OK;
}

int linear_check(int dtype, int nc, int64_t batch, int64_t in, int64_t out) {
  return matmul_check(dtype, batch, out, in, 1, nc);
}

int bwd_check(int dtype, int nc, int64_t batch, int64_t in, int64_t out) {
  const int st = linear_check(dtype, nc, batch, in, out);
  if (st != MCF_OK) return st;
  if (in > ((int64_t)1 << 20) || out > ((int64_t)1 << 20)) return MCF_E_SHAPE;
  return MCF_OK;
}

int distill_check(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, double temperature) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc)) return MCF_E_NC;
  if (rows < 0 || vocab < 1 || k < 0 || k > 1024) return MCF_E_SHAPE;
  if (rows >= ((int64_t)1 << 31) || vocab > ((int64_t)1 << 30) || !elems_fit(rows, vocab)) return MCF_E_SHAPE;
  const float t = (float)temperature;
  if (!(t > 0.0f) || !isfinite(t) || !isfinite(2.0f / t)) return MCF_E_ARG;
  return MCF_OK;
}

struct Span {
  const void *p;
  int64_t bytes;
};

// Whether any of the outputs overlaps an input or another output.
template <int NO, int NI>
bool outputs_overlap(const Span (&outs)[NO], const Span (&ins)[NI]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlap(outs[o].p, outs[o].bytes, ins[i].p, ins[i].bytes)) return true;
    for (int p = o + 1; p < NO; ++p)
      if (overlap(outs[o].p, outs[o].bytes, outs[p].p, outs[p].bytes)) return true;
  }
  return false;
}

int workspace_check(const void *workspace, int64_t given, int64_t needed) {
  if (needed <= 0) return MCF_OK;
  if (!workspace) return MCF_E_NULL;
  if (given < needed || !aligned(workspace, 16)) return MCF_E_ARG;
  return MCF_OK;
}

}  // namespace

extern "C" {

int mc_mx4_quantize(int dtype, int nc_in, int nc, int64_t rows, int64_t n, const void *x, void *codes, void *scales,
                    void *stream) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc_in) || !nc_ok(nc)) return MCF_E_NC;
  const int st = tensor_check(rows, n);
  if (st != MCF_OK) return st;
  if (rows == 0 || n == 0) return MCF_OK;
  if (!x || !codes || !scales) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const Span outs[2] = {{codes, codes_bytes(nc, rows, n)}, {scales, scales_bytes(nc, rows, n)}};
  const Span ins[1] = {{x, nc_in * rows * n * elem_size(dtype)}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_mx4_quantize(dtype, nc_in, nc, rows, n, x, codes, scales, (hipStream_t)stream));
}

int mc_mx4_dequantize(int dtype, int nc, int64_t rows, int64_t n, const void *codes, const void *scales, void *out,
                      void *stream) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc)) return MCF_E_NC;
  const int st = tensor_check(rows, n);
  if (st != MCF_OK) return st;
  if (rows == 0 || n == 0) return MCF_OK;
  if (!codes || !scales || !out) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const Span outs[1] = {{out, rows * n * elem_size(dtype)}};
  const Span ins[2] = {{codes, codes_bytes(nc, rows, n)}, {scales, scales_bytes(nc, rows, n)}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_mx4_dequantize(dtype, nc, rows, n, codes, scales, out, (hipStream_t)stream));
}

int64_t mc_mx4_matmul_workspace(int dtype, int64_t M, int64_t N, int64_t K, int a_nc, int b_nc) {
  const int st = matmul_check(dtype, M, N, K, a_nc, b_nc);
  if (st != MCF_OK) return st;
  return M == 0 || N == 0 ? 0 : mcf::mx4_matmul_workspace_bytes(M, N, K, a_nc, b_nc);
}

int mc_mx4_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales, int a_nc,
                  const void *b_codes, const void *b_scales, int b_nc, void *workspace, int64_t workspace_bytes,
                  void *C, void *stream) {
  const int st = matmul_check(dtype, M, N, K, a_nc, b_nc);
  if (st != MCF_OK) return st;
  if (M == 0 || N == 0) return MCF_OK;
  if (!C || (K > 0 && (!a_codes || !a_scales || !b_codes || !b_scales))) return MCF_E_NULL;
  if (!aligned(a_codes, 16) || !aligned(b_codes, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4))
    return MCF_E_ARG;
  const int64_t wb = mcf::mx4_matmul_workspace_bytes(M, N, K, a_nc, b_nc);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const Span outs[2] = {{C, M * N * elem_size(dtype)}, {workspace, wb}};
  const Span ins[4] = {{a_codes, codes_bytes(a_nc, M, K)}, {a_scales, scales_bytes(a_nc, M, K)},
                       {b_codes, codes_bytes(b_nc, N, K)}, {b_scales, scales_bytes(b_nc, N, K)}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_mx4_matmul(dtype, M, N, K, a_codes, a_scales, a_nc, b_codes, b_scales, b_nc,
                                           workspace, C, (hipStream_t)stream));
}

int64_t mc_mx4_linear_fwd_workspace(int dtype, int nc, int64_t batch, int64_t in, int64_t out) {
  const int st = linear_check(dtype, nc, batch, in, out);
  if (st != MCF_OK) return st;
  return batch == 0 || out == 0 ? 0 : mcf::mx4_linear_workspace_bytes(dtype, nc, batch, in, out);
}

int mc_mx4_linear_fwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                      const void *scales, const void *b, void *workspace, int64_t workspace_bytes, void *y,
                      void *stream) {
  const int st = linear_check(dtype, nc, batch, in, out);
  if (st != MCF_OK) return st;
  if (batch == 0 || out == 0) return MCF_OK;
  if (!y || (in > 0 && (!x || !codes || !scales))) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const int64_t wb = mcf::mx4_linear_workspace_bytes(dtype, nc, batch, in, out);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const int64_t es = elem_size(dtype);
  const Span outs[2] = {{y, batch * out * es}, {workspace, wb}};
  const Span ins[4] = {{x, batch * in * es}, {codes, codes_bytes(nc, out, in)}, {scales, scales_bytes(nc, out, in)},
                       {b, out * es}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_mx4_linear(dtype, nc, batch, in, out, x, codes, scales, b, workspace, y,
                                           (hipStream_t)stream));
}

int64_t mc_mx4_linear_bwd_workspace(int dtype, int nc, int64_t batch, int64_t in, int64_t out) {
  const int st = bwd_check(dtype, nc, batch, in, out);
  if (st != MCF_OK) return st;
  return mcf::mx4_linear_bwd_workspace_bytes(dtype, nc, batch, in, out, batch > 0 && in > 0, in > 0 && out > 0,
                                             out > 0);
}

int mc_mx4_linear_bwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                      const void *scales, const void *dY, void *dX, void *dW, void *db, void *workspace,
                      int64_t workspace_bytes, void *stream) {
  const int st = bwd_check(dtype, nc, batch, in, out);
  if (st != MCF_OK) return st;
  // outputs with no elements are not computed
  if (batch == 0 || in == 0) dX = nullptr;
  if (out == 0 || in == 0) dW = nullptr;
  if (out == 0) db = nullptr;
  if (!dX && !dW && !db) return MCF_OK;
  if (batch > 0 && out > 0 && !dY) return MCF_E_NULL;
  if (dX && out > 0 && (!codes || !scales)) return MCF_E_NULL;
  if (dW && batch > 0 && !x) return MCF_E_NULL;
  if (dX && (!aligned(codes, 16) || !aligned(scales, 4))) return MCF_E_ARG;
  const int64_t wb = mcf::mx4_linear_bwd_workspace_bytes(dtype, nc, batch, in, out, dX != nullptr, dW != nullptr,
                                                         db != nullptr);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const int64_t es = elem_size(dtype);
  const Span outs[4] = {{dX, batch * in * es}, {dW, out * in * es}, {db, out * es}, {workspace, wb}};
  const Span ins[4] = {{x, dW ? batch * in * es : 0},
                       {codes, dX ? codes_bytes(nc, out, in) : 0},
                       {scales, dX ? scales_bytes(nc, out, in) : 0},
                       {dY, batch * out * es}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_mx4_linear_bwd(dtype, nc, batch, in, out, x, codes, scales, dY, dX, dW, db, workspace,
                                               (hipStream_t)stream));
}

int64_t mc_distill_workspace(int64_t rows, int64_t vocab) {
  const int st = distill_check(MCF_F32, 1, rows, vocab, 0, 1.0);
  return st != MCF_OK ? st : mcf::distill_workspace_bytes(rows, vocab);
}

static int distill(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                   const void *t, double temperature, const void *g, void *workspace, int64_t workspace_bytes,
                   void *loss, void *stats, void *dz, bool grad, void *stream) {
  const int st = distill_check(dtype, nc, rows, vocab, k, temperature);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!z || !loss || (grad && !dz) || (k > 0 && (!ids || !t))) return MCF_E_NULL;
  if (!aligned(ids, 4) || !aligned(g, 4) || !aligned(loss, 4) || !aligned(stats, 4)) return MCF_E_ARG;
  const int64_t wb = mcf::distill_workspace_bytes(rows, vocab), es = elem_size(dtype);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const Span outs[4] = {{loss, 4 * rows}, {stats, 8 * rows}, {dz, rows * vocab * es}, {workspace, wb}};
  const Span ins[4] = {{z, nc * rows * vocab * es}, {ids, rows * k * 4}, {t, rows * k * es}, {g, rows * 4}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_distill(dtype, nc, rows, vocab, k, z, ids, t, temperature, nullptr, g, workspace, loss,
                                        stats, dz, (hipStream_t)stream));
}

int mc_distill_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                   const void *t, double temperature, void *workspace, int64_t workspace_bytes, void *loss,
                   void *stats, void *stream) {
  return distill(dtype, nc, rows, vocab, k, z, ids, t, temperature, nullptr, workspace, workspace_bytes, loss, stats,
                 nullptr, false, stream);
}

int mc_distill_fwd_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                       const void *t, double temperature, const void *g, void *workspace, int64_t workspace_bytes,
                       void *loss, void *dz, void *stream) {
  return distill(dtype, nc, rows, vocab, k, z, ids, t, temperature, g, workspace, workspace_bytes, loss, nullptr, dz,
                 true, stream);
}

int mc_distill_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                   const void *t, double temperature, const void *stats, const void *g, void *dz, void *stream) {
  const int st = distill_check(dtype, nc, rows, vocab, k, temperature);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!z || !stats || !dz || (k > 0 && (!ids || !t))) return MCF_E_NULL;
  if (!aligned(ids, 4) || !aligned(g, 4) || !aligned(stats, 4)) return MCF_E_ARG;
  const int64_t es = elem_size(dtype);
  const Span outs[1] = {{dz, rows * vocab * es}};
  const Span ins[5] = {{z, nc * rows * vocab * es}, {ids, rows * k * 4}, {t, rows * k * es}, {g, rows * 4},
                       {stats, 8 * rows}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_distill(dtype, nc, rows, vocab, k, z, ids, t, temperature, stats, g, nullptr, nullptr,
                                        nullptr, dz, (hipStream_t)stream));
}

}  // extern "C"
