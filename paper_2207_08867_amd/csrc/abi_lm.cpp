// abi_lm.cpp -- the extern "C" entry points of the RMS norm, of 8-bit tensors and of the log probabilities
// of tokens: argument validation, aliasing rules and dispatch to the kernel launchers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "abi_checks.hpp"
#include "int8.hpp"
#include "mcf_internal.hpp"

namespace {

constexpr int64_t ROW_MAX = (int64_t)1 << 30;  // elements of a row

int64_t codes_bytes(int64_t rows, int64_t n) { return rows * mcf::int8_pitch(n); }

// rows x n of a plain, MC or 8-bit tensor, of up to 4 planes.
int rows_check(int64_t rows, int64_t n) {
  if (rows < 0 || n < 0 || rows > ((int64_t)1 << 40) || n > ROW_MAX) return MCF_E_SHAPE;
  return elems_fit(rows, mcf::int8_pitch(n)) ? MCF_OK : MCF_E_SHAPE;
}

int norm_check(int dtype, int nc, int64_t rows, int64_t n, double eps) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc)) return MCF_E_NC;
  const int st = rows_check(rows, n);
  if (st != MCF_OK) return st;
  if (n < 1) return MCF_E_SHAPE;
  return eps >= 0.0 && isfinite(eps) ? MCF_OK : MCF_E_ARG;
}

// A norm's call with the outputs given (bytes 0: not that call's).
int norm_call(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w, double eps,
              void *h_out, void *y, void *codes, void *scales, bool int8, void *stream) {
  const int st = norm_check(dtype, nc, rows, n, eps);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!h || (x && !h_out) || (int8 ? !codes || !scales : !y)) return MCF_E_NULL;
  if (!x && h_out) return MCF_E_ARG;
  if (int8 && (!aligned(codes, 16) || !aligned(scales, 4))) return MCF_E_ARG;
  const int64_t es = elem_size(dtype), plane = rows * n * es;
  const Span outs[4] = {{h_out, nc * plane}, {y, plane}, {codes, codes_bytes(rows, n)}, {scales, 4 * rows}};
  // in place: the stream behind the addition may be the stream itself
  const Span ins[3] = {{h_out == h ? nullptr : h, nc * plane}, {x, plane}, {w, n * es}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_rmsnorm(dtype, nc, rows, n, h, x, w, eps, h_out, y, codes, scales, true,
                                        (hipStream_t)stream));
}

// The exact sums stay below 2^31 while K 127^2 does.
constexpr int64_t K_MAX = 131072;

int matmul_check(int dtype, int64_t M, int64_t N, int64_t K) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (M < 0 || N < 0 || K < 0) return MCF_E_SHAPE;
  if (M > ((int64_t)1 << 20) || N > ((int64_t)1 << 24) || K > K_MAX) return MCF_E_SHAPE;
  return MCF_OK;
}

int logprobs_check(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, int64_t top, double temperature) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc)) return MCF_E_NC;
  if (rows < 0 || vocab < 1 || given < 0 || given > mcf::LOGP_GIVEN || top < 0 || top > mcf::LOGP_TOP) return MCF_E_SHAPE;
  if (rows >= ((int64_t)1 << 31) || vocab > ROW_MAX || !elems_fit(rows, vocab)) return MCF_E_SHAPE;
  const float t = (float)temperature;
  if (!(t > 0.0f) || !isfinite(t) || !isfinite(2.0f / t)) return MCF_E_ARG;
  return MCF_OK;
}

}  // namespace

extern "C" {

int mc_rmsnorm_fwd(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w, double eps,
                   void *h_out, void *y, void *stream) {
  return norm_call(dtype, nc, rows, n, h, x, w, eps, h_out, y, nullptr, nullptr, false, stream);
}

int mc_rmsnorm_int8(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w, double eps,
                    void *h_out, void *codes, void *scales, void *stream) {
  return norm_call(dtype, nc, rows, n, h, x, w, eps, h_out, nullptr, codes, scales, true, stream);
}

int64_t mc_rmsnorm_bwd_workspace(int dtype, int64_t rows, int64_t n) {
  const int st = norm_check(dtype, 1, rows, n, 0.0);
  return st != MCF_OK ? st : mcf::rmsnorm_bwd_workspace_bytes(dtype, rows, n);
}

int mc_rmsnorm_bwd(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *w, const void *dy,
                   const void *g, double eps, void *dh, void *dw, void *workspace, int64_t workspace_bytes,
                   void *stream) {
  const int st = norm_check(dtype, nc, rows, n, eps);
  if (st != MCF_OK) return st;
  if (rows == 0) dh = nullptr;
  if (!dh && !dw) return MCF_OK;
  if (rows > 0 && (!h || !dy)) return MCF_E_NULL;
  const int64_t wb = dw ? mcf::rmsnorm_bwd_workspace_bytes(dtype, rows, n) : 0;
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const int64_t es = elem_size(dtype), plane = rows * n * es;
  const Span outs[3] = {{dh, plane}, {dw, n * es}, {workspace, wb}};
  const Span ins[4] = {{h, nc * plane}, {w, n * es}, {dy, plane}, {g, plane}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_rmsnorm_bwd(dtype, nc, rows, n, h, w, dy, g, eps, dh, dw, workspace,
                                            (hipStream_t)stream));
}

int mc_int8_quantize(int dtype, int nc_in, int64_t rows, int64_t n, const void *x, void *codes, void *scales,
                     void *stream) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  if (!nc_ok(nc_in)) return MCF_E_NC;
  const int st = rows_check(rows, n);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!scales || (n > 0 && (!x || !codes))) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const Span outs[2] = {{codes, codes_bytes(rows, n)}, {scales, 4 * rows}};
  const Span ins[1] = {{x, nc_in * rows * n * elem_size(dtype)}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_rmsnorm(dtype, nc_in, rows, n, x, nullptr, nullptr, 0.0, nullptr, nullptr, codes, scales,
                                        false, (hipStream_t)stream));
}

int mc_int8_dequantize(int dtype, int64_t rows, int64_t n, const void *codes, const void *scales, void *out,
                       void *stream) {
  if (!plain_format(dtype)) return MCF_E_DTYPE;
  const int st = rows_check(rows, n);
  if (st != MCF_OK) return st;
  if (rows == 0 || n == 0) return MCF_OK;
  if (!codes || !scales || !out) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const Span outs[1] = {{out, rows * n * elem_size(dtype)}};
  const Span ins[2] = {{codes, codes_bytes(rows, n)}, {scales, 4 * rows}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_int8_dequantize(dtype, rows, n, codes, scales, out, (hipStream_t)stream));
}

int64_t mc_int8_matmul_workspace(int dtype, int64_t M, int64_t N, int64_t K) {
  const int st = matmul_check(dtype, M, N, K);
  if (st != MCF_OK) return st;
  return M == 0 || N == 0 ? 0 : mcf::int8_matmul_workspace_bytes(M, N, K);
}

int mc_int8_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales,
                   const void *b_codes, const void *b_scales, const void *bias, void *workspace,
                   int64_t workspace_bytes, void *C, void *stream) {
  const int st = matmul_check(dtype, M, N, K);
  if (st != MCF_OK) return st;
  if (M == 0 || N == 0) return MCF_OK;
  if (!C || !a_scales || !b_scales || (K > 0 && (!a_codes || !b_codes))) return MCF_E_NULL;
  if (!aligned(a_codes, 16) || !aligned(b_codes, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4))
    return MCF_E_ARG;
  const int64_t wb = mcf::int8_matmul_workspace_bytes(M, N, K), es = elem_size(dtype);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const Span outs[2] = {{C, M * N * es}, {workspace, wb}};
  const Span ins[5] = {{a_codes, codes_bytes(M, K)}, {a_scales, 4 * M}, {b_codes, codes_bytes(N, K)},
                       {b_scales, 4 * N}, {bias, N * es}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_int8_matmul(dtype, M, N, K, a_codes, a_scales, b_codes, b_scales, bias, workspace, C,
                                            (hipStream_t)stream));
}

int64_t mc_int8_linear_fwd_workspace(int dtype, int64_t batch, int64_t in, int64_t out) {
  const int st = matmul_check(dtype, batch, out, in);
  if (st != MCF_OK) return st;
  return batch == 0 || out == 0 ? 0 : mcf::int8_linear_workspace_bytes(batch, in, out);
}

int mc_int8_linear_fwd(int dtype, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                       const void *scales, const void *b, void *workspace, int64_t workspace_bytes, void *y,
                       void *stream) {
  const int st = matmul_check(dtype, batch, out, in);
  if (st != MCF_OK) return st;
  if (batch == 0 || out == 0) return MCF_OK;
  if (!y || !scales || (in > 0 && (!x || !codes))) return MCF_E_NULL;
  if (!aligned(codes, 16) || !aligned(scales, 4)) return MCF_E_ARG;
  const int64_t wb = mcf::int8_linear_workspace_bytes(batch, in, out), es = elem_size(dtype);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const Span outs[2] = {{y, batch * out * es}, {workspace, wb}};
  const Span ins[4] = {{x, batch * in * es}, {codes, codes_bytes(out, in)}, {scales, 4 * out}, {b, out * es}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_int8_linear(dtype, batch, in, out, x, codes, scales, b, workspace, y,
                                            (hipStream_t)stream));
}

int64_t mc_logprobs_workspace(int64_t rows, int64_t vocab, int64_t top) {
  const int st = logprobs_check(MCF_F32, 1, rows, vocab, 0, top, 1.0);
  return st != MCF_OK ? st : mcf::logprobs_workspace_bytes(rows, vocab, top);
}

int mc_logprobs_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, int64_t top, const void *z,
                    const void *ids, double temperature, void *workspace, int64_t workspace_bytes, void *logp,
                    void *entropy, void *top_ids, void *top_logp, void *stats, void *stream) {
  const int st = logprobs_check(dtype, nc, rows, vocab, given, top, temperature);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!z || (given > 0 && (!ids || !logp)) || (top > 0 && (!top_ids || !top_logp))) return MCF_E_NULL;
  if (!aligned(ids, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(top_ids, 4) || !aligned(top_logp, 4) ||
      !aligned(stats, 4))
    return MCF_E_ARG;
  const int64_t wb = mcf::logprobs_workspace_bytes(rows, vocab, top);
  const int ws = workspace_check(workspace, workspace_bytes, wb);
  if (ws != MCF_OK) return ws;
  const Span outs[6] = {{logp, 4 * rows * given}, {entropy, 4 * rows},  {top_ids, 4 * rows * top},
                        {top_logp, 4 * rows * top}, {stats, 12 * rows}, {workspace, wb}};
  const Span ins[2] = {{z, nc * rows * vocab * elem_size(dtype)}, {ids, 4 * rows * given}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_logprobs_fwd(dtype, nc, rows, vocab, given, top, z, ids, temperature, workspace, logp,
                                             entropy, top_ids, top_logp, stats, (hipStream_t)stream));
}

int mc_logprobs_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, const void *z, const void *ids,
                    double temperature, const void *stats, const void *g, const void *g_entropy, void *dz,
                    void *stream) {
  const int st = logprobs_check(dtype, nc, rows, vocab, given, 0, temperature);
  if (st != MCF_OK) return st;
  if (rows == 0) return MCF_OK;
  if (!z || !stats || !dz || (given > 0 && !ids)) return MCF_E_NULL;
  if (!aligned(ids, 4) || !aligned(stats, 4) || !aligned(g, 4) || !aligned(g_entropy, 4)) return MCF_E_ARG;
  const int64_t es = elem_size(dtype);
  const Span outs[1] = {{dz, rows * vocab * es}};
  const Span ins[5] = {{z, nc * rows * vocab * es}, {ids, 4 * rows * given}, {stats, 12 * rows},
                       {g, 4 * rows * given}, {g_entropy, 4 * rows}};
  if (outputs_overlap(outs, ins)) return MCF_E_ALIAS;
  return hip_status(mcf::launch_logprobs_bwd(dtype, nc, rows, vocab, given, z, ids, temperature, stats, g, g_entropy, dz,
                                             (hipStream_t)stream));
}

}  // extern "C"
