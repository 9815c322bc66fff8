/*
 * mcf.h -- C ABI of the MI355X (gfx950) multi-component floating-point library.
 *
 * Arithmetic follows "MCTensor: A High-Precision Deep Learning Library with
 * Multi-Component Floating-Point" (arXiv 2207.08867).  A multi-component (MC) value
 * is an unevaluated sum x = x_0 + x_1 + ... + x_{nc-1} of nc floating-point
 * components of one format, largest first (Section 2, the MCF expansion equation).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Memory.  All tensor pointers are DEVICE pointers owned by the caller; the library
 *   allocates nothing per call and keeps no state besides two static per-device
 *   arrays: a binary16 exponential table (128 KiB, built on the first mc_exp call on
 *   a device) and the 8 MiB scratch of mc_matmul_splitk_noalloc.  Calls that need
 *   scratch memory (mc_matmul_splitk, mc_matmul_exact, mc_linreg_gd_step, the MXFP4
 *   products, the distillation loss, the norm's gradients, the 8-bit products, the log
 *   probabilities) take a caller-owned workspace.
 * Layout.  Dense, component-major ("planar"): component c of element i of an MC
 *   array of n elements is at element offset c*n + i.  A plain tensor is one plane.
 *   Matrices are row-major inside each plane.  The paper's interleaved layout
 *   (components in the last dimension) converts with a transpose on the caller side.
 * Formats.  MCF_F16 = IEEE binary16 components, MCF_F32 = IEEE binary32, MCF_F64 =
 *   IEEE binary64 (the paper's MC float64).  Every step of every algorithm is one IEEE
 *   round-to-nearest-even operation in the component format with gradual underflow;
 *   FMA appears only where the algorithm names it (Two-Prod); component division is
 *   correctly rounded; the component exponentials are correctly rounded in every
 *   format.  mc_matmul_exact takes MCF_F16 only.
 *   MCF_F16S = binary16 components with scaled low components (Section 2.4 names
 *   scaling the smaller components as the way past binary16's smallest subnormal):
 *   component c is stored as the binary16 number y_c and stands for 2^(-11 c) y_c.
 *   The algorithms are the same, with every quantity at a level and every rounding
 *   taken in the binary16 format of its level, fl_l(v) = 2^(-11 l) RN16(2^(11 l) v):
 *   the operands of an operation share a level (component i of an operand is at
 *   level i; a product is at the sum of its factors' levels), the errors of Two-Sum
 *   and Two-Prod and the carry built from them are at the next level, and a value
 *   Simple-Renorm moves to an earlier slot j is rounded into level j.  Only
 *   operations whose operands pair equal levels take MCF_F16S: mc_add (MC, MC
 *   only), mc_mul (MC, T and T, MC only), mc_matmul (MC x MC by the level-aligned
 *   parts described there) and mc_linear_fwd; every other call returns MCF_E_DTYPE.
 *   Non-finite components are outside this format's contract.
 * Operand kinds.  Binary operations take an MC value and a plain tensor in either
 *   order, or two MC values (Section 2.1).  The flags x_mc / y_mc / a_mc / b_mc are 1
 *   for an MC operand of nc planes and 0 for a plain tensor of one plane; at least
 *   one operand must be MC.  Results always have nc components.
 * nc.  1 <= nc <= 4.
 * Streams.  Work is enqueued on `stream` (a hipStream_t; NULL = the null stream) and
 *   runs asynchronously; nothing synchronises.  Calls on different streams are
 *   independent.  The library is reentrant.
 * Graph capture.  A call launches kernels only (no allocation, memset or
 *   synchronisation), so it may be captured into a HIP graph on `stream` -- except
 *   the first binary16 mc_exp call on a device, which builds the exponential table and
 *   waits for it; make that call once before capturing.
 * Aliasing.  Elementwise calls allow `out` to be exactly `x` or `y` (in place);
 *   any other overlap of out with an input is rejected (MCF_E_ALIAS).  Matrix calls
 *   reject any overlap of the output with an input.
 * Degenerate sizes.  n = 0 (or M*N = 0) returns MCF_OK without launching; a
 *   reduction length of 0 gives +0 in every output component.
 * Size limits.  Each entry point states its own; in addition every matrix of a
 *   product (M*K, K*N, M*N elements per plane) must stay below 2^50 elements, else
 *   MCF_E_SHAPE.
 * Errors.  Every call returns MCF_OK (0) or a negative mcf_status; on error nothing
 *   is launched.  Launch failures are reported as MCF_E_HIP.  Input values are not
 *   inspected: non-finite components propagate by IEEE rules.
 */
#ifndef MCF_H
#define MCF_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* MCF_BF16 (bfloat16) is taken by the mc_mx4_*, mc_distill_*, mc_rmsnorm_*, mc_int8_* and
 * mc_logprobs_* calls alone; those take MCF_F16, MCF_BF16 and MCF_F32. */
typedef enum { MCF_F16 = 0, MCF_F32 = 1, MCF_F64 = 2, MCF_F16S = 3, MCF_BF16 = 4 } mcf_dtype;

typedef enum {
  MCF_OK = 0,
  MCF_E_NULL = -1,  /* a required pointer is NULL */
  MCF_E_NC = -2,    /* nc (or nc_out) out of range */
  MCF_E_SHAPE = -3, /* negative size, or a size the kernels cannot index */
  MCF_E_DTYPE = -4, /* unknown format, or an operation not provided for it */
  MCF_E_ALIAS = -5, /* output overlaps an input in a way that is not allowed */
  MCF_E_HIP = -6,   /* the HIP runtime reported an error */
  MCF_E_ARG = -7,   /* any other invalid argument (operand kinds, mode) */
  MCF_E_SCRATCH = -8 /* the call needs more than the library's static scratch */
} mcf_status;

/* Addition (Section 2.1; Appendix A.2.1).
 *   (MC, MC): Add-MCN -- per component, Two-Sum of the operands, Two-Sum with the
 *             carry, carry = fl(e1 + e2); the nc+1 terms pass through Simple-Renorm.
 *   (MC, T), (T, MC): Grow-ExpN -- a chain of Two-Sums from the last component up,
 *             then Simple-Renorm to nc components.
 * x, y: [nc or 1][n]; out: [nc][n]. */
int mc_add(int dtype, int nc, int64_t n, const void *x, int x_mc, const void *y, int y_mc, void *out,
           void *stream);

/* Multiplication (Section 2.1; Appendix A.2.1).
 *   (MC, T), (T, MC): ScalingN without expand -- per component Two-Prod (FMA
 *             variant), Two-Sum with the carry, carry = fl(e1 + e2); Simple-Renorm.
 *   (MC, MC): Mult-MCN, fast version -- Renormalize(Div-MCN(x, Renormalize(
 *             Div-MCN((1, 0, ..., 0), y)))).
 * x, y: [nc or 1][n]; out: [nc][n]. */
int mc_mul(int dtype, int nc, int64_t n, const void *x, int x_mc, const void *y, int y_mc, void *out,
           void *stream);

/* Division (Appendix A.2.1).
 *   (MC, MC): Div-MCN -- long division: q = fl(x_0 / y_0), then nc times
 *             x = Add-MCN(x, -ScalingN(y, q)), q = fl(x_0 / y_0); the nc+1 quotient
 *             digits pass through Simple-Renorm.
 *   (T, MC):  DivN -- the dividend is padded with zero components.
 *   (MC, T):  Div-MCN with the divisor padded with zero components.
 * x, y: [nc or 1][n]; out: [nc][n]. */
int mc_div(int dtype, int nc, int64_t n, const void *x, int x_mc, const void *y, int y_mc, void *out,
           void *stream);

/* Multiplication, Mult-MCN-Slow (Appendix A.2.1), for two MC operands: p = fl(x_0 y_0)
 * is the first product digit; nc times the remainder x = Add-MCN(x, -DivN(p, y)) is
 * formed and its next digit p = fl(x_0 y_0) taken; the nc+1 digits pass through
 * Simple-Renorm.  x, y, out: [nc][n]; out may be x or y exactly. */
int mc_mul_slow(int dtype, int nc, int64_t n, const void *x, const void *y, void *out, void *stream);

/* Square, Square-MCN (Appendix A.2.1).  The printed first step fl(2^{x_0}) is read as
 * fl(x_0 x_0), the square's leading term: h = (fl(x_0 x_0), 0, ..., 0), then
 * h = Grow-ExpN(h, fl(2 x_0 x_1)) (the addend is zero when nc = 1).  As printed, the
 * result is accurate to about one unit of x_0^2 (the rounding of x_0^2 and the terms
 * x_1^2, x_0 x_2, ... are not carried).  x, out: [nc][n]; out == x allowed. */
int mc_square(int dtype, int nc, int64_t n, const void *x, void *out, void *stream);

/* Exponential, Exp-MCN (Appendix A.2.1): h = exp(x_0) (one component), then for
 * i = 1 .. nc-1, h = ScalingN(h, exp(x_i), expand) growing h by one component per
 * step.  The component exponential is correctly rounded in every format (binary16
 * by table lookup; binary32 from a binary64 evaluation, with a double-double one
 * where that lies too close to a rounding boundary; binary64 by a double-double
 * table-driven evaluation, with a 192-bit fixed-point one where that lies too close
 * to a rounding boundary).  x, out: [nc][n]; out == x allowed. */
int mc_exp(int dtype, int nc, int64_t n, const void *x, void *out, void *stream);

/* Renormalization (Appendix A.2.1).
 *   mode 0: Renormalize (Priest variant): a top-down Two-Sum sweep s = x_0 (+) x_1 ...
 *           collecting the errors t_i, then a second sweep s, e = Two-Sum(s, t_i)
 *           that emits s whenever e != 0; the final s is emitted too; the first
 *           nc_out emitted values are returned, +0 padded.
 *   mode 1: Simple-Renorm: the first nc_out non-zero components in order, +0 padded.
 * 1 <= nc_out <= nc_in <= 4.  x: [nc_in][n]; out: [nc_out][n] (out == x allowed
 * only when nc_out == nc_in). */
int mc_renorm(int dtype, int nc_in, int nc_out, int64_t n, const void *x, void *out, int mode, void *stream);

/* Matrix product C = A B (Appendix A.2.2, MM-MCN; MV-MCN is N = 1 and Dot-MCN is
 * M = N = 1).  Each output is accumulated in MM-MCN order: acc = ScalingN(A_i0,
 * B_0j), then acc = Add-MCN(acc, ScalingN(A_ik, B_kj)) for k = 1 .. K-1, so the
 * result is reproducible and independent of the launch geometry.  With both
 * operands MC (not defined by the paper, whose matrix operators multiply an MC
 * matrix by a plain one) the product is taken by linearity over the components of
 * B: C = MM(A, B^(0)) (+) MM(A, B^(1)) (+) ... with (+) = Add-MCN.
 * MCF_F16S, both operands MC: B^(b) is at level b, so the part A B^(b) has levels
 * b, b+1, ..., of which the format keeps those below nc: the part is MM-MCN over the
 * first nc - b components of A with nc - b components at levels b .. nc-1, and the
 * parts, each placed at its levels (b leading zero components), are added left to
 * right: C = P_0 (+) (0, P_1) (+) (0, 0, P_2) ...
 * A: [nc or 1][M][K], B: [nc or 1][K][N], C: [nc][M][N]. */
int mc_matmul(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, int a_mc, const void *B,
              int b_mc, void *C, void *stream);

/* Pruned product of two MC matrices, a faster contraction with the accuracy class of
 * mc_matmul (Section 2.2 leaves faster MC products open).  The component products
 * A^(a) B^(b) with a + b >= nc are of the order of u^nc relative to A B -- the size of
 * MM-MCN's own error -- and are left out: component b of B multiplies the first
 * nc - b components of A, in MM-MCN order with nc - b components,
 *   C = MM_nc(A, B^(0)) (+) MM_{nc-1}(A[:nc-1], B^(1)) (+) ... (+) MM_1(A[:1], B^(nc-1)),
 * each part zero-padded to nc components, (+) = Add-MCN left to right.  A fixed
 * function of the inputs (reproducible on any launch geometry) but not mc_matmul's
 * bits: the error bound |C - C*| <= 4 K u^nc (|A||B|) is what it shares.  At nc = 3 it
 * needs 48 essential operations per multiply-add against mc_matmul's 102.
 * A: [nc][M][K], B: [nc][K][N], C: [nc][M][N], C not overlapping A or B. */
int mc_matmul_pruned(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, const void *B, void *C,
                     void *stream);

/* Batched and broadcast matrix products, BMM-MCN and 4DMM-MCN (Appendix A.2.2): for
 * every batch index (i1, i2) in [0, B1) x [0, B2), the matrices of A and B at that
 * index are multiplied exactly as mc_matmul multiplies its operands (MM-MCN order;
 * both MC: by linearity over the components of B).  A batch dimension of size 1
 * broadcast against a larger one (torch.matmul semantics) is a batch stride of 0.
 * A: component plane c starts at A + c*a_plane (elements); the matrix of batch
 *   (i1, i2) starts a_s1*i1 + a_s2*i2 elements into each plane and is [M][K]
 *   row-major.  B likewise, [K][N], with b_plane, b_s1, b_s2.  Every stride is >= 0
 *   and each plane must hold every batch's matrix: (B1-1)*s1 + (B2-1)*s2 + rows*cols
 *   <= plane (else MCF_E_SHAPE); the caller provides planes * plane elements.
 * C: dense [nc][B1][B2][M][N]; it must not overlap A or B.
 * Sizes as mc_matmul; B1, B2 >= 0; B1 * B2 * M * N below 2^40. */
int mc_matmul_batched(int dtype, int nc, int64_t B1, int64_t B2, int64_t M, int64_t N, int64_t K, const void *A,
                      int a_mc, int64_t a_plane, int64_t a_s1, int64_t a_s2, const void *B, int b_mc,
                      int64_t b_plane, int64_t b_s1, int64_t b_s2, void *C, void *stream);

/* AddMM-MCN (Appendix A.2.2): C = Add-MCN(ScalingN(A B, alpha), ScalingN(Y, beta)),
 * the product taken exactly as mc_matmul (any operand kinds), both ScalingN without
 * expand (so the result has nc components).
 * Y: MC, [nc][M][N] (y_rows = M) or [nc][N] added to every row (y_rows = 1).
 * alpha, beta: plain scalars that must be exactly representable in the component
 *   format (else MCF_E_ARG).
 * A: [nc or 1][M][K], B: [nc or 1][K][N], C: [nc][M][N], not overlapping A, B or Y. */
int mc_addmm(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, int a_mc, const void *B, int b_mc,
             const void *Y, int64_t y_rows, double alpha, double beta, void *C, void *stream);

/* K-split matrix product, for reductions that are long compared with the number of
 * outputs (Dot-MCN, MV-MCN, small products).  Section 2.2 of the paper notes that an
 * accurate sum of N MC values can be had in O(nc log N) depth; this entry point
 * computes the following log-depth variant of MM-MCN, fixed by the slice count S
 * alone (never by the device or the launch):
 *   the reduction steps are dealt round-robin to S slices, slice s taking
 *   k = s, s + S, s + 2S, ...; each slice is summed in MM-MCN order; the S slice
 *   sums are combined by a pairwise Add-MCN tree -- at each level entry q of the
 *   next level is Add-MCN(entry 2q, entry 2q+1), an odd last entry moves up
 *   unchanged.  With both operands MC, one such product per component of B,
 *   combined left to right with Add-MCN (as mc_matmul).
 * S = 1 gives exactly mc_matmul's result.  Other S give a result of the same
 * accuracy class (the error bound of MM-MCN holds) but not the same bits.
 * slices: S, at most 2^20 (else MCF_E_ARG); values above K are taken as K;
 *   slices <= 0 selects mc_matmul_splitk_slices(M, N, K).
 * workspace: device memory of at least mc_matmul_splitk_workspace(...) bytes (the
 *   partial tree roots: G = ceil(S / 256) entries of planes x nc x M x N components
 *   when S > 256; planes = nc for MC x MC, else 1), owned
 *   by the caller, not overlapping A, B or C; may be NULL when that size is 0.  Its
 *   contents on entry do not matter; calls sharing a workspace must not overlap
 *   in time.  Too small: MCF_E_ARG; NULL when needed: MCF_E_NULL.
 * A: [nc or 1][M][K], B: [nc or 1][K][N], C: [nc][M][N] (C must not overlap A or B);
 * M * N below 2^31. */
int mc_matmul_splitk(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, int a_mc, const void *B,
                     int b_mc, int64_t slices, void *workspace, int64_t workspace_bytes, void *C, void *stream);

/* Allocation-free form of mc_matmul_splitk, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same arguments, result and rules as mc_matmul_splitk, but the partial
 * tree roots go to a static per-device scratch array inside the library (8 MiB,
 * held by every device the library runs on until the process ends) instead of a
 * caller workspace; the call allocates nothing.
 * Limit: calls whose mc_matmul_splitk_workspace(...) exceeds 8 MiB (8388608 bytes)
 *   return MCF_E_SCRATCH and launch nothing.  With the default slice count the roots
 *   take at most 1 MiB (binary64, nc = 4, MC x MC), so the limit binds only for
 *   large explicit slice counts on many outputs.
 * Sharing: every call on a device uses that device's one scratch array, so calls on
 *   one device that overlap in time (different streams, or different host threads)
 *   race and give undefined results; serialise them.  The contents left by earlier
 *   calls do not matter (nothing is read before it is written).
 * The device is the one that runs `stream` (the current device for NULL).  The first
 * call on a device looks up the array's device address (no allocation). */
int mc_matmul_splitk_noalloc(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, int a_mc,
                             const void *B, int b_mc, int64_t slices, void *C, void *stream);

/* Default slice count of mc_matmul_splitk, a function of the shape only: enough
 * slices for about 2^20 lanes in total (ceil(2^20 / (M N))), at most K / 64 (so a
 * slice holds at least 64 terms when K allows), at most 2^20, at least 1.
 * Negative sizes: MCF_E_SHAPE. */
int64_t mc_matmul_splitk_slices(int64_t M, int64_t N, int64_t K);

/* Workspace bytes mc_matmul_splitk needs for these arguments (0 when none), or a
 * negative mcf_status for arguments mc_matmul_splitk would reject. */
int64_t mc_matmul_splitk_workspace(int dtype, int nc, int64_t M, int64_t N, int64_t K, int a_mc, int b_mc,
                                   int64_t slices);

/* Exact MC product for binary16 components, rounded into nc components.  An MC
 * number is the unevaluated sum of its components (Section 2.1), so every output has
 * one exact value P_ij = sum_k (sum_c A^(c)_ik)(sum_c B^(c)_kj), the quantity that
 * MM-MCN (Section 2.2) approximates within about 4 K u^nc sum_k |A_ik||B_kj|
 * (Section 2.4).  This call returns P_ij split by successive round-to-nearest-even
 * into binary16: c_0 = RN(P), c_1 = RN(P - c_0), ..., so the components never
 * overlap and their sum is within half an ulp of c_{nc-1} (at most 2^-25 absolute
 * in the subnormal range) of P.  Not mc_matmul's bits: a different, more accurate
 * result.  The contraction runs on the int8 matrix cores: each entry is an exact
 * integer multiple of 2^-24, cut into 8-bit digits whose products are summed
 * exactly.
 * dtype: MCF_F16 only (else MCF_E_DTYPE).
 * Special values (input values ARE inspected here): an output whose row of A or
 *   column of B holds an infinite or NaN component is NaN in every component; if
 *   |P| rounds above 65504 the result is (+-inf, +0, ..., +0); an exact zero gives +0
 *   in every component, a non-zero P that rounds to zero keeps its sign.
 * A: [nc or 1][M][K]; B: [nc or 1][K][N], or [nc or 1][N][K] when b_trans = 1 (a
 *   linear layer's weight); C: [nc][M][N], not overlapping A or B.
 * workspace: device memory of at least mc_matmul_exact_workspace(...) bytes, owned by
 *   the caller, not overlapping A, B or C (else MCF_E_ALIAS); contents on entry do
 *   not matter; calls sharing a workspace must not overlap in time.  Too small:
 *   MCF_E_ARG; NULL: MCF_E_NULL.
 * Sizes: M, N <= 2^31, K <= 2^29, (M + N) K <= 2^40 and M N <= 2^38 (else
 *   MCF_E_SHAPE). */
int mc_matmul_exact(int dtype, int nc, int64_t M, int64_t N, int64_t K, const void *A, int a_mc, const void *B,
                    int b_mc, int b_trans, void *workspace, int64_t workspace_bytes, void *C, void *stream);

/* Exact MC-Linear forward for binary16 components: y = x W^T + b with the exact value
 * of every output (x plain, W and b MC; Section 2.3's layer) split into nc components
 * by successive rounding, as mc_matmul_exact -- the bias is added to the exact sum
 * before the split.  An output whose column of W or bias holds an infinite or NaN
 * component, or whose row of x does, is NaN in every component.
 * x: [batch][in] (plain), W: [nc][out][in], b: [nc][out] or NULL, y: [nc][batch][out]
 * (not overlapping x, W, b or the workspace).
 * workspace: as mc_matmul_exact, at least mc_matmul_exact_workspace(dtype, nc, batch,
 *   out, in) bytes.  dtype: MCF_F16 only.  Sizes as mc_matmul_exact with M = batch,
 *   N = out, K = in. */
int mc_linear_fwd_exact(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *W,
                        const void *b, void *workspace, int64_t workspace_bytes, void *y, void *stream);

/* Workspace bytes mc_matmul_exact needs (about 6 (M + N) K bytes of digit planes,
 * plus 16 M N ceil(K / 16384) bytes of partial sums when K > 16384), or a negative
 * mcf_status for
 * sizes it would reject. */
int64_t mc_matmul_exact_workspace(int dtype, int nc, int64_t M, int64_t N, int64_t K);

/* MC-Linear forward (Section 2.3): y = x W^T (+ b).  The weight and bias are MC,
 * the input is a plain tensor; each output accumulates ScalingN(W[o][i], x[t][i])
 * over i in MM-MCN order, then adds the bias with Add-MCN.
 * x: [batch][in] (plain), W: [nc][out][in], b: [nc][out] or NULL,
 * y: [nc][batch][out]. */
int mc_linear_fwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *W,
                  const void *b, void *y, void *stream);

/* MC-Linear backward (the layer of Section 2.3, y = x W^T + b): given the gradient dY
 * of the loss with respect to y, computes
 *   dX = dY W          [batch][in]  (MM-MCN; dY MC: by linearity over W's components)
 *   dW = dY^T x        [out][in]    (MM-MCN over the batch index, in batch order)
 *   db = sum_t dY[t]   [out]        (Add-MCN of the rows of dY in batch order: MM-MCN
 *                                    against a column of ones, ScalingN by 1 being exact)
 * The paper keeps the gradient of an MC value as a plain tensor -- the gradient of
 * its leading component (Section 2.1) -- and takes it from automatic differentiation;
 * here the gradients are MC values whose leading components are those plain
 * gradients, accumulated with MM-MCN's error propagation.  A plain dY (dy_mc = 0)
 * enters dW and db as an MC value with +0 low components.
 * x: [batch][in] plain; W: [nc][out][in]; dY: [nc or 1][batch][out] (dy_mc 1 or 0);
 * dX: [nc][batch][in], dW: [nc][out][in], db: [nc][out] -- each may be NULL (not
 * computed); outputs must not overlap the inputs, each other or the workspace.
 * workspace: device memory of at least mc_linear_bwd_workspace(...) bytes when dW or
 *   db is requested, owned by the caller, not overlapping the inputs; contents on entry do
 *   not matter; calls sharing it must not overlap in time.  Too small: MCF_E_ARG; NULL when
 *   needed: MCF_E_NULL.  The size covers every gradient and kind of dY: dY^T in nc planes,
 *   then x with a column of ones appended and the [dW | db] product, which gives both in one
 *   pass.  A call may touch less of it, or none: a plain dY stages one plane, and results of
 *   few outputs (any size at nc = 1, and db alone) read dY and x as they are stored.
 * dtype: MCF_F16, MCF_F32, MCF_F64.  Sizes: batch, out <= 2^20, in <= 2^30 (and the
 * product limits of mc_matmul). */
int mc_linear_bwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *W,
                  const void *dY, int dy_mc, void *dX, void *dW, void *db, void *workspace, int64_t workspace_bytes,
                  void *stream);

/* Workspace bytes mc_linear_bwd needs when dW or db is requested, or a negative
 * mcf_status for sizes it would reject. */
int64_t mc_linear_bwd_workspace(int dtype, int nc, int64_t batch, int64_t in, int64_t out);

/* One gradient-descent step of the paper's linear-regression precision experiment
 * (Section 2.4): an MC-Linear layer without bias, W (out = 1 row of d weights), fitted
 * to targets y with the mean-squared error L(W) = (1/n) sum_i (x_i . W - y_i)^2.
 * The paper leaves the optimizer step unprinted and defines the gradient of an MC value
 * as the plain gradient of its leading component (Section 2.1).  This call computes, in
 * stream order:
 *   yhat = MC-Linear(X, W) (MM-MCN order, as mc_linear_fwd);
 *   r = Grow-ExpN(yhat, y_neg), the MC residual;
 *   G = r^T X and RR = r . r, each by the K-split product with its default slice count
 *     (mc_matmul_splitk_slices);
 *   per weight j: g = ScalingN(G_j, fl(2/n)); grad_j = the leading component of g;
 *     W_j = Grow-ExpN(W_j, fl(-lr * grad_j)) (one rounding of the product);
 *   loss = ScalingN(RR, fl(1/n)), the loss at W before the update.
 * fl(2/n), fl(1/n): the binary64 quotients rounded once to the component format;
 * fl(-lr): the binary64 value -lr rounded to the component format.
 * X: [n][d] plain; y_neg: [n] plain, the NEGATED targets (-y); W: [nc][d] MC, updated
 *   in place; loss: [nc] MC, or NULL.  W and loss must not overlap each other, X, y_neg
 *   or the workspace.
 * workspace: device memory of at least mc_linreg_workspace(...) bytes, owned by the
 *   caller (contents on entry do not matter; steps sharing it must not overlap in
 *   time).  Too small: MCF_E_ARG.
 * Sizes: n >= 1, d >= 1, n <= 2^30, d <= 2^20, n d <= 2^40. */
int mc_linreg_gd_step(int dtype, int nc, int64_t n, int64_t d, const void *X, const void *y_neg, void *W, double lr,
                      void *workspace, int64_t workspace_bytes, void *loss, void *stream);

/* Workspace bytes mc_linreg_gd_step needs, or a negative mcf_status for arguments it
 * would reject. */
int64_t mc_linreg_workspace(int dtype, int nc, int64_t n, int64_t d);

/* ---------------------------------------------------------------------------------
 * Microscaled 4-bit (MXFP4) tensors
 *
 * An MXFP4 number is an E2M1 element (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives)
 * times the power of two of its block: 32 elements along a row share one E8M0 scale
 * (byte s stands for 2^(s - 127), 255 for NaN).  An MXFP4 tensor of nc components is the
 * sum of nc of them, each the rounding of what the components before it leave -- an MC
 * value (Section 2) whose component format has 4 bits.  1 <= nc <= 4.
 * Layout of a tensor of `rows` rows of n elements, G = ceil(n / 128) groups of four blocks:
 *   codes:  [nc][rows][64 G] bytes, element i of a row in byte i / 2, the low half for even
 *           i; zeros past n; 16-byte aligned.
 *   scales: [nc][G][rows][4] bytes, block b of group q of row r at byte 4 (q rows + r) + b of
 *           its component; zeros for blocks wholly past n; 4-byte aligned.
 * Sums of the products are held in binary32; results are rounded once to the call's format.
 * Non-finite inputs propagate by IEEE rules through the products of the single components:
 * with one component an infinity in x or dY gives y and dX what the whole numbers give,
 * whatever the number of rows.  It may give NaN in place of an infinity where the weight has
 * several components (infinity times a component that is 0 or of the other sign), and in dW of
 * binary32, whose two factors are both split.
 * Workspaces: device memory of at least the matching ..._workspace(...) bytes, 16-byte
 * aligned, owned by the caller, not overlapping the other arguments; may be NULL when that
 * size is 0; contents on entry do not matter; calls sharing one must not overlap in time.
 * Too small or misaligned: MCF_E_ARG; NULL when needed: MCF_E_NULL.
 */

/* Quantisation.  The exact value v of an element (with nc_in > 1 the sum of its planes, in
 * binary64 where binary32 does not hold it) is split into nc components: with a the largest
 * magnitude of its block and X = max(floor(log2 a) - 2, -127), the component is v 2^-X
 * rounded to nearest E2M1, ties to even, at most 6, times 2^X, and v minus it is the next
 * component's value.  A block with an infinity or NaN gets the scale 255 and zero codes in
 * every component.
 * x: [nc_in][rows][n]; codes and scales as above.  ceil(rows / 16) ceil(n / 128)
 * below 2^31. */
int mc_mx4_quantize(int dtype, int nc_in, int nc, int64_t rows, int64_t n, const void *x, void *codes, void *scales,
                    void *stream);

/* Reading back: out = the sum of the components in binary32, the last one first, rounded to
 * the format.  out: [rows][n]. */
int mc_mx4_dequantize(int dtype, int nc, int64_t rows, int64_t n, const void *codes, const void *scales, void *out,
                      void *stream);

/* C = A B^T of two MXFP4 tensors (a_nc and b_nc components) on the scaled matrix
 * instructions.  A: M rows of K, B: N rows of K, C: [M][N] in the call's format.
 * M <= 2^20, N <= 2^24, K <= 2^22. */
int mc_mx4_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales, int a_nc,
                  const void *b_codes, const void *b_scales, int b_nc, void *workspace, int64_t workspace_bytes,
                  void *C, void *stream);
int64_t mc_mx4_matmul_workspace(int dtype, int64_t M, int64_t N, int64_t K, int a_nc, int b_nc);

/* Linear layer of a plain input with an MXFP4 weight: y = x W^T (+ b).
 * x: [batch][in]; codes, scales: W, `out` rows of `in`, nc components; b: [out] or NULL;
 * y: [batch][out].  batch <= 2^20, in <= 2^22, out <= 2^24. */
int mc_mx4_linear_fwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                      const void *scales, const void *b, void *workspace, int64_t workspace_bytes, void *y,
                      void *stream);
int64_t mc_mx4_linear_fwd_workspace(int dtype, int nc, int64_t batch, int64_t in, int64_t out);

/* Its gradients, given that of the loss with respect to y:
 *   dX = dY W      [batch][in]
 *   dW = dY^T x    [out][in]   the gradient with respect to the numbers W stands for, which
 *                              a straight-through rule hands to the weight it was made from
 *   db = sum_t dY  [out]
 * dX, dW and db may each be NULL (not computed); codes and scales are needed for dX only, x
 * for dW only.  dY: [batch][out].  batch, in, out <= 2^20. */
int mc_mx4_linear_bwd(int dtype, int nc, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                      const void *scales, const void *dY, void *dX, void *dW, void *db, void *workspace,
                      int64_t workspace_bytes, void *stream);
int64_t mc_mx4_linear_bwd_workspace(int dtype, int nc, int64_t batch, int64_t in, int64_t out);

/* ---------------------------------------------------------------------------------
 * Distillation from a teacher's top logits
 *
 * A row has the student's logits z_j, j < vocab, and up to k teacher entries (ids_i, t_i),
 * in any order.  With p the softmax over the row's used entries of t_i / T and q the softmax
 * over the row of z_j / T:
 *   loss  = T^2 sum_i p_i (log p_i - log q_{ids_i})
 *   dz_j  = g T (q_j - sum of the p_i with ids_i = j)       (g: the row's upstream gradient)
 * An entry with ids_i outside [0, vocab) is unused; a row with no used entry, or with none
 * above -inf, has loss 0 and gradient 0.  A logit of -inf has q_j = 0; a teacher entry with
 * p_i > 0 there makes the loss +inf.  Statistics and sums are binary32.
 * z: plain [rows][vocab], or (nc > 1) an MC value [nc][rows][vocab] whose planes are summed
 *   in binary32, the last one first; its gradient is plain, that of the sum (Section 2.1).
 * ids: int32 [rows][k]; t: [rows][k] in z's format; 0 <= k <= 1024 (may be NULL for k = 0).
 * temperature: finite and above 2^-127, as a binary32 number.  loss: binary32 [rows], which has T^2.
 * stats: binary32 [rows][2], the row's largest logit m and sum_j exp((z_j - m) / T).
 * g: binary32 [rows], or NULL for ones.  dz: [rows][vocab] in z's format.
 * No output may overlap an input or another output.  rows < 2^31, 1 <= vocab <= 2^30. */

/* loss, and stats for the backward call (stats may be NULL).  workspace: at least
 * mc_distill_workspace(rows, vocab) bytes, under the rules above. */
int mc_distill_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                   const void *t, double temperature, void *workspace, int64_t workspace_bytes, void *loss,
                   void *stats, void *stream);

/* dz from the forward call's stats. */
int mc_distill_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                   const void *t, double temperature, const void *stats, const void *g, void *dz, void *stream);

/* Both in one pass over z, for a g that is known beforehand (1 / rows for a mean). */
int mc_distill_fwd_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t k, const void *z, const void *ids,
                       const void *t, double temperature, const void *g, void *workspace, int64_t workspace_bytes,
                       void *loss, void *dz, void *stream);
int64_t mc_distill_workspace(int64_t rows, int64_t vocab);

/* ---------------------------------------------------------------------------------
 * 8-bit tensors, the RMS norm that makes them, and their products
 *
 * An 8-bit tensor of `rows` rows of n elements, P = n rounded up to a multiple of 128:
 *   codes:  [rows][P] signed bytes from -127 to 127, zeros past n; 16-byte aligned.
 *   scales: [rows] binary32.  Element i of a row stands for code_i times the row's scale.
 * Quantisation of a row p: with m its largest magnitude, code_i = 127 p_i / m rounded to the
 *   nearest integer, ties to even (the binary64 quotient fl(fl(127 p_i) / m)), scale = m / 127
 *   rounded once; a row of zeros has the scale 0.  A row with an infinity or NaN, or whose scale
 *   passes binary32's range, has the scale NaN and zero codes.
 * n <= 2^30; rows times P below 2^50.  Workspaces as for the MXFP4 calls. */

/* x: plain [rows][n] or (nc_in > 1) an MC value [nc_in][rows][n], of which the planes' sum in
 * binary64, the last one first, is quantised. */
int mc_int8_quantize(int dtype, int nc_in, int64_t rows, int64_t n, const void *x, void *codes, void *scales,
                     void *stream);

/* Reading back: out [rows][n] = code times scale in binary32, rounded to the format. */
int mc_int8_dequantize(int dtype, int64_t rows, int64_t n, const void *codes, const void *scales, void *out,
                       void *stream);

/* C = A B^T (+ bias) of two 8-bit tensors.  A: M rows of K (tokens), B: N rows of K (a weight's
 * output channels), bias: [N] of the call's format or NULL, C: [M][N] in the call's format.  The
 * integers' products are summed exactly; C_ij = (sum a_i) b_j + bias_j in binary32 (sum, a_i and b_j
 * the scales of the rows), rounded once to the format: a row's result does not depend on
 * the other rows.  M <= 2^20, N <= 2^24, K <= 131072. */
int mc_int8_matmul(int dtype, int64_t M, int64_t N, int64_t K, const void *a_codes, const void *a_scales,
                   const void *b_codes, const void *b_scales, const void *bias, void *workspace,
                   int64_t workspace_bytes, void *C, void *stream);
int64_t mc_int8_matmul_workspace(int dtype, int64_t M, int64_t N, int64_t K);

/* Linear layer of a plain input with an 8-bit weight: y = x W^T (+ b), each row of x quantised as
 * above; the same numbers as mc_int8_quantize and mc_int8_matmul.
 * x: [batch][in]; codes, scales: W, `out` rows of `in`; b: [out] or NULL; y: [batch][out].
 * batch <= 2^20, in <= 131072, out <= 2^24. */
int mc_int8_linear_fwd(int dtype, int64_t batch, int64_t in, int64_t out, const void *x, const void *codes,
                       const void *scales, const void *b, void *workspace, int64_t workspace_bytes, void *y,
                       void *stream);
int64_t mc_int8_linear_fwd_workspace(int dtype, int64_t batch, int64_t in, int64_t out);

/* Root-mean-square norm of the rows of a residual stream, a layer's output x added to it first.
 *   s = the planes of h summed in binary64, the last one first, plus x;
 *   h_out = s split by successive rounding into nc planes (each through binary32 into the format;
 *           nothing is left of a value past its range); v = the planes' sum again;
 *   r = 1 / sqrt(sum of v_i^2 / n + eps);
 *   y_i = v_i w_i r, rounded to the format.
 * Without x, v is the sum of h's planes and h_out must be NULL.
 * h: [nc][rows][n] (a plain stream: nc = 1); x: [rows][n] or NULL; w: [n] or NULL for ones; h_out:
 * [nc][rows][n], may be h itself (in place); y: [rows][n].  Everything between the loads and the
 * roundings is binary64, but that y of a plain 16-bit stream is rounded from a binary32 number
 * within 2^-23 of v_i w_i r, relative to it, or within 2^-140 where v_i w_i is below 2^-126.  A row's
 * result does not depend on the other rows.  A row of zeros with eps = 0 has r = inf and so NaN.
 * n >= 1, eps >= 0 and finite. */
int mc_rmsnorm_fwd(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w, double eps,
                   void *h_out, void *y, void *stream);

/* The same with the output as an 8-bit tensor: the quantisation of p_i = v_i w_i, of which the
 * codes are a fixed function, with the scale r max |p| / 127. */
int mc_rmsnorm_int8(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *x, const void *w, double eps,
                    void *h_out, void *codes, void *scales, void *stream);

/* The gradients of mc_rmsnorm_fwd, given dy, that of the loss with respect to y, and g, the
 * gradient that reaches the stream behind the addition from elsewhere (NULL for none):
 *   dh = g + r (w dy - v r^2 sum(v w dy) / n)   [rows][n]  with respect to that stream, and so to
 *                                                          h and to x alike (plain, Section 2.1)
 *   dw = sum over the rows of dy v r            [n]
 * h: the stream the norm was taken of (h_out where x was added).  dh and dw may each be NULL (not
 * computed); the workspace is needed for dw.  Sums over rows are joined in a fixed order. */
int mc_rmsnorm_bwd(int dtype, int nc, int64_t rows, int64_t n, const void *h, const void *w, const void *dy,
                   const void *g, double eps, void *dh, void *dw, void *workspace, int64_t workspace_bytes,
                   void *stream);
int64_t mc_rmsnorm_bwd_workspace(int dtype, int64_t rows, int64_t n);

/* ---------------------------------------------------------------------------------
 * Log probabilities of tokens
 *
 * With q the softmax over a row of z_j / T, j < vocab:
 *   logp_i = log q_{ids_i}, of `given` tokens a row; 0 for an id outside [0, vocab) (no token);
 *   entropy = -sum_j q_j log q_j;
 *   the `top` most likely tokens, in the order (z descending, j ascending), and their log q.  Past
 *   the last logit above -inf the id is -1 and the log probability -inf.
 * A logit of -inf has q_j = 0 and log q_j = -inf.  A row of nothing but -inf: log probabilities
 * -inf, entropy 0, no alternatives, gradient 0.  A row with a NaN or +inf: NaN everywhere, ids -1.
 * z: plain [rows][vocab], or (nc > 1) an MC value [nc][rows][vocab] whose planes are summed in
 *   binary32, the last one first; its gradient is plain, that of the sum (Section 2.1).
 * ids: int32 [rows][given], 0 <= given <= 1024, in any order, also equal ones.
 * temperature: finite and above 2^-127, as a binary32 number.  At a very small one the entropy has
 *   terms near binary32's smallest numbers, and so an error of up to vocab 2^-149 / temperature beside
 *   that of its roundings.
 * logp: binary32 [rows][given]; entropy: binary32 [rows] or NULL; top_ids: int32 and top_logp:
 *   binary32 [rows][top], 0 <= top <= 128.
 * stats: binary32 [rows][3] or NULL, for the gradient: the row's largest logit m, L = log sum_j
 *   exp((z_j - m) / T), and entropy - L.
 * Statistics and sums are binary32, summed in an order that depends on rows and vocab alone; the log
 * probability of a token the row is sure of, and the gradient there, keep their relative accuracy.
 * No output may overlap an input or another output.  rows < 2^31, 1 <= vocab <= 2^30.  Workspace as
 * for the MXFP4 calls. */
int mc_logprobs_fwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, int64_t top, const void *z,
                    const void *ids, double temperature, void *workspace, int64_t workspace_bytes, void *logp,
                    void *entropy, void *top_ids, void *top_logp, void *stats, void *stream);
int64_t mc_logprobs_workspace(int64_t rows, int64_t vocab, int64_t top);

/* The gradient dz [rows][vocab], in z's format, of sum_i g_i logp_i + g_entropy entropy over each row:
 *   dz_j = (sum of the g_i with ids_i = j - q_j (sum of all used g_i + g_entropy (log q_j + entropy))) / T.
 * g: binary32 [rows][given] or NULL for ones; g_entropy: binary32 [rows] or NULL for zeros. */
int mc_logprobs_bwd(int dtype, int nc, int64_t rows, int64_t vocab, int64_t given, const void *z, const void *ids,
                    double temperature, const void *stats, const void *g, const void *g_entropy, void *dz,
                    void *stream);

/* Human-readable name of a status code (static storage). */
const char *mc_status_str(int status);

#ifdef __cplusplus
}
#endif

#endif /* MCF_H */
