/*
 * bpdq.h -- C ABI of the BPDQ per-layer quantization pass for AMD MI355X (gfx950).
 *
 * BPDQ (Bit-Plane Decomposition Quantization on a variable grid) represents a linear
 * layer's weight as   What = REP(C_0) + sum_{i=1..k} REP(C_i) (.) B_i   (paper Eq. 1):
 * k binary planes B_i and k+1 real coefficients per (row, group of g input channels),
 * chosen to minimise || (W - What) X ||_F^2 = tr((W - What) H (W - What)^T)  (Eq. 2).
 *
 * Conventions
 *  - Every pointer is a DEVICE pointer owned by the caller unless marked "host".
 *    The library allocates nothing: scratch comes from the caller's workspace `ws`
 *    (256-byte aligned, at least *_workspace_bytes() long).
 *  - Every call only enqueues work on `stream` (a hipStream_t passed as void*; NULL is
 *    the default stream) and returns without synchronising.  Calls on one stream are
 *    ordered; a workspace must not be shared by calls that can run concurrently.
 *  - Matrices are dense row-major fp32 unless stated.
 *  - Return value: 0 = enqueued; -n = argument number n (1-based) is invalid;
 *    BPDQ_ERR_LAUNCH = a HIP call failed.  Numerical failure of bpdq_prepare is reported
 *    through its device-side `info`, LAPACK style.
 *  - Results are deterministic: no floating-point atomics anywhere.
 */
#ifndef BPDQ_H
#define BPDQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BPDQ_ERR_LAUNCH (-100)
#define BPDQ_GRID_VARIABLE 0
#define BPDQ_GRID_UNIFORM 1

/* Knobs of the method (paper Sec. 4.1: k in {2,3,4}, g in {64,128,256}, 10 iterations,
 * alpha = 1e-4). */
typedef struct bpdq_params {
  int   bits;           /* k, number of bit-planes: 1..4                                      */
  int   group;          /* g: 32, 64, 128 or 256 (256 only with bits <= 3); must divide d_in  */
  int   block;          /* lazy-update block B; the effective block is max(B, g); g | B       */
  int   refine_iters;   /* T >= 0 iterations of (bit-plane update, refit, delta correction);
                           0 keeps the initialisation + one fit (Sec. 3.2)                    */
  float alpha;          /* relative ridge of the coefficient fit (Sec. 3.2, end): the
                           (k+1)x(k+1) normal matrix G gets alpha*tr(G)/(k+1) on its diagonal */
  int   grid;           /* BPDQ_GRID_VARIABLE: the method (variable grid, Sec. 3).
                           BPDQ_GRID_UNIFORM: the fixed-grid comparator of App. A -- levels
                           lo + s*{0..2^k-1} per (row, group) from the group's min/max, one
                           sweep, no fit (GPTQ on a uniform grid); refine_iters and alpha are
                           ignored, the coefficients returned are (lo, s, 2s, ...).             */
  int   coef_fp16;      /* storage precision of the coefficients (Table 1 counts 16 bits each).
                           0: fp32 throughout.  1: every coefficient is rounded to IEEE half
                           (nearest even, in one step from the fp64 fit; a fixed grid's from fp32)
                           right after its fit, so the levels of the next bit-plane
                           update, What, E*, the scores and the compensation all belong to the
                           values that are stored; `coefs` still holds floats, each exactly a
                           half (bpdq_coefs_to_fp16 is then lossless).  Magnitudes above 65504
                           would become infinite: scale such a layer first.                    */
} bpdq_params;

/* Library version (major*10000 + minor*100 + patch). */
int bpdq_version(void);

/* ---- step 1: calibration Hessian (Sec. 3.1, text under Eq. 2: H = X X^T) ---------------
 * H += scale * Xc^T Xc for one chunk of tokens.
 *   Xc : n_tok x d_in, one token per row, row stride ldx floats (>= d_in).  This is the
 *        paper's X (d_in x N, one token per column) in column-major storage.
 *   H  : d_in x d_in.  Only the upper triangle (j >= i) is accumulated; pass
 *        symmetrize != 0 (e.g. on the last chunk) to mirror it into the lower triangle.
 *   scale : 2 reproduces the customary H = 2 X X^T; any positive factor gives the same
 *        planes and coefficients.
 *   ws : split-K partial sums and, for the default entry, the activations re-encoded as halves;
 *        bpdq_hessian_workspace_bytes(n_tok, d_in) bytes serve any of the three entries
 *        (about 4 * n_tok * d_in bytes plus the partial tiles).
 *        That size is not monotonic in n_tok: a short call on a narrow layer is cut into more slices
 *        than a longer one.  The default entry also accepts a workspace that does not hold those
 *        slices but holds coarser ones (sized for a longer call, say); see below.  Its small calls
 *        (below) leave ws untouched, but ask for the same sizes, so that a program need not know
 *        which calls are small.
 * Requirements: d_in % 4 == 0, ldx % 4 == 0, Xc and H 16-byte aligned, ws 256-byte aligned, n_tok >= 0.
 * Returns 0, or a negative code naming the offending argument (-1 Xc, -2 n_tok, -3 d_in,
 * -4 ldx, -6 H, -8 ws, -9 ws_bytes); nothing is launched then.
 *
 * Three kernels compute the same update; each result is bit-reproducible from call to call, they
 * are not bit-identical to one another (they differ by rounding), and each is checked against the
 * fp64 definition to 1e-5 relative Frobenius error.  The slices, hence the last bits, follow from
 * n_tok and d_in alone with any workspace of at least bpdq_hessian_workspace_bytes(n_tok, d_in)
 * bytes; on a smaller one that is accepted they are the coarser slices, the same in every such call.
 * bpdq_hessian_accumulate (the fastest) runs on the fp16 matrix cores: a streaming pre-pass finds
 *   every channel's largest magnitude in the call, scales the channel by the power of two that
 *   brings it into [2^13, 2^14) and cuts every scaled value into two halves h + l (22 significant
 *   bits, fewer where the value is below 2^-16 of the channel's largest, of which the error is 2^-38 at most); a product is
 *   the sum of the three half products of weight >= 2^-11, accumulated in fp32, and the result is scaled back exactly.  The
 *   error of a product of values above 2^-15 of their channels' largest is below 2^-21 of it -- above the 2^-24 of an fp32
 *   product, far below the rounding of the fp32 accumulation over thousands of tokens.
 *   Launches of n_tok * d_in >= 2^27 (a call of up to 524288 tokens, of up to 8192 on a layer of 1024 tiles or more, is one
 *   launch) scale a channel by the largest of every 16th token instead: that factor is the same or larger, so the halves are
 *   as fine or finer, and no value is lost, because channels with a value that leaves the half range under it are scaled
 *   again by the largest of all tokens.  The time of such a call depends on the activations: at 262144 x 3584 9.5 ms with the
 *   scales of all tokens, 9.0 without outliers that the sample missed, up to 10.5 where every channel has one.
 *   Small calls (up to 64 tokens on 3072 channels, 256 on 2048, 512 on 704, 1024 on 512, 2048
 *   on 320, less some that the above does sooner) are one launch on the fp32 matrix cores instead: fp32
 *   products (2^-24) of the channels scaled in the same way, in chains of at most 32 tokens.  Which of
 *   the two follows from n_tok and d_in alone.
 *   Assumes finite X (an infinity or NaN yields NaN in its row and column).
 * bpdq_hessian_accumulate_bf16x3 runs on the bf16 matrix cores without a pre-pass: every value is
 *   cut exactly into three bf16 pieces inside the kernel and a product is the sum of the six piece
 *   products of weight >= 2^-16 (error below 2^-24 of a product).  About 1.5 times slower.
 *   Assumes |x| < 2^127.
 * bpdq_hessian_accumulate_f32 runs on the fp32 matrix cores (about 2.4 times slower). */
size_t bpdq_hessian_workspace_bytes(int n_tok, int d_in);
int bpdq_hessian_accumulate(const float* Xc, int n_tok, int d_in, int ldx, float scale,
                            float* H, int symmetrize, void* ws, size_t ws_bytes, void* stream);
int bpdq_hessian_accumulate_bf16x3(const float* Xc, int n_tok, int d_in, int ldx, float scale,
                                   float* H, int symmetrize, void* ws, size_t ws_bytes,
                                   void* stream);
int bpdq_hessian_accumulate_f32(const float* Xc, int n_tok, int d_in, int ldx, float scale,
                                float* H, int symmetrize, void* ws, size_t ws_bytes,
                                void* stream);

/* The same call with the kernel chosen by number, for measurement: ev_begin / ev_end (hipEvent_t
 * as void*, created by the caller with timing enabled, or NULL) are recorded on `stream`
 * immediately before the first and immediately after the last launch of the tile-product kernel
 * (a call of at most 524288 tokens on a layer of fewer than 1024 tiles is one launch: then the two
 * events bracket that kernel alone, without the pre-pass before it and the reduction after it; of a
 * small call of the default entry they bracket its one launch, which is all of it).
 * Return codes as above with every argument number one higher (-1: unknown kernel). */
#define BPDQ_HESSIAN_F16X2 0
#define BPDQ_HESSIAN_BF16X3 1
#define BPDQ_HESSIAN_F32 2
int bpdq_hessian_accumulate_timed(int kernel, const float* Xc, int n_tok, int d_in, int ldx,
                                  float scale, float* H, int symmetrize, void* ws, size_t ws_bytes,
                                  void* stream, void* ev_begin, void* ev_end);

/* ---- step 2: damping and U = chol(H^-1) (Sec. 3.1, "Quantization Error Compensation") ---
 * Reads the upper triangle of H.  Channels with H_ii == 0 are marked dead[i] = 1 and get
 * H_ii = 1.  Then lambda = damp * mean_i(H_ii), Ht = H + lambda I, and U is the upper
 * triangular matrix with positive diagonal such that Ht^-1 = U^T U.
 *   U    : d_in x d_in fp32, full matrix written (strictly lower part = 0); may alias H.
 *   dead : d_in bytes.
 *   info : one device int: 0, or the 1-based index of the first column whose pivot was not
 *          positive (Ht not positive definite; U is then undefined).  The columns are taken from
 *          the last to the first.
 * The factorisation runs in fp64 inside ws.  From 65 to 12288 columns a workspace of
 * 12 d_in^2 bytes and a little (what other widths ask for) is accepted too where the size asked for is
 * larger: the same U to the rounding of fp64, up to 1.6 times slower. */
size_t bpdq_prepare_workspace_bytes(int d_in);
int bpdq_prepare(const float* H, int d_in, float damp, float* U, unsigned char* dead,
                 int* info, void* ws, size_t ws_bytes, void* stream);

/* ---- steps 3-4: the group/column sweep with lazy block updates (Sec. 3.2, 3.3, App. B.3) -
 * For every block of max(B, g) columns, left to right, and every group of g columns in it:
 * 8-bit round-to-nearest initialisation of the planes from the group's current working
 * weights (Eq. 5), coefficient fit in the metric of the local factor (Eq. 6), then
 * refine_iters times: column-wise nearest-level bit-plane update with error propagation
 * (Eq. 3-4, 7-8), coefficient refit, delta correction (Eq. 9); the iterate with the smallest
 * ||E_group||_F^2 is kept (the initial state counts as iterate 0; ties keep the earliest).
 * Its propagation error reaches the columns not yet quantized exactly as
 * W'[:, end:] -= E_blk U[blk, end:] per block (and E* U[grp, rest of block] inside a block):
 * one GEMM per block for the far columns, applied one block late and overlapped with the next
 * sweep, while the groups of the next block read the pending terms directly from the kept E*.
 *   W       : d_out x d_in, read only.
 *   U, dead : from bpdq_prepare (dead may be NULL).
 *   planes  : uint32 [bits][d_out][d_in/32]; column c of plane B_i (i = 1..bits) is bit
 *             (c % 32) of word planes[i-1][r][c/32], least significant bit first.
 *   coefs   : float [bits+1][d_out][d_in/g]; index 0 is the bias C_0.
 *   W_hat   : float d_out x d_in, or NULL.  Equal to bpdq_dequant(planes, coefs) bit for bit.
 *   grp_err : double [d_in/g], ||E_group||_F^2 of the kept iterate; their sum is the layer
 *             objective tr((W-What) Ht (W-What)^T) (App. B.2).
 *   grp_iter: int [d_in/g], index of the kept iterate (0..refine_iters).
 * Requirements: d_in % group == 0, d_in % 32 == 0, group | max(block, group). */
size_t bpdq_quantize_workspace_bytes(int d_out, int d_in, const bpdq_params* p /* host */);
int bpdq_quantize_layer(const float* W, int d_out, int d_in, const float* U,
                        const unsigned char* dead, const bpdq_params* p /* host */,
                        uint32_t* planes, float* coefs, float* W_hat, double* grp_err,
                        int* grp_iter, void* ws, size_t ws_bytes, void* stream);

/* The lazy block update on its own (Eq. 4 applied to a whole block of finished columns, App. B.3
 * tail form), as bpdq_quantize_layer applies it inside the sweep:
 *     Wp[:, c_begin:c_end] -= E_blk U[k0:k0+Kd, c_begin:c_end]
 * on the fp32 matrix cores, in place.
 *   Et : the block's propagation coordinates, transposed: Kd x lde, row k holds E[:, k0 + k] for all
 *        d_out rows (lde >= d_out; the lde - d_out padding entries of a row are read and ignored).
 *   U  : the factor from bpdq_prepare, leading dimension ldu;  Wp: d_out x ldw working weights.
 * Requirements: lde, ldu multiples of 4; Et, U 16-byte aligned; c_begin, c_end multiples of 4.
 * Exposed for parity tests and for measuring this GEMM by itself. */
int bpdq_block_update(const float* Et, int lde, int Kd, const float* U, int ldu, int k0, float* Wp,
                      int ldw, int d_out, int c_begin, int c_end, void* stream);

/* Layers that share one input (q/k/v, up/gate) share H and U; stacked by rows they go through the
 * sweep in one call.  Every formula of the method is row-wise; only the choice of the kept
 * iterate is made per weight matrix (Sec. 3.3), so it is made per layer here:
 *   W       : the layers stacked by rows, d_out rows in all; planes / coefs / W_hat likewise.
 *   seg_end : host array of n_seg (1..8) ascending row boundaries, seg_end[n_seg-1] == d_out;
 *             every layer but the last must have a multiple of 16 rows.
 *   grp_err, grp_iter : [n_seg][d_in/g].
 * The results equal those of n_seg separate bpdq_quantize_layer calls bit for bit; the workspace
 * is bpdq_quantize_workspace_bytes(d_out, d_in, p). */
int bpdq_quantize_layers(const float* W, int d_out, int d_in, const float* U,
                         const unsigned char* dead, const bpdq_params* p /* host */, int n_seg,
                         const int* seg_end /* host */, uint32_t* planes, float* coefs,
                         float* W_hat, double* grp_err, int* grp_iter, void* ws, size_t ws_bytes,
                         void* stream);

/* ---- storage format helpers (Eq. 1) -------------------------------------------------------
 * codes : uint8 d_out x d_in, bit (i-1) of a code is B_i.  planes as above. */
int bpdq_pack_planes(const unsigned char* codes, int d_out, int d_in, int bits,
                     uint32_t* planes, void* stream);
/* W_hat[r][c] = ((C_0 + b_1 C_1) + b_2 C_2) + ... evaluated in fp32 in this order. */
int bpdq_dequant(const uint32_t* planes, const float* coefs, int d_out, int d_in, int bits,
                 int group, float* W_hat, void* stream);

/* Storage format with 16-bit coefficients: k plane bits per weight plus (k+1) halves per
 * (row, group), i.e. k + 16 (k+1) / g bits per weight (the BPW column of Table 1).
 * bpdq_coefs_to_fp16: out[i] = half(coefs[i]), round to nearest even, n values (uint16 bit
 * patterns).  bpdq_dequant_fp16: as bpdq_dequant with the coefficients read as halves; the sum
 * is evaluated in fp32 in the same order, so for a layer quantized with coef_fp16 = 1 it
 * reproduces that call's W_hat bit for bit. */
int bpdq_coefs_to_fp16(const float* coefs, long n, uint16_t* out, void* stream);
int bpdq_dequant_fp16(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in,
                      int bits, int group, float* W_hat, void* stream);

/* ---- serving side: y = What x for one token, straight from the stored format (Sec. 5) -------
 * Eq. 1 regrouped per (row, group G):
 *   y_r = sum_G ( C_0[r,G] S(G) + sum_i C_i[r,G] sum_{c in G} B_i[r,c] x_c ),  S(G) = sum_{c in G} x_c
 * so a weight costs no multiply: the inner sums come from a table of the 16 partial sums of every
 * 4 consecutive x values.  The planes are read once (bits/8 bytes per weight), the coefficients
 * as halves; fp32 accumulation in a fixed order.
 *   planes : as above;  coefs_h : half [bits+1][d_out][d_in/g];  x : float d_in;  y : float d_out.
 * Requirements: d_in % 32 == 0, 32 | group | d_in, x 16-byte aligned. */
int bpdq_gemv(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in, int bits,
              int group, const float* x, float* y, void* stream);

/* ---- serving side: the product for any number of tokens, with what surrounds it ---------------
 * Y[t][r] = act( sum_c What[r][c] X[t][c] + bias[r] ) + residual[t][r],  What as in bpdq_dequant_fp16 (Eq. 1), straight
 * from the stored planes and coefficients.
 *   X : n_tok x d_in, row stride ldx;  bias : d_out or NULL;  residual : n_tok x d_out, row stride ldr, or NULL;
 *   Y : n_tok x d_out, row stride ldy.  All of one type, BPDQ_F16 or BPDQ_BF16 (uint16 bit patterns); strides in elements.
 *   act : BPDQ_ACT_*; GELU is v Phi(v), GELU_TANH its approximation by tanh, SILU v / (1 + exp(-v)), each in fp32 with a relative error below
 *   2^-16, and 2^-21 of the exponential's argument where that is larger.
 * What is evaluated in fp32 and rounded once to fp16; X in bf16 is scaled by a power of two per token and taken as fp16, which changes no
 * value above 2^-29 of the token's largest; the products are exact, sums, bias, activation and residual fp32; Y is rounded once.
 * (A level of a row beyond 65504 becomes infinite.)  A NaN or infinity in a row of X reaches that row of Y alone.
 * (For one fp32 token without any of that bpdq_gemv is quicker.)
 * Y may be the residual itself (same address and stride); other overlaps are not allowed.  The result of a token does not
 * depend on the others of the call beyond the choice of kernel by n_tok, which changes the order of sums.
 * From 33 tokens on X is brought into the order of the matrix instructions first, in ws: 256-byte aligned,
 * bpdq_linear_workspace_bytes() bytes (0 for fewer tokens, ws may be NULL then).
 * Requirements: d_in % 32 == 0, 32 | group | d_in; any alignment of the elements (X aligned to 16 bytes with ldx % 8 == 0,
 * and planes likewise with d_in % 128 == 0, are quicker).  n_tok = 0 launches nothing.
 * Returns 0, or a negative code naming the argument (-1 planes, -2 coefs_h, -3 d_out, -4 d_in, -5 bits, -6 group, -7 X,
 * -8 n_tok, -9 ldx, -10 dtype, -11 bias, -12 act, -13 residual, -14 ldr, -15 Y, -16 ldy, -17 ws, -18 ws_bytes). */
#define BPDQ_F32 0
#define BPDQ_F16 1
#define BPDQ_BF16 2
#define BPDQ_ACT_NONE 0
#define BPDQ_ACT_RELU 1
#define BPDQ_ACT_GELU 2
#define BPDQ_ACT_GELU_TANH 3
#define BPDQ_ACT_SILU 4
size_t bpdq_linear_workspace_bytes(int n_tok, int d_in);
int bpdq_linear(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in, int bits, int group,
                const void* X, int n_tok, long ldx, int dtype, const void* bias, int act,
                const void* residual, long ldr, void* Y, long ldy, void* ws, size_t ws_bytes, void* stream);

/* The two projections of a gated feed-forward block in one call:
 *   Y[t][f] = act( sum_c Wgate[f][c] X[t][c] + bias[f] ) * ( sum_c Wup[f][c] X[t][c] + bias[d_out + f] ),
 * f < d_out, from two layers stacked by rows (2 d_out rows, gate first), as bpdq_quantize_layers leaves layers that share one input.
 *   planes : [bits][2 d_out][d_in/32];  coefs_h : [bits+1][2 d_out][d_in/group];  bias : 2 d_out values or NULL;  Y : n_tok x d_out, row stride ldy.
 * Types, activations, precision, workspace (bpdq_linear_workspace_bytes) and requirements are those of bpdq_linear; neither projection is rounded
 * before the product.  (One token of up to 8192 columns: weights are not rounded to fp16 either, and X in bf16 keeps all its bits, so its result is a little
 * nearer than that of the same token among others.)  Y must not overlap X.  A plane (2 d_out x d_in bits) has to be below 4 GiB.
 * Returns 0, or a negative code naming the argument (-1 planes, -2 coefs_h, -3 d_out, -4 d_in, -5 bits, -6 group, -7 X,
 * -8 n_tok, -9 ldx, -10 dtype, -11 bias, -12 act, -13 Y, -14 ldy, -15 ws, -16 ws_bytes). */
int bpdq_gated_linear(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in, int bits, int group,
                      const void* X, int n_tok, long ldx, int dtype, const void* bias, int act, void* Y, long ldy,
                      void* ws, size_t ws_bytes, void* stream);

/* ---- serving side: the norm before a product --------------------------------------------------
 *   S[t] = X[t] + residual[t],    Y[t][c] = S[t][c] / sqrt( mean_c S[t][c]^2 + eps ) * (offset + weight[c])
 *   X : n_tok x d, row stride ldx, of type dtype (BPDQ_F32, BPDQ_F16 or BPDQ_BF16), and so weight (d values, or NULL: ones, with offset 0 as they are)
 *   and Y (row stride ldy);  residual : NULL, or n_tok x d, row stride ldr, of type rdtype: dtype or BPDQ_F32;  S : NULL, or the sum in the
 *   residual's type, row stride lds (only with a residual).
 * The sum is fp32 and is rounded once for S; Y comes from it unrounded, its squares summed in fp64, the rest fp32, Y rounded once.  A row with a
 * NaN or an infinity gets NaN (at an infinity) and zeros or NaN elsewhere; other rows do not see it.
 * S may be the residual or X, and Y may be X (same address, type and stride); other overlaps are not allowed.
 * Requirements: 1 <= d <= 65536; eps >= 2^-126; offset and eps finite; any alignment of the elements (16 bytes, strides too, is quicker); n_tok
 * times the threads of a row (d / 16 rounded up to whole wavefronts, 1024 at most) below 2^32.  n_tok = 0 launches nothing.
 * Returns 0, or a negative code naming the argument (-1 X, -2 n_tok, -3 d, -4 ldx, -5 dtype, -6 residual, -7 ldr, -8 rdtype, -9 S, -10 lds,
 * -11 weight, -12 offset, -13 eps, -14 Y, -15 ldy). */
int bpdq_rms_norm(const void* X, int n_tok, int d, long ldx, int dtype, const void* residual, long ldr, int rdtype, void* S,
                  long lds, const void* weight, float offset, float eps, void* Y, long ldy, void* stream);
/* The same with Y in 8 bits, as it is kept or sent: codes[t][c] = rint(y / scale) in [-127, 127] (row stride ldc), y before any rounding, with one scale
 * for a row (group = 0) or for each `group` (32, 64, 128 or 256, a divisor of d) of its channels: scales[t][c / group], dense,
 * max(amax, 2^-96) * (1/127), amax the largest |y| of the group.  A row with a NaN or an infinity gets scales of NaN, and so does a group with a y that
 * is NaN or infinite by its weight; codes under a scale of NaN say nothing.
 * Returns as above (-14 group, -15 codes, -16 ldc, -17 scales). */
int bpdq_rms_norm_q8(const void* X, int n_tok, int d, long ldx, int dtype, const void* residual, long ldr, int rdtype, void* S,
                     long lds, const void* weight, float offset, float eps, int group, int8_t* codes, long ldc, float* scales,
                     void* stream);

/* ---- serving side: rotary positions ---------------------------------------------------------------
 * Turns channel pair i of every head of Q and K at position p by the angle p freq[i]:
 *   (a, b) -> mscale (a cos - b sin, b cos + a sin),   i < rot / 2; channels from rot on are passed on as they are.
 *   layout : BPDQ_ROTARY_HALF pairs (i, i + rot/2), BPDQ_ROTARY_INTERLEAVED pairs (2i, 2i+1).  inverse != 0 turns back (by -p freq[i]).
 *   freq : rot / 2 doubles on the GPU, radians per position;  pos, tok_start, n_seq, n_tok, max_tok : as in bpdq_kv_write, the call's next user:
 *   row tok_start[b] + i is at position pos[b] + i.  Rows of a sequence with pos < 0, and rows that no sequence names, are left alone.
 *   Q : n_tok rows of n_q heads of head_dim values, row stride ldq, into Q_out (row stride ldqo);  K likewise (n_kv = 0: none).
 *   dtype : BPDQ_F32, BPDQ_F16 or BPDQ_BF16.  Q_out may be Q and K_out may be K (same stride); other overlaps are not allowed.
 * The angle is formed in fp64, so far positions are as good as near ones (2^-24 of a turn); the rotation is fp32, rounded once.
 * Requirements: rot even, 2 <= rot <= head_dim <= 512; n_seq <= 65535; any alignment of the elements.
 * n_seq = 0, n_tok = 0, max_tok = 0 or no heads launches nothing.
 * Returns 0, or a negative code naming the argument (-1 freq, -2 rot, -3 layout, -4 mscale, -6 pos, -7 tok_start, -8 n_seq, -9 n_tok,
 * -10 max_tok, -11 Q, -12 ldq, -13 n_q, -14 K, -15 ldk, -16 n_kv, -17 head_dim, -18 dtype, -19 Q_out, -20 ldqo, -21 K_out, -22 ldko). */
#define BPDQ_ROTARY_HALF 0
#define BPDQ_ROTARY_INTERLEAVED 1
int bpdq_rotary(const double* freq, int rot, int layout, float mscale, int inverse, const int* pos, const int* tok_start,
                int n_seq, int n_tok, int max_tok, const void* Q, long ldq, int n_q, const void* K, long ldk, int n_kv,
                int head_dim, int dtype, void* Q_out, long ldqo, void* K_out, long ldko, void* stream);
/* The frequencies of the usual scalings, on the host: with f_i = base^(-2i/rot),
 *   PLAIN f_i;  LINEAR f_i / factor;  NTK the base times factor^(rot/(rot-2)) (rot > 2);
 *   YARN f_i for pairs that make `high` or more turns in `original` positions, f_i / factor for `low` or fewer, and a ramp over the pairs between
 *   (pairs counted down and up to whole ones), *mscale = 0.1 log(factor) + 1;
 *   BANDS the same ends with a ramp over the number of turns.
 * freq : rot / 2 doubles;  mscale : NULL, or the factor for bpdq_rotary (1 but for YARN).  factor >= 1; 0 < low < high.
 * Returns 0, or a negative code naming the argument (-1 rot, -2 base, -3 scaling, -4 factor, -5 low, -6 high, -7 original, -8 freq). */
#define BPDQ_ROTARY_PLAIN 0
#define BPDQ_ROTARY_LINEAR 1
#define BPDQ_ROTARY_NTK 2
#define BPDQ_ROTARY_YARN 3
#define BPDQ_ROTARY_BANDS 4
int bpdq_rotary_frequencies(int rot, double base, int scaling, double factor, double low, double high, int original,
                            double* freq /* host */, double* mscale /* host */);

/* ---- serving side: the next token ------------------------------------------------------------------
 * For each row of logits (n_tok x n_vocab, row stride ldl, of type dtype), with M its largest value, T = temperature and w_i = exp((x_i - M) / T):
 *   top_k  keeps the k largest values;
 *   top_p  keeps of these, in descending order, the fewest whose weights add up to at least top_p times theirs in all (one at least);
 *   min_p  keeps of these what has w_i >= min_p (more than 1 counts as 1);
 *   token  = the lowest kept index i with  sum_{kept j <= i} w_j  >  u * sum_{kept j} w_j;   prob = w_i over that sum.
 * Of equal values the lower index comes first.  T must be above 0: any other T (a NaN too) asks for the largest value, prob 1.  top_k <= 0, top_p >= 1 or
 * NaN and min_p <= 0 or NaN keep all.  u in [0, 1); below (or NaN) counts as 0, from 1 on as the last.
 *   temperature, top_k, top_p, min_p : n_tok values each, or NULL (T = 1; nobody asks).  u : n_tok floats.
 *   token : n_tok ints;  prob : NULL or n_tok floats.  (The workspace is some 43 KB a row.)
 * A value of minus infinity or NaN is not there; a row where nothing is there gets token -1 and prob 0.  Plus infinities share the row equally.
 * Weights are counted in units of 2^-43 of the largest (a token below half a unit is never drawn and adds nothing), their sums are exact, and the
 * result is the same from run to run.
 * Requirements: n_tok <= 32768, n_vocab <= 2^20; ws 256-byte aligned, of bpdq_sample_workspace_bytes() bytes; any alignment of the elements.  n_tok = 0 launches nothing.
 * Returns 0, or a negative code naming the argument (-1 logits, -2 n_tok, -3 n_vocab, -4 ldl, -5 dtype, -6 temperature, -7 top_k, -8 top_p,
 * -9 min_p, -10 u, -11 token, -12 prob, -13 ws, -14 ws_bytes). */
size_t bpdq_sample_workspace_bytes(int n_tok, int n_vocab);
int bpdq_sample(const void* logits, int n_tok, int n_vocab, long ldl, int dtype, const float* temperature, const int* top_k,
                const float* top_p, const float* min_p, const float* u, int* token, float* prob, void* ws, size_t ws_bytes,
                void* stream);

/* ---- serving side: keys and values in 8 bits --------------------------------------------------
 * The cache is in pages of `page` tokens.  A page and key head hold page * head_dim codes of K, as many of V, and one fp32
 * scale of each; a value is (code - 128) * scale, code - 128 in [-127, 127].  Which page holds which tokens of which
 * sequence is the caller's: row b of `page_table` (n_seq x max_pages ints) lists the pages of sequence b in order, so token
 * t of it is slot t % page of page page_table[b][t / page].
 * Layout of the head_dim * page bytes of a page and head: tiles of 64 tokens, in the order in which the matrix
 * instructions take them; token t = 16 g + 4 u + i of a tile (g, u, i in 0..3):
 *   K : [tile][u][d / 64][d % 64 / 16][g][i][d % 16]          V : [tile][d / 16][g][d % 16][t % 16]
 */
typedef struct bpdq_kv_cache {
  uint8_t* k;          /* [n_pages][n_kv][page * head_dim], 16-byte aligned */
  uint8_t* v;          /* likewise */
  float* k_scale;      /* [n_pages][n_kv] */
  float* v_scale;
  int n_pages;
  int n_kv;            /* key/value heads */
  int page;            /* tokens per page: 64, 128 or 256 */
  int head_dim;        /* 64, 128 or 256 */
} bpdq_kv_cache;

/* Quantizes new tokens into the cache.  Rows tok_start[b] .. tok_start[b+1]-1 of K and V (n_tok rows of n_kv heads of head_dim
 * values, row strides ldk, ldv in elements, of type dtype: BPDQ_F32, BPDQ_F16 or BPDQ_BF16) become tokens pos[b] ... of
 * sequence b.  max_tok: at least the largest count of a sequence.
 * Scale and codes, per page and head, in fp32:
 *   - the first slot of the page is among the new tokens: scale = max(amax, 2^-96) * (1/127), amax the largest magnitude of
 *     the page's new tokens; what the page held before is gone.
 *   - else the scale doubles until the new tokens fit: scale' = scale * 2^j, the smallest j >= 0 with amax <= 127 scale 2^j, and the
 *     codes of the tokens before become rint((code - 128) / 2^j) + 128.  Doubling bounds what repeated rounding can do: however many
 *     calls fill a page, no value is further than one step (scale) from what was written.
 *   code = rint(x * (1 / scale)) + 128, ties to even, clamped to 1..255.
 * A new token with a NaN or an infinity makes the scale of its page and head NaN, so all tokens of that page and head read as
 * NaN until the page is written from its first slot again.  Slots behind the last token written hold no promise.
 * A page must not belong to two sequences that the same call writes.  A sequence with pos < 0, tokens beyond max_pages pages, rows
 * beyond n_tok and pages outside [0, n_pages) are left out.
 * Requirements: k, v 16-byte aligned; n_seq <= 65535.  n_seq = 0, n_tok = 0 or max_tok = 0 launches nothing.
 * Returns 0, or a negative code naming the argument (-1 cache, -2 page_table, -3 max_pages, -4 n_seq, -5 pos, -6 tok_start,
 * -7 n_tok, -8 max_tok, -9 K, -10 ldk, -11 V, -12 ldv, -13 dtype). */
int bpdq_kv_write(const bpdq_kv_cache* cache /* host */, const int* page_table, int max_pages, int n_seq,
                  const int* pos, const int* tok_start, int n_tok, int max_tok, const void* K, long ldk,
                  const void* V, long ldv, int dtype, void* stream);
/* The inverse: tokens pos[b] .. of sequence b into rows tok_start[b] .. tok_start[b+1]-1 of K and V, (code - 128) * scale
 * rounded to dtype (so in fp16 what lies within half a step of 65504 may read as an infinity).  Tokens that bpdq_kv_write would leave out read as zero (rows of a sequence with pos < 0 and rows that no
 * sequence names are left alone).  Arguments and return codes as above. */
int bpdq_kv_read(const bpdq_kv_cache* cache /* host */, const int* page_table, int max_pages, int n_seq,
                 const int* pos, const int* tok_start, int n_tok, int max_tok, void* K, long ldk, void* V,
                 long ldv, int dtype, void* stream);

/* Attention of new tokens over the cache.  Sequence b has kv_len[b] tokens in the cache; its queries are rows q_start[b] ..
 * q_start[b+1]-1 of Q (n_tok rows of n_q heads of head_dim values, row stride ldq), n of them, the last of them at position
 * kv_len[b] - 1.  n_kv must divide n_q; query head h reads key head h / (n_q / n_kv).
 *   out[i][h] = sum_t p_t v_t,  p = softmax over the visible t of scale * <q_i, k_t>
 * Token t is visible to query i, at position p = kv_len - n + i, if t < kv_len, and t <= p where causal != 0, and t > p - window
 * where window > 0.  A query that sees nothing gets zeros.  What is not visible is not looked at: neither its codes nor, on a page
 * without visible tokens, the page's scale.
 *   Q, out : BPDQ_F16 or BPDQ_BF16;  lse : NULL, or n_tok x n_q floats: log of the sum of exp(scale <q, k>), -inf for a query that
 *   sees nothing.
 *   max_q, max_kv : at least the largest count of queries and of cached tokens of a sequence; all sequences are laid out by them (single
 *   tokens in one call with a long chunk go through the kernel for many rows, their caches unsplit: in a call of their own they are quicker),
 *   and longer sequences are cut to them.  max_kv <= max_pages * page and 2^30.
 * Scores and sums are fp32 on exact products (Q in bf16 is scaled by a power of two per row and head and taken as fp16, where a value
 * below 2^-31 of the row's largest may lose bits); the unnormalised probabilities are rounded to fp16 for the product with V: for
 * max_q * n_q / n_kv <= 32 with 11 bits where they are above 2^-14 of the row's maximum so far, for more rows times their page's scale of V,
 * with 11 bits where that product is above 2^-21 of the row's largest so far, and with fewer below; out is rounded
 * once.  A call's result does not change from run to run; the split of long caches depends on n_seq,
 * max_q, n_q, n_kv, head_dim, max_kv and window alone.  The cache's scales must not be negative (bpdq_kv_write's are not).
 * Pages outside [0, n_pages) count as not visible.
 * Requirements: n_seq <= 65535; max_q * (n_q / n_kv) <= 2^24; ws 256-byte aligned, of bpdq_kv_attention_workspace_bytes() bytes
 * (0 where nothing is split, ws may be NULL then).  out must not overlap Q.
 * Returns 0, or a negative code naming the argument (-1 cache, -2 page_table, -3 max_pages, -4 n_seq, -5 kv_len, -6 q_start,
 * -7 n_tok, -8 max_q, -9 max_kv, -10 Q, -11 ldq, -12 n_q, -13 dtype, -14 scale, -16 window, -17 out, -18 ldo, -20 ws,
 * -21 ws_bytes). */
size_t bpdq_kv_attention_workspace_bytes(int n_seq, int max_q, int max_kv, int n_q, int n_kv, int head_dim, int window);
int bpdq_kv_attention(const bpdq_kv_cache* cache /* host */, const int* page_table, int max_pages, int n_seq,
                      const int* kv_len, const int* q_start, int n_tok, int max_q, int max_kv, const void* Q,
                      long ldq, int n_q, int dtype, float scale, int causal, int window, void* out, long ldo,
                      float* lse, void* ws, size_t ws_bytes, void* stream);

/* ---- channel ordering around the pass (Sec. 4.1) --------------------------------------------
 * The pass quantizes the columns left to right; a caller that wants another order permutes W and
 * H first and carries `perm` with the stored layer.
 * bpdq_channel_order: perm[i] = original index of the channel at position i.
 *   group_size = 1: channels in descending order of H_jj (GPTQ's desc_act, Sec. 4.1); equal
 *     values keep their index order.
 *   group_size = g (divides d_in): every block of g consecutive channels stays together and in
 *     order, blocks sorted by the descending sum of their H_jj (fp64, index order) -- a
 *     group-preserving stand-in for the reordering the paper's experiments take from another
 *     paper, not that method.
 *   H: d_in x d_in, only the diagonal is read.  perm: d_in ints.  ws: 8-byte aligned,
 *   bpdq_channel_order_workspace_bytes(d_in) bytes.
 * bpdq_gather_columns:   Wp[r][i] = W[r][perm[i]]            (Wp must not alias W)
 * bpdq_scatter_columns:  W[r][perm[i]] = Wp[r][i]            (inverse; e.g. W_hat back in place)
 * bpdq_gather_symmetric: Hp[i][j] = H[perm[i]][perm[j]]      (H full/symmetrized; no aliasing)
 * perm must be a permutation of 0..d_in-1 (not checked). */
size_t bpdq_channel_order_workspace_bytes(int d_in);
int bpdq_channel_order(const float* H, int d_in, int group_size, int* perm, void* ws,
                       size_t ws_bytes, void* stream);
/* bpdq_channel_order for callers that cannot allocate device memory and have no workspace to
 * hand over (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * same arguments and result, the sort keys live in a 256 KB device array built into the library
 * (one copy per GPU, held until the process ends).  No hipMalloc / hipFree, no workspace.
 *   Limit: d_in / group_size <= 32768 keys; more returns -2 and launches nothing.
 *   All calls on one GPU share that array: calls that may overlap on one GPU (different streams,
 *   different host threads) race and must be serialised by the caller.  Nothing of an earlier
 *   call's contents enters a later result.
 * Returns 0, -1 H, -2 d_in (or too many keys), -3 group_size, -4 perm, BPDQ_ERR_LAUNCH. */
int bpdq_channel_order_noalloc(const float* H, int d_in, int group_size, int* perm, void* stream);
int bpdq_gather_columns(const float* W, int d_out, int d_in, const int* perm, float* Wp,
                        void* stream);
int bpdq_scatter_columns(const float* Wp, int d_out, int d_in, const int* perm, float* W,
                         void* stream);
int bpdq_gather_symmetric(const float* H, int d_in, const int* perm, float* Hp, void* stream);

/* ---- measurement probes (not part of the method) ---------------------------------------------
 * Ceilings of the GPU the library runs on, for quoting a kernel against what the hardware
 * sustains as well as against its published peak.
 * bpdq_probe_mfma: a register-only loop of one matrix-core instruction, no memory traffic:
 *   kind 0 v_mfma_f32_32x32x2_f32, 1 v_mfma_f32_32x32x16_bf16, 2 v_mfma_f32_32x32x16_f16,
 *   3 v_mfma_f64_16x16x4_f64, 4 v_mfma_i32_32x32x32_i8 (ops instead of flops; normal operands are
 *   round(32 z) clamped to +-127);  data 0 zeros, 1 ones, 2 standard normal operand values (the
 *   sustained clock depends on the operand bits that toggle);  waves_per_simd 1 or 2;
 *   `groups` work-groups (256 = one per compute unit) of 4 * waves_per_simd wavefronts, each
 *   issuing 8 * iters instructions on a 2 x 4 grid of independent accumulator tiles (fp64: 16 * iters
 *   on 4 x 4).
 *   out: device floats, groups * 256 * waves_per_simd of them (keeps the results alive).
 *   flops (host, may be NULL): receives the flops the launch performs.  Time it with events.
 * bpdq_probe_copy: dst[i] = src[i], n_floats (multiple of 4) floats, 16-byte aligned: the plain
 *   streaming copy HBM counters and bandwidth are scaled by. */
int bpdq_probe_mfma(int kind, int data, int waves_per_simd, int groups, int iters, float* out,
                    double* flops /* host */, void* stream);
int bpdq_probe_copy(const float* src, float* dst, long n_floats, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BPDQ_H */
