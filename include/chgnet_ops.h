/*
 * chgnet_ops.h - operators of the training step for models of the caller's own.
 *
 * Pieces of the step in chgnet.h, and what a deep network out of them needs around
 * them, as calls on plain arrays. The first two: the gate of the
 * gated MLP (GatedMLP of Eq. 4-6: LayerNorm, SiLU and sigmoid, product) with an
 * 8-bit checkpoint of its input for the backward pass, and the embedding lookup
 * (Eq. 2) with a scale, and its gradient. chgnet_step, chgnet_forward and
 * chgnet_backward keep their pre-activations in the same checkpoint with
 * chgnet_hparams.act_bits = 8, and sum the element table's gradient with
 * chgnet_embed_backward's kernels on large batches. Then: norms, the residual
 * connection around a block with its gate and dropout, dropout alone, and matrices
 * in 8-bit floating point with their products, for linear layers.
 *
 * The conventions of chgnet.h hold: device pointers owned by the caller, no
 * allocation, work enqueued on `stream` of the current device, error codes,
 * results bitwise reproducible run to run (no floating-point atomics). No call
 * waits on the host, so all of them can be captured into a HIP graph; calls
 * that may overlap in time need workspaces of their own (a replayed graph uses
 * the workspace it was captured with). Workspace contents need no
 * initialisation and hold nothing between calls.
 *
 * Arrays of `dtype` hold fp32, bf16 or fp16 values, aligned to their size;
 * arithmetic and sums are fp32, rounded once where a result is stored in 16
 * bits. ld* are row strides in values, at least the row's width. Outputs must
 * not overlap inputs or each other. Widths and strides that are multiples of 4
 * values, with arrays on 16-byte boundaries, take vector loads. Zero rows
 * (tokens) are valid: no row is written, gradients of the whole are zero (or
 * unchanged with `accumulate`).
 */
#ifndef CHGNET_OPS_H
#define CHGNET_OPS_H

#include "chgnet.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CHGNET_F32 0
#define CHGNET_BF16 1
#define CHGNET_F16 2

/* Gate, forward. z [rows, 2d] (columns core | gate), ln [4, d] fp32: the
 * LayerNorm scale and shift g_c, b_c of the core and g_g, b_g of the gate, as
 * they follow each other in the flat parameter vector:
 *   phi = SiLU(LN(core) g_c + b_c) * sigmoid(LN(gate) g_g + b_g)   [rows, d]
 * with LN(x) = (x - mean) / sqrt(var + 1e-5) over the row's d values, mean and
 * variance in fp32. Where the variance passes fp32's range (a deviation of 1.8e19)
 * LN(x) is 0 and no gradient passes it, in both passes. The mean is off by its
 * rounding: values far from zero for their deviation (or that of 1e-5) have an
 * LN(x) that is off by some 1e-7 of their ratio. 1 <= d <= 1024.
 *
 * With codes != NULL also the checkpoint for chgnet_gate_backward: codes
 * [rows, 2d] bytes and step [rows, 2] fp32 (8-byte aligned). For each half x of
 * a row:
 *   step = max((max x - min x) * fl(1/255), 2^-100)
 *   code = round_to_even((x - min x) * fl(1/step))
 * (difference and quotient rounded to fp32, the product exact), so that
 * min x + code * step is within step/2 of x up to fp32 rounding. min x is not
 * kept: the LayerNorm takes it out. It is 2d + 8 bytes a row in place of 8d. A
 * half with a value that is not finite, or whose max - min is above fp32's
 * range, has a step that is not finite, and dz of its row and the LayerNorm
 * gradients are then NaN. codes == NULL (then step too): inference, nothing is
 * kept and phi has the same bits as with codes on a 4-byte boundary. */
int chgnet_gate_forward(int64_t rows, int32_t d, int32_t dtype, const void* z, int64_t ldz, const float* ln,
                        void* phi, int64_t ldphi, uint8_t* codes, float* step, void* stream);

/* Gate, backward, at the values that the checkpoint holds: dz [rows, 2d] from
 * dphi [rows, d] (both of `dtype`), and dln [4, d] fp32 = the gradients of ln,
 * added to what it holds with accumulate != 0, else overwritten. ws: at least
 * chgnet_gate_backward_workspace(rows, d) bytes, 16-byte aligned. */
int chgnet_gate_backward_workspace(int64_t rows, int32_t d, size_t* bytes);
int chgnet_gate_backward(int64_t rows, int32_t d, int32_t dtype, const uint8_t* codes, const float* step,
                         const float* ln, const void* dphi, int64_t lddphi, void* dz, int64_t lddz, float* dln,
                         int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Embedding lookup: out [n, d] row i = scale * table row (tok[i] - first), table
 * [vocab, d]; zeros where tok[i] - first is not in 0 .. vocab - 1 (padding).
 * first = 1 takes atomic numbers. tok int32, n >= 0, 1 <= d <= 65536,
 * 1 <= vocab < 2^31, first >= 0. */
int chgnet_embed_forward(int64_t n, int32_t d, int64_t vocab, int32_t dtype, const int32_t* tok, int32_t first,
                         const void* table, int64_t ldtable, float scale, void* out, int64_t ldout, void* stream);

/* Gradient of the table: dtable [vocab, d] fp32, row v = scale * sum of dout [n,
 * d] over the i with tok[i] - first = v (added to what it holds with accumulate
 * != 0), summed in fp32 in an order fixed by the sizes, the arrays' alignment and
 * the tokens. Tokens outside the table add nothing. n <= 2^30. ws: at least
 * chgnet_embed_backward_workspace(n, d, vocab) bytes, 16-byte aligned. */
int chgnet_embed_backward_workspace(int64_t n, int32_t d, int64_t vocab, size_t* bytes);
int chgnet_embed_backward(int64_t n, int32_t d, int64_t vocab, int32_t dtype, const int32_t* tok, int32_t first,
                          const void* dout, int64_t lddout, float scale, float* dtable, int64_t lddtable,
                          int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Norms of rows x [rows, d], n(x):
 *   CHGNET_NORM_RMS    x r,           r = 1 / sqrt(mean(x^2) + eps)
 *   CHGNET_NORM_LAYER  (x - mean) r,  r = 1 / sqrt(var + eps)
 *   CHGNET_NORM_NONE   x (where a call says so)
 * with sums in fp32. Where the mean square (the variance) passes fp32's range
 * n(x) is 0 and no gradient passes it. 1 <= d <= 16384, 1e-20 <= eps <= 1,
 * rows < 2^32. Parameters are fp32, one row [d] (scale) or two [2, d] (scale,
 * shift), at any float. */
#define CHGNET_NORM_NONE 0
#define CHGNET_NORM_RMS 1
#define CHGNET_NORM_LAYER 2

/* h = w[0] n(x) + w[1], and its gradients: dx from dh, dw [w_rows, d] fp32, added
 * to what it holds with accumulate != 0. ws: at least
 * chgnet_residual_backward_workspace(rows, d, w_rows) bytes, 16-byte aligned. */
int chgnet_norm_forward(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, int32_t kind, const float* w,
                        int32_t w_rows, float eps, void* h, int64_t ldh, void* stream);
int chgnet_residual_backward_workspace(int64_t rows, int32_t d, int32_t param_rows, size_t* bytes);
int chgnet_norm_backward(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, int32_t kind, const float* w,
                         int32_t w_rows, float eps, const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dw,
                         int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Residual connection around a block: its stream x [rows, d], its output f, and
 * the norms after it and before the next block:
 *   t = post[0] n_post(f) + post[1]
 *   y = alpha x + beta Drop(sigmoid(gate) t)
 *   h = pre[0] n_pre(y) + pre[1]        (y as it is stored)
 * post NULL (post_kind then CHGNET_NORM_NONE): t = f; with post and
 * CHGNET_NORM_NONE a learned scale. gate: pre-activations, [rows, gate_cols] with
 * gate_cols = d or 1 (one for the row), or NULL: no gate. pre NULL: no h. Drop is
 * chgnet_dropout's with p, seed, call and step (p = 0: none); what it drops of f and
 * gate has no part in y or in any gradient but through the norm's statistics. */
typedef struct chgnet_residual {
  int32_t post_kind, post_rows; /* CHGNET_NORM_*, rows of post */
  int32_t pre_kind, pre_rows;
  int32_t gate_cols;
  float alpha, beta, eps, p;
  uint64_t seed, call;
  const int64_t* step; /* on the GPU, 8-byte aligned, or NULL */
} chgnet_residual;

int chgnet_residual_forward(int64_t rows, int32_t d, int32_t dtype, const chgnet_residual* cfg, const void* x, int64_t ldx,
                            const void* f, int64_t ldf, const void* gate, int64_t ldgate, const float* post,
                            const float* pre, void* y, int64_t ldy, void* h, int64_t ldh, void* stream);

/* Its gradients from those of y (dy; NULL: zero) and of h (dh, with pre): dx, df,
 * dgate (with gate), and in fp32 dpost and dpre (with post and pre), added to what
 * they hold with accumulate != 0. Nothing of the forward pass is kept but y, which
 * is read with pre; f is read with post or gate. ws: at least
 * chgnet_residual_backward_workspace(rows, d, rows of post + rows of pre) bytes,
 * 16-byte aligned. */
int chgnet_residual_backward(int64_t rows, int32_t d, int32_t dtype, const chgnet_residual* cfg, const void* y, int64_t ldy,
                             const void* f, int64_t ldf, const void* gate, int64_t ldgate, const float* post,
                             const float* pre, const void* dy, int64_t lddy, const void* dh, int64_t lddh, void* dx,
                             int64_t lddx, void* df, int64_t lddf, void* dgate, int64_t lddgate, float* dpost, float* dpre,
                             int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Dropout of x [rows, d]: out = x / (1 - q) where a value is kept, else 0, with q
 * = p rounded to a multiple of 2^-16; q = 1 keeps none. Value (i, j) is kept if
 * its 16 bits are at least 2^16 q: half j % 2 (low first) of word (j % 8) / 2 of
 * Philox4x32-10 (Salmon et al., SC 2011) with the counter (j / 8, i, low and high
 * word of n) and the key (low and high word of seed), n = call + *step (mod 2^64;
 * step on the GPU, or NULL: 0). The same seed and n give the same mask, whatever
 * the type, width, strides and launch: the call on the upstream gradient is the
 * backward pass, and a graph that adds to *step draws anew at each replay. rows <
 * 2^32, 1 <= d <= 2^30, 0 <= p <= 1. */
int chgnet_dropout(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, float p, uint64_t seed,
                   uint64_t call, const int64_t* step, void* out, int64_t ldout, void* stream);

/* A matrix [rows, cols] in 8-bit floating point: codes (e4m3: 4 bits of
 * exponent, 3 of mantissa, largest 448) and for each block of block_rows (1 or
 * 128) x 128 of them an exponent byte, 2^(byte - 127), 255 for NaN:
 *   value[i][j] = code[i][j] 2^(scale[i / block_rows][j / 128] - 127)
 * Codes of a row follow each other, rows are ld bytes apart (a multiple of 16, on
 * 16-byte boundaries); where cols is no multiple of 16 the bytes up to the next one
 * are 0 (chgnet_fp8_quantize writes them). Scale rows are ld_scale bytes apart (a
 * multiple of 4, on 4-byte boundaries) and are read in words of 4. Strides are at most
 * 2^23, rows < 2^31, 0 <= cols <= 2^23; without columns there is nothing to read. */
typedef struct chgnet_fp8 {
  int64_t rows, cols;
  uint8_t* codes;
  int64_t ld;
  uint8_t* scale;
  int64_t ld_scale;
  int32_t block_rows;
} chgnet_fp8;

/* Quantises x [rows, cols] into q, and its transpose [cols, rows] into t, whose
 * blocks of 128 run along the rows of x; either may be NULL. A block's scale is
 * the least power of two by which its largest magnitude is at most 448, but at
 * least 2^-126; codes are rounded to nearest, ties to even. A block with a value that
 * is not finite has the scale NaN. With block_rows = 128 both forms hold the same
 * values. rows <= 2^23; with t or block_rows = 128 fewer than 2^40 values. */
int chgnet_fp8_quantize(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ldx, const chgnet_fp8* q,
                        const chgnet_fp8* t, void* stream);

/* out [M, N] of `dtype` = a b^T for a [M, K] and b [N, K], summed in fp32, added to
 * what it holds with accumulate != 0. A linear layer's y = x w^T, dx = dy w and dw =
 * dy^T x are this with the forms of chgnet_fp8_quantize: (x, w), (dy, w^T), (dy^T,
 * x^T). For 16-bit results the products of a block are added eight at a time, cut
 * off at 2^-13 of the largest one's power of two (of normal values some 2e-5 of a
 * result); for fp32 results they are exact, for values that are fp32 numbers (past
 * its largest they count as infinite, below 2^-126 they may count as 0). ws: at least
 * chgnet_fp8_matmul_workspace(M, N, K) bytes, 16-byte aligned (none where that is 0). */
int chgnet_fp8_matmul_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes);
int chgnet_fp8_matmul(const chgnet_fp8* a, const chgnet_fp8* b, int32_t dtype, void* out, int64_t ldout, int accumulate,
                      void* ws, size_t ws_bytes, void* stream);

/* Linear layer: out [rows, N] = q(x) w^T for x [rows, K] and w [N, K], where q(x) is
 * x as chgnet_fp8_quantize has it with block_rows = 1; out has x's dtype, summed
 * as chgnet_fp8_matmul does for that type (to fp32's last place of 16-bit x: that call
 * with fp32 results). rows <= 2^23. ws: at least chgnet_fp8_linear_workspace(rows, N, K)
 * bytes, 16-byte aligned. */
int chgnet_fp8_linear_workspace(int64_t rows, int64_t n, int64_t k, size_t* bytes);
int chgnet_fp8_linear(int64_t rows, int32_t dtype, const void* x, int64_t ldx, const chgnet_fp8* w, void* out,
                      int64_t ldout, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CHGNET_OPS_H */
