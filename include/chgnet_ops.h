/*
 * chgnet_ops.h - operators of the training step for models of the caller's own.
 *
 * Two pieces of the step in chgnet.h as calls on plain arrays: the gate of the
 * gated MLP (GatedMLP of Eq. 4-6: LayerNorm, SiLU and sigmoid, product) with an
 * 8-bit checkpoint of its input for the backward pass, and the embedding lookup
 * (Eq. 2) with a scale, and its gradient. chgnet_step, chgnet_forward and
 * chgnet_backward keep their pre-activations in the same checkpoint with
 * chgnet_hparams.act_bits = 8, and sum the element table's gradient with
 * chgnet_embed_backward's kernels on large batches.
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

#ifdef __cplusplus
}
#endif
#endif /* CHGNET_OPS_H */
