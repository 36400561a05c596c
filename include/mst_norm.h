/*
 * mst_norm.h -- C ABI of what stands between the mini-sequence blocks
 *               (hand-written HIP for gfx950 / MI355X): the norm before a
 *               block, the gated and scaled residual after it (with a norm of
 *               its own or without), both in one pass, their gradients, and
 *               8-bit checkpoints of activations that the gradients read.
 *
 * With X the residual stream [S, d], O what a block gave, all per row r and
 * column j (L = gate_rows: rows that share a row of the gate):
 *
 *   norm(x)_j = x_j * rstd,  rstd = (mean_j x_j^2 + eps)^(-1/2)
 *   before a block   H = norm(X) * (w_offset + w_pre)
 *   after it         Y = X + scale * gate[r / L] * N
 *                    N = norm(O) * (w_offset + w_post)   (normalize != 0), or O
 *   between blocks   Y as above, then H = norm(Y) * (w_offset + w_pre)
 *
 * and, given gradients of H and Y, with ~w = w_offset + w and a hat on what is
 * divided by its root mean square:
 *
 *   before   a = dH * ~w_pre;      dX = dres + rstd * (a - ^X * mean_j(a * ^X))
 *            dw_pre = sum_r dH * ^X
 *   after    e = scale * gate * dY;  b = e * ~w_post
 *            dO = rstd * (b - ^O * mean_j(b * ^O))       (or e without the norm)
 *            dw_post = sum_r e * ^O;  dgate[g] = sum_{r / L = g} scale * dY * N
 *            (the gradient of X is dY itself)
 *   between  dY = dres + the gradient through the norm as above, then the rest
 *            with this dY, before it is rounded to the stream's type
 *
 * The checkpoint of a tensor [S, d] holds a signed 8-bit code per entry and a
 * scale per block of 32 columns (the last block of a row is shorter where
 * d % 32 != 0):
 *
 *   exps  [S, ceil(d / 32)]   byte E; the block's scale is 2^(E - 127), the
 *                             smallest such (E >= 0) that is more than the
 *                             block's largest magnitude / 127.5
 *   codes [S, d]              entry / scale to the nearest integer, ties to
 *                             even: -127 .. 127
 *
 * Both divisions and products by a power of two are exact, so the error is half
 * a step: at most 1 / 127.5 of the block's largest magnitude, or, with E = 0
 * (largest magnitudes below 127.5 * 2^-127), at most 2^-128.  The codes are a
 * function of the tensor alone, and what a code stands for fits bf16 without a
 * second rounding: 33 bytes for 32 entries.  A block with a NaN, an infinity or
 * a magnitude from 127.5 * 2^121 on (3.39e38, which would be rounded to 2^128) has
 * E = 255 and stands for NaN throughout (its codes are unspecified).
 *
 * Conventions (where not said otherwise, those of mst_lmhead.h)
 *   - Every pointer is a DEVICE pointer owned by the caller.  The calls only
 *     enqueue kernels on `stream` (capturable into a HIP graph after one eager
 *     call in the process); they allocate nothing and keep nothing.  Nothing
 *     but the checkpoint is handed from a forward to a backward call.  A
 *     workspace must not be shared by calls (or replays of graphs) that may run
 *     at the same time.
 *   - stream_type: type of the residual stream (X, Y, dres, dX, dY), MST_TYPE_BF16
 *     or MST_TYPE_FP32.  H, O, dH, dO, weights and gates are bf16, gradients of
 *     weights and gates fp32 (each fully overwritten).  Everything is computed
 *     in fp32 and rounded once; a row's sum of squares has to be a finite fp32
 *     number.  Sums over rows have a fixed order that depends on S, d, the gate's
 *     rows and the call alone (no atomics: bit-identical across calls).
 *   - A weight pointer that may be NULL stands for ones: the norm then has the
 *     factor w_offset + 1, and its gradient's pointer must be NULL too.
 *   - Where a backward call takes a tensor or its checkpoint, exactly one of the
 *     two is given (both of codes and exps, or neither).
 *   - Tensors are row-major without padding.  Requirements: 1 <= S < 2^30;
 *     8 <= d <= MST_NORM_MAX_D, d % 8 == 0, S * d <= 2^36; eps, scale and
 *     w_offset finite, eps >= 2^-100; gate_rows >= 1 with a gate (which has
 *     ceil(S / gate_rows) rows), 0 without; all tensors 16-byte
 *     aligned but exps (any), workspace 256-byte aligned.
 *   - An output may be the very memory of an input of S * d entries of the same
 *     size (Y of X, dX of dres, ...); no output may overlap anything otherwise.
 *   - Return value: MST_OK or a negative error code of mst_lmhead.h, found on
 *     the host before anything is launched; MST_ERR_BAD_ARGUMENT for values out
 *     of range, pointers that exclude or need each other, and overlaps.
 */
#ifndef MST_NORM_H
#define MST_NORM_H

#include "mst_lmhead.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MST_TYPE_BF16 = 0, MST_TYPE_FP32 = 1 };

#define MST_NORM_MAX_D 16384

/* host: "mst-norm <version> (gfx950)" */
const char* mst_norm_version(void);

/*
 * Bytes of workspace of the three backward calls (host, pure): partial sums over rows.  gate_rows: as in the
 * call, 0 without a gate (and for mst_prenorm_bwd).  The calls without one (forward, checkpoints) need none.
 */
mst_status mst_norm_workspace_bytes(int64_t S, int64_t d, int64_t gate_rows, size_t* bytes);

/*
 * Checkpoint of X [S, d] of type `type`, and back: the tensor of type `type` that the checkpoint stands for
 * (the same values in either type).
 */
mst_status mst_ckpt_pack(const void* X, int32_t type, int64_t S, int64_t d, int8_t* codes, uint8_t* exps, void* stream);
mst_status mst_ckpt_unpack(const int8_t* codes, const uint8_t* exps, int64_t S, int64_t d, void* X, int32_t type, void* stream);

/*
 * Norm before a block.
 *   X  [S, d] stream type    w_pre [d] bf16 or NULL    H [S, d] bf16, out
 *   codes, exps   out, both NULL or both given: the checkpoint of X
 * mst_prenorm_rebuild: H again from that checkpoint.
 */
mst_status mst_prenorm_fwd(const void* X, int32_t stream_type, const void* w_pre, float w_offset, float eps,
                           int64_t S, int64_t d, void* H, int8_t* codes, uint8_t* exps, void* stream);
mst_status mst_prenorm_rebuild(const int8_t* codes, const uint8_t* exps, const void* w_pre, float w_offset, float eps,
                               int64_t S, int64_t d, void* H, void* stream);

/*
 * Its gradients.
 *   dH [S, d] bf16; X or its checkpoint; dres [S, d] stream type or NULL: what reaches X around the block
 *   dX [S, d] stream type, out;  dw_pre [d] fp32, out (NULL with w_pre NULL)
 */
mst_status mst_prenorm_bwd(const void* dH, const void* X, const int8_t* codes, const uint8_t* exps, const void* dres,
                           int32_t stream_type, const void* w_pre, float w_offset, float eps, int64_t S, int64_t d,
                           void* workspace, size_t workspace_bytes, void* dX, float* dw_pre, void* stream);

/*
 * Gated and scaled residual after a block.
 *   O [S, d] bf16;  X [S, d] stream type;  gate [ceil(S / gate_rows), d] bf16 or NULL (ones; gate_rows = 0)
 *   normalize   whether O passes a norm of weight w_post ([d] bf16 or NULL; NULL without the norm)
 *   Y [S, d] stream type, out;  codes, exps: as above, the checkpoint of O
 */
mst_status mst_residual_fwd(const void* O, const void* X, int32_t stream_type, int32_t normalize, const void* w_post,
                            float w_offset, float eps, const void* gate, int64_t gate_rows, float scale,
                            int64_t S, int64_t d, void* Y, int8_t* codes, uint8_t* exps, void* stream);

/*
 * Its gradients.  O or its checkpoint: neither is needed (or looked at) without norm and gate.
 *   dY [S, d] stream type;  dO [S, d] bf16, out
 *   dw_post [d] fp32, out, NULL where w_post is;  dgate [ceil(S / gate_rows), d] fp32, out, NULL where gate is
 */
mst_status mst_residual_bwd(const void* dY, int32_t stream_type, const void* O, const int8_t* codes, const uint8_t* exps,
                            int32_t normalize, const void* w_post, float w_offset, float eps,
                            const void* gate, int64_t gate_rows, float scale, int64_t S, int64_t d,
                            void* workspace, size_t workspace_bytes, void* dO, float* dw_post, float* dgate, void* stream);

/*
 * The end of one block and the begin of the next in one pass: mst_residual_fwd, then mst_prenorm_fwd of its Y (H is formed
 * from Y before Y is rounded, the checkpoint of Y from Y as it is stored).  Both norms have the same w_offset and eps.
 */
mst_status mst_residual_prenorm_fwd(const void* O, const void* X, int32_t stream_type, int32_t normalize, const void* w_post,
                                    const void* gate, int64_t gate_rows, float scale, const void* w_pre,
                                    float w_offset, float eps, int64_t S, int64_t d, void* Y, void* H,
                                    int8_t* codes_o, uint8_t* exps_o, int8_t* codes_y, uint8_t* exps_y, void* stream);

/*
 * Its gradients: mst_prenorm_bwd, whose dX is dY here, then mst_residual_bwd with this dY (before it is rounded).  Y and O:
 * each the tensor or its checkpoint.
 */
mst_status mst_residual_prenorm_bwd(const void* dH, const void* dres, int32_t stream_type,
                                    const void* Y, const int8_t* codes_y, const uint8_t* exps_y,
                                    const void* O, const int8_t* codes_o, const uint8_t* exps_o,
                                    int32_t normalize, const void* w_post, const void* gate, int64_t gate_rows, float scale,
                                    const void* w_pre, float w_offset, float eps, int64_t S, int64_t d,
                                    void* workspace, size_t workspace_bytes, void* dY, void* dO,
                                    float* dw_pre, float* dw_post, float* dgate, void* stream);

/*
 * How a backward call goes over the rows (host, pure; a test aid; prenorm: 0 for mst_residual_bwd): info = {threads of
 * a workgroup, teams of lanes in it that hold a row each, rows that a team takes in turn, workgroups, 1 where a team takes
 * whole rows of the gate}.
 */
mst_status mst_norm_bwd_info(int64_t S, int64_t d, int64_t gate_rows, int32_t prenorm, int64_t* info);

#ifdef __cplusplus
}
#endif
#endif /* MST_NORM_H */
