/*
 * head.h -- a projection head trained on and served beside an index, in
 * libpvs.so.
 *
 * The index of pvs.h holds vectors that a learned head makes of an encoder's
 * hidden rows.  These operators train such a head against the items of a
 * collection and serve it for single queries and for many:
 *   - softmax cross entropy of rows over the items (a large vocabulary), in
 *     pieces of the vocabulary, without keeping the logits, and its gradients;
 *   - rows kept in 8 bits between the forward and the backward pass, by the
 *     per-vector quantizer of Sec. 2.3.1, and the backward steps that read them;
 *   - distillation: the same softmax against a teacher's distribution over a list of
 *     items of each row, and its gradients;
 *   - rows of a table by their ids, scaled, and the table's gradient;
 *   - products of a few rows with weights kept in 4 bits, with group scales, and of any
 *     number of rows with both operands in microscaled 4-bit floating point.
 * The paper has no counterpart to them.
 *
 * Conventions:
 *   - Every matrix is in DEVICE memory, row-major with a leading dimension
 *     `ld` in elements (>= its columns); element types are pvs_dtype, held
 *     as the native bf16, f16 or float32.  Sums are float32; the tensor cores
 *     cut the sum of each step of 16 terms to 24 bits, where float32 arithmetic
 *     rounds.  A pointer is aligned to its elements where nothing else is said.
 *   - Every call queues its work on `cuda_stream` (a cudaStream_t; NULL: the
 *     legacy default stream) of the current device and returns; nothing is
 *     allocated and nothing waited for, so calls can be captured into a CUDA
 *     graph (but for the first call on a device, which sets it up).
 *   - Scratch is the caller's: the *_workspace call says how many bytes the
 *     operator wants for the same arguments (256-byte aligned device memory).
 *     It may be used again once the call's work is done.
 *   - A call returns PVS_ERR_INVALID for arguments that it can see to be
 *     wrong (sizes, null or misaligned pointers, unknown types, too small a workspace)
 *     and then queues nothing, PVS_ERR_CUDA where a CUDA call fails.  What
 *     only the device sees is said for each operator.  A device-side wait
 *     that runs out ends its kernel; the next call on that device that has
 *     work to queue, or pvs_head_status, then returns PVS_ERR_TIMEOUT once, and
 *     queues nothing: what was queued before it has no valid outputs.  (The
 *     status is the device's: whichever thread asks next has it.)
 */
#ifndef PVS_HEAD_H_
#define PVS_HEAD_H_

#include <stddef.h>
#include <stdint.h>

#include "pvs.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pvs_dtype { PVS_BF16 = 0, PVS_F16 = 1, PVS_F32 = 2 } pvs_dtype;

typedef enum pvs_act {
    PVS_ACT_NONE = 0,
    PVS_ACT_GELU = 1          /* x Phi(x), Phi the normal distribution function; +inf
                                 at +inf, NaN at -inf (-inf times 0) and at NaN.
                                 Its Phi is off by at most 7.5e-8 for bf16 and f16,
                                 in float32 by (x^2 + 6) 2^-23 of itself */
} pvs_act;

/* PVS_OK, or the status of an operator whose device-side wait ran out on the
 * current device since this was last asked (cleared by asking). */
pvs_status pvs_head_status(void);

/* Limit, in nanoseconds, of each wait of the tensor-core products that are
 * queued from now on on the current device (default and maximum 2e9, i.e. 2 s).
 * 0 makes every such wait give up at once unless what it waits for is already
 * there, which lets tests reach PVS_ERR_TIMEOUT without a fault.  A product's
 * waits for its own copies in flight always keep the 2 s limit.  A CUDA graph
 * keeps the limit that it was captured with. */
pvs_status pvs_head_set_wait_limit(int64_t ns);

/* ---------------------------------------------------------------------------
 * Softmax cross entropy.  For T = rows rows x_t and V = items vectors w_j of
 * `dim` elements, a = scale and b = bias (zeros where null):
 *     l_tj   = a <x_t, w_j> + b_j
 *     loss_t = ln(sum_j exp(l_tj)) - l_{t, targets[t]}
 * An item whose bias is -inf (a deleted one, a false negative) is not in the
 * softmax, whatever its vector holds, NaN and infinities too.
 *   - targets[t] == ignore_index: loss 0 and no gradient, whatever the row
 *     holds.  Any other target outside [0, items): the loss is NaN, and so
 *     are the gradients that the row reaches.
 *   - no item in the softmax: every loss is 0, and no gradient.
 *   - the target itself masked: loss +inf, and no gradient through the target.
 * NaN and overflows elsewhere reach the outputs as in that formula, but that
 * finite biases beyond 2.3e38 in size count as 2.36e38 (one of the lowest value at a
 * target gives its own loss).
 * bf16 and f16 products are exact.  float32 operands enter the logits as pairs
 * of f16 with a power of two for each row and item, and the gradients as three
 * bf16 parts; what is left out of a product is about 2^-22 of it.
 * Up to 16 float32 rows of dim <= 1024 are multiplied in float32 as they are.
 * ------------------------------------------------------------------------ */
typedef struct pvs_xent_args {
    const void* x;            /* [rows x dim], leading dimension ldx           */
    const void* w;            /* [items x dim], leading dimension ldw          */
    const int64_t* targets;   /* [rows]                                        */
    const float* bias;        /* [items] or null                               */
    int64_t rows, items;      /* rows, items <= 2^31 - 2^16; items >= 1           */
    int64_t ldx, ldw;
    int64_t ignore_index;
    int32_t dim;              /* 1 .. 32767                                    */
    int32_t dtype;            /* pvs_dtype of x, w and their gradients         */
    float scale;              /* a > 0, a normal float32                       */
    int32_t reserved;         /* 0                                             */
} pvs_xent_args;

/* Bytes of scratch for pvs_xent_forward (backward = 0) or pvs_xent_backward
 * (1) of these arguments.  Forward: copies of rows that are not 16-bit and aligned
 * and of 1 GB of such items, and 8 bytes for each row and 256 items of a block of rows
 * (1 GB, or 1,024 rows). */
pvs_status pvs_xent_workspace(const pvs_xent_args* args, int32_t backward, size_t* bytes);

/* loss [rows] and stats [rows x 4], both float32, stats 16-byte aligned.  A
 * row's stats are for the backward pass: m and s with sum_j exp(l_tj) = s 2^m (m
 * the largest l_tj / ln 2), dloss_t / dl of the target, and the target's
 * l / ln 2. */
pvs_status pvs_xent_forward(const pvs_xent_args* args, float* loss, float* stats,
                            void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The gradients of sum_t grad_loss[t] loss_t: dx [rows x dim] (leading
 * dimension lddx) and dw [items x dim] (lddw), of the operands' type, each
 * rounded once from its float32 sum; either may be null.  The logits are
 * computed again, a piece of the items at a time, and G = dloss/dl of the
 * piece is kept in the workspace: in two bf16 parts for bf16, in two f16 parts
 * after a common scaling to the largest |grad_loss| for f16 (2^-15 of each entry is
 * lost, next to nothing of what rounding dx and dw loses), for float32 in three bf16
 * parts (up to 16 rows of dim <= 1024: in float32).  G takes 1 GB at most, or 1,024
 * items' where that is more. */
pvs_status pvs_xent_backward(const pvs_xent_args* args, const float* stats,
                             const float* grad_loss, void* dx, int64_t lddx, void* dw,
                             int64_t lddw, void* workspace, size_t workspace_bytes,
                             void* cuda_stream);

/* ---------------------------------------------------------------------------
 * Distillation: a row's target is a teacher's distribution over the items of its list (its
 * `top` best, say).  With l_tj as above, slots k of ids i_tk and teacher logits z_tk, and
 * c = teacher_scale:
 *     p_tk   = exp(c z_tk) / sum_k exp(c z_tk)
 *     loss_t = sum_k p_tk (ln p_tk - l_{t, i_tk} + ln(sum_j exp(l_tj)))
 * the divergence of the student's softmax over all items from the teacher's over the list;
 * dloss_t / dl_tj = softmax(l_t)_j - sum_{k: i_tk = j} p_tk.
 *   - a slot whose id is ignore_index, whose c z_tk is -inf, or whose item's bias is -inf (an
 *     item that was deleted after the list was made) is not in the list: the others share its part.
 *   - no slot in the list: loss 0 and no gradient, whatever the row holds.
 *   - any other id outside [0, items): the loss is NaN, and so are the gradients that the row
 *     reaches.
 *   - an id that a list has twice: its slots' shares add up.
 * Biases, overflows and types are as in the softmax cross entropy.
 * ------------------------------------------------------------------------ */
typedef struct pvs_distill_args {
    pvs_xent_args student;    /* targets are not used; ignore_index is that of ids   */
    const int64_t* ids;       /* [rows x top] without gaps                           */
    const void* logits;       /* [rows x top] without gaps                           */
    int32_t top;              /* 1 .. 1024                                           */
    int32_t teacher_dtype;    /* pvs_dtype of logits                                 */
    float teacher_scale;      /* c > 0, a normal float32                             */
    int32_t reserved;         /* 0                                                   */
} pvs_distill_args;

/* Bytes of scratch of the two calls, as pvs_xent_workspace; forward, 10 more for each slot and 2
 * for each row and 256 items of a block of rows. */
pvs_status pvs_distill_workspace(const pvs_distill_args* args, int32_t backward, size_t* bytes);

/* loss [rows], stats [rows x 4] (16-byte aligned) and hits [rows x top], all float32.  stats
 * and hits are for the backward pass: a row's m and s with sum_j exp(l_tj) = s 2^m, 0 and
 * -inf; and dloss_t / dl of each slot's item, 2 for a slot that is not in the list. */
pvs_status pvs_distill_forward(const pvs_distill_args* args, float* loss, float* stats, float* hits,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The gradients of sum_t grad_loss[t] loss_t, as pvs_xent_backward's; logits and teacher_scale
 * are not used (teacher_scale is checked). */
pvs_status pvs_distill_backward(const pvs_distill_args* args, const float* stats, const float* hits,
                                const float* grad_loss, void* dx, int64_t lddx, void* dw,
                                int64_t lddw, void* workspace, size_t workspace_bytes,
                                void* cuda_stream);

/* ---------------------------------------------------------------------------
 * Rows kept in 8 bits.  Row r of x [rows x cols] is kept as Sec. 2.3.1 keeps
 * a vector, its scale to within a last bit: s_r = RN(max|x| RN(1 / 127)) (1 for a
 * zero row, the smallest positive float32 where that underflows), z =
 * round_half_away(RN(x / s_r)) clipped to [-127, 127]; it stands for s_r z.  A row with a NaN or an infinity gets the
 * scale NaN and codes 0: all that it stands for is NaN.
 * 0 <= rows <= 2^31 - 2^16, 1 <= cols <= 32767.
 * ------------------------------------------------------------------------ */

/* codes int8 [rows x cols] and scales float32 [rows], and, where act is not
 * PVS_ACT_NONE, y = act(x) in x's type (else y is not used, and may be null). */
pvs_status pvs_ckpt_store(const void* x, int64_t ldx, int64_t rows, int32_t cols, int32_t dtype,
                          int32_t act, int8_t* codes, int64_t ldcodes, float* scales, void* y,
                          int64_t ldy, void* cuda_stream);

/* out = s z, in out's type. */
pvs_status pvs_ckpt_load(const int8_t* codes, int64_t ldcodes, const float* scales, int64_t rows,
                         int32_t cols, void* out, int64_t ldout, int32_t dtype,
                         void* cuda_stream);

/* dx = dy act'(s z): the gradient before an activation whose input was kept.
 * dy and dx share a type. */
pvs_status pvs_ckpt_act_backward(const void* dy, int64_t lddy, const int8_t* codes,
                                 int64_t ldcodes, const float* scales, int64_t rows, int32_t cols,
                                 int32_t dtype, int32_t act, void* dx, int64_t lddx,
                                 void* cuda_stream);

/* Weight gradient of a linear layer y = x W^T whose input was kept:
 *     dw[n, k] = sum_r dy[r, n] s_r z[r, k],  dw [out_cols x cols] in dy's type.
 * bf16: dy is an exact operand, and s_r z the other in two bf16 parts (2^-15 of a term
 * is lost).  Else the codes are exact operands, and dy s_r is in two bf16 parts for f16,
 * three for float32.  Operands are laid out in the workspace a piece of the rows at a
 * time: 1 GB of them, and 2 GB of float32 sums, or 4,096 rows and one dw in float32
 * where that is more. */
pvs_status pvs_ckpt_grad_workspace(int64_t rows, int32_t out_cols, int32_t cols, int32_t dtype,
                                   size_t* bytes);
pvs_status pvs_ckpt_grad_weight(const void* dy, int64_t lddy, const int8_t* codes,
                                int64_t ldcodes, const float* scales, int64_t rows,
                                int32_t out_cols, int32_t cols, int32_t dtype, void* dw,
                                int64_t lddw, void* workspace, size_t workspace_bytes,
                                void* cuda_stream);

/* ---------------------------------------------------------------------------
 * 4-bit weights.  A row of `cols` weights is padded to kp, a multiple of 128,
 * and cut into groups of 32, 64 or 128: s = RN_bf16(RN(max|w| RN(1 / 7))) (1 for a
 * group of zeros, the smallest positive bf16 where that underflows; NaN, with
 * codes 0, where the group holds a NaN or an infinity), q =
 * round_half_away(RN(w / s)) clipped to [-7, 7], kept as q + 8; padding is 8.
 * codes: uint8 [rows x kp / 2] without gaps, 16-byte aligned.  A block of 128
 * weights is 64 bytes, laid out for the tensor cores' operand: byte
 * 16 t + 4 i + b (0 <= t, i, b < 4) holds weight 32 i + 8 t + 2 b in its low
 * half and the next one in its high half.
 * scales: bf16 [rows x kp / group] without gaps, 8-byte aligned.
 * 0 <= rows <= 2^31 - 2^16, 1 <= cols <= 32767.
 * ------------------------------------------------------------------------ */
pvs_status pvs_wq_pack(const void* w, int64_t ldw, int64_t rows, int32_t cols, int32_t dtype,
                       int32_t group, uint8_t* codes, void* scales, void* cuda_stream);

/* out [rows x cols] = s q, in out's type. */
pvs_status pvs_wq_unpack(const uint8_t* codes, const void* scales, int64_t rows, int32_t cols,
                         int32_t group, void* out, int64_t ldout, int32_t dtype,
                         void* cuda_stream);

/* y [batch x rows] = x [batch x cols] times the transposed weights, in x's
 * type, 0 <= batch <= 64 (written for single queries and a few: the weights
 * are read once for 32 bf16, 16 f16 or 10 float32 rows).  x enters as one, two
 * or three bf16 parts (exact), codes are exact, sums float32. */
pvs_status pvs_wq_matvec(const void* x, int64_t ldx, int32_t batch, const uint8_t* codes,
                         const void* scales, int64_t rows, int32_t cols, int32_t group,
                         int32_t dtype, void* y, int64_t ldy, void* cuda_stream);

/* ---------------------------------------------------------------------------
 * Microscaled 4-bit rows, for products of any number of rows on the tensor cores.  An element
 * is kept as one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign (e2m1), in units of a scale that
 * `group` neighbours of a row share; columns are padded with zeros to kp, a multiple of 128:
 *   group 32   scale 2^(floor(log2 max|x|) - 2), clipped to 2^-127 from below (zero groups too),
 *              as its exponent with bias 127; 255 (NaN) for a group that holds a NaN or an
 *              infinity, with codes 0.
 *   group 16   each row has a power of two r = 2^(floor(log2 max|x_row|) - 10), 2^-126 at least (1
 *              for a zero row; NaN, with scales and codes 0, for a row that holds a NaN or an
 *              infinity), and a group the scale s = RN_e4m3(RN(max|x| RN(1 / 6)) / r), in units of r
 *              (of float32's 2^23 significands one, which lies beside a border of e4m3, gets the scale
 *              on its other side than max|x| / 6 would; none of 16 bits does).
 * An element is the nearest of those values to x / scale, of two the one with an even code,
 * 6 beyond 6; 0 where the scale is 0.
 * codes: uint8 [rows x kp / 2] without gaps, 16-byte aligned; the lower half of a byte comes first,
 * bit 3 of a half is the sign.
 * scales: uint8, 16-byte aligned, as the tensor cores take them: blocks of 512 bytes
 * [ceil(rows / 128)][kp / (4 group)], each the four scales of 4 group columns of 128 rows, those
 * of row 32 i + j from byte 16 j + 4 i; zeros for rows that are not there.
 * row_scales: float32 [rows] for group 16; not used for 32.
 * 0 <= rows <= 2^31 - 2^16, 1 <= cols <= 32767.
 * ------------------------------------------------------------------------ */
pvs_status pvs_mx_pack(const void* x, int64_t ldx, int64_t rows, int32_t cols, int32_t dtype,
                       int32_t group, uint8_t* codes, uint8_t* scales, float* row_scales,
                       void* cuda_stream);

/* out [rows x cols] = what codes stand for, in out's type. */
pvs_status pvs_mx_unpack(const uint8_t* codes, const uint8_t* scales, const float* row_scales,
                         int64_t rows, int32_t cols, int32_t group, void* out, int64_t ldout,
                         int32_t dtype, void* cuda_stream);

/* y [batch x rows] in x's type = x [batch x cols], put into the weights' format as pvs_mx_pack
 * does, times the transposed weights [rows x cols]: products of codes are exact, sums float32,
 * y rounded once from them (group 16: from the sum times both row scales, right wherever that is a
 * float32; group 32: its scales are in the sums, which are infinite or NaN where one leaves
 * float32's range on its way).  Scratch: x in that format, and float32 sums of a few units of y
 * where k is split. */
pvs_status pvs_mx_workspace(int64_t batch, int64_t rows, int32_t cols, int32_t group, size_t* bytes);
pvs_status pvs_mx_matmul(const void* x, int64_t ldx, int64_t batch, const uint8_t* codes,
                         const uint8_t* scales, const float* row_scales, int64_t rows, int32_t cols,
                         int32_t group, int32_t dtype, void* y, int64_t ldy, void* workspace,
                         size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------
 * Rows of a table by their ids, for the tokens or items that a head is fed with:
 *     y_t = scale w[ids[t]]                          [rows x dim], in w's type
 * and the table's gradient
 *     dw_v = scale sum_{t: ids[t] = v} dy_t          [items x dim], in dy's type
 * for a row of the table that no id names, zeros.  Each output is rounded once; a
 * sum is float32, of whole stretches of the order of t, and the same in every call.
 *   - ids[t] == ignore_index: a row of zeros, and no gradient, whatever dy_t holds.
 *   - any other id outside [0, items): a row of NaN, and no gradient.
 * 0 <= rows <= 2^31 - 2^16, 1 <= items <= 2^31 - 2^16, 1 <= dim <= 32767; scale finite.
 * Outputs may not overlap inputs.
 * ------------------------------------------------------------------------ */
pvs_status pvs_embed_forward(const void* w, int64_t ldw, int64_t items, int32_t dim, int32_t dtype,
                             const int64_t* ids, int64_t rows, float scale, int64_t ignore_index,
                             void* y, int64_t ldy, void* cuda_stream);

/* Scratch of the gradient: 16 bytes an id at most, 4 KB for every 1,024 of more than 8,192
 * ids, and two float32 rows and 4 bytes for every 32 ids (for every 8 of few). */
pvs_status pvs_embed_workspace(int64_t rows, int64_t items, int32_t dim, size_t* bytes);
pvs_status pvs_embed_backward(const void* dy, int64_t lddy, const int64_t* ids, int64_t rows,
                              int64_t items, int32_t dim, int32_t dtype, float scale,
                              int64_t ignore_index, void* dw, int64_t lddw, void* workspace,
                              size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* PVS_HEAD_H_ */
