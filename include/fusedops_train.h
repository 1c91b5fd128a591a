/*
 * fusedops_train.h - operators of a language model's training step that stand next to the
 * fused templates of fusedops.h (same library, same conventions):
 *   fused_block_norm / fused_block_norm_grad  a residual block's epilogue and the next block's norm, row by row
 *   fused_grad_norm / fused_grad_clip         the global norm of many tensors, and clipping by it
 *   fused_adamw                               AdamW over many tensors, scaled by a factor that stays on the device
 *
 * Conventions, as in fusedops.h: matrix data, vectors, `result`, `factor` and `ws` are DEVICE
 * pointers of the caller; the structs are HOST memory, copied at launch, free on return.  Calls
 * are asynchronous on `stream`, allocate nothing, never synchronise, and return FO_OK or a
 * negative fo_status; on an error nothing was launched.  Sums are deterministic: their order is
 * fixed by the sizes, the alignments and the GPU.  Workspaces are prepared once with fo_workspace_init().
 *
 * Element types: the templates' float64, and float32, bfloat16 and float16 as models use them.
 * Arithmetic, statistics and sums are in 32 bits (in 64 where a type is float64); a result in
 * fewer bits is rounded once, to nearest, when it is stored.
 */
#ifndef FUSEDOPS_TRAIN_H
#define FUSEDOPS_TRAIN_H

#include "fusedops.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FO_F64 = 0, FO_F32 = 1, FO_BF16 = 2, FO_F16 = 3 };

/* --------------------------------------------------------------- block norm
 * For every row i of rows x cols matrices, in one pass:
 *     z = norm(f_i; post)                      (post.kind == FO_NORM_NONE: z = f_i)
 *     u = scale * col_scale (.) act(gate) (.) z
 *     h = x_i + u                              (x NULL: h = u;  f NULL: h = x_i, nothing of the above)
 *     y = norm(h; pre)
 * with   norm(t) = (t - mu) * r (.) weight + bias,   r = 1 / sqrt(mean((t - mu)^2) + eps),
 * mu the row's mean for FO_NORM_LAYER and 0 for FO_NORM_RMS: the norm after a block, its gate, the
 * residual scale, the addition to the residual stream, and the norm before the next block.
 * y is computed from h before h is rounded.
 *
 * Types: x and h have `stream_type`; f, gate and y have `block_type`; weights, biases and
 * col_scale have `vec_type`.  Pairs (stream, block): both the same, or FO_F32 with FO_BF16 or
 * FO_F16.  vec_type: block_type, or FO_F32 with a 16-bit block_type.
 * Matrices are row-major with leading dimension ld >= cols (element (i, j) at p[i * ld + j]).
 * gate: FO_AT_CELL: rows x cols; FO_AT_ROW: one value per row at gate[i * ld_gate];
 * FO_AT_COL: one value per column, contiguous; NULL: no gate.  Vectors are contiguous.
 * h and y are NULL where they are not wanted; h may be x itself (same pointer and ld).
 * stats: NULL or 4 x rows values (float, or double where block_type is FO_F64), contiguous: mu and r
 * of the post norm, mu and r of the pre norm, zeros for a norm that is not there and for rows without columns.
 * The gradient needs them.
 * Any address of an element and any ld works (another address: FO_ERR_UNSUPPORTED).  Fast is a call of which
 * every row begins and ends on a piece: 16 bytes of the block's type, as many elements of the stream's (32 bytes
 * of FO_F32 beside a 16-bit block), with vectors at 16-byte boundaries; one matrix or vector that does not takes
 * the whole call the slower way.
 * cols <= FO_BLOCK_NORM_MAX_COLS, else FO_ERR_UNSUPPORTED.  A single token is the call with rows = 1.
 * A row that holds a NaN or an infinity affects that row alone.
 */
#define FO_BLOCK_NORM_MAX_COLS 32768
enum { FO_NORM_NONE = 0, FO_NORM_RMS = 1, FO_NORM_LAYER = 2 };
enum { FO_ACT_LINEAR = 0, FO_ACT_SIGMOID = 1, FO_ACT_SILU = 2, FO_ACT_TANH = 3 };

typedef struct fo_norm {
    int32_t kind;               /* FO_NORM_* */
    int32_t reserved;
    double eps;                 /* >= 0 */
    const void *weight;         /* cols values, or NULL for ones */
    const void *bias;           /* cols values, or NULL for zeros */
} fo_norm;

typedef struct fo_block_norm {
    int64_t rows, cols;
    int32_t stream_type, block_type, vec_type;
    int32_t gate_access, gate_act, reserved;
    const void *x, *f, *gate, *col_scale;
    int64_t ld_x, ld_f, ld_gate;
    double scale;
    fo_norm post, pre;
    void *h, *y, *stats;
    int64_t ld_h, ld_y;
} fo_block_norm;

int fused_block_norm(const fo_block_norm *a, void *stream);

/* ------------------------------------------------- gradient of the block norm
 * Given dh and dy, the gradients of h and y (either may be NULL: zero), and the forward pass's
 * inputs, h and stats, with n = (t - mu) * r the normalised row of the norm in question:
 *     t   = dh + r (a - n mean(a n) - [layer: mean(a)]),  a = dy (.) pre.weight,  n of h
 *     dx  = t;      dpre_weight = sum_i dy n;      dpre_bias = sum_i dy
 *     q   = scale * t;      dcol_scale = sum_i q act(gate) z;      q' = q col_scale
 *     dgate = q' z act'(gate), summed over what the gate is shared by
 *     d   = q' act(gate);   df = d through the post norm, as t above (post.kind none: d)
 *     dpost_weight = sum_i d n;   dpost_bias = sum_i d,   n of f
 * f NULL: only dx and the pre norm's gradients.  x itself is not needed; h only where a pre norm is.
 * Every output may be NULL.  dx has stream_type; df and dgate of a gate per element have block_type; the
 * summed gradients (dgate per row or column, dcol_scale, weights, biases) are float, or double
 * where block_type is FO_F64.  dx may be dh itself.  Types, layouts and limits as above.
 */
typedef struct fo_block_norm_grad {
    int64_t rows, cols;
    int32_t stream_type, block_type, vec_type;
    int32_t gate_access, gate_act, reserved;
    const void *dh, *dy, *h, *f, *gate, *col_scale, *stats;
    int64_t ld_dh, ld_dy, ld_h, ld_f, ld_gate;
    double scale;
    fo_norm post, pre;
    void *dx, *df, *dgate;
    int64_t ld_dx, ld_df, ld_dgate;     /* ld_dgate: gate per element only */
    void *dcol_scale, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
} fo_block_norm_grad;

int fused_block_norm_grad(const fo_block_norm_grad *a, void *ws, size_t ws_bytes, void *stream);
/* Bytes of scratch (0 on invalid sizes or types). */
size_t fused_block_norm_grad_workspace_bytes(int64_t rows, int64_t cols, int block_type);

/* ------------------------------------------- global gradient norm, and clipping
 * Over `count` tensors of n values each (any addresses of elements, any sizes, zero among them):
 *     norm   = sqrt(sum g^2)  (FO_NORM_L2)   or   max |g|  (FO_NORM_MAX), over all of them
 *     factor = min(1, max_norm / (norm + eps))
 *     out    = factor * g
 * result[0] = norm, result[1] = factor, of result_type FO_F32 or FO_F64, on the device.
 * fused_grad_norm writes `result` only (`out` is not looked at); fused_grad_clip also every `out`,
 * which may be `in` itself - a clip in place whose factor is 1 writes nothing.
 * The tensors of a call share in_type and out_type.  16-bit and 32-bit values are squared and
 * added in 32 bits for a few neighbouring values (at most 32) and in 64 bits over these; values whose
 * 32-bit sum would leave the normal range are added in 64 bits from the start, so gradients near either end
 * of the range have their norm too.  A NaN anywhere makes norm and factor NaN; an infinity makes the norm infinite
 * and, with a finite max_norm, the factor zero (out: zero, NaN where the infinity was).
 */
enum { FO_NORM_L2 = 0, FO_NORM_MAX = 1 };

typedef struct fo_tensor {
    const void *in;
    void *out;
    int64_t n;
} fo_tensor;

int fused_grad_norm(const fo_tensor *t, int count, int in_type, int norm_kind, double max_norm, double eps,
                    void *result, int result_type, void *ws, size_t ws_bytes, void *stream);
int fused_grad_clip(const fo_tensor *t, int count, int in_type, int out_type, int norm_kind, double max_norm,
                    double eps, void *result, int result_type, void *ws, size_t ws_bytes, void *stream);
size_t fused_grad_workspace_bytes(void);

/* -------------------------------------------------------------------- AdamW
 * For every tensor of the list, element by element (c = *factor, or 1 where factor is NULL):
 *     g' = c g;   m' = beta1 m + (1 - beta1) g';   v' = beta2 v + (1 - beta2) g'^2
 *     p' = p - lr (m' / (1 - beta1^step) / (sqrt(v' / (1 - beta2^step)) + eps) + decay p)
 * p, m and v are float (double where grad_type is FO_F64); `weights` (NULL, or of weight_type, a
 * 16-bit type) takes p' rounded.  Each output may be its input.  `factor` is result + 1 of a
 * gradient norm, of factor_type, so clipping needs no pass of its own over the gradients.
 * decay is each tensor's own.  step >= 1.
 */
typedef struct fo_adam_tensor {
    const void *p, *g, *m, *v;
    void *p_out, *m_out, *v_out, *weights;
    int64_t n;
    double decay;
} fo_adam_tensor;

int fused_adamw(const fo_adam_tensor *t, int count, int grad_type, int weight_type, double lr, double beta1,
                double beta2, double eps, int64_t step, const void *factor, int factor_type, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FUSEDOPS_TRAIN_H */
