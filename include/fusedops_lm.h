/*
 * fusedops_lm.h - operators of a language model's step that lie between the block norms of fusedops_train.h (same library,
 * same conventions, types and status codes):
 *   fused_head_norm / fused_head_norm_grad   norms of the heads' queries and keys and their rotation by position
 *   fused_scan / fused_scan_grad             a gated linear recurrence over the tokens
 *   fused_distill / _grad / _step            the distillation loss from a teacher's top logits, its gradient, both at once
 *
 * Arithmetic, statistics, states and sums are in 32 bits (in 64 where a type is float64); a result in fewer bits is rounded
 * once, to nearest, when it is stored.  Results are deterministic: the order of every sum is fixed by the sizes, the
 * alignments and the GPU.  Strides are in elements and not negative.
 */
#ifndef FUSEDOPS_LM_H
#define FUSEDOPS_LM_H

#include "fusedops_train.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FO_I32 = 16, FO_I64 = 17 };     /* integer types, beside FO_F64 .. FO_F16 */

/* ------------------------------------------------- head norms with rotation
 * For every vector x of `dim` values, of each head of each token, in one pass over up to two tensors (queries and keys):
 *     u = (x - mu) * r (.) weight + bias            as in fused_block_norm; kind FO_NORM_NONE: u = x
 *     y = u with its first 2 * pairs values turned, the rest as it is:
 *         (y_a, y_b) = (u_a cos - u_b sin,  u_b cos + u_a sin)   for every pair j = (a, b):
 *         FO_PAIR_HALVES: a = j, b = pairs + j;    FO_PAIR_NEIGHBOURS: a = 2 j, b = 2 j + 1
 *     cos = cos_table[position * ld_cos + j], sin alike, the position being the token's on the pair's axis: pairs are
 *     divided into `axes` sections, one behind the other, of section[k] pairs with the token's k-th position.
 * A position outside the table (negative, or >= rows) makes what it turns NaN.
 * Norm and weights are each tensor's own and shared by its heads.  Element (b, t, h, i) of a tensor is at
 * p[b * batch + t * token + h * head + i] (i: neighbours).  `y` may be `x` itself with the same strides.
 * vec_type (weights, biases): `type`, or FO_F32 with a 16-bit type.  Tables: float (double where type is FO_F64).
 * positions: int32 or int64, at positions[k * axis + b * batch + t * token], any strides (0 among them).
 * dim <= FO_HEAD_MAX_DIM and batch * tokens * heads < 2^31, else FO_ERR_UNSUPPORTED.  A decoding step is the call with
 * tokens = 1.  Any address of an element and any stride works; fast are vectors that begin at 8- or 16-byte boundaries and whose
 * rotated part (FO_PAIR_HALVES: each half of it) is a whole number of these.
 */
#define FO_HEAD_MAX_DIM 512
#define FO_MAX_AXES 4
enum { FO_PAIR_HALVES = 0, FO_PAIR_NEIGHBOURS = 1 };

typedef struct fo_strides {
    int64_t batch, token, head;
} fo_strides;

typedef struct fo_rotation {
    int32_t pairs;                       /* 0: no rotation, nothing else is looked at */
    int32_t pairing, axes, position_type;
    int32_t section[FO_MAX_AXES];        /* their sum is `pairs` */
    int64_t rows, ld_cos, ld_sin;
    const void *cos_table, *sin_table;
    const void *positions;
    int64_t position_axis, position_batch, position_token;
} fo_rotation;

typedef struct fo_heads {
    int64_t heads;
    const void *x;
    void *y;
    fo_strides x_at, y_at;
    fo_norm norm;
} fo_heads;

typedef struct fo_head_norm {
    int64_t batch, tokens;
    int32_t dim, type, vec_type, count;  /* count: tensors, 1 or 2 */
    fo_heads t[2];
    fo_rotation rotation;
} fo_head_norm;

int fused_head_norm(const fo_head_norm *a, void *stream);

/* The gradient from dy: with g = dy turned back, n = (x - mu) r,  a = g (.) weight
 *     dx = r (a - n mean(a n) - [layer: mean(a)])      (kind FO_NORM_NONE: g, and x may be NULL)
 *     dweight = sum g n,   dbias = sum g               over all tokens and heads; float (double for FO_F64), or NULL
 * Statistics are computed again from x.  dx may be dy or x itself with the same strides.
 */
typedef struct fo_heads_grad {
    int64_t heads;
    const void *dy, *x;
    void *dx;
    fo_strides dy_at, x_at, dx_at;
    fo_norm norm;
    void *dweight, *dbias;
} fo_heads_grad;

typedef struct fo_head_norm_grad {
    int64_t batch, tokens;
    int32_t dim, type, vec_type, count;
    fo_heads_grad t[2];
    fo_rotation rotation;
} fo_head_norm_grad;

int fused_head_norm_grad(const fo_head_norm_grad *a, void *ws, size_t ws_bytes, void *stream);
/* Bytes of scratch (0 on an invalid dim or type). */
size_t fused_head_norm_grad_workspace_bytes(int dim, int type);

/* ------------------------------------------------- gated linear recurrence
 * For every sequence b and channel c, over its tokens t:
 *     h_t = a_t h_{t-1} + m(a_t) x_t,      h_{-1} = state (NULL: zero)
 *     a = gate (FO_DECAY_VALUE), sigmoid(gate) (FO_DECAY_SIGMOID), exp(gate) (FO_DECAY_EXP)
 *     m = 1 (FO_MIX_ONE), 1 - a (FO_MIX_REST), sqrt(1 - a^2) (FO_MIX_ROOT; NaN where |a| > 1)
 * reset[b * reset_batch + t * reset_token] != 0 (bytes; NULL: nowhere): nothing of h_{t-1} enters h_t, whatever it holds.
 * lengths[b] (int32 or int64; NULL: `tokens`), taken into 0 .. tokens: behind a sequence's end x and gate are not looked at,
 * and h is zero there.  last (NULL, or batch x channels) = h at the end: of the last token, or the state without tokens;
 * `last` may be `state`.  1 - a is computed without the cancellation; 16-bit x goes through the hardware's
 * exponential, reciprocal and root, whatever the gate's type: the smaller of a sigmoid and 1 - a is off by some (10 + |gate|) 2^-23 of itself,
 * the larger is rounded to 32 bits.
 * Element (b, t, c) of x, gate, h is at p[b * batch + t * token + c].  state and last: float (double for FO_F64), contiguous.
 * Products of the decays over parts of the sequence are formed in 32 bits (64 for FO_F64): where they overflow, which takes decays above 1, or
 * where a state is infinite, h may be NaN.  It is NaN, too, should the CTAs that share a sequence lose each other.
 * gate_type: `type`, or FO_F32 with a 16-bit type.  channels <= FO_SCAN_MAX_CHANNELS, tokens <= FO_SCAN_MAX_TOKENS.  h may be
 * x itself.  A decoding step is the call with tokens = 1.
 */
#define FO_SCAN_MAX_CHANNELS (1 << 28)
#define FO_SCAN_MAX_TOKENS (1 << 30)
enum { FO_DECAY_VALUE = 0, FO_DECAY_SIGMOID = 1, FO_DECAY_EXP = 2 };
enum { FO_MIX_ONE = 0, FO_MIX_REST = 1, FO_MIX_ROOT = 2 };

typedef struct fo_rows {
    int64_t batch, token;                /* strides */
} fo_rows;

typedef struct fo_scan {
    int64_t batch, tokens, channels;
    int32_t type, gate_type, decay, mix;
    const void *x, *gate, *state, *reset, *lengths;
    fo_rows x_at, gate_at, reset_at;
    int32_t lengths_type, reserved;
    void *h, *last;
    fo_rows h_at;
} fo_scan;

int fused_scan(const fo_scan *a, void *ws, size_t ws_bytes, void *stream);
/* Bytes of scratch for fused_scan and fused_scan_grad of so many tokens; 0: none is needed, and ws may be NULL. */
size_t fused_scan_workspace_bytes(int64_t tokens);

/* The gradient from dh and dlast (either may be NULL: zero) and the forward pass's inputs and h:
 *     l_t = dh_t + a_{t+1} l_{t+1}   (dlast where the sequence ends; nothing through a reset)
 *     dx = m l,   dgate = l (h_{t-1} + m'(a) x) a'(gate),   dstate = a_0 l_0 (dlast without tokens)
 * dx has `type`, dgate gate_type; both are zero behind a sequence's end.  dstate: float (double for FO_F64), or NULL.
 * x may be NULL with FO_MIX_ONE.  dx and dgate overlap none of the inputs.
 */
typedef struct fo_scan_grad {
    int64_t batch, tokens, channels;
    int32_t type, gate_type, decay, mix;
    const void *dh, *dlast, *x, *gate, *h, *state, *reset, *lengths;
    fo_rows dh_at, x_at, gate_at, h_at, reset_at;
    int32_t lengths_type, reserved;
    void *dx, *dgate, *dstate;
    fo_rows dx_at, dgate_at;
} fo_scan_grad;

int fused_scan_grad(const fo_scan_grad *a, void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------- distillation from a teacher's top logits
 * For every row z of `vocab` logits, with q = softmax(z / temperature) and the teacher's `top` entries (id_k, v_k):
 *     tail NULL:  p = softmax(v / temperature) over the entries;      loss = sum_k p_k (log p_k - log q_{id_k})
 *     tail given: p_k = exp(v_k / temperature - tail), the teacher's own shares (tail: the log-sum-exp of its whole row over
 *                 temperature), P = max(0, 1 - sum p) and Q = 1 - sum q_{id_k} all that is outside the entries;
 *                 loss as above + P log(P / Q); where Q is zero as a number of 64 bits (the entries are all the row, or the rest is
 *                 masked) a P of at most 1 / 32 is what the rounding of v and tail has left, and taken as zero; a larger one makes the
 *                 loss infinite
 * An entry with a negative id is none; one with an id >= vocab makes the row NaN.  Entries with the same id are one place of q
 * with several shares.  Without entries the first form's loss is zero; p_k = 0 adds nothing.
 * Gradient, times dloss of the row (float; NULL: 1):
 *     dz_j = (q_j S - p_j) / temperature at an entry's place (p_j: the sum of its shares),   S = sum p + P
 *     dz_j = q_j (S - P / Q) / temperature elsewhere
 * fused_distill writes loss and stats (either may be NULL), fused_distill_grad dz from stats and dloss, fused_distill_step loss
 * and dz in one pass over the logits.  The two with dloss do not look at a row whose dloss is zero: its dz, and the step's loss, are zero.
 * loss, stats, dloss, tail: float (double where type is FO_F64).  stats: 3 x rows, contiguous: the largest logit, the sum of
 * exp((z - largest) / temperature), and S - P / Q, below sum p where P is not zero; where P / Q is above
 * 2^60, minus the sum, and log(P / Q).
 * ids: int32 or int64; ids and values have rows of ld_ids, ld_values >= top.
 * values_type: `type`, or FO_F32 with a 16-bit type.  What concerns the entries is computed in 64 bits.
 * dz may be the logits themselves.  Any address of an element and any ld >= vocab works; fast are logits and dz whose rows lie at
 * the same offset from a 16-byte boundary.
 * 1e-300 <= temperature <= 1e300, top <= FO_DISTILL_MAX_TOP and vocab <= FO_DISTILL_MAX_VOCAB, else FO_ERR_UNSUPPORTED.
 */
#define FO_DISTILL_MAX_TOP 1024
#define FO_DISTILL_MAX_VOCAB (1 << 20)

typedef struct fo_distill {
    int64_t rows, vocab, top;
    int32_t type, values_type, ids_type, reserved;
    double temperature;
    const void *logits, *ids, *values, *tail, *dloss;
    int64_t ld_logits, ld_ids, ld_values;
    void *loss, *stats, *dz;             /* stats: written by fused_distill, read by fused_distill_grad */
    int64_t ld_dz;
} fo_distill;

int fused_distill(const fo_distill *a, void *stream);
int fused_distill_grad(const fo_distill *a, void *stream);
int fused_distill_step(const fo_distill *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FUSEDOPS_LM_H */
