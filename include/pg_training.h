/*
 * pg_training.h - the local half of decentralized SGD for all simulated workers at once.
 *
 * Algorithm 1 of the paper needs a gradient G_i of every worker before pg_round_sgd can take it.
 * These calls compute the forward and backward pass of a residual block for N workers in one
 * launch each: every worker has its own tokens and its own weights (the leading, "batch" axis
 * below), as its parameter stack has its own matrices.  Activations of all workers share one
 * GPU, so what a backward pass needs is kept in 8 bits.
 *
 * Conventions (those of powergossip.h, and)
 *   - The calls need no context.  They allocate nothing; a call that needs scratch has a
 *     ..._workspace_bytes() beside it and takes workspace and size (16-byte aligned device memory,
 *     free again when the enqueued work has run).
 *   - All work is enqueued on `stream`; nothing waits.  Device-side time-outs are reported by
 *     pg_training_status.
 *   - Arguments come in one struct per call.  All pointers in it are device pointers of the
 *     current device.  A matrix is row-major: `ld` elements from row to row, `stride` elements from
 *     worker to worker; an operand all workers share has stride 0.  Outputs of different workers
 *     must not overlap.  An optional matrix or vector is left out by a null pointer.
 *   - 16-bit elements are bf16 or fp16 (`dtype`), the same for all 16-bit matrices of a call;
 *     biases, gains, statistics and parameter gradients are fp32, as the parameter stack is.
 *   - Sums, statistics and products are held in fp32 and rounded once, where a result is stored.  (The
 *     tensor cores cut sums off instead of rounding them: of a weight gradient's size that is under
 *     1e-6, as for an fp32 product, and up to 5e-6 where all products have the same sign.)
 *   - tokens = 0 and batch = 0 are valid: outputs per token are empty, sums over tokens are zero.
 *   - A NaN or an infinity in an input reaches the outputs that depend on it, and no others; in the
 *     8-bit form it takes its block of 32 values with it (below).
 *   - Rows may start on any element.  Where they start on 16-byte boundaries the kernels take their
 *     fastest path; elsewhere 16-byte pieces of memory that hold at least one element of a row are
 *     read whole, and what else is in them is not used.  Outputs are written to their own elements only.
 *   - PG_ERR_INVALID: sizes out of range, a required pointer missing, misaligned, on the host or
 *     on another device, ld below the row length, rows of an output that overlap from worker to worker.
 *     Nothing is launched then.  That different operands do not overlap (but for what may be in place)
 *     is up to the caller.
 */
#ifndef PG_TRAINING_H_
#define PG_TRAINING_H_

#include "powergossip.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { PG_BF16 = 0, PG_F16 = 1 };

/* Activations a(z), with s(v) = 1 / (1 + exp(-v)):  NONE z,  RELU max(z, 0),
 * GELU z s(2 sqrt(2/pi) (z + 0.044715 z^3)) (the tanh form),  SILU z s(z).
 * The slope of RELU at 0 is 0. */
enum { PG_ACT_NONE = 0, PG_ACT_RELU = 1, PG_ACT_GELU = 2, PG_ACT_SILU = 3 };

/* A batch of row-major matrices; element type as stated where it is used. */
typedef struct pg_matrix {
    void *data;
    int64_t ld;      /* elements from row to row      */
    int64_t stride;  /* elements from worker to worker */
} pg_matrix;

/*
 * A batch of matrices in 8 bits.  32 neighbouring values of a row form a block with one power of
 * two:  value = q * 2^(scale - 127),  q in -127..127.  The writer takes
 *     scale - 127 = max(floor(log2(max |v| in the block)) - 6, least)
 *     q           = v * 2^-(scale - 127) rounded to nearest, ties to even, clamped to +-127
 * with least = -126 for bf16 and -24 for fp16 (whose own step that is), so that every value the
 * form stands for is exact in 16 bits, where it is in the type's range (a result that goes to 8 bits
 * from fp32 may be beyond fp16's, and reads back as an infinity).  A block that holds a NaN or an infinity gets scale 255
 * and reads back as NaN.  A row has ceil(cols / 32) scales; the last block may be short.
 * values: 16-byte aligned, ld and stride multiples of 16 (bytes from row to row, worker to worker).
 */
typedef struct pg_matrix8 {
    int8_t *values;
    uint8_t *scales;
    int64_t ld, stride;              /* of values, in bytes */
    int64_t scale_ld, scale_stride;  /* of scales, in bytes */
} pg_matrix8;

/* ------------------------------------------------------------------ norm */
/*
 * Residual addition and root-mean-square norm, row by row (tokens x cols per worker):
 *     s = x + residual;  rstd = (mean(s^2) + eps)^(-1/2);  y = s * rstd * gain
 * h gets s rounded to 16 bits (the next residual stream; may be x or residual in place), y the
 * result.  At most 16384 columns (PG_ERR_TOO_LARGE).  With y8, the 8-bit form of the result is written too and y holds the values it stands
 * for: the layer behind the norm then sees in its forward pass what its weight gradient will read.
 * h8 gets the 8-bit form of h as it is stored, in 16 bits (what pg_checkpoint_write makes of it), the checkpoint
 * that pg_add_rms_norm_grad reads.
 */
typedef struct pg_norm_args {
    int32_t dtype, batch, tokens, cols;
    float eps;                 /* finite, >= 0 */
    pg_matrix x;               /* 16-bit */
    pg_matrix residual;        /* 16-bit, optional */
    const float *gain;         /* cols per worker, optional (1) */
    int64_t gain_stride;
    pg_matrix h;               /* out, 16-bit, optional */
    pg_matrix y;               /* out, 16-bit, optional */
    pg_matrix8 y8;             /* out, optional */
    pg_matrix8 h8;             /* out, optional */
    float *rstd;               /* out, batch x tokens, optional */
} pg_norm_args;
PG_API int pg_add_rms_norm(const pg_norm_args *args, void *stream);

/*
 * Its gradient.  With u = h rstd and a = dy gain:
 *     dx = rstd (a - u mean(a u)) + dh          (also the gradient of `residual`)
 *     dgain = sum over tokens of dy u           (added to what is there with accumulate)
 * h is the stored sum, in 16 bits or as its 8-bit checkpoint (exactly one of h and h8).  At most
 * 16384 columns: PG_ERR_TOO_LARGE from the call and from its workspace query.
 */
typedef struct pg_norm_grad_args {
    int32_t dtype, batch, tokens, cols;
    int32_t accumulate;        /* 0: dgain is overwritten, 1: added to */
    pg_matrix dy;              /* 16-bit */
    pg_matrix h;               /* 16-bit, or */
    pg_matrix8 h8;
    const float *rstd;         /* batch x tokens */
    const float *gain;         /* optional (1) */
    int64_t gain_stride;
    pg_matrix dh;              /* 16-bit, optional: gradient that reaches h on the residual path */
    pg_matrix dx;              /* out, 16-bit; may be dy or dh in place */
    float *dgain;              /* out, cols per worker, optional */
    int64_t dgain_stride;
} pg_norm_grad_args;
PG_API int pg_add_rms_norm_grad_workspace_bytes(const pg_norm_grad_args *args, size_t *bytes_out);
PG_API int pg_add_rms_norm_grad(const pg_norm_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Residual addition and layer norm:
 *     s = x + residual;  mean = mean(s);  rstd = (mean((s - mean)^2) + eps)^(-1/2);  y = (s - mean) rstd gain + bias
 * Otherwise as pg_add_rms_norm.  With eps = 0 a row of equal values has no result.
 */
typedef struct pg_layer_norm_args {
    int32_t dtype, batch, tokens, cols;
    float eps;                 /* finite, >= 0 */
    pg_matrix x;               /* 16-bit */
    pg_matrix residual;        /* 16-bit, optional */
    const float *gain;         /* cols per worker, optional (1) */
    int64_t gain_stride;
    const float *bias;         /* cols per worker, optional (0) */
    int64_t bias_stride;
    pg_matrix h;               /* out, 16-bit, optional */
    pg_matrix y;               /* out, 16-bit, optional */
    pg_matrix8 y8;             /* out, optional */
    pg_matrix8 h8;             /* out, optional */
    float *mean;               /* out, batch x tokens, optional */
    float *rstd;               /* out, batch x tokens, optional */
} pg_layer_norm_args;
PG_API int pg_add_layer_norm(const pg_layer_norm_args *args, void *stream);

/*
 * Its gradient.  With u = (h - mean) rstd and a = dy gain:
 *     dx = rstd (a - mean(a) - u mean(a u)) + dh    (also the gradient of `residual`)
 *     dgain = sum over tokens of dy u,  dbias = sum over tokens of dy      (added to with accumulate)
 * Otherwise as pg_add_rms_norm_grad.
 */
typedef struct pg_layer_norm_grad_args {
    int32_t dtype, batch, tokens, cols;
    int32_t accumulate;        /* 0: dgain and dbias are overwritten, 1: added to */
    pg_matrix dy;              /* 16-bit */
    pg_matrix h;               /* 16-bit, or */
    pg_matrix8 h8;
    const float *mean;         /* batch x tokens */
    const float *rstd;         /* batch x tokens */
    const float *gain;         /* optional (1) */
    int64_t gain_stride;
    pg_matrix dh;              /* 16-bit, optional: gradient that reaches h on the residual path */
    pg_matrix dx;              /* out, 16-bit; may be dy or dh in place */
    float *dgain;              /* out, cols per worker, optional */
    int64_t dgain_stride;
    float *dbias;              /* out, cols per worker, optional */
    int64_t dbias_stride;
} pg_layer_norm_grad_args;
PG_API int pg_add_layer_norm_grad_workspace_bytes(const pg_layer_norm_grad_args *args, size_t *bytes_out);
PG_API int pg_add_layer_norm_grad(const pg_layer_norm_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------- linear */
/*
 * z = x W^T + bias;  y = a(z) + residual, for every worker: x tokens x in, W out x in (a layer of
 * the stack: rows = out, cols = in), y tokens x out.  z8, if given, gets the 8-bit form of z for
 * pg_activation_grad (16-bit dtype decides its smallest step).
 * Unless there are very few tokens, rows of x or W that are not 16-byte aligned (ld or stride not a multiple of 8
 * elements, or such a pointer) are first copied to aligned rows in the workspace; otherwise none is
 * needed.  The same goes for the operands of the two gradients below.
 */
typedef struct pg_linear_args {
    int32_t dtype, activation, batch, tokens, in_features, out_features;
    pg_matrix x;               /* 16-bit, tokens x in */
    pg_matrix weight;          /* 16-bit, out x in */
    const float *bias;         /* out per worker, optional */
    int64_t bias_stride;
    pg_matrix residual;        /* 16-bit, tokens x out, optional */
    pg_matrix y;               /* out, 16-bit, tokens x out; may be residual in place */
    pg_matrix8 z8;             /* out, optional */
} pg_linear_args;
PG_API int pg_linear_workspace_bytes(const pg_linear_args *args, size_t *bytes_out);
PG_API int pg_linear(const pg_linear_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* dx = dz W + residual: the gradient of x, with what reaches x on another path added. */
typedef struct pg_input_grad_args {
    int32_t dtype, batch, tokens, in_features, out_features;
    pg_matrix dz;              /* 16-bit, tokens x out */
    pg_matrix weight;          /* 16-bit, out x in */
    pg_matrix residual;        /* 16-bit, tokens x in, optional */
    pg_matrix dx;              /* out, 16-bit, tokens x in; may be residual in place */
} pg_input_grad_args;
PG_API int pg_linear_input_grad_workspace_bytes(const pg_input_grad_args *args, size_t *bytes_out);
PG_API int pg_linear_input_grad(const pg_input_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* dW = dz^T x in fp32, straight into a gradient buffer's layout (pg_stack_offset): overwritten, or
 * added to with accumulate.  x is a 16-bit matrix or an 8-bit checkpoint (exactly one of x, x8) whose values
 * are in the 16-bit type's range, as those written from that type are. */
typedef struct pg_weight_grad_args {
    int32_t dtype, batch, tokens, in_features, out_features;
    int32_t accumulate;
    pg_matrix dz;              /* 16-bit, tokens x out */
    pg_matrix x;               /* 16-bit, tokens x in, or */
    pg_matrix8 x8;
    pg_matrix dweight;         /* out, fp32, out x in */
} pg_weight_grad_args;
PG_API int pg_linear_weight_grad_workspace_bytes(const pg_weight_grad_args *args, size_t *bytes_out);
PG_API int pg_linear_weight_grad(const pg_weight_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/*
 * dz = dy a'(z) and dbias = sum over tokens of dz (before dz is rounded), z read from its 8-bit
 * checkpoint; z8 may be left out for PG_ACT_NONE.  dbias is added to with accumulate.
 */
typedef struct pg_activation_grad_args {
    int32_t dtype, activation, batch, tokens, cols;
    int32_t accumulate;
    pg_matrix dy;              /* 16-bit */
    pg_matrix8 z8;
    pg_matrix dz;              /* out, 16-bit, optional; may be dy in place */
    float *dbias;              /* out, cols per worker, optional */
    int64_t dbias_stride;
} pg_activation_grad_args;
PG_API int pg_activation_grad(const pg_activation_grad_args *args, void *stream);

/* ---------------------------------------------------------- sequences */
/*
 * Operators along tokens.  A worker's tokens are `sequences` sequences of `length` tokens, one after another: row
 * s length + t of a matrix is token t of sequence s.  With `lengths` (int32, batch x sequences) only the first lengths[s] tokens of a
 * sequence are there (0 to length; other values count as the nearer of these): what the inputs hold behind them is not used, and
 * the outputs' rows are zero there, as are what they would add to a sum.  A state, if given, is what came before a sequence's first
 * token (zeros, if not); state_out gets what comes before the next one, and may be `state` in place.  Gradients stop at states,
 * as in truncated back-propagation.  At most 524288 channels (PG_ERR_TOO_LARGE).
 */

/*
 * Causal convolution of every channel with `width` taps of its own, 2 to 4:
 *     z_t = bias + sum over j of weight[j] x_{t - width + 1 + j},   y_t = a(z_t)
 * activation is PG_ACT_NONE or PG_ACT_SILU.  The state is the last width - 1 inputs, the oldest first.
 */
typedef struct pg_conv_args {
    int32_t dtype, activation, batch, sequences, length, channels, width;
    pg_matrix x;               /* 16-bit, tokens x channels */
    pg_matrix weight;          /* fp32, channels x width */
    const float *bias;         /* channels per worker, optional */
    int64_t bias_stride;
    const int32_t *lengths;    /* batch x sequences, optional */
    const void *state;         /* 16-bit, batch x sequences x (width - 1) x channels, optional */
    void *state_out;           /* out, the same, optional */
    pg_matrix y;               /* out, 16-bit, tokens x channels */
} pg_conv_args;
PG_API int pg_causal_conv(const pg_conv_args *args, void *stream);

/* Its gradient: dx, and with dz = dy a'(z) the sums over tokens dweight[j] of dz_t x_{t - width + 1 + j} and dbias of dz. */
typedef struct pg_conv_grad_args {
    int32_t dtype, activation, batch, sequences, length, channels, width;
    int32_t accumulate;        /* 0: dweight and dbias are overwritten, 1: added to */
    pg_matrix dy;              /* 16-bit, tokens x channels */
    pg_matrix x;
    pg_matrix weight;
    const float *bias;
    int64_t bias_stride;
    const int32_t *lengths;
    const void *state;
    pg_matrix dx;              /* out, 16-bit, tokens x channels */
    pg_matrix dweight;         /* out, fp32, channels x width, optional */
    float *dbias;              /* out, channels per worker, optional */
    int64_t dbias_stride;
} pg_conv_grad_args;
PG_API int pg_causal_conv_grad_workspace_bytes(const pg_conv_grad_args *args, size_t *bytes_out);
PG_API int pg_causal_conv_grad(const pg_conv_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Selective scan, for every channel and `states` states (at most 64, PG_ERR_TOO_LARGE):
 *     D_t = log(1 + exp(delta_t + delta_bias))
 *     h_t = exp(D_t a) h_{t-1} + D_t u_t b_t,   y_t = (sum over states of c_t h_t + skip u_t) s(z_t) z_t
 * with s as above; without z the last factors are left out.  u, delta, z and y have a column per channel, b and c one per state, a
 * is fp32, channels x states (a layer of the stack), and not positive where states are to decay; -inf forgets a state at every token.
 * States are fp32.
 * Where there are few sequences they are cut into chunks that run side by side, whose states the workspace joins.
 */
typedef struct pg_scan_args {
    int32_t dtype, batch, sequences, length, channels, states;
    pg_matrix u;               /* 16-bit, tokens x channels */
    pg_matrix delta;           /* 16-bit, tokens x channels */
    pg_matrix a;               /* fp32, channels x states */
    pg_matrix b;               /* 16-bit, tokens x states */
    pg_matrix c;               /* 16-bit, tokens x states */
    pg_matrix z;               /* 16-bit, tokens x channels, optional */
    const float *delta_bias;   /* channels per worker, optional (0) */
    int64_t delta_bias_stride;
    const float *skip;         /* channels per worker, optional (0) */
    int64_t skip_stride;
    const int32_t *lengths;    /* batch x sequences, optional */
    const float *state;        /* batch x sequences x channels x states, optional */
    float *state_out;          /* out, the same, optional */
    pg_matrix y;               /* out, 16-bit, tokens x channels */
} pg_scan_args;
PG_API int pg_selective_scan_workspace_bytes(const pg_scan_args *args, size_t *bytes_out);
PG_API int pg_selective_scan(const pg_scan_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* Its gradient, from the inputs alone (states are computed once more).  db and dc are sums over channels, da, dskip and ddelta_bias sums over
 * tokens. */
typedef struct pg_scan_grad_args {
    int32_t dtype, batch, sequences, length, channels, states;
    int32_t accumulate;        /* 0: da, dskip and ddelta_bias are overwritten, 1: added to */
    pg_matrix dy;              /* 16-bit, tokens x channels */
    pg_matrix u;
    pg_matrix delta;
    pg_matrix a;
    pg_matrix b;
    pg_matrix c;
    pg_matrix z;
    const float *delta_bias;
    int64_t delta_bias_stride;
    const float *skip;
    int64_t skip_stride;
    const int32_t *lengths;
    const float *state;
    pg_matrix du;              /* out, 16-bit, tokens x channels */
    pg_matrix ddelta;          /* out, 16-bit, tokens x channels: of delta, before the softplus */
    pg_matrix da;              /* out, fp32, channels x states */
    pg_matrix db;              /* out, 16-bit, tokens x states */
    pg_matrix dc;              /* out, 16-bit, tokens x states */
    pg_matrix dz;              /* out, 16-bit, tokens x channels; with z */
    float *dskip;              /* out, channels per worker, optional */
    int64_t dskip_stride;
    float *ddelta_bias;        /* out, channels per worker, optional */
    int64_t ddelta_bias_stride;
} pg_scan_grad_args;
PG_API int pg_selective_scan_grad_workspace_bytes(const pg_scan_grad_args *args, size_t *bytes_out);
PG_API int pg_selective_scan_grad(const pg_scan_grad_args *args, void *workspace, size_t workspace_bytes, void *stream);

/* -------------------------------------------------------------- loss */
/*
 * Loss of a row of logits x against a teacher's top logits, and against a label: with tau = temperature,
 *     p = softmax(teacher / tau) over the list's entries,  q = softmax(x / tau) over all classes
 *     loss = alpha tau^2 sum p (log p - log q)  +  (1 - alpha) (log sum exp(x) - x[label])
 * The first term is there with top > 0, the second with labels; a weight of 0 leaves a term out.  Rows whose label is no class
 * (negative, or too large) have no second term.  Entries whose id is no class do not count, nor do those whose logit is -inf;
 * a row without any other has no first term.  A row of no terms has a loss and a gradient of 0, whatever its logits are.  An id
 * may occur more than once: each entry counts.  A logit x of -inf has probability 0 (and an infinite loss, where p is not 0); a row
 * of nothing else, or with a NaN or +inf, gives NaN.
 * lse gets log sum exp(x) and log sum exp(x / tau) of every row; the first is 0 where the call has no second term, the second where it has no first.
 *
 * The gradient dloss (alpha tau (q - p) + (1 - alpha) (softmax(x) - [label])) goes to dlogits: by pg_distillation_loss
 * together with the loss, reading the logits once (to 100000 classes with lists to 100 entries; twice above), or by pg_distillation_loss_grad from lse,
 * which it reads (and whose step, 2^-24 of its size, is the error of the probabilities' logarithms then).  At most 1024 entries in a
 * list (PG_ERR_TOO_LARGE); the gradient's time goes with the square of their number from some 100 on.
 */
typedef struct pg_distillation_args {
    int32_t dtype, batch, tokens, classes, top;
    float temperature;         /* 1e-30 to 1e30 */
    float alpha;               /* 0 to 1 */
    pg_matrix logits;          /* 16-bit, tokens x classes */
    pg_matrix ids;             /* int32, tokens x top: classes */
    pg_matrix teacher;         /* 16-bit, tokens x top: their logits */
    const int32_t *labels;     /* batch x tokens, optional */
    const float *dloss;        /* batch x tokens, optional (1) */
    float *loss;               /* out, batch x tokens, optional; not of _grad */
    float *lse;                /* batch x tokens x 2: out, optional; read by _grad */
    pg_matrix dlogits;         /* out, 16-bit, tokens x classes, optional but of _grad; may be logits in place */
} pg_distillation_args;
PG_API int pg_distillation_loss(const pg_distillation_args *args, void *stream);
PG_API int pg_distillation_loss_grad(const pg_distillation_args *args, void *stream);

/* ------------------------------------------------------------ checkpoints */
/* tokens x cols per worker between 16 bits and the 8-bit form. */
typedef struct pg_checkpoint_args {
    int32_t dtype, batch, tokens, cols;
    pg_matrix x;               /* 16-bit: read by _write, written by _read */
    pg_matrix8 x8;
} pg_checkpoint_args;
PG_API int pg_checkpoint_write(const pg_checkpoint_args *args, void *stream);
PG_API int pg_checkpoint_read(const pg_checkpoint_args *args, void *stream);

/*
 * Wait for `stream` and report whether a bounded device-side wait of these kernels gave up on the
 * current device since the last call (PG_ERR_TIMEOUT), then clear the word.  PG_OK otherwise.  A wait
 * gives up after two seconds; the outputs of its call are not valid then, and nothing else says so: ask
 * before results are used, as after a training step.  There is one word per device, for all streams:
 * whoever asks first is told, and has to take every call since the last answer for the one.
 */
PG_API int pg_training_status(void *stream);

/*
 * Self-test of the bounded wait: a block waits, for a millisecond at most, on a barrier that nothing
 * arrives on.  Waits for `stream` and returns PG_ERR_TIMEOUT when that was reported (the expected
 * outcome), PG_OK if not.  Clears the word, as pg_training_status does.
 */
PG_API int pg_selftest_training_timeout(void *stream);

/*
 * Self-test of the bounds-checked build, whose training kernels look every address up in the operands of
 * their call (accesses outside are skipped, and pg_training_status returns PG_ERR_BOUNDS; one call at
 * a time on a device): a kernel asks the check about the word behind an operand, without touching it.
 * Waits for `stream` and returns PG_ERR_BOUNDS from a library built with -DPG_BOUNDS_CHECK, PG_OK from
 * the regular one.  Clears the word.
 */
PG_API int pg_selftest_training_bounds(void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PG_TRAINING_H_ */
