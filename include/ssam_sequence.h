/* ssam_sequence.h -- filters and scans along time, channel by channel or with a matrix per head for a state, and the norm
 * around them: the parts of a state space layer of a language model, in the C ABI's manner (every convention of ssam.h holds
 * here too, except where a line below says otherwise).
 *
 * Data: rows are tokens, channels lie side by side.  A tensor of rows is described by ssam_rows: the address of row 0's
 * channel 0, and the elements from one row, and from one sequence, to the next; the channels of a row are contiguous.
 * Element types: SSAM_F32, SSAM_F16, SSAM_BF16 (dtype); arithmetic, states and sums are fp32, results are rounded once.
 * No alignment beyond the element's is asked for.  Parameters live in device memory (they are learned).
 *
 * Sequences are described by ssam_sequences, in one of three forms:
 *   - batch: d_begin = d_end = NULL; sequence s is the rows 0 .. rows-1 at  d + s * batch;
 *   - padded batch: d_begin = NULL, d_end = lengths; sequence s is the rows 0 .. d_end[s]-1 at  d + s * batch;
 *   - packed: sequence s is the rows d_begin[s] .. d_end[s]-1 of one tensor of `rows` rows (batch strides unused);
 *     d_begin is ascending and sequences do not overlap, so an array of S+1 offsets serves as both (d_end = d_begin + 1).
 * d_begin and d_end are device arrays that the kernels read: values are held to 0 .. rows there, a sequence may be empty,
 * and rows that belong to no sequence are neither read into a result nor written.  Sequences of the packed form that
 * overlap or descend give undefined values (no access outside the tensors).
 *
 * A workspace belongs to one call until that call's work has finished; two calls in flight, or two captured graphs that
 * may run at the same time, must not share one.  Results do not depend on what a workspace held.  All sums over rows
 * and channels are added in a fixed order, so results are the same from run to run.
 *
 * Infinities and NaN stay where the definitions have them: rows of no sequence, an absent skip, and what kernels hold beyond the
 * last row, state or channel add nothing, not even zero times an infinity.  (A single row's decay below 2^-126 counts as 0, which
 * times an infinite state is NaN.)
 *
 * Tensors may reach over 2^59 elements at most, from the first to behind the last (SSAM_ERR_DIM).
 *
 * An output may overlap neither an input nor another output (SSAM_ERR_ALIAS) except where a comment allows it; tensors
 * that are column ranges of one buffer, of whole sequences or with all sequences' rows in turn, do not overlap.
 */
#ifndef SSAM_SEQUENCE_H_
#define SSAM_SEQUENCE_H_

#include "ssam.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SSAM_MAX_TAPS 8        /* longest filter of ssam_conv1d                               */
#define SSAM_MAX_STATES 64     /* states per channel of ssam_scan_selective                    */
#define SSAM_MARK_ROWS 16      /* ssam_scan_selective: rows from one mark to the next          */
#define SSAM_DELTA_ROWS 64     /* ssam_scan_delta: rows that are taken together                */
#define SSAM_MAX_KEY 256       /* ssam_scan_delta: longest key                                 */

typedef struct {
    void *d;                   /* device; NULL: not there (where a tensor is optional)         */
    long long batch, row;      /* elements, >= 0                                               */
} ssam_rows;

typedef struct {
    int sequences;             /* >= 0; of a batch, sequences x rows <= 2^40                   */
    int rows;                  /* batch forms: rows of a sequence; packed: rows of the tensor  */
    const int *d_begin, *d_end;
} ssam_sequences;

/* Per-channel causal filter along time, with bias, an optional SiLU and carried rows:
 *     p_t = bias + sum_{j < taps} weight[c][j] * x_{t - taps + 1 + j},    y_t = silu ? p_t / (1 + exp(-p_t)) : p_t
 * x at t < 0 comes from d_state, [sequences][taps-1][channels] in dtype, oldest row first (zeros without one).  d_final
 * receives the last taps-1 rows of each sequence, old state included, in the same layout: the state of a call that goes
 * on; it may be d_state itself.  weight: [channels][taps], bias: [channels] or NULL, both param_dtype (dtype or
 * SSAM_F32), contiguous. */
typedef struct {
    int dtype, param_dtype, channels, taps, silu;
    ssam_sequences seq;
    ssam_rows in, out;
    const void *d_weight, *d_bias, *d_state;
    void *d_final;
} ssam_conv1d_args;
int ssam_conv1d(const ssam_conv1d_args *args, void *hip_stream);

/* Gradients of ssam_conv1d.  grad_out: gradient of its result; d_grad_final (may be NULL): of its d_final.  grad_in and
 * d_grad_state are in dtype, d_grad_weight and d_grad_bias in param_dtype; each may be absent (NULL).  d_grad_state is
 * the gradient of d_state, or of the zeros that stand for it.  d_work: ssam_conv1d_backward_workspace_bytes(args)
 * bytes (0 where neither parameter's gradient is asked for), 16-byte aligned. */
typedef struct {
    int dtype, param_dtype, channels, taps, silu;
    ssam_sequences seq;
    ssam_rows in, grad_out, grad_in;
    const void *d_weight, *d_bias, *d_state, *d_grad_final;
    void *d_grad_weight, *d_grad_bias, *d_grad_state;
    void *d_work;
    size_t work_bytes;
} ssam_conv1d_backward_args;
int ssam_conv1d_backward(const ssam_conv1d_backward_args *args, void *hip_stream);
size_t ssam_conv1d_backward_workspace_bytes(const ssam_conv1d_backward_args *args);

/* ssam_conv1d for one more row of each of `rows` sequences.  Their states are slots of a pool, slot i at
 * d_state + i * slot_stride elements, [taps-1][channels] contiguous, updated in place.  d_slots (device, `rows` ints;
 * NULL: row r has slot r) names the slot of each row; a row whose slot is outside 0 .. slots-1 is passed over (its
 * output stays as it was), and rows that name the same slot are taken in order, as successive rows of one sequence. */
typedef struct {
    int dtype, param_dtype, channels, taps, silu;
    int rows, slots;
    const int *d_slots;
    ssam_rows in, out;         /* batch strides unused                                         */
    const void *d_weight, *d_bias;
    void *d_state;
    long long slot_stride;     /* elements of dtype, >= (taps-1) * channels                    */
} ssam_conv1d_step_args;
int ssam_conv1d_step(const ssam_conv1d_step_args *args, void *hip_stream);

/* Scan with decay chosen by the input: for every channel c (of group g = c / (channels / groups)) and state n < states
 *     d_t = softplus ? log(1 + exp(dt_t + dt_bias)) : dt_t + dt_bias
 *     h_t[n] = exp(d_t * a[c][n]) * h_{t-1}[n] + d_t * in_t * b_t[g][n]
 *     y_t = sum_n c_t[g][n] * h_t[n] + skip[c] * in_t,      out_t = gate ? y_t * gate_t / (1 + exp(-gate_t)) : y_t
 * in, dt, gate (optional), out: rows of `channels` elements; b, c: rows of groups x states elements, the states of a
 * group contiguous, b_group / c_group elements from one group to the next.  a: [channels][states]; skip, dt_bias:
 * [channels] or NULL; d_state, d_final: [sequences][channels][states], the state before the first and after the last row
 * (zeros / not stored where NULL; d_final may be d_state); all of these fp32, contiguous.
 * Of sequences of more than one row, rows lie at most 2^24 elements apart (SSAM_ERR_DIM), here and for the gradients.
 * d_marks (NULL: not wanted): the state before rows 0, 16, 32 .. of every sequence, what ssam_scan_selective_backward
 * starts from; ssam_scan_selective_marks(args) entries of [channels][states] floats, one for each 16 rows and sequence.
 * d_work: ssam_scan_selective_workspace_bytes(args) bytes, 16-byte aligned (NULL where that is 0): [channels][states + 1] floats for each piece
 * of cut sequences, however many shorter sequences lie among them.
 * Schedules: one launch where sequences and channels fill the device; otherwise sequences are cut along time: the state
 * that each piece adds, the states between the pieces, then all rows (three launches). */
typedef struct {
    int dtype, channels, states, groups, softplus;
    ssam_sequences seq;
    ssam_rows in, dt, gate, out, b, c;
    long long b_group, c_group;
    const float *d_a, *d_skip, *d_dt_bias, *d_state;
    float *d_final, *d_marks;
    void *d_work;
    size_t work_bytes;
} ssam_scan_selective_args;
int ssam_scan_selective(const ssam_scan_selective_args *args, void *hip_stream);
size_t ssam_scan_selective_workspace_bytes(const ssam_scan_selective_args *args);
long long ssam_scan_selective_marks(const ssam_scan_selective_args *args);   /* host only; 0 for invalid arguments */

/* Gradients of ssam_scan_selective, from the same inputs and its marks.  grad_out: gradient of its result;
 * d_grad_final (may be NULL): of its d_final.  grad_in, grad_dt, grad_gate, grad_b, grad_c are in dtype (grad_b and
 * grad_c contiguous within a row, [groups][states]), the others fp32 in the layout of what they belong to; each may be
 * absent (NULL).  d_grad_dt_bias is the sum of grad_dt over the rows, d_grad_state the gradient of d_state.  groups x
 * states must be below 2^27 (SSAM_ERR_DIM).
 * d_work: ssam_scan_selective_backward_workspace_bytes(args) bytes, 16-byte aligned: as above, for grad_b and grad_c 2 x groups x states floats a
 * row and 64 or 128 channels, for the parameters [channels][states + 2] floats a piece (of at most 2^15 blocks of 64 or 128 channels). */
typedef struct {
    int dtype, channels, states, groups, softplus;
    ssam_sequences seq;
    ssam_rows in, dt, gate, b, c, grad_out;
    long long b_group, c_group;
    const float *d_a, *d_skip, *d_dt_bias, *d_marks, *d_grad_final;
    ssam_rows grad_in, grad_dt, grad_gate, grad_b, grad_c;
    float *d_grad_a, *d_grad_skip, *d_grad_dt_bias, *d_grad_state;
    void *d_work;
    size_t work_bytes;
} ssam_scan_selective_backward_args;
int ssam_scan_selective_backward(const ssam_scan_selective_backward_args *args, void *hip_stream);
size_t ssam_scan_selective_backward_workspace_bytes(const ssam_scan_selective_backward_args *args);

/* ssam_scan_selective for one more row of each of `rows` sequences; slots as in ssam_conv1d_step, slot i at
 * d_state + i * slot_stride floats, [channels][states] contiguous, updated in place. */
typedef struct {
    int dtype, channels, states, groups, softplus;
    int rows, slots;
    const int *d_slots;
    ssam_rows in, dt, gate, out, b, c;   /* batch strides unused                               */
    long long b_group, c_group;
    const float *d_a, *d_skip, *d_dt_bias;
    float *d_state;
    long long slot_stride;     /* floats, >= channels * states                                 */
} ssam_scan_selective_step_args;
int ssam_scan_selective_step(const ssam_scan_selective_step_args *args, void *hip_stream);

/* Scan whose state is a matrix per head, corrected by every row (the gated delta rule).  For every head h, which uses key head
 * h / (heads / key_heads), with the state S [key_dim][value_dim] of the row before:
 *     S' = exp(g_t) S,    u = beta_t (v_t - S'^T k_t),    S = S' + k_t u^T,    out_t = scale S^T q_t
 * unit != 0: q_t and k_t are divided by sqrt(their squares' sum + 1e-6) first.  q, k: rows of key_heads x key_dim elements, v and
 * out: of heads x value_dim, a head's elements contiguous, *_head elements from one head to the next; g, beta: rows of `heads`
 * floats (g.d NULL: no decay).  d_state, d_final: [sequences][heads][key_dim][value_dim] floats, the state before the first and
 * after the last row (zeros / not stored where NULL; d_final may be d_state).  g below -1000 counts as -1000, whose exponential is 0; where
 * a sum of positive g over neighbouring rows passes 88, its exponential is infinite.
 * Rows are taken 64 at a time: a value that is not finite makes the other rows of its 64, of its head, NaN too (rows behind them
 * follow from the state); rows of no sequence reach nothing.
 * d_marks (NULL: not wanted): what ssam_scan_delta_backward starts from, ssam_scan_delta_marks(args) entries of
 * [heads][key_dim + 64][value_dim] floats: for each 64 rows and sequence the state before them and what the rows correct it by.
 * Operands of the matrix products are held as pairs of fp16, scaled by powers of two: with an error of 2^-22 of a value or 2^-35 of the largest that
 * shares its power of two, whichever is more.  Those are a value's 64 rows (of v, the corrections and their gradients), a state's column, a row
 * of q or k in fp32: where sizes differ by more than 2^13, the small ones have fewer bits, also if a decay between the rows parts them.  q and k in bf16 are
 * exact down to 2^-27 of a row's largest element and at most 2^-34 of that off below; in fp16 they are taken as they are.
 * key_dim is at most SSAM_MAX_KEY (SSAM_ERR_SHAPE), heads x value_dim at most 2^24; of sequences of more than one row, and of a step's
 * rows, rows lie at most 2^24 elements apart, here and for the gradients (SSAM_ERR_DIM).
 * d_work: ssam_scan_delta_workspace_bytes(args) bytes, 16-byte aligned.
 * Schedules: two launches, the 64 rows' own matrices for all of them at once, then the state's way through them, a block for each head and
 * 64 of its values (fp32, where there are many: 128). */
typedef struct {
    int dtype, heads, key_heads, key_dim, value_dim, unit;
    float scale;
    ssam_sequences seq;
    ssam_rows q, k, v, out, g, beta;
    long long q_head, k_head, v_head, out_head;
    const float *d_state;
    float *d_final, *d_marks;
    void *d_work;
    size_t work_bytes;
} ssam_scan_delta_args;
int ssam_scan_delta(const ssam_scan_delta_args *args, void *hip_stream);
size_t ssam_scan_delta_workspace_bytes(const ssam_scan_delta_args *args);
long long ssam_scan_delta_marks(const ssam_scan_delta_args *args);   /* host only; 0 for invalid arguments */

/* Gradients of ssam_scan_delta, from the same inputs and its marks.  grad_out: gradient of its result; d_grad_final (may be
 * NULL): of its d_final.  grad_q, grad_k, grad_v are in dtype, a row's elements contiguous, grad_g and grad_beta rows of `heads`
 * floats; each may be absent (NULL).  d_grad_state is the gradient of d_state, or of the zeros that stand for it.
 * d_work: ssam_scan_delta_backward_workspace_bytes(args) bytes, 16-byte aligned. */
typedef struct {
    int dtype, heads, key_heads, key_dim, value_dim, unit;
    float scale;
    ssam_sequences seq;
    ssam_rows q, k, v, grad_out, g, beta;
    long long q_head, k_head, v_head, grad_out_head;
    const float *d_marks, *d_grad_final;
    ssam_rows grad_q, grad_k, grad_v, grad_g, grad_beta;
    float *d_grad_state;
    void *d_work;
    size_t work_bytes;
} ssam_scan_delta_backward_args;
int ssam_scan_delta_backward(const ssam_scan_delta_backward_args *args, void *hip_stream);
size_t ssam_scan_delta_backward_workspace_bytes(const ssam_scan_delta_backward_args *args);

/* ssam_scan_delta for one more row of each of `rows` sequences; slots as in ssam_conv1d_step, slot i at
 * d_state + i * slot_stride floats, [heads][key_dim][value_dim] contiguous, updated in place. */
typedef struct {
    int dtype, heads, key_heads, key_dim, value_dim, unit;
    float scale;
    int rows, slots;
    const int *d_slots;
    ssam_rows q, k, v, out, g, beta;   /* batch strides unused                                 */
    long long q_head, k_head, v_head, out_head;
    float *d_state;
    long long slot_stride;     /* floats, >= heads * key_dim * value_dim                       */
} ssam_scan_delta_step_args;
int ssam_scan_delta_step(const ssam_scan_delta_step_args *args, void *hip_stream);

/* Root-mean-square norm of the groups of a row, width = channels / groups elements each:
 *     s = in + residual, rounded to dtype (in where there is no residual);   y = s / sqrt(mean(s^2) + eps) * weight
 *     out = gate ? y * gate / (1 + exp(-gate)) : y
 * `sequences` x `rows` rows (a batch's strides count from sequence to sequence).  sum (may be absent, or residual itself) receives s;
 * the norm is that of s as it is stored, so that s is all that the gradients need.  weight: [width] in param_dtype (dtype or
 * SSAM_F32), NULL: ones.  width is at most 32768 (SSAM_ERR_SHAPE).
 * ssam_rms_norm_e4m3: out is in 8 bits (e4m3, 448 at most) with a scale for every `block` channels, a divisor of width, 16 at least
 * or the whole of it (SSAM_ERR_SHAPE):
 *     scale = max over the block of |y| / 448 (at least 2^-126; 1 where all are zero),   out = y / scale, rounded to nearest
 * d_scales: [sequences * rows][channels / block] floats; out's strides count bytes.  The quotient is that of s * weight * gate's factor and the block's
 * largest of them, from which the root has gone: halves between two codes are met as such and go to the even one. */
typedef struct {
    int dtype, param_dtype, channels, groups, block;   /* block: ssam_rms_norm_e4m3 only         */
    int sequences, rows;
    float eps;                 /* >= 0                                                         */
    ssam_rows in, residual, sum, gate, out;
    const void *d_weight;
    float *d_scales;           /* ssam_rms_norm_e4m3 only                                      */
} ssam_rms_norm_args;
int ssam_rms_norm(const ssam_rms_norm_args *args, void *hip_stream);
int ssam_rms_norm_e4m3(const ssam_rms_norm_args *args, void *hip_stream);

/* Gradients of ssam_rms_norm.  in: what was normalised (its sum, where it had a residual); grad_out: gradient of its result;
 * grad_sum (may be absent): of its sum, which is added to grad_in.  grad_in, that of in and of residual alike, and grad_gate are in
 * dtype, d_grad_weight in param_dtype; each may be absent (NULL).
 * d_work: ssam_rms_norm_backward_workspace_bytes(args) bytes (0 without d_grad_weight), 16-byte aligned. */
typedef struct {
    int dtype, param_dtype, channels, groups;
    int sequences, rows;
    float eps;
    ssam_rows in, gate, grad_out, grad_sum, grad_in, grad_gate;
    const void *d_weight;
    void *d_grad_weight;
    void *d_work;
    size_t work_bytes;
} ssam_rms_norm_backward_args;
int ssam_rms_norm_backward(const ssam_rms_norm_backward_args *args, void *hip_stream);
size_t ssam_rms_norm_backward_workspace_bytes(const ssam_rms_norm_backward_args *args);

#ifdef __cplusplus
}
#endif
#endif /* SSAM_SEQUENCE_H_ */
