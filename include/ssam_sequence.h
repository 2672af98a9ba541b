/* ssam_sequence.h -- filters and scans along time, channel by channel: the two halves of a state space layer of a
 * language model, in the C ABI's manner (every convention of ssam.h holds here too, except where a line below says
 * otherwise).
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

#ifdef __cplusplus
}
#endif
#endif /* SSAM_SEQUENCE_H_ */
