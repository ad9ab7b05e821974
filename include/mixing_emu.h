/*
 * mixing_emu.h -- C ABI of the token mixing operators of libsgemm_emu.so:
 * rotary positions and the gated delta rule.  Status codes, streams, graph
 * capture, threads and ownership of memory are as in sgemm_emu.h.
 */
#ifndef MIXING_EMU_H
#define MIXING_EMU_H

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "sgemm_emu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Conventions --------------------------------------------------------
 * Plane rotations by position and the gated delta rule: the operators of a
 * linear-attention layer, built on the same ground as the entries above (a
 * rotary position is a Givens rotation of pairs of a head; the delta rule
 * multiplies a state by one decayed reflector I - beta k k^T per token; the
 * decays' running sums are a scan; the products of a chunk are emulated in
 * FP32 on fp16 matrix instructions).
 *
 * Tensors are (batch, token, head, element) views with element strides for
 * the first three; the last dimension is contiguous.  Input strides may be
 * zero (broadcast); an output's elements must be apart (ERR_STRIDE).  Spans
 * of outputs must not overlap spans of inputs (ERR_ALIAS) except where noted, and
 * two outputs must not share elements (ERR_ALIAS); their spans may overlap where they lie
 * between each other with the same strides (slices of one buffer).
 * Elements are aligned to their size; with 16-byte aligned rows the loads are vectors. */
#define SGEMM_EMU_F32 0
#define SGEMM_EMU_BF16 1
#define SGEMM_EMU_F16 2

typedef struct {
    void* p;
    int64_t batch, token, head; /* element strides */
} sgemm_emu_view_t;

/*
 * Rotary positions on one or two tensors in one launch.  For every token with
 * position p and every head x, the first `rot` elements are turned in pairs
 * by the table's angles and the others copied:
 *   (y_a, y_b) = (x_a cos - x_b sin, x_a sin + x_b cos),
 * cos = cos_table[p][i], sin = sin_table[p][i] (row-major table_rows x rot/2,
 * FP32), pair i being elements (2i, 2i+1) if `interleaved`, else
 * (i, i + rot/2).  `inverse` turns back (sin negated): the gradient of the
 * rotation, and its inverse.  Computed in FP32, rounded once to the type.
 *   positions: device int32 (position_bytes 4) or int64 (8), position of
 *     token (b, t) at b*position_batch + t*position_token; NULL: t + offset.
 *   A position outside the table gives NaN in the rotated elements.
 *   x[1].p == NULL or heads[1] == 0: one tensor only.
 *   y[i] may be x[i] itself (same pointer and strides: in place).
 * Errors: _DIM (also a negative offset), _UNSUPPORTED (rot odd, < 0 or > size;
 * dtype or position_bytes unknown; more than 2^31 - 1 tokens in all, or elements
 * of a token),
 * _NULL, _STRIDE, _ALIAS, _HIP.
 */
typedef struct {
    int32_t dtype, batch, tokens, size, rot, interleaved, inverse, table_rows;
    int32_t heads[2];
    sgemm_emu_view_t x[2], y[2];
    const float* cos_table;
    const float* sin_table;
    const void* positions;
    int64_t position_batch, position_token, offset;
    int32_t position_bytes, reserved;
} rotary_emu_t;

int rotary_emu(const rotary_emu_t* a, hipStream_t stream);

/*
 * The tables of rotary_emu: for p in [0, rows), i in [0, rot/2), with
 *   f_i = base^(-2i/rot),   r_i = original f_i / 2 pi  (turns over the original length),
 *   w_i = min(1, max(0, (r_i - low) / (high - low)))   (low < high), else 0,
 *   f'_i = f_i (w_i + (1 - w_i) / factor),
 *   cos_table[p][i] = amplitude cos(p f'_i), sin_table[p][i] = amplitude sin(p f'_i).
 * factor 1: plain positions.  factor > 1 with low == high: all frequencies
 * divided by factor (positions interpolated).  With low < high the pairs that
 * turn more than `high` times over the original length keep their frequency,
 * those that turn less than `low` times are interpolated, and the ramp
 * joins them.  Angles are formed and reduced in FP64, so the entries are
 * within one rounding of FP32 at any position.
 * Errors: _DIM (rows or rot negative, rot odd), _UNSUPPORTED (base <= 0,
 * factor <= 0, low > high, a value that is not finite), _NULL, _ALIAS, _HIP.
 */
int rotary_emu_table(int rows, int rot, double base, double factor, double original, double low,
                     double high, double amplitude, float* cos_table, float* sin_table,
                     hipStream_t stream);

/*
 * The gated delta rule.  q, k: (batch, tokens, k_heads, k_size); v, o: (batch,
 * tokens, v_heads, v_size), all of one dtype; g, beta: (batch, tokens, v_heads)
 * FP32 (their views' `head` stride is that of the last dimension).  Value head h reads
 * key head h / (v_heads / k_heads).  Per sequence and value head a state S
 * (k_size x v_size, FP32) goes from token to token:
 *   S_t = e^{g_t} S_{t-1} + k_t u_t^T,   u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t),
 *   o_t = scale S_t^T q_t.
 * g.p == NULL: no decay; beta.p == NULL: beta = 1.  g <= 0 is expected; decays below
 * e^-200 (g = -infinity too) count as zero.  States and gradients of states
 * are contiguous (sequence, v_heads, k_size, v_size) FP32.
 *   cu_seqlens NULL: `batch` sequences of `tokens` tokens.
 *   else: packed sequences; the views' batch stride is not used, `tokens` is the
 *     number of rows in all, and sequence n is rows cu_seqlens[n] to
 *     cu_seqlens[n+1] - 1 (device, int32, batch + 1 values, not decreasing; values outside
 *     [0, tokens] are clamped to it; where they decrease, results are unspecified, and
 *     nothing outside the tensors is touched).  Rows of no sequence are not written.
 * initial: states before the first tokens, or NULL (zero).
 * workspace: device memory, 256-byte aligned, at least what the _workspace query
 *   for the same arguments returns (0 for up to 16 tokens that are not packed, which
 *   go token by token); its contents need not be kept.
 * Sizes: k_size <= 128, v_size <= 65536, token strides <= 2^22 (of q, k, v, o
 * and their gradients; the recurrent form takes any), k_heads divides v_heads.
 * Empty sequences leave final = initial.  A value that is not finite reaches what the
 * recurrence takes it to: no earlier token, other sequence, head or, if it is in
 * v or a state, column.
 * Errors: _DIM, _UNSUPPORTED (dtype, sizes and strides above, head counts, more than
 * 2^21 chunks x value heads, or sequences x value heads x groups of 64 value columns; of 32
 * where float32 outputs of more than 16 tokens have keys above 64),
 * _NULL, _STRIDE, _ALIAS, _HIP.
 */
typedef struct {
    int32_t dtype, batch, tokens, k_heads, v_heads, k_size, v_size;
    float scale;
    const int32_t* cu_seqlens;
    sgemm_emu_view_t q, k, v, g, beta, o;
    const float* initial;
    float* final_state; /* may be NULL, or == initial */
    void* workspace;
    int64_t workspace_bytes;
} delta_emu_forward_t;

/* Bytes of workspace, or a negative error; pointers are not looked at except
 * for being NULL. */
int64_t delta_emu_forward_workspace(const delta_emu_forward_t* a);
int delta_emu_forward(const delta_emu_forward_t* a, hipStream_t stream);

/* The gradient: from d_o (like o) and dfinal (gradient of the final states, or
 * NULL) to dq, dk, dv (the inputs' type), dg, dbeta (FP32; p NULL: not
 * wanted) and dinitial (or NULL).  Sums over the value heads of a key head and over
 * tokens are in FP32 in a fixed order.  dinitial may be dfinal.  A value of d_o or dfinal
 * that is not finite reaches no later token (nor other sequence, head or, in dv and
 * dinitial, column); where q, k, v, g, beta or a state is not, any gradient of that sequence's
 * key head may not be. */
typedef struct {
    int32_t dtype, batch, tokens, k_heads, v_heads, k_size, v_size;
    float scale;
    const int32_t* cu_seqlens;
    sgemm_emu_view_t q, k, v, g, beta, d_o;
    sgemm_emu_view_t dq, dk, dv, dg, dbeta;
    const float* initial;
    const float* dfinal;
    float* dinitial;
    void* workspace;
    int64_t workspace_bytes;
} delta_emu_backward_t;

int64_t delta_emu_backward_workspace(const delta_emu_backward_t* a);
int delta_emu_backward(const delta_emu_backward_t* a, hipStream_t stream);

/* The recurrent form: `tokens` tokens of each of `batch` sequences, one after
 * another, on states that are updated in place: sequence b's state is
 * state + slot * state_stride, slot = slots[b] (device, int32) or b if slots is
 * NULL.  A slot outside [0, n_slots) leaves the sequence out (o = 0 there); slots
 * that occur are different ones.  state_stride >= v_heads * k_size * v_size.
 * No workspace.  For single tokens and a few drafted ones: every token costs a
 * pass over the state's registers. */
typedef struct {
    int32_t dtype, batch, tokens, k_heads, v_heads, k_size, v_size;
    float scale;
    sgemm_emu_view_t q, k, v, g, beta, o;
    float* state;
    int64_t state_stride;
    const int32_t* slots;
    int32_t n_slots, reserved;
} delta_emu_step_t;

int delta_emu_step(const delta_emu_step_t* a, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MIXING_EMU_H */
