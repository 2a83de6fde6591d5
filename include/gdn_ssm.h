/*
 * gdn_ssm.h -- C ABI of the short causal convolution and the selective state
 * space scan in libgdn_tailreplay.so (MI355X, gfx950), each for packed
 * sequences and for one token per sequence.
 *
 * Hybrid models put one of two recurrences behind a short convolution.  The
 * gated delta rule is in gdn_tail_replay.h; this is the other one, a state
 * space layer with input-dependent steps.  For every packed sequence n and
 * head h, with group gh = h / (H / G) and, per token t,
 *     delta = softplus(dt_t + dt_bias),   alpha = exp(-exp(a_log) delta),
 *     M_t = alpha M_{t-1} + B_t (delta x_t)^T        (d_state x head_dim, fp32)
 *     y_t = M_t^T C_t + d_skip x_t.
 * As with the delta rule, a state may be rebuilt by scanning only a tail of the
 * matched prefix from the zero state.
 *
 * Conventions as in gdn_tail_replay.h (device pointers unless named _host,
 * caller-owned buffers, host-side validation before anything is enqueued,
 * everything on `stream`, capturable, no allocation), and:
 *   - Rows.  Token rows may be strided: ld_* is the distance of two tokens'
 *     rows in elements, so that a call reads its columns out of a projection's
 *     rows; at most 2^23.  Inside a row the elements are dense.
 *   - Rows at or behind cu_seqlens[N] are neither read nor written.
 *   - An input that is not finite reaches outputs of its own sequence only.
 *     In gdn_ssm_scan it may reach every output of its 64-token chunk
 *     (counted from the sequence's first token) and all later ones; in
 *     gdn_causal_conv the outputs whose taps it meets.
 */
#ifndef GDN_SSM_H
#define GDN_SSM_H

#include "gdn_tail_replay.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { GDN_ACT_NONE = 0, GDN_ACT_SILU = 1 } gdn_activation;

typedef struct {
  int32_t num_seqs;     /* N >= 0                                            */
  int32_t channels;     /* C >= 1                                            */
  int32_t taps;         /* W: 2, 3 or 4                                      */
  int32_t dtype;        /* gdn_dtype of x, y and the histories               */
  int32_t activation;   /* gdn_activation                                    */
  int64_t ld_x;         /* elements between token rows of x, >= C            */
  int64_t ld_y;         /* elements between token rows of y, >= C            */
} gdn_conv_shape;

/*
 * Causal depthwise convolution of packed sequences:
 *     y[t, c] = act(bias[c] + sum_j weight[c, j] x[t - W + 1 + j, c]),
 * where the W - 1 rows before a sequence's first token are history_in[n] (zeros
 * when history_in is NULL).
 *   x [T, C] (rows ld_x apart), y [T, C] (rows ld_y apart): dtype;
 *   weight [C, W] fp32; bias [C] fp32, NULL = none;
 *   history_in, history_out [N, W - 1, C] dtype, oldest row first.
 * history_out (NULL = not written) receives the last W - 1 rows of history_in
 * followed by the sequence, which is what the next call or gdn_causal_conv_step
 * starts from; it may equal history_in and must not otherwise overlap it.  y
 * must not overlap x (columns of the same rows that do not meet are allowed
 * when ld_x == ld_y), nor either of them a history.
 * Any alignment of the element type is accepted; 16-byte aligned pointers with
 * C, ld_x and ld_y multiples of 16 bytes take the 16-byte accesses.
 */
gdn_status gdn_causal_conv(const gdn_conv_shape* shape, const int32_t* cu_seqlens_host,
                           const int32_t* cu_seqlens, const void* x, const float* weight,
                           const float* bias, const void* history_in, void* y,
                           void* history_out, void* stream);

/*
 * The same for one token per sequence: x [N, C], y [N, C].  history_in NULL =
 * zeros; history_out is required and may equal history_in.
 */
gdn_status gdn_causal_conv_step(const gdn_conv_shape* shape, const void* x, const float* weight,
                                const float* bias, const void* history_in, void* y,
                                void* history_out, void* stream);

typedef struct {
  int32_t num_seqs;     /* N >= 0                                            */
  int32_t num_heads;    /* H >= 1: heads of x, dt, y and the state           */
  int32_t num_groups;   /* G >= 1: heads of B and C; H % G == 0              */
  int32_t d_state;      /* rows of the state, 64 or 128                      */
  int32_t head_dim;     /* columns of the state, 64 or 128                   */
  int32_t dtype;        /* gdn_dtype of x, B, C and y                        */
  int32_t dt_dtype;     /* gdn_dtype of dt: GDN_F32 or the same as dtype     */
  int64_t ld_x;         /* elements between token rows, >= H head_dim        */
  int64_t ld_dt;        /* >= H                                              */
  int64_t ld_b;         /* >= G d_state                                      */
  int64_t ld_c;         /* >= G d_state                                      */
  int64_t ld_y;         /* >= H head_dim                                     */
} gdn_ssm_shape;        /* ld_c and ld_y are looked at only where y is given */

/* Workspace bytes of gdn_ssm_scan, with or without y (0 where the sequences run unsplit). */
gdn_status gdn_ssm_workspace_size(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host,
                                  size_t* bytes);

/*
 * The scan of packed sequences, from state_in (NULL = zero state):
 *   x [T, H, head_dim], B, C [T, G, d_state], y [T, H, head_dim]: dtype;
 *   dt [T, H]: dt_dtype; a_log [H] fp32; d_skip, dt_bias [H] fp32, NULL = 0;
 *   state_in, state_out [N, H, d_state, head_dim] fp32.
 * y NULL = no outputs (the state alone, as where a tail is replayed; C and
 * d_skip are not read then and may be NULL); state_out NULL = not written
 * (one of the two is required where there are tokens).  state_out may equal state_in and must not
 * otherwise overlap it, nor another input; y must not overlap an input or a
 * state.  A zero-length sequence writes its state_in (or zeros) to state_out.
 * x, B, C, y and the states must be 16-byte aligned, the row strides of x, B, C
 * and y multiples of 16 bytes (GDN_ERR_UNSUPPORTED otherwise).
 * workspace: at least gdn_ssm_workspace_size bytes, 256-byte aligned; NULL is
 * accepted where that is 0.
 */
gdn_status gdn_ssm_scan(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host,
                        const int32_t* cu_seqlens, const void* x, const void* dt,
                        const float* a_log, const void* B, const void* C, const float* d_skip,
                        const float* dt_bias, const float* state_in, void* y, float* state_out,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * One token per sequence (T = N): the state is advanced once, y and state_out
 * are required, state_out may equal state_in.  One kernel, no workspace.
 * Alignment as for gdn_ssm_scan.
 */
gdn_status gdn_ssm_step(const gdn_ssm_shape* shape, const void* x, const void* dt,
                        const float* a_log, const void* B, const void* C, const float* d_skip,
                        const float* dt_bias, const float* state_in, void* y, float* state_out,
                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_SSM_H */
