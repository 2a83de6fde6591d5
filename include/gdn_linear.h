/*
 * gdn_linear.h -- C ABI of linear attention with a fixed decay for each head in
 * libgdn_tailreplay.so (MI355X, gfx950), for packed sequences and for one token
 * per sequence.
 *
 * The simplest of the recurrences of hybrid models.  For every packed sequence n
 * and value head h, with key/query head kh = h / (Hv / Hk):
 *     M_t = exp(g_h) M_{t-1} + k_t v_t^T        (d_k x d_v, fp32)
 *     o_t = scale M_t^T q_t.
 * As with the delta rule (gdn_tail_replay.h), a state may be rebuilt by replaying
 * only a tail of the matched prefix from the zero state.
 *
 * Conventions as in gdn_ssm.h: strided token rows, rows at or behind
 * cu_seqlens[N] left alone, an input that is not finite reaches outputs of its
 * own sequence only (every output of its 64-token chunk and all later ones).
 * g <= 0 is assumed, not checked; a decay below 2^-150 a token is taken as that.
 */
#ifndef GDN_LINEAR_H
#define GDN_LINEAR_H

#include "gdn_tail_replay.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t num_seqs;     /* N >= 0                                            */
  int32_t num_k_heads;  /* Hk >= 1: heads of q and k                         */
  int32_t num_v_heads;  /* Hv >= 1: heads of v, g, o and state; Hv % Hk == 0 */
  int32_t d_k;          /* key head dimension, 64 or 128                     */
  int32_t d_v;          /* value head dimension, 64 or 128                   */
  int32_t dtype;        /* gdn_dtype of q, k, v and o                        */
  float scale;          /* finite                                            */
  int64_t ld_q;         /* elements between token rows, >= Hk d_k            */
  int64_t ld_k;         /* >= Hk d_k                                         */
  int64_t ld_v;         /* >= Hv d_v                                         */
  int64_t ld_o;         /* >= Hv d_v                                         */
} gdn_linear_shape;     /* ld_q and ld_o are looked at only where o is given */

/* Workspace bytes of gdn_linear_attention, with or without o (0 where the sequences run unsplit). */
gdn_status gdn_linear_attention_workspace_size(const gdn_linear_shape* shape, const int32_t* cu_seqlens_host,
                                               size_t* bytes);

/*
 * Packed sequences, from state_in (NULL = zero state):
 *   q, k [T, Hk, d_k], v, o [T, Hv, d_v]: dtype; g [Hv] fp32;
 *   state_in, state_out [N, Hv, d_k, d_v] fp32.
 * o NULL = no outputs (the states alone, as where a tail is replayed; q is not
 * read then and may be NULL); state_out NULL = not written (one of the two is
 * required where there are tokens).  state_out may equal state_in and must not
 * otherwise overlap it, nor another input; o must not overlap an input or a
 * state.  A zero-length sequence writes its state_in (or zeros) to state_out.
 * q, k, v, o and the states must be 16-byte aligned, row strides multiples of 16
 * bytes (GDN_ERR_UNSUPPORTED otherwise).  workspace: at least
 * gdn_linear_attention_workspace_size bytes, 256-byte aligned; NULL is accepted
 * where that is 0.
 */
gdn_status gdn_linear_attention(const gdn_linear_shape* shape, const int32_t* cu_seqlens_host,
                                const int32_t* cu_seqlens, const void* q, const void* k, const void* v,
                                const float* g, const float* state_in, void* o, float* state_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * One token per sequence (T = N): the state is advanced once, o and state_out
 * are required, state_out may equal state_in.  One kernel, no workspace.
 */
gdn_status gdn_linear_attention_step(const gdn_linear_shape* shape, const void* q, const void* k,
                                     const void* v, const float* g, const float* state_in, void* o,
                                     float* state_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_LINEAR_H */
