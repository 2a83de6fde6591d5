/*
 * gdn_attn.h -- C ABI of a hybrid model's full-attention layer at a prefix hit
 * in libgdn_tailreplay.so (MI355X, gfx950): the pages that its keys and values
 * lie in, norm and rotation of queries and keys on their way there, and the
 * attention of a batch that shares a prefix.
 *
 * Pages.  A cache holds num_pages pages of page_size tokens; token row r of
 * page p is slot p * page_size + r.  A sequence's tokens lie in the pages of its
 * row of a block table, in order: its token i in page table[n][i / page_size],
 * row i % page_size.  An entry outside [0, num_pages) is no page: tokens there
 * are not written and not seen.
 *
 * Conventions as in gdn_tail_replay.h (device pointers unless named _host,
 * caller-owned buffers, host-side validation before anything is enqueued,
 * everything on `stream`, capturable, no allocation), and:
 *   - Rows of q, k, v and outputs may be strided, ld_* elements apart (at most
 *     2^23); the heads of a row are dense.  Rows at or behind cu_seqlens[N] are
 *     left alone.
 *   - lens, block tables, slots and positions are read on the device alone, so
 *     a captured step can be replayed while they advance.
 */
#ifndef GDN_ATTN_H
#define GDN_ATTN_H

#include "gdn_tail_replay.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ pages */
typedef struct {
  int32_t num_seqs;     /* N >= 0                                            */
  int32_t table_width;  /* W >= 1: entries of a block table's row            */
  int32_t page_size;    /* tokens of a page, >= 1                            */
  int32_t num_free;     /* F >= 0: entries of free_pages                     */
  int32_t first;        /* position of a sequence's own token 0 (>= 0): the
                           length of a prefix that lies elsewhere            */
} gdn_pages_shape;

/* Workspace bytes of gdn_extend_pages. */
gdn_status gdn_extend_pages_workspace_size(const gdn_pages_shape* shape, const int32_t* cu_seqlens_host,
                                           size_t* bytes);

/*
 * Makes room for the new tokens of every sequence, packed by cu_seqlens.
 * Sequence n holds lens_in[n] tokens and gets q = cu[n + 1] - cu[n] more:
 *   lens_out[n]  = lens_in[n] + q;
 *   table_out[n] = table_in[n] with the entries from ceil(lens_in / page_size) up
 *                  to ceil(lens_out / page_size) taken from free_pages, in order
 *                  of the sequences, from entry taken_in[0] on;
 *   taken_out[0] = taken_in[0] + the pages that all sequences take;
 *   slots[t], positions[t] of new token t, the i-th of sequence n: the slot of
 *                  its token lens_in + i, and first + lens_in + i.
 * Where the free list ends (taken_out > F then) an entry is -1.  A table row
 * holds W entries: what would lie behind them is not taken.  Tokens without a
 * page get slot -1, also where a slot would pass 2^31 - 1.
 *   table_in, table_out [N, W] int32; lens_in, lens_out [N] int32 (negative
 *   values count as 0, sums stop at 2^31 - 1); free_pages [F] int32; taken_in
 *   [1] int32 (NULL = 0; negative = 0), taken_out [1] int32; slots, positions
 *   [T] int32.
 * Each output may equal its input (updated in place) and must not otherwise
 * overlap an input or another output.  workspace: at least
 * gdn_extend_pages_workspace_size bytes, 256-byte aligned.
 */
gdn_status gdn_extend_pages(const gdn_pages_shape* shape, const int32_t* cu_seqlens_host,
                            const int32_t* cu_seqlens, const int32_t* table_in, const int32_t* lens_in,
                            const int32_t* free_pages, const int32_t* taken_in, int32_t* table_out,
                            int32_t* lens_out, int32_t* taken_out, int32_t* slots, int32_t* positions,
                            void* workspace, size_t workspace_bytes, void* stream);

/* --------------------------------------------- norm and rotation, into pages */
typedef struct {
  int32_t num_tokens;    /* T >= 0                                           */
  int32_t num_heads;     /* Hq >= 1                                          */
  int32_t num_kv_heads;  /* Hkv >= 1                                         */
  int32_t head_dim;      /* D: 64 or 128                                     */
  int32_t dtype;         /* gdn_dtype of q, k, v, their outputs and the caches */
  int32_t rotary_dim;    /* R: the first R of D are rotated; multiple of 16  */
  int32_t interleaved;   /* 0: pairs (i, i + R/2); 1: pairs (2 i, 2 i + 1)   */
  int32_t num_positions; /* P >= 1: rows of cos_sin                          */
  float eps;             /* of the norms, >= 0                               */
  int32_t num_pages, page_size;     /* of the caches, where they are given   */
  int64_t ld_q, ld_k, ld_v;         /* elements between token rows           */
  int64_t ld_q_out, ld_k_out;
  int64_t k_page, k_token, k_head;  /* elements between pages, tokens of a page and heads of k_cache */
  int64_t v_page, v_token, v_head;  /* and of v_cache                        */
} gdn_qk_shape;

/*
 * Per head of q and k: x <- x rsqrt(mean(x^2) + eps) w (where w is given), then
 * the first R elements are rotated by the token's row c | s of cos_sin: pair p
 * (a, b) becomes (a c_p - b s_p, b c_p + a s_p).  q goes to q_out, k to k_out
 * and/or into k_cache at the token's slot; v is copied into v_cache there.
 *   q [T, Hq, D], k, v [T, Hkv, D]; positions [T] int32; cos_sin [P, R] fp32
 *   (R/2 cosines, then R/2 sines); q_weight, k_weight [D] fp32, both or neither
 *   (NULL = no norm); k_cache, v_cache pages of [page_size, Hkv, D] with the
 *   strides of the shape; slots [T] int32, required with a cache.
 * k_out, the caches and v may be NULL: v and v_cache go together, and k_out or
 * k_cache is required.  q_out may equal q and k_out equal k (rotated in place, at
 * equal strides); outputs must not otherwise overlap an input or each other.
 * A token whose slot is no row of the cache is not written there.  A token whose
 * position is outside [0, P) is skipped whole: none of its outputs is written.
 * Two tokens with one slot leave either's rows there.
 * Pointers other than slots and positions must be 16-byte aligned, strides
 * multiples of 16 bytes (GDN_ERR_UNSUPPORTED otherwise).
 */
gdn_status gdn_qk_norm_rope(const gdn_qk_shape* shape, const void* q, const void* k, const void* v,
                            const int32_t* positions, const float* cos_sin, const float* q_weight,
                            const float* k_weight, const int32_t* slots, void* q_out, void* k_out,
                            void* k_cache, void* v_cache, void* stream);

/* ------------------------------------------------------------- attention */
typedef struct {
  int32_t num_seqs;      /* N >= 0                                           */
  int32_t num_heads;     /* Hq >= 1: query heads; head h reads K/V head h / (Hq / Hkv) */
  int32_t num_kv_heads;  /* Hkv >= 1; Hq % Hkv == 0                          */
  int32_t head_dim;      /* D: 64 or 128                                     */
  int32_t dtype;         /* gdn_dtype of q, out and the caches               */
  int32_t num_pages, page_size;
  int32_t table_width;   /* W >= 1                                           */
  int32_t prefix_len;    /* P >= 0: tokens that all sequences share          */
  int32_t max_len;       /* no sequence holds more own tokens than this: a
                            length above it counts as max_len, one below 0 as
                            0; at most W page_size, 0 = that.  Work is cut by
                            it: to be given where tables are much wider      */
  float scale;           /* finite                                           */
  int64_t ld_q, ld_out;
  int64_t k_page, k_token, k_head;  /* elements between pages, tokens of a page and heads */
  int64_t v_page, v_token, v_head;
} gdn_attn_shape;

/* Workspace bytes of gdn_prefix_attention. */
gdn_status gdn_prefix_attention_workspace_size(const gdn_attn_shape* shape, const int32_t* cu_seqlens_host,
                                               size_t* bytes);

/*
 * For every packed query t, the i-th of the q_n of sequence n, and head h:
 *   out[t, h] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q[t, h] . k_j),
 * over the P tokens of the shared prefix and the sequence's own tokens
 * j <= lens[n] - q_n + i: its queries are its last tokens, whose keys and values
 * are in the cache already.  With P = 0 this is plain causal attention over
 * pages.  A query that sees no token gets zeros; one all of whose scores are -inf
 * has no output, 0 / 0, and gets NaN.
 *   q, out [T, Hq, D]; k_cache, v_cache as in gdn_qk_norm_rope; table [N, W]
 *   int32; lens [N] int32; prefix_pages [ceil(P / page_size)] int32.
 * Scores and sums are fp32 (so the values that a query sees must not add up to
 * 2^128 or more: the sums are formed at weights up to 1 and divided at the end);
 * for bf16 the weights w enter the second product rounded to bf16.  What lies in
 * a cache where no query looks (behind a sequence's last token, in other pages)
 * has no effect, whatever its bits; a key or value that is not finite reaches the
 * queries that see it, and no others.
 * out must not overlap q or the caches.  q, out and the caches must be 16-byte
 * aligned, strides multiples of 16 bytes (GDN_ERR_UNSUPPORTED otherwise).
 * workspace: at least gdn_prefix_attention_workspace_size bytes, 256-byte aligned.
 */
gdn_status gdn_prefix_attention(const gdn_attn_shape* shape, const int32_t* cu_seqlens_host,
                                const int32_t* cu_seqlens, const void* q, const void* k_cache,
                                const void* v_cache, const int32_t* table, const int32_t* lens,
                                const int32_t* prefix_pages, void* out, void* workspace,
                                size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_ATTN_H */
