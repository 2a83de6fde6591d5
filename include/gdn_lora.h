/*
 * gdn_lora.h -- C ABI of low-rank adapters beside a shared projection in
 * libgdn_tailreplay.so (MI355X, gfx950).
 *
 * Requests of one batch share a projection's weights, and each may carry an
 * adapter of its own.  For every token t of packed sequence n with adapter
 * a = adapters[n]:
 *     out[t] = base[t] + scales[a] (x[t] A_a^T) B_a^T,
 * and out[t] = base[t] where a = -1 (no adapter).  `base` is what the shared
 * projection gave.
 *
 * Conventions as in gdn_tail_replay.h; token rows may be strided and rows at or
 * behind cu_seqlens[N] are left alone, as in gdn_ssm.h.  x A^T is summed in
 * fp32; for fp32 outputs it enters the second product with 24 bits, for bf16
 * outputs with 16.  A token whose x A^T is not finite gets outputs that are not
 * (NaN also where the formula gives an infinity), and no other token does.
 */
#ifndef GDN_LORA_H
#define GDN_LORA_H

#include "gdn_tail_replay.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t num_seqs;      /* N >= 0                                           */
  int32_t num_adapters;  /* >= 0                                             */
  int32_t hidden;        /* K: columns of x, multiple of 8                   */
  int32_t width;         /* M >= 1: columns of base and out                  */
  int32_t rank;          /* R: multiple of 8, at most 128; smaller adapters
                            are padded with zero rows                        */
  int32_t out_dtype;     /* gdn_dtype of base and out                        */
  int64_t ld_x;          /* elements between token rows, >= K, multiple of 8 */
  int64_t ld_base;       /* >= M                                             */
  int64_t ld_out;        /* >= M                                             */
} gdn_lora_shape;

/* Workspace bytes of gdn_lora_add. */
gdn_status gdn_lora_workspace_size(const gdn_lora_shape* shape, const int32_t* cu_seqlens_host,
                                   size_t* bytes);

/*
 *   x [T, K] bf16; lora_a [num_adapters, R, K] bf16; lora_b [num_adapters, M, R]
 *   bf16; scales [num_adapters] fp32, NULL = 1; base, out [T, M] out_dtype;
 *   adapters_host, adapters [N] int32: the adapter of each sequence, -1 = none;
 *   the caller guarantees that the device copy holds the same values.
 * out may equal base (with ld_out == ld_base): the adapters are then added in
 * place and rows without one are not touched.  It must not otherwise overlap
 * base, nor x.
 * x, lora_a and lora_b must be 16-byte aligned (GDN_ERR_UNSUPPORTED otherwise).
 * workspace: at least gdn_lora_workspace_size bytes, 256-byte aligned.
 */
gdn_status gdn_lora_add(const gdn_lora_shape* shape, const int32_t* cu_seqlens_host,
                        const int32_t* cu_seqlens, const int32_t* adapters_host,
                        const int32_t* adapters, const void* base, const void* x,
                        const void* lora_a, const void* lora_b, const float* scales, void* out,
                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GDN_LORA_H */
