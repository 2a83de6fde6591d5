"""MI355X-native Gated DeltaNet tail replay (Tail-Replay, arXiv 2608.30310).

On a prefix-cache hit of a hybrid model, every GDN recurrent state is rebuilt
by replaying only the last r tokens of the matched prefix from a zero state
(paper Section 3, Eq. 2); the same chunked kernels then continue over the new
suffix and emit its outputs, and a decode-step kernel advances the state by
one generated token.  A whole linear-attention layer (projections,
convolution, norms and gates around the recurrence) can be replayed from the
cached hiddens as well.  Beside these stand the layer's other operators: the
short causal convolution with its history, the selective state space scan, linear
attention with a decay for each head (each for prompts and for single tokens) and
low-rank adapters beside a shared projection; and the group's full-attention
layer: pages and slots from lengths, norm and rotation into the pages, attention
of a batch that shares a prefix.  The work runs in hand-written HIP kernels for gfx950
(the projections through hipBLASLt) behind the C ABI declared in
``include/gdn_tail_replay.h``, ``include/gdn_la_block.h``,
``include/gdn_ssm.h``, ``include/gdn_linear.h``, ``include/gdn_lora.h`` and
``include/gdn_attn.h``; this package is a thin binding
of that library.
"""
from .binding import (GDNError, LIB_PATH, chunk_forward, decode_step, la_block_replay,
                      la_block_stage_names, la_block_workspace_size, load_library, noalloc_scratch_bytes,
                      replay_forward, replay_forward_stage_names, replay_forward_workspace_size,
                      replay_len, stage_names, tail_replay, tail_replay_noalloc, workspace_size)
from .layer_ops import (causal_conv, causal_conv_step, linear_attention, linear_attention_step, lora_add, ssm_scan,
                        ssm_step)
from .attn_ops import extend_pages, prefix_attention, qk_norm_rope

__all__ = ["GDNError", "LIB_PATH", "causal_conv", "causal_conv_step", "chunk_forward", "decode_step", "extend_pages",
           "la_block_replay", "la_block_stage_names", "la_block_workspace_size", "linear_attention",
           "linear_attention_step", "load_library", "lora_add", "noalloc_scratch_bytes", "prefix_attention",
           "qk_norm_rope", "replay_forward", "replay_forward_stage_names", "replay_forward_workspace_size", "replay_len",
           "ssm_scan", "ssm_step", "stage_names", "tail_replay", "tail_replay_noalloc", "workspace_size"]
