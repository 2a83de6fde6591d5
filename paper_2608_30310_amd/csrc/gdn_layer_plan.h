// Host-side validation and planning of the recurrent layer's other operators
// (gdn_ssm.h, gdn_lora.h).  Pure C++ (no HIP), like gdn_plan.h.
#pragma once

#include <cstddef>
#include <cstdint>
#include <string>

#include "gdn_lora.h"
#include "gdn_ssm.h"

namespace gdn {

// State columns of a workgroup of the state space scan (bf16, fp32), where a B/C
// group has that many heads to share them; fewer heads otherwise, and where
// make_ssm_plan says so.  bf16, 256 columns (one workgroup on a CU) and 128 (two):
// 16 sequences of 2048 tokens, 32 heads of 128 x 128, 251 and 354 us; one of 8192,
// 64 heads of 64 x 128, 105 and 124.
constexpr int32_t kSsmCols = 256, kSsmColsF32 = 128;
// Sequences that the scan's workgroups rank by themselves, one a lane.
constexpr int32_t kSsmOrdered = 64;

// Packed sequences cut into tiles of `tile` tokens, each sequence from its own
// start: tile j of sequence n is slot cu[n] / tile + n + j.  The map is
// injective and every sequence has a slot of its own, the empty ones too; at
// most N slots stay unused.  The kernels find a slot's sequence from cu alone.
inline int64_t tile_slots(int64_t tokens, int64_t seqs, int64_t tile) { return seqs > 0 ? tokens / tile + seqs : 0; }

// Validates the host copy of the offsets; *tokens = cu[N], *longest = the
// longest sequence.
gdn_status check_seqlens(int32_t n, const int32_t* cu, int64_t* tokens, int64_t* longest, std::string* err);

gdn_status check_conv(const gdn_conv_shape* s, std::string* err);
// outputs: y is given (ld_c and ld_y are not looked at otherwise)
gdn_status check_ssm(const gdn_ssm_shape* s, std::string* err, bool outputs = true);

// How gdn_ssm_scan runs: which heads share a workgroup and whether sequences
// are worked on in segments.
struct SsmPlan {
  int64_t tokens = 0, longest = 0;
  int32_t heads_per_group = 1;   // heads of a workgroup
  int32_t seg_tokens = 0;        // 0: whole sequences
  bool ordered = false;          // whole sequences, more than the chip holds: the longest first
  int64_t slots = 0;             // segments (an empty sequence has one), or sequences
  size_t off_decay = 0;          // workspace: states [slots, H, d_state, head_dim], then decays [slots, H]
  size_t bytes = 0;
};
gdn_status make_ssm_plan(const gdn_ssm_shape* s, const int32_t* cu, SsmPlan* p, std::string* err, bool outputs = true,
                         int64_t least_segment = 1);   // chunks of a segment at least

gdn_status check_lora(const gdn_lora_shape* s, std::string* err);

struct LoraPlan {
  int64_t tokens = 0;
  // tokens of a tile of the first and of the second product (32, 64 in the second
  // where there are many, 16 in both where there are few) and their slots
  int32_t down_tile = 0, up_tile = 0;
  int64_t down_slots = 0, up_slots = 0;
  int32_t parts = 1;   // pieces of the first product's contraction over K
  size_t bytes = 0;          // workspace: partial x A^T, fp32 [parts, tokens, rank]
};
gdn_status make_lora_plan(const gdn_lora_shape* s, const int32_t* cu, LoraPlan* p, std::string* err);

// Two row-strided regions of `rows` rows: a starts at pa, has wa bytes in each
// row and lda bytes between rows.  False only where no byte is in both: their
// extents do not meet, or the strides are equal and the rows' windows never meet.
bool rows_overlap(const void* pa, int64_t wa, int64_t lda, const void* pb, int64_t wb, int64_t ldb, int64_t rows);
// Two flat regions.
bool overlap(const void* pa, size_t na, const void* pb, size_t nb);

}  // namespace gdn
