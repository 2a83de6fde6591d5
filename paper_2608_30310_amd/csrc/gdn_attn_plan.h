// Host-side validation and planning of the full-attention layer's operators
// (gdn_attn.h).  Pure C++ (no HIP), like gdn_plan.h.
#pragma once

#include <cstddef>
#include <cstdint>
#include <string>

#include "gdn_attn.h"
#include "gdn_layer_plan.h"

namespace gdn {

// New tokens of a workgroup of gdn_extend_pages.
constexpr int32_t kPageTokens = 1024;

struct PagesPlan {
  int64_t tokens = 0;
  int64_t slots = 0;    // workgroups: tiles of kPageTokens new tokens, one at least for each sequence
  size_t bytes = 0;     // workspace: three int32 per sequence
};
gdn_status make_pages_plan(const gdn_pages_shape* s, const int32_t* cu, PagesPlan* p, std::string* err);

// k_out, k_cache: given (their fields are looked at); v: v and v_cache are
gdn_status check_qk(const gdn_qk_shape* s, bool k_out, bool k_cache, bool v, std::string* err);

gdn_status check_attn(const gdn_attn_shape* s, std::string* err);

// Rows (one query head of one token, the heads of a K/V head next to each other)
// of a wave, and of a workgroup whose waves take rows of their own.
constexpr int32_t kPlanRows = 32, kPlanTile = 128;
// Keys of a tile of the line that waves share, sequences that it may have, and K/V heads (a
// wave for each at least).
constexpr int32_t kPlanLineTile = 32, kPlanLineSeqs = 1024, kPlanLineHeads = 1024;

// Up to so many partial results of a row a wave joins them by itself.
constexpr int32_t kPlanFewParts = 8;

// How gdn_prefix_attention runs.  Shared items: tiles of all packed rows against
// `shared_splits` pieces of the prefix.  Own items: tiles of a sequence's rows
// against `own_splits` pieces of its own tokens, and against the whole prefix
// before them where there are no shared items.
struct AttnPlan {
  int64_t tokens = 0, longest = 0;
  int32_t groups = 1;        // query heads of a K/V head
  int32_t max_len = 0;       // own tokens of a sequence at most
  int64_t rows = 0;          // tokens * groups
  int32_t shared_splits = 0, shared_chunk = 0;
  int64_t shared_tiles = 0, shared_items = 0;
  int32_t own_tile = kPlanTile, own_splits = 1, own_chunk = 0;
  int64_t own_slots = 0, own_items = 0;
  int32_t shared_wt = kPlanTile / kPlanRows;   // wave tiles of a shared item; 1: it is a wave's
  // few rows a sequence: stream_waves waves from workgroup stream_first on share all
  // sequences' own tokens out in equal parts
  bool stream = false;
  int32_t stream_first = 0, stream_waves = 0;
  int64_t grid = 0;
  bool joined = false;       // items leave partial results, which a second kernel joins
  bool spread = false;       // many of them: its waves share out the parts
  size_t off_ml = 0, off_line = 0;   // workspace: partial outputs, their maxima and sums, the line
  size_t bytes = 0;
};
gdn_status make_attn_plan(const gdn_attn_shape* s, const int32_t* cu, AttnPlan* p, std::string* err);

// Elements from a cache's first to behind its last.
int64_t cache_extent(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int64_t page, int64_t token,
                     int64_t head);
// Whether two caches of the same strides, whose extents may meet, share no byte:
// at some of the strides the windows of the two never meet.
bool caches_apart(const void* pa, const void* pb, int64_t elt, int32_t pages, int32_t page_size, int32_t heads, int32_t dim,
                  int64_t page, int64_t token, int64_t head);

}  // namespace gdn
