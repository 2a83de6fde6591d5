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

// cached: a cache is given (its fields are looked at); k_out, v: k_out, v and v_cache are given
gdn_status check_qk(const gdn_qk_shape* s, bool k_out, bool k_cache, bool v, std::string* err);

gdn_status check_attn(const gdn_attn_shape* s, std::string* err);

struct AttnPlan {
  int64_t tokens = 0, longest = 0;
  int32_t max_len = 0;   // own tokens of a sequence at most
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
