// The adapters' call as the layer block makes it (gdn_lora.hip): gdn_lora_add with
// the distance of two adapters in lora_b given, so that a projection of some of
// the rows takes some of B's.
#pragma once

#include <cstddef>
#include <cstdint>

#include "gdn_lora.h"

namespace gdn {

// b_stride: elements between two adapters' lora_b (width x rank where it is whole)
gdn_status lora_run(const gdn_lora_shape* shape, const int32_t* cu_host, const int32_t* cu,
                    const int32_t* adapters_host, const int32_t* adapters, const void* base, const void* x,
                    const void* lora_a, const void* lora_b, int64_t b_stride, const float* scales, void* out,
                    void* workspace, size_t workspace_bytes, void* stream);

}  // namespace gdn
