// Device helpers for packed sequences of any length: the sequence of a tile
// slot, element runs of a row, softplus.
#pragma once

#include "gdn_block.h"

namespace gdn {

// Largest n in [0, N) with cu[n] / tile + n <= slot: the sequence whose tiles
// slot `slot` is among.  The wave looks at 64 candidates at a time, so up to 64
// sequences take one load's latency.  Uniform over the wave.
__device__ __forceinline__ int slot_seq(const int32_t* __restrict__ cu, int n_seqs, int slot, int tile) {
  const int lane = threadIdx.x % kWave;
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int at = lo + lane * step;
    const bool below = at < hi && cu[at] / tile + at <= slot;
    const int found = __popcll(__ballot(below));   // lane 0 holds lo, which is below
    lo += (found - 1) * step;
    hi = min(hi, lo + step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// N consecutive elements of a row, by 16-byte accesses where the caller says
// that the run starts at a multiple of 16 bytes (N elements are 16 bytes then),
// else N = 1.
template <typename T, int N>
__device__ __forceinline__ void store_run(T* __restrict__ p, const float (&x)[N]) {
  if constexpr (N == 1) {
    if constexpr (sizeof(T) == 2) *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[0]));   // nearest even, NaN kept
    else *p = x[0];
  } else if constexpr (sizeof(T) == 2) {
    static_assert(N == 8, "16 bytes");
    store8(p, x);
  } else {
    static_assert(N == 4, "16 bytes");
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  }
}

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x| <= 1.  With u the rounded
// 1 + e, log(1 + e) = log(u) e / (u - 1) to within the logarithm's own rounding.
__device__ __forceinline__ float softplus_f(float x) {
  const float e = __builtin_amdgcn_exp2f(-1.44269504088896f * fabsf(x));
  const float u = 1.0f + e, d = u - 1.0f;
  const float l = __builtin_amdgcn_logf(u) * 0.693147180559945f;   // v_log_f32 is base 2
  return fmaxf(x, 0.0f) + (d == 0.0f ? e : l * (e * __builtin_amdgcn_rcpf(d)));
}

// dt is fp32 or has the element type
__device__ __forceinline__ float load_dt(const void* __restrict__ dt, bool bf16, int64_t i) {
  return bf16 ? bf2f(static_cast<const uint16_t*>(dt)[i]) : static_cast<const float*>(dt)[i];
}

}  // namespace gdn
