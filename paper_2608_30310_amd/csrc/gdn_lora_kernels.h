// Kernels of the low-rank adapters (C ABI in gdn_lora.h).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

constexpr int kLoraThreads = 256;

// u[t, r] = scale x[t] . A[r] in fp32: a wave per (token, r).
__global__ __launch_bounds__(kLoraThreads)
void k_lora_down(int32_t tokens, int32_t n_seqs, const int32_t* __restrict__ cu, const int32_t* __restrict__ adapters,
                 int32_t n_adapters, int32_t K, int32_t R, const uint16_t* __restrict__ x, int64_t ldx,
                 const uint16_t* __restrict__ A, const float* __restrict__ scales, float* __restrict__ u) {
  const int lane = threadIdx.x % kWave;
  const int waves = gridDim.x * (kLoraThreads / kWave);
  for (int64_t i = blockIdx.x * (kLoraThreads / kWave) + threadIdx.x / kWave; i < static_cast<int64_t>(tokens) * R;
       i += waves) {
    const int t = static_cast<int>(i / R), r = static_cast<int>(i % R);
    const int a = adapters[seq_of(cu, n_seqs, t)];
    if (a < 0 || a >= n_adapters) continue;
    float s = 0.0f;
    for (int k = lane; k < K; k += kWave)
      s = fmaf(bf2f(x[t * ldx + k]), bf2f(A[(static_cast<int64_t>(a) * R + r) * K + k]), s);
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) s += __shfl_xor(s, off, kWave);
    if (lane == 0) u[i] = (scales ? scales[a] : 1.0f) * s;
  }
}

// out[t, m] = base[t, m] + u[t] . B[m]: a thread per element.
template <typename T>
__global__ __launch_bounds__(kLoraThreads)
void k_lora_up(int32_t tokens, int32_t n_seqs, const int32_t* __restrict__ cu, const int32_t* __restrict__ adapters,
               int32_t n_adapters, int32_t M, int32_t R, const float* __restrict__ u, const uint16_t* __restrict__ B,
               const T* base, int64_t ldbase, T* out, int64_t ldout) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kLoraThreads + threadIdx.x; i < static_cast<int64_t>(tokens) * M;
       i += static_cast<int64_t>(gridDim.x) * kLoraThreads) {
    const int t = static_cast<int>(i / M), m = static_cast<int>(i % M);
    const int a = adapters[seq_of(cu, n_seqs, t)];
    const float was = load_elt(base, t * ldbase + m);
    float s[1] = {was};
    if (a >= 0 && a < n_adapters)
      for (int r = 0; r < R; ++r)
        s[0] = fmaf(u[static_cast<int64_t>(t) * R + r], bf2f(B[(static_cast<int64_t>(a) * M + m) * R + r]), s[0]);
    store_run<T, 1>(out + t * ldout + m, s);
  }
}

}  // namespace gdn
