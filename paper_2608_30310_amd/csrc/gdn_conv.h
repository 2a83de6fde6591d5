// The short causal convolution (gdn_ssm.h), for packed sequences and for one
// token per sequence.  W multiply-adds per element read and written: HBM bound.
// fp32 arithmetic whatever the element type, one rounding at the store.
//
// Measured, bf16, 4 taps, 8192 channels: 8192 tokens 57 us (4.7 TB/s; a copy of
// as many bytes 49 to 55), 256 single tokens 8.0 us (4.2 TB/s with their
// histories), one single token 2.7 us, a launch.  771 fp32 channels, whose rows
// are not 16-byte aligned, 2700 tokens: 7.5 us.
#pragma once

#include <type_traits>

#include "gdn_varlen.h"

namespace gdn {

constexpr int kConvThreads = 256;
constexpr int kConvLanes = 32;                          // channel groups of a workgroup
constexpr int kConvRows = kConvThreads / kConvLanes;    // token rows of a workgroup
// channels of a thread: 16 bytes of them, or one where rows are not aligned
template <typename T, bool ALIGNED>
constexpr int conv_vec() { return ALIGNED ? 16 / static_cast<int>(sizeof(T)) : 1; }
// tokens of a workgroup's tile when each thread takes tpt of them
constexpr int conv_tile(int tpt) { return kConvRows * tpt; }

// A thread's channels of one row as they lie in memory: 16 bytes, or one element.
// They become floats only where they are used: converted at the load, each row
// waits for its own (8192 tokens 101 us so, 57 kept raw).
template <typename T, int VEC>
struct Chans {
  typedef typename std::conditional<VEC == 1, T, u32x4>::type Raw;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ void clear() {
    if constexpr (VEC == 1) raw = T(0);
    else raw = u32x4{0u, 0u, 0u, 0u};
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (VEC == 1) return load_elt(&raw, 0);
    else return vec_elt<T>(raw, e);
  }
};

// The taps and the bias of a thread's channels.  c0 + VEC <= C for every thread
// that stores; the others take the last channels'.
template <int VEC, int W>
__device__ __forceinline__ void load_taps(const float* __restrict__ w, const float* __restrict__ bias, int c0,
                                          float (&tap)[W][VEC], float (&b)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
#pragma unroll
    for (int j = 0; j < W; ++j) tap[j][e] = w[static_cast<int64_t>(c0 + e) * W + j];
    b[e] = bias ? bias[c0 + e] : 0.0f;
  }
}

template <int VEC, bool SILU>
__device__ __forceinline__ void activate(float (&acc)[VEC]) {
  if constexpr (SILU) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = silu_f(acc[e]);
  }
}

// Workgroup: 32 channel groups x 8 rows of TPT consecutive tokens; a thread
// loads the TPT + W - 1 rows that its tokens need once, all of them before
// anything waits.  blockIdx.x % slabs is its channel slab for good (the taps stay
// in registers), its tiles are the slots from blockIdx.x / slabs in steps of
// gridDim.x / slabs.
// The rows before a sequence and the history after it belong to the sequence's
// first tile, so history_out may be history_in: that workgroup alone touches
// them, and it reads before it writes.
template <typename T, int VEC, int W, int TPT, bool SILU>
__global__ __launch_bounds__(kConvThreads)
void k_causal_conv(int32_t slots, int32_t slabs, int32_t n_seqs, const int32_t* __restrict__ cu, int32_t C,
                   const T* __restrict__ x, int64_t ldx, const float* __restrict__ w, const float* __restrict__ bias,
                   const T* hist_in, T* __restrict__ y, int64_t ldy, T* hist_out) {
  constexpr int H = W - 1;
  constexpr int TILE = conv_tile(TPT);
  typedef Chans<T, VEC> Row;
  const int tid = threadIdx.x;
  const int row = tid / kConvLanes;
  const int slab = blockIdx.x % slabs;
  const int mine = (slab * kConvLanes + tid % kConvLanes) * VEC;
  const bool any = mine < C;              // C is a multiple of VEC
  const int c0 = any ? mine : C - VEC;    // the others load the last channels and store nothing
  float tap[W][VEC], b[VEC];
  load_taps<VEC, W>(w, bias, c0, tap, b);
  const int step = gridDim.x / slabs;
  for (int slot = blockIdx.x / slabs; slot < slots; slot += step) {   // uniform per workgroup
    const int n = slot_seq(cu, n_seqs, slot, TILE);
    const int start = cu[n], len = cu[n + 1] - start;
    const int j = slot - (start / TILE + n);
    if (j > 0 && j * TILE >= len) continue;   // an unused slot
    const int t0 = j * TILE + row * TPT;
    const T* xs = x + static_cast<int64_t>(start) * ldx + c0;
    const int64_t hbase = static_cast<int64_t>(n) * H * C + c0;
    Row u[TPT + H];
    if (len > 0) {
#pragma unroll
      for (int r = 0; r < TPT + H; ++r) u[r].load(xs + static_cast<int64_t>(min(max(t0 - H + r, 0), len - 1)) * ldx);
    }
    if (j == 0) {   // uniform: rows before the sequence, and the history after it
#pragma unroll
      for (int r = 0; r < TPT + H; ++r) {
        const int t = t0 - H + r;
        if (t < 0) {
          if (hist_in) u[r].load(hist_in + hbase + static_cast<int64_t>(H + t) * C);
          else u[r].clear();
        }
      }
      if (hist_out) {
        // rows len .. len + H - 1 of (history | sequence)
        Row h[H];
        if (any && row == 0) {
#pragma unroll
          for (int r = 0; r < H; ++r) {
            const int t = len - H + r;
            if (t >= 0) h[r].load(xs + static_cast<int64_t>(t) * ldx);
            else if (hist_in) h[r].load(hist_in + hbase + static_cast<int64_t>(H + t) * C);
            else h[r].clear();
          }
        }
        __syncthreads();   // every row's history_in is in registers
        if (any && row == 0) {
#pragma unroll
          for (int r = 0; r < H; ++r) h[r].store(hist_out + hbase + static_cast<int64_t>(r) * C);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TPT; ++i) {
      if (!any || t0 + i >= len) continue;
      float acc[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        acc[e] = b[e];
#pragma unroll
        for (int k = 0; k < W; ++k) acc[e] = fmaf(tap[k][e], u[i + k].get(e), acc[e]);
      }
      activate<VEC, SILU>(acc);
      store_run<T, VEC>(y + static_cast<int64_t>(start + t0 + i) * ldy + mine, acc);
    }
  }
}

// One token per sequence: a thread takes VEC channels of the sequences from
// blockIdx.y in steps of gridDim.y, its taps in registers.  It reads its
// history before it writes it, so the two may be one.
template <typename T, int VEC, int W, bool SILU>
__global__ __launch_bounds__(kConvThreads)
void k_causal_conv_step(int32_t n_seqs, int32_t C, const T* __restrict__ x, int64_t ldx, const float* __restrict__ w,
                        const float* __restrict__ bias, const T* hist_in, T* __restrict__ y, int64_t ldy,
                        T* hist_out) {
  constexpr int H = W - 1;
  typedef Chans<T, VEC> Row;
  const int c0 = (blockIdx.x * blockDim.x + threadIdx.x) * VEC;
  if (c0 >= C) return;
  float tap[W][VEC], b[VEC];
  Row u[W];
  const auto fetch = [&](int n) {
    const int64_t hbase = static_cast<int64_t>(n) * H * C + c0;
#pragma unroll
    for (int r = 0; r < H; ++r) {
      if (hist_in) u[r].load(hist_in + hbase + static_cast<int64_t>(r) * C);
      else u[r].clear();
    }
    u[H].load(x + static_cast<int64_t>(n) * ldx + c0);
  };
  fetch(blockIdx.y);   // beside the taps
  load_taps<VEC, W>(w, bias, c0, tap, b);
  for (int n = blockIdx.y; n < n_seqs; n += gridDim.y) {
    if (n != static_cast<int>(blockIdx.y)) fetch(n);
    const int64_t hbase = static_cast<int64_t>(n) * H * C + c0;
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      acc[e] = b[e];
#pragma unroll
      for (int k = 0; k < W; ++k) acc[e] = fmaf(tap[k][e], u[k].get(e), acc[e]);
    }
    activate<VEC, SILU>(acc);
#pragma unroll
    for (int r = 0; r < H; ++r) u[r + 1].store(hist_out + hbase + static_cast<int64_t>(r) * C);
    store_run<T, VEC>(y + static_cast<int64_t>(n) * ldy + c0, acc);
  }
}

}  // namespace gdn
