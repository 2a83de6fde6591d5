// Kernels of the selective state space recurrence (C ABI in
// gdn_ssm.h).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

constexpr int kSsmThreads = 256;
constexpr int kSsmWaves = kSsmThreads / kWave;

// dt is fp32 or has the element type
__device__ __forceinline__ float load_dt(const void* __restrict__ dt, bool bf16, int64_t i) {
  return bf16 ? bf2f(static_cast<const uint16_t*>(dt)[i]) : static_cast<const float*>(dt)[i];
}

// One step of a token: log alpha and delta.  log alpha is held above -104: e^-104
// rounds to zero in fp32, and sums of it over a chunk stay finite.
__device__ __forceinline__ void step_of(float dt, float dt_bias, float neg_a, float& log_alpha, float& delta) {
  delta = softplus_f(dt + dt_bias);
  log_alpha = fmaxf(neg_a * delta, -104.0f);
}

// A workgroup per (sequence, head) walks the tokens with the state in
// registers: thread t owns the four columns 4 (t % (DV / 4)).. of row part
// t / (DV / 4), as in k_decode.
template <typename T, int DK, int DV>
__global__ __launch_bounds__(kSsmThreads)
void k_ssm_walk(int32_t heads, int32_t groups, const int32_t* __restrict__ cu, const T* __restrict__ x, int64_t ldx,
                const void* __restrict__ dt, bool dt_bf16, int64_t ld_dt, const float* __restrict__ a_log,
                const T* __restrict__ B, int64_t ldb, const T* __restrict__ Cm, int64_t ldc,
                const float* __restrict__ d_skip, const float* __restrict__ dt_bias, const float* state_in,
                T* __restrict__ y, int64_t ldy, float* state_out) {
  constexpr int CQ = DV / 4;
  constexpr int RP = kSsmThreads / CQ;
  constexpr int RPT = DK / RP;
  __shared__ f32x4 red[kSsmWaves][CQ];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lane = tid % kWave;
  const int cq = tid % CQ, rp = tid / CQ;
  const int h = blockIdx.x % heads, n = blockIdx.x / heads;
  const int gh = h / (heads / groups);
  const int64_t sbase = (static_cast<int64_t>(n) * heads + h) * DK * DV + 4 * cq;
  f32x4 m[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i)
    m[i] = state_in ? *reinterpret_cast<const f32x4*>(state_in + sbase + static_cast<int64_t>(rp * RPT + i) * DV)
                    : zero4();
  const float neg_a = -expf(a_log[h]), bias = dt_bias ? dt_bias[h] : 0.0f, skip = d_skip ? d_skip[h] : 0.0f;
  for (int64_t t = cu[n]; t < cu[n + 1]; ++t) {
    float xv[4], bv[RPT], cv[RPT], la, delta;
    step_of(load_dt(dt, dt_bf16, t * ld_dt + h), bias, neg_a, la, delta);
    const float alpha = expf(la);
    load_run<T, 4>(x + t * ldx + h * DV + 4 * cq, xv);
    load_run<T, RPT>(B + t * ldb + gh * DK + rp * RPT, bv);
    if (y) load_run<T, RPT>(Cm + t * ldc + gh * DK + rp * RPT, cv);
    f32x4 p = zero4();
#pragma unroll
    for (int i = 0; i < RPT; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        m[i][c] = fmaf(bv[i], delta * xv[c], alpha * m[i][c]);
        if (y) p[c] = fmaf(cv[i], m[i][c], p[c]);
      }
    if (y) {
      __syncthreads();   // the last token's sums have been read
      const f32x4 o = decode_reduce<CQ>(p, red, lane, wave, cq);
      if (rp == 0) {
#pragma unroll
        for (int c = 0; c < 4; ++c) store_elt(y, t * ldy + h * DV + 4 * cq + c, fmaf(skip, xv[c], o[c]));
      }
    }
  }
  if (state_out) {
#pragma unroll
    for (int i = 0; i < RPT; ++i)
      *reinterpret_cast<f32x4*>(state_out + sbase + static_cast<int64_t>(rp * RPT + i) * DV) = m[i];
  }
}

// One token per sequence: read and write the state once.  HBM bound (8 bytes
// per state element against three multiply-adds); streaming accesses, since a
// layer's state comes back only after every other layer's.
template <typename T, int DK, int DV>
__global__ __launch_bounds__(kSsmThreads)
void k_ssm_step(int32_t heads, int32_t groups, const T* __restrict__ x, int64_t ldx, const void* __restrict__ dt,
                bool dt_bf16, int64_t ld_dt, const float* __restrict__ a_log, const T* __restrict__ B, int64_t ldb,
                const T* __restrict__ Cm, int64_t ldc, const float* __restrict__ d_skip,
                const float* __restrict__ dt_bias, const float* state_in, T* __restrict__ y, int64_t ldy,
                float* state_out) {
  constexpr int CQ = DV / 4;
  constexpr int RP = kSsmThreads / CQ;
  constexpr int RPT = DK / RP;
  __shared__ f32x4 red[kSsmWaves][CQ];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lane = tid % kWave;
  const int cq = tid % CQ, rp = tid / CQ;
  const int h = blockIdx.x % heads, n = blockIdx.x / heads;
  const int gh = h / (heads / groups);
  const int64_t sbase = (static_cast<int64_t>(n) * heads + h) * DK * DV + 4 * cq;
  f32x4 m[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i)
    m[i] = state_in ? __builtin_nontemporal_load(
                          reinterpret_cast<const f32x4*>(state_in + sbase + static_cast<int64_t>(rp * RPT + i) * DV))
                    : zero4();
  float xv[4], bv[RPT], cv[RPT], la, delta;
  load_run<T, 4>(x + n * ldx + h * DV + 4 * cq, xv);
  load_run<T, RPT>(B + n * ldb + gh * DK + rp * RPT, bv);
  load_run<T, RPT>(Cm + n * ldc + gh * DK + rp * RPT, cv);
  step_of(load_dt(dt, dt_bf16, n * ld_dt + h), dt_bias ? dt_bias[h] : 0.0f, -expf(a_log[h]), la, delta);
  const float alpha = expf(la), skip = d_skip ? d_skip[h] : 0.0f;
  f32x4 p = zero4();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      m[i][c] = fmaf(bv[i], delta * xv[c], alpha * m[i][c]);
      p[c] = fmaf(cv[i], m[i][c], p[c]);
    }
    __builtin_nontemporal_store(m[i], reinterpret_cast<f32x4*>(state_out + sbase + static_cast<int64_t>(rp * RPT + i) * DV));
  }
  const f32x4 o = decode_reduce<CQ>(p, red, lane, wave, cq);
  if (rp == 0) {
#pragma unroll
    for (int c = 0; c < 4; ++c) store_elt(y, n * ldy + h * DV + 4 * cq + c, fmaf(skip, xv[c], o[c]));
  }
}

}  // namespace gdn
