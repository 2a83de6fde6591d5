// The state space recurrence for one token per sequence (C ABI in gdn_ssm.h).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

constexpr int kSsmThreads = 256;
constexpr int kSsmWaves = kSsmThreads / kWave;

// One token per sequence: read and write the state once.  HBM bound (8 bytes
// per state element against three multiply-adds); streaming accesses, since a
// layer's state comes back only after every other layer's.  A workgroup takes a
// head of a sequence, a thread four neighbouring columns of DK DV / 1024 rows,
// so that all its loads are in flight together.  64 heads of 64 x 128: 128
// sequences 83 us (539 MB, 6.5 TB/s, part of the state still in the last-level
// cache; a copy of as many bytes 99 to 110), one sequence 3.9 us.
// FIXED: the same for linear attention with a decay for each head (gdn_linear.h):
// delta = 1, a_log is log alpha, the output is scaled.
template <typename T, int DK, int DV, bool FIXED = false>
__global__ __launch_bounds__(kSsmThreads)
void k_ssm_step(int32_t heads, int32_t groups, const T* __restrict__ x, int64_t ldx, const void* __restrict__ dt,
                bool dt_bf16, int64_t ld_dt, const float* __restrict__ a_log, const T* __restrict__ B, int64_t ldb,
                const T* __restrict__ Cm, int64_t ldc, const float* __restrict__ d_skip,
                const float* __restrict__ dt_bias, const float* state_in, T* __restrict__ y, int64_t ldy,
                float* state_out, float scale) {
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
  float xv[4], bv[RPT], cv[RPT];
  load_run<T, 4>(x + n * ldx + h * DV + 4 * cq, xv);
  load_run<T, RPT>(B + n * ldb + gh * DK + rp * RPT, bv);
  load_run<T, RPT>(Cm + n * ldc + gh * DK + rp * RPT, cv);
  const float delta = FIXED ? 1.0f : softplus_f(load_dt(dt, dt_bf16, n * ld_dt + h) + (dt_bias ? dt_bias[h] : 0.0f));
  const float alpha = expf(FIXED ? a_log[h] : -expf(a_log[h]) * delta), skip = !FIXED && d_skip ? d_skip[h] : 0.0f;
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
    for (int c = 0; c < 4; ++c) store_elt(y, n * ldy + h * DV + 4 * cq + c, FIXED ? scale * o[c] : fmaf(skip, xv[c], o[c]));
  }
}

}  // namespace gdn
