// Launches of the chunked scan and its single-token step, of the state space
// recurrence (gdn_ssm.h) and, with FIXED, of linear attention (gdn_linear.h).
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "gdn_layer_plan.h"
#include "gdn_plan.h"
#include "gdn_ssm_scan.h"
#include "gdn_ssm_step.h"

namespace gdn {
namespace {

inline gdn_status sfail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

inline gdn_status slaunched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return sfail(GDN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return GDN_OK;
}

struct SsmArgs {
  const gdn_ssm_shape* s;
  const SsmPlan* p;   // NULL: one token per sequence
  const int32_t* cu;
  int64_t tokens;
  const void* x;
  const void* dt;
  const float* a_log;
  const void* B;
  const void* C;
  const float* d_skip;
  const float* dt_bias;
  const float* state_in;
  void* y;
  float* state_out;
  char* ws;
  hipStream_t stream;
  float scale = 1.0f;   // of the outputs (FIXED)
};

template <typename T, int DK, int DV, bool FIXED>
gdn_status launch_step(const SsmArgs& a) {
  const gdn_ssm_shape& s = *a.s;
  hipLaunchKernelGGL((k_ssm_step<T, DK, DV, FIXED>), dim3(static_cast<uint32_t>(s.num_seqs) * s.num_heads), dim3(kSsmThreads),
                     0, a.stream, s.num_heads, s.num_groups, static_cast<const T*>(a.x), s.ld_x, a.dt,
                     s.dt_dtype == GDN_BF16, s.ld_dt, a.a_log, static_cast<const T*>(a.B), s.ld_b,
                     static_cast<const T*>(a.C), s.ld_c, a.d_skip, a.dt_bias, a.state_in, static_cast<T*>(a.y), s.ld_y,
                     a.state_out, a.scale);
  return slaunched(FIXED ? "linear attention step launch" : "state space step launch");
}

template <typename T, int DK, int DV, int CT, int NW, bool FIXED>
gdn_status launch_scan(const SsmArgs& a) {
  const gdn_ssm_shape& s = *a.s;
  const SsmPlan& p = *a.p;
  SsmScanArgs k{s.num_seqs, s.num_heads, s.num_groups, p.seg_tokens, a.scale, p.ordered, a.cu, a.x, a.dt, a.B, a.C,
                s.ld_x, s.ld_dt, s.ld_b, s.ld_c, s.ld_y, s.dt_dtype == GDN_BF16, a.a_log, a.d_skip, a.dt_bias,
                a.state_in, a.y, a.state_out, reinterpret_cast<f32x4*>(a.ws),
                reinterpret_cast<float*>(a.ws + p.off_decay)};
  const dim3 grid(static_cast<uint32_t>(p.slots * (s.num_heads / p.heads_per_group))), block(NW * kWave);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, a.stream, k); };
  if (p.seg_tokens == 0) {
    if (a.y) run(k_ssm_scan<T, DK, DV, CT, NW, SsmMode::kWhole, true, FIXED>);
    else run(k_ssm_scan<T, DK, DV, CT, NW, SsmMode::kWhole, false, FIXED>);
    return slaunched(FIXED ? "linear attention launch" : "state space scan launch");
  }
  run(k_ssm_scan<T, DK, DV, CT, NW, SsmMode::kLocal, false, FIXED>);
  const int64_t vecs = static_cast<int64_t>(s.num_seqs) * s.num_heads * DK * DV / 4;
  const dim3 jgrid(static_cast<uint32_t>((vecs + 255) / 256));
  if (a.y) {
    hipLaunchKernelGGL((k_ssm_join<DK, DV, CT, NW, true>), jgrid, dim3(256), 0, a.stream, k);
    run(k_ssm_scan<T, DK, DV, CT, NW, SsmMode::kJoined, true, FIXED>);
  } else {
    hipLaunchKernelGGL((k_ssm_join<DK, DV, CT, NW, false>), jgrid, dim3(256), 0, a.stream, k);
  }
  return slaunched(FIXED ? "linear attention launch" : "state space scan launch");
}

template <typename T, int DK, int DV, bool FIXED>
gdn_status launch_ssm(const SsmArgs& a) {
  if (!a.p) return launch_step<T, DK, DV, FIXED>(a);
  constexpr int CT = 2, WPH = DV / (16 * CT);   // waves of a head
  constexpr int share = (sizeof(T) == 2 ? kSsmCols : kSsmColsF32) / DV;
  const int heads = a.p->heads_per_group;
  if constexpr (share >= 4)
    if (heads == 4) return launch_scan<T, DK, DV, CT, 4 * WPH, FIXED>(a);
  if constexpr (share >= 2)
    if (heads == 2) return launch_scan<T, DK, DV, CT, 2 * WPH, FIXED>(a);
  return launch_scan<T, DK, DV, CT, WPH, FIXED>(a);
}

template <typename T, bool FIXED>
gdn_status ssm_dims(const SsmArgs& a) {
  if (a.s->d_state == 64) return a.s->head_dim == 64 ? launch_ssm<T, 64, 64, FIXED>(a) : launch_ssm<T, 64, 128, FIXED>(a);
  return a.s->head_dim == 64 ? launch_ssm<T, 128, 64, FIXED>(a) : launch_ssm<T, 128, 128, FIXED>(a);
}

}  // namespace
}  // namespace gdn
