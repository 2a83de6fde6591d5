// The selective state space scan and its single-token step: validation and
// launches (C ABI in gdn_ssm.h).
#include <hip/hip_runtime.h>

#include <string>

#include "gdn_layer_plan.h"
#include "gdn_plan.h"
#include "gdn_ssm_kernels.h"

namespace gdn {
namespace {

gdn_status sfail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

gdn_status slaunched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return sfail(GDN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return GDN_OK;
}

struct SsmArgs {
  const gdn_ssm_shape* s;
  const int32_t* cu;   // NULL: one token per sequence
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
  hipStream_t stream;
};

template <typename T, int DK, int DV>
gdn_status launch_ssm(const SsmArgs& a) {
  const gdn_ssm_shape& s = *a.s;
  const bool dt_bf16 = s.dt_dtype == GDN_BF16;
  const uint32_t blocks = static_cast<uint32_t>(s.num_seqs) * s.num_heads;
  if (!a.cu) {
    hipLaunchKernelGGL((k_ssm_step<T, DK, DV>), dim3(blocks), dim3(kSsmThreads), 0, a.stream, s.num_heads,
                       s.num_groups, static_cast<const T*>(a.x), s.ld_x, a.dt, dt_bf16, s.ld_dt, a.a_log,
                       static_cast<const T*>(a.B), s.ld_b, static_cast<const T*>(a.C), s.ld_c, a.d_skip, a.dt_bias,
                       a.state_in, static_cast<T*>(a.y), s.ld_y, a.state_out);
    return slaunched("state space step launch");
  }
  hipLaunchKernelGGL((k_ssm_walk<T, DK, DV>), dim3(blocks), dim3(kSsmThreads), 0, a.stream, s.num_heads, s.num_groups,
                     a.cu, static_cast<const T*>(a.x), s.ld_x, a.dt, dt_bf16, s.ld_dt, a.a_log,
                     static_cast<const T*>(a.B), s.ld_b, static_cast<const T*>(a.C), s.ld_c, a.d_skip, a.dt_bias,
                     a.state_in, static_cast<T*>(a.y), s.ld_y, a.state_out);
  return slaunched("state space scan launch");
}

template <typename T>
gdn_status ssm_dims(const SsmArgs& a) {
  if (a.s->d_state == 64) return a.s->head_dim == 64 ? launch_ssm<T, 64, 64>(a) : launch_ssm<T, 64, 128>(a);
  return a.s->head_dim == 64 ? launch_ssm<T, 128, 64>(a) : launch_ssm<T, 128, 128>(a);
}

gdn_status ssm_impl(const SsmArgs& a) {
  const gdn_ssm_shape& s = *a.s;
  if (!a.a_log) return sfail(GDN_ERR_NULL_ARG, "a_log is NULL");
  if (a.tokens > 0 && (!a.x || !a.dt || !a.B || (a.y && !a.C)))
    return sfail(GDN_ERR_NULL_ARG, "x, dt, B (and C where y is given) must be non-NULL");
  const auto misaligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; };
  if (misaligned(a.x) || misaligned(a.B) || (a.y && misaligned(a.C)) || misaligned(a.y) || misaligned(a.state_in) ||
      misaligned(a.state_out))
    return sfail(GDN_ERR_UNSUPPORTED, "x, B, C, y and the states must be 16-byte aligned");
  const int64_t e = s.dtype == GDN_BF16 ? 2 : 4, edt = s.dt_dtype == GDN_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(a.dt) % edt != 0) return sfail(GDN_ERR_UNSUPPORTED, "dt must be aligned to its elements");
  const size_t states = static_cast<size_t>(s.num_seqs) * s.num_heads * s.d_state * s.head_dim * sizeof(float);
  if (a.state_in && a.state_out && a.state_in != a.state_out && overlap(a.state_in, states, a.state_out, states))
    return sfail(GDN_ERR_BAD_SHAPE, "state_out overlaps state_in without being equal");
  if (a.y && a.tokens > 0) {
    const int64_t wy = static_cast<int64_t>(s.num_heads) * s.head_dim * e, wb = static_cast<int64_t>(s.num_groups) * s.d_state * e;
    if (rows_overlap(a.y, wy, s.ld_y * e, a.x, wy, s.ld_x * e, a.tokens) ||
        rows_overlap(a.y, wy, s.ld_y * e, a.B, wb, s.ld_b * e, a.tokens) ||
        rows_overlap(a.y, wy, s.ld_y * e, a.C, wb, s.ld_c * e, a.tokens) ||
        rows_overlap(a.y, wy, s.ld_y * e, a.dt, s.num_heads * edt, s.ld_dt * edt, a.tokens))
      return sfail(GDN_ERR_BAD_SHAPE, "y overlaps an input");
  }
  return s.dtype == GDN_BF16 ? ssm_dims<uint16_t>(a) : ssm_dims<float>(a);
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_ssm_workspace_size(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  if (!bytes) return gdn::sfail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  gdn_status st = gdn::check_ssm(shape, &err);
  int64_t tokens = 0, longest = 0;
  if (st == GDN_OK) st = gdn::check_seqlens(shape->num_seqs, cu_seqlens_host, &tokens, &longest, &err);
  if (st != GDN_OK) return gdn::sfail(st, err);
  *bytes = 0;
  return GDN_OK;
}

gdn_status gdn_ssm_scan(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                        const void* x, const void* dt, const float* a_log, const void* B, const void* C,
                        const float* d_skip, const float* dt_bias, const float* state_in, void* y, float* state_out,
                        void* workspace, size_t workspace_bytes, void* stream) {
  std::string err;
  gdn_status st = gdn::check_ssm(shape, &err);
  int64_t tokens = 0, longest = 0;
  if (st == GDN_OK) st = gdn::check_seqlens(shape->num_seqs, cu_seqlens_host, &tokens, &longest, &err);
  if (st != GDN_OK) return gdn::sfail(st, err);
  if (shape->num_seqs == 0) return GDN_OK;
  if (!cu_seqlens) return gdn::sfail(GDN_ERR_NULL_ARG, "cu_seqlens (device) is NULL");
  if (!y && !state_out) return gdn::sfail(GDN_ERR_NULL_ARG, "y and state_out are both NULL");
  return gdn::ssm_impl({shape, cu_seqlens, tokens, x, dt, a_log, B, C, d_skip, dt_bias, state_in, y, state_out,
                        static_cast<hipStream_t>(stream)});
}

gdn_status gdn_ssm_step(const gdn_ssm_shape* shape, const void* x, const void* dt, const float* a_log, const void* B,
                        const void* C, const float* d_skip, const float* dt_bias, const float* state_in, void* y,
                        float* state_out, void* stream) {
  std::string err;
  const gdn_status st = gdn::check_ssm(shape, &err);
  if (st != GDN_OK) return gdn::sfail(st, err);
  if (shape->num_seqs == 0) return GDN_OK;
  if (!y || !state_out) return gdn::sfail(GDN_ERR_NULL_ARG, "y and state_out must be non-NULL");
  return gdn::ssm_impl({shape, nullptr, shape->num_seqs, x, dt, a_log, B, C, d_skip, dt_bias, state_in, y, state_out,
                        static_cast<hipStream_t>(stream)});
}

}  // extern "C"
