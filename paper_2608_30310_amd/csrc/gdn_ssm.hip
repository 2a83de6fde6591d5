// The selective state space scan and its single-token step: validation and
// launches (C ABI in gdn_ssm.h).
#include "gdn_ssm_launch.h"

namespace gdn {
namespace {

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
  if (a.tokens > 0) {
    const int64_t wy = static_cast<int64_t>(s.num_heads) * s.head_dim * e, wb = static_cast<int64_t>(s.num_groups) * s.d_state * e;
    const struct { const void* p; int64_t width, ld; } in[] = {
        {a.x, wy, s.ld_x * e}, {a.B, wb, s.ld_b * e}, {a.y ? a.C : nullptr, wb, s.ld_c * e}, {a.dt, s.num_heads * edt, s.ld_dt * edt}};
    for (const auto& r : in) {
      if (!r.p) continue;
      if (a.y && rows_overlap(a.y, wy, s.ld_y * e, r.p, r.width, r.ld, a.tokens))
        return sfail(GDN_ERR_BAD_SHAPE, "y overlaps an input");
      if (a.state_out && overlap(a.state_out, states, r.p, (a.tokens - 1) * r.ld + r.width))
        return sfail(GDN_ERR_BAD_SHAPE, "state_out overlaps an input");
    }
    const size_t ey = (a.tokens - 1) * s.ld_y * e + wy;
    if (a.y && ((a.state_in && overlap(a.state_in, states, a.y, ey)) || (a.state_out && overlap(a.state_out, states, a.y, ey))))
      return sfail(GDN_ERR_BAD_SHAPE, "y overlaps a state");
  }
  return s.dtype == GDN_BF16 ? ssm_dims<uint16_t, false>(a) : ssm_dims<float, false>(a);
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_ssm_workspace_size(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  if (!bytes) return gdn::sfail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  gdn::SsmPlan p;
  const gdn_status st = gdn::make_ssm_plan(shape, cu_seqlens_host, &p, &err, false);
  if (st != GDN_OK) return gdn::sfail(st, err);
  *bytes = p.bytes;
  return GDN_OK;
}

gdn_status gdn_ssm_scan(const gdn_ssm_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                        const void* x, const void* dt, const float* a_log, const void* B, const void* C,
                        const float* d_skip, const float* dt_bias, const float* state_in, void* y, float* state_out,
                        void* workspace, size_t workspace_bytes, void* stream) {
  std::string err;
  gdn::SsmPlan p;
  const gdn_status st = gdn::make_ssm_plan(shape, cu_seqlens_host, &p, &err, y != nullptr);
  if (st != GDN_OK) return gdn::sfail(st, err);
  if (shape->num_seqs == 0 || (p.tokens == 0 && !state_out)) return GDN_OK;
  if (!cu_seqlens) return gdn::sfail(GDN_ERR_NULL_ARG, "cu_seqlens (device) is NULL");
  if (!y && !state_out) return gdn::sfail(GDN_ERR_NULL_ARG, "y and state_out are both NULL");
  if (p.bytes > 0 && !workspace) return gdn::sfail(GDN_ERR_WORKSPACE, "workspace is NULL");
  if (workspace_bytes < p.bytes)
    return gdn::sfail(GDN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(p.bytes) + " bytes, got " +
                                             std::to_string(workspace_bytes));
  if (p.bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % gdn::kAlign != 0)
    return gdn::sfail(GDN_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return gdn::ssm_impl({shape, &p, cu_seqlens, p.tokens, x, dt, a_log, B, C, d_skip, dt_bias, state_in, y, state_out,
                        static_cast<char*>(workspace), static_cast<hipStream_t>(stream)});
}

gdn_status gdn_ssm_step(const gdn_ssm_shape* shape, const void* x, const void* dt, const float* a_log, const void* B,
                        const void* C, const float* d_skip, const float* dt_bias, const float* state_in, void* y,
                        float* state_out, void* stream) {
  std::string err;
  const gdn_status st = gdn::check_ssm(shape, &err);
  if (st != GDN_OK) return gdn::sfail(st, err);
  if (shape->num_seqs == 0) return GDN_OK;
  if (!y || !state_out) return gdn::sfail(GDN_ERR_NULL_ARG, "y and state_out must be non-NULL");
  return gdn::ssm_impl({shape, nullptr, nullptr, shape->num_seqs, x, dt, a_log, B, C, d_skip, dt_bias, state_in, y,
                        state_out, nullptr, static_cast<hipStream_t>(stream)});
}

}  // extern "C"
