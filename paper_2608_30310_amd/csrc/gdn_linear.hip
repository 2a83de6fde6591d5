// Linear attention with a decay for each head: validation and launches (C ABI in
// gdn_linear.h).  The chunked scan and the step are the state space recurrence's,
// with k for B, v for x, q for C and steps that are all the same.
// 32 heads of 128 x 128: 16 sequences of 128 to 2048 tokens 185 us (bound by the longest
// one's chunks in sequence), a token for each of 128 sequences 89 (540 MB, 6.1 TB/s).
#include "gdn_linear.h"

#include <cmath>

#include "gdn_ssm_launch.h"

namespace gdn {
namespace {

// States alone: a segment of one chunk costs the pass that joins the segments more than it
// spares the walk (819 tokens of 32 heads of 128 x 128 24.5 us by ones, 20.7 by twos; 2048 of
// 4 heads 19.6 and 15.7; with outputs 34.2 and 36.0).  No more segments than with outputs,
// whose workspace is enough.
constexpr int64_t kAloneSegment = 2;

gdn_status check_linear(const gdn_linear_shape* s, bool outputs, gdn_ssm_shape* as, std::string* err) {
  const auto bad = [&](const char* what, gdn_status st) {
    *err = what;
    return st;
  };
  if (!s) return bad("shape is NULL", GDN_ERR_NULL_ARG);
  if (s->num_seqs < 0) return bad("num_seqs must be >= 0", GDN_ERR_BAD_SHAPE);
  if (s->num_k_heads < 1 || s->num_v_heads < 1) return bad("head counts must be >= 1", GDN_ERR_BAD_SHAPE);
  if (s->num_v_heads % s->num_k_heads != 0)
    return bad("num_v_heads must be a multiple of num_k_heads", GDN_ERR_BAD_SHAPE);
  if (s->num_v_heads > 65535) return bad("num_v_heads must be <= 65535", GDN_ERR_UNSUPPORTED);
  const auto dim = [](int32_t d) { return d == 64 || d == 128; };
  if (!dim(s->d_k) || !dim(s->d_v)) return bad("d_k and d_v must each be 64 or 128", GDN_ERR_UNSUPPORTED);
  if (s->dtype != GDN_F32 && s->dtype != GDN_BF16) return bad("dtype must be GDN_F32 or GDN_BF16", GDN_ERR_UNSUPPORTED);
  if (!std::isfinite(s->scale)) return bad("scale must be finite", GDN_ERR_BAD_SHAPE);
  const int64_t wk = static_cast<int64_t>(s->num_k_heads) * s->d_k, wv = static_cast<int64_t>(s->num_v_heads) * s->d_v;
  const int64_t vec = s->dtype == GDN_BF16 ? 8 : 4;
  const struct { const char* name; int64_t ld, least; bool used; } rows[] = {
      {"ld_q", s->ld_q, wk, outputs}, {"ld_k", s->ld_k, wk, true}, {"ld_v", s->ld_v, wv, true}, {"ld_o", s->ld_o, wv, outputs}};
  for (const auto& r : rows) {
    if (!r.used) continue;
    if (r.ld < r.least) {
      *err = std::string(r.name) + " must be at least " + std::to_string(r.least);
      return GDN_ERR_BAD_SHAPE;
    }
    if (r.ld > int64_t{1} << 23 || r.ld % vec != 0) {
      *err = std::string(r.name) + " must be a multiple of 16 bytes, at most 2^23 elements";
      return GDN_ERR_UNSUPPORTED;
    }
  }
  *as = {s->num_seqs, s->num_v_heads, s->num_k_heads, s->d_k, s->d_v, s->dtype, GDN_F32, s->ld_v, s->num_v_heads, s->ld_k,
         s->ld_q, s->ld_o};
  return GDN_OK;
}

gdn_status linear_impl(const SsmArgs& a) {
  const gdn_ssm_shape& s = *a.s;
  if (!a.a_log) return sfail(GDN_ERR_NULL_ARG, "g is NULL");
  if (a.tokens > 0 && (!a.x || !a.B || (a.y && !a.C)))
    return sfail(GDN_ERR_NULL_ARG, "k, v (and q where o is given) must be non-NULL");
  const void* q = a.y ? a.C : nullptr;
  for (const void* p : {a.x, a.B, q, static_cast<const void*>(a.y), static_cast<const void*>(a.state_in),
                        static_cast<const void*>(a.state_out)})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
      return sfail(GDN_ERR_UNSUPPORTED, "q, k, v, o and the states must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(a.a_log) % 4 != 0) return sfail(GDN_ERR_UNSUPPORTED, "g must be aligned to its elements");
  const int64_t e = s.dtype == GDN_BF16 ? 2 : 4;
  const size_t states = static_cast<size_t>(s.num_seqs) * s.num_heads * s.d_state * s.head_dim * sizeof(float);
  const size_t ng = s.num_heads * sizeof(float);
  if (a.state_in && a.state_out && a.state_in != a.state_out && overlap(a.state_in, states, a.state_out, states))
    return sfail(GDN_ERR_BAD_SHAPE, "state_out overlaps state_in without being equal");
  if (a.state_out && overlap(a.state_out, states, a.a_log, ng)) return sfail(GDN_ERR_BAD_SHAPE, "state_out overlaps an input");
  if (a.tokens > 0) {
    const int64_t wv = static_cast<int64_t>(s.num_heads) * s.head_dim * e, wk = static_cast<int64_t>(s.num_groups) * s.d_state * e;
    const struct { const void* p; int64_t width, ld; } in[] = {{a.x, wv, s.ld_x * e}, {a.B, wk, s.ld_b * e}, {q, wk, s.ld_c * e}};
    for (const auto& r : in) {
      if (!r.p) continue;
      if (a.y && rows_overlap(a.y, wv, s.ld_y * e, r.p, r.width, r.ld, a.tokens))
        return sfail(GDN_ERR_BAD_SHAPE, "o overlaps an input");
      if (a.state_out && overlap(a.state_out, states, r.p, (a.tokens - 1) * r.ld + r.width))
        return sfail(GDN_ERR_BAD_SHAPE, "state_out overlaps an input");
    }
    const size_t ey = a.y ? (a.tokens - 1) * s.ld_y * e + wv : 0;
    if (a.y && ((a.state_in && overlap(a.state_in, states, a.y, ey)) || (a.state_out && overlap(a.state_out, states, a.y, ey))))
      return sfail(GDN_ERR_BAD_SHAPE, "o overlaps a state");
    if (a.y && overlap(a.y, ey, a.a_log, ng)) return sfail(GDN_ERR_BAD_SHAPE, "o overlaps an input");
  }
  return s.dtype == GDN_BF16 ? ssm_dims<uint16_t, true>(a) : ssm_dims<float, true>(a);
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_linear_attention_workspace_size(const gdn_linear_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  using namespace gdn;
  if (!bytes) return sfail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  SsmPlan p;
  gdn_ssm_shape as;
  gdn_status st = check_linear(shape, false, &as, &err);
  if (st == GDN_OK) st = make_ssm_plan(&as, cu_seqlens_host, &p, &err, false);
  if (st != GDN_OK) return sfail(st, err);
  *bytes = p.bytes;
  return GDN_OK;
}

gdn_status gdn_linear_attention(const gdn_linear_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                                const void* q, const void* k, const void* v, const float* g, const float* state_in, void* o,
                                float* state_out, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace gdn;
  std::string err;
  SsmPlan p;
  gdn_ssm_shape as;
  gdn_status st = check_linear(shape, o != nullptr, &as, &err);
  if (st == GDN_OK) st = make_ssm_plan(&as, cu_seqlens_host, &p, &err, o != nullptr, o ? 1 : kAloneSegment);
  if (st != GDN_OK) return sfail(st, err);
  if (shape->num_seqs == 0 || (p.tokens == 0 && !state_out)) return GDN_OK;
  if (!cu_seqlens) return sfail(GDN_ERR_NULL_ARG, "cu_seqlens (device) is NULL");
  if (!o && !state_out) return sfail(GDN_ERR_NULL_ARG, "o and state_out are both NULL");
  if (p.bytes > 0 && !workspace) return sfail(GDN_ERR_WORKSPACE, "workspace is NULL");
  if (workspace_bytes < p.bytes)
    return sfail(GDN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(p.bytes) + " bytes, got " +
                                        std::to_string(workspace_bytes));
  if (p.bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return sfail(GDN_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return linear_impl({&as, &p, cu_seqlens, p.tokens, v, nullptr, g, k, q, nullptr, nullptr, state_in, o, state_out,
                      static_cast<char*>(workspace), static_cast<hipStream_t>(stream), shape->scale});
}

gdn_status gdn_linear_attention_step(const gdn_linear_shape* shape, const void* q, const void* k, const void* v, const float* g,
                                     const float* state_in, void* o, float* state_out, void* stream) {
  using namespace gdn;
  std::string err;
  gdn_ssm_shape as;
  gdn_status st = check_linear(shape, true, &as, &err);
  if (st == GDN_OK) st = check_ssm(&as, &err);
  if (st != GDN_OK) return sfail(st, err);
  if (shape->num_seqs == 0) return GDN_OK;
  if (!o || !state_out) return sfail(GDN_ERR_NULL_ARG, "o and state_out must be non-NULL");
  return linear_impl({&as, nullptr, nullptr, shape->num_seqs, v, nullptr, g, k, q, nullptr, nullptr, state_in, o, state_out,
                      nullptr, static_cast<hipStream_t>(stream), shape->scale});
}

}  // extern "C"
