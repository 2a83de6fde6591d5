// Attention over a shared prefix and own pages: validation and launches (C ABI
// in gdn_attn.h).
#include "gdn_attn_kernels.h"

#include <string>

#include "gdn_attn_plan.h"
#include "gdn_plan.h"

namespace gdn {
namespace {

gdn_status afail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

template <typename T, int D>
gdn_status launch_attn(const AttnArgs& a, hipStream_t stream) {
  const int64_t units = static_cast<int64_t>(a.tokens) * a.heads, nw = kAttnThreads / kWave;
  hipLaunchKernelGGL((k_attn<T, D>), dim3(static_cast<uint32_t>((units + nw - 1) / nw)), dim3(kAttnThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return afail(GDN_ERR_HIP, std::string("attention launch: ") + hipGetErrorString(e));
  return GDN_OK;
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_prefix_attention_workspace_size(const gdn_attn_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  if (!bytes) return gdn::afail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  gdn::AttnPlan p;
  const gdn_status st = gdn::make_attn_plan(shape, cu_seqlens_host, &p, &err);
  if (st != GDN_OK) return gdn::afail(st, err);
  *bytes = p.bytes;
  return GDN_OK;
}

gdn_status gdn_prefix_attention(const gdn_attn_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                                const void* q, const void* k_cache, const void* v_cache, const int32_t* table,
                                const int32_t* lens, const int32_t* prefix_pages, void* out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  using namespace gdn;
  std::string err;
  AttnPlan p;
  const gdn_status st = make_attn_plan(shape, cu_seqlens_host, &p, &err);
  if (st != GDN_OK) return afail(st, err);
  const gdn_attn_shape& s = *shape;
  if (s.num_seqs == 0 || p.tokens == 0) return GDN_OK;
  if (!cu_seqlens || !q || !k_cache || !v_cache || !table || !lens || !out)
    return afail(GDN_ERR_NULL_ARG, "cu_seqlens, q, the caches, table, lens and out must be non-NULL");
  if (s.prefix_len > 0 && !prefix_pages) return afail(GDN_ERR_NULL_ARG, "prefix_pages is NULL");
  for (const void* x : {q, k_cache, v_cache, static_cast<const void*>(out)})
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0) return afail(GDN_ERR_UNSUPPORTED, "q, out and the caches must be 16-byte aligned");
  for (const int32_t* x : {cu_seqlens, table, lens, prefix_pages})
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0)
      return afail(GDN_ERR_UNSUPPORTED, "cu_seqlens, table, lens and prefix_pages must be aligned to their elements");
  const int64_t e = s.dtype == GDN_BF16 ? 2 : 4, w = s.num_heads * static_cast<int64_t>(s.head_dim) * e;
  if (rows_overlap(out, w, s.ld_out * e, q, w, s.ld_q * e, p.tokens)) return afail(GDN_ERR_BAD_SHAPE, "out overlaps q");
  const size_t on = static_cast<size_t>((p.tokens - 1) * s.ld_out * e + w), i4 = sizeof(int32_t);
  const struct { const void* p; int64_t n; const char* name; } in[] = {
      {k_cache, e * cache_extent(s.num_pages, s.page_size, s.num_kv_heads, s.head_dim, s.k_page, s.k_token, s.k_head), "k_cache"},
      {v_cache, e * cache_extent(s.num_pages, s.page_size, s.num_kv_heads, s.head_dim, s.v_page, s.v_token, s.v_head), "v_cache"},
      {table, static_cast<int64_t>(i4) * s.num_seqs * s.table_width, "table"}, {lens, static_cast<int64_t>(i4) * s.num_seqs, "lens"},
      {prefix_pages, static_cast<int64_t>(i4) * ((static_cast<int64_t>(s.prefix_len) + s.page_size - 1) / s.page_size), "prefix_pages"}};
  for (const auto& r : in)
    if (r.p && overlap(out, on, r.p, static_cast<size_t>(r.n))) return afail(GDN_ERR_BAD_SHAPE, std::string("out overlaps ") + r.name);
  if (p.bytes > 0 && !workspace) return afail(GDN_ERR_WORKSPACE, "workspace is NULL");
  if (workspace_bytes < p.bytes)
    return afail(GDN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(p.bytes) + " bytes, got " +
                                        std::to_string(workspace_bytes));
  if (p.bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return afail(GDN_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const AttnArgs a{s.num_seqs, s.num_heads, s.num_kv_heads, s.num_pages, s.page_size, s.table_width, s.prefix_len, p.max_len,
                   static_cast<int32_t>(p.tokens), s.scale, cu_seqlens, table, lens, prefix_pages, q, k_cache, v_cache, out,
                   s.ld_q, s.ld_out, s.k_page, s.k_token, s.k_head, s.v_page, s.v_token, s.v_head};
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  if (s.dtype == GDN_BF16) return s.head_dim == 64 ? launch_attn<uint16_t, 64>(a, hs) : launch_attn<uint16_t, 128>(a, hs);
  return s.head_dim == 64 ? launch_attn<float, 64>(a, hs) : launch_attn<float, 128>(a, hs);
}

}  // extern "C"
