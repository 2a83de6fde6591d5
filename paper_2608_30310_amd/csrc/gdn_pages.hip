// Pages and slots from lengths, norm and rotation into pages: validation and
// launches (C ABI in gdn_attn.h).
#include "gdn_pages.h"

#include <string>

#include "gdn_attn_plan.h"
#include "gdn_plan.h"

namespace gdn {
namespace {

gdn_status pfail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

gdn_status plaunched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return pfail(GDN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return GDN_OK;
}

struct Region {
  const void* p;
  int64_t width, ld, rows;   // bytes of a row, between rows, and rows
  size_t bytes() const { return rows > 0 ? static_cast<size_t>((rows - 1) * ld + width) : 0; }
};

bool meet(const Region& a, const Region& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
  if (a.rows == b.rows && a.rows > 1) return rows_overlap(a.p, a.width, a.ld, b.p, b.width, b.ld, a.rows);
  return overlap(a.p, a.bytes(), b.p, b.bytes());
}

template <typename T, int D, int R>
gdn_status launch_qk_rows(const QkArgs& a, bool interleaved, hipStream_t stream) {
  constexpr int rows = R * kWave / (D / 8);   // of a wave
  const uint32_t chunks = static_cast<uint32_t>((a.heads + (a.v ? 2 : 1) * a.kv_heads + rows - 1) / rows);
  const dim3 grid(static_cast<uint32_t>((static_cast<int64_t>(a.tokens) * chunks + kQkWaves - 1) / kQkWaves));
  if (interleaved) hipLaunchKernelGGL((k_qk_norm_rope<T, D, true, R>), grid, dim3(kQkThreads), 0, stream, a, chunks);
  else hipLaunchKernelGGL((k_qk_norm_rope<T, D, false, R>), grid, dim3(kQkThreads), 0, stream, a, chunks);
  return plaunched("norm and rotation launch");
}

// With few tokens every row gets lanes of its own, with many a wave keeps a token's
// cosines over its rows.
template <typename T, int D>
gdn_status launch_qk(const QkArgs& a, bool interleaved, hipStream_t stream) {
  const int64_t waves = static_cast<int64_t>(a.tokens) * (a.heads + (a.v ? 2 : 1) * a.kv_heads) / (kWave / (D / 8));
  return waves < kQkManyWaves ? launch_qk_rows<T, D, 1>(a, interleaved, stream) : launch_qk_rows<T, D, 4>(a, interleaved, stream);
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_extend_pages_workspace_size(const gdn_pages_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  if (!bytes) return gdn::pfail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  gdn::PagesPlan p;
  const gdn_status st = gdn::make_pages_plan(shape, cu_seqlens_host, &p, &err);
  if (st != GDN_OK) return gdn::pfail(st, err);
  *bytes = p.bytes;
  return GDN_OK;
}

gdn_status gdn_extend_pages(const gdn_pages_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                            const int32_t* table_in, const int32_t* lens_in, const int32_t* free_pages,
                            const int32_t* taken_in, int32_t* table_out, int32_t* lens_out, int32_t* taken_out,
                            int32_t* slots, int32_t* positions, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace gdn;
  std::string err;
  PagesPlan p;
  const gdn_status st = make_pages_plan(shape, cu_seqlens_host, &p, &err);
  if (st != GDN_OK) return pfail(st, err);
  const gdn_pages_shape& s = *shape;
  if (!taken_out) return pfail(GDN_ERR_NULL_ARG, "taken_out is NULL");
  if (s.num_seqs > 0 && (!cu_seqlens || !table_in || !lens_in || !table_out || !lens_out))
    return pfail(GDN_ERR_NULL_ARG, "cu_seqlens, the tables and the lengths must be non-NULL");
  if (s.num_free > 0 && !free_pages) return pfail(GDN_ERR_NULL_ARG, "free_pages is NULL");
  if (p.tokens > 0 && (!slots || !positions)) return pfail(GDN_ERR_NULL_ARG, "slots and positions must be non-NULL");
  const size_t e = sizeof(int32_t), table = e * s.num_seqs * s.table_width, lens = e * s.num_seqs, toks = e * p.tokens;
  const struct { const void* p; size_t n; const char* name; } in[] = {
      {table_in, table, "table_in"}, {lens_in, lens, "lens_in"}, {taken_in, e, "taken_in"},
      {free_pages, e * s.num_free, "free_pages"}, {cu_seqlens, lens + e, "cu_seqlens"}},
      out[] = {{table_out, table, "table_out"}, {lens_out, lens, "lens_out"}, {taken_out, e, "taken_out"},
               {slots, toks, "slots"}, {positions, toks, "positions"}};
  for (const auto& r : in)
    if (reinterpret_cast<uintptr_t>(r.p) % e != 0) return pfail(GDN_ERR_UNSUPPORTED, std::string(r.name) + " must be aligned to its elements");
  for (int i = 0; i < 5; ++i) {
    const auto& o = out[i];
    if (reinterpret_cast<uintptr_t>(o.p) % e != 0) return pfail(GDN_ERR_UNSUPPORTED, std::string(o.name) + " must be aligned to its elements");
    if (!o.p) continue;
    for (int j = 0; j < 5; ++j) {
      if (in[j].p && !(i == j && i < 3 && o.p == in[j].p) && overlap(o.p, o.n, in[j].p, in[j].n))
        return pfail(GDN_ERR_BAD_SHAPE, std::string(o.name) + " overlaps " + in[j].name);
      if (j < i && out[j].p && overlap(o.p, o.n, out[j].p, out[j].n))
        return pfail(GDN_ERR_BAD_SHAPE, std::string(o.name) + " overlaps " + out[j].name);
    }
  }
  if (p.bytes > 0 && !workspace) return pfail(GDN_ERR_WORKSPACE, "workspace is NULL");
  if (workspace_bytes < p.bytes)
    return pfail(GDN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(p.bytes) + " bytes, got " +
                                        std::to_string(workspace_bytes));
  if (p.bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return pfail(GDN_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  int32_t* ws = static_cast<int32_t*>(workspace);
  const int64_t n = s.num_seqs;
  const PagesArgs a{s.num_seqs, s.table_width, s.page_size, s.num_free, s.first, cu_seqlens, table_in, lens_in, free_pages,
                    taken_in, table_out, lens_out, taken_out, slots, positions, ws, ws + n, ws + 2 * n};
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  const dim3 fill(static_cast<uint32_t>(p.slots));
  if (n > 0 && n <= kPagesFew && lens_out != lens_in && taken_out != taken_in) {
    hipLaunchKernelGGL((k_pages_fill<kPageTokens, false>), fill, dim3(kPagesThreads), 0, hs, a);
  } else {
    hipLaunchKernelGGL(k_pages_plan, dim3(1), dim3(kPagesPlanThreads), 0, hs, a);
    if (n > 0) hipLaunchKernelGGL((k_pages_fill<kPageTokens, true>), fill, dim3(kPagesThreads), 0, hs, a);
  }
  return plaunched("pages launch");
}

gdn_status gdn_qk_norm_rope(const gdn_qk_shape* shape, const void* q, const void* k, const void* v, const int32_t* positions,
                            const float* cos_sin, const float* q_weight, const float* k_weight, const int32_t* slots,
                            void* q_out, void* k_out, void* k_cache, void* v_cache, void* stream) {
  using namespace gdn;
  std::string err;
  const gdn_status st = check_qk(shape, k_out != nullptr, k_cache != nullptr, v_cache != nullptr, &err);
  if (st != GDN_OK) return pfail(st, err);
  const gdn_qk_shape& s = *shape;
  if (s.num_tokens == 0) return GDN_OK;
  if (!q || !k || !positions || !cos_sin || !q_out) return pfail(GDN_ERR_NULL_ARG, "q, k, positions, cos_sin and q_out must be non-NULL");
  if (!k_out && !k_cache) return pfail(GDN_ERR_NULL_ARG, "k_out and k_cache are both NULL");
  if (!v != !v_cache) return pfail(GDN_ERR_NULL_ARG, "v and v_cache go together");
  if (v && !k_cache) return pfail(GDN_ERR_NULL_ARG, "v_cache is given without k_cache");
  if (k_cache && !slots) return pfail(GDN_ERR_NULL_ARG, "slots is NULL");
  if (!q_weight != !k_weight) return pfail(GDN_ERR_NULL_ARG, "q_weight and k_weight go together");
  for (const void* p : {q, k, v, static_cast<const void*>(cos_sin), static_cast<const void*>(q_weight),
                        static_cast<const void*>(k_weight), static_cast<const void*>(q_out), static_cast<const void*>(k_out),
                        static_cast<const void*>(k_cache), static_cast<const void*>(v_cache)})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
      return pfail(GDN_ERR_UNSUPPORTED, "q, k, v, cos_sin, the weights, the outputs and the caches must be 16-byte aligned");
  for (const void* p : {static_cast<const void*>(positions), static_cast<const void*>(slots)})
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return pfail(GDN_ERR_UNSUPPORTED, "positions and slots must be aligned to their elements");
  const int64_t e = s.dtype == GDN_BF16 ? 2 : 4, D = s.head_dim, T = s.num_tokens;
  const int64_t wq = s.num_heads * D * e, wk = s.num_kv_heads * D * e;
  const auto cache = [&](const void* p, int64_t pg, int64_t tk, int64_t hd) {
    const int64_t n = p ? e * cache_extent(s.num_pages, s.page_size, s.num_kv_heads, s.head_dim, pg, tk, hd) : 0;
    return Region{p, n, n, p ? 1 : 0};
  };
  const Region in[] = {{q, wq, s.ld_q * e, T}, {k, wk, s.ld_k * e, T}, {v, wk, s.ld_v * e, v ? T : 0},
                       {positions, 4 * T, 4 * T, 1}, {slots, 4 * T, 4 * T, k_cache ? 1 : 0},
                       {cos_sin, 4 * int64_t{s.rotary_dim} * s.num_positions, 0, 1},
                       {q_weight, 4 * D, 0, q_weight ? 1 : 0}, {k_weight, 4 * D, 0, k_weight ? 1 : 0}};
  const Region kc = cache(k_cache, s.k_page, s.k_token, s.k_head), vc = cache(v_cache, s.v_page, s.v_token, s.v_head);
  const Region out[] = {{q_out, wq, s.ld_q_out * e, T}, {k_out, wk, s.ld_k_out * e, k_out ? T : 0}, kc, vc};
  const char* names[] = {"q_out", "k_out", "k_cache", "v_cache"};
  const auto apart = [&] {   // keys and values of one allocation, in turns
    return s.k_page == s.v_page && s.k_token == s.v_token && s.k_head == s.v_head &&
           caches_apart(k_cache, v_cache, e, s.num_pages, s.page_size, s.num_kv_heads, s.head_dim, s.k_page, s.k_token, s.k_head);
  };
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 8; ++j) {
      const bool same = (i == 0 && j == 0 && q_out == q && s.ld_q_out == s.ld_q) || (i == 1 && j == 1 && k_out == k && s.ld_k_out == s.ld_k);
      if (!same && meet(out[i], in[j])) return pfail(GDN_ERR_BAD_SHAPE, std::string(names[i]) + " overlaps an input");
    }
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j]) && !(i == 3 && j == 2 && apart()))
        return pfail(GDN_ERR_BAD_SHAPE, std::string(names[i]) + " overlaps " + names[j]);
  }
  const QkArgs a{s.num_tokens, s.num_heads, s.num_kv_heads, s.rotary_dim, s.num_positions,
                 k_cache ? s.num_pages * s.page_size : 0, k_cache ? s.page_size : 1, s.eps, q, k, v, s.ld_q, s.ld_k, s.ld_v,
                 s.ld_q_out, s.ld_k_out, positions, cos_sin, q_weight, k_weight, slots, q_out, k_out, k_cache, v_cache,
                 s.k_page, s.k_token, s.k_head, s.v_page, s.v_token, s.v_head};
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  const bool il = s.interleaved != 0;
  if (s.dtype == GDN_BF16) return D == 64 ? launch_qk<uint16_t, 64>(a, il, hs) : launch_qk<uint16_t, 128>(a, il, hs);
  return D == 64 ? launch_qk<float, 64>(a, il, hs) : launch_qk<float, 128>(a, il, hs);
}

}  // extern "C"
