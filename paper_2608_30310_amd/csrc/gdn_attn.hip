// Attention over a shared prefix and own pages: validation and launches (C ABI
// in gdn_attn.h).
#include "gdn_attn_kernels.h"

#include <algorithm>
#include <cmath>
#include <limits>
#include <string>

#include "gdn_attn_plan.h"
#include "gdn_plan.h"

namespace gdn {
namespace {

gdn_status afail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

// Whether a few rows that are `units` of 16 bytes apart have 32-bit offsets.
bool a_stride_fits(int64_t units) { return units < int64_t{1} << 24; }

template <typename T, int D>
gdn_status launch_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  static_assert(kAttnRows == kPlanRows && kAttnTile == kPlanTile && kLineTile == kPlanLineTile && kStreamSeqs == kPlanLineSeqs,
                "the plan's tiles");
  hipLaunchKernelGGL((k_attn<T, D>), dim3(static_cast<uint32_t>(p.grid)), dim3(kAttnThreads), 0, stream, a);
  if (p.joined) {
    const uint32_t tiles = static_cast<uint32_t>((p.rows + kAttnRows - 1) / kAttnRows * a.kv_heads);
    if (p.spread) hipLaunchKernelGGL((k_attn_join<T, D, true>), dim3(tiles * (D / 8)), dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((k_attn_join<T, D, false>), dim3(tiles), dim3(kAttnThreads), 0, stream, a);
  }
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
  // n / d = mulhi(n, m) >> (l - 1) for n < 2^31: m = 2^(31 + l) / d rounded up, l = ceil(log2 d)
  int l = 0;
  while ((int64_t{1} << l) < s.page_size) ++l;
  const uint32_t mul = l ? static_cast<uint32_t>((uint64_t{1} << (31 + l)) / s.page_size + 1) : 0;
  const int64_t vec = 16 / e;
  const auto units = [&](int64_t stride) { return static_cast<uint32_t>(stride / vec); };
  AttnArgs a{};
  a.n_seqs = s.num_seqs, a.kv_heads = s.num_kv_heads, a.groups = p.groups, a.num_pages = s.num_pages;
  a.page_size = s.page_size, a.width = s.table_width, a.prefix_len = s.prefix_len, a.max_len = p.max_len;
  a.page_mul = mul, a.page_shift = l ? l - 1 : 0;
  // (not below the least normal number: a masked score of -inf stays one)
  a.scale2 = std::max(std::fabs(s.scale) * 1.44269504088896f, std::numeric_limits<float>::min());
  // rows of a DMA: 1 KiB of rows
  const int64_t rows = 1024 / (s.head_dim * e);
  const bool near = a_stride_fits(s.k_token / vec) && a_stride_fits(s.v_token / vec);
  a.dma_in_page = s.page_size % rows == 0 && near;
  a.part_in_page = s.page_size % (s.dtype == GDN_BF16 ? kPartRows : kPartRowsF32) == 0 && near;
  a.flip = std::signbit(s.scale) ? 0x80000000u : 0u;
  a.shared_splits = p.shared_splits, a.shared_chunk = p.shared_chunk;
  a.shared_tiles = static_cast<int32_t>(p.shared_tiles), a.shared_items = static_cast<int32_t>(p.shared_items);
  a.own_tile = p.own_tile, a.own_splits = p.own_splits, a.own_chunk = p.own_chunk;
  a.own_slots = static_cast<int32_t>(p.own_slots), a.rows = static_cast<int32_t>(p.rows);
  a.shared_wt = p.shared_wt, a.stream = p.stream, a.stream_first = p.stream_first, a.stream_waves = p.stream_waves;
  a.cu = cu_seqlens, a.table = table, a.lens = lens, a.prefix_pages = prefix_pages;
  a.q = q, a.k = k_cache, a.v = v_cache, a.out = out, a.ldq = s.ld_q, a.ldo = s.ld_out;
  a.kp = units(s.k_page), a.kt = units(s.k_token), a.vp = units(s.v_page), a.vt = units(s.v_token);
  a.kh = s.k_head * e, a.vh = s.v_head * e;
  if (p.joined) {
    a.part = static_cast<f32x4*>(workspace);
    a.part_ml = reinterpret_cast<f32x2*>(static_cast<char*>(workspace) + p.off_ml);
    a.line = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + p.off_line);
  }
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  if (s.dtype == GDN_BF16) return s.head_dim == 64 ? launch_attn<uint16_t, 64>(a, p, hs) : launch_attn<uint16_t, 128>(a, p, hs);
  return s.head_dim == 64 ? launch_attn<float, 64>(a, p, hs) : launch_attn<float, 128>(a, p, hs);
}

}  // extern "C"
