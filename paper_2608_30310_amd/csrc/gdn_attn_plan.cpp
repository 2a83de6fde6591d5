// Host-side validation and planning (see gdn_attn_plan.h).
#include "gdn_attn_plan.h"

#include "gdn_plan.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace gdn {
namespace {

constexpr int64_t kMaxInt = std::numeric_limits<int32_t>::max();
constexpr int64_t kMaxStride = int64_t{1} << 23;

// Workgroups of the attention that the chip holds at once: two a CU, but one where a
// workgroup's tiles (fp32, heads of 128) fill its LDS.  The fewest keys of a piece of a
// split range, in fp32 (a quarter of the rate) half as many.
constexpr int64_t kAttnPlaces = 512, kLeastChunk = 256;

gdn_status bad(std::string* err, const std::string& what, gdn_status st = GDN_ERR_BAD_SHAPE) {
  *err = what;
  return st;
}

gdn_status check_types(int32_t dim, int32_t dtype, std::string* err) {
  if (dim != 64 && dim != 128) return bad(err, "head_dim must be 64 or 128", GDN_ERR_UNSUPPORTED);
  if (dtype != GDN_F32 && dtype != GDN_BF16) return bad(err, "dtype must be GDN_F32 or GDN_BF16", GDN_ERR_UNSUPPORTED);
  return GDN_OK;
}

gdn_status check_ld(const char* name, int64_t ld, int64_t least, int64_t vec, std::string* err) {
  if (ld < least) return bad(err, std::string(name) + " must be at least " + std::to_string(least));
  if (ld > kMaxStride) return bad(err, std::string(name) + " must be at most 2^23", GDN_ERR_UNSUPPORTED);
  if (ld % vec != 0) return bad(err, std::string(name) + " must be a multiple of 16 bytes", GDN_ERR_UNSUPPORTED);
  return GDN_OK;
}

constexpr int64_t kMaxExtent = int64_t{1} << 48;   // elements between the rows of a cache: offsets in bytes fit 64 bits

// Strides of a cache: its rows of `dim` elements are apart; in 16 bytes they fit 31 bits.
gdn_status check_cache(const char* name, int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int64_t page,
                       int64_t token, int64_t head, int64_t vec, std::string* err) {
  if (pages < 1 || page_size < 1) return bad(err, "num_pages and page_size must be >= 1");
  if (static_cast<int64_t>(pages) * page_size > kMaxInt)
    return bad(err, "a cache must hold at most 2^31 - 1 tokens", GDN_ERR_UNSUPPORTED);
  struct { int64_t stride, count; } d[3] = {{page, pages}, {token, page_size}, {head, heads}};
  for (const auto& x : d) {
    if (x.stride < 0) return bad(err, std::string("strides of ") + name + " must not be negative");
    if (x.stride / vec >= int64_t{1} << 31) return bad(err, std::string("strides of ") + name + " must be below 2^31 x 16 bytes", GDN_ERR_UNSUPPORTED);
    if (x.stride % vec != 0)
      return bad(err, std::string("strides of ") + name + " must be multiples of 16 bytes", GDN_ERR_UNSUPPORTED);
  }
  std::sort(d, d + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
  int64_t extent = dim;   // of what lies inside one step of the next larger stride
  for (const auto& x : d) {
    if (x.count == 1) continue;
    if (x.stride < extent) return bad(err, std::string("rows of ") + name + " overlap");
    if (x.count - 1 > kMaxExtent / x.stride) return bad(err, std::string(name) + " is too large", GDN_ERR_UNSUPPORTED);
    extent += (x.count - 1) * x.stride;
  }
  return GDN_OK;
}

}  // namespace

int64_t cache_extent(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int64_t page, int64_t token,
                     int64_t head) {
  return (pages - 1) * page + (page_size - 1) * token + (heads - 1) * head + dim;
}

bool caches_apart(const void* pa, const void* pb, int64_t elt, int32_t pages, int32_t page_size, int32_t heads, int32_t dim,
                  int64_t page, int64_t token, int64_t head) {
  const int64_t whole = elt * cache_extent(pages, page_size, heads, dim, page, token, head);
  if (!overlap(pa, static_cast<size_t>(whole), pb, static_cast<size_t>(whole))) return true;
  struct { int64_t stride, count; } d[3] = {{page, pages}, {token, page_size}, {head, heads}};
  std::sort(d, d + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
  int64_t inner = dim;   // extent of what repeats at this stride
  for (int i = 0; i < 3; ++i) {
    if (d[i].count == 1) continue;
    bool regular = d[i].stride > 0;
    for (int j = i + 1; j < 3; ++j) regular = regular && (d[j].count == 1 || d[j].stride % d[i].stride == 0);
    const int64_t step = d[i].stride * elt;
    if (regular && !rows_overlap(pa, inner * elt, step, pb, inner * elt, step, whole / step + 1)) return true;
    inner += (d[i].count - 1) * d[i].stride;
  }
  return false;
}

gdn_status make_pages_plan(const gdn_pages_shape* s, const int32_t* cu, PagesPlan* plan, std::string* err) {
  if (!s) return bad(err, "shape is NULL", GDN_ERR_NULL_ARG);
  if (s->num_seqs < 0 || s->num_free < 0 || s->first < 0)
    return bad(err, "num_seqs, num_free and first must be >= 0");
  if (s->table_width < 1 || s->page_size < 1) return bad(err, "table_width and page_size must be >= 1");
  if (static_cast<int64_t>(s->num_seqs) * s->table_width > kMaxInt)
    return bad(err, "num_seqs * table_width too large", GDN_ERR_UNSUPPORTED);
  PagesPlan p;
  int64_t longest = 0;
  const gdn_status st = check_seqlens(s->num_seqs, cu, &p.tokens, &longest, err);
  if (st != GDN_OK) return st;
  p.slots = tile_slots(p.tokens, s->num_seqs, kPageTokens);
  if (p.slots > kMaxInt / 256) return bad(err, "too many sequences for one call", GDN_ERR_UNSUPPORTED);
  p.bytes = (3 * sizeof(int32_t) * static_cast<size_t>(s->num_seqs) + kAlign - 1) / kAlign * kAlign;
  *plan = p;
  return GDN_OK;
}

gdn_status check_qk(const gdn_qk_shape* s, bool k_out, bool k_cache, bool v, std::string* err) {
  if (!s) return bad(err, "shape is NULL", GDN_ERR_NULL_ARG);
  if (s->num_tokens < 0) return bad(err, "num_tokens must be >= 0");
  if (s->num_heads < 1 || s->num_kv_heads < 1) return bad(err, "head counts must be >= 1");
  if (s->num_heads > 65535 || s->num_kv_heads > 65535) return bad(err, "head counts must be <= 65535", GDN_ERR_UNSUPPORTED);
  gdn_status st = check_types(s->head_dim, s->dtype, err);
  if (st != GDN_OK) return st;
  if (s->rotary_dim < 16 || s->rotary_dim > s->head_dim || s->rotary_dim % 16 != 0)
    return bad(err, "rotary_dim must be a multiple of 16, at most head_dim", GDN_ERR_UNSUPPORTED);
  if (s->interleaved != 0 && s->interleaved != 1) return bad(err, "interleaved must be 0 or 1");
  if (s->num_positions < 1) return bad(err, "num_positions must be >= 1");
  if (!(s->eps >= 0.0f) || std::isinf(s->eps)) return bad(err, "eps must be >= 0 and finite");
  const int64_t vec = s->dtype == GDN_BF16 ? 8 : 4, D = s->head_dim;
  const struct { const char* name; int64_t ld, least; bool used; } rows[] = {
      {"ld_q", s->ld_q, s->num_heads * D, true},           {"ld_k", s->ld_k, s->num_kv_heads * D, true},
      {"ld_v", s->ld_v, s->num_kv_heads * D, v},           {"ld_q_out", s->ld_q_out, s->num_heads * D, true},
      {"ld_k_out", s->ld_k_out, s->num_kv_heads * D, k_out}};
  for (const auto& r : rows)
    if (r.used && (st = check_ld(r.name, r.ld, r.least, vec, err)) != GDN_OK) return st;
  if (k_cache)
    st = check_cache("k_cache", s->num_pages, s->page_size, s->num_kv_heads, s->head_dim, s->k_page, s->k_token, s->k_head,
                     vec, err);
  if (st == GDN_OK && v)
    st = check_cache("v_cache", s->num_pages, s->page_size, s->num_kv_heads, s->head_dim, s->v_page, s->v_token, s->v_head,
                     vec, err);
  if (st != GDN_OK) return st;
  if (static_cast<int64_t>(s->num_tokens) * (s->num_heads + 2 * static_cast<int64_t>(s->num_kv_heads)) > kMaxInt)
    return bad(err, "too many tokens for one call", GDN_ERR_UNSUPPORTED);
  return GDN_OK;
}

gdn_status check_attn(const gdn_attn_shape* s, std::string* err) {
  if (!s) return bad(err, "shape is NULL", GDN_ERR_NULL_ARG);
  if (s->num_seqs < 0) return bad(err, "num_seqs must be >= 0");
  if (s->num_heads < 1 || s->num_kv_heads < 1) return bad(err, "head counts must be >= 1");
  if (s->num_heads % s->num_kv_heads != 0) return bad(err, "num_heads must be a multiple of num_kv_heads");
  if (s->num_heads > 65535) return bad(err, "num_heads must be <= 65535", GDN_ERR_UNSUPPORTED);
  gdn_status st = check_types(s->head_dim, s->dtype, err);
  if (st != GDN_OK) return st;
  if (s->table_width < 1) return bad(err, "table_width must be >= 1");
  if (s->prefix_len < 0 || s->max_len < 0) return bad(err, "prefix_len and max_len must be >= 0");
  if (!std::isfinite(s->scale)) return bad(err, "scale must be finite");
  const int64_t vec = s->dtype == GDN_BF16 ? 8 : 4, width = static_cast<int64_t>(s->num_heads) * s->head_dim;
  if ((st = check_ld("ld_q", s->ld_q, width, vec, err)) != GDN_OK) return st;
  if ((st = check_ld("ld_out", s->ld_out, width, vec, err)) != GDN_OK) return st;
  if ((st = check_cache("k_cache", s->num_pages, s->page_size, s->num_kv_heads, s->head_dim, s->k_page, s->k_token,
                        s->k_head, vec, err)) != GDN_OK)
    return st;
  if ((st = check_cache("v_cache", s->num_pages, s->page_size, s->num_kv_heads, s->head_dim, s->v_page, s->v_token,
                        s->v_head, vec, err)) != GDN_OK)
    return st;
  const int64_t room = static_cast<int64_t>(s->table_width) * s->page_size;
  if (s->max_len > room) return bad(err, "max_len must be at most table_width * page_size");
  if ((s->max_len ? s->max_len : room) > (kMaxInt >> 1) || s->prefix_len > (kMaxInt >> 1))
    return bad(err, "prefix_len and own tokens must be below 2^30", GDN_ERR_UNSUPPORTED);
  return GDN_OK;
}

gdn_status make_attn_plan(const gdn_attn_shape* s, const int32_t* cu, AttnPlan* plan, std::string* err) {
  gdn_status st = check_attn(s, err);
  AttnPlan p;
  if (st == GDN_OK) st = check_seqlens(s->num_seqs, cu, &p.tokens, &p.longest, err);
  if (st != GDN_OK) return st;
  p.max_len = s->max_len ? s->max_len : s->table_width * s->page_size;
  p.groups = s->num_heads / s->num_kv_heads;
  if (p.tokens * s->num_heads > kMaxInt) return bad(err, "too many tokens for one call", GDN_ERR_UNSUPPORTED);
  const int64_t G = p.groups, H = s->num_kv_heads, N = s->num_seqs, P = s->prefix_len;
  p.rows = p.tokens * G;
  p.own_tile = p.longest * G <= kPlanRows ? kPlanRows : kPlanTile;
  int64_t tiles = 0;
  for (int64_t n = 0; n < N; ++n) tiles += ((static_cast<int64_t>(cu[n + 1]) - cu[n]) * G + p.own_tile - 1) / p.own_tile;
  p.own_slots = tile_slots(p.rows, N, p.own_tile);
  const bool bf16 = s->dtype == GDN_BF16;
  const int64_t least_chunk = bf16 ? kLeastChunk : kLeastChunk / 2;
  // A range of keys in as many pieces as are expected to end soonest, in us: a workgroup's
  // tiles of 64 keys one after the other, with one workgroup a CU or two; the joining's
  // launch, and each piece's partial results written and read.  Measured, 32 / 4 bf16 heads
  // of 128: prompts of 512 and 1024 tokens 23 and 39 us in two pieces, 20 and 31 in one; three
  // suffixes of up to 300 tokens behind 2000 shared ones 56 with two pieces of the prefix, 60
  // with one; fp32, 8 heads of 64, 20 suffixes of up to 200 tokens behind 1001: 99 and 115.
  const double scale = s->head_dim / 128.0, alone = scale * (bf16 ? 1.5 : 11.6), beside = scale * (bf16 ? 2.2 : 19.2);
  const double part = static_cast<double>(p.rows) * H * s->head_dim * 8 / 4.5e6;
  const auto pieces = [=](int64_t keys, int64_t items, int64_t most, bool joined, int32_t* splits, int32_t* chunk) {
    most = std::max<int64_t>(1, std::min((keys + least_chunk - 1) / least_chunk, most));
    double best = 0.0;
    for (int64_t n = 1; n <= most; ++n) {
      const int64_t each = std::max<int64_t>(64, ((keys + n - 1) / n + 63) / 64 * 64), got = std::max<int64_t>(1, (keys + each - 1) / each);
      const double cost = (items * got > kAttnPlaces / 2 ? beside : alone) * static_cast<double>(each / 64) +
                          (got > 1 && !joined ? 5.0 : 0.0) + part * static_cast<double>(got);
      if (n > 1 && cost >= best) continue;
      best = cost;
      *chunk = static_cast<int32_t>(each);
      *splits = static_cast<int32_t>(got);
    }
  };
  const int64_t line = N * H * ((p.max_len + static_cast<int64_t>(kPlanLineTile) - 1) / kPlanLineTile);   // tiles at most
  p.stream = p.own_tile == kPlanRows && N <= kPlanLineSeqs && H <= kPlanLineHeads && line <= int64_t{1} << 30;
  // (fp32's single tokens wait for memory with half as many waves: 161 us, 175 with all)
  const int64_t places = bf16 || (!p.stream && s->head_dim == 64) ? kAttnPlaces : kAttnPlaces / 2;
  constexpr int64_t waves = kPlanTile / kPlanRows;   // of a workgroup
  // (without rows there are no tiles to share places out to)
  if (P > 0 && p.rows > 0 && (p.stream || tiles * H < places || p.rows < tiles * p.own_tile * 3 / 5)) {
    p.shared_tiles = (p.rows + kPlanTile - 1) / kPlanTile;
    if (p.stream && p.rows <= kPlanRows) {
      // a wave's items, as many tiles each as balance their walk with the joining (see line_shares)
      p.shared_wt = 1;
      const int64_t keys = (P + kPlanLineTile - 1) / kPlanLineTile;
      const int64_t least = static_cast<int64_t>(std::ceil(std::sqrt(static_cast<double>(keys) / 32)));
      const int64_t n = std::max<int64_t>(1, std::min(places * waves / H, keys / std::max<int64_t>(1, least)));
      const int64_t each = (keys + n - 1) / n;
      p.shared_chunk = static_cast<int32_t>(each * kPlanLineTile);
      p.shared_splits = static_cast<int32_t>((keys + each - 1) / each);
    } else {
      if (p.stream) {
        // one workgroup a CU: the other place is for own items, which wait for memory while
        // these compute
        const int64_t n = std::max<int64_t>(1, std::min((P + least_chunk - 1) / least_chunk, places / 2 / (p.shared_tiles * H)));
        p.shared_chunk = static_cast<int32_t>(std::max<int64_t>(64, ((P + n - 1) / n + 63) / 64 * 64));
        p.shared_splits = static_cast<int32_t>((P + p.shared_chunk - 1) / p.shared_chunk);
      } else {
        // with room for the own items beside them, unless that leaves the prefix whole
        pieces(P, p.shared_tiles * H, std::max<int64_t>(2, places / 2 / (p.shared_tiles * H)), true, &p.shared_splits, &p.shared_chunk);
      }
    }
    p.shared_items = p.shared_tiles * H * p.shared_splits;
  }
  size_t own_tiles = 0;   // wave tiles of the own items' partial results
  if (p.stream) {
    // workgroups of their own for the own tokens while there is room, else all take both
    const int64_t wanted = (std::max<int64_t>(1, std::min(places * waves, line)) + waves - 1) / waves;
    const int64_t shared = p.shared_wt == 1 ? (p.shared_items + waves - 1) / waves : p.shared_items;
    const bool apart = shared + wanted <= places;
    p.stream_first = apart ? static_cast<int32_t>(shared) : 0;
    p.stream_waves = static_cast<int32_t>(wanted * waves);
    p.grid = apart ? shared + wanted : places;
    p.joined = true;
    own_tiles = 2 * static_cast<size_t>(p.stream_waves) + static_cast<size_t>(N * H);
  } else {
    if (P == 0 || p.shared_items > 0) pieces(p.max_len, tiles * H, places / std::max<int64_t>(1, tiles * H), p.shared_items > 0, &p.own_splits, &p.own_chunk);
    else p.own_chunk = (p.max_len + 63) / 64 * 64;
    p.own_items = p.own_slots * H * p.own_splits;
    p.joined = p.shared_items > 0 || p.own_splits > 1;
    p.grid = p.shared_items + p.own_items;
    own_tiles = static_cast<size_t>(p.own_items) * (p.own_tile / kPlanRows);
  }
  if (p.grid > kMaxInt / 256 || p.rows / kPlanRows * H * (s->head_dim / 8) > kMaxInt / 256)
    return bad(err, "too many tokens for one call", GDN_ERR_UNSUPPORTED);
  p.spread = p.stream || p.shared_splits + p.own_splits > kPlanFewParts;
  if (p.joined) {
    const size_t parts = static_cast<size_t>(p.shared_items) * p.shared_wt + own_tiles;
    p.off_ml = parts * kPlanRows * s->head_dim * sizeof(float);
    p.off_line = p.off_ml + parts * kPlanRows * 2 * sizeof(float);
    p.bytes = p.off_line + (p.stream ? (static_cast<size_t>(N) + 1 + p.tokens) * sizeof(int32_t) : 0);
    p.bytes = (p.bytes + kAlign - 1) / kAlign * kAlign;
  }
  *plan = p;
  return GDN_OK;
}

}  // namespace gdn
