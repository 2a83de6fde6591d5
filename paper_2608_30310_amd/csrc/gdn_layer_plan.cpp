// Host-side validation and planning (see gdn_layer_plan.h).
#include "gdn_layer_plan.h"

#include "gdn_plan.h"

#include <algorithm>
#include <functional>
#include <limits>

namespace gdn {
namespace {

constexpr int64_t kMaxGrid = std::numeric_limits<int32_t>::max();
// a tile's rows are addressed with 32-bit byte offsets: 64 rows of 2^23 fp32 elements
constexpr int64_t kMaxStride = int64_t{1} << 23;

constexpr int64_t kSsmPlaces = 256;   // workgroups of the state space scan that the chip holds at once, one per CU

// Workgroups that the first product of the adapters aims at: 64 sequences of 8
// tokens, rank 16, 16.5 us; 18.6 with 128, 17.1 with 512.
constexpr int64_t kLoraGroups = 256;

int64_t chunks_of(const int32_t* cu, int64_t n) { return (static_cast<int64_t>(cu[n + 1]) - cu[n] + 63) / 64; }

constexpr int64_t kXcds = 8;

// Chunks after which the last of n <= kSsmOrdered sequences ends: the longest
// first, dealt to the XCDs there and back, `lanes` of them at once on each, where the
// next starts as one ends.
double longest_first(const int32_t* cu, int64_t n, int64_t lanes) {
  int64_t chunks[kSsmOrdered];
  for (int64_t i = 0; i < n; ++i) chunks[i] = chunks_of(cu, i);
  std::sort(chunks, chunks + n, std::greater<int64_t>());
  int64_t end = 0;
  for (int64_t x = 0; x < kXcds; ++x) {
    int64_t busy[kSsmOrdered] = {};   // a heap, the lane that is free first in front
    for (int64_t row = 0; row * kXcds < n; ++row) {
      const int64_t r = row * kXcds + (row % 2 != 0 && (row + 1) * kXcds <= n ? kXcds - 1 - x : x);
      if (r >= n) continue;
      std::pop_heap(busy, busy + lanes, std::greater<int64_t>());
      end = std::max(end, busy[lanes - 1] += chunks[r]);
      std::push_heap(busy, busy + lanes, std::greater<int64_t>());
    }
  }
  return static_cast<double>(end);
}

bool known_dtype(int32_t d) { return d == GDN_F32 || d == GDN_BF16; }

gdn_status check_stride(const char* name, int64_t ld, int64_t least, std::string* err) {
  if (ld < least) { *err = std::string(name) + " must be at least " + std::to_string(least); return GDN_ERR_BAD_SHAPE; }
  if (ld > kMaxStride) { *err = std::string(name) + " must be at most 2^23"; return GDN_ERR_UNSUPPORTED; }
  return GDN_OK;
}

}  // namespace

gdn_status check_seqlens(int32_t n, const int32_t* cu, int64_t* tokens, int64_t* longest, std::string* err) {
  if (!cu) { *err = "cu_seqlens_host is NULL"; return GDN_ERR_NULL_ARG; }
  if (cu[0] != 0) { *err = "cu_seqlens_host[0] must be 0"; return GDN_ERR_BAD_SEQLENS; }
  int64_t top = 0;
  for (int32_t i = 0; i < n; ++i) {
    const int64_t len = static_cast<int64_t>(cu[i + 1]) - cu[i];
    if (len < 0) { *err = "cu_seqlens_host must be non-decreasing"; return GDN_ERR_BAD_SEQLENS; }
    top = std::max(top, len);
  }
  *tokens = cu[n];
  *longest = top;
  return GDN_OK;
}

gdn_status check_conv(const gdn_conv_shape* s, std::string* err) {
  if (!s) { *err = "shape is NULL"; return GDN_ERR_NULL_ARG; }
  if (s->num_seqs < 0) { *err = "num_seqs must be >= 0"; return GDN_ERR_BAD_SHAPE; }
  if (s->channels < 1) { *err = "channels must be >= 1"; return GDN_ERR_BAD_SHAPE; }
  if (s->taps < 2 || s->taps > 4) { *err = "taps must be 2, 3 or 4"; return GDN_ERR_UNSUPPORTED; }
  if (!known_dtype(s->dtype)) { *err = "dtype must be GDN_F32 or GDN_BF16"; return GDN_ERR_UNSUPPORTED; }
  if (s->activation != GDN_ACT_NONE && s->activation != GDN_ACT_SILU) {
    *err = "activation must be GDN_ACT_NONE or GDN_ACT_SILU";
    return GDN_ERR_UNSUPPORTED;
  }
  const gdn_status st = check_stride("ld_x", s->ld_x, s->channels, err);
  return st != GDN_OK ? st : check_stride("ld_y", s->ld_y, s->channels, err);
}

gdn_status check_ssm(const gdn_ssm_shape* s, std::string* err, bool outputs) {
  if (!s) { *err = "shape is NULL"; return GDN_ERR_NULL_ARG; }
  if (s->num_seqs < 0) { *err = "num_seqs must be >= 0"; return GDN_ERR_BAD_SHAPE; }
  if (s->num_heads < 1 || s->num_groups < 1) { *err = "head counts must be >= 1"; return GDN_ERR_BAD_SHAPE; }
  if (s->num_heads % s->num_groups != 0) {
    *err = "num_heads must be a multiple of num_groups";
    return GDN_ERR_BAD_SHAPE;
  }
  if (s->num_heads > 65535) { *err = "num_heads must be <= 65535"; return GDN_ERR_UNSUPPORTED; }
  const auto dim = [](int32_t d) { return d == 64 || d == 128; };
  if (!dim(s->d_state) || !dim(s->head_dim)) {
    *err = "d_state and head_dim must each be 64 or 128";
    return GDN_ERR_UNSUPPORTED;
  }
  if (!known_dtype(s->dtype)) { *err = "dtype must be GDN_F32 or GDN_BF16"; return GDN_ERR_UNSUPPORTED; }
  if (s->dt_dtype != GDN_F32 && s->dt_dtype != s->dtype) {
    *err = "dt_dtype must be GDN_F32 or the same as dtype";
    return GDN_ERR_UNSUPPORTED;
  }
  const int64_t H = s->num_heads, G = s->num_groups, vec = s->dtype == GDN_BF16 ? 8 : 4;
  struct { const char* name; int64_t ld, least; bool used, aligned; } rows[] = {
      {"ld_x", s->ld_x, H * s->head_dim, true, true},
      {"ld_dt", s->ld_dt, H, true, false},
      {"ld_b", s->ld_b, G * s->d_state, true, true},
      {"ld_c", s->ld_c, G * s->d_state, outputs, true},
      {"ld_y", s->ld_y, H * s->head_dim, outputs, true}};
  for (const auto& r : rows) {
    if (!r.used) continue;
    if (const gdn_status st = check_stride(r.name, r.ld, r.least, err); st != GDN_OK) return st;
  }
  for (const auto& r : rows)
    if (r.used && r.aligned && r.ld % vec != 0) {
      *err = std::string(r.name) + " must be a multiple of 16 bytes";
      return GDN_ERR_UNSUPPORTED;
    }
  if (static_cast<int64_t>(s->num_seqs) * H > kMaxGrid / 256) {
    *err = "num_seqs * num_heads too large";
    return GDN_ERR_UNSUPPORTED;
  }
  return GDN_OK;
}

gdn_status make_ssm_plan(const gdn_ssm_shape* s, const int32_t* cu, SsmPlan* plan, std::string* err, bool outputs,
                         int64_t least_segment) {
  gdn_status st = check_ssm(s, err, outputs);
  SsmPlan p;
  if (st == GDN_OK) st = check_seqlens(s->num_seqs, cu, &p.tokens, &p.longest, err);
  if (st != GDN_OK) return st;
  const int64_t H = s->num_heads, N = s->num_seqs;
  const bool bf16 = s->dtype == GDN_BF16;
  int32_t share = (bf16 ? kSsmCols : kSsmColsF32) / s->head_dim;
  while (H / s->num_groups % share != 0) share /= 2;
  // Whole sequences: the longest one, or what the places' shares of the work come to.
  const int64_t longest = (p.longest + 63) / 64;
  int64_t chunks = 0;
  for (int64_t n = 0; n < N; ++n) chunks += chunks_of(cu, n);
  // More sequences than fit at once start with the longest, unless there is so much
  // work that the last one's length does not matter (us, 32 heads of 128 x 128: 24
  // sequences of 1 to 1000 tokens 146, as they come 196; 40 of 1 to 800 187 and 215; 64
  // of 1 to 300 151 and 139).
  const auto orderable = [&](int64_t groups) {
    return N * groups > kSsmPlaces && N <= kSsmOrdered && groups <= kSsmPlaces / kXcds &&
           2 * longest * kSsmPlaces >= chunks * groups;
  };
  const auto whole = [&](int64_t groups) {
    if (N * groups <= kSsmPlaces) return static_cast<double>(longest);
    if (orderable(groups)) return longest_first(cu, N, std::min<int64_t>(kSsmOrdered, kSsmPlaces / kXcds / groups));
    return std::max(static_cast<double>(longest), static_cast<double>(chunks * groups) / kSsmPlaces);
  };
  // Whole sequences end with the longest one, or with the work per place; in
  // segments the work is even, but every chunk is walked twice (once for the
  // states alone), the segments' states pass through memory and there are two
  // launches more.  In chunks of the whole walk (~6.5 us for bf16 inputs): whole
  // 0.8 + the chunks; segments 2.5 + 1.5 x a segment's chunks + 0.0093 x their
  // number.  Measured, 64 heads of 64 x 128, one sequence of 2, 3, 8, 24 and 128
  // chunks: whole 18, 25, 55, 152 and 776 us, segments 24, 26, 37, 44 and 105;
  // 32 heads of 128 x 128, 8 sequences of 8 and 16, 4 of 64: 58, 104 and 397, 73, 110 and 190.
  int64_t groups = H / share;   // workgroups of a sequence
  double best = 0.8 + whole(groups);
  p.heads_per_group = share;
  p.slots = N;
  // Half the heads a workgroup, whole sequences: twice the CUs at 0.77 of the time
  // a chunk.  Measured, 64 heads of 64 x 128: one sequence of 1, 2 and 3 chunks
  // 9.6, 14.4 and 19.4 us by twos, 12.2, 18.4 and 24.5 by fours; 8 of 1, 3 and 13:
  // 14.5, 25.5 and 72.9, 16.6, 29.8 and 89.7; but 32 of 32 chunks 676, 486.  And 32 heads
  // of 128 x 128, 16 of 2 to 32 chunks: 202 one by one, 223 by twos.
  if (bf16 && share * s->head_dim == kSsmCols)
    if (const double cost = 0.7 + 0.77 * whole(2 * groups); cost < best) {
      best = cost;
      p.heads_per_group = share / 2;
    }
  const int64_t least = std::max<int64_t>(1, (chunks * groups + kSsmPlaces - 1) / kSsmPlaces);
  int64_t seg = 0;
  const bool joinable = N * H * s->d_state * s->head_dim / 4 <= kMaxGrid;   // a thread of the join takes four elements
  for (int64_t more = 0; joinable && more <= 4 && least + more * ((least + 3) / 4) < longest; ++more) {
    const int64_t try_seg = std::max(least_segment, least + more * ((least + 3) / 4));
    int64_t segs = 0;
    for (int64_t n = 0; n < N; ++n) segs += std::max<int64_t>(1, (chunks_of(cu, n) + try_seg - 1) / try_seg);
    const int64_t rounds = (segs * groups + kSsmPlaces - 1) / kSsmPlaces;
    const double cost = 2.5 + 1.5 * static_cast<double>(try_seg * rounds) + 0.0093 * static_cast<double>(segs * groups);
    if (cost < best) {
      best = cost;
      seg = try_seg;
      p.slots = segs;
      p.heads_per_group = share;
    }
  }
  groups = H / p.heads_per_group;
  p.ordered = seg == 0 && orderable(groups);
  if (seg > 0) {
    p.seg_tokens = static_cast<int32_t>(64 * seg);
    const size_t state = static_cast<size_t>(H) * s->d_state * s->head_dim * sizeof(float);
    p.off_decay = static_cast<size_t>(p.slots) * state;   // a multiple of 256
    p.bytes = (p.off_decay + static_cast<size_t>(p.slots) * H * sizeof(float) + kAlign - 1) / kAlign * kAlign;
  }
  if (p.slots * groups > kMaxGrid / 1024) {
    *err = "too many segments";
    return GDN_ERR_UNSUPPORTED;
  }
  *plan = p;
  return GDN_OK;
}

gdn_status check_lora(const gdn_lora_shape* s, std::string* err) {
  if (!s) { *err = "shape is NULL"; return GDN_ERR_NULL_ARG; }
  if (s->num_seqs < 0 || s->num_adapters < 0) {
    *err = "num_seqs and num_adapters must be >= 0";
    return GDN_ERR_BAD_SHAPE;
  }
  if (s->hidden < 1 || s->width < 1 || s->rank < 1) {
    *err = "hidden, width and rank must be >= 1";
    return GDN_ERR_BAD_SHAPE;
  }
  if (s->hidden % 8 != 0) { *err = "hidden must be a multiple of 8"; return GDN_ERR_UNSUPPORTED; }
  if (s->rank % 8 != 0 || s->rank > 128) {
    *err = "rank must be a multiple of 8, at most 128";
    return GDN_ERR_UNSUPPORTED;
  }
  if (!known_dtype(s->out_dtype)) { *err = "out_dtype must be GDN_F32 or GDN_BF16"; return GDN_ERR_UNSUPPORTED; }
  gdn_status st = check_stride("ld_x", s->ld_x, s->hidden, err);
  if (st == GDN_OK) st = check_stride("ld_base", s->ld_base, s->width, err);
  if (st == GDN_OK) st = check_stride("ld_out", s->ld_out, s->width, err);
  if (st != GDN_OK) return st;
  if (s->ld_x % 8 != 0) { *err = "ld_x must be a multiple of 8"; return GDN_ERR_UNSUPPORTED; }
  return GDN_OK;
}

gdn_status make_lora_plan(const gdn_lora_shape* s, const int32_t* cu, LoraPlan* plan, std::string* err) {
  gdn_status st = check_lora(s, err);
  LoraPlan p;
  int64_t longest = 0;
  if (st == GDN_OK) st = check_seqlens(s->num_seqs, cu, &p.tokens, &longest, err);
  if (st != GDN_OK) return st;
  // Small tiles where larger ones would be mostly empty, or too few for the CUs.
  // Measured (2048 -> 12352, us), tiles of 16 tokens and of 32 and 64: 64 sequences of 1, 8
  // and 32 tokens at rank 16 12.3, 16.5 and 30.6, 16.6, 20.4 and 28.6; at rank 64 8 of 32
  // tokens 17.4, 23.3, one of 819 27.8, 31.1, 8 of 128 33.5 both, of 512 88, 61.
  // Second product, tiles of 32 and of 64: 64 sequences of 32 tokens 26.7, 35.1, at rank
  // 64 8 of 512 56.6, 58.9, of 1500 182.7, 162.3.
  const bool tokenwise = p.tokens <= std::max<int64_t>(1024, 16 * static_cast<int64_t>(s->num_seqs));
  p.down_tile = tokenwise ? 16 : 32;
  p.up_tile = tokenwise ? 16 : p.tokens > 6144 && p.tokens >= 64 * static_cast<int64_t>(s->num_seqs) ? 64 : 32;
  p.down_slots = tile_slots(p.tokens, s->num_seqs, p.down_tile);
  p.up_slots = tile_slots(p.tokens, s->num_seqs, p.up_tile);
  // x A^T in parts of K until there are workgroups for every CU (64 sequences of 4
  // tokens, rank 16: 14.1 us in four parts, 15.7 in one), each with at least two
  // 32-wide steps for each of its four waves.  Every column tile reads every part,
  // so no more than 1 KB of them a token (8 x 32 tokens, rank 64: 15.6 us in 4 parts,
  // 17.6 in 8, 20.9 in one; one sequence of 1500 36.8 in 4, 38.7 in 6).
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(s->hidden / 256, 256 / s->rank));
  p.parts = static_cast<int32_t>(std::min(most, std::max<int64_t>(1, kLoraGroups / std::max<int64_t>(1, p.down_slots))));
  const int64_t tiles = (static_cast<int64_t>(s->width) + 255) / 256;
  if (p.down_slots * p.parts > kMaxGrid / 256 || p.up_slots * tiles > kMaxGrid / 256) {
    *err = "too many tokens for one call";
    return GDN_ERR_UNSUPPORTED;
  }
  p.bytes = (static_cast<size_t>(p.parts) * p.tokens * s->rank * sizeof(float) + kAlign - 1) / kAlign * kAlign;
  *plan = p;
  return GDN_OK;
}

bool overlap(const void* pa, size_t na, const void* pb, size_t nb) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(pa), b = reinterpret_cast<uintptr_t>(pb);
  return na > 0 && nb > 0 && a < b + nb && b < a + na;
}

bool rows_overlap(const void* pa, int64_t wa, int64_t lda, const void* pb, int64_t wb, int64_t ldb, int64_t rows) {
  if (rows < 1) return false;
  const size_t na = static_cast<size_t>((rows - 1) * lda + wa), nb = static_cast<size_t>((rows - 1) * ldb + wb);
  if (!overlap(pa, na, pb, nb)) return false;
  if (lda != ldb) return true;
  // windows [0, wa) and [d, d + wb) of a circle of lda bytes
  const int64_t gap = static_cast<int64_t>(reinterpret_cast<uintptr_t>(pb) - reinterpret_cast<uintptr_t>(pa));
  const int64_t d = ((gap % lda) + lda) % lda;
  return d < wa || d + wb > lda;
}

}  // namespace gdn
