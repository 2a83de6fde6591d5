// Attention over a shared prefix and each sequence's own pages on the matrix
// cores (C ABI in gdn_attn.h).
//
// Rows.  The Hq / Hkv query heads of a K/V head read the same keys, so a row of
// a tile is one head of one token, r = token * G + head % G, and keys are read
// once for all of them.  A work item is a tile of rows, one K/V head and a range
// of keys: of the prefix, of a sequence's own tokens, or of both one after the
// other.
//
// A tile of scores is formed transposed, S^T = K Q^T (32 x 32 x 16 products): a
// lane holds one row's scores, 16 keys of 32 (the other half wave the rest), so
// maximum and sum are per lane but for one exchange of halves, and the scores'
// registers are, key for key, the operand of O^T = V^T P^T.  Which keys lie in
// which registers does not matter to that product as long as V's operand has them
// in the same order.  One pass, with the running maximum m and sum l of each row:
//   p = 2^(s - m),  l += sum p,  O += p V,  out = O / l,
// where m is 8 above a maximum and moves (and O and l are scaled) only when weights or a
// tile's sum of them pass 1: weights are 2^-8 at first and never above 1, so that no sum of
// values grows beyond that of the values themselves.
#pragma once

#include <type_traits>

#include "gdn_varlen.h"

namespace gdn {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / kWave;
constexpr int kAttnRows = 32;                        // of a wave
constexpr int kAttnTile = kAttnRows * kAttnWaves;    // of a workgroup whose waves take rows of their own
constexpr int kPartRows = 16, kPartRowsF32 = 8;      // rows of such a workgroup's K/V tiles that a wave loads

constexpr int kStreamSeqs = 1024;                    // sequences of a line (see there)

struct AttnArgs {
  int32_t n_seqs, kv_heads, groups, num_pages, page_size, width, prefix_len, max_len;
  uint32_t page_mul;      // n / page_size = mulhi(n, page_mul) >> page_shift (page_size > 1)
  int32_t page_shift;
  float scale2;           // |scale| log2 e
  uint32_t flip;          // sign bits of the queries where scale is negative
  int32_t dma_in_page;    // the rows of a DMA never lie in two pages, and their offsets fit 32 bits
  int32_t part_in_page;   // so do those of a wave's part of a workgroup's tile
  // items: shared ones over the prefix alone, all rows packed (shared_splits 0: none), then own ones
  int32_t shared_splits, shared_chunk, shared_tiles, shared_items;
  int32_t own_tile, own_splits, own_chunk, own_slots;
  int32_t shared_wt;      // wave tiles of a shared item: kAttnWaves, or 1 (a wave's)
  // stream (see there): stream_waves waves from workgroup stream_first on share the own tokens out
  int32_t stream, stream_first, stream_waves;
  int32_t* line;          // [N + 1], then the sequence of each token [T], for the joining kernel
  int32_t rows;           // T G
  const int32_t* cu;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* prefix_pages;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  int64_t ldq, ldo;
  uint32_t kp, kt, vp, vt;   // strides of the caches' pages and tokens, in 16 bytes
  int64_t kh, vh;            // of their heads, in bytes
  // partial results of the items: shared ones, then own ones
  f32x4* part;            // [item][wave tile][D / 8][lane]: four columns of a row
  f32x2* part_ml;         // [item][wave tile][32]: m and l of a row
};

// Branches that registers are not to be allotted for (rare loops would come before
// the ones around them).
__device__ __forceinline__ bool rarely(bool x) { return __builtin_expect(x, 0); }

// ---------------------------------------------------------------- operands
// 32 x 32 x 16 products: lane (h, r) supplies elements 8 h + j (j = 0..7) of row r
// of either operand and holds rows 8 (i / 4) + 4 h + i % 4 (i = 0..15) of column r.
template <typename T>
struct Mm;
template <>
struct Mm<uint16_t> {
  typedef bf16x8 R;
  static __device__ __forceinline__ f32x16 mul(const R& a, const R& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // p: eight weights, rounded to bf16 as the product takes them, and their sums: of what
  // enters the product, so that the rounding of a weight is one of numerator and
  // denominator alike; two at a time.  Outputs are within 2.0e-3 to 2.4e-3 of 64 bits that
  // way, 1.5e-3 to 1.7e-3 of which are the output's own rounding; weights in two parts would
  // take half as many products again.
  static __device__ __forceinline__ R pack(const float (&p)[8], float (&sum)[4]) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 x = {p[2 * j], p[2 * j + 1]};
      const bf16x2 y = __builtin_convertvector(x, bf16x2), one = {1.0f, 1.0f};
      w[j] = __builtin_bit_cast(uint32_t, y);
      sum[j] = __builtin_amdgcn_fdot2_f32_bf16(y, one, sum[j], false);
    }
    return __builtin_bit_cast(R, w);
  }
  static __device__ __forceinline__ R flip(const R& a, uint32_t sign) {
    u32x4 w = __builtin_bit_cast(u32x4, a);
    w ^= sign | sign >> 16;
    return __builtin_bit_cast(R, w);
  }
};
template <>
struct Mm<float> {
  typedef f32x8 R;
  static __device__ __forceinline__ f32x16 mul(const R& a, const R& b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ R pack(const float (&p)[8], float (&sum)[4]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j % 4] += p[j];
    return R{p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]};
  }
  static __device__ __forceinline__ R flip(const R& a, uint32_t sign) {
    R r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = __uint_as_float(__float_as_uint(a[j]) ^ sign);
    return r;
  }
};

// The lane, for what is made of it anew for each tile instead of being kept in registers
// over the tiles.
__device__ __forceinline__ int lane_now() {
  int x = threadIdx.x;
  asm volatile("" : "+v"(x));
  return static_cast<uint32_t>(x) % kWave;
}

// Rows of D elements in LDS as they lie in memory, 16-byte piece p of row r at
// p ^ swz(r).  The swizzle is a permutation of the low row bits, so the operand
// reads of K (32 rows of one piece) meet every bank once; those of V (four rows
// of four pieces, transposed on the way) do because rows 0..3 differ in the high
// bits of the piece.  (fp32: rows r and r + 4 differ in the highest, for V's
// 4-byte reads.)
template <typename T, int D>
struct KvRows {
  static constexpr int kPitch = D * static_cast<int>(sizeof(T));
  static constexpr int kPieces = kPitch / 16;
  static constexpr int kRowsPerDma = kWave / kPieces;   // a DMA moves 64 pieces
  static __device__ __forceinline__ constexpr int swz(int r) {
    if (sizeof(T) == 4) return (r & 7) << 1 | (r >> 3 & 1);
    return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
  static __device__ __forceinline__ int at(int r, int piece) { return r * kPitch + ((piece ^ swz(r)) << 4); }
  // Operand of 32 rows, elements 16 u + 8 h ..: `at` is at(r, h) for lane (h, r) (fp32:
  // of 4-byte elements, at(r, 2 h)), turned by kFragStep u; r multiples of 16 above, the
  // swizzle is the same.
  static constexpr int kFragStep = 2 * 16 * static_cast<int>(sizeof(T)) / 2;
  static __device__ __forceinline__ int frag_start(int lane) { return at(lane % 32, lane / 32 * static_cast<int>(sizeof(T)) / 2); }
  static __device__ __forceinline__ typename Mm<T>::R frag_at(const char* base, int at) {
    if constexpr (sizeof(T) == 2) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(base + at));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(base + at);
      const f32x4 b = *reinterpret_cast<const f32x4*>(base + (at ^ 16));
      return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  }
  // Operand of 16 rows, transposed: column 32 dt + lane % 32 of rows 8 (j / 4) + 4 h + j % 4,
  // j = 0..7.  col_start: where a lane's first read begins for dt = 0.
  static __device__ __forceinline__ int col_start(int lane) {
    const int h = lane / 32;
    if constexpr (sizeof(T) == 2) return at(4 * h + lane % 16 / 4, lane / 16 % 2 * 2 + lane % 4 / 2) + lane % 2 * 8;
    else return at(4 * h, lane % 32 / 4) + lane % 4 * 4;
  }
  static __device__ __forceinline__ typename Mm<T>::R col_frag(const char* base, int at, int dt) {
    if constexpr (sizeof(T) == 2) {
      // four pieces on is the bits 4 dt of the piece; eight rows on turn it by swz(8)
      const u32x2 a = lds_read_tr16(base + (at ^ 64 * dt));
      const u32x2 b = lds_read_tr16(base + (at ^ 64 * dt ^ 16 * swz(8)) + 8 * kPitch);
      return join_halves(a, b);
    } else {
      f32x8 x;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = 8 * (j / 4) + j % 4;   // bits apart from those of 4 h
        x[j] = *reinterpret_cast<const float*>(base + (at ^ 128 * dt ^ 16 * swz(row)) + row * kPitch);
      }
      return x;
    }
  }
};

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }
// A piece of a row with its infinities and NaNs replaced by zero.
template <typename T>
__device__ __forceinline__ u32x4 finite_only(u32x4 w) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 2) {
      const bool lo = (w[j] & 0x7F80u) == 0x7F80u, hi = (w[j] & 0x7F800000u) == 0x7F800000u;
      w[j] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
    } else {
      w[j] = not_finite(__uint_as_float(w[j])) ? 0u : w[j];
    }
  }
  return w;
}

// The larger of a lane's value and its counterpart's in the other half wave, and their sum.
__device__ __forceinline__ float half_max(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// ---------------------------------------------------------------- keys
// The keys that an item walks: `count0` tokens of the prefix from `first0` on, then
// `count1` of a sequence's own from `first1` on.
struct KeyRange {
  const int32_t* list0;
  const int32_t* list1;
  int first0, count0, first1, count1;
};
// A tile of KT of them: tokens base .. of a list of pages, `count` of them left in
// their part of the range.
struct KeyTile {
  const int32_t* list;
  int base, count;
  bool own;
};
__device__ __forceinline__ void key_part(const KeyRange& k, KeyTile& t) {   // t.own: into the second part
  t.list = t.own ? k.list1 : k.list0;
  t.base = t.own ? k.first1 : k.first0;
  t.count = t.own ? k.count1 : k.count0;
}
__device__ __forceinline__ KeyTile first_tile(const KeyRange& k) {
  KeyTile t;
  t.own = k.count0 <= 0;
  key_part(k, t);
  return t;
}
// KT tokens on; no tile where its count is not positive.
template <int KT>
__device__ __forceinline__ void next_tile(const KeyRange& k, KeyTile& t) {
  t.base += KT;
  t.count -= KT;
  if (t.count <= 0 && !t.own) {
    t.own = true;
    key_part(k, t);
  }
}

// Loads into LDS that the compiler does not count: it would wait for all of them
// before the next transposing read of LDS, which may be of another buffer.  Whoever
// reads what they write waits by wait_dma or wait_dma_but first.
__device__ __forceinline__ uint32_t lds_address(lds_byte* p) {
  return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)));
}
// Two waits that the compiler does not add inside a string: one instruction between the
// write of M0 and the load that takes its place in LDS from it; and five between a vector
// instruction's write of a scalar register (a lane read) and a load that takes its address
// from it, but none where a scalar move lies between.  (16 suffixes and the single tokens
// take as long with them as without.)
__device__ __forceinline__ void async_piece(const void* src, lds_byte* dst) {   // 16 bytes a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(dst)), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ void async_piece(uint64_t base, uint32_t off, lds_byte* dst) {   // from a uniform base
  uint64_t at;
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0"
               : "=&s"(at) : "s"(lds_address(dst)), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void async_word(const void* src, lds_byte* dst) {   // 4 bytes a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_address(dst)), "v"(src) : "memory", "m0");
}

// What the loop over tiles needs of the arguments: each value a register of its own
// (left in the tuples that they are loaded in, they do not fit the scalar registers and
// every use restores a whole tuple).
template <typename X>
__device__ __forceinline__ X apart(X x) {
  static_assert(sizeof(X) == 4 || sizeof(X) == 8, "one or two registers");
  if constexpr (sizeof(X) == 4) {
    uint32_t u = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(uint32_t, x));
    asm("" : "+s"(u));
    return __builtin_bit_cast(X, u);
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u)),
             hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
    asm("" : "+s"(lo), "+s"(hi));
    return __builtin_bit_cast(X, static_cast<uint64_t>(hi) << 32 | lo);
  }
}
// Where a K/V head's rows are in the caches, and a lane's place in a DMA of
// kRowsPerDma rows: the swizzle is linear over XOR, so piece p of row r + j (r a
// multiple of kRowsPerDma) comes from piece (p ^ swz(j)) ^ swz(r).
template <typename T, int D>
struct CacheAt {
  uint64_t k, v;
  uint32_t kp, kt, vp, vt, page_mul;
  int page_shift, page_size, num_pages, dma_in_page, part_in_page;
  __device__ __forceinline__ CacheAt(const AttnArgs& a, int kvh) {
    k = apart(reinterpret_cast<uint64_t>(a.k) + kvh * a.kh);
    v = apart(reinterpret_cast<uint64_t>(a.v) + kvh * a.vh);
    kp = apart(a.kp), kt = apart(a.kt), vp = apart(a.vp), vt = apart(a.vt), page_mul = apart(a.page_mul);
    page_shift = apart(a.page_shift), page_size = apart(a.page_size), num_pages = apart(a.num_pages);
    dma_in_page = apart(a.dma_in_page), part_in_page = apart(a.part_in_page);
  }
  // The page index of token base + lane % KT of a tile (lanes behind its end: of its
  // last token), and the token's row there.
  template <int KT>
  __device__ __forceinline__ int page_index(const KeyTile& t, int* row) const {
    const int key = t.base + min(lane_now() % KT, t.count - 1);
    const int c = page_size == 1 ? key : static_cast<int>(__umulhi(key, page_mul) >> page_shift);
    *row = key - c * page_size;
    return c;
  }
  // The page numbers come through LDS, 64 of a wave's own.
  template <int KT>
  __device__ __forceinline__ void ask_pages(const KeyTile& t, lds_byte* to) const {
    int row;
    async_word(t.list + page_index<KT>(t, &row), to);
  }
  // Addresses of the rows of a tile, one a lane, and which of them are there; rows that
  // are not have the cache's first.
  struct RowsAt { uint64_t k, v; };
  template <int KT>
  __device__ __forceinline__ RowsAt find_rows(const KeyTile& t, const lds_byte* numbers, uint64_t* there) const {
    const int lane = lane_now();
    int row;
    page_index<KT>(t, &row);
    const int page = page_of(numbers);
    const bool ok = lane < min(KT, t.count) && page >= 0 && page < num_pages;
    *there = __ballot(ok);
    const uint32_t p = ok ? page : 0, r = ok ? row : 0;
    const auto far = [](uint32_t x, uint32_t y) { return static_cast<uint64_t>(x) * y; };
    return {k + 16 * (far(p, kp) + far(r, kt)), v + 16 * (far(p, vp) + far(r, vt))};
  }
  // Which rows of a tile are there, of the lane's page number.
  static __device__ __forceinline__ int page_of(const lds_byte* numbers) {
    return ((const __attribute__((address_space(3))) int32_t*)numbers)[lane_now()];
  }
  template <int KT>
  __device__ __forceinline__ uint64_t rows_there(const KeyTile& t, int page) const {
    constexpr uint64_t kAll = KT == 64 ? ~0ull : (1ull << (KT % 64)) - 1;
    const uint64_t valid = __ballot(static_cast<uint32_t>(page) < static_cast<uint32_t>(num_pages));
    return valid & (t.count >= KT ? kAll : (1ull << t.count) - 1);
  }
  // Address of row `key` of a tile, in page number `page`; of the cache's first unless ok.
  __device__ __forceinline__ uint64_t row_at(uint64_t from, uint32_t page_step, uint32_t step, int key, int page, bool ok) const {
    const uint32_t c = page_size == 1 ? key : __umulhi(key, page_mul) >> page_shift;
    const uint32_t p = ok ? page : 0, r = ok ? key - c * page_size : 0;
    return from + 16 * (static_cast<uint64_t>(p) * page_step + static_cast<uint64_t>(r) * step);
  }
};

__device__ __forceinline__ KeyRange apart_range(const KeyRange& k) {
  return {reinterpret_cast<const int32_t*>(apart(reinterpret_cast<uint64_t>(k.list0))),
          reinterpret_cast<const int32_t*>(apart(reinterpret_cast<uint64_t>(k.list1))), apart(k.first0), apart(k.count0),
          apart(k.first1), apart(k.count1)};
}

__device__ __forceinline__ uint64_t uniform_at(uint64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), lane),
                 hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), lane);
  return static_cast<uint64_t>(hi) << 32 | lo;
}
__device__ __forceinline__ uint64_t lane_at(uint64_t x, int lane) {
  const uint32_t lo = __shfl(static_cast<uint32_t>(x), lane, kWave), hi = __shfl(static_cast<uint32_t>(x >> 32), lane, kWave);
  return static_cast<uint64_t>(hi) << 32 | lo;
}

// DMA of rows [i0, i0 + N) kRowsPerDma of a tile into LDS; `stride`: of the rows, kt or vt.
// Where a DMA's rows lie in one page they are read from its first row's address on:
// rows behind the last token that way too, which are in the page and masked later.
template <typename T, int D, int N>
__device__ __forceinline__ void load_rows(const CacheAt<T, D>& c, uint64_t rows_at, uint32_t stride, lds_byte* to, int i0) {
  typedef KvRows<T, D> Rows;
  constexpr int RPD = Rows::kRowsPerDma;
  const int lane = lane_now(), j = lane / Rows::kPieces;
  const uint32_t piece = 16 * (lane % Rows::kPieces ^ Rows::swz(j)), row_off = 16 * j * stride;
  if (!rarely(!c.dma_in_page)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = (i0 + i) * RPD;
      async_piece(uniform_at(rows_at, r), row_off + (piece ^ 16 * Rows::swz(r)), to + (i0 + i) * 1024);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = (i0 + i) * RPD;
      const uint64_t at = lane_at(rows_at, r + j);
      async_piece(reinterpret_cast<const void*>(at + (piece ^ 16 * Rows::swz(r))), to + (i0 + i) * 1024);
    }
  }
}

// A wave's part of a workgroup's tile, N DMAs: rows N kRowsPerDma wave and on.  Where they
// lie in one page their address is a scalar, and vector instructions are left for the
// offsets of the pieces alone (the matrix unit leaves room for four a product, so each
// counts: 16 suffixes behind 8192 tokens 2.74 ms with an address for every row, 2.58 with one).
// `from`, `page_step`, `step`: of keys or values.
template <typename T, int D, int N, int KT>
__device__ __forceinline__ void load_part(const CacheAt<T, D>& c, uint64_t from, uint32_t page_step, uint32_t step, uint32_t row_off,
                                          uint32_t piece, int base, int page, uint64_t there, lds_byte* to, int wave) {
  typedef KvRows<T, D> Rows;
  constexpr int RPD = Rows::kRowsPerDma, P = N * RPD;
  to += N * wave * 1024;
  const int turn = 16 * Rows::swz(P * wave);
  if (!rarely(!c.part_in_page)) {
    const bool ok = there >> (P * wave) & 1;
    uint64_t at = c.row_at(from, page_step, step, base + P * wave, __builtin_amdgcn_readlane(page, P * wave), ok);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      async_piece(at, row_off + (piece ^ (turn ^ 16 * Rows::swz(RPD * i))), to + i * 1024);
      at += static_cast<uint64_t>(16 * RPD) * step;
    }
  } else {
    const int lane = lane_now(), r = lane % KT;
    const uint64_t rows = c.row_at(from, page_step, step, base + r, page, there >> r & 1);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t at = lane_at(rows, P * wave + RPD * i + lane / Rows::kPieces);
      async_piece(reinterpret_cast<const void*>(at + (piece ^ (turn ^ 16 * Rows::swz(RPD * i)))), to + i * 1024);
    }
  }
}

// Values of rows that are not there count as zeros.  drop: some rows of the item do
// not see some keys (weight zero), so what is not finite must not enter the products
// either; returns whether there was any in this thread's part (of `threads` threads),
// for add_dropped.
template <typename T, int D, int KT>
__device__ __forceinline__ bool clean_values(char* vl, uint64_t there, bool drop, int thread, int threads) {
  typedef KvRows<T, D> Rows;
  bool odd = false;
  asm volatile("" : "+v"(thread));
#pragma unroll 1
  for (int p = (drop ? 0 : __builtin_ctzll(~there)) * Rows::kPieces + thread; p < KT * Rows::kPieces; p += threads) {
    u32x4* at = reinterpret_cast<u32x4*>(vl + 16 * p);
    if (!(there >> (p / Rows::kPieces) & 1)) {
      *at = u32x4{0, 0, 0, 0};
    } else if (drop) {
      const u32x4 w = *at, f = finite_only<T>(w);
      if (w[0] != f[0] || w[1] != f[1] || w[2] != f[2] || w[3] != f[3]) {
        odd = true;
        *at = f;
      }
    }
  }
  return odd;
}

// ---------------------------------------------------------------- a wave's rows
constexpr float kSlack = 8.0f;   // m is so far above the maximum that it was taken at
template <typename T, int D>
struct AttnWave {
  typedef KvRows<T, D> Rows;
  typedef typename Mm<T>::R R;
  R q[D / 16];
  f32x16 o[D / 32];   // O^T: columns 32 dt + .. of row lane % 32
  float m, l;         // l: this half wave's part
  int frag0, col0;    // where the lane's operands of a tile's K and V begin
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    m = -INFINITY;
    l = 0.0f;
    frag0 = Rows::frag_start(threadIdx.x % kWave);
    col0 = Rows::col_start(threadIdx.x % kWave);
  }
  __device__ __forceinline__ void load_q(const T* row, uint32_t flip, int h) {
#pragma unroll
    for (int u = 0; u < D / 16; ++u) {
      float x[8];
      if constexpr (sizeof(T) == 2) {
        q[u] = Mm<T>::flip(__builtin_bit_cast(R, *reinterpret_cast<const u32x4*>(row + 16 * u + 8 * h)), flip);
      } else {
        load_run<T, 8>(row + 16 * u + 8 * h, x);
        q[u] = Mm<T>::flip(R{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}, flip);
      }
    }
  }
  // The rows' maxima over NB blocks of scores; O and l follow where one moves, by more than
  // `slack` (the same in both halves of a row).
  template <int NB>
  __device__ __forceinline__ void raise(const f32x16 (&s)[NB], float scale2, float slack) {
    float t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = s[0][k];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i % 4] = fmaxf(t[i % 4], s[b][i]);
    const float top = fmaf(half_max(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]))), scale2, kSlack);
    // each row by itself: what one row meets does not change another's rounding
    const bool moves = top > m + slack || m == -INFINITY;
    if (rarely(__any(moves))) {
      const float next = moves ? fmaxf(m, top) : m;
      const float keep = moves ? __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.0f : next)) : 1.0f;
      m = next;
      l *= keep;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] *= keep;
    }
  }
  // Scores of 16 keys into weights, two parts of four; p[k]: operand of 16 keys.  The scores stay.
  template <int NB>
  __device__ __forceinline__ void weigh4(const f32x16 (&s)[NB], R (&p)[2 * NB], float (&w)[8], int i0, float scale2, float at,
                                         float (&sum)[4]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[i0 % 8 + k] = __builtin_amdgcn_exp2f(fmaf(s[i0 / 16][i0 % 16 + k], scale2, -at));
    if (i0 % 8 == 4) p[i0 / 8] = Mm<T>::pack(w, sum);
  }
  // All of a tile; returns the sum of the weights (of this half wave).
  template <int NB>
  __device__ __forceinline__ float weigh(const f32x16 (&s)[NB], R (&p)[2 * NB], float scale2) const {
    const float at = m == -INFINITY ? 0.0f : m;
    float sum[4] = {}, w[8];
#pragma unroll
    for (int i = 0; i < 16 * NB; i += 4) weigh4(s, p, w, i, scale2, at, sum);
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // S^T of the tile's NB blocks of 32 keys; operands are read a step ahead of their
  // products.  With WEIGH the scores `s` become weights meanwhile (returned: their sum):
  // matrix and vector instructions take turns.
  template <int NB, bool WEIGH>
  __device__ __forceinline__ float scores(const char* kl, f32x16 (&next)[NB], const f32x16 (&s)[NB], R (&p)[2 * NB], float scale2,
                                          int lane) const {
    constexpr int U = D / 16, E = 16 * NB / U;   // scores for each step
    int first = frag0;
    asm volatile("" : "+v"(first));   // one value that the steps turn, not an expression for each
    R kf[2][NB];
    const auto load = [&](int u) {
#pragma unroll
      for (int b = 0; b < NB; ++b) kf[u & 1][b] = Rows::frag_at(kl + 32 * b * Rows::kPitch, first ^ Rows::kFragStep * u);
    };
    const float at = m == -INFINITY ? 0.0f : m;
    float sum[4] = {}, w[8];
    load(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u + 1 < U) load(u + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x16 zero;
#pragma unroll
        for (int i = 0; i < 16; ++i) zero[i] = 0.0f;
        next[b] = Mm<T>::mul(kf[u & 1][b], q[u], u == 0 ? zero : next[b]);
      }
      if constexpr (WEIGH) {
#pragma unroll
        for (int e = 0; e < (E + 3) / 4; ++e)
          if (E >= 4 || u % (4 / E) == 0) weigh4(s, p, w, E >= 4 ? E * u + 4 * e : 4 * (u / (4 / E)), scale2, at, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(sum[k]));   // made here, not where they are used first
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // O^T += V^T P^T over the tile's NB blocks of 32 keys
  template <int NB>
  __device__ __forceinline__ void values(const char* vl, const R (&p)[2 * NB], int lane) {
    constexpr int DT = D / 32, S = 2 * NB;
    int at = col0;
    asm volatile("" : "+v"(at));
    R vf[2][DT];
    const auto load = [&](int s) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vf[s & 1][dt] = Rows::col_frag(vl + 16 * s * Rows::kPitch, at, dt);
    };
    load(0);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (s + 1 < S) load(s + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = Mm<T>::mul(vf[s & 1][dt], p[s], o[dt]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // Scores of keys that the lane's row does not see: limit keys of the tile may be
  // seen, of those that are `there`.
  template <int NB>
  __device__ __forceinline__ void mask(f32x16 (&s)[NB], int limit, uint64_t there, int lane) {
    int h4 = lane / 32 * 4;
    asm volatile("" : "+v"(h4));   // what follows is made here, not kept in registers over the tiles
    const int left = limit - h4;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const uint32_t bits = static_cast<uint32_t>(there >> (32 * b)) >> h4;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i / 4) + i % 4;
        s[b][i] = 32 * b + key < left && (bits >> key & 1) ? s[b][i] : -INFINITY;
      }
    }
  }
};

// Waits for this wave's LDS accesses; keeps memory accesses on their side of it.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// ---------------------------------------------------------------- items
template <typename T, int D>
struct AttnLds {
  typedef KvRows<T, D> Rows;
  static constexpr int kTileKeys = kAttnWaves * (sizeof(T) == 2 ? kPartRows : kPartRowsF32);   // of a workgroup whose waves take rows of their own
  static constexpr int kTileBytes = kTileKeys * Rows::kPitch;
  static constexpr int kOwnBytes = 32 * Rows::kPitch;          // tiles of a wave that takes keys of its own
  static constexpr int kOffV = 2 * kTileBytes;                 // two of K, then two of V
  static constexpr int kRows = 4 * kTileBytes;
  static constexpr int kKeys = 2 * kAttnWaves * kOwnBytes;
  static constexpr int kMerge = kAttnWaves * D * kAttnRows * 4 + kAttnWaves * kAttnRows * 8;
  static constexpr int kMost = kRows > kKeys ? (kRows > kMerge ? kRows : kMerge) : (kKeys > kMerge ? kKeys : kMerge);
  static constexpr int kOffOdd = kMost;                        // a flag for each wave
  static constexpr int kOffPages = kOffOdd + 64;               // 64 page numbers for each wave
  static constexpr int kOffLine = kOffPages + 4 * kAttnThreads;
  static constexpr int kBytes = kOffLine + 12 * kStreamSeqs + 8;
};

// The kernel's arguments, loaded anew: what is used at the end alone is not kept in
// scalar registers over the loop.
__device__ __forceinline__ AttnArgs args_again() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttnArgs*)p;
}

struct AttnItem {
  int kvh;
  int row0;            // first row, counted over all packed rows
  int rows;            // of the item, from row0 on
  int len, tail;       // own tokens; row r of the item is token (row0 + r) / G, and sees own tokens below
  int first_row;       // tail + 1 + (row0 + r - first_row) / G
  KeyRange keys;
  int64_t part;        // its first wave tile among the partial results; < 0: it writes out
};

// Own tokens that row r of the item sees.
__device__ __forceinline__ int own_limit(const AttnItem& it, int groups, int r) {
  const int i = static_cast<int>(static_cast<uint32_t>(it.row0 - it.first_row + r) / static_cast<uint32_t>(groups));
  return max(min(it.tail + 1 + i, it.len), 0);
}

// The own tokens that every row of the item sees; INT_MAX if that is all there are.
__device__ __forceinline__ int least_limit(const AttnArgs& a, const AttnItem& it) {
  const int least = __builtin_amdgcn_readfirstlane(own_limit(it, a.groups, 0));
  return least < it.keys.first1 + it.keys.count1 ? least : INT_MAX;
}

// The token and query head of row r of the item.
struct RowAt { int64_t token; int head; };
__device__ __forceinline__ RowAt row_at(const AttnArgs& a, const AttnItem& it, int r) {
  const uint32_t row = it.row0 + r, token = row / static_cast<uint32_t>(a.groups);
  return {token, static_cast<int>(it.kvh * a.groups + (row - token * a.groups))};
}

// Adds the values that clean_values dropped to the outputs of the rows that see them:
// a weight is positive, so what is not finite stays itself.  Own keys from the first
// tile (of kt) that not all rows see; `limit`: the own keys that the lane's row sees;
// o: NT column blocks from dt0 on.  Rare, so small rather than fast.
template <typename T, int D, int NT>
__device__ __forceinline__ void add_dropped(const AttnArgs& a, const AttnItem& it, f32x16 (&o)[NT], int dt0, int limit, int kt,
                                            int lane) {
  const int end = it.keys.first1 + it.keys.count1;
  const char* head = static_cast<const char*>(a.v) + it.kvh * a.vh;
#pragma unroll 1
  for (int key = it.keys.first1 + max(own_limit(it, a.groups, 0) - it.keys.first1, 0) / kt * kt; key < end; ++key) {
    asm volatile("" : "+v"(lane));   // addresses are made here, not kept in registers over the keys
    const int page = it.keys.list1[key / a.page_size];
    if (page < 0 || page >= a.num_pages) continue;
    const T* row = reinterpret_cast<const T*>(
        head + 16 * (static_cast<uint64_t>(page) * a.vp + static_cast<uint64_t>(key % a.page_size) * a.vt));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = load_elt(row, 32 * (dt0 + t) + 8 * (i / 4) + 4 * (lane / 32) + i % 4);
        if (key < limit && not_finite(x)) o[t][i] += x;
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
  }
}

// The sum of a row's weights is zero where it sees no token, whose output is zero, and
// where all of its scores are -inf, which has none: 0 / 0.  The latter's sum becomes a NaN.
// Rare: whether any of the `tokens` first tokens of a list of pages lies in a page that is there.
__device__ __forceinline__ bool any_there(const AttnArgs& a, const int32_t* list, int tokens) {
#pragma unroll 1
  for (int c = 0; c * static_cast<int64_t>(a.page_size) < tokens; ++c)
    if (static_cast<uint32_t>(list[c]) < static_cast<uint32_t>(a.num_pages)) return true;
  return false;
}
__device__ __forceinline__ float sum_or_none(const AttnArgs& a, const int32_t* prefix, int count, const int32_t* own, int limit, float l) {
  if (l != 0.0f) return l;
  return any_there(a, prefix, count) || any_there(a, own, limit) ? __builtin_nanf("") : 0.0f;
}

template <typename T, int D>
__device__ __forceinline__ void store_out(const AttnArgs& a, const AttnItem& it, const f32x16& o, int dt, float l, int r, int lane) {
  if (r >= it.rows) return;
  const RowAt at = row_at(a, it, r);
  T* out = static_cast<T*>(a.out) + at.token * a.ldo + static_cast<int64_t>(at.head) * D + 32 * dt + 4 * (lane / 32);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = l == 0.0f ? 0.0f : o[4 * i4 + i] * inv;
    if constexpr (sizeof(T) == 2) {
      u32x2 w;
      w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2], x[3]}), bf16x2));
      *reinterpret_cast<u32x2*>(out + 8 * i4) = w;
    } else {
      *reinterpret_cast<f32x4*>(out + 8 * i4) = f32x4{x[0], x[1], x[2], x[3]};
    }
  }
}

// Results of wave tile `wt` of the item (rows 32 wt ..): out, or partial results.
template <typename T, int D>
__device__ __forceinline__ void put_columns(const AttnArgs& a, const AttnItem& it, int wt, const f32x16& o, int dt, float m, float l,
                                            int lane) {
  const int r = kAttnRows * wt + lane % 32;
  if (it.part < 0) {
    store_out<T, D>(a, it, o, dt, l, r, lane);
    return;
  }
  if (r >= it.rows) return;
  f32x4* p = a.part + ((it.part + wt) * (D / 8) + 4 * dt) * kWave + lane;
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) p[i4 * kWave] = f32x4{o[4 * i4], o[4 * i4 + 1], o[4 * i4 + 2], o[4 * i4 + 3]};
  if (dt == 0 && lane < 32) a.part_ml[(it.part + wt) * kAttnRows + lane] = f32x2{m, l};
}

// Waves take rows of their own and share tiles of keys, 64 for bf16 (two buffers each of K
// and V are 64 KB, so two workgroups fit a CU: with one 3.59 ms instead of 2.58).  Bound by
// the matrix cores and the vector instructions beside them, whose shares add up to most
// of the cycles (50 % and 155 instructions a tile), at the clock that the power limit
// leaves: 16 suffixes behind 8192 tokens 985 to 1068 TFLOP/s from card to card, a prompt of
// 8192 tokens 956 to 1033 (916 in the first 25 ms, until the clock has settled), 16 fp32
// suffixes of 1024 behind 4096 115.
template <typename T, int D>
__device__ __forceinline__ void attend_rows(const AttnArgs& a, const AttnItem& it, const CacheAt<T, D>& cache, char* lds) {
  typedef AttnLds<T, D> L;
  typedef typename L::Rows Rows;
  constexpr int KT = L::kTileKeys, NB = KT / 32, N = KT / Rows::kRowsPerDma / kAttnWaves;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int w0 = kAttnRows * wave, r = min(w0 + lane % 32, it.rows - 1);
  const RowAt mine_at = row_at(a, it, r);
  AttnWave<T, D> w;
  w.load_q(static_cast<const T*>(a.q) + mine_at.token * a.ldq + static_cast<int64_t>(mine_at.head) * D, a.flip, lane / 32);
  w.clear();
  const bool idle = w0 >= it.rows;
  const int mine = own_limit(it, a.groups, r);
  const int first = least_limit(a, it);   // of the workgroup, then the wave's least
  const int least = __builtin_amdgcn_readfirstlane(own_limit(it, a.groups, min(w0, it.rows - 1)));
  lds_byte* dst = (lds_byte*)lds;
  uint32_t* odd = reinterpret_cast<uint32_t*>(lds + L::kOffOdd);   // values were dropped
  if (threadIdx.x == 0) *odd = 0;
  const float scale2 = apart(a.scale2);
  const KeyRange keys = apart_range(it.keys);
  lds_byte* numbers = dst + L::kOffPages + 4 * kWave * wave;
  uint32_t piece, k_off, v_off;   // the lane's piece of a DMA, and where its row begins
  {
    const int j = lane / Rows::kPieces;
    piece = 16 * (lane % Rows::kPieces ^ Rows::swz(j)), k_off = 16 * j * cache.kt, v_off = 16 * j * cache.vt;
  }
  constexpr uint64_t kAll = KT == 64 ? ~0ull : (1ull << (KT % 64)) - 1;
  // While a tile's scores become weights and its values are added, the next one's
  // scores are formed, the next one's V and the K of the one after that come in, and
  // the page numbers of one more.  K and V of tile t lie in buffers t % 2.
  struct State { int base; bool own, any; uint64_t there; };
  State d0{}, d1{};   // the tile whose scores are formed, and the one whose K is here
  int page1 = 0;      // the lane's page number of d1
  KeyTile walk = first_tile(keys);
  if (walk.count > 0) cache.template ask_pages<KT>(walk, numbers);
  f32x16 sa[NB], sb[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) sa[b] = f32x16{};
  typename Mm<T>::R p[2 * NB];
  // SIDE: the buffers of d0's V; s: its scores, then those of d1 in `next`
  const auto step = [&](auto side, f32x16 (&s)[NB], f32x16 (&next)[NB]) {
    constexpr int SIDE = decltype(side)::value;
    wait_dma();
    lds_barrier();
    State d2{};
    int page2 = 0;
    if (d1.any)
      load_part<T, D, N, KT>(cache, cache.v, cache.vp, cache.vt, v_off, piece, d1.base, page1, d1.there,
                             dst + L::kOffV + (SIDE ^ 1) * L::kTileBytes, wave);
    if (walk.count > 0) {
      page2 = cache.page_of(numbers);
      d2.there = cache.template rows_there<KT>(walk, page2);
      load_part<T, D, N, KT>(cache, cache.k, cache.kp, cache.kt, k_off, piece, walk.base, page2, d2.there,
                             dst + SIDE * L::kTileBytes, wave);
      d2.base = walk.base;
      d2.own = walk.own;
      d2.any = true;
      next_tile<KT>(keys, walk);
      if (walk.count > 0) cache.template ask_pages<KT>(walk, numbers);
    }
    const char* kl = lds + (SIDE ^ 1) * L::kTileBytes;
    char* vl = lds + L::kOffV + SIDE * L::kTileBytes;
    // tiles that some rows of the workgroup do not see whole
    const bool partly = d0.own && first < d0.base + KT;
    if (rarely(d0.any && (d0.there != kAll || partly))) {
      if (clean_values<T, D, KT>(vl, d0.there, partly, threadIdx.x, kAttnThreads)) *odd = 1;
      lds_barrier();
      if (d0.there != kAll || least < d0.base + KT) w.mask(s, d0.own ? mine - d0.base : KT, d0.there, lane);
    }
    if (!idle) {
      // The maximum is looked at only where a row has none yet, or where weights turn out to
      // be large (a row's sum over a tile's half above 1, whose maximum becomes the largest
      // score then): the scores are there until then.
      // 35 vector instructions a tile less, and the moves that kept the scores (16 suffixes
      // behind 8192 tokens 2.64 -> 2.55 ms).
      // Without a tile d0 weights are made of whatever was there, without a tile d1 scores,
      // and not looked at.
      if (rarely(d0.any && __any(w.m == -INFINITY))) w.raise(s, scale2, kSlack);
      const bool scored = sizeof(T) == 2 || d1.any;   // (fp32's scores cost too much to be formed of nothing)
      float sum = 0.0f;
      if (scored) sum = w.template scores<NB, true>(kl, next, s, p, scale2, lane);
      if (d0.any) {
        if (rarely(!scored || __any(sum > 1.0f))) {
          w.raise(s, scale2, !scored ? kSlack : half_max(sum) > 1.0f ? 0.0f : INFINITY);
          sum = w.weigh(s, p, scale2);
        }
        w.l += sum;
        w.template values<NB>(vl, p, lane);
      }
    }
    d0 = d1;
    d1 = d2;
    page1 = page2;
  };
  while (true) {
    step(std::integral_constant<int, 0>(), sa, sb);
    if (!(d0.any || d1.any)) break;
    step(std::integral_constant<int, 1>(), sb, sa);
    if (!(d0.any || d1.any)) break;
  }
  lds_barrier();
  if (idle) return;
  w.l = half_sum(w.l);
  const AttnArgs e = args_again();
  if (rarely(__builtin_amdgcn_readfirstlane(*odd) != 0)) add_dropped<T, D>(e, it, w.o, 0, mine, KT, lane);
  if (rarely(it.part < 0 && __any(w.l == 0.0f))) w.l = sum_or_none(e, it.keys.list0, it.keys.count0, it.keys.list1, mine, w.l);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) put_columns<T, D>(e, it, wave, w.o[dt], dt, w.m, w.l, lane);
}

// At most 32 rows.  join: the waves take every fourth tile of the keys each, and their
// results are joined; else the item is this wave's alone.  Nothing but loads counts: a
// tile's K and V pass through LDS of the wave's own without a barrier, eight waves a CU keep
// up to 128 KB on the way.  128 single tokens behind up to 2047 own and 8192 shared ones:
// 90 us for 405 MB beside the shared items' products, 5 of them until the first tiles come
// (72 for the DMA alone).
template <typename T, int D>
__device__ __forceinline__ void attend_keys(const AttnArgs& a, const AttnItem& it, const CacheAt<T, D>& cache, bool join, char* lds) {
  typedef AttnLds<T, D> L;
  typedef typename L::Rows Rows;
  constexpr int KT = 32, N = KT / Rows::kRowsPerDma;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int r = min(lane % 32, it.rows - 1);
  const RowAt mine_at = row_at(a, it, r);
  AttnWave<T, D> w;
  w.load_q(static_cast<const T*>(a.q) + mine_at.token * a.ldq + static_cast<int64_t>(mine_at.head) * D, a.flip, lane / 32);
  w.clear();
  const int mine = own_limit(it, a.groups, r), least = least_limit(a, it);
  const char* kl = lds + wave * 2 * L::kOwnBytes;
  char* vl = lds + wave * 2 * L::kOwnBytes + L::kOwnBytes;
  lds_byte* kd = (lds_byte*)lds + wave * 2 * L::kOwnBytes;
  lds_byte* vd = kd + L::kOwnBytes;
  const float scale2 = apart(a.scale2);
  const KeyRange keys = apart_range(it.keys);
  bool odd = false;   // values were dropped
  const int step = join ? kAttnWaves : 1;
  lds_byte* numbers = (lds_byte*)lds + L::kOffPages + 4 * kWave * wave;
  constexpr uint64_t kAll = 0xFFFFFFFFull;
  // K of the next tile is on its way while the weights are made, its V while the next
  // scores are; pages are looked up a tile further ahead, between the two
  KeyTile cur{}, next = first_tile(keys);
  const auto skip = [&](int n) {
    for (int i = 0; i < n && next.count > 0; ++i) next_tile<KT>(keys, next);
  };
  skip(join ? wave : 0);
  uint64_t there = 0;
  bool any = false;
  if (next.count > 0) {
    cache.template ask_pages<KT>(next, numbers);
    wait_dma();
  }
  while (any || next.count > 0) {
    const bool now = any;
    const KeyTile was = cur;
    const uint64_t was_there = there;
    if (now) wait_dma_but<N>();   // its K and the next one's pages are here, V may be on its way
    f32x16 s[1];
    typename Mm<T>::R p[2];
    if (now) (void)w.template scores<1, false>(kl, s, s, p, scale2, lane);
    wait_lds();
    any = next.count > 0;
    typename CacheAt<T, D>::RowsAt at{};
    bool asked = false;
    if (any) {
      at = cache.template find_rows<KT>(next, numbers, &there);
      load_rows<T, D, N>(cache, at.k, cache.kt, kd, 0);
      cur = next;
      skip(step);
      asked = next.count > 0;
      if (asked) cache.template ask_pages<KT>(next, numbers);
    }
    if (now) {
      const int limit = was.own ? mine - was.base : KT;
      const bool whole = was_there == kAll && (!was.own || least >= was.base + KT);
      if (rarely(!whole)) w.mask(s, limit, was_there, lane);
      w.raise(s, scale2, kSlack);
      w.l += w.weigh(s, p, scale2);
      if (asked) wait_dma_but<N + 1>();
      else if (any) wait_dma_but<N>();
      else wait_dma();
      if (rarely(!whole)) {
        odd |= clean_values<T, D, KT>(vl, was_there, was.own && least < was.base + KT, lane, kWave);
        wait_lds();
      }
      w.template values<1>(vl, p, lane);
      wait_lds();
    }
    if (any) load_rows<T, D, N>(cache, at.v, cache.vt, vd, 0);
  }
  w.l = half_sum(w.l);
  odd = __any(odd);
  if (!join) {
    const AttnArgs e = args_again();
    if (rarely(odd)) add_dropped<T, D>(e, it, w.o, 0, mine, KT, lane);
    if (rarely(it.part < 0 && __any(w.l == 0.0f))) w.l = sum_or_none(e, it.keys.list0, it.keys.count0, it.keys.list1, mine, w.l);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) put_columns<T, D>(e, it, 0, w.o[dt], dt, w.m, w.l, lane);
    return;
  }
  // the waves' results into one: every wave's maximum, then the scaled sums of 32 columns a wave
  uint32_t* odds = reinterpret_cast<uint32_t*>(lds + L::kOffOdd);
  f32x4* os = reinterpret_cast<f32x4*>(lds);   // [wave][D / 8][lane]
  f32x2* mls = reinterpret_cast<f32x2*>(lds + kAttnWaves * D * kAttnRows * 4);
  lds_barrier();
  if (lane == 0) odds[wave] = odd;
  if (lane < 32) mls[wave * kAttnRows + lane] = f32x2{w.m, w.l};
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      os[(wave * (D / 8) + 4 * dt + i4) * kWave + lane] =
          f32x4{w.o[dt][4 * i4], w.o[dt][4 * i4 + 1], w.o[dt][4 * i4 + 2], w.o[dt][4 * i4 + 3]};
  lds_barrier();
  if (wave >= D / 32) return;
  float m = -INFINITY, l = 0.0f, f[kAttnWaves];
#pragma unroll
  for (int x = 0; x < kAttnWaves; ++x) m = fmaxf(m, mls[x * kAttnRows + lane % 32][0]);
  const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int x = 0; x < kAttnWaves; ++x) {
    const f32x2 ml = mls[x * kAttnRows + lane % 32];
    f[x] = __builtin_amdgcn_exp2f(ml[0] - base);
    l = fmaf(f[x], ml[1], l);
  }
  f32x16 o[1];
#pragma unroll
  for (int i4 = 0; i4 < 4; ++i4) {
    f32x4 sum = zero4();
#pragma unroll
    for (int x = 0; x < kAttnWaves; ++x) {
      const f32x4 p = os[(x * (D / 8) + 4 * wave + i4) * kWave + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = fmaf(f[x], p[i], sum[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) o[0][4 * i4 + i] = sum[i];
  }
#pragma unroll
  for (int x = 0; x < kAttnWaves; ++x) odd |= odds[x] != 0;
  const AttnArgs e = args_again();
  if (rarely(__builtin_amdgcn_readfirstlane(odd))) add_dropped<T, D>(e, it, o, wave, mine, KT, lane);
  if (rarely(it.part < 0 && __any(l == 0.0f))) l = sum_or_none(e, it.keys.list0, it.keys.count0, it.keys.list1, mine, l);
  put_columns<T, D>(e, it, 0, o[0], wave, m, l, lane);
}

// Largest n in [0, N) with cu[n] G / tile + n <= slot (see slot_seq).
__device__ __forceinline__ int row_slot_seq(const int32_t* __restrict__ cu, int n_seqs, int slot, int groups, int tile) {
  const int lane = threadIdx.x % kWave;
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int at = lo + lane * step;
    const bool below = at < hi && static_cast<int64_t>(cu[at]) * groups / tile + at <= slot;
    const int found = __popcll(__ballot(below));
    lo += (found - 1) * step;
    hi = min(hi, lo + step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Batches of a few rows a sequence (own_tile 32: single tokens): lengths differ, and
// the last long sequence would keep the memory waiting.  So the own tokens of all
// sequences, in tiles of 32 keys, are one line, of which each wave takes an equal share for
// one K/V head: the end of one sequence's, all of some, the beginning of another's.  The
// waves of a workgroup take the heads of the same tokens, which lie beside each other in
// memory (128 single tokens 104.5 us with every head's tiles after one another, 101.7 so).
// Waves work alone, without barriers, so that the start of
// one share (offsets, pages, first rows: one memory access after another) hides behind
// the others' loads.  A sequence that is one wave's is done (or one part of it is, where
// there is a prefix); of one that is shared out each wave leaves its part: the first of
// them at 2 wave + 1, the others at 2 wave.
constexpr int kLineTile = 32;

// The line of one K/V head: tiles[n] before sequence n (which has one where it has
// queries but no tokens), tiles[N] in all; and the sequences' first tokens and lengths.
struct Line {
  int* tiles;
  int* cu;
  int* lens;
};
template <typename T, int D>
__device__ __forceinline__ Line line_at(char* lds) {
  int* p = reinterpret_cast<int*>(lds + AttnLds<T, D>::kOffLine);
  return {p, p + kStreamSeqs + 1, p + 2 * kStreamSeqs + 2};
}
// `keep`: for the joining kernel as well.
template <typename T, int D>
__device__ __forceinline__ void lay_line(const AttnArgs& a, char* lds, bool keep) {
  const Line line = line_at<T, D>(lds);
  int* sums = reinterpret_cast<int*>(lds);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int total = 0;
  for (int n0 = 0; n0 < a.n_seqs; n0 += kAttnThreads) {
    const int n = n0 + threadIdx.x;
    int mine = 0;
    if (n < a.n_seqs) {
      const int start = a.cu[n], end = a.cu[n + 1], len = min(max(a.lens[n], 0), a.max_len);
      if (end > start) mine = max(1, (len + kLineTile - 1) / kLineTile);
      line.cu[n] = start;
      line.lens[n] = len;
      if (n == a.n_seqs - 1) line.cu[n + 1] = end;
      if (keep)
        for (int t = start; t < end; ++t) a.line[a.n_seqs + 1 + t] = n;
    }
    int up_to = mine;   // inclusive sums over the wave
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int up = __shfl_up(up_to, off, kWave);
      up_to += lane >= off ? up : 0;
    }
    if (lane == kWave - 1) sums[wave] = up_to;
    lds_barrier();
    int before = total;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      before += w < wave ? sums[w] : 0;
      total += sums[w];
    }
    if (n < a.n_seqs) {
      line.tiles[n] = before + up_to - mine;
      if (keep) a.line[n] = before + up_to - mine;
    }
    lds_barrier();
  }
  if (threadIdx.x == 0) {
    line.tiles[a.n_seqs] = total;
    if (keep) a.line[a.n_seqs] = total;
  }
  lds_barrier();
}
// Shares of a line of `total` tiles, each taken by a wave for every K/V head: no more than
// leave each as many tiles as balance its walk with the joining of the parts (a tile of a
// lonely wave takes about 1.3 us, 16 parts of a row 0.6).
__device__ __forceinline__ int line_shares(const AttnArgs& a, int total) {
  const int least = max(1, static_cast<int>(ceilf(sqrtf(static_cast<float>(total) / (32.0f * a.n_seqs)))));
  const uint32_t most = static_cast<uint32_t>(total + least - 1) / static_cast<uint32_t>(least);
  return __builtin_amdgcn_readfirstlane(min(static_cast<int>(most), a.stream_waves / a.kv_heads));
}
// Equal shares, the first ones a tile longer where it does not come out even.
__device__ __forceinline__ int share_start(uint32_t tiles, uint32_t shares, int s) {
  return s * static_cast<int>(tiles / shares) + min(s, static_cast<int>(tiles % shares));
}
__device__ __forceinline__ int share_of(uint32_t tiles, uint32_t shares, uint32_t t) {   // the share that holds tile t
  const uint32_t each = tiles / shares, longer = tiles % shares, behind = longer * (each + 1);
  return static_cast<int>(t < behind ? t / (each + 1) : longer + (t - behind) / each);
}

// The items of a wave, one after another; those of a workgroup come to all of its waves.
struct AttnWork {
  int shared, shared_step;   // the next shared item
  int at, end;               // what is left of the share of the line
  int wave, kvh;             // of the line
  bool own_first;
};
enum class AttnKind { kNone, kRows, kKeys, kWave };

__device__ __forceinline__ void shared_item(const AttnArgs& a, int b, AttnItem& it) {
  // [split][row tile][K/V head]
  it.kvh = b % a.kv_heads;
  const int u = b / a.kv_heads, tile = u % a.shared_tiles, split = u / a.shared_tiles;
  it.row0 = tile * kAttnTile;
  it.rows = min(kAttnTile, a.rows - it.row0);
  it.len = it.tail = 0;
  it.first_row = it.row0;
  const int first = split * a.shared_chunk;
  it.keys = {a.prefix_pages, nullptr, first, min(a.shared_chunk, a.prefix_len - first), 0, 0};
  it.part = ((static_cast<int64_t>(split) * a.shared_tiles + tile) * a.kv_heads + it.kvh) * a.shared_wt;
}
__device__ __forceinline__ bool own_item(const AttnArgs& a, int b, AttnItem& it) {
  // [slot, the last first][split][K/V head]
  it.kvh = b % a.kv_heads;
  const int u = b / a.kv_heads, split = u % a.own_splits, slot = a.own_slots - 1 - u / a.own_splits;
  const int n = row_slot_seq(a.cu, a.n_seqs, slot, a.groups, a.own_tile);
  const int start = a.cu[n], count = a.cu[n + 1] - start;
  it.first_row = start * a.groups;
  const int from = (slot - (it.first_row / a.own_tile + n)) * a.own_tile;
  const int left = count * a.groups - from;
  if (left <= 0) return false;
  it.row0 = it.first_row + from;
  it.rows = min(a.own_tile, left);
  it.len = min(max(a.lens[n], 0), a.max_len);
  it.tail = it.len - count;
  const int end = own_limit(it, a.groups, it.rows - 1);
  const int64_t first = static_cast<int64_t>(split) * a.own_chunk;
  const int64_t own = min(static_cast<int64_t>(a.own_chunk), end - first);
  it.keys = {a.prefix_pages, a.table + static_cast<int64_t>(n) * a.width, 0, a.shared_items == 0 ? a.prefix_len : 0,
             static_cast<int>(first), static_cast<int>(max(own, static_cast<int64_t>(0)))};
  it.part = a.part ? static_cast<int64_t>(a.shared_items) * a.shared_wt +
                         ((static_cast<int64_t>(slot) * a.own_splits + split) * a.kv_heads + it.kvh) * (a.own_tile / kAttnRows)
                   : -1;
  return true;
}
__device__ __forceinline__ void line_item(const AttnArgs& a, const Line& line, AttnWork& w, AttnItem& it) {
  // the last sequence that begins at the tile or before it; 64 candidates at a time
  const int t = w.at, lane = threadIdx.x % kWave;
  int lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const int found = __popcll(__ballot(at < hi && line.tiles[min(at, hi)] <= t));
    lo += (found - 1) * step;
    hi = min(hi, lo + step);
  }
  const int n = __builtin_amdgcn_readfirstlane(lo);
  const int begin = __builtin_amdgcn_readfirstlane(line.tiles[n]),
            tiles = __builtin_amdgcn_readfirstlane(line.tiles[n + 1]) - begin;
  const int off = t - begin, take = min(w.end - t, tiles - off);
  it.kvh = w.kvh;
  const int start = __builtin_amdgcn_readfirstlane(line.cu[n]),
            count = __builtin_amdgcn_readfirstlane(line.cu[n + 1]) - start;
  it.row0 = it.first_row = start * a.groups;
  it.rows = count * a.groups;
  it.len = __builtin_amdgcn_readfirstlane(line.lens[n]);
  it.tail = it.len - count;
  const int first = off * kLineTile;
  it.keys = {nullptr, a.table + static_cast<int64_t>(n) * a.width, 0, 0, first, min(take * kLineTile, it.len - first)};
  const int64_t base = static_cast<int64_t>(a.shared_items) * a.shared_wt;
  if (take < tiles) it.part = base + 2 * w.wave + (off == 0);
  else it.part = a.shared_items ? base + 2 * a.stream_waves + static_cast<int64_t>(n) * a.kv_heads + it.kvh : -1;
  w.at += take;
}
__device__ __forceinline__ AttnKind next_item(const AttnArgs& a, const Line& line, AttnWork& w, AttnItem& it) {
  const bool shared = w.shared < a.shared_items, own = w.at < w.end;
  if (shared && !(own && w.own_first)) {
    shared_item(a, w.shared, it);
    w.shared += w.shared_step;
    return a.shared_wt == 1 ? AttnKind::kWave : it.rows > kAttnRows ? AttnKind::kRows : AttnKind::kKeys;
  }
  if (!own) return AttnKind::kNone;
  if (a.stream) {
    line_item(a, line, w, it);
    return AttnKind::kWave;
  }
  w.at = w.end;
  if (!own_item(a, static_cast<int>(blockIdx.x) - a.shared_items, it)) return AttnKind::kNone;
  return it.rows > kAttnRows ? AttnKind::kRows : AttnKind::kKeys;
}

template <typename T, int D>
__global__ __launch_bounds__(kAttnThreads, sizeof(T) == 2 ? 2 : 1)
void k_attn(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[AttnLds<T, D>::kBytes];
  const Line line = line_at<T, D>(lds);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), group = blockIdx.x;
  AttnWork work{};
  work.shared = a.shared_wt == 1 ? kAttnWaves * group + wave : group;
  work.shared_step = a.shared_wt == 1 ? kAttnWaves * gridDim.x : gridDim.x;
  if (!a.stream) {
    work.end = group >= a.shared_items;   // one own item, or none
    if (work.end) work.shared = a.shared_items;
    else work.shared_step = a.shared_items;
  } else {
    if (group >= a.stream_first && kAttnWaves * (group - a.stream_first) < a.stream_waves) {
      if (a.stream_first > 0) work.shared = a.shared_items;   // there are others for these
      lay_line<T, D>(a, lds, group == a.stream_first);
      const int total = __builtin_amdgcn_readfirstlane(line.tiles[a.n_seqs]);
      // the waves of a workgroup walk the same tokens' K/V heads, which lie beside each other
      const int shares = line_shares(a, total);
      work.wave = kAttnWaves * (group - a.stream_first) + wave;
      const int share = static_cast<int>(static_cast<uint32_t>(work.wave) / static_cast<uint32_t>(a.kv_heads));
      work.kvh = work.wave - share * a.kv_heads;
      if (share < shares) {
        work.at = share_start(total, shares, share);
        work.end = share_start(total, shares, share + 1);
      }
    }
    // shared items compute, own ones wait for memory: half of the workgroups begin with
    // the one, half with the other
    work.own_first = group >= static_cast<int>(gridDim.x) / 2;
  }
  while (true) {
    const AttnArgs e = args_again();
    AttnItem it;
    const AttnKind kind = next_item(e, line, work, it);
    if (kind == AttnKind::kNone) break;
    const CacheAt<T, D> cache(e, it.kvh);
    if (kind != AttnKind::kWave) lds_barrier();   // the LDS of the item before has been read
    if (kind == AttnKind::kRows) attend_rows<T, D>(e, it, cache, lds);
    else attend_keys<T, D>(e, it, cache, kind == AttnKind::kKeys, lds);
    if (kind != AttnKind::kWave) lds_barrier();
  }
}

// The items' partial results of a row into one.  A workgroup takes 32 packed rows of a
// K/V head, lane (h, r) four columns of row r at a time.  SPREAD, for many parts: one of the
// D / 8 groups of columns a workgroup, a wave every fourth part (11 us for 128 single tokens of
// 32 heads with 12 parts each, 32 MB; 5 for one: a chain of loads).  Else a wave takes a quarter
// of the columns and all parts (two parts of 512 tokens, 17 MB: 5.9 us, 15 the other way).
// kAttnAhead parts' loads are in flight at a time.
constexpr int kAttnAhead = 4;
template <typename T, int D, bool SPREAD>
__global__ __launch_bounds__(kAttnThreads)
void k_attn_join(AttnArgs a) {
  constexpr int COLS = SPREAD ? 1 : D / 8 / kAttnWaves, AHEAD = SPREAD ? kAttnAhead : kAttnAhead / 2;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int unit = SPREAD ? blockIdx.x / (D / 8) : blockIdx.x, col = SPREAD ? blockIdx.x % (D / 8) : COLS * wave;
  const int kvh = unit % a.kv_heads, wt = unit / a.kv_heads;
  const bool there = wt * kAttnRows + lane % 32 < a.rows;
  const int row = there ? wt * kAttnRows + lane % 32 : a.rows - 1;
  const int token = static_cast<int>(static_cast<uint32_t>(row) / static_cast<uint32_t>(a.groups));
  int lo = 0;   // the sequence of the token: the first whose end lies behind it
  if (a.stream) {
    lo = a.line[a.n_seqs + 1 + token];
  } else {
    int hi = a.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.cu[mid + 1] > token) hi = mid;
      else lo = mid + 1;
    }
  }
  const int first = a.cu[lo] * a.groups, rs = row - first;
  // where the row is among the wave tiles of part s: those of the shared items are these
  // rows, those of the own ones are found by sequence
  const int64_t shared0 = (static_cast<int64_t>(wt / a.shared_wt) * a.kv_heads + kvh) * a.shared_wt + wt % a.shared_wt,
                shared_step = static_cast<int64_t>(a.shared_tiles) * a.kv_heads * a.shared_wt,
                base = static_cast<int64_t>(a.shared_items) * a.shared_wt;
  int64_t own0, own_step;   // the first of the own parts (what follows: a step behind), and the steps
  int own = a.own_splits;
  if (a.stream) {
    const int before = a.line[lo], mine = a.line[lo + 1] - before, total = a.line[a.n_seqs];
    const int shares = line_shares(a, total), w0 = share_of(total, shares, before);
    own = share_of(total, shares, before + mine - 1) - w0 + 1;
    own_step = 2 * a.kv_heads;
    own0 = own == 1 ? base + 2 * a.stream_waves + static_cast<int64_t>(lo) * a.kv_heads + kvh
                    : base + 2 * (static_cast<int64_t>(w0) * a.kv_heads + kvh);   // (its first part one behind)
  } else {
    const int slot = first / a.own_tile + lo + rs / a.own_tile;
    own_step = static_cast<int64_t>(a.kv_heads) * (a.own_tile / kAttnRows);
    own0 = base + (static_cast<int64_t>(slot) * a.own_splits * a.kv_heads + kvh) * (a.own_tile / kAttnRows) +
           rs % a.own_tile / kAttnRows;
  }
  const bool split = a.stream && own > 1;
  const bool done = a.stream && own == 1 && a.shared_splits == 0;   // its item wrote it out
  const int parts = there && !done ? a.shared_splits + own : 0;
  int most = parts;   // over the lanes
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) most = max(most, __shfl_xor(most, off, kWave));
  most = __builtin_amdgcn_readfirstlane(most);
  if (most == 0) return;
  const int own_row = a.stream ? rs : rs % kAttnRows;
  float m = -INFINITY, l = 0.0f;
  f32x4 sum[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) sum[c] = zero4();
  constexpr int STEP = SPREAD ? kAttnWaves : 1;
  for (int s0 = SPREAD ? wave : 0; s0 < most; s0 += STEP * AHEAD) {
    f32x2 ml[AHEAD];
    f32x4 x[AHEAD][COLS];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int s = max(min(s0 + STEP * k, parts - 1), 0), so = s - a.shared_splits;
      const int64_t t = so < 0 ? shared0 + s * shared_step : own0 + so * own_step + (split && so == 0);
      const int r = so < 0 ? lane % 32 : own_row;
      ml[k] = f32x2{-INFINITY, 0.0f};
#pragma unroll
      for (int c = 0; c < COLS; ++c) x[k][c] = zero4();
      if (s0 + STEP * k < parts) {
        ml[k] = a.part_ml[t * kAttnRows + r];
#pragma unroll
        for (int c = 0; c < COLS; ++c) x[k][c] = a.part[(t * (D / 8) + col + c) * kWave + lane / 32 * 32 + r];
      }
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, ml[k][0]);
    const float at = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - at);
    m = top;
    l *= keep;
#pragma unroll
    for (int c = 0; c < COLS; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[c][i] *= keep;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      // (a part without weights too: a value that is not finite counts at a weight of nothing)
      const float f = __builtin_amdgcn_exp2f(ml[k][0] - at);
      l = fmaf(f, ml[k][1], l);
#pragma unroll
      for (int c = 0; c < COLS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[c][i] = fmaf(f, x[k][c][i], sum[c][i]);
    }
  }
  if constexpr (SPREAD) {
    __shared__ f32x4 sums[kAttnWaves][kWave];
    __shared__ f32x2 mls[kAttnWaves][kWave];
    sums[wave][lane] = sum[0];
    mls[wave][lane] = f32x2{m, l};
    lds_barrier();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) m = fmaxf(m, mls[w][lane][0]);
    const float at = m == -INFINITY ? 0.0f : m;
    l = 0.0f;
    sum[0] = zero4();
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const f32x2 ml = mls[w][lane];
      const float f = __builtin_amdgcn_exp2f(ml[0] - at);
      l = fmaf(f, ml[1], l);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[0][i] = fmaf(f, sums[w][lane][i], sum[0][i]);
    }
  }
  if (parts == 0) return;
  if (rarely(__any(l == 0.0f))) {
    const int count = a.cu[lo + 1] - a.cu[lo], len = min(max(a.lens[lo], 0), a.max_len);
    l = sum_or_none(a, a.prefix_pages, a.prefix_len, a.table + static_cast<int64_t>(lo) * a.width,
                    max(min(len - count + 1 + (token - a.cu[lo]), len), 0), l);
  }
  const int head = kvh * a.groups + (row - token * a.groups);
  T* out = static_cast<T*>(a.out) + token * a.ldo + static_cast<int64_t>(head) * D + 8 * col + 4 * (lane / 32);
  const float inv = 1.0f / l;
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = l == 0.0f ? 0.0f : sum[c][i] * inv;
    if constexpr (sizeof(T) == 2) {
      u32x2 w;
      w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[0], y[1]}), bf16x2));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[2], y[3]}), bf16x2));
      *reinterpret_cast<u32x2*>(out + 8 * c) = w;
    } else {
      *reinterpret_cast<f32x4*>(out + 8 * c) = f32x4{y[0], y[1], y[2], y[3]};
    }
  }
}

}  // namespace gdn
