// The chunked selective state space scan on the matrix cores.
//
// A workgroup holds the states of a few heads of one sequence (or of one
// segment of it) in registers and walks its 64-token chunks.  With G the
// chunk's inclusive cumulative log alpha and M0 the state before it,
//   y  = diag(e^G) C M0 + ((C B^T) o L o delta_j) x + d_skip x,
//   M <- e^{G_last} M0 + B^T diag(e^{G_last - G_j} delta_j) x,
//   L_ij = e^{G_i - G_j} for j <= i.
// A wave owns 16 CT state columns of one head; the waves of a head share the
// decayed products P = (C B^T) o L o delta_j through LDS, and the heads of a
// workgroup, which are of one B/C group, share the B and C rows and C B^T.
//
// What bounds it: a chunk is a chain (rows into LDS, C B^T, P, P x) between
// products on the state, and matrix and vector instructions of a SIMD's waves
// hardly overlap.  Measured, bf16: 16 sequences of 128 to 2048 tokens, 32
// heads of 128 x 128, 198 us (498 MB, 2.5 TB/s); one of 32768 tokens, 64 heads of
// 64 x 128, in segments 342 us: 117 for the segments' states, 12 for the join
// and 226 for the outputs at best, each more where the chip's power limit lowers
// its clock.  States alone: 82 and 119 us.  Of the outputs' time, found by leaving out one stage's arithmetic:
// the split of M into parts 35, the products on M 42, the state's update 37, P 34,
// the stores 23, the loads 16, C B^T 11.  fp32 inputs go through k = 4 products
// (2048 tokens, 4 heads of 64 x 64: 23 us a call in segments).
#pragma once

#include <type_traits>

#include "gdn_varlen.h"

namespace gdn {

constexpr int kSsmChunk = 64;

// ---------------------------------------------------------------- operands
// Matrix operands of an element type: R is an operand taken from the inputs as
// it is; F2 and F3 carry fp32 values.  bf16 inputs: F2 is two bf16 parts (within
// 2^-16 of the value), for what ends in a bf16 output; F3 is three (24 bits),
// for the states.  fp32 inputs: every operand is the fp32 value itself, and a
// k = 32 product is eight k = 4 ones (slot 8 g + j of the k step is element j of
// lane group g, so operands are laid out as for bf16).
template <typename T>
struct Mx;

// x rounded to a bf16 pair, and what the rounding left of it (exact).
__device__ __forceinline__ uint32_t round_pair(f32x2& x) {
  const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
  x[0] -= __uint_as_float(h << 16);
  x[1] -= __uint_as_float(h & 0xFFFF0000u);
  return h;
}
__device__ __forceinline__ uint32_t last_pair(const f32x2& x) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

template <>
struct Mx<uint16_t> {
  typedef bf16x8 R;
  struct F2 { R part[2]; };
  struct F3 { R part[3]; };
  template <int N>
  static __device__ __forceinline__ void split(const float (&v)[8], R (&part)[N]) {
    u32x4 w[N];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      f32x2 x = {v[2 * p], v[2 * p + 1]};
#pragma unroll
      for (int k = 0; k < N - 1; ++k) w[k][p] = round_pair(x);
      w[N - 1][p] = last_pair(x);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) part[k] = __builtin_bit_cast(R, w[k]);
  }
  // an F2 operand in LDS: 64 lanes x 16 bytes of high parts, then of low parts
  static constexpr int kF2Bytes = 2048;
  static __device__ __forceinline__ void put4(char* frag, int slot, int half, const float (&v)[4]) {
    u32x2 hi, lo;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f32x2 x = {v[2 * p], v[2 * p + 1]};
      hi[p] = round_pair(x);
      lo[p] = last_pair(x);
    }
    *reinterpret_cast<u32x2*>(frag + 16 * slot + 8 * half) = hi;
    *reinterpret_cast<u32x2*>(frag + 1024 + 16 * slot + 8 * half) = lo;
  }
  static __device__ __forceinline__ F2 get(const char* frag, int lane) {
    F2 f;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      f.part[k] = __builtin_bit_cast(R, *reinterpret_cast<const u32x4*>(frag + 1024 * k + 16 * lane));
    return f;
  }
  static __device__ __forceinline__ float elt(const R& r, int j) {
    const u32x4 w = __builtin_bit_cast(u32x4, r);
    return __uint_as_float((j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16));
  }
  static __device__ __forceinline__ f32x4 mul(const R& a, const R& b, f32x4 c) { return mma(a, b, c); }
};

template <>
struct Mx<float> {
  typedef f32x8 R;
  struct F2 { R part[1]; };
  struct F3 { R part[1]; };
  static __device__ __forceinline__ void split(const float (&v)[8], R (&part)[1]) {
    part[0] = R{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  }
  static constexpr int kF2Bytes = 2048;   // 64 lanes x 32 bytes
  static __device__ __forceinline__ void put4(char* frag, int slot, int half, const float (&v)[4]) {
    *reinterpret_cast<f32x4*>(frag + 32 * slot + 16 * half) = f32x4{v[0], v[1], v[2], v[3]};
  }
  static __device__ __forceinline__ F2 get(const char* frag, int lane) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(frag + 32 * lane);
    const f32x4 b = *reinterpret_cast<const f32x4*>(frag + 32 * lane + 16);
    return {{R{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}}};
  }
  static __device__ __forceinline__ float elt(const R& r, int j) { return r[j]; }
  static __device__ __forceinline__ f32x4 mul(const R& a, const R& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};
template <typename F>
constexpr int parts_of() { return sizeof(F::part) / sizeof(typename std::remove_extent<decltype(F::part)>::type); }

// ---------------------------------------------------------------- token rows in LDS
// 64 rows of D elements.  bf16: 16-byte pieces swizzled as key rows are
// (row_swz: 16-byte operand reads without bank conflicts, transposing reads with
// the fewest there are).  fp32: rows padded by 16 bytes.
template <typename T, int D>
struct RowsLds {
  static constexpr int kPieces = D * static_cast<int>(sizeof(T)) / 16;   // of a row
  static constexpr int kPitch = sizeof(T) == 2 ? 2 * D : 4 * D + 16;
  static constexpr int kBytes = kSsmChunk * kPitch;
  // The swizzle repeats every 16 rows, so a row's address may be taken from any
  // row a multiple of 16 above it.
  static __device__ __forceinline__ int at(int row, int piece) {
    if constexpr (sizeof(T) == 2) return row * kPitch + ((piece ^ row_swz<kPitch>(row)) << 4);
    else return row * kPitch + (piece << 4);
  }
  // elements 8 e8 .. + 7 of row `up` + row, up a multiple of 16
  static __device__ __forceinline__ typename Mx<T>::R row_frag(const char* base, int up, int row, int e8) {
    base += up * kPitch;
    if constexpr (sizeof(T) == 2) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(base + at(row, e8)));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(base + at(row, 2 * e8));
      const f32x4 b = *reinterpret_cast<const f32x4*>(base + at(row, 2 * e8 + 1));
      return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  }
  // rows up + 8 g + j (j = 0..7; up a multiple of 32) of column col32 + 8 (c / 4) + 4 half + c % 4, for lane (g, c)
  static __device__ __forceinline__ typename Mx<T>::R col_frag(const char* base, int up, int col32, int half, int g,
                                                               int c) {
    base += up * kPitch;
    if constexpr (sizeof(T) == 2) {
      // lane 4 t + q of a group of 16 supplies four elements of row t, columns 8 q ..; lane i receives
      // column 8 (i / 4) + i % 4 of rows 0..3
      const int row = 8 * g + c / 4, piece = col32 / 8 + c % 4;
      const u32x2 a = lds_read_tr16(base + at(row, piece) + 8 * half);
      const u32x2 b = lds_read_tr16(base + at(row + 4, piece) + 8 * half);
      return join_halves(a, b);
    } else {
      const float* p = reinterpret_cast<const float*>(base + 8 * g * kPitch) + col32 + 8 * (c / 4) + 4 * half + c % 4;
      f32x8 r;
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = p[j * (kPitch / 4)];
      return r;
    }
  }
  // writes elements 8 e8 .. + 7 of row `up` + row
  static __device__ __forceinline__ void put8(char* base, int up, int row, int e8, const float (&x)[8]) {
    base += up * kPitch;
    if constexpr (sizeof(T) == 2) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 pair = {x[2 * j], x[2 * j + 1]};
        w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2));
      }
      *reinterpret_cast<u32x4*>(base + at(row, e8)) = w;
    } else {
      *reinterpret_cast<f32x4*>(base + at(row, 2 * e8)) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4*>(base + at(row, 2 * e8 + 1)) = f32x4{x[4], x[5], x[6], x[7]};
    }
  }
  // address of row + k STEP
  template <int STEP>
  static __device__ __forceinline__ int at_step(int row, int k, int piece) {
    if constexpr (STEP % 16 == 0) return at(row, piece) + k * STEP * kPitch;
    else return at(row + k * STEP, piece);
  }
};

// Raw buffer of `bytes` bytes: a load behind its end gives zero, a store is dropped.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}

// Per head and chunk, in base 2: with l the inclusive cumulative log alpha inside
// a token's 16-token tile and s what is left of the tile after it, e^{G_i - G_j}
// = 2^(l_i - l_j) within a tile and 2^l_i 2^between 2^s_j across tiles, three
// factors of at most one, so no factor overflows.  Across tiles exponents are sums
// of terms of one sign.  Within a tile they are the difference of two sums that
// may be far longer (l reaches -2400, where fp32 steps by 2^-12: outputs off by
// 1e-4): l is summed in 64 bits there and kept as two floats, whose differences
// are as good as the sum of the steps between.
struct HeadScalars {
  float high[kSsmChunk];   // l rounded
  float low[kSsmChunk];    // l - high
  float same[kSsmChunk];   // log2 delta - low
  float row[kSsmChunk];    // 2^l
  float past[kSsmChunk];   // 2^s delta
  float pre[kSsmChunk];    // e^G
  float suf[kSsmChunk];    // e^{G_last - G} delta
  float between[10];       // 2^(log2 alpha summed over the tiles between those of tile pair t), see tile_rows
  float total;             // e^{G_last}
  float pad[5];
};

// Lane exchanges inside a DPP row of 16 lanes; a lane without a source gets 0.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Inclusive sums along the row: SHIFT 0x110 (row_shr) from its start, 0x100 (row_shl) from its end.
template <int SHIFT>
__device__ __forceinline__ float row_scan(float x) {
  x += dpp<SHIFT + 1>(x);
  x += dpp<SHIFT + 2>(x);
  x += dpp<SHIFT + 4>(x);
  x += dpp<SHIFT + 8>(x);
  return x;
}
// The same from the row's start, in 64 bits.
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double row_scan_wide(double x) {
  x += dpp<0x111>(x);
  x += dpp<0x112>(x);
  x += dpp<0x114>(x);
  x += dpp<0x118>(x);
  return x;
}
__device__ __forceinline__ float read_lane(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// Sequences cut into segments of `tokens`, an empty one into one: the sequence n
// and its segment j that segment number `unit` is, counted over all of them.
// The wave looks at 64 sequences at a time; uniform over the wave.
struct SegmentAt { int n, j; };
__device__ __forceinline__ int segments_of(const int32_t* __restrict__ cu, int n_seqs, int i, int tokens) {
  return i < n_seqs ? max(1, (cu[i + 1] - cu[i] + tokens - 1) / tokens) : 0;
}
__device__ __forceinline__ int wave_scan(int x) {   // inclusive sums over the wave
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int up = __shfl_up(x, off, kWave);
    x += lane >= off ? up : 0;
  }
  return x;
}
__device__ __forceinline__ SegmentAt segment_at(const int32_t* __restrict__ cu, int n_seqs, int tokens, int unit) {
  const int lane = threadIdx.x % kWave;
  for (int n0 = 0;; n0 += kWave) {   // unit is below the number of segments
    const int sum = wave_scan(segments_of(cu, n_seqs, n0 + lane, tokens));
    const int total = __builtin_amdgcn_readlane(sum, kWave - 1);
    if (unit < total || n0 + kWave >= n_seqs) {
      const int k = min(static_cast<int>(__popcll(__ballot(sum <= unit))), kWave - 1);
      const int before = k > 0 ? __builtin_amdgcn_readlane(sum, max(k - 1, 0)) : 0;
      return {min(n0 + k, n_seqs - 1), unit - before};
    }
    unit -= total;
  }
}
// Segments of the sequences before n.
__device__ __forceinline__ int segments_before(const int32_t* __restrict__ cu, int n, int tokens) {
  const int lane = threadIdx.x % kWave;
  int total = 0;
  for (int n0 = 0; n0 < n; n0 += kWave)
    total += __builtin_amdgcn_readlane(wave_scan(segments_of(cu, n, n0 + lane, tokens)), kWave - 1);
  return total;
}

// The sequence of rank r by chunks, the longest first, equal ones as they come;
// at most 64 sequences.  Uniform over the wave.
__device__ __forceinline__ int nth_longest(const int32_t* __restrict__ cu, int n_seqs, int r) {
  const int lane = threadIdx.x % kWave;
  const int mine = lane < n_seqs ? (cu[lane + 1] - cu[lane] + kSsmChunk - 1) / kSsmChunk : -1;
  int rank = 0;
  for (int j = 0; j < n_seqs; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    rank += other > mine || (other == mine && j < lane) ? 1 : 0;
  }
  return max(__ffsll(static_cast<unsigned long long>(__ballot(lane < n_seqs && rank == r))) - 1, 0);
}

struct SsmScanArgs {
  int32_t n_seqs, heads, groups, seg_tokens;
  float scale;    // of the outputs (fixed decays)
  bool ordered;   // kWhole: unit r is the sequence of rank r
  const int32_t* cu;
  const void* x;
  const void* dt;
  const void* B;
  const void* C;
  int64_t ldx, ld_dt, ldb, ldc, ldy;
  bool dt_bf16;
  const float* a_log;   // fixed decays: log alpha
  const float* d_skip;
  const float* dt_bias;
  const float* state_in;
  void* y;
  float* state_out;
  f32x4* seg_state;     // [segment, head group, wave, tile, lane]
  float* seg_decay;     // [segment, head]: log2 of a segment's decay
};

// kWhole: a unit is a sequence, from state_in to y (where given) and state_out.
// kLocal: a unit is a segment from the zero state to seg_state and seg_decay.
// kJoined: a unit is a segment from seg_state to y.
enum class SsmMode { kWhole, kLocal, kJoined };

// 2^e of an exponent in 64 bits: as good as exp2's own rounding whatever |e|.
__device__ __forceinline__ float exp2_wide(double e) {
  const float high = static_cast<float>(e), low = static_cast<float>(e - high);
  const float p = __builtin_amdgcn_exp2f(high);
  return fmaf(p, low * 0.693147180559945f, p);
}

template <typename T, int DK, int DV, int CT, int NW, bool OUT>
struct SsmLayout {
  static constexpr int kThreads = NW * kWave;
  static constexpr int kCols = 16 * CT;               // state columns of a wave
  static constexpr int kWavesPerHead = DV / kCols;
  static constexpr int kHeads = NW / kWavesPerHead;   // heads of a workgroup
  static constexpr int kTiles = DK / 16 * CT;         // accumulator tiles of a wave's state
  typedef RowsLds<T, DK> KRows;
  typedef RowsLds<T, DV> XRows;
  static constexpr int kPFrags = 6;                   // (row tile ti, k step kk <= ti / 2)
  static constexpr int kPBytes = kPFrags * Mx<T>::kF2Bytes;
  static constexpr int kOffB = 0;
  static constexpr int kOffC = kOffB + KRows::kBytes;
  static constexpr int kOffX = kOffC + (OUT ? KRows::kBytes : 0);
  static constexpr int kOffP = kOffX + kHeads * XRows::kBytes;
  static constexpr int kOffCb = kOffP + (OUT ? kHeads * kPBytes : 0);   // C B^T: 10 tiles, 16 bytes a lane
  static constexpr int kOffS = kOffCb + (OUT ? 10 * 1024 : 0);
  static constexpr int kBytes = kOffS + kHeads * static_cast<int>(sizeof(HeadScalars));
  static_assert(NW % kWavesPerHead == 0 && kHeads <= NW, "whole heads");
  static_assert(kSsmChunk * KRows::kPieces % kThreads == 0 && kSsmChunk * XRows::kPieces * kHeads % kThreads == 0,
                "whole pieces per thread");
};

// Row and first column of state tile (td, ct) of lane (g, c); see strow.
__device__ __forceinline__ int ssm_col(int ct, int c) { return 32 * (ct >> 1) + 8 * (c / 4) + 4 * (ct & 1) + c % 4; }

// Waves of a SIMD that the registers are kept for: two for bf16 inputs, where a
// CU's LDS holds enough workgroups.  Whole sequences with outputs and 128 state
// rows want more than 256 registers, for which four waves a workgroup can give up
// the second one: 32 heads of 128 x 128, one a workgroup, 8 sequences of 512 tokens
// 47 us with one, 66 with two, 16 of 2048 334 and 383 (71 registers spilled).
template <typename T, int DK, int NW, SsmMode MODE, bool OUT, int BYTES>
constexpr int ssm_waves() {
  if (sizeof(T) != 2 || 160 * 1024 / BYTES * NW / 4 < 2) return 1;
  return MODE == SsmMode::kWhole && OUT && DK == 128 && NW <= 4 ? 1 : 2;
}

// FIXED: linear attention with a decay for each head (gdn_linear.h), M <- alpha M +
// k v^T, y = scale M^T q: x is v, B is k, C is q, a step has delta = 1 and there is
// no dt.  The scalars of a whole chunk are the same for every chunk, so they are
// made once, from exponents in 64 bits, and again for a sequence's last, shorter one.
template <typename T, int DK, int DV, int CT, int NW, SsmMode MODE, bool OUT, bool FIXED = false>
__global__ __launch_bounds__(NW * kWave, (ssm_waves<T, DK, NW, MODE, OUT, SsmLayout<T, DK, DV, CT, NW, OUT>::kBytes>()))
void k_ssm_scan(SsmScanArgs a) {
  typedef SsmLayout<T, DK, DV, CT, NW, OUT> L;
  typedef typename L::KRows KRows;
  typedef typename L::XRows XRows;
  typedef Mx<T> X;
  typedef typename X::R R;
  constexpr int KB = kSsmChunk * KRows::kPieces / L::kThreads;                 // pieces per thread
  constexpr int KX = kSsmChunk * XRows::kPieces * L::kHeads / L::kThreads;
  constexpr int XP = XRows::kPieces * L::kHeads;                               // pieces of a token's heads
  __shared__ __attribute__((aligned(1024))) char lds[L::kBytes];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lane = tid % kWave;
  const int g = lane / 16, c = lane % 16;
  const int hgs = a.heads / L::kHeads;
  const int unit = xcd_cluster_remap(blockIdx.x, gridDim.x, hgs);
  const int hg = unit % hgs, slot = unit / hgs;
  int n = slot, first = 0;
  if constexpr (MODE == SsmMode::kWhole) {
    // a sequence's workgroups go to one XCD, its neighbours' to the next: every other
    // row of eight backwards, so that the first XCD does not get the longest of each
    if (a.ordered) {
      const int rank = (slot & kXcds) && (slot | (kXcds - 1)) < a.n_seqs ? slot ^ (kXcds - 1) : slot;
      n = __builtin_amdgcn_readfirstlane(nth_longest(a.cu, a.n_seqs, rank));
    }
  } else {
    const SegmentAt at = segment_at(a.cu, a.n_seqs, a.seg_tokens, slot);
    n = at.n;
    first = at.j * a.seg_tokens;
  }
  const int start = __builtin_amdgcn_readfirstlane(a.cu[n]);
  const int seq_len = __builtin_amdgcn_readfirstlane(a.cu[n + 1]) - start;
  const int len = MODE == SsmMode::kWhole ? seq_len : min(a.seg_tokens, seq_len - first);
  const int64_t t0 = static_cast<int64_t>(start) + first;
  const int h0 = hg * L::kHeads, gh = h0 / (a.heads / a.groups);
  const int hl = wave / L::kWavesPerHead, head = h0 + hl;
  const int p0 = (wave % L::kWavesPerHead) * L::kCols;   // this wave's first column of its head

  const T* xb = static_cast<const T*>(a.x) + t0 * a.ldx + static_cast<int64_t>(h0) * DV;
  const T* bb = static_cast<const T*>(a.B) + t0 * a.ldb + static_cast<int64_t>(gh) * DK;
  const T* cb = OUT ? static_cast<const T*>(a.C) + t0 * a.ldc + static_cast<int64_t>(gh) * DK : nullptr;
  HeadScalars* sc = reinterpret_cast<HeadScalars*>(lds + L::kOffS);

  // the state
  f32x4 m[DK / 16][CT];
  const int64_t sbase = (static_cast<int64_t>(n) * a.heads + head) * DK * DV;
  f32x4* seg = a.seg_state + (static_cast<int64_t>(slot) * hgs * NW + hg * NW + wave) * L::kTiles * kWave + lane;
#pragma unroll
  for (int td = 0; td < DK / 16; ++td)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      if constexpr (MODE == SsmMode::kJoined) {
        m[td][ct] = seg[(td * CT + ct) * kWave];
      } else if (MODE == SsmMode::kWhole && a.state_in) {
#pragma unroll
        for (int i = 0; i < 4; ++i) m[td][ct][i] = a.state_in[sbase + strow(td, g, i) * DV + p0 + ssm_col(ct, c)];
      } else {
        m[td][ct] = zero4();
      }
    }

  const float neg_a2 = !FIXED && wave < L::kHeads ? -expf(a.a_log[h0 + wave]) * 1.44269504088896f : 0.0f;
  const float dt_bias = !FIXED && wave < L::kHeads && a.dt_bias ? a.dt_bias[h0 + wave] : 0.0f;
  const float skip = !FIXED && OUT && a.d_skip ? a.d_skip[head] : 0.0f;
  double rate = 0.0;   // log2 alpha (FIXED)
  if (FIXED && wave < L::kHeads) {
    rate = static_cast<double>(a.a_log[h0 + wave]) * 1.4426950408889634;
    if (rate < -150.0) rate = -150.0;   // as below
  }
  float log_total = 0.0f;   // of the whole segment (kLocal)

  // A thread's pieces of a chunk: rows tid / pieces + k (threads / pieces).  A
  // chunk is a buffer from its first row: its offsets fit 32 bits (row strides
  // are at most 2^23 elements), rows behind the sequence's last one read as zero.
  constexpr uint32_t E = sizeof(T);
  u32x4 pb[KB], pc[OUT ? KB : 1], px[KX];
  uint32_t pdt = 0;   // dt as loaded
  const uint32_t ldb = static_cast<uint32_t>(a.ldb) * E, ldc = static_cast<uint32_t>(a.ldc) * E,
                 ldx = static_cast<uint32_t>(a.ldx) * E, ldy = static_cast<uint32_t>(a.ldy) * E;
  const uint32_t rowk = tid / KRows::kPieces, colk = tid % KRows::kPieces, rowx = tid / XP, colx = tid % XP;
  constexpr uint32_t KSTEP = L::kThreads / KRows::kPieces, XSTEP = L::kThreads / XP;   // rows from k to k + 1
  static_assert(KSTEP * KRows::kPieces == L::kThreads && XSTEP * XP == L::kThreads, "whole rows per step");
  const auto x_at = [&](int k) {   // where piece k of x lies in LDS
    return L::kOffX + static_cast<int>(colx / XRows::kPieces) * XRows::kBytes +
           XRows::template at_step<XSTEP>(rowx, k, colx % XRows::kPieces);
  };
  const auto fetch = [&](int at) {
    const uint32_t rows = min(kSsmChunk, len - at);
    uint32_t vb = rowk * ldb + colk * 16, vc = rowk * ldc + colk * 16, vx = rowx * ldx + colx * 16;
    asm volatile("" : "+v"(vb), "+v"(vc), "+v"(vx));   // added to here, not kept in a register per piece
    const __amdgpu_buffer_rsrc_t rb = rows_buffer(bb + at * a.ldb, (rows - 1) * ldb + DK * E);
#pragma unroll
    for (int k = 0; k < KB; ++k) pb[k] = __builtin_amdgcn_raw_buffer_load_b128(rb, vb + k * KSTEP * ldb, 0, 0);
    if constexpr (OUT) {
      const __amdgpu_buffer_rsrc_t rc = rows_buffer(cb + at * a.ldc, (rows - 1) * ldc + DK * E);
#pragma unroll
      for (int k = 0; k < KB; ++k) pc[k] = __builtin_amdgcn_raw_buffer_load_b128(rc, vc + k * KSTEP * ldc, 0, 0);
    }
    const __amdgpu_buffer_rsrc_t rx = rows_buffer(xb + at * a.ldx, (rows - 1) * ldx + L::kHeads * DV * E);
#pragma unroll
    for (int k = 0; k < KX; ++k) px[k] = __builtin_amdgcn_raw_buffer_load_b128(rx, vx + k * XSTEP * ldx, 0, 0);
    if (!FIXED && wave < L::kHeads) {
      const int64_t base = (t0 + at) * a.ld_dt + h0 + wave;
      const uint32_t off = min(static_cast<uint32_t>(lane), rows - 1) * static_cast<uint32_t>(a.ld_dt);
      if (a.dt_bf16) pdt = (static_cast<const uint16_t*>(a.dt) + base)[off];
      else pdt = (static_cast<const uint32_t*>(a.dt) + base)[off];
    }
  };

  if constexpr (OUT) {
    // the halves of P's diagonal operands that lie above the diagonal
    if (wave % L::kWavesPerHead == 0) {
      char* pf = lds + L::kOffP + hl * L::kPBytes;
      const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      X::put4(pf, 32 + lane % 32, lane / 32, zero);
      X::put4(pf + 3 * X::kF2Bytes, 32 + lane % 32, lane / 32, zero);
    }
  }
  // The outputs of the chunk at `at`, which lie where its x lay.  A thread takes
  // the very pieces that it writes the next chunk's x to, so no barrier comes
  // between.
  const auto write_y = [&](int at) {
    const uint32_t rows = min(kSsmChunk, len - at);
    const __amdgpu_buffer_rsrc_t ry = rows_buffer(static_cast<T*>(a.y) + (t0 + at) * a.ldy + static_cast<int64_t>(h0) * DV,
                                                  (rows - 1) * ldy + L::kHeads * DV * E);
    uint32_t vy = rowx * ldy + colx * 16;
    asm volatile("" : "+v"(vy));
#pragma unroll
    for (int k = 0; k < KX; ++k)
      __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(lds + x_at(k)), ry, vy + k * XSTEP * ldy, 0, 0);
  };
  if (len > 0) fetch(0);
  for (int at = 0; at < len; at += kSsmChunk) {
    const int rows = min(kSsmChunk, len - at);
    if (OUT && at > 0) write_y(at - kSsmChunk);
    // registers -> LDS
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      *reinterpret_cast<u32x4*>(lds + L::kOffB + KRows::template at_step<KSTEP>(rowk, k, colk)) = pb[k];
      if constexpr (OUT) *reinterpret_cast<u32x4*>(lds + L::kOffC + KRows::template at_step<KSTEP>(rowk, k, colk)) = pc[k];
    }
#pragma unroll
    for (int k = 0; k < KX; ++k) *reinterpret_cast<u32x4*>(lds + x_at(k)) = px[k];
    if (FIXED && wave < L::kHeads && (at == 0 || rows < kSsmChunk)) {
      // this head's decays, a token per lane: its tile holds `in_tile` tokens, `upto` of them up to this one
      const int in_tile = max(0, min(16, rows - 16 * g)), upto = min(c + 1, in_tile), behind = max(0, rows - 1 - lane);
      const bool there = lane < rows;
      HeadScalars& o = sc[wave];
      if constexpr (OUT) {
        const double wide = rate * upto;
        const float high = static_cast<float>(wide), low = static_cast<float>(wide - high);
        o.high[lane] = high;
        o.low[lane] = low;
        o.same[lane] = there ? -low : -INFINITY;
        o.row[lane] = exp2_wide(wide) * a.scale;
        o.past[lane] = there ? exp2_wide(rate * (in_tile - upto)) : 0.0f;
        o.pre[lane] = exp2_wide(rate * min(lane + 1, rows)) * a.scale;
        // the tokens of the tiles between those of tile pair t, see tile_rows
        if (lane < 10) {
          const int t1 = max(0, min(16, rows - 16)), t2 = max(0, min(16, rows - 32));
          o.between[lane] = exp2_wide(rate * (lane == 3 ? t1 : lane == 6 ? t1 + t2 : lane == 7 ? t2 : 0));
        }
      }
      o.suf[lane] = there ? exp2_wide(rate * behind) : 0.0f;
      if (lane == 0) o.total = exp2_wide(rate * rows);
    }
    if (!FIXED && wave < L::kHeads) {
      // this head's steps, a token per lane
      float delta = 0.0f, la = 0.0f;
      if (lane < rows) {
        delta = softplus_f(__uint_as_float(a.dt_bf16 ? pdt << 16 : pdt) + dt_bias);
        la = neg_a2 * delta;
        if (la < -150.0f) la = -150.0f;   // 2^-150 rounds to zero, and sums of it stay finite; NaN stays NaN
      }
      // sums over the 16-token tiles (a tile is a DPP row): up to the token, and behind it
      const float l = row_scan<0x110>(la), s = row_scan<0x100>(dpp<0x101>(la));
      const float q0 = read_lane(l, 15), q1 = read_lane(l, 31), q2 = read_lane(l, 47), q3 = read_lane(l, 63);
      const float before = g == 0 ? 0.0f : g == 1 ? q0 : g == 2 ? q0 + q1 : q0 + q1 + q2;
      const float after = g == 3 ? 0.0f : g == 2 ? q3 : g == 1 ? q2 + q3 : q1 + (q2 + q3);
      HeadScalars& o = sc[wave];
      int place = lane;
      asm volatile("" : "+v"(place));   // addresses are made here, not kept in registers over the chunks
      if constexpr (OUT) {
        const double wide = row_scan_wide(la);
        const float high = static_cast<float>(wide), low = static_cast<float>(wide - high);
        o.high[place] = high;
        o.low[place] = low;
        o.same[place] = __log2f(delta) - low;
        o.row[place] = __builtin_amdgcn_exp2f(l);
        o.past[place] = __builtin_amdgcn_exp2f(s) * delta;
        o.pre[place] = __builtin_amdgcn_exp2f(before + l);
        if (place < 10)
          o.between[place] = __builtin_amdgcn_exp2f(place == 3 ? q1 : place == 6 ? q1 + q2 : place == 7 ? q2 : 0.0f);
      }
      o.suf[place] = __builtin_amdgcn_exp2f(s + after) * delta;
      const float sum = (q0 + q1) + (q2 + q3);
      log_total += sum;
      if (lane == 0) o.total = __builtin_amdgcn_exp2f(sum);
    }
    lds_barrier();
    const HeadScalars& hs = sc[hl];
    const char* xt = lds + L::kOffX + hl * XRows::kBytes;
    char* pt = lds + L::kOffP + hl * L::kPBytes;

    constexpr int KK = DK / 32;
    constexpr int N2 = parts_of<typename X::F2>();
    // the state that kJoined carries ends in outputs alone (the join has written the final one)
    typedef typename std::conditional<MODE == SsmMode::kJoined, typename X::F2, typename X::F3>::type FS;
    constexpr int NS = parts_of<FS>();
    R xf[2][CT];
    const auto load_x = [&] {   // tokens 32 kk + 8 g + j of column ct
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) xf[kk][ct] = XRows::col_frag(xt, 32 * kk, p0 + 32 * (ct >> 1), ct & 1, g, c);
    };

    // Operands are read one step ahead of the products that take them: the
    // scheduling barriers keep the reads in front (left to itself the compiler
    // waits for every read right after it).
    const auto tile_rows = [](int t, int& ti, int& tj) {   // tile t of the lower triangle
      ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3;
      tj = t - ti * (ti + 1) / 2;
    };
    f32x4 yt[4][OUT ? CT : 1];   // y^T tiles: rows are state columns, columns are tokens
    if constexpr (OUT) {
      // C B^T by 16 x 16 tiles of the lower triangle, one after another over the
      // workgroup's waves: a lane's accumulator is four columns j of row i
      int first = wave;
      asm volatile("" : "+s"(first));   // tile addresses are made here, not kept in registers over the chunks
      constexpr int CB = (10 + NW - 1) / NW;
#pragma unroll
      for (int k = 0; k < CB; ++k) {
        const int t = first + k * NW;
        if (10 % NW != 0 && t >= 10) break;
        int ti, tj;
        tile_rows(t, ti, tj);
        R tb[KK], tc[KK];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          tb[kk] = KRows::row_frag(lds + L::kOffB, 16 * tj, c, 4 * kk + g);
          tc[kk] = KRows::row_frag(lds + L::kOffC, 16 * ti, c, 4 * kk + g);
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 acc = zero4();
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) acc = X::mul(tb[kk], tc[kk], acc);
        *reinterpret_cast<f32x4*>(lds + L::kOffCb + 1024 * t + 16 * lane) = acc;
      }
      R cf[2][4];
      const auto load_c = [&](int kk) {
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) cf[kk & 1][ti] = KRows::row_frag(lds + L::kOffC, 16 * ti, c, 4 * kk + g);
      };
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) yt[ti][ct] = zero4();
      typename X::F2 mf[2][CT];
      const auto split_m = [&](int kk) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] = m[2 * kk][ct][j];
            v[4 + j] = m[2 * kk + 1][ct][j];
          }
          X::split(v, mf[kk & 1][ct].part);
        }
      };
      load_c(0);
      split_m(0);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) load_c(kk + 1);
        else load_x();
        __builtin_amdgcn_sched_barrier(0);
        if (kk + 1 < KK) split_m(kk + 1);   // beside the products
#pragma unroll
        for (int k = 0; k < N2; ++k)
#pragma unroll
          for (int ti = 0; ti < 4; ++ti)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) yt[ti][ct] = X::mul(mf[kk & 1][ct].part[k], cf[kk & 1][ti], yt[ti][ct]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) {
        const float e = hs.pre[16 * ti + c];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) yt[ti][ct][i] *= e;
      }
      lds_barrier();   // C B^T is whole
      // P^T = (C B^T o L o delta)^T, the head's tiles shared by its waves: the four
      // values of a lane are half of one lane's operand for x^T P^T
      constexpr int WPH = L::kWavesPerHead, ND = 4 / WPH, NO = (6 + WPH - 1) / WPH;   // tiles on and below the diagonal
      static_assert(4 % WPH == 0, "diagonal tiles per wave");
      int own = wave % WPH;
      asm volatile("" : "+s"(own));
      int gg = g, cc = c;
      asm volatile("" : "+v"(gg), "+v"(cc));   // so are the places of the exponents
      f32x4 cd[ND], hd[ND], jd[ND], co[NO];
      float ed[ND], ld[ND], eo[NO];
      int ti_o[NO], tj_o[NO];
#pragma unroll
      for (int k = 0; k < ND; ++k) {
        const int ti = own + k * WPH;
        cd[k] = *reinterpret_cast<const f32x4*>(lds + L::kOffCb + 1024 * (ti * (ti + 3) / 2) + 16 * lane);
        hd[k] = *reinterpret_cast<const f32x4*>(hs.high + 16 * ti + 4 * gg);
        jd[k] = *reinterpret_cast<const f32x4*>(hs.same + 16 * ti + 4 * gg);
        ed[k] = hs.high[16 * ti + cc];
        ld[k] = hs.low[16 * ti + cc];
      }
#pragma unroll
      for (int k = 0; k < NO; ++k) {
        const int o = min(own + k * WPH, 5);   // (1,0) (2,0) (2,1) (3,0) (3,1) (3,2)
        ti_o[k] = o < 1 ? 1 : o < 3 ? 2 : 3;
        tj_o[k] = o - ti_o[k] * (ti_o[k] - 1) / 2;
        const int t = ti_o[k] * (ti_o[k] + 1) / 2 + tj_o[k];
        co[k] = *reinterpret_cast<const f32x4*>(lds + L::kOffCb + 1024 * t + 16 * lane);
        eo[k] = hs.row[16 * ti_o[k] + c] * hs.between[t];
      }
      __builtin_amdgcn_sched_barrier(0);
      const auto put = [&](int ti, int tj, const float (&v)[4]) {
        X::put4(pt + (ti < 2 ? ti : 2 * ti - 2 + tj / 2) * X::kF2Bytes, 16 * (2 * (tj & 1) + g / 2) + c, g & 1, v);
      };
#pragma unroll
      for (int k = 0; k < ND; ++k) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p = cd[k][r] * __builtin_amdgcn_exp2f((ed[k] - hd[k][r]) + (ld[k] + jd[k][r]));
          if (FIXED) p *= a.scale;
          v[r] = 4 * g + r < c ? p : 4 * g + r == c ? p + skip : 0.0f;   // d_skip x rides on the diagonal
        }
        put(own + k * WPH, own + k * WPH, v);
      }
#pragma unroll
      for (int k = 0; k < NO; ++k) {
        // (read here: with the operands above it would be a register too many)
        const f32x4 jo = *reinterpret_cast<const f32x4*>(hs.past + 16 * tj_o[k] + 4 * g);
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = co[k][r] * (eo[k] * jo[r]);
        if (6 % WPH == 0 || own + k * WPH < 6) put(ti_o[k], tj_o[k], v);
      }
    } else {
      load_x();
    }
    // the next chunk's rows are on their way from here on (not earlier: the
    // operands above need the registers)
    if (at + kSsmChunk < len) fetch(at + kSsmChunk);

    // M <- e^{G_last} M + B^T (diag(suf) x)
    constexpr int TS = 2, STEPS = DK / 16 / TS;   // state row tiles of a step, steps for each kk
    R bt[2][TS];
    FS wx[CT];
    const auto load_b = [&](int step) {
#pragma unroll
      for (int t = 0; t < TS; ++t)
        bt[step & 1][t] = KRows::col_frag(lds + L::kOffB, 32 * (step / STEPS), 32 * (step % STEPS), t, g, c);
    };
    const auto weigh_x = [&](int kk) {
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(hs.suf + 32 * kk + 8 * g);
      const f32x4 w1 = *reinterpret_cast<const f32x4*>(hs.suf + 32 * kk + 8 * g + 4);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (j < 4 ? w0[j & 3] : w1[j & 3]) * X::elt(xf[kk][ct], j);
        X::split(v, wx[ct].part);
      }
    };
    // (not after the last chunk of a segment whose state ends there)
    if (MODE != SsmMode::kJoined || at + kSsmChunk < len) {
      const float total = hs.total;
      load_b(0);
      __builtin_amdgcn_sched_barrier(0);
      weigh_x(0);
#pragma unroll
      for (int td = 0; td < DK / 16; ++td)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) m[td][ct][i] *= total;
#pragma unroll
      for (int step = 0; step < 2 * STEPS; ++step) {
        if (step + 1 < 2 * STEPS) load_b(step + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (step == STEPS) weigh_x(1);
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
          for (int t = 0; t < TS; ++t)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              f32x4& acc = m[step % STEPS * TS + t][ct];
              acc = X::mul(bt[step & 1][t], wx[ct].part[k], acc);
            }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (OUT) {
      lds_barrier();   // P is whole
      // y^T += x^T P^T, and out
      typename X::F2 pf[L::kPFrags];
#pragma unroll
      for (int f = 0; f < L::kPFrags; ++f) pf[f] = X::get(pt + f * X::kF2Bytes, lane);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < N2; ++k)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int ti = 2 * kk; ti < 4; ++ti)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
              yt[ti][ct] = X::mul(xf[kk][ct], pf[ti < 2 ? ti : 2 * ti - 2 + kk].part[k], yt[ti][ct]);
      // over the chunk's x, which every wave has in registers by now; write_y sends
      // whole token rows from there (a wave's own 64-byte pieces of 16 rows per
      // store kept the CU's memory path busy more than twice as long)
      char* yl = lds + L::kOffX + hl * XRows::kBytes;
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int b = 0; b < CT / 2; ++b) {
          float o[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = yt[ti][2 * b + j / 4][j & 3];
          XRows::put8(yl, 16 * ti, c, (p0 + 32 * b) / 8 + g, o);
        }
    }
    lds_barrier();   // the chunk's LDS has been read, its outputs are whole
  }
  if (OUT && len > 0) write_y((len - 1) / kSsmChunk * kSsmChunk);

  if constexpr (MODE == SsmMode::kLocal) {
#pragma unroll
    for (int td = 0; td < DK / 16; ++td)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) seg[(td * CT + ct) * kWave] = m[td][ct];
    if (wave < L::kHeads && lane == 0)
      a.seg_decay[static_cast<int64_t>(slot) * a.heads + h0 + wave] = FIXED ? static_cast<float>(rate * len) : log_total;
  } else if (MODE == SsmMode::kWhole && a.state_out) {
#pragma unroll
    for (int td = 0; td < DK / 16; ++td)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.state_out[sbase + strow(td, g, i) * DV + p0 + ssm_col(ct, c)] = m[td][ct][i];
  }
}

// The segments' states become their starts: per sequence and state element,
//   start_0 = state_in,  start_{j+1} = decay_j start_j + local_j,
// the last of them state_out (where wanted).  With JOIN the starts replace the
// local states, for kJoined.  A thread takes one accumulator element (four rows
// of a column) of one sequence.  Bound by the states' bytes: 13 segments of 64
// heads of 64 x 128, 54 MB both ways, 10 us.
template <int DK, int DV, int CT, int NW, bool JOIN>
__global__ __launch_bounds__(256)
void k_ssm_join(SsmScanArgs a) {
  constexpr int kWavesPerHead = DV / (16 * CT);
  constexpr int kTiles = DK / 16 * CT;
  static_assert(kWavesPerHead * kTiles * kWave % 256 == 0, "whole blocks per sequence");
  const int per_seq = a.heads * kWavesPerHead * kTiles * kWave;   // f32x4 of a sequence's states
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;   // per_seq is a multiple of 256: one n per block
  const int n = __builtin_amdgcn_readfirstlane(static_cast<int>(i / per_seq)), e = static_cast<int>(i % per_seq);
  const int lane = e % kWave, tile = e / kWave % kTiles, w = e / (kWave * kTiles);   // w: wave of the sequence
  const int head = w / kWavesPerHead;
  const int td = tile / CT, ct = tile % CT, g = lane / 16, c = lane % 16;
  const int64_t sbase = (static_cast<int64_t>(n) * a.heads + head) * DK * DV + (w % kWavesPerHead) * 16 * CT + ssm_col(ct, c);
  f32x4 run = zero4();
  if (a.state_in) {
#pragma unroll
    for (int r = 0; r < 4; ++r) run[r] = a.state_in[sbase + strow(td, g, r) * DV];
  }
  const int start = a.cu[n], len = a.cu[n + 1] - start;
  const int64_t slot0 = segments_before(a.cu, n, a.seg_tokens);
  const int segs = max(1, (len + a.seg_tokens - 1) / a.seg_tokens);
  // eight segments' loads are in flight at a time
  constexpr int AHEAD = 8;
  f32x4* p = a.seg_state + slot0 * per_seq + e;
  const float* dec = a.seg_decay + slot0 * a.heads + head;
  for (int j0 = 0; j0 < segs; j0 += AHEAD) {
    f32x4 local[AHEAD];
    float decay[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t j = min(j0 + k, segs - 1);
      local[k] = p[j * per_seq];
      decay[k] = dec[j * a.heads];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (j0 + k >= segs) break;
      if (JOIN) p[(j0 + k) * static_cast<int64_t>(per_seq)] = run;
      const float d = __builtin_amdgcn_exp2f(decay[k]);
#pragma unroll
      for (int r = 0; r < 4; ++r) run[r] = fmaf(d, run[r], local[k][r]);   // an empty segment: decay 1, local 0
    }
  }
  if (a.state_out) {
#pragma unroll
    for (int r = 0; r < 4; ++r) a.state_out[sbase + strow(td, g, r) * DV] = run[r];
  }
}

}  // namespace gdn
