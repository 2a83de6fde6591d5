// The chunked selective state space scan on the matrix cores.
//
// A workgroup holds the states of a few heads of one sequence (or of one
// segment of it) in registers and walks its 64-token chunks.  With G the
// chunk's inclusive cumulative log alpha and M0 the state before it,
//   y  = diag(e^G) C M0 + ((C B^T) o L o delta_j) x + d_skip x,
//   M <- e^{G_last} M0 + B^T diag(e^{G_last - G_j} delta_j) x,
//   L_ij = e^{G_i - G_j} for j <= i.
// C B^T is computed once per chunk for all of the workgroup's heads (they share
// a B/C group), everything else per wave: a wave owns 16 CT state columns of
// one head.
#pragma once

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

template <>
struct Mx<uint16_t> {
  typedef bf16x8 R;
  typedef Frag F2;
  struct F3 { bf16x8 hi, mid, lo; };
  static __device__ __forceinline__ F2 f2(const float (&v)[8]) { return split8(v); }
  static __device__ __forceinline__ F3 f3(const float (&v)[8]) {
    F3 f;
    u32x4 hi, mid, lo;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const f32x2 x = {v[2 * p], v[2 * p + 1]};
      const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
      const f32x2 d = {x[0] - __uint_as_float(h << 16), x[1] - __uint_as_float(h & 0xFFFF0000u)};
      const uint32_t m = __builtin_bit_cast(uint32_t, __builtin_convertvector(d, bf16x2));
      const f32x2 e = {d[0] - __uint_as_float(m << 16), d[1] - __uint_as_float(m & 0xFFFF0000u)};
      hi[p] = h;
      mid[p] = m;
      lo[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(e, bf16x2));
    }
    f.hi = __builtin_bit_cast(bf16x8, hi);
    f.mid = __builtin_bit_cast(bf16x8, mid);
    f.lo = __builtin_bit_cast(bf16x8, lo);
    return f;
  }
  static __device__ __forceinline__ float elt(const R& r, int j) {
    const u32x4 w = __builtin_bit_cast(u32x4, r);
    return __uint_as_float((j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16));
  }
  static __device__ __forceinline__ f32x4 rr(const R& a, const R& b, f32x4 c) { return mma(a, b, c); }
  static __device__ __forceinline__ f32x4 fr(const F2& a, const R& b, f32x4 c) { return mma(a.lo, b, mma(a.hi, b, c)); }
  static __device__ __forceinline__ f32x4 rf(const R& a, const F2& b, f32x4 c) { return mma(a, b.lo, mma(a, b.hi, c)); }
  static __device__ __forceinline__ f32x4 rf3(const R& a, const F3& b, f32x4 c) {
    return mma(a, b.lo, mma(a, b.mid, mma(a, b.hi, c)));
  }
};

template <>
struct Mx<float> {
  typedef f32x8 R;
  typedef f32x8 F2;
  typedef f32x8 F3;
  static __device__ __forceinline__ f32x8 f2(const float (&v)[8]) {
    return f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  }
  static __device__ __forceinline__ f32x8 f3(const float (&v)[8]) { return f2(v); }
  static __device__ __forceinline__ float elt(const R& r, int j) { return r[j]; }
  static __device__ __forceinline__ f32x4 rr(const R& a, const R& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x4 fr(const F2& a, const R& b, f32x4 c) { return rr(a, b, c); }
  static __device__ __forceinline__ f32x4 rf(const R& a, const F2& b, f32x4 c) { return rr(a, b, c); }
  static __device__ __forceinline__ f32x4 rf3(const R& a, const F3& b, f32x4 c) { return rr(a, b, c); }
};

// ---------------------------------------------------------------- token rows in LDS
// 64 rows of D elements.  bf16: 16-byte pieces swizzled as key rows are
// (row_swz: 16-byte operand reads without bank conflicts, transposing reads with
// the fewest there are).  fp32: rows padded by 16 bytes.
template <typename T, int D>
struct RowsLds {
  static constexpr int kPieces = D * static_cast<int>(sizeof(T)) / 16;   // of a row
  static constexpr int kPitch = sizeof(T) == 2 ? 2 * D : 4 * D + 16;
  static constexpr int kBytes = kSsmChunk * kPitch;
  static __device__ __forceinline__ int at(int row, int piece) {
    if constexpr (sizeof(T) == 2) return row * kPitch + ((piece ^ row_swz<kPitch>(row)) << 4);
    else return row * kPitch + (piece << 4);
  }
  // elements 8 e8 .. + 7 of a row
  static __device__ __forceinline__ typename Mx<T>::R row_frag(const char* base, int row, int e8) {
    if constexpr (sizeof(T) == 2) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(base + at(row, e8)));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(base + at(row, 2 * e8));
      const f32x4 b = *reinterpret_cast<const f32x4*>(base + at(row, 2 * e8 + 1));
      return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  }
  // rows row0 + 8 g + j (j = 0..7) of column col32 + 8 (c / 4) + 4 half + c % 4, for lane (g, c)
  static __device__ __forceinline__ typename Mx<T>::R col_frag(const char* base, int row0, int col32, int half, int g,
                                                               int c) {
    if constexpr (sizeof(T) == 2) {
      // lane 4 t + q of a group of 16 supplies four elements of row t, columns 8 q ..; lane i receives
      // column 8 (i / 4) + i % 4 of rows 0..3
      const int row = row0 + 8 * g + c / 4, piece = col32 / 8 + c % 4;
      const u32x2 a = lds_read_tr16(base + at(row, piece) + 8 * half);
      const u32x2 b = lds_read_tr16(base + at(row + 4, piece) + 8 * half);
      return join_halves(a, b);
    } else {
      const float* p = reinterpret_cast<const float*>(base + (row0 + 8 * g) * kPitch) + col32 + 8 * (c / 4) + 4 * half + c % 4;
      f32x8 r;
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = p[j * (kPitch / 4)];
      return r;
    }
  }
};

// Per head and chunk, base-2 logarithms: with l the inclusive cumulative log
// alpha inside a token's 16-token tile and s what is left of the tile after it,
// e^{G_i - G_j} = 2^(l_i - l_j) within a tile and 2^(l_i + between + s_j) across
// tiles: sums of terms of one sign, never the difference of two long ones.
struct HeadScalars {
  float l[kSsmChunk];      // l
  float same[kSsmChunk];   // log2 delta - l
  float past[kSsmChunk];   // log2 delta + s
  float pre[kSsmChunk];    // e^G
  float suf[kSsmChunk];    // e^{G_last - G} delta
  float tile[4];           // log2 alpha summed over each tile
  float total;             // e^{G_last}
  float log_total;         // G_last, base 2
  float pad[2];
};

struct SsmScanArgs {
  int32_t n_seqs, heads, groups, seg_tokens;
  const int32_t* cu;
  const void* x;
  const void* dt;
  const void* B;
  const void* C;
  int64_t ldx, ld_dt, ldb, ldc, ldy;
  bool dt_bf16;
  const float* a_log;
  const float* d_skip;
  const float* dt_bias;
  const float* state_in;
  void* y;
  float* state_out;
  f32x4* seg_state;     // [slot, head group, wave, tile, lane]
  float* seg_decay;     // [slot, head]: log2 of a segment's decay
};

// kWhole: a unit is a sequence, from state_in to y (where given) and state_out.
// kLocal: a unit is a segment from the zero state to seg_state and seg_decay.
// kJoined: a unit is a segment from seg_state to y and, the last one, state_out.
enum class SsmMode { kWhole, kLocal, kJoined };

template <typename T, int DK, int DV, int CT, int NW, bool OUT>
struct SsmLayout {
  static constexpr int kThreads = NW * kWave;
  static constexpr int kCols = 16 * CT;               // state columns of a wave
  static constexpr int kWavesPerHead = DV / kCols;
  static constexpr int kHeads = NW / kWavesPerHead;   // heads of a workgroup
  static constexpr int kTiles = DK / 16 * CT;         // accumulator tiles of a wave's state
  typedef RowsLds<T, DK> KRows;
  typedef RowsLds<T, DV> XRows;
  static constexpr int kCbPitch = kSsmChunk + 4;
  static constexpr int kOffB = 0;
  static constexpr int kOffC = kOffB + KRows::kBytes;
  static constexpr int kOffX = kOffC + (OUT ? KRows::kBytes : 0);
  static constexpr int kOffCb = kOffX + kHeads * XRows::kBytes;
  static constexpr int kOffS = kOffCb + (OUT ? kSsmChunk * kCbPitch * 4 : 0);
  static constexpr int kBytes = kOffS + kHeads * static_cast<int>(sizeof(HeadScalars));
  static_assert(NW % kWavesPerHead == 0 && kHeads <= NW, "whole heads");
  static_assert(kSsmChunk * KRows::kPieces % kThreads == 0 && kSsmChunk * XRows::kPieces * kHeads % kThreads == 0,
                "whole pieces per thread");
};

// Row and first column of state tile (td, ct) of lane (g, c); see strow.
__device__ __forceinline__ int ssm_col(int ct, int c) { return 32 * (ct >> 1) + 8 * (c / 4) + 4 * (ct & 1) + c % 4; }

template <typename T, int DK, int DV, int CT, int NW, SsmMode MODE, bool OUT>
__global__ __launch_bounds__(NW * kWave)
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
  if constexpr (MODE != SsmMode::kWhole) n = slot_seq(a.cu, a.n_seqs, slot, a.seg_tokens);
  const int start = a.cu[n], seq_len = a.cu[n + 1] - start;
  if constexpr (MODE != SsmMode::kWhole) {
    const int64_t at = static_cast<int64_t>(slot - (start / a.seg_tokens + n)) * a.seg_tokens;
    if (at > 0 && at >= seq_len) return;   // an unused slot
    first = static_cast<int>(at);
  }
  const int len = MODE == SsmMode::kWhole ? seq_len : min(a.seg_tokens, seq_len - first);
  const bool last = first + len >= seq_len;
  if (MODE == SsmMode::kLocal && OUT == false && last && a.y) return;   // the joined pass ends there by itself
  const int64_t t0 = static_cast<int64_t>(start) + first;
  const int h0 = hg * L::kHeads, gh = h0 / (a.heads / a.groups);
  const int hl = wave / L::kWavesPerHead, head = h0 + hl;
  const int p0 = (wave % L::kWavesPerHead) * L::kCols;   // this wave's first column of its head

  const T* xb = static_cast<const T*>(a.x) + t0 * a.ldx + static_cast<int64_t>(h0) * DV;
  const T* bb = static_cast<const T*>(a.B) + t0 * a.ldb + static_cast<int64_t>(gh) * DK;
  const T* cb = OUT ? static_cast<const T*>(a.C) + t0 * a.ldc + static_cast<int64_t>(gh) * DK : nullptr;
  HeadScalars* sc = reinterpret_cast<HeadScalars*>(lds + L::kOffS);
  float* cbm = reinterpret_cast<float*>(lds + L::kOffCb);

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

  const float neg_a2 = wave < L::kHeads ? -expf(a.a_log[h0 + wave]) * 1.44269504088896f : 0.0f;
  const float dt_bias = wave < L::kHeads && a.dt_bias ? a.dt_bias[h0 + wave] : 0.0f;
  const float skip = OUT && a.d_skip ? a.d_skip[head] : 0.0f;
  float log_total = 0.0f;   // of the whole segment (kLocal)

  u32x4 pb[KB], pc[OUT ? KB : 1], px[KX];
  float pdt = 0.0f;
  // Rows behind the last token repeat it: their steps are zero, so what is
  // multiplied with it vanishes, and their outputs are not written.
  auto fetch = [&](int at) {
    const int rows = min(kSsmChunk, len - at);
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int i = tid + k * L::kThreads, row = min(i / KRows::kPieces, rows - 1), piece = i % KRows::kPieces;
      pb[k] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(bb + (at + row) * a.ldb) + piece * 16);
      if constexpr (OUT)
        pc[k] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(cb + (at + row) * a.ldc) + piece * 16);
    }
#pragma unroll
    for (int k = 0; k < KX; ++k) {
      const int i = tid + k * L::kThreads, row = min(i / XP, rows - 1), piece = i % XP;
      px[k] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(xb + (at + row) * a.ldx) + piece * 16);
    }
    if (wave < L::kHeads) pdt = load_dt(a.dt, a.dt_bf16, (t0 + at + min(lane, rows - 1)) * a.ld_dt + h0 + wave);
  };

  if (len > 0) fetch(0);
  for (int at = 0; at < len; at += kSsmChunk) {
    const int rows = min(kSsmChunk, len - at);
    // registers -> LDS
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int i = tid + k * L::kThreads, row = i / KRows::kPieces, piece = i % KRows::kPieces;
      *reinterpret_cast<u32x4*>(lds + L::kOffB + KRows::at(row, piece)) = pb[k];
      if constexpr (OUT) *reinterpret_cast<u32x4*>(lds + L::kOffC + KRows::at(row, piece)) = pc[k];
    }
#pragma unroll
    for (int k = 0; k < KX; ++k) {
      const int i = tid + k * L::kThreads, row = i / XP, piece = i % XP;
      *reinterpret_cast<u32x4*>(lds + L::kOffX + (piece / XRows::kPieces) * XRows::kBytes +
                                XRows::at(row, piece % XRows::kPieces)) = px[k];
    }
    if (wave < L::kHeads) {
      // this head's steps, a token per lane
      float delta = 0.0f, la = 0.0f;
      if (lane < rows) {
        delta = softplus_f(pdt + dt_bias);
        la = fmaxf(neg_a2 * delta, -150.0f);   // 2^-150 rounds to zero
      }
      float l = la, s = la;
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) {
        const float up = __shfl_up(l, off, 16), down = __shfl_down(s, off, 16);
        l += c >= off ? up : 0.0f;
        s += c + off < 16 ? down : 0.0f;
      }
      s = __shfl_down(s, 1, 16);
      if (c == 15) s = 0.0f;
      const float q0 = __shfl(l, 15, kWave), q1 = __shfl(l, 31, kWave), q2 = __shfl(l, 47, kWave), q3 = __shfl(l, 63, kWave);
      const float before = g == 0 ? 0.0f : g == 1 ? q0 : g == 2 ? q0 + q1 : q0 + q1 + q2;
      const float after = g == 3 ? 0.0f : g == 2 ? q3 : g == 1 ? q2 + q3 : q1 + (q2 + q3);
      const float ld = __log2f(delta);
      HeadScalars& o = sc[wave];
      o.l[lane] = l;
      o.same[lane] = ld - l;
      o.past[lane] = ld + s;
      o.pre[lane] = __builtin_amdgcn_exp2f(before + l);
      o.suf[lane] = __builtin_amdgcn_exp2f(s + after) * delta;
      if (c == 15) o.tile[g] = l;
      const float sum = (q0 + q1) + (q2 + q3);
      log_total += sum;
      if (lane == 0) o.total = __builtin_amdgcn_exp2f(sum);
    }
    __syncthreads();
    if (at + kSsmChunk < len) fetch(at + kSsmChunk);
    const HeadScalars& hs = sc[hl];
    const char* xt = lds + L::kOffX + hl * XRows::kBytes;

    if constexpr (OUT) {
      // C B^T, lower triangle of 16 x 16 tiles, transposed through the
      // accumulators: a lane holds four columns j of row i
      for (int t = wave; t < 10; t += NW) {
        const int ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, tj = t - ti * (ti + 1) / 2;
        f32x4 acc = zero4();
#pragma unroll
        for (int kk = 0; kk < DK / 32; ++kk)
          acc = X::rr(KRows::row_frag(lds + L::kOffB, 16 * tj + c, 4 * kk + g),
                      KRows::row_frag(lds + L::kOffC, 16 * ti + c, 4 * kk + g), acc);
        *reinterpret_cast<f32x4*>(cbm + (16 * ti + c) * L::kCbPitch + 16 * tj + 4 * g) = acc;
      }
      __syncthreads();
    }

    // x as an operand: tokens 32 kk + 8 g + j of column ct
    R xf[2][CT];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) xf[kk][ct] = XRows::col_frag(xt, 32 * kk, p0 + 32 * (ct >> 1), ct & 1, g, c);

    if constexpr (OUT) {
      // y^T tiles: rows are state columns, columns are tokens
      f32x4 yt[4][CT];
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) yt[ti][ct] = zero4();
#pragma unroll
      for (int kk = 0; kk < DK / 32; ++kk) {
        typename X::F2 mf[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] = m[2 * kk][ct][j];
            v[4 + j] = m[2 * kk + 1][ct][j];
          }
          mf[ct] = X::f2(v);
        }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          const R cf = KRows::row_frag(lds + L::kOffC, 16 * ti + c, 4 * kk + g);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) yt[ti][ct] = X::fr(mf[ct], cf, yt[ti][ct]);
        }
      }
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) {
        const float e = hs.pre[16 * ti + c];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) yt[ti][ct][i] *= e;
      }
      // + x^T P^T
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) {
        const float li = hs.l[16 * ti + c];
#pragma unroll
        for (int kk = 0; kk <= ti / 2; ++kk) {
          const int tj = 2 * kk + (g >> 1);
          const int j0 = 32 * kk + 8 * g;
          float between = 0.0f;
          if (tj + 1 < ti) between += hs.tile[ti - 1];
          if (tj + 2 < ti) between += hs.tile[ti - 2];
          const float* src = tj < ti ? hs.past : hs.same;
          const f32x4 b0 = *reinterpret_cast<const f32x4*>(src + j0), b1 = *reinterpret_cast<const f32x4*>(src + j0 + 4);
          const float* row = cbm + (16 * ti + c) * L::kCbPitch + j0;
          const f32x4 s0 = *reinterpret_cast<const f32x4*>(row), s1 = *reinterpret_cast<const f32x4*>(row + 4);
          const float e = li + between;
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float p = (j < 4 ? s0[j & 3] : s1[j & 3]) * __builtin_amdgcn_exp2f(e + (j < 4 ? b0[j & 3] : b1[j & 3]));
            v[j] = j0 + j <= 16 * ti + c ? p : 0.0f;
          }
          const typename X::F2 pf = X::f2(v);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) yt[ti][ct] = X::rf(xf[kk][ct], pf, yt[ti][ct]);
        }
      }
      // + d_skip x, and out
      T* yb = static_cast<T*>(a.y) + (t0 + at) * a.ldy + static_cast<int64_t>(head) * DV + p0;
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) {
        const int i = 16 * ti + c;
#pragma unroll
        for (int b = 0; b < CT / 2; ++b) {
          const R xr = XRows::row_frag(xt, i, (p0 + 32 * b) / 8 + g);
          float o[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = fmaf(skip, X::elt(xr, j), yt[ti][2 * b + j / 4][j & 3]);
          if (i < rows) store8(yb + i * a.ldy + 32 * b + 8 * g, o);
        }
      }
    }

    // M <- e^{G_last} M + B^T (diag(suf) x)
    const float total = hs.total;
#pragma unroll
    for (int td = 0; td < DK / 16; ++td)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) m[td][ct][i] *= total;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(hs.suf + 32 * kk + 8 * g);
      const f32x4 w1 = *reinterpret_cast<const f32x4*>(hs.suf + 32 * kk + 8 * g + 4);
      typename X::F3 wx[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (j < 4 ? w0[j & 3] : w1[j & 3]) * X::elt(xf[kk][ct], j);
        wx[ct] = X::f3(v);
      }
#pragma unroll
      for (int td = 0; td < DK / 16; ++td) {
        const R bt = KRows::col_frag(lds + L::kOffB, 32 * kk, 32 * (td >> 1), td & 1, g, c);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) m[td][ct] = X::rf3(bt, wx[ct], m[td][ct]);
      }
    }
    __syncthreads();   // the chunk's LDS has been read
  }

  if constexpr (MODE == SsmMode::kLocal) {
#pragma unroll
    for (int td = 0; td < DK / 16; ++td)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) seg[(td * CT + ct) * kWave] = m[td][ct];
    if (wave < L::kHeads && lane == 0) a.seg_decay[static_cast<int64_t>(slot) * a.heads + h0 + wave] = log_total;
  } else if (last && a.state_out) {
#pragma unroll
    for (int td = 0; td < DK / 16; ++td)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.state_out[sbase + strow(td, g, i) * DV + p0 + ssm_col(ct, c)] = m[td][ct][i];
  }
}

// The segments' states become their starts: per sequence and state element,
//   start_0 = state_in,  start_{j+1} = decay_j start_j + local_j.
// With JOIN the starts replace the local states (the last segment's is not
// read); without, only the last state is wanted and goes to state_out.  A thread
// takes one accumulator element (four rows of a column) of one sequence.
template <int DK, int DV, int CT, int NW, bool JOIN>
__global__ __launch_bounds__(256)
void k_ssm_join(SsmScanArgs a) {
  constexpr int kWavesPerHead = DV / (16 * CT);
  constexpr int kTiles = DK / 16 * CT;
  const int per_seq = a.heads * kWavesPerHead * kTiles * kWave;   // f32x4 of a sequence's states
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(a.n_seqs) * per_seq) return;
  const int n = static_cast<int>(i / per_seq), e = static_cast<int>(i % per_seq);
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
  const int64_t slot0 = start / a.seg_tokens + n;
  const int segs = max(1, (len + a.seg_tokens - 1) / a.seg_tokens);
  for (int j = 0; j < segs; ++j) {
    f32x4* p = a.seg_state + (slot0 + j) * per_seq + e;
    if (JOIN && j == segs - 1) {
      *p = run;
      return;
    }
    if (j * static_cast<int64_t>(a.seg_tokens) < len) {
      const f32x4 local = *p;
      const float decay = __builtin_amdgcn_exp2f(a.seg_decay[(slot0 + j) * a.heads + head]);
      if (JOIN) *p = run;
#pragma unroll
      for (int r = 0; r < 4; ++r) run[r] = fmaf(decay, run[r], local[r]);
    }
  }
  if (!JOIN) {
#pragma unroll
    for (int r = 0; r < 4; ++r) a.state_out[sbase + strow(td, g, r) * DV] = run[r];
  }
}

}  // namespace gdn
