// Kernels of the low-rank adapters (C ABI in gdn_lora.h).  Two launches:
//   k_lora_down  u[t] = s_a x[t] A_a^T, fp32, in the workspace
//   k_lora_up    out[t] = base[t] + u[t] B_a^T
// Both are matrix products whose operands lie along their contraction in memory
// (rows of x, A and B), so a lane's 16 bytes of a row are an MFMA operand as
// they are loaded, without a pass through LDS.  The work is HBM's: at rank 64 a
// projected element costs 128 multiply-adds against reading and writing it.
//
// Measured, 2048 -> 12352, on inputs that are not in the last-level cache: bf16,
// 4324 tokens of 8 requests at rank 64, 19 and 64 us (the second kernel moves 214
// MB of base and out, 3.3 TB/s; 238 MB in all, which a copy moves in 44 to 49),
// fp32 19 and 119; 64 single tokens at rank 16 5.9 and 9.1 us (16 MB, most of it A
// and B).  With the same inputs call after call, as for the figures below, part of
// them stays in that cache: 16 and 48 us.  The first kernel has 143 workgroups
// there for 256 CUs, each bound by its loads' way through L2: eight waves instead of
// four, or neighbouring steps a wave, left it at 16.0 us.
//
// Tokens go by tiles of 16 TT inside a sequence (its adapter is the tile's).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

constexpr int kLoraThreads = 256;
constexpr int kLoraWaves = kLoraThreads / kWave;
constexpr int kLoraWaveCols = 64;                          // output columns of a wave of k_lora_up
constexpr int kLoraCols = kLoraWaves * kLoraWaveCols;      // of a workgroup
constexpr int lora_tile(int tt) { return 16 * tt; }

struct LoraArgs {
  int32_t n_seqs, n_adapters, K, M, R, parts;   // parts: pieces of K, a partial u each
  int64_t tokens;
  const int32_t* cu;
  const int32_t* adapters;
  const uint16_t* x;
  int64_t ldx;
  const uint16_t* A;
  const uint16_t* B;
  int64_t b_stride;   // elements between two adapters' B
  const float* scales;
  const void* base;
  int64_t ldbase;
  void* out;
  int64_t ldout;
  float* u;   // [parts, tokens, R]
};

// The tile's sequence, first token, token count and adapter (-1: none).
struct LoraTile { int64_t t0; int rows, adapter; };
template <int TT>
__device__ __forceinline__ LoraTile lora_tile_of(const LoraArgs& a, int slot) {
  const int n = slot_seq(a.cu, a.n_seqs, slot, lora_tile(TT));
  const int start = a.cu[n], len = a.cu[n + 1] - start;
  const int at = (slot - (start / lora_tile(TT) + n)) * lora_tile(TT);
  const int id = a.adapters[n];
  return {static_cast<int64_t>(start) + at, min(len - at, lora_tile(TT)), id < a.n_adapters ? id : -1};
}

__device__ __forceinline__ bf16x8 lora_load(const uint16_t* p) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p));
}
__device__ __forceinline__ bf16x8 lora_zero() { return __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u}); }

// grid: slots x parts.  Wave w takes the 32-wide steps w, w + 4, .. of its part
// of K; the waves' sums meet in LDS.  RT = row tiles of A (R <= 16 RT).
template <int TT, int RT>
__global__ __launch_bounds__(kLoraThreads)
void k_lora_down(LoraArgs a) {
  __shared__ f32x4 sum[kLoraWaves / 2][TT * RT][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g = lane / 16, c = lane % 16;
  const int part = blockIdx.x % a.parts;
  const LoraTile t = lora_tile_of<TT>(a, blockIdx.x / a.parts);
  if (t.rows <= 0 || t.adapter < 0) return;   // uniform
  // rows behind the last repeat it: their sums are not stored
  const uint16_t* xr[TT];
  const uint16_t* ar[RT];
#pragma unroll
  for (int i = 0; i < TT; ++i) xr[i] = a.x + (t.t0 + min(16 * i + c, t.rows - 1)) * a.ldx + 8 * g;
#pragma unroll
  for (int i = 0; i < RT; ++i)
    ar[i] = a.A + (static_cast<int64_t>(t.adapter) * a.R + min(16 * i + c, a.R - 1)) * a.K + 8 * g;
  f32x4 acc[TT][RT];
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = zero4();
  const int steps = (a.K + 31) / 32;
  const int per = (steps + a.parts - 1) / a.parts;
  const int end = min(steps, (part + 1) * per);
  // four steps' loads are in flight together
  constexpr int AHEAD = 4;
  for (int k = part * per + wave; k < end; k += AHEAD * kLoraWaves) {
    bf16x8 xf[AHEAD][TT], af[AHEAD][RT];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) {
      // a step behind the last one, or columns behind K (a multiple of 8), count as zero;
      // what is loaded for them is the row's start
      const int kn = k + n * kLoraWaves;
      const bool in = kn < end && 32 * kn + 8 * g < a.K;
      const int off = in ? 32 * kn : -8 * g;
#pragma unroll
      for (int i = 0; i < TT; ++i) xf[n][i] = lora_load(xr[i] + off);
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        af[n][j] = lora_load(ar[j] + off);
        if (!in) af[n][j] = lora_zero();
      }
#pragma unroll
      for (int i = 0; i < TT; ++i)
        if (!in) xf[n][i] = lora_zero();
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < AHEAD; ++n)
#pragma unroll
      for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = mma(af[n][j], xf[n][i], acc[i][j]);   // rows r, columns tokens
  }
  // waves 2 and 3 hand over to 0 and 1, then 1 to 0: a fixed order
#pragma unroll
  for (int half = kLoraWaves / 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) sum[wave - half][i * RT + j][lane] = acc[i][j];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] += sum[wave][i * RT + j][lane][e];
    __syncthreads();
  }
  if (wave != 0) return;
  const float s = a.scales ? a.scales[t.adapter] : 1.0f;
  float* u = a.u + (part * a.tokens + t.t0) * a.R;
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int r = 16 * j + 4 * g;
      if (16 * i + c < t.rows && r < a.R)
        *reinterpret_cast<f32x4*>(u + static_cast<int64_t>(16 * i + c) * a.R + r) =
            f32x4{s * acc[i][j][0], s * acc[i][j][1], s * acc[i][j][2], s * acc[i][j][3]};
    }
}

// Eight output columns of a token: read as they lie (the value is made of them
// after the products, so the load stays in flight), by streaming 16-byte accesses
// (base and out pass once), or one by one where rows are not aligned.
template <typename T, bool WIDE>
struct Cols8 {
  static constexpr int kVecs = 8 * static_cast<int>(sizeof(T)) / 16;
  u32x4 raw[kVecs];
  __device__ __forceinline__ void load(const T* p, int) {
#pragma unroll
    for (int j = 0; j < kVecs; ++j) raw[j] = reinterpret_cast<const u32x4*>(p)[j];
  }
  __device__ __forceinline__ float get(int e) const {
    constexpr int E = 16 / static_cast<int>(sizeof(T));
    return vec_elt<T>(raw[e / E], e % E);
  }
  static __device__ __forceinline__ void store(T* p, int, const float (&v)[8]) {
    u32x4 w[kVecs];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 2) {
        const f32x2 pair = {v[2 * j], v[2 * j + 1]};
        w[0][j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2));
      } else {
        w[0][j] = __float_as_uint(v[j]);
        w[1][j] = __float_as_uint(v[4 + j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kVecs; ++j) reinterpret_cast<u32x4*>(p)[j] = w[j];
  }
};
template <typename T>
struct Cols8<T, false> {
  T raw[8];
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) raw[e] = p[e];
  }
  __device__ __forceinline__ float get(int e) const { return load_elt(raw, e); }
  static __device__ __forceinline__ void store(T* p, int n, const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float one[1] = {v[e]};
      if (e < n) store_run<T, 1>(p + e, one);
    }
  }
};

// w rounded to bf16; w keeps what the rounding left (exact).
__device__ __forceinline__ bf16x8 round_off8(float (&w)[8]) {
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const f32x2 pair = {w[2 * p], w[2 * p + 1]};
    r[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2));
    w[2 * p] -= __uint_as_float(r[p] << 16);
    w[2 * p + 1] -= __uint_as_float(r[p] & 0xFFFF0000u);
  }
  return __builtin_bit_cast(bf16x8, r);
}

// Tiles of bf16 tokens pass through LDS, so that base and out move as whole rows
// of 512 bytes: 4324 tokens 47.5 us, 52 by 64-byte pieces of 16 rows from the lanes.
// (Those of fp32 are 128 bytes.)
constexpr int kLoraPitch = 2 * kLoraCols + 64;
template <typename T, int TT, bool WIDE>
constexpr bool lora_rows() { return sizeof(T) == 2 && WIDE; }

// grid: slots x column tiles, an XCD takes neighbouring ones (they share u, and
// the adapter's B stays in its L2).  A workgroup: a token tile x 256 columns, 64
// of them a wave's, KS steps over the rank.  The tile's u goes through LDS once
// for the four waves, as operands of bf16 parts: two (within 2^-16) where the
// outputs are bf16, three (24 bits) where they are fp32.  A tile's rows of B are
// taken in the order in which a lane ends up with eight neighbouring columns of
// a token.  Rows through LDS: registers for as many waves as it holds workgroups
// (left alone the compiler reads all of a tile ahead, with one wave a SIMD 81 us
// for those 47.5).
template <typename T, int TT, int KS, bool WIDE>
__global__ __launch_bounds__(kLoraThreads, (lora_rows<T, TT, WIDE>() ? (TT == 4 ? (KS < 4 ? 3 : 2) : 4) : 1))
void k_lora_up(LoraArgs a) {
  constexpr int NP = sizeof(T) == 2 ? 2 : 3;
  __shared__ bf16x8 uf[TT * KS][NP][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g = lane / 16, c = lane % 16;
  const int tiles = (a.M + kLoraCols - 1) / kLoraCols;
  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const LoraTile t = lora_tile_of<TT>(a, unit / tiles);
  const bool adapted = t.adapter >= 0;
  if (t.rows <= 0 || (!adapted && a.out == a.base)) return;   // uniform
  const int m0 = unit % tiles * kLoraCols + wave * kLoraWaveCols;   // may lie behind M: the wave then only helps with u
  constexpr int BLOCKS = kLoraWaveCols / 32;
  const T* base = static_cast<const T*>(a.base) + t.t0 * a.ldbase;
  T* out = static_cast<T*>(a.out) + t.t0 * a.ldout;
  // everything that is read is on its way before anything waits
  constexpr bool ROWS = lora_rows<T, TT, WIDE>();
  constexpr int PIECES = kLoraCols / 8, STEP = kLoraThreads / PIECES, NPC = ROWS ? lora_tile(TT) / STEP : 1;
  __shared__ __attribute__((aligned(16))) char tile[ROWS ? lora_tile(TT) * kLoraPitch : 16];
  const int prow = threadIdx.x / PIECES, pcol = threadIdx.x % PIECES;
  const int pm = unit % tiles * kLoraCols + 8 * pcol;
  u32x4 piece[NPC];
  Cols8<T, WIDE> was[ROWS ? 1 : TT][BLOCKS];
  if constexpr (ROWS) {
#pragma unroll
    for (int k = 0; k < NPC; ++k)
      if (prow + k * STEP < t.rows && pm < a.M)
        piece[k] = *reinterpret_cast<const u32x4*>(base + (prow + k * STEP) * a.ldbase + pm);
  } else {
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        const int row = 16 * i + c, m = m0 + 32 * b + 8 * g;
        if (row < t.rows && m < a.M) was[i][b].load(base + row * a.ldbase + m, a.M - m);
      }
  }
  bf16x8 bf[BLOCKS][2][KS];
  if (adapted) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int m = min(m0 + 32 * b + 8 * (c / 4) + 4 * h + c % 4, a.M - 1);
        const uint16_t* p = a.B + t.adapter * a.b_stride + static_cast<int64_t>(m) * a.R + 8 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) bf[b][h][k] = 32 * k + 8 * g < a.R ? lora_load(p + 32 * k) : lora_zero();
      }
#pragma unroll
    for (int f = 0; f < TT * KS; f += kLoraWaves) {
      if (f + wave >= TT * KS) break;
      const int i = (f + wave) / KS, k = (f + wave) % KS;
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = 0.0f;
      if (32 * k + 8 * g < a.R) {
        const float* p = a.u + (t.t0 + min(16 * i + c, t.rows - 1)) * a.R + 32 * k + 8 * g;
        for (int s = 0; s < a.parts; ++s) {
          float q[8];
          load_run<float, 8>(p + s * a.tokens * a.R, q);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] += q[e];
        }
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) uf[f + wave][p][lane] = round_off8(w);
    }
  }
  if constexpr (ROWS) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < NPC; ++k)
      *reinterpret_cast<u32x4*>(tile + (prow + k * STEP) * kLoraPitch + 16 * pcol) = piece[k];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    if constexpr (ROWS) __builtin_amdgcn_sched_barrier(0);
    f32x4 acc[BLOCKS][2];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[b][h] = zero4();
    if (adapted) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const bf16x8 u = uf[i * KS + k][p][lane];
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[b][h] = mma(bf[b][h][k], u, acc[b][h]);   // rows columns, columns tokens
        }
      }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int row = 16 * i + c, m = m0 + 32 * b + 8 * g;
      float v[8];
      if constexpr (ROWS) {
        if (!adapted) continue;
        T* place = reinterpret_cast<T*>(tile + row * kLoraPitch) + wave * kLoraWaveCols + 32 * b + 8 * g;
        was[0][b].load(place, 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = was[0][b].get(e) + acc[b][e / 4][e % 4];
        Cols8<T, WIDE>::store(place, 8, v);
      } else {
        if (row >= t.rows || m >= a.M) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = adapted ? was[i][b].get(e) + acc[b][e / 4][e % 4] : was[i][b].get(e);
        Cols8<T, WIDE>::store(out + row * a.ldout + m, a.M - m, v);
      }
    }
  }
  if constexpr (ROWS) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NPC; ++k)
      if (prow + k * STEP < t.rows && pm < a.M)
        *reinterpret_cast<u32x4*>(out + (prow + k * STEP) * a.ldout + pm) =
            *reinterpret_cast<const u32x4*>(tile + (prow + k * STEP) * kLoraPitch + 16 * pcol);
  }
}

}  // namespace gdn
