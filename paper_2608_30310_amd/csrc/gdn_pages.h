// Pages and slots from lengths, and norm and rotation of queries and keys on
// their way into the pages (C ABI in gdn_attn.h).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

// ---------------------------------------------------------------- pages
struct PagesArgs {
  int32_t n_seqs, width, page_size, num_free, first;
  const int32_t* cu;
  const int32_t* table_in;
  const int32_t* lens_in;
  const int32_t* free_pages;
  const int32_t* taken_in;
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* taken_out;
  int32_t* slots;
  int32_t* positions;
  int32_t* have;    // workspace [N]: pages that a sequence holds already
  int32_t* index;   // [N]: where its new pages begin in free_pages
  int32_t* held;    // [N]: its tokens before the call
};
constexpr int32_t kMaxToken = 0x7FFFFFFF;

__device__ __forceinline__ int32_t pages_of(int64_t tokens, int32_t page_size, int32_t width) {
  const int64_t p = (tokens + page_size - 1) / page_size;
  return static_cast<int32_t>(p < width ? p : width);
}
__device__ __forceinline__ int32_t clamp_token(int64_t x) { return static_cast<int32_t>(x < kMaxToken ? x : kMaxToken); }

__device__ __forceinline__ int wave_sums(int x) {   // inclusive sums over the wave
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int up = __shfl_up(x, off, kWave);
    x += lane >= off ? up : 0;
  }
  return x;
}

// What sequence n holds, and takes.
struct PagesNeed { int32_t held, have, more, len; };
__device__ __forceinline__ PagesNeed pages_need(const PagesArgs& a, int n) {
  const int32_t held = max(a.lens_in[n], 0), have = pages_of(held, a.page_size, a.width);
  const int32_t len = clamp_token(static_cast<int64_t>(held) + (a.cu[n + 1] - a.cu[n]));
  return {held, have, pages_of(len, a.page_size, a.width) - have, len};
}

// One workgroup: the exclusive sums of what the sequences take.  The old lengths
// go to the workspace, since lens_out may be lens_in.
constexpr int kPagesPlanThreads = 1024;
__global__ __launch_bounds__(kPagesPlanThreads)
void k_pages_plan(PagesArgs a) {
  constexpr int NW = kPagesPlanThreads / kWave;
  __shared__ int sums[NW];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  int64_t base = a.taken_in ? max(a.taken_in[0], 0) : 0;
  for (int n0 = 0; n0 < a.n_seqs; n0 += kPagesPlanThreads) {
    const int n = n0 + tid;
    PagesNeed mine{};
    if (n < a.n_seqs) mine = pages_need(a, n);
    const int up_to = wave_sums(mine.more);
    if (lane == kWave - 1) sums[wave] = up_to;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < NW; ++w) {
      before += w < wave ? sums[w] : 0;
      all += sums[w];
    }
    if (n < a.n_seqs) {
      a.have[n] = mine.have;
      a.index[n] = clamp_token(base + before + up_to - mine.more);
      a.held[n] = mine.held;
      a.lens_out[n] = mine.len;
    }
    base += all;
    __syncthreads();
  }
  if (tid == 0) a.taken_out[0] = clamp_token(base);
}

// A workgroup takes TILE new tokens of a sequence, the first of a sequence its
// table row too.  Where table_out is table_in, entries below `have` are only read
// and those from it on only written.  PLANNED: behind k_pages_plan; else a workgroup
// sums up by itself what the sequences before its own take, which needs the old lengths
// and the old `taken` to stay, and spares a launch where there are few sequences (256
// single tokens: 12.9 -> 10.4 us a call, the kernels 5.5 -> 4.3).
constexpr int kPagesThreads = 256, kPagesFew = 1024;
template <int TILE, bool PLANNED>
__global__ __launch_bounds__(kPagesThreads)
void k_pages_fill(PagesArgs a) {
  const int tid = threadIdx.x;
  const int n = slot_seq(a.cu, a.n_seqs, blockIdx.x, TILE);
  const int start = a.cu[n], count = a.cu[n + 1] - start;
  const int64_t from = (static_cast<int64_t>(blockIdx.x) - (start / TILE + n)) * TILE;   // first new token of the tile
  int32_t have, index, held;
  if constexpr (PLANNED) {
    have = a.have[n], index = a.index[n], held = a.held[n];
  } else {
    __shared__ int sums[kPagesThreads / kWave];
    const PagesNeed mine = pages_need(a, n);
    int64_t base = a.taken_in ? max(a.taken_in[0], 0) : 0;
    int before = 0;
    for (int i = tid; i < n; i += kPagesThreads) before += pages_need(a, i).more;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) before += __shfl_xor(before, off, kWave);
    if (tid % kWave == 0) sums[tid / kWave] = before;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPagesThreads / kWave; ++w) base += sums[w];
    have = mine.have, index = clamp_token(base), held = mine.held;
    if (from == 0 && tid == 0) {
      a.lens_out[n] = mine.len;
      if (n == a.n_seqs - 1) a.taken_out[0] = clamp_token(base + mine.more);
    }
  }
  const int64_t row = static_cast<int64_t>(n) * a.width;
  const auto page_at = [&](int32_t c) {
    if (c < have) return a.table_in[row + c];
    const int64_t i = static_cast<int64_t>(index) + (c - have);
    return i < a.num_free ? a.free_pages[i] : -1;
  };
  if (from == 0) {
    const int32_t need = pages_of(clamp_token(static_cast<int64_t>(held) + count), a.page_size, a.width);
    const bool in_place = a.table_in == a.table_out;
    for (int c = in_place ? have + tid : tid; c < (in_place ? need : a.width); c += kPagesThreads)
      a.table_out[row + c] = c < need ? page_at(c) : a.table_in[row + c];
  }
  const int64_t end = from + TILE < count ? from + TILE : count;
  for (int64_t i = from + tid; i < end; i += kPagesThreads) {
    const int64_t at = held + i, c = at / a.page_size;
    const int32_t page = c < a.width ? page_at(static_cast<int32_t>(c)) : -1;
    const int64_t slot = static_cast<int64_t>(page) * a.page_size + (at - c * a.page_size);
    a.slots[start + i] = page >= 0 && slot <= kMaxToken ? static_cast<int32_t>(slot) : -1;
    a.positions[start + i] = clamp_token(a.first + at);
  }
}

// ---------------------------------------------------------------- norm and rotation
struct QkArgs {
  int32_t tokens, heads, kv_heads, rotary, num_positions, slots_end, page_size;
  float eps;
  const void* q;
  const void* k;
  const void* v;
  int64_t ldq, ldk, ldv, ldqo, ldko;
  const int32_t* positions;
  const float* cos_sin;
  const float* q_weight;
  const float* k_weight;
  const int32_t* slots;
  void* q_out;
  void* k_out;
  void* k_cache;
  void* v_cache;
  int64_t kp, kt, kh, vp, vt, vh;
};

// A thread takes eight elements of a head row, D / 8 neighbouring lanes a row; a wave up
// to R rows each of one token, whose cosines and sines it keeps.  All rows are asked for
// before the first is used.
constexpr int kQkThreads = 256, kQkWaves = kQkThreads / kWave;
// From here on (waves at one row for a lane) a wave takes four rows: the keys and queries
// of 820 tokens, 32 + 4 + 4 heads of 128, take 7.0 us with one and 8.2 with four, of 8192
// tokens 48 and 38 (with two or five as with four).
constexpr int64_t kQkManyWaves = 16384;
template <typename T, int D, bool INTERLEAVED, int R>
__global__ __launch_bounds__(kQkThreads)
void k_qk_norm_rope(QkArgs a, uint32_t chunks) {
  constexpr int LPR = D / 8, ROWS = kWave / LPR, V = sizeof(T) / 2;   // V: 16-byte pieces of eight elements
  const uint32_t id = __builtin_amdgcn_readfirstlane(blockIdx.x * kQkWaves + threadIdx.x / kWave);
  const int t = static_cast<int>(id / chunks), c = static_cast<int>(id % chunks);
  if (t >= a.tokens) return;
  const int lane = threadIdx.x % LPR, heads = a.heads + (a.v ? 2 : 1) * a.kv_heads;
  const int pos = a.positions[t], slot = a.k_cache ? a.slots[t] : -1;
  if (pos < 0 || pos >= a.num_positions) return;
  const int from = c * R * ROWS + threadIdx.x % kWave / LPR;
  u32x4 raw[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int u = min(from + i * ROWS, heads - 1);
    const T* src = u < a.heads ? static_cast<const T*>(a.q) + t * a.ldq + u * D
                   : u < a.heads + a.kv_heads ? static_cast<const T*>(a.k) + t * a.ldk + (u - a.heads) * D
                                              : static_cast<const T*>(a.v) + t * a.ldv + (u - a.heads - a.kv_heads) * D;
#pragma unroll
    for (int j = 0; j < V; ++j) raw[i][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 8 * lane) + j);
  }
  const int half = a.rotary / 2;
  const bool turned = 8 * lane < a.rotary, first = 8 * lane < half;
  constexpr int NC = INTERLEAVED ? 4 : 8;
  float co[NC] = {}, si[NC] = {};
  if (turned) {
    const float* cs = a.cos_sin + static_cast<int64_t>(pos) * a.rotary + (INTERLEAVED ? 4 * lane : 8 * lane - (first ? 0 : half));
    load_run<float, NC>(cs, co);
    load_run<float, NC>(cs + half, si);
  }
  // a pair's other element: 8 * half elements on, or back
  const int other = INTERLEAVED || !turned ? lane : first ? lane + half / 8 : lane - half / 8;
  const int64_t page = slot < 0 ? 0 : static_cast<uint32_t>(slot) / static_cast<uint32_t>(a.page_size);
  const int64_t in_page = slot < 0 ? 0 : slot - page * a.page_size;
  const bool kept = slot >= 0 && slot < a.slots_end;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int u = from + i * ROWS;
    if (u >= heads) return;   // whole rows of lanes leave together
    const bool is_q = u < a.heads, is_v = u >= a.heads + a.kv_heads;
    const int h = is_q ? u : is_v ? u - a.heads - a.kv_heads : u - a.heads;
    if (is_v) {
      if (kept) {
        u32x4* to = reinterpret_cast<u32x4*>(static_cast<T*>(a.v_cache) + page * a.vp + in_page * a.vt + h * a.vh + 8 * lane);
#pragma unroll
        for (int j = 0; j < V; ++j) to[j] = raw[i][j];
      }
      continue;
    }
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = vec_elt<T>(raw[i][j / (8 / V)], j % (8 / V));
    if (a.q_weight) {
      float s = 0.0f, w[8];
      load_run<float, 8>((is_q ? a.q_weight : a.k_weight) + 8 * lane, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], s);
#pragma unroll
      for (int off = 1; off < LPR; off <<= 1) s += __shfl_xor(s, off, LPR);
      const float r = rsqrtf(s * (1.0f / D) + a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * r * w[j];
    }
    if constexpr (INTERLEAVED) {
      if (turned) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const float e = x[2 * p], o = x[2 * p + 1];
          x[2 * p] = e * co[p] - o * si[p];
          x[2 * p + 1] = o * co[p] + e * si[p];
        }
      }
    } else {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = __shfl(x[j], other, LPR);
      if (turned) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = first ? x[j] * co[j] - y[j] * si[j] : x[j] * co[j] + y[j] * si[j];
      }
    }
    if (is_q) {
      store8(static_cast<T*>(a.q_out) + t * a.ldqo + h * D + 8 * lane, x);
    } else {
      if (a.k_out) store8(static_cast<T*>(a.k_out) + t * a.ldko + h * D + 8 * lane, x);
      if (kept) store8(static_cast<T*>(a.k_cache) + page * a.kp + in_page * a.kt + h * a.kh + 8 * lane, x);
    }
  }
}

}  // namespace gdn
