// Attention over a shared prefix and each sequence's own pages (C ABI in
// gdn_attn.h).
#pragma once

#include "gdn_varlen.h"

namespace gdn {

struct AttnArgs {
  int32_t n_seqs, heads, kv_heads, num_pages, page_size, width, prefix_len, max_len, tokens;
  float scale;
  const int32_t* cu;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* prefix_pages;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  int64_t ldq, ldo, kp, kt, kh, vp, vt, vh;
};

// A wave takes one query head of one token and 64 keys at a time, a key a lane
// for the scores, D / 64 columns a lane for the values.
constexpr int kAttnThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kAttnThreads)
void k_attn(AttnArgs a) {
  constexpr int NW = kAttnThreads / kWave, C = D / 64;
  __shared__ float qs[NW][D];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * NW + wave;
  if (unit >= static_cast<int64_t>(a.tokens) * a.heads) return;
  const int t = static_cast<int>(unit / a.heads), h = static_cast<int>(unit % a.heads), kvh = h / (a.heads / a.kv_heads);
  // the sequence of token t: the first whose end lies behind it
  int lo = 0, hi = a.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (a.cu[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  const int n = lo, len = min(max(a.lens[n], 0), a.max_len);
  const int own = max(min(len, len - (a.cu[n + 1] - t) + 1), 0);   // own tokens that the query sees
  const T* q = static_cast<const T*>(a.q) + t * a.ldq + h * D;
  for (int d = lane; d < D; d += kWave) qs[wave][d] = load_elt(q, d);
  __builtin_amdgcn_wave_barrier();
  float top = -INFINITY, sum = 0.0f, acc[C] = {};
  const auto walk = [&](const int32_t* pages, int count) {
    for (int j0 = 0; j0 < count; j0 += kWave) {
      const int j = j0 + lane;
      const int page = j < count ? pages[j / a.page_size] : -1, r = j % a.page_size;
      const bool seen = page >= 0 && page < a.num_pages;
      float s = -INFINITY;
      if (seen) {
        const T* k = static_cast<const T*>(a.k) + page * a.kp + r * a.kt + kvh * a.kh;
        s = 0.0f;
        for (int d = 0; d < D; d += 8) {
          float x[8];
          load_run<T, 8>(k + d, x);
          for (int e = 0; e < 8; ++e) s = fmaf(x[e], qs[wave][d + e], s);
        }
        s *= a.scale;
      }
      float m = s;
      for (int off = 1; off < kWave; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
      const float next = fmaxf(top, m), at = next == -INFINITY ? 0.0f : next;
      const float keep = expf(top - at), p = seen ? expf(s - at) : 0.0f;
      top = next;
      float ps = p;
      for (int off = 1; off < kWave; off <<= 1) ps += __shfl_xor(ps, off, kWave);
      sum = sum * keep + ps;
      for (int c = 0; c < C; ++c) acc[c] *= keep;
      for (int i = 0; i < kWave; ++i) {
        const int pg = __shfl(page, i, kWave), ri = __shfl(r, i, kWave);
        const float w = __shfl(p, i, kWave);
        if (pg < 0 || pg >= a.num_pages) continue;
        const T* v = static_cast<const T*>(a.v) + pg * a.vp + ri * a.vt + kvh * a.vh + C * lane;
        for (int c = 0; c < C; ++c) acc[c] = fmaf(w, load_elt(v, c), acc[c]);
      }
    }
  };
  walk(a.prefix_pages, a.prefix_len);
  walk(a.table + static_cast<int64_t>(n) * a.width, own);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* o = static_cast<T*>(a.out) + t * a.ldo + h * D + C * lane;
  for (int c = 0; c < C; ++c) {
    const float x[1] = {acc[c] * inv};
    store_run<T, 1>(o + c, x);
  }
}

}  // namespace gdn
