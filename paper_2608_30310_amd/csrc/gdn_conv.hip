// The short causal convolution: validation and launches (C ABI in gdn_ssm.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "gdn_conv.h"
#include "gdn_layer_plan.h"
#include "gdn_plan.h"

namespace gdn {
namespace {

gdn_status cfail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

gdn_status claunched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cfail(GDN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return GDN_OK;
}

constexpr int64_t kMaxGrid = 0x7fffffff / kConvThreads;   // work items of a grid dimension fit 32 bits

struct ConvArgs {
  const gdn_conv_shape* s;
  const int32_t* cu;
  int64_t tokens;
  const void* x;
  const float* w;
  const float* bias;
  const void* hist_in;
  void* y;
  void* hist_out;
  hipStream_t stream;
};

template <typename T, int VEC, int W, bool SILU>
gdn_status launch_conv(const ConvArgs& a) {
  const gdn_conv_shape& s = *a.s;
  const int64_t slabs = (s.channels + kConvLanes * VEC - 1) / (kConvLanes * VEC);
  if (!a.cu) {   // one token per sequence
    const int64_t threads = (s.channels + VEC - 1) / VEC;
    const int block = 64;
    const int64_t bx = (threads + block - 1) / block;
    // a thread keeps its taps over its sequences: 128, 256 and 1024 of 8192 channels
    // take 5.8, 7.9 and 23 us in 1024 workgroups, 6.8, 11.5 and 43 in 256, 7.2, 12.0 and 24 in 4096
    const int64_t by = std::min<int64_t>(s.num_seqs, std::max<int64_t>(1, 1024 / bx));
    hipLaunchKernelGGL((k_causal_conv_step<T, VEC, W, SILU>), dim3(static_cast<uint32_t>(bx), static_cast<uint32_t>(by)),
                       dim3(block), 0, a.stream, s.num_seqs, s.channels, static_cast<const T*>(a.x), s.ld_x, a.w,
                       a.bias, static_cast<const T*>(a.hist_in), static_cast<T*>(a.y), s.ld_y,
                       static_cast<T*>(a.hist_out));
    return claunched("convolution step launch");
  }
  // Eight tokens a thread (11 rows read for 8 written) as soon as half the CUs have
  // a workgroup, else one: 8192 channels, 64, 128, 512 and 8192 tokens take 5.5,
  // 5.6, 7.3 and 56 us with eight, 4.6, 5.6, 12.2 and 63 with one.
  const bool many = tile_slots(a.tokens, s.num_seqs, conv_tile(8)) * slabs >= 128;
  const int64_t slots = tile_slots(a.tokens, s.num_seqs, conv_tile(many ? 8 : 1));
  if (slots > 0x7fffffff) return cfail(GDN_ERR_UNSUPPORTED, "too many token tiles");
  // a workgroup keeps its taps over its tiles; 4096 of them end evenly (16384 tokens
  // 108 us, with 2048 111, with 1024 113)
  const int64_t rows = std::min(slots, std::max<int64_t>(1, 4096 / slabs));
  if (rows * slabs > kMaxGrid) return cfail(GDN_ERR_UNSUPPORTED, "too many channels");
  auto kernel = many ? k_causal_conv<T, VEC, W, 8, SILU> : k_causal_conv<T, VEC, W, 1, SILU>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(rows * slabs)), dim3(kConvThreads), 0, a.stream,
                     static_cast<int32_t>(slots), static_cast<int32_t>(slabs), s.num_seqs, a.cu, s.channels,
                     static_cast<const T*>(a.x), s.ld_x, a.w, a.bias, static_cast<const T*>(a.hist_in),
                     static_cast<T*>(a.y), s.ld_y, static_cast<T*>(a.hist_out));
  return claunched("convolution launch");
}

template <typename T, int VEC, int W>
gdn_status conv_act(const ConvArgs& a) {
  return a.s->activation == GDN_ACT_SILU ? launch_conv<T, VEC, W, true>(a) : launch_conv<T, VEC, W, false>(a);
}

template <typename T, int VEC>
gdn_status conv_taps(const ConvArgs& a) {
  switch (a.s->taps) {
    case 2: return conv_act<T, VEC, 2>(a);
    case 3: return conv_act<T, VEC, 3>(a);
    default: return conv_act<T, VEC, 4>(a);
  }
}

template <typename T>
gdn_status conv_align(const ConvArgs& a) {
  constexpr int V = conv_vec<T, true>();
  const gdn_conv_shape& s = *a.s;
  bool wide = s.channels % V == 0 && s.ld_x % V == 0 && s.ld_y % V == 0;
  for (const void* p : {a.x, static_cast<const void*>(a.y), a.hist_in, static_cast<const void*>(a.hist_out)})
    wide = wide && reinterpret_cast<uintptr_t>(p) % 16 == 0;
  return wide ? conv_taps<T, V>(a) : conv_taps<T, 1>(a);
}

// cu == nullptr: one token per sequence
gdn_status conv_impl(const ConvArgs& a) {
  const gdn_conv_shape& s = *a.s;
  const int64_t e = s.dtype == GDN_BF16 ? 2 : 4;
  if (!a.w) return cfail(GDN_ERR_NULL_ARG, "weight is NULL");
  if (a.tokens > 0 && (!a.x || !a.y)) return cfail(GDN_ERR_NULL_ARG, "x and y must be non-NULL");
  for (const void* p : {a.x, static_cast<const void*>(a.y), a.hist_in, static_cast<const void*>(a.hist_out)})
    if (reinterpret_cast<uintptr_t>(p) % e != 0)
      return cfail(GDN_ERR_UNSUPPORTED, "x, y and the histories must be aligned to their elements");
  const size_t hb = static_cast<size_t>(s.num_seqs) * (s.taps - 1) * s.channels * e;
  if (a.hist_in != a.hist_out && a.hist_in && a.hist_out && overlap(a.hist_in, hb, a.hist_out, hb))
    return cfail(GDN_ERR_BAD_SHAPE, "history_out overlaps history_in without being equal");
  if (a.tokens > 0) {
    const int64_t row = s.channels * e;
    const int64_t ex = (a.tokens - 1) * s.ld_x * e + row, ey = (a.tokens - 1) * s.ld_y * e + row;
    if (rows_overlap(a.x, row, s.ld_x * e, a.y, row, s.ld_y * e, a.tokens))
      return cfail(GDN_ERR_BAD_SHAPE, "y overlaps x");
    if ((a.hist_in && overlap(a.hist_in, hb, a.y, ey)) || (a.hist_out && overlap(a.hist_out, hb, a.y, ey)) ||
        (a.hist_out && overlap(a.hist_out, hb, a.x, ex)))
      return cfail(GDN_ERR_BAD_SHAPE, "a history overlaps x or y");
  }
  return s.dtype == GDN_BF16 ? conv_align<uint16_t>(a) : conv_align<float>(a);
}

}  // namespace
}  // namespace gdn

extern "C" {

gdn_status gdn_causal_conv(const gdn_conv_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                           const void* x, const float* weight, const float* bias, const void* history_in, void* y,
                           void* history_out, void* stream) {
  std::string err;
  gdn_status st = gdn::check_conv(shape, &err);
  int64_t tokens = 0, longest = 0;
  if (st == GDN_OK) st = gdn::check_seqlens(shape->num_seqs, cu_seqlens_host, &tokens, &longest, &err);
  if (st != GDN_OK) return gdn::cfail(st, err);
  if (shape->num_seqs == 0 || (tokens == 0 && !history_out)) return GDN_OK;
  if (!cu_seqlens) return gdn::cfail(GDN_ERR_NULL_ARG, "cu_seqlens (device) is NULL");
  return gdn::conv_impl({shape, cu_seqlens, tokens, x, weight, bias, history_in, y, history_out,
                         static_cast<hipStream_t>(stream)});
}

gdn_status gdn_causal_conv_step(const gdn_conv_shape* shape, const void* x, const float* weight, const float* bias,
                                const void* history_in, void* y, void* history_out, void* stream) {
  std::string err;
  const gdn_status st = gdn::check_conv(shape, &err);
  if (st != GDN_OK) return gdn::cfail(st, err);
  if (shape->num_seqs == 0) return GDN_OK;
  if (!history_out) return gdn::cfail(GDN_ERR_NULL_ARG, "history_out is NULL");
  return gdn::conv_impl({shape, nullptr, shape->num_seqs, x, weight, bias, history_in, y, history_out,
                         static_cast<hipStream_t>(stream)});
}

}  // extern "C"
