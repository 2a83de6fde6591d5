// Low-rank adapters beside a shared projection: validation and launches (C ABI
// in gdn_lora.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "gdn_layer_plan.h"
#include "gdn_lora_call.h"
#include "gdn_lora_kernels.h"
#include "gdn_plan.h"

namespace gdn {
namespace {

gdn_status lfail(gdn_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

gdn_status llaunched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return lfail(GDN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return GDN_OK;
}

template <typename T, int TT, bool WIDE>
void launch_up(const LoraArgs& k, int64_t slots, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(slots * ((k.M + kLoraCols - 1) / kLoraCols)));
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kLoraThreads), 0, stream, k); };
  if (k.R <= 32) run(k_lora_up<T, TT, 1, WIDE>);
  else if (k.R <= 64) run(k_lora_up<T, TT, 2, WIDE>);
  else run(k_lora_up<T, TT, 4, WIDE>);
}

template <int TT>
void launch_down(const LoraArgs& k, int64_t slots, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(slots * k.parts));
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kLoraThreads), 0, stream, k); };
  if (k.R <= 16) run(k_lora_down<TT, 1>);
  else if (k.R <= 32) run(k_lora_down<TT, 2>);
  else if (k.R <= 64) run(k_lora_down<TT, 4>);
  else run(k_lora_down<TT, 8>);
}

template <typename T>
gdn_status launch_lora(const LoraArgs& k, const LoraPlan& p, bool any, bool wide, hipStream_t stream) {
  if (any) {
    if (p.down_tile == lora_tile(2)) launch_down<2>(k, p.down_slots, stream);
    else launch_down<1>(k, p.down_slots, stream);
  }
  const auto up = [&](auto tt) {
    if (wide) launch_up<T, tt.value, true>(k, p.up_slots, stream);
    else launch_up<T, tt.value, false>(k, p.up_slots, stream);
  };
  if (p.up_tile == lora_tile(4)) up(std::integral_constant<int, 4>{});
  else if (p.up_tile == lora_tile(2)) up(std::integral_constant<int, 2>{});
  else up(std::integral_constant<int, 1>{});
  return llaunched("adapter launch");
}

}  // namespace

gdn_status lora_run(const gdn_lora_shape* s, const int32_t* cu_host, const int32_t* cu, const int32_t* adapters_host,
                    const int32_t* adapters, const void* base, const void* x, const void* A, const void* B,
                    int64_t b_stride, const float* scales, void* out, void* workspace, size_t workspace_bytes,
                    void* stream_ptr) {
  std::string err;
  LoraPlan p;
  const gdn_status st = make_lora_plan(s, cu_host, &p, &err);
  if (st != GDN_OK) return lfail(st, err);
  const int64_t tokens = p.tokens;
  if (s->num_seqs == 0) return GDN_OK;
  if (tokens > 0 && !adapters_host) return lfail(GDN_ERR_NULL_ARG, "adapters_host is NULL");
  bool any = false;
  for (int32_t n = 0; adapters_host && n < s->num_seqs; ++n) {
    if (adapters_host[n] < -1 || adapters_host[n] >= s->num_adapters)
      return lfail(GDN_ERR_BAD_SHAPE, "adapters_host must hold -1 or an adapter's index");
    any = any || (adapters_host[n] >= 0 && cu_host[n + 1] > cu_host[n]);
  }
  if (tokens == 0) return GDN_OK;
  if (!cu || !adapters) return lfail(GDN_ERR_NULL_ARG, "cu_seqlens and adapters (device) must be non-NULL");
  if (!base || !out) return lfail(GDN_ERR_NULL_ARG, "base and out must be non-NULL");
  if (any && (!x || !A || !B)) return lfail(GDN_ERR_NULL_ARG, "x, lora_a and lora_b must be non-NULL");
  const auto off = [](const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; };
  if (off(x, 16) || off(A, 16) || off(B, 16)) return lfail(GDN_ERR_UNSUPPORTED, "x, lora_a and lora_b must be 16-byte aligned");
  const int64_t e = s->out_dtype == GDN_BF16 ? 2 : 4, row = s->width * e;
  if (off(base, e) || off(out, e)) return lfail(GDN_ERR_UNSUPPORTED, "base and out must be aligned to their elements");
  if (base == out ? s->ld_base != s->ld_out : rows_overlap(base, row, s->ld_base * e, out, row, s->ld_out * e, tokens))
    return lfail(GDN_ERR_BAD_SHAPE, "out overlaps base without being equal");
  if (x && rows_overlap(x, s->hidden * 2, s->ld_x * 2, out, row, s->ld_out * e, tokens))
    return lfail(GDN_ERR_BAD_SHAPE, "out overlaps x");
  if (!workspace) return lfail(GDN_ERR_WORKSPACE, "workspace is NULL");
  if (workspace_bytes < p.bytes)
    return lfail(GDN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(p.bytes) + " bytes, got " +
                                        std::to_string(workspace_bytes));
  if (off(workspace, kAlign)) return lfail(GDN_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (!any && base == out) return GDN_OK;
  const LoraArgs k{s->num_seqs, s->num_adapters, s->hidden, s->width, s->rank, p.parts,
                   tokens, cu, adapters, static_cast<const uint16_t*>(x), s->ld_x, static_cast<const uint16_t*>(A),
                   static_cast<const uint16_t*>(B), b_stride, scales, base, s->ld_base, out, s->ld_out,
                   static_cast<float*>(workspace)};
  const hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
  const int64_t vec = 16 / e;
  const bool wide = s->width % vec == 0 && s->ld_base % vec == 0 && s->ld_out % vec == 0 && s->width % 8 == 0 &&
                    !off(base, 16) && !off(out, 16);
  return s->out_dtype == GDN_BF16 ? launch_lora<uint16_t>(k, p, any, wide, stream)
                                  : launch_lora<float>(k, p, any, wide, stream);
}

}  // namespace gdn

extern "C" {

gdn_status gdn_lora_workspace_size(const gdn_lora_shape* shape, const int32_t* cu_seqlens_host, size_t* bytes) {
  if (!bytes) return gdn::lfail(GDN_ERR_NULL_ARG, "bytes is NULL");
  std::string err;
  gdn::LoraPlan p;
  const gdn_status st = gdn::make_lora_plan(shape, cu_seqlens_host, &p, &err);
  if (st != GDN_OK) return gdn::lfail(st, err);
  *bytes = p.bytes;
  return GDN_OK;
}

gdn_status gdn_lora_add(const gdn_lora_shape* shape, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens,
                        const int32_t* adapters_host, const int32_t* adapters, const void* base, const void* x,
                        const void* lora_a, const void* lora_b, const float* scales, void* out, void* workspace,
                        size_t workspace_bytes, void* stream) {
  const int64_t b_stride = shape ? static_cast<int64_t>(shape->width) * shape->rank : 0;
  return gdn::lora_run(shape, cu_seqlens_host, cu_seqlens, adapters_host, adapters, base, x, lora_a, lora_b, b_stride,
                       scales, out, workspace, workspace_bytes, stream);
}

}  // extern "C"
