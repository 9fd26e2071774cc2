// libonebitlamb: host side of the gradient's norm and its clipping (include/ob_layer.h) -- contexts, tables of segments, argument
// validation and launches.  The kernels live in ob_clip_kernels.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ob_clip_kernels.h"
#include "ob_host.h"
#include "ob_layer.h"

using namespace obl;

struct ob_clip_ctx {
  int device = -1;
  int64_t n = 0;
  int layers = 0, segments = 0;
  float eps = 0, grad_scale = 1;
  void* mem = nullptr;
  size_t bytes = 0;
  Segment* d_segments = nullptr;
  int* d_first = nullptr;
  double *d_sums = nullptr, *d_layer_sums = nullptr;
  unsigned* d_ticket = nullptr;
  std::string hip_err;
  ~ob_clip_ctx() {
    if (mem) (void)hipFree(mem);
  }
};

namespace {

// Segments up to which the workgroups that apply the factor add them up themselves
constexpr int FEW_SEGMENTS = 1024;

size_t room(size_t bytes) { return (bytes + 255) / 256 * 256; }

ClipArgs args_of(const ob_clip_ctx* ctx, float* norm, float* layer_norms, float max_norm) {
  return ClipArgs{ctx->d_sums, ctx->d_first, ctx->d_layer_sums, ctx->d_ticket, norm, layer_norms, ctx->layers, ctx->segments, ctx->grad_scale, ctx->eps, max_norm};
}

void launch_squares(const ob_clip_ctx* ctx, const void* grad, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)ctx->segments);
  if (!ctx->segments) return;
  if (dtype == OB_F32) hipLaunchKernelGGL(k_clip_squares<F32>, grid, dim3(256), 0, s, ctx->d_segments, grad, ctx->d_sums);
  else if (dtype == OB_F16) hipLaunchKernelGGL(k_clip_squares<F16>, grid, dim3(256), 0, s, ctx->d_segments, grad, ctx->d_sums);
  else hipLaunchKernelGGL(k_clip_squares<BF16>, grid, dim3(256), 0, s, ctx->d_segments, grad, ctx->d_sums);
}

template <int IN, bool NORM>
void launch_apply_from(const ClipApplyArgs& p, int out_dtype, unsigned grid, hipStream_t s) {
  if (out_dtype == OB_F32) hipLaunchKernelGGL((k_clip_apply<IN, F32, NORM>), dim3(grid), dim3(256), 0, s, p);
  else if (out_dtype == OB_F16) hipLaunchKernelGGL((k_clip_apply<IN, F16, NORM>), dim3(grid), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((k_clip_apply<IN, BF16, NORM>), dim3(grid), dim3(256), 0, s, p);
}
template <bool NORM>
void launch_apply(const ClipApplyArgs& p, int in_dtype, int out_dtype, hipStream_t s) {
  const int64_t span = in_dtype == OB_F32 ? 4096 : 8192;
  const unsigned grid = (unsigned)std::max<int64_t>(p.apply ? (p.n + span - 1) / span : std::min((p.norm.layers + 3) / 4, 256), 1);
  if (in_dtype == OB_F32) launch_apply_from<F32, NORM>(p, out_dtype, grid, s);
  else if (in_dtype == OB_F16) launch_apply_from<F16, NORM>(p, out_dtype, grid, s);
  else launch_apply_from<BF16, NORM>(p, out_dtype, grid, s);
}

// The norm where norm_dst is not NULL, and with `apply` the clipped gradient
ob_status call(ob_clip_ctx* ctx, const void* grad, int dtype, float* norm_dst, float* layer_norms, const float* norm_src, bool apply, float max_norm, void* out,
               int out_dtype, void* hip_stream) {
  if (!any_dtype(dtype) || (apply && (!any_dtype(out_dtype) || !(max_norm >= 0)))) return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (ctx->n && (!grad || (apply && !out))) return OB_ERR_NULL;
  if (off_element(grad, dtype) || off(norm_dst, 4) || off(layer_norms, 4) || off(norm_src, 4) || (apply && off_element(out, out_dtype))) return OB_ERR_ALIGN;
  if (apply && ctx->n && out == grad && out_dtype != dtype) return OB_ERR_ARG;
  apply = apply && ctx->n;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool few = ctx->segments <= FEW_SEGMENTS;
  ClipApplyArgs p{args_of(ctx, norm_dst ? norm_dst : const_cast<float*>(norm_src), layer_norms, max_norm), grad, out, ctx->n, apply, out == grad};
  if (norm_dst) {
    launch_squares(ctx, grad, dtype, s);
    if (few) launch_apply<true>(p, dtype, apply ? out_dtype : dtype, s);
    else hipLaunchKernelGGL(k_clip_norm, dim3((unsigned)((ctx->layers + 3) / 4)), dim3(256), 0, s, p.norm);
  }
  if (apply && !(norm_dst && few)) launch_apply<false>(p, dtype, out_dtype, s);
  return hip_ok(ctx, hipGetLastError(), "k_clip") ? OB_OK : OB_ERR_HIP;
}

}  // namespace

extern "C" {

ob_status ob_clip_create(const ob_clip_config* cfg, ob_clip_ctx** out) {
  if (!cfg || !out) return OB_ERR_NULL;
  *out = nullptr;
  if (!cfg->layer_offsets) return OB_ERR_NULL;
  if (cfg->num_layers < 1 || cfg->num_layers > ((int64_t)1 << 22) || !(cfg->eps >= 0) || !std::isfinite(cfg->eps) || !(cfg->grad_scale > 0) ||
      !std::isfinite(cfg->grad_scale) || cfg->layer_offsets[0] != 0)
    return OB_ERR_ARG;
  for (int64_t l = 0; l < cfg->num_layers; ++l)
    if (cfg->layer_offsets[l + 1] < cfg->layer_offsets[l]) return OB_ERR_ARG;
  const int64_t n = cfg->layer_offsets[cfg->num_layers];
  if (n > ((int64_t)1 << 35)) return OB_ERR_ARG;
  ob_clip_ctx* ctx = nullptr;
  try {
    ctx = new ob_clip_ctx();
    ctx->n = n;
    ctx->layers = (int)cfg->num_layers;
    ctx->eps = cfg->eps;
    ctx->grad_scale = cfg->grad_scale;
    // Segments of 2048 elements, or twice as many as long as there would be over 4096 of them; from 32768 elements on, over 2^22 (a grid
    // counts its threads in 32 bits, and a tensor's last segment may be a short one)
    int64_t span = 2048;
    while (n / span > (span < 32768 ? 4096 : (int64_t)1 << 22)) span *= 2;
    std::vector<Segment> segments;
    std::vector<int> first;
    first.reserve(cfg->num_layers + 1);
    for (int64_t l = 0; l < cfg->num_layers; ++l) {
      first.push_back((int)segments.size());
      for (int64_t at = cfg->layer_offsets[l]; at < cfg->layer_offsets[l + 1]; at += span)
        segments.push_back(Segment{at, (int32_t)std::min(span, cfg->layer_offsets[l + 1] - at), (int32_t)l});
    }
    first.push_back((int)segments.size());
    ctx->segments = (int)segments.size();
    const size_t a = room(segments.size() * sizeof(Segment)), b = room(first.size() * sizeof(int)), c = room(segments.size() * sizeof(double)),
                 d = room(cfg->num_layers * sizeof(double));
    ctx->bytes = a + b + c + d + 256;
    hipError_t e = hipGetDevice(&ctx->device);
    if (e == hipSuccess) e = hipMalloc(&ctx->mem, ctx->bytes);
    if (e == hipSuccess) {
      char* const m = static_cast<char*>(ctx->mem);
      ctx->d_segments = reinterpret_cast<Segment*>(m);
      ctx->d_first = reinterpret_cast<int*>(m + a);
      ctx->d_sums = reinterpret_cast<double*>(m + a + b);
      ctx->d_layer_sums = reinterpret_cast<double*>(m + a + b + c);
      ctx->d_ticket = reinterpret_cast<unsigned*>(m + a + b + c + d);
      const unsigned zero = 0;
      if (!segments.empty()) e = hipMemcpy(ctx->d_segments, segments.data(), segments.size() * sizeof(Segment), hipMemcpyHostToDevice);
      if (e == hipSuccess) e = hipMemcpy(ctx->d_first, first.data(), first.size() * sizeof(int), hipMemcpyHostToDevice);
      if (e == hipSuccess) e = hipMemcpy(ctx->d_ticket, &zero, sizeof zero, hipMemcpyHostToDevice);
    }
    if (e != hipSuccess) {
      delete ctx;
      return OB_ERR_HIP;
    }
  } catch (...) {
    delete ctx;
    return OB_ERR_SIZE;
  }
  *out = ctx;
  return OB_OK;
}

void ob_clip_destroy(ob_clip_ctx* ctx) { delete ctx; }
size_t ob_clip_workspace_bytes(const ob_clip_ctx* ctx) { return ctx ? ctx->bytes : 0; }
const char* ob_clip_last_hip_error(const ob_clip_ctx* ctx) { return ctx ? ctx->hip_err.c_str() : ""; }

ob_status ob_clip_norm(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, float* norm, float* layer_norms, void* hip_stream) {
  if (!ctx || !norm) return OB_ERR_NULL;
  return call(ctx, grad, grad_dtype, norm, layer_norms, nullptr, false, 0.0f, nullptr, OB_F32, hip_stream);
}

ob_status ob_clip_apply(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, const float* norm, float max_norm, void* out, ob_dtype out_dtype,
                        void* hip_stream) {
  if (!ctx || !norm) return OB_ERR_NULL;
  return call(ctx, grad, grad_dtype, nullptr, nullptr, norm, true, max_norm, out, out_dtype, hip_stream);
}

ob_status ob_clip_norm_apply(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, float max_norm, float* norm, float* layer_norms, void* out,
                             ob_dtype out_dtype, void* hip_stream) {
  if (!ctx || !norm) return OB_ERR_NULL;
  return call(ctx, grad, grad_dtype, norm, layer_norms, nullptr, true, max_norm, out, out_dtype, hip_stream);
}

}  // extern "C"
