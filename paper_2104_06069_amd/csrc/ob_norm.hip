// libonebitlamb: host side of the root-mean-square norm (include/ob_layer.h) -- contexts, argument validation and launches.  The
// kernels live in ob_norm_kernels.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

#include "ob_host.h"
#include "ob_layer.h"
#include "ob_norm_kernels.h"

using namespace obl;

struct ob_norm_ctx {
  ob_norm_config cfg;
  int device = -1;
  int most_parts = 1;      // workgroups of k_norm_backward that there is room for
  size_t bytes = 0;
  float* d_partial = nullptr;
  std::string hip_err;
  ~ob_norm_ctx() {
    if (d_partial) (void)hipFree(d_partial);
  }
};

namespace {

constexpr int64_t MOST_N = 16384, MOST_LD = (int64_t)1 << 31;

template <int V>
using Int = std::integral_constant<int, V>;

// f(type of x, type of h)
template <class F>
ob_status with_types(const ob_norm_config& c, F f) {
  if (c.dtype == OB_F32) return f(Int<F32>{}, Int<F32>{});
  if (c.dtype == OB_F16) return c.res_dtype == OB_F32 ? f(Int<F16>{}, Int<F32>{}) : f(Int<F16>{}, Int<F16>{});
  return c.res_dtype == OB_F32 ? f(Int<BF16>{}, Int<F32>{}) : f(Int<BF16>{}, Int<BF16>{});
}

// f(threads of a row, pieces of a thread): one piece each where a workgroup has threads for that, so that a row is one trip to
// memory and many rows are under way (forward 16384 x 2048: 42.8 us, four pieces of a wavefront 44.4; backward 57.9, four pieces 95).
// What the weight's gradient takes of the registers speaks for wavefronts of their own with rows up to 1024 (32768 rows: the same time as
// with two wavefronts a row), and above 8192 there are not threads enough.
template <class F>
ob_status with_forward_size(int64_t n, F f) {
  if (n <= 512) return f(Int<64>{}, Int<1>{});
  if (n <= 1024) return f(Int<128>{}, Int<1>{});
  if (n <= 2048) return f(Int<256>{}, Int<1>{});
  if (n <= 4096) return f(Int<512>{}, Int<1>{});
  if (n <= 8192) return f(Int<1024>{}, Int<1>{});
  return f(Int<512>{}, Int<4>{});
}
template <class F>
ob_status with_backward_size(int64_t n, F f) {
  if (n <= 512) return f(Int<64>{}, Int<1>{});
  if (n <= 1024) return f(Int<64>{}, Int<2>{});
  if (n <= 2048) return f(Int<256>{}, Int<1>{});
  if (n <= 4096) return f(Int<512>{}, Int<1>{});
  if (n <= 8192) return f(Int<1024>{}, Int<1>{});
  return f(Int<512>{}, Int<4>{});
}

// rows that a workgroup of k_norm_backward has at a time
int sets_of(int64_t n) { return n <= 1024 ? 8 : n <= 2048 ? 2 : 1; }
// and workgroups of it, as many as the card runs at once (16384 x 2048 with 256 / 512 / 768 / 1024 of them: 81.4 / 62.3 / 57.9 / 68.9 us; 32768 x 1024,
// where two wavefronts' registers less fit: 512 / 768: 61.8 / 74.4; binary32 16384 x 2048: 113 / 136)
int parts_of(int64_t n, bool f32) { return !f32 && (n <= 512 || (n > 1024 && n <= 4096)) ? 768 : 512; }

bool rows_wrong(int64_t ld, int64_t n) { return ld < n || ld >= MOST_LD; }

}  // namespace

extern "C" {

ob_status ob_norm_create(const ob_norm_config* cfg, ob_norm_ctx** out) {
  if (!cfg || !out) return OB_ERR_NULL;
  *out = nullptr;
  if (cfg->n < 1 || cfg->n > MOST_N || !any_dtype(cfg->dtype) || (cfg->res_dtype != cfg->dtype && cfg->res_dtype != OB_F32) ||
      !any_dtype(cfg->weight_dtype) || !(cfg->eps >= 0) || !std::isfinite(cfg->eps))
    return OB_ERR_ARG;
  ob_norm_ctx* ctx = new (std::nothrow) ob_norm_ctx();
  if (!ctx) return OB_ERR_ARG;
  ctx->cfg = *cfg;
  hipError_t e = hipGetDevice(&ctx->device);
  ctx->most_parts = parts_of(cfg->n, cfg->dtype == OB_F32);
  ctx->bytes = (size_t)ctx->most_parts * cfg->n * sizeof(float);
  if (e == hipSuccess) e = hipMalloc(&ctx->d_partial, ctx->bytes);
  if (e != hipSuccess) {
    delete ctx;
    return OB_ERR_HIP;
  }
  *out = ctx;
  return OB_OK;
}

void ob_norm_destroy(ob_norm_ctx* ctx) { delete ctx; }
size_t ob_norm_workspace_bytes(const ob_norm_ctx* ctx) { return ctx ? ctx->bytes : 0; }
const char* ob_norm_last_hip_error(const ob_norm_ctx* ctx) { return ctx ? ctx->hip_err.c_str() : ""; }

ob_status ob_norm_forward(ob_norm_ctx* ctx, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, int64_t rows,
                          void* h, int64_t ldh, void* y, int64_t ldy, void* data, int64_t ld, void* scales, int64_t ld_scales, int32_t format,
                          float* rstd, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  const ob_norm_config& c = ctx->cfg;
  const int64_t blocks = (c.n + BLOCK8 - 1) / BLOCK8;
  if (rows < 0 || rows > 0x7fffffff || rows_wrong(ldx, c.n) || (residual && (rows_wrong(ldr, c.n) || rows_wrong(ldh, c.n))) ||
      (y && rows_wrong(ldy, c.n)) || (data && (ld % BLOCK8 || rows_wrong(ld, c.n) || ld_scales % 4 || rows_wrong(ld_scales, blocks))) ||
      (data && format != OB_E4M3 && format != OB_E5M2))
    return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!rows) return OB_OK;
  if (!x || (residual && !h) || (!y && !data) || (data && !scales)) return OB_ERR_NULL;
  if (off_element(x, c.dtype) || off_element(residual, c.res_dtype) || (residual && off_element(h, c.res_dtype)) || off_element(weight, c.weight_dtype) ||
      off_element(y, c.dtype) || off(data, 16) || (data && off(scales, 4)) || off(rstd, 4))
    return OB_ERR_ALIGN;
  NormArgs p{x, residual, weight, h, y, static_cast<uint8_t*>(data), static_cast<uint8_t*>(scales), rstd, ldx, ldr, ldh, ldy, ld, ld_scales,
             (int)rows, (int)c.n, c.weight_dtype, format, c.eps};
  const auto part = [](auto* from, int64_t rows, int64_t ld, int size) { return from ? reinterpret_cast<decltype(from)>((uintptr_t)from + rows * ld * size) : nullptr; };
  return with_types(c, [&](auto X, auto H) {
    return with_forward_size(c.n, [&](auto T, auto C) {
      constexpr int NT = T < 256 ? 256 : T;
      constexpr int64_t MOST = ((int64_t)1 << 31) / T;      // rows of a launch: a grid counts its threads in 32 bits
      for (int64_t first = 0; first < rows; first += MOST) {
        NormArgs q = p;
        q.rows = (int)std::min(MOST, rows - first);
        q.x = part(p.x, first, ldx, elem_size(c.dtype));
        q.residual = part(p.residual, first, ldr, elem_size(c.res_dtype));
        q.h = part(p.h, first, ldh, elem_size(c.res_dtype));
        q.y = part(p.y, first, ldy, elem_size(c.dtype));
        q.data = part(p.data, first, ld, 1);
        q.scales = part(p.scales, first, ld_scales, 1);
        q.rstd = part(p.rstd, first, 1, 4);
        hipLaunchKernelGGL((k_norm_forward<X, H, T, C>), dim3((unsigned)((q.rows + NT / T - 1) / (NT / T))), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), q);
      }
      return hip_ok(ctx, hipGetLastError(), "k_norm_forward") ? OB_OK : OB_ERR_HIP;
    });
  });
}

ob_status ob_norm_backward(ob_norm_ctx* ctx, const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* rstd, const void* weight,
                           const void* dres, int64_t lddres, int64_t rows, void* dh, int64_t lddh, float* dweight, int32_t accumulate, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  const ob_norm_config& c = ctx->cfg;
  if (rows < 0 || rows > 0x7fffffff || rows_wrong(lddy, c.n) || rows_wrong(ldh, c.n) || (dres && rows_wrong(lddres, c.n)) || (dh && rows_wrong(lddh, c.n)))
    return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!dh && !dweight) return OB_ERR_NULL;
  if (rows && (!dy || !h || !rstd)) return OB_ERR_NULL;
  if (off_element(dy, c.dtype) || off_element(h, c.res_dtype) || off(rstd, 4) || off_element(weight, c.weight_dtype) || off_element(dres, c.res_dtype) ||
      off_element(dh, c.res_dtype) || off(dweight, 4))
    return OB_ERR_ALIGN;
  const int sets = sets_of(c.n);
  const int parts = (int)std::max<int64_t>(std::min<int64_t>((rows + sets - 1) / sets, ctx->most_parts), 1);
  NormGradArgs p{dy, h, weight, dres, rstd, dh, dweight, ctx->d_partial, lddy, ldh, lddres, lddh, (int)rows, (int)c.n, c.weight_dtype, accumulate != 0};
  if (!rows && !dweight) return OB_OK;      // (without rows one workgroup writes zeros to dweight, or adds them)
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return with_types(c, [&](auto X, auto H) {
    return with_backward_size(c.n, [&](auto T, auto C) {
      hipLaunchKernelGGL((k_norm_backward<X, H, T, C>), dim3((unsigned)parts), dim3(norm_grad_threads<T>()), 0, s, p);
      if (dweight && parts > 1)
        hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((c.n + 63) / 64)), dim3(SHARES * 64), 0, s, ctx->d_partial, parts, (int)c.n, p.accumulate, dweight);
      return hip_ok(ctx, hipGetLastError(), "k_norm_backward") ? OB_OK : OB_ERR_HIP;
    });
  });
}

}  // extern "C"
