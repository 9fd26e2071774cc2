// libonebitlamb: host side of the linear layer in 8 bits (include/ob_layer.h) -- contexts, argument validation and launches.  The
// kernels live in ob_linear8_kernels.h and ob_mm8.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "ob_host.h"
#include "ob_layer.h"
#include "ob_linear8_kernels.h"
#include "ob_linear8_plan.h"

using namespace obl;

struct ob_linear8_ctx {
  ob_linear8_config cfg;
  int device = -1;
  size_t bytes = 0;
  float* d_partial = nullptr;
  std::string hip_err;
  ~ob_linear8_ctx() {
    if (d_partial) (void)hipFree(d_partial);
  }
};

namespace {

constexpr int64_t MOST = (int64_t)1 << 22;      // rows, columns and distances between rows: a tile's offsets are 32-bit

// Tiles by their side (ob_linear8_plan.h)
template <int KIND>
using Tile8 = std::conditional_t<KIND == W256, Shape<256, 256, 64, 2, 4>, std::conditional_t<KIND == W128, Shape<128, 128, 64, 2, 2>, Shape<64, 64, 64, 2, 2, KIND == TEAMS64 ? 4 : 3, KIND == TEAMS64 ? 2 : 1>>>;

template <int FORMAT, int OUT>
ob_status launch_flow(ob_linear8_ctx* ctx, const Product8Args& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.a.rows + 255) / 256) * ((p.b.rows + 255) / 256);
  hipLaunchKernelGGL((k_product8_flow<FORMAT, OUT>), dim3((unsigned)std::min<int64_t>((tiles + 7) / 8 * 8, CUS8)), dim3(256), (Flow8<FORMAT, OUT>::LDS_BYTES), s, p);
  return hip_ok(ctx, hipGetLastError(), "k_product8_flow") ? OB_OK : OB_ERR_HIP;
}

template <class S, int FORMAT, bool WIDE>
ob_status launch_product(ob_linear8_ctx* ctx, const Product8Args& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.a.rows + S::BM - 1) / S::BM) * ((p.b.rows + S::BN - 1) / S::BN) * p.parts;
  if ((tiles + 8) * S::NT > 0x7fffffff) return OB_ERR_SIZE;      // (a grid counts its threads in 32 bits)
  hipLaunchKernelGGL((k_product8<S, FORMAT, WIDE>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(S::NT), (Product8<S, FORMAT, WIDE>::LDS_BYTES), s, p);
  if (p.parts > 1) {
    const int64_t fours = (int64_t)p.a.rows * ((p.b.rows + 3) / 4);
    hipLaunchKernelGGL(k_product8_join, dim3((unsigned)((fours + 255) / 256)), dim3(256), 0, s, p);
  }
  return hip_ok(ctx, hipGetLastError(), "k_product8") ? OB_OK : OB_ERR_HIP;
}

// f(kind, format, wide)
template <class F>
auto with_product(int kind, int format, bool wide, F f) {
  const auto with_kind = [&](auto format, auto wide) {
    if (kind == W256) return f(std::integral_constant<int, W256>{}, format, wide);
    if (kind == W128) return f(std::integral_constant<int, W128>{}, format, wide);
    if (kind == TEAMS64) return f(std::integral_constant<int, TEAMS64>{}, format, wide);
    return f(std::integral_constant<int, W64>{}, format, wide);
  };
  const auto with_format = [&](auto format) { return wide ? with_kind(format, std::true_type{}) : with_kind(format, std::false_type{}); };
  return format == OB_E4M3 ? with_format(std::integral_constant<int, E4M3>{}) : with_format(std::integral_constant<int, E5M2>{});
}

// f(format, type of the results, ADD_F32 among them)
template <class F>
auto with_flow(int format, int out, F f) {
  const auto with_out = [&](auto format) {
    if (out == OB_F32) return f(format, std::integral_constant<int, F32>{});
    if (out == ADD_F32) return f(format, std::integral_constant<int, ADD_F32>{});
    if (out == OB_F16) return f(format, std::integral_constant<int, F16>{});
    return f(format, std::integral_constant<int, BF16>{});
  };
  return format == OB_E4M3 ? with_out(std::integral_constant<int, E4M3>{}) : with_out(std::integral_constant<int, E5M2>{});
}

hipError_t allow_products() {
  hipError_t e = hipSuccess;
  for (int kind = 0; kind < KINDS8; ++kind)
    for (const int format : {E4M3, E5M2})
      for (const bool wide : {false, true})
        if (e == hipSuccess)
          e = with_product(kind, format, wide, [](auto k, auto f, auto w) { return allow_lds(k_product8<Tile8<k>, f, w>, Product8<Tile8<k>, f, w>::LDS_BYTES); });
  for (const int format : {E4M3, E5M2})
    for (const int out : {(int)F32, (int)F16, (int)BF16, ADD_F32})
      if (e == hipSuccess) e = with_flow(format, out, [](auto f, auto o) { return allow_lds(k_product8_flow<f, o>, Flow8<f, o>::LDS_BYTES); });
  return e;
}

template <int R, int DTYPE, bool WIDE>
void launch_few(const FewArgs& f, hipStream_t s) {
  const FewPlan8 plan = few_plan8(f.p.b.rows, f.p.slabs);
  const dim3 grid((unsigned)((f.p.b.rows + plan.columns - 1) / plan.columns));
  if (plan.columns == 32) hipLaunchKernelGGL((k_product8_few<R, 2, 8, DTYPE, WIDE>), grid, dim3(512), 0, s, f);
  else if (plan.waves == 8) hipLaunchKernelGGL((k_product8_few<R, 1, 8, DTYPE, WIDE>), grid, dim3(512), 0, s, f);
  else hipLaunchKernelGGL((k_product8_few<R, 1, 16, DTYPE, WIDE>), grid, dim3(1024), 0, s, f);
}
template <bool WIDE>
void launch_few(const FewArgs& f, int x_dtype, hipStream_t s) {
  if (x_dtype == OB_F32) launch_few<1, F32, WIDE>(f, s);
  else if (x_dtype == OB_F16) launch_few<1, F16, WIDE>(f, s);
  else if (x_dtype == OB_BF16) launch_few<1, BF16, WIDE>(f, s);
  else if (f.p.a.rows <= 16) launch_few<1, NONE, WIDE>(f, s);
  else launch_few<2, NONE, WIDE>(f, s);
}

struct Given {      // an operand as a call has it
  const void* p;
  int64_t ld;
  const void* scales;
  int64_t ld_scales;
};
bool wrong(const Given& g, int64_t depth) { return g.ld % BLOCK8 || g.ld < depth || g.ld > MOST || g.ld_scales % 4 || g.ld_scales < (depth + BLOCK8 - 1) / BLOCK8 || g.ld_scales > MOST; }
bool misplaced(const Given& g) { return off(g.p, 16) || off(g.scales, 4); }

// out [rows, cols] = a [rows, depth] b [cols, depth]^T
ob_status product(ob_linear8_ctx* ctx, const Given& a, int format, const Given& b, bool b_square, int64_t rows, int64_t cols, int64_t depth, void* out,
                  int64_t ldo, int out_dtype, bool accumulate, void* hip_stream) {
  if (wrong(a, depth) || wrong(b, depth) || ldo < cols || ldo > MOST || !any_dtype(out_dtype) || (accumulate && out_dtype != OB_F32) ||
      (format != OB_E4M3 && format != OB_E5M2))
    return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!rows || !cols) return OB_OK;
  if (!out || (depth && (!a.p || !a.scales || !b.p || !b.scales))) return OB_ERR_NULL;
  if (misplaced(a) || misplaced(b) || off_element(out, out_dtype)) return OB_ERR_ALIGN;
  Product8Args p;
  p.a = Operand8{static_cast<const uint8_t*>(a.p), static_cast<const uint8_t*>(a.scales), a.ld, a.ld_scales, (int)rows, 0};
  p.b = Operand8{static_cast<const uint8_t*>(b.p), static_cast<const uint8_t*>(b.scales), b.ld, b.ld_scales, (int)cols, b_square ? 7 : 0};
  p.out = out;
  p.partial = ctx->d_partial;
  p.ldo = ldo;
  p.slabs = (int)((depth + BLOCK8 - 1) / BLOCK8);
  p.out_dtype = out_dtype;
  p.accumulate = accumulate;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (few8(rows, p.slabs)) {
    p.parts = 1;
    const FewArgs f{p, nullptr, 0, (int)depth, format};
    if (out_dtype == OB_F32) launch_few<true>(f, NONE, s);
    else launch_few<false>(f, NONE, s);
    return hip_ok(ctx, hipGetLastError(), "k_product8_few") ? OB_OK : OB_ERR_HIP;
  }
  const bool wide = out_dtype == OB_F32, eights = cols % 8 == 0 && ldo % 8 == 0 && !off(out, 16) && ldo <= ((int64_t)1 << 20);
  const Plan8 plan = plan8(rows, cols, p.slabs, wide, eights && p.slabs >= 2);
  p.parts = plan.parts;
  if (plan.kind == FLOW256) return with_flow(format, accumulate ? ADD_F32 : out_dtype, [&](auto f, auto o) { return launch_flow<f, o>(ctx, p, s); });
  return with_product(plan.kind, format, wide, [&](auto k, auto f, auto w) { return launch_product<Tile8<k>, f, w>(ctx, p, s); });
}

template <int DTYPE>
void launch_quantize(const QuantizeArgs& p, bool square, hipStream_t s) {
  const int64_t blocks = (int64_t)p.rows * ((p.cols + BLOCK8 - 1) / BLOCK8);
  // Past the caches where the numbers fill most of the 256 MB behind them.  Through / past them, us, to rows and transpose of bfloat16: 32768 x 8192
  // (512 MB) 238 / 182, 16384 x 8192 113 / 94, 24576 x 4096 (192 MB) 82 / 72, 32768 x 2048 (128 MB) 49.7 / 51.5; rows alone 139 / 129, 71 / 63, 51 / 48,
  // 31.5 / 32.3.
  const bool past = (int64_t)p.rows * p.cols * (DTYPE == F32 ? 4 : 2) > (int64_t)128 << 20;
  if (!square && !p.data_t && blocks <= (int64_t)1 << 28) {      // (a grid counts its threads in 32 bits)
    // One block a lane group / four, us: 4096 x 512 (16384 blocks) 3.3 / 3.7, 4096 x 1024 4.4 / 4.3, 4096 x 2048 6.9 / 6.1: where every CU has workgroups either way, the
    // loads of four in flight count for more.
    if (blocks <= 32 * 1024) hipLaunchKernelGGL((k_quantize8_rows<DTYPE, 1, false>), dim3((unsigned)((blocks + 15) / 16)), dim3(256), 0, s, p);
    else if (past) hipLaunchKernelGGL((k_quantize8_rows<DTYPE, 4, true>), dim3((unsigned)((blocks + 63) / 64)), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_quantize8_rows<DTYPE, 4, false>), dim3((unsigned)((blocks + 63) / 64)), dim3(256), 0, s, p);
    return;
  }
  const dim3 grid((unsigned)((p.cols + BLOCK8 - 1) / BLOCK8), (unsigned)((p.rows + BLOCK8 - 1) / BLOCK8));
  if (square) hipLaunchKernelGGL((k_quantize8<DTYPE, true, false>), grid, dim3(256), 0, s, p);
  else if (past) hipLaunchKernelGGL((k_quantize8<DTYPE, false, true>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((k_quantize8<DTYPE, false, false>), grid, dim3(256), 0, s, p);
}

}  // namespace

extern "C" {

ob_status ob_linear8_create(const ob_linear8_config* cfg, ob_linear8_ctx** out) {
  if (!cfg || !out) return OB_ERR_NULL;
  *out = nullptr;
  const int64_t most = (int64_t)1 << 20;
  if (cfg->k < 1 || cfg->k > most || cfg->n < 1 || cfg->n > most || cfg->max_rows < 0 || cfg->max_rows > MOST) return OB_ERR_ARG;
  ob_linear8_ctx* ctx = new (std::nothrow) ob_linear8_ctx();
  if (!ctx) return OB_ERR_ARG;
  ctx->cfg = *cfg;
  hipError_t e = hipGetDevice(&ctx->device);
  if (e == hipSuccess) e = allow_products();
  ctx->bytes = (size_t)WORKSPACE8;
  if (e == hipSuccess) e = hipMalloc(&ctx->d_partial, ctx->bytes);
  if (e != hipSuccess) {
    delete ctx;
    return OB_ERR_HIP;
  }
  *out = ctx;
  return OB_OK;
}

void ob_linear8_destroy(ob_linear8_ctx* ctx) { delete ctx; }
size_t ob_linear8_workspace_bytes(const ob_linear8_ctx* ctx) { return ctx ? ctx->bytes : 0; }
const char* ob_linear8_last_hip_error(const ob_linear8_ctx* ctx) { return ctx ? ctx->hip_err.c_str() : ""; }

ob_status ob_linear8_quantize(ob_linear8_ctx* ctx, const void* src, ob_dtype src_dtype, int64_t lds, int64_t rows, int64_t cols, int32_t form,
                              int32_t format, int32_t format_t, void* data, int64_t ld, void* scales, int64_t ld_scales, void* data_t, int64_t ld_t,
                              void* scales_t, int64_t ld_scales_t, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  const bool square = form == OB_BLOCK_SQUARE;
  if (rows < 0 || rows > MOST || cols < 0 || cols > MOST || lds < cols || lds > MOST || !any_dtype(src_dtype) || (!square && form != OB_BLOCK_ROWS) ||
      (data && (wrong(Given{data, ld, scales, ld_scales}, cols) || (format != OB_E4M3 && format != OB_E5M2))) ||
      (data_t && (wrong(Given{data_t, ld_t, scales_t, ld_scales_t}, rows) || (format_t != OB_E4M3 && format_t != OB_E5M2))) ||
      (square && data && data_t && format != format_t))
    return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!rows || !cols) return OB_OK;
  if (!src || (data && !scales) || (data_t && !scales_t) || (!data && !data_t)) return OB_ERR_NULL;
  if (off_element(src, src_dtype) || off(data, 16) || off(data_t, 16) || (data && off(scales, 4)) || (data_t && off(scales_t, 4))) return OB_ERR_ALIGN;
  const QuantizeArgs p{src, lds, (int)rows, (int)cols, format, format_t, static_cast<uint8_t*>(data), static_cast<uint8_t*>(scales),
                       static_cast<uint8_t*>(data_t), static_cast<uint8_t*>(scales_t), ld, ld_scales, ld_t, ld_scales_t};
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (src_dtype == OB_F32) launch_quantize<F32>(p, square, s);
  else if (src_dtype == OB_F16) launch_quantize<F16>(p, square, s);
  else launch_quantize<BF16>(p, square, s);
  return hip_ok(ctx, hipGetLastError(), "k_quantize8") ? OB_OK : OB_ERR_HIP;
}

ob_status ob_linear8_forward(ob_linear8_ctx* ctx, const void* x, int64_t ldx, const void* x_scales, int64_t ldx_scales, int32_t x_format, const void* w,
                             int64_t ldw, const void* w_scales, int64_t ldw_scales, int64_t rows, void* y, int64_t ldy, ob_dtype y_dtype, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  if (rows < 0 || rows > ctx->cfg.max_rows) return OB_ERR_ARG;
  return product(ctx, Given{x, ldx, x_scales, ldx_scales}, x_format, Given{w, ldw, w_scales, ldw_scales}, true, rows, ctx->cfg.n, ctx->cfg.k, y, ldy, y_dtype,
                 false, hip_stream);
}

ob_status ob_linear8_forward_few(ob_linear8_ctx* ctx, const void* x, ob_dtype x_dtype, int64_t ldx, int32_t x_format, const void* w, int64_t ldw,
                                 const void* w_scales, int64_t ldw_scales, int64_t rows, void* y, int64_t ldy, ob_dtype y_dtype, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  const int64_t k = ctx->cfg.k, n = ctx->cfg.n;
  const Given g{w, ldw, w_scales, ldw_scales};
  if (rows < 0 || rows > ctx->cfg.max_rows || ldx < k || ldx > MOST || wrong(g, k) || ldy < n || ldy > MOST || !any_dtype(x_dtype) || !any_dtype(y_dtype) ||
      (x_format != OB_E4M3 && x_format != OB_E5M2))
    return OB_ERR_ARG;
  if (rows > OB_LINEAR8_FEW_ROWS) return OB_ERR_SIZE;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!rows) return OB_OK;
  if (!x || !w || !w_scales || !y) return OB_ERR_NULL;
  if (off_element(x, x_dtype) || misplaced(g) || off_element(y, y_dtype)) return OB_ERR_ALIGN;
  FewArgs f;
  f.p.a = Operand8{nullptr, nullptr, 0, 0, (int)rows, 0};
  f.p.b = Operand8{static_cast<const uint8_t*>(w), static_cast<const uint8_t*>(w_scales), ldw, ldw_scales, (int)n, 7};
  f.p.out = y;
  f.p.partial = nullptr;
  f.p.ldo = ldy;
  f.p.slabs = (int)((k + BLOCK8 - 1) / BLOCK8);
  f.p.parts = 1;
  f.p.out_dtype = y_dtype;
  f.p.accumulate = false;
  f.x = x;
  f.ldx = ldx;
  f.k = (int)k;
  f.format = x_format;
  if (y_dtype == OB_F32) launch_few<true>(f, x_dtype, static_cast<hipStream_t>(hip_stream));
  else launch_few<false>(f, x_dtype, static_cast<hipStream_t>(hip_stream));
  return hip_ok(ctx, hipGetLastError(), "k_product8_few") ? OB_OK : OB_ERR_HIP;
}

ob_status ob_linear8_input_grad(ob_linear8_ctx* ctx, const void* dy, int64_t lddy, const void* dy_scales, int64_t lddy_scales, int32_t dy_format, const void* w_t,
                                int64_t ldw_t, const void* w_t_scales, int64_t ldw_t_scales, int64_t rows, void* dx, int64_t lddx, ob_dtype dx_dtype,
                                void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  if (rows < 0 || rows > ctx->cfg.max_rows) return OB_ERR_ARG;
  return product(ctx, Given{dy, lddy, dy_scales, lddy_scales}, dy_format, Given{w_t, ldw_t, w_t_scales, ldw_t_scales}, true, rows, ctx->cfg.k, ctx->cfg.n, dx,
                 lddx, dx_dtype, false, hip_stream);
}

ob_status ob_linear8_weight_grad(ob_linear8_ctx* ctx, const void* dy_t, int64_t lddy_t, const void* dy_t_scales, int64_t lddy_t_scales, int32_t dy_format,
                                 const void* x_t, int64_t ldx_t, const void* x_t_scales, int64_t ldx_t_scales, int64_t rows, void* dw, int64_t lddw,
                                 ob_dtype dw_dtype, int32_t accumulate, void* hip_stream) {
  if (!ctx) return OB_ERR_NULL;
  if (rows < 0 || rows > ctx->cfg.max_rows) return OB_ERR_ARG;
  return product(ctx, Given{dy_t, lddy_t, dy_t_scales, lddy_t_scales}, dy_format, Given{x_t, ldx_t, x_t_scales, ldx_t_scales}, false, ctx->cfg.n, ctx->cfg.k, rows,
                 dw, lddw, dw_dtype, accumulate != 0, hip_stream);
}

}  // extern "C"
