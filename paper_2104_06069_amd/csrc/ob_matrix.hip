// libonebitlamb: host side of the matrix operators (include/ob_matrix.h) -- contexts, tile lists, argument validation and
// launches.  The kernels live in ob_matrix_kernels.h and ob_mm.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <string>
#include <type_traits>
#include <vector>

#include "ob_matrix.h"
#include "ob_matrix_kernels.h"

using namespace obm;

namespace {

template <int KIND, int BK>
using Tile = Shape<side_of(KIND), side_of(KIND), KIND == DEEP ? 64 : BK, 2, KIND == T256 ? 4 : 2,
                   KIND == DEEP ? (BK == 32 ? 4 : 8) : KIND == T64 ? 3 : 2, KIND == DEEP ? 2 : 1>;

template <class F>
auto with_tile(int kind, F f) {
  switch (kind) {
    case T256: return f(std::integral_constant<int, T256>{});
    case T128: return f(std::integral_constant<int, T128>{});
    case T64: return f(std::integral_constant<int, T64>{});
    default: return f(std::integral_constant<int, DEEP>{});
  }
}

inline int elem_size(int dtype) { return dtype == OB_F32 ? 4 : 2; }
inline bool off_element(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_size(dtype) != 0; }
inline bool at16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
inline bool any_dtype(int d) { return d == OB_F32 || d == OB_F16 || d == OB_BF16; }

template <class Ctx>
bool hip_ok(Ctx* ctx, hipError_t e, const char* what) {
  if (e == hipSuccess) return true;
  try {
    ctx->hip_err = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return false;
}

bool on_device(int device) {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && dev == device;
}

// A kernel may ask for more than 64 KB of LDS once it has been told.
template <class K>
hipError_t allow_lds(K* kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

}  // namespace

// ---- expert layers -------------------------------------------------------------------------------------------------
struct ob_experts_ctx {
  ob_experts_config cfg;
  int device = -1;
  // weight_grad with more than one workgroup a tile of 64 x 64: the most of them there is room for
  int parts = 1;
  void* mem = nullptr;
  size_t bytes = 0;
  float* d_partial = nullptr;
  ~ob_experts_ctx() {
    if (mem) (void)hipFree(mem);
  }
  std::string hip_err;
};

namespace {

template <class S, bool BF, int FB, int MODE>
ob_status launch_rows(ob_experts_ctx* ctx, const RowsArgs& p, hipStream_t stream) {
  const int64_t tiles = ((int64_t)p.groups.rows / S::BM + std::min<int64_t>(p.groups.n, p.groups.rows)) * ((p.width + S::BN - 1) / S::BN);
  const int64_t grid = (tiles + 7) / 8 * 8 + (S::BM == 256 ? CUS : 0);      // (with the split tiles of the last round)
  if (grid > 0x7fffffff) return OB_ERR_SIZE;
  hipLaunchKernelGGL((k_experts_rows<S, BF, FB, MODE>), dim3((unsigned)grid), dim3(S::NT), (Product<S, BF, KC, FB, 1, 1, MODE>::LDS_BYTES), stream, p);
  return hip_ok(ctx, hipGetLastError(), "k_experts_rows") ? OB_OK : OB_ERR_HIP;
}

template <bool BF, int FB, int MODE>
ob_status launch_few_rows(ob_experts_ctx* ctx, const RowsArgs& p, hipStream_t stream) {
  using F = FewRows<BF, FB, MODE>;
  const int64_t tiles = ((int64_t)p.groups.rows / F::BM + std::min<int64_t>(p.groups.n, p.groups.rows)) * ((p.width + F::BN - 1) / F::BN);
  const int64_t grid = (tiles + 7) / 8 * 8;
  if (grid > 0x7fffffff) return OB_ERR_SIZE;
  hipLaunchKernelGGL((k_experts_few_rows<BF, FB, MODE>), dim3((unsigned)grid), dim3(256), (F::LDS_BYTES), stream, p);
  return hip_ok(ctx, hipGetLastError(), "k_experts_few_rows") ? OB_OK : OB_ERR_HIP;
}

template <class S, bool BF, int MODE>
ob_status launch_weights(ob_experts_ctx* ctx, const WeightsArgs& p, hipStream_t stream) {
  const int64_t tiles = (int64_t)((p.height + S::BM - 1) / S::BM) * ((p.width + S::BN - 1) / S::BN);      // of a group
  const int64_t grid = (tiles + 7) / 8 * 8 * p.groups.n * p.parts;
  if (grid > 0x7fffffff) return OB_ERR_SIZE;
  hipLaunchKernelGGL((k_experts_weights<S, BF, MODE>), dim3((unsigned)grid), dim3(S::NT), (Product<S, BF, KS, KS, 1, 1, MODE>::LDS_BYTES), stream, p);
  if (p.parts > 1) hipLaunchKernelGGL((k_experts_join<BF, MODE>), dim3((unsigned)(tiles * p.groups.n)), dim3(BLOCK), 0, stream, p);
  return hip_ok(ctx, hipGetLastError(), "k_experts_weights") ? OB_OK : OB_ERR_HIP;
}

// f(kind, mode), for a kind of kind_of()
template <class F>
auto with_tile_and_mode(int kind, bool direct, F f) {
  if (!direct) {
    if (kind == T128) return f(std::integral_constant<int, T128>{}, std::integral_constant<int, ANY>{});
    return f(std::integral_constant<int, T64>{}, std::integral_constant<int, ANY>{});
  }
  return with_tile(kind, [&](auto n) { return f(n, std::integral_constant<int, TAIL>{}); });
}

template <bool BF, int MODE>
hipError_t allow_few_rows() {
  const hipError_t e = allow_lds(k_experts_few_rows<BF, KC, MODE>, FewRows<BF, KC, MODE>::LDS_BYTES);
  return e == hipSuccess ? allow_lds(k_experts_few_rows<BF, KS, MODE>, FewRows<BF, KS, MODE>::LDS_BYTES) : e;
}
template <bool BF>
hipError_t allow_experts() {
  hipError_t e = allow_few_rows<BF, TAIL>();
  if (e == hipSuccess) e = allow_few_rows<BF, ANY>();
  for (int kind = 0; kind < KINDS; ++kind)
    for (const bool direct : {false, true}) {
      if (e != hipSuccess) return e;
      e = with_tile_and_mode(kind_of(kind, direct), direct, [&](auto n, auto mode) {
        using S = Tile<n, 64>;
        hipError_t e = allow_lds(k_experts_rows<S, BF, KC, mode>, Product<S, BF, KC, KC, 1, 1, mode>::LDS_BYTES);
        if (e == hipSuccess) e = allow_lds(k_experts_rows<S, BF, KS, mode>, Product<S, BF, KC, KS, 1, 1, mode>::LDS_BYTES);
        if (e == hipSuccess) e = allow_lds(k_experts_weights<S, BF, mode>, Product<S, BF, KS, KS, 1, 1, mode>::LDS_BYTES);
        return e;
      });
    }
  return e;
}

constexpr int64_t MAX_LD = (int64_t)1 << 22;      // a tile's offsets are 32-bit

ob_status rows_call(ob_experts_ctx* ctx, const void* a, int64_t lda, const void* w, const int32_t* offsets, int64_t rows,
                    void* out, int64_t ldo, int out_dtype, bool transposed, void* hip_stream) {
  if (!ctx || !offsets) return OB_ERR_NULL;
  const ob_experts_config& c = ctx->cfg;
  const int64_t depth = transposed ? c.n : c.k, width = transposed ? c.k : c.n;
  if (rows < 0 || rows > c.max_rows || lda < depth || ldo < width || lda >= MAX_LD || ldo >= MAX_LD) return OB_ERR_ARG;
  if (out_dtype != c.dtype && out_dtype != OB_F32) return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (!w || (rows && (!a || !out))) return OB_ERR_NULL;
  if (off_element(a, c.dtype) || off_element(w, c.dtype) || off_element(out, out_dtype) || off_element(offsets, OB_F32)) return OB_ERR_ALIGN;
  if (rows == 0) return OB_OK;
  RowsArgs p;
  p.groups = Groups{offsets, c.num_groups, (int)rows};
  p.a = static_cast<const uint16_t*>(a);
  p.w = static_cast<const uint16_t*>(w);
  p.out = out;
  p.lda = lda;
  p.ldo = ldo;
  p.w_stride = c.w_stride;
  p.depth = (int)depth;
  p.width = (int)width;
  p.out_dtype = out_dtype;
  p.ldw = c.w_layout == OB_EXPERTS_KN ? c.n : c.k;
  const bool strided = (c.w_layout == OB_EXPERTS_KN) != transposed;      // W's columns, as the product has them, are its rows in memory
  p.a_direct = at16(a) && lda % 8 == 0;
  p.w_direct = at16(w) && p.ldw % 8 == 0 && c.w_stride % 8 == 0 && (!strided || width % 8 == 0);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool direct = p.a_direct && p.w_direct;
  const RowsPlan plan = rows_plan(c.num_groups, rows, depth, width, direct);
  if (plan.few) {
    const auto few = [&](auto mode) {
      if (c.dtype == OB_BF16) return strided ? launch_few_rows<true, KS, mode>(ctx, p, s) : launch_few_rows<true, KC, mode>(ctx, p, s);
      return strided ? launch_few_rows<false, KS, mode>(ctx, p, s) : launch_few_rows<false, KC, mode>(ctx, p, s);
    };
    return direct ? few(std::integral_constant<int, TAIL>{}) : few(std::integral_constant<int, ANY>{});
  }
  return with_tile_and_mode(plan.kind, direct, [&](auto n, auto mode) {
    using S = Tile<n, 64>;
    if (c.dtype == OB_BF16) return strided ? launch_rows<S, true, KS, mode>(ctx, p, s) : launch_rows<S, true, KC, mode>(ctx, p, s);
    return strided ? launch_rows<S, false, KS, mode>(ctx, p, s) : launch_rows<S, false, KC, mode>(ctx, p, s);
  });
}

}  // namespace

extern "C" {

ob_status ob_experts_create(const ob_experts_config* cfg, ob_experts_ctx** out) {
  if (!cfg || !out) return OB_ERR_NULL;
  *out = nullptr;
  const int64_t most = (int64_t)1 << 20;
  if (cfg->num_groups < 1 || cfg->num_groups > 65536 || (cfg->dtype != OB_F16 && cfg->dtype != OB_BF16) ||
      (cfg->w_layout != OB_EXPERTS_KN && cfg->w_layout != OB_EXPERTS_NK) || cfg->reserved != 0 || cfg->k < 1 || cfg->k > most ||
      cfg->n < 1 || cfg->n > most || cfg->max_rows < 0 || cfg->max_rows > ((int64_t)1 << 26) ||
      (cfg->w_stride != 0 && cfg->w_stride < cfg->k * cfg->n) || cfg->w_stride > ((int64_t)1 << 44))
    return OB_ERR_ARG;
  ob_experts_ctx* ctx = new (std::nothrow) ob_experts_ctx();
  if (!ctx) return OB_ERR_ARG;
  ctx->cfg = *cfg;
  if (!ctx->cfg.w_stride) ctx->cfg.w_stride = cfg->k * cfg->n;
  hipError_t e = hipGetDevice(&ctx->device);
  if (e == hipSuccess) e = cfg->dtype == OB_BF16 ? allow_experts<true>() : allow_experts<false>();
  ctx->parts = most_parts(cfg->num_groups, cfg->k, cfg->n, cfg->max_rows);
  if (e == hipSuccess && ctx->parts > 1) {
    const int64_t tiles = cfg->num_groups * ((cfg->k + 63) / 64) * ((cfg->n + 63) / 64);
    ctx->bytes = (size_t)tiles * ctx->parts * 64 * 64 * sizeof(float);
    e = hipMalloc(&ctx->mem, ctx->bytes);
    ctx->d_partial = static_cast<float*>(ctx->mem);
  }
  if (e != hipSuccess) {
    delete ctx;
    return OB_ERR_HIP;
  }
  *out = ctx;
  return OB_OK;
}

void ob_experts_destroy(ob_experts_ctx* ctx) { delete ctx; }
size_t ob_experts_workspace_bytes(const ob_experts_ctx* ctx) { return ctx ? ctx->bytes : 0; }
const char* ob_experts_last_hip_error(const ob_experts_ctx* ctx) { return ctx ? ctx->hip_err.c_str() : ""; }

ob_status ob_experts_forward(ob_experts_ctx* ctx, const void* x, int64_t ldx, const void* w, const int32_t* offsets, int64_t rows,
                             void* y, int64_t ldy, ob_dtype y_dtype, void* hip_stream) {
  return rows_call(ctx, x, ldx, w, offsets, rows, y, ldy, y_dtype, false, hip_stream);
}

ob_status ob_experts_input_grad(ob_experts_ctx* ctx, const void* dy, int64_t lddy, const void* w, const int32_t* offsets, int64_t rows,
                                void* dx, int64_t lddx, ob_dtype dx_dtype, void* hip_stream) {
  return rows_call(ctx, dy, lddy, w, offsets, rows, dx, lddx, dx_dtype, true, hip_stream);
}

ob_status ob_experts_weight_grad(ob_experts_ctx* ctx, const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets,
                                 int64_t rows, void* dw, ob_dtype dw_dtype, int32_t accumulate, void* hip_stream) {
  if (!ctx || !offsets || !dw) return OB_ERR_NULL;
  const ob_experts_config& c = ctx->cfg;
  if (rows < 0 || rows > c.max_rows || ldx < c.k || lddy < c.n || ldx >= MAX_LD || lddy >= MAX_LD) return OB_ERR_ARG;
  if ((dw_dtype != (ob_dtype)c.dtype && dw_dtype != OB_F32) || (accumulate && dw_dtype != OB_F32)) return OB_ERR_ARG;
  if (!on_device(ctx->device)) return OB_ERR_ARG;
  if (rows && (!x || !dy)) return OB_ERR_NULL;
  if (off_element(x, c.dtype) || off_element(dy, c.dtype) || off_element(dw, dw_dtype) || off_element(offsets, OB_F32)) return OB_ERR_ALIGN;
  WeightsArgs p;
  p.groups = Groups{offsets, c.num_groups, (int)rows};
  const bool kn = c.w_layout == OB_EXPERTS_KN;
  p.a = static_cast<const uint16_t*>(kn ? x : dy);
  p.b = static_cast<const uint16_t*>(kn ? dy : x);
  p.lda = kn ? ldx : lddy;
  p.ldb = kn ? lddy : ldx;
  p.height = (int)(kn ? c.k : c.n);
  p.width = (int)(kn ? c.n : c.k);
  p.out = dw;
  p.out_stride = c.w_stride;
  p.out_dtype = dw_dtype;
  p.accumulate = accumulate != 0;
  p.a_direct = at16(p.a) && p.lda % 8 == 0 && p.height % 8 == 0;
  p.b_direct = at16(p.b) && p.ldb % 8 == 0 && p.width % 8 == 0;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool direct = p.a_direct && p.b_direct;
  const WeightsPlan plan = weights_plan(c.num_groups, rows, p.height, p.width, ctx->parts, direct);
  p.parts = plan.parts;
  p.partial = ctx->d_partial;
  return with_tile_and_mode(plan.kind, direct, [&](auto n, auto mode) {
    using S = Tile<n, 64>;
    return c.dtype == OB_BF16 ? launch_weights<S, true, mode>(ctx, p, s) : launch_weights<S, false, mode>(ctx, p, s);
  });
}

}  // extern "C"

// ---- orthogonalised update -----------------------------------------------------------------------------------------
struct ob_muon_ctx {
  int device = -1;
  int steps = 0, nesterov = 0, precision = OB_F32;
  float eps = 0, beta = 0, weight_decay = 0;
  std::vector<float> coefficients;      // 3 * steps
  int64_t n = 0;                        // elements of the flat buffers
  int mats = 0, square_tiles = 0;
  bool norms = false;                   // a launch of k_muon_norms
  int small_lds = 0;                    // not 0: the whole list in k_polar_small, with this much LDS
  std::vector<Part> parts;
  int64_t x_plane = 0, e_plane = 0;     // elements
  void* mem = nullptr;
  size_t bytes = 0;
  Matrix* d_mats = nullptr;
  SquareTile* d_square = nullptr;
  double* d_sums = nullptr;
  Inverse* d_inv = nullptr;
  uint16_t* d_x[2] = {nullptr, nullptr};
  uint16_t* d_e[5] = {};                // S or E, B, Y, and two of Q
  std::string hip_err;
  ~ob_muon_ctx() {
    if (mem) (void)hipFree(mem);
  }
};

namespace {

template <class T>
size_t room(size_t count) {
  return (std::max<size_t>(count * sizeof(T), 1) + 1023) / 1024 * 1024;
}

template <int N, int TERMS>
hipError_t allow_muon() {
  using S = Tile<N, TERMS == 2 ? 32 : 64>;
  hipError_t e = allow_lds(k_polar_symmetric<S, TERMS, false>, Product<S, false, KC, KC, TERMS, TERMS, WHOLE>::LDS_BYTES);
  if (e == hipSuccess) e = allow_lds(k_polar_symmetric<S, TERMS, true>, Product<S, false, KC, KC, TERMS, TERMS, WHOLE>::LDS_BYTES);
  const int bytes = Product<Tile<N, 32>, false, KC, KS, TERMS, 2, WHOLE>::LDS_BYTES;
  if (e == hipSuccess) e = allow_lds(k_polar_apply<Tile<N, 32>, TERMS, false>, bytes);
  if (e == hipSuccess) e = allow_lds(k_polar_apply<Tile<N, 32>, TERMS, true>, bytes);
  return e;
}

template <int TERMS, bool FROM_X>
void symmetric(const Part& part, const SymmetricArgs& a, int products, hipStream_t s) {
  with_tile(part.sym_tile, [&](auto n) {
    using S = Tile<n, TERMS == 2 ? 32 : 64>;
    using P = Product<S, false, KC, KC, TERMS, TERMS, WHOLE>;
    hipLaunchKernelGGL((k_polar_symmetric<S, TERMS, FROM_X>), dim3((unsigned)part.tiles[FROM_X ? GRAM : SYMMETRIC].size(), products), dim3(S::NT), P::LDS_BYTES, s, a);
  });
}
template <int TERMS>
void apply(const Part& part, const ApplyArgs& a, bool last, hipStream_t s) {
  with_tile(part.apply_tile, [&](auto n) {
    using S = Tile<n, 32>;
    using P = Product<S, false, KC, KS, TERMS, 2, WHOLE>;
    if (last) hipLaunchKernelGGL((k_polar_apply<S, TERMS, true>), dim3((unsigned)part.tiles[APPLY].size()), dim3(S::NT), P::LDS_BYTES, s, a);
    else hipLaunchKernelGGL((k_polar_apply<S, TERMS, false>), dim3((unsigned)part.tiles[APPLY].size()), dim3(S::NT), P::LDS_BYTES, s, a);
  });
}

void follow_s(ob_muon_ctx* ctx, const Part& part, const Finish& finish, hipStream_t stream) {
  uint16_t* const S = ctx->d_e[0];
  uint16_t* const Y = ctx->d_e[2];
  int cur = 0;
  for (int first = 0, n; first < ctx->steps; first += n) {
    n = steps_from(ctx->coefficients, ctx->precision == OB_F32, first);
    SymmetricArgs g{part.d_tiles[GRAM], ctx->d_x[cur], {}, nullptr, {S}, ctx->x_plane, ctx->e_plane, {S_UNIT / (X_UNIT * X_UNIT)}, 0.0f, 0.0f};
    symmetric<2, true>(part, g, 1, stream);
    double most = 1.0;      // what Q's elements can come to
    for (int k = first; k < first + n; ++k)
      most *= std::max(1.0, (double)std::fabs(ctx->coefficients[3 * k]));
    const float q_unit = (float)std::exp2(std::min(8.0, std::floor(std::log2(32768.0 / most))));
    uint16_t* q = ctx->d_e[3];
    for (int k = first; k < first + n; ++k) {
      const float a = ctx->coefficients[3 * k], b = ctx->coefficients[3 * k + 1], c = ctx->coefficients[3 * k + 2];
      const bool start = k == first, end = k == first + n - 1;
      // the first B is Q; it is kept in Q's unit
      uint16_t* const B = start ? q : ctx->d_e[1];
      const float unit = start ? q_unit : E_UNIT;
      symmetric<2, false>(part, SymmetricArgs{part.d_tiles[SYMMETRIC], S, {S}, S, {B}, 0, ctx->e_plane, {c * unit / (S_UNIT * S_UNIT)}, b * unit / S_UNIT, a * unit},
                          1, stream);
      SymmetricArgs p{part.d_tiles[SYMMETRIC], B, {}, nullptr, {}, 0, ctx->e_plane, {}, 0.0f, 0.0f};
      int products = 0;
      if (!end) {
        p.b[products] = S;
        p.out[products] = Y;
        p.mul[products++] = 1.0f / unit;
      }
      if (!start) {
        uint16_t* const next = q == ctx->d_e[3] ? ctx->d_e[4] : ctx->d_e[3];
        p.b[products] = q;
        p.out[products] = next;
        p.mul[products++] = 1.0f / unit;
        q = next;
      }
      if (products) symmetric<2, false>(part, p, products, stream);
      if (!end) symmetric<2, false>(part, SymmetricArgs{part.d_tiles[SYMMETRIC], Y, {B}, nullptr, {S}, 0, ctx->e_plane, {1.0f / unit}, 0.0f, 0.0f}, 1, stream);
    }
    apply<2>(part, ApplyArgs{part.d_tiles[APPLY], ctx->d_mats, q, ctx->d_x[cur], ctx->d_x[cur ^ 1], ctx->e_plane, ctx->x_plane, 1.0f / q_unit, finish},
             first + n == ctx->steps, stream);
    cur ^= 1;
  }
}

template <int TERMS>
void step_by_step(ob_muon_ctx* ctx, const Part& part, const Finish& finish, hipStream_t stream) {
  uint16_t* const E = ctx->d_e[0];
  uint16_t* const B = ctx->d_e[1];
  for (int k = 0; k < ctx->steps; ++k) {
    const float a = ctx->coefficients[3 * k], b = ctx->coefficients[3 * k + 1], c = ctx->coefficients[3 * k + 2];
    const float per_gram = E_UNIT / (X_UNIT * X_UNIT);
    SymmetricArgs g{part.d_tiles[GRAM], ctx->d_x[k & 1], {}, nullptr, {E}, ctx->x_plane, ctx->e_plane, {per_gram}, 0.0f, 0.0f};
    Shifted form = {};
    if (c != 0.0f) {
      form = shifted(a, b, c);
      g.diag = -form.t * E_UNIT;
    } else {      // B = a + b S from the first product alone
      g.out[0] = B;
      g.mul[0] = b * per_gram;
      g.diag = a * E_UNIT;
    }
    symmetric<TERMS, true>(part, g, 1, stream);
    if (c != 0.0f) {
      symmetric<TERMS, false>(part, SymmetricArgs{part.d_tiles[SYMMETRIC], E, {E}, form.linear != 0.0f ? E : nullptr, {B}, 0, ctx->e_plane, {c / E_UNIT},
                                                  form.linear, form.constant * E_UNIT}, 1, stream);
    }
    apply<TERMS>(part, ApplyArgs{part.d_tiles[APPLY], ctx->d_mats, B, ctx->d_x[k & 1], ctx->d_x[(k & 1) ^ 1], ctx->e_plane, ctx->x_plane, 1.0f / E_UNIT, finish},
                 k + 1 == ctx->steps, stream);
  }
}

// u -> the working X, and its Newton-Schulz steps, the last of which ends in `finish`
ob_status run_list(ob_muon_ctx* ctx, Direction d, float* m_out, const Finish& finish, hipStream_t s) {
  if (ctx->small_lds) {
    SmallArgs a{ctx->d_mats, d, m_out, finish, ctx->eps, ctx->steps, {}};
    std::copy(ctx->coefficients.begin(), ctx->coefficients.end(), a.coefficients);
    hipLaunchKernelGGL(k_polar_small, dim3(ctx->mats), dim3(SMALL_NT), ctx->small_lds, s, a);
    return hip_ok(ctx, hipGetLastError(), "k_polar_small") ? OB_OK : OB_ERR_HIP;
  }
  hipLaunchKernelGGL(k_muon_moments, dim3(ctx->square_tiles), dim3(BLOCK), 0, s, ctx->d_square, ctx->d_mats, d, m_out, ctx->d_sums);
  if (ctx->norms) hipLaunchKernelGGL(k_muon_norms, dim3(ctx->mats), dim3(BLOCK), 0, s, ctx->d_mats, ctx->d_sums, ctx->eps, ctx->d_inv);
  hipLaunchKernelGGL(k_muon_pack, dim3(ctx->square_tiles), dim3(BLOCK), 0, s, ctx->d_square, ctx->d_mats, d, ctx->norms ? ctx->d_inv : nullptr,
                     ctx->d_sums, ctx->eps, ctx->d_x[0], ctx->x_plane);
  for (const Part& part : ctx->parts) {
    if (part.follow_s) follow_s(ctx, part, finish, s);
    else if (part.terms == 2) step_by_step<2>(ctx, part, finish, s);
    else step_by_step<1>(ctx, part, finish, s);
  }
  return hip_ok(ctx, hipGetLastError(), "the orthogonaliser's kernels") ? OB_OK : OB_ERR_HIP;
}

ob_status create(const ob_muon_config* cfg, ob_muon_ctx* ctx) {
  ctx->steps = cfg->steps;
  ctx->nesterov = cfg->nesterov != 0;
  ctx->precision = cfg->precision;
  ctx->eps = cfg->eps;
  ctx->beta = cfg->beta;
  ctx->weight_decay = cfg->weight_decay;
  for (int k = 0; k < cfg->steps; ++k)
    for (int e = 0; e < 3; ++e) ctx->coefficients.push_back(cfg->coefficients[3 * std::min(k, cfg->num_coefficients - 1) + e]);
  ctx->n = cfg->layer_offsets[cfg->num_layers];
  std::vector<Matrix> mats;
  std::vector<SquareTile> square;
  int64_t xs = 0, es = 0;
  for (int64_t l = 0; l < cfg->num_layers; ++l) {
    const int64_t size = cfg->layer_offsets[l + 1] - cfg->layer_offsets[l], rows = cfg->layer_rows[l];
    if (rows == 0 || size == 0) continue;
    const int64_t cols = size / rows;
    Matrix m{};
    m.at = cfg->layer_offsets[l];
    m.rows = (int)rows;
    m.cols = (int)cols;
    m.tall = rows > cols;
    const int64_t side = SIDE;
    m.mp = (int)((std::min(rows, cols) + side - 1) / side * side);
    m.np = (int)((std::max(rows, cols) + side - 1) / side * side);
    m.scale = cfg->layer_scale ? cfg->layer_scale[l] : (float)(0.2 * std::sqrt((double)std::max(rows, cols)));
    m.x = xs;
    m.e = es;
    xs += (int64_t)m.mp * m.np;
    es += (int64_t)m.mp * m.mp;
    const int64_t tiles = (int64_t)(m.mp / SIDE) * (m.np / SIDE);
    if ((int64_t)square.size() + tiles > ((int64_t)1 << 30)) return OB_ERR_SIZE;
    m.tile0 = (int)square.size();
    m.tiles = (int)tiles;
    for (int64_t r = 0; r < rows; r += SIDE)
      for (int64_t c = 0; c < cols; c += SIDE) square.push_back(SquareTile{(int)mats.size(), (int)r, (int)c});
    mats.push_back(m);
  }
  if (mats.empty()) return OB_ERR_ARG;
  int largest_m = 0, largest_n = 0;
  for (const Matrix& m : mats) {
    largest_m = std::max(largest_m, m.mp);
    largest_n = std::max(largest_n, m.np);
  }
  if (largest_m <= SMALL_M && largest_n <= SMALL_N) {
    ctx->small_lds = (2 * SMALL_M * largest_n + 2 * SMALL_M * SMALL_M) * 2;
    if (!hip_ok(ctx, allow_lds(k_polar_small, ctx->small_lds), "hipFuncSetAttribute")) return OB_ERR_HIP;
    xs = es = 0;      // no working matrices outside of LDS
    square.clear();
  }
  if (!ctx->small_lds) ctx->parts = parts_of(mats, ctx->coefficients, cfg->precision == OB_F32);
  for (const Part& part : ctx->parts)
    for (const auto& table : part.tiles)
      if (table.size() > 0x7fffffff) return OB_ERR_SIZE;
  for (int kind = 0; kind < KINDS; ++kind) {
    hipError_t e = with_tile(kind, [&](auto n) { return allow_muon<n, 2>(); });
    if (e == hipSuccess) e = with_tile(kind, [&](auto n) { return allow_muon<n, 1>(); });
    if (!hip_ok(ctx, e, "hipFuncSetAttribute")) return OB_ERR_HIP;
  }
  ctx->mats = (int)mats.size();
  ctx->norms = norms_apart(mats);
  ctx->square_tiles = (int)square.size();
  ctx->x_plane = xs;
  ctx->e_plane = es;
  size_t total = 0;
  auto place = [&](size_t bytes) {
    const size_t at = total;
    total += bytes;
    return at;
  };
  const size_t at_mats = place(room<Matrix>(mats.size())), at_square = place(room<SquareTile>(square.size()));
  std::vector<size_t> at_table;
  for (const Part& part : ctx->parts)
    for (const auto& table : part.tiles) at_table.push_back(place(room<ListTile>(table.size())));
  const size_t at_sums = place(room<double>(square.size())), at_inv = place(room<Inverse>(mats.size()));
  const size_t at_x0 = place(room<uint16_t>(2 * xs)), at_x1 = place(room<uint16_t>(2 * xs));
  size_t at_e[5];
  for (size_t& at : at_e) at = place(room<uint16_t>(2 * es));
  if (!hip_ok(ctx, hipGetDevice(&ctx->device), "hipGetDevice") || !hip_ok(ctx, hipMalloc(&ctx->mem, total), "hipMalloc")) return OB_ERR_HIP;
  ctx->bytes = total;
  unsigned char* const base = static_cast<unsigned char*>(ctx->mem);
  ctx->d_mats = reinterpret_cast<Matrix*>(base + at_mats);
  ctx->d_square = reinterpret_cast<SquareTile*>(base + at_square);
  ctx->d_sums = reinterpret_cast<double*>(base + at_sums);
  ctx->d_inv = reinterpret_cast<Inverse*>(base + at_inv);
  ctx->d_x[0] = reinterpret_cast<uint16_t*>(base + at_x0);
  ctx->d_x[1] = reinterpret_cast<uint16_t*>(base + at_x1);
  for (int i = 0; i < 5; ++i) ctx->d_e[i] = reinterpret_cast<uint16_t*>(base + at_e[i]);
  bool ok = hip_ok(ctx, hipMemcpy(ctx->d_mats, mats.data(), mats.size() * sizeof(Matrix), hipMemcpyHostToDevice), "hipMemcpy") &&
                  hip_ok(ctx, hipMemcpy(ctx->d_square, square.data(), square.size() * sizeof(SquareTile), hipMemcpyHostToDevice), "hipMemcpy");
  size_t next = 0;
  for (Part& part : ctx->parts)
    for (const int k : {0, 1, 2}) {
      part.d_tiles[k] = reinterpret_cast<ListTile*>(base + at_table[next++]);
      ok = ok && hip_ok(ctx, hipMemcpy(part.d_tiles[k], part.tiles[k].data(), part.tiles[k].size() * sizeof(ListTile), hipMemcpyHostToDevice), "hipMemcpy");
    }
  return ok ? OB_OK : OB_ERR_HIP;
}

}  // namespace

extern "C" {

ob_status ob_muon_create(const ob_muon_config* cfg, ob_muon_ctx** out) {
  if (!cfg || !out) return OB_ERR_NULL;
  *out = nullptr;
  if (!cfg->layer_offsets || !cfg->layer_rows || !cfg->coefficients) return OB_ERR_NULL;
  if (cfg->num_layers < 1 || cfg->num_layers > 0x7fffffff || cfg->steps < 1 || cfg->steps > 64 || cfg->num_coefficients < 1 || cfg->num_coefficients > cfg->steps ||
      !(cfg->eps >= 0.0f) || !(cfg->beta >= 0.0f && cfg->beta < 1.0f) || !(cfg->weight_decay >= 0.0f) || !std::isfinite(cfg->eps) ||
      !std::isfinite(cfg->weight_decay) || (cfg->precision != OB_F32 && cfg->precision != OB_F16) || cfg->layer_offsets[0] != 0)
    return OB_ERR_ARG;
  for (int i = 0; i < cfg->num_coefficients; ++i) {      // (B's elements have a binary16 unit)
    const float* const k = cfg->coefficients + 3 * i;
    if (!(std::fabs(k[0]) + std::fabs(k[1]) + std::fabs(k[2]) <= 100.0f)) return OB_ERR_ARG;
  }
  for (int64_t l = 0; l < cfg->num_layers; ++l) {
    const int64_t size = cfg->layer_offsets[l + 1] - cfg->layer_offsets[l], rows = cfg->layer_rows[l];
    if (size < 0 || cfg->layer_offsets[l + 1] > ((int64_t)1 << 40) || rows < 0 || (rows && size % rows != 0)) return OB_ERR_ARG;
    // 32-bit offsets inside a tile, tile numbers of 16 bits
    if (rows && (rows > ((int64_t)1 << 20) || size / rows > ((int64_t)1 << 20))) return OB_ERR_SIZE;
    if (cfg->layer_scale && !std::isfinite(cfg->layer_scale[l])) return OB_ERR_ARG;
  }
  ob_muon_ctx* ctx = nullptr;
  try {
    ctx = new ob_muon_ctx();
    const ob_status s = create(cfg, ctx);
    if (s != OB_OK) {
      delete ctx;
      return s;
    }
  } catch (const std::exception&) {      // (out of host memory)
    delete ctx;
    return OB_ERR_ARG;
  }
  *out = ctx;
  return OB_OK;
}

void ob_muon_destroy(ob_muon_ctx* ctx) { delete ctx; }
size_t ob_muon_workspace_bytes(const ob_muon_ctx* ctx) { return ctx ? ctx->bytes : 0; }
const char* ob_muon_last_hip_error(const ob_muon_ctx* ctx) { return ctx ? ctx->hip_err.c_str() : ""; }

ob_status ob_muon_orthogonalize(ob_muon_ctx* ctx, const void* src, ob_dtype src_dtype, void* out, ob_dtype out_dtype, void* hip_stream) {
  if (!ctx || !src || !out) return OB_ERR_NULL;
  if (!any_dtype(src_dtype) || !any_dtype(out_dtype) || !on_device(ctx->device)) return OB_ERR_ARG;
  if (off_element(src, src_dtype) || off_element(out, out_dtype)) return OB_ERR_ALIGN;
  return run_list(ctx, Direction{src, nullptr, src_dtype, 0, 1.0f, 0.0f, 0.0f}, nullptr, Finish{nullptr, out, out_dtype, 0.0f, 0.0f},
                  static_cast<hipStream_t>(hip_stream));
}

ob_status ob_muon_step(ob_muon_ctx* ctx, float* x, float* m, const void* grad, ob_dtype grad_dtype, float grad_scale, float lr, void* x_lp,
                       ob_dtype x_dtype, void* hip_stream) {
  if (!ctx || !x || !m) return OB_ERR_NULL;
  if ((grad && !any_dtype(grad_dtype)) || (x_lp && x_dtype != OB_F16 && x_dtype != OB_BF16) || !std::isfinite(lr) || !std::isfinite(grad_scale) ||
      !on_device(ctx->device))
    return OB_ERR_ARG;
  if (off_element(x, OB_F32) || off_element(m, OB_F32) || (grad && off_element(grad, grad_dtype)) || (x_lp && off_element(x_lp, x_dtype))) return OB_ERR_ALIGN;
  return run_list(ctx, Direction{grad, m, grad ? (int)grad_dtype : F32, ctx->nesterov, grad_scale, ctx->beta, 1.0f - ctx->beta}, m,
                  Finish{x, x_lp, (int)x_dtype, lr, 1.0f - lr * ctx->weight_decay}, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
