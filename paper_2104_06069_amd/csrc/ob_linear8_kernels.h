// Kernels of the linear layer in 8 bits (include/ob_layer.h), on the tiles of ob_mm8.h.  Included by ob_linear8.hip only.
#pragma once

#include "ob_mm8.h"

namespace obl {

// ---- to 8 bits -----------------------------------------------------------------------------------------------------
struct QuantizeArgs {
  const void* src;
  int64_t lds;
  int rows, cols, format, format_t;
  uint8_t *data, *scales, *data_t, *scales_t;
  int64_t ld, ld_scales, ld_t, ld_scales_t;
};

template <bool PAST>
__device__ __forceinline__ void write8(uint8_t* p, v2i q) {
  if constexpr (PAST) __builtin_nontemporal_store(q, reinterpret_cast<v2i*>(p));
  else *reinterpret_cast<v2i*>(p) = q;
}

// Column e of eight rows' eight numbers
template <int DTYPE>
__device__ __forceinline__ Raw8<DTYPE> column(const Raw8<DTYPE> (&v)[8], int e) {
  Raw8<DTYPE> r;
  if constexpr (DTYPE == F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.lo[i] = e < 4 ? v[i].lo[e & 3] : v[i].hi[e & 3];
      r.hi[i] = e < 4 ? v[i + 4].lo[e & 3] : v[i + 4].hi[e & 3];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.h[i] = v[i].h[e];
  }
  return r;
}

// A workgroup takes 128 x 128 numbers, a thread eight adjacent rows by eight adjacent columns of them: a row's block is that of
// sixteen adjacent lanes, a column's that of sixteen lanes one from each group of those, four in a wavefront.  The transposed
// bytes are turned in LDS, so that both results go out 128 bytes of a row at a time; there the 16-byte pieces of a column are permuted by the
// column's number, or the lanes of a row would meet in one bank.  PAST (the rule is launch_quantize's): numbers are read and rows written past the
// caches; the transposed bytes are not, which are 128 of a row at a time.
template <int DTYPE, bool SQUARE, bool PAST>
__global__ __launch_bounds__(256) void k_quantize8(QuantizeArgs p) {
  using Magnitudes = typename Raw8<DTYPE>::Magnitudes;
  __shared__ __align__(16) uint8_t turned[BLOCK8 * BLOCK8];
  __shared__ __align__(16) Magnitudes most_of[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rg = tid >> 4, cg = tid & 15;
  const int r0 = blockIdx.y * BLOCK8, c0 = blockIdx.x * BLOCK8, left = p.cols - c0 - cg * 8, below = p.rows - r0 - rg * 8;
  Raw8<DTYPE> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i].template load<PAST>(p.src, (int64_t)(r0 + rg * 8 + i) * p.lds + c0 + cg * 8, i < below ? left : 0);
  Magnitudes rows, cols = v[0].magnitudes();      // of this thread's eight rows, and columns
  rows[0] = highest(cols);
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const Magnitudes m = v[i].magnitudes();
    rows[i] = highest(m);
    cols = __builtin_elementwise_max(cols, m);
  }
  const auto of_wave = [&](Magnitudes m) {      // lanes of the same columns
#pragma unroll
    for (int d = 32; d >= 16; d >>= 1) {
      Magnitudes o;
      int w[sizeof(m) / 4];
      __builtin_memcpy(w, &m, sizeof(m));
#pragma unroll
      for (int& k : w) k = __shfl_xor(k, d);
      __builtin_memcpy(&o, w, sizeof(m));
      m = __builtin_elementwise_max(m, o);
    }
    return m;
  };
  if constexpr (SQUARE) {
    cols = of_wave(highest_of_16(cols));
    if (lane == 0) most_of[wave][0] = cols;
    __syncthreads();
    const auto m = highest(__builtin_elementwise_max(__builtin_elementwise_max(most_of[0][0], most_of[1][0]), __builtin_elementwise_max(most_of[2][0], most_of[3][0])));
#pragma unroll
    for (int e = 0; e < 8; ++e) rows[e] = cols[e] = m;
  } else {
    rows = highest_of_16(rows);
    if (p.data_t) {
      cols = of_wave(cols);
      if (lane < 16) most_of[wave][cg] = cols;
      __syncthreads();
      cols = __builtin_elementwise_max(__builtin_elementwise_max(most_of[0][cg], most_of[1][cg]), __builtin_elementwise_max(most_of[2][cg], most_of[3][cg]));
    }
  }
  if (p.data) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int byte = scale_byte(Raw8<DTYPE>::of_binary32(rows[i]), p.format);
      const v2i q = bytes8(v[i], byte, p.format, left);
      if (i < below) {
        const int64_t row = r0 + rg * 8 + i;
        write8<PAST>(p.data + row * p.ld + c0 + cg * 8, q);
        if (cg == 0 && (!SQUARE || (rg == 0 && i == 0))) p.scales[(SQUARE ? row / BLOCK8 : row) * p.ld_scales + blockIdx.x] = (uint8_t)byte;
      }
    }
  }
  if (p.data_t) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int byte = scale_byte(Raw8<DTYPE>::of_binary32(cols[e]), p.format_t);
      *reinterpret_cast<v2i*>(turned + (cg * 8 + e) * BLOCK8 + (rg / 2 ^ (cg & 7)) * 16 + rg % 2 * 8) = bytes8(column(v, e), byte, p.format_t, below);
      if (rg == 0 && e < left) {
        const int64_t col = c0 + cg * 8 + e;
        if (!SQUARE) p.scales_t[col * p.ld_scales_t + blockIdx.y] = (uint8_t)byte;
        else if (cg == 0 && e == 0) p.scales_t[col / BLOCK8 * p.ld_scales_t + blockIdx.y] = (uint8_t)byte;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = j * 32 + tid / 8, piece = tid % 8;
      if (c0 + col < p.cols)
        *reinterpret_cast<v4i*>(p.data_t + (int64_t)(c0 + col) * p.ld_t + r0 + piece * 16) = *reinterpret_cast<const v4i*>(turned + col * BLOCK8 + (piece ^ (col >> 3 & 7)) * 16);
    }
  }
}

// Rows alone: a block of 128 to sixteen lanes, EACH blocks of them, wherever they lie: more workgroups than tiles, and no exchange between wavefronts.  With
// tiles / so: 1777 x 1000 5.0 / 3.4 us, 32768 x 2048 35.3 / 31.5, 32768 x 8192 140 / 126.
template <int DTYPE, int EACH, bool PAST>
__global__ __launch_bounds__(256) void k_quantize8_rows(QuantizeArgs p) {
  constexpr int GROUP = 16 * EACH;      // blocks of a workgroup
  const int blocks = (p.cols + BLOCK8 - 1) / BLOCK8, l = threadIdx.x & 15;
  const int64_t first = (int64_t)blockIdx.x * GROUP, row0 = first / blocks;
  const int rest = (int)(first - row0 * blocks);
  int64_t row[EACH];
  int block[EACH];
  Raw8<DTYPE> v[EACH];
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int at = rest + u * 16 + (threadIdx.x >> 4), down = at / blocks;
    row[u] = row0 + down;
    block[u] = at - down * blocks;
    v[u].template load<PAST>(p.src, row[u] * p.lds + block[u] * BLOCK8 + l * 8, row[u] < p.rows ? p.cols - block[u] * BLOCK8 - l * 8 : 0);
  }
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int byte = scale_byte(Raw8<DTYPE>::of_binary32(highest_of_16(highest(v[u].magnitudes()))), p.format);
    if (row[u] < p.rows) {
      write8<PAST>(p.data + row[u] * p.ld + block[u] * BLOCK8 + l * 8, bytes8(v[u], byte, p.format, p.cols - block[u] * BLOCK8 - l * 8));
      if (l == 0) p.scales[row[u] * p.ld_scales + block[u]] = (uint8_t)byte;
    }
  }
}

// ---- products --------------------------------------------------------------------------------------------------------
struct Product8Args {
  Operand8 a, b;
  void* out;
  float* partial;      // [parts, rows, cols], with parts > 1
  int64_t ldo;
  int slabs, parts, out_dtype;
  bool accumulate;
};

extern __shared__ __align__(1024) uint16_t lds_of_product8[];

template <class S, int FORMAT, bool WIDE>
__global__ __launch_bounds__(S::NT, 2) void k_product8(Product8Args p) {
  using P = Product8<S, FORMAT, WIDE>;
  const int nm = (p.a.rows + S::BM - 1) / S::BM, nn = (p.b.rows + S::BN - 1) / S::BN, tiles = nm * nn;
  const int at = tile_of_workgroup(blockIdx.x, tiles * p.parts);
  if (at < 0) return;
  int tm, tn;
  tile_in_bands(at % tiles, nm, nn, &tm, &tn);
  const int part = at / tiles, first = (int)((int64_t)p.slabs * part / p.parts), end = (int)((int64_t)p.slabs * (part + 1) / p.parts);
  const int r0 = tm * S::BM, c0 = tn * S::BN;
  typename P::Acc acc = {};
  P::run(p.a, p.b, r0, c0, first, end - first, reinterpret_cast<uint8_t*>(lds_of_product8), acc);
  const int rows = p.a.rows, cols = p.b.rows;
  if (p.parts > 1) {
    store_tile<S, true>(acc, lds_of_product8, p.partial + (int64_t)part * rows * cols, F32, cols, r0, c0, rows, cols, 0, 0);
  } else if constexpr (WIDE) {
    if (p.accumulate) {
      Results<S>::by_rows(acc, lds_of_product8, [&](int r, int c, v4f v) {
        r += r0;
        c += c0;
        if (r < rows) store4(p.out, F32, (int64_t)r * p.ldo + c, cols - c, v + load4(p.out, F32, (int64_t)r * p.ldo + c, cols - c));
      });
    } else {
      store_tile<S, true>(acc, lds_of_product8, p.out, F32, p.ldo, r0, c0, rows, cols, 0, 0);
    }
  } else if (p.out_dtype == BF16) {
    store_tile<S, true>(acc, lds_of_product8, p.out, BF16, p.ldo, r0, c0, rows, cols, 0, 0);
  } else {
    store_tile<S, false>(acc, lds_of_product8, p.out, F16, p.ldo, r0, c0, rows, cols, 0, 0);
  }
}

// Workgroups that stay (Flow8): tiles id, id + gridDim.x, ..
template <int FORMAT, int OUT>
__global__ __launch_bounds__(256, 1) void k_product8_flow(Product8Args p) {
  const int nm = (p.a.rows + 255) / 256, nn = (p.b.rows + 255) / 256, tiles = nm * nn, per = (tiles + 7) / 8;
  int id = blockIdx.x;
  Flow8<FORMAT, OUT>::run(p.a, p.b, p.slabs, p.out, p.ldo, reinterpret_cast<uint8_t*>(lds_of_product8), [&](int* r, int* c) {
    for (*r = *c = -1; id >> 3 < per; id += gridDim.x) {
      const int t = tile_of_workgroup(id, tiles);
      if (t < 0) continue;
      tile_in_bands(t, nm, nn, r, c);
      *r *= 256;
      *c *= 256;
      id += gridDim.x;
      return;
    }
  });
}

// The parts of a product's sums, in their order
__global__ __launch_bounds__(256) void k_product8_join(Product8Args p) {
  const int64_t rows = p.a.rows, cols = p.b.rows, fours = (cols + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= rows * fours) return;
  const int64_t r = at / fours, c = at % fours * 4;
  const int left = (int)min(cols - c, (int64_t)4);
  v4f sum = load4(p.partial, F32, r * cols + c, left);
  for (int k = 1; k < p.parts; ++k) sum += load4(p.partial, F32, (k * rows + r) * cols + c, left);
  if (p.accumulate) sum += load4(p.out, F32, r * p.ldo + c, left);
  store4(p.out, p.out_dtype, r * p.ldo + c, left, sum);
}

// The same for a few rows, where what counts is how fast the other operand is read.  A workgroup has up to 16 R rows and 16 J columns, its
// wavefronts share out the slabs of K and load each operand's 32 bytes a lane straight into registers, two slabs under way at once; their sums
// are added in a fixed order at the end.
struct FewArgs {
  Product8Args p;
  const void* x;      // where a is not in 8 bits yet (up to 16 rows): every workgroup makes it so itself, as k_quantize8 does
  int64_t ldx;
  int k, format;      // columns of x; a's format
};

// A lane's pieces q and q + 4 of a row's block, in 8 bits, and the block's scale
template <int DTYPE>
__device__ __forceinline__ void quantized_fragment(const FewArgs& f, int row, int slab, int lane, v8i& to, int& scale) {
  Raw8<DTYPE> v[4];
  unsigned most = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int at = slab * BLOCK8 + (lane >> 4) * 16 + (u & 1) * 8 + (u >> 1) * 64;
    v[u].load(f.x, row * f.ldx + at, f.k - at);
    most = max(most, highest(v[u].magnitudes()));
  }
#pragma unroll
  for (int d = 32; d >= 16; d >>= 1) most = max(most, (unsigned)__shfl_xor((int)most, d));
  scale = scale_byte(Raw8<DTYPE>::of_binary32(most), f.format);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int at = slab * BLOCK8 + (lane >> 4) * 16 + (u & 1) * 8 + (u >> 1) * 64;
    const v2i q = bytes8(v[u], scale, f.format, f.k - at);
    to[u * 2] = q.x;
    to[u * 2 + 1] = q.y;
  }
}

constexpr int NONE = 3;      // (of types: a is in 8 bits)
template <int R, int J, int WAVES, int DTYPE, bool WIDE>
__global__ __launch_bounds__(WAVES * 64) void k_product8_few(FewArgs f) {
  constexpr int STRIDE = 16 * J + 4, AHEAD = 2;
  __shared__ __align__(16) float sums[WAVES][16 * R * STRIDE];
  const Product8Args& p = f.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * 16 * J, rows = p.a.rows, cols = p.b.rows;
  const uint8_t *a[R], *b[J], *sa[R], *sb[J];
  int row[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    row[r] = min(r * 16 + i, rows - 1);
    a[r] = p.a.p + row[r] * p.a.ld + q * 16;
    sa[r] = p.a.scales + (row[r] >> p.a.shift) * p.a.ld_scales;
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = min(c0 + j * 16 + i, cols - 1);
    b[j] = p.b.p + c * p.b.ld + q * 16;
    sb[j] = p.b.scales + (c >> p.b.shift) * p.b.ld_scales;
  }
  const auto fragment = [](const uint8_t* at) {
    const v4i lo = *reinterpret_cast<const v4i*>(at), hi = *reinterpret_cast<const v4i*>(at + 64);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  v4f acc[R][J] = {};
  for (int t0 = wave; t0 < p.slabs; t0 += WAVES * AHEAD) {
    v8i fa[AHEAD][R], fb[AHEAD][J];
    int ea[AHEAD][R], eb[AHEAD][J];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int t = min(t0 + u * WAVES, p.slabs - 1);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        fb[u][j] = fragment(b[j] + (int64_t)t * BLOCK8);
        eb[u][j] = sb[j][t];
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (DTYPE == NONE) {
          fa[u][r] = fragment(a[r] + (int64_t)t * BLOCK8);
          ea[u][r] = sa[r][t];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (t0 + u * WAVES >= p.slabs) break;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (DTYPE != NONE) quantized_fragment<DTYPE>(f, row[r], t0 + u * WAVES, lane, fa[u][r], ea[u][r]);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          if constexpr (!WIDE) {
            acc[r][j] = f.format == E4M3 ? mma8<E4M3>(fb[u][j], eb[u][j], fa[u][r], ea[u][r], acc[r][j]) : mma8<E5M2>(fb[u][j], eb[u][j], fa[u][r], ea[u][r], acc[r][j]);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const v8s wb = widened<E4M3>(fb[u][j][2 * k], fb[u][j][2 * k + 1], scale_value(eb[u][j]));
              const v8s wa = f.format == E4M3 ? widened<E4M3>(fa[u][r][2 * k], fa[u][r][2 * k + 1], scale_value(ea[u][r]))
                                              : widened<E5M2>(fa[u][r][2 * k], fa[u][r][2 * k + 1], scale_value(ea[u][r]));
              acc[r][j] = mma<true>(wb, wa, acc[r][j]);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < J; ++j) *reinterpret_cast<v4f*>(&sums[wave][(r * 16 + i) * STRIDE + j * 16 + q * 4]) = acc[r][j];
  __syncthreads();
  for (int at = threadIdx.x; at < R * 16 * 4 * J; at += WAVES * 64) {
    const int r = at / (4 * J), c = at % (4 * J) * 4, left = cols - c0 - c;
    if (r >= rows || left <= 0) continue;
    v4f v = *reinterpret_cast<const v4f*>(&sums[0][r * STRIDE + c]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += *reinterpret_cast<const v4f*>(&sums[w][r * STRIDE + c]);
    const int64_t to = r * p.ldo + c0 + c;
    if (p.accumulate) v += load4(p.out, F32, to, left);
    store4(p.out, p.out_dtype, to, left, v);
  }
}

}  // namespace obl
