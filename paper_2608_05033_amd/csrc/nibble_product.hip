// sd_nibble_product: Y[m, n] = sum_k X(m, k) W(n, k) + bias[n] for two 4-bit
// tables, and sd_expert_product: the same where each row of Y is one row of X
// through the weights of the expert it was sorted to.
//
// A wave's 16 x 16 tile over 128 k: lane (r, g) = (lane % 16, lane / 16) holds a
// whole block of row r of each side, its 32 codes in 16 bytes and its scale byte,
// which is what v_mfma_scale_f32_16x16x128_f8f6f4 takes.  W is the first operand,
// so a lane ends with four neighbouring n of one row m.
//
// Products of e2m1 codes are multiples of 1/4 up to 36, so that the unit, which
// drops what lies far under the largest product of a run, drops nothing within a
// block: sums of blocks of one scale are exact.  Measured over random codes, one
// instruction is off by at most 2.1e-7 of the magnitudes summed, also where the
// blocks' scales differ by 2^80 or the sum so far is 10^6 times the products.
#include "nibble.h"
#include "tiles.h"

namespace {

using namespace nibble;

struct Operand {
  const uint8_t *codes, *scales;
  int64_t ld, rows;
};

// Rows of Y sorted by expert: those of expert e are offsets[e] .. offsets[e + 1] - 1
// and use rows e * n .. of W; the rows from offsets[experts] on are zeros.
struct Sorted {
  const int32_t *offsets, *source;  // source: X's row for each of Y's; null: X is sorted too
  int32_t experts;
  int64_t total;  // rows of Y
};

struct Frag {
  u32x4 v;
  uint32_t s;
};

__device__ inline f32x4 multiply(const Frag &w, const Frag &x, f32x4 acc) {
  const i32x8 a = {(int)w.v[0], (int)w.v[1], (int)w.v[2], (int)w.v[3], 0, 0, 0, 0};
  const i32x8 b = {(int)x.v[0], (int)x.v[1], (int)x.v[2], (int)x.v[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)w.s, 0, (int)x.s);
}

// Block 4 kg + g of one row; zeros past the last block.
__device__ inline void load_frag(const Operand &p, int64_t row, int32_t kg, int g, int32_t blocks, Frag &f) {
  f.v = u32x4{0, 0, 0, 0};
  f.s = 127;
  if (4 * kg + g < blocks) {
    f.v = *reinterpret_cast<const u32x4 *>(p.codes + row * p.ld + (4 * kg + g) * 16);
    f.s = p.scales[((int64_t)kg * p.rows + row) * 4 + g];
  }
}

// Which rows the tile of rows `tile` (BM rows each, the experts' one after the
// other, then the rows that have none) covers: [m0, m1) of Y, and its expert;
// expert -1: zeros; false: there is no such tile.  For a whole wave.  Offsets are
// taken as far as they ascend within Y.
__device__ inline bool find_tile(const Sorted &s, uint32_t tile, int bm, int64_t &m0, int64_t &m1, int32_t &expert) {
  const int lane = threadIdx.x & 63;
  const auto at = [&](int32_t e) {
    const int64_t o = s.offsets[e];
    return o < 0 ? 0 : o > s.total ? s.total : o;
  };
  uint32_t before = 0;
  for (int32_t e0 = 0; e0 <= s.experts; e0 += 64) {
    const int32_t e = e0 + lane;
    int64_t b = 0, end = 0;
    if (e <= s.experts) {
      b = at(e);
      end = e == s.experts ? s.total : at(e + 1);
    }
    const uint32_t own = end > b ? (uint32_t)((end - b + bm - 1) / bm) : 0u;
    uint32_t upto = own;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = (uint32_t)__shfl_up((int)upto, d);
      if (lane >= d) upto += o;
    }
    const uint32_t whole = before + (uint32_t)__shfl((int)upto, 63);
    if (tile < whole) {
      const bool mine = tile < before + upto && tile >= before + upto - own;
      const int who = __ffsll((unsigned long long)__ballot(mine)) - 1;
      const int64_t lo = __shfl((int)b, who), hi = __shfl((int)end, who);
      const uint32_t first = before + (uint32_t)__shfl((int)(upto - own), who);
      expert = e0 + who < s.experts ? e0 + who : -1;
      m0 = lo + (int64_t)(tile - first) * bm;
      m1 = m0 + bm < hi ? m0 + bm : hi;
      return true;
    }
    before = whole;
  }
  return false;
}

// Zeros to rows [m0, m1) and columns [n0, n1) of Y, by the whole workgroup.
template <typename T>
__device__ inline void clear_rows(T *Y, int64_t stride, int64_t m0, int64_t m1, int64_t n0, int64_t n1) {
  const int64_t wide = n1 - n0;
  for (int64_t i = threadIdx.x; i < (m1 - m0) * wide; i += blockDim.x)
    Y[(m0 + i / wide) * stride + n0 + i % wide] = (T)0.0f;
}

// MF x NF tiles of 16 x 16 by one workgroup, operands straight from memory: KW
// waves each take every KW-th group of 128 k and join their sums in shared memory.
template <typename T, int MF, int NF, int KW, bool EXPERTS>
__global__ __launch_bounds__(KW * 64) void k_nibble_rows(Operand X, Operand W, Sorted sorted,
                                                         const float *__restrict__ bias, T *__restrict__ Y,
                                                         int64_t stride, int64_t rows, int64_t n, int32_t blocks,
                                                         int32_t ng, int32_t nt) {
  __shared__ f32x4 part[KW][MF * NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  int64_t m0 = (int64_t)(workgroup() / (uint32_t)nt) * (MF * 16), m1 = rows;
  const int64_t n0 = (int64_t)(workgroup() % (uint32_t)nt) * (NF * 16);
  int64_t w0 = 0;
  if constexpr (EXPERTS) {
    int32_t expert;
    if (!find_tile(sorted, workgroup() / (uint32_t)nt, MF * 16, m0, m1, expert)) return;
    if (expert < 0) {
      clear_rows(Y, stride, m0, m1, n0, n0 + NF * 16 < n ? n0 + NF * 16 : n);
      return;
    }
    w0 = expert * n;
    if (bias) bias += w0;
  }
  if (m0 >= m1) return;
  f32x4 acc[MF][NF] = {};
  int64_t xrow[MF], wrow[NF];  // rows past the last read the last one
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    int64_t row = m0 + i * 16 + r;
    row = row < m1 ? row : m1 - 1;
    if constexpr (EXPERTS) {
      if (sorted.source) {
        const int64_t from = sorted.source[row];
        row = from < 0 ? 0 : from < X.rows ? from : X.rows - 1;
      }
    }
    xrow[i] = row;
  }
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int64_t row = n0 + col_of<kWoven<T, NF>>(j, r);
    wrow[j] = w0 + (row < n ? row : n - 1);
  }
  for (int32_t kg = wave; kg < ng; kg += KW) {
    Frag x[MF], w[NF];
#pragma unroll
    for (int i = 0; i < MF; ++i) load_frag(X, xrow[i], kg, g, blocks, x[i]);
#pragma unroll
    for (int j = 0; j < NF; ++j) load_frag(W, wrow[j], kg, g, blocks, w[j]);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[i][j] = multiply(w[j], x[i], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) part[wave][i * NF + j][lane] = acc[i][j];
  __syncthreads();
  // wave i adds up and writes row group i
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    if (i != wave) continue;
    f32x4 sum[1][NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      sum[0][j] = part[0][i * NF + j][lane];
#pragma unroll
      for (int t = 1; t < KW; ++t) sum[0][j] += part[t][i * NF + j][lane];
    }
    store_tiles<1, NF>(sum, m0 + i * 16, n0, m1, n, bias, Y, stride);
  }
}

struct Call {
  Operand x, w;
  Sorted sorted;
  const float *bias;
  int64_t stride, rows, n;
  int32_t blocks, ng;
};

// Tiles of bm rows: as many as there are, or for sorted rows at most as many as there can be.
template <bool EXPERTS>
int64_t row_tiles(const Call &c, int64_t bm) {
  if (!EXPERTS) return ceil_div(c.rows, bm);
  const int64_t parts = c.sorted.experts + 1 < c.rows ? c.sorted.experts + 1 : c.rows;  // that are not empty
  return (c.rows - parts) / bm + parts;
}

template <typename T, int MF, int NF, int KW, bool EXPERTS>
int rows_launch(const Call &c, T *y, hipStream_t s) {
  static_assert(MF <= KW, "a wave for each row group");
  const int64_t nt = ceil_div(c.n, NF * 16), wgs = row_tiles<EXPERTS>(c, MF * 16) * nt;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_nibble_rows<T, MF, NF, KW, EXPERTS>), grid_of(wgs), dim3(KW * 64), 0, s, c.x, c.w, c.sorted,
                     c.bias, y, c.stride, c.rows, c.n, c.blocks, c.ng, (int32_t)nt);
  return launched();
}

template <typename T, bool EXPERTS>
int product_as(const Call &c, void *Y, hipStream_t s) {
  return rows_launch<T, 2, 2, 4, EXPERTS>(c, static_cast<T *>(Y), s);
}
template <bool EXPERTS>
int product(const Call &c, void *Y, int32_t type, void *stream) {
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? product_as<float, EXPERTS>(c, Y, s)
         : type == SD_TYPE_F16 ? product_as<f16, EXPERTS>(c, Y, s)
                               : product_as<bf16, EXPERTS>(c, Y, s);
}

Operand operand(const sd_nibble_t *p) { return Operand{p->codes, p->scales, p->ld, p->rows}; }

}  // namespace

extern "C" int sd_nibble_product_size(int64_t rows, int64_t cols, int64_t n, size_t *bytes) {
  if (!bytes || rows < 0 || cols < 0 || n < 0) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || n > kMaxRows || cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  *bytes = 0;
  return SD_OK;
}

extern "C" int sd_nibble_product(const sd_nibble_t *X, const sd_nibble_t *W, const float *bias, void *Y, int32_t type,
                                 int64_t row_stride, void *workspace, size_t bytes, void *stream) {
  int st = check_nibble(X);
  if (st == SD_OK) st = check_nibble(W);
  if (st == SD_OK && X->cols != W->cols) st = SD_ERR_INVALID_VALUE;
  if (st == SD_OK) st = check_table(Y, type, X->rows, W->rows, row_stride);
  if (st == SD_OK && bias && !aligned_to(bias, 4)) st = SD_ERR_INVALID_VALUE;
  size_t need = 0;
  if (st == SD_OK) st = sd_nibble_product_size(X->rows, X->cols, W->rows, &need);
  if (st == SD_OK && need > 0 && (!workspace || bytes < need || !aligned_to(workspace, 16)))
    st = SD_ERR_INVALID_VALUE;
  if (st != SD_OK) return st;
  if (X->rows == 0 || W->rows == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  const Call c{operand(X), operand(W), Sorted{}, bias, row_stride, X->rows, W->rows, (int32_t)col_blocks(X->cols),
               (int32_t)groups_of(X->cols)};
  return product<false>(c, Y, type, stream);
}

extern "C" int sd_expert_product(const sd_nibble_t *X, const sd_nibble_t *W, const sd_route_t *route, int32_t sorted,
                                 const float *bias, void *Y, int32_t type, int64_t row_stride, void *stream) {
  int st = check_nibble(X);
  if (st == SD_OK) st = check_nibble(W);
  if (st == SD_OK) st = check_route(route);
  if (st != SD_OK) return st;
  const int64_t total = route->rows * route->k;
  if (X->cols != W->cols || W->rows % route->experts != 0 || X->rows != (sorted ? total : route->rows) ||
      (sorted != 0 && sorted != 1))
    return SD_ERR_INVALID_VALUE;
  const int64_t n = W->rows / route->experts;
  if ((st = check_table(Y, type, total, n, row_stride)) != SD_OK) return st;
  if (bias && !aligned_to(bias, 4)) return SD_ERR_INVALID_VALUE;
  if (total == 0 || n == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  const Call c{operand(X), operand(W), Sorted{route->offsets, sorted ? nullptr : route->source, route->experts, total},
               bias, row_stride, total, n, (int32_t)col_blocks(X->cols), (int32_t)groups_of(X->cols)};
  return product<true>(c, Y, type, stream);
}
