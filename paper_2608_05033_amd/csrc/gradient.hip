// sd_pack_gradient: dW[c, n] = sum_r value_X(r, c) G[r, n], X in 8 bits.
//
// The sum runs over the rows, so both operands are needed with neighbouring
// rows in one register: a thread reads the same columns of eight rows and
// writes them as eight consecutive 16-bit values of one column to shared memory.
// Codes become bf16 with their scale, which is exact (at most 4 significant
// bits times a power of two).  G in bf16 is used as it is; f16 and f32 are cut
// into two and three bf16 terms (8 significant bits each), which hold all of
// the 11 and 24 bits, and v_mfma_f32_16x16x32_bf16 sums the products in 32 bits.
// Workgroups share a tile's rows; their sums go to the workspace and a second
// kernel adds them in a fixed order.
#include "dense.h"

namespace {

using namespace dense;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kRows = 32;   // rows of a step
constexpr int kTileC = 128; // columns of X per tile: one block, so one scale a row
constexpr int kTileN = 64;  // columns of G per tile
constexpr int kPad = 8;     // 16-bit values between the columns in shared memory beyond kRows

template <typename T>
constexpr int terms() {
  return sizeof(T) == 4 ? 3 : __is_same(T, f16) ? 2 : 1;
}

template <int FMT>
__device__ inline bf16x2 to_bf16(uint32_t w, float s, bool hi) {
  if constexpr (FMT == SD_PACK_E4M3)
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
  else
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false);
}

// The leading 8 significant bits of v (the upper half of its 32), and v without
// them, which is exact.  Cutting never overflows as rounding up could; infinities
// and NaN go whole into the first term.
__device__ inline uint32_t cut(float &v) {
  const uint32_t b = __float_as_uint(v);
  const uint32_t top = v == v ? b & 0xffff0000u : 0x7fc00000u;
  v = (b & 0x7f800000u) == 0x7f800000u ? 0.0f : v - __uint_as_float(top);
  return top;
}

// Rows [r0, r1) of one tile by one workgroup: out[kTileC][kTileN] sums.
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void k_gradient(const uint8_t *__restrict__ codes,
                                                       const uint8_t *__restrict__ scales, int64_t ld, int64_t rows,
                                                       int32_t cols, const T *__restrict__ G, int64_t stride,
                                                       int32_t n, int32_t nt, int32_t splits, int64_t split_rows,
                                                       float *__restrict__ out, int64_t out_split) {
  constexpr int TERMS = terms<T>();
  constexpr int LD = kRows + kPad;
  __shared__ __align__(16) bf16 sx[kTileC * LD];
  __shared__ __align__(16) bf16 sg[TERMS][kTileN * LD];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r16 = lane & 15, g4 = lane >> 4;
  const int32_t split = blockIdx.x % (uint32_t)splits, tile = blockIdx.x / (uint32_t)splits;
  const int32_t ct = tile / nt, c0 = ct * kTileC, n0 = (tile % nt) * kTileN;
  const int64_t r0 = (int64_t)split * split_rows;
  const int64_t r1 = r0 + split_rows < rows ? r0 + split_rows : rows;
  // wave w: columns [64 (w / 2), +64) of X, [32 (w % 2), +32) of G
  f32x4 acc[4][2] = {};
  // X: 32 threads over the tile's columns (4 codes each), 8 groups of 4 rows; G: 64 threads over columns, 4 of 8 rows
  const int xc = (t & 31) * 4, xr = (t >> 5) * 4;
  const int gc = t & 63, gr = (t >> 6) * 8;
  const int32_t k16 = (cols + 15) & ~15;
  const bool x_in = c0 + xc < k16, g_in = n0 + gc < n;
  for (int64_t r = r0; r < r1; r += kRows) {
    bf16x2 lo[4], hi[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = r + xr + u;
      uint32_t w = 0;
      float s = 0.0f;
      if (row < r1 && x_in) {
        w = *reinterpret_cast<const uint32_t *>(codes + row * ld + c0 + xc);
        s = scale_value(scales[(int64_t)ct * rows + row]);
      }
      lo[u] = to_bf16<FMT>(w, s, false);
      hi[u] = to_bf16<FMT>(w, s, true);
    }
    float gv[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t row = r + gr + u;
      gv[u] = row < r1 && g_in ? (float)G[row * stride + n0 + gc] : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      sx[(xc + 0) * LD + xr + u] = lo[u][0];
      sx[(xc + 1) * LD + xr + u] = lo[u][1];
      sx[(xc + 2) * LD + xr + u] = hi[u][0];
      sx[(xc + 3) * LD + xr + u] = hi[u][1];
    }
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      u32x4 o;
#pragma unroll
      for (int u = 0; u < 8; u += 2) o[u / 2] = (cut(gv[u]) >> 16) | cut(gv[u + 1]);
      *reinterpret_cast<u32x4 *>(&sg[k][gc * LD + gr]) = o;
    }
    __syncthreads();
    bf16x8 a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a[i] = *reinterpret_cast<const bf16x8 *>(&sx[((wave >> 1) * 64 + i * 16 + r16) * LD + g4 * 8]);
#pragma unroll
    for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bf16x8 b = *reinterpret_cast<const bf16x8 *>(&sg[k][((wave & 1) * 32 + j * 16 + r16) * LD + g4 * 8]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b, acc[i][j], 0, 0, 0);
      }
  }
  float *o = out + split * out_split;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t c = c0 + (wave >> 1) * 64 + i * 16 + g4 * 4 + u, q = n0 + (wave & 1) * 32 + j * 16 + r16;
        if (c < cols && q < n) o[(int64_t)c * n + q] = acc[i][j][u];
      }
}

__global__ __launch_bounds__(kThreads) void k_gradient_join(const float *__restrict__ part, int64_t size,
                                                            int32_t splits, float *__restrict__ dw) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < size; i += (int64_t)gridDim.x * kThreads) {
    float sum = 0.0f;
    for (int32_t s = 0; s < splits; ++s) sum += part[s * size + i];
    dw[i] = sum;
  }
}

struct Split {
  int64_t tiles, split_rows;
  int32_t nt, splits;
};
// Two workgroups per compute unit over all tiles; a part of at least 8 steps.
Split split_of(int64_t rows, int64_t cols, int64_t n) {
  Split p{};
  p.nt = (int32_t)ceil_div(n, kTileN);
  p.tiles = blocks_of(cols) * p.nt;
  int64_t want = ceil_div(2ll * cu_count(), p.tiles > 0 ? p.tiles : 1);
  const int64_t most = ceil_div(rows, 8 * kRows);
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.split_rows = ceil_div(ceil_div(rows, want), kRows) * kRows;
  if (p.split_rows < kRows) p.split_rows = kRows;
  p.splits = (int32_t)ceil_div(rows, p.split_rows);
  if (p.splits < 1) p.splits = 1;
  return p;
}

template <typename T, int FMT>
int gradient(const sd_packed_t *X, const void *G, int64_t n, int64_t stride, float *dW, float *ws, const Split &p,
             hipStream_t s) {
  const int64_t wgs = p.tiles * p.splits, size = X->cols * n;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  float *out = p.splits > 1 ? ws : dW;
  hipLaunchKernelGGL((k_gradient<T, FMT>), dim3((uint32_t)wgs), dim3(kThreads), 0, s, X->codes, X->scales, X->ld,
                     X->rows, (int32_t)X->cols, static_cast<const T *>(G), stride, (int32_t)n, p.nt, p.splits,
                     p.split_rows, out, size);
  if (p.splits > 1) {
    const int64_t join = ceil_div(size, kThreads);
    hipLaunchKernelGGL(k_gradient_join, dim3((uint32_t)(join < 65536 ? join : 65536)), dim3(kThreads), 0, s, ws, size,
                       p.splits, dW);
  }
  return launched();
}
template <typename T>
int gradient_as(const sd_packed_t *X, const void *G, int64_t n, int64_t stride, float *dW, float *ws, const Split &p,
                hipStream_t s) {
  return X->format == SD_PACK_E4M3 ? gradient<T, SD_PACK_E4M3>(X, G, n, stride, dW, ws, p, s)
                                   : gradient<T, SD_PACK_E5M2>(X, G, n, stride, dW, ws, p, s);
}

size_t workspace_of(const Split &p, int64_t cols, int64_t n) {
  return p.splits > 1 ? 4 * (size_t)p.splits * (size_t)cols * (size_t)n : 0;
}

}  // namespace

extern "C" int sd_pack_gradient_size(int64_t rows, int64_t cols, int64_t n, size_t *bytes) {
  if (!bytes || rows < 0 || cols < 0 || n < 0) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || cols > kMaxRows - 1024 || n > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  *bytes = workspace_of(split_of(rows, cols, n), cols, n);
  return SD_OK;
}

extern "C" int sd_pack_gradient(const sd_packed_t *X, const void *G, int32_t type, int64_t n, int64_t row_stride,
                                float *dW, void *workspace, size_t bytes, void *stream) {
  int st = check_packed(X);
  if (st != SD_OK) return st;
  if (n < 0) return SD_ERR_INVALID_VALUE;
  if (n > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if ((st = check_table(G, type, X->rows, n, row_stride)) != SD_OK) return st;
  if (X->cols == 0 || n == 0) return SD_OK;
  const Split p = split_of(X->rows, X->cols, n);
  const size_t need = workspace_of(p, X->cols, n);
  if (!dW || !aligned_to(dW, 4) || bytes < need || (need > 0 && (!workspace || !aligned_to(workspace, 16))))
    return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float *ws = static_cast<float *>(workspace);
  return type == SD_TYPE_F32   ? gradient_as<float>(X, G, n, row_stride, dW, ws, p, s)
         : type == SD_TYPE_F16 ? gradient_as<f16>(X, G, n, row_stride, dW, ws, p, s)
                               : gradient_as<bf16>(X, G, n, row_stride, dW, ws, p, s);
}
