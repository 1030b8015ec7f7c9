// sd_pack_gradient: dW[c, n] = sum_r value_X(r, c) G[r, n], X in 8 bits.
//
// The sum runs over the rows, so both operands are needed with neighbouring
// rows in one register: a thread reads the same columns of eight rows and
// writes them as eight consecutive 16-bit values of one column to shared memory.
// Codes become bf16 with their scale (at most 4 significant bits times a power of
// two).  G in bf16 is used as it is; f16 and f32 are cut into two and three bf16
// terms (8 significant bits each), which hold all of the 11 and 24 bits, and
// v_mfma_f32_16x16x32_bf16 sums the products in 32 bits.  All of that is exact as
// far as bf16 reaches, down to multiples of 2^-133.
// Workgroups share a tile's rows; their sums go to the workspace and a second
// kernel adds them in a fixed order.
// 262144 x 128 codes with 64 columns of fp32 take 28 us and the join 4: 3.7 TB/s,
// bound by the bytes and by cutting G into its terms.  50021 x 601 with 129 columns
// of bf16 take 35 and 7, where the last column of G costs a whole tile.
#include "dense.h"

namespace {

using namespace dense;

constexpr int kThreads = 256;
constexpr int kRows = 64;   // rows of a step
constexpr int kTileC = 128; // columns of X per tile: one block, so one scale a row

template <typename T>
constexpr int terms() {
  return sizeof(T) == 4 ? 3 : __is_same(T, f16) ? 2 : 1;
}

// v without its leading 8 significant bits (the upper half of its 32), which is
// exact: the next term.  Cutting never overflows as rounding up could.
// Infinities and NaN are whole in the first term (the quiet bit is in the upper
// half), nothing is left of them.
__device__ inline float rest_of(float v) {
  const float r = v - __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  return r == r ? r : 0.0f;
}
// The upper halves of a and b side by side.
__device__ inline uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// Shared memory holds columns of kRows 16-bit values, in units of 8 rows.  The
// unit's place is mixed with the column's, so that 16 neighbouring columns read
// at one unit, and every fourth column written at one, touch different banks.
__device__ inline int place(int col, int unit) {
  return (col * (kRows / 8) + (unit ^ ((col >> 1) & 7) ^ ((col >> 4) & 1))) * 8;
}

// Rows [r0, r1) of one kTileC x TN tile by one workgroup.  The next step's rows
// are read into registers while this step's products run.
template <typename T, int FMT, int TN>
__global__ __launch_bounds__(kThreads) void k_gradient(const uint8_t *__restrict__ codes,
                                                       const uint8_t *__restrict__ scales, int64_t ld, int64_t rows,
                                                       int32_t cols, const T *__restrict__ G, int64_t stride,
                                                       int32_t n, int32_t nt, uint32_t tiles, uint32_t wgs,
                                                       int64_t split_rows, float *__restrict__ out,
                                                       int64_t out_split) {
  constexpr int TERMS = terms<T>();
  constexpr int NJ = TN / 32;                              // 16-column products per wave
  constexpr int GC = 4 / sizeof(T), GU = TN / (32 * GC);  // G: columns (one word) and units of 8 rows per thread
  __shared__ __align__(16) bf16 sx[kTileC * kRows];
  __shared__ __align__(16) bf16 sg[TERMS][TN * kRows];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r16 = lane & 15, g4 = lane >> 4;
  if (workgroup() >= wgs) return;
  // a split's tiles, which read the same rows, run on one XCD
  const uint32_t at = xcd_place(workgroup(), wgs);
  const int32_t split = at / tiles, tile = at % tiles;
  const int32_t ct = tile / nt, c0 = ct * kTileC, n0 = (tile % nt) * TN;
  const int64_t r0 = (int64_t)split * split_rows;
  const int64_t r1 = r0 + split_rows < rows ? r0 + split_rows : rows;
  // wave w: columns [64 (w / 2), +64) of X, [TN / 2 (w % 2), +TN / 2) of G
  f32x4 acc[4][NJ] = {};
  // X: 4 codes (one word) of 8 rows per thread
  const int xc = (t & 31) * 4, xu = t >> 5;
  const int gc = t % (TN / GC) * GC, gu = t / (TN / GC) * GU;
  const int32_t k16 = (cols + 15) & ~15;
  // Columns past the last read the last ones' place: their sums go nowhere.  A
  // word that holds the last column as its first is read one column earlier and
  // shifted when it is used.
  const int32_t xcol = c0 + xc < k16 ? c0 + xc : k16 - 4;
  const int32_t gcol = n0 + gc, gword = gcol + GC <= n ? gcol : n - GC;
  const int gshift = gword < gcol ? 16 : 0;
  const uint8_t *xp = codes + xcol + xu * 8 * ld, *sp = scales + (int64_t)ct * rows + xu * 8;
  const T *gp = G + gword + gu * 8 * stride;
  uint32_t xw[8], gw[GU][8], shift = 0;
  Span<uint8_t, 8> xs;
  auto fetch = [&](int64_t r) {
    const uint8_t *xr = xp + r * ld, *sr = sp + r;
    const T *gr = gp + r * stride;
    if (r + kRows <= r1 && n >= GC) {
#pragma unroll
      for (int u = 0; u < 8; ++u) xw[u] = *reinterpret_cast<const uint32_t *>(xr + u * ld);
      xs = *reinterpret_cast<const Span<uint8_t, 8> *>(sr);
#pragma unroll
      for (int u = 0; u < GU * 8; ++u)
        gw[u / 8][u % 8] = reinterpret_cast<const Span<uint32_t, 1, sizeof(T)> *>(gr + u * stride)->v[0];
      shift = gshift;
    } else {
      const int xl = (int)(r1 - r) - xu * 8, gl = (int)(r1 - r) - gu * 8;  // rows left for this thread
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        xw[u] = u < xl ? *reinterpret_cast<const uint32_t *>(xr + u * ld) : 0u;
        xs.v[u] = u < xl ? sr[u] : (uint8_t)127;
      }
#pragma unroll
      for (int u = 0; u < GU * 8; ++u) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < GC; ++j)
          if (u < gl && gcol + j < n) {
            const T *p = G + gcol + j + (r + gu * 8 + u) * stride;
            if constexpr (GC == 1)
              w = *reinterpret_cast<const uint32_t *>(p);
            else
              w |= (uint32_t)*reinterpret_cast<const uint16_t *>(p) << (16 * j);
          }
        gw[u / 8][u % 8] = w;
      }
      shift = 0;
    }
  };
  if (r0 < r1) fetch(r0);
  for (int64_t r = r0; r < r1; r += kRows) {
    __syncthreads();
    {
      // four columns of eight rows: pairs of rows side by side
      bf16x2 lo[8], hi[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float s = scale_value(xs.v[u]);
        lo[u] = to_bf16<FMT>(xw[u], s, false);
        hi[u] = to_bf16<FMT>(xw[u], s, true);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 o;
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = j < 2 ? lo[u][j & 1] : hi[u][j & 1];
        *reinterpret_cast<bf16x8 *>(&sx[place(xc + j, xu)]) = o;
      }
    }
    if constexpr (GC > 1) {
#pragma unroll
      for (int u = 0; u < GU * 8; ++u) gw[u / 8][u % 8] >>= shift;
    }
#pragma unroll
    for (int k = 0; k < GU; ++k) {
      if constexpr (TERMS == 1) {
        u32x4 even, odd;
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
          even[u / 2] = __builtin_amdgcn_perm(gw[k][u + 1], gw[k][u], 0x05040100u);
          odd[u / 2] = __builtin_amdgcn_perm(gw[k][u + 1], gw[k][u], 0x07060302u);
        }
        *reinterpret_cast<u32x4 *>(&sg[0][place(gc, gu + k)]) = even;
        *reinterpret_cast<u32x4 *>(&sg[0][place(gc + 1, gu + k)]) = odd;
      } else {
#pragma unroll
        for (int j = 0; j < GC; ++j) {
          float v[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            if constexpr (GC == 1)
              v[u] = __builtin_canonicalizef(__uint_as_float(gw[k][u]));
            else
              v[u] = (float)__builtin_bit_cast(f16, (uint16_t)(gw[k][u] >> (16 * j)));
          }
#pragma unroll
          for (int q = 0; q < TERMS; ++q) {
            u32x4 o;
#pragma unroll
            for (int u = 0; u < 8; u += 2) o[u / 2] = upper_halves(v[u], v[u + 1]);
            *reinterpret_cast<u32x4 *>(&sg[q][place(gc + j, gu + k)]) = o;
            if (q + 1 < TERMS)
#pragma unroll
              for (int u = 0; u < 8; ++u)
                v[u] = q == 0 ? rest_of(v[u]) : v[u] - __uint_as_float(__float_as_uint(v[u]) & 0xffff0000u);
          }
        }
      }
    }
    __syncthreads();
    if (r + kRows < r1) fetch(r + kRows);
#pragma unroll
    for (int h = 0; h < kRows / 32; ++h) {
      bf16x8 a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        a[i] = *reinterpret_cast<const bf16x8 *>(&sx[place((wave >> 1) * 64 + i * 16 + r16, h * 4 + g4)]);
#pragma unroll
      for (int q = TERMS - 1; q >= 0; --q)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const bf16x8 b =
              *reinterpret_cast<const bf16x8 *>(&sg[q][place((wave & 1) * (TN / 2) + j * 16 + r16, h * 4 + g4)]);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b, acc[i][j], 0, 0, 0);
        }
    }
  }
  float *o = out + split * out_split;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int32_t c = c0 + (wave >> 1) * 64 + i * 16 + g4 * 4 + u, q = n0 + (wave & 1) * (TN / 2) + j * 16 + r16;
        if (c < cols && q < n) o[(int64_t)c * n + q] = acc[i][j][u];
      }
}

// Sixteen threads share an output, each adding every sixteenth part.
constexpr int kJoinOut = 64, kJoinWays = 16;
__global__ __launch_bounds__(kJoinOut *kJoinWays) void k_gradient_join(const float *__restrict__ part, int64_t size,
                                                                       int32_t splits, float *__restrict__ dw) {
  __shared__ float sums[kJoinWays][kJoinOut];
  const int o = threadIdx.x % kJoinOut, way = threadIdx.x / kJoinOut;
  for (int64_t base = (int64_t)blockIdx.x * kJoinOut; base < size; base += (int64_t)gridDim.x * kJoinOut) {
    float sum = 0.0f;
    if (base + o < size) {
#pragma unroll 8
      for (int32_t s = way; s < splits; s += kJoinWays) sum += part[s * size + base + o];
    }
    sums[way][o] = sum;
    __syncthreads();
    if (way == 0 && base + o < size) {
#pragma unroll
      for (int w = 1; w < kJoinWays; ++w) sum += sums[w][o];
      dw[base + o] = sum;
    }
    __syncthreads();
  }
}

struct Split {
  int64_t tiles, split_rows;
  int32_t nt, splits, tn;
};
// Two workgroups per compute unit over all tiles; a part of at least 4 steps.
// Columns of G a tile: 128 of 16-bit G where more than 64 are there, so that X is
// read half as often; 64 of fp32, whose three terms fill the registers and shared
// memory.  Measured in us, 64 and 128 columns:
//   rows x columns x n         fp32        f16         bf16
//   262144 x 128 x 128       47   63     36   38     30   30
//   50021 x 601 x 129        58  101     48   52     39   39
//   20000 x 1024 x 256       54   76     47   44     39   36
//   8000 x 2048 x 1024      176  230    152  134    127  106
Split split_of(int64_t rows, int64_t cols, int64_t n, bool wide_type) {
  Split p{};
  p.tn = n > 64 && !wide_type ? 128 : 64;
  p.nt = (int32_t)ceil_div(n, p.tn);
  p.tiles = blocks_of(cols) * p.nt;
  int64_t want = 2ll * cu_count() / (p.tiles > 0 ? p.tiles : 1);
  const int64_t most = ceil_div(rows, 4 * kRows);
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
  auto *kernel = k_gradient<T, FMT, 64>;
  if constexpr (sizeof(T) == 2)
    if (p.tn == 128) kernel = k_gradient<T, FMT, 128>;
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, X->codes, X->scales, X->ld,
                     X->rows, (int32_t)X->cols, static_cast<const T *>(G), stride, (int32_t)n, p.nt,
                     (uint32_t)p.tiles, (uint32_t)wgs, p.split_rows, out, size);
  if (p.splits > 1) {
    const int64_t join = ceil_div(size, kJoinOut);
    hipLaunchKernelGGL(k_gradient_join, dim3((uint32_t)(join < 65536 ? join : 65536)), dim3(kJoinOut * kJoinWays), 0,
                       s, ws, size, p.splits, dW);
  }
  return launched();
}
template <typename T>
int gradient_as(const sd_packed_t *X, const void *G, int64_t n, int64_t stride, float *dW, float *ws, const Split &p,
                hipStream_t s) {
  return X->format == SD_PACK_E4M3 ? gradient<T, SD_PACK_E4M3>(X, G, n, stride, dW, ws, p, s)
                                   : gradient<T, SD_PACK_E5M2>(X, G, n, stride, dW, ws, p, s);
}

// Enough for any type of G.
size_t workspace_of(int64_t rows, int64_t cols, int64_t n) {
  const int32_t a = split_of(rows, cols, n, true).splits, b = split_of(rows, cols, n, false).splits, most = a > b ? a : b;
  return most > 1 ? 4 * (size_t)most * (size_t)cols * (size_t)n : 0;
}

}  // namespace

extern "C" int sd_pack_gradient_size(int64_t rows, int64_t cols, int64_t n, size_t *bytes) {
  if (!bytes || rows < 0 || cols < 0 || n < 0) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || cols > kMaxRows - 1024 || n > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  *bytes = workspace_of(rows, cols, n);
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
  const Split p = split_of(X->rows, X->cols, n, type == SD_TYPE_F32);
  const size_t need = workspace_of(X->rows, X->cols, n);
  if (!dW || !aligned_to(dW, 4) || bytes < need || (need > 0 && (!workspace || !aligned_to(workspace, 16))))
    return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float *ws = static_cast<float *>(workspace);
  return type == SD_TYPE_F32   ? gradient_as<float>(X, G, n, row_stride, dW, ws, p, s)
         : type == SD_TYPE_F16 ? gradient_as<f16>(X, G, n, row_stride, dW, ws, p, s)
                               : gradient_as<bf16>(X, G, n, row_stride, dW, ws, p, s);
}
