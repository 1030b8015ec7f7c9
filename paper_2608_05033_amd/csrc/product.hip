// sd_pack_product: Y[m, n] = sum_k X(m, k) W(n, k) + bias[n] for two packed
// matrices, on the matrix units.
//
// A wave's 16 x 16 tile over one block of 128 k: lane (r, g) = (lane % 16,
// lane / 16) holds 32 codes of row r of each side, and its row's scale byte.
// Which 32 of the 128 a lane group holds does not matter as long as both sides
// agree, since one scale covers them all.  W is the first operand, so a lane
// ends with four neighbouring n of one row m and writes them in one store.
//
// Two instruction forms (measured on this card against 64 bits, normal values):
//  * 16-bit results: v_mfma_scale_f32_16x16x128_f8f6f4, codes and scales as they
//    are.  It aligns the 128 products of a step to the largest and drops what
//    is below, 1.6e-5 of the result in 2-norm: under a tenth of an f16 rounding.
//  * 32-bit results: the codes become bf16, exactly (4 or 3 significant bits and
//    a power of two), and v_mfma_f32_16x16x32_bf16 sums in 32 bits (1.2e-7).
#include "dense.h"

namespace {

using namespace dense;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Operand {
  const uint8_t *codes, *scales;
  int64_t ld, rows;
};

template <int FMT>
__device__ inline bf16x2 to_bf16(uint32_t w, float s, bool hi) {
  if constexpr (FMT == SD_PACK_E4M3)
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
  else
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false);
}

// 32 codes of one row in a block, and the block's scale byte.
struct Frag {
  i32x8 v;
  uint32_t s;
};
// Eight of them as bf16 values.
template <int FMT>
__device__ inline bf16x8 bf16_of(const Frag &f, int q) {
  const float s = scale_value(f.s);
  bf16x8 o;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t w = (uint32_t)f.v[2 * q + j];
    const bf16x2 lo = to_bf16<FMT>(w, s, false), hi = to_bf16<FMT>(w, s, true);
    o[4 * j] = lo[0];
    o[4 * j + 1] = lo[1];
    o[4 * j + 2] = hi[0];
    o[4 * j + 3] = hi[1];
  }
  return o;
}

template <int WF, int XF>
__device__ inline f32x4 mfma_scaled(const Frag &w, const Frag &x, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, c, WF == SD_PACK_E5M2, XF == SD_PACK_E5M2, 0,
                                                          (int)w.s, 0, (int)x.s);
}

// Codes [32 g, 32 g + 32) of block kb of one row; zero past the row's last 16.
__device__ inline void load_frag(const Operand &p, int64_t row, int32_t kb, int g, int32_t k16, Frag &f) {
  const int32_t at = kb * kBlock + g * 32;
  const uint8_t *q = p.codes + row * p.ld + at;
  u32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
  if (at < k16) a = *reinterpret_cast<const u32x4 *>(q);
  if (at + 16 < k16) b = *reinterpret_cast<const u32x4 *>(q + 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f.v[i] = (int)a[i];
    f.v[4 + i] = (int)b[i];
  }
  f.s = p.scales[kb * p.rows + row];
}

// MF x NF tiles of 16 x 16 per wave, operands straight from memory.  KW waves
// share a tile, each taking every KW-th block of k, and join their sums in
// shared memory; with KW = 1 the four waves of a workgroup take four tiles.
template <typename T, int XF, int WF, int MF, int NF, int KW>
__global__ __launch_bounds__(KW > 4 ? KW * 64 : 256) void k_product_rows(Operand X, Operand W,
                                                                         const float *__restrict__ bias,
                                                                         T *__restrict__ Y, int64_t stride,
                                                                         int32_t k16, int32_t nb, int32_t nt) {
  constexpr int WAVES = KW > 4 ? KW : 4, TILES = WAVES / KW;
  __shared__ f32x4 part[KW > 1 ? WAVES : 1][MF * NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t m0 = ((int64_t)(blockIdx.x / (uint32_t)nt) * TILES + wave / KW) * (MF * 16);
  const int64_t n0 = (int64_t)(blockIdx.x % (uint32_t)nt) * (NF * 16);
  f32x4 acc[MF][NF] = {};
  for (int32_t kb = wave % KW; kb < nb; kb += KW) {
    Frag x[MF], w[NF];
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const int64_t row = m0 + i * 16 + r;
      load_frag(X, row < X.rows ? row : X.rows - 1, kb, g, k16, x[i]);
    }
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      const int64_t row = n0 + j * 16 + r;
      load_frag(W, row < W.rows ? row : W.rows - 1, kb, g, k16, w[j]);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = mfma_scaled<WF, XF>(w[j], x[i], acc[i][j]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        bf16x8 xb[MF], wb[NF];
#pragma unroll
        for (int i = 0; i < MF; ++i) xb[i] = bf16_of<XF>(x[i], q);
#pragma unroll
        for (int j = 0; j < NF; ++j) wb[j] = bf16_of<WF>(w[j], q);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
          for (int j = 0; j < NF; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j], xb[i], acc[i][j], 0, 0, 0);
      }
    }
  }
  if constexpr (KW > 1) {
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) part[wave][i * NF + j][lane] = acc[i][j];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      f32x4 sum = acc[i][j];
      if constexpr (KW > 1) {
        if ((i * NF + j) % KW != wave) continue;
        sum = part[0][i * NF + j][lane];
        for (int t = 1; t < KW; ++t) sum += part[t][i * NF + j][lane];
      }
      const int64_t m = m0 + i * 16 + r, n = n0 + j * 16 + g * 4;
      if (m >= X.rows || n >= W.rows) continue;
      float out[4];
      const int left = W.rows - n < 4 ? (int)(W.rows - n) : 4;
#pragma unroll
      for (int t = 0; t < 4; ++t) out[t] = sum[t] + (bias && t < left ? bias[n + t] : 0.0f);
      T *q = Y + m * stride + n;
      if (left == 4)
        store_span(q, out);
      else
        store_part(q, left, out);
    }
}

template <typename T, int XF, int WF, int MF, int NF, int KW>
int rows_launch(const Operand &x, const Operand &w, const float *bias, T *y, int64_t stride, int32_t k16, int32_t nb,
                hipStream_t s) {
  constexpr int WAVES = KW > 4 ? KW : 4, TILES = WAVES / KW;
  const int64_t nt = ceil_div(w.rows, NF * 16), wgs = ceil_div(x.rows, MF * 16 * TILES) * nt;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_product_rows<T, XF, WF, MF, NF, KW>), dim3((uint32_t)wgs), dim3(WAVES * 64), 0, s, x, w, bias,
                     y, stride, k16, nb, (int32_t)nt);
  return launched();
}

template <typename T, int XF, int WF>
int product(const sd_packed_t *X, const sd_packed_t *W, const float *bias, void *Y, int64_t stride, hipStream_t s) {
  const Operand x{X->codes, X->scales, X->ld, X->rows}, w{W->codes, W->scales, W->ld, W->rows};
  const int32_t k16 = (int32_t)(ceil_div(X->cols, 16) * 16), nb = (int32_t)blocks_of(X->cols);
  T *y = static_cast<T *>(Y);
  if (x.rows <= 16) return rows_launch<T, XF, WF, 1, 1, 8>(x, w, bias, y, stride, k16, nb, s);
  return rows_launch<T, XF, WF, 4, 4, 1>(x, w, bias, y, stride, k16, nb, s);
}
template <typename T>
int product_as(const sd_packed_t *X, const sd_packed_t *W, const float *bias, void *Y, int64_t stride, hipStream_t s) {
  if (X->format == SD_PACK_E4M3)
    return W->format == SD_PACK_E4M3 ? product<T, SD_PACK_E4M3, SD_PACK_E4M3>(X, W, bias, Y, stride, s)
                                     : product<T, SD_PACK_E4M3, SD_PACK_E5M2>(X, W, bias, Y, stride, s);
  return W->format == SD_PACK_E4M3 ? product<T, SD_PACK_E5M2, SD_PACK_E4M3>(X, W, bias, Y, stride, s)
                                   : product<T, SD_PACK_E5M2, SD_PACK_E5M2>(X, W, bias, Y, stride, s);
}

}  // namespace

extern "C" int sd_pack_product(const sd_packed_t *X, const sd_packed_t *W, const float *bias, void *Y, int32_t type,
                               int64_t row_stride, void *stream) {
  int st = check_packed(X);
  if (st == SD_OK) st = check_packed(W);
  if (st == SD_OK && X->cols != W->cols) st = SD_ERR_INVALID_VALUE;
  if (st == SD_OK) st = check_table(Y, type, X->rows, W->rows, row_stride);
  if (st == SD_OK && bias && !aligned_to(bias, 4)) st = SD_ERR_INVALID_VALUE;
  if (st != SD_OK) return st;
  if (X->rows == 0 || W->rows == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? product_as<float>(X, W, bias, Y, row_stride, s)
         : type == SD_TYPE_F16 ? product_as<f16>(X, W, bias, Y, row_stride, s)
                               : product_as<bf16>(X, W, bias, Y, row_stride, s);
}
