// Results of the matrix units on their way to memory, shared by the products.
#pragma once

#include "dense.h"

namespace dense {

// Where row rho of a wave's tile j lies among its rows of W (columns of Y).  For
// 16-bit results two tiles are woven so that a lane's four columns of each are
// eight neighbours, written in one store of 16 bytes.
template <typename T, int NF>
constexpr bool kWoven = sizeof(T) == 2 && NF % 2 == 0;
template <bool WOVEN>
__device__ constexpr int col_of(int j, int rho) {
  return WOVEN ? j / 2 * 32 + rho / 4 * 8 + j % 2 * 4 + rho % 4 : j * 16 + rho;
}

// A wave's MF x NF tiles from (m0, n0) on, with the bias, as far as they are inside Y: lane (r, g) holds
// four neighbouring n from 4 g on of row r of each.
template <int MF, int NF, typename T>
__device__ inline void store_tiles(const f32x4 (&acc)[MF][NF], int64_t m0, int64_t n0, int64_t rows, int64_t cols,
                                   const float *__restrict__ bias, T *__restrict__ Y, int64_t stride) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  constexpr bool WOVEN = kWoven<T, NF>;
  constexpr int RUN = WOVEN ? 8 : 4;  // neighbouring columns of a lane
  float b[NF][4] = {};
  if (bias) {
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t n = n0 + col_of<WOVEN>(j, g * 4 + t);
        b[j][t] = n < cols ? bias[n] : 0.0f;
      }
  }
  T *y = Y + (m0 + r) * stride + n0;
  if (n0 + NF * 16 <= cols) {  // the same for the wave: a row's lines are written one after the other
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      if (m0 + i * 16 + r < rows) {
#pragma unroll
        for (int j = 0; j < NF; j += RUN / 4) {
          float out[RUN];
#pragma unroll
          for (int t = 0; t < RUN; ++t) out[t] = acc[i][j + t / 4][t % 4] + b[j + t / 4][t % 4];
          store_span(y + i * 16 * stride + col_of<WOVEN>(j, g * 4), out);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < NF; j += RUN / 4) {
    if (n0 + (j + RUN / 4) * 16 <= cols) {  // the same for the wave
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        float out[RUN];
#pragma unroll
        for (int t = 0; t < RUN; ++t) out[t] = acc[i][j + t / 4][t % 4] + b[j + t / 4][t % 4];
        if (m0 + i * 16 + r < rows) store_span(y + i * 16 * stride + col_of<WOVEN>(j, g * 4), out);
      }
    } else if (n0 + j * 16 < cols) {
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int t = 0; t < RUN; ++t) {
          const int n = col_of<WOVEN>(j, g * 4) + t;
          if (m0 + i * 16 + r < rows && n0 + n < cols)
            y[i * 16 * stride + n] = rounded<T>(acc[i][j + t / 4][t % 4] + b[j + t / 4][t % 4]);
        }
    }
  }
}

}  // namespace dense
