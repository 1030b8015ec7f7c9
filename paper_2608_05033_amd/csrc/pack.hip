// sd_pack / sd_unpack: dense tables to 8 bits and back.
//
// value(r, c) = f8(code(r, c)) * 2^(s(c / 128, r) - 127).  The scale of a row's
// block of 128 columns is the least power of two that brings its largest finite
// magnitude into the format's range, so both directions are exact up to the one
// rounding to the format (nearest, ties to even).
#include "dense.h"

namespace dense {

int cu_count() {
  constexpr int kMaxDevices = 64;
  static int32_t cached[kMaxDevices];  // 0: not asked yet; every writer stores the same value
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)hipGetLastError();
    return sd::kDefaultCUs;
  }
  int32_t n = __atomic_load_n(&cached[dev], __ATOMIC_RELAXED);
  if (n == 0) {
    int v = 0;
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) {
      (void)hipGetLastError();
      v = sd::kDefaultCUs;
    }
    n = v;
    __atomic_store_n(&cached[dev], n, __ATOMIC_RELAXED);
  }
  return n;
}

}  // namespace dense

namespace {

using namespace dense;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // row blocks in flight per lane group

// A group of 128 / V lanes takes one row's block of 128 columns: V neighbouring
// columns per lane (16 bytes), the block's maximum over the lanes, V codes per
// lane back.  Bound by the bytes read and written; four blocks per group are in
// flight: 262144 x 128 fp32 take 25 us, 6.6 TB/s of bytes that the 256 MB Infinity
// Cache partly serves.  COLS: consecutive elements of a row lie together (else any strides,
// each lane's elements read one by one).
template <typename T, int FMT, bool COLS>
__global__ __launch_bounds__(kThreads) void k_pack(const T *__restrict__ x, int64_t row_stride, int64_t col_stride,
                                                   int64_t rows, int32_t cols, int32_t nb, uint8_t *__restrict__ codes,
                                                   int64_t ld, uint8_t *__restrict__ scales) {
  constexpr int V = 16 / sizeof(T), LANES = kBlock / V, GROUPS = kThreads / LANES;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int64_t first = (int64_t)workgroup() * (GROUPS * kUnroll);
  const int64_t r0 = first / nb;
  const uint32_t b0 = (uint32_t)(first - r0 * nb);
  float v[kUnroll][V];
  int64_t row[kUnroll];
  int32_t blk[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t at = b0 + u * GROUPS + group;
    row[u] = r0 + at / (uint32_t)nb;
    blk[u] = at % (uint32_t)nb;
    const int32_t c = blk[u] * kBlock + lane * V;
    const int left = row[u] < rows ? cols - c : 0;
    if constexpr (COLS) {
      const T *p = x + row[u] * row_stride + c;
      if (left >= V)
        load_span(p, v[u]);
      else
        load_part(p, left, v[u]);
    } else {
      const T *p = x + row[u] * row_stride + c * col_stride;
#pragma unroll
      for (int i = 0; i < V; ++i) v[u][i] = i < left ? (float)p[i * col_stride] : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t s = scale_byte<FMT>(largest_finite(v[u], V, LANES));
    const float inv = inverse_scale(s);
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
      w[i] = encode4<FMT>(v[u][4 * i] * inv, v[u][4 * i + 1] * inv, v[u][4 * i + 2] * inv, v[u][4 * i + 3] * inv);
    if (row[u] >= rows) continue;
    const int32_t c = blk[u] * kBlock + lane * V;
    if (c < ((cols + 15) & ~15)) {
      uint8_t *p = codes + row[u] * ld + c;
      if constexpr (V == 4)
        *reinterpret_cast<uint32_t *>(p) = w[0];
      else
        *reinterpret_cast<u32x2 *>(p) = u32x2{w[0], w[V / 4 - 1]};
    }
    if (lane == 0) scales[(int64_t)blk[u] * rows + row[u]] = (uint8_t)s;
  }
}

// Lanes along a row, four codes each.  Bound by the bytes written: 262144 x 128 to
// bf16 take 22 us, 4.5 TB/s.
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void k_unpack(const uint8_t *__restrict__ codes, int64_t ld,
                                                     const uint8_t *__restrict__ scales, int64_t rows, int32_t cols,
                                                     int32_t quads, T *__restrict__ y, int64_t row_stride) {
  const int64_t first = (int64_t)workgroup() * (kThreads * kUnroll);
  const int64_t r0 = first / quads;
  const uint32_t q0 = (uint32_t)(first - r0 * quads);
  uint32_t w[kUnroll];
  float s[kUnroll];
  int64_t row[kUnroll];
  int32_t col[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t at = q0 + u * kThreads + threadIdx.x;
    row[u] = r0 + at / (uint32_t)quads;
    col[u] = (int32_t)(at % (uint32_t)quads) * 4;
    w[u] = 0;
    s[u] = 0;
    if (row[u] < rows) {
      w[u] = *reinterpret_cast<const uint32_t *>(codes + row[u] * ld + col[u]);
      s[u] = scale_value(scales[(int64_t)(col[u] / kBlock) * rows + row[u]]);
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (row[u] >= rows) continue;
    float v[4];
    decode4<FMT>(w[u], v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= s[u];
    T *p = y + row[u] * row_stride + col[u];
    const int left = cols - col[u];
    if (left >= 4)
      store_span(p, v);
    else
      store_part(p, left, v);
  }
}

template <typename T, int FMT>
int pack_as(const T *x, int64_t row_stride, int64_t col_stride, const sd_packed_t *out, hipStream_t s) {
  constexpr int per_wg = kThreads / (kBlock * (int)sizeof(T) / 16) * kUnroll;
  const int64_t nb = blocks_of(out->cols), wgs = ceil_div(out->rows * nb, per_wg);
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  auto *kernel = col_stride == 1 ? k_pack<T, FMT, true> : k_pack<T, FMT, false>;
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, x, row_stride, col_stride, out->rows,
                     (int32_t)out->cols, (int32_t)nb, out->codes, out->ld, out->scales);
  return launched();
}
template <typename T>
int pack_any(const void *x, int64_t row_stride, int64_t col_stride, const sd_packed_t *out, hipStream_t s) {
  const T *p = static_cast<const T *>(x);
  return out->format == SD_PACK_E4M3 ? pack_as<T, SD_PACK_E4M3>(p, row_stride, col_stride, out, s)
                                     : pack_as<T, SD_PACK_E5M2>(p, row_stride, col_stride, out, s);
}

template <typename T>
int unpack_as(const sd_packed_t *x, void *y, int64_t row_stride, hipStream_t s) {
  const int64_t quads = ceil_div(x->cols, 4), wgs = ceil_div(x->rows * quads, kThreads * kUnroll);
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  auto *kernel = x->format == SD_PACK_E4M3 ? k_unpack<T, SD_PACK_E4M3> : k_unpack<T, SD_PACK_E5M2>;
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, x->codes, x->ld, x->scales, x->rows,
                     (int32_t)x->cols, (int32_t)quads, static_cast<T *>(y), row_stride);
  return launched();
}

}  // namespace

extern "C" int sd_pack(const void *x, int32_t type, int64_t row_stride, int64_t col_stride, const sd_packed_t *out,
                       void *stream) {
  int st = check_packed(out);
  if (st != SD_OK) return st;
  if (!type_ok(type) || row_stride < 0 || col_stride < 0) return SD_ERR_INVALID_VALUE;
  if (row_stride > (1ll << 40) || col_stride > (1ll << 31)) return SD_ERR_OVERFLOW;
  if (out->rows == 0 || out->cols == 0) return SD_OK;
  if (!x || !aligned_to(x, type_bytes(type))) return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? pack_any<float>(x, row_stride, col_stride, out, s)
         : type == SD_TYPE_F16 ? pack_any<f16>(x, row_stride, col_stride, out, s)
                               : pack_any<bf16>(x, row_stride, col_stride, out, s);
}

extern "C" int sd_unpack(const sd_packed_t *x, void *y, int32_t type, int64_t row_stride, void *stream) {
  int st = check_packed(x);
  if (st != SD_OK) return st;
  if ((st = check_table(y, type, x->rows, x->cols, row_stride)) != SD_OK) return st;
  if (x->rows == 0 || x->cols == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? unpack_as<float>(x, y, row_stride, s)
         : type == SD_TYPE_F16 ? unpack_as<f16>(x, y, row_stride, s)
                               : unpack_as<bf16>(x, y, row_stride, s);
}
