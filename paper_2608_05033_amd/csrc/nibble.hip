// sd_nibble_pack / sd_nibble_unpack: dense tables to 4 bits and back.
//
// value(r, c) = e2m1(code(r, c)) * 2^(s(c / 32, r) - 127).  The scale of a row's
// block of 32 columns is the least power of two that brings its largest magnitude
// to at most 6, the format's largest number, so nothing is cut off and both
// directions are exact up to the one rounding (nearest, ties to even).  The format
// has no NaN and no infinity of its own: a block that holds one gets the scale
// byte 255, which makes all of it NaN here and in the matrix units.
#include "nibble.h"

namespace {

using namespace nibble;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // row groups in flight per lane group

// V elements of a row, of which `left` lie inside the table; all or none where rows are
// EVEN, of whole spans.  Else a row's end is read with what lies behind it where the
// next row does; the last row's element by element, and a table's of rows so close or
// few that V elements from its first pass its end.  What is asked for (`ask`, of many
// rows in a row) is converted and cut off (`take`) later: done at once, each row waited
// for its own.
template <typename T, bool EVEN>
struct Ends {
  static constexpr int V = 16 / sizeof(T);
  const T *x;
  int64_t row_stride, rows;
  int32_t cols;
  struct Some {
    Span<T, V> span;
    const T *p;
    int left;
    bool whole;
  };
  __device__ inline bool any_whole() const { return cols >= V || (rows > 1 && row_stride >= V); }
  __device__ inline Some ask(int64_t row, int32_t c) const {
    Some o;
    o.p = x + row * row_stride + c;
    o.left = row < rows ? cols - c : 0;
    o.span = Span<T, V>{};
    if constexpr (EVEN) {
      if (o.left > 0) o.span = *reinterpret_cast<const Span<T, V> *>(o.p);
      return o;
    }
    o.whole = o.left >= V || (o.left > 0 && row + 1 < rows && row_stride >= V);
    if (any_whole()) o.span = *reinterpret_cast<const Span<T, V> *>(o.whole ? o.p : x);
    return o;
  }
  __device__ inline void take(const Some &o, float (&v)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = EVEN || i < o.left ? (float)o.span.v[i] : 0.0f;
    if (!EVEN && o.left > 0 && !o.whole) load_part(o.p, o.left, v);
  }
};

// A group of WIDE / V lanes takes one row's group of 128 columns, of which there are
// at most WIDE: V neighbouring columns per lane (16 bytes), the largest bits of each
// block over its 32 / V lanes, V codes per lane back.  Bound by the bytes, four groups
// in flight: 262144 x 128 fp32 take 24 us, 6.3 TB/s of bytes that the 256 MB Infinity
// Cache partly serves; 563394 x 127 bf16 35.  COLS: consecutive elements of a row lie together (else any
// strides, each lane's elements read one by one).
template <typename T, int WIDE, bool COLS, bool EVEN>
__global__ __launch_bounds__(kThreads) void k_nibble_pack(const T *__restrict__ x, int64_t row_stride,
                                                          int64_t col_stride, int64_t rows, int32_t cols, int32_t ng,
                                                          uint8_t *__restrict__ codes, int64_t ld,
                                                          uint8_t *__restrict__ scales) {
  constexpr int V = 16 / sizeof(T), LANES = WIDE / V, GROUPS = kThreads / LANES, SHARE = kCols / V;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int64_t first = (int64_t)workgroup() * (GROUPS * kUnroll);
  const int64_t r0 = first / ng;
  const uint32_t g0 = (uint32_t)(first - r0 * ng);
  const Ends<T, EVEN> ends{x, row_stride, rows, cols};
  typename Ends<T, EVEN>::Some some[kUnroll];
  float v[kUnroll][V];
  int64_t row[kUnroll];
  int32_t grp[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t at = g0 + u * GROUPS + group;
    row[u] = r0 + at / (uint32_t)ng;
    grp[u] = at % (uint32_t)ng;
    const int32_t c = grp[u] * kGroup + lane * V;
    if constexpr (COLS) {
      some[u] = ends.ask(row[u], c);
    } else {
      const int left = row[u] < rows ? cols - c : 0;
      const T *p = x + row[u] * row_stride + c * col_stride;
#pragma unroll
      for (int i = 0; i < V; ++i) v[u][i] = i < left ? (float)p[i * col_stride] : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if constexpr (COLS) ends.take(some[u], v[u]);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t bits = __float_as_uint(v[u][i]) & 0x7fffffffu;
      most = most > bits ? most : bits;
    }
    const uint32_t s = scale_byte(group_max_bits(most, SHARE));
    const float scale = scale_value(s);
    uint32_t w = encode2<0>(0u, v[u][0], v[u][1], scale);
    w = encode2<1>(w, v[u][2], v[u][3], scale);
    if constexpr (V == 8) {
      w = encode2<2>(w, v[u][4], v[u][5], scale);
      w = encode2<3>(w, v[u][6], v[u][7], scale);
    }
    if (s == kNanScale) w = 0;
    if (row[u] >= rows) continue;
    const int32_t c = grp[u] * kGroup + lane * V;
    if (c < ((cols + kCols - 1) & ~(kCols - 1))) {
      uint8_t *p = codes + row[u] * ld + c / 2;
      if constexpr (V == 4)
        *reinterpret_cast<uint16_t *>(p) = (uint16_t)w;
      else
        *reinterpret_cast<uint32_t *>(p) = w;
    }
    if (lane % SHARE == 0) {
      uint8_t *p = scales + ((int64_t)grp[u] * rows + row[u]) * 4;
      if constexpr (WIDE == 32) {
        *reinterpret_cast<uint32_t *>(p) = s | 0x7f7f7f00u;
      } else {
        p[lane / SHARE] = (uint8_t)s;
        if constexpr (WIDE == 64) p[2 + lane / SHARE] = 127;
      }
    }
  }
}

// The same where consecutive rows lie closer than consecutive columns (a
// transposed table): lanes along the rows, a whole block for each lane, the four
// blocks of a group for the four waves.  Bound by the bytes: 2^18 x 256 fp32 take
// 55 us, 5.5 TB/s; with groups of a row spread over the XCDs, which then each write
// parts of its lines, 74.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_nibble_pack_across(const T *__restrict__ x, int64_t row_stride,
                                                                 int64_t col_stride, int64_t rows, int32_t cols,
                                                                 int32_t ng, uint8_t *__restrict__ codes, int64_t ld,
                                                                 uint8_t *__restrict__ scales, uint32_t wgs) {
  if (workgroup() >= wgs) return;
  // neighbouring groups of a row share lines, and run on one XCD
  const uint32_t at = xcd_place(workgroup(), wgs);
  const int64_t strip = at / (uint32_t)ng;
  const int32_t grp = at % (uint32_t)ng;
  const int block = threadIdx.x >> 6;
  const int64_t row = strip * 64 + (threadIdx.x & 63);
  if (row >= rows) return;
  const int32_t c = grp * kGroup + block * kCols;
  const int left = cols - c;
  float v[kCols];
  const T *p = x + row * row_stride + c * col_stride;
  if (left >= kCols) {
#pragma unroll
    for (int i = 0; i < kCols; ++i) v[i] = (float)p[i * col_stride];
  } else {
#pragma unroll
    for (int i = 0; i < kCols; ++i) v[i] = i < left ? (float)p[i * col_stride] : 0.0f;
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kCols; ++i) {
    const uint32_t bits = __float_as_uint(v[i]) & 0x7fffffffu;
    most = most > bits ? most : bits;
  }
  const uint32_t s = scale_byte(most);
  const float scale = scale_value(s);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t q = encode2<0>(0u, v[8 * i], v[8 * i + 1], scale);
    q = encode2<1>(q, v[8 * i + 2], v[8 * i + 3], scale);
    q = encode2<2>(q, v[8 * i + 4], v[8 * i + 5], scale);
    q = encode2<3>(q, v[8 * i + 6], v[8 * i + 7], scale);
    w[i] = s == kNanScale ? 0 : q;
  }
  if (left > 0) *reinterpret_cast<u32x4 *>(codes + row * ld + c / 2) = w;
  scales[((int64_t)grp * rows + row) * 4 + block] = (uint8_t)s;
}

// A table and its transpose from one reading, of consecutive elements in a row.
// A workgroup takes 128 rows x 128 columns, a wave 32 of the rows: it packs them along
// the columns as k_nibble_pack does, leaves them in shared memory and takes them
// column by column, so that a lane has a block of the transpose.  The four waves'
// blocks of a column leave together, 64 bytes of codes and a word of scales.  Bound by
// the bytes, two workgroups a compute unit for fp32: 2^18 x 256 take 71 us with calls in
// a row, 4.8 TB/s, where the two ways one after the other take 102; in a training step,
// behind other tables, 85.
template <typename T, bool EVEN>
__global__ __launch_bounds__(kThreads) void k_nibble_pack_both(const T *__restrict__ x, int64_t row_stride,
                                                               int64_t rows, int32_t cols, int32_t ng,
                                                               uint8_t *__restrict__ codes, int64_t ld,
                                                               uint8_t *__restrict__ scales,
                                                               uint8_t *__restrict__ codes_t, int64_t ld_t,
                                                               uint8_t *__restrict__ scales_t, uint32_t strips,
                                                               uint32_t wgs) {
  constexpr int V = 16 / sizeof(T), LANES = kGroup / V, SHARE = kCols / V, AT_ONCE = 64 / LANES, STEPS = 32 / AT_ONCE;
  // by whole words: an odd number of them between rows, so that neither way of reading meets itself
  constexpr int PITCH = kGroup + 4 / (int)sizeof(T);
  __shared__ __align__(16) T tile[4][32 * PITCH];
  __shared__ __align__(16) u32x4 blocks[4][kGroup];
  __shared__ __align__(4) uint8_t bytes[kGroup][4];  // read as words
  const int t = threadIdx.x, wave = t >> 6, l = t & 63, lane = l % LANES, down = l / LANES;
  if (workgroup() >= wgs) return;
  // neighbouring strips share lines of the transpose, and run on one XCD
  const uint32_t at = xcd_place(workgroup(), wgs);
  const int64_t strip = at % strips, row0 = strip * 128 + wave * 32;
  const int32_t grp = at / strips;
  const int32_t c = grp * kGroup + lane * V;
  const Ends<T, EVEN> ends{x, row_stride, rows, cols};
  typename Ends<T, EVEN>::Some some[STEPS];
#pragma unroll
  for (int u = 0; u < STEPS; ++u) some[u] = ends.ask(row0 + u * AT_ONCE + down, c);
#pragma unroll
  for (int u = 0; u < STEPS; ++u) {
    const int64_t row = row0 + u * AT_ONCE + down;
    float v[V];
    ends.take(some[u], v);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t bits = __float_as_uint(v[i]) & 0x7fffffffu;
      most = most > bits ? most : bits;
    }
    const uint32_t s = scale_byte(group_max_bits(most, SHARE));
    const float scale = scale_value(s);
    uint32_t w = encode2<0>(0u, v[0], v[1], scale);
    w = encode2<1>(w, v[2], v[3], scale);
    if constexpr (V == 8) {
      w = encode2<2>(w, v[4], v[5], scale);
      w = encode2<3>(w, v[6], v[7], scale);
    }
    if (s == kNanScale) w = 0;
    T *q = &tile[wave][(u * AT_ONCE + down) * PITCH + lane * V];
#pragma unroll
    for (int i = 0; i < V; ++i) q[i] = (T)v[i];
    if (row < rows) {
      if (c < ((cols + kCols - 1) & ~(kCols - 1))) {
        uint8_t *o = codes + row * ld + c / 2;
        if constexpr (V == 4)
          *reinterpret_cast<uint16_t *>(o) = (uint16_t)w;
        else
          *reinterpret_cast<uint32_t *>(o) = w;
      }
      if (lane % SHARE == 0) scales[((int64_t)grp * rows + row) * 4 + lane / SHARE] = (uint8_t)s;
    }
  }
  wave_order();  // the lanes' rows, before others read them
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // column h * 64 + l of the wave's 32 rows
    float d[kCols];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      d[i] = (float)tile[wave][i * PITCH + h * 64 + l];
      const uint32_t bits = __float_as_uint(d[i]) & 0x7fffffffu;
      most = most > bits ? most : bits;
    }
    const uint32_t s = scale_byte(most);
    const float scale = scale_value(s);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t q = encode2<0>(0u, d[8 * i], d[8 * i + 1], scale);
      q = encode2<1>(q, d[8 * i + 2], d[8 * i + 3], scale);
      q = encode2<2>(q, d[8 * i + 4], d[8 * i + 5], scale);
      q = encode2<3>(q, d[8 * i + 6], d[8 * i + 7], scale);
      w[i] = s == kNanScale ? 0 : q;
    }
    blocks[wave][h * 64 + l] = w;
    bytes[h * 64 + l][wave] = (uint8_t)s;
  }
  __syncthreads();
  // blocks of 32 rows that there are; four threads a column
  const int64_t have = (rows - strip * 128 + 31) / 32;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int column = h * 64 + t / 4, part = t & 3;
    const int64_t col = (int64_t)grp * kGroup + column;
    if (col < cols && part < have)
      *reinterpret_cast<u32x4 *>(codes_t + col * ld_t + strip * 64 + part * 16) = blocks[part][column];
  }
  const int64_t col = (int64_t)grp * kGroup + t;
  if (t < kGroup && col < cols)
    *reinterpret_cast<uint32_t *>(scales_t + (strip * cols + col) * 4) = *reinterpret_cast<const uint32_t *>(bytes[t]);
}

// Lanes along a row, eight codes each.  Bound by the bytes written: 262144 x 128 to
// bf16 take 14 us, 6 TB/s of bytes that the caches partly serve.  END 1: a row's last lane begins eight columns before its
// end, so that all write whole spans; its codes lie in two words and may lie in two
// blocks.  END 2: rows of fewer than eight columns.
template <typename T, int END>
__global__ __launch_bounds__(kThreads) void k_nibble_unpack(const uint8_t *__restrict__ codes, int64_t ld,
                                                            const uint8_t *__restrict__ scales, int64_t rows,
                                                            int32_t cols, int32_t octs, T *__restrict__ y,
                                                            int64_t row_stride) {
  const int64_t first = (int64_t)workgroup() * (kThreads * kUnroll);
  const int64_t r0 = first / octs;
  const uint32_t q0 = (uint32_t)(first - r0 * octs);
  uint32_t w[kUnroll], w1[kUnroll], s[kUnroll], s1[kUnroll];
  int64_t row[kUnroll];
  int32_t col[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t at = q0 + u * kThreads + threadIdx.x;
    row[u] = r0 + at / (uint32_t)octs;
    col[u] = (int32_t)(at % (uint32_t)octs) * 8;
    if (END == 1 && col[u] > cols - 8) col[u] = cols - 8;
    w[u] = w1[u] = 0;
    s[u] = s1[u] = 127;
    if (row[u] < rows) {
      const uint8_t *p = codes + row[u] * ld;
      const auto scale_at = [&](int32_t c) {
        return (uint32_t)scales[((int64_t)(c / kGroup) * rows + row[u]) * 4 + c / kCols % 4];
      };
      w[u] = *reinterpret_cast<const uint32_t *>(p + col[u] / 8 * 4);
      s[u] = scale_at(col[u]);
      if constexpr (END == 1) {
        w1[u] = *reinterpret_cast<const uint32_t *>(p + (col[u] + 7) / 8 * 4);
        s1[u] = scale_at(col[u] + 7);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (row[u] >= rows) continue;
    const auto value_of = [](uint32_t b) {
      return b == kNanScale ? __uint_as_float(0x7fc00000u) : scale_value(b);
    };
    const float scale = value_of(s[u]);
    uint32_t codes8 = w[u];
    if constexpr (END == 1)
      codes8 = (uint32_t)((((uint64_t)w1[u] << 32) | w[u]) >> (4 * (col[u] & 7)));
    float v[8];
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes8, 1.0f, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes8, 1.0f, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes8, 1.0f, 2);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes8, 1.0f, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
    if constexpr (END == 1) {
      const float scale1 = value_of(s1[u]);
      const int turn = kCols - (col[u] & (kCols - 1));  // the first of the next block
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= i < turn ? scale : scale1;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= scale;
    }
    T *p = y + row[u] * row_stride + col[u];
    if constexpr (END == 2)
      store_part(p, cols, v);
    else
      store_span(p, v);
  }
}

template <typename T, bool COLS, bool EVEN>
auto pack_kernel(int wide) {
  return wide == 32   ? k_nibble_pack<T, 32, COLS, EVEN>
         : wide == 64 ? k_nibble_pack<T, 64, COLS, EVEN>
                      : k_nibble_pack<T, 128, COLS, EVEN>;
}

template <typename T>
int pack_any(const void *x, int64_t row_stride, int64_t col_stride, const sd_nibble_t *out, hipStream_t s) {
  const T *p = static_cast<const T *>(x);
  const int64_t ng = groups_of(out->cols);
  const bool across = col_stride != 1 && row_stride < col_stride;
  const int wide = out->cols <= 32 ? 32 : out->cols <= 64 ? 64 : 128;
  const int64_t per_wg = kThreads / (wide * (int)sizeof(T) / 16) * kUnroll;
  const int64_t wgs = across ? ceil_div(out->rows, 64) * ng : ceil_div(out->rows * ng, per_wg);
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  if (across) {
    hipLaunchKernelGGL(k_nibble_pack_across<T>, grid_of(wgs), dim3(kThreads), 0, s, p, row_stride, col_stride,
                       out->rows, (int32_t)out->cols, (int32_t)ng, out->codes, out->ld, out->scales, (uint32_t)wgs);
    return launched();
  }
  const bool even = out->cols % (16 / sizeof(T)) == 0;
  auto *kernel = col_stride != 1 ? pack_kernel<T, false, false>(wide)
                 : even          ? pack_kernel<T, true, true>(wide)
                                 : pack_kernel<T, true, false>(wide);
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, p, row_stride, col_stride, out->rows,
                     (int32_t)out->cols, (int32_t)ng, out->codes, out->ld, out->scales);
  return launched();
}

template <typename T>
int both_any(const void *x, int64_t row_stride, const sd_nibble_t *out, const sd_nibble_t *out_t, hipStream_t s) {
  const int64_t ng = groups_of(out->cols), wgs = ceil_div(out->rows, 128) * ng;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  auto *kernel = out->cols % (16 / sizeof(T)) == 0 ? k_nibble_pack_both<T, true> : k_nibble_pack_both<T, false>;
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, static_cast<const T *>(x), row_stride, out->rows,
                     (int32_t)out->cols, (int32_t)ng, out->codes, out->ld, out->scales, out_t->codes, out_t->ld,
                     out_t->scales, (uint32_t)(wgs / ng), (uint32_t)wgs);
  return launched();
}

template <typename T>
int unpack_as(const sd_nibble_t *x, void *y, int64_t row_stride, hipStream_t s) {
  const int64_t octs = ceil_div(x->cols, 8), wgs = ceil_div(x->rows * octs, kThreads * kUnroll);
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  auto *kernel = x->cols % 8 == 0 ? k_nibble_unpack<T, 0> : x->cols > 8 ? k_nibble_unpack<T, 1> : k_nibble_unpack<T, 2>;
  hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(kThreads), 0, s, x->codes, x->ld, x->scales, x->rows,
                     (int32_t)x->cols, (int32_t)octs, static_cast<T *>(y), row_stride);
  return launched();
}

}  // namespace

extern "C" int sd_nibble_pack(const void *x, int32_t type, int64_t row_stride, int64_t col_stride,
                              const sd_nibble_t *out, void *stream) {
  int st = check_nibble(out);
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

extern "C" int sd_nibble_pack_both(const void *x, int32_t type, int64_t row_stride, int64_t col_stride,
                                   const sd_nibble_t *out, const sd_nibble_t *out_t, void *stream) {
  int st = check_nibble(out);
  if (st == SD_OK) st = check_nibble(out_t);
  if (st == SD_OK && (out_t->rows != out->cols || out_t->cols != out->rows)) st = SD_ERR_INVALID_VALUE;
  if (st != SD_OK) return st;
  if (row_stride > (1ll << 31)) return SD_ERR_OVERFLOW;
  // One after the other where rows fill little of k_nibble_pack_both's 128 columns and the second launch does
  // not count: 500000 x 50 fp32 take 43 us so and 67 at once, 1000000 x 64 bf16 54 and 54, 516016 x 75 62 and 47.
  if (col_stride != 1 || (out->cols <= 64 && out->rows >= (1 << 17))) {
    st = sd_nibble_pack(x, type, row_stride, col_stride, out, stream);
    return st == SD_OK ? sd_nibble_pack(x, type, col_stride, row_stride, out_t, stream) : st;
  }
  if (!type_ok(type) || row_stride < 0) return SD_ERR_INVALID_VALUE;
  if (out->rows == 0 || out->cols == 0) return SD_OK;
  if (!x || !aligned_to(x, type_bytes(type))) return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? both_any<float>(x, row_stride, out, out_t, s)
         : type == SD_TYPE_F16 ? both_any<f16>(x, row_stride, out, out_t, s)
                               : both_any<bf16>(x, row_stride, out, out_t, s);
}

extern "C" int sd_nibble_unpack(const sd_nibble_t *x, void *y, int32_t type, int64_t row_stride, void *stream) {
  int st = check_nibble(x);
  if (st != SD_OK) return st;
  if ((st = check_table(y, type, x->rows, x->cols, row_stride)) != SD_OK) return st;
  if (x->rows == 0 || x->cols == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? unpack_as<float>(x, y, row_stride, s)
         : type == SD_TYPE_F16 ? unpack_as<f16>(x, y, row_stride, s)
                               : unpack_as<bf16>(x, y, row_stride, s);
}
