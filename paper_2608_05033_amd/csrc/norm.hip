// sd_group_norm / sd_group_norm_backward: group norm with an activation over
// segments of rows, channels last.
//
//   xh = (x - mean) rstd, z = xh w + b, y = act(z), with mean and
//   rstd = (var + eps)^-1/2 over a segment's rows and a group's channels.
//   dz = dy act'(z), dh = dz w:
//   dx = rstd (dh - mean(dh) - xh mean(dh xh)), dw = sum dz xh, db = sum dz.
//
// Rows are cut into chunks of equal length whatever the segments are; a chunk's
// part of a segment is a piece, numbered chunk + segment (both only grow along
// the rows, so no two pieces share a number).  One kernel leaves sums per piece
// and channel, one joins them per segment and group in 64 bits, one applies the
// result, chunks in reverse so that what the first pass read last is still in
// the Infinity Cache.  Bound by the bytes moved: x is read twice and written once.
// 2400000 x 128 fp32, 8-bit copy kept: sums 208 us, apply 559 us (4.9 TB/s); backward
// 289 us and 561 us.
//
// Short segments take one launch instead: a team of threads holds a segment's
// rows in registers, adds them up in shared memory and applies the result.  100003
// rows of 96 bf16 in 3001 segments take 36 us: three workgroups fit a compute unit,
// so there are four rounds of some 9 us, each a chain of offsets, rows, two joins and
// the stores, which few waves hide.  37 rows of 64 fp32 take 6 us.
//
// Every sum has a fixed order: results do not change from run to run.
#include "dense.h"

namespace {

using namespace dense;

constexpr int kThreads = 256;
constexpr int V = 4;         // channels per lane
constexpr int kBatch = 4;    // rows of a lane in flight: 4 (backward sums) to 8 waves per SIMD fit the registers

// What every kernel needs of the call.
struct Shape {
  int64_t rows, segments, len;  // len: rows of each segment where offsets is null
  const int32_t *offsets;
  int32_t channels, groups, per_group;
  int32_t chunk_rows, chunks, tx, ty;
  int32_t share;   // lanes that add up one group's channels
  int32_t across;  // of a team's, those side by side on channels
  // A slab of tx * V channels leaves sums for the groups that it has a part of, at
  // group + slab of a piece's slots: both only grow along the channels.
  int32_t slots;
  // Short segments: teams of tx * ty threads, wgs workgroups; 0: chunks are used.
  int32_t wgs;
  bool one_row;  // each thread keeps one row of a segment, as many as the caller says there are
  float eps;
  const float *weight, *bias;
};

__device__ inline int64_t seg_begin(const Shape &p, int64_t s) { return p.offsets ? p.offsets[s] : s * p.len; }
// The segment that holds row r: the last one that begins at or before it.
__device__ inline int64_t seg_of(const Shape &p, int64_t r) {
  if (!p.offsets) return r / p.len;
  int64_t lo = 0, hi = p.segments;  // offsets[lo] <= r < offsets[hi]
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) >> 1;
    if (p.offsets[mid] <= r)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Rows [lo, hi) of segment s inside rows [r0, r1); calls f(s, lo, hi) for each
// segment that has some.
template <typename F>
__device__ inline void for_pieces(const Shape &p, int64_t r0, int64_t r1, F f) {
  for (int64_t s = seg_of(p, r0); s < p.segments; ++s) {
    const int64_t b = seg_begin(p, s), e = seg_begin(p, s + 1);
    if (b >= r1) break;
    const int64_t lo = b > r0 ? b : r0, hi = e < r1 ? e : r1;
    if (lo < hi) f(s, lo, hi);
  }
}

// This thread's rows of [lo, hi), every ty_count-th: f(row, count) for kBatch of
// them at a time (row, row + ty_count, ...) while all threads have that many, then
// one by one.
template <int N>
struct Count {
  static constexpr int value = N;
};
template <typename F>
__device__ inline void for_rows(int64_t lo, int64_t hi, int ty, int ty_count, F f) {
  int64_t r = lo;
  for (; r + ty_count * kBatch <= hi; r += ty_count * kBatch) f(r + ty, Count<kBatch>());
  for (r += ty; r < hi; r += ty_count) f(r, Count<1>());
}

// ---- where x comes from: dense rows, or 8-bit codes and their scales.  N rows
// from r on, `step` apart, V channels from c on; all of them are there.  Where
// channels come in whole vectors (`whole`, the same for all threads) the loads
// stand together without conditions; a lane past the last channel reads the
// first, for nothing. ----
template <typename T>
struct Dense {
  T *p;
  uint32_t stride;  // below 2^31, as rows are: one 32-bit product a row
  bool stream;      // written past the caches
  __device__ T *at(int64_t r) const { return p + (uint64_t)(uint32_t)r * stride; }
  template <int N>
  __device__ void load(int64_t r, int64_t step, int32_t c, int left, bool whole, float (&v)[N][V]) const {
    if (whole) {
      const T *q = at(r) + (left > 0 ? c : 0);
#pragma unroll
      for (int u = 0; u < N; ++u) load_span(q + u * step * stride, v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) load_part(at(r + u * step) + c, left, v[u]);
    }
  }
  // Rows past `last` read one before, for nothing.
  template <int N>
  __device__ void load_to(int64_t last, int64_t r, int64_t step, int32_t c, int left, bool whole,
                          float (&v)[N][V]) const {
    if (whole) {
      const T *q = at(r < last ? r : last) + (left > 0 ? c : 0);
#pragma unroll
      for (int u = 0; u < N; ++u) load_span(r + u * step <= last ? q + u * step * stride : q, v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) load_part(at(r + u * step < last ? r + u * step : last) + c, left, v[u]);
    }
  }
  template <int N>
  __device__ void store(int64_t r, int64_t step, int32_t c, int left, bool whole, const float (&v)[N][V]) const {
    T *q = at(r) + c;
    if (whole && stream) {
      if (left > 0)
#pragma unroll
        for (int u = 0; u < N; ++u) stream_span(q + u * step * stride, v[u]);
    } else if (whole) {
      if (left > 0)
#pragma unroll
        for (int u = 0; u < N; ++u) store_span(q + u * step * stride, v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) store_part(q + u * step * stride, left, v[u]);
    }
  }
};
template <int FMT>
struct Codes {
  const uint8_t *codes, *scales;
  int64_t ld, rows;
  template <int N>
  __device__ void load_to(int64_t last, int64_t r, int64_t step, int32_t c, int left, bool, float (&v)[N][V]) const {
    const int32_t at = left > 0 ? c : 0;  // codes are there up to a multiple of 16
    const uint8_t *q = codes + at, *sq = scales + (int64_t)(at / kBlock) * rows;
    uint32_t w[N], s[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t row = r + u * step < last ? r + u * step : last;
      w[u] = *reinterpret_cast<const uint32_t *>(q + row * ld);
      s[u] = sq[row];
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float f = scale_value(s[u]);
      decode4<FMT>(w[u], v[u]);
#pragma unroll
      for (int i = 0; i < V; ++i) v[u][i] *= f;
    }
  }
  template <int N>
  __device__ void load(int64_t r, int64_t step, int32_t c, int left, bool whole, float (&v)[N][V]) const {
    load_to(INT64_MAX, r, step, c, left, whole, v);
  }
};

// ---- activations; NaN stays NaN ----
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
// The normal distribution's tail beyond |z|, 0.5 erfc(|z| / sqrt 2), from its
// density e = exp(-z^2 / 2): Abramowitz and Stegun, Handbook of Mathematical
// Functions, 7.1.26, absolute error 1.5e-7 in erf.  A quarter of the operations
// of the library's erf, whose two ranges both run in a wave.
__device__ inline float normal_tail(float z, float e) {
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * 0.70710678f * fabsf(z));
  const float q = 0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f)));
  return 0.5f * t * q * e;
}
template <int ACT>
__device__ inline float act(float z) {
  if constexpr (ACT == SD_ACT_RELU) return z < 0.0f ? 0.0f : z;
  if constexpr (ACT == SD_ACT_SILU) return z * sigmoid(z);
  if constexpr (ACT == SD_ACT_GELU) {
    const float tail = normal_tail(z, __expf(-0.5f * z * z));
    return z * (z < 0.0f ? tail : 1.0f - tail);
  }
  return z;
}
template <int ACT>
__device__ inline float act_slope(float z) {
  if constexpr (ACT == SD_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
  if constexpr (ACT == SD_ACT_SILU) {
    const float s = sigmoid(z);
    return s * (1.0f + z * (1.0f - s));
  }
  if constexpr (ACT == SD_ACT_GELU) {
    const float e = __expf(-0.5f * z * z), tail = normal_tail(z, e);
    return (z < 0.0f ? tail : 1.0f - tail) + z * e * 0.39894228f;
  }
  return 1.0f;
}

// ------------------------------------------------------------- forward -----
// What the numbers of a segment and group are counted from: the first of them
// (0 where that is not finite).  Its distance from the mean is no more than
// sqrt(n) deviations, so the variance, a difference of sums counted from here,
// keeps n 2^-53 of itself however large the mean is, and is 0 where all n
// numbers are the same.
template <typename T>
__device__ inline float origin_of(const Shape &p, const Dense<const T> &x, int64_t first_row, int32_t first_channel) {
  const int64_t row = first_row < 0 ? 0 : first_row < p.rows ? first_row : p.rows - 1;
  const float v = (float)x.at(row)[first_channel];
  return fabsf(v) < __builtin_inff() ? v : 0.0f;
}
// Of a lane's channels, whose groups begin at `first`; one where they share a group.
template <typename T>
__device__ inline void origins_of(const Shape &p, const Dense<const T> &x, int64_t first_row, const int32_t (&first)[V],
                                  float (&k)[V]) {
  if (p.per_group % V == 0) {  // the same for all threads
    const float v = origin_of(p, x, first_row, first[0]);
#pragma unroll
    for (int i = 0; i < V; ++i) k[i] = v;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) k[i] = origin_of(p, x, first_row, first[i]);
  }
}

// Per piece and group: the sums of x and x^2, counted from the segment's origin, in
// 64 bits.  The three 64-bit operations per element take less time than loading it.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_stats(Shape p, Dense<const T> x, double2 *__restrict__ part) {
  __shared__ double2 s_sum[kThreads][V];
  const int tx = threadIdx.x % p.tx, ty = threadIdx.x / p.tx, TY = p.ty;
  const int32_t c = (blockIdx.y * p.tx + tx) * V;
  const int left = p.channels - c;
  const bool whole = p.channels % V == 0;
  const int64_t r0 = (int64_t)blockIdx.x * p.chunk_rows;
  const int64_t r1 = r0 + p.chunk_rows < p.rows ? r0 + p.chunk_rows : p.rows;
  int32_t group_first[V];
#pragma unroll
  for (int i = 0; i < V; ++i) group_first[i] = i < left ? (c + i) / p.per_group * p.per_group : 0;
  for_pieces(p, r0, r1, [&](int64_t s, int64_t lo, int64_t hi) {
    double a[V] = {}, b[V] = {};
    float origin[V];
    origins_of(p, x, seg_begin(p, s), group_first, origin);
    for_rows(lo, hi, ty, TY, [&](int64_t row, auto count) {
      constexpr int N = decltype(count)::value;
      float v[N][V];
      x.load(row, TY, c, left, whole, v);
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const double d = (double)v[u][i] - (double)origin[i];
          a[i] += d;
          b[i] = fma(d, d, b[i]);
        }
    });
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[t][i] = double2{a[i], b[i]};
    __syncthreads();
    for (int h = TY / 2; h > 0; h /= 2) {
      if (ty < h) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const double2 o = s_sum[t + h * p.tx][i];
          s_sum[t][i] = double2{a[i] += o.x, b[i] += o.y};
        }
      }
      __syncthreads();
    }
    // s_sum[0 .. tx) holds the slab's channels in order; a few lanes per group add them up
    double2 *out = part + (blockIdx.x + s) * p.slots;
    const double2 *in = &s_sum[0][0];
    const int32_t first = blockIdx.y * p.tx * V, last = p.channels - first < p.tx * V ? p.channels : first + p.tx * V;
    const int32_t g0 = first / p.per_group, g1 = (last - 1) / p.per_group;
    for (int32_t k = t / p.share; k <= g1 - g0; k += blockDim.x / p.share) {
      const int32_t lo_c = (g0 + k) * p.per_group, hi_c = lo_c + p.per_group;
      const int32_t from = lo_c > first ? lo_c : first, to = hi_c < last ? hi_c : last;
      double sum = 0, square = 0;
      for (int32_t q = from + t % p.share; q < to; q += p.share) {
        sum += in[q - first].x;
        square += in[q - first].y;
      }
      for (int d = 1; d < p.share; d *= 2) {
        sum += __shfl_xor(sum, d);
        square += __shfl_xor(square, d);
      }
      if (t % p.share == 0) out[g0 + k + blockIdx.y] = double2{sum, square};
    }
    __syncthreads();
  });
}

// Sum over the workgroup's threads, the same in every thread.
__device__ inline double wg_sum(double v, double *lds) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  if (blockDim.x == 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0;
  for (uint32_t w = 0; w < blockDim.x / 64; ++w) t += lds[w];
  return t;
}

// From sums counted from `origin`; one: 1 over the count.  The variance and eps are
// rounded to 32 bits once they are added, over an even power of two: numbers of 2^64
// and more, and of 2^-64 and less, have variances past that range, and rstd fits it.
__device__ inline void write_stats(const Shape &p, double sum, double square, double one, float origin, float *mean,
                                   float *rstd) {
  const double mu = sum * one, var = square * one - mu * mu;
  *mean = (float)((double)origin + mu);
  const double v = (var < 0.0 ? 0.0 : var) + (double)p.eps;
  const int half = __builtin_amdgcn_frexp_exp(v) >> 1;  // 0 for 0, infinity and NaN
  *rstd = __builtin_ldexpf(1.0f / sqrtf((float)__builtin_ldexp(v, -2 * half)), -half);
}

// The chunks that hold rows [b, e).
__device__ inline bool chunks_of(const Shape &p, int64_t b, int64_t e, int64_t *c0, int64_t *c1) {
  if (e <= b) return false;
  *c0 = b / p.chunk_rows;
  *c1 = (e - 1) / p.chunk_rows;
  *c0 = *c0 < 0 ? 0 : *c0;
  *c1 = *c1 >= p.chunks ? p.chunks - 1 : *c1;
  return *c0 <= *c1;
}

template <typename T>
__global__ void k_norm_join(Shape p, Dense<const T> x, const double2 *__restrict__ part, float *__restrict__ mean,
                            float *__restrict__ rstd) {
  __shared__ double lds[16];
  const int32_t slab = p.tx * V;
  for (int64_t at = blockIdx.x; at < p.segments * p.groups; at += gridDim.x) {
    const int64_t s = at / p.groups;
    const int32_t g = (int32_t)(at - s * p.groups);
    const int64_t b = seg_begin(p, s), e = seg_begin(p, s + 1);
    const int32_t k0 = g + g * p.per_group / slab, k1 = g + ((g + 1) * p.per_group - 1) / slab;
    double sum = 0, square = 0;
    float origin = 0.0f;
    int64_t c0, c1;
    if (chunks_of(p, b, e, &c0, &c1)) {
      origin = origin_of(p, x, b, g * p.per_group);
#pragma unroll 4
      for (int64_t c = c0 + threadIdx.x; c <= c1; c += blockDim.x)
        for (int32_t k = k0; k <= k1; ++k) {
          const double2 v = part[(c + s) * p.slots + k];
          sum += v.x;
          square += v.y;
        }
    }
    sum = wg_sum(sum, lds);
    square = wg_sum(square, lds);
    if (threadIdx.x == 0)
      write_stats(p, sum, square, 1.0 / (e > b ? (double)(e - b) * p.per_group : 1.0), origin, mean + at, rstd + at);
    __syncthreads();
  }
}

// Where a kernel writes 8-bit copies; codes is null where it does not.
struct Packs {
  uint8_t *codes, *scales;
  int64_t ld;
};
template <int FMT>
__device__ inline void store_packed(const Packs &o, int64_t rows, int64_t r, int32_t c, int32_t channels, int tx,
                                    int width, const float (&v)[V]) {
  const uint32_t most = largest_finite(v, channels - c, width);
  const uint32_t s = scale_byte<FMT>(most);
  const float inv = inverse_scale(s);
  if (c < ((channels + 15) & ~15)) {
    float u[V];
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = c + i < channels ? v[i] * inv : 0.0f;
    *reinterpret_cast<uint32_t *>(o.codes + r * o.ld + c) = encode4<FMT>(u[0], u[1], u[2], u[3]);
  }
  if (tx % (kBlock / V) == 0 && c < channels) o.scales[(int64_t)(c / kBlock) * rows + r] = (uint8_t)s;
}

// Mean, rstd * weight and bias of a lane's channels.
struct Coeff {
  float mean[V], scale[V], shift[V];
};
__device__ inline void load_coeff(const Shape &p, const float *mean, const float *rstd, int64_t s, int32_t c, int left,
                                  Coeff &k, float (&rs)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (i < left) {
      const int64_t g = s * p.groups + (c + i) / p.per_group;
      rs[i] = rstd[g];
      k.mean[i] = mean[g];
      k.scale[i] = rs[i] * (p.weight ? p.weight[c + i] : 1.0f);
      k.shift[i] = p.bias ? p.bias[c + i] : 0.0f;
    } else {
      rs[i] = k.mean[i] = k.scale[i] = k.shift[i] = 0.0f;
    }
  }
}

template <typename T, int ACT, int XF, int YF>
__global__ __launch_bounds__(kThreads) void k_norm_apply(Shape p, Dense<const T> x, const float *__restrict__ mean,
                                                         const float *__restrict__ rstd, Dense<T> y, Packs xo,
                                                         Packs yo) {
  const int tx = threadIdx.x % p.tx, ty = threadIdx.x / p.tx, TY = p.ty;
  const int32_t c = (blockIdx.y * p.tx + tx) * V;
  const int left = p.channels - c;
  const bool whole = p.channels % V == 0;
  const int width = p.tx < kBlock / V ? p.tx : kBlock / V;
  const int64_t r0 = (int64_t)(p.chunks - 1 - blockIdx.x) * p.chunk_rows;
  const int64_t r1 = r0 + p.chunk_rows < p.rows ? r0 + p.chunk_rows : p.rows;
  for_pieces(p, r0, r1, [&](int64_t s, int64_t lo, int64_t hi) {
    Coeff k;
    float rs[V];
    load_coeff(p, mean, rstd, s, c, left, k, rs);
    // the lanes of a row take its last rows together: they share its 8-bit scale
    for_rows(lo, hi, ty, TY, [&](int64_t row, auto count) {
      constexpr int N = decltype(count)::value;
      float v[N][V];
      x.load(row, TY, c, left, whole, v);
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int64_t at = row + u * TY;
        if constexpr (XF != 0) store_packed<XF>(xo, p.rows, at, c, p.channels, tx, width, v[u]);
#pragma unroll
        for (int i = 0; i < V; ++i) v[u][i] = act<ACT>((v[u][i] - k.mean[i]) * k.scale[i] + k.shift[i]);
        if constexpr (YF != 0) store_packed<YF>(yo, p.rows, at, c, p.channels, tx, width, v[u]);
      }
      if (y.p) y.store(row, TY, c, left, whole, v);
    });
  });
}

// ------------------------------------------------------------ backward -----
// Per piece and channel, and per chunk and channel: sums of dz and dz xh.
template <typename T, typename X, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_sums(Shape p, X x, Dense<const T> dy, const float *__restrict__ mean,
                                                        const float *__restrict__ rstd, float *__restrict__ part,
                                                        float *__restrict__ total) {
  __shared__ float s_a[kThreads][V], s_b[kThreads][V];
  const int tx = threadIdx.x % p.tx, ty = threadIdx.x / p.tx, TY = p.ty;
  const int32_t c = (blockIdx.y * p.tx + tx) * V;
  const int left = p.channels - c;
  const bool whole = p.channels % V == 0;
  const int64_t r0 = (int64_t)blockIdx.x * p.chunk_rows;
  const int64_t r1 = r0 + p.chunk_rows < p.rows ? r0 + p.chunk_rows : p.rows;
  float ta[V] = {}, tb[V] = {};
  // sums over the workgroup's rows into the threads of ty = 0
  auto reduce = [&](float (&a)[V], float (&b)[V]) {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s_a[t][i] = a[i];
      s_b[t][i] = b[i];
    }
    __syncthreads();
    for (int h = TY / 2; h > 0; h /= 2) {
      if (ty < h) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s_a[t][i] = a[i] += s_a[t + h * p.tx][i];
          s_b[t][i] = b[i] += s_b[t + h * p.tx][i];
        }
      }
      __syncthreads();
    }
  };
  auto write = [&](float *o, const float (&a)[V], const float (&b)[V]) {
    if (ty != 0 || left <= 0) return;
    if (left >= V) {
      store_span(o, a);
      store_span(o + p.channels, b);
    } else {
      store_part(o, left, a);
      store_part(o + p.channels, left, b);
    }
  };
  for_pieces(p, r0, r1, [&](int64_t s, int64_t lo, int64_t hi) {
    Coeff k;
    float rs[V];
    load_coeff(p, mean, rstd, s, c, left, k, rs);
    float a[V] = {}, b[V] = {};
    for_rows(lo, hi, ty, TY, [&](int64_t row, auto count) {
      constexpr int N = decltype(count)::value;
      float xv[N][V], dv[N][V];
      x.load(row, TY, c, left, whole, xv);
      dy.load(row, TY, c, left, whole, dv);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float sa = 0.0f, sb = 0.0f;  // a batch by itself: fewer additions on the way to the sum
#pragma unroll
        for (int u = 0; u < N; ++u) {
          const float d = xv[u][i] - k.mean[i];
          const float dz = dv[u][i] * act_slope<ACT>(d * k.scale[i] + k.shift[i]);
          sa += dz;
          sb += dz * (d * rs[i]);
        }
        a[i] += sa;
        b[i] += sb;
      }
    });
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ta[i] += a[i];
      tb[i] += b[i];
    }
    reduce(a, b);
    write(part + (blockIdx.x + s) * 2 * (int64_t)p.channels + c, a, b);
  });
  reduce(ta, tb);
  write(total + (int64_t)blockIdx.x * 2 * p.channels + c, ta, tb);
}

// Workgroups [0, joins): mean(dh) and mean(dh xh) per segment and group; the
// others: dweight and dbias of kJoinCols channels over all chunks.
constexpr int kJoinCols = 8;
__global__ void k_norm_join_back(Shape p, int32_t joins, const float *__restrict__ part,
                                 const float *__restrict__ total, float *__restrict__ m1, float *__restrict__ m2,
                                 float *__restrict__ dweight, float *__restrict__ dbias) {
  __shared__ double lds[16];
  __shared__ double s_a[1024], s_b[1024];
  if ((int32_t)blockIdx.x >= joins) {
    const int lane = threadIdx.x % kJoinCols, row = threadIdx.x / kJoinCols, step = blockDim.x / kJoinCols;
    const int32_t c = (blockIdx.x - joins) * kJoinCols + lane;
    double a = 0, b = 0;
    if (c < p.channels) {
#pragma unroll 8
      for (int32_t k = row; k < p.chunks; k += step) {
        a += total[(int64_t)k * 2 * p.channels + c];
        b += total[((int64_t)k * 2 + 1) * p.channels + c];
      }
    }
    s_a[threadIdx.x] = a;
    s_b[threadIdx.x] = b;
    __syncthreads();
    for (int h = step / 2; h > 0; h /= 2) {
      if (row < h) {
        s_a[threadIdx.x] += s_a[threadIdx.x + h * kJoinCols];
        s_b[threadIdx.x] += s_b[threadIdx.x + h * kJoinCols];
      }
      __syncthreads();
    }
    if (row == 0 && c < p.channels) {
      if (dbias) dbias[c] = (float)s_a[threadIdx.x];
      if (dweight) dweight[c] = (float)s_b[threadIdx.x];
    }
    return;
  }
  for (int64_t at = blockIdx.x; at < p.segments * p.groups; at += joins) {
    const int64_t s = at / p.groups;
    const int32_t g = (int32_t)(at - s * p.groups);
    const int64_t b = seg_begin(p, s), e = seg_begin(p, s + 1);
    const float *base = part + s * 2 * (int64_t)p.channels + (int64_t)g * p.per_group;
    const float *w = p.weight ? p.weight + (int64_t)g * p.per_group : nullptr;
    const double count = e > b ? (double)(e - b) * p.per_group : 1.0;
    double a = 0, q = 0;
    int64_t c0, c1;
    if (chunks_of(p, b, e, &c0, &c1)) {
      // lanes over the group's channels, the rest of the workgroup over chunks
      const int lane = threadIdx.x % p.share, row = threadIdx.x / p.share, step = blockDim.x / p.share;
      for (int32_t i = lane; i < p.per_group; i += p.share) {
        const double wi = w ? (double)w[i] : 1.0;
        double ai = 0, qi = 0;
#pragma unroll 4
        for (int64_t k = c0 + row; k <= c1; k += step) {
          ai += base[k * 2 * p.channels + i];
          qi += base[(k * 2 + 1) * p.channels + i];
        }
        a += wi * ai;
        q += wi * qi;
      }
    }
    a = wg_sum(a, lds);
    q = wg_sum(q, lds);
    if (threadIdx.x == 0) {
      m1[at] = (float)(a / count);
      m2[at] = (float)(q / count);
    }
    __syncthreads();
  }
}

template <typename T, typename X, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_grad(Shape p, X x, Dense<const T> dy, const float *__restrict__ mean,
                                                        const float *__restrict__ rstd, const float *__restrict__ m1,
                                                        const float *__restrict__ m2, Dense<T> dx) {
  const int tx = threadIdx.x % p.tx, ty = threadIdx.x / p.tx, TY = p.ty;
  const int32_t c = (blockIdx.y * p.tx + tx) * V;
  const int left = p.channels - c;
  const bool whole = p.channels % V == 0;
  if (left <= 0) return;
  const int64_t r0 = (int64_t)(p.chunks - 1 - blockIdx.x) * p.chunk_rows;
  const int64_t r1 = r0 + p.chunk_rows < p.rows ? r0 + p.chunk_rows : p.rows;
  for_pieces(p, r0, r1, [&](int64_t s, int64_t lo, int64_t hi) {
    Coeff k;
    float rs[V], a1[V], a2[V];
    load_coeff(p, mean, rstd, s, c, left, k, rs);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t g = s * p.groups + (i < left ? (c + i) / p.per_group : 0);
      a1[i] = m1[g] * rs[i];
      a2[i] = m2[g] * rs[i];
    }
    for_rows(lo, hi, ty, TY, [&](int64_t row, auto count) {
      constexpr int N = decltype(count)::value;
      float xv[N][V], dv[N][V];
      x.load(row, TY, c, left, whole, xv);
      dy.load(row, TY, c, left, whole, dv);
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = xv[u][i] - k.mean[i];
          const float dz = dv[u][i] * act_slope<ACT>(d * k.scale[i] + k.shift[i]);
          dv[u][i] = dz * k.scale[i] - a1[i] - d * rs[i] * a2[i];  // rstd^2 by itself may not fit 32 bits
        }
      dx.store(row, TY, c, left, whole, dv);
    });
  });
}

// ------------------------------------------------------ short segments -----
constexpr int kHeld = 8;  // rows of a lane that stay in registers
// Waves a SIMD: without the limit the compiler takes registers for two, and 100003 rows
// of 96 bf16 in 3001 segments take 43 us a call instead of 34.
constexpr int kTeamWaves = 3;

template <int N>
__device__ inline float (&first_of(float (&v)[N][V]))[1][V] {
  return *reinterpret_cast<float(*)[1][V]>(&v[0]);
}

// Adds a team's values, items[ty][tx * V], group by group: `share` lanes to a
// group, `across` of them over its channels; f(group, sums) in one lane of them.
template <typename S, typename F>
__device__ inline void team_sums(const Shape &p, const S *items, int t, F f) {
  const int team = p.tx * p.ty, row = p.tx * V;
  const int down = p.share / p.across, lane = t & (p.share - 1);
  for (int32_t g = t / p.share; g < p.groups; g += team / p.share) {
    double a = 0, b = 0;
    for (int32_t y = lane / p.across; y < p.ty; y += down)
      for (int32_t q = lane & (p.across - 1); q < p.per_group; q += p.across) {
        const S v = items[y * row + g * p.per_group + q];
        a += v.x;
        b += v.y;
      }
    for (int d = 1; d < p.share; d *= 2) {
      a += __shfl_xor(a, d);
      b += __shfl_xor(b, d);
    }
    if (lane == 0) f(g, a, b);
  }
}

// A team per segment.  Its first kHeld rows a lane are read once and kept; what a
// longer segment has beyond them is read again, from L2.
template <typename T, int ACT, int XF, int YF>
__global__ __launch_bounds__(kThreads, kTeamWaves) void k_norm_team(Shape p, Dense<const T> x,
                                                                    float *__restrict__ mean, float *__restrict__ rstd,
                                                                    Dense<T> y, Packs xo, Packs yo) {
  __shared__ double2 s_sum[kThreads][V];
  __shared__ float2 s_stat[kThreads * V];
  __shared__ float s_origin[kThreads * V];
  const int team = p.tx * p.ty, which = threadIdx.x / team, teams = blockDim.x / team, t = threadIdx.x % team;
  const int tx = t % p.tx, ty = t / p.tx, TY = p.ty;
  const int32_t c = tx * V, left = p.channels - c, width = p.tx < kBlock / V ? p.tx : kBlock / V;
  const bool whole = p.channels % V == 0;
  float2 *stat = s_stat + which * p.groups;
  const int most = p.one_row ? TY : TY * kHeld;  // rows that are kept
  float weight[V], shift[V];
  int32_t group[V], group_first[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    weight[i] = p.weight && i < left ? p.weight[c + i] : 1.0f;
    shift[i] = p.bias && i < left ? p.bias[c + i] : 0.0f;
    group[i] = i < left ? (c + i) / p.per_group : 0;
    group_first[i] = group[i] * p.per_group;
  }
  for (int64_t s0 = (int64_t)blockIdx.x * teams; s0 < p.segments; s0 += (int64_t)gridDim.x * teams) {
    const int64_t s = s0 + which;
    const bool here = s < p.segments;
    int64_t lo = here ? seg_begin(p, s) : 0, hi = here ? seg_begin(p, s + 1) : 0;
    lo = lo < 0 ? 0 : lo;
    hi = hi > p.rows ? p.rows : hi;
    const int64_t mid = lo + most < hi ? lo + most : hi;
    const double one = 1.0 / (hi > lo ? (double)(hi - lo) * p.per_group : 1.0);
    float v[kHeld][V], origin[V] = {};
    double a[V] = {}, b[V] = {};
    if (lo < hi) origins_of(p, x, lo, group_first, origin);
    auto add = [&](const float (&u)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float o = origin[i];
        asm volatile("" : "+v"(o));  // widened at each use: four registers instead of eight
        const double d = (double)u[i] - (double)o;
        a[i] += d;
        b[i] = fma(d, d, b[i]);
      }
    };
    const int64_t last = mid > 0 ? mid - 1 : 0;
    if (p.one_row) {  // the same for all threads
      if (p.rows > 0) x.load_to(last, lo + ty, TY, c, left, whole, first_of(v));
      if (lo + ty < mid) add(v[0]);
    } else {
      if (p.rows > 0) x.load_to(last, lo + ty, TY, c, left, whole, v);
#pragma unroll
      for (int u = 0; u < kHeld; ++u)
        if (lo + ty + u * TY < mid) add(v[u]);
    }
    if (mid < hi)
      for_rows(mid, hi, ty, TY, [&](int64_t row, auto count) {
        constexpr int N = decltype(count)::value;
        float w[N][V];
        x.load(row, TY, c, left, whole, w);
#pragma unroll
        for (int u = 0; u < N; ++u) add(w[u]);
      });
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[threadIdx.x][i] = double2{a[i], b[i]};
    if (ty == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i)  // one lane has a group's first channel
        if (i < left && c + i == group_first[i]) s_origin[which * p.groups + group[i]] = origin[i];
    }
    __syncthreads();
    if (here)
      team_sums(p, &s_sum[which * team][0], t, [&](int32_t g, double sum, double square) {
        float m, r;
        write_stats(p, sum, square, one, s_origin[which * p.groups + g], &m, &r);
        stat[g] = float2{m, r};
        mean[s * p.groups + g] = m;
        rstd[s * p.groups + g] = r;
      });
    __syncthreads();
    if (lo >= hi) continue;
    Coeff k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 st = stat[group[i]];
      k.mean[i] = st.x;
      k.scale[i] = st.y * weight[i];
      k.shift[i] = shift[i];
    }
    auto finish = [&](int64_t row, float (&u)[1][V]) {
      if constexpr (XF != 0) store_packed<XF>(xo, p.rows, row, c, p.channels, tx, width, u[0]);
#pragma unroll
      for (int i = 0; i < V; ++i) u[0][i] = act<ACT>((u[0][i] - k.mean[i]) * k.scale[i] + k.shift[i]);
      if constexpr (YF != 0) store_packed<YF>(yo, p.rows, row, c, p.channels, tx, width, u[0]);
      if (y.p) y.store(row, 0, c, left, whole, u);
    };
    if (lo + ty < mid) finish(lo + ty, first_of(v));
    if (!p.one_row) {
#pragma unroll
      for (int u = 1; u < kHeld; ++u) {
        const int64_t row = lo + ty + u * TY;
        if (row < mid) finish(row, *reinterpret_cast<float(*)[1][V]>(&v[u]));
      }
    }
    if (mid < hi)
      for_rows(mid, hi, ty, TY, [&](int64_t row, auto count) {
        constexpr int N = decltype(count)::value;
        float w[N][V];
        x.load(row, TY, c, left, whole, w);
#pragma unroll
        for (int u = 0; u < N; ++u) finish(row + u * TY, *reinterpret_cast<float(*)[1][V]>(&w[u]));
      });
  }
}

// The gradients the same way; a workgroup leaves its segments' sums of dz and
// dz xh per channel in total.
template <typename T, typename X, int ACT>
__global__ __launch_bounds__(kThreads) void k_norm_team_grad(Shape p, X x, Dense<const T> dy, const float *__restrict__ mean,
                                                             const float *__restrict__ rstd, Dense<T> dx,
                                                             float *__restrict__ total) {
  constexpr int kHeldBack = kHeld / 2;
  __shared__ float2 s_sum[kThreads][V];
  __shared__ float2 s_stat[kThreads * V];
  const int team = p.tx * p.ty, which = threadIdx.x / team, teams = blockDim.x / team, t = threadIdx.x % team;
  const int tx = t % p.tx, ty = t / p.tx, TY = p.ty;
  const int32_t c = tx * V, left = p.channels - c;
  const bool whole = p.channels % V == 0;
  float2 *stat = s_stat + which * p.groups;
  const int most = p.one_row ? TY : TY * kHeldBack;  // rows that are kept
  float w[V], ta[V] = {}, tb[V] = {};
#pragma unroll
  for (int i = 0; i < V; ++i) w[i] = i >= left ? 0.0f : p.weight ? p.weight[c + i] : 1.0f;
  for (int64_t s0 = (int64_t)blockIdx.x * teams; s0 < p.segments; s0 += (int64_t)gridDim.x * teams) {
    const int64_t s = s0 + which;
    const bool here = s < p.segments;
    int64_t lo = here ? seg_begin(p, s) : 0, hi = here ? seg_begin(p, s + 1) : 0;
    lo = lo < 0 ? 0 : lo;
    hi = hi > p.rows ? p.rows : hi;
    const int64_t mid = lo + most < hi ? lo + most : hi;
    Coeff k;
    float rs[V];
    load_coeff(p, mean, rstd, here ? s : 0, c, left, k, rs);
    float d[kHeldBack][V], dz[kHeldBack][V], a[V] = {}, b[V] = {};
    // xh and dz of one row in place of x and dy
    auto shape = [&](float (&xv)[V], float (&dv)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float off = xv[i] - k.mean[i];
        dv[i] *= act_slope<ACT>(off * k.scale[i] + k.shift[i]);
        xv[i] = off * rs[i];
      }
    };
    const int64_t last = mid > 0 ? mid - 1 : 0;
    if (p.one_row && p.rows > 0) {  // the same for all threads
      x.load_to(last, lo + ty, TY, c, left, whole, first_of(d));
      dy.load_to(last, lo + ty, TY, c, left, whole, first_of(dz));
    } else if (p.rows > 0) {
      x.load_to(last, lo + ty, TY, c, left, whole, d);
      dy.load_to(last, lo + ty, TY, c, left, whole, dz);
    }
    auto add = [&](int u) {
      shape(d[u], dz[u]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        a[i] += dz[u][i];
        b[i] += dz[u][i] * d[u][i];
      }
    };
    if (lo + ty < mid) add(0);
    if (!p.one_row) {
#pragma unroll
      for (int u = 1; u < kHeldBack; ++u)
        if (lo + ty + u * TY < mid) add(u);
    }
    if (mid < hi)
      for_rows(mid, hi, ty, TY, [&](int64_t row, auto count) {
        constexpr int N = decltype(count)::value;
        float xv[N][V], dv[N][V], sa[V] = {}, sb[V] = {};
        x.load(row, TY, c, left, whole, xv);
        dy.load(row, TY, c, left, whole, dv);
#pragma unroll
        for (int u = 0; u < N; ++u) {
          shape(xv[u], dv[u]);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            sa[i] += dv[u][i];
            sb[i] += dv[u][i] * xv[u][i];
          }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          a[i] += sa[i];
          b[i] += sb[i];
        }
      });
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ta[i] += a[i];
      tb[i] += b[i];
      s_sum[threadIdx.x][i] = float2{w[i] * a[i], w[i] * b[i]};
    }
    __syncthreads();
    if (here)
      team_sums(p, &s_sum[which * team][0], t, [&](int32_t g, double sa, double sb) {
        const double count = hi > lo ? (double)(hi - lo) * p.per_group : 1.0;
        stat[g] = float2{(float)(sa / count), (float)(sb / count)};
      });
    __syncthreads();
    if (lo >= hi || left <= 0) continue;
    float a1[V], a2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 st = i < left ? stat[(c + i) / p.per_group] : float2{0, 0};
      a1[i] = st.x * rs[i];
      a2[i] = st.y * rs[i];
    }
    auto finish = [&](int64_t row, const float (&xv)[V], const float (&dv)[V]) {
      float out[1][V];
#pragma unroll
      for (int i = 0; i < V; ++i) out[0][i] = dv[i] * k.scale[i] - a1[i] - xv[i] * a2[i];
      dx.store(row, 0, c, left, whole, out);
    };
    if (lo + ty < mid) finish(lo + ty, d[0], dz[0]);
    if (!p.one_row) {
#pragma unroll
      for (int u = 1; u < kHeldBack; ++u) {
        const int64_t row = lo + ty + u * TY;
        if (row < mid) finish(row, d[u], dz[u]);
      }
    }
    if (mid < hi)
      for_rows(mid, hi, ty, TY, [&](int64_t row, auto count) {
        constexpr int N = decltype(count)::value;
        float xv[N][V], dv[N][V];
        x.load(row, TY, c, left, whole, xv);
        dy.load(row, TY, c, left, whole, dv);
#pragma unroll
        for (int u = 0; u < N; ++u) {
          shape(xv[u], dv[u]);
          finish(row + u * TY, xv[u], dv[u]);
        }
      });
  }
  // the workgroup's sums over its lane rows
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) s_sum[threadIdx.x][i] = float2{ta[i], tb[i]};
  __syncthreads();
  for (int h = blockDim.x / p.tx / 2; h > 0; h /= 2) {
    if ((int)threadIdx.x < h * p.tx) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 o = s_sum[threadIdx.x + h * p.tx][i];
        s_sum[threadIdx.x][i].x += o.x;
        s_sum[threadIdx.x][i].y += o.y;
      }
    }
    __syncthreads();
  }
  for (int32_t i = threadIdx.x; i < p.channels; i += blockDim.x) {
    const float2 o = (&s_sum[0][0])[i];
    total[(int64_t)blockIdx.x * 2 * p.channels + i] = o.x;
    total[((int64_t)blockIdx.x * 2 + 1) * p.channels + i] = o.y;
  }
}

// ---------------------------------------------------------------- host -----
int check(const sd_norm_t *d) {
  if (!d || d->rows < 0 || d->channels < 1 || d->groups < 1 || d->segments < 0 || d->longest < 0 ||
      !type_ok(d->type) || d->activation < SD_ACT_NONE || d->activation > SD_ACT_GELU || d->reserved != 0 ||
      !(d->eps >= 0.0f))
    return SD_ERR_INVALID_VALUE;
  if (d->channels % d->groups != 0) return SD_ERR_INVALID_VALUE;
  if (!aligned_to(d->offsets, 4) || !aligned_to(d->weight, 4) || !aligned_to(d->bias, 4)) return SD_ERR_INVALID_VALUE;
  if (d->rows > kMaxRows || d->segments > kMaxRows || d->channels > (1 << 24)) return SD_ERR_OVERFLOW;
  if (!d->offsets && d->rows > 0 && (d->segments < 1 || d->rows % d->segments != 0)) return SD_ERR_INVALID_VALUE;
  if (d->offsets && d->rows > 0 && d->segments < 1) return SD_ERR_INVALID_VALUE;
  return SD_OK;
}

// Lanes for a row, with the 8-bit copies' bytes up to a multiple of 16.
int64_t lanes_of(int32_t channels) { return ceil_div(channels, 16) * (16 / V); }

// Rows of the longest segment as far as the caller says; all of them else.
int64_t longest_of(const sd_norm_t *d) {
  if (!d->offsets) return d->segments > 0 ? d->rows / d->segments : 0;
  return d->longest > 0 && d->longest < d->rows ? d->longest : d->rows;
}

// Lanes over channels: a power of two, or whole blocks of 32 lanes, so that a
// row's block of 128 columns lies in aligned lanes of one wave.
// Short segments, of at most kTeamBytes, go to teams: a power of two of threads,
// with as many lane rows as a segment of the mean length keeps busy.  Else chunks:
// four workgroups per compute unit, all resident at once, each thread a batch of
// rows at least.
constexpr int64_t kTeamBytes = 128 << 10;
Shape shape_of(const sd_norm_t *d, bool back) {
  Shape p{};
  p.rows = d->rows;
  p.segments = d->segments;
  p.len = d->segments > 0 ? d->rows / d->segments : 0;
  p.offsets = d->offsets;
  p.channels = d->channels;
  p.groups = d->groups;
  p.per_group = d->channels / d->groups;
  p.eps = d->eps;
  p.weight = d->weight;
  p.bias = d->bias;
  const int64_t lanes = lanes_of(d->channels);
  int32_t tx = 1;
  while (tx < 32 && tx < lanes) tx *= 2;
  if (lanes > 32) tx = (int32_t)(lanes > kThreads ? kThreads : ceil_div(lanes, 32) * 32);
  if (lanes <= kThreads && longest_of(d) * d->channels * type_bytes(d->type) <= kTeamBytes && d->segments > 0) {
    while (tx & (tx - 1)) tx += 32;
    const int64_t held = back ? kHeld / 2 : kHeld, mean = ceil_div(d->rows, d->segments);
    p.tx = tx;
    p.ty = 1;
    while (p.ty * 2 * tx <= kThreads && p.ty * held < mean) p.ty *= 2;
    const int32_t team = p.tx * p.ty;
    p.share = 1;
    while (p.share < 64 && p.share * 2 <= team && p.share * 2 * p.groups <= team) p.share *= 2;
    p.across = 1;
    while (p.across * 2 <= p.share && p.across * 2 <= p.per_group) p.across *= 2;
    p.one_row = longest_of(d) <= p.ty;
    // what a thread needs of its channels is read once for all its segments; the
    // gradients' sums over all segments are kept per workgroup
    const int64_t wgs = ceil_div(d->segments, kThreads / team), most = (back ? 4ll : 6ll) * cu_count();
    p.wgs = (int32_t)(wgs < most ? wgs : most);
    p.chunks = p.wgs;
    return p;
  }
  p.tx = tx;
  p.ty = 1;
  while (p.ty * 2 * tx <= kThreads) p.ty *= 2;
  const int64_t slabs = ceil_div(lanes, tx);
  p.slots = p.groups + (int32_t)slabs - 1;
  // lanes that share a group's channels: a power of two that the workgroup's threads come out even in
  // (160 and 224 of them leave half a wave)
  p.share = 1;
  while (p.share < 64 && p.share * 4 <= p.per_group && p.tx * p.ty % (p.share * 2) == 0) p.share *= 2;
  const int64_t step = (int64_t)p.ty * kBatch;
  const int64_t want = 4ll * cu_count() / slabs;
  int64_t rows = ceil_div(d->rows, want > 0 ? want : 1);
  rows = ceil_div(rows > 0 ? rows : 1, step) * step;
  p.chunk_rows = (int32_t)(rows > kMaxRows ? kMaxRows : rows);
  p.chunks = (int32_t)ceil_div(d->rows, p.chunk_rows);
  return p;
}
uint32_t slabs_of(const Shape &p) { return (uint32_t)ceil_div(lanes_of(p.channels), p.tx); }
size_t part_bytes(const Shape &p) { return 8 * (size_t)(p.chunks + p.segments) * (size_t)p.channels; }
size_t stats_bytes(const Shape &p) { return p.wgs ? 0 : 16 * (size_t)(p.chunks + p.segments) * (size_t)p.slots; }
size_t total_bytes(const Shape &p) { return 8 * (size_t)p.chunks * (size_t)p.channels; }
size_t back_bytes(const Shape &p) {
  if (p.wgs) return total_bytes(p);
  return part_bytes(p) + total_bytes(p) + 8 * (size_t)p.segments * (size_t)p.groups;
}
// Workgroups and threads of a joining kernel: one workgroup per segment and
// group, wide where there are few of them.
uint32_t join_wgs(const Shape &p) {
  const int64_t n = p.segments * (int64_t)p.groups;
  return (uint32_t)(n < (1 << 20) ? n : (1 << 20));
}
uint32_t join_threads(const Shape &p) {
  return (!p.wgs && p.segments * (int64_t)p.groups >= 1024) || p.chunks < 8 ? 64 : 1024;
}

// A result of 64 MB or more leaves the Infinity Cache to the table that the second
// pass reads again: a training step of 262144 x 128 fp32 takes 190 us, and 219 us
// with ordinary stores.
template <typename T>
bool streamed(const Shape &p) {
  return p.rows * p.channels * (int64_t)sizeof(T) >= 64 << 20;
}

template <typename T, int ACT, int XF, int YF>
void apply(const Shape &p, Dense<const T> x, float *mean, float *rstd, Dense<T> y, Packs xo, Packs yo, hipStream_t s) {
  if (p.wgs) {
    hipLaunchKernelGGL((k_norm_team<T, ACT, XF, YF>), dim3(p.wgs), dim3(kThreads), 0, s, p, x, mean, rstd, y,
                       xo, yo);
    return;
  }
  hipLaunchKernelGGL((k_norm_apply<T, ACT, XF, YF>), dim3(p.chunks, slabs_of(p)), dim3(p.tx * p.ty), 0, s, p, x, mean,
                     rstd, y, xo, yo);
}
template <typename T, int ACT, int XF>
void apply_y(int yf, const Shape &p, Dense<const T> x, float *mean, float *rstd, Dense<T> y, Packs xo, Packs yo,
             hipStream_t s) {
  if (yf == SD_PACK_E4M3)
    apply<T, ACT, XF, SD_PACK_E4M3>(p, x, mean, rstd, y, xo, yo, s);
  else if (yf == SD_PACK_E5M2)
    apply<T, ACT, XF, SD_PACK_E5M2>(p, x, mean, rstd, y, xo, yo, s);
  else
    apply<T, ACT, XF, 0>(p, x, mean, rstd, y, xo, yo, s);
}
template <typename T, int ACT>
void apply_x(int xf, int yf, const Shape &p, Dense<const T> x, float *mean, float *rstd, Dense<T> y, Packs xo,
             Packs yo, hipStream_t s) {
  if (xf == SD_PACK_E4M3)
    apply_y<T, ACT, SD_PACK_E4M3>(yf, p, x, mean, rstd, y, xo, yo, s);
  else if (xf == SD_PACK_E5M2)
    apply_y<T, ACT, SD_PACK_E5M2>(yf, p, x, mean, rstd, y, xo, yo, s);
  else
    apply_y<T, ACT, 0>(yf, p, x, mean, rstd, y, xo, yo, s);
}

template <typename T>
int forward(const Shape &p, int32_t activation, const void *x, int64_t x_stride, void *y, int64_t y_stride,
            const sd_packed_t *xp, const sd_packed_t *yp, float *mean, float *rstd, double2 *part, hipStream_t s) {
  const Dense<const T> in{static_cast<const T *>(x), (uint32_t)x_stride, false};
  const Dense<T> out{static_cast<T *>(y), (uint32_t)y_stride, streamed<T>(p)};
  const Packs none{nullptr, nullptr, 0};
  const Packs xo = xp ? Packs{xp->codes, xp->scales, xp->ld} : none;
  const Packs yo = yp ? Packs{yp->codes, yp->scales, yp->ld} : none;
  const int xf = xp ? xp->format : 0, yf = yp ? yp->format : 0;
  if (!p.wgs && p.chunks > 0)
    hipLaunchKernelGGL((k_norm_stats<T>), dim3(p.chunks, slabs_of(p)), dim3(p.tx * p.ty), 0, s, p, in, part);
  if (!p.wgs && join_wgs(p) > 0)
    hipLaunchKernelGGL((k_norm_join<T>), dim3(join_wgs(p)), dim3(join_threads(p)), 0, s, p, in, part, mean, rstd);
  if (p.chunks > 0) {
    if (activation == SD_ACT_RELU)
      apply_x<T, SD_ACT_RELU>(xf, yf, p, in, mean, rstd, out, xo, yo, s);
    else if (activation == SD_ACT_SILU)
      apply_x<T, SD_ACT_SILU>(xf, yf, p, in, mean, rstd, out, xo, yo, s);
    else if (activation == SD_ACT_GELU)
      apply_x<T, SD_ACT_GELU>(xf, yf, p, in, mean, rstd, out, xo, yo, s);
    else
      apply_x<T, SD_ACT_NONE>(xf, yf, p, in, mean, rstd, out, xo, yo, s);
  }
  return launched();
}

template <typename T, typename X, int ACT>
int backward_as(const Shape &p, X x, Dense<const T> dy, const float *mean, const float *rstd, Dense<T> dx,
                float *dweight, float *dbias, float *ws, hipStream_t s) {
  if (p.wgs) {
    hipLaunchKernelGGL((k_norm_team_grad<T, X, ACT>), dim3(p.wgs), dim3(kThreads), 0, s, p, x, dy, mean, rstd, dx,
                       ws);
    if (dweight || dbias)
      hipLaunchKernelGGL(k_norm_join_back, dim3((uint32_t)ceil_div(p.channels, kJoinCols)), dim3(join_threads(p)), 0, s,
                         p, 0, nullptr, ws, nullptr, nullptr, dweight, dbias);
    return launched();
  }
  float *part = ws, *total = part + part_bytes(p) / 4, *m1 = total + total_bytes(p) / 4,
        *m2 = m1 + p.segments * p.groups;
  const dim3 grid(p.chunks, slabs_of(p)), threads(p.tx * p.ty);
  if (p.chunks > 0)
    hipLaunchKernelGGL((k_norm_sums<T, X, ACT>), grid, threads, 0, s, p, x, dy, mean, rstd, part, total);
  hipLaunchKernelGGL(k_norm_join_back, dim3(join_wgs(p) + (uint32_t)ceil_div(p.channels, kJoinCols)),
                     dim3(join_threads(p)), 0, s, p, (int32_t)join_wgs(p), part, total, m1, m2, dweight, dbias);
  if (p.chunks > 0)
    hipLaunchKernelGGL((k_norm_grad<T, X, ACT>), grid, threads, 0, s, p, x, dy, mean, rstd, m1, m2, dx);
  return launched();
}
template <typename T, typename X>
int backward_act(int32_t activation, const Shape &p, X x, Dense<const T> dy, const float *mean, const float *rstd,
                 Dense<T> dx, float *dweight, float *dbias, float *ws, hipStream_t s) {
  if (activation == SD_ACT_RELU)
    return backward_as<T, X, SD_ACT_RELU>(p, x, dy, mean, rstd, dx, dweight, dbias, ws, s);
  if (activation == SD_ACT_SILU)
    return backward_as<T, X, SD_ACT_SILU>(p, x, dy, mean, rstd, dx, dweight, dbias, ws, s);
  if (activation == SD_ACT_GELU)
    return backward_as<T, X, SD_ACT_GELU>(p, x, dy, mean, rstd, dx, dweight, dbias, ws, s);
  return backward_as<T, X, SD_ACT_NONE>(p, x, dy, mean, rstd, dx, dweight, dbias, ws, s);
}
template <typename T>
int backward(int32_t activation, const Shape &p, const void *x, int64_t x_stride, const sd_packed_t *xp,
             const void *dy, int64_t dy_stride, const float *mean, const float *rstd, void *dx, int64_t dx_stride,
             float *dweight, float *dbias, float *ws, hipStream_t s) {
  const Dense<const T> in{static_cast<const T *>(x), (uint32_t)x_stride, false}, g{static_cast<const T *>(dy), (uint32_t)dy_stride, false};
  const Dense<T> out{static_cast<T *>(dx), (uint32_t)dx_stride, streamed<T>(p)};
  if (!xp) return backward_act<T>(activation, p, in, g, mean, rstd, out, dweight, dbias, ws, s);
  if (xp->format == SD_PACK_E4M3)
    return backward_act<T>(activation, p, Codes<SD_PACK_E4M3>{xp->codes, xp->scales, xp->ld, xp->rows}, g, mean, rstd,
                           out, dweight, dbias, ws, s);
  return backward_act<T>(activation, p, Codes<SD_PACK_E5M2>{xp->codes, xp->scales, xp->ld, xp->rows}, g, mean, rstd,
                         out, dweight, dbias, ws, s);
}

int check_copy(const sd_norm_t *d, const sd_packed_t *p) {
  if (!p) return SD_OK;
  const int st = check_packed(p);
  if (st != SD_OK) return st;
  return p->rows == d->rows && p->cols == d->channels ? SD_OK : SD_ERR_INVALID_VALUE;
}

}  // namespace

extern "C" int sd_group_norm_size(const sd_norm_t *d, size_t *forward, size_t *backward) {
  const int st = check(d);
  if (st != SD_OK) return st;
  if (!forward && !backward) return SD_ERR_INVALID_VALUE;
  if (forward) *forward = stats_bytes(shape_of(d, false));
  if (backward) *backward = back_bytes(shape_of(d, true));
  return SD_OK;
}

extern "C" int sd_group_norm(const sd_norm_t *d, const void *x, int64_t x_stride, void *y, int64_t y_stride,
                             const sd_packed_t *x_packed, const sd_packed_t *y_packed, float *mean, float *rstd,
                             void *workspace, size_t bytes, void *stream) {
  int st = check(d);
  if (st != SD_OK) return st;
  if ((st = check_table(x, d->type, d->rows, d->channels, x_stride)) != SD_OK) return st;
  if (y && (st = check_table(y, d->type, d->rows, d->channels, y_stride)) != SD_OK) return st;
  if ((st = check_copy(d, x_packed)) != SD_OK || (st = check_copy(d, y_packed)) != SD_OK) return st;
  if (!y && !y_packed && d->rows > 0) return SD_ERR_INVALID_VALUE;
  if (d->segments > 0 && (!mean || !rstd)) return SD_ERR_INVALID_VALUE;
  if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return SD_ERR_INVALID_VALUE;
  const Shape p = shape_of(d, false);
  if (bytes < stats_bytes(p) || (stats_bytes(p) > 0 && (!workspace || !aligned_to(workspace, 16))))
    return SD_ERR_INVALID_VALUE;
  if (d->segments == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  double2 *part = static_cast<double2 *>(workspace);
  return d->type == SD_TYPE_F32
             ? forward<float>(p, d->activation, x, x_stride, y, y_stride, x_packed, y_packed, mean, rstd, part, s)
         : d->type == SD_TYPE_F16
             ? forward<f16>(p, d->activation, x, x_stride, y, y_stride, x_packed, y_packed, mean, rstd, part, s)
             : forward<bf16>(p, d->activation, x, x_stride, y, y_stride, x_packed, y_packed, mean, rstd, part, s);
}

extern "C" int sd_group_norm_backward(const sd_norm_t *d, const void *dy, int64_t dy_stride, const void *x,
                                      int64_t x_stride, const sd_packed_t *x_packed, const float *mean,
                                      const float *rstd, void *dx, int64_t dx_stride, float *dweight, float *dbias,
                                      void *workspace, size_t bytes, void *stream) {
  int st = check(d);
  if (st != SD_OK) return st;
  if ((st = check_table(dy, d->type, d->rows, d->channels, dy_stride)) != SD_OK) return st;
  if ((st = check_table(dx, d->type, d->rows, d->channels, dx_stride)) != SD_OK) return st;
  if ((st = check_copy(d, x_packed)) != SD_OK) return st;
  if (!x_packed && (st = check_table(x, d->type, d->rows, d->channels, x_stride)) != SD_OK) return st;
  if (x && x_packed) return SD_ERR_INVALID_VALUE;
  if (d->segments > 0 && (!mean || !rstd)) return SD_ERR_INVALID_VALUE;
  if (!aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(dweight, 4) || !aligned_to(dbias, 4))
    return SD_ERR_INVALID_VALUE;
  const Shape p = shape_of(d, true);
  if (bytes < back_bytes(p) || (back_bytes(p) > 0 && (!workspace || !aligned_to(workspace, 16))))
    return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float *ws = static_cast<float *>(workspace);
  return d->type == SD_TYPE_F32 ? backward<float>(d->activation, p, x, x_stride, x_packed, dy, dy_stride, mean, rstd,
                                                  dx, dx_stride, dweight, dbias, ws, s)
         : d->type == SD_TYPE_F16 ? backward<f16>(d->activation, p, x, x_stride, x_packed, dy, dy_stride, mean, rstd,
                                                  dx, dx_stride, dweight, dbias, ws, s)
                                  : backward<bf16>(d->activation, p, x, x_stride, x_packed, dy, dy_stride, mean, rstd,
                                                   dx, dx_stride, dweight, dbias, ws, s);
}
