// sd_route, sd_dispatch, sd_combine: entries (row t, slot j) sorted by the expert
// that each was given, the rows brought there and the results brought back.
//
// A stable counting sort: position(t, j) = offsets[e] + the number of entries of
// expert e before (t, j).  Entries without an expert are one more kind behind the
// last.  A wave counts a run of neighbouring entries 64 at a time; lanes of equal
// kind find each other with one ballot for each bit of the kind, and a lane's rank
// among them is the number of such lanes before it.  Nothing depends on the order
// in which waves run.
#include <type_traits>

#include "nibble.h"

namespace {

using namespace nibble;

constexpr int64_t kMaxRuns = 1024;    // runs of entries that are counted apart
constexpr int64_t kRun = 512;         // entries of a run at least
constexpr int64_t kOneGroup = 8192;   // entries that one workgroup sorts by itself
constexpr int kWaves = 16;            // of it
constexpr int kKindsAlone = 960;      // kinds whose counters for 16 waves and whose sums fit 64 KiB

__device__ inline uint32_t kind_of(const void *chosen, int wide, int64_t i, uint32_t experts) {
  const int64_t e = wide ? static_cast<const int64_t *>(chosen)[i] : (int64_t) static_cast<const int32_t *>(chosen)[i];
  return e >= 0 && e < (int64_t)experts ? (uint32_t)e : experts;
}
// The lanes whose kind is this lane's.
__device__ inline uint64_t same_kind(uint32_t kind, int bits, bool there) {
  uint64_t mask = __ballot(there);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((kind >> b) & 1);
    mask &= (kind >> b) & 1 ? set : ~set;
  }
  return mask;
}

// Counts of each kind among entries [begin, end), by one wave.
__device__ inline void count_run(const void *chosen, int wide, uint32_t experts, int64_t begin, int64_t end,
                                 uint32_t *counts) {
  for (int64_t i = begin + (threadIdx.x & 63); i < end; i += 64)
    atomicAdd(&counts[kind_of(chosen, wide, i, experts)], 1u);
}
// Positions of entries [begin, end), by one wave: next[kind] is the position of
// its next entry.
__device__ inline void place_run(const void *chosen, int wide, uint32_t experts, int bits, int32_t k, int64_t begin,
                                 int64_t end, uint32_t *next, int32_t *place, int32_t *source) {
  const int lane = threadIdx.x & 63;
  for (int64_t i0 = begin; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool there = i < end;
    const uint32_t kind = there ? kind_of(chosen, wide, i, experts) : 0u;
    const uint64_t same = same_kind(kind, bits, there);
    if (there) {
      const int before = __popcll(same & ((1ull << lane) - 1));
      const uint32_t at = next[kind] + (uint32_t)before;
      __builtin_amdgcn_wave_barrier();  // every lane has read before one writes
      if (before == 0) next[kind] = at + (uint32_t)__popcll(same);
      const bool kept = kind < experts;
      place[i] = kept ? (int32_t)at : -1;
      source[at] = kept ? (int32_t)(i / k) : -1;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Sums of v over the threads before this one, of up to 1024; `sums` holds 16.
__device__ inline uint32_t sum_before(uint32_t v, uint32_t *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_up((int)upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += sums[w];
  return before + upto - v;
}

// All of it in one launch, for few entries.
__global__ __launch_bounds__(kWaves * 64) void k_route_few(const void *__restrict__ chosen, int wide, int64_t entries,
                                                           int32_t k, int32_t experts, int bits,
                                                           int32_t *__restrict__ offsets, int32_t *__restrict__ place,
                                                           int32_t *__restrict__ source, int64_t run) {
  extern __shared__ uint32_t few_lds[];  // counters [waves][kinds]
  __shared__ uint32_t sums[kWaves];
  const int kinds = experts + 1, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < kWaves * kinds; i += kWaves * 64) few_lds[i] = 0;
  __syncthreads();
  const int64_t begin = wave * run, end = begin + run < entries ? begin + run : entries;
  uint32_t *mine = few_lds + wave * kinds;
  count_run(chosen, wide, experts, begin, end, mine);
  __syncthreads();
  const int kind = threadIdx.x;
  uint32_t total = 0;
  if (kind < kinds)
    for (int w = 0; w < kWaves; ++w) total += few_lds[w * kinds + kind];
  uint32_t at = sum_before(total, sums);
  if (kind < kinds) {
    offsets[kind] = (int32_t)at;
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = few_lds[w * kinds + kind];
      few_lds[w * kinds + kind] = at;
      at += c;
    }
  }
  __syncthreads();
  place_run(chosen, wide, experts, bits, k, begin, end, mine, place, source);
}

// Four runs a workgroup: counts[kind][run].
__global__ __launch_bounds__(256) void k_route_count(const void *__restrict__ chosen, int wide, int64_t entries,
                                                     int32_t experts, uint32_t *__restrict__ counts, int64_t run,
                                                     int32_t runs) {
  extern __shared__ uint32_t count_lds[];  // [4][kinds]
  const int kinds = experts + 1, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < 4 * kinds; i += 256) count_lds[i] = 0;
  __syncthreads();
  const int32_t r0 = blockIdx.x * 4, own = r0 + wave;
  const int64_t begin = own * run, end = begin + run < entries ? begin + run : entries;
  count_run(chosen, wide, experts, begin, end, count_lds + wave * kinds);
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * kinds; i += 256)
    if (r0 + i % 4 < runs) counts[(int64_t)(i / 4) * runs + r0 + i % 4] = count_lds[i % 4 * kinds + i / 4];
}
// A workgroup of 1024 for each kind: its counts become sums over the runs before,
// and their sum.
__global__ __launch_bounds__(1024) void k_route_sum(uint32_t *__restrict__ counts, int32_t runs,
                                                    uint32_t *__restrict__ totals) {
  __shared__ uint32_t sums[16];
  uint32_t *mine = counts + (int64_t)blockIdx.x * runs;
  const uint32_t v = (int)threadIdx.x < runs ? mine[threadIdx.x] : 0u;
  const uint32_t at = sum_before(v, sums);
  if ((int)threadIdx.x < runs) mine[threadIdx.x] = at;
  if (threadIdx.x == 1023) totals[blockIdx.x] = at + v;
}
__global__ __launch_bounds__(256) void k_route_place(const void *__restrict__ chosen, int wide, int64_t entries,
                                                     int32_t k, int32_t experts, int bits,
                                                     const uint32_t *__restrict__ counts,
                                                     const uint32_t *__restrict__ totals, int64_t run, int32_t runs,
                                                     int32_t *__restrict__ offsets, int32_t *__restrict__ place,
                                                     int32_t *__restrict__ source) {
  extern __shared__ uint32_t place_lds[];  // [4][kinds]
  __shared__ uint32_t sums[4];
  const int kinds = experts + 1, wave = threadIdx.x >> 6;
  // every kind's first position, 16 kinds a thread (4096 kinds at most)
  uint32_t own = 0;
  for (int i = 0; i < 16; ++i) {
    const int kind = threadIdx.x * 16 + i;
    if (kind < kinds) own += totals[kind];
  }
  uint32_t at = sum_before(own, sums);
  for (int i = 0; i < 16; ++i) {
    const int kind = threadIdx.x * 16 + i;
    if (kind >= kinds) break;
    if (blockIdx.x == 0) offsets[kind] = (int32_t)at;
    for (int w = 0; w < 4; ++w) {
      const int32_t r = blockIdx.x * 4 + w;
      place_lds[w * kinds + kind] = at + (r < runs ? counts[(int64_t)kind * runs + r] : 0u);
    }
    at += totals[kind];
  }
  __syncthreads();
  const int64_t begin = (int64_t)(blockIdx.x * 4 + wave) * run, end = begin + run < entries ? begin + run : entries;
  place_run(chosen, wide, experts, bits, k, begin, end, place_lds + wave * kinds, place, source);
}

// Offsets of no entries.
__global__ void k_route_none(int32_t *offsets, int32_t experts) {
  for (int i = threadIdx.x; i <= experts; i += blockDim.x) offsets[i] = 0;
}

int64_t run_of(int64_t entries) {
  const int64_t run = ceil_div(ceil_div(entries, kMaxRuns), 64) * 64;
  return run > kRun ? run : kRun;
}
bool few(int64_t entries, int32_t experts) { return entries <= kOneGroup && experts + 1 <= kKindsAlone; }

// ------------------------------------------------------- rows to and back ---
// A team of LANES lanes for each row t; 16 bytes of it a lane and step.
constexpr int kThreads = 256;

// y[place[t, j]] = x[t]; rows of y that no entry is sorted to (those behind the
// last expert's) become zeros.
template <typename T, int LANES>
__global__ __launch_bounds__(kThreads) void k_dispatch(const T *__restrict__ x, int64_t x_stride, int64_t rows,
                                                       int32_t k, int32_t cols, const int32_t *__restrict__ place,
                                                       const int32_t *__restrict__ source, T *__restrict__ y,
                                                       int64_t y_stride) {
  constexpr int V = 16 / sizeof(T);
  const int64_t t = (int64_t)workgroup() * (kThreads / LANES) + threadIdx.x / LANES;
  if (t >= rows) return;
  const int64_t total = rows * k;
  const int32_t *p = place + t * k, *s = source + t * k;
  for (int32_t c = threadIdx.x % LANES * V; c < cols; c += LANES * V) {
    float v[V];
    const float none[V] = {};
    const int left = cols - c;
    if (left >= V)
      load_span(x + t * x_stride + c, v);
    else
      load_part(x + t * x_stride + c, left, v);
    for (int32_t j = 0; j < k; ++j) {
      const int64_t to = p[j];
      if (to >= 0 && to < total) {
        if (left >= V)
          store_span(y + to * y_stride + c, v);
        else
          store_part(y + to * y_stride + c, left, v);
      }
      if (s[j] < 0) {
        if (left >= V)
          store_span(y + (t * k + j) * y_stride + c, none);
        else
          store_part(y + (t * k + j) * y_stride + c, left, none);
      }
    }
  }
}

// out[t] = sum over j, in this order, of weights[t, j] y[place[t, j]].
template <typename T, int LANES, bool WEIGHTS>
__global__ __launch_bounds__(kThreads) void k_combine(const T *__restrict__ y, int64_t y_stride, int64_t rows,
                                                      int32_t k, int32_t cols, const int32_t *__restrict__ place,
                                                      const float *__restrict__ weights, T *__restrict__ out,
                                                      int64_t out_stride) {
  constexpr int V = 16 / sizeof(T);
  const int64_t t = (int64_t)workgroup() * (kThreads / LANES) + threadIdx.x / LANES;
  if (t >= rows) return;
  const int64_t total = rows * k;
  const int32_t *p = place + t * k;
  for (int32_t c = threadIdx.x % LANES * V; c < cols; c += LANES * V) {
    float sum[V] = {};
    const int left = cols - c;
    for (int32_t j = 0; j < k; ++j) {
      const int64_t from = p[j];
      if (from < 0 || from >= total) continue;
      float v[V];
      if (left >= V)
        load_span(y + from * y_stride + c, v);
      else
        load_part(y + from * y_stride + c, left, v);
      const float w = WEIGHTS ? weights[t * k + j] : 1.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = WEIGHTS ? fmaf(w, v[i], sum[i]) : sum[i] + v[i];
    }
    if (left >= V)
      store_span(out + t * out_stride + c, sum);
    else
      store_part(out + t * out_stride + c, left, sum);
  }
}

// dy[place[t, j]] = weights[t, j] dout[t], zeros in rows that no entry is sorted
// to; dweights[t, j] = the dot product of dout[t] and y[place[t, j]].
template <typename T, int LANES>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const T *__restrict__ dout, int64_t dout_stride,
                                                               const T *__restrict__ y, int64_t y_stride, int64_t rows,
                                                               int32_t k, int32_t cols,
                                                               const int32_t *__restrict__ place,
                                                               const int32_t *__restrict__ source,
                                                               const float *__restrict__ weights, T *__restrict__ dy,
                                                               int64_t dy_stride, float *__restrict__ dweights) {
  constexpr int V = 16 / sizeof(T);
  const int64_t t = (int64_t)workgroup() * (kThreads / LANES) + threadIdx.x / LANES;
  if (t >= rows) return;
  const int lane = threadIdx.x % LANES;
  const int64_t total = rows * k;
  for (int32_t j = 0; j < k; ++j) {
    const int64_t at = place[t * k + j];
    const bool there = at >= 0 && at < total, clear = dy && source[t * k + j] < 0;
    const float w = weights ? weights[t * k + j] : 1.0f;
    float dot = 0.0f;
    for (int32_t c = lane * V; c < cols; c += LANES * V) {
      const int left = cols - c;
      if (there) {
        float d[V];
        if (left >= V)
          load_span(dout + t * dout_stride + c, d);
        else
          load_part(dout + t * dout_stride + c, left, d);
        if (dweights) {
          float v[V];
          if (left >= V)
            load_span(y + at * y_stride + c, v);
          else
            load_part(y + at * y_stride + c, left, v);
#pragma unroll
          for (int i = 0; i < V; ++i) dot = fmaf(d[i], v[i], dot);
        }
        if (dy) {
#pragma unroll
          for (int i = 0; i < V; ++i) d[i] *= w;
          if (left >= V)
            store_span(dy + at * dy_stride + c, d);
          else
            store_part(dy + at * dy_stride + c, left, d);
        }
      }
      if (clear) {
        const float none[V] = {};
        if (left >= V)
          store_span(dy + (t * k + j) * dy_stride + c, none);
        else
          store_part(dy + (t * k + j) * dy_stride + c, left, none);
      }
    }
    if (dweights) {
#pragma unroll
      for (int d = LANES / 2; d > 0; d /= 2) dot += __shfl_xor(dot, d);
      if (lane == 0) dweights[t * k + j] = dot;
    }
  }
}

// Calls f with the number of lanes for rows of `cols` elements: a power of two up to a wave.
template <typename T, typename F>
int with_lanes(int64_t cols, const F &f) {
  const int64_t steps = ceil_div(cols * (int64_t)sizeof(T), 16);
  if (steps > 32) return f(std::integral_constant<int, 64>());
  if (steps > 16) return f(std::integral_constant<int, 32>());
  if (steps > 8) return f(std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 8>());
}

template <typename T>
int dispatch_as(const sd_route_t *r, const void *x, int64_t cols, int64_t x_stride, void *y, int64_t y_stride,
                hipStream_t s) {
  return with_lanes<T>(cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_dispatch<T, L>), grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s,
                       static_cast<const T *>(x), x_stride, r->rows, r->k, (int32_t)cols, r->place, r->source,
                       static_cast<T *>(y), y_stride);
    return launched();
  });
}
template <typename T>
int combine_as(const sd_route_t *r, const void *y, int64_t cols, int64_t y_stride, const float *weights, void *out,
               int64_t out_stride, hipStream_t s) {
  return with_lanes<T>(cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    auto *kernel = weights ? k_combine<T, L, true> : k_combine<T, L, false>;
    hipLaunchKernelGGL(kernel, grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s,
                       static_cast<const T *>(y), y_stride, r->rows, r->k, (int32_t)cols, r->place, weights,
                       static_cast<T *>(out), out_stride);
    return launched();
  });
}
template <typename T>
int backward_as(const sd_route_t *r, const void *dout, int64_t cols, int64_t dout_stride, const void *y,
                int64_t y_stride, const float *weights, void *dy, int64_t dy_stride, float *dweights, hipStream_t s) {
  return with_lanes<T>(cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_combine_backward<T, L>), grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s,
                       static_cast<const T *>(dout), dout_stride, static_cast<const T *>(y), y_stride, r->rows, r->k,
                       (int32_t)cols, r->place, r->source, weights, static_cast<T *>(dy), dy_stride, dweights);
    return launched();
  });
}

}  // namespace

extern "C" int sd_route_size(int64_t rows, int32_t k, int32_t experts, size_t *bytes) {
  if (!bytes || rows < 0 || k < 1 || experts < 1) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || rows * k > kMaxRows) return SD_ERR_OVERFLOW;
  if (experts > kMaxExperts) return SD_ERR_UNSUPPORTED;
  const int64_t entries = rows * k;
  *bytes = entries == 0 || few(entries, experts)
               ? 0
               : (size_t)((ceil_div(entries, run_of(entries)) + 1) * (experts + 1) * 4 + 15) / 16 * 16;
  return SD_OK;
}

extern "C" int sd_route(const void *chosen, int32_t index_bytes, const sd_route_t *out, void *workspace, size_t bytes,
                        void *stream) {
  int st = check_route(out);
  if (st != SD_OK) return st;
  size_t need = 0;
  if ((st = sd_route_size(out->rows, out->k, out->experts, &need)) != SD_OK) return st;
  if (index_bytes != 4 && index_bytes != 8) return SD_ERR_INVALID_VALUE;
  const int64_t entries = out->rows * out->k;
  if (entries > 0 && (!chosen || !aligned_to(chosen, index_bytes))) return SD_ERR_INVALID_VALUE;
  if (need > 0 && (!workspace || bytes < need || !aligned_to(workspace, 16))) return SD_ERR_INVALID_VALUE;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int wide = index_bytes == 8, kinds = out->experts + 1;
  if (entries == 0) {
    hipLaunchKernelGGL(k_route_none, dim3(1), dim3(256), 0, s, out->offsets, out->experts);
    return launched();
  }
  int bits = 0;
  while ((1 << bits) < kinds) ++bits;
  if (few(entries, out->experts)) {
    const int64_t run = ceil_div(ceil_div(entries, kWaves), 64) * 64;
    hipLaunchKernelGGL(k_route_few, dim3(1), dim3(kWaves * 64), (size_t)kWaves * kinds * 4, s, chosen, wide, entries,
                       out->k, out->experts, bits, out->offsets, out->place, out->source, run);
    return launched();
  }
  const int64_t run = run_of(entries);
  const int32_t runs = (int32_t)ceil_div(entries, run);
  uint32_t *counts = static_cast<uint32_t *>(workspace), *totals = counts + (int64_t)kinds * runs;
  const uint32_t wgs = (uint32_t)ceil_div(runs, 4);
  const size_t lds = (size_t)4 * kinds * 4;
  hipLaunchKernelGGL(k_route_count, dim3(wgs), dim3(256), lds, s, chosen, wide, entries, out->experts, counts, run,
                     runs);
  if ((st = launched()) != SD_OK) return st;
  hipLaunchKernelGGL(k_route_sum, dim3((uint32_t)kinds), dim3(1024), 0, s, counts, runs, totals);
  if ((st = launched()) != SD_OK) return st;
  hipLaunchKernelGGL(k_route_place, dim3(wgs), dim3(256), lds, s, chosen, wide, entries, out->k, out->experts, bits,
                     counts, totals, run, runs, out->offsets, out->place, out->source);
  return launched();
}

extern "C" int sd_dispatch(const sd_route_t *route, const void *x, int32_t type, int64_t cols, int64_t x_stride,
                           void *y, int64_t y_stride, void *stream) {
  int st = check_route(route);
  if (st != SD_OK) return st;
  if (cols < 0) return SD_ERR_INVALID_VALUE;
  if (cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if ((st = check_table(x, type, route->rows, cols, x_stride)) != SD_OK) return st;
  if ((st = check_table(y, type, route->rows * route->k, cols, y_stride)) != SD_OK) return st;
  if (route->rows == 0 || cols == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? dispatch_as<float>(route, x, cols, x_stride, y, y_stride, s)
         : type == SD_TYPE_F16 ? dispatch_as<f16>(route, x, cols, x_stride, y, y_stride, s)
                               : dispatch_as<bf16>(route, x, cols, x_stride, y, y_stride, s);
}

extern "C" int sd_combine(const sd_route_t *route, const void *y, int32_t type, int64_t cols, int64_t y_stride,
                          const float *weights, void *out, int64_t out_stride, void *stream) {
  int st = check_route(route);
  if (st != SD_OK) return st;
  if (cols < 0) return SD_ERR_INVALID_VALUE;
  if (cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if ((st = check_table(y, type, route->rows * route->k, cols, y_stride)) != SD_OK) return st;
  if ((st = check_table(out, type, route->rows, cols, out_stride)) != SD_OK) return st;
  if (weights && !aligned_to(weights, 4)) return SD_ERR_INVALID_VALUE;
  if (route->rows == 0 || cols == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? combine_as<float>(route, y, cols, y_stride, weights, out, out_stride, s)
         : type == SD_TYPE_F16 ? combine_as<f16>(route, y, cols, y_stride, weights, out, out_stride, s)
                               : combine_as<bf16>(route, y, cols, y_stride, weights, out, out_stride, s);
}

extern "C" int sd_combine_backward(const sd_route_t *route, const void *dout, int32_t type, int64_t cols,
                                   int64_t dout_stride, const void *y, int64_t y_stride, const float *weights,
                                   void *dy, int64_t dy_stride, float *dweights, void *stream) {
  int st = check_route(route);
  if (st != SD_OK) return st;
  if (cols < 0) return SD_ERR_INVALID_VALUE;
  if (cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  const int64_t total = route->rows * route->k;
  if ((st = check_table(dout, type, route->rows, cols, dout_stride)) != SD_OK) return st;
  if (dweights && (st = check_table(y, type, total, cols, y_stride)) != SD_OK) return st;
  if (dy && (st = check_table(dy, type, total, cols, dy_stride)) != SD_OK) return st;
  if ((weights && !aligned_to(weights, 4)) || (dweights && !aligned_to(dweights, 4))) return SD_ERR_INVALID_VALUE;
  if (total == 0 || (!dweights && (!dy || cols == 0))) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32
             ? backward_as<float>(route, dout, cols, dout_stride, y, y_stride, weights, dy, dy_stride, dweights, s)
         : type == SD_TYPE_F16
             ? backward_as<f16>(route, dout, cols, dout_stride, y, y_stride, weights, dy, dy_stride, dweights, s)
             : backward_as<bf16>(route, dout, cols, dout_stride, y, y_stride, weights, dy, dy_stride, dweights, s);
}
