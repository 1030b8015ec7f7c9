// sd_route, sd_dispatch, sd_combine: entries (row t, slot j) sorted by the expert
// that each was given, the rows brought there and the results brought back.
//
// A stable counting sort: position(t, j) = offsets[e] + the number of entries of
// expert e before (t, j).  Entries without an expert are one more kind behind the
// last.  A wave counts a run of neighbouring entries 64 at a time; lanes of equal
// kind find each other with one ballot for each bit of the kind, and a lane's rank
// among them is the number of such lanes before it.  Nothing depends on the order
// in which waves run.  Up to 8192 entries take one launch (74 entries 3.8 us, 8192
// 10), more three (calls in a row: 2^19 entries of 8 experts 13 us, 2^22 33; as the
// first of a pass, with entries from memory, 2^15 to 2^19 take 17 to 20): latency of
// launches and loads, the entries' bytes would take 2 and 13.
#include <type_traits>

#include "nibble.h"

namespace {

using namespace nibble;

constexpr int64_t kMaxRuns = 4096;    // runs of entries that are counted apart
constexpr int64_t kRun = 512;         // entries of a run at least
constexpr int64_t kOneGroup = 8192;   // entries that one workgroup sorts by itself: 10 us; 16384 take 17, three launches 12
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

// A wave's run of entries [begin, end), 64 at a time, kinds read ahead for kAhead such steps.
constexpr int kAhead = 8;
struct Kinds {
  uint32_t v[kAhead];
};
__device__ inline Kinds read_kinds(const void *chosen, int wide, uint32_t experts, int64_t first, int64_t end) {
  const int64_t i = first + (threadIdx.x & 63);
  Kinds k;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) k.v[u] = i + u * 64 < end ? kind_of(chosen, wide, i + u * 64, experts) : 0u;
  return k;
}
// Counts of each kind among the entries from `first` on.  Atomics of shared memory, also where eight experts
// put them behind each other: finding equals first took 14 us instead of 12 for 16384 entries and more.
__device__ inline void count_kinds(const Kinds &k, int64_t first, int64_t end, uint32_t *counts) {
  const int64_t i = first + (threadIdx.x & 63);
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (i + u * 64 < end) atomicAdd(&counts[k.v[u]], 1u);
}
// Their positions: next[kind] is the position of its next entry.
__device__ inline void place_kinds(const Kinds &kinds, uint32_t experts, int bits, int32_t k, int64_t first,
                                   int64_t end, uint32_t *next, int32_t *place, int32_t *source) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    if (first + u * 64 >= end) break;  // the same for the wave
    const int64_t i = first + u * 64 + lane;
    const uint32_t kind = kinds.v[u];
    const bool there = i < end;
    const uint64_t same = same_kind(kind, bits, there);
    if (there) {
      const int before = __popcll(same & ((1ull << lane) - 1));
      const uint32_t at = next[kind] + (uint32_t)before;
      wave_order();  // every lane has read before one writes
      if (before == 0) next[kind] = at + (uint32_t)__popcll(same);
      const bool kept = kind < experts;
      place[i] = kept ? (int32_t)at : -1;
      source[at] = kept ? (int32_t)((uint32_t)i / (uint32_t)k) : -1;
    }
    wave_order();  // and it has been written before one reads again
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

// All of it in one launch, for few entries: a wave's run is what it reads ahead.
static_assert(kOneGroup <= (int64_t)kWaves * 64 * kAhead);
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
  const Kinds own = read_kinds(chosen, wide, experts, begin, end);  // the whole run
  count_kinds(own, begin, end, mine);
  __syncthreads();
  const int kind = threadIdx.x;
  uint32_t c[kWaves], total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) c[w] = kind < kinds ? few_lds[w * kinds + kind] : 0u;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) total += c[w];
  uint32_t at = sum_before(total, sums);
  if (kind < kinds) {
    offsets[kind] = (int32_t)at;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      few_lds[w * kinds + kind] = at;
      at += c[w];
    }
  }
  __syncthreads();
  place_kinds(own, experts, bits, k, begin, end, mine, place, source);
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
  for (int64_t first = begin; first < end; first += 64 * kAhead)
    count_kinds(read_kinds(chosen, wide, experts, first, end), first, end, count_lds + wave * kinds);
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * kinds; i += 256)
    if (r0 + i % 4 < runs) counts[(int64_t)(i / 4) * runs + r0 + i % 4] = count_lds[i % 4 * kinds + i / 4];
}
// A workgroup of 1024 for each kind: its counts become sums over the runs before,
// and their sum.
__global__ __launch_bounds__(1024) void k_route_sum(uint32_t *__restrict__ counts, int32_t runs,
                                                    uint32_t *__restrict__ totals) {
  constexpr int EACH = kMaxRuns / 1024;
  __shared__ uint32_t sums[16];
  uint32_t *mine = counts + (int64_t)blockIdx.x * runs;
  const int first = threadIdx.x * EACH;
  uint32_t v[EACH], own = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) v[i] = first + i < runs ? mine[first + i] : 0u;
#pragma unroll
  for (int i = 0; i < EACH; ++i) own += v[i];
  uint32_t at = sum_before(own, sums);
  if (threadIdx.x == 1023) totals[blockIdx.x] = at + own;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (first + i < runs) mine[first + i] = at;
    at += v[i];
  }
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
  // every kind's first position, 256 kinds at a time
  uint32_t before = 0;
  for (int first = 0; first < kinds; first += 256) {
    const int kind = first + threadIdx.x;
    const uint32_t own = kind < kinds ? totals[kind] : 0u;
    const uint32_t *c = counts + (int64_t)kind * runs + blockIdx.x * 4;
    uint32_t runs_before[4];
#pragma unroll
    for (int w = 0; w < 4; ++w)
      runs_before[w] = kind < kinds && (int32_t)(blockIdx.x * 4) + w < runs ? c[w] : 0u;
    const uint32_t at = before + sum_before(own, sums);
    if (kind < kinds) {
      if (blockIdx.x == 0) offsets[kind] = (int32_t)at;
#pragma unroll
      for (int w = 0; w < 4; ++w) place_lds[w * kinds + kind] = at + runs_before[w];
    }
    before += sums[0] + sums[1] + sums[2] + sums[3];
    __syncthreads();  // the sums are free again
  }
  __syncthreads();
  const int64_t begin = (int64_t)(blockIdx.x * 4 + wave) * run, end = begin + run < entries ? begin + run : entries;
  for (int64_t first = begin; first < end; first += 64 * kAhead)
    place_kinds(read_kinds(chosen, wide, experts, first, end), experts, bits, k, first, end, place_lds + wave * kinds,
                place, source);
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
// A team of LANES lanes for each row t; 16 bytes of it a lane and step.  Entries
// are taken KB at a time, whose rows are read (or written) together; with k <= KB
// their places are read once.  A step takes V columns, the 16 bytes or, of shorter
// rows, the most that they have; a row's last step begins V columns before its end and
// does some columns twice, with the same results.
constexpr int kThreads = 256;

// The team's row and place in it, and the places of entries (t, j0 ..), -1 for none.
template <int LANES>
struct Team {
  int64_t t;
  int lane;
  __device__ Team() : t((int64_t)workgroup() * (kThreads / LANES) + threadIdx.x / LANES), lane(threadIdx.x % LANES) {}
};
template <int KB>
struct Places {
  int32_t at[KB];
  __device__ void read(const int32_t *place, int64_t t, int32_t k, int32_t j0, int64_t total) {
#pragma unroll
    for (int u = 0; u < KB; ++u) {
      const int32_t p = j0 + u < k ? place[t * k + j0 + u] : -1;
      at[u] = p < total ? p : -1;
    }
  }
};
// y[place[t, j]] = x[t]; rows of y that no entry is sorted to (those behind the
// last expert's) become zeros.  Bound by the bytes, each row of x read once: 2^18 x
// 128 fp32 to two experts each take 70 us, 5.8 TB/s with what the caches serve.
template <typename T, int LANES, int KB, int V>
__global__ __launch_bounds__(kThreads) void k_dispatch(const T *__restrict__ x, int64_t x_stride, int64_t rows,
                                                       int32_t k, int32_t cols, const int32_t *__restrict__ place,
                                                       const int32_t *__restrict__ source, T *__restrict__ y,
                                                       int64_t y_stride) {
  const Team<LANES> team;
  const int64_t t = team.t;
  if (t >= rows) return;
  Places<KB> p;
  uint32_t clear = 0;
  auto read = [&](int32_t j0) {
    p.read(place, t, k, j0, rows * k);
    clear = 0;
#pragma unroll
    for (int u = 0; u < KB; ++u) clear |= (j0 + u < k && source[t * k + j0 + u] < 0 ? 1u : 0u) << u;
  };
  if (k <= KB) read(0);
  for (int32_t c0 = team.lane * V; c0 < cols; c0 += LANES * V) {
    const int32_t c = c0 > cols - V ? cols - V : c0;
    float v[V];
    const float none[V] = {};
    load_span(x + t * x_stride + c, v);
    for (int32_t j0 = 0; j0 < k; j0 += KB) {
      if (k > KB) read(j0);
#pragma unroll
      for (int u = 0; u < KB; ++u)
        if (p.at[u] >= 0) store_span(y + p.at[u] * y_stride + c, v);
      if (clear) {
#pragma unroll
        for (int u = 0; u < KB; ++u)
          if (clear >> u & 1) store_span(y + (t * k + j0 + u) * y_stride + c, none);
      }
    }
  }
}

// out[t] = sum over j, in this order, of weights[t, j] y[place[t, j]].  Bound by the
// bytes: 83 us at those sizes (74 to 92), 4.9 TB/s.
template <typename T, int LANES, int KB, int V>
__global__ __launch_bounds__(kThreads) void k_combine(const T *__restrict__ y, int64_t y_stride, int64_t rows,
                                                      int32_t k, int32_t cols, const int32_t *__restrict__ place,
                                                      const float *__restrict__ weights, T *__restrict__ out,
                                                      int64_t out_stride) {
  const Team<LANES> team;
  const int64_t t = team.t;
  if (t >= rows) return;
  Places<KB> p;
  float w[KB];
  auto read = [&](int32_t j0) {
    p.read(place, t, k, j0, rows * k);
#pragma unroll
    for (int u = 0; u < KB; ++u) w[u] = weights && j0 + u < k ? weights[t * k + j0 + u] : 1.0f;
  };
  if (k <= KB) read(0);
  for (int32_t c0 = team.lane * V; c0 < cols; c0 += LANES * V) {
    const int32_t c = c0 > cols - V ? cols - V : c0;
    float sum[V] = {};
    for (int32_t j0 = 0; j0 < k; j0 += KB) {
      if (k > KB) read(j0);
      float v[KB][V];
#pragma unroll
      for (int u = 0; u < KB; ++u)
        if (p.at[u] >= 0) load_span(y + p.at[u] * y_stride + c, v[u]);
#pragma unroll
      for (int u = 0; u < KB; ++u)
        if (p.at[u] >= 0) {
#pragma unroll
          for (int i = 0; i < V; ++i) sum[i] = fmaf(w[u], v[u][i], sum[i]);
        }
    }
    store_span(out + t * out_stride + c, sum);
  }
}

// dy[place[t, j]] = weights[t, j] dout[t], zeros in rows that no entry is sorted
// to; dweights[t, j] = the dot product of dout[t] and y[place[t, j]].  One reading of
// dout and y serves both: 120 us at those sizes, 5.6 TB/s.
template <typename T, int LANES, int KB, int V>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const T *__restrict__ dout, int64_t dout_stride,
                                                               const T *__restrict__ y, int64_t y_stride, int64_t rows,
                                                               int32_t k, int32_t cols,
                                                               const int32_t *__restrict__ place,
                                                               const int32_t *__restrict__ source,
                                                               const float *__restrict__ weights, T *__restrict__ dy,
                                                               int64_t dy_stride, float *__restrict__ dweights) {
  const Team<LANES> team;
  const int64_t t = team.t;
  if (t >= rows) return;
  for (int32_t j0 = 0; j0 < k; j0 += KB) {
    Places<KB> p;
    p.read(place, t, k, j0, rows * k);
    uint32_t clear = 0;
    float w[KB], dot[KB] = {};
#pragma unroll
    for (int u = 0; u < KB; ++u) {
      w[u] = weights && j0 + u < k ? weights[t * k + j0 + u] : 1.0f;
      clear |= (dy && j0 + u < k && source[t * k + j0 + u] < 0 ? 1u : 0u) << u;
    }
    for (int32_t c0 = team.lane * V; c0 < cols; c0 += LANES * V) {
      const int32_t c = c0 > cols - V ? cols - V : c0;
      float d[V], v[KB][V];
      load_span(dout + t * dout_stride + c, d);
      if (dweights) {
#pragma unroll
        for (int u = 0; u < KB; ++u)
          if (p.at[u] >= 0) load_span(y + p.at[u] * y_stride + c, v[u]);
#pragma unroll
        for (int u = 0; u < KB; ++u)
          if (p.at[u] >= 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)  // columns that the step before has done count once
              if (c + i >= c0) dot[u] = fmaf(d[i], v[u][i], dot[u]);
          }
      }
      if (dy) {
#pragma unroll
        for (int u = 0; u < KB; ++u)
          if (p.at[u] >= 0) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = w[u] * d[i];
            store_span(dy + p.at[u] * dy_stride + c, o);
          }
        if (clear) {
          const float none[V] = {};
#pragma unroll
          for (int u = 0; u < KB; ++u)
            if (clear >> u & 1) store_span(dy + (t * k + j0 + u) * dy_stride + c, none);
        }
      }
    }
    if (dweights) {
#pragma unroll
      for (int u = 0; u < KB; ++u) {
#pragma unroll
        for (int s = LANES / 2; s > 0; s /= 2) dot[u] += __shfl_xor(dot[u], s);
        if (team.lane == 0 && j0 + u < k) dweights[t * k + j0 + u] = dot[u];
      }
    }
  }
}

// Calls f(lanes, entries at a time, columns of a step) for rows of `cols`
// elements: lanes for a whole row up to 32, then 64.  Measured in us (to the experts, back,
// gradients), calls in a row, whose rows the caches hold in part (with rows from memory
// 20011, 4, 601 bf16 take 32, 38 and 60):
//   rows, entries of each, columns     8 lanes       16           32           64
//   262144, 2, 128 fp32               82, 78, 136  75, 73, 125  76, 71, 119  104, 83, 146
//   262144, 2, 129 fp32             165, 121, 246 116, 92, 197  93, 81, 157  116, 94, 171
//   20011, 4, 601 bf16                32, 27, 63   27, 26, 55   24, 25, 47   23, 24, 49
//   100000, 8, 64 bf16                21, 24, 56   24, 32, 97   37, 56, 187
template <int MOST, typename T, typename F>
int with_shape(int64_t cols, int32_t k, const F &f) {
  constexpr int V = 16 / sizeof(T);
  const int64_t steps = ceil_div(cols, V);
  const auto entries = [&](auto l, auto v) {
    if (k == 1) return f(l, std::integral_constant<int, 1>(), v);
    if (k == 2) return f(l, std::integral_constant<int, 2>(), v);
    if (k <= 4 || MOST == 4) return f(l, std::integral_constant<int, 4>(), v);
    return f(l, std::integral_constant<int, MOST>(), v);
  };
  constexpr std::integral_constant<int, V> whole{};
  if (steps > 48) return entries(std::integral_constant<int, 64>(), whole);
  if (steps > 16) return entries(std::integral_constant<int, 32>(), whole);
  if (steps > 8) return entries(std::integral_constant<int, 16>(), whole);
  if (steps > 2) return entries(std::integral_constant<int, 8>(), whole);
  if (cols >= V) return entries(std::integral_constant<int, 2>(), whole);
  if (V == 8 && cols >= 4) return entries(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
  if (cols >= 2) return entries(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
  return entries(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
}

template <typename T>
int dispatch_as(const sd_route_t *r, const void *x, int64_t cols, int64_t x_stride, void *y, int64_t y_stride,
                hipStream_t s) {
  return with_shape<8, T>(cols, r->k, [&](auto lanes, auto kb, auto v) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_dispatch<T, L, decltype(kb)::value, decltype(v)::value>),
                       grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s, static_cast<const T *>(x),
                       x_stride, r->rows, r->k, (int32_t)cols, r->place, r->source, static_cast<T *>(y), y_stride);
    return launched();
  });
}
template <typename T>
int combine_as(const sd_route_t *r, const void *y, int64_t cols, int64_t y_stride, const float *weights, void *out,
               int64_t out_stride, hipStream_t s) {
  return with_shape<8, T>(cols, r->k, [&](auto lanes, auto kb, auto v) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_combine<T, L, decltype(kb)::value, decltype(v)::value>),
                       grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s, static_cast<const T *>(y),
                       y_stride, r->rows, r->k, (int32_t)cols, r->place, weights, static_cast<T *>(out), out_stride);
    return launched();
  });
}
template <typename T>
int backward_as(const sd_route_t *r, const void *dout, int64_t cols, int64_t dout_stride, const void *y,
                int64_t y_stride, const float *weights, void *dy, int64_t dy_stride, float *dweights, hipStream_t s) {
  return with_shape<4, T>(cols, r->k, [&](auto lanes, auto kb, auto v) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_combine_backward<T, L, decltype(kb)::value, decltype(v)::value>),
                       grid_of(ceil_div(r->rows, kThreads / L)), dim3(kThreads), 0, s, static_cast<const T *>(dout),
                       dout_stride, static_cast<const T *>(y), y_stride, r->rows, r->k, (int32_t)cols, r->place,
                       r->source, weights, static_cast<T *>(dy), dy_stride, dweights);
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
