// Shared by the dense operators' translation units: element types, unaligned
// vector access, the 8-bit formats, and argument checks.  Nothing here is part
// of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "sd_internal.h"

namespace dense {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;  // columns that share a scale
constexpr int64_t kMaxRows = (1ll << 31) - 1;

inline int64_t blocks_of(int64_t cols) { return (cols + kBlock - 1) / kBlock; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// N elements of T at any address that T's own alignment allows: gfx950 takes
// wide loads and stores at element alignment.
template <typename T, int N, int ALIGN = sizeof(T)>
struct __attribute__((packed, aligned(ALIGN))) Span {
  T v[N];
};

template <int N, typename T>
__device__ inline void load_span(const T *p, float (&out)[N]) {
  const Span<T, N> s = *reinterpret_cast<const Span<T, N> *>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = (float)s.v[i];
}
// The first `count` of N elements; zero for the others.
template <int N, typename T>
__device__ inline void load_part(const T *p, int count, float (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = i < count ? (float)p[i] : 0.0f;
}
// v rounded to T from its 32 bits.  Without the barrier the compiler may fuse the
// operation that makes v with an f16 rounding in some places and not in others,
// and one value would round differently from call to call.
template <typename T>
__device__ inline T rounded(float v) {
  if constexpr (__is_same(T, f16)) asm("" : "+v"(v));
  return (T)v;
}
template <int N, typename T>
__device__ inline void store_span(T *p, const float (&in)[N]) {
  Span<T, N> s;
#pragma unroll
  for (int i = 0; i < N; ++i) s.v[i] = rounded<T>(in[i]);
  *reinterpret_cast<Span<T, N> *>(p) = s;
}
// The same past the caches, for tables that are larger than them: what is read
// next then stays where it is.
template <int N, typename T>
__device__ inline void stream_span(T *p, const float (&in)[N]) {
  constexpr int WORDS = N * sizeof(T) / 4;
  typedef uint32_t words __attribute__((ext_vector_type(WORDS), aligned(sizeof(T))));
  Span<T, N> s;
#pragma unroll
  for (int i = 0; i < N; ++i) s.v[i] = rounded<T>(in[i]);
  words w;
  __builtin_memcpy(&w, &s, sizeof(w));
  __builtin_nontemporal_store(w, reinterpret_cast<words *>(p));
}
template <int N, typename T>
__device__ inline void store_part(T *p, int count, const float (&in)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < count) p[i] = rounded<T>(in[i]);
}

// ---- 8-bit formats.  A block's scale is 2^(s - 127), s its byte: the least
// power of two that brings the largest finite magnitude to at most 1.75 * 2^8
// (e4m3) or 1.75 * 2^15 (e5m2).  Powers of two multiply exactly, so the codes
// follow from the values alone. ----
template <int FMT>
__device__ inline uint32_t scale_byte(uint32_t max_bits) {
  if (max_bits == 0) return 127;
  const int e = (int)(max_bits >> 23) - (FMT == SD_PACK_E4M3 ? 8 : 15) + ((max_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;
}
// 2^(127 - s); s comes from scale_byte (at most 247).
__device__ inline float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127) for s in [0, 254].
__device__ inline float scale_value(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }

template <int FMT>
__device__ inline uint32_t encode4(float a, float b, float c, float d) {
  int w;
  if constexpr (FMT == SD_PACK_E4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
  }
  return (uint32_t)w;
}
// The four codes of w, unscaled.
template <int FMT>
__device__ inline void decode4(uint32_t w, float (&out)[4]) {
  f32x2 lo, hi;
  if constexpr (FMT == SD_PACK_E4M3) {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
  }
  out[0] = lo[0];
  out[1] = lo[1];
  out[2] = hi[0];
  out[3] = hi[1];
}

// Two of w's codes, the lower or the upper ones, times the scale s.
template <int FMT>
__device__ inline bf16x2 to_bf16(uint32_t w, float s, bool hi) {
  if constexpr (FMT == SD_PACK_E4M3)
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
  else
    return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true)
              : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false);
}

// v of another lane: quad_perm and mirror forms of the data-parallel primitives.
template <int CTRL>
__device__ inline float dpp(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Largest value over aligned groups of `width` lanes (a power of two up to 32);
// NaN counts as nothing.  Each step takes the largest of another half that
// already agrees within itself: pairs, quads, mirrored halves of 8 and 16, and
// 16 lanes swapped against their neighbours.
__device__ inline float group_max(float v, int width) {
  if (width >= 2) v = fmaxf(v, dpp<0xb1>(v));
  if (width >= 4) v = fmaxf(v, dpp<0x4e>(v));
  if (width >= 8) v = fmaxf(v, dpp<0x141>(v));
  if (width >= 16) v = fmaxf(v, dpp<0x140>(v));
  if (width >= 32) {
    const uint32_t b = __float_as_uint(v);
    const u32x2 p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return v;
}
// The largest finite magnitude of the first `count` of N values in each lane of
// groups of `width` lanes, as its bits.
template <int N>
__device__ inline uint32_t largest_finite(const float (&v)[N], int count, int width) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = fmaxf(most, i < count ? fabsf(v[i]) : 0.0f);
  most = group_max(most, width);
  if (__any(__float_as_uint(most) >= 0x7f800000u)) {  // an infinity somewhere in the wave: once more without them
    most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
      most = fmaxf(most, i < count && (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u ? fabsf(v[i]) : 0.0f);
    most = group_max(most, width);
  }
  return __float_as_uint(most);
}

// What a wave's lanes wrote to shared memory before is there for all of them after it, and what they read
// before has been read: the unit takes a wave's accesses in order, so this is no instruction, only the order
// that the compiler keeps to.
__device__ inline void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Workgroup b of n as a place in a list of which each of the eight XCDs takes a
// contiguous run: workgroups go to the XCDs in turn, and neighbours in the list
// then share an L2.
__device__ inline uint32_t xcd_place(uint32_t b, uint32_t n) {
  const uint32_t x = b & 7, j = b >> 3, whole = n >> 3, more = n & 7;
  return x * whole + (x < more ? x : more) + j;
}

// This workgroup's number in a grid of grid_of().
__device__ inline uint32_t workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

// ------------------------------------------------------------ host side ---
// A launch holds fewer than 2^32 threads along a dimension: workgroups (of at most
// 1024 threads, fewer than 2^31 of them) past 2^21 go along a second one.  The last
// row of such a grid has some too many, which find no work.
inline dim3 grid_of(int64_t wgs) {
  constexpr int64_t kAlong = 1 << 21;
  return wgs <= kAlong ? dim3((uint32_t)wgs) : dim3((uint32_t)kAlong, (uint32_t)ceil_div(wgs, kAlong));
}
inline bool type_ok(int32_t t) { return t == SD_TYPE_F32 || t == SD_TYPE_F16 || t == SD_TYPE_BF16; }
inline int64_t type_bytes(int32_t t) { return t == SD_TYPE_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// A packed matrix's own fields; pointers may be null where there are no codes.
inline int check_packed(const sd_packed_t *p) {
  if (!p || p->rows < 0 || p->cols < 0 || (p->format != SD_PACK_E4M3 && p->format != SD_PACK_E5M2) ||
      p->reserved != 0)
    return SD_ERR_INVALID_VALUE;
  if (p->rows > kMaxRows || p->cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if (p->ld % 16 != 0 || p->ld < ceil_div(p->cols, 16) * 16) return SD_ERR_INVALID_VALUE;
  if (p->ld > (1ll << 40)) return SD_ERR_OVERFLOW;
  if (p->rows > 0 && p->cols > 0 && (!p->codes || !p->scales || !aligned_to(p->codes, 16)))
    return SD_ERR_INVALID_VALUE;
  return SD_OK;
}
// Rows of `cols` elements, `stride` elements apart, at a pointer of its type's alignment.
inline int check_table(const void *p, int32_t type, int64_t rows, int64_t cols, int64_t stride) {
  if (!type_ok(type)) return SD_ERR_INVALID_VALUE;
  if (rows == 0 || cols == 0) return SD_OK;
  if (!p || !aligned_to(p, type_bytes(type)) || (rows > 1 && stride < cols)) return SD_ERR_INVALID_VALUE;
  if (stride > INT32_MAX) return SD_ERR_OVERFLOW;
  return SD_OK;
}
// SD_ERR_NO_DEVICE without a GPU, SD_OK else.  Asked until there is one.
inline int have_device() {
  static bool found = false;
  if (__atomic_load_n(&found, __ATOMIC_RELAXED)) return SD_OK;
  int count = 0;
  if (hipGetDeviceCount(&count) != hipSuccess || count <= 0) {
    (void)hipGetLastError();
    return SD_ERR_NO_DEVICE;
  }
  __atomic_store_n(&found, true, __ATOMIC_RELAXED);
  return SD_OK;
}
inline int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SD_OK : sd::report_hip_error((int)e);
}
// Compute units of the current device (256 where it cannot be asked).
int cu_count();

}  // namespace dense
