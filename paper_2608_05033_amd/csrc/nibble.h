// The 4-bit format: e2m1 codes, two in a byte, and a power of two for each row
// and block of 32 columns.  Shared by the packing and the products.
#pragma once

#include "dense.h"

namespace nibble {

using namespace dense;

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kCols = 32;              // columns that share a scale: 16 bytes of codes
constexpr int kGroup = 128;             // columns whose four scale bytes lie together
constexpr uint32_t kNanScale = 255;     // a block that held a NaN or an infinity

inline int64_t col_blocks(int64_t cols) { return ceil_div(cols, kCols); }
inline int64_t groups_of(int64_t cols) { return ceil_div(cols, kGroup); }

// The scale's byte for a block whose largest magnitude has these bits: the least
// power of two with magnitude <= 6 = 1.5 * 2^2 times it, 2^-127 at least; 1 for
// zeros.  Infinities and NaN have the largest bits of all.
__device__ inline uint32_t scale_byte(uint32_t max_bits) {
  if (max_bits == 0) return 127;
  if (max_bits >= 0x7f800000u) return kNanScale;
  const int e = (int)(max_bits >> 23) - 2 + ((max_bits & 0x7fffffu) > 0x400000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;
}
// The codes of a and b over the scale s, in byte SEL of `old`; to nearest, ties to even.
template <int SEL>
__device__ inline uint32_t encode2(uint32_t old, float a, float b, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, s, SEL);
}
// Largest of aligned groups of `width` lanes (4 or 8).
__device__ inline uint32_t group_max_bits(uint32_t v, int width) {
  const auto step = [&](uint32_t o) { v = v > o ? v : o; };
  step(__float_as_uint(dpp<0xb1>(__uint_as_float(v))));
  step(__float_as_uint(dpp<0x4e>(__uint_as_float(v))));
  if (width >= 8) step(__float_as_uint(dpp<0x141>(__uint_as_float(v))));
  return v;
}

// A table's fields; pointers may be null where there are no codes.
inline int check_nibble(const sd_nibble_t *p) {
  if (!p || p->rows < 0 || p->cols < 0 || p->reserved != 0) return SD_ERR_INVALID_VALUE;
  if (p->rows > kMaxRows || p->cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if (p->ld % 16 != 0 || p->ld < col_blocks(p->cols) * 16) return SD_ERR_INVALID_VALUE;
  if (p->ld > (1ll << 40)) return SD_ERR_OVERFLOW;
  if (p->rows > 0 && p->cols > 0 &&
      (!p->codes || !p->scales || !aligned_to(p->codes, 16) || !aligned_to(p->scales, 4)))
    return SD_ERR_INVALID_VALUE;
  return SD_OK;
}
// A route's fields.
constexpr int32_t kMaxExperts = 4095;
inline int check_route(const sd_route_t *r) {
  if (!r || r->rows < 0 || r->k < 1 || r->experts < 1) return SD_ERR_INVALID_VALUE;
  if (r->rows > kMaxRows || r->rows * r->k > kMaxRows) return SD_ERR_OVERFLOW;
  if (r->experts > kMaxExperts) return SD_ERR_UNSUPPORTED;
  if (!r->offsets || !aligned_to(r->offsets, 4)) return SD_ERR_INVALID_VALUE;
  if (r->rows > 0 && (!r->place || !r->source || !aligned_to(r->place, 4) || !aligned_to(r->source, 4)))
    return SD_ERR_INVALID_VALUE;
  return SD_OK;
}

}  // namespace nibble
