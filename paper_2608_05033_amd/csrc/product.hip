// sd_pack_product: Y[m, n] = sum_k X(m, k) W(n, k) + bias[n] for two packed
// matrices, on the matrix units.
//
// A wave's 16 x 16 tile over one block of 128 k: lane (r, g) = (lane % 16,
// lane / 16) holds 32 codes of row r of each side, and its row's scale byte.
// Which 32 of the 128 a lane group holds does not matter as long as both sides
// agree, since one scale covers them all.  W is the first operand, so a lane
// ends with four neighbouring n of one row m and writes them in one store.
//
// The codes become bf16 with their scale (4 or 3 significant bits and a power of
// two: exact as far as bf16 reaches, to multiples of 2^-133), and
// v_mfma_f32_16x16x32_bf16 sums in 32 bits: 1.2e-7 of the result in 2-norm on
// normal values.  The matrix units' 8-bit forms, scaled or not, run at twice the
// rate but are not used: in each run of 8 neighbouring k they drop what lies under
// 2^-13 of the run's largest product, taken by the codes' stored exponents.
// Measured, that is 1.5e-5 of the result on normal values, 2e-3 of the magnitudes
// summed where a run's codes differ widely, and all of a result that is left when
// larger terms cancel.
#include "tiles.h"

namespace {

using namespace dense;

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Operand {
  const uint8_t *codes, *scales;
  int64_t ld, rows;
};

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

// Chunks of 16 codes g and g + 4 of block kb of one row; zero past the row's last.
__device__ inline void load_frag(const Operand &p, int64_t row, int32_t kb, int g, int32_t k16, Frag &f) {
  const int32_t at = kb * kBlock + g * 16;
  const uint8_t *q = p.codes + row * p.ld + at;
  u32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
  if (at < k16) a = *reinterpret_cast<const u32x4 *>(q);
  if (at + 64 < k16) b = *reinterpret_cast<const u32x4 *>(q + 64);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f.v[i] = (int)a[i];
    f.v[4 + i] = (int)b[i];
  }
  f.s = p.scales[kb * p.rows + row];
}

// What stands in for the codes past a row's end.
__device__ __align__(16) uint8_t kZeros[16];

// MF x NF tiles of 16 x 16 by one workgroup, operands straight from memory: KW
// waves each take every KW-th block of k and join their sums in shared memory.
// Bound by the latency of the loads: one row of 4096 by 4096 x 4096 takes 6 us,
// 2.8 TB/s of W.
template <typename T, int XF, int WF, int MF, int NF, int KW>
__global__ __launch_bounds__(KW * 64) void k_product_rows(Operand X, Operand W,
                                                                         const float *__restrict__ bias,
                                                                         T *__restrict__ Y, int64_t stride,
                                                                         int32_t k16, int32_t nb, int32_t nt) {
  __shared__ f32x4 part[KW][MF * NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)(workgroup() / (uint32_t)nt) * (MF * 16);
  const int64_t n0 = (int64_t)(workgroup() % (uint32_t)nt) * (NF * 16);
  if (m0 >= X.rows) return;
  f32x4 acc[MF][NF] = {};
  int64_t xrow[MF], wrow[NF];  // rows past the last read the last one
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t row = m0 + i * 16 + r;
    xrow[i] = row < X.rows ? row : X.rows - 1;
  }
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int64_t row = n0 + col_of<kWoven<T, NF>>(j, r);
    wrow[j] = row < W.rows ? row : W.rows - 1;
  }
  auto load = [&](int32_t kb, Frag (&x)[MF], Frag (&w)[NF]) {
#pragma unroll
    for (int i = 0; i < MF; ++i) load_frag(X, xrow[i], kb, g, k16, x[i]);
#pragma unroll
    for (int j = 0; j < NF; ++j) load_frag(W, wrow[j], kb, g, k16, w[j]);
  };
  auto multiply = [&](const Frag (&x)[MF], const Frag (&w)[NF]) {
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
  };
  // the next block is on its way while this one's products run
  Frag x0[MF], w0[NF], x1[MF], w1[NF];
  int32_t kb = wave;
  if (kb < nb) load(kb, x0, w0);
  while (kb < nb) {
    if (kb + KW < nb) load(kb + KW, x1, w1);
    multiply(x0, w0);
    kb += KW;
    if (kb >= nb) break;
    if (kb + KW < nb) load(kb + KW, x0, w0);
    multiply(x1, w1);
    kb += KW;
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) part[wave][i * NF + j][lane] = acc[i][j];
  __syncthreads();
  // wave i adds up and writes row group i
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    if (i != wave) continue;
    f32x4 sum[1][NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      sum[0][j] = part[0][i * NF + j][lane];
#pragma unroll
      for (int t = 1; t < KW; ++t) sum[0][j] += part[t][i * NF + j][lane];
    }
    store_tiles<1, NF>(sum, m0 + i * 16, n0, X.rows, W.rows, bias, Y, stride);
  }
}

// BM x BN tiles (rows of X by rows of W), operands through shared memory: WM x WN
// waves, each (BM / WM) x (BN / WN).  Two buffers hold a block of 128 k each; the
// next block's codes go from memory straight to shared memory (16 bytes a lane)
// while this block's products run.  Rows lie 128 bytes apart, their eight 16-byte
// chunks mixed with the row so that 16 rows read at one chunk touch all banks;
// the mixing is done on the memory side, since a wave's 64 lanes write 1 KiB in
// order.  Scale bytes lie by lane, the tile's 16-row groups side by side, so one
// read serves all of a lane's products.  Bound by the matrix units and the
// conversions to bf16: 8192 cubed in 760 to 890 us, 1.3 PFLOP/s.
template <typename T, int XF, int WF, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64) void k_product_tile(Operand X, Operand W, const float *__restrict__ bias,
                                                              T *__restrict__ Y, int64_t stride, int32_t k16,
                                                              int32_t nb, int32_t mt, int32_t nt) {
  constexpr int THREADS = WM * WN * 64, MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int ROWS = BM + BN, CHUNKS = ROWS * 8 / THREADS;  // 16-byte chunks per thread and block
  static_assert(MF % 4 == 0 && NF % 4 == 0 && ROWS * 8 % THREADS == 0, "scales are read four at a time");
  // two objects and not an array of two: reads of one then need not wait for what is on its way to the other
  __shared__ __align__(16) uint8_t codes_a[ROWS * kBlock], codes_b[ROWS * kBlock];
  __shared__ __align__(16) uint8_t scales_a[16][ROWS / 16], scales_b[16][ROWS / 16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r = lane & 15, g = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;
  const uint32_t tiles = (uint32_t)mt * (uint32_t)nt;
  if (workgroup() >= tiles) return;
  const uint32_t at = xcd_place(workgroup(), tiles);
  // tiles in bands of 8 along m: neighbours in the list share X's and W's rows
  const uint32_t band = at / (8u * nt), left = mt - band * 8u < 8u ? mt - band * 8u : 8u;
  const uint32_t in_band = at - band * 8u * nt;
  const int64_t m0 = (int64_t)(band * 8u + in_band % left) * BM, n0 = (int64_t)(in_band / left) * BN;

  // Chunk i of thread t: row i * THREADS / 8 + t / 8 of the tile (X's rows first),
  // place t % 8.  Rows past the last read the last one.
  static_assert(THREADS % 128 == 0 && BM % (THREADS / 8) == 0, "one operand and one mixing for a thread's chunks");
  constexpr int XC = BM / (THREADS / 8);  // of them, chunks of X
  constexpr bool WOVEN = kWoven<T, NF>;
  // a row's chunks are mixed with 8 rows' worth of its place: bits 1 to 3, or for woven rows 1, 3 and 4
  const int xchunk = ((t & 7) ^ ((t >> 4) & 7)) * 16;
  const int wchunk = WOVEN ? ((t & 7) ^ (((t >> 4) & 1) | ((t >> 6) & 3) << 1)) * 16 : xchunk;
  const uint8_t *xbase = X.codes + m0 * X.ld, *wbase = W.codes + n0 * W.ld;
  uint32_t off[CHUNKS];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int row = (i < XC ? i : i - XC) * (THREADS / 8) + t / 8;
    const int64_t most = i < XC ? X.rows - 1 - m0 : W.rows - 1 - n0;
    off[i] = (uint32_t)(row < most ? row : most) * (uint32_t)(i < XC ? X.ld : W.ld) + (i < XC ? xchunk : wchunk);
  }
  const uint8_t *ssrc[(ROWS + THREADS - 1) / THREADS];
  int64_t sstep[(ROWS + THREADS - 1) / THREADS];
#pragma unroll
  for (int i = 0; i * THREADS < ROWS; ++i) {
    const int row = i * THREADS + t;
    const Operand &p = row < BM ? X : W;
    const int64_t want = row < BM ? m0 + row : n0 + row - BM, have = want < p.rows ? want : p.rows - 1;
    ssrc[i] = p.scales + have;
    sstep[i] = p.rows;
  }
  uint8_t sv[(ROWS + THREADS - 1) / THREADS];
  // 16 bytes a lane of block kb; past the rows' last 16 bytes, zeros.
  auto fetch_chunk = [&](int32_t kb, int i, uint8_t *codes) {
    const uint8_t *p = (i < XC ? xbase : wbase) + (int64_t)kb * kBlock + off[i];
    if ((i < XC ? xchunk : wchunk) >= k16 - kb * kBlock) p = kZeros;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(p),
                                     (__attribute__((address_space(3))) void *)(&codes[(i * THREADS + wave * 64) * 16]),
                                     16, 0, 0);
  };
  auto fetch_scales = [&](int32_t kb) {
#pragma unroll
    for (int i = 0; i * THREADS < ROWS; ++i)
      if (ROWS % THREADS == 0 || i * THREADS + t < ROWS) sv[i] = ssrc[i][kb * sstep[i]];
  };
  auto store_scales = [&](uint8_t (*scales)[ROWS / 16]) {
#pragma unroll
    for (int i = 0; i * THREADS < ROWS; ++i) {
      const int row = i * THREADS + t;
      if (ROWS % THREADS == 0 || row < ROWS) {
        const bool woven = WOVEN && row >= BM;
        const int rho = woven ? (row >> 3 & 3) * 4 + (row & 3) : row & 15;
        const int group = woven ? row >> 5 << 1 | (row >> 2 & 1) : row >> 4;
        scales[rho][group] = sv[i];
      }
    }
  };
  // A lane's two chunks of its row in a group of 16 rows: places g and g + 4, mixed.
  // The mixing of row r of a group of 16 is r / 2 in either order of rows.
  const int place = (g ^ ((r >> 1) & 7)) * 16;
  const int xlo = (wm * MF * 16 + r) * kBlock + place;
  const int wlo = (BM + wn * NF * 16 + col_of<WOVEN>(0, r)) * kBlock + place;
  auto frag = [&](const uint8_t *codes, int at, int row) {
    const u32x4 a = *reinterpret_cast<const u32x4 *>(codes + at + row * kBlock);
    const u32x4 b = *reinterpret_cast<const u32x4 *>(codes + (at ^ 64) + row * kBlock);
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f.v[i] = (int)a[i];
      f.v[4 + i] = (int)b[i];
    }
    return f;
  };

  f32x4 acc[MF][NF] = {};
  // One block's products from (codes, scales).  The next one is asked for a part at a time between
  // the products: a wave that asks for all of it at once waits until the last request is taken.
  auto step = [&](int32_t kb, const uint8_t *codes, const uint8_t (*scales)[ROWS / 16], uint8_t *codes_next,
                  uint8_t (*scales_next)[ROWS / 16]) {
    constexpr int PARTS = CHUNKS / (MF / 2);
    static_assert(CHUNKS % (MF / 2) == 0, "the first half of the products asks for the next block");
    const int32_t next = kb + 1 < nb ? kb + 1 : kb;  // after the last block: that one again, for nothing
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): what this wave asked for is in shared memory
    __syncthreads();                     // every wave's part of this block is there, the other buffer is free
    fetch_scales(next);
    uint32_t sx[MF / 4], sw[NF / 4];
#pragma unroll
    for (int i = 0; i < MF / 4; ++i) sx[i] = *reinterpret_cast<const uint32_t *>(&scales[r][wm * MF + 4 * i]);
#pragma unroll
    for (int i = 0; i < NF / 4; ++i) sw[i] = *reinterpret_cast<const uint32_t *>(&scales[r][BM / 16 + wn * NF + 4 * i]);
    Frag w[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      w[j] = frag(codes, wlo, col_of<WOVEN>(j, 0));
      w[j].s = (sw[j / 4] >> (8 * (j % 4))) & 255;
    }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      Frag x = frag(codes, xlo, i * 16);
      x.s = (sx[i / 4] >> (8 * (i % 4))) & 255;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x8 xb = bf16_of<XF>(x, q);
#pragma unroll
        for (int j = 0; j < NF; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of<WF>(w[j], q), xb, acc[i][j], 0, 0, 0);
      }
      if (i < MF / 2) {
#pragma unroll
        for (int q = 0; q < PARTS; ++q) fetch_chunk(next, i * PARTS + q, codes_next);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    store_scales(scales_next);
  };
  if (nb > 0) {
    fetch_scales(0);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) fetch_chunk(0, i, codes_a);
    store_scales(scales_a);
  }
  for (int32_t kb = 0; kb < nb; kb += 2) {
    step(kb, codes_a, scales_a, codes_b, scales_b);
    if (kb + 1 < nb) step(kb + 1, codes_b, scales_b, codes_a, scales_a);
  }
  __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing is on its way to shared memory when the workgroup ends
  store_tiles<MF, NF>(acc, m0 + wm * MF * 16, n0 + wn * NF * 16, X.rows, W.rows, bias, Y, stride);
}

// Long tables times few columns: all of W (up to NF * 16 columns of Y, kNarrowBlocks
// blocks of k) stays in shared memory, and each wave takes strips of 16 rows of X
// straight from memory, the next strip's codes on their way while this one's
// products run.  Bound by writing Y: 262144 x 128 x 128, 32-bit results, take 32 us,
// 5.2 TB/s.
constexpr int kNarrowBlocks = 4;
template <typename T, int XF, int WF, int NF>
__global__ __launch_bounds__(256) void k_product_narrow(Operand X, Operand W, const float *__restrict__ bias,
                                                        T *__restrict__ Y, int64_t stride, int32_t k16, int32_t nb,
                                                        int64_t strips) {
  constexpr int ROWS = NF * 16;
  constexpr bool WOVEN = kWoven<T, NF>;
  extern __shared__ __align__(16) uint8_t narrow_lds[];  // codes [nb][ROWS][128], then scales [nb][16][NF]
  uint8_t *codes = narrow_lds, *scales = narrow_lds + nb * ROWS * kBlock;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r = lane & 15, g = lane >> 4;
  for (int i = t; i < nb * ROWS * 8; i += 256) {
    const int place = i & 7, row = (i >> 3) % ROWS, kb = (i >> 3) / ROWS;
    const int rho = WOVEN ? (row >> 3 & 3) * 4 + (row & 3) : row & 15;
    const int at = (place ^ (rho >> 1)) * 16 + kb * kBlock;
    u32x4 v = {0, 0, 0, 0};
    if (row < W.rows && at < k16) v = *reinterpret_cast<const u32x4 *>(W.codes + row * W.ld + at);
    *reinterpret_cast<u32x4 *>(codes + i * 16) = v;
  }
  for (int i = t; i < nb * ROWS; i += 256) {
    const int j = i % NF, rho = i / NF % 16, kb = i / ROWS, row = col_of<WOVEN>(j, rho);
    scales[i] = row < W.rows ? W.scales[kb * W.rows + row] : 127;
  }
  __syncthreads();
  const int wlo = col_of<WOVEN>(0, r) * kBlock + (g ^ (r >> 1)) * 16;
  const int64_t step = (int64_t)gridDim.x * 4;
  auto load = [&](int64_t strip, int32_t kb) {
    const int64_t row = strip * 16 + r;
    Frag f;
    load_frag(X, row < X.rows ? row : X.rows - 1, kb, g, k16, f);
    return f;
  };
  int64_t strip = (int64_t)blockIdx.x * 4 + wave;
  if (strip >= strips) return;
  Frag next = load(strip, 0);
  for (; strip < strips; strip += step) {
    f32x4 acc[1][NF] = {};
    for (int32_t kb = 0; kb < nb; ++kb) {
      const Frag x = next;
      if (kb + 1 < nb)
        next = load(strip, kb + 1);
      else if (strip + step < strips)
        next = load(strip + step, 0);
      uint32_t sw[NF / 4];
#pragma unroll
      for (int i = 0; i < NF / 4; ++i) sw[i] = *reinterpret_cast<const uint32_t *>(scales + (kb * 16 + r) * NF + 4 * i);
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int p = wlo + (kb * ROWS + col_of<WOVEN>(j, 0)) * kBlock;
        const u32x4 a = *reinterpret_cast<const u32x4 *>(codes + p);
        const u32x4 b = *reinterpret_cast<const u32x4 *>(codes + (p ^ 64));
        Frag w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w.v[i] = (int)a[i];
          w.v[4 + i] = (int)b[i];
        }
        w.s = (sw[j / 4] >> (8 * (j % 4))) & 255;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of<WF>(w, q), bf16_of<XF>(x, q), acc[0][j], 0, 0, 0);
      }
    }
    store_tiles<1, NF>(acc, strip * 16, 0, X.rows, W.rows, bias, Y, stride);
  }
}

template <typename T, int XF, int WF, int NF>
int narrow_launch(const Operand &x, const Operand &w, const float *bias, T *y, int64_t stride, int32_t k16, int32_t nb,
                  hipStream_t s) {
  const int64_t strips = ceil_div(x.rows, 16), most = 8ll * cu_count();
  const int64_t wgs = ceil_div(strips, 4) < most ? ceil_div(strips, 4) : most;
  const size_t lds = (size_t)nb * NF * 16 * (kBlock + 1);
  hipLaunchKernelGGL((k_product_narrow<T, XF, WF, NF>), dim3((uint32_t)wgs), dim3(256), lds, s, x, w, bias, y, stride,
                     k16, nb, strips);
  return launched();
}

template <typename T, int XF, int WF, int MF, int NF, int KW>
int rows_launch(const Operand &x, const Operand &w, const float *bias, T *y, int64_t stride, int32_t k16, int32_t nb,
                hipStream_t s) {
  static_assert(MF <= KW, "a wave for each row group");
  const int64_t nt = ceil_div(w.rows, NF * 16), wgs = ceil_div(x.rows, MF * 16) * nt;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_product_rows<T, XF, WF, MF, NF, KW>), grid_of(wgs), dim3(KW * 64), 0, s, x, w, bias,
                     y, stride, k16, nb, (int32_t)nt);
  return launched();
}

template <typename T, int XF, int WF, int BM, int BN, int WM, int WN>
int tile_launch(const Operand &x, const Operand &w, const float *bias, T *y, int64_t stride, int32_t k16, int32_t nb,
                hipStream_t s) {
  const int64_t mt = ceil_div(x.rows, BM), nt = ceil_div(w.rows, BN);
  if (mt * nt > INT32_MAX) return SD_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_product_tile<T, XF, WF, BM, BN, WM, WN>), grid_of(mt * nt), dim3(WM * WN * 64), 0, s,
                     x, w, bias, y, stride, k16, nb, (int32_t)mt, (int32_t)nt);
  return launched();
}

template <typename T, int XF, int WF>
int product(const sd_packed_t *X, const sd_packed_t *W, const float *bias, void *Y, int64_t stride, hipStream_t s) {
  const Operand x{X->codes, X->scales, X->ld, X->rows}, w{W->codes, W->scales, W->ld, W->rows};
  const int32_t k16 = (int32_t)(ceil_div(X->cols, 16) * 16), nb = (int32_t)blocks_of(X->cols);
  T *y = static_cast<T *>(Y);
  // The largest tile that still gives three compute units in four a workgroup: a
  // larger tile reads less for each product, and with fewer workgroups than that
  // the sum over k is what takes time, so more waves have to share it.  Measured
  // in us, 16-bit results, this choice and its neighbours:
  //   rows x columns x k   256x256  128x128  64x64  32x64  32x32  16x16
  //   4096 x 4096 x 4096       104      156    308    417
  //   2048 x 2048 x 2048        49       24     52     64     79    120
  //   256 x 4096 x 4096         88       39     22     28     36     61
  //   4096 x 128 x 4096         87       38     23     16     20     33
  //   64 x 4096 x 4096          86       38     21     15     11     18
  //   1 x 4096 x 4096           86       38     18     12      8      7
  // 256 x 256 only where its edges cost little against 128 x 128: 300 columns of
  // 100000 rows (700 of k, 32-bit results) take 120 us with it and 76 us without.
  const int64_t enough = 3 * cu_count() / 4;
  const auto tiles = [&](int64_t bm, int64_t bn) { return ceil_div(x.rows, bm) * ceil_div(w.rows, bn); };
  // the large tiles keep row offsets in 32 bits
  const bool near = x.ld <= (1 << 23) && w.ld <= (1 << 23);
  if (near && tiles(256, 256) >= enough && 32 * tiles(256, 256) <= 9 * tiles(128, 128))
    return tile_launch<T, XF, WF, 256, 256, 2, 4>(x, w, bias, y, stride, k16, nb, s);
  // W in shared memory for long tables of few columns: 1000000 x 47 of 64 k, 32-bit
  // results, take 63 us so and 88 us with 128 x 128 tiles.  That kernel reads a block
  // ahead, so there has to be one.
  if (nb > 0 && nb <= kNarrowBlocks && w.rows <= 128 && x.rows >= 64 * enough)
    return w.rows <= 64 ? narrow_launch<T, XF, WF, 4>(x, w, bias, y, stride, k16, nb, s)
                        : narrow_launch<T, XF, WF, 8>(x, w, bias, y, stride, k16, nb, s);
  if (near && tiles(128, 128) >= enough)
    return tile_launch<T, XF, WF, 128, 128, 2, 2>(x, w, bias, y, stride, k16, nb, s);
  if (tiles(64, 64) >= enough) return rows_launch<T, XF, WF, 4, 4, 4>(x, w, bias, y, stride, k16, nb, s);
  if (tiles(32, 64) >= enough) return rows_launch<T, XF, WF, 2, 4, 8>(x, w, bias, y, stride, k16, nb, s);
  if (tiles(32, 32) >= enough) return rows_launch<T, XF, WF, 2, 2, 8>(x, w, bias, y, stride, k16, nb, s);
  return rows_launch<T, XF, WF, 1, 1, 8>(x, w, bias, y, stride, k16, nb, s);
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
