// sd_nibble_product: Y[m, n] = sum_k X(m, k) W(n, k) + bias[n] for two 4-bit
// tables, and sd_expert_product: the same where each row of Y is one row of X
// through the weights of the expert it was sorted to.
//
// The matrix unit takes a block of a row from each lane: its 32 codes in 16 bytes
// and its scale byte.  Few rows run products of 16 x 16 x 128 (16 rows, 4 blocks),
// large tiles of 32 x 32 x 64 (32 rows, 2 blocks).  W is the first operand, so a lane
// ends with runs of four neighbouring n of one row m.
//
// Products of e2m1 codes are multiples of 1/4 up to 36, so that the unit, which
// drops what lies far under the largest product of a run, drops nothing within a
// block: sums of blocks of one scale are exact.  Measured over random codes, one
// instruction is off by at most 2.1e-7 of the magnitudes summed, also where the
// blocks' scales differ by 2^80 or the sum so far is 10^6 times the products.
//
// With operands in registers the 32 x 32 form reaches 9.4 PFLOP/s on zeros and 6.7 on
// random codes, where power lets the clock fall to 1.65 GHz; the 16 x 16 form 6.9 on
// zeros.  6.7 is what the large products are held against.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "nibble.h"
#include "tiles.h"

namespace {

using namespace nibble;

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Operand {
  const uint8_t *codes, *scales;
  int64_t ld, rows;
};

// Rows of Y sorted by expert: those of expert e are offsets[e] .. offsets[e + 1] - 1
// and use rows e * n .. of W; the rows from offsets[experts] on are zeros.
struct Sorted {
  const int32_t *offsets, *source;  // source: X's row for each of Y's; null: X is sorted too
  int32_t experts;
  int64_t total;  // rows of Y
};

struct Frag {
  u32x4 v;
  uint32_t s;
};

__device__ inline f32x4 multiply(const Frag &w, const Frag &x, f32x4 acc) {
  const i32x8 a = {(int)w.v[0], (int)w.v[1], (int)w.v[2], (int)w.v[3], 0, 0, 0, 0};
  const i32x8 b = {(int)x.v[0], (int)x.v[1], (int)x.v[2], (int)x.v[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)w.s, 0, (int)x.s);
}

// Block 4 kg + g of one row; zeros past the last block.
__device__ inline void load_frag(const Operand &p, int64_t row, int32_t kg, int g, int32_t blocks, Frag &f) {
  f.v = u32x4{0, 0, 0, 0};
  f.s = 127;
  if (4 * kg + g < blocks) {
    f.v = *reinterpret_cast<const u32x4 *>(p.codes + row * p.ld + (4 * kg + g) * 16);
    f.s = p.scales[((int64_t)kg * p.rows + row) * 4 + g];
  }
}

// Which rows a tile of rows (BM rows each, the experts' one after the other, then the
// rows that have none) covers: [m0, m1) of Y, and its expert; expert -1: zeros; false:
// there is no such tile.  The tile is tile_of(tiles that there are), which are counted
// if COUNTED and given as 0 else.  For a whole wave, with the same results in all its
// lanes, kept in scalar registers.  Offsets are taken as far as they ascend within Y.
template <bool COUNTED, typename F>
__device__ inline bool find_tile(const Sorted &s, int bm, const F &tile_of, int64_t &m0, int64_t &m1,
                                 int32_t &expert) {
  const int lane = threadIdx.x & 63;
  const auto at = [&](int32_t e) {
    const int32_t o = s.offsets[e];
    return o < 0 ? 0 : o > s.total ? (int32_t)s.total : o;
  };
  // an expert's rows and tiles
  int32_t b, end;
  const auto own_of = [&](int32_t e) {
    b = end = 0;
    if (e <= s.experts) {
      b = at(e);
      end = e == s.experts ? (int32_t)s.total : at(e + 1);
    }
    return end > b ? ((uint32_t)(end - b) + bm - 1) / (uint32_t)bm : 0u;
  };
  // 64 experts, one a lane: its tiles, those up to its last; the sum of all
  uint32_t own, upto;
  const auto scan = [&](int32_t e0) {
    upto = own = own_of(e0 + lane);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = (uint32_t)__shfl_up((int)upto, d);
      if (lane >= d) upto += o;
    }
    return (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  };
  int32_t e0 = 0;
  uint32_t before = 0, whole, all = 0;
  if (COUNTED && s.experts >= 64) {
    uint32_t some = 0;
    for (int32_t e = lane; e <= s.experts; e += 64) some += own_of(e);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) some += (uint32_t)__shfl_xor((int)some, d);
    all = (uint32_t)__builtin_amdgcn_readfirstlane((int)some);
  }
  whole = scan(0);
  if (COUNTED && s.experts < 64) all = whole;
  const uint32_t tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)tile_of(all));
  while (tile >= before + whole) {
    before += whole;
    e0 += 64;
    if (e0 > s.experts) return false;
    whole = scan(e0);
  }
  const bool mine = tile < before + upto && tile >= before + upto - own;
  const int who = __ffsll((unsigned long long)__ballot(mine)) - 1;
  if (who < 0) return false;  // offsets that fall and rise until their sums pass 32 bits
  const int32_t lo = __builtin_amdgcn_readlane(b, who), hi = __builtin_amdgcn_readlane(end, who);
  const uint32_t first = before + (uint32_t)__builtin_amdgcn_readlane((int)(upto - own), who);
  expert = e0 + who < s.experts ? e0 + who : -1;
  m0 = lo + (int64_t)(tile - first) * bm;
  m1 = m0 + bm < hi ? m0 + bm : hi;
  return true;
}

// Zeros to rows [m0, m1) and columns [n0, n1) of Y, by the whole workgroup.
template <typename T>
__device__ inline void clear_rows(T *Y, int64_t stride, int64_t m0, int64_t m1, int64_t n0, int64_t n1) {
  const int64_t wide = n1 - n0;
  for (int64_t i = threadIdx.x; i < (m1 - m0) * wide; i += blockDim.x)
    Y[(m0 + i / wide) * stride + n0 + i % wide] = (T)0.0f;
}

// MF x NF tiles of 16 x 16 by one workgroup, operands straight from memory: KW
// waves each take every KW-th pair of groups of 128 k and join their sums in shared
// memory.  Lane (r, g) = (lane % 16, lane / 16) takes block g of a group of row r.
// Bound by the latency of the loads where there are few tiles: 1 x 4096 x 4096 takes
// 3.7 us with calls in a row (2.4 TB/s of W) and 4.4 with W from memory, the launch
// itself 2; by W's bytes where there are many: 16 rows through 8 of 64 experts of 1024 x
// 2048 take 15, 4.6 TB/s.
// ALONG: the waves take a tile each, KW neighbouring ones, and the whole sum.
template <typename T, int MF, int NF, int KW, bool EXPERTS, bool ALONG>
__global__ __launch_bounds__(KW * 64) void k_nibble_rows(Operand X, Operand W, Sorted sorted,
                                                         const float *__restrict__ bias, T *__restrict__ Y,
                                                         int64_t stride, int64_t rows, int64_t n, int32_t blocks,
                                                         int32_t ng, int32_t nt) {
  __shared__ f32x4 part[ALONG ? 1 : KW][MF * NF][64];
  constexpr int WIDE = NF * 16 * (ALONG ? KW : 1);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  int64_t m0 = (int64_t)(workgroup() / (uint32_t)nt) * (MF * 16), m1 = rows;
  const int64_t first = (int64_t)(workgroup() % (uint32_t)nt) * WIDE, n0 = first + (ALONG ? wave * NF * 16 : 0);
  int64_t w0 = 0;
  if constexpr (EXPERTS) {
    int32_t expert;
    const uint32_t tile = workgroup() / (uint32_t)nt;
    if (!find_tile<false>(sorted, MF * 16, [=](uint32_t) { return tile; }, m0, m1, expert)) return;
    if (expert < 0) {
      clear_rows(Y, stride, m0, m1, first, first + WIDE < n ? first + WIDE : n);
      return;
    }
    w0 = expert * n;
    if (bias) bias += w0;
  }
  if (m0 >= m1 || n0 >= n) return;
  f32x4 acc[MF][NF] = {};
  int64_t xrow[MF], wrow[NF];  // rows past the last read the last one
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    int64_t row = m0 + i * 16 + r;
    row = row < m1 ? row : m1 - 1;
    if constexpr (EXPERTS) {
      if (sorted.source) {
        const int64_t from = sorted.source[row];
        row = from < 0 ? 0 : from < X.rows ? from : X.rows - 1;
      }
    }
    xrow[i] = row;
  }
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int64_t row = n0 + col_of<kWoven<T, NF>>(j, r);
    wrow[j] = w0 + (row < n ? row : n - 1);
  }
  // Two neighbouring groups at a time, the whole line that holds them; the next two are on their way while
  // these ones' products run.
  struct Operands {
    Frag x[2][MF], w[2][NF];
  };
  auto load = [&](int32_t pair, Operands &o) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < MF; ++i) load_frag(X, xrow[i], 2 * pair + h, g, blocks, o.x[h][i]);
#pragma unroll
      for (int j = 0; j < NF; ++j) load_frag(W, wrow[j], 2 * pair + h, g, blocks, o.w[h][j]);
    }
  };
  auto multiply_all = [&](const Operands &o) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = multiply(o.w[h][j], o.x[h][i], acc[i][j]);
  };
  Operands a, b;
  constexpr int STEP = ALONG ? 1 : KW;
  const int32_t pairs = (ng + 1) / 2;
  int32_t pair = ALONG ? 0 : wave;
  if (pair < pairs) load(pair, a);
  while (pair < pairs) {
    if (pair + STEP < pairs) load(pair + STEP, b);
    multiply_all(a);
    pair += STEP;
    if (pair >= pairs) break;
    if (pair + STEP < pairs) load(pair + STEP, a);
    multiply_all(b);
    pair += STEP;
  }
  if constexpr (ALONG) {
    store_tiles<MF, NF>(acc, m0, n0, m1, n, bias, Y, stride);
    return;
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) part[ALONG ? 0 : wave][i * NF + j][lane] = acc[i][j];
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
      for (int t = 1; t < (ALONG ? 1 : KW); ++t) sum[0][j] += part[t][i * NF + j][lane];
    }
    store_tiles<1, NF>(sum, m0 + i * 16, n0, m1, n, bias, Y, stride);
  }
}

// s_waitcnt's operand: all of the wave's reads of shared memory are back, and all
// but the last `left` of what it asked for from memory.
__device__ constexpr int wait_until(int left) { return (left & 15) | (left >> 4) << 14 | 0x70; }

// BM x BN tiles (rows of X by rows of W), operands through shared memory: WM x WN
// waves, each (BM / WM) x (BN / WN) in products of 32 x 32 x 64.
//
// A buffer holds 256 k (a stage), 128 bytes of every row: whole lines, which the caches
// hand out at twice the rate of their halves (34 and 18 TB/s over the card).  What is
// asked for goes from memory straight to shared memory; with two buffers a stage is
// asked for as soon as the one before the last has been read, with four, where only
// 128 rows a side leave room, two stages earlier.  A stage has four products per 32 x
// 32 tile.  While one runs, the next one's operands come from shared memory; the
// requests for the next stage are woven in between, one behind each product, since a
// wave that asks for all at once waits until the last request is taken.  The one
// barrier of a stage stands before its last product, whose operands are there already.
//
// Rows of codes lie 128 bytes apart, their eight blocks mixed with the row so that 16
// rows read at one block touch all banks (no conflicts counted); the mixing is done on
// the memory side, since a wave's 64 lanes write 1 KiB in order.  Lane (r, g) = (lane %
// 32, lane / 32) takes blocks 4 g .. 4 g + 3 of a row, so that one word holds all the
// scale bytes it needs of the row; these words lie by lane, the tile's 32-row groups
// side by side, and one read serves several products.
//
// A wave's results go through shared memory in their own type, 32 rows at a time, so
// that whole lines are written.
//
// Bound by the matrix units at the clock that power allows, and by what the requests
// take from them: 8192 cubed to bf16 takes 250 us and up to 320 as the clock falls, 4.4
// to 3.4 PFLOP/s, of which a tile's 32 stages take 60 (2850 cycles each at 1.5 to 1.65
// GHz, 2112 of them products), the way in 2.4 and the way out 4.  2048 cubed takes 9.4.
// With one buffer four workgroups share a compute unit and cover each other's waits.
//
// 256 x 256 tiles use all 512 registers of a lane, and of 16-bit results 16, of fp32
// ones 8 more lie in scratch (68 and 36 bytes a lane), used outside of the sum's loop
// alone.
template <typename T, int BM, int BN, int BUFFERS, bool EXPERTS>
__global__ __launch_bounds__(256, BUFFERS == 1 ? 3 : 1) void k_nibble_tile(Operand X, Operand W, Sorted sorted,
                                                             const float *__restrict__ bias, T *__restrict__ Y,
                                                             int64_t stride, int64_t rows, int64_t n, int32_t blocks,
                                                             int32_t stages, int32_t mt, int32_t nt,
                                                             int32_t split_stages, int64_t split_stride) {
  constexpr int THREADS = 256, WM = 2, WN = 2, MF = BM / WM / 32, NF = BN / WN / 32;
  constexpr int ROWS = BM + BN, CHUNKS = ROWS * 8 / THREADS, SCALES = 2 * ROWS / THREADS;
  constexpr int BUFFER = ROWS * 136, PITCH = NF * 32 + 16 / (int)sizeof(T);  // PITCH: between a wave's rows of results
  static_assert(ROWS % THREADS == 0 && BM % (THREADS / 8) == 0 && BM % 64 == 0, "one operand for a wave's requests");
  static_assert((BUFFERS == 1 ? 4 : 2) * 32 * PITCH * (int)sizeof(T) <= BUFFER, "the waves' results in the buffers");
  // objects of their own and no array: reads of one then need not wait for what is on its way to another
  __shared__ __align__(16) uint8_t buffer_a[BUFFER], buffer_b[BUFFERS > 1 ? BUFFER : 16];
  __shared__ __align__(16) uint8_t buffer_c[BUFFERS == 4 ? BUFFER : 16], buffer_d[BUFFERS == 4 ? BUFFER : 16];
  __shared__ __align__(16) float shared_bias[BN];
  const int t = threadIdx.x, lane = t & 63, r = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WN, wn = wave % WN;
  const uint32_t tiles = (uint32_t)mt * (uint32_t)nt, split = workgroup() / tiles;
  const int32_t first = split * split_stages, last = first + split_stages < stages ? first + split_stages : stages;
  if (first >= last && split > 0) return;
  Y += split * split_stride;
  // The place of workgroup wg of `mtiles` rows of tiles, in bands of 8 along m: neighbours in the list share X's
  // and W's rows
  int64_t n0 = 0;
  const auto place = [&](uint32_t wg, uint32_t mtiles) -> uint32_t {
    if (wg >= mtiles * (uint32_t)nt) return ~0u;
    const uint32_t at = xcd_place(wg, mtiles * (uint32_t)nt), band = at / (8u * nt);
    const uint32_t left = mtiles - band * 8u < 8u ? mtiles - band * 8u : 8u, in_band = at - band * 8u * nt;
    n0 = (int64_t)(in_band / left) * BN;
    return band * 8u + in_band % left;
  };
  int64_t m0, m1 = rows, w0 = 0;
  if constexpr (EXPERTS) {
    // The tiles that there are, and not those that there could be, go to all XCDs alike: 1024 rows to 2 of 16
    // experts, 4096 x 4096, take 39 us, not 56.
    int32_t expert;
    if (!find_tile<true>(sorted, BM, [&](uint32_t all) { return place(workgroup(), all); }, m0, m1, expert)) return;
    if (expert < 0) {
      clear_rows(Y, stride, m0, m1, n0, n0 + BN < n ? n0 + BN : n);
      return;
    }
    w0 = expert * n;
    if (bias) bias += w0;
  } else {
    m0 = (int64_t)place(workgroup() - split * tiles, mt) * BM;
  }
  // X's and W's rows for one of the tile, counted from the first; past the last one, that
  const int32_t xlast = (int32_t)(m1 - m0 < BM ? m1 - m0 : BM) - 1, wlast = (int32_t)(n - n0 < BN ? n - n0 : BN) - 1;
  const bool gathered = EXPERTS && sorted.source;
  const int64_t xfirst = gathered ? 0 : m0, wfirst = w0 + n0;
  const auto x_row = [&](int row) -> uint32_t {
    row = row < xlast ? row : xlast;
    if (!gathered) return row;
    const int32_t from = sorted.source[m0 + row];
    return from < 0 ? 0 : from < X.rows ? from : X.rows - 1;
  };
  const auto w_row = [&](int row) -> uint32_t { return row < wlast ? row : wlast; };

  // Block i of thread t: row i * THREADS / 8 + t / 8 of the tile (X's rows first), place t % 8.
  constexpr int XC = BM / (THREADS / 8);  // of them, X's
  const int chunk = (t & 7) ^ ((t >> 4) & 7);
  const uint8_t *xbase = X.codes + xfirst * X.ld, *wbase = W.codes + wfirst * W.ld;
  uint32_t off[CHUNKS];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int row = (i < XC ? i : i - XC) * (THREADS / 8) + t / 8;
    off[i] = i < XC ? x_row(row) * (uint32_t)X.ld : w_row(row) * (uint32_t)W.ld;
  }
  // Scale word i of thread t: place i * THREADS + t of [g][X's, then W's][wave row or column][r][product].
  const uint8_t *ssrc[SCALES];
#pragma unroll
  for (int i = 0; i < SCALES; ++i) {
    const bool of_x = (i * THREADS + wave * 64) % ROWS < BM;
    const int u = (i * THREADS + t) % ROWS - (of_x ? 0 : BM), f = of_x ? MF : NF;
    const int row = (u / (32 * f) * f + u % f) * 32 + u / f % 32;
    ssrc[i] = of_x ? X.scales + (xfirst + x_row(row)) * 4 : W.scales + (wfirst + w_row(row)) * 4;
  }
  // Part `part` of four of stage st; past the last stage: that one again, for nothing; past a row's last block
  // or group of scales: that one again
  auto fetch = [&](int32_t st, int part, uint8_t *buffer) {
    st = st < last ? st : last - 1;
    const uint32_t block = st * 8 + chunk < blocks ? st * 8 + chunk : blocks - 1;
#pragma unroll
    for (int i = part * CHUNKS / 4; i < (part + 1) * CHUNKS / 4; ++i)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void *)((i < XC ? xbase : wbase) + (off[i] + block * 16)),
          (__attribute__((address_space(3))) void *)(&buffer[(i * THREADS + wave * 64) * 16]), 16, 0, 0);
#pragma unroll
    for (int i = part * SCALES / 4; i < (part + 1) * SCALES / 4; ++i) {
      const int at = i * THREADS + wave * 64, u = at % ROWS;
      const int64_t group = st * 2 + (at >= ROWS && st * 2 + 1 < (blocks + 3) / 4 ? 1 : 0);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void *)(ssrc[i] + group * ((u < BM ? X.rows : W.rows) * 4)),
          (__attribute__((address_space(3))) void *)(&buffer[ROWS * 128 + at * 4]), 4, 0, 0);
    }
  };

  struct Operands {
    i32x8 x[MF], w[NF];
  };
  struct Scales {
    uint32_t x[MF], w[NF];
  };
  // Where a lane's block of its row lies: the mixing of a row is bits 1 to 3 of its number.
  const int xlo = (wm * MF * 32 + r) * 128, wlo = (BM + wn * NF * 32 + r) * 128, mix = (r >> 1) & 7;
  const int xs = ROWS * 128 + (g * ROWS + (wm * 32 + r) * MF) * 4;
  const int ws = ROWS * 128 + (g * ROWS + BM + (wn * 32 + r) * NF) * 4;
  auto load = [&](const uint8_t *buffer, int h, Operands &o) {
    const int place = ((4 * g + h) ^ mix) * 16;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(buffer + wlo + j * 32 * 128 + place);
      o.w[j] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(buffer + xlo + i * 32 * 128 + place);
      o.x[i] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
    }
  };
  // Blocks past the last, whose codes are another's, get the scale 2^-127 on both sides:
  // what they add is under 2^-240.
  auto load_scales = [&](const uint8_t *buffer, int32_t st, Scales &o) {
    const int32_t have = st < last ? blocks - (st * 8 + g * 4) : 0;
    const uint32_t mask = have >= 4 ? ~0u : have <= 0 ? 0u : (1u << (8 * have)) - 1;
#pragma unroll
    for (int i = 0; i < MF; ++i) o.x[i] = *reinterpret_cast<const uint32_t *>(buffer + xs + i * 4) & mask;
#pragma unroll
    for (int j = 0; j < NF; ++j) o.w[j] = *reinterpret_cast<const uint32_t *>(buffer + ws + j * 4) & mask;
  };
  f32x16 acc[MF][NF] = {};
  auto multiply_all = [&](const Operands &o, const Scales &s, auto h) {
    constexpr int H = decltype(h)::value;
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(o.w[j], o.x[i], acc[i][j], 4, 4, H, (int)s.w[j], H,
                                                                    (int)s.x[i]);
  };
  Operands a, b;
  Scales s, s_next;
  // The order within a fourth of a stage: a read of shared memory behind every product, or two and a request
  // to memory.
  auto weave = [&](auto requests) {
    constexpr int R = decltype(requests)::value, READS = MF + NF, BOTH = READS > R ? READS : R;
#pragma unroll
    for (int i = 0; i < BOTH; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
      if (i < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // a read of shared memory
      if (i < R) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // a request
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int ASKED = CHUNKS + SCALES, HALF = ASKED / 2;
  auto stage = [&](int32_t st, uint8_t *buffer, const uint8_t *buffer_next, uint8_t *buffer_before) {
    load(buffer, 1, b);
    fetch(st + BUFFERS - 1, 2, buffer_before);
    fetch(st + BUFFERS - 1, 3, buffer_before);
    multiply_all(a, s, std::integral_constant<int, 0>());
    weave(std::integral_constant<int, HALF>());
    load(buffer, 2, a);
    multiply_all(b, s, std::integral_constant<int, 1>());
    weave(std::integral_constant<int, 0>());
    load(buffer, 3, b);
    multiply_all(a, s, std::integral_constant<int, 2>());
    weave(std::integral_constant<int, 0>());
    // This wave's part of the next stage is there; behind the barrier every wave's is, and nobody reads this
    // stage's buffer any more.
    __builtin_amdgcn_s_waitcnt(wait_until(BUFFERS > 2 ? (BUFFERS - 2) * ASKED : 0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    load(buffer_next, 0, a);
    load_scales(buffer_next, st + 1, s_next);
    fetch(st + BUFFERS, 0, buffer);
    fetch(st + BUFFERS, 1, buffer);
    multiply_all(b, s, std::integral_constant<int, 3>());
    weave(std::integral_constant<int, HALF>());
    s = s_next;
  };
  if constexpr (BUFFERS == 1) {  // other workgroups of the compute unit have work while this one waits
    for (int32_t st = first; st < last; ++st) {
#pragma unroll
      for (int part = 0; part < 4; ++part) fetch(st, part, buffer_a);
      __builtin_amdgcn_s_waitcnt(wait_until(0));
      __syncthreads();
      load_scales(buffer_a, st, s);
      load(buffer_a, 0, a);
      multiply_all(a, s, std::integral_constant<int, 0>());
      load(buffer_a, 1, a);
      multiply_all(a, s, std::integral_constant<int, 1>());
      load(buffer_a, 2, a);
      multiply_all(a, s, std::integral_constant<int, 2>());
      load(buffer_a, 3, a);
      multiply_all(a, s, std::integral_constant<int, 3>());
      __syncthreads();
    }
  } else if (first < last) {
    auto fetch_half = [&](int32_t st, int half, uint8_t *buffer) {
      fetch(st, 2 * half, buffer);
      fetch(st, 2 * half + 1, buffer);
    };
    fetch_half(first, 0, buffer_a);
    fetch_half(first, 1, buffer_a);
    if constexpr (BUFFERS == 4) {
      fetch_half(first + 1, 0, buffer_b);
      fetch_half(first + 1, 1, buffer_b);
      fetch_half(first + 2, 0, buffer_c);
      fetch_half(first + 2, 1, buffer_c);
      fetch_half(first + 3, 0, buffer_d);
    } else {
      fetch_half(first + 1, 0, buffer_b);
    }
    __builtin_amdgcn_s_waitcnt(wait_until(BUFFERS > 2 ? (BUFFERS - 2) * ASKED + HALF : HALF));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(buffer_a, 0, a);
    load_scales(buffer_a, first, s);
    // Rounds of all buffers, then the rest: with no path on which a stage of a round is skipped the compiler
    // sees which requests are still under way for which buffer, and waits for no others.
    int32_t st = first;
    if constexpr (MF * NF == 16) {  // no registers for a stage more: the last one may be of blocks past the last
      for (; st < last; st += 2) {
        stage(st, buffer_a, buffer_b, buffer_b);
        stage(st + 1, buffer_b, buffer_a, buffer_a);
      }
    } else if constexpr (BUFFERS == 2) {
      for (; st + 2 <= last; st += 2) {
        stage(st, buffer_a, buffer_b, buffer_b);
        stage(st + 1, buffer_b, buffer_a, buffer_a);
      }
      if (st < last) stage(st, buffer_a, buffer_b, buffer_b);
    } else {
      for (; st + 4 <= last; st += 4) {
        stage(st, buffer_a, buffer_b, buffer_d);
        stage(st + 1, buffer_b, buffer_c, buffer_a);
        stage(st + 2, buffer_c, buffer_d, buffer_b);
        stage(st + 3, buffer_d, buffer_a, buffer_c);
      }
      if (st < last) {
        stage(st, buffer_a, buffer_b, buffer_d);
        if (st + 1 < last) {
          stage(st + 1, buffer_b, buffer_c, buffer_a);
          if (st + 2 < last) stage(st + 2, buffer_c, buffer_d, buffer_b);
        }
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(wait_until(0));  // nothing is on its way to shared memory any more, from no wave
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // The bias, by way of shared memory: every lane needs 16 of each 32 columns'.  Added (zeros without one) where the
  // results leave, so that the accumulators stay in one place: 8192 x 8192 x 2048 to fp32 in 256 x 256 tiles takes
  // 113 us with one, and took 138.  Large tiles of 16-bit results add it here: 8192 cubed without a bias takes 242 us
  // so and 247 with it added late, and 260 with one.
  constexpr bool LATE = MF * NF != 16 || sizeof(T) == 4;
  f32x4 add[NF][4] = {};
  if (bias) {
    if (t < BN) shared_bias[t] = n0 + t < n ? bias[n0 + t] : 0.0f;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(shared_bias + (wn * NF + j) * 32 + q * 8 + g * 4);
        if constexpr (LATE) {
          add[j][q] = v;
        } else {
#pragma unroll
          for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int p = 0; p < 4; ++p) acc[i][j][4 * q + p] += v[p];
          __builtin_amdgcn_sched_barrier(0);  // one at a time: the accumulators leave few registers
        }
      }
  }
  // Results in Y's type, 32 rows of the wave's columns: a lane leaves four neighbours of its row at a time and
  // takes 16 bytes of a row for the memory.
  T *mine = reinterpret_cast<T *>(BUFFERS == 1 ? buffer_a + wave * (32 * PITCH * sizeof(T))
                                               : (wave < 2 ? buffer_a : buffer_b) + wave % 2 * (32 * PITCH * sizeof(T)));
  constexpr int V = 16 / sizeof(T), LANES = NF * 32 / V, STEP = 64 / LANES;  // columns of a lane, lanes of a row
  const int vr = lane / LANES, vc = lane % LANES * V;
  const int64_t c = n0 + wn * NF * 32 + vc;
  const int there = n - c < V ? (int)(n - c) : V;
  T *y = Y + (m0 + wm * MF * 32 + vr) * stride + c;
  auto put = [&](int i) {
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = j * 32 + q * 8 + g * 4;
        Span<T, 4, 4 * sizeof(T)> o;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          if constexpr (LATE)
            o.v[p] = rounded<T>(acc[i][j][4 * q + p] + add[j][q][p]);
          else
            o.v[p] = rounded<T>(acc[i][j][4 * q + p]);
        }
        *reinterpret_cast<Span<T, 4, 4 * sizeof(T)> *>(mine + r * PITCH + at) = o;
      }
    wave_order();  // before other lanes take them
    __builtin_amdgcn_sched_barrier(0);
  };
  auto get = [&](int row) { return *reinterpret_cast<const Span<T, V, 16> *>(mine + row * PITCH + vc); };
  if (m0 + BM <= m1 && n0 + BN <= n) {  // a whole tile: no conditions between the reads and the writes
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      put(i);
#pragma unroll
      for (int k = 0; k < 32 / STEP; ++k) {
        const auto o = get(k * STEP + vr);
        *reinterpret_cast<Span<T, V> *>(y + (i * 32 + k * STEP) * stride) = *reinterpret_cast<const Span<T, V> *>(&o);
      }
      wave_order();  // they have been taken before the next ones come
      __builtin_amdgcn_sched_barrier(0);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t m = m0 + (wm * MF + i) * 32;
    put(i);
    for (int k = 0; k < 32 / STEP; ++k) {
      if (m + k * STEP + vr >= m1) continue;
      const auto o = get(k * STEP + vr);
      T *to = y + (i * 32 + k * STEP) * stride;
      if (there == V) {
        *reinterpret_cast<Span<T, V> *>(to) = *reinterpret_cast<const Span<T, V> *>(&o);
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q)
          if (q < there) to[q] = o.v[q];
      }
    }
    wave_order();
  }
}

// Y = the sum of the parts that workgroups of a split sum left + bias: TEAM threads for four columns, each
// every TEAM-th part, then the threads' sums, all in one order.  64 parts of 256 x 128 take 4 us, 2.1 TB/s.
template <typename T, int TEAM>
__global__ __launch_bounds__(256) void k_nibble_join(const float *__restrict__ parts, int32_t splits, int64_t rows,
                                                     int64_t n, const float *__restrict__ bias, T *__restrict__ Y,
                                                     int64_t stride) {
  constexpr int QUADS = 256 / TEAM;
  __shared__ f32x4 sums[TEAM][QUADS];
  const int own = threadIdx.x % QUADS, team = threadIdx.x / QUADS;
  const int64_t quads = (n + 3) / 4, at = (int64_t)workgroup() * QUADS + own, m = at / quads, c = at % quads * 4;
  const int there = m >= rows ? 0 : n - c < 4 ? (int)(n - c) : 4;
  const float *p = parts + (team * rows + m) * n + c;
  float sum[4] = {};
  if (there == 4) {
#pragma unroll 4
    for (int32_t i = team; i < splits; i += TEAM, p += TEAM * rows * n) {
      float v[4];
      load_span(p, v);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += v[q];
    }
  } else {
    for (int32_t i = team; i < splits; i += TEAM, p += TEAM * rows * n) {
      float v[4];
      load_part(p, there, v);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += v[q];
    }
  }
  if constexpr (TEAM > 1) {
    sums[team][own] = f32x4{sum[0], sum[1], sum[2], sum[3]};
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int i = 1; i < TEAM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += sums[i][own][q];
  }
  if (there == 0) return;
  if (bias) {
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] += q < there ? bias[c + q] : 0.0f;
  }
  if (there == 4)
    store_span(Y + m * stride + c, sum);
  else
    store_part(Y + m * stride + c, there, sum);
}

struct Call {
  Operand x, w;
  Sorted sorted;
  const float *bias;
  int64_t stride, rows, n;
  int32_t blocks, ng;
  float *parts;  // workspace of a split sum
};

enum Form {
  kTile256 = SD_NIBBLE_TILE_256,
  kTile128 = SD_NIBBLE_TILE_128,
  kTile128Deep = SD_NIBBLE_TILE_128_DEEP,
  kTile128Short = SD_NIBBLE_TILE_128_SHORT,
  kRows32 = SD_NIBBLE_ROWS_32,
  kRows16 = SD_NIBBLE_ROWS_16,
  kRows16Short = SD_NIBBLE_ROWS_16_SHORT,
  kRows16Along = SD_NIBBLE_ROWS_16_ALONG
};
struct Plan {
  Form form;
  int32_t splits, split_stages;
};

// Tiles of bm rows: as many as there are, or for rows sorted by expert at most as many as there can be.
int64_t row_tiles(int64_t rows, int32_t experts, int64_t bm) {
  if (experts == 0) return ceil_div(rows, bm);
  const int64_t parts = experts + 1 < rows ? experts + 1 : rows;  // that are not empty
  return (rows - parts) / bm + parts;
}

// Measured in us, 16-bit results, launches in a row (256 compute units; 128 x 128 with the better number of
// buffers; "s": such tiles with the sum in so many parts, joined by a second launch):
//   rows x columns x k      256x256   128x128  32x32  16x16   s4    s16   s64   s128
//   8192 x 8192 x 8192          251       301   2234
//   8192 x 8192 x 512            50        36    273    304
//   4096 x 4096 x 4096           40        44    282    559
//   2048 x 2048 x 2048           17       9.4     41     73
//   1000 x 1000 x 1000           15       7.0    9.1     12
//   256 x 4096 x 4096            23        11     21     37    20    36
//   64 x 4096 x 4096             24        11    7.1     11    12    22
//   512 x 512 x 4096             23        10    7.2     11    11    18
//   1 x 4096 x 4096              23        10    5.7    3.8     9    13
//   262144 x 128 x 128           52        17    111    103
//   1000000 x 20 x 128          214        54    164    115
//   512 x 512 x 32768           144        55     40     72    22    20    43
//   64 x 64 x 65536             266       103     71     37    33    15    11     11
//   256 x 128 x 262144         1094       405    278    141   108    34    19     21
// A stage of 256 k takes a lone 128 x 128 tile 0.5 us, and the parts go to memory and back at about
// 2.5 TB/s: that gives the number of parts.  So it is for operands that the caches hold; 256 x 128 x 262144 in a
// training step, whose operands come from memory, takes 69 parts 24 + 4 us, on 138 of the compute units.
//
// Rows sorted by expert, us, launches in a row (rows of X, experts of each, experts, columns x k; 16 x 16 with
// the best of sums shared by the waves or not):
//                              256x256   128x128  32x32  16x16
//   4096, 2, 16, 4096 x 4096        111       104    632    870
//   1024, 2, 16, 4096 x 4096         44        39    172    228
//   64, 2, 16, 4096 x 4096           35        26     38     28
//   16, 2, 16, 4096 x 4096           35        25     36     27
//   64, 8, 64, 1024 x 2048           26        17     27     17
//   16, 8, 64, 1024 x 2048           21        15     23     15
//   1, 8, 64, 1024 x 2048            17         9    5.3    4.4
Plan plan_of(int64_t rows, int32_t experts, int64_t n, int64_t cols, int32_t type, bool near) {
  const int64_t cus = cu_count(), stages = ceil_div(cols, 256);
  // of rows sorted by expert the tiles there will be: half a tile too many for each expert
  const auto tiles = [&](int64_t bm, int64_t bn) {
    const int64_t mt = ceil_div(rows, bm);
    return (experts == 0 ? mt : std::min<int64_t>(mt + experts / 2, rows)) * ceil_div(n, bn);
  };
  const auto whole = [&](Form f) { return Plan{f, 1, (int32_t)stages}; };
  // A wave for each 16 x 32 where the sum is short and what the waves read twice is little, us with it and
  // without: 3000 x 300 x 100 3.8 and 6.1, 1000 x 1000 x 256 4.2 and 5.2, but 1500 x 1500 x 256 7.2 and 5.8;
  // 16 x 131072 x 300 5.7 and 9.4.  Of rows sorted by expert, where each has few of them: 2000 to 100 experts,
  // 1000 x 100, 7.3 and 11.9; 600 to 64, 1024 x 512, 6.2 and 7.8, x 768 10.1 and 8.7.
  const int64_t waves = tiles(16, 32), thin = std::min(rows, n);
  const bool spread = 2 * waves >= 9 * cus, few = rows <= 8 * (int64_t)experts;  // few rows of each expert
  if (experts > 0 ? spread && (rows * stages <= 24 * (int64_t)experts || (few && stages <= 8))
                  : stages <= 3 && waves >= 2 * cus && (thin <= 16 || waves * ceil_div(cols, 128) <= 30 * cus))
    return whole(kRows16Along);
  if (near && (!few || spread)) {
    // Large tiles, us with them and with one buffer of 128 x 128: 4096 x 4096 x 2048 25.5 and 26.2 to bf16, 30.6 and
    // 30.6 to fp32, 8192 x 8192 x 2048 111 and 100 to fp32, 4096 cubed 44 and 49.  Of rows sorted by expert, whose
    // tiles begin with two more loads, where they are many: 16384 rows to 2 of 16, 4096 x 4096, 364 and 368, 8192 to
    // 2 of 8 179 and 178, 4096 to 2 of 16 111 and 104.  Not where they cover much more than there is.
    const int64_t large = tiles(256, 256);
    if (stages >= (type == SD_TYPE_F32 ? 12 : 8) && 4 * large >= 3 * cus && 32 * large <= 9 * tiles(128, 128) &&
        (experts == 0 || large * stages >= 80 * cus))
      return whole(kTile256);
    const int64_t t = tiles(128, 128);
    // 256 x 2048 x 1000 takes 4.8 us in tiles of 32 x 32 and 5.4 of 128 x 128, 512 x 1024 x 4096 11.5 and 10.2;
    // 20000 x 16 x 4096 13.8 of 16 x 16 and 16.4.
    const bool wide = rows > 64 && n > 64 && t >= cus / 8 && (stages > 8 || tiles(32, 32) > 2 * cus);
    const bool many = t >= cus / 2 && (experts > 0 || thin > 16 || t >= 2 * cus);
    if (experts == 0 && !many && stages >= (wide ? 32 : 64)) {
      const int64_t best = (int64_t)std::sqrt(0.5 * stages / ((double)rows * n * 8 / 2.5e6));
      const int64_t splits = std::min(std::min(cus / t, stages / 4), best);
      if (splits > 1) {
        const int64_t each = ceil_div(stages, splits);
        return Plan{kTile128Deep, (int32_t)ceil_div(stages, each), (int32_t)each};
      }
    }
    // Buffers for 128 x 128: one, and four workgroups a compute unit, where there are more tiles than units or
    // the sum is short (3000 x 3000 x 3000 takes 30, 33 and 35 us with one, two and four, 533036 x 44 x 26 33,
    // 47 and 86); four where the sum is long (2048 x 2048 x 8192 29 with two, 25 with four), else two (2048
    // cubed 11.5, 9.4 and 9.9).  Of rows sorted by expert the tiles are fewer than thought: 16 rows to 4 of 16
    // experts, 4096 x 8192, 44 with two, 53 with one.
    if (wide || many || few) {
      const bool one = stages <= 2 || (experts > 0 && stages >= 16 ? t > 2 * cus : t > cus);
      return whole(one ? kTile128Short : stages >= 24 && t <= cus ? kTile128Deep : kTile128);
    }
  }
  if (rows > 16 && n > 16 && tiles(32, 32) >= cus && !few) return whole(kRows32);
  // Four waves share the sum where it is short or workgroups come in numbers, as for 32 x 32 always (512 x 512 x
  // 4096 7.1 us, with eight 7.2, 400 x 1000 x 1500 5.4 and 7.9), else eight: 1500 x 1500 x 1500 takes 23 and 33 us
  // in tiles of 16 x 16, 1 x 4096 x 4096 3.9 and 3.7.
  return whole(stages <= 4 || tiles(16, 16) >= 2 * cus ? kRows16Short : kRows16);
}
size_t parts_bytes(const Plan &p, int64_t rows, int64_t n) {
  return p.splits > 1 ? (size_t)p.splits * rows * n * 4 : 0;
}

template <typename T, int MF, int NF, int KW, bool EXPERTS, bool ALONG = false>
int rows_launch(const Call &c, T *y, hipStream_t s) {
  static_assert(MF <= KW, "a wave for each row group");
  const int64_t nt = ceil_div(c.n, NF * 16 * (ALONG ? KW : 1));
  const int64_t wgs = row_tiles(c.rows, EXPERTS ? c.sorted.experts : 0, MF * 16) * nt;
  if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_nibble_rows<T, MF, NF, KW, EXPERTS, ALONG>), grid_of(wgs), dim3(KW * 64), 0, s, c.x, c.w,
                     c.sorted, c.bias, y, c.stride, c.rows, c.n, c.blocks, c.ng, (int32_t)nt);
  return launched();
}

template <typename T, int BM, int BN, int BUFFERS, bool EXPERTS>
int tile_launch(const Call &c, const Plan &p, T *y, hipStream_t s) {
  const int64_t mt = row_tiles(c.rows, EXPERTS ? c.sorted.experts : 0, BM), nt = ceil_div(c.n, BN);
  if (mt * nt > INT32_MAX / p.splits) return SD_ERR_OVERFLOW;
  const bool parts = p.splits > 1;
  hipLaunchKernelGGL((k_nibble_tile<T, BM, BN, BUFFERS, EXPERTS>), grid_of(mt * nt * p.splits), dim3(256), 0, s, c.x,
                     c.w, c.sorted, parts ? nullptr : c.bias, y, parts ? c.n : c.stride, c.rows, c.n, c.blocks,
                     (c.ng + 1) / 2, (int32_t)mt, (int32_t)nt, p.split_stages, c.rows * c.n);
  return launched();
}

template <typename T, bool EXPERTS>
int product_as(const Call &c, const Plan &p, void *Y, hipStream_t s) {
  T *y = static_cast<T *>(Y);
  if (p.splits > 1) {
    int st = tile_launch<float, 128, 128, 4, false>(c, p, c.parts, s);
    if (st != SD_OK) return st;
    const int team = p.splits >= 16 ? 8 : 1;
    const int64_t wgs = ceil_div(c.rows * ceil_div(c.n, 4), 256 / team);
    if (wgs > INT32_MAX) return SD_ERR_OVERFLOW;
    auto *kernel = team == 8 ? k_nibble_join<T, 8> : k_nibble_join<T, 1>;
    hipLaunchKernelGGL(kernel, grid_of(wgs), dim3(256), 0, s, c.parts, p.splits, c.rows, c.n, c.bias, y, c.stride);
    return launched();
  }
  switch (p.form) {
    case kTile256: return tile_launch<T, 256, 256, 2, EXPERTS>(c, p, y, s);
    case kTile128: return tile_launch<T, 128, 128, 2, EXPERTS>(c, p, y, s);
    case kTile128Deep: return tile_launch<T, 128, 128, 4, EXPERTS>(c, p, y, s);
    case kTile128Short: return tile_launch<T, 128, 128, 1, EXPERTS>(c, p, y, s);
    case kRows32: return rows_launch<T, 2, 2, 4, EXPERTS>(c, y, s);
    case kRows16: return rows_launch<T, 1, 1, 8, EXPERTS>(c, y, s);
    case kRows16Short: return rows_launch<T, 1, 1, 4, EXPERTS>(c, y, s);
    default: return rows_launch<T, 1, 2, 4, EXPERTS, true>(c, y, s);
  }
}
template <bool EXPERTS>
int product(const Call &c, const Plan &p, void *Y, int32_t type, void *stream) {
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == SD_TYPE_F32   ? product_as<float, EXPERTS>(c, p, Y, s)
         : type == SD_TYPE_F16 ? product_as<f16, EXPERTS>(c, p, Y, s)
                               : product_as<bf16, EXPERTS>(c, p, Y, s);
}

// The large tiles keep the distance of a tile's rows in 32 bits.
bool near_rows(const sd_nibble_t *p) { return p->ld <= (1 << 23); }
// Of rows sorted by expert, X's from anywhere, and so their distance from its first one.
bool near_entries(int64_t ld, int64_t rows) { return rows <= (1ll << 32) / (ld > 0 ? ld : 1); }

Operand operand(const sd_nibble_t *p) { return Operand{p->codes, p->scales, p->ld, p->rows}; }

}  // namespace

extern "C" int sd_nibble_product_size(int64_t rows, int64_t cols, int64_t n, size_t *bytes) {
  if (!bytes || rows < 0 || cols < 0 || n < 0) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || n > kMaxRows || cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  // results of any type: it has no say in how a sum is split
  *bytes = rows == 0 || n == 0 ? 0 : parts_bytes(plan_of(rows, 0, n, cols, SD_TYPE_BF16, true), rows, n);
  return SD_OK;
}

extern "C" int sd_nibble_product_form(int64_t rows, int64_t cols, int64_t n, int32_t experts, int32_t type,
                                      int32_t *form, int32_t *parts) {
  if (!form || !parts || rows < 1 || cols < 0 || n < 1 || experts < 0 || !type_ok(type)) return SD_ERR_INVALID_VALUE;
  if (rows > kMaxRows || n > kMaxRows || cols > kMaxRows - 1024) return SD_ERR_OVERFLOW;
  if (experts > kMaxExperts) return SD_ERR_UNSUPPORTED;
  const int64_t ld = col_blocks(cols) * 16;
  const bool near = ld <= (1 << 23) && (experts == 0 || near_entries(ld, rows));
  const Plan p = plan_of(rows, experts, n, cols, type, near);
  *form = p.form;
  *parts = p.splits;
  return SD_OK;
}

extern "C" int sd_nibble_product(const sd_nibble_t *X, const sd_nibble_t *W, const float *bias, void *Y, int32_t type,
                                 int64_t row_stride, void *workspace, size_t bytes, void *stream) {
  int st = check_nibble(X);
  if (st == SD_OK) st = check_nibble(W);
  if (st == SD_OK && X->cols != W->cols) st = SD_ERR_INVALID_VALUE;
  if (st == SD_OK) st = check_table(Y, type, X->rows, W->rows, row_stride);
  if (st == SD_OK && bias && !aligned_to(bias, 4)) st = SD_ERR_INVALID_VALUE;
  size_t need = 0;
  if (st == SD_OK) st = sd_nibble_product_size(X->rows, X->cols, W->rows, &need);
  if (st == SD_OK && need > 0 && (!workspace || bytes < need || !aligned_to(workspace, 16)))
    st = SD_ERR_INVALID_VALUE;
  if (st != SD_OK) return st;
  if (X->rows == 0 || W->rows == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  const Plan p = plan_of(X->rows, 0, W->rows, X->cols, type, near_rows(X) && near_rows(W));
  const Call c{operand(X), operand(W), Sorted{}, bias, row_stride, X->rows, W->rows, (int32_t)col_blocks(X->cols),
               (int32_t)groups_of(X->cols), static_cast<float *>(workspace)};
  return product<false>(c, p, Y, type, stream);
}

extern "C" int sd_expert_product(const sd_nibble_t *X, const sd_nibble_t *W, const sd_route_t *route, int32_t sorted,
                                 const float *bias, void *Y, int32_t type, int64_t row_stride, void *stream) {
  int st = check_nibble(X);
  if (st == SD_OK) st = check_nibble(W);
  if (st == SD_OK) st = check_route(route);
  if (st != SD_OK) return st;
  const int64_t total = route->rows * route->k;
  if (X->cols != W->cols || W->rows % route->experts != 0 || X->rows != (sorted ? total : route->rows) ||
      (sorted != 0 && sorted != 1))
    return SD_ERR_INVALID_VALUE;
  const int64_t n = W->rows / route->experts;
  if ((st = check_table(Y, type, total, n, row_stride)) != SD_OK) return st;
  if (bias && !aligned_to(bias, 4)) return SD_ERR_INVALID_VALUE;
  if (total == 0 || n == 0) return SD_OK;
  if ((st = have_device()) != SD_OK) return st;
  const bool near = near_rows(W) && near_entries(X->ld, X->rows);
  const Plan p = plan_of(total, route->experts, n, X->cols, type, near);
  const Call c{operand(X), operand(W), Sorted{route->offsets, sorted ? nullptr : route->source, route->experts, total},
               bias, row_stride, total, n, (int32_t)col_blocks(X->cols), (int32_t)groups_of(X->cols), nullptr};
  return product<true>(c, p, Y, type, stream);
}
