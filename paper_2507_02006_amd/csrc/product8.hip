// Product of two matrices held in 8 bits with a scale for each 128 values of k
// (gfx950): Y = A B^T,
//   y_ij = sum_b sA(i, b) sB(j, b) sum_{k in b} a_ik b_jk.
//
// The inner sums run on the matrix cores; each block's sums are multiplied with
// its scales and added in vector registers, one multiply-add a value and block where
// B's scale is one for 128 rows.  B's rows are the matrix cores' rows and A's their
// columns, so that a lane holds results of one row of A and has one scale of it.
//
// How exact the inner sums are: the 8-bit products of the matrix cores add eight
// neighbours of k in fixed point, cut off 2^-13 below the largest of the eight (found
// by sums of a large and a small product; the eights are then added in fp32), which
// leaves the sums of a block of normally distributed values 1.3e-5 of their size off.
// That is below the rounding of a result of 16 bits (2^-9 and 2^-12 on average) and
// far above fp32's: for fp32 results, and where few rows leave the matrix cores idle
// anyway, the codes are converted to bf16, which holds them exactly, and multiplied
// at half the rate with sums that are fp32's.
//
// Two forms.  Up to 16 rows of A: bound by B's bytes, which go from memory to the
// matrix cores' registers, no LDS; a workgroup owns 16 rows of B and its wavefronts
// share k.  Else tiles: stages of 128 k go from global memory straight to LDS.  Where
// an operand's rows are not chunks of 16 bytes it is copied so first.  Where there are few
// tiles k is split over workgroups, whose partial sums a second launch adds in a fixed
// order.
//
// What is rounded to fewer bits: nothing but Y, once (the codes are the operands).
//
// Measured: 16384 x 8192 x 4096, 128 x 128 scales, bf16 550 us (2000 TFLOP/s, with random
// codes; the power limit holds the clock below what codes of one value reach, 468 us), with
// a scale for each row of B 725; 5 x 8192 x 2048 6 us (2.7 TB/s); 1000 x 520 x 65537, row scales, fp32 in bf16 products 117 us
// and 42 for copies and sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "layers.h"
#include "rows8.h"
#include "tile.h"

namespace aires {
namespace kern {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_el1 __attribute__((aligned(1)));

struct Args {
  Held x, w;        // A (rows of Y) and B (columns of Y)
  Mat y;
  float* part;      // [split][rows][columns] sums, or NULL
  int64_t k, steps; // k (in tiles: a multiple of 16), steps of 128 k
  int64_t per;      // steps of a split
};

__device__ __forceinline__ i32x8 join(i32x4 lo, i32x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// Codes [8 part, 8 part + 8) of 16 in bf16.
__device__ __forceinline__ bf16x8 widen(i32x4 c, int part) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const int lo = c[2 * part], hi = c[2 * part + 1];
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// Bytes [0, 16) of p, of which the first `have` are there (others: 0).
__device__ __forceinline__ i32x4 load16(const uint8_t* p, int64_t have) {
  if (have >= 16) return *reinterpret_cast<const i32x4_el1*>(p);
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int b = 0; b < 15; ++b)
    if (b < have) v[b / 4] |= (int)((uint32_t)p[b] << (8 * (b & 3)));
  return v;
}

// The same of a row that has 16 bytes before p + have: loaded as one chunk that ends with
// the row and moved to its place.
__device__ __forceinline__ i32x4 load16_moved(const uint8_t* p, int64_t have) {
  const int by = have >= 16 ? 0 : have <= 0 ? 16 : 16 - (int)have;
  const i32x4 w = *reinterpret_cast<const i32x4_el1*>(have >= 16 ? p : p + have - 16);
  uint64_t lo = (uint64_t)(uint32_t)w[1] << 32 | (uint32_t)w[0], hi = (uint64_t)(uint32_t)w[3] << 32 | (uint32_t)w[2];
  if (by >= 8) {
    lo = hi;
    hi = 0;
  }
  const int bits = (by & 7) * 8;
  lo = by == 16 ? 0 : bits == 0 ? lo : lo >> bits | hi << (64 - bits);
  hi = hi >> bits;
  return i32x4{(int)(uint32_t)lo, (int)(uint32_t)(lo >> 32), (int)(uint32_t)hi, (int)(uint32_t)(hi >> 32)};
}

__device__ __forceinline__ void store_y(const Args& a, int64_t row, int64_t col, const float (&v)[4]) {
  if (row >= a.y.rows || col >= a.y.cols) return;
  void* const to = a.y.data;
  const int64_t at = row * a.y.ld + col;
  const int t = a.y.type;
  if (col + 4 <= a.y.cols) {
    if (t == DT_F32) store4<DT_F32>(to, at, v);
    else if (t == DT_BF16) store4<DT_BF16>(to, at, v);
    else store4<DT_F16>(to, at, v);
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (col + q < a.y.cols) store1(to, t, at + q, v[q]);
  }
}

// ------------------------------------------------------------------- tiles

// One operand's share of a stage: SPAN rows of 128 k.  Load j of a wavefront fills
// 1 KB, 8 rows, of the stage; its 16-byte chunks are placed XORed with their row
// so that neither writes nor reads of LDS meet bank conflicts.  Rows past the last repeat it (their results
// are not used).
template <int SPAN, int WAVES>
struct Share {
  static constexpr int COUNT = SPAN / 8 / WAVES;
  static_assert(SPAN % (8 * WAVES) == 0, "a wavefront loads whole parts");
  const uint8_t* base;  // first row of the tile, advanced along k
  int64_t ld, left;     // left: k that there are from the next stage's first on
  int last;             // last row that there is
  uint32_t off;         // of this lane in the first part

  __device__ static int row(int wave, int lane) { return wave * 8 + lane / 8; }
  __device__ static int chunk(int wave, int lane) { return ((lane % 8) ^ (row(wave, lane) / 2 % 8)) * 16; }

  __device__ void init(const Held& h, int64_t r0, int64_t k0, int64_t k, int wave, int lane) {
    base = h.codes + r0 * h.ld + k0;
    ld = h.ld;
    left = k - k0;
    last = h.rows - 1 - r0 < SPAN ? (int)(h.rows - 1 - r0) : SPAN;
    off = (uint32_t)(row(wave, lane) * ld + chunk(wave, lane));
  }
  // Straight to LDS.  k past the last repeats the row's last chunk (the other operand
  // holds zeros there).
  __device__ __forceinline__ void issue(char* lds, int wave, int lane) {
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const uint8_t* from = reinterpret_cast<const uint8_t*>(
        ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32) |
        (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b));
    const auto load = [&](int j, const uint8_t* p) {
      __builtin_amdgcn_global_load_lds((global_void*)p, (lds_void*)(lds + (j * WAVES + wave) * 1024), 16, 0, 0);
    };
    if (last >= SPAN - 1 && left >= 128) {
#pragma unroll
      for (int j = 0; j < COUNT; ++j, from += WAVES * 8 * ld) load(j, from + off);
    } else {
      const int at = chunk(wave, lane), c = at < left ? at : (int)left - 16;
#pragma unroll
      for (int j = 0; j < COUNT; ++j) {
        const int r = row(wave, lane) + j * WAVES * 8;
        load(j, from + (uint32_t)((r < last ? r : last) * ld + c));
      }
    }
    base += 128;
    left -= 128;
  }
};

// Where a lane reads its row's chunk h of 128 k, h = 0..3: 16 k each of the lane's half
// (32 rows on: the same place 4 KB on).
__device__ __forceinline__ uint32_t place_of(int first, int lane) {
  const int r = first + (lane & 31);
  return (uint32_t)(r * 128 + (((lane >> 5) ^ (r / 2 % 8)) << 4));
}

// TW x TX: rows of B and of A in a tile, WW x WX a wavefront's.  ROWS: B has scales
// for each row.  WIDE: the products are made in bf16.
template <int TW, int TX, int WW, int WX, int STAGES, bool ROWS, bool WIDE>
struct Tile8 {
  static constexpr int WAVES = TW / WW * (TX / WX), THREADS = 64 * WAVES;
  static constexpr int MT = WW / 32, NT = WX / 32;
  static constexpr int STAGE = (TW + TX) * 128;
  // Scales of four steps at a time, [step][row], twice: a row's lie next to each other
  // in memory, and each line that is fetched for them gives four.
  static constexpr int SCALES = (TW + TX) * 16, LDS = STAGES * STAGE + 2 * SCALES;
  static constexpr int SHARES = (TW + TX) / 64;  // of 64 rows
  static_assert(SHARES <= WAVES, "a wavefront loads one share of the scales");
  static_assert(WW <= BLOCK8, "a wavefront's rows of B share a scale");
  typedef Share<TW, WAVES> ShareW;
  typedef Share<TX, WAVES> ShareX;
  static constexpr int LOADS = ShareW::COUNT + ShareX::COUNT;

  static __device__ __forceinline__ void run(const Args& a, int64_t w0, int64_t x0, int64_t s0, int64_t s1, char* lds,
                                             f32x16 (&acc)[MT][NT]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ww = wave / (TX / WX), wx0 = wave % (TX / WX) * WX;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const uint32_t at_w = place_of(ww * WW, lane), at_x = TW * 128 + place_of(wx0, lane);
    const int total = (int)(s1 - s0);
    // this wavefront's share of the scales: 64 rows of the tile, B's first (where there
    // are more wavefronts than shares, some write the same to the same place)
    const int sp = wave % SHARES;
    const bool of_w = sp < TW / 64;
    const Held& h = of_w ? a.w : a.x;
    const int64_t h0 = of_w ? w0 : x0, hr = h0 + (of_w ? sp : sp - TW / 64) * 64 + lane;
    const float* const scale = h.scales + h0 / h.tile * h.lds + s0;
    const uint32_t scale_off = (uint32_t)(((hr < h.rows ? hr : h.rows - 1) / h.tile - h0 / h.tile) * h.lds * 4);
    // (steps past the last repeat it)
    const auto issue_scales = [&](int group) {
      char* to = lds + STAGES * STAGE + (group & 1) * SCALES + sp * 256;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int s = group * 4 + q < total ? group * 4 + q : total - 1;
        __builtin_amdgcn_global_load_lds((global_void*)(reinterpret_cast<const char*>(scale + s) + scale_off),
                                         (lds_void*)(to + q * (TW + TX) * 4), 4, 0, 0);
      }
    };
    ShareW sw;
    ShareX sx;
    sw.init(a.w, w0, s0 * 128, a.k, wave, lane);
    sx.init(a.x, x0, s0 * 128, a.k, wave, lane);
    const auto issue = [&](int stage) {
      char* to = lds + stage * STAGE;
      sw.issue(to, wave, lane);
      sx.issue(to + TW * 128, wave, lane);
    };
    issue_scales(0);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
      if (s < total) issue(s);
    int cur = 0;
    for (int s = 0; s < total; ++s) {
      // this step's loads are the oldest ones; the reads of the step before are
      // done in every wavefront before any overwrites their stage
      if (s + STAGES - 2 < total) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS * (STAGES - 2)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      char* const codes_w = lds + cur * STAGE;
      const int tail = (int)((a.k - (s0 + s) * 128) / 16);  // chunks there are
      if (tail < 8) {
        // what was loaded past the last k counts 0 (A's finite codes there, or NaNs of a
        // row that has one anyway, are multiplied with B's zeros)
        for (int i = threadIdx.x; i < TW * 8; i += THREADS)
          if (i % 8 >= tail) *reinterpret_cast<i32x4*>(codes_w + (i / 8) * 128 + (((i % 8) ^ (i / 16 % 8)) << 4)) = i32x4{0, 0, 0, 0};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      if (s + STAGES - 1 < total) issue(cur == 0 ? STAGES - 1 : cur - 1);
      // (the other half was last read before this step's barrier)
      if (s % 4 == 0 && s + 4 < total) issue_scales(s / 4 + 1);
      const float* const scales = reinterpret_cast<const float*>(lds + STAGES * STAGE + (s / 4 & 1) * SCALES) + s % 4 * (TW + TX);
      const uint32_t stage_w = (uint32_t)(cur * STAGE) + at_w, stage_x = (uint32_t)(cur * STAGE) + at_x;
      const auto read = [&](uint32_t at, int block, int h) {  // (stages lie at multiples of 256)
        return *reinterpret_cast<const i32x4*>(lds + (at ^ (h << 5)) + block * 4096);
      };
      float f[NT];
      const float fw = ROWS ? 1.f : scales[ww * WW];
      i32x4 cx[4][NT];      // this lane's codes of A: chunks of 16 k
      bf16x8 wx[WIDE ? 8 : 1][NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        f[j] = scales[TW + wx0 + j * 32 + (lane & 31)] * fw;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          cx[h][j] = read(stage_x, j, h);
          if constexpr (WIDE) {
            wx[2 * h][j] = widen(cx[h][j], 0);
            wx[2 * h + 1][j] = widen(cx[h][j], 1);
          }
        }
      }
      // Products of a 32 x 32 block run while the sums of the one before are scaled.
      f32x16 t[2];
      float row[ROWS ? 16 : 1];  // the scales of this lane's rows
      const auto scale_sums = [&](int i, int j) {
        if constexpr (ROWS)
          if (j == 0)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 v = *reinterpret_cast<const f32x4*>(scales + ww * WW + i * 32 + 8 * q + 4 * (lane >> 5));
              row[4 * q] = v[0]; row[4 * q + 1] = v[1]; row[4 * q + 2] = v[2]; row[4 * q + 3] = v[3];
            }
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] += t[(i * NT + j) & 1][r] * (ROWS ? row[ROWS ? r : 0] * f[j] : f[j]);
      };
      i32x4 cw[2][4];
      const auto read_w = [&](int i) {
#pragma unroll
        for (int h = 0; h < 4; ++h) cw[i & 1][h] = read(stage_w, i, h);
      };
      read_w(0);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (!WIDE)
          if (i + 1 < MT) read_w(i + 1);
        bf16x8 w[WIDE ? 8 : 1];
        if constexpr (WIDE)
#pragma unroll
          for (int h = 0; h < 8; ++h) w[h] = widen(cw[i & 1][h / 2], h % 2);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          f32x16& p = t[(i * NT + j) & 1];
          if constexpr (WIDE) {
#pragma unroll
            for (int h = 0; h < 8; ++h)
              p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[h], wx[h][j], h ? p : f32x16{}, 0, 0, 0);
            if (j == 0 && i + 1 < MT) read_w(i + 1);
          } else {
            const i32x4* const c = cw[i & 1];
            p = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(c[0], c[1]), join(cx[0][j], cx[1][j]), f32x16{}, 0, 0, 0, 0, 0, 0);
            p = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(c[2], c[3]), join(cx[2][j], cx[3][j]), p, 0, 0, 0, 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
          if (j > 0) scale_sums(i, j - 1);
          else if (i > 0) scale_sums(i - 1, NT - 1);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      scale_sums(MT - 1, NT - 1);
      cur = cur == STAGES - 1 ? 0 : cur + 1;
    }
  }

  // Results in type Y to rows [r0, rows) and columns [c0, cols) of a matrix whose row
  // `first` is the tile's matrix's first.
  template <int Y>
  static __device__ __forceinline__ void write(const f32x16 (&acc)[MT][NT], char* to, int64_t first, int64_t ld, int64_t r0,
                                               int64_t c0, int64_t rows, int64_t cols, char* lds) {
    constexpr int SIZE = dtype_bytes(Y), ROW = WW * SIZE + 16, LANES = WW * SIZE / 16, EACH = 16 / SIZE;
    static_assert(WAVES * WX * ROW <= LDS, "a tile's results fit the stages' LDS");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int ww = wave / (TX / WX), wx = wave % (TX / WX);
    char* const mine = lds + wave * WX * ROW;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          char* p = mine + (j * 32 + (lane & 31)) * ROW + (i * 32 + 8 * q + 4 * (lane >> 5)) * SIZE;
          if constexpr (Y == DT_F32) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
          else store4<Y>(p, 0, v);
        }
    wave_sync();
    const int64_t col = c0 + ww * WW + lane % LANES * EACH;
    const int64_t have = cols - col;
#pragma unroll 4
    for (int r = lane / LANES; r < WX; r += 64 / LANES) {
      const int64_t row = r0 + wx * WX + r;
      if (row >= rows || have <= 0) continue;
      const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * ROW + lane % LANES * 16);
      char* const at = to + ((first + row) * ld + col) * SIZE;
      if (have >= EACH) {
        store_vec<true>(reinterpret_cast<u32x4_el2*>(at), (u32x4_el2)v);
      } else if constexpr (Y == DT_F32) {
#pragma unroll
        for (int q = 0; q < EACH - 1; ++q)
          if (q < have) reinterpret_cast<uint32_t*>(at)[q] = v[q];
      } else {
#pragma unroll
        for (int q = 0; q < EACH - 1; ++q)
          if (q < have) reinterpret_cast<uint16_t*>(at)[q] = (uint16_t)(v[q / 2] >> (16 * (q & 1)));
      }
    }
  }
};

template <int TW, int TX, int WW, int WX, int STAGES, bool ROWS, bool WIDE>
__global__ __launch_bounds__(TW / WW * (TX / WX) * 64, 2) void k_tiles8(Args a) {
  typedef Tile8<TW, TX, WW, WX, STAGES, ROWS, WIDE> T;
  __shared__ __attribute__((aligned(16))) char lds[T::LDS];
  int64_t ty, tx;
  place_tile(blockIdx.x, (a.y.rows + TX - 1) / TX, (a.y.cols + TW - 1) / TW, 8, ty, tx);
  const int64_t s0 = blockIdx.y * a.per, s1 = s0 + a.per < a.steps ? s0 + a.per : a.steps;
  f32x16 acc[T::MT][T::NT];
  T::run(a, tx * TW, ty * TX, s0, s1, lds, acc);
  // Each wavefront's results through LDS, so that rows of Y are written in runs of
  // its WW columns.
  const bool part = a.part != nullptr;
  const int type = part ? (int)DT_F32 : a.y.type;
  char* const to = static_cast<char*>(part ? (void*)a.part : a.y.data);
  const int64_t ld = part ? a.y.cols : a.y.ld, r0 = ty * TX, c0 = tx * TW;
  const int64_t first = part ? (int64_t)blockIdx.y * a.y.rows : 0;
  __syncthreads();  // the stages' LDS changes its use
  if constexpr (TW < 256)  // (the largest tiles have 16-bit results and share no k)
    if (type == DT_F32) return T::template write<DT_F32>(acc, to, first, ld, r0, c0, a.y.rows, a.y.cols, lds);
  if (type == DT_BF16) T::template write<DT_BF16>(acc, to, first, ld, r0, c0, a.y.rows, a.y.cols, lds);
  else T::template write<DT_F16>(acc, to, first, ld, r0, c0, a.y.rows, a.y.cols, lds);
}

// Y: the splits' sums.  Four values a lane; SHARES of a workgroup's wavefronts each add
// every SHARES-th split, and their sums are added in their order: eight where there are few
// values and as many splits, which waits for memory less often (181 x 38 in 17 splits 5.2 us
// against 12; 1000 x 520 in 12 splits 7.2 against 6.5).  (64 MB of sums at most: 32-bit
// places.)
template <int SHARES>
__global__ __launch_bounds__(256) void k_join8(Mat y, const float* part, int splits) {
  __shared__ float sums[SHARES - 1 ? SHARES - 1 : 1][256 / SHARES][4];
  constexpr int LANES = 256 / SHARES;
  const uint32_t cols = (uint32_t)y.cols, values = (uint32_t)y.rows * cols;
  const int lane = threadIdx.x % LANES, share = threadIdx.x / LANES;
  const uint32_t i = (blockIdx.x * LANES + lane) * 4;
  const int have = i >= values ? 0 : values - i < 4 ? (int)(values - i) : 4;
  float v[4] = {};
  if (have == 4) {
#pragma unroll 4
    for (int s = share; s < splits; s += SHARES) {
      float x[4];
      load4<DT_F32>(part + (int64_t)s * values, i, x);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += x[q];
    }
  } else {
    for (int s = share; s < splits; s += SHARES)
      for (int q = 0; q < have; ++q) v[q] += part[(int64_t)s * values + i + q];
  }
  if constexpr (SHARES > 1) {
    if (share > 0)
#pragma unroll
      for (int q = 0; q < 4; ++q) sums[share - 1][lane][q] = v[q];
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int u = 0; u < SHARES - 1; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += sums[u][lane][q];
  }
  const uint32_t row = i / cols, col = i % cols;
  if (col + 4 <= cols && have == 4) {
    const int64_t at = row * y.ld + col;
    if (y.type == DT_F32) store4<DT_F32>(y.data, at, v);
    else if (y.type == DT_BF16) store4<DT_BF16>(y.data, at, v);
    else store4<DT_F16>(y.data, at, v);
  } else {
    for (int q = 0; q < have; ++q) {
      const uint32_t r = (i + q) / cols;
      store1(y.data, y.type, r * y.ld + (i + q - r * cols), v[q]);
    }
  }
}

// -------------------------------------------------------------- few rows of A

struct Codes {  // of a lane: chunks of 16 k
  i32x4 c[2];
};

constexpr int ROW_WAVES = 8;
constexpr int kFewRows = 16;

// All rows of A against 16 rows of B a workgroup; its wavefronts (eight; four and sixteen
// make no difference) take steps of 128 k in turn, two at a time.  A lane holds 32 k of its row: chunks of 16 bytes, 64 bytes
// apart, so that a load covers 64 contiguous bytes of a row.  (With two or four times
// 16 rows of A the tiles are faster: 17 x 8192 x 8192 18 us against 23, 64 x 8192 x 2048 9
// against 16.)
// ODD: rows begin at any address (the first at a multiple of 4).  The words that a chunk's
// bytes lie in are loaded and moved to their places, five words a chunk: a load of 16 bytes
// at an odd address takes several times as long (2 x 4868 x 5311 15 us, 23 by such loads;
// at multiples of 4 it makes no difference).
template <bool ROWS, bool ODD>
__global__ __launch_bounds__(64 * ROW_WAVES) void k_rows8(Args a) {
  __shared__ float sums[ROW_WAVES][64][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w0 = (int64_t)blockIdx.x * 16;
  const auto clamp = [](int64_t r, const Held& h) { return r < h.rows ? r : h.rows - 1; };
  const int64_t xr = clamp(lane & 15, a.x);
  const uint8_t* const wp = a.w.codes + clamp(w0 + (lane & 15), a.w) * a.w.ld + (lane >> 4) * 16;
  const uint8_t* const xp = a.x.codes + xr * a.x.ld + (lane >> 4) * 16;
  const float* const xs = a.x.scales + xr * a.x.lds;
  const float* ws[ROWS ? 4 : 1];
#pragma unroll
  for (int q = 0; q < (ROWS ? 4 : 1); ++q)
    ws[q] = a.w.scales + clamp(ROWS ? w0 + (lane >> 4) * 4 + q : w0, a.w) / a.w.tile * a.w.lds;
  f32x4 acc = {};
  const auto step = [&](int64_t s, const Codes& w, const Codes& x) {
    float f[ROWS ? 4 : 1];
#pragma unroll
    for (int q = 0; q < (ROWS ? 4 : 1); ++q) f[q] = ws[q][s];
    const float fx = xs[s];
    f32x4 v = {};
#pragma unroll
    for (int h = 0; h < 4; ++h)
      v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.c[h / 2], h % 2), widen(x.c[h / 2], h % 2), v, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] = fmaf(v[q], f[ROWS ? q : 0] * fx, acc[q]);
  };
  const auto words = [&](const uint8_t* p) {
    const uint32_t by = (uint32_t)reinterpret_cast<uintptr_t>(p) & 3;
    const uint32_t* const q = reinterpret_cast<const uint32_t*>(p - by);
    const u32x4 w = *reinterpret_cast<const u32x4_el4*>(q);
    const uint32_t last = q[4];
    i32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = (int)__builtin_amdgcn_alignbyte(i < 3 ? w[i < 3 ? i + 1 : 3] : last, w[i], by);
    return c;
  };
  const auto whole = [&](const uint8_t* p, int64_t s) {
    if constexpr (ODD) return Codes{words(p + s * 128), words(p + s * 128 + 64)};
    return Codes{*reinterpret_cast<const i32x4_el1*>(p + s * 128), *reinterpret_cast<const i32x4_el1*>(p + s * 128 + 64)};
  };
  // (the words of a chunk end at most 4 bytes behind it: those are the row's own)
  const int64_t full = ODD ? (a.k >= 4 ? a.k - 4 : 0) / 128 : a.k / 128;
  int64_t s = wave;
  for (; s + ROW_WAVES < full; s += 2 * ROW_WAVES) {
    const int64_t u = s + ROW_WAVES;
    const Codes w0v = whole(wp, s), w1v = whole(wp, u), x0v = whole(xp, s), x1v = whole(xp, u);
    step(s, w0v, x0v);
    step(u, w1v, x1v);
  }
  for (; s < a.steps; s += ROW_WAVES) {
    const int64_t have = a.k - s * 128 - (lane >> 4) * 16;
    const auto some = [&](const uint8_t* p, auto load) { return Codes{load(p + s * 128, have), load(p + s * 128 + 64, have - 64)}; };
    if (a.k >= 16) step(s, some(wp, load16_moved), some(xp, load16_moved));
    else step(s, some(wp, load16), some(xp, load16));
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) sums[wave][lane][q] = acc[q];
  __syncthreads();
  if (wave != 0) return;
  float v[4] = {};
#pragma unroll
  for (int u = 0; u < ROW_WAVES; ++u)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += sums[u][lane][q];
  store_y(a, lane & 15, w0 + (lane >> 4) * 4, v);
}

__global__ __launch_bounds__(256) void k_zero8(Mat y) {
  const int64_t values = y.rows * y.cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < values; i += (int64_t)gridDim.x * 256)
    store1(y.data, y.type, i / y.cols * y.ld + i % y.cols, 0.f);
}

// Rows of codes as chunks of 16 bytes, zeros past the last column (1520 x 65537: 36 us, 5.6
// TB/s; the tiles read codes that lie so straight to LDS, which by way of registers took
// more of them than there are).
// Both operands in one launch; one that is not copied has no rows here.
__global__ __launch_bounds__(256) void k_pack8(Held a, Held b, uint8_t* to, int64_t chunks) {
  const int64_t total = (a.rows + b.rows) * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / chunks, c = i % chunks * 16;
    const uint8_t* const row = r < a.rows ? a.codes + r * a.ld : b.codes + (r - a.rows) * b.ld;
    reinterpret_cast<i32x4*>(to)[i] = load16(row + c, a.cols - c);
  }
}

// What a product of these sizes is made with.
struct Way {
  int tile;        // rows of A and of B in a tile; 0: few rows of A
  int64_t splits, per;
};

constexpr int64_t kPartBytes = int64_t(64) << 20;

// Tiles of 256 where there are enough for the chip (not where B's rows have scales of their
// own, or the products are wide: those need the registers: 16384 x 8192 x 4096 722 us against
// 798), of 128 where there are enough of those (2048 x 2048 x 2048 17 us, 22 with 64, 26
// with 128 and k in two), else of 64 (300 x 4096 x 2048 12.5 us, 15 with 128); k is split
// where there are few tiles and many steps (256 x 256 x 8192 14 us in 8 shares, 31 in
// one; 300 x 1024 x 1024 6.5 in one, 9 in two), and with much work in tiles of 128 (1000 x 520 x
// 65536).
Way way_of(int64_t m, int64_t n, int64_t k, bool rows, bool wide) {
  const int64_t steps = (k + 127) / 128;
  if (m <= kFewRows) return {0, 1, steps};
  const auto tiles = [&](int64_t t) { return (m + t - 1) / t * ((n + t - 1) / t); };
  if (!rows && !wide && tiles(256) >= 200) return {256, 1, steps};
  if (tiles(128) >= 192) return {128, 1, steps};
  const bool much = tiles(128) * steps >= 4096;
  const int tile = much ? 128 : 64;
  // (two workgroups of tiles of 128 to a CU: one more than 512 of them takes twice the time)
  const int64_t fill = much ? 512 / tiles(128) : tiles(64) <= 160 ? (512 + tiles(64) / 2) / tiles(64) : 1;
  int64_t splits = std::max<int64_t>(1, std::min({fill, steps / 8, kPartBytes / (m * n * 4)}));
  const int64_t per = (steps + splits - 1) / splits;
  splits = (steps + per - 1) / per;
  return {tile, splits, per};
}

template <int TW, int TX, int WW, int WX, int STAGES, bool ROWS, bool WIDE>
hipError_t launch(const Args& a, const Way& w, hipStream_t s) {
  const int64_t tiles = (a.y.rows + TX - 1) / TX * ((a.y.cols + TW - 1) / TW);
  const dim3 grid((unsigned)tiles, (unsigned)w.splits);
  k_tiles8<TW, TX, WW, WX, STAGES, ROWS, WIDE><<<grid, TW / WW * (TX / WX) * 64, 0, s>>>(a);
  return hipGetLastError();
}

template <bool ROWS, bool WIDE>
hipError_t launch(const Args& a, const Way& w, hipStream_t s) {
  if constexpr (!ROWS && !WIDE)
    if (w.tile == 256) return launch<256, 256, 128, 64, 2, ROWS, WIDE>(a, w, s);
  if (w.tile == 128) return launch<128, 128, 64, 64, 2, ROWS, WIDE>(a, w, s);
  return launch<64, 64, 32, 32, 3, ROWS, WIDE>(a, w, s);
}

// Whether h's rows are chunks of 16 bytes, and the bytes of a copy that is.
bool chunks(const Held& h) {
  return reinterpret_cast<uintptr_t>(h.codes) % 16 == 0 && h.cols % 16 == 0 && (h.ld % 16 == 0 || h.rows == 1);
}
int64_t packed_bytes(const Held& h) { return chunks(h) ? 0 : h.rows * ((h.cols + 15) / 16 * 16); }

// Operands that are copied, to `to`.
hipError_t pack(Held& a, Held& b, uint8_t* to, hipStream_t s) {
  const int64_t of_a = packed_bytes(a), of_b = packed_bytes(b), chunks = (a.cols + 15) / 16;
  if (of_a + of_b == 0) return hipSuccess;
  Held x = a, y = b;
  if (of_a == 0) x.rows = 0;
  if (of_b == 0) y.rows = 0;
  k_pack8<<<(unsigned)std::min<int64_t>(((of_a + of_b) / 16 + 255) / 256, 1 << 16), 256, 0, s>>>(x, y, to, chunks);
  if (of_a) a.codes = to, a.ld = chunks * 16;
  if (of_b) b.codes = to + of_a, b.ld = chunks * 16;
  return hipGetLastError();
}

}  // namespace

int64_t matmul8_workspace(const Held& A, const Held& B, int type) {
  const int64_t m = A.rows, n = B.rows, k = A.cols;
  if (m == 0 || n == 0 || k == 0) return 0;
  const Way w = way_of(m, n, k, B.tile == 1, type == DT_F32);
  const int64_t part = w.splits > 1 ? (w.splits * m * n * (int64_t)sizeof(float) + 15) / 16 * 16 : 0;
  return part + (w.tile ? packed_bytes(A) + packed_bytes(B) : 0);
}

hipError_t matmul8(const Held& A, const Held& B, const Mat& Y, void* ws, hipStream_t s) {
  const int64_t m = Y.rows, n = Y.cols, k = A.cols;
  if (m == 0 || n == 0) return hipSuccess;
  if (k == 0) {
    k_zero8<<<(unsigned)std::min<int64_t>((m * n + 255) / 256, 1 << 16), 256, 0, s>>>(Y);
    return hipGetLastError();
  }
  const bool rows = B.tile == 1, wide = Y.type == DT_F32;
  const Way w = way_of(m, n, k, rows, wide);
  Args a{A, B, Y, nullptr, k, (k + 127) / 128, w.per};
  if (w.tile == 0) {
    const dim3 grid((unsigned)((n + 15) / 16));
    const auto at4 = [](const Held& h) { return reinterpret_cast<uintptr_t>(h.codes) % 4 == 0; };
    const auto rows4 = [](const Held& h) { return h.ld % 4 == 0 || h.rows == 1; };
    const bool odd = at4(A) && at4(B) && !(rows4(A) && rows4(B));
    if (rows && odd) k_rows8<true, true><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    else if (rows) k_rows8<true, false><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    else if (odd) k_rows8<false, true><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    else k_rows8<false, false><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    return hipGetLastError();
  }
  uint8_t* place = static_cast<uint8_t*>(ws);
  if (w.splits > 1) {
    a.part = static_cast<float*>(ws);
    place += (w.splits * m * n * (int64_t)sizeof(float) + 15) / 16 * 16;
  }
  hipError_t e = pack(a.x, a.w, place, s);
  if (e != hipSuccess) return e;
  a.k = (k + 15) / 16 * 16;
  if (rows) e = wide ? launch<true, true>(a, w, s) : launch<true, false>(a, w, s);
  else e = wide ? launch<false, true>(a, w, s) : launch<false, false>(a, w, s);
  if (e != hipSuccess || w.splits == 1) return e;
  const int64_t quads = (m * n + 3) / 4;
  if (w.splits >= 8 && quads <= 65536) k_join8<8><<<(unsigned)((quads + 31) / 32), 256, 0, s>>>(Y, a.part, (int)w.splits);
  else k_join8<1><<<(unsigned)((quads + 255) / 256), 256, 0, s>>>(Y, a.part, (int)w.splits);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
