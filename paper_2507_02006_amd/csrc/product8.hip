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
// Three forms.  Up to 64 rows of A ("rows"): bound by B's bytes, which go from
// memory to the matrix cores' registers, no LDS; a workgroup owns 16 rows of B and
// its wavefronts share k.  Else tiles: stages of 128 k go from global memory
// straight to LDS, their 16-byte chunks placed as in tile.h.  Where the
// operands' rows are not chunks of 16 bytes they go through registers, which
// put zeros past the last k.  Where there are few tiles k is split over
// workgroups, whose partial sums a second launch adds in a fixed order.
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
  int64_t k, steps; // steps of 128 k
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

__device__ __forceinline__ void store_y(const Args& a, int64_t row, int64_t col, int split, const float (&v)[4]) {
  if (row >= a.y.rows || col >= a.y.cols) return;
  const bool part = a.part != nullptr;
  void* const to = part ? a.part : a.y.data;
  const int64_t at = part ? ((int64_t)split * a.y.rows + row) * a.y.cols + col : row * a.y.ld + col;
  const int t = part ? (int)DT_F32 : a.y.type;
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

// One operand's share of a stage through registers: SPAN rows of 128 k.
template <int SPAN, int WAVES>
struct Copier {
  static constexpr int TOTAL = SPAN / 8, COUNT = (TOTAL + WAVES - 1) / WAVES;
  const uint8_t* base;
  int64_t left;
  uint32_t off[COUNT];
  int at[COUNT];
  i32x4 held[COUNT];

  __device__ void init(const Held& h, int64_t r0, int64_t k0, int64_t k, int wave, int lane) {
    base = h.codes + r0 * h.ld + k0;
    left = k - k0;
    const int64_t last = h.rows - 1 - r0;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const int r = part_of<TOTAL, WAVES>(j, wave) * 8 + lane / 8;
      at[j] = ((lane % 8) ^ (r / 2 % 8)) * 16;
      off[j] = (uint32_t)((r < last ? r : last) * h.ld + at[j]);
    }
  }
  __device__ __forceinline__ void load() {
#pragma unroll
    for (int j = 0; j < COUNT; ++j) held[j] = load16(base + off[j], left - at[j]);
    base += 128;
    left -= 128;
  }
  __device__ __forceinline__ void store(char* lds, int wave, int lane) const {
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
      *reinterpret_cast<i32x4*>(lds + part_of<TOTAL, WAVES>(j, wave) * 1024 + lane * 16) = held[j];
  }
};

// TW x TX: rows of B and of A in a tile, WW x WX a wavefront's.  ROWS: B has scales
// for each row.  DIRECT: rows are chunks of 16 bytes and go straight to LDS.  WIDE:
// the products are made in bf16.
template <int TW, int TX, int WW, int WX, int STAGES, bool ROWS, bool DIRECT, bool WIDE>
struct Tile8 {
  static constexpr int WAVES = TW / WW * (TX / WX), THREADS = 64 * WAVES;
  static constexpr int MT = WW / 32, NT = WX / 32;
  static constexpr int CODES = (TW + TX) * 128, STAGE = CODES + (TW + TX) * 4, LDS = STAGES * STAGE;
  static constexpr int SCALES = (TW + TX) / 64;  // loads of 64 scales
  static_assert(SCALES <= WAVES, "a wavefront loads 64 scales a stage");
  static_assert(WW <= BLOCK8, "a wavefront's rows of B share a scale");
  static constexpr int LOADS = Stager<TW, WAVES, false>::COUNT + Stager<TX, WAVES, false>::COUNT + 1;

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
    const Reader<TW, WW, false> rw(ww * WW, lane);
    const Reader<TX, WX, false> rx(wx0, lane);
    const int total = (int)(s1 - s0);
    // this wavefront's scales: 64 rows of the tile, B's first
    const int sp = wave % SCALES;
    const float* scale;
    {
      const bool of_w = sp < TW / 64;
      const Held& h = of_w ? a.w : a.x;
      const int64_t r = (of_w ? w0 + sp * 64 : x0 + (sp - TW / 64) * 64) + lane;
      scale = h.scales + (r < h.rows ? r : h.rows - 1) / h.tile * h.lds + s0;
    }
    Stager<TW, WAVES, false> sw;
    Stager<TX, WAVES, false> sx;
    Copier<TW, WAVES> copy_w;
    Copier<TX, WAVES> copy_x;
    float held = 0.f;
    if constexpr (DIRECT) {
      const Panel pw{reinterpret_cast<const uint16_t*>(a.w.codes), a.w.ld / 2, a.w.rows, a.k / 2};
      const Panel px{reinterpret_cast<const uint16_t*>(a.x.codes), a.x.ld / 2, a.x.rows, a.k / 2};
      sw.init(pw, w0, s0 * 64, wave, lane);
      sx.init(px, x0, s0 * 64, wave, lane);
    } else {
      copy_w.init(a.w, w0, s0 * 128, a.k, wave, lane);
      copy_x.init(a.x, x0, s0 * 128, a.k, wave, lane);
    }
    auto issue = [&](int stage) {  // DIRECT
      char* to = lds + stage * STAGE;
      if (sw.left < BK) {
        const Panel pw{nullptr, a.w.ld / 2, a.w.rows, a.k / 2}, px{nullptr, a.x.ld / 2, a.x.rows, a.k / 2};
        sw.place(pw, w0, wave, lane);
        sx.place(px, x0, wave, lane);
      }
      sw.issue(to, wave);
      sx.issue(to + TW * 128, wave);
      __builtin_amdgcn_global_load_lds((global_void*)scale, (lds_void*)(to + CODES + sp * 256), 4, 0, 0);
      sw.base += sw.step;
      sx.base += sx.step;
      sw.left -= BK;
      sx.left -= BK;
      ++scale;
    };
    auto load = [&]() {  // not DIRECT
      copy_w.load();
      copy_x.load();
      held = *scale++;
    };
    auto store = [&](int stage) {
      char* to = lds + stage * STAGE;
      copy_w.store(to, wave, lane);
      copy_x.store(to + TW * 128, wave, lane);
      reinterpret_cast<float*>(to + CODES)[sp * 64 + lane] = held;
    };
    if constexpr (DIRECT) {
#pragma unroll
      for (int s = 0; s < STAGES - 1; ++s)
        if (s < total) issue(s);
    } else {
      load();
      store(0);
      if (total > 1) load();
    }
    int cur = 0;
    for (int s = 0; s < total; ++s) {
      // this step's loads are the oldest ones; the reads of the step before are
      // done in every wavefront before any overwrites their stage
      if constexpr (DIRECT) {
        if (s + STAGES - 2 < total) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS * (STAGES - 2)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      } else {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      char* const codes_w = lds + cur * STAGE;
      if constexpr (DIRECT) {
        const int tail = (int)((a.k - (s0 + s) * 128) / 16);  // chunks there are
        if (tail < 8) {
          // what was loaded past the last k counts 0 (A's finite codes there, or
          // NaNs of a row that has one anyway, are multiplied with B's zeros)
          for (int i = threadIdx.x; i < TW * 8; i += THREADS)
            if (i % 8 >= tail) *reinterpret_cast<i32x4*>(codes_w + (i / 8) * 128 + (((i % 8) ^ (i / 16 % 8)) << 4)) = i32x4{0, 0, 0, 0};
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
        if (s + STAGES - 1 < total) issue(cur == 0 ? STAGES - 1 : cur - 1);
      }
      const char* const codes_x = codes_w + TW * 128;
      const float* const scales = reinterpret_cast<const float*>(codes_w + CODES);
      float f[NT];
      const float fw = ROWS ? 1.f : scales[ww * WW];
      i32x4 cx[4][NT];      // this lane's codes of A: chunks of 16 k
      bf16x8 wx[WIDE ? 8 : 1][NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        f[j] = scales[TW + wx0 + j * 32 + (lane & 31)] * fw;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          cx[h][j] = __builtin_bit_cast(i32x4, rx.get(codes_x, j, h));
          if constexpr (WIDE) {
            wx[2 * h][j] = widen(cx[h][j], 0);
            wx[2 * h + 1][j] = widen(cx[h][j], 1);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        i32x4 cw[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) cw[h] = __builtin_bit_cast(i32x4, rw.get(codes_w, i, h));
        f32x4 row[4];  // ROWS: the scales of this lane's rows
        if constexpr (ROWS)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            row[q] = *reinterpret_cast<const f32x4*>(scales + ww * WW + i * 32 + 8 * q + 4 * (lane >> 5));
        f32x16 t[NT];
        if constexpr (WIDE) {
#pragma unroll
          for (int h = 0; h < 8; ++h) {
            const bf16x8 w = widen(cw[h / 2], h % 2);
#pragma unroll
            for (int j = 0; j < NT; ++j)
              t[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, wx[h][j], h ? t[j] : f32x16{}, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int j = 0; j < NT; ++j)
            t[j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(cw[0], cw[1]), join(cx[0][j], cx[1][j]), f32x16{}, 0, 0, 0, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < NT; ++j)
            t[j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(cw[2], cw[3]), join(cx[2][j], cx[3][j]), t[j], 0, 0, 0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if constexpr (ROWS) acc[i][j][r] += t[j][r] * (row[r / 4][r % 4] * f[j]);
            else acc[i][j][r] += t[j][r] * f[j];
          }
      }
      if constexpr (!DIRECT)
        if (s + 1 < total) {
          store(cur ^ 1);
          if (s + 2 < total) load();
        }
      cur = cur == STAGES - 1 ? 0 : cur + 1;
    }
  }
};

template <int TW, int TX, int WW, int WX, int STAGES, bool ROWS, bool DIRECT, bool WIDE>
__global__ __launch_bounds__(TW / WW * (TX / WX) * 64) void k_tiles8(Args a) {
  typedef Tile8<TW, TX, WW, WX, STAGES, ROWS, DIRECT, WIDE> T;
  static_assert(DIRECT || STAGES == 2, "through registers: two stages");
  __shared__ __attribute__((aligned(16))) char lds[T::LDS];
  int64_t ty, tx;
  place_tile(blockIdx.x, (a.y.rows + TX - 1) / TX, (a.y.cols + TW - 1) / TW, 8, ty, tx);
  const int64_t s0 = blockIdx.y * a.per, s1 = s0 + a.per < a.steps ? s0 + a.per : a.steps;
  f32x16 acc[T::MT][T::NT];
  T::run(a, tx * TW, ty * TX, s0, s1, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ww = wave / (TX / WX), wx = wave % (TX / WX);
#pragma unroll
  for (int j = 0; j < T::NT; ++j) {
    const int64_t row = ty * TX + wx * WX + j * 32 + (lane & 31);
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        store_y(a, row, tx * TW + ww * WW + i * 32 + 8 * q + 4 * (lane >> 5), blockIdx.y, v);
      }
  }
}

// Y: the splits' sums, added in their order.
__global__ __launch_bounds__(256) void k_join8(Mat y, const float* part, int splits) {
  const int64_t values = y.rows * y.cols;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < values; i += (int64_t)gridDim.x * 1024) {
    float v[4] = {};
    const int have = values - i < 4 ? (int)(values - i) : 4;
    for (int s = 0; s < splits; ++s) {
      const float* p = part + s * values + i;
      if (have == 4) {
        float x[4];
        load4<DT_F32>(p, 0, x);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += x[q];
      } else {
        for (int q = 0; q < have; ++q) v[q] += p[q];
      }
    }
    int64_t row = i / y.cols, col = i % y.cols;
    for (int q = 0; q < have; ++q) {
      store1(y.data, y.type, row * y.ld + col, v[q]);
      if (++col == y.cols) {
        col = 0;
        ++row;
      }
    }
  }
}

// -------------------------------------------------------------- few rows of A

struct Codes {  // of a lane: chunks of 16 k
  i32x4 c[2];
};

constexpr int ROW_WAVES = 8;
constexpr int kFewRows = 64;

// XT x 16 rows of A against 16 rows of B a workgroup; its wavefronts take steps
// of 128 k in turn, two at a time.  A lane holds 32 k of its row: chunks of 16 bytes,
// 64 bytes apart, so that a load covers 64 contiguous bytes of a row.
template <int XT, bool ROWS>
__global__ __launch_bounds__(64 * ROW_WAVES) void k_rows8(Args a) {
  __shared__ float sums[ROW_WAVES][XT][64][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w0 = (int64_t)blockIdx.x * 16;
  const int64_t wr = w0 + (lane & 15) < a.w.rows ? w0 + (lane & 15) : a.w.rows - 1;
  const uint8_t* const wp = a.w.codes + wr * a.w.ld + (lane >> 4) * 16;
  const uint8_t* xp[XT];
  const float* xs[XT];
  const float* ws[ROWS ? 4 : 1];
#pragma unroll
  for (int t = 0; t < XT; ++t) {
    const int64_t r = t * 16 + (lane & 15) < a.x.rows ? t * 16 + (lane & 15) : a.x.rows - 1;
    xp[t] = a.x.codes + r * a.x.ld + (lane >> 4) * 16;
    xs[t] = a.x.scales + r * a.x.lds;
  }
#pragma unroll
  for (int q = 0; q < (ROWS ? 4 : 1); ++q) {
    const int64_t r = ROWS ? w0 + (lane >> 4) * 4 + q : w0;
    ws[q] = a.w.scales + (r < a.w.rows ? r : a.w.rows - 1) / a.w.tile * a.w.lds;
  }
  f32x4 acc[XT] = {};
  const auto step = [&](int64_t s, const Codes& w, const Codes (&x)[XT]) {
    float f[ROWS ? 4 : 1];
#pragma unroll
    for (int q = 0; q < (ROWS ? 4 : 1); ++q) f[q] = ws[q][s];
#pragma unroll
    for (int t = 0; t < XT; ++t) {
      const float fx = xs[t][s];
      f32x4 v = {};
#pragma unroll
      for (int h = 0; h < 4; ++h)
        v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.c[h / 2], h % 2), widen(x[t].c[h / 2], h % 2), v, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[t][q] += v[q] * (f[ROWS ? q : 0] * fx);
    }
  };
  const auto whole = [&](const uint8_t* p, int64_t s) {
    return Codes{*reinterpret_cast<const i32x4_el1*>(p + s * 128), *reinterpret_cast<const i32x4_el1*>(p + s * 128 + 64)};
  };
  const int64_t full = a.k / 128;
  int64_t s = wave;
  for (; s + ROW_WAVES < full; s += 2 * ROW_WAVES) {
    const int64_t u = s + ROW_WAVES;
    const Codes w0v = whole(wp, s), w1v = whole(wp, u);
    Codes x0v[XT], x1v[XT];
#pragma unroll
    for (int t = 0; t < XT; ++t) {
      x0v[t] = whole(xp[t], s);
      x1v[t] = whole(xp[t], u);
    }
    step(s, w0v, x0v);
    step(u, w1v, x1v);
  }
  for (; s < a.steps; s += ROW_WAVES) {
    const int64_t have = a.k - s * 128 - (lane >> 4) * 16;
    Codes x[XT];
#pragma unroll
    for (int t = 0; t < XT; ++t) x[t] = Codes{load16(xp[t] + s * 128, have), load16(xp[t] + s * 128 + 64, have - 64)};
    step(s, Codes{load16(wp + s * 128, have), load16(wp + s * 128 + 64, have - 64)}, x);
  }
#pragma unroll
  for (int t = 0; t < XT; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[wave][t][lane][q] = acc[t][q];
  __syncthreads();
  for (int i = threadIdx.x; i < XT * 64; i += 64 * ROW_WAVES) {
    const int t = i / 64, l = i % 64;
    float v[4] = {};
#pragma unroll
    for (int u = 0; u < ROW_WAVES; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += sums[u][t][l][q];
    store_y(a, t * 16 + (l & 15), w0 + (l >> 4) * 4, 0, v);
  }
}

__global__ __launch_bounds__(256) void k_zero8(Mat y) {
  const int64_t values = y.rows * y.cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < values; i += (int64_t)gridDim.x * 256)
    store1(y.data, y.type, i / y.cols * y.ld + i % y.cols, 0.f);
}

// What a product of these sizes is made with.
struct Way {
  int tile;        // rows of A and of B in a tile; 0: few rows of A
  int64_t splits, per;
};

constexpr int64_t kPartBytes = int64_t(64) << 20;

Way way_of(int64_t m, int64_t n, int64_t k, bool direct, bool wide) {
  const int64_t steps = (k + 127) / 128;
  if (m <= kFewRows) return {0, 1, steps};
  const auto tiles = [&](int64_t t) { return (m + t - 1) / t * ((n + t - 1) / t); };
  if (direct && !wide && tiles(256) >= 200) return {256, 1, steps};
  const int tile = tiles(128) >= 256 || steps >= 64 ? 128 : 64;
  const int64_t want = 512 / tiles(tile);
  int64_t splits = std::max<int64_t>(1, std::min({want, steps / 8, kPartBytes / (m * n * 4)}));
  const int64_t per = (steps + splits - 1) / splits;
  splits = (steps + per - 1) / per;
  return {tile, splits, per};
}

template <int TW, int TX, int WW, int WX, int STAGES, bool DIRECT, bool WIDE>
hipError_t launch(const Args& a, const Way& w, hipStream_t s) {
  const int64_t tiles = (a.y.rows + TX - 1) / TX * ((a.y.cols + TW - 1) / TW);
  const dim3 grid((unsigned)tiles, (unsigned)w.splits);
  constexpr int threads = TW / WW * (TX / WX) * 64;
  if (a.w.tile == 1) k_tiles8<TW, TX, WW, WX, STAGES, true, DIRECT, WIDE><<<grid, threads, 0, s>>>(a);
  else k_tiles8<TW, TX, WW, WX, STAGES, false, DIRECT, WIDE><<<grid, threads, 0, s>>>(a);
  return hipGetLastError();
}

template <bool WIDE>
hipError_t launch(const Args& a, const Way& w, bool direct, hipStream_t s) {
  if (w.tile == 128)
    return direct ? launch<128, 128, 64, 64, 2, true, WIDE>(a, w, s) : launch<128, 128, 64, 64, 2, false, WIDE>(a, w, s);
  return direct ? launch<64, 64, 32, 32, 3, true, WIDE>(a, w, s) : launch<64, 64, 32, 32, 2, false, WIDE>(a, w, s);
}

// Rows that are chunks of 16 bytes.
bool chunks(const Held& h) {
  return reinterpret_cast<uintptr_t>(h.codes) % 16 == 0 && h.cols % 16 == 0 && (h.ld % 16 == 0 || h.rows == 1);
}

}  // namespace

int64_t matmul8_workspace(int64_t m, int64_t n, int64_t k) {
  if (m == 0 || n == 0 || k == 0) return 0;
  int64_t most = 0;
  for (int i = 0; i < 4; ++i) {
    const Way w = way_of(m, n, k, i & 1, i & 2);
    if (w.splits > 1) most = std::max(most, w.splits * m * n * (int64_t)sizeof(float));
  }
  return most;
}

hipError_t matmul8(const Held& A, const Held& B, const Mat& Y, void* ws, hipStream_t s) {
  const int64_t m = Y.rows, n = Y.cols, k = A.cols;
  if (m == 0 || n == 0) return hipSuccess;
  if (k == 0) {
    k_zero8<<<(unsigned)std::min<int64_t>((m * n + 255) / 256, 1 << 16), 256, 0, s>>>(Y);
    return hipGetLastError();
  }
  const bool direct = chunks(A) && chunks(B);
  const bool wide = Y.type == DT_F32;
  const Way w = way_of(m, n, k, direct, wide);
  Args a{A, B, Y, w.splits > 1 ? static_cast<float*>(ws) : nullptr, k, (k + 127) / 128, w.per};
  if (w.tile == 0) {
    const dim3 grid((unsigned)((n + 15) / 16));
    const int xt = m <= 16 ? 1 : m <= 32 ? 2 : 4;
    if (B.tile == 1) {
      if (xt == 1) k_rows8<1, true><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
      else if (xt == 2) k_rows8<2, true><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
      else k_rows8<4, true><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    } else {
      if (xt == 1) k_rows8<1, false><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
      else if (xt == 2) k_rows8<2, false><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
      else k_rows8<4, false><<<grid, 64 * ROW_WAVES, 0, s>>>(a);
    }
    return hipGetLastError();
  }
  hipError_t e;
  if (w.tile == 256) e = launch<256, 256, 128, 64, 2, true, false>(a, w, s);
  else e = wide ? launch<true>(a, w, direct, s) : launch<false>(a, w, direct, s);
  if (e != hipSuccess || w.splits == 1) return e;
  k_join8<<<(unsigned)std::min<int64_t>((m * n + 1023) / 1024, 2048), 256, 0, s>>>(Y, a.part, (int)w.splits);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
