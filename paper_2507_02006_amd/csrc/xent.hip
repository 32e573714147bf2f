// Softmax cross entropy of scores H W^T against labels, with both gradients,
// without storing the scores (gfx950).
//
// With z = H W^T and s_i = log sum_j exp(z_ij): row_loss_i = s_i - z_i,label,
// dz_ij = scale (exp(z_ij - s_i) - [j = label(i)]) for labelled rows and 0 for
// others, dH = dz W, dW = dz^T H.  2 T V D flops make the scores and as many
// each gradient.  The scores are made twice, 8 T V D in all: once for each
// tile's row maxima and sums of exponentials, joined to those of the row, and the
// labels' scores, which the tile that holds them writes (the loss of a row whose
// label dominates is a difference of equal numbers: they have to be the same
// ones), and once more in pieces of the table for dz, which goes to the workspace in 16
// bits (a piece fits the 256 MB cache) and is read by both gradient products.
//
// dz of 16-bit operands is rounded to their 16 bits, the matrix cores' other
// operand being of those; its error is of the size of the gradients' own rounding
// to that type.  Against 64 bits both together are 1.0 to 1.24 times the latter
// where scores are spread, and 1.0 to 1.75 times where nearly every label
// dominates its row, whose dz is then two numbers that cancel (six sizes from 300
// x 64 x 100 to 100 x 200 x 60013, bf16 and fp16).  A second plane of dz would
// remove it and double the gradients' products, half of a call's time.
//
// All four products run on the matrix cores (tile.h).  fp32 operands are
// split into three bf16 planes, whose sum is exact, and six of the nine
// products of planes are added: what is left out is below fp32's own
// rounding.  Scores are laid out with the table along the accumulator's
// registers, so that a lane holds 64 scores of one row and its maximum and sum
// need a single exchange between lanes.
//
// What bounds it is the matrix cores where rows, columns and table are all
// long.  8192 rows, 100003 x 512 table, bf16, both gradients: 3.54 ms a call among
// others; traced one by one, 3.85 in all, the first scores take 934 us
// (900 TFLOP/s), the seven pieces' dz 160 us each (750) and their gradients 254
// (950).  4099 rows, 30011 x 256, f32: 1.49 ms; traced, 346 us (182 TFLOP/s), three
// pieces' dz 176 each (119; 36 bytes a lane spilled) and gradients 250 (168).
#include "train.h"

#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "device.h"
#include "tile.h"
#include "xent.h"

namespace aires {
namespace kern {
namespace {

constexpr int TV = 256;  // table entries of a tile of scores
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // dz of one piece of the table
constexpr int64_t kCopyBytes = int64_t(1) << 30;     // packed rows of the table
// dz in fp16, which is 1 at most, is held times this: as high as fp16 goes.  A
// probability keeps its 11 bits down to 2^-29 (times 2^10: to 2^-24, which a
// large gradient scale brings into an fp16 result's range).
constexpr float F16_UP = 32768.f;

// ---------------------------------------------------------------- operands

// Rows of X and Y at a stride of `width` columns, zeros past the end: 16-bit
// values as they are, fp32 as three planes of bf16 (tile.h).  The first
// `first` workgroups take X.
struct Pack {
  Mat X, Y;
  uint16_t *x, *y;
  int64_t width;
  unsigned first;
};

template <bool PLANES>
__global__ __launch_bounds__(256) void k_pack(Pack a) {
  const bool is_x = blockIdx.x < a.first;
  const Mat X = is_x ? a.X : a.Y;
  uint16_t* const to = is_x ? a.x : a.y;
  const int64_t width = a.width, per = width / 4, total = X.rows * per;
  const int64_t b = is_x ? blockIdx.x : blockIdx.x - a.first, step = is_x ? a.first : gridDim.x - a.first;
  for (int64_t i = b * 256 + threadIdx.x; i < total; i += step * 256) {
    const int64_t r = i / per, c = (i - r * per) * 4, at = r * X.ld + c;
    if constexpr (!PLANES) {
      const uint16_t* x = static_cast<const uint16_t*>(X.data);
      u16x4_el v = {0, 0, 0, 0};
      if (c + 4 <= X.cols) v = *reinterpret_cast<const u16x4_el*>(x + at);
      else
        for (int k = 0; k < 4; ++k)
          if (c + k < X.cols) v[k] = x[at + k];
      *reinterpret_cast<u16x4_el*>(to + r * width + c) = v;
    } else {
      float x[4];
      if (c + 4 <= X.cols) load4<DT_F32>(X.data, at, x);
      else
        for (int k = 0; k < 4; ++k) x[k] = c + k < X.cols ? load1<DT_F32>(X.data, at + k) : 0.f;
      uint16_t* out = to + r * width * 3 + c / 16 * 48 + c % 16;
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        u16x4_el v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = f32_to_bf16(x[k]);
          x[k] -= bf16_to_f32(v[k]);
        }
        *reinterpret_cast<u16x4_el*>(out + p * 16) = v;
      }
    }
  }
}

// ------------------------------------------------------------------ scores

// The loss, and what dz is multiplied with, from workgroups' losses and
// labelled rows in a fixed order, by one workgroup.
struct Total {
  const double2* sums; int64_t n;
  int mean; float grad_scale;
  float* scale; float* loss;
};

template <int THREADS>
__device__ __forceinline__ void total_loss(const Total& a) {
  __shared__ double2 buf[THREADS / 64];
  double2 v = {0, 0};
  for (int64_t i = threadIdx.x; i < a.n; i += THREADS) {
    v.x += a.sums[i].x;
    v.y += a.sums[i].y;
  }
  v = wave_sum2(v);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < THREADS / 64; ++i) {
      v.x += buf[i].x;
      v.y += buf[i].y;
    }
    const double div = a.mean && v.y > 0 ? v.y : 1.0;
    *a.scale = (float)(a.grad_scale / div);
    *a.loss = (float)(v.x / div);
  }
}

__global__ __launch_bounds__(256) void k_total(Total a) { total_loss<256>(a); }

struct Scores {
  Panel W, H;
  int64_t T, V, v0, v1;   // the piece [v0, v1) of the table
  int steps;
  float2* part;           // [tile][t]: maximum, sum
  float* target;          // labels' scores
  const float* top; const float* inv;  // of whole rows
  const void* labels; int i64;
  uint16_t* dz; int64_t ldz;  // of 16-bit elements
  uint32_t* ticket;       // cleared here for the workgroups of k_rows
  Total total;            // n > 0: made by a workgroup more, the first one
};

// TT rows of H a tile.  256: eight wavefronts of 128 x 64; 128: of 64 x 64;
// 32: four of 64 x 32, two workgroups a CU, for the few rows whose scores only
// cost the reading of the table (T = 1, 262144 x 512 bf16: 41 us against 71
// with 256 rows).
template <int TT, int TYPE>
using ScoreTile = std::conditional_t<TYPE == DT_F32, Tile3<TV, TT, TT == 32 ? 64 : 128, TT == 32 ? 32 : 64, TT == 256 ? 3 : 2, false, false>,
                                     Tile<TV, TT, TT == 256 ? 128 : 64, TT == 32 ? 32 : 64, false, false, TYPE == DT_F16>>;

constexpr int score_threads(int type, int TT) { return TT == 256 || (TT == 128 && type != DT_F32) ? 512 : 256; }

template <bool GRAD, int TYPE, int TT>
__global__ __launch_bounds__(score_threads(TYPE, TT), 2) void k_scores(Scores s) {
  constexpr bool F16 = TYPE == DT_F16;
  constexpr int PLANES = TYPE == DT_F32 ? 3 : 1;
  using T_ = ScoreTile<TT, TYPE>;
  constexpr int SPAN = T_::MT * 32, NWM = TV / SPAN;  // table entries of a wavefront, wavefronts along the table
  __shared__ __attribute__((aligned(16))) char lds[T_::LDS];
  if (GRAD && s.total.n > 0 && blockIdx.x == 0) return total_loss<T_::THREADS>(s.total);
  int64_t vt, tt;
  place_tile(blockIdx.x - (GRAD && s.total.n > 0 ? 1 : 0), (s.v1 - s.v0 + TV - 1) / TV, (s.T + TT - 1) / TT, 8, vt, tt);
  const int64_t v0 = s.v0 + vt * TV, t0 = tt * TT;
  f32x16 acc[T_::MT][T_::NT];
  // Labels, as they come: they are on their way during the products.
  uint32_t low[GRAD ? 1 : T_::NT], high[GRAD ? 1 : T_::NT];
  if constexpr (!GRAD) {
#pragma unroll
    for (int j = 0; j < T_::NT; ++j) {
      const int64_t t = t0 + T_::col(j), at = t < s.T ? t : s.T - 1;
      const uint32_t* const l = static_cast<const uint32_t*>(s.labels) + (s.i64 ? 2 * at : at);
      low[j] = l[0];
      high[j] = l[s.i64 ? 1 : 0];
    }
    // They stay before the stages' loads, which are waited for by their number.
    asm volatile("" ::: "memory");
  }
  T_::run(s.W, v0, s.H, t0, 0, s.steps, lds, acc);
  const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / (T_::WAVES / NWM);
  __syncthreads();  // the stages' LDS changes its use

  if constexpr (!GRAD) {
    if (v0 + TV > s.V) {
#pragma unroll
      for (int i = 0; i < T_::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (v0 + T_::row(i, r) >= s.V)
#pragma unroll
            for (int j = 0; j < T_::NT; ++j) acc[i][j][r] = -INFINITY;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *s.ticket = 0;
    float2* others = reinterpret_cast<float2*>(lds);  // of the wavefronts after the first along the table
#pragma unroll
    for (int j = 0; j < T_::NT; ++j) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < T_::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float from = top == -INFINITY ? 0.f : top;  // a NaN still reaches the sum
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < T_::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += exp_from(acc[i][j][r], from);
      sum += __shfl_xor(sum, 32);
      const int c = T_::col(j);
      // the label's score, where it is among this wavefront's, by the lane that has it
      const int64_t label = s.i64 && high[j] != 0 ? -1 : (int64_t)(int32_t)low[j];
      const int64_t first = v0 + wm * SPAN;
      const bool mine = label >= first && label < first + SPAN && label < s.V && ((label >> 2) & 1) == lane >> 5;
      if (__any(mine)) {
        const int at = mine ? (int)(label - v0) : -1;
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < T_::MT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) z = T_::row(i, r) == at ? acc[i][j][r] : z;
        if (mine && t0 + c < s.T) s.target[t0 + c] = z;
      }
      if (wm > 0 && lane < 32) others[(wm - 1) * TT + c] = make_float2(top, sum);
      acc[0][j][0] = top;
      acc[0][j][1] = sum;
    }
    __syncthreads();
    if (wm == 0 && lane < 32)
#pragma unroll
      for (int j = 0; j < T_::NT; ++j) {
        const int c = T_::col(j);
        float m = acc[0][j][0], x = acc[0][j][1];
#pragma unroll
        for (int w = 0; w < NWM - 1; ++w) join(m, x, others[w * TT + c].x, others[w * TT + c].y);
        if (t0 + c < s.T) s.part[vt * s.T + t0 + c] = make_float2(m, x);
      }
  } else {
#pragma unroll
    for (int j = 0; j < T_::NT; ++j) {
      const int64_t t = t0 + T_::col(j);
      const int64_t label = t < s.T ? label_at(s.labels, s.i64, t) : -1;
      const bool there = label >= 0 && label < s.V;
      const float top = there ? s.top[t] : 0.f, inv = there ? s.inv[t] * (F16 ? F16_UP : 1.f) : 0.f;
#pragma unroll
      for (int i = 0; i < T_::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = exp_from(acc[i][j][r], top) * inv;
          acc[i][j][r] = there ? p : 0.f;  // a score that is no number stays out of rows without a label
        }
      const int64_t first = v0 + wm * SPAN;
      if (__any(there && label >= first && label < first + SPAN)) {
        const int at = there && label >= first && label < first + SPAN ? (int)(label - v0) : -1;
#pragma unroll
        for (int i = 0; i < T_::MT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (T_::row(i, r) == at) acc[i][j][r] -= F16 ? F16_UP : 1.f;
      }
    }
    if (v0 + TV > s.v1) {
#pragma unroll
      for (int i = 0; i < T_::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (v0 + T_::row(i, r) >= s.v1)
#pragma unroll
            for (int j = 0; j < T_::NT; ++j) acc[i][j][r] = 0.f;
    }
    // Each wavefront through LDS of its own, 32 rows at a time, so that rows of
    // dz are written 256 bytes (three planes of 64 entries: 384) at a time.
    constexpr int IS = PLANES == 1 ? T_::MT : 2;  // tiles of 32 entries at once
    constexpr int ROW = IS * 64 * PLANES, CH = ROW / 16;
    static_assert(T_::WAVES * 32 * ROW <= T_::LDS && T_::MT % IS == 0, "dz is staged in the stages' LDS");
    char* mine = lds + (threadIdx.x >> 6) * (32 * ROW);
    const int c32 = lane & 31;
#pragma unroll
    for (int j = 0; j < T_::NT; ++j)
#pragma unroll
      for (int i0 = 0; i0 < T_::MT; i0 += IS) {
#pragma unroll
        for (int i = 0; i < IS; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = acc[i0 + i][j][q * 4 + k];
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
              u16x4_el v;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                v[k] = F16 ? f32_to_f16(x[k]) : f32_to_bf16(x[k]);
                if constexpr (PLANES > 1) x[k] -= bf16_to_f32(v[k]);
              }
              // 16 columns of a plane are two chunks
              const int ch = (2 * i + (q >> 1)) * (2 * PLANES) + 2 * p + (q & 1);
              *reinterpret_cast<uint64_t*>(mine + c32 * ROW + ((ch ^ (c32 & 7)) << 4) + (lane >> 5) * 8) =
                  __builtin_bit_cast(uint64_t, v);
            }
          }
        wave_sync();
        uint16_t* to = s.dz + (t0 + T_::col(j) - c32) * s.ldz + (v0 - s.v0 + wm * SPAN + i0 * 32) * PLANES;
        for (int it = lane; it < 32 * CH; it += 64) {
          const int r = it / CH, ch = it % CH;
          *reinterpret_cast<uint4*>(to + r * s.ldz + ch * 8) =
              *reinterpret_cast<const uint4*>(mine + r * ROW + ((ch ^ (r & 7)) << 4));
        }
        wave_sync();
      }
    // The products of 16-bit operands read 64 rows of dz a step: behind an odd
    // number of tiles of 32 the other half of the last step is zeros.
    if constexpr (PLANES == 1 && TT < BK)
      if (tt == (s.T - 1) / TT && (t0 + TT) % BK != 0)
        for (int it = threadIdx.x; it < (BK - TT) * (TV / 8); it += T_::THREADS)
          *reinterpret_cast<uint4*>(s.dz + (t0 + TT + it / (TV / 8)) * s.ldz + (v0 - s.v0) + it % (TV / 8) * 8) =
              make_uint4(0, 0, 0, 0);
  }
}

// ---------------------------------------------------------- rows and loss

struct Rows {
  int64_t T, V;
  const void* labels; int i64;
  const float2* part; int64_t tiles;
  const float* target;
  float* top; float* inv; float* row_loss;
  double2* sums;      // a workgroup's losses and labelled rows
  uint32_t* ticket;   // with it the last workgroup to finish adds up the loss
  Total total;
};

// Maximum and sum of each row from its tiles', and its loss: ROWS rows a
// workgroup, SLICES threads to a row's tiles.  With a ticket the last workgroup
// to finish adds up the loss.  7 us for one row's 1024 tiles, and for 8192 rows of
// 391.
template <int ROWS, int SLICES>
__global__ __launch_bounds__(ROWS * SLICES) void k_rows(Rows a) {
  static_assert(ROWS <= 64, "the rows' losses are one wavefront's");
  constexpr int THREADS = ROWS * SLICES;
  __shared__ float2 buf[SLICES][ROWS];
  __shared__ bool last;
  const int tid = threadIdx.x, r = tid % ROWS, slice = tid / ROWS;
  const int64_t T = a.T, t = (int64_t)blockIdx.x * ROWS + r;
  int64_t label = -1;
  float target = 0.f;  // (without a label: what the array happens to hold)
  if (slice == 0 && t < T) {
    label = label_at(a.labels, a.i64, t);
    target = a.target[t];
  }
  float m = -INFINITY, s = 0.f;
  if (t < T) {
#pragma unroll 8
    for (int64_t i = slice; i < a.tiles; i += SLICES) {
      const float2 p = a.part[i * T + t];
      join(m, s, p.x, p.y);
    }
  }
  buf[slice][r] = make_float2(m, s);
  __syncthreads();
  for (int o = SLICES / 2; o > 0; o >>= 1) {
    if (slice < o) {
      join(m, s, buf[slice + o][r].x, buf[slice + o][r].y);
      buf[slice][r] = make_float2(m, s);
    }
    __syncthreads();
  }
  if (tid < 64) {
    double2 mine = {0, 0};
    if (slice == 0 && t < T) {
      const bool there = label >= 0 && label < a.V;
      const float x = there ? loss_of(m, s, target) : 0.f;
      a.top[t] = m;
      a.inv[t] = 1.f / s;
      a.row_loss[t] = x;
      mine = {x, there ? 1.0 : 0.0};
    }
    mine = wave_sum2(mine);
    if (tid == 0) {
      a.sums[blockIdx.x] = mine;
      // the share is visible to whoever draws a later number
      last = (a.ticket && gridDim.x == 1) ||
             (a.ticket && __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1);
    }
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  total_loss<THREADS>(a.total);
}

// Rows of a workgroup: 8 with 128 threads each for few rows, 16 with 64 where
// a row has many tiles, 64 with 4 where it has few or the launch would be too
// large.
int rows_of(int64_t T, int64_t tiles) { return T <= 2048 ? 8 : tiles >= 32 && T <= (1 << 24) ? 16 : 64; }

}  // namespace

int64_t rows_and_loss_workspace(int64_t T) { return 16 * std::max<int64_t>(1, (T + 7) / 8); }

namespace {

// The rows; Total's n is 0 where the loss has been added up with them.
Total rows_of_all(const XentArgs& x, const float2* part, int64_t tiles, const float* target, float* top, float* inv,
                  float* row_loss, void* sums, uint32_t* ticket, float grad_scale, float* scale, hipStream_t s) {
  const int64_t T = x.H.rows;
  const int rows = rows_of(T, tiles);
  const unsigned blocks = (unsigned)std::max<int64_t>(1, (T + rows - 1) / rows);
  // A ticket costs 20 ns a workgroup, one after the other, another launch 5 us.
  const bool drawn = ticket && blocks <= 128;
  Total total{(double2*)sums, blocks, x.mean, grad_scale, scale, x.loss};
  const Rows rw{T, x.W.rows, x.labels, x.labels_i64, part, tiles, target, top, inv, row_loss, (double2*)sums,
                drawn ? ticket : nullptr, total};
  if (rows == 8) k_rows<8, 128><<<blocks, 1024, 0, s>>>(rw);
  else if (rows == 16) k_rows<16, 64><<<blocks, 1024, 0, s>>>(rw);
  else k_rows<64, 4><<<blocks, 256, 0, s>>>(rw);
  if (drawn) total.n = 0;
  return total;
}

}  // namespace

void rows_and_loss(const XentArgs& x, const float2* part, int64_t tiles, const float* target, float* top, float* inv,
                   float* row_loss, void* sums, uint32_t* ticket, float grad_scale, float* scale, hipStream_t s) {
  const Total total = rows_of_all(x, part, tiles, target, top, inv, row_loss, sums, ticket, grad_scale, scale, s);
  if (total.n > 0) k_total<<<1, 256, 0, s>>>(total);
}

namespace {

// --------------------------------------------------------------- gradients

// out(m, n) = scale sum_k A(m, k) B(n, k), in `slices` shares of k.
struct Product {
  Panel A, B;
  int64_t ny, nx, rows, cols;  // tiles, and what is there of the result
  int steps, per, slices;      // of BK; steps of a slice
  float* part; int64_t ldp;    // fp32 sums [slice][rows][ldp], or NULL:
  int add;                     //   added to what is there
  void* out; int64_t ldo;      // the result itself
  int type;
  int64_t blocks() const { return ny * nx * slices; }
};

struct Gradients {
  Product dh, dw;
  int64_t first_dw;  // workgroups before it make dH
  const float* scale;
};

template <class T_, int G>
__device__ __forceinline__ void product(const Product& p, int64_t b, const float* scale, char* lds) {
  int64_t y, x;
  place_tile(b, p.ny * p.slices, p.nx, 8, y, x);
  const int slice = (int)(y / p.ny);
  const int64_t m0 = (y - slice * p.ny) * G, n0 = x * G;
  const int s0 = slice * p.per, s1 = s0 + p.per < p.steps ? s0 + p.per : p.steps;
  f32x16 acc[T_::MT][T_::NT];
  T_::run(p.A, m0, p.B, n0, s0, s1, lds, acc);
  // Through LDS, 32 rows of the wavefront's part at a time, so that rows are
  // written 256 bytes (fp32) at a time.
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int W = T_::NT * 32;
  float* mine = reinterpret_cast<float*>(lds) + wave * (32 * W);
  const float k = p.part ? 1.f : *scale;
  float* part = p.part ? p.part + slice * p.rows * p.ldp : nullptr;
  const int64_t row0 = m0 + wave / (G / W) * (T_::MT * 32), n = n0 + wave % (G / W) * W + lane % (W / 4) * 4;
  __syncthreads();  // the stages' LDS changes its use
#pragma unroll
  for (int i = 0; i < T_::MT; ++i) {
#pragma unroll
    for (int j = 0; j < T_::NT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        mine[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * W + j * 32 + (lane & 31)] = acc[i][j][r];
    wave_sync();
    for (int r = lane / (W / 4); r < 32; r += 64 / (W / 4)) {
      const int64_t m = row0 + i * 32 + r;
      if (m >= p.rows || n >= p.cols) continue;
      const float4 v = *reinterpret_cast<const float4*>(mine + r * W + lane % (W / 4) * 4);
      float x[4] = {v.x * k, v.y * k, v.z * k, v.w * k};
      if (part) {
        float4* at = reinterpret_cast<float4*>(part + m * p.ldp + n);
        if (p.add) {
          const float4 o = *at;
          x[0] += o.x; x[1] += o.y; x[2] += o.z; x[3] += o.w;
        }
        *at = make_float4(x[0], x[1], x[2], x[3]);
      } else if (n + 4 <= p.cols) {
        if (p.type == DT_F32) store4<DT_F32>(p.out, m * p.ldo + n, x);
        else if (p.type == DT_BF16) store4<DT_BF16>(p.out, m * p.ldo + n, x);
        else store4<DT_F16>(p.out, m * p.ldo + n, x);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (n + c < p.cols) store1(p.out, p.type, m * p.ldo + n + c, x[c]);
      }
    }
    wave_sync();
  }
}

// G x G tiles: 256 by eight wavefronts of 128 x 64, or 128 by four of 64 x 64
// (two workgroups a CU).
template <int TYPE, int G, bool AK>
using GradientTile = std::conditional_t<TYPE == DT_F32, Tile3<G, G, G / 2, 64, 3, AK, true>,
                                        Tile<G, G, G / 2, 64, AK, true, TYPE == DT_F16>>;

template <int TYPE, int G>
__global__ __launch_bounds__(G == 256 ? 512 : 256, 2) void k_gradients(Gradients g) {
  using TH = GradientTile<TYPE, G, false>;
  using TW = GradientTile<TYPE, G, true>;
  __shared__ __attribute__((aligned(16))) char lds[TH::LDS];
  if ((int64_t)blockIdx.x < g.first_dw) product<TH, G>(g.dh, blockIdx.x, g.scale, lds);
  else product<TW, G>(g.dw, blockIdx.x - g.first_dw, g.scale, lds);
}

template <int TYPE>
void gradients(const Gradients& g, int G, hipStream_t s) {
  const unsigned grid = (unsigned)(g.first_dw + g.dw.blocks());
  if (G == 256) k_gradients<TYPE, 256><<<grid, 512, 0, s>>>(g);
  else k_gradients<TYPE, 128><<<grid, 256, 0, s>>>(g);
}

// out = scale times the sum of the slices; GROUPS threads to an element's
// slices (16 where there are many).
template <int GROUPS>
__device__ __forceinline__ void finish_part(const Finish& f, float k, int64_t b, int64_t blocks, float4* buf) {
  constexpr int ITEMS = 256 / GROUPS;
  const int64_t per = (f.cols + 3) / 4, total = f.rows * per;
  const int item = threadIdx.x % ITEMS, group = threadIdx.x / ITEMS;
  for (int64_t i0 = b * ITEMS; i0 < total; i0 += blocks * ITEMS) {
    const int64_t i = i0 + item, r = i / per, c = (i - r * per) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < total) {
#pragma unroll 4
      for (int s = group; s < f.slices; s += GROUPS) {
        const float4 v = *reinterpret_cast<const float4*>(f.part + (s * f.rows + r) * f.ldp + c);
        x.x += v.x; x.y += v.y; x.z += v.z; x.w += v.w;
      }
    }
    if constexpr (GROUPS > 1) {
      buf[threadIdx.x] = x;
      __syncthreads();
      if (group == 0)
        for (int q = 1; q < GROUPS; ++q) {
          const float4 v = buf[q * ITEMS + item];
          x.x += v.x; x.y += v.y; x.z += v.z; x.w += v.w;
        }
      __syncthreads();
    }
    if (group != 0 || i >= total) continue;
    const float o[4] = {x.x * k, x.y * k, x.z * k, x.w * k};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < f.cols) store1(f.out, f.type, r * f.ldo + c + j, o[j]);
  }
}

// The loss from workgroups' shares and labelled rows, in a fixed order.
__device__ __forceinline__ void sum_shares(const double2* sums, int n, int mean, float* loss, double2* buf) {
  double2 x = {0, 0};
  for (int i = threadIdx.x; i < n; i += 256) {
    x.x += sums[i].x;
    x.y += sums[i].y;
  }
  x = wave_sum2(x);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int i = 1; i < 4; ++i) {
    x.x += buf[i].x;
    x.y += buf[i].y;
  }
  *loss = (float)(mean && x.y > 0 ? x.x / x.y : x.x);
}

// Up to two gradients and the loss in one launch: workgroups of the first, of
// the second, and one.
struct FinishAll {
  Finish a, b;
  unsigned first, second;
  const float* scale;
  const double2* sums; int nsums, mean;
  float* loss;
};

__global__ __launch_bounds__(256) void k_finish(FinishAll f) {
  __shared__ float4 buf[256];
  if (blockIdx.x >= f.first + f.second) return sum_shares(f.sums, f.nsums, f.mean, f.loss, reinterpret_cast<double2*>(buf));
  const bool is_a = blockIdx.x < f.first;
  const Finish w = is_a ? f.a : f.b;
  const int64_t b = is_a ? blockIdx.x : blockIdx.x - f.first, blocks = is_a ? f.first : f.second;
  const float k = *f.scale;
  if (w.slices > 8) finish_part<16>(w, k, b, blocks, buf);
  else finish_part<1>(w, k, b, blocks, buf);
}

}  // namespace

void finish(const Finish& a, const Finish& b, const float* scale, const double2* sums, int nsums, int mean,
            float* loss, hipStream_t s) {
  auto blocks = [](const Finish& f) {
    const int64_t items = f.part ? f.rows * ((f.cols + 3) / 4) : 0, per = f.slices > 8 ? 16 : 256;
    return (unsigned)std::min<int64_t>(8192, (items + per - 1) / per);
  };
  const FinishAll f{a, b, blocks(a), blocks(b), scale, sums, nsums, mean, loss};
  const unsigned grid = f.first + f.second + (sums ? 1 : 0);
  if (grid) k_finish<<<grid, 256, 0, s>>>(f);
}

namespace {

__global__ __launch_bounds__(256) void k_zero(void* out, int type, int64_t rows, int64_t cols, int64_t ld) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256)
    store1(out, type, i / cols * ld + i % cols, 0.f);
}

// -------------------------------------------------------------------- host

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
unsigned grid_of(int64_t items, int64_t per) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(16384, (items + per - 1) / per));
}

// Sizes and places in the workspace.
struct Layout {
  int64_t width, planes, step;         // columns and planes of the packed operands, k of a step
  int64_t copy;                        // table entries that the workspace has room to pack
  int TT, G;                           // tiles
  int64_t piece, Tp, ldz;              // table entries of a piece, rows of dz and their stride
  int dh_per, dh_slices, dw_per, dw_slices;
  int64_t ticket, scale, target, top, inv, rows, sums, part, h, w, dh, dw, dz, bytes;
};

void slices_of(int steps, int64_t ideal, int& per, int& slices) {
  slices = (int)std::max<int64_t>(1, (steps + ideal / 2) / ideal);
  per = std::max(1, (steps + slices - 1) / slices);
  slices = std::max(1, (steps + per - 1) / per);
}

// Rows of a tile of scores: no more than there are, as many as still make a
// tile for every other CU (500 x 2000 scores, 64 columns, f32: the whole call 80
// us so, 102 in tiles of 256 rows), and not 256 where that leaves a seventh or more
// of them empty that 128 would not (loss of 258 x 124296 scores, 423 columns, f32:
// 329 us so, 360 with 256; 1100 x 60000, 512 columns, bf16, with gradients: 384 with
// 128, 370 with 256).
int score_rows(int64_t T, int64_t V) {
  for (int TT : {256, 128})
    if (T > TT / 2 && up(T, TT) / TT * (up(V, TV) / TV) >= 128 && 7 * up(T, 128) > 6 * up(T, TT)) return TT;
  return 32;
}

Layout layout_of(int64_t T, int64_t D, int64_t V, int type, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  l.planes = type == DT_F32 ? 3 : 1;
  l.step = type == DT_F32 ? 16 : BK;
  l.width = up(D, l.step);
  l.TT = score_rows(T, V);
  l.Tp = up(T, std::max<int64_t>(l.TT, l.step));
  l.ticket = take(4);
  l.scale = take(4);
  l.target = take(4 * T);
  l.top = take(4 * T);
  l.inv = take(4 * T);
  l.rows = take(4 * T);
  l.sums = take(rows_and_loss_workspace(T));
  l.part = take(8 * T * (up(V, TV) / TV));
  l.h = take(2 * l.planes * T * l.width);
  // A table whose copy would be larger than kCopyBytes is packed in pieces, once
  // for the first scores and again for dz: the workspace does not grow with it.
  const bool whole = 2 * l.planes * l.width * V <= kCopyBytes;
  l.copy = whole ? std::max<int64_t>(V, 1) : std::max<int64_t>(TV, kCopyBytes / (2 * l.planes * l.width) / TV * TV);
  if (grads) {
    const int64_t most = std::min(std::max<int64_t>(TV, kPieceBytes / (2 * l.planes * std::max<int64_t>(l.Tp, 1)) / TV * TV),
                                  up(l.copy, TV));
    const int64_t pieces = std::max<int64_t>(1, (V + most - 1) / most);
    l.piece = up((V + pieces - 1) / pieces, TV);  // (of one size: a small last one costs more than its share)
    if (!whole) l.copy = l.piece;
    const int dh_steps = (int)(up(std::min(l.piece, V), l.step) / l.step), dw_steps = (int)(up(T, l.step) / l.step);
    // Shares of k of about equal length, one workgroup a CU with large tiles,
    // two with small ones; none shorter than `least` steps.  Small tiles where
    // a side would leave half of a large one empty, or where large ones do not
    // make twice that share for every CU (300 x 130 x 3000 bf16: 54 us for the
    // call with large ones, 44 with small ones; 4099 x 256 x 30011 f32 1581 and
    // 1893).
    const int64_t least = l.planes == 1 ? 4 : 8;
    auto work = [&](int64_t G) {
      const int64_t nx = up(D, G) / G;
      return up(T, G) / G * nx * dh_steps + up(std::min(l.piece, V), G) / G * nx * dw_steps;
    };
    l.G = std::min({T, D, V}) <= 128 || work(256) < 256 * 2 * least ? 128 : 256;
    const int64_t ideal = std::max<int64_t>(least, work(l.G) / (l.G == 256 ? 256 : 512));
    slices_of(dh_steps, ideal, l.dh_per, l.dh_slices);
    slices_of(dw_steps, ideal, l.dw_per, l.dw_slices);
    if (l.dh_slices > 1 || l.piece < V) l.dh = take(4 * l.dh_slices * T * l.width);
    if (l.dw_slices > 1) l.dw = take(4 * l.dw_slices * l.piece * l.width);
    l.ldz = l.planes * l.piece + 64;
    l.dz = take(2 * l.Tp * l.ldz);
  }
  l.w = take(2 * l.planes * std::min(l.copy, V) * l.width);
  l.bytes = at;
  return l;
}

// Whether the tiles can read X as it lies.  Of the two operands of the scores
// one has to hold zeros up to the next multiple of BK columns: H (whole), which
// is the smaller one as a rule.
bool lies_well(const Mat& X, const Layout& l, bool whole) {
  return l.planes == 1 && X.cols % (whole ? l.step : 8) == 0 && X.ld % 8 == 0 && X.ld < (int64_t(1) << 22) &&
         (reinterpret_cast<uintptr_t>(X.data) & 15) == 0;
}

// Rows of X, and of Y where that has any, packed to x and y.
void pack(const Mat& X, const Mat& Y, const Layout& l, char* x, char* y, hipStream_t s) {
  Pack a{X, Y, (uint16_t*)x, (uint16_t*)y, l.width, 0};
  a.first = grid_of(X.rows * (l.width / 4), 1024);
  const unsigned grid = a.first + (Y.rows > 0 ? grid_of(Y.rows * (l.width / 4), 1024) : 0);
  if (l.planes == 1) k_pack<false><<<grid, 256, 0, s>>>(a);
  else k_pack<true><<<grid, 256, 0, s>>>(a);
}

// The operands as they lie, else packed into the workspace with zeros past
// their columns; a table that is packed in pieces is left to piece_of.
void panels_of(const Mat& H, const Mat& W, const Layout& l, char* ws, Panel& h, Panel& w, hipStream_t s) {
  const bool ph = !lies_well(H, l, true), pw = !lies_well(W, l, false) && l.copy >= W.rows;
  auto panel = [&](const Mat& X, bool packed, int64_t at) {
    return packed ? Panel{reinterpret_cast<uint16_t*>(ws + at), l.planes * l.width, X.rows, l.width}
                  : Panel{static_cast<const uint16_t*>(X.data), X.ld, X.rows, X.cols};
  };
  h = panel(H, ph, l.h);
  w = panel(W, pw, l.w);
  const Mat none{};
  if (ph && pw) pack(H, W, l, ws + l.h, ws + l.w, s);
  else if (ph) pack(H, none, l, ws + l.h, nullptr, s);
  else if (pw) pack(W, none, l, ws + l.w, nullptr, s);
}

// Packs entries [v0, v0 + n) of a table that is packed in pieces and points w at
// them by their numbers in the whole table.
void piece_of(const Mat& W, const Layout& l, char* ws, int64_t v0, int64_t n, Panel& w, hipStream_t s) {
  if (l.copy >= W.rows || lies_well(W, l, false)) return;
  Mat some = W;
  some.data = (char*)W.data + v0 * W.ld * dtype_bytes(W.type);
  some.rows = n;
  pack(some, Mat{}, l, ws + l.w, nullptr, s);
  w = Panel{reinterpret_cast<uint16_t*>(ws + l.w) - v0 * l.planes * l.width, l.planes * l.width, v0 + n, l.width};
}

template <bool GRAD, int TYPE>
void scores(const Scores& sc, int TT, hipStream_t s) {
  const unsigned grid = (unsigned)(up(sc.v1 - sc.v0, TV) / TV * (up(sc.T, TT) / TT)) + (sc.total.n > 0 ? 1 : 0);
  if (TT == 32) k_scores<GRAD, TYPE, 32><<<grid, 256, 0, s>>>(sc);
  else if (TT == 128) k_scores<GRAD, TYPE, 128><<<grid, score_threads(TYPE, 128), 0, s>>>(sc);
  else k_scores<GRAD, TYPE, 256><<<grid, 512, 0, s>>>(sc);
}

template <bool GRAD>
void scores(const Scores& sc, int type, int TT, hipStream_t s) {
  if (type == DT_F32) scores<GRAD, DT_F32>(sc, TT, s);
  else if (type == DT_BF16) scores<GRAD, DT_BF16>(sc, TT, s);
  else scores<GRAD, DT_F16>(sc, TT, s);
}

}  // namespace

int64_t linear_xent_workspace(int64_t T, int64_t D, int64_t V, int type, bool grads) {
  if (xent_few_fits(T, D, V)) return xent_few_workspace(T, D, V, grads);
  if (xent_rows_fits(T, D, V, type, grads)) return xent_rows_workspace(T, D, V, grads);
  return layout_of(T, D, V, type, grads).bytes;
}

hipError_t linear_xent(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dW.data != nullptr || x.dH.data != nullptr;
  const int type = x.H.type;
  const bool f16 = type == DT_F16;
  if (xent_few_fits(T, D, V)) return xent_few(x, s);
  if (xent_rows_fits(T, D, V, type, grads)) return xent_rows(x, s);
  const Layout l = layout_of(T, D, V, type, grads);
  char* ws = static_cast<char*>(x.ws);
  float* scale = (float*)(ws + l.scale);
  Scores sc{};
  if (T > 0) {
    panels_of(x.H, x.W, l, ws, sc.H, sc.W, s);
    sc.T = T; sc.V = V;
    sc.steps = (int)(l.width / l.step);
    sc.labels = x.labels; sc.i64 = x.labels_i64;
    sc.ticket = (uint32_t*)(ws + l.ticket);
    sc.target = (float*)(ws + l.target);
    // (a launch holds fewer than 2^32 threads)
    const int64_t most = std::min(std::max<int64_t>(1, (int64_t(1) << 22) / (up(T, l.TT) / l.TT)) * TV,
                                  lies_well(x.W, l, false) ? up(V, TV) : up(l.copy, TV));
    for (int64_t v0 = 0; v0 < V; v0 += most) {
      sc.v0 = v0; sc.v1 = std::min(V, v0 + most);
      piece_of(x.W, l, ws, v0, sc.v1 - v0, sc.W, s);
      sc.part = (float2*)(ws + l.part) + v0 / TV * T;
      scores<false>(sc, type, l.TT, s);
    }
  }
  float *top = (float*)(ws + l.top), *inv = (float*)(ws + l.inv);
  // fp16 dz is held times F16_UP
  const float gs = x.grad_scale * (f16 ? 1.f / F16_UP : 1.f);
  float* row_loss = x.row_loss ? x.row_loss : (float*)(ws + l.rows);
  const float2* part = (float2*)(ws + l.part);
  const float* target = (float*)(ws + l.target);
  const int64_t tiles = up(V, TV) / TV;
  if (grads && T > 0)  // dz does not need the loss: it is made next to it
    sc.total = rows_of_all(x, part, tiles, target, top, inv, row_loss, ws + l.sums, nullptr, gs, scale, s);
  else
    rows_and_loss(x, part, tiles, target, top, inv, row_loss, ws + l.sums, (uint32_t*)(ws + l.ticket), gs, scale, s);
  if (!grads) return hipGetLastError();
  if (T == 0) {
    if (V > 0 && D > 0) k_zero<<<grid_of(V * D, 1024), 256, 0, s>>>(x.dW.data, type, V, D, x.dW.ld);
    return hipGetLastError();
  }
  sc.top = top; sc.inv = inv;
  sc.dz = (uint16_t*)(ws + l.dz);
  sc.ldz = l.ldz;
  const Panel dz{sc.dz, l.ldz, l.Tp, l.piece};
  const int64_t nx = up(D, l.G) / l.G;
  const int size = dtype_bytes(type);
  for (int64_t v0 = 0; v0 < V; v0 += l.piece) {
    const int64_t n = std::min(l.piece, V - v0);
    sc.v0 = v0; sc.v1 = v0 + n;
    piece_of(x.W, l, ws, v0, n, sc.W, s);
    scores<true>(sc, type, l.TT, s);
    sc.total.n = 0;
    Gradients g{};
    g.scale = scale;
    Panel w = sc.W;
    w.data += v0 * w.ld;
    w.rows = n;
    g.dh = Product{dz, w, up(T, l.G) / l.G, nx, T, D, (int)(up(n, l.step) / l.step), l.dh_per, 0,
                   l.dh ? (float*)(ws + l.dh) : nullptr, l.width, v0 > 0, x.dH.data, x.dH.ld, type};
    g.dh.slices = (g.dh.steps + l.dh_per - 1) / l.dh_per;
    Mat out = x.dW;
    out.data = (char*)x.dW.data + v0 * x.dW.ld * size;
    g.dw = Product{dz, sc.H, up(n, l.G) / l.G, nx, n, D, (int)(up(T, l.step) / l.step), l.dw_per, l.dw_slices,
                   l.dw ? (float*)(ws + l.dw) : nullptr, l.width, 0, out.data, out.ld, type};
    g.first_dw = g.dh.blocks();
    if (type == DT_F32) gradients<DT_F32>(g, l.G, s);
    else if (type == DT_BF16) gradients<DT_BF16>(g, l.G, s);
    else gradients<DT_F16>(g, l.G, s);
    Finish dh{}, dw{};
    if (l.dw) dw = Finish{(float*)(ws + l.dw), l.dw_slices, n, D, l.width, out.data, type, out.ld};
    if (l.dh && v0 + n == V) dh = Finish{(float*)(ws + l.dh), l.dh_slices, T, D, l.width, x.dH.data, type, x.dH.ld};
    finish(dh, dw, scale, nullptr, 0, 0, nullptr, s);
  }
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
