// Products of many streamed rows S with at most 64 kept rows K, and what the
// cross entropy does with them, in one pass over S (gfx950): S is H and K the
// table where there are few classes, S the table and K H where there are few
// rows.
//
// With a short side the products are small and what bounds the work is the
// bytes of S (and of its gradient), so each row is read once and everything
// that it is needed for happens while a workgroup holds it: scores z = S K^T,
// dz, dS = dz K and its share of dK = dz^T S.
//
// Every wavefront owns DT tiles of 16 columns: it alone reads them of S, with
// its columns of K in registers for the scores and for dS, and sums its columns
// of dK in the accumulators over all its rows.  The wavefronts meet only over
// the scores: each writes its share of the sum over columns to LDS, and reads
// dz there.  Rows go from global memory to registers (the scores' operand),
// from there through the wavefront's own LDS to the layout of dK's operand,
// while the next block's are on their way.  A workgroup's dK is written once,
// at the end; a second launch adds them up in a fixed order.
//
// Products run on the matrix cores, the scores of 16-bit rows in those bits (16
// x 16 x 16), everything else in fp32 (16 x 16 x 4): nothing is rounded on its
// way.  A lane's k within a step is free as long as
// both operands agree on it: k = 16 i + 4 (lane / 16) + j for step j of group i,
// so that a lane's four steps are one 16-byte read.  Strides that are 4 modulo
// 16 words keep both directions of reading free of bank conflicts.
//
// Measured, loss and both gradients, 150001 x 256, 41 classes: the call takes 140 us in f32
// (308 MB at 2.2 TB/s), of which the three products, of 48 classes as they are
// padded, keep the matrix cores busy for 71, and 106 us in bf16 (135 with scores
// in fp32).  The rest is waiting where the wavefronts meet over the scores.  The
// shapes with gradients and the most tiles keep part of them in scratch memory:
// that one in f32 104 bytes a lane, 32 rows by 1024 columns 568.
#pragma once
#include <type_traits>

#include "dense.h"
#include "device.h"
#include "xent.h"

namespace aires {
namespace kern {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// 16 columns of 16-bit rows, four a lane
template <int TYPE>
__device__ __forceinline__ f32x4 mfma16(s16x4 a, s16x4 b, f32x4 c) {
  if constexpr (TYPE == DT_BF16) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
}

// CLASSES: softmax along the kept rows, loss; TRAIN: and both gradients.
// STATS: maximum and sum of exponentials along the streamed rows; DZ: both
// gradients from those of the whole table.
enum FewMode : int { FEW_CLASSES, FEW_CLASSES_TRAIN, FEW_STATS, FEW_DZ };

struct Few {
  Mat S, K, dS;
  int D, NK, Dp;                    // columns, kept rows, columns up to a multiple of 16
  const void* labels; int i64;      // of H's rows
  float* scale;                     // what dz is multiplied with: written by CLASSES, read by DZ
  uint32_t* ticket;                 // cleared by STATS
  float* part;                      // [workgroup][NK][Dp]: shares of dK
  // CLASSES
  const int* counts; int ncounts;   // TRAIN: labelled rows; ncounts = 0: counted here
  int mean; float grad_scale;
  float* row_loss;
  double2* sums;                    // a workgroup's losses and labelled rows
  // STATS, DZ
  float2* stats;                    // [workgroup][NK]: maximum, sum
  float* target;                    // scores of the kept rows' labels: written by STATS
  const float* top; const float* inv;
};

// KT tiles of 16 kept rows, DT tiles of 16 columns to each of WAVES
// wavefronts, RT tiles of 16 streamed rows a block; TYPE: of S, K and dS.  Two
// wavefronts a SIMD: two workgroups of four a CU, whose meetings do not coincide, where their
// registers hold KT DT <= 12 tiles, else one of eight.
template <int KT, int DT, int WAVES, int RT, int MODE, int TYPE>
__global__ __launch_bounds__(WAVES * 64, 2) void k_few(Few a) {
  constexpr bool WIDE = TYPE == DT_F32;
  constexpr bool GRAD = MODE == FEW_CLASSES_TRAIN || MODE == FEW_DZ;
  constexpr bool CLASSES = MODE == FEW_CLASSES || MODE == FEW_CLASSES_TRAIN;
  constexpr int THREADS = WAVES * 64, TB = RT * 16, ZS = KT * 16 + 4, HS = DT * 16 + 4;
  __shared__ __attribute__((aligned(16))) float z[WAVES][TB][ZS];
  __shared__ __attribute__((aligned(16))) float dz[GRAD ? TB : 1][ZS];
  __shared__ __attribute__((aligned(16))) float hall[GRAD ? WAVES : 1][GRAD ? TB : 1][HS];
  __shared__ int totals[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, q = lane >> 4;
  const int p16 = tid & 15;                         // kept rows p16 + 16 k are this thread's between the products
  float(*const h)[HS] = hall[GRAD ? wave : 0];
  const int64_t N = a.S.rows;
  const int D = a.D, NK = a.NK;

  const int c0 = wave * DT * 16;

  // Rows n16 of each row tile, columns 4 q ... of each column tile, as they
  // come: converting them waits for them, so that is left to their use.  Rows
  // past the end repeat the last one, whose dz is not used again, columns the
  // last group of four, which meets zeros of K (so an infinity in it makes its
  // row's scores NaN: W has none, and a row of H with one has no finite loss); of
  // a group that D cuts the values past D are taken out at their use (in the last
  // rows they might lie past the array: read one by one there).
  using E = std::conditional_t<WIDE, float, uint16_t>;
  using Raw = std::conditional_t<WIDE, f32x4_el, u16x4_el>;
  Raw raw[RT][DT];
  constexpr int PASSES = TB * 16 / THREADS > 0 ? TB * 16 / THREADS : 1;
  int64_t lab[CLASSES ? PASSES : 1];                // of the rows that this thread takes between the products
  const int last = (D - 1) & ~3;
  auto fetch = [&](int64_t r0) {
    if constexpr (CLASSES)
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int64_t r = r0 + (tid >> 4) + p * (THREADS / 16);
        lab[p] = label_at(a.labels, a.i64, r < N ? r : N - 1);
      }
    auto each = [&](auto get) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int64_t r = r0 + rt * 16 + n16, row = (r < N ? r : N - 1) * a.S.ld;
#pragma unroll
        for (int d = 0; d < DT; ++d) raw[rt][d] = get(row, c0 + d * 16 + 4 * q);
      }
    };
    const E* const from = static_cast<const E*>(a.S.data);
    if (D % 4 == 0 || r0 + TB + 4 <= N)
      each([&](int64_t row, int c) { return *reinterpret_cast<const Raw*>(from + row + (c < last ? c : last)); });
    else
      each([&](int64_t row, int c) {
        Raw v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = from[row + (c + k < D ? c + k : D - 1)];
        return v;
      });
  };
  auto number = [](E x) {
    if constexpr (WIDE) return x;
    else if constexpr (TYPE == DT_BF16) return bf16_to_f32(x);
    else return f16_to_f32(x);
  };
  auto values = [&](Raw v) { return f32x4{number(v[0]), number(v[1]), number(v[2]), number(v[3])}; };

  // The first rows are asked for before anything else: the kept rows, and what
  // is known of them, come at the same time.
  const int64_t blocks = (N + TB - 1) / TB;
  int64_t b = blockIdx.x;
  if (b < blocks) fetch(b * TB);

  // this wavefront's columns of K, for the scores (row n16, columns 4 q ...)
  // and for dS (rows 16 i + 4 q + j, column n16)
  // (none of the loads conditional: they are in flight together)
  std::conditional_t<WIDE, float[4], s16x4> wn[KT][DT];  // (no vectors of f32: the products take single registers)
  float wk[GRAD ? DT : 1][KT][4];
  f32x4 acc[GRAD ? KT : 1][DT];
  auto keep = [&]() {
    auto at = [&](int v, int c) {
      const E x = static_cast<const E*>(a.K.data)[(int64_t)(v < NK ? v : NK - 1) * a.K.ld + (c < D ? c : D - 1)];
      return (v < NK) & (c < D) ? x : E(0);  // (&: a branch would take the load with it)
    };
#pragma unroll
    for (int v = 0; v < KT; ++v)
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          wn[v][d][j] = at(v * 16 + n16, c0 + d * 16 + 4 * q + j);
          if constexpr (GRAD) wk[d][v][j] = number(at(16 * v + 4 * q + j, c0 + d * 16 + n16));
        }
  };
  keep();
  if constexpr (GRAD)
#pragma unroll
    for (int v = 0; v < KT; ++v)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[v][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  // what this thread knows of its kept rows (H's, where those are kept)
  float top[KT], inv[KT];
  int64_t label[KT];
#pragma unroll
  for (int k = 0; k < KT; ++k) {
    const int t = p16 + 16 * k;
    top[k] = MODE == FEW_STATS ? -INFINITY : 0.f;
    inv[k] = 0.f;  // STATS: the sum
    label[k] = -1;
    if constexpr (!CLASSES)
      if (t < NK) {
        const int64_t l = label_at(a.labels, a.i64, t);
        if (l >= 0 && l < N) {
          label[k] = l;
          if constexpr (MODE == FEW_DZ) {
            top[k] = a.top[t];
            inv[k] = a.inv[t];
          }
        }
      }
  }

  float scale = 1.f;
  if constexpr (MODE == FEW_CLASSES_TRAIN) {
    int c = 0;
    if (a.ncounts == 0) {
      for (int64_t t = tid; t < N; t += THREADS) {
        const int64_t l = label_at(a.labels, a.i64, t);
        c += l >= 0 && l < NK;
      }
    } else if (wave == 0) {
      for (int i = lane; i < a.ncounts; i += 64) c += a.counts[i];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
    if (lane == 0) totals[wave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) c += totals[w];
    scale = (float)(a.grad_scale / (a.mean && c > 0 ? (double)c : 1.0));
    if (blockIdx.x == 0 && tid == 0) *a.scale = scale;
  }
  if constexpr (MODE == FEW_DZ) scale = *a.scale;
  if constexpr (MODE == FEW_STATS)
    if (blockIdx.x == 0 && tid == 0) *a.ticket = 0;  // for the workgroups that join the statistics

  double2 loss = {0, 0};
  for (; b < blocks; b += gridDim.x) {
    const int64_t r0 = b * TB;
    // Four wavefronts make their places in LDS anew each time: kept, they push
    // other values to scratch memory (150001 x 256, 41 classes, f32: 140 us, 149
    // with them kept; eight, whose registers spill either way, 412 and 376 with 60
    // rows, 500 columns).
    int here = tid;
    if constexpr (WAVES == 4) asm("" : "+v"(here));
    const int n16 = here & 15, q = (here >> 4) & 3, p16 = n16;
    // scores over this wavefront's columns
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x4 s[KT];
#pragma unroll
      for (int v = 0; v < KT; ++v) s[v] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if constexpr (WIDE) {
          f32x4 x = values(raw[rt][d]);
          if (D % 4 != 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = c0 + d * 16 + 4 * q + j < D ? x[j] : 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < KT; ++v) s[v] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], wn[v][d][j], s[v], 0, 0, 0);
          if constexpr (GRAD) *reinterpret_cast<f32x4*>(&h[rt * 16 + n16][d * 16 + 4 * q]) = x;
        } else {
          Raw x = raw[rt][d];
          if (D % 4 != 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = c0 + d * 16 + 4 * q + j < D ? x[j] : E(0);
#pragma unroll
          for (int v = 0; v < KT; ++v) s[v] = mfma16<TYPE>(__builtin_bit_cast(s16x4, x), wn[v][d], s[v]);
          if constexpr (GRAD) *reinterpret_cast<f32x4*>(&h[rt * 16 + n16][d * 16 + 4 * q]) = values(x);
        }
      }
#pragma unroll
      for (int v = 0; v < KT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[wave][rt * 16 + 4 * q + r][v * 16 + n16] = s[v][r];
    }
    int64_t now[CLASSES ? PASSES : 1];
    if constexpr (CLASSES)
#pragma unroll
      for (int p = 0; p < PASSES; ++p) now[p] = lab[p];
    if (b + gridDim.x < blocks) fetch((b + gridDim.x) * TB);
    __syncthreads();

    // 16 threads a row
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = (tid >> 4) + p * (THREADS / 16);
      if (TB * 16 < THREADS && r >= TB) break;
      const int64_t row = r0 + r;
      float y[KT];
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        y[k] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) y[k] += z[w][r][p16 + k * 16];
      }
      if constexpr (CLASSES) {  // softmax and loss
        const int64_t l = row < N ? now[p] : -1;
        const bool there = l >= 0 && l < NK;
        float big = -INFINITY, target = 0.f;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          const int v = p16 + k * 16;
          if (v == l) target = y[k];
          if (v >= NK) y[k] = -INFINITY;
          big = fmaxf(big, y[k]);
        }
        big = group16_max_f32(big);
        target = group_sum_f32<16>(target);
        const float from = big == -INFINITY ? 0.f : big;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          y[k] = exp_from(y[k], from);
          sum += y[k];
        }
        sum = group_sum_f32<16>(sum);
        if constexpr (GRAD) {
          const float one = 1.f / sum;
#pragma unroll
          for (int k = 0; k < KT; ++k) {
            const int v = p16 + k * 16;
            dz[r][v] = there && v < NK ? y[k] * one - (v == l ? 1.f : 0.f) : 0.f;
          }
        }
        if (p16 == 0 && row < N) {
          const float x = there ? loss_of(big, sum, target) : 0.f;
          a.row_loss[row] = x;
          loss.x += x;
          loss.y += there ? 1.0 : 0.0;
        }
      }
      if constexpr (MODE == FEW_STATS) {
        if (row < N)
#pragma unroll
          for (int k = 0; k < KT; ++k) {
            const float up = fmaxf(top[k], y[k]), from = up == -INFINITY ? 0.f : up;
            inv[k] = (top[k] == up ? inv[k] : inv[k] * exp_from(top[k], up)) + exp_from(y[k], from);
            top[k] = up;
            if (row == label[k]) a.target[p16 + k * 16] = y[k];
          }
      }
      if constexpr (MODE == FEW_DZ) {
#pragma unroll
        for (int k = 0; k < KT; ++k)
          dz[r][p16 + k * 16] = row < N && label[k] >= 0
                                    ? exp_from(y[k], top[k]) * inv[k] - (row == label[k] ? 1.f : 0.f)
                                    : 0.f;
      }
    }
    __syncthreads();

    if constexpr (GRAD) {
      // dS, 16 columns by 16 rows: four columns of a row a lane
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KT; ++i) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(&dz[rt * 16 + n16][16 * i + 4 * q]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(wk[d][i][j], y[j], o[d], 0, 0, 0);
        }
        const int64_t row = r0 + rt * 16 + n16;
        if (row < N) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const int c = c0 + d * 16 + 4 * q;
            const float y[4] = {o[d][0] * scale, o[d][1] * scale, o[d][2] * scale, o[d][3] * scale};
            const int64_t at = row * a.dS.ld + c;
            if (c + 4 <= D) {
              if constexpr (WIDE) store4<DT_F32>(a.dS.data, at, y);
              else if (a.dS.type == DT_BF16) store4<DT_BF16>(a.dS.data, at, y);
              else store4<DT_F16>(a.dS.data, at, y);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (c + k < D) store1(a.dS.data, a.dS.type, at + k, y[k]);
            }
          }
        }
      }
      // dK
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 16 * i + 4 * q + j;
          float y[KT];
#pragma unroll
          for (int v = 0; v < KT; ++v) y[v] = dz[k][v * 16 + n16];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const float g = h[k][d * 16 + n16];
#pragma unroll
            for (int v = 0; v < KT; ++v) acc[v][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[v], g, acc[v][d], 0, 0, 0);
          }
        }
    }
  }

  if constexpr (GRAD) {
    float* part = a.part + (int64_t)blockIdx.x * NK * a.Dp;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const int c = c0 + d * 16 + n16;
      if (c >= a.Dp) continue;
#pragma unroll
      for (int v = 0; v < KT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = v * 16 + 4 * q + r;
          if (row < NK) part[(int64_t)row * a.Dp + c] = acc[v][d][r];
        }
    }
  }

  if constexpr (MODE == FEW_STATS) {  // joined over the threads with the same kept rows
    __syncthreads();
    float2* const all = reinterpret_cast<float2*>(&z[0][0][0]);
    static_assert(sizeof(float2) * KT * THREADS <= sizeof(z), "statistics fit the scores' LDS");
#pragma unroll
    for (int k = 0; k < KT; ++k) all[k * THREADS + tid] = make_float2(top[k], inv[k]);
    __syncthreads();
    if (tid < KT * 16 && tid < NK) {
      const float2* mine = all + (tid >> 4) * THREADS + (tid & 15);
      float m = mine[0].x, s = mine[0].y;
      for (int i = 16; i < THREADS; i += 16) join(m, s, mine[i].x, mine[i].y);
      a.stats[(int64_t)blockIdx.x * NK + tid] = make_float2(m, s);
    }
  }

  if constexpr (CLASSES) {
    __shared__ double2 sums[WAVES];
    loss = wave_sum2(loss);
    if (lane == 0) sums[wave] = loss;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < WAVES; ++i) {
        loss.x += sums[i].x;
        loss.y += sums[i].y;
      }
      a.sums[blockIdx.x] = loss;
    }
  }
}

// Tiles of 16 columns a wavefront, wavefronts of a workgroup, row tiles of a
// block; DT = 0 where the shape does not fit.
struct FewShape {
  int KT, DT, waves, RT;
};

inline FewShape few_shape(int64_t D, int64_t NK) {
  if (D > 1024 || NK > 64) return {0, 0, 0, 0};
  const int KT = (int)((NK + 15) / 16), tiles = (int)((D + 15) / 16), DT4 = (tiles + 3) / 4, DT8 = (tiles + 7) / 8;
  // (three tiles take the kernels for four)
  const int four = DT4 == 3 ? 4 : DT4, eight = DT8 <= 2 ? 2 : DT8 <= 4 ? 4 : 8;
  if (four <= 4 && KT * four <= 12) return {KT, four, 4, 2};
  if (eight <= 4) return {KT, eight, 8, 2};
  return KT <= 2 ? FewShape{KT, 8, 8, 1} : FewShape{0, 0, 0, 0};
}

// Workgroups: two of four wavefronts a CU or one of eight, also where a pass
// without gradients would leave room for more (150001 x 256, 41 classes, bf16,
// loss alone: 40 us, 47 with twice as many).
inline int64_t few_groups(const FewShape& f, int64_t rows) {
  const int64_t blocks = (rows + f.RT * 16 - 1) / (f.RT * 16);
  const int64_t fill = 256 * (f.waves == 4 ? 2 : 1);
  return std::max<int64_t>(1, std::min<int64_t>(fill, blocks));
}

template <int KT, int MODE, int TYPE>
void few_launch(const FewShape& f, const Few& a, unsigned grid, hipStream_t s) {
  if (f.waves == 4) {
    if (f.DT == 1) k_few<KT, 1, 4, 2, MODE, TYPE><<<grid, 256, 0, s>>>(a);
    else if (f.DT == 2) k_few<KT, 2, 4, 2, MODE, TYPE><<<grid, 256, 0, s>>>(a);
    else if constexpr (KT <= 3) k_few<KT, 4, 4, 2, MODE, TYPE><<<grid, 256, 0, s>>>(a);
  } else {
    if constexpr (KT == 4)
      if (f.DT == 2) k_few<KT, 2, 8, 2, MODE, TYPE><<<grid, 512, 0, s>>>(a);  // (fewer tiles: four wavefronts)
    if (f.DT == 4) k_few<KT, 4, 8, 2, MODE, TYPE><<<grid, 512, 0, s>>>(a);
    else if constexpr (KT <= 2)
      if (f.DT == 8) k_few<KT, 8, 8, 1, MODE, TYPE><<<grid, 512, 0, s>>>(a);
  }
}

// (16-bit rows come kept by 32 at most, by 16 with gradients: xent_rows_fits)
template <int MODE>
void few_launch(const FewShape& f, const Few& a, unsigned grid, hipStream_t s) {
  auto of = [&](auto t) {
    constexpr int TYPE = decltype(t)::value;
    constexpr int MOST = TYPE == DT_F32 || MODE == FEW_CLASSES || MODE == FEW_CLASSES_TRAIN ? 4 : MODE == FEW_STATS ? 2 : 1;
    if (f.KT == 1) few_launch<1, MODE, TYPE>(f, a, grid, s);
    else if constexpr (MOST >= 2) {
      if (f.KT == 2) few_launch<2, MODE, TYPE>(f, a, grid, s);
      else if constexpr (MOST >= 4) {
        if (f.KT == 3) few_launch<3, MODE, TYPE>(f, a, grid, s);
        else few_launch<4, MODE, TYPE>(f, a, grid, s);
      }
    }
  };
  if (a.S.type == DT_F32) of(std::integral_constant<int, DT_F32>{});
  else if (a.S.type == DT_BF16) of(std::integral_constant<int, DT_BF16>{});
  else of(std::integral_constant<int, DT_F16>{});
}

}  // namespace
}  // namespace kern
}  // namespace aires
