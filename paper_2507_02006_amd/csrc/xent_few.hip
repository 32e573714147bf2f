// Softmax cross entropy against few classes (at most 64), loss and both
// gradients in one pass over the rows (gfx950).
//
// With few classes the products are small and what bounds the work is the
// bytes of H and dH, so each row is read once and everything that it is needed
// for happens while a workgroup holds it: scores z = H W^T, the row's softmax
// and loss, dH = dz W and its share of dW = dz^T H.
//
// Every wavefront owns DT tiles of 16 columns: it alone reads them of H, with
// its columns of W in registers for the scores and for dH, and sums its
// columns of dW in the accumulators over all its rows.  The wavefronts meet
// only over the scores: each writes its share of the sum over columns to LDS,
// and reads dz there.  Rows go from global memory to registers (the scores'
// operand), from there through the wavefront's own LDS to the layout of dW's
// operand, while the next block's are on their way.  A workgroup's dW is
// written once, at the end; a second launch adds them up in a fixed order.
//
// Products run in fp32 on the matrix cores (16 x 16 x 4) for every type: fp32
// rows are not rounded anywhere.  A lane's k within a step is free as long as
// both operands agree on it: k = 16 i + 4 (lane / 16) + j for step j of group i,
// so that a lane's four steps are one 16-byte read.  Strides that are 4 modulo
// 16 words keep both directions of reading free of bank conflicts.
#include "xent.h"

#include <algorithm>

#include "dense.h"
#include "device.h"

namespace aires {
namespace kern {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int ROWS = 32;            // of a block
constexpr int COUNT_BLOCK = 1024;   // labels a workgroup of k_count looks at, at least
constexpr int MAX_COUNTS = 256;

struct Few {
  Mat H, W, dH;
  const void* labels; int i64;
  const int* counts; int ncounts;
  int mean; float grad_scale;
  float* scale; float* loss; float* row_loss;
  double* sums; uint32_t* ticket;
  float* part;                      // [workgroup][V][Dp], NULL without gradients
  int D, V, Dp;
};

// Labelled rows among each workgroup's share.
__global__ __launch_bounds__(256) void k_count(const void* labels, int i64, int64_t T, int64_t V, int* counts,
                                               uint32_t* ticket) {
  __shared__ int buf[4];
  int n = 0;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < T; t += (int64_t)gridDim.x * 256) {
    const int64_t l = label_at(labels, i64, t);
    n += l >= 0 && l < V;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    counts[blockIdx.x] = buf[0] + buf[1] + buf[2] + buf[3];
    if (blockIdx.x == 0) *ticket = 0;
  }
}

// VT tiles of 16 classes, DT tiles of 16 columns to each of WAVES wavefronts.
// Two wavefronts a SIMD: two workgroups of four a CU, whose meetings do not
// coincide, where their registers hold VT DT <= 12 tiles, else one of eight.
template <int VT, int DT, int WAVES, bool GRAD>
__global__ __launch_bounds__(WAVES * 64, 2) void k_few(Few a) {
  constexpr int THREADS = WAVES * 64, TB = ROWS, RT = TB / 16, ZS = VT * 16 + 4, HS = DT * 16 + 4;
  __shared__ __attribute__((aligned(16))) float z[WAVES][TB][ZS];
  __shared__ __attribute__((aligned(16))) float dz[TB][ZS];
  __shared__ __attribute__((aligned(16))) float hall[GRAD ? WAVES : 1][TB][HS];
  __shared__ int total;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, q = lane >> 4;
  float(*const h)[HS] = hall[GRAD ? wave : 0];
  const int64_t T = a.H.rows;
  const int D = a.D, V = a.V;

  if (wave == 0) {
    int c = 0;
    for (int i = lane; i < a.ncounts; i += 64) c += a.counts[i];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
    if (lane == 0) total = c;
  }
  __syncthreads();
  const double div = a.mean ? (double)(total > 0 ? total : 1) : 1.0;
  const float scale = (float)(a.grad_scale / div);  // what dz is multiplied with
  if (blockIdx.x == 0 && tid == 0) *a.scale = scale;

  // this wavefront's columns of W, for the scores (class n16, columns 4 q ...)
  // and for dH (classes 16 i + 4 q + j, column n16)
  const int c0 = wave * DT * 16;
  auto w = [&](int v, int c) { return v < V && c < D ? load1(a.W.data, a.W.type, (int64_t)v * a.W.ld + c) : 0.f; };
  float wn[VT][DT][4], wk[GRAD ? DT : 1][VT][4];
  f32x4 acc[GRAD ? VT : 1][DT];
#pragma unroll
  for (int v = 0; v < VT; ++v)
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
      for (int j = 0; j < 4; ++j) wn[v][d][j] = w(v * 16 + n16, c0 + d * 16 + 4 * q + j);
      if constexpr (GRAD) {
#pragma unroll
        for (int j = 0; j < 4; ++j) wk[d][v][j] = w(16 * v + 4 * q + j, c0 + d * 16 + n16);
        acc[v][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }

  // rows n16 of each row tile, columns 4 q ... of each column tile
  float x[RT][DT][4];
  auto fetch = [&](int64_t t0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int64_t t = t0 + rt * 16 + n16;
        const int c = c0 + d * 16 + 4 * q;
        const int64_t at = t * a.H.ld + c;
        if (t < T && c + 4 <= D) {
          if (a.H.type == DT_F32) load4<DT_F32>(a.H.data, at, x[rt][d]);
          else if (a.H.type == DT_BF16) load4<DT_BF16>(a.H.data, at, x[rt][d]);
          else load4<DT_F16>(a.H.data, at, x[rt][d]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[rt][d][k] = t < T && c + k < D ? load1(a.H.data, a.H.type, at + k) : 0.f;
        }
      }
  };

  const int64_t blocks = (T + TB - 1) / TB;
  double loss = 0;
  int64_t b = blockIdx.x;
  if (b < blocks) fetch(b * TB);
  for (; b < blocks; b += gridDim.x) {
    const int64_t t0 = b * TB;
    // scores over this wavefront's columns
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x4 s[VT];
#pragma unroll
      for (int v = 0; v < VT; ++v) s[v] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int v = 0; v < VT; ++v)
            s[v] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[rt][d][j], wn[v][d][j], s[v], 0, 0, 0);
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[wave][rt * 16 + 4 * q + r][v * 16 + n16] = s[v][r];
      if constexpr (GRAD) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
          *reinterpret_cast<f32x4*>(&h[rt * 16 + n16][d * 16 + 4 * q]) =
              f32x4{x[rt][d][0], x[rt][d][1], x[rt][d][2], x[rt][d][3]};
      }
    }
    if (b + gridDim.x < blocks) fetch((b + gridDim.x) * TB);
    __syncthreads();

    // softmax and loss: 16 threads a row
#pragma unroll
    for (int r = tid >> 4; r < TB; r += THREADS / 16) {
      const int p = tid & 15;
      const int64_t t = t0 + r;
      const int64_t label = t < T ? label_at(a.labels, a.i64, t) : -1;
      const bool there = label >= 0 && label < V;
      float y[VT], top = -INFINITY, target = 0.f;
#pragma unroll
      for (int k = 0; k < VT; ++k) {
        const int v = p + k * 16;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += z[w][r][v];
        y[k] = v < V ? s : -INFINITY;
        top = fmaxf(top, y[k]);
        if (v == label) target = s;
      }
      top = group16_max_f32(top);
      target = group_sum_f32<16>(target);
      const float top2 = top * LOG2E, from = top2 == -INFINITY ? 0.f : top2;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < VT; ++k) {
        y[k] = exp2_fast(fmaf(y[k], LOG2E, -from));
        sum += y[k];
      }
      sum = group_sum_f32<16>(sum);
      if constexpr (GRAD) {
        const float inv = 1.f / sum;
#pragma unroll
        for (int k = 0; k < VT; ++k) {
          const int v = p + k * 16;
          dz[r][v] = there && v < V ? y[k] * inv - (v == label ? 1.f : 0.f) : 0.f;
        }
      }
      if (p == 0 && t < T) {
        const float l = there ? (top2 + log2f(sum)) * LN2 - target : 0.f;
        a.row_loss[t] = l;
        loss += l;
      }
    }
    __syncthreads();

    if constexpr (GRAD) {
      // dH, 16 columns by 16 rows: four columns of a row a lane
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(&dz[rt * 16 + n16][16 * i + 4 * q]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(wk[d][i][j], y[j], o[d], 0, 0, 0);
        }
        const int64_t t = t0 + rt * 16 + n16;
        if (t < T) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const int c = c0 + d * 16 + 4 * q;
            const float y[4] = {o[d][0] * scale, o[d][1] * scale, o[d][2] * scale, o[d][3] * scale};
            const int64_t at = t * a.dH.ld + c;
            if (c + 4 <= D) {
              if (a.dH.type == DT_F32) store4<DT_F32>(a.dH.data, at, y);
              else if (a.dH.type == DT_BF16) store4<DT_BF16>(a.dH.data, at, y);
              else store4<DT_F16>(a.dH.data, at, y);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (c + k < D) store1(a.dH.data, a.dH.type, at + k, y[k]);
            }
          }
        }
      }
      // dW
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 16 * i + 4 * q + j;
          float y[VT];
#pragma unroll
          for (int v = 0; v < VT; ++v) y[v] = dz[k][v * 16 + n16];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const float g = h[k][d * 16 + n16];
#pragma unroll
            for (int v = 0; v < VT; ++v) acc[v][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[v], g, acc[v][d], 0, 0, 0);
          }
        }
    }
  }

  if constexpr (GRAD) {
    float* part = a.part + (int64_t)blockIdx.x * V * a.Dp;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const int c = c0 + d * 16 + n16;
      if (c >= a.Dp) continue;
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = v * 16 + 4 * q + r;
          if (row < V) part[(int64_t)row * a.Dp + c] = acc[v][d][r];
        }
    }
  }

  // the workgroup's loss; the last workgroup adds them up in order
  __shared__ double sums[THREADS];
  __shared__ bool last;
  auto add_up = [&](double x) {
    sums[tid] = x;
    __syncthreads();
    for (int o = THREADS / 2; o > 0; o >>= 1) {
      if (tid < o) sums[tid] += sums[tid + o];
      __syncthreads();
    }
  };
  add_up(loss);
  if (tid == 0) {
    a.sums[blockIdx.x] = sums[0];
    last = gridDim.x == 1 ||
           __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  loss = 0;
  for (int i = tid; i < (int)gridDim.x; i += THREADS) loss += a.sums[i];
  add_up(loss);
  if (tid == 0) *a.loss = (float)(sums[0] / div);
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Tiles of 16 columns a wavefront and wavefronts of a workgroup.
struct Shape {
  int DT, waves;
};

Shape shape_of(int64_t D, int64_t V) {
  const int VT = (int)((V + 15) / 16), tiles = (int)((D + 15) / 16), DT = (tiles + 3) / 4;
  if (DT <= 4 && VT * DT <= 12) return {DT, 4};
  return {(tiles + 7) / 8, 8};
}

int64_t groups_of(int64_t T, int64_t D, int64_t V) {
  return std::max<int64_t>(1, std::min<int64_t>(shape_of(D, V).waves == 4 ? 512 : 256, (T + ROWS - 1) / ROWS));
}

struct Layout {
  int64_t counts, ticket, scale, rows, sums, part, bytes;
};

Layout layout_of(int64_t T, int64_t D, int64_t V, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  const int64_t g = groups_of(T, D, V);
  l.counts = take(4 * MAX_COUNTS);
  l.ticket = take(4);
  l.scale = take(4);
  l.rows = take(4 * T);
  l.sums = take(8 * g);
  if (grads) l.part = take(4 * g * V * up(D, 16));
  l.bytes = at;
  return l;
}

template <int VT, int DT, int WAVES>
void launch(const Few& f, unsigned grid, bool grads, hipStream_t s) {
  if (grads) k_few<VT, DT, WAVES, true><<<grid, WAVES * 64, 0, s>>>(f);
  else k_few<VT, DT, WAVES, false><<<grid, WAVES * 64, 0, s>>>(f);
}

template <int VT>
void launch(const Few& f, unsigned grid, bool grads, hipStream_t s) {
  const Shape sh = shape_of(f.D, f.V);
  if (sh.waves == 4) {
    if (sh.DT == 1) launch<VT, 1, 4>(f, grid, grads, s);
    else if (sh.DT == 2) launch<VT, 2, 4>(f, grid, grads, s);
    else if (sh.DT == 3) launch<VT, 3, 4>(f, grid, grads, s);
    else if constexpr (VT <= 3) launch<VT, 4, 4>(f, grid, grads, s);
  } else {
    if constexpr (VT == 4)
      if (sh.DT == 2) launch<VT, 2, 8>(f, grid, grads, s);  // (fewer classes: four wavefronts)
    if (sh.DT == 3) launch<VT, 3, 8>(f, grid, grads, s);
    else if (sh.DT == 4) launch<VT, 4, 8>(f, grid, grads, s);
  }
}

}  // namespace

bool xent_few_fits(int64_t T, int64_t D, int64_t V) { return T > 0 && V <= 64 && D <= 512; }

int64_t xent_few_workspace(int64_t T, int64_t D, int64_t V, bool grads) { return layout_of(T, D, V, grads).bytes; }

hipError_t xent_few(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dW.data != nullptr || x.dH.data != nullptr;
  const Layout l = layout_of(T, D, V, grads);
  char* ws = static_cast<char*>(x.ws);
  Few f{};
  f.H = x.H; f.W = x.W; f.dH = x.dH;
  f.labels = x.labels; f.i64 = x.labels_i64;
  f.counts = (const int*)(ws + l.counts);
  f.ncounts = (int)std::min<int64_t>(MAX_COUNTS, (T + COUNT_BLOCK - 1) / COUNT_BLOCK);
  f.mean = x.mean; f.grad_scale = x.grad_scale;
  f.scale = (float*)(ws + l.scale); f.loss = x.loss;
  f.row_loss = x.row_loss ? x.row_loss : (float*)(ws + l.rows);
  f.sums = (double*)(ws + l.sums); f.ticket = (uint32_t*)(ws + l.ticket);
  f.part = grads ? (float*)(ws + l.part) : nullptr;
  f.D = (int)D; f.V = (int)V; f.Dp = (int)up(D, 16);
  k_count<<<(unsigned)f.ncounts, 256, 0, s>>>(x.labels, x.labels_i64, T, V, (int*)(ws + l.counts), f.ticket);
  const unsigned grid = (unsigned)groups_of(T, D, V);
  const int VT = (f.V + 15) / 16;
  if (VT == 1) launch<1>(f, grid, grads, s);
  else if (VT == 2) launch<2>(f, grid, grads, s);
  else if (VT == 3) launch<3>(f, grid, grads, s);
  else launch<4>(f, grid, grads, s);
  if (grads) finish(f.part, (int)grid, V, D, f.Dp, f.scale, x.dW.data, x.dW.type, x.dW.ld, s);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
