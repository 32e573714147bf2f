// Softmax cross entropy of scores H W^T against labels, with both gradients,
// without storing the scores (gfx950).
//
// With z = H W^T, s_i = log sum_j exp(z_ij): row_loss_i = s_i - z_i,label and
// dz_ij = scale (exp(z_ij - s_i) - [j = label(i)]) for labelled rows, 0 for
// others; dH = dz W, dW = dz^T H.  Scores are computed twice: once for the
// maxima and sums of exponentials of each tile's rows, joined to s, and once
// more in pieces of the table for dz, which goes to the workspace for the
// two gradient products.
#include "train.h"

#include <algorithm>

#include "dense.h"

namespace aires {
namespace kern {
namespace {

constexpr int TILE = 64, KSTEP = 16, BLOCK = 256;
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // dz of one piece of the table

__device__ __forceinline__ int64_t label_at(const void* labels, int i64, int64_t i) {
  return i64 ? static_cast<const int64_t*>(labels)[i] : (int64_t)static_cast<const int32_t*>(labels)[i];
}

// acc[i][j] += sum_k A(m0 + 4 ty + i, k) B(n0 + 4 tx + j, k): element (r, k)
// of an operand is at data[r * row + k * step].
struct Operand {
  const void* data;
  int type;
  int64_t rows, row, step;
};

__device__ __forceinline__ void tile_product(const Operand& A, int64_t m0, const Operand& B, int64_t n0, int64_t K,
                                             float (&a)[KSTEP][TILE + 4], float (&b)[KSTEP][TILE + 4],
                                             float (&acc)[4][4]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  for (int64_t k0 = 0; k0 < K; k0 += KSTEP) {
    for (int e = threadIdx.x; e < KSTEP * TILE; e += BLOCK) {
      // neighbouring threads along the operand's contiguous direction
      const int ra = A.step == 1 ? e / KSTEP : e % TILE, ka = A.step == 1 ? e % KSTEP : e / TILE;
      a[ka][ra] = m0 + ra < A.rows && k0 + ka < K ? load1(A.data, A.type, (m0 + ra) * A.row + (k0 + ka) * A.step) : 0.f;
      const int rb = B.step == 1 ? e / KSTEP : e % TILE, kb = B.step == 1 ? e % KSTEP : e / TILE;
      b[kb][rb] = n0 + rb < B.rows && k0 + kb < K ? load1(B.data, B.type, (n0 + rb) * B.row + (k0 + kb) * B.step) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KSTEP; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += a[k][ty * 4 + i] * b[k][tx * 4 + j];
    __syncthreads();
  }
}

struct Scores {
  Operand H, W;
  int64_t D;
  const void* labels; int i64;
  float2* part;      // [tile of the table][t]: maximum, sum of exp(z - maximum)
  float* target;     // z of the row's label
  const float* lse;
  const float* count;
  float grad_scale;
  int64_t v0, v1;    // piece of the table
  float* dz; int64_t ldz;
};

// Tile of scores: statistics of its rows (GRAD false) or dz.
template <bool GRAD>
__global__ __launch_bounds__(BLOCK) void k_scores(Scores s) {
  __shared__ float a[KSTEP][TILE + 4], b[KSTEP][TILE + 4];
  const int64_t t0 = (int64_t)blockIdx.y * TILE, v0 = s.v0 + (int64_t)blockIdx.x * TILE;
  Operand W = s.W;
  W.rows = s.v1;
  float acc[4][4];
  tile_product(s.H, t0, W, v0, s.D, a, b, acc);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + ty * 4 + i;
    const bool row = t < s.H.rows;
    const int64_t label = row ? label_at(s.labels, s.i64, t) : -1;
    if constexpr (GRAD) {
      if (!row) continue;
      const bool there = label >= 0 && label < s.W.rows;
      const float scale = there ? s.grad_scale / s.count[0] : 0.f, lse = s.lse[t];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t v = v0 + tx * 4 + j;
        if (v < s.v1)
          s.dz[t * s.ldz + (v - s.v0)] = there ? scale * (expf(acc[i][j] - lse) - (v == label ? 1.f : 0.f)) : 0.f;
      }
    } else {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t v = v0 + tx * 4 + j;
        if (v < s.v1) top = fmaxf(top, acc[i][j]);
        if (v == label && v < s.v1) s.target[t] = acc[i][j];
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (v0 + tx * 4 + j < s.v1) sum += top == -INFINITY && acc[i][j] == top ? 0.f : expf(acc[i][j] - top);
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor(sum, o);
      if (row && tx == 0) s.part[(int64_t)blockIdx.x * s.H.rows + t] = make_float2(top, sum);
    }
  }
}

// s_i of each row from its tiles' statistics; row_loss.
__global__ __launch_bounds__(BLOCK) void k_rows(Scores s, int64_t tiles, float* lse, float* row_loss) {
  const int64_t t = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
  if (t >= s.H.rows) return;
  float top = -INFINITY, sum = 0.f;
  for (int64_t i = 0; i < tiles; ++i) {
    const float2 p = s.part[i * s.H.rows + t];
    const float up = fmaxf(top, p.x);
    // exp(-inf - -inf) is no number: a side without a score adds nothing
    sum = (top == -INFINITY ? 0.f * sum : sum * expf(top - up)) + (p.x == -INFINITY ? p.y : p.y * expf(p.x - up));
    top = up;
  }
  const float l = top + logf(sum);
  lse[t] = l;
  const int64_t label = label_at(s.labels, s.i64, t);
  row_loss[t] = label >= 0 && label < s.W.rows ? l - s.target[t] : 0.f;
}

// loss and the divisor c, by one workgroup in a fixed order.
__global__ __launch_bounds__(1024) void k_loss(const void* labels, int i64, int64_t T, int64_t V, int mean,
                                               const float* row_loss, float* count, float* loss) {
  __shared__ double sums[1024];
  __shared__ int64_t counts[1024];
  double x = 0;
  int64_t n = 0;
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    const int64_t l = label_at(labels, i64, t);
    if (l >= 0 && l < V) {
      ++n;
      x += row_loss[t];
    }
  }
  sums[threadIdx.x] = x;
  counts[threadIdx.x] = n;
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) {
      sums[threadIdx.x] += sums[threadIdx.x + o];
      counts[threadIdx.x] += counts[threadIdx.x + o];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double c = mean ? (double)(counts[0] > 0 ? counts[0] : 1) : 1.0;
    *count = (float)c;
    *loss = (float)(sums[0] / c);
  }
}

// out (+)= A B^T; the first piece overwrites, the last rounds to `type`.
__global__ __launch_bounds__(BLOCK) void k_product(Operand A, Operand B, int64_t K, float* sum, int add, void* out,
                                                   int type, int64_t ldo) {
  __shared__ float a[KSTEP][TILE + 4], b[KSTEP][TILE + 4];
  const int64_t m0 = (int64_t)blockIdx.y * TILE, n0 = (int64_t)blockIdx.x * TILE;
  float acc[4][4];
  tile_product(A, m0, B, n0, K, a, b, acc);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= A.rows || n >= B.rows) continue;
      float x = acc[i][j];
      if (add) x += sum[m * B.rows + n];
      if (out) store1(out, type, m * ldo + n, x);
      else sum[m * B.rows + n] = x;
    }
}

__global__ void k_zero(void* out, int type, int64_t rows, int64_t cols, int64_t ld) {
  for (int64_t i = (int64_t)blockIdx.x * BLOCK + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * BLOCK)
    store1(out, type, i / cols * ld + i % cols, 0.f);
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
unsigned tiles_of(int64_t n) { return (unsigned)((n + TILE - 1) / TILE); }

struct Layout {
  int64_t count, lse, target, rows, part, dh, dz, bytes, piece;
};

Layout layout_of(int64_t T, int64_t D, int64_t V, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  l.count = take(4);
  l.lse = take(4 * T);
  l.target = take(4 * T);
  l.rows = take(4 * T);
  l.part = take(8 * T * tiles_of(V));
  if (grads) {
    l.piece = std::min(up(V, TILE), std::max<int64_t>(TILE, kPieceBytes / 4 / std::max<int64_t>(T, 1) / TILE * TILE));
    l.dh = take(4 * T * D);
    l.dz = take(4 * T * l.piece);
  }
  l.bytes = at;
  return l;
}

}  // namespace

int64_t linear_xent_workspace(int64_t T, int64_t D, int64_t V, int, bool grads) {
  return layout_of(T, D, V, grads).bytes;
}

hipError_t linear_xent(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dH.data || x.dW.data;
  const Layout l = layout_of(T, D, V, grads);
  char* ws = static_cast<char*>(x.ws);
  float* count = (float*)(ws + l.count);
  float* row_loss = x.row_loss ? x.row_loss : (float*)(ws + l.rows);
  if (T > 0) {
    Scores sc{};
    sc.H = Operand{x.H.data, x.H.type, T, x.H.ld, 1};
    sc.W = Operand{x.W.data, x.W.type, V, x.W.ld, 1};
    sc.D = D;
    sc.labels = x.labels; sc.i64 = x.labels_i64;
    sc.part = (float2*)(ws + l.part);
    sc.target = (float*)(ws + l.target);
    sc.v0 = 0; sc.v1 = V;
    k_scores<false><<<dim3(tiles_of(V), tiles_of(T)), BLOCK, 0, s>>>(sc);
    float* lse = (float*)(ws + l.lse);
    k_rows<<<(unsigned)((T + BLOCK - 1) / BLOCK), BLOCK, 0, s>>>(sc, tiles_of(V), lse, row_loss);
    sc.lse = lse;
    sc.count = count;
    sc.grad_scale = x.grad_scale;
    k_loss<<<1, 1024, 0, s>>>(x.labels, x.labels_i64, T, V, x.mean, row_loss, count, x.loss);
    if (grads) {
      sc.dz = (float*)(ws + l.dz);
      float* dh = (float*)(ws + l.dh);
      for (int64_t v0 = 0; v0 < V; v0 += l.piece) {
        const int64_t n = std::min(l.piece, V - v0);
        sc.v0 = v0; sc.v1 = v0 + n; sc.ldz = n;
        k_scores<true><<<dim3(tiles_of(n), tiles_of(T)), BLOCK, 0, s>>>(sc);
        const int size = dtype_bytes(x.W.type);
        const bool last = v0 + n == V;
        k_product<<<dim3(tiles_of(D), tiles_of(T)), BLOCK, 0, s>>>(
            Operand{sc.dz, DT_F32, T, n, 1},
            Operand{(const char*)x.W.data + v0 * x.W.ld * size, x.W.type, D, 1, x.W.ld}, n, dh, v0 > 0,
            last ? x.dH.data : nullptr, x.dH.type, x.dH.ld);
        k_product<<<dim3(tiles_of(D), tiles_of(n)), BLOCK, 0, s>>>(
            Operand{sc.dz, DT_F32, n, 1, n}, Operand{x.H.data, x.H.type, D, 1, x.H.ld}, T, nullptr, 0,
            (char*)x.dW.data + v0 * x.dW.ld * size, x.dW.type, x.dW.ld);
      }
    }
  } else {
    k_loss<<<1, 1024, 0, s>>>(nullptr, 0, 0, V, x.mean, nullptr, count, x.loss);
    if (grads && V > 0 && D > 0)
      k_zero<<<(unsigned)std::min<int64_t>(4096, (V * D + BLOCK - 1) / BLOCK), BLOCK, 0, s>>>(x.dW.data, x.dW.type, V, D, x.dW.ld);
  }
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
