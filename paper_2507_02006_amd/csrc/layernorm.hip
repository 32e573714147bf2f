// Layer norm over the rows of a dense matrix, forward and backward (gfx950).
//
// Forward: mu = sum x / n, r = (sum (x - mu)^2 / n + eps)^-1/2,
// y = (x - mu) r gamma + beta.  Backward: with xh = (x - mu) r and
// g = dy gamma, dx = r (g - mean(g) - xh mean(g xh)); dgamma = sum over rows
// of dy xh, dbeta = sum over rows of dy.  A handful of operations per value:
// bound by the bytes of X, Y, dY and dX, which are read and written once.
//
// A team of L lanes (or a workgroup, for wide rows) holds its row in
// registers, 4 E columns a lane, so both sums of the forward pass (the
// deviations are summed around the mean) and the three of the backward pass
// need one read.  Teams walk over rows, with gamma and beta in registers;
// in the backward pass each lane also sums dy xh and dy of its columns over
// its rows.  Those partial sums are joined per workgroup, written once and
// summed by a second launch in a fixed order.
//
// Measured: forward 262144 x 512, f32 -> bf16, 149 us (5.4 TB/s); backward with
// dgamma and dbeta, 1048576 x 256, dY bf16, X and dX f32, 473 us (5.7 TB/s);
// 4001 x 6001, f16, 57 us (2.5 TB/s: a 16-bit chunk is converted in the branch that
// guards its load, so each is waited for before the next is asked for, four a
// row here; and the wavefronts that share a row meet over its sums).  128 x 64
// takes 3 us, which is a launch.
#include "train.h"

#include <algorithm>

#include "dense.h"
#include "device.h"

namespace aires {
namespace kern {
namespace {

constexpr int TEAM_BLOCK = 256;    // threads of a workgroup of teams
constexpr int MAX_BLOCK = 1024;    // threads of a workgroup that shares a row
constexpr int MAX_E = 8;           // chunks of four columns a lane holds
// Widest rows held in registers: 1024 threads have 128 registers each, and the
// backward pass holds five rows' worth.  (The widest forward shape, E = 8 by a
// workgroup, keeps three of its 96 values in scratch memory.)
constexpr int64_t kForwardCols = (int64_t)MAX_BLOCK * MAX_E * 4;
constexpr int64_t kBackwardCols = (int64_t)MAX_BLOCK * 4 * 4;

struct Args {
  const void* x; int64_t ldx; int xt;
  const void* dy; int64_t lddy; int dyt;
  void* out; int64_t ldo; int ot;      // Y or dX (NULL: not wanted)
  const void* gamma; const void* beta; int wt;
  float* mean; float* rstd;            // written by the forward pass
  const float* cmean; const float* crstd;
  float* part;                         // backward: [workgroup][2][n], or NULL
  void* dgamma; void* dbeta;           // written directly by a single workgroup
  int64_t m; int n; float eps, inv_n;
};

// Sums of K values over a team, in every lane.  L = 0: over the workgroup,
// through `buf` (two halves used in turn, so one barrier a call is enough).
template <int L, int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float* buf, int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = group_sum_f32<L == 0 ? 64 : L>(v[k]);
  if constexpr (L == 0) {
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    float* b = buf + (turn & 1) * (2 * (MAX_BLOCK / 64));
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) b[wave * K + k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += b[w * K + k];
  }
}

// A lane's columns of one row: chunk e holds 4 columns from (e W + lane) 4.
template <int T, int E, bool ONCE>
__device__ __forceinline__ void load_row_t(const void* p, int64_t at, int n, int lane, int W, float (&x)[E][4]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = (e * W + lane) * 4;
    if (c + 4 <= n) {
      load4<T, ONCE>(p, at + c, x[e]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) x[e][k] = c + k < n ? load1<T>(p, at + c + k) : 0.f;
    }
  }
}

template <int E, bool ONCE = false>
__device__ __forceinline__ void load_row(const void* p, int t, int64_t at, int n, int lane, int W, float (&x)[E][4]) {
  if (t == DT_F32) load_row_t<DT_F32, E, ONCE>(p, at, n, lane, W, x);
  else if (t == DT_BF16) load_row_t<DT_BF16, E, ONCE>(p, at, n, lane, W, x);
  else load_row_t<DT_F16, E, ONCE>(p, at, n, lane, W, x);
}

template <int T, int E, bool ONCE>
__device__ __forceinline__ void store_row_t(void* p, int64_t at, int n, int lane, int W, const float (&x)[E][4]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = (e * W + lane) * 4;
    if (c + 4 <= n) {
      store4<T, ONCE>(p, at + c, x[e]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < n) store1<T>(p, at + c + k, x[e][k]);
    }
  }
}

template <int E, bool ONCE = false>
__device__ __forceinline__ void store_row(void* p, int t, int64_t at, int n, int lane, int W, const float (&x)[E][4]) {
  if (t == DT_F32) store_row_t<DT_F32, E, ONCE>(p, at, n, lane, W, x);
  else if (t == DT_BF16) store_row_t<DT_BF16, E, ONCE>(p, at, n, lane, W, x);
  else store_row_t<DT_F16, E, ONCE>(p, at, n, lane, W, x);
}

template <int E>
__device__ __forceinline__ void load_weight(const void* p, int t, float fill, int n, int lane, int W,
                                            float (&x)[E][4]) {
  if (p) {
    load_row<E>(p, t, 0, n, lane, W, x);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[e][k] = fill;
  }
}

template <int L>
struct Team {
  int lane, W;
  int64_t first, step;
  __device__ Team() {
    if constexpr (L == 0) {
      lane = threadIdx.x; W = blockDim.x; first = blockIdx.x; step = gridDim.x;
    } else {
      constexpr int teams = TEAM_BLOCK / L;
      lane = threadIdx.x % L; W = L;
      first = (int64_t)blockIdx.x * teams + threadIdx.x / L; step = (int64_t)gridDim.x * teams;
    }
  }
};

template <int L, int E, bool ONCE>
__global__ __launch_bounds__(L == 0 ? MAX_BLOCK : TEAM_BLOCK) void k_ln_forward(Args a) {
  __shared__ float buf[L == 0 ? 4 * (MAX_BLOCK / 64) : 1];
  const Team<L> tm;
  const int n = a.n;
  int turn = 0;
  float g[E][4], b[E][4];
  load_weight<E>(a.gamma, a.wt, 1.f, n, tm.lane, tm.W, g);
  load_weight<E>(a.beta, a.wt, 0.f, n, tm.lane, tm.W, b);
  for (int64_t row = tm.first; row < a.m; row += tm.step) {
    float x[E][4];
    load_row<E, ONCE>(a.x, a.xt, row * a.ldx, n, tm.lane, tm.W, x);
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[0] += x[e][k];
    team_sum<L>(s, buf, turn);
    const float mu = s[0] / (float)n;  // exact where the sum and the mean are
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (e * tm.W + tm.lane) * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[e][k] -= mu;
        s[0] += c + k < n ? x[e][k] * x[e][k] : 0.f;
      }
    }
    team_sum<L>(s, buf, turn);
    const float r = 1.f / sqrtf(s[0] * a.inv_n + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[e][k] = x[e][k] * r * g[e][k] + b[e][k];
    store_row<E, ONCE>(a.out, a.ot, row * a.ldo, n, tm.lane, tm.W, x);
    if (a.mean && tm.lane == 0) {
      a.mean[row] = mu;
      a.rstd[row] = r;
    }
  }
}

// Joins the lanes' column sums of a workgroup's teams and writes them: to the
// partial sums of this workgroup, or (one workgroup in the launch) to dst.
template <int L, int E>
__device__ __forceinline__ void join_columns(float (&acc)[E][4], int which, const Args& a, float* buf) {
  const int n = a.n;
  float* part = a.part ? a.part + ((int64_t)blockIdx.x * 2 + which) * n : nullptr;
  void* dst = which ? a.dbeta : a.dgamma;
  if (!dst) return;
  if constexpr (L == 0) {
    if (part) store_row_t<DT_F32, E, false>(part, 0, n, threadIdx.x, blockDim.x, acc);
    else store_row<E>(dst, a.wt, 0, n, threadIdx.x, blockDim.x, acc);
  } else {
    constexpr int cols = L * E * 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int o = L; o < 64; o <<= 1) acc[e][k] += __shfl_xor(acc[e][k], o);
        if (lane < L) buf[wave * cols + (e * L + lane) * 4 + k] = acc[e][k];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += TEAM_BLOCK) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < TEAM_BLOCK / 64; ++w) v += buf[w * cols + c];
      if (c < n) {
        if (part) part[c] = v;
        else store1(dst, a.wt, c, v);
      }
    }
    __syncthreads();
  }
}

template <int L, int E, bool ONCE>
__global__ __launch_bounds__(L == 0 ? MAX_BLOCK : TEAM_BLOCK) void k_ln_backward(Args a) {
  __shared__ float buf[L == 0 ? 4 * (MAX_BLOCK / 64) : (TEAM_BLOCK / 64) * L * E * 4];
  const Team<L> tm;
  const int n = a.n;
  int turn = 0;
  float g[E][4], sg[E][4] = {}, sb[E][4] = {};
  load_weight<E>(a.gamma, a.wt, 1.f, n, tm.lane, tm.W, g);
  for (int64_t row = tm.first; row < a.m; row += tm.step) {
    float x[E][4], dy[E][4];
    load_row<E>(a.x, a.xt, row * a.ldx, n, tm.lane, tm.W, x);
    load_row<E>(a.dy, a.dyt, row * a.lddy, n, tm.lane, tm.W, dy);
    const float mu = a.cmean[row], r = a.crstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (e * tm.W + tm.lane) * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // columns past the end hold x = dy = 0; their xh is not used
        x[e][k] = c + k < n ? (x[e][k] - mu) * r : 0.f;
        sg[e][k] += dy[e][k] * x[e][k];
        sb[e][k] += dy[e][k];
        dy[e][k] *= g[e][k];
        s[0] += dy[e][k];
        s[1] += dy[e][k] * x[e][k];
      }
    }
    if (!a.out) continue;
    team_sum<L>(s, buf, turn);
    const float m1 = s[0] * a.inv_n, m2 = s[1] * a.inv_n;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) dy[e][k] = r * (dy[e][k] - m1 - x[e][k] * m2);
    store_row<E, ONCE>(a.out, a.ot, row * a.ldo, n, tm.lane, tm.W, dy);
  }
  if (!a.dgamma && !a.dbeta) return;
  __syncthreads();  // buf changes its use
  join_columns<L, E>(sg, 0, a, buf);
  join_columns<L, E>(sb, 1, a, buf);
}

// Rows wider than a workgroup's registers are read again for each sum.
__global__ __launch_bounds__(MAX_BLOCK) void k_ln_forward_wide(Args a) {
  __shared__ float buf[4 * (MAX_BLOCK / 64)];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) s[0] += load1(a.x, a.xt, row * a.ldx + c);
    team_sum<0>(s, buf, turn);
    const float mu = s[0] / (float)a.n;
    s[0] = 0.f;
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) {
      const float d = load1(a.x, a.xt, row * a.ldx + c) - mu;
      s[0] += d * d;
    }
    team_sum<0>(s, buf, turn);
    const float r = 1.f / sqrtf(s[0] * a.inv_n + a.eps);
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) {
      const float d = load1(a.x, a.xt, row * a.ldx + c) - mu;
      store1(a.out, a.ot, row * a.ldo + c,
             d * r * (a.gamma ? load1(a.gamma, a.wt, c) : 1.f) + (a.beta ? load1(a.beta, a.wt, c) : 0.f));
    }
    if (a.mean && threadIdx.x == 0) {
      a.mean[row] = mu;
      a.rstd[row] = r;
    }
  }
}

__global__ __launch_bounds__(MAX_BLOCK) void k_ln_backward_wide(Args a) {
  __shared__ float buf[4 * (MAX_BLOCK / 64)];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    const float mu = a.cmean[row], r = a.crstd[row];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) {
      const float g = load1(a.dy, a.dyt, row * a.lddy + c) * (a.gamma ? load1(a.gamma, a.wt, c) : 1.f);
      s[0] += g;
      s[1] += g * ((load1(a.x, a.xt, row * a.ldx + c) - mu) * r);
    }
    team_sum<0>(s, buf, turn);
    const float m1 = s[0] * a.inv_n, m2 = s[1] * a.inv_n;
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) {
      const float g = load1(a.dy, a.dyt, row * a.lddy + c) * (a.gamma ? load1(a.gamma, a.wt, c) : 1.f);
      const float xh = (load1(a.x, a.xt, row * a.ldx + c) - mu) * r;
      store1(a.out, a.ot, row * a.ldo + c, r * (g - m1 - xh * m2));
    }
  }
}

// Column sums of wide rows: a thread owns a column, blockIdx.y a run of rows.
__global__ __launch_bounds__(TEAM_BLOCK) void k_ln_columns_wide(Args a) {
  const int64_t c = (int64_t)blockIdx.x * TEAM_BLOCK + threadIdx.x;
  if (c >= a.n) return;
  const int64_t per = (a.m + gridDim.y - 1) / gridDim.y;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < a.m ? r0 + per : a.m;
  float sg = 0.f, sb = 0.f;
  for (int64_t row = r0; row < r1; ++row) {
    const float dy = load1(a.dy, a.dyt, row * a.lddy + c);
    sg += dy * ((load1(a.x, a.xt, row * a.ldx + c) - a.cmean[row]) * a.crstd[row]);
    sb += dy;
  }
  a.part[((int64_t)blockIdx.y * 2) * a.n + c] = sg;
  a.part[((int64_t)blockIdx.y * 2 + 1) * a.n + c] = sb;
}

// dgamma and dbeta: the workgroups' partial sums, 32 shares of them side by
// side for 32 columns, added in a fixed order.  count = 0 writes zeros.  A launch
// holds fewer than 2^32 threads along a side, so more than kColumnBlocks groups of
// columns are gone through in turn.
constexpr int64_t kColumnBlocks = int64_t(1) << 20;

__global__ __launch_bounds__(1024) void k_ln_columns(const float* part, int64_t count, int n, void* dgamma,
                                                     void* dbeta, int wt) {
  __shared__ float buf[32][33];
  const int c = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int which = blockIdx.y;
  for (int64_t at = (int64_t)blockIdx.x * 32; at < n; at += (int64_t)gridDim.x * 32) {
    const int64_t col = at + c;
    float v = 0.f;
    if (col < n) {
#pragma unroll 8
      for (int64_t i = w; i < count; i += 32) v += part[(i * 2 + which) * n + col];
    }
    buf[w][c] = v;
    __syncthreads();
    if (w == 0 && col < n) {
      v = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) v += buf[i][c];
      void* dst = which ? dbeta : dgamma;
      if (dst) store1(dst, wt, col, v);
    }
    __syncthreads();
  }
}

// Statistics of rows without columns: those of a row of equal values, 0.
__global__ __launch_bounds__(TEAM_BLOCK) void k_ln_no_columns(float* mean, float* rstd, int64_t m, float eps) {
  for (int64_t i = (int64_t)blockIdx.x * TEAM_BLOCK + threadIdx.x; i < m; i += (int64_t)gridDim.x * TEAM_BLOCK) {
    mean[i] = 0.f;
    rstd[i] = 1.f / sqrtf(eps);
  }
}

// Lanes a row, chunks of four columns a lane, threads of a workgroup.
struct Shape {
  int L, E, threads;
};

Shape shape_of(int64_t n) {
  const int64_t chunks = (n + 3) / 4;
  if (chunks <= 8) return {8, 1, TEAM_BLOCK};
  if (chunks <= 16) return {16, 1, TEAM_BLOCK};
  if (chunks <= 32) return {16, 2, TEAM_BLOCK};
  if (chunks <= 64) return {32, 2, TEAM_BLOCK};
  if (chunks <= 128) return {64, 2, TEAM_BLOCK};
  if (chunks <= 256) return {64, 4, TEAM_BLOCK};
  if (chunks <= 512) return {64, 8, TEAM_BLOCK};
  const int E = chunks <= 2048 ? 2 : chunks <= 4096 ? 4 : 8;
  const int64_t lanes = (chunks + E - 1) / E;
  return {0, E, (int)((lanes + 63) / 64 * 64)};
}

#define LN_LAUNCH(kernel, L_, E_)                                              \
  do {                                                                         \
    if (once) kernel<L_, E_, true><<<g_, b_, 0, s>>>(a);                       \
    else kernel<L_, E_, false><<<g_, b_, 0, s>>>(a);                           \
  } while (0)
#define LN_DISPATCH(kernel, sh, grid, widest)                                  \
  do {                                                                         \
    const dim3 g_((unsigned)(grid)), b_((unsigned)(sh).threads);               \
    if ((sh).L == 8) LN_LAUNCH(kernel, 8, 1);                                  \
    else if ((sh).L == 16 && (sh).E == 1) LN_LAUNCH(kernel, 16, 1);            \
    else if ((sh).L == 16) LN_LAUNCH(kernel, 16, 2);                           \
    else if ((sh).L == 32) LN_LAUNCH(kernel, 32, 2);                           \
    else if ((sh).L == 64 && (sh).E == 2) LN_LAUNCH(kernel, 64, 2);            \
    else if ((sh).L == 64 && (sh).E == 4) LN_LAUNCH(kernel, 64, 4);            \
    else if ((sh).L == 64) LN_LAUNCH(kernel, 64, 8);                           \
    else if ((sh).E == 2) LN_LAUNCH(kernel, 0, 2);                             \
    else if ((sh).E == 4) LN_LAUNCH(kernel, 0, 4);                             \
    else widest;                                                               \
  } while (0)

// An array that the second-level caches (8 x 4 MB) cannot keep is read and
// written past them: forward, 262144 x 512 f32 -> bf16, 150 us against 162,
// backward, 4001 x 6001 f16, 57 against 61 with stores of dX alone (its loads
// past them cost that again).
bool too_large_to_keep(const Mat& m) { return m.rows * m.cols * dtype_bytes(m.type) > (int64_t(32) << 20); }

int64_t rows_at_once(const Shape& sh) { return sh.L == 0 ? 1 : TEAM_BLOCK / sh.L; }

// Workgroups of the backward pass: what fills the chip, but eight rows a team
// at least once there are many rows (each workgroup writes 2 n partial sums).
int64_t backward_groups(int64_t m, int64_t n) {
  if (n > kBackwardCols) return std::max<int64_t>(1, std::min<int64_t>(32, m / 8));
  const Shape sh = shape_of(n);
  const int64_t rows = rows_at_once(sh);
  const int64_t need = (m + rows - 1) / rows;
  const int64_t fill = sh.L == 0 ? 256 * std::max(1, 1536 / sh.threads) : 1024;
  return std::max<int64_t>(1, std::min({need, fill, std::max<int64_t>(256, need / 8)}));
}

}  // namespace

hipError_t layer_norm(const Mat& X, const void* gamma, const void* beta, int wt, float eps, const Mat& Y, float* mean,
                      float* rstd, hipStream_t s) {
  if (X.rows == 0 || (X.cols == 0 && !mean)) return hipSuccess;
  if (X.cols == 0) {
    k_ln_no_columns<<<(unsigned)std::min<int64_t>((X.rows + TEAM_BLOCK - 1) / TEAM_BLOCK, 1 << 16), TEAM_BLOCK, 0, s>>>(
        mean, rstd, X.rows, eps);
    return hipGetLastError();
  }
  Args a{};
  a.x = X.data; a.ldx = X.ld; a.xt = X.type;
  a.out = Y.data; a.ldo = Y.ld; a.ot = Y.type;
  a.gamma = gamma; a.beta = beta; a.wt = wt;
  a.mean = mean; a.rstd = rstd;
  a.m = X.rows; a.n = (int)X.cols; a.eps = eps; a.inv_n = (float)(1.0 / (double)X.cols);
  if (X.cols > kForwardCols) {
    k_ln_forward_wide<<<(unsigned)std::min<int64_t>(a.m, 1 << 20), MAX_BLOCK, 0, s>>>(a);
    return hipGetLastError();
  }
  const Shape sh = shape_of(X.cols);
  const int64_t rows = rows_at_once(sh);
  const int64_t grid = std::min<int64_t>((a.m + rows - 1) / rows, sh.L == 0 ? 256 * std::max(1, 2048 / sh.threads) : 2048);
  const bool once = too_large_to_keep(X);
  LN_DISPATCH(k_ln_forward, sh, grid, LN_LAUNCH(k_ln_forward, 0, 8));
  return hipGetLastError();
}

int64_t layer_norm_workspace(int64_t m, int64_t n) {
  if (m == 0 || n == 0) return 0;
  return backward_groups(m, n) * 2 * n * (int64_t)sizeof(float);
}

hipError_t layer_norm_backward(const Mat& dY, const Mat& X, const float* mean, const float* rstd, const void* gamma,
                               int wt, const Mat& dX, void* dgamma, void* dbeta, float* ws, hipStream_t s) {
  const bool weights = dgamma || dbeta;
  const int n = (int)X.cols;
  const dim3 cgrid((unsigned)std::min<int64_t>(((int64_t)n + 31) / 32, kColumnBlocks), 2);
  if (n == 0 || (X.rows == 0 && !weights)) return hipSuccess;
  if (X.rows == 0) {
    k_ln_columns<<<cgrid, 1024, 0, s>>>(nullptr, 0, n, dgamma, dbeta, wt);
    return hipGetLastError();
  }
  Args a{};
  a.x = X.data; a.ldx = X.ld; a.xt = X.type;
  a.dy = dY.data; a.lddy = dY.ld; a.dyt = dY.type;
  a.out = dX.data; a.ldo = dX.ld; a.ot = dX.type;
  a.gamma = gamma; a.wt = wt;
  a.cmean = mean; a.crstd = rstd;
  a.dgamma = dgamma; a.dbeta = dbeta;
  a.m = X.rows; a.n = n; a.inv_n = (float)(1.0 / (double)n);
  const int64_t groups = backward_groups(a.m, n);
  const bool wide = n > kBackwardCols;
  a.part = weights && (groups > 1 || wide) ? ws : nullptr;
  if (wide) {
    if (weights) k_ln_columns_wide<<<dim3((unsigned)((n + TEAM_BLOCK - 1) / TEAM_BLOCK), (unsigned)groups), TEAM_BLOCK, 0, s>>>(a);
    if (a.out) k_ln_backward_wide<<<(unsigned)std::min<int64_t>(a.m, 1 << 20), MAX_BLOCK, 0, s>>>(a);
  } else {
    const Shape sh = shape_of(n);
    const bool once = too_large_to_keep(X);
    LN_DISPATCH(k_ln_backward, sh, groups, (void)0);  // (kBackwardCols: E is 4 at most)
  }
  if (a.part) k_ln_columns<<<cgrid, 1024, 0, s>>>(a.part, groups, n, dgamma, dbeta, wt);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
