// Root-mean-square norm of rows with a residual stream's addition, forward (in
// a float type or in 8 bits) and backward (gfx950).
//
// Forward: s = x + r as it is stored, q = (sum s^2 / n + eps)^-1/2,
// y = s q gamma.  Backward: with sh = s q and g = dy gamma,
// dx = q (g - sh mean(g sh)) + ds; dgamma = sum over rows of dy sh.  A handful
// of operations per value: bound by the bytes of the arrays, each read and
// written once.
//
// A team of L lanes (a workgroup for wide rows) holds its row in registers,
// 8 E columns a lane, and walks over rows with gamma in registers too.  16 lanes
// hold the 128 columns that share a scale in 8 bits, so a block's maximum is four
// lane exchanges.  In the backward pass each lane also sums dy sh of its columns
// over its rows; these partial sums are joined per workgroup, written once and
// summed by a second launch in a fixed order.
//
// Sums, statistics and the products between them are fp32.  What is rounded to fewer bits:
// S and Y to the types asked for, once each; Y in 8 bits from fp32.
//
// Measured: 262144 x 512 with a residual, bf16, Y in 8 bits 168 us (5.6 TB/s); backward
// pass of 4001 x 6001, fp16, 47 us (4.1 TB/s) and 5 for its second launch; one row of 512
// 2.4 us.
#include "layers.h"

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "rows8.h"

namespace aires {
namespace kern {
namespace {

constexpr int TEAM_BLOCK = 256;    // threads of a workgroup of teams
constexpr int MAX_BLOCK = 1024;    // threads of a workgroup that shares a row
// Two kinds of those (L = 0 and 1 where a team has L lanes): up to 512 threads have
// 256 registers each, 1024 have 128.
constexpr int group_threads(int L) { return L == 1 ? MAX_BLOCK / 2 : MAX_BLOCK; }
// Widest rows held in registers (1024 threads have 128 registers each).
constexpr int64_t kRegisterCols = (int64_t)MAX_BLOCK * 2 * 8;

struct Args {
  const void* x; int64_t ldx; int xt;     // X; backward: the normalised rows S
  const void* r; int64_t ldr; int rt;     // residual; backward: dS
  const void* dy; int64_t lddy; int dyt;
  void* s; int64_t lds; int st;
  void* out; int64_t ldo; int ot;         // Y or dX
  uint8_t* codes; int64_t ldc;            // Y in 8 bits
  float* scales; int64_t ldsc;
  const void* gamma; int wt;
  float* rstd; const float* crstd;
  float* part; void* dgamma;
  int64_t m; int n; float eps, inv_n;
};

// Sum over a team, in every lane.  L < 8: over the workgroup, through `buf` (two
// halves used in turn, so one barrier a call is enough).
template <int L>
__device__ __forceinline__ float team_sum(float v, float* buf, int& turn) {
  v = group_sum_f32<L < 8 ? 64 : L>(v);
  if constexpr (L < 8) {
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    float* b = buf + (turn & 1) * (MAX_BLOCK / 64);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) b[wave] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < waves; ++w) v += b[w];
  }
  return v;
}

template <int L>
struct Team {
  int lane, W;
  int64_t first, step;
  __device__ Team() {
    if constexpr (L < 8) {
      lane = threadIdx.x; W = blockDim.x; first = blockIdx.x; step = gridDim.x;
    } else {
      constexpr int teams = TEAM_BLOCK / L;
      lane = threadIdx.x % L; W = L;
      first = (int64_t)blockIdx.x * teams + threadIdx.x / L; step = (int64_t)gridDim.x * teams;
    }
  }
  // first column of chunk e
  __device__ int col(int e) const { return (e * W + lane) * 8; }
};

template <int T, int E, typename M, typename R>
__device__ __forceinline__ void load_row(const void* p, int t, int64_t at, int n, const M& tm, R (&x)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) load_raw<T != MIXED>(p, type_of<T>(t), at + tm.col(e), n - tm.col(e), row_of<T>(n), x[e]);
}

// A lane's eight columns of a row in fp32 (zeros past the last).
template <typename R>
__device__ __forceinline__ void values_of(R& r, int t, int have, int n, float (&x)[8]) {
  settle(r, t, have, n);
  convert(r, t, x);
}

template <int E, typename T>
__device__ __forceinline__ void load_gamma(const Args& a, const T& tm, float (&g)[E][8]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (a.gamma) {
      Raw8 r;
      load_raw(a.gamma, a.wt, tm.col(e), a.n - tm.col(e), a.n, r);
      values_of(r, a.wt, a.n - tm.col(e), a.n, g[e]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) g[e][k] = 1.f;
    }
  }
}

// Columns [c, c + 8) of y in 8 bits; every lane of a group of 16 takes part.
__device__ __forceinline__ void store_codes(const Args& a, int64_t row, int c, const float (&y)[8]) {
  float big = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) big = fmaxf(big, c + k < a.n ? finite_abs(y[k]) : 0.f);
  float scale, inv;
  block_scale(group16_max_f32(big), scale, inv);
  if (c >= a.n) return;
  if (c % BLOCK8 == 0) a.scales[row * a.ldsc + c / BLOCK8] = scale;
  u32x2_el1 w;
  w[0] = encode4(scaled(y[0], inv), scaled(y[1], inv), scaled(y[2], inv), scaled(y[3], inv));
  w[1] = encode4(scaled(y[4], inv), scaled(y[5], inv), scaled(y[6], inv), scaled(y[7], inv));
  uint8_t* to = a.codes + row * a.ldc + c;
  if (c + 8 <= a.n) {
    *reinterpret_cast<u32x2_el1*>(to) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (c + k < a.n) to[k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
  }
}

// T: the type of X, R, S and Y (or MIXED).  The next row is asked for before this one
// is used.
template <int L, int E, int T, bool RESIDUAL, bool CODES>
__global__ __launch_bounds__(L < 8 ? group_threads(L) : TEAM_BLOCK) void k_rms_forward(Args a) {
  __shared__ float buf[L < 8 ? 2 * (MAX_BLOCK / 64) : 1];
  const Team<L> tm;
  const int n = a.n, n8 = row_of<T>(n);
  const bool residual = T == MIXED ? a.r != nullptr : RESIDUAL, codes = T == MIXED ? a.codes != nullptr : CODES;
  int turn = 0;
  float g[E][8];
  Raw<T> xr[E], rr[E];
  const auto load = [&](int64_t row) {  // (past the last row: the last again)
    row = row < a.m ? row : a.m - 1;
    load_row<T>(a.x, a.xt, row * a.ldx, n, tm, xr);
    if (residual) load_row<T>(a.r, a.rt, row * a.ldr, n, tm, rr);
  };
  load(tm.first);
  load_gamma<E>(a, tm, g);
  for (int64_t row = tm.first; row < a.m; row += tm.step) {
    float x[E][8], sum[L == 64 ? E : 1] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int have = n - tm.col(e);
      values_of(xr[e], type_of<T>(a.xt), have, n8, x[e]);
      if (residual) {
        float r[8];
        values_of(rr[e], type_of<T>(a.rt), have, n8, r);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[e][k] += r[k];
      }
    }
    if constexpr (T != MIXED) load(row + tm.step);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (residual) {
        Raw<T> p;
        pack(x[e], type_of<T>(a.st), p);
        store_raw<T != MIXED>(a.s, type_of<T>(a.st), row * a.lds + tm.col(e), n - tm.col(e), p);
        convert(p, type_of<T>(a.st), x[e]);  // the norm is that of what is stored
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[L == 64 ? e : 0] += x[e][k] * x[e][k];
    }
    // (a wavefront's chunks in the order in which several wavefronts' are added: the same
    // bits with a residual and without)
    float all = team_sum<L>(sum[0], buf, turn);
    if constexpr (L == 64)
#pragma unroll
      for (int e = 1; e < E; ++e) all += team_sum<L>(sum[e], buf, turn);
    const float q = 1.f / sqrtf(all * a.inv_n + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[e][k] = x[e][k] * q * g[e][k];
      const int c = tm.col(e);
      if constexpr (L != 8)
        if (codes) {
          store_codes(a, row, c, x[e]);
          continue;
        }
      Raw<T> p;
      pack(x[e], type_of<T>(a.ot), p);
      store_raw<T != MIXED>(a.out, type_of<T>(a.ot), row * a.ldo + c, n - c, p);
    }
    if (a.rstd && tm.lane == 0) a.rstd[row] = q;
    if constexpr (T == MIXED) load(row + tm.step);
  }
}

// Rows wider than a workgroup's registers are read again for the result: S by
// the threads that wrote it.  (The second reading comes from the caches: 256 x 20000 with a
// residual, bf16, 13 us.)
__global__ __launch_bounds__(MAX_BLOCK) void k_rms_forward_wide(Args a) {
  __shared__ float buf[2 * (MAX_BLOCK / 64)];
  int turn = 0;
  const int chunks = (a.n + 7) / 8, whole = (chunks + 15) / 16 * 16;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    float sum = 0.f;
    for (int i = threadIdx.x; i < chunks; i += MAX_BLOCK) {
      const int c = i * 8;
      Raw8 p;
      float x[8];
      load_raw(a.x, a.xt, row * a.ldx + c, a.n - c, a.n, p);
      values_of(p, a.xt, a.n - c, a.n, x);
      if (a.r) {
        float r[8];
        load_raw(a.r, a.rt, row * a.ldr + c, a.n - c, a.n, p);
        values_of(p, a.rt, a.n - c, a.n, r);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] += r[k];
        pack(x, a.st, p);
        store_raw(a.s, a.st, row * a.lds + c, a.n - c, p);
        convert(p, a.st, x);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += x[k] * x[k];
    }
    const float q = 1.f / sqrtf(team_sum<0>(sum, buf, turn) * a.inv_n + a.eps);
    for (int i = threadIdx.x; i < whole; i += MAX_BLOCK) {
      const int c = i * 8;
      Raw8 p;
      float x[8], g[8];
      // (a chunk past the row's end holds zeros, whatever its load brings)
      if (a.r) load_raw(a.s, a.st, row * a.lds + c, a.n - c, a.n, p);
      else load_raw(a.x, a.xt, row * a.ldx + c, a.n - c, a.n, p);
      values_of(p, a.r ? a.st : a.xt, a.n - c, a.n, x);
      if (a.gamma) {
        load_raw(a.gamma, a.wt, c, a.n - c, a.n, p);
        values_of(p, a.wt, a.n - c, a.n, g);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = x[k] * q * (a.gamma ? g[k] : 1.f);
      if (a.codes) {
        store_codes(a, row, c, x);
      } else {
        pack(x, a.ot, p);
        store_raw(a.out, a.ot, row * a.ldo + c, a.n - c, p);
      }
    }
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = q;
  }
}

// Joins the lanes' column sums of a workgroup's teams and writes them: to the
// partial sums of this workgroup, or (one workgroup in the launch) to dgamma.
template <int L, int E>
__device__ __forceinline__ void join_columns(float (&acc)[E][8], const Args& a, const Team<L>& tm, float* buf) {
  const int n = a.n;
  float* part = a.part ? a.part + (int64_t)blockIdx.x * n : nullptr;
  if constexpr (L < 8) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = tm.col(e), t = part ? (int)DT_F32 : a.wt;
      Raw8 p;
      pack(acc[e], t, p);
      store_raw(part ? part : a.dgamma, t, c, n - c, p);
    }
  } else {
    constexpr int cols = L * E * 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int o = L; o < 64; o <<= 1) acc[e][k] += __shfl_xor(acc[e][k], o);
        if (lane < L) buf[wave * cols + (e * L + lane) * 8 + k] = acc[e][k];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols && c < n; c += TEAM_BLOCK) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < TEAM_BLOCK / 64; ++w) v += buf[w * cols + c];
      if (part) part[c] = v;
      else store1(a.dgamma, a.wt, c, v);
    }
  }
}

// T: the type of S, dY, dS and dX (or MIXED); PAST: dS is given.
template <int L, int E, int T, bool PAST>
__global__ __launch_bounds__(L < 8 ? group_threads(L) : TEAM_BLOCK) void k_rms_backward(Args a) {
  __shared__ float buf[L < 8 ? 2 * (MAX_BLOCK / 64) : (TEAM_BLOCK / 64) * L * E * 8];
  const Team<L> tm;
  const int n = a.n, n8 = row_of<T>(n);
  const bool past = T == MIXED ? a.r && a.out : PAST;
  int turn = 0;
  float g[E][8], acc[E][8] = {};
  Raw<T> xr[E], yr[E], sr[E];
  float q = 0.f;
  const auto load = [&](int64_t row) {  // (past the last row: the last again)
    row = row < a.m ? row : a.m - 1;
    load_row<T>(a.x, a.xt, row * a.ldx, n, tm, xr);
    load_row<T>(a.dy, a.dyt, row * a.lddy, n, tm, yr);
    q = a.crstd[row];
  };
  const auto load_past = [&](int64_t row) {
    row = row < a.m ? row : a.m - 1;
    if (past) load_row<T>(a.r, a.rt, row * a.ldr, n, tm, sr);
  };
  // the next row is asked for before this one is used (1024 threads have no
  // registers for that)
  constexpr bool EARLY = T != MIXED && (L != 0 || E == 1);
  if constexpr (EARLY) {
    load(tm.first);
    load_past(tm.first);
  }
  load_gamma<E>(a, tm, g);
  for (int64_t row = tm.first; row < a.m; row += tm.step) {
    float x[E][8], dy[E][8], ds[PAST || T == MIXED ? E : 1][8], sum = 0.f;
    if constexpr (!EARLY) {
      load(row);
      load_past(row);
    }
    const float rq = q;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int have = n - tm.col(e);
      values_of(xr[e], type_of<T>(a.xt), have, n8, x[e]);
      values_of(yr[e], type_of<T>(a.dyt), have, n8, dy[e]);
    }
    if constexpr (EARLY) load(row + tm.step);
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[e][k] *= rq;
        acc[e][k] += dy[e][k] * x[e][k];
        dy[e][k] *= g[e][k];
        sum += dy[e][k] * x[e][k];
      }
    }
    if (a.out) {
      const float mean = team_sum<L>(sum, buf, turn) * a.inv_n;
#pragma unroll
      for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int k = 0; k < 8; ++k) dy[e][k] = rq * (dy[e][k] - x[e][k] * mean);
        if (past) {
          values_of(sr[e], type_of<T>(a.rt), n - tm.col(e), n8, ds[PAST || T == MIXED ? e : 0]);
#pragma unroll
          for (int k = 0; k < 8; ++k) dy[e][k] += ds[PAST || T == MIXED ? e : 0][k];
        }
      }
      if constexpr (EARLY) load_past(row + tm.step);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        Raw<T> p;
        pack(dy[e], type_of<T>(a.ot), p);
        store_raw<T != MIXED>(a.out, type_of<T>(a.ot), row * a.ldo + tm.col(e), n - tm.col(e), p);
      }
    }
  }
  if (!a.dgamma) return;
  join_columns<L, E>(acc, a, tm, buf);
}

// Backward pass of such rows, a column a thread and step (256 x 20000, bf16, with the
// weights' gradient 65 us in three launches).
__global__ __launch_bounds__(MAX_BLOCK) void k_rms_backward_wide(Args a) {
  __shared__ float buf[2 * (MAX_BLOCK / 64)];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
    const float q = a.crstd[row];
    float sum = 0.f;
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK)
      sum += load1(a.dy, a.dyt, row * a.lddy + c) * (a.gamma ? load1(a.gamma, a.wt, c) : 1.f) *
             (load1(a.x, a.xt, row * a.ldx + c) * q);
    const float mean = team_sum<0>(sum, buf, turn) * a.inv_n;
    for (int c = threadIdx.x; c < a.n; c += MAX_BLOCK) {
      const float g = load1(a.dy, a.dyt, row * a.lddy + c) * (a.gamma ? load1(a.gamma, a.wt, c) : 1.f);
      const float d = q * (g - load1(a.x, a.xt, row * a.ldx + c) * q * mean);
      store1(a.out, a.ot, row * a.ldo + c, a.r ? d + load1(a.r, a.rt, row * a.ldr + c) : d);
    }
  }
}

// Column sums of wide rows: a thread owns a column, blockIdx.y a run of rows.
__global__ __launch_bounds__(TEAM_BLOCK) void k_rms_columns_wide(Args a) {
  const int64_t c = (int64_t)blockIdx.x * TEAM_BLOCK + threadIdx.x;
  if (c >= a.n) return;
  const int64_t per = (a.m + gridDim.y - 1) / gridDim.y;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < a.m ? r0 + per : a.m;
  float v = 0.f;
  for (int64_t row = r0; row < r1; ++row)
    v += load1(a.dy, a.dyt, row * a.lddy + c) * (load1(a.x, a.xt, row * a.ldx + c) * a.crstd[row]);
  a.part[(int64_t)blockIdx.y * a.n + c] = v;
}

// dgamma: the workgroups' partial sums, 32 shares of them side by side for 32
// columns, added in a fixed order.  count = 0 writes zeros.  (512 sums of 6001 columns: 5
// us for 12 MB.)
__global__ __launch_bounds__(1024) void k_rms_columns(const float* part, int64_t count, int n, void* dgamma, int wt) {
  __shared__ float buf[32][33];
  const int c = threadIdx.x & 31, w = threadIdx.x >> 5;
  for (int64_t at = (int64_t)blockIdx.x * 32; at < n; at += (int64_t)gridDim.x * 32) {
    const int64_t col = at + c;
    float v = 0.f;
    if (col < n) {
#pragma unroll 8
      for (int64_t i = w; i < count; i += 32) v += part[i * n + col];
    }
    buf[w][c] = v;
    __syncthreads();
    if (w == 0 && col < n) {
      v = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) v += buf[i][c];
      store1(dgamma, wt, col, v);
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(TEAM_BLOCK) void k_rms_no_columns(float* rstd, int64_t m, float eps) {
  for (int64_t i = (int64_t)blockIdx.x * TEAM_BLOCK + threadIdx.x; i < m; i += (int64_t)gridDim.x * TEAM_BLOCK)
    rstd[i] = 1.f / sqrtf(eps);
}

// Lanes a row, chunks of eight columns a lane, threads of a workgroup.
struct Shape {
  int L, E, threads;
};

// A wavefront holds its row where a lane has `most` chunks of it at most, else several
// share it.  More than that leaves no registers for the next row's loads: 8192 x 2048 with a
// residual 26 us with four wavefronts a row, 35 with one (bf16), 61 and 75 (fp32); fp32
// without one 30 and 37; types that are looked at as it runs, X in bf16 and R in fp32, 41 and
// 61, and 8192 x 1024 20 and 24.  32768 x 2048 in bf16 without a residual: 51 and 46.
Shape shape_of(int64_t n, bool codes, int most) {
  const int64_t chunks = (n + 7) / 8;
  if (chunks <= 8 && !codes) return {8, 1, TEAM_BLOCK};
  if (chunks <= 16) return {16, 1, TEAM_BLOCK};
  if (chunks <= 32) return {32, 1, TEAM_BLOCK};
  if (chunks <= 64) return {64, 1, TEAM_BLOCK};
  if (chunks <= 128 && most >= 2) return {64, 2, TEAM_BLOCK};
  if (chunks <= 256 && most >= 4) return {64, 4, TEAM_BLOCK};
  const int E = chunks <= MAX_BLOCK ? 1 : 2;
  const int threads = (int)(((chunks + E - 1) / E + 63) / 64 * 64);
  return {threads <= MAX_BLOCK / 2 ? 1 : 0, E, threads};
}

// One of a kernel's shapes; f(L, E) launches it.
template <int V>
using Int = std::integral_constant<int, V>;
template <bool BACK, typename F>
void with_shape(const Shape& sh, F f) {
  if (sh.L == 8) f(Int<8>(), Int<1>());
  else if (sh.L == 16) f(Int<16>(), Int<1>());
  else if (sh.L == 32) f(Int<32>(), Int<1>());
  else if (sh.L == 64 && sh.E == 1) f(Int<64>(), Int<1>());
  else if (sh.L == 64 && sh.E == 2) f(Int<64>(), Int<2>());
  else if (sh.L == 64) f(Int<64>(), Int<BACK ? 2 : 4>());  // (the backward pass has two at most)
  else if (sh.L == 1) f(Int<1>(), Int<1>());
  else if (sh.E == 1) f(Int<0>(), Int<1>());
  else f(Int<0>(), Int<2>());
}

// The type that all of these have, or MIXED: a kernel for one type knows how many loads
// and stores are on their way and waits for none too many (4001 x 6001, fp16, backward 47
// us, 66 with dY in bf16).  (Rows of fewer than eight values are left to the
// kernels for mixed types.)
int common_type(int64_t n, std::initializer_list<const Mat*> all) {
  int t = -1;
  for (const Mat* m : all)
    if (m->data) t = t < 0 || t == m->type ? m->type : MIXED;
  return n < 8 ? MIXED : t;
}

int64_t rows_at_once(const Shape& sh) { return sh.L < 8 ? 1 : TEAM_BLOCK / sh.L; }

// Workgroups of the backward pass: what fills the chip, but eight rows a team
// at least once there are 512 (each workgroup writes n partial sums: 8192 x 2048 in
// bf16 32 us so, 35 with four rows; 2110 x 1564 15 us in 512 workgroups, 18 in 256).
int64_t backward_groups(int64_t m, int64_t n) {
  if (n > kRegisterCols) return std::max<int64_t>(1, std::min<int64_t>(32, m / 8));
  const Shape sh = shape_of(n, false, 2);
  const int64_t rows = rows_at_once(sh);
  const int64_t need = (m + rows - 1) / rows;
  const int64_t fill = sh.L < 8 ? 256 * std::max(1, 1536 / sh.threads) : 1024;
  return std::max<int64_t>(1, std::min({need, fill, std::max<int64_t>(512, need / 8)}));
}

}  // namespace

hipError_t rms_norm(const Mat& X, const Mat& R, const void* gamma, int wt, float eps, const Mat& S, const Mat& Y,
                    const Held& Y8, float* rstd, hipStream_t s) {
  if (X.rows == 0 || (X.cols == 0 && !rstd)) return hipSuccess;
  if (X.cols == 0) {
    k_rms_no_columns<<<(unsigned)std::min<int64_t>((X.rows + TEAM_BLOCK - 1) / TEAM_BLOCK, 1 << 16), TEAM_BLOCK, 0, s>>>(
        rstd, X.rows, eps);
    return hipGetLastError();
  }
  Args a{};
  a.x = X.data; a.ldx = X.ld; a.xt = X.type;
  a.r = R.data; a.ldr = R.ld; a.rt = R.type;
  a.s = S.data; a.lds = S.ld; a.st = S.type;
  a.out = Y.data; a.ldo = Y.ld; a.ot = Y.type;
  a.codes = Y8.codes; a.ldc = Y8.ld; a.scales = Y8.scales; a.ldsc = Y8.lds;
  a.gamma = gamma; a.wt = wt;
  a.rstd = rstd;
  a.m = X.rows; a.n = (int)X.cols; a.eps = eps; a.inv_n = (float)(1.0 / (double)X.cols);
  if (X.cols > kRegisterCols) {
    k_rms_forward_wide<<<(unsigned)std::min<int64_t>(a.m, 1 << 20), MAX_BLOCK, 0, s>>>(a);
    return hipGetLastError();
  }
  const int type = common_type(a.n, {&X, &R, &S, &Y});
  const Shape sh = shape_of(X.cols, a.codes != nullptr, type == MIXED ? 1 : type == DT_F32 || a.r ? 2 : 4);
  const int64_t rows = rows_at_once(sh);
  const int64_t grid = std::min<int64_t>((a.m + rows - 1) / rows, sh.L < 8 ? 256 * std::max(1, 2048 / sh.threads) : 2048);
  // (eight lanes hold no block of 128 columns: their kernels have no codes)
  const dim3 g((unsigned)grid), b((unsigned)sh.threads);
  with_shape<false>(sh, [&](auto l, auto e) {
    constexpr int L = decltype(l)::value, E = decltype(e)::value;
    // (what a lane may hold: see shape_of)
    const auto typed = [&](auto t) {
      constexpr int T = decltype(t)::value;
      if constexpr (E <= (T == DT_F32 ? 2 : 4)) {
        if (a.codes) {
          if constexpr (L != 8) {
            if constexpr (E <= 2)
              if (a.r) return k_rms_forward<L, E, T, true, true><<<g, b, 0, s>>>(a);
            k_rms_forward<L, E, T, false, true><<<g, b, 0, s>>>(a);
          }
        } else {
          if constexpr (E <= 2)
            if (a.r) return k_rms_forward<L, E, T, true, false><<<g, b, 0, s>>>(a);
          k_rms_forward<L, E, T, false, false><<<g, b, 0, s>>>(a);
        }
      }
    };
    switch (type) {
      case DT_F32: return typed(Int<DT_F32>());
      case DT_BF16: return typed(Int<DT_BF16>());
      case DT_F16: return typed(Int<DT_F16>());
      default:
        if constexpr (E == 1 || L == 0) k_rms_forward<L, E, MIXED, false, false><<<g, b, 0, s>>>(a);
    }
  });
  return hipGetLastError();
}

int64_t rms_norm_workspace(int64_t m, int64_t n) {
  if (m == 0 || n == 0) return 0;
  return backward_groups(m, n) * n * (int64_t)sizeof(float);
}

hipError_t rms_norm_backward(const Mat& dY, const Mat& S, const float* rstd, const void* gamma, int wt, const Mat& dS,
                             const Mat& dX, void* dgamma, float* ws, hipStream_t s) {
  const int n = (int)S.cols;
  // a launch holds fewer than 2^32 threads along a side
  const unsigned cgrid = (unsigned)std::min<int64_t>(((int64_t)n + 31) / 32, 1 << 20);
  if (n == 0 || (S.rows == 0 && !dgamma)) return hipSuccess;
  if (S.rows == 0) {
    k_rms_columns<<<cgrid, 1024, 0, s>>>(nullptr, 0, n, dgamma, wt);
    return hipGetLastError();
  }
  Args a{};
  a.x = S.data; a.ldx = S.ld; a.xt = S.type;
  a.dy = dY.data; a.lddy = dY.ld; a.dyt = dY.type;
  a.r = dS.data; a.ldr = dS.ld; a.rt = dS.type;
  a.out = dX.data; a.ldo = dX.ld; a.ot = dX.type;
  a.gamma = gamma; a.wt = wt;
  a.crstd = rstd;
  a.dgamma = dgamma;
  a.m = S.rows; a.n = n; a.inv_n = (float)(1.0 / (double)n);
  if (!a.out && !dgamma) return hipSuccess;
  const int64_t groups = backward_groups(a.m, n);
  const bool wide = n > kRegisterCols;
  a.part = dgamma && (groups > 1 || wide) ? ws : nullptr;
  if (wide) {
    if (dgamma) k_rms_columns_wide<<<dim3((unsigned)((n + TEAM_BLOCK - 1) / TEAM_BLOCK), (unsigned)groups), TEAM_BLOCK, 0, s>>>(a);
    if (a.out) k_rms_backward_wide<<<(unsigned)std::min<int64_t>(a.m, 1 << 20), MAX_BLOCK, 0, s>>>(a);
  } else {
    const Shape sh = shape_of(n, false, 2);
    const dim3 g((unsigned)groups), b((unsigned)sh.threads);
    with_shape<true>(sh, [&](auto l, auto e) {
      constexpr int L = decltype(l)::value, E = decltype(e)::value;
      const auto typed = [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (a.r && a.out) k_rms_backward<L, E, T, true><<<g, b, 0, s>>>(a);
        else k_rms_backward<L, E, T, false><<<g, b, 0, s>>>(a);
      };
      switch (common_type(n, {&S, &dY, &dS, &dX})) {
        case DT_F32: return typed(Int<DT_F32>());
        case DT_BF16: return typed(Int<DT_BF16>());
        case DT_F16: return typed(Int<DT_F16>());
        default: k_rms_backward<L, E, MIXED, false><<<g, b, 0, s>>>(a);
      }
    });
  }
  if (a.part) k_rms_columns<<<cgrid, 1024, 0, s>>>(a.part, groups, n, dgamma, wt);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
