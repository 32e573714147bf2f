// Log probabilities of labels, entropy and the most probable classes of rows of
// scores, and the gradient of the scores (gfx950).
//
// With m the row's maximum, s = sum exp(z - m) and w = sum (z - m) exp(z - m):
//   lse = m + log s,  logp = (z_label - m) - log s,  entropy = log s - w / s;
// dz_j = dlogp ([j = label] - p_j) - dentropy p_j (log p_j + entropy).
// One pass over the scores, a running maximum per lane with the sums raised or
// lowered to it; about a dozen operations a score, an exponential among them:
// bound by the scores' bytes, near the rate of exponentials for 16-bit ones.
//
// Rows of up to 2048 scores are held in the registers of 8 to 64 lanes; the
// highest scores are taken out one after the other.  Longer rows are streamed by
// a workgroup each, or by several where there are few rows, which a second launch
// joins.  There every wavefront keeps its highest scores as a list over its
// lanes and looks at a chunk of 512 scores only where one is above the list's
// last; chunks come in rising order of columns, so equal scores stay in the order
// of their index.  Scores are compared as integers of the same order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "layers.h"
#include "rows8.h"

namespace aires {
namespace kern {
namespace {

constexpr int BLOCK = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.402823466e38f;
constexpr int NONE = (int)0x80000000;  // key of no score: below that of -infinity

// Integers in the order of the scores (0 and -0 are equal, a NaN is +infinity).
__device__ __forceinline__ int key_of(float z) {
  const int b = __float_as_int(z + 0.f);
  return z != z ? 0x7f800000 : b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float score_of(int key) { return __int_as_float(key ^ (key >> 31 & 0x7fffffff)); }

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }

// Running statistics of a part of a row.  m starts at the lowest finite number,
// so that scores of -infinity subtract to -infinity and count 0.
struct Stats {
  float m, s, w;
};
constexpr Stats EMPTY = {LOWEST, 0.f, 0.f};

// The same sums around another maximum.
__device__ __forceinline__ void raise(Stats& t, float m) {
  const float d = fmaxf(t.m - m, LOWEST), f = exp_of(d);
  t.w = f > 0.f ? f * (t.w + d * t.s) : 0.f * t.s;  // (0 s: a NaN stays)
  t.s *= f;
  t.m = m;
}

__device__ __forceinline__ void add(Stats& t, float z) {
  const float d = z - t.m, e = exp_of(d);
  t.s += e;
  t.w += fmaxf(d, LOWEST) * e;
}

__device__ __forceinline__ Stats merge(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m);
  raise(b, m);
  return Stats{m, a.s + b.s, a.w + b.w};
}

template <int W>
__device__ __forceinline__ float group_max(float v) {
  v = fmaxf(v, dpp_f32<0xB1>(v));
  v = fmaxf(v, dpp_f32<0x4E>(v));
  v = fmaxf(v, dpp_f32<0x141>(v));
  if constexpr (W >= 16) v = fmaxf(v, dpp_f32<0x140>(v));
  if constexpr (W >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  if constexpr (W == 64) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

template <int CTRL>
__device__ __forceinline__ int dpp_i32(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, false);
}

template <int W, bool MAX>
__device__ __forceinline__ int group_best(int v) {
  const auto op = [](int a, int b) { return MAX ? (a > b ? a : b) : (a < b ? a : b); };
  v = op(v, dpp_i32<0xB1>(v));
  v = op(v, dpp_i32<0x4E>(v));
  v = op(v, dpp_i32<0x141>(v));
  if constexpr (W >= 16) v = op(v, dpp_i32<0x140>(v));
  if constexpr (W == 32) v = op(v, __shfl_xor(v, 16));
  if constexpr (W == 64)  // one lane of each row of 16, in scalar registers
    v = op(op(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
           op(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
  return v;
}

struct Args {
  const void* z; int64_t ldz; int zt;
  int64_t t; int v;
  const void* labels; int i64;
  int top;
  float *logp, *entropy, *lse, *top_logp;
  int64_t* top_index;
  // parts of a row: columns each, their number, statistics and lists of all parts
  int per, parts;
  Stats* stats; uint64_t* lists;
};

__device__ __forceinline__ int64_t label_of(const void* labels, int i64, int64_t row) {
  return i64 ? static_cast<const int64_t*>(labels)[row] : static_cast<const int32_t*>(labels)[row];
}

// What a row's statistics give.
__device__ __forceinline__ void finish_row(const Args& a, int64_t row, const Stats& t, float log_s) {
  if (a.lse) a.lse[row] = t.m + log_s;
  if (a.entropy) a.entropy[row] = t.s == 0.f ? 0.f : log_s - t.w / t.s;
  if (a.labels) {
    const int64_t y = label_of(a.labels, a.i64, row);
    float p = 0.f;
    if (y >= 0 && y < a.v) {
      const float z = load1(a.z, a.zt, row * a.ldz + y);
      p = t.s == 0.f ? -__builtin_inff() : (z - t.m) - log_s;
    }
    a.logp[row] = p;
  }
}

__device__ __forceinline__ void store_top(const Args& a, int64_t row, int at, float z, int col, const Stats& t, float log_s) {
  a.top_logp[row * a.top + at] = t.s == 0.f ? -__builtin_inff() : (z - t.m) - log_s;
  a.top_index[row * a.top + at] = col;
}

// ------------------------------------------------------------- short rows

// L lanes hold a row, 8 E scores a lane: chunk e is columns (e L + lane) 8 on.
template <int L, int E, int T>
__global__ __launch_bounds__(BLOCK) void k_logp_short(Args a) {
  const int zt = type_of<T>(a.zt), n8 = row_of<T>(a.v);
  constexpr int TEAMS = BLOCK / L;
  const int lane = threadIdx.x % L;
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / L; row < a.t; row += (int64_t)gridDim.x * TEAMS) {
    Raw<T> r[E];
    float z[E][8];
    Stats t = EMPTY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (e * L + lane) * 8;
      load_raw(a.z, zt, row * a.ldz + c, a.v - c, n8, r[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      settle(r[e], zt, a.v - (e * L + lane) * 8, n8);
      convert(r[e], zt, z[e]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if ((e * L + lane) * 8 + k >= a.v) z[e][k] = -__builtin_inff();
        t.m = fmaxf(t.m, z[e][k]);
      }
    }
    t.m = group_max<L>(t.m);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 8; ++k) add(t, z[e][k]);
    t.s = group_sum_f32<L>(t.s);
    t.w = group_sum_f32<L>(t.w);
    const float log_s = logf(t.s);
    if (lane == 0) finish_row(a, row, t, log_s);
    if (a.top == 0) continue;
    int key[E][8];
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < 8; ++k) key[e][k] = (e * L + lane) * 8 + k < a.v ? key_of(z[e][k]) : NONE;
    float mine = 0.f;  // what the round of this lane's number found
    int mine_col = 0;
    for (int i = 0; i < a.top; ++i) {
      int best = NONE;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < 8; ++k) best = key[e][k] > best ? key[e][k] : best;
      best = group_best<L, true>(best);
      int col = 0x7fffffff;
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
#pragma unroll
        for (int k = 7; k >= 0; --k) col = key[e][k] == best ? (e * L + lane) * 8 + k : col;
      col = group_best<L, false>(col);
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < 8; ++k) key[e][k] = (e * L + lane) * 8 + k == col ? NONE : key[e][k];
      if (lane == i % L) {
        mine = score_of(best);
        mine_col = col;
      }
      if (i % L == L - 1 || i == a.top - 1) {
        const int first = i / L * L;
        if (first + lane <= i) store_top(a, row, first + lane, mine, mine_col, t, log_s);
      }
    }
  }
}

// -------------------------------------------------------------- long rows

// A score and its column as one number: higher scores first, then lower columns.
__device__ __forceinline__ uint64_t entry_of(int key, int col) {
  return (uint64_t)((uint32_t)key ^ 0x80000000u) << 32 | ~(uint32_t)col;
}

// The highest of the wavefront's entries (0: none), in every lane.
__device__ __forceinline__ uint64_t wave_best(uint64_t v) {
  const int hi = group_best<64, true>((int)((uint32_t)(v >> 32) ^ 0x80000000u));
  const bool at = (int)((uint32_t)(v >> 32) ^ 0x80000000u) == hi;
  const int lo = group_best<64, true>(at ? (int)((uint32_t)v ^ 0x80000000u) : NONE);
  return (uint64_t)((uint32_t)hi ^ 0x80000000u) << 32 | ((uint32_t)lo ^ 0x80000000u);
}

// The wavefront's `top` highest entries, highest first: lane i gets the i-th (0 if
// there are not so many).  buf: 64 entries of LDS of the wavefront's own.  The
// top-th highest of the lanes' best entries is a bound that the wanted ones are not
// below; what is not below it, `top` entries and few more in any order but
// a sorted one, is ranked by comparing each with all.  (One by one, `top` times a maximum
// over the wavefront: 0.3 us each, where two rankings take about 0.6.)
template <int E>
__device__ __forceinline__ uint64_t wave_top(const uint64_t (&x)[E], int top, uint64_t* buf) {
  const int lane = threadIdx.x & 63;
  uint64_t best = x[0];
#pragma unroll
  for (int e = 1; e < E; ++e) best = x[e] > best ? x[e] : best;
  wave_sync();
  buf[lane] = best;
  wave_sync();
  int rank = 0;
#pragma unroll 16
  for (int l = 0; l < 64; ++l) rank += buf[l] > best;
  // (entries are different from each other)
  const uint64_t at = __ballot(rank == top - 1 && best != 0);
  uint64_t bound = 1;
  if (at) {
    const int l = __ffsll((unsigned long long)at) - 1;
    bound = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(best >> 32), l) << 32 |
            (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)best, l);
  }
  int mine = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) mine += x[e] >= bound;
  const int upto = wave_incl_scan(mine), total = wave_last(upto);
  uint64_t out = 0;
  if (total <= 64) {
    wave_sync();
    int place = upto - mine;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (x[e] >= bound) buf[place++] = x[e];
    wave_sync();
    const uint64_t y = lane < total ? buf[lane] : 0;
    rank = 0;
    for (int l = 0; l < total; ++l) rank += buf[l] > y;
    wave_sync();
    if (lane < total) buf[rank] = y;
    wave_sync();
    out = lane < total && lane < top ? buf[lane] : 0;
  } else {
    uint64_t left[E];
#pragma unroll
    for (int e = 0; e < E; ++e) left[e] = x[e];
    for (int i = 0; i < top; ++i) {
      best = left[0];
#pragma unroll
      for (int e = 1; e < E; ++e) best = left[e] > best ? left[e] : best;
      best = wave_best(best);
#pragma unroll
      for (int e = 0; e < E; ++e) left[e] = left[e] == best ? 0 : left[e];
      out = lane == i ? best : out;
    }
  }
  return out;
}

// The same of `count` entries in memory.
template <int E>
__device__ __forceinline__ uint64_t take_top(const uint64_t* from, int count, int top, uint64_t* buf) {
  const int lane = threadIdx.x & 63;
  uint64_t x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = e * 64 + lane < count ? from[e * 64 + lane] : 0;
  return wave_top(x, top, buf);
}

__device__ __forceinline__ void store_entry(const Args& a, int64_t row, int at, uint64_t entry, const Stats& t, float log_s) {
  store_top(a, row, at, score_of((int)((uint32_t)(entry >> 32) ^ 0x80000000u)), (int)~(uint32_t)entry, t, log_s);
}

// The wavefront's highest scores: lane i holds the i-th.
struct List {
  int key, col, count, last;  // last: the lowest key of a full list, or NONE
  __device__ List() : key(NONE), col(0), count(0), last(NONE) {}

  // The chunk that begins at column `first` of this lane.  More than two new scores are
  // ranked together with the list, fewer put in their places one by one.
  __device__ __forceinline__ void take(const float (&z)[8], int first, int end, int top, uint64_t* buf) {
    const int lane = threadIdx.x & 63;
    int k[8], best = NONE;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      k[j] = first + j < end ? key_of(z[j]) : NONE;
      best = k[j] > best ? k[j] : best;
    }
    if (__popcll(__ballot(best > last)) > 2) {
      uint64_t x[9];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = k[j] == NONE ? 0 : entry_of(k[j], first + j);
      x[8] = lane < count ? entry_of(key, col) : 0;
      const uint64_t y = wave_top(x, top, buf);
      key = (int)((uint32_t)(y >> 32) ^ 0x80000000u);  // (none: NONE)
      col = (int)~(uint32_t)y;
      count = __popcll(__ballot(y != 0));
      if (count == top) last = __builtin_amdgcn_readlane(key, top - 1);
      return;
    }
    while (true) {
      const int most = group_best<64, true>(best);
      if (most <= last) break;  // (a list that is not full ends with NONE)
      const int owner = __ffsll((unsigned long long)__ballot(best == most)) - 1;
      int at = 0;
#pragma unroll
      for (int j = 7; j >= 0; --j) at = k[j] == most ? j : at;
      const int c = __builtin_amdgcn_readlane(first + at, owner);
      // equal scores that are there already have lower columns
      const int place = __popcll(__ballot(lane < count && key >= most));
      const int pk = dpp_move<0x138, 0xf>(key), pc = dpp_move<0x138, 0xf>(col);
      key = lane > place ? pk : lane == place ? most : key;
      col = lane > place ? pc : lane == place ? c : col;
      count += count < top;
      if (count == top) last = __builtin_amdgcn_readlane(key, top - 1);
      at = lane == owner ? at : 8;
      best = NONE;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        k[j] = j == at ? NONE : k[j];
        best = k[j] > best ? k[j] : best;
      }
    }
  }
};

// A workgroup streams columns [part * per, + per) of a row.
template <bool TOP, int T>
__global__ __launch_bounds__(BLOCK) void k_logp_long(Args a) {
  const int zt = type_of<T>(a.zt), n8 = row_of<T>(a.v);
  constexpr int WAVES = BLOCK / 64;
  __shared__ Stats stats[WAVES];
  __shared__ uint64_t lists[TOP ? WAVES * 64 : 1], bufs[TOP ? WAVES : 1][64];
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int begin = part * a.per, end = a.v - begin < a.per ? a.v : begin + a.per;
  const int64_t base = row * a.ldz;
  Stats t = EMPTY;
  List list;
  Raw<T> next;
  // (a chunk past the row's end is moved back into the row, one past the part's not)
  load_raw<true>(a.z, zt, base + begin + (int)threadIdx.x * 8, a.v - begin - (int)threadIdx.x * 8, n8, next);
  for (int at = begin; at < end; at += BLOCK * 8) {
    Raw<T> now = next;
    const int c = at + threadIdx.x * 8;
    load_raw<true>(a.z, zt, base + c + BLOCK * 8, a.v - c - BLOCK * 8, n8, next);
    float z[8];
    settle(now, zt, a.v - c, n8);
    convert(now, zt, z);
    if (c + 8 > end)
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k >= end) z[k] = -__builtin_inff();
    float most = z[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) most = fmaxf(most, z[k]);
    if (__any(most > t.m)) raise(t, fmaxf(t.m, most));
#pragma unroll
    for (int k = 0; k < 8; ++k) add(t, z[k]);
    if constexpr (TOP)
      // (a NaN, which no comparison sees, has made the sum one)
      if (__any(list.count < a.top || t.s != t.s || key_of(most) > list.last)) list.take(z, c, end, a.top, bufs[wave]);
  }
  // the lanes' statistics, then the wavefronts'
  {
    const float m = group_max<64>(t.m);
    raise(t, m);
    t.s = group_sum_f32<64>(t.s);
    t.w = group_sum_f32<64>(t.w);
  }
  if (lane == 0) stats[wave] = t;
  if constexpr (TOP) {
    if (lane < a.top) lists[wave * a.top + lane] = list.key == NONE ? 0 : entry_of(list.key, list.col);
  }
  __syncthreads();
  if (wave != 0) return;
  t = stats[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) t = merge(t, stats[w]);
  const float log_s = logf(t.s);
  if (a.parts == 1) {
    if (lane == 0) finish_row(a, row, t, log_s);
    if constexpr (TOP) {
      const uint64_t x = take_top<4>(lists, WAVES * a.top, a.top, bufs[0]);
      if (lane < a.top) store_entry(a, row, lane, x, t, log_s);
    }
  } else {
    if (lane == 0) a.stats[blockIdx.x] = t;
    if constexpr (TOP) {
      const uint64_t x = take_top<4>(lists, WAVES * a.top, a.top, bufs[0]);
      if (lane < a.top) a.lists[(int64_t)blockIdx.x * a.top + lane] = x;
    }
  }
}

constexpr int kMostEntries = 1024;  // of all parts of a row
constexpr int kMostParts = 64;

// The parts of a row, one wavefront a row.
__global__ __launch_bounds__(64) void k_logp_join(Args a) {
  __shared__ uint64_t buf[64];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  Stats t = lane < a.parts ? a.stats[row * a.parts + lane] : EMPTY;
  raise(t, group_max<64>(t.m));
  t.s = group_sum_f32<64>(t.s);
  t.w = group_sum_f32<64>(t.w);
  const float log_s = logf(t.s);
  if (lane == 0) finish_row(a, row, t, log_s);
  if (a.top > 0) {
    const uint64_t x = take_top<kMostEntries / 64>(a.lists + row * a.parts * a.top, a.parts * a.top, a.top, buf);
    if (lane < a.top) store_entry(a, row, lane, x, t, log_s);
  }
}

// ---------------------------------------------------------------- gradient

struct Back {
  const void* z; int64_t ldz; int zt;
  void* dz; int64_t ldd; int dt;
  int64_t t; int v;
  const void* labels; int i64;
  const float *lse, *entropy, *dlogp, *dentropy;
};

// L lanes a row (a workgroup for long rows, blockIdx.y of gridDim.y runs of it).
// T: the type of Z and dZ (or MIXED).
template <int L, int T>
__global__ __launch_bounds__(BLOCK) void k_logp_back(Back a) {
  constexpr int TEAMS = BLOCK / L;
  const int zt = type_of<T>(a.zt), dt = type_of<T>(a.dt), n8 = row_of<T>(a.v);
  const int lane = threadIdx.x % L;
  const int64_t first = ((int64_t)blockIdx.y * L + lane) * 8, step = (int64_t)gridDim.y * L * 8;
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / L; row < a.t; row += (int64_t)gridDim.x * TEAMS) {
    const float lse = a.lse[row], db = a.dentropy ? a.dentropy[row] : 0.f, h = a.dentropy ? a.entropy[row] : 0.f;
    int64_t y = -1;
    float da = 0.f;
    if (a.dlogp) {
      y = label_of(a.labels, a.i64, row);
      if (y >= 0 && y < a.v) da = a.dlogp[row];
      else y = -1;
    }
    const bool none = lse == -__builtin_inff();
    Raw<T> next;
    load_raw<T != MIXED>(a.z, zt, row * a.ldz + first, (int)(a.v - first), n8, next);
    for (int64_t c = first; c < a.v; c += step) {
      Raw<T> r = next;
      load_raw<T != MIXED>(a.z, zt, row * a.ldz + c + step, (int)(a.v - c - step), n8, next);
      float z[8];
      settle(r, zt, (int)(a.v - c), n8);
      convert(r, zt, z);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float lp = z[k] - lse, p = exp_of(lp);
        float d = p == 0.f ? 0.f : -p * (da + db * (lp + h));
        d = c + k == y ? d + da : d;
        z[k] = none ? 0.f : d;
      }
      pack(z, dt, r);
      store_raw<T != MIXED>(a.dz, dt, row * a.ldd + c, a.v - c, r);
    }
  }
}

constexpr int64_t kShortCols = 2048;

// f(type) with the type as a constant (rows of fewer than eight scores: MIXED).
template <typename F>
void with_type(int t, int64_t v, F f) {
  if (v < 8 || t == MIXED) f(std::integral_constant<int, MIXED>());
  else if (t == DT_F32) f(std::integral_constant<int, DT_F32>());
  else if (t == DT_BF16) f(std::integral_constant<int, DT_BF16>());
  else f(std::integral_constant<int, DT_F16>());
}

// Workgroups that share a row: where rows are fewer than what fills the chip, as
// many as have a step of columns each, of which the lists can be joined.
int parts_of(int64_t t, int64_t v, int top) {
  if (v <= kShortCols || t >= 512) return 1;
  const int64_t steps = (v + BLOCK * 8 - 1) / (BLOCK * 8);
  const int64_t most = std::min<int64_t>(kMostParts, top > 0 ? kMostEntries / top : kMostParts);
  const int64_t parts = std::max<int64_t>(1, std::min({steps, most, (1024 + t - 1) / t}));
  const int64_t per = (steps + parts - 1) / parts;
  return (int)((steps + per - 1) / per);
}

}  // namespace

int64_t log_probs_workspace(int64_t t, int64_t v, int top) {
  const int64_t parts = parts_of(t, v, top);
  if (t == 0 || parts == 1) return 0;
  return t * parts * ((int64_t)sizeof(Stats) + top * (int64_t)sizeof(uint64_t)) + 16;
}

hipError_t log_probs(const LogProbs& x, void* ws, hipStream_t s) {
  if (x.Z.rows == 0) return hipSuccess;
  Args a{};
  a.z = x.Z.data; a.ldz = x.Z.ld; a.zt = x.Z.type;
  a.t = x.Z.rows; a.v = (int)x.Z.cols;
  a.labels = x.labels; a.i64 = x.labels_i64;
  a.top = x.top;
  a.logp = x.logp; a.entropy = x.entropy; a.lse = x.lse; a.top_logp = x.top_logp; a.top_index = x.top_index;
  a.parts = 1;
  const auto grid = [&](int lanes) {
    const int64_t rows = BLOCK / lanes;
    return dim3((unsigned)std::min<int64_t>((a.t + rows - 1) / rows, 1 << 20));
  };
  if (a.v <= kShortCols) {
    with_type(a.zt, a.v, [&](auto type) {
      constexpr int T = decltype(type)::value;
      if (a.v <= 64) k_logp_short<8, 1, T><<<grid(8), BLOCK, 0, s>>>(a);
      else if (a.v <= 128) k_logp_short<16, 1, T><<<grid(16), BLOCK, 0, s>>>(a);
      else if (a.v <= 256) k_logp_short<32, 1, T><<<grid(32), BLOCK, 0, s>>>(a);
      else if (a.v <= 512) k_logp_short<64, 1, T><<<grid(64), BLOCK, 0, s>>>(a);
      else if (a.v <= 1024) k_logp_short<64, 2, T><<<grid(64), BLOCK, 0, s>>>(a);
      else k_logp_short<64, 4, T><<<grid(64), BLOCK, 0, s>>>(a);
    });
    return hipGetLastError();
  }
  a.parts = parts_of(a.t, a.v, a.top);
  const int64_t steps = ((int64_t)a.v + BLOCK * 8 - 1) / (BLOCK * 8);
  a.per = (int)((steps + a.parts - 1) / a.parts * (BLOCK * 8));
  a.lists = static_cast<uint64_t*>(ws);
  a.stats = reinterpret_cast<Stats*>(a.lists + a.t * a.parts * a.top);
  const int64_t groups = a.t * a.parts;
  // a launch holds fewer than 2^32 threads
  constexpr int64_t kMost = int64_t(1) << 23;
  for (int64_t r0 = 0; r0 < a.t; r0 += kMost) {  // (parts = 1 where there are so many)
    Args b = a;
    if (groups > kMost) {
      b.z = static_cast<const char*>(a.z) + r0 * a.ldz * dtype_bytes(a.zt);
      b.t = std::min<int64_t>(a.t - r0, kMost);
      if (a.labels) b.labels = static_cast<const char*>(a.labels) + r0 * (a.i64 ? 8 : 4);
      if (a.logp) b.logp += r0;
      if (a.entropy) b.entropy += r0;
      if (a.lse) b.lse += r0;
      if (a.top_logp) b.top_logp += r0 * a.top;
      if (a.top_index) b.top_index += r0 * a.top;
    }
    const dim3 g((unsigned)(b.t * b.parts));
    with_type(a.zt, a.v, [&](auto type) {
      constexpr int T = decltype(type)::value;
      if (a.top > 0) k_logp_long<true, T><<<g, BLOCK, 0, s>>>(b);
      else k_logp_long<false, T><<<g, BLOCK, 0, s>>>(b);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.parts > 1) k_logp_join<<<(unsigned)a.t, 64, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t log_probs_backward(const Mat& Z, const void* labels, int labels_i64, const float* lse, const float* entropy,
                              const float* dlogp, const float* dentropy, const Mat& dZ, hipStream_t s) {
  if (Z.rows == 0 || Z.cols == 0) return hipSuccess;
  Back a{Z.data, Z.ld, Z.type, dZ.data, dZ.ld, dZ.type, Z.rows, (int)Z.cols, labels, labels_i64, lse, entropy, dlogp, dentropy};
  const auto go = [&](auto wide, auto type, int64_t shares) {
    constexpr int L = decltype(wide)::value;
    const int64_t rows = BLOCK / L;
    const dim3 g((unsigned)std::min<int64_t>((a.t + rows - 1) / rows, 1 << 20), (unsigned)shares);
    k_logp_back<L, decltype(type)::value><<<g, BLOCK, 0, s>>>(a);
  };
  with_type(a.zt == a.dt ? a.zt : MIXED, a.v, [&](auto type) {
    if (a.v <= 64) return go(std::integral_constant<int, 8>(), type, 1);
    if (a.v <= 128) return go(std::integral_constant<int, 16>(), type, 1);
    if (a.v <= 512) return go(std::integral_constant<int, 64>(), type, 1);
    const int64_t steps = ((int64_t)a.v + BLOCK * 8 - 1) / (BLOCK * 8);
    go(std::integral_constant<int, BLOCK>(), type, std::min<int64_t>(steps, std::max<int64_t>(1, (4096 + a.t - 1) / a.t)));
  });
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
