// Log probabilities of labels, entropy and the most probable classes of rows of
// scores, and the gradient of the scores (gfx950).
//
// With m the row's maximum, s = sum exp(z - m) and w = sum (z - m) exp(z - m):
//   lse = m + log s,  logp = (z_label - m) - log s,  entropy = log s - w / s;
// dz_j = dlogp ([j = label] - p_j) - dentropy p_j (log p_j + entropy).
// lse in fp32 is off by up to half a step of its own, which far from zero is more than
// the rest of p's error (3e-5 of p at 1000): what its rounding leaves is handed on too.
// One pass over the scores, a running maximum per lane with the sums raised or
// lowered to it; about a dozen operations a score, an exponential among them:
// bound by the scores' bytes, near the rate of exponentials for 16-bit ones.
//
// Rows of up to 512 scores are held in the registers of 8 to 64 lanes, and a few
// highest scores are taken out one after the other.  Longer rows are streamed, by
// a wavefront or a workgroup each, or by several workgroups where there are few rows,
// which a second launch joins.  There every wavefront keeps its highest scores as a
// list over its lanes and looks at a chunk of 512 scores only where one is above the
// list's last; chunks come in rising order of columns, so equal scores stay in the
// order of their index.  Scores are compared as integers of the same order.
//
// Statistics are fp32; what is rounded to fewer bits is dz alone, to the type asked for.
//
// Measured: 150001 x 41 in fp32, 5 alternatives, 17 us (2.2 TB/s: five rounds over a
// wavefront's eight rows; 8 without alternatives); 3 x 262144 in bf16, 10 alternatives, 9 us and 4 for the join (the
// way to memory, six times one after the other); gradient of 4099 x 30011 in bf16 114 us
// (4.3 TB/s; 98 at 30016 columns, whose rows lie at multiples of 16 bytes).
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
// A few alternatives: taken out one after the other.
constexpr int kFewTop = 8;
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
  float *logp, *entropy, *lse, *rest, *top_logp;
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
  const float lse = t.m + log_s;
  if (a.lse) a.lse[row] = lse;
  if (a.rest) {  // what the sum's rounding leaves, exactly
    const float b = lse - t.m;
    a.rest[row] = finite_f32(lse) ? (t.m - (lse - b)) + (log_s - b) : 0.f;
  }
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

// --------------------------------------------------- highest of a wavefront

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

__device__ __forceinline__ int key_of_entry(uint64_t x) { return (int)((uint32_t)(x >> 32) ^ 0x80000000u); }

// The wavefront's `top` highest entries, highest first: lane i gets the i-th (0 if
// there are not so many).  buf: 64 entries of LDS of the wavefront's own.  No wanted
// score is below the top-th highest of the lanes' best ones; what is not below that,
// `top` entries and few more in any order but a sorted one, is ranked by comparing
// each with all.  The best ones' top-th is found by ranking too where there are more than
// a few (50000 x 2000 in bf16: 20 alternatives 127 us, 156 by taking out; 5 115 and 110).
template <int E>
__device__ __forceinline__ uint64_t wave_top(const uint64_t (&x)[E], int top, uint64_t* buf) {
  const int lane = threadIdx.x & 63;
  uint64_t best = x[0];
#pragma unroll
  for (int e = 1; e < E; ++e) best = x[e] > best ? x[e] : best;
  int bound = NONE, rest = key_of_entry(best);
  if (top <= kFewTop) {
    for (int i = 0; i < top; ++i) {
      bound = group_best<64, true>(rest);
      rest = lane == __ffsll((unsigned long long)__ballot(rest == bound)) - 1 ? NONE : rest;
    }
  } else {
    int* const keys = reinterpret_cast<int*>(buf);
    wave_sync();
    keys[lane] = rest;
    wave_sync();
    int rank = 0;
#pragma unroll 16
    for (int l = 0; l < 64; ++l) rank += keys[l] > rest;
    bound = group_best<64, false>(rank < top ? rest : 0x7fffffff);
  }
  // (an entry that is none is below all)
  const uint32_t least = bound == NONE ? 1u : (uint32_t)bound ^ 0x80000000u;
  int mine = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) mine += (uint32_t)(x[e] >> 32) >= least;
  const int upto = wave_incl_scan(mine), total = wave_last(upto);
  uint64_t out = 0;
  if (total <= 64) {
    wave_sync();
    int place = upto - mine;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if ((uint32_t)(x[e] >> 32) >= least) buf[place++] = x[e];
    wave_sync();
    const uint64_t y = lane < total ? buf[lane] : 0;
    int rank = 0;  // (entries are different from each other)
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

// ------------------------------------------------------------- short rows

// L lanes hold a row, eight scores a lane.  MANY: a wavefront ranks more than a few
// alternatives (20 of 100000 x 500 in bf16: 97 us, 225 by taking them out; 5: 88).
template <int L, int T, bool MANY = false>
__global__ __launch_bounds__(BLOCK) void k_logp_short(Args a) {
  static_assert(!MANY || L == 64);
  constexpr int TEAMS = BLOCK / L;
  __shared__ uint64_t bufs[MANY ? TEAMS : 1][64];
  const int zt = type_of<T>(a.zt), n8 = row_of<T>(a.v);
  const int lane = threadIdx.x % L, first = lane * 8;
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / L; row < a.t; row += (int64_t)gridDim.x * TEAMS) {
    Raw<T> r;
    float z[8];
    Stats t = EMPTY;
    load_raw(a.z, zt, row * a.ldz + first, a.v - first, n8, r);
    settle(r, zt, a.v - first, n8);
    convert(r, zt, z);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (first + k >= a.v) z[k] = -__builtin_inff();
      t.m = fmaxf(t.m, z[k]);
    }
    t.m = group_max<L>(t.m);
#pragma unroll
    for (int k = 0; k < 8; ++k) add(t, z[k]);
    t.s = group_sum_f32<L>(t.s);
    t.w = group_sum_f32<L>(t.w);
    const float log_s = logf(t.s);
    if (lane == 0) finish_row(a, row, t, log_s);
    if (a.top == 0) continue;
    int key[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) key[k] = first + k < a.v ? key_of(z[k]) : NONE;
    if constexpr (MANY) {
      uint64_t x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = key[k] == NONE ? 0 : entry_of(key[k], first + k);
      const uint64_t best = wave_top(x, a.top, bufs[threadIdx.x / L]);
      if (lane < a.top) store_entry(a, row, lane, best, t, log_s);
      continue;
    }
    float mine = 0.f;  // what the round of this lane's number found
    int mine_col = 0;
    for (int i = 0; i < a.top; ++i) {
      int best = NONE;
#pragma unroll
      for (int k = 0; k < 8; ++k) best = key[k] > best ? key[k] : best;
      best = group_best<L, true>(best);
      int col = 0x7fffffff;
#pragma unroll
      for (int k = 7; k >= 0; --k) col = key[k] == best ? first + k : col;
      col = group_best<L, false>(col);
#pragma unroll
      for (int k = 0; k < 8; ++k) key[k] = first + k == col ? NONE : key[k];
      if (lane == i % L) {
        mine = score_of(best);
        mine_col = col;
      }
      if (i % L == L - 1 || i == a.top - 1) {
        const int begin = i / L * L;
        if (begin + lane <= i) store_top(a, row, begin + lane, mine, mine_col, t, log_s);
      }
    }
  }
}

// -------------------------------------------------------------- long rows

// The wavefront's highest scores: lane i holds the i-th as an entry.  Scores above the
// last of a full list wait in LDS and are ranked together with it when 64 do not hold
// them.
struct List {
  uint64_t entry;
  int last, waiting;  // last: the lowest key of a full list, or NONE
  __device__ List() : entry(0), last(NONE), waiting(0) {}

  template <int E>
  __device__ __forceinline__ void rank(const uint64_t (&x)[E], int top, uint64_t* buf) {
    entry = wave_top(x, top, buf);
    waiting = 0;
    last = __builtin_amdgcn_readlane(key_of_entry(entry), top - 1);  // (no entry: NONE)
  }

  // The chunk that begins at column `first` of this lane.  floor: a key below which no
  // score is wanted.  Equal scores that are there already have lower columns.
  __device__ __forceinline__ void take(const float (&z)[8], int first, int end, int floor, int top, uint64_t* wait, uint64_t* buf) {
    const int lane = threadIdx.x & 63;
    int k[8], total = waiting;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      k[j] = first + j < end ? key_of(z[j]) : NONE;
      k[j] = k[j] >= floor ? k[j] : NONE;
      total += __popcll(__ballot(k[j] > last));
    }
    if (total <= 64) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t who = __ballot(k[j] > last);
        const int at = waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        if (k[j] > last) wait[at] = entry_of(k[j], first + j);
        waiting += __popcll(who);
      }
      return;
    }
    wave_sync();
    uint64_t x[10];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = k[j] == NONE ? 0 : entry_of(k[j], first + j);
    x[8] = entry;
    x[9] = lane < waiting ? wait[lane] : 0;
    rank(x, top, buf);
  }

  __device__ __forceinline__ void finish(int top, const uint64_t* wait, uint64_t* buf) {
    if (waiting == 0) return;
    wave_sync();
    const uint64_t x[2] = {entry, (int)(threadIdx.x & 63) < waiting ? wait[threadIdx.x & 63] : 0};
    rank(x, top, buf);
  }
};

// A workgroup of W threads streams columns [part * per, + per) of a row.  Its
// wavefronts tell each other how high the scores of a full list are.  TOP: NO, LISTS, or
// ONE, the highest score alone, of which each lane keeps its own (1500 x 16000 in fp16 21
// us, 26 with lists).
constexpr int NO = 0, ONE = 1, LISTS = 2;
template <int W, int TOP, int T>
__global__ __launch_bounds__(W) void k_logp_long(Args a) {
  constexpr int WAVES = W / 64;
  __shared__ Stats stats[WAVES];
  __shared__ uint64_t lists[TOP == LISTS ? WAVES * 64 : WAVES], bufs[TOP != NO ? WAVES : 1][64], waits[TOP == LISTS ? WAVES : 1][64];
  __shared__ int floor_of;
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int begin = part * a.per, end = a.v - begin < a.per ? a.v : begin + a.per;
  const int64_t base = row * a.ldz;
  Stats t = EMPTY;
  List list;
  int high = NONE, high_col = 0;
  if constexpr (TOP == LISTS && WAVES > 1) {
    if (threadIdx.x == 0) floor_of = NONE;
    __syncthreads();
  }
  Raw<T> next;
  // (a chunk past the row's end is moved back into the row, one past the part's not)
  load_raw<true>(a.z, T, base + begin + (int)threadIdx.x * 8, a.v - begin - (int)threadIdx.x * 8, 8, next);
  for (int at = begin; at < end; at += W * 8) {
    Raw<T> now = next;
    const int c = at + threadIdx.x * 8;
    load_raw<true>(a.z, T, base + c + W * 8, a.v - c - W * 8, 8, next);
    float z[8];
    settle(now, T, a.v - c, 8);
    convert(now, T, z);
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
    if constexpr (TOP == ONE)
      // (a NaN, as below)
      if (__any(high == NONE || t.s != t.s || key_of(most) > high)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int key = c + k < end ? key_of(z[k]) : NONE;
          high_col = key > high ? c + k : high_col;
          high = key > high ? key : high;
        }
      }
    if constexpr (TOP == LISTS)
      // (a NaN, which no comparison sees, has made the sum one)
      if (__any(list.last == NONE || t.s != t.s || key_of(most) > list.last)) {
        int floor = NONE;
        if constexpr (WAVES > 1) floor = __hip_atomic_load(&floor_of, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        const int before = list.last;
        list.take(z, c, end, floor, a.top, waits[wave], bufs[wave]);
        if constexpr (WAVES > 1)
          if (list.last != before && lane == 0) atomicMax(&floor_of, list.last);
      }
  }
  // the lanes' statistics, then the wavefronts'
  {
    const float m = group_max<64>(t.m);
    raise(t, m);
    t.s = group_sum_f32<64>(t.s);
    t.w = group_sum_f32<64>(t.w);
  }
  uint64_t best = 0;
  if constexpr (TOP == ONE) best = wave_best(high == NONE ? 0 : entry_of(high, high_col));
  if constexpr (TOP == LISTS) {
    list.finish(a.top, waits[wave], bufs[wave]);
    best = list.entry;
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) stats[wave] = t;
    if constexpr (TOP != NO) {
      if (lane < a.top) lists[wave * a.top + lane] = best;
    }
    __syncthreads();
    if (wave != 0) return;
    t = stats[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) t = merge(t, stats[w]);
    if constexpr (TOP != NO) best = take_top<WAVES>(lists, WAVES * a.top, a.top, bufs[0]);
  }
  const float log_s = logf(t.s);
  if (a.parts == 1) {
    if (lane == 0) finish_row(a, row, t, log_s);
    if (TOP != NO && lane < a.top) store_entry(a, row, lane, best, t, log_s);
  } else {
    if (lane == 0) a.stats[blockIdx.x] = t;
    if (TOP != NO && lane < a.top) a.lists[(int64_t)blockIdx.x * a.top + lane] = best;
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
  const float *lse, *rest, *entropy, *dlogp, *dentropy;
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
    const float lse = a.lse[row], rest = a.rest ? a.rest[row] : 0.f, db = a.dentropy ? a.dentropy[row] : 0.f;
    // log p = z - lse - rest: the rest is taken off in the exponential's multiply-add, and
    // off the entropy for log p + entropy
    const float off = -rest * LOG2E, h = (a.dentropy ? a.entropy[row] : 0.f) - rest;
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
        const float lp = z[k] - lse, p = __builtin_amdgcn_exp2f(fmaf(lp, LOG2E, off));
        float d = p == 0.f ? 0.f : -p * (da + db * (lp + h));
        d = c + k == y ? d + da : d;
        z[k] = none ? 0.f : d;
      }
      pack(z, dt, r);
      store_raw<T != MIXED>(a.dz, dt, row * a.ldd + c, a.v - c, r);
    }
  }
}

// Rows held in registers (64 lanes of eight scores); longer ones are streamed.
constexpr int64_t kShortCols = 512;

// f(type) with the type as a constant.
template <typename F>
void with_type(int t, F f) {
  if (t == DT_F32) f(std::integral_constant<int, DT_F32>());
  else if (t == DT_BF16) f(std::integral_constant<int, DT_BF16>());
  else f(std::integral_constant<int, DT_F16>());
}

// Rows that a wavefront streams by itself: of up to 2048 scores, or 16384 where there are
// enough rows to fill the chip with them (10 alternatives, 3770 x 16000 in bf16: 56 us, 67
// with workgroups; 20 alternatives, 1500 x 16000: 43, 37).
constexpr int64_t kWaveCols = 2048, kManyWaveCols = 16384, kManyRows = 2048;

// Workgroups that share a row: where rows are fewer than what fills the chip, as
// many as have a step of columns each, of which the lists can be joined (37 x 258440 in bf16,
// 5 alternatives: 21 us with 1024 workgroups, 23 with 2048; 679 x 20159, 20 alternatives: 26
// with a workgroup a row, 37 with two or more).
int parts_of(int64_t t, int64_t v, int top) {
  if (t == 0 || v <= kWaveCols || t >= 512) return 1;
  const int64_t steps = (v + BLOCK * 8 - 1) / (BLOCK * 8);
  const int64_t most = std::min<int64_t>(kMostParts, top > 0 ? kMostEntries / top : kMostParts);
  const int64_t parts = std::max<int64_t>(1, std::min({steps, most, (1024 + t - 1) / t}));
  const int64_t per = (steps + parts - 1) / parts;
  return (int)((steps + per - 1) / per);
}

}  // namespace

int64_t log_probs_workspace(int64_t t, int64_t v, int top) {
  const int64_t parts = parts_of(t, v, top);
  if (parts == 1) return 0;
  return t * parts * ((int64_t)sizeof(Stats) + top * (int64_t)sizeof(uint64_t)) + 16;
}

hipError_t log_probs(const LogProbs& x, void* ws, hipStream_t s) {
  if (x.Z.rows == 0) return hipSuccess;
  Args a{};
  a.z = x.Z.data; a.ldz = x.Z.ld; a.zt = x.Z.type;
  a.t = x.Z.rows; a.v = (int)x.Z.cols;
  a.labels = x.labels; a.i64 = x.labels_i64;
  a.top = x.top;
  a.logp = x.logp; a.entropy = x.entropy; a.lse = x.lse; a.rest = x.rest; a.top_logp = x.top_logp; a.top_index = x.top_index;
  a.parts = 1;
  const auto grid = [&](int lanes) {
    const int64_t rows = BLOCK / lanes;
    return dim3((unsigned)std::min<int64_t>((a.t + rows - 1) / rows, 1 << 20));
  };
  if (a.v < 8) {
    k_logp_short<8, MIXED><<<grid(8), BLOCK, 0, s>>>(a);
    return hipGetLastError();
  }
  if (a.v <= kShortCols) {
    with_type(a.zt, [&](auto type) {
      constexpr int T = decltype(type)::value;
      if (a.v <= 64) k_logp_short<8, T><<<grid(8), BLOCK, 0, s>>>(a);
      else if (a.v <= 128) k_logp_short<16, T><<<grid(16), BLOCK, 0, s>>>(a);
      else if (a.v <= 256) k_logp_short<32, T><<<grid(32), BLOCK, 0, s>>>(a);
      else if (a.top <= kFewTop) k_logp_short<64, T><<<grid(64), BLOCK, 0, s>>>(a);
      else k_logp_short<64, T, true><<<grid(64), BLOCK, 0, s>>>(a);
    });
    return hipGetLastError();
  }
  const bool wave = a.v <= kWaveCols || (a.v <= kManyWaveCols && a.t >= kManyRows);
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
      if (a.rest) b.rest += r0;
      if (a.top_logp) b.top_logp += r0 * a.top;
      if (a.top_index) b.top_index += r0 * a.top;
    }
    const dim3 g((unsigned)(b.t * b.parts));
    with_type(a.zt, [&](auto type) {
      constexpr int T = decltype(type)::value;
      const auto go = [&](auto top) {
        constexpr int TOP = decltype(top)::value;
        if (wave) k_logp_long<64, TOP, T><<<g, 64, 0, s>>>(b);
        else k_logp_long<BLOCK, TOP, T><<<g, BLOCK, 0, s>>>(b);
      };
      if (a.top == 0) go(std::integral_constant<int, NO>());
      else if (a.top == 1) go(std::integral_constant<int, ONE>());
      else go(std::integral_constant<int, LISTS>());
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.parts > 1) k_logp_join<<<(unsigned)a.t, 64, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t log_probs_backward(const Mat& Z, const void* labels, int labels_i64, const float* lse, const float* rest,
                              const float* entropy, const float* dlogp, const float* dentropy, const Mat& dZ,
                              hipStream_t s) {
  if (Z.rows == 0 || Z.cols == 0) return hipSuccess;
  Back a{Z.data, Z.ld, Z.type, dZ.data, dZ.ld, dZ.type, Z.rows, (int)Z.cols, labels, labels_i64, lse, rest, entropy, dlogp, dentropy};
  const auto go = [&](auto wide, auto type, int64_t shares) {
    constexpr int L = decltype(wide)::value;
    const int64_t rows = BLOCK / L;
    const dim3 g((unsigned)std::min<int64_t>((a.t + rows - 1) / rows, 1 << 20), (unsigned)shares);
    k_logp_back<L, decltype(type)::value><<<g, BLOCK, 0, s>>>(a);
  };
  const auto typed = [&](auto type) {
    if (a.v <= 64) return go(std::integral_constant<int, 8>(), type, 1);
    if (a.v <= 128) return go(std::integral_constant<int, 16>(), type, 1);
    if (a.v <= 256) return go(std::integral_constant<int, 32>(), type, 1);
    if (a.v <= 512) return go(std::integral_constant<int, 64>(), type, 1);
    const int64_t steps = ((int64_t)a.v + BLOCK * 8 - 1) / (BLOCK * 8);
    go(std::integral_constant<int, BLOCK>(), type, std::min<int64_t>(steps, std::max<int64_t>(1, (4096 + a.t - 1) / a.t)));
  };
  if (a.v < 8 || a.zt != a.dt) typed(std::integral_constant<int, MIXED>());
  else with_type(a.zt, typed);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
