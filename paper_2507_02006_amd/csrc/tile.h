// Matrix-core tile products of 16-bit operands (gfx950, wave64).
//
// acc(m, n) = sum_k A(m, k) B(n, k) for a tile of TM x TN, each wavefront
// WM x WN of it in 32 x 32 x 16 MFMAs.  An operand is either K-contiguous (row
// m holds its k) or K-major (row k holds its m); both are staged as they lie
// in memory, 64 k a step, by loads that go from global memory straight to
// LDS (no registers, no transposed copies).  K-contiguous fragments are read
// 16 bytes a lane; K-major ones with the transposing LDS read, which hands a
// lane four k of its column.  16-byte chunks are placed XORed with their row
// so that neither read meets bank conflicts (256 bytes a cycle: 16 lanes of
// 16 bytes, 32 of 8): the swap is made on the global address of each lane,
// since the destination of such a load is fixed.
//
// Two stages.  Fragments are read one group of products ahead; before the last
// group of a stage the wavefronts meet once, which frees the stage for the
// loads after the next and lets the next stage's first fragments be read under
// that group.  What bounds it is the way from L2 to the CU (64 bytes a cycle):
// 256 x 256 takes 32 bytes a cycle at the matrix cores' full rate, 256 x 128
// 48.  Measured alone, bf16, 8192 x 2048 x 32768: 1372 TFLOP/s with both
// operands K-contiguous, 1005 with one or both K-major; 256 x 128 with 32 k a
// stage and three stages 969.  (Under such load the clock is near 1.9 GHz, at
// which the matrix cores reach 2 PFLOP/s.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aires {
namespace kern {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A 16-bit operand in memory, rows 16-byte aligned, `cols` a multiple of 8.
// K-contiguous: `rows` are m, `cols` k; k past `cols` repeats the row's last
// chunk (the other operand holds zeros there, so that chunk has to be finite).  K-major: `rows` are k, `cols` m.
struct Panel {
  const uint16_t* data;
  int64_t ld, rows, cols;
};

constexpr int BK = 64;  // k of a stage

template <bool F16>
__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) void global_void;

// Load j of a wavefront fills 1 KB of the stage.  Where the stage has fewer
// than every wavefront's share, the last one is loaded more than once.
template <int TOTAL, int WAVES>
__device__ __forceinline__ int part_of(int j, int wave) {
  const int i = j * WAVES + wave;
  return TOTAL % WAVES == 0 || i < TOTAL ? i : TOTAL - 1;
}

// A wavefront's loads of a stage, straight to LDS: a scalar base and a 32-bit
// offset a lane, so no vector arithmetic a load.
template <int TOTAL, int WAVES, int COUNT>
__device__ __forceinline__ void load_parts(const char* base, const uint32_t (&off)[COUNT], char* lds, int wave) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const char* from = reinterpret_cast<const char*>(
      ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32) |
      (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b));
#pragma unroll
  for (int j = 0; j < COUNT; ++j) {
    uint32_t o = off[j];
    asm("" : "+v"(o));
    __builtin_amdgcn_global_load_lds((global_void*)(from + o), (lds_void*)(lds + part_of<TOTAL, WAVES>(j, wave) * 1024), 16, 0,
                                     0);
  }
}

// One operand's share of a stage: SPAN x BK elements, 1 KB an instruction.
template <int SPAN, int WAVES, bool KMAJOR>
struct Stager {
  static constexpr int TOTAL = SPAN * BK / 512, COUNT = (TOTAL + WAVES - 1) / WAVES;  // loads, a wavefront's
  static constexpr int CHUNKS = KMAJOR ? SPAN / 8 : BK / 8;  // 16-byte chunks a row
  static constexpr int ROWS = 64 / CHUNKS;                   // rows an instruction
  static_assert(ROWS >= 1, "a load holds whole rows");
  const char* base;      // first row of the tile, advanced along k
  int64_t step;          // bytes a step
  uint32_t off[COUNT];
  int64_t ld2;           // bytes a row
  int64_t left;          // k that there are from the next stage's first on

  // m0: first m of the tile (m0 < extent of m); k0: first k, a multiple of BK
  __device__ void init(const Panel& p, int64_t m0, int64_t k0, int wave, int lane) {
    const char* d = reinterpret_cast<const char*>(p.data);
    ld2 = p.ld * 2;
    base = d + (KMAJOR ? k0 * ld2 + m0 * 2 : m0 * ld2 + k0 * 2);
    step = KMAJOR ? BK * ld2 : BK * 2;
    left = (KMAJOR ? p.rows : p.cols) - k0;
    place(p, m0, wave, lane);
  }
  // Offsets within a stage.  m past the end repeats the last one (its results
  // are not used), and so does k (the other operand holds zeros there).
  __device__ void place(const Panel& p, int64_t m0, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const int r = part_of<TOTAL, WAVES>(j, wave) * ROWS + lane / CHUNKS;
      if constexpr (KMAJOR) {
        const int64_t last = p.cols - 8 - m0;
        const int c = ((lane % CHUNKS) ^ ((r & 3) * 4)) * 8;
        off[j] = (uint32_t)((r < left ? r : left - 1) * ld2 + (c < last ? c : last) * 2);
      } else {
        const int64_t last = p.rows - 1 - m0;
        const int c = ((lane % CHUNKS) ^ (r / (16 / CHUNKS) % CHUNKS)) * 8;
        off[j] = (uint32_t)((r < last ? r : last) * ld2 + (c < left ? c : left - 8) * 2);
      }
    }
  }
  __device__ __forceinline__ void issue(char* lds, int wave) const { load_parts<TOTAL, WAVES>(base, off, lds, wave); }
};

// Fragment reads of one operand: SPAN rows of m staged, W of them this
// wavefront's, from `first` on.
template <int SPAN, int W, bool KMAJOR>
struct Reader {
  uint32_t at[KMAJOR ? W / 32 : BK / 16];
  __device__ Reader(int first, int lane) {
    if constexpr (!KMAJOR) {
      constexpr int chunks = BK / 8;
      const int r = first + (lane & 31);
#pragma unroll
      for (int kk = 0; kk < BK / 16; ++kk)
        at[kk] = (uint32_t)(r * (BK * 2) + (((kk * 2 + (lane >> 5)) ^ (r / (16 / chunks) % chunks)) << 4));
    } else {
      const int g = lane >> 4, i = lane & 15;
      const int k = 8 * (g >> 1) + i / 4;
      const int c = first / 8 + (g & 1) * 2 + ((i & 3) >> 1);
#pragma unroll
      for (int t = 0; t < W / 32; ++t)
        at[t] = (uint32_t)(k * (SPAN * 2) + (((c + 4 * t) ^ ((i / 4) * 4)) << 4) + (i & 1) * 8);
    }
  }
  // rows [32 t, 32 t + 32) of the wavefront's span, k [16 kk, 16 kk + 16)
  __device__ __forceinline__ s16x8 get(const char* lds, int t, int kk) const {
    if constexpr (!KMAJOR) {
      return *reinterpret_cast<const s16x8*>(lds + at[kk] + t * (32 * BK * 2));
    } else {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const char* p = lds + at[t] + kk * 16 * (SPAN * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * (SPAN * 2)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

template <int TM, int TN, int WM, int WN, bool AK, bool BK_, bool F16>
struct Tile {
  static constexpr int WAVES = TM / WM * (TN / WN), THREADS = 64 * WAVES;
  static constexpr int MT = WM / 32, NT = WN / 32;
  static constexpr int STAGE = (TM + TN) * BK * 2, LDS = 2 * STAGE;
  static constexpr int LOADS = Stager<TM, WAVES, AK>::COUNT + Stager<TN, WAVES, BK_>::COUNT;  // a wavefront's, a stage

  static constexpr int STEP = BK;  // k of a step

  // Products over steps [s0, s1).
  static __device__ __forceinline__ void run(const Panel& A, int64_t m0, const Panel& B, int64_t n0, int s0, int s1,
                                             char* lds, f32x16 (&acc)[MT][NT]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (TN / WN), wn = wave % (TN / WN);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    Stager<TM, WAVES, AK> sa;
    Stager<TN, WAVES, BK_> sb;
    const Reader<TM, WM, AK> ra(wm * WM, lane);
    const Reader<TN, WN, BK_> rb(wn * WN, lane);
    sa.init(A, m0, (int64_t)s0 * BK, wave, lane);
    sb.init(B, n0, (int64_t)s0 * BK, wave, lane);
    const int total = s1 - s0;
    auto issue = [&](int stage) {
      if (sa.left < BK) sa.place(A, m0, wave, lane);
      if (sb.left < BK) sb.place(B, n0, wave, lane);
      char* to = lds + stage * STAGE;
      sa.issue(to, wave);
      sb.issue(to + TM * BK * 2, wave);
      sa.base += sa.step;
      sb.base += sb.step;
      sa.left -= BK;
      sb.left -= BK;
    };
    s16x8 fa[2][MT], fb[2][NT];
    auto read = [&](int stage, int kk) {
      const char* a = lds + stage * STAGE;
      const char* b = a + TM * BK * 2;
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[kk & 1][i] = ra.get(a, i, kk);
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[kk & 1][j] = rb.get(b, j, kk);
    };
    issue(0);
    if (total > 1) {
      issue(1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(0, 0);
    constexpr int KK = BK / 16;
    static_assert(KK % 2 == 0, "a stage's first fragments go to the same registers");
    for (int s = 0; s < total; ++s) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) {
          read(s & 1, kk + 1);
        } else if (s + 1 < total) {
          // the next stage has arrived, and this one's reads are done in every
          // wavefront once all are here: it takes the loads after the next's
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          read((s + 1) & 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);  // reads first: they return under the products
        if (kk + 1 == KK && s + 2 < total) issue(s & 1);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma<F16>(fa[kk & 1][i], fb[kk & 1][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // m and n of register r of acc[i][j] within the tile
  static __device__ __forceinline__ int row(int i, int r) {
    const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / (TN / WN);
    return wm * WM + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
  }
  static __device__ __forceinline__ int col(int j) {
    const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) % (TN / WN);
    return wn * WN + j * 32 + (lane & 31);
  }
};

// ------------------------------------------------------------ fp32 products

// An fp32 operand is three bf16 planes (x = x0 + x1 + x2 exactly), laid out
// [row][column / 16][plane][16], so that 16 columns of all planes are 96
// contiguous bytes in either reading.  Of the nine products of planes the six
// that are not below fp32's own rounding are added, small ones first.  A stage
// holds 16 k of all three planes: every byte that comes to LDS takes part in
// two products on average, which halves the loads and LDS reads of six
// separate products (scores of 4099 x 30011, 256 columns: 337 us, 187 TFLOP/s of
// fp32; 394 as six passes over the planes; a library's fp32 product reaches 153
// on large squares).

// One operand's share of a stage: SPAN x 16 x 3 planes, 6 SPAN chunks.
template <int SPAN, int WAVES, bool KMAJOR>
struct Stager3 {
  static constexpr int TOTAL = SPAN * 6 / 64, COUNT = (TOTAL + WAVES - 1) / WAVES;
  const char* base;
  int64_t step, ld2, left;
  uint32_t off[COUNT];

  // p.ld in 16-bit elements, p.rows and p.cols in rows and fp32 columns
  __device__ void init(const Panel& p, int64_t m0, int64_t k0, int wave, int lane) {
    const char* d = reinterpret_cast<const char*>(p.data);
    ld2 = p.ld * 2;
    base = d + (KMAJOR ? k0 * ld2 + m0 * 6 : m0 * ld2 + k0 * 6);
    step = KMAJOR ? 16 * ld2 : 96;
    left = (KMAJOR ? p.rows : p.cols) - k0;
    place(p, m0, wave, lane);
  }
  // As in Stager; k past the end of a K-contiguous row is there (zeros).
  __device__ void place(const Panel& p, int64_t m0, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const int i = part_of<TOTAL, WAVES>(j, wave) * 64 + lane;
      if constexpr (KMAJOR) {
        const int64_t last = (p.cols - m0) / 16 * 6 - 1;  // chunks there are
        const int r = i / (SPAN * 3 / 8), c = (i % (SPAN * 3 / 8)) ^ ((r & 3) * 4);
        off[j] = (uint32_t)((r < left ? r : left - 1) * ld2 + (c < last ? c : last) * 16);
      } else {
        const int64_t last = p.rows - 1 - m0;
        const int r = i / 6, c = (i % 6) ^ ((r >> 3) & 1);
        off[j] = (uint32_t)((r < last ? r : last) * ld2 + c * 16);
      }
    }
  }
};

template <int SPAN, int W, bool KMAJOR>
struct Reader3 {
  uint32_t at[KMAJOR ? W / 32 : 1];
  int odd;
  __device__ Reader3(int first, int lane) {
    if constexpr (!KMAJOR) {
      const int r = first + (lane & 31);  // (32 rows on: the same swap)
      odd = (r >> 3) & 1;
      at[0] = (uint32_t)(r * 96 + (((lane >> 5) ^ odd) << 4));
    } else {
      const int g = lane >> 4, i = lane & 15;
      odd = 0;
#pragma unroll
      for (int t = 0; t < W / 32; ++t)
        at[t] = (uint32_t)((8 * (g >> 1) + i / 4) * (SPAN * 6) + (i & 1) * 8) |
                (uint32_t)(((first + 32 * t) / 16 + (g & 1)) * 6 + ((i & 3) >> 1)) << 20;
    }
  }
  // rows [32 t, 32 t + 32) of the wavefront's span in one plane
  __device__ __forceinline__ s16x8 get(const char* lds, int t, int plane, int lane) const {
    if constexpr (!KMAJOR) {
      return *reinterpret_cast<const s16x8*>(lds + at[0] + t * (32 * 96) + plane * 32);
    } else {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const uint32_t c = (at[t] >> 20) + plane * 2;
      const char* p = lds + (at[t] & 0xfffff) + ((c ^ (((lane & 15) / 4) * 4)) << 4);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * (SPAN * 6)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

template <int TM, int TN, int WM, int WN, int STAGES, bool AK, bool BK_>
struct Tile3 {
  static constexpr int WAVES = TM / WM * (TN / WN), THREADS = 64 * WAVES;
  static constexpr int MT = WM / 32, NT = WN / 32;
  static constexpr int STAGE = (TM + TN) * 96, LDS = STAGES * STAGE;
  static constexpr int STEP = 16;
  static constexpr int LOADS = Stager3<TM, WAVES, AK>::COUNT + Stager3<TN, WAVES, BK_>::COUNT;

  static __device__ __forceinline__ void run(const Panel& A, int64_t m0, const Panel& B, int64_t n0, int s0, int s1,
                                             char* lds, f32x16 (&acc)[MT][NT]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (TN / WN), wn = wave % (TN / WN);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    Stager3<TM, WAVES, AK> sa;
    Stager3<TN, WAVES, BK_> sb;
    const Reader3<TM, WM, AK> ra(wm * WM, lane);
    const Reader3<TN, WN, BK_> rb(wn * WN, lane);
    sa.init(A, m0, (int64_t)s0 * STEP, wave, lane);
    sb.init(B, n0, (int64_t)s0 * STEP, wave, lane);
    const int total = s1 - s0;
    auto issue = [&](int stage) {
      if constexpr (AK)
        if (sa.left < STEP) sa.place(A, m0, wave, lane);
      if constexpr (BK_)
        if (sb.left < STEP) sb.place(B, n0, wave, lane);
      char* to = lds + stage * STAGE;
      load_parts<sa.TOTAL, WAVES>(sa.base, sa.off, to, wave);
      load_parts<sb.TOTAL, WAVES>(sb.base, sb.off, to + TM * 96, wave);
      sa.base += sa.step;
      sb.base += sb.step;
      sa.left -= STEP;
      sb.left -= STEP;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
      if (s < total) issue(s);
    int cur = 0;
    for (int s = 0; s < total; ++s) {
      // this step's loads are the oldest ones; the reads of the step before
      // are done before any wavefront overwrites their stage
      if (s + STAGES - 2 < total) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS * (STAGES - 2)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const char* a = lds + cur * STAGE;
      const char* b = a + TM * 96;
      s16x8 fa[3][MT], fb[3][NT];
      // in the order of their use
      auto read = [&](int p, int q) {
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[p][i] = ra.get(a, i, p, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[q][j] = rb.get(b, j, q, lane);
      };
      auto multiply = [&](int p, int q) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma<false>(fa[p][i], fb[q][j], acc[i][j]);
      };
      read(2, 0);
      read(0, 2);
      __builtin_amdgcn_sched_barrier(0);
      if (s + STAGES - 1 < total) issue(cur == 0 ? STAGES - 1 : cur - 1);
      multiply(2, 0);
      __builtin_amdgcn_sched_barrier(0);
      read(1, 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, 2);
      multiply(1, 1);
      multiply(1, 0);
      multiply(0, 1);
      multiply(0, 0);
      cur = cur == STAGES - 1 ? 0 : cur + 1;
    }
  }

  // m and n of register r of acc[i][j] within the tile
  static __device__ __forceinline__ int row(int i, int r) {
    const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 6) / (TN / WN);
    return wm * WM + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
  }
  static __device__ __forceinline__ int col(int j) {
    const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) % (TN / WN);
    return wn * WN + j * 32 + (lane & 31);
  }
};

// Workgroups go round-robin to the 8 XCDs: give each XCD one run of tiles, in
// groups of `group` rows by all columns, so that its L2 sees the same panels
// again.  b of total -> (y, x) in a grid of ny by nx.
__device__ __forceinline__ void place_tile(int64_t b, int64_t ny, int64_t nx, int group, int64_t& y, int64_t& x) {
  const int64_t total = ny * nx, per = total / 8, more = total % 8, xcd = b % 8;
  const int64_t id = xcd * per + (xcd < more ? xcd : more) + b / 8;
  const int64_t band = id / (group * nx), first = band * group;
  const int64_t high = ny - first < group ? ny - first : group, in = id - band * group * nx;
  y = first + in % high;
  x = in / high;
}

}  // namespace
}  // namespace kern
}  // namespace aires
