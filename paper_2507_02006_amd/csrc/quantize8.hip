// Matrices held in 8 bits: e4m3 codes with a scale for 128 values of a row or
// for 128 x 128 values, as the matrix lies and transposed (gfx950).
//
// Per block: scale = max |x| / 448, code = x (448 / max |x|) to nearest even.
// Every value is read once and each code written once, for about a dozen
// operations a value and order: bound by bytes.
//
// As it lies with scales for each row: 16 lanes hold a block, a workgroup 128 blocks
// that follow each other in memory, so a block's maximum is four lane exchanges.
// Else a workgroup holds a tile of 128 x 128 in registers, a thread 8 rows by 8
// columns of it: 16 lanes hold a row of the tile, so a row's maximum is four lane
// exchanges, and a column's is the thread's own, two lane exchanges and one
// exchange between the four wavefronts.  Both orders come from one read of the
// matrix.  The transposed codes go through LDS, eight of a column at a time,
// their place exchanged with the column's number against bank conflicts, and are
// written as rows of 128 bytes.
//
// Measured, X in bf16: 65536 x 1000, scales along rows, both orders 56 us (4.8 TB/s); 16384 x
// 4096 as it lies 36 us (5.6 TB/s), 128 x 128 scales, both orders, 50 us (5.4 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "layers.h"
#include "rows8.h"

namespace aires {
namespace kern {
namespace {

constexpr int BLOCK = 256;

struct Args {
  const void* x; int64_t ldx; int xt;
  int64_t m, n;
  Held q, t;
};

// Magnitudes of a row's eight values as integers of the same order (signs cut
// off): packed pairs of 16-bit ones, or eight of 32 bits.  What is not finite is
// above all others.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

template <bool HALF>
struct Sizes {
  uint32_t v[HALF ? 4 : 8] = {};

  template <typename R>
  __device__ __forceinline__ void add(const R& r) {
    if constexpr (HALF) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v[k]),
                                                                      __builtin_bit_cast(u16x2, r.lo[k] & 0x7fff7fffu)));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = max(v[k], r.lo[k] & 0x7fffffffu);
        v[k + 4] = max(v[k + 4], r.hi[k] & 0x7fffffffu);
      }
    }
  }
  // value k's, as an integer
  __device__ __forceinline__ uint32_t bits(int k) const {
    if constexpr (HALF) return v[k / 2] >> (16 * (k & 1)) & 0xffffu;
    else return v[k];
  }
  __device__ __forceinline__ uint32_t most() const {
    uint32_t m = bits(0);
#pragma unroll
    for (int k = 1; k < 8; ++k) m = max(m, bits(k));
    return m;
  }
};

template <bool HALF>
__device__ __forceinline__ bool is_finite(uint32_t bits, int t) {
  return bits < (!HALF ? 0x7f800000u : t == DT_BF16 ? 0x7f80u : 0x7c00u);
}
template <bool HALF>
__device__ __forceinline__ float size_of(uint32_t bits, int t) {
  if constexpr (!HALF) return __uint_as_float(bits);
  return t == DT_BF16 ? bf16_to_f32((uint16_t)bits) : f16_to_f32((uint16_t)bits);
}

// Largest finite magnitude of a row's eight values.
template <bool HALF, typename R>
__device__ __forceinline__ float magnitude(const R& r, int t) {
  Sizes<HALF> z;
  z.add(r);
  const uint32_t most = z.most();
  if (is_finite<HALF>(most, t)) return size_of<HALF>(most, t);
  float x[8], big = 0.f;
  convert(r, t, x);
#pragma unroll
  for (int k = 0; k < 8; ++k) big = fmaxf(big, finite_abs(x[k]));
  return big;
}

// Largest value over the wavefront's lanes that hold the same columns.
__device__ __forceinline__ float max_over_rows(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// ROWS, COLUMNS: which orders are written; TILES: one scale a tile; T: X's
// type.  A value that is not finite is NaN or an infinity after its product
// with the inverse scale too, and the conversion makes both NaN.
template <bool ROWS, bool COLUMNS, bool TILES, int T>
__global__ __launch_bounds__(BLOCK) void k_quantize(Args a) {
  typedef Raw<T> Raw;
  constexpr bool HALF = T == DT_BF16 || T == DT_F16;
  const int xt = T == MIXED ? (int)DT_F32 : T, n8 = row_of<T>((int)a.n);  // (MIXED: made fp32 below)
  __shared__ float big_of[BLOCK / 64][BLOCK8];
  __shared__ float inverse_of[BLOCK8];
  __shared__ uint64_t turned[COLUMNS ? BLOCK8 * 16 : 1];
  const int j = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int64_t wide = (a.n + BLOCK8 - 1) / BLOCK8, tiles = (a.m + BLOCK8 - 1) / BLOCK8 * wide;
  for (int64_t id = blockIdx.x; id < tiles; id += gridDim.x) {
    // workgroups go round-robin to the 8 XCDs: each gets a run of tiles, whose
    // neighbours share lines where rows are no multiples of 128 bytes
    const int64_t per = tiles / 8, at = id < per * 8 ? id % 8 * per + id / 8 : id;
    const int64_t r0 = at / wide * BLOCK8, c0 = at % wide * BLOCK8;
    const int64_t row = r0 + g * 8, col = c0 + j * 8;
    Raw x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)  // (rows past the last: the last again)
      load_raw<true>(a.x, type_of<T>(a.xt), (row + i < a.m ? row + i : a.m - 1) * a.ldx + col, (int)(a.n - col), n8, x[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      settle(x[i], type_of<T>(a.xt), (int)(a.n - col), n8);
      if constexpr (T == MIXED) {
        float v[8];
        convert(x[i], a.xt, v);
        pack(v, DT_F32, x[i]);
      }
      if (row + i >= a.m) x[i] = Raw{};
    }
    float big[8] = {}, inv_tile = 0.f;
    if constexpr (TILES || COLUMNS) {
      Sizes<HALF> z;
#pragma unroll
      for (int i = 0; i < 8; ++i) z.add(x[i]);
#pragma unroll
      for (int k = 0; k < 8; ++k) big[k] = size_of<HALF>(z.bits(k), xt);
      if (!is_finite<HALF>(z.most(), xt)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) big[k] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v[8];
          convert(x[i], xt, v);
#pragma unroll
          for (int k = 0; k < 8; ++k) big[k] = fmaxf(big[k], finite_abs(v[k]));
        }
      }
    }
    if constexpr (TILES) {
      float most = big[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) most = fmaxf(most, big[k]);
      most = max_over_rows(group16_max_f32(most));
      if ((threadIdx.x & 63) == 0) big_of[wave][0] = most;
      __syncthreads();
      most = fmaxf(fmaxf(big_of[0][0], big_of[1][0]), fmaxf(big_of[2][0], big_of[3][0]));
      float scale;
      block_scale(most, scale, inv_tile);
      if (threadIdx.x == 0) {
        if (ROWS) a.q.scales[r0 / BLOCK8 * a.q.lds + c0 / BLOCK8] = scale;
        if (COLUMNS) a.t.scales[c0 / BLOCK8 * a.t.lds + r0 / BLOCK8] = scale;
      }
    } else if constexpr (COLUMNS) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float most = max_over_rows(big[k]);
        if ((threadIdx.x & 63) < 16) big_of[wave][j * 8 + k] = most;
      }
      __syncthreads();
      if (threadIdx.x < BLOCK8) {
        const int c = threadIdx.x;
        float scale, inv;
        block_scale(fmaxf(fmaxf(big_of[0][c], big_of[1][c]), fmaxf(big_of[2][c], big_of[3][c])), scale, inv);
        inverse_of[c] = inv;
        if (c0 + c < a.n) a.t.scales[(c0 + c) * a.t.lds + r0 / BLOCK8] = scale;
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) made_again(x[i]);
    if constexpr (ROWS) {
      // eight of the 16 lanes of a row make the quotients of its eight rows
      float inverse = 0.f;
      if constexpr (!TILES) {
        float mine = 0.f, scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float most = group16_max_f32(magnitude<HALF>(x[i], xt));
          mine = (j & 7) == i ? most : mine;
        }
        block_scale(mine, scale, inverse);
        if (j < 8 && row + j < a.m) a.q.scales[(row + j) * a.q.lds + c0 / BLOCK8] = scale;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) made_again(x[i]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
        convert(x[i], xt, v);
        const float inv = TILES ? inv_tile : __shfl(inverse, (threadIdx.x & 48) + i);
        u32x2_el1 w;
        w[0] = encode4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        w[1] = encode4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
        if (row + i < a.m) {
          uint8_t* to = a.q.codes + (row + i) * a.q.ld + col;
          if (col + 8 <= a.n) {
            *reinterpret_cast<u32x2_el1*>(to) = w;
          } else {
#pragma unroll
            for (int k = 0; k < 7; ++k)
              if (col + k < a.n) to[k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
          }
        }
      }
    }
    if constexpr (ROWS && COLUMNS)
#pragma unroll
      for (int i = 0; i < 8; ++i) made_again(x[i]);
    if constexpr (COLUMNS) {
      // rows of four at a time: their codes of each column are one word
      uint32_t word[2][8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) convert(x[h * 4 + i], xt, v[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float inv = TILES ? inv_tile : inverse_of[j * 8 + k];
          word[h][k] = encode4(v[0][k] * inv, v[1][k] * inv, v[2][k] * inv, v[3][k] * inv);
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) turned[(j * 8 + k) * 16 + (g ^ j)] = (uint64_t)word[1][k] << 32 | word[0][k];
      __syncthreads();
      // 16 lanes write the 128 codes of a column
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = i * 16 + g;
        const int64_t to_row = c0 + c, to_col = r0 + j * 8;
        if (to_row >= a.n || to_col >= a.m) continue;
        const uint64_t w = turned[c * 16 + (j ^ (c >> 3))];
        uint8_t* to = a.t.codes + to_row * a.t.ld + to_col;
        if (to_col + 8 <= a.m) {
          *reinterpret_cast<u32x2_el1*>(to) = u32x2_el1{(uint32_t)w, (uint32_t)(w >> 32)};
        } else {
#pragma unroll
          for (int k = 0; k < 7; ++k)
            if (to_col + k < a.m) to[k] = (uint8_t)(w >> (8 * k));
        }
      }
    }
    if constexpr (TILES || COLUMNS) __syncthreads();  // the next tile overwrites what is shared
  }
}

// X as it lies, a scale for each block of a row.  (The tiles' kernel, whose
// reads are runs of 256 bytes, took 54 us for 65536 x 1000 in bf16, this 35.)
template <int T>
__global__ __launch_bounds__(BLOCK) void k_quantize_rows(Args a) {
  const int lane = threadIdx.x & 63, j = threadIdx.x & 15, g = threadIdx.x >> 4, n8 = row_of<T>((int)a.n);
  const int64_t wide = (a.n + BLOCK8 - 1) / BLOCK8, blocks = a.m * wide;
  const int64_t rows16 = 16 / wide, rest16 = 16 % wide;  // 16 blocks on
  for (int64_t at = (int64_t)blockIdx.x * 128 + g; at - g < blocks; at += (int64_t)gridDim.x * 128) {
    int64_t row = at / wide, block = at % wide, to[8];
    Raw<T> x[8];
    float mine = 0.f, scale, inverse;
    int have[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t col = block * BLOCK8 + j * 8;
      const bool in = row < a.m;
      to[i] = in ? row * a.q.ld + col : -1;
      have[i] = (int)(a.n - col);
      load_raw<true>(a.x, type_of<T>(a.xt), (in ? row : a.m - 1) * a.ldx + col, have[i], n8, x[i]);
      row += rows16;
      block += rest16;
      if (block >= wide) {
        block -= wide;
        ++row;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      settle(x[i], type_of<T>(a.xt), have[i], n8);
      if constexpr (T == MIXED) {
        float v[8];
        convert(x[i], a.xt, v);
        pack(v, DT_F32, x[i]);
      }
      const float most = group16_max_f32(magnitude<T == DT_BF16 || T == DT_F16>(x[i], T == MIXED ? (int)DT_F32 : T));
      mine = (j & 7) == i ? most : mine;
    }
    // eight of the 16 lanes make the quotients of the group's eight blocks
    block_scale(mine, scale, inverse);
    const int64_t own = at + (j & 7) * 16;
    if (j < 8 && own < blocks) a.q.scales[own / wide * a.q.lds + own % wide] = scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) made_again(x[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[8];
      convert(x[i], T == MIXED ? (int)DT_F32 : T, v);
      const float inv = __shfl(inverse, (lane & 48) + i);
      u32x2_el1 w;
      w[0] = encode4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      w[1] = encode4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
      if (to[i] < 0) continue;
      if (have[i] >= 8) {
        *reinterpret_cast<u32x2_el1*>(a.q.codes + to[i]) = w;
      } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
          if (k < have[i]) a.q.codes[to[i] + k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
      }
    }
  }
}

}  // namespace

hipError_t quantize8(const Mat& X, const Held& Q, const Held& Qt, hipStream_t s) {
  if (X.rows == 0 || X.cols == 0 || (!Q.codes && !Qt.codes)) return hipSuccess;
  Args a{X.data, X.ld, X.type, X.rows, X.cols, Q, Qt};
  const int64_t tiles = (X.rows + BLOCK8 - 1) / BLOCK8 * ((X.cols + BLOCK8 - 1) / BLOCK8);
  const dim3 grid((unsigned)std::min<int64_t>(tiles, 1 << 20));
  const bool many = (Q.codes ? Q.tile : Qt.tile) == BLOCK8;
  const auto orders = [&](auto tiles, auto type) {
    constexpr bool M = decltype(tiles)::value;
    constexpr int T = decltype(type)::value;
    if (Q.codes && Qt.codes) {
      k_quantize<true, true, M, T><<<grid, BLOCK, 0, s>>>(a);
    } else if (Q.codes) {
      if constexpr (M) k_quantize<true, false, M, T><<<grid, BLOCK, 0, s>>>(a);
      else k_quantize_rows<T><<<(unsigned)std::min<int64_t>((X.rows * ((X.cols + BLOCK8 - 1) / BLOCK8) + 127) / 128, 1 << 20), BLOCK, 0, s>>>(a);
    } else k_quantize<false, true, M, T><<<grid, BLOCK, 0, s>>>(a);
  };
  const auto typed = [&](auto tiles) {
    if (X.cols < 8) orders(tiles, std::integral_constant<int, MIXED>());
    else if (X.type == DT_F32) orders(tiles, std::integral_constant<int, DT_F32>());
    else if (X.type == DT_BF16) orders(tiles, std::integral_constant<int, DT_BF16>());
    else orders(tiles, std::integral_constant<int, DT_F16>());
  };
  if (many) typed(std::true_type());
  else typed(std::false_type());
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
