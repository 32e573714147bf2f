// Matrices held in 8 bits: e4m3 codes with a scale for 128 values of a row or
// for 128 x 128 values, as the matrix lies and transposed (gfx950).
//
// Per block: scale = max |x| / 448, code = x (448 / max |x|) to nearest even.
// Every value is read once and each code written once, for about a dozen
// operations a value and order: bound by bytes.
//
// A workgroup holds a tile of 128 x 128 in registers, a thread 8 rows by 8
// columns of it: 16 lanes hold a row of the tile, so a row's maximum is four lane
// exchanges, and a column's is the thread's own, two lane exchanges and one
// exchange between the four wavefronts.  Both orders come from one read of the
// matrix.  The transposed codes go through LDS, eight of a column at a time,
// their place exchanged with the column's number against bank conflicts, and are
// written as rows of 128 bytes.
#include <hip/hip_runtime.h>

#include <algorithm>

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

__device__ __forceinline__ float magnitude(const float (&x)[8]) {
  float big = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) big = fmaxf(big, finite_abs(x[k]));
  return big;
}

// Largest value over the wavefront's lanes that hold the same columns.
__device__ __forceinline__ float max_over_rows(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// ROWS, COLUMNS: which orders are written; TILES: one scale a tile.
template <bool ROWS, bool COLUMNS, bool TILES>
__global__ __launch_bounds__(BLOCK) void k_quantize(Args a) {
  __shared__ float big_of[BLOCK / 64][BLOCK8];
  __shared__ float inverse_of[BLOCK8];
  __shared__ uint64_t turned[COLUMNS ? BLOCK8 * 16 : 1];
  const int j = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int64_t wide = (a.n + BLOCK8 - 1) / BLOCK8, tiles = (a.m + BLOCK8 - 1) / BLOCK8 * wide;
  for (int64_t at = blockIdx.x; at < tiles; at += gridDim.x) {
    const int64_t r0 = at / wide * BLOCK8, c0 = at % wide * BLOCK8;
    const int64_t row = r0 + g * 8, col = c0 + j * 8;
    Raw8 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) load_raw<true>(a.x, a.xt, (row + i) * a.ldx + col, row + i < a.m ? a.n - col : 0, x[i]);
    float big[8] = {}, inv_tile = 0.f;
    if constexpr (TILES || COLUMNS) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
        convert(x[i], a.xt, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) big[k] = fmaxf(big[k], finite_abs(v[k]));
      }
    }
    if constexpr (TILES) {
      float most = max_over_rows(group16_max_f32(magnitude(big)));
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
    if constexpr (ROWS) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8], inv = inv_tile;
        convert(x[i], a.xt, v);
        if constexpr (!TILES) {
          float scale;
          block_scale(group16_max_f32(magnitude(v)), scale, inv);
          if (j == 0 && row + i < a.m) a.q.scales[(row + i) * a.q.lds + c0 / BLOCK8] = scale;
        }
        u32x2_el1 w;
        w[0] = encode4(scaled(v[0], inv), scaled(v[1], inv), scaled(v[2], inv), scaled(v[3], inv));
        w[1] = encode4(scaled(v[4], inv), scaled(v[5], inv), scaled(v[6], inv), scaled(v[7], inv));
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
    if constexpr (COLUMNS) {
      // rows of four at a time: their codes of each column are one word
      uint32_t word[2][8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) convert(x[h * 4 + i], a.xt, v[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float inv = TILES ? inv_tile : inverse_of[j * 8 + k];
          word[h][k] = encode4(scaled(v[0][k], inv), scaled(v[1][k], inv), scaled(v[2][k], inv), scaled(v[3][k], inv));
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

}  // namespace

hipError_t quantize8(const Mat& X, const Held& Q, const Held& Qt, hipStream_t s) {
  if (X.rows == 0 || X.cols == 0 || (!Q.codes && !Qt.codes)) return hipSuccess;
  Args a{X.data, X.ld, X.type, X.rows, X.cols, Q, Qt};
  const int64_t tiles = (X.rows + BLOCK8 - 1) / BLOCK8 * ((X.cols + BLOCK8 - 1) / BLOCK8);
  const dim3 grid((unsigned)std::min<int64_t>(tiles, 1 << 20));
  const bool many = (Q.codes ? Q.tile : Qt.tile) == BLOCK8;
  if (Q.codes && Qt.codes) {
    if (many) k_quantize<true, true, true><<<grid, BLOCK, 0, s>>>(a);
    else k_quantize<true, true, false><<<grid, BLOCK, 0, s>>>(a);
  } else if (Q.codes) {
    if (many) k_quantize<true, false, true><<<grid, BLOCK, 0, s>>>(a);
    else k_quantize<true, false, false><<<grid, BLOCK, 0, s>>>(a);
  } else {
    if (many) k_quantize<false, true, true><<<grid, BLOCK, 0, s>>>(a);
    else k_quantize<false, true, false><<<grid, BLOCK, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
