// Rows of dense arrays held in registers, eight columns a lane and chunk, and
// blocks of 8-bit codes with a scale (gfx950, wave64).
//
// A chunk of a row is loaded as it lies (one 16-byte load of 16-bit values, two
// of fp32) and converted at its use, so that the loads of several arrays are all
// on their way before the first is waited for.
#pragma once
#include <type_traits>

#include "dense.h"
#include "device.h"

namespace aires {
namespace kern {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_el4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_el2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_el1 __attribute__((ext_vector_type(2), aligned(1)));

// A kernel is built for one type of its rows, so that what it loads and stores is
// counted at build time and nothing is waited for but what is used (MIXED: types
// are looked at as it runs, and rows may have fewer than eight values).
constexpr int MIXED = 3;
template <int T>
__device__ __forceinline__ constexpr int type_of(int t) { return T == MIXED ? t : T; }
template <int T>
__device__ __forceinline__ constexpr int row_of(int n) { return T == MIXED ? n : 8; }

// Eight values as they lie: 32-bit ones in both words, 16-bit ones in lo.
struct Raw8 {
  u32x4 lo, hi;
};

// The same where every type is of 16 bits: half the registers, so that more loads
// can be on their way.
struct Raw8Half {
  u32x4 lo;
};

template <int T>
using Raw = std::conditional_t<T == DT_BF16 || T == DT_F16, Raw8Half, Raw8>;

// Values [i, i + 8) of p in two steps: the load, and settle() where they are used.
// `have` is how many there are from i on, `n` how many in the whole row.  A chunk
// that passes the row's end is loaded moved back to the last eight, so that every
// lane makes the same load whatever its columns, and no load waits for another;
// settle() moves the values to their places and fills up with zeros.
template <bool ONCE = false>
__device__ __forceinline__ void load_raw(const void* p, int t, int64_t i, int have, int n, Raw8& r) {
  if (n >= 8) {
    i += have < 8 ? have - 8 : 0;
    if (t == DT_F32) {
      const uint32_t* q = static_cast<const uint32_t*>(p) + i;
      r.lo = load_vec<ONCE>(reinterpret_cast<const u32x4_el4*>(q));
      r.hi = load_vec<ONCE>(reinterpret_cast<const u32x4_el4*>(q + 4));
    } else {
      r.lo = load_vec<ONCE>(reinterpret_cast<const u32x4_el2*>(static_cast<const uint16_t*>(p) + i));
    }
  } else {  // (a row that has no eight values)
    r.lo = r.hi = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < have) {
        if (t == DT_F32) {
          if (k < 4) r.lo[k] = static_cast<const uint32_t*>(p)[i + k];
          else r.hi[k - 4] = static_cast<const uint32_t*>(p)[i + k];
        } else {
          r.lo[k / 2] |= (uint32_t)static_cast<const uint16_t*>(p)[i + k] << (16 * (k & 1));
        }
      }
  }
}

template <bool ONCE = false>
__device__ __forceinline__ void load_raw(const void* p, int, int64_t i, int have, int n, Raw8Half& r) {
  Raw8 x;
  load_raw<ONCE>(p, DT_F16, i, have, n, x);
  r.lo = x.lo;
}

// Words moved down by `by` halves of a word, zeros after them.
__device__ __forceinline__ void move_halves(u32x4& w, int by) {
  uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
  if (by >= 4) {
    lo = hi;
    hi = 0;
    by -= 4;
  }
  const int bits = by * 16;
  lo = by >= 4 ? 0 : bits == 0 ? lo : lo >> bits | hi << (64 - bits);
  hi = by >= 4 ? 0 : hi >> bits;
  w = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

__device__ __forceinline__ void settle(Raw8& r, int t, int have, int n) {
  const int by = have < 0 ? 8 : 8 - have;
  if (n < 8 || !__any(by > 0)) return;
  if (by <= 0) return;
  if (t == DT_F32) {
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = r.lo[k];
      w[k + 4] = r.hi[k];
    }
#pragma unroll
    for (int s = 1; s < 8; s *= 2)
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = by & s ? (k + s < 8 ? w[k + s < 8 ? k + s : 0] : 0) : w[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r.lo[k] = by >= 8 ? 0 : w[k];
      r.hi[k] = by >= 8 ? 0 : w[k + 4];
    }
  } else {
    move_halves(r.lo, by);
  }
}

__device__ __forceinline__ void settle(Raw8Half& r, int, int have, int n) {
  const int by = have < 0 ? 8 : 8 - have;
  if (n < 8 || !__any(by > 0)) return;
  if (by > 0) move_halves(r.lo, by);
}

__device__ __forceinline__ void convert(const Raw8& r, int t, float (&x)[8]) {
  if (t == DT_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = __uint_as_float(r.lo[k]);
      x[k + 4] = __uint_as_float(r.hi[k]);
    }
  } else if (t == DT_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(r.lo[k] << 16);
      x[2 * k + 1] = __uint_as_float(r.lo[k] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = f16_to_f32((uint16_t)r.lo[k]);
      x[2 * k + 1] = f16_to_f32((uint16_t)(r.lo[k] >> 16));
    }
  }
}

// x in the words of type t (one rounding, to nearest even).
__device__ __forceinline__ void pack(const float (&x)[8], int t, Raw8& r) {
  if (t == DT_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r.lo[k] = __float_as_uint(x[k]);
      r.hi[k] = __float_as_uint(x[k + 4]);
    }
  } else if (t == DT_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r.lo[k] = f32_to_bf16(x[2 * k]) | (uint32_t)f32_to_bf16(x[2 * k + 1]) << 16;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) r.lo[k] = f32_to_f16(x[2 * k]) | (uint32_t)f32_to_f16(x[2 * k + 1]) << 16;
  }
}

__device__ __forceinline__ void convert(const Raw8Half& r, int t, float (&x)[8]) {
  convert(Raw8{r.lo, r.lo}, t == DT_F16 ? (int)DT_F16 : (int)DT_BF16, x);
}

template <bool ONCE = false>
__device__ __forceinline__ void store_raw(void* p, int t, int64_t i, int64_t have, const Raw8& r) {
  if (have <= 0) return;
  if (t == DT_F32) {
    uint32_t* q = static_cast<uint32_t*>(p) + i;
    if (have >= 8) {
      store_vec<ONCE>(reinterpret_cast<u32x4_el4*>(q), (u32x4_el4)r.lo);
      store_vec<ONCE>(reinterpret_cast<u32x4_el4*>(q + 4), (u32x4_el4)r.hi);
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < have) q[k] = k < 4 ? r.lo[k] : r.hi[k - 4];
    }
  } else {
    uint16_t* q = static_cast<uint16_t*>(p) + i;
    if (have >= 8) {
      store_vec<ONCE>(reinterpret_cast<u32x4_el2*>(q), (u32x4_el2)r.lo);
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < have) q[k] = (uint16_t)(r.lo[k / 2] >> (16 * (k & 1)));
    }
  }
}

__device__ __forceinline__ void pack(const float (&x)[8], int t, Raw8Half& r) {
  Raw8 w;
  pack(x, t == DT_F16 ? (int)DT_F16 : (int)DT_BF16, w);
  r.lo = w.lo;
}
template <bool ONCE = false>
__device__ __forceinline__ void store_raw(void* p, int, int64_t i, int64_t have, const Raw8Half& r) {
  store_raw<ONCE>(p, DT_F16, i, have, Raw8{r.lo, r.lo});
}

// The words as if read anew: what was made of them before is made again rather
// than kept in registers.
__device__ __forceinline__ void made_again(Raw8& r) { asm volatile("" : "+v"(r.lo), "+v"(r.hi)); }
__device__ __forceinline__ void made_again(Raw8Half& r) { asm volatile("" : "+v"(r.lo)); }

// Matrices held in 8 bits: runs of BLOCK8 values of a row share a scale.
constexpr int BLOCK8 = 128;
constexpr float TOP8 = 448.f;       // largest e4m3 number
constexpr float TINY8 = 0x1p-110f;  // a block with no larger value is held as zeros

__device__ __forceinline__ bool finite_f32(float x) { return fabsf(x) <= 3.402823466e38f; }

__device__ __forceinline__ float finite_abs(float x) { return finite_f32(x) ? fabsf(x) : 0.f; }

// A block's scale, and what its values are multiplied with, from its largest
// finite magnitude.
__device__ __forceinline__ void block_scale(float big, float& scale, float& inverse) {
  const bool used = big >= TINY8;
  scale = used ? big / TOP8 : 0.f;
  inverse = used ? TOP8 / big : 0.f;
}

// A value times its block's inverse scale, NaN if it was not finite (a block of
// zeros holds no finite value to multiply).
__device__ __forceinline__ float scaled(float x, float inverse) {
  return finite_f32(x) ? x * inverse : __uint_as_float(0x7fc00000u);
}

// Four values to codes, the first in the lowest byte, to nearest even.  In units
// of its scale a value is at most 448 (1 + 2^-22), which rounds to 448.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}

}  // namespace
}  // namespace kern
}  // namespace aires
