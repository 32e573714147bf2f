// Rows of dense arrays held in registers, eight columns a lane and chunk, and
// blocks of 8-bit codes with a scale (gfx950, wave64).
//
// A chunk of a row is loaded as it lies (one 16-byte load of 16-bit values, two
// of fp32) and converted at its use, so that the loads of several arrays are all
// on their way before the first is waited for.
#pragma once
#include "dense.h"
#include "device.h"

namespace aires {
namespace kern {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_el4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_el2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_el1 __attribute__((ext_vector_type(2), aligned(1)));

// Eight values as they lie: 32-bit ones in both words, 16-bit ones in lo.
struct Raw8 {
  u32x4 lo, hi;
};

// Values [i, i + 8) of p, of which the first `have` are there (others: 0).
template <bool ONCE = false>
__device__ __forceinline__ void load_raw(const void* p, int t, int64_t i, int64_t have, Raw8& r) {
  r.lo = r.hi = u32x4{0, 0, 0, 0};
  if (t == DT_F32) {
    const uint32_t* q = static_cast<const uint32_t*>(p) + i;
    if (have >= 8) {
      r.lo = load_vec<ONCE>(reinterpret_cast<const u32x4_el4*>(q));
      r.hi = load_vec<ONCE>(reinterpret_cast<const u32x4_el4*>(q + 4));
    } else if (have > 0) {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < have) {
          if (k < 4) r.lo[k] = q[k];
          else r.hi[k - 4] = q[k];
        }
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + i;
    if (have >= 8) {
      r.lo = load_vec<ONCE>(reinterpret_cast<const u32x4_el2*>(q));
    } else if (have > 0) {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < have) r.lo[k / 2] |= (uint32_t)q[k] << (16 * (k & 1));
    }
  }
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
