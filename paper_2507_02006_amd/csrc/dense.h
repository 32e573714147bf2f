// Device helpers for dense arrays of fp32, bf16 and fp16 (gfx950, wave64).
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aires {
namespace kern {

enum DType : int { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };  // aires_dtype

__host__ __device__ constexpr int dtype_bytes(int t) { return t == DT_F32 ? 4 : 2; }

namespace {

// Four values at the alignment of one: global memory takes 8- and 16-byte
// accesses at any element boundary, so rows need no alignment of their own.
typedef float f32x4_el __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_el __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_to_f32(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
__device__ __forceinline__ float f16_to_f32(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
__device__ __forceinline__ uint16_t f32_to_bf16(float x) {  // to nearest even
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ uint16_t f32_to_f16(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

template <int T>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  if constexpr (T == DT_F32) return static_cast<const float*>(p)[i];
  const uint16_t u = static_cast<const uint16_t*>(p)[i];
  return T == DT_BF16 ? bf16_to_f32(u) : f16_to_f32(u);
}

template <int T>
__device__ __forceinline__ void store1(void* p, int64_t i, float x) {
  if constexpr (T == DT_F32) static_cast<float*>(p)[i] = x;
  else static_cast<uint16_t*>(p)[i] = T == DT_BF16 ? f32_to_bf16(x) : f32_to_f16(x);
}

__device__ __forceinline__ float load1(const void* p, int t, int64_t i) {
  return t == DT_F32 ? load1<DT_F32>(p, i) : t == DT_BF16 ? load1<DT_BF16>(p, i) : load1<DT_F16>(p, i);
}

__device__ __forceinline__ void store1(void* p, int t, int64_t i, float x) {
  if (t == DT_F32) store1<DT_F32>(p, i, x);
  else if (t == DT_BF16) store1<DT_BF16>(p, i, x);
  else store1<DT_F16>(p, i, x);
}

// ONCE: the value is not needed again soon; it does not push others out of
// the caches.
template <bool ONCE, typename V>
__device__ __forceinline__ V load_vec(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, typename V>
__device__ __forceinline__ void store_vec(V* p, V v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}

template <int T, bool ONCE = false>
__device__ __forceinline__ void load4(const void* p, int64_t i, float x[4]) {
  if constexpr (T == DT_F32) {
    const f32x4_el v = load_vec<ONCE>(reinterpret_cast<const f32x4_el*>(static_cast<const float*>(p) + i));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = v[k];
  } else {
    const u16x4_el v = load_vec<ONCE>(reinterpret_cast<const u16x4_el*>(static_cast<const uint16_t*>(p) + i));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = T == DT_BF16 ? bf16_to_f32(v[k]) : f16_to_f32(v[k]);
  }
}

template <int T, bool ONCE = false>
__device__ __forceinline__ void store4(void* p, int64_t i, const float x[4]) {
  if constexpr (T == DT_F32) {
    f32x4_el v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = x[k];
    store_vec<ONCE>(reinterpret_cast<f32x4_el*>(static_cast<float*>(p) + i), v);
  } else {
    u16x4_el v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = T == DT_BF16 ? f32_to_bf16(x[k]) : f32_to_f16(x[k]);
    store_vec<ONCE>(reinterpret_cast<u16x4_el*>(static_cast<uint16_t*>(p) + i), v);
  }
}

}  // namespace
}  // namespace kern
}  // namespace aires
