// AdamW over many tensors in one launch, moments in 32 or in 8 bits (gfx950).
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr / (1 - b1^k) m / (sqrt(v) / sqrt(1 - b2^k) + eps).
//
// Every value is read and written once: 28 bytes with fp32 gradients and
// 32-bit moments, 14 with bf16 gradients and 8-bit moments, for about 15
// operations (80 with 8-bit moments: conversions, the block's maximum, random
// rounding), so bandwidth bounds it.  The tensors' descriptors travel as
// kernel arguments; a workgroup finds its tensor from its number and updates
// 4096 values, all of whose loads are issued before the first is used.
// Measured: 32-bit moments, bf16 gradients and copies, 262144 x 512 values, 630
// us (6.0 TB/s of 28 bytes a value); 8-bit moments, bf16 gradients, 1048576 x
// 256 values, 620 to 640 us (5.9 to 6.1 TB/s of 14 bytes a value); 19 tensors of
// 1.4 million values in all, f32, 7 us.
//
// 8-bit moments: blocks of 256 values share a scale, so that a block is four
// values a lane of one wavefront and its maximum a scan within the registers.
// m is held as e4m3.  v is held as e5m2: as a square it needs the exponents.
// Both are rounded at random in proportion to the distance: v moves by a
// thousandth a step where neighbouring codes are an eighth to a quarter apart,
// so rounding to nearest would never let it move.
#include "train.h"

#include <algorithm>
#include <cmath>

#include "dense.h"
#include "device.h"

#pragma clang fp contract(off)

namespace aires {
namespace kern {
namespace {

constexpr int BLOCK = 256;            // threads of a workgroup; values that share a scale
constexpr int PER = 4;                // vectors of four values a lane updates
constexpr int CHUNK = BLOCK * 4 * PER;  // values a workgroup updates
constexpr int MAX_TENSORS = 40;       // descriptors that fit the kernel arguments

struct Table {
  AdamWTensor t[MAX_TENSORS];
  uint32_t first[MAX_TENSORS + 1];    // first workgroup of each tensor
  int count;
  AdamWStep o;
};
static_assert(sizeof(Table) <= 4096, "kernel arguments hold 4 KiB");

// The tensor that this workgroup updates, and the workgroup's number in it.
__device__ __forceinline__ int find(const Table& tab, uint32_t b) {
  int lo = 0, hi = tab.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tab.first[mid] <= b) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int T, int STRIDE>
__device__ __forceinline__ void load_all_t(const void* p, int64_t i, float (&x)[PER][4]) {
#pragma unroll
  for (int q = 0; q < PER; ++q) load4<T, true>(p, i + q * STRIDE, x[q]);
}

template <int STRIDE>
__device__ __forceinline__ void load_all(const void* p, int t, int64_t i, float (&x)[PER][4]) {
  if (t == DT_F32) load_all_t<DT_F32, STRIDE>(p, i, x);
  else if (t == DT_BF16) load_all_t<DT_BF16, STRIDE>(p, i, x);
  else load_all_t<DT_F16, STRIDE>(p, i, x);
}

template <int T, int STRIDE>
__device__ __forceinline__ void store_all_t(void* p, int64_t i, const float (&x)[PER][4]) {
#pragma unroll
  for (int q = 0; q < PER; ++q) store4<T, true>(p, i + q * STRIDE, x[q]);
}

template <int STRIDE>
__device__ __forceinline__ void store_all(void* p, int t, int64_t i, const float (&x)[PER][4]) {
  if (t == DT_F32) store_all_t<DT_F32, STRIDE>(p, i, x);
  else if (t == DT_BF16) store_all_t<DT_BF16, STRIDE>(p, i, x);
  else store_all_t<DT_F16, STRIDE>(p, i, x);
}

// New moments, and the parameter from them.  The square root and the
// reciprocal are the hardware's, within one unit in the last place; the square
// root takes denormal numbers for 0, so small ones are raised by 2^64 before.
__device__ __forceinline__ void update(const AdamWStep& o, float g, float& p, float& m, float& v) {
  g *= o.grad_scale;
  m = m * o.beta1 + g * o.one_beta1;
  v = v * o.beta2 + (g * g) * o.one_beta2;
  const bool low = v < 0x1p-96f;
  const float root = __builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.f);
  const float den = root * o.inv_root + o.eps;
  p = p * o.decay - o.rate * (m * __builtin_amdgcn_rcpf(den));
}

__global__ __launch_bounds__(BLOCK) void k_adamw_32(Table tab) {
  const int k = find(tab, blockIdx.x);
  const AdamWTensor& t = tab.t[k];
  const int64_t base = (int64_t)(blockIdx.x - tab.first[k]) * CHUNK;
  float* const m_ = static_cast<float*>(t.m);
  float* const v_ = static_cast<float*>(t.v);
  if (base + CHUNK <= t.n) {
    const int64_t i = base + threadIdx.x * 4;
    float p[PER][4], g[PER][4], m[PER][4], v[PER][4];
    load_all<4 * BLOCK>(t.g, t.gt, i, g);
    load_all_t<DT_F32, 4 * BLOCK>(m_, i, m);
    load_all_t<DT_F32, 4 * BLOCK>(v_, i, v);
    load_all<4 * BLOCK>(t.p, t.pt, i, p);
#pragma unroll
    for (int q = 0; q < PER; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) update(tab.o, g[q][j], p[q][j], m[q][j], v[q][j]);
    store_all_t<DT_F32, 4 * BLOCK>(m_, i, m);
    store_all_t<DT_F32, 4 * BLOCK>(v_, i, v);
    store_all<4 * BLOCK>(t.p, t.pt, i, p);
    if (t.c) store_all<4 * BLOCK>(t.c, t.ct, i, p);
    return;
  }
  for (int64_t i = base + threadIdx.x; i < t.n; i += BLOCK) {
    float p = load1(t.p, t.pt, i), m = m_[i], v = v_[i];
    update(tab.o, load1(t.g, t.gt, i), p, m, v);
    m_[i] = m;
    v_[i] = v;
    store1(t.p, t.pt, i, p);
    if (t.c) store1(t.c, t.ct, i, p);
  }
}

// ------------------------------------------------------------ 8-bit moments

constexpr float TINY = 0x1p-110f;  // blocks below are held as zeros
constexpr float TOP_M = 448.f, TOP_V = 57344.f;

typedef uint32_t u32_any __attribute__((aligned(1)));

template <bool SECOND>
__device__ __forceinline__ void decode(uint32_t c, float s, float (&x)[4]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  f2 lo, hi;
  if constexpr (SECOND) {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8(c, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8(c, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  }
  x[0] = lo.x * s; x[1] = lo.y * s; x[2] = hi.x * s; x[3] = hi.y * s;
}

template <bool SECOND>
__device__ __forceinline__ uint32_t encode(const float (&x)[4]) {
  int c = 0;
  if constexpr (SECOND) {
    c = __builtin_amdgcn_cvt_pk_bf8_f32(x[0], x[1], c, false);
    c = __builtin_amdgcn_cvt_pk_bf8_f32(x[2], x[3], c, true);
  } else {
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], c, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c, true);
  }
  return (uint32_t)c;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// Largest finite magnitude of the wavefront's values (patterns of values
// that are not negative order as integers do).
__device__ __forceinline__ float block_max(const float (&x)[4]) {
  float big = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) big = fmaxf(big, finite(x[j]) ? fabsf(x[j]) : 0.f);
  return __uint_as_float((uint32_t)wave_last(wave_scan_op<false>((int)__float_as_uint(big))));
}

// x (in units of the block's scale) to a code above or below it, with 16
// random bits r: they are added below the mantissa bits that stay (DROP go),
// so the carry rounds up in proportion.  Below the smallest normal code the
// codes are evenly spaced; adding that code's value there lines the mantissa
// up with them.
template <bool SECOND>
__device__ __forceinline__ float round_code(float x, uint32_t r) {
  constexpr int DROP = SECOND ? 21 : 20;
  constexpr float LEAST = SECOND ? 0x1p-14f : 0x1p-6f, TOP = SECOND ? TOP_V : TOP_M;
  const float a = fminf(fabsf(x), TOP);
  const float off = a < LEAST ? LEAST : 0.f;
  const uint32_t bits = __float_as_uint(a + off) + ((r << (DROP - 16)) | (1u << (DROP - 17)));
  float q = fminf(__uint_as_float(bits & ~((1u << DROP) - 1)) - off, TOP);
  if constexpr (SECOND) q = fmaxf(q, a > 0.f ? 0x1p-16f : 0.f);
  return finite(x) ? copysignf(q, x) : __uint_as_float(0x7fc00000u);
}

// 32 random bits of a value: two multiply-and-fold rounds over its index.
__device__ __forceinline__ uint32_t noise(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7C2E9D35u;
  x = (x ^ (x >> 15)) * 0x6A8F3B47u;
  return x ^ (x >> 16);
}
constexpr uint32_t kIndexStep = 0x9E3779B1u;

__global__ __launch_bounds__(BLOCK) void k_adamw_8(Table tab) {
  const int k = find(tab, blockIdx.x);
  const AdamWTensor& t = tab.t[k];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // this wavefront's PER blocks
  const int64_t base = (int64_t)(blockIdx.x - tab.first[k]) * CHUNK + wave * (PER * BLOCK);
  if (base >= t.n) return;
  const int64_t i0 = base + lane * 4;
  uint8_t* const mc = static_cast<uint8_t*>(t.m);
  uint8_t* const vc = static_cast<uint8_t*>(t.v);
  const bool whole = base + PER * BLOCK <= t.n;
  float p[PER][4], g[PER][4];
  uint32_t cm[PER], cv[PER];
  float sm[PER], sv[PER];
  if (whole) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      cm[q] = load_vec<true>(reinterpret_cast<const u32_any*>(mc + i0 + q * BLOCK));
      cv[q] = load_vec<true>(reinterpret_cast<const u32_any*>(vc + i0 + q * BLOCK));
      sm[q] = t.ms[base / BLOCK + q];
      sv[q] = t.vs[base / BLOCK + q];
    }
    load_all<BLOCK>(t.g, t.gt, i0, g);
    load_all<BLOCK>(t.p, t.pt, i0, p);
  } else {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const bool some = base + q * BLOCK < t.n;
      cm[q] = cv[q] = 0;
      sm[q] = some ? t.ms[base / BLOCK + q] : 0.f;
      sv[q] = some ? t.vs[base / BLOCK + q] : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t i = i0 + q * BLOCK + j;
        const bool in = i < t.n;
        g[q][j] = in ? load1(t.g, t.gt, i) : 0.f;
        p[q][j] = in ? load1(t.p, t.pt, i) : 0.f;
        if (in) {
          cm[q] |= (uint32_t)mc[i] << (8 * j);
          cv[q] |= (uint32_t)vc[i] << (8 * j);
        }
      }
    }
  }
  float m[PER][4], v[PER][4], big = 0.f;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    decode<false>(cm[q], sm[q], m[q]);
    decode<true>(cv[q], sv[q], v[q]);
#pragma unroll
    for (int j = 0; j < 4; ++j) update(tab.o, g[q][j], p[q][j], m[q][j], v[q][j]);
    // lane 2 q keeps block q's largest first moment, lane 2 q + 1 its second
    const float bm = block_max(m[q]), bv = block_max(v[q]);
    big = lane == 2 * q ? bm : lane == 2 * q + 1 ? bv : big;
  }
  // All scales and their inverses at once: the division is what they cost.  Both
  // are rounded as torch rounds such quotients on the device (x / constant as a
  // product with its reciprocal, constant / x as one with x's): rounded once
  // instead, codes next to a boundary come out otherwise than there.
  const bool used = big >= TINY;
  const float top = lane & 1 ? TOP_V : TOP_M, one = lane & 1 ? 1.f / TOP_V : 1.f / TOP_M;
  const float scale = used ? big * one : 0.f, inverse = used ? 1.f / big * top : 0.f;
  auto of = [](float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const float im = of(inverse, 2 * q), iv = of(inverse, 2 * q + 1);
    sm[q] = of(scale, 2 * q);
    sv[q] = of(scale, 2 * q + 1);
    const uint32_t x0 = (uint32_t)(i0 + q * BLOCK) * kIndexStep + t.seed;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t r = noise(x0 + j * kIndexStep);
      m[q][j] = round_code<false>(m[q][j] * im, r & 0xffffu);
      v[q][j] = round_code<true>(v[q][j] * iv, r >> 16);
    }
    cm[q] = encode<false>(m[q]);
    cv[q] = encode<true>(v[q]);
  }
  if (whole) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      store_vec<true, u32_any>(reinterpret_cast<u32_any*>(mc + i0 + q * BLOCK), cm[q]);
      store_vec<true, u32_any>(reinterpret_cast<u32_any*>(vc + i0 + q * BLOCK), cv[q]);
    }
    store_all<BLOCK>(t.p, t.pt, i0, p);
    if (t.c) store_all<BLOCK>(t.c, t.ct, i0, p);
  } else {
#pragma unroll
    for (int q = 0; q < PER; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t i = i0 + q * BLOCK + j;
        if (i < t.n) {
          mc[i] = (uint8_t)(cm[q] >> (8 * j));
          vc[i] = (uint8_t)(cv[q] >> (8 * j));
          store1(t.p, t.pt, i, p[q][j]);
          if (t.c) store1(t.c, t.ct, i, p[q][j]);
        }
      }
  }
  if (lane == 0)
#pragma unroll
    for (int q = 0; q < PER; ++q)
      if (base + q * BLOCK < t.n) {
        t.ms[base / BLOCK + q] = sm[q];
        t.vs[base / BLOCK + q] = sv[q];
      }
}

}  // namespace

uint32_t adamw_seed(uint32_t seed, int64_t tensor) {
  return (seed + (uint32_t)tensor * 0x632BE5ABu) * 0x85157AF5u;
}

hipError_t adamw(const AdamWTensor* tensors, int64_t count, const AdamWStep& step, hipStream_t s) {
  constexpr int64_t kMost = int64_t(1) << 23;  // workgroups of a launch (2^31 threads), and of a tensor at most
  for (int eight = 0; eight < 2; ++eight) {
    Table tab;
    tab.o = step;
    tab.count = 0;
    tab.first[0] = 0;
    auto launch = [&]() {
      if (tab.count == 0) return hipSuccess;
      if (eight) k_adamw_8<<<tab.first[tab.count], BLOCK, 0, s>>>(tab);
      else k_adamw_32<<<tab.first[tab.count], BLOCK, 0, s>>>(tab);
      tab.count = 0;
      return hipGetLastError();
    };
    for (int64_t k = 0; k < count; ++k) {
      if ((tensors[k].ms != nullptr) != (eight != 0) || tensors[k].n == 0) continue;
      const int64_t groups = (tensors[k].n + CHUNK - 1) / CHUNK;
      if (tab.count == MAX_TENSORS || (tab.count && tab.first[tab.count] + groups > kMost)) {
        const hipError_t e = launch();
        if (e != hipSuccess) return e;
      }
      tab.t[tab.count] = tensors[k];
      tab.first[tab.count + 1] = tab.first[tab.count] + (uint32_t)groups;
      ++tab.count;
    }
    const hipError_t e = launch();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace kern
}  // namespace aires
