// Norm over the gradients of many tensors, and gradients brought to a norm of
// max_norm at most (gfx950).
//
//   norm = sqrt(sum g^2),  scale = max_norm / norm where norm > max_norm, else 1.
//
// Every value is read once, and once more and written where gradients are
// clipped: bandwidth bounds it.  Squares and sums are in 64 bits: the square of
// an fp32 value is exact there and overflows at no size, and a conversion and a
// 64-bit multiply-add a value are a small part of the time its bytes take.  The
// tensors' descriptors travel as kernel arguments; a workgroup finds its tensor
// from its number, sums a span of it and writes one partial sum; a second launch
// adds those in a fixed order.  Where there are few, each workgroup that scales
// gradients adds them by itself instead (the same sum in each).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "layers.h"
#include "rows8.h"

namespace aires {
namespace kern {
namespace {

constexpr int BLOCK = 256;               // threads of a workgroup
constexpr int MAX_TENSORS = 96;          // descriptors that fit the kernel arguments
constexpr int64_t kGroups = 4096;        // workgroups over all tensors, about
constexpr int64_t kFewPartials = 1024;   // partial sums that every workgroup adds by itself
// Chunks of eight values a lane reads at once: four, or one where the tensors are so
// small that more workgroups hide more of the way to memory.
constexpr int64_t chunk_of(int per) { return BLOCK * 8 * per; }
constexpr int64_t kSmall = kFewPartials * chunk_of(1);

struct Table {
  GradTensor t[MAX_TENSORS];
  uint32_t first[MAX_TENSORS + 1];       // first workgroup of each tensor
  int count;
  int64_t span;                          // values a workgroup goes through
};
static_assert(sizeof(Table) <= 3968, "kernel arguments hold 4 KiB");

struct Final {
  const double* part;
  int64_t parts;
  double max_norm;
  float* norm;
  float* scale;
};

__device__ __forceinline__ int find(const Table& tab, uint32_t b) {
  int lo = 0, hi = tab.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tab.first[mid] <= b) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sum over the workgroup, in every thread.
__device__ __forceinline__ double block_sum(double v, double* buf) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += buf[w];
  return v;
}

template <int PER, bool ONCE>
__device__ __forceinline__ void load_chunk(const GradTensor& t, int64_t at, int64_t end, Raw8 (&r)[PER]) {
#pragma unroll
  for (int q = 0; q < PER; ++q) load_raw<ONCE>(t.g, t.gt, at + q * BLOCK * 8, end - at - q * BLOCK * 8, r[q]);
}

template <int PER>
__global__ __launch_bounds__(BLOCK) void k_grad_squares(Table tab, double* part) {
  __shared__ double buf[BLOCK / 64];
  const int k = find(tab, blockIdx.x);
  const GradTensor& t = tab.t[k];
  const int64_t begin = (int64_t)(blockIdx.x - tab.first[k]) * tab.span;
  const int64_t end = begin + tab.span < t.n ? begin + tab.span : t.n;
  double sum = 0.0;
  for (int64_t at = begin + threadIdx.x * 8; at < end; at += chunk_of(PER)) {
    Raw8 r[PER];
    load_chunk<PER, (PER > 1)>(t, at, end, r);
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      float x[8];
      convert(r[q], t.gt, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += (double)x[j] * (double)x[j];
    }
  }
  sum = block_sum(sum, buf);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The partial sums, in an order of their number alone.
__device__ __forceinline__ double add_parts(const Final& f, double* buf) {
  double v = 0.0;
  for (int64_t i = threadIdx.x; i < f.parts; i += blockDim.x) v += f.part[i];
  return block_sum(v, buf);
}

// A NaN gives NaN (the comparison is false), an infinity 0.
__device__ __forceinline__ float scale_of(double sum, double max_norm) {
  const double norm = sqrt(sum);
  return norm <= max_norm ? 1.f : (float)(max_norm / norm);
}

__global__ __launch_bounds__(BLOCK) void k_grad_norm(Final f) {
  __shared__ double buf[BLOCK / 64];
  const double sum = add_parts(f, buf);
  if (threadIdx.x == 0) {
    *f.norm = (float)sqrt(sum);
    if (f.scale) *f.scale = scale_of(sum, f.max_norm);
  }
}

// out = g * scale, scale from the partial sums or (parts = 0) from memory.  The
// first gradients are asked for before it.
template <int PER>
__global__ __launch_bounds__(BLOCK) void k_grad_scale(Table tab, Final f) {
  __shared__ double buf[BLOCK / 64];
  const int k = find(tab, blockIdx.x);
  const GradTensor& t = tab.t[k];
  const int64_t begin = (int64_t)(blockIdx.x - tab.first[k]) * tab.span;
  const int64_t end = begin + tab.span < t.n ? begin + tab.span : t.n;
  int64_t at = begin + threadIdx.x * 8;
  Raw8 r[PER];
  load_chunk<PER, (PER > 1)>(t, at, end, r);
  float scale;
  if (f.parts > 0) {
    const double sum = add_parts(f, buf);
    scale = scale_of(sum, f.max_norm);
    if (f.norm && blockIdx.x == 0 && threadIdx.x == 0) *f.norm = (float)sqrt(sum);
  } else {
    scale = *f.scale;
  }
  if (scale == 1.f && t.out == t.g) return;
  while (at < end) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      float x[8];
      convert(r[q], t.gt, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= scale;
      Raw8 p;
      pack(x, t.ot, p);
      store_raw<(PER > 1)>(t.out, t.ot, at + q * BLOCK * 8, end - at - q * BLOCK * 8, p);
    }
    at += chunk_of(PER);
    if (at < end) load_chunk<PER, (PER > 1)>(t, at, end, r);
  }
}

// Values a workgroup goes through: at most kGroups workgroups, and one for each tensor.
int64_t span_of(int64_t total, int64_t chunk) {
  const int64_t each = (total + kGroups - 1) / kGroups;
  return std::max<int64_t>(1, (each + chunk - 1) / chunk) * chunk;
}

// Launches over all tensors, a table of them at a time; `go` gets the number
// of workgroups before this launch.
template <typename F>
hipError_t for_tables(const GradTensor* tensors, int64_t count, int64_t span, F go) {
  Table tab;
  tab.span = span;
  tab.count = 0;
  tab.first[0] = 0;
  int64_t before = 0;
  for (int64_t k = 0; k <= count; ++k) {
    if (tab.count > 0 && (k == count || tab.count == MAX_TENSORS)) {
      const uint32_t groups = tab.first[tab.count];
      go(tab, groups, before);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      before += groups;
      tab.count = 0;
    }
    if (k == count || tensors[k].n == 0) continue;
    tab.t[tab.count] = tensors[k];
    tab.first[tab.count + 1] = tab.first[tab.count] + (uint32_t)((tensors[k].n + span - 1) / span);
    ++tab.count;
  }
  return hipSuccess;
}

}  // namespace

// (spans that no tensor fills are one a tensor at most; the last place is the scale's)
int64_t grad_norm_workspace(int64_t count) { return (kGroups + count + 1) * (int64_t)sizeof(double); }

hipError_t grad_norm(const GradTensor* tensors, int64_t count, double max_norm, float* norm, float* scale, bool clip,
                     void* ws, hipStream_t s) {
  double* part = static_cast<double*>(ws);
  int64_t total = 0;
  for (int64_t k = 0; k < count; ++k) total += tensors[k].n;
  const bool small = total <= kSmall;
  const int64_t span = span_of(total, chunk_of(small ? 1 : 4));
  Final f{part, 0, max_norm, norm, scale};
  hipError_t e = for_tables(tensors, count, span, [&](const Table& tab, uint32_t groups, int64_t before) {
    if (small) k_grad_squares<1><<<groups, BLOCK, 0, s>>>(tab, part + before);
    else k_grad_squares<4><<<groups, BLOCK, 0, s>>>(tab, part + before);
    f.parts = before + groups;
  });
  if (e != hipSuccess) return e;
  if (!clip || f.parts == 0 || f.parts > kFewPartials) {
    if (clip) f.scale = reinterpret_cast<float*>(part + kGroups + count);
    k_grad_norm<<<1, BLOCK, 0, s>>>(f);
    e = hipGetLastError();
    if (e != hipSuccess || !clip || f.parts == 0) return e;
    f.parts = 0;
  }
  return for_tables(tensors, count, span, [&](const Table& tab, uint32_t groups, int64_t before) {
    Final g = f;
    if (before > 0) g.norm = nullptr;
    if (small) k_grad_scale<1><<<groups, BLOCK, 0, s>>>(tab, g);
    else k_grad_scale<4><<<groups, BLOCK, 0, s>>>(tab, g);
  });
}

}  // namespace kern
}  // namespace aires
