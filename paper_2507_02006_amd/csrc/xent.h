// Shared by the cross entropy's kernels: xent.hip (any table),
// xent_few.hip (few classes) and xent_rows.hip (few rows).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "train.h"

namespace aires {
namespace kern {

// out (rows x cols of `type`) = *scale times the sum of fp32 slices
// [slice][rows][ldp], in a fixed order; ldp a multiple of 4.  part NULL: none.
struct Finish {
  const float* part; int slices;
  int64_t rows, cols, ldp;
  void* out; int type; int64_t ldo;
};

// Both, and the loss from `sums` (losses, labelled rows) where that is given, in
// one launch.
void finish(const Finish& a, const Finish& b, const float* scale, const double2* sums, int nsums, int mean, float* loss,
            hipStream_t s);

// Rows' maxima, inverse sums and losses from the statistics [tile][t] of
// `tiles` tiles of the table and the scores `target` of the labels, the loss, and
// *scale = grad_scale / c.  *ticket is 0 before; sums: rows_and_loss_workspace(T)
// bytes.
int64_t rows_and_loss_workspace(int64_t T);
void rows_and_loss(const XentArgs& x, const float2* part, int64_t tiles, const float* target, float* top, float* inv,
                   float* row_loss, void* sums, uint32_t* ticket, float grad_scale, float* scale, hipStream_t s);

// Few rows, few classes: whether this shape takes that path, its workspace, and the
// call.
bool xent_few_fits(int64_t T, int64_t D, int64_t V);
int64_t xent_few_workspace(int64_t T, int64_t D, int64_t V, bool grads);
hipError_t xent_few(const XentArgs& x, hipStream_t s);
bool xent_rows_fits(int64_t T, int64_t D, int64_t V, int type, bool grads);
int64_t xent_rows_workspace(int64_t T, int64_t D, int64_t V, bool grads);
hipError_t xent_rows(const XentArgs& x, hipStream_t s);

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

__device__ __forceinline__ int64_t label_at(const void* labels, int i64, int64_t i) {
  return i64 ? static_cast<const int64_t*>(labels)[i] : (int64_t)static_cast<const int32_t*>(labels)[i];
}

// exp(z - top).  The difference is taken first: it is exact where it is small
// and 0 at the maximum, whatever the scores' size, so that a row's sum is 1 and
// what the others add.
__device__ __forceinline__ float exp_from(float z, float top) { return __builtin_amdgcn_exp2f((z - top) * LOG2E); }

// log sum_j exp(z_j) - target from the maximum and the sum of exp(z_j - top).
// top and target are of one size: their difference is taken before the logarithm
// is added, and is exact where the loss is small.  Not negative.
__device__ __forceinline__ float loss_of(float top, float sum, float target) {
  return (top - target) + log2f(sum) * LN2;
}

__device__ __forceinline__ double2 wave_sum2(double2 v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    v.x += __shfl_xor(v.x, o);
    v.y += __shfl_xor(v.y, o);
  }
  return v;
}

// Joins two (maximum, sum of exponentials); equal maxima (of minus infinity too)
// need no scaling.
__device__ __forceinline__ void join(float& m, float& s, float m1, float s1) {
  const float top = fmaxf(m, m1);
  s = (m == top ? s : s * exp_from(m, top)) + (m1 == top ? s1 : s1 * exp_from(m1, top));
  m = top;
}

}  // namespace
}  // namespace kern
}  // namespace aires
