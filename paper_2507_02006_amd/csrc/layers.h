// Launchers of the operators of layers on top of the aggregated features:
// norm with a residual stream, matrices held in 8 bits and their product, log
// probabilities, gradient norm (gfx950).  Arguments are checked by the entry
// points in layers.cpp.
#pragma once
#include "train.h"

namespace aires {
namespace kern {

// A matrix held in 8 bits: e4m3 codes, one scale for `tile` rows of 128 columns.
struct Held {
  uint8_t* codes;
  float* scales;
  int64_t rows, cols, ld, lds;
  int tile;
};

// root-mean-square norm; R.data, Y.data, Y8.codes, dS.data: NULL where there is none
hipError_t rms_norm(const Mat& X, const Mat& R, const void* gamma, int wt, float eps, const Mat& S, const Mat& Y,
                    const Held& Y8, float* rstd, hipStream_t s);
int64_t rms_norm_workspace(int64_t m, int64_t n);
hipError_t rms_norm_backward(const Mat& dY, const Mat& S, const float* rstd, const void* gamma, int wt, const Mat& dS,
                             const Mat& dX, void* dgamma, float* ws, hipStream_t s);

// X in 8 bits, as it lies and transposed (codes NULL: not wanted)
hipError_t quantize8(const Mat& X, const Held& Q, const Held& Qt, hipStream_t s);
int64_t matmul8_workspace(const Held& A, const Held& B, int type);  // of Y
hipError_t matmul8(const Held& A, const Held& B, const Mat& Y, void* ws, hipStream_t s);

// log probabilities
struct LogProbs {
  Mat Z;
  const void* labels; int labels_i64;
  int top;
  float *logp, *entropy, *lse, *rest;  // rest: what lse's rounding leaves
  float* top_logp; int64_t* top_index;
};
int64_t log_probs_workspace(int64_t t, int64_t v, int top);
hipError_t log_probs(const LogProbs& a, void* ws, hipStream_t s);
hipError_t log_probs_backward(const Mat& Z, const void* labels, int labels_i64, const float* lse, const float* rest,
                              const float* entropy, const float* dlogp, const float* dentropy, const Mat& dZ,
                              hipStream_t s);

// norm over many gradients
struct GradTensor {
  const void* g; void* out;
  int64_t n;
  uint8_t gt, ot;  // DType of g and out
};
int64_t grad_norm_workspace(int64_t count);
hipError_t grad_norm(const GradTensor* tensors, int64_t count, double max_norm, float* norm, float* scale, bool clip,
                     void* ws, hipStream_t s);

}  // namespace kern
}  // namespace aires
