// Launchers of the training operators (dense rows, gfx950).  Arguments are
// checked by the entry points in train.cpp.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aires {
namespace kern {

struct Mat {  // row-major device matrix; type: DType
  void* data;
  int64_t rows, cols, ld;
  int type;
};

// layer norm
hipError_t layer_norm(const Mat& X, const void* gamma, const void* beta, int wt, float eps, const Mat& Y, float* mean,
                      float* rstd, hipStream_t s);
int64_t layer_norm_workspace(int64_t m, int64_t n);
hipError_t layer_norm_backward(const Mat& dY, const Mat& X, const float* mean, const float* rstd, const void* gamma,
                               int wt, const Mat& dX, void* dgamma, void* dbeta, float* ws, hipStream_t s);

// softmax cross entropy of H W^T
struct XentArgs {
  Mat H, W, dH, dW;  // dH, dW: data NULL without gradients
  const void* labels;
  int labels_i64, mean;
  float grad_scale;
  float* loss; float* row_loss;  // row_loss may be NULL
  void* ws;
};
int64_t linear_xent_workspace(int64_t T, int64_t D, int64_t V, int type, bool grads);
hipError_t linear_xent(const XentArgs& x, hipStream_t s);

// AdamW: moments in 32 bits, or in 8 where ms and vs are given
struct AdamWTensor {
  void* p; const void* g; void* m; void* v;
  float* ms; float* vs;
  void* c;
  int64_t n;
  uint32_t seed;
  uint8_t pt, gt, ct;  // DType of p, g and c
};
struct AdamWStep {
  float beta1, one_beta1, beta2, one_beta2, eps, decay, rate, inv_root, grad_scale;
};
// What the rounding of a tensor's 8-bit moments is drawn from.
uint32_t adamw_seed(uint32_t seed, int64_t tensor);
// device_scale: a factor of the gradients in device memory, or NULL.
hipError_t adamw(const AdamWTensor* tensors, int64_t count, const AdamWStep& step, const float* device_scale,
                 hipStream_t s);

}  // namespace kern
}  // namespace aires
