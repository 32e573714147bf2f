// Softmax cross entropy against few classes (at most 64): one pass over H with
// the table kept (few.h), which makes each row's softmax, its loss and both
// gradients.
#include <algorithm>

#include "few.h"

namespace aires {
namespace kern {
namespace {

constexpr int COUNT_BLOCK = 1024;   // labels a workgroup of k_count looks at, at least
constexpr int MAX_COUNTS = 256;
constexpr int COUNT_ALL = 4096;    // so few labels every workgroup of k_few counts by itself: a launch less

// Labelled rows among each workgroup's share.
__global__ __launch_bounds__(256) void k_count(const void* labels, int i64, int64_t T, int64_t V, int* counts) {
  __shared__ int buf[4];
  int n = 0;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < T; t += (int64_t)gridDim.x * 256) {
    const int64_t l = label_at(labels, i64, t);
    n += l >= 0 && l < V;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = buf[0] + buf[1] + buf[2] + buf[3];
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Layout {
  int64_t counts, scale, rows, sums, part, bytes;
};

Layout layout_of(int64_t T, int64_t D, int64_t V, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  const int64_t g = few_groups(few_shape(D, V), T);
  l.counts = take(4 * MAX_COUNTS);
  l.scale = take(4);
  l.rows = take(4 * T);
  l.sums = take(16 * g);
  if (grads) l.part = take(4 * g * V * up(D, 16));
  l.bytes = at;
  return l;
}

}  // namespace

bool xent_few_fits(int64_t T, int64_t D, int64_t V) { return T > 0 && few_shape(D, V).DT > 0; }

int64_t xent_few_workspace(int64_t T, int64_t D, int64_t V, bool grads) { return layout_of(T, D, V, grads).bytes; }

hipError_t xent_few(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dW.data != nullptr || x.dH.data != nullptr;
  const Layout l = layout_of(T, D, V, grads);
  char* ws = static_cast<char*>(x.ws);
  Few f{};
  f.S = x.H; f.K = x.W; f.dS = x.dH;
  f.D = (int)D; f.NK = (int)V; f.Dp = (int)up(D, 16);
  f.labels = x.labels; f.i64 = x.labels_i64;
  f.scale = (float*)(ws + l.scale);
  f.part = grads ? (float*)(ws + l.part) : nullptr;
  f.counts = (const int*)(ws + l.counts);
  // (the gradients need the number of labelled rows first)
  f.ncounts = grads && T > COUNT_ALL ? (int)std::min<int64_t>(MAX_COUNTS, (T + COUNT_BLOCK - 1) / COUNT_BLOCK) : 0;
  f.mean = x.mean; f.grad_scale = x.grad_scale;
  f.row_loss = x.row_loss ? x.row_loss : (float*)(ws + l.rows);
  f.sums = (double2*)(ws + l.sums);
  if (f.ncounts > 0) k_count<<<(unsigned)f.ncounts, 256, 0, s>>>(x.labels, x.labels_i64, T, V, (int*)(ws + l.counts));
  const FewShape sh = few_shape(D, V);
  const unsigned grid = (unsigned)few_groups(sh, T);
  Finish dw{};
  if (!grads) {
    few_launch<FEW_CLASSES>(sh, f, grid, s);
  } else {
    few_launch<FEW_CLASSES_TRAIN>(sh, f, grid, s);
    dw = Finish{f.part, (int)grid, V, D, f.Dp, x.dW.data, x.dW.type, x.dW.ld};
  }
  finish(dw, Finish{}, f.scale, f.sums, (int)grid, x.mean, x.loss, s);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
