// Softmax cross entropy of few rows (at most 64) against a table: passes over
// the table with H kept (few.h), one for the rows' maxima and sums of
// exponentials, one for the gradients.  Unlike the tiles of xent.hip it takes
// the table as it lies: fp32, or rows at any alignment.
#include <algorithm>

#include "few.h"

namespace aires {
namespace kern {
namespace {

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Layout {
  int64_t ticket, scale, target, top, inv, rows, sums, stats, part, bytes;
};

Layout layout_of(int64_t T, int64_t D, int64_t V, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  const int64_t g = few_groups(few_shape(D, T), V);
  l.ticket = take(4);
  l.scale = take(4);
  l.target = take(4 * T);
  l.top = take(4 * T);
  l.inv = take(4 * T);
  l.rows = take(4 * T);
  l.sums = take(rows_and_loss_workspace(T));
  l.stats = take(8 * g * T);
  if (grads) l.part = take(4 * g * T * up(D, 16));
  l.bytes = at;
  return l;
}

}  // namespace

// fp32 tables would be split into planes (16 bytes moved for each 4), tables
// of an odd number of columns copied (6 for 2): with few rows that is the whole
// work.  16-bit tables that the tiles read as they lie stay with them, and so do
// calls whose gradients, fp32 products here, cost more than the copy.  Loss, and
// loss and gradients, in us, here and in tiles:
//   f32, 60013 x 256:   1 row 20, 53 and 49, 110;  32 rows 31, 82 and 50, 117;
//                       64 rows 43, 118 and 53, 132 (60013 x 333: 65, 233 and 66, 183)
//   f16, 60013 x 333:  16 rows 30, 79 and 33, 83;  32 rows 34, 103 and 34, 84;
//                       64 rows 43, 165 and 34, 85
//   f16, 261215 x 815: 16 rows 150, 469 and 283, 682;  32 rows 168, 782 and 283, 681
bool xent_rows_fits(int64_t T, int64_t D, int64_t V, int type, bool grads) {
  if (T < 1 || few_shape(D, T).DT == 0) return false;
  return type == DT_F32 ? T <= 64 : D % 8 != 0 && T <= (grads ? 16 : 32);
}

int64_t xent_rows_workspace(int64_t T, int64_t D, int64_t V, bool grads) { return layout_of(T, D, V, grads).bytes; }

hipError_t xent_rows(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dW.data != nullptr || x.dH.data != nullptr;
  const Layout l = layout_of(T, D, V, grads);
  char* ws = static_cast<char*>(x.ws);
  const FewShape sh = few_shape(D, T);
  const unsigned grid = (unsigned)few_groups(sh, V);
  Few f{};
  f.S = x.W; f.K = x.H; f.dS = x.dW;
  f.D = (int)D; f.NK = (int)T; f.Dp = (int)up(D, 16);
  f.labels = x.labels; f.i64 = x.labels_i64;
  f.scale = (float*)(ws + l.scale); f.ticket = (uint32_t*)(ws + l.ticket);
  f.part = grads ? (float*)(ws + l.part) : nullptr;
  f.stats = (float2*)(ws + l.stats);
  f.target = (float*)(ws + l.target);
  f.top = (const float*)(ws + l.top); f.inv = (const float*)(ws + l.inv);
  few_launch<FEW_STATS>(sh, f, grid, s);
  rows_and_loss(x, f.stats, grid, f.target, (float*)(ws + l.top), (float*)(ws + l.inv),
                x.row_loss ? x.row_loss : (float*)(ws + l.rows), ws + l.sums, f.ticket, x.grad_scale, f.scale, s);
  if (grads) {
    few_launch<FEW_DZ>(sh, f, grid, s);
    finish(Finish{f.part, (int)grid, T, D, f.Dp, x.dH.data, x.dH.type, x.dH.ld}, Finish{}, f.scale, nullptr, 0, 0, nullptr, s);
  }
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
