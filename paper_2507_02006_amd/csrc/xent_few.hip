// Softmax cross entropy against few classes (at most 64), loss and both
// gradients in one pass over the rows (gfx950).
//
// With few classes the products are small and what bounds the work is the
// bytes of H and dH, so each row is read once and everything that it is needed
// for happens while it is in LDS: scores z = H W^T, the row's softmax and
// loss, dH = dz W and its share of dW = dz^T H.  A workgroup holds W in LDS and
// takes blocks of TB rows in turn, the next block's rows on their way to
// registers meanwhile; dW stays in the accumulators until the end, when each
// workgroup writes its sum for a second launch to add up in a fixed order.
//
// Products run in fp32 on the matrix cores (16 x 16 x 4) for every type: fp32
// rows are not rounded anywhere.  A lane's k within a step is free as long as
// both operands agree on it, so four steps' values come in one 16-byte read:
// k = 16 i + 4 (lane / 16) + j for step j of group i.  With row strides that
// are 4 modulo 8 words the same order also keeps the reads along columns
// (dW) free of bank conflicts.
#include "xent.h"

#include <algorithm>

#include "dense.h"
#include "device.h"

namespace aires {
namespace kern {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 512, WAVES = 8;
constexpr int COUNT_BLOCK = 1024;   // labels a workgroup of k_count looks at, at least
constexpr int MAX_COUNTS = 256;
constexpr int64_t LDS_BYTES = 160 * 1024;

struct Few {
  Mat H, W, dH;
  const void* labels; int i64;
  const int* counts; int ncounts;
  int mean; float grad_scale;
  float* scale; float* loss; float* row_loss;
  double* sums; uint32_t* ticket;
  float* part;                      // [workgroup][V][Dp], NULL without gradients
  int D, V, Dp;
};

// Labelled rows among each workgroup's share.
__global__ __launch_bounds__(256) void k_count(const void* labels, int i64, int64_t T, int64_t V, int* counts,
                                               uint32_t* ticket) {
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
  if (threadIdx.x == 0) {
    counts[blockIdx.x] = buf[0] + buf[1] + buf[2] + buf[3];
    if (blockIdx.x == 0) *ticket = 0;
  }
}

// Words of LDS: W, a block of H, partial scores, dz.
constexpr int words(int VT, int TB, int Dp) {
  return (VT * 16 + TB) * (Dp + 4) + (WAVES / (TB / 16) + 1) * TB * (VT * 16 + 4);
}

// VT tiles of 16 classes, DT tiles of 16 columns a wavefront, TB rows a block.
template <int VT, int DT, int TB, bool GRAD>
__global__ __launch_bounds__(THREADS, 2) void k_few(Few a) {
  constexpr int Vp = VT * 16, ZS = Vp + 4;         // classes; stride of score rows
  constexpr int RT = TB / 16, KS = WAVES / RT;     // row tiles, shares of k
  constexpr int PF = TB * DT / 16;                 // 4-column chunks a thread fetches
  constexpr int PER = THREADS / TB, CW = Vp / PER; // threads and classes a thread of a row
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int Dp = a.Dp, HS = Dp + 4;
  float* const w = lds;                            // [Vp][HS]
  float* const h = w + Vp * HS;                    // [TB][HS]
  float* const z = h + TB * HS;                    // [KS][TB][ZS]
  float* const dz = z + KS * TB * ZS;              // [TB][ZS]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, q = lane >> 4;
  const int64_t T = a.H.rows;
  const int D = a.D, V = a.V, groups = Dp / 16;

  // what dz is multiplied with
  __shared__ int total;
  if (wave == 0) {
    int c = 0;
    for (int i = lane; i < a.ncounts; i += 64) c += a.counts[i];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
    if (lane == 0) total = c;
  }
  for (int i = tid; i < Vp * (Dp / 4); i += THREADS) {
    const int r = i / (Dp / 4), c = (i - r * (Dp / 4)) * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[r * HS + c + k] = r < V && c + k < D ? load1(a.W.data, a.W.type, (int64_t)r * a.W.ld + c + k) : 0.f;
  }
  __syncthreads();
  const double div = a.mean ? (double)(total > 0 ? total : 1) : 1.0;
  const float scale = (float)(a.grad_scale / div);
  if (blockIdx.x == 0 && tid == 0) *a.scale = scale;

  // W as dH's operand stays in registers: columns of this wavefront's tiles
  float wk[GRAD ? DT : 1][VT][4];
  f32x4 acc[GRAD ? VT : 1][DT];
  if constexpr (GRAD) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        const int tile = wave + d * WAVES;
#pragma unroll
        for (int j = 0; j < 4; ++j) wk[d][i][j] = tile < groups ? w[(16 * i + 4 * q + j) * HS + tile * 16 + n16] : 0.f;
        acc[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
  }

  // this thread's chunks of a block of H
  const int per_row = Dp / 4;
  float next[PF][4];
  auto fetch = [&](int64_t t0) {
#pragma unroll
    for (int e = 0; e < PF; ++e) {
      const int i = e * THREADS + tid, r = i / per_row, c = (i - r * per_row) * 4;
      const int64_t t = t0 + r, at = t * a.H.ld + c;
      const bool in = r < TB && t < T;
      if (in && c + 4 <= D) {
        if (a.H.type == DT_F32) load4<DT_F32>(a.H.data, at, next[e]);
        else if (a.H.type == DT_BF16) load4<DT_BF16>(a.H.data, at, next[e]);
        else load4<DT_F16>(a.H.data, at, next[e]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) next[e][k] = in && c + k < D ? load1(a.H.data, a.H.type, at + k) : 0.f;
      }
    }
  };

  const int64_t blocks = (T + TB - 1) / TB;
  double loss = 0;
  int64_t b = blockIdx.x;
  if (b < blocks) fetch(b * TB);
  for (; b < blocks; b += gridDim.x) {
    const int64_t t0 = b * TB;
#pragma unroll
    for (int e = 0; e < PF; ++e) {
      const int i = e * THREADS + tid, r = i / per_row, c = (i - r * per_row) * 4;
      if (r < TB) *reinterpret_cast<f32x4*>(h + r * HS + c) = f32x4{next[e][0], next[e][1], next[e][2], next[e][3]};
    }
    __syncthreads();
    if (b + gridDim.x < blocks) fetch((b + gridDim.x) * TB);

    {  // scores of 16 rows over this wavefront's share of k
      const int rt = wave % RT, ks = wave / RT;
      const int i0 = groups * ks / KS, i1 = groups * (ks + 1) / KS;
      f32x4 s[VT];
#pragma unroll
      for (int v = 0; v < VT; ++v) s[v] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int i = i0; i < i1; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(h + (rt * 16 + n16) * HS + 16 * i + 4 * q);
#pragma unroll
        for (int v = 0; v < VT; ++v) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(w + (v * 16 + n16) * HS + 16 * i + 4 * q);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[v] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], s[v], 0, 0, 0);
        }
      }
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[(ks * TB + rt * 16 + 4 * q + r) * ZS + v * 16 + n16] = s[v][r];
    }
    __syncthreads();

    {  // softmax and loss: PER threads a row, CW classes each
      const int r = tid / PER, p = tid % PER;
      const int64_t t = t0 + r;
      const int64_t label = t < T ? label_at(a.labels, a.i64, t) : -1;
      const bool there = label >= 0 && label < V;
      float x[CW], top = -INFINITY, target = 0.f;
#pragma unroll
      for (int k = 0; k < CW; ++k) {
        const int v = p + k * PER;
        float s = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s += z[(ks * TB + r) * ZS + v];
        x[k] = v < V ? s : -INFINITY;
        top = fmaxf(top, x[k]);
        if (v == label) target = s;
      }
#pragma unroll
      for (int o = 1; o < PER; o <<= 1) {
        top = fmaxf(top, __shfl_xor(top, o));
        target += __shfl_xor(target, o);
      }
      const float top2 = top * LOG2E, from = top2 == -INFINITY ? 0.f : top2;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < CW; ++k) {
        x[k] = exp2_fast(fmaf(x[k], LOG2E, -from));
        sum += x[k];
      }
#pragma unroll
      for (int o = 1; o < PER; o <<= 1) sum += __shfl_xor(sum, o);
      if constexpr (GRAD) {
        const float inv = 1.f / sum;
#pragma unroll
        for (int k = 0; k < CW; ++k) {
          const int v = p + k * PER;
          dz[r * ZS + v] = there && v < V ? x[k] * inv - (v == label ? 1.f : 0.f) : 0.f;
        }
      }
      if (p == 0 && t < T) {
        const float l = there ? (top2 + log2f(sum)) * LN2 - target : 0.f;
        a.row_loss[t] = l;
        loss += l;
      }
    }
    __syncthreads();

    if constexpr (GRAD) {
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int tile = wave + d * WAVES;
        if (tile >= groups) continue;
        // dH, 16 columns by 16 rows: four columns of a row a lane
        const int c = tile * 16 + 4 * q;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < VT; ++i) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(dz + (rt * 16 + n16) * ZS + 16 * i + 4 * q);
#pragma unroll
            for (int j = 0; j < 4; ++j) o = __builtin_amdgcn_mfma_f32_16x16x4f32(wk[d][i][j], y[j], o, 0, 0, 0);
          }
          const int64_t t = t0 + rt * 16 + n16;
          if (t < T) {
            const float x[4] = {o[0] * scale, o[1] * scale, o[2] * scale, o[3] * scale};
            const int64_t at = t * a.dH.ld + c;
            if (c + 4 <= D) {
              if (a.dH.type == DT_F32) store4<DT_F32>(a.dH.data, at, x);
              else if (a.dH.type == DT_BF16) store4<DT_BF16>(a.dH.data, at, x);
              else store4<DT_F16>(a.dH.data, at, x);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (c + k < D) store1(a.dH.data, a.dH.type, at + k, x[k]);
            }
          }
        }
        // dW
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int k = 16 * i + 4 * q + j;
            const float y = h[k * HS + tile * 16 + n16];
#pragma unroll
            for (int v = 0; v < VT; ++v)
              acc[v][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(dz[k * ZS + v * 16 + n16], y, acc[v][d], 0, 0, 0);
          }
      }
      __syncthreads();  // h and dz are free
    }
  }

  if constexpr (GRAD) {
    float* part = a.part + (int64_t)blockIdx.x * V * Dp;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const int tile = wave + d * WAVES;
      if (tile >= groups) continue;
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = v * 16 + 4 * q + r;
          if (row < V) part[(int64_t)row * Dp + tile * 16 + n16] = acc[v][d][r];
        }
    }
  }

  // the workgroup's loss; the last workgroup adds them up in order
  __shared__ double sums[THREADS];
  __shared__ bool last;
  auto add_up = [&](double x) {
    sums[tid] = x;
    __syncthreads();
    for (int o = THREADS / 2; o > 0; o >>= 1) {
      if (tid < o) sums[tid] += sums[tid + o];
      __syncthreads();
    }
  };
  add_up(loss);
  if (tid == 0) {
    a.sums[blockIdx.x] = sums[0];
    last = gridDim.x == 1 ||
           __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  loss = 0;
  for (int i = tid; i < (int)gridDim.x; i += THREADS) loss += a.sums[i];
  add_up(loss);
  if (tid == 0) *a.loss = (float)(sums[0] / div);
}

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Whether a block of TB rows fits LDS next to W and the kernel's own arrays,
// and the registers (64 rows of more than 384 columns do not).
constexpr bool fits(int VT, int TB, int Dp) {
  return (TB == 32 || Dp <= 384) && (int64_t)words(VT, TB, Dp) * 4 + THREADS * 8 + 64 <= LDS_BYTES;
}

// Rows a block: 64, or 32 where a wider W leaves no room for more; 0: neither.
int rows_of(int64_t D, int64_t V) {
  if (V > 64 || D > 512) return 0;
  const int VT = (int)((V + 15) / 16), Dp = (int)up(D, 16);
  return fits(VT, 64, Dp) ? 64 : fits(VT, 32, Dp) ? 32 : 0;
}

int64_t groups_of(int64_t T, int TB) { return std::max<int64_t>(1, std::min<int64_t>(256, (T + TB - 1) / TB)); }

struct Layout {
  int64_t counts, ticket, scale, rows, sums, part, bytes;
};

Layout layout_of(int64_t T, int64_t D, int64_t V, bool grads) {
  Layout l{};
  int64_t at = 0;
  auto take = [&](int64_t n) {
    const int64_t here = at;
    at = up(at + n, 256);
    return here;
  };
  const int64_t g = groups_of(T, rows_of(D, V));
  l.counts = take(4 * MAX_COUNTS);
  l.ticket = take(4);
  l.scale = take(4);
  l.rows = take(4 * T);
  l.sums = take(8 * g);
  if (grads) l.part = take(4 * g * V * up(D, 16));
  l.bytes = at;
  return l;
}

template <int VT, int DT, int TB>
hipError_t launch(const Few& f, unsigned grid, bool grads, hipStream_t s) {
  // widths of DT tiles a wavefront: from the first to `most`, where rows_of gives TB
  constexpr int first = (DT - 1) * WAVES * 16 + 16, most = DT * WAVES * 16;
  if constexpr (fits(VT, TB, first) && (TB == 64 || !fits(VT, 64, most))) {
    const int bytes = words(VT, TB, f.Dp) * 4;
    auto run = [&](auto kernel) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
      if (e != hipSuccess) return e;
      kernel<<<grid, THREADS, bytes, s>>>(f);
      return hipGetLastError();
    };
    return grads ? run(k_few<VT, DT, TB, true>) : run(k_few<VT, DT, TB, false>);
  } else {
    return hipErrorInvalidConfiguration;  // no width comes here
  }
}

template <int VT, int TB>
hipError_t launch(const Few& f, unsigned grid, bool grads, hipStream_t s) {
  const int DT = (f.Dp / 16 + WAVES - 1) / WAVES;
  return DT == 1   ? launch<VT, 1, TB>(f, grid, grads, s)
         : DT == 2 ? launch<VT, 2, TB>(f, grid, grads, s)
         : DT == 3 ? launch<VT, 3, TB>(f, grid, grads, s)
                   : launch<VT, 4, TB>(f, grid, grads, s);
}

template <int TB>
hipError_t launch(const Few& f, unsigned grid, bool grads, hipStream_t s) {
  const int VT = (f.V + 15) / 16;
  return VT == 1   ? launch<1, TB>(f, grid, grads, s)
         : VT == 2 ? launch<2, TB>(f, grid, grads, s)
         : VT == 3 ? launch<3, TB>(f, grid, grads, s)
                   : launch<4, TB>(f, grid, grads, s);
}

}  // namespace

bool xent_few_fits(int64_t T, int64_t D, int64_t V) { return T > 0 && rows_of(D, V) > 0; }

int64_t xent_few_workspace(int64_t T, int64_t D, int64_t V, bool grads) { return layout_of(T, D, V, grads).bytes; }

hipError_t xent_few(const XentArgs& x, hipStream_t s) {
  const int64_t T = x.H.rows, D = x.H.cols, V = x.W.rows;
  const bool grads = x.dW.data != nullptr || x.dH.data != nullptr;
  const Layout l = layout_of(T, D, V, grads);
  char* ws = static_cast<char*>(x.ws);
  Few f{};
  f.H = x.H; f.W = x.W; f.dH = x.dH;
  f.labels = x.labels; f.i64 = x.labels_i64;
  f.counts = (const int*)(ws + l.counts);
  f.ncounts = (int)std::min<int64_t>(MAX_COUNTS, (T + COUNT_BLOCK - 1) / COUNT_BLOCK);
  f.mean = x.mean; f.grad_scale = x.grad_scale;
  f.scale = (float*)(ws + l.scale); f.loss = x.loss;
  f.row_loss = x.row_loss ? x.row_loss : (float*)(ws + l.rows);
  f.sums = (double*)(ws + l.sums); f.ticket = (uint32_t*)(ws + l.ticket);
  f.part = grads ? (float*)(ws + l.part) : nullptr;
  f.D = (int)D; f.V = (int)V; f.Dp = (int)up(D, 16);
  k_count<<<(unsigned)f.ncounts, 256, 0, s>>>(x.labels, x.labels_i64, T, V, (int*)(ws + l.counts), f.ticket);
  const int TB = rows_of(D, V);
  const unsigned grid = (unsigned)groups_of(T, TB);
  const hipError_t e = TB == 64 ? launch<64>(f, grid, grads, s) : launch<32>(f, grid, grads, s);
  if (e != hipSuccess) return e;
  if (grads) finish(f.part, (int)grid, V, D, f.Dp, f.scale, x.dW.data, x.dW.type, x.dW.ld, s);
  return hipGetLastError();
}

}  // namespace kern
}  // namespace aires
