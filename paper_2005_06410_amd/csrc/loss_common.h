// Shared by the losses (loss.hip, loss_grad.hip): a column's targets, and the launch of
// the product Z = F X whose sums end in a loss instead of in memory.
#pragma once

#include "linear_common.h"
#include "linear_product.h"
#include "loss.h"

namespace linear {

// The classes of a column that have a target weight: one label, or the teacher's
// entries sorted by class.  bin[b] is the first entry of class 128 b or later, so that
// a wave (at most 128 rows, inside one bin) finds its entries with one load.
struct Targets {
  const void* label;        // t labels, or nullptr with a list
  int wide;                 // labels are 64 bits
  int64_t ignore;
  const int* index;         // [t][k]
  const float* weight;      // [t][k]
  const uint16_t* bin;      // [t][bins + 1]
  const int* count;         // [t]: entries that count, or -1 where one is invalid
  int k, bins;
};

constexpr int kBin = 128;

// Columns of one workgroup that goes on from partial products.
constexpr int kSpan = 8;

__device__ inline int64_t label_of(const Targets& y, int n) {
  return y.wide ? static_cast<const int64_t*>(y.label)[n] : (int64_t)static_cast<const int*>(y.label)[n];
}

// The entries of one column among the classes c0 .. c0 + rows of a wave, one lane taking
// every step-th from the `from`-th on; the row and weight of its first are loaded ahead (the
// row lies outside 0 .. rows for a neighbour in its bin).
struct Entries {
  int lo, hi;
  int64_t row;
  float weight;

  // Asks for column n's entries; nothing where it is not `there`.
  __device__ void find(const Targets& y, int n, bool there, int64_t c0, int rows) {
    lo = hi = 0;
    row = -1;
    weight = 1.0f;
    if (!there) return;
    if (y.label) {
      row = label_of(y, n) - c0;
      hi = row >= 0 && row < rows;
    } else {
      const uint16_t* b = y.bin + (int64_t)n * (y.bins + 1) + c0 / kBin;
      lo = b[0];
      hi = b[1];
    }
  }
  // The first entry itself, by a list; for several columns after find() of all, so that
  // their loads wait together.
  template <bool WEIGHT> __device__ void first(const Targets& y, int n, int64_t c0, int from) {
    lo += from;
    if (!y.label && lo < hi) {
      row = (int64_t)y.index[(int64_t)n * y.k + lo] - c0;
      if (WEIGHT) weight = y.weight[(int64_t)n * y.k + lo];
    }
  }
  // f(entry, row, weight) for those that are in the rows
  template <bool WEIGHT, class F> __device__ void each(const Targets& y, int n, int64_t c0, int rows, int step, F f) const {
    int64_t r = row;
    float w = weight;
    for (int e = lo; e < hi; e += step) {
      if (e > lo) {
        r = (int64_t)y.index[(int64_t)n * y.k + e] - c0;
        if (WEIGHT) w = y.weight[(int64_t)n * y.k + e];
      }
      if (r >= 0 && r < rows) f(e, (int)r, w);
    }
  }
};

// Z (M x N) = F X + bias for one piece of the classes, times 1 / T.
struct LossProduct : Product {
  const void* bias;         // M values or nullptr
  float scale;              // 1 / T
  int64_t row0;             // the piece's first class
  Targets y;
  // forward: maximum and sum of exponentials of each wave's rows, [row parts][N], and
  // the targets' logits, [N] or [N][k]
  float2* sums;
  float* at;
  // gradients
  const float* lse;         // N
  const float* w;           // N: g T (16-bit types: times a factor for all); 0 where nothing counts
  void* dZ;
  int64_t lddz;             // M rounded up to whole vectors
  float* db;                // [column parts][M] sums of dZ's rows, or nullptr
  // where workgroups share contractions: [splits][N][M] partial products, and what the
  // forward call gives
  float* shares;
  int64_t kn;
  float temperature2;
  float* loss;
  float* lse_out;
};

namespace {

// The row of a wave's tile that acc[i][.][r] holds in lane group q: as write_tile()
// lays them out.
template <int VA> __device__ inline int row_of(int i, int r, int q) {
  return VA == 1 ? 16 * i + 4 * q + r : 16 * (i / VA * VA) + VA * (4 * q + r) + i % VA;
}

template <class END, class R> __global__ __launch_bounds__(R::NT, 2) void loss_ring_kernel(LossProduct p) {
  R::template run<END>(p);
}
template <class END, class T, bool AKC> __global__ __launch_bounds__(512) void loss_wide_kernel(LossProduct p) {
  wide_run<T, AKC, true, false, END>(p);
}

// f(whether Z / T is the sums as they are)
template <class F> __device__ inline void by_plain(const LossProduct& p, F f) {
  if (!p.bias && p.scale == 1.0f)
    f(std::integral_constant<bool, true>{});
  else
    f(std::integral_constant<bool, false>{});
}

// bias / T of a lane's rows, zeros without one.
template <class T, int VA, int WM> __device__ inline void bias_of(const LossProduct& p, int m0, int q, float (&bias)[WM][4]) {
  const T* b = static_cast<const T*>(p.bias);
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) bias[i][r] = b ? p.scale * (float)b[min(m0 + row_of<VA>(i, r, q), p.M - 1)] : 0.0f;
}

// Z / T of the cnt >= 1 classes m .. m + V of column n from partial products, -inf for
// those behind.
template <class T, int V> __device__ inline void shared_logits(const LossProduct& p, int splits, int n, int m, int cnt, float* z) {
  const float* from = p.shares + (int64_t)n * p.M + m;
#pragma unroll
  for (int i = 0; i < V; ++i) z[i] = 0.0f;
  for (int k = 0; k < splits; ++k, from += (int64_t)p.N * p.M) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      if (cnt >= V) {
        float w[4];
        load_vec(from + i, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i + j] += w[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i + j] += from[min(i + j, cnt - 1)];
      }
    }
  }
  const T* b = static_cast<const T*>(p.bias);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    z[i] = z[i] * p.scale + (b ? p.scale * (float)b[m + min(i, cnt - 1)] : 0.0f);
    if (i >= cnt) z[i] = -INFINITY;
  }
}

// How a piece's product is computed.  Its sums end in the kernel where they are whole;
// where workgroups share the contractions of a small product, they are written as partial
// products (fp32) and a second kernel goes on from these.
struct LossPlan {
  Route route;
  Shape shape;
  int rows, cols;           // of a wave's tile (cols of the second kernel where splits > 1)
  int splits;
};

// 80 columns of 1000 classes from 4096 features, fp32: 33 us whole, 15 + 4 in four shares.
// The second kernel takes a workgroup for each column, so that columns are to be neither few nor long.
LossPlan loss_plan(int dtype, bool a_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K) {
  static constexpr int wm[kShapes] = {8, 4, 4, 4, 2, 2, 2, 4, 4, 1, 2, 1}, wn[kShapes] = {4, 4, 2, 2, 2, 2, 2, 2, 1, 1, 5, 5};
  LossPlan l;
  l.route = route_of(dtype, a_kc, true, a, b, M, N, K, false);
  l.shape = kSquare2;
  l.splits = 1;
  if (l.route.width == 0) {
    l.rows = 64;
    l.cols = N > 64 ? 64 : N <= 16 ? 16 : 64;
    return l;
  }
  const Plan whole = plan_of(dtype, 16, a_kc, true, M, N, K, true);
  if (N >= 32 && M <= 8192) {
    const Plan shared = plan_of(dtype, 16, a_kc, true, M, N, K);
    if (shared.splits > 1 && shared.us < whole.us) {
      l.splits = shared.splits;
      l.rows = kBin;
      l.cols = kSpan;
      return l;
    }
  }
  l.shape = whole.shape;
  l.rows = 16 * wm[l.shape];
  l.cols = 16 * wn[l.shape];
  return l;
}

int64_t share_bytes(const LossPlan& l, int64_t M, int64_t N) { return l.splits > 1 ? up256(l.splits * M * N * 4) : 0; }

template <class END, class R> hipError_t launch_loss_ring(LossProduct p, hipStream_t s) {
  p.mtiles = (p.M + R::MT - 1) / R::MT;
  p.ntiles = (p.N + R::NTILE - 1) / R::NTILE;
  const hipError_t e = ltlt::ensure_dynamic_lds((const void*)loss_ring_kernel<END, R>, R::LDS);
  if (e != hipSuccess) return e;
  loss_ring_kernel<END, R><<<dim3((unsigned)((int64_t)p.mtiles * p.ntiles)), R::NT, R::LDS, s>>>(p);
  return hipGetLastError();
}

template <class END, class T, bool AKC> hipError_t launch_loss_shape(Shape shape, LossProduct p, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (shape == kWide) {
      p.mtiles = (p.M + 255) / 256;
      p.ntiles = (p.N + 255) / 256;
      auto k = loss_wide_kernel<END, T, AKC>;
      const hipError_t e = ltlt::ensure_dynamic_lds((const void*)k, 2 * kWideBuffer);
      if (e != hipSuccess) return e;
      k<<<dim3((unsigned)((int64_t)p.mtiles * p.ntiles)), 512, 2 * kWideBuffer, s>>>(p);
      return hipGetLastError();
    }
  } else {
    if (shape == kSlim80) return launch_loss_ring<END, Ring<T, AKC, true, 1, 5, 1, 1, 8, 4, 3, 16>>(p, s);
    if (shape == kRow80) return launch_loss_ring<END, Ring<T, AKC, true, 2, 5, 1, 1, 4, 2, 2, 16>>(p, s);
  }
  if (shape == kSquare4) return launch_loss_ring<END, Ring<T, AKC, true, 4, 2, 2, 4, 1, 1, 4, 16>>(p, s);
  if (shape == kTall) return launch_loss_ring<END, Ring<T, AKC, true, 4, 2, 2, 2, 1, 1, 3, 16>>(p, s);
  if (shape == kSmall) return launch_loss_ring<END, Ring<T, AKC, true, 2, 2, 2, 2, 1, 1, 4, 16>>(p, s);
  if (shape == kQuad64) return launch_loss_ring<END, Ring<T, AKC, true, 2, 2, 2, 2, 2, 2, 4, 16>>(p, s);
  if (shape == kBlock32) return launch_loss_ring<END, Ring<T, AKC, true, 2, 2, 1, 1, 4, 4, 4, 16>>(p, s);
  if (shape == kNarrow32) return launch_loss_ring<END, Ring<T, AKC, true, 4, 2, 1, 1, 4, 4, 3, 16>>(p, s);
  if (shape == kNarrow16) return launch_loss_ring<END, Ring<T, AKC, true, 4, 1, 1, 1, 4, 4, 3, 16>>(p, s);
  if constexpr (AKC) {
    if (shape == kThin16) return launch_loss_ring<END, Ring<T, AKC, true, 1, 1, 1, 1, 8, 8, 4, 16>>(p, s);
  }
  return launch_loss_ring<END, Ring<T, AKC, true, 4, 4, 2, 2, 1, 1, 2, 16>>(p, s);
}

template <class END, class T, bool AKC> hipError_t launch_loss_registers(const LossProduct& p, hipStream_t s) {
  if (p.N > 64) return launch_loss_ring<END, Ring<T, AKC, true, 4, 4, 2, 2, 1, 1, 2, 0>>(p, s);
  if (p.N <= 16) return launch_loss_ring<END, Ring<T, AKC, true, 4, 1, 1, 1, 4, 4, 2, 0>>(p, s);
  return launch_loss_ring<END, Ring<T, AKC, true, 4, 4, 1, 1, 4, 4, 2, 0>>(p, s);
}

// The product and its end; copies of operands that need them go to `ws`.
template <class END, class T> hipError_t launch_loss_typed(int dtype, bool a_kc, LossProduct p, char* ws, hipStream_t s) {
  const LossPlan l = loss_plan(dtype, a_kc, p.a, p.b, p.M, p.N, p.K);
  p.splits = 1;
  p.part = nullptr;
  set_extents(p);
  if (l.route.width == 0) {
    true_extents(p);
    return a_kc ? launch_loss_registers<END, T, true>(p, s) : launch_loss_registers<END, T, false>(p, s);
  }
  hipError_t e = copy_operands<T>(dtype, l.route, a_kc, true, p, ws, s);
  if (e != hipSuccess) return e;
  if (l.splits > 1) {
    Product part = p;
    part.splits = l.splits;
    part.part = p.shares;
    part.a = part.b = Lines::kDirect;
    e = launch_product_part(dtype, a_kc, true, part, s);
    return e == hipSuccess ? END::template from_shares<T>(p, l.splits, s) : e;
  }
  return a_kc ? launch_loss_shape<END, T, true>(l.shape, p, s) : launch_loss_shape<END, T, false>(l.shape, p, s);
}

template <class END> hipError_t launch_loss(int dtype, bool a_kc, const LossProduct& p, char* ws, hipStream_t s) {
  switch (dtype) {
    case LINEAR_F32: return launch_loss_typed<END, float>(dtype, a_kc, p, ws, s);
    case LINEAR_BF16: return launch_loss_typed<END, bf16>(dtype, a_kc, p, ws, s);
    default: return launch_loss_typed<END, f16>(dtype, a_kc, p, ws, s);
  }
}

}  // namespace

// loss.hip.  A call's arguments that both directions have, and their checks.
struct LossCall {
  int dtype;
  int64_t kn, ci, t;
  const void* F;
  int f_order;
  int64_t ldf;
  const void* X;
  int64_t ldx;
  const void* bias;
  // labels
  const void* labels;
  int64_t ignore;
  // teacher (k > 0)
  int k;
  const void* top;
  int ttype;
  int64_t ldtop;
  const void* index;
  int64_t ldi;
  double temperature;
  int itype;
};

// 0, or the argument's number (negative) of dtype .. bias (arguments 1 .. 10).
int check_loss_layer(const LossCall& c);
// The same from k on (argument 11).
int check_teacher(const LossCall& c);

// The teacher's lists in a workspace: bytes, and the launch that makes them.
int64_t list_bytes(int64_t kn, int64_t t, int k);
hipError_t launch_lists(const LossCall& c, char* ws, Targets& y, hipStream_t s);

}  // namespace linear
