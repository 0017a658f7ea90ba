// Losses over a layer's outputs, gradients: for one piece of the classes after the
// other, Z = F X + bias again with dZ = w (p - q) in the product's epilogue, then
// dF = dZ X^T of the piece and its share of dX = F^T dZ, which is added up in fp32.
//
// Bound by the three products: a piece of 16384 classes of 4096 features by 8192 tokens bf16
// takes 843 us with dZ, 893 for dF and 862 for dX (1300, 1230 and 1280 TFLOP/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "loss_common.h"

namespace linear {
namespace {

// dZ from partial products, and the sums of its rows over kSpan = 8 columns: 32 vectors of
// a workgroup, each of whose eight groups of 32 lanes has a column.  Bound by latency, so
// that nothing follows in one thread (64 columns a workgroup: 22 us instead of 5 at 80
// columns of 1000 classes).
template <class T> __global__ __launch_bounds__(256) void shared_dz_kernel(LossProduct p, int splits) {
  constexpr int V = kVec<T>;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, m = (blockIdx.x * 32 + x) * V, cnt = p.M - m;
  static_assert(kSpan == 8, "a column for each group of lanes");
  const int n = blockIdx.y * kSpan + y;
  float d[V];
#pragma unroll
  for (int i = 0; i < V; ++i) d[i] = 0.0f;
  if (cnt > 0 && n < p.N) {
    const float w = p.w[n], lse = p.lse[n];
    Entries entries;
    entries.find(p.y, n, w != 0.0f, p.row0 + m / kBin * kBin, kBin);
    entries.first<true>(p.y, n, p.row0 + m / kBin * kBin, 0);
    shared_logits<T, V>(p, splits, n, m, cnt, d);
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = w == 0.0f || i >= cnt ? 0.0f : w * exp_of<T>(d[i] - lse);
    entries.each<true>(p.y, n, p.row0 + m / kBin * kBin, kBin, 1, [&](int, int row, float q) {
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] -= m % kBin + i == row && i < cnt ? w * q : 0.0f;
    });
    store_vec(static_cast<T*>(p.dZ) + (int64_t)n * p.lddz + m, d);
  }
  if (!p.db) return;
  __shared__ float sh[8][32 * V];
#pragma unroll
  for (int i = 0; i < V; ++i) sh[y][x * V + i] = d[i];
  __syncthreads();
  for (int r = threadIdx.x; r < 32 * V; r += 256) {
    const int k = blockIdx.x * 32 * V + r;
    if (k >= p.M) break;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sh[i][r];
    p.db[(int64_t)blockIdx.y * p.M + k] = s;
  }
}

// Ends a wave's tile with dZ, and with the sums of its rows for dbias.  A column whose
// w is 0 is written as zeros, whatever Z is there.  dZ goes through LDS, 16 columns at a
// time, so that it is stored as whole vectors; there the targets' weights are taken off.
struct SlopeEnd {
  using P = LossProduct;
  template <class T> static hipError_t from_shares(const P& p, int splits, hipStream_t s) {
    const int width = 32 * kVec<T>;
    shared_dz_kernel<T><<<dim3((unsigned)((p.M + width - 1) / width), (unsigned)((p.N + kSpan - 1) / kSpan)), 256, 0, s>>>(p, splits);
    return hipGetLastError();
  }
  template <class T, int VA, int VB, bool STREAM, int WM, int WN>
  static __device__ void tile(const P& p, int, int m0, int n0, int lane, char* lds, f4 (&acc)[WM][WN]) {
    static_assert(VB == 1, "X's contraction is contiguous");
    constexpr int ROWS = 16 * WM, S = ROWS + 4, V = kVec<T>, PER = ROWS / V;
    if (m0 >= p.M || n0 >= p.N) return;
    float* st = reinterpret_cast<float*>(lds);
    const int q = lane >> 4, l16 = lane & 15;
    Entries entries[WN];
    float w[WN], lse[WN];
#pragma unroll
    for (int j = 0; j < WN; ++j) {
      const int n = n0 + 16 * j + l16;
      entries[j].find(p.y, n, n < p.N, p.row0 + m0, ROWS);
      w[j] = n < p.N ? p.w[n] : 0.0f;
      lse[j] = n < p.N ? p.lse[n] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < WN; ++j) entries[j].template first<true>(p.y, n0 + 16 * j + l16, p.row0 + m0, 0);
    by_plain(p, [&](auto plain) {
      if constexpr (!decltype(plain)::value) {
        float bias[WM][4];
        bias_of<T, VA>(p, m0, q, bias);
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = acc[i][j][r] * p.scale + bias[i][r];
      }
    });
    float total[V];
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < WN; ++j) {
      const int n = n0 + 16 * j + l16;
#pragma unroll
      for (int i = 0; i < WM; ++i) {
        float d[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          d[r] = w[j] == 0.0f ? 0.0f : w[j] * exp_of<T>(acc[i][j][r] - lse[j]);
        if constexpr (VA == 1) {
          *reinterpret_cast<f4*>(st + l16 * S + 16 * i + 4 * q) = f4{d[0], d[1], d[2], d[3]};
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) st[l16 * S + row_of<VA>(i, r, q)] = d[r];
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (q == 0 && w[j] != 0.0f) {               // one lane a column: equal classes one after the other
        entries[j].template each<true>(p.y, n, p.row0 + m0, ROWS, 1, [&](int, int row, float weight) { st[l16 * S + row] -= w[j] * weight; });
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int x = lane; x < PER * 16; x += 64) {
        const int col = x / PER, row = (x % PER) * V;
        const int c = n0 + 16 * j + col, m = m0 + row;
        if (c >= p.N || m >= p.M) continue;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          const f4 a = *reinterpret_cast<const f4*>(st + col * S + row + i);
          v[i] = a[0], v[i + 1] = a[1], v[i + 2] = a[2], v[i + 3] = a[3];
        }
        if (m + V > p.M) {
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = m + i < p.M ? v[i] : 0.0f;
        }
        store_vec(static_cast<T*>(p.dZ) + (int64_t)c * p.lddz + m, v);
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] += v[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (!p.db) return;
    // lanes PER apart have the same rows of other columns
#pragma unroll
    for (int d = PER; d < 64; d <<= 1)
#pragma unroll
      for (int i = 0; i < V; ++i) total[i] += __shfl_xor(total[i], d);
    float* to = p.db + (int64_t)(n0 / (16 * WN)) * p.M + m0 + lane * V;
    if (lane < PER) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (m0 + lane * V + i < p.M) to[i] = total[i];
    }
  }
};

// w of every column: g T, 0 where the column does not count, NaN where its target is
// invalid.  16-bit types (one workgroup): times the factor that puts the largest finite
// |g| T of the columns that count at 2^15; its inverse goes to `back`.  fp16: no dZ, which is
// at most |g| T, overflows, and the lower end loses at most 2^-39 of it.  Both: where every
// column has the same g, as for a mean, a target's dZ = g (p - 1) then lies just below a
// power of two unless p is large, where a rounding is relatively smallest; it has most of
// the rounding's part of the gradients' error (10007 x 1001 by 777 fp16: 2.3e-4 of the
// gradients' norm; a power of two that leaves g at 1.3 2^14: 3.5e-4; the results' own
// rounding alone: 2.1e-4).
template <bool SCALED>
__global__ __launch_bounds__(1024) void column_kernel(int t, int64_t kn, const float* __restrict__ g, int ginc, float temperature,
                                                      Targets y, float* __restrict__ w, float* __restrict__ back) {
  auto value = [&](int n) {
    const float v = g[(int64_t)n * ginc] * temperature;
    if (v == 0.0f) return 0.0f;
    if (y.label) {
      const int64_t label = label_of(y, n);
      return label == y.ignore ? 0.0f : label < 0 || label >= kn ? NAN : v;
    }
    return y.count[n] == 0 ? 0.0f : y.count[n] < 0 ? NAN : v;
  };
  float scale = 1.0f;
  if constexpr (SCALED) {
    __shared__ float sh[16];
    float top = 0.0f;
#pragma unroll 4
    for (int n = threadIdx.x; n < t; n += 1024) {
      const float v = fabsf(value(n));
      top = fmaxf(top, v < INFINITY ? v : 0.0f);
    }
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = top;
    __syncthreads();
    top = sh[threadIdx.x & 15];
    for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    // both within fp32's normal values
    if (top > 0.0f) scale = 32768.0f / fmaxf(top, 1e-33f);
    if (threadIdx.x == 0) *back = 1.0f / scale;
  }
#pragma unroll 4
  for (int64_t n = (int64_t)blockIdx.x * 1024 + threadIdx.x; n < t; n += (int64_t)gridDim.x * 1024)
    w[n] = value((int)n) * scale;
}

// X as the products take it: lines of whole vectors with zeros behind, and zeros in
// the columns with w = 0.  One read and one write.
template <class T>
__global__ __launch_bounds__(256) void input_kernel(int ci, int64_t t, const T* __restrict__ X, int64_t ldx,
                                                    const float* __restrict__ w, T* __restrict__ to, int64_t ldto) {
  constexpr int V = kVec<T>;
  const int64_t per = ldto / V, total = per * t;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
    const int64_t n = x / per;
    const int at = (int)(x - n * per) * V;
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.0f;
    if (w[n] != 0.0f) {
      const T* q = X + n * ldx + at;
      if (at + V <= ci) {
        load_vec(q, v);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (at + i < ci) v[i] = (float)q[i];
      }
    }
    store_vec(to + n * ldto + at, v);
  }
}

// dbias of a piece: its column parts added in a fixed order.
template <class T>
__global__ __launch_bounds__(256) void row_sum_kernel(int M, int parts, const float* __restrict__ part,
                                                      const float* __restrict__ back, T* __restrict__ dbias) {
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, m = blockIdx.x * 32 + x;
  __shared__ float sh[8][32];
  float s = 0.0f;
  if (m < M) {
#pragma unroll 8
    for (int i = y; i < parts; i += 8) s += part[(int64_t)i * M + m];
  }
  sh[y][x] = s;
  __syncthreads();
  if (y > 0 || m >= M) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += sh[i][x];
  if (sizeof(T) == 2) s *= *back;
  dbias[m] = (T)s;
}

// Classes of a piece: at most 8192, or as many as make 256 MB of dZ where these are more; with several
// pieces they are dealt out evenly (10007 by 8192 tokens fp32: 5120 and 4887).  A piece adds its share of dX
// to memory and starts four launches; dZ is a piece's workspace.  131072 classes by 8192
// tokens bf16, loss and gradients: 27.8 ms with 4096 classes a piece, 26.6 with 8192, 26.2
// with 16384 (256 MB), 26.1 with 32768, 25.9 with 65536 (1 GB, half of what the logits would
// take).  Multiples of 256 (whole tiles, whole bins).
constexpr int64_t kPieceRows = 8192, kPieceBytes = 256ll << 20;

int64_t piece_rows(int dtype, int64_t kn, int64_t t) {
  const int64_t most = std::min<int64_t>(1 << 20, std::max<int64_t>(kPieceRows, kPieceBytes / (std::max<int64_t>(t, 1) * type_size(dtype))));
  const int64_t pieces = std::max<int64_t>(1, ceil_div(kn, most));
  return ceil_div(std::max<int64_t>(1, ceil_div(kn, pieces)), 256) * 256;
}

// The workspace, in order, for the outputs that are wanted: one that is left out never
// adds to it.
struct Backward {
  int64_t rows = 0, pieces = 0;    // classes of a piece (the last has fewer)
  bool copy_x = false, copy_f = false;
  int64_t ldx = 0;                 // of X's copy
  int64_t lddz = 0;
  Lines x, f, d;                   // as the products find them
  int splits = 1;                  // of dX's partial products (several pieces)
  int64_t back = 0, lists = 0, xcopy = 0, fcopy = 0, dz = 0, db = 0, dx = 0, shares = 0, product = 0, bytes = 0;
};

int64_t whole(int dtype, int64_t n) { return std::max<int64_t>(padded(dtype, n), 1); }

bool far_lines(int dtype, int64_t len) {
  const int64_t n = whole(dtype, len);
  return lines_of(dtype, nullptr, n, n) == Lines::kFar;
}

// The lines of a piece of F of `rows` classes.
Lines piece_lines(int dtype, int f_order, bool copied, Lines f, int64_t ci, int64_t rows) {
  const int64_t len = whole(dtype, f_order ? ci : rows);
  return copied ? lines_of(dtype, nullptr, len, len) : f;
}

Backward backward_layout(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, Lines f, Lines x, bool want_dx,
                         bool want_df) {
  Backward w;
  const int64_t size = type_size(dtype);
  w.rows = piece_rows(dtype, kn, t);
  w.pieces = std::max<int64_t>(1, ceil_div(kn, w.rows));
  const int64_t most = std::min(kn, w.rows);
  w.ldx = whole(dtype, ci);
  w.copy_x = want_df || (x != Lines::kDirect && !far_lines(dtype, ci));
  w.x = w.copy_x ? lines_of(dtype, nullptr, w.ldx, w.ldx) : x;
  w.copy_f = f != Lines::kDirect && !far_lines(dtype, f_order ? ci : most);
  w.f = piece_lines(dtype, f_order, w.copy_f, f, ci, most);
  w.lddz = whole(dtype, most);
  w.d = lines_of(dtype, nullptr, w.lddz, w.lddz);
  w.back = up256(t * 4);
  w.lists = w.back + 256;
  w.xcopy = w.lists + (k ? list_bytes(kn, t, k) : 0);
  w.fcopy = w.xcopy + (w.copy_x ? up256(w.ldx * t * size) : 0);
  w.dz = w.fcopy + (w.copy_f ? up256((f_order ? w.ldx * most : w.lddz * ci) * size) : 0);
  w.db = w.dz + up256(w.lddz * t * size);
  int64_t parts = 0;                                        // of dbias: over the pieces' sizes
  int64_t product = 0, shares = 0;
  const int64_t last = kn - (w.pieces - 1) * w.rows;
  for (int64_t rows : {most, last}) {
    const Lines fl = piece_lines(dtype, f_order, w.copy_f, f, ci, rows);
    const LossPlan l = loss_plan(dtype, f_order == 1, fl, w.x, rows, t, ci);
    parts = std::max(parts, ceil_div(t, l.cols) * rows);
    shares = std::max(shares, share_bytes(l, rows, t));
    if (want_dx && w.pieces == 1) product = std::max(product, product_workspace(dtype, f_order == 0, true, fl, w.d, ci, t, rows));
    if (want_df)
      product = std::max(product, f_order ? product_workspace(dtype, false, false, w.x, w.d, ci, rows, t)
                                          : product_workspace(dtype, false, false, w.d, w.x, rows, ci, t));
  }
  w.dx = w.db + up256(parts * 4);
  w.product = w.dx;
  if (want_dx && w.pieces > 1) {
    w.splits = product_splits(dtype, f_order == 0, true, w.f, w.d, ci, t, most);
    w.product += up256(w.splits * ci * t * 4);
  }
  w.shares = w.product;                                     // read before the products that follow
  w.bytes = w.product + std::max(product, shares);
  return w;
}

struct Wanted {
  const float* lse;
  const float* g;
  int ginc;
  void* dX;
  int64_t lddx;
  void* dF;
  int64_t lddf;
  void* dbias;
};

Backward layout_of(const LossCall& c, const Wanted& o) {
  return backward_layout(c.dtype, c.kn, c.ci, c.t, c.f_order, c.k, lines_of(c.dtype, c.F, c.ldf, c.f_order ? c.ci : c.kn),
                         lines_of(c.dtype, c.X, c.ldx, c.ci), o.dX, o.dF);
}

template <class T> hipError_t loss_backward(const LossCall& c, const Wanted& o, char* ws, hipStream_t s) {
  const Backward w = layout_of(c, o);
  const int size = (int)sizeof(T), order = c.f_order;
  hipError_t e = hipSuccess;
  Targets y{c.labels, c.itype == LOSS_I64, c.ignore, nullptr, nullptr, nullptr, nullptr, 0, 0};
  if (c.k && c.t > 0) e = launch_lists(c, ws + w.lists, y, s);
  if (e != hipSuccess) return e;
  float* wc = reinterpret_cast<float*>(ws);
  float* back = sizeof(T) == 2 ? reinterpret_cast<float*>(ws + w.back) : nullptr;
  {
    constexpr bool scaled = sizeof(T) == 2;
    const int blocks = scaled ? 1 : (int)std::min<int64_t>(std::max<int64_t>(1, ceil_div(c.t, 1024)), 1024);
    column_kernel<scaled><<<dim3((unsigned)blocks), 1024, 0, s>>>((int)c.t, c.kn, o.g, o.ginc, (float)c.temperature, y, wc, back);
    e = hipGetLastError();
  }
  const void* X = c.X;
  int64_t ldx = c.ldx;
  int x_rows = (int)c.ci;                              // as the products load it
  if (e == hipSuccess && w.copy_x && c.t > 0 && c.ci > 0) {
    T* to = reinterpret_cast<T*>(ws + w.xcopy);
    const int64_t vecs = w.ldx / kVec<T> * c.t;
    input_kernel<T><<<dim3((unsigned)std::min<int64_t>(ceil_div(vecs, 256), 8192)), 256, 0, s>>>(
        (int)c.ci, c.t, static_cast<const T*>(c.X), c.ldx, wc, to, w.ldx);
    e = hipGetLastError();
    X = to;
    ldx = w.ldx;
    x_rows = (int)w.ldx;
  }
  Product dx{};
  for (int64_t piece = 0; piece < w.pieces && e == hipSuccess; ++piece) {
    const int64_t row0 = piece * w.rows, rows = std::min(w.rows, c.kn - row0);
    const T* F = c.F ? static_cast<const T*>(c.F) + (order ? row0 * c.ldf : row0) : nullptr;
    int64_t ldf = c.ldf;
    const int64_t line = order ? c.ci : rows, lines = order ? rows : c.ci;
    int f_line = (int)line;                            // as loaded
    if (w.copy_f && line > 0 && lines > 0) {
      const Copy copy{F, ws + w.fcopy, c.ldf, whole(c.dtype, line), lines, (int)line};
      const int blocks = (int)std::min<int64_t>(ceil_div(lines * (copy.to_ld / kVec<T>), 256), 4096);
      pad_kernel<T><<<dim3((unsigned)blocks), 256, 0, s>>>(copy, copy, blocks);
      if ((e = hipGetLastError()) != hipSuccess) break;
      F = reinterpret_cast<const T*>(ws + w.fcopy);
      ldf = copy.to_ld;
      f_line = (int)copy.to_ld;
    }
    const Lines fl = piece_lines(c.dtype, order, w.copy_f, w.f, c.ci, rows);
    const int64_t lddz = whole(c.dtype, rows);
    const Lines dl = lines_of(c.dtype, nullptr, lddz, lddz);
    char* dz = ws + w.dz;
    if (rows > 0 && c.t > 0) {
      LossProduct p{};
      p.A = F;
      p.lda = ldf;
      p.B = X;
      p.ldb = ldx;
      p.M = (int)rows;
      p.N = (int)c.t;
      p.K = (int)c.ci;
      (order ? p.aK : p.arows) = f_line;
      p.bK = x_rows;
      p.a = fl;
      p.b = w.x;
      p.bias = c.bias ? static_cast<const T*>(c.bias) + row0 : nullptr;
      p.scale = (float)(1.0 / c.temperature);
      p.row0 = row0;
      p.y = y;
      p.lse = o.lse;
      p.w = wc;
      p.dZ = dz;
      p.lddz = lddz;
      p.db = o.dbias ? reinterpret_cast<float*>(ws + w.db) : nullptr;
      p.shares = reinterpret_cast<float*>(ws + w.shares);
      if ((e = launch_loss_typed<SlopeEnd, T>(c.dtype, order == 1, p, nullptr, s)) != hipSuccess) break;
    }
    if (o.dbias && rows > 0) {
      const int parts = (int)ceil_div(c.t, loss_plan(c.dtype, order == 1, fl, w.x, rows, c.t, c.ci).cols);
      row_sum_kernel<T><<<dim3((unsigned)ceil_div(rows, 32)), 256, 0, s>>>((int)rows, parts, reinterpret_cast<const float*>(ws + w.db),
                                                                          back, static_cast<T*>(o.dbias) + row0);
      if ((e = hipGetLastError()) != hipSuccess) break;
    }
    if (o.dF) {
      // with kn fastest dZ X^T; with ci fastest its transpose X dZ^T
      Product p{};
      p.A = order ? X : dz;
      p.lda = order ? ldx : lddz;
      p.B = order ? dz : X;
      p.ldb = order ? lddz : ldx;
      p.M = (int)(order ? c.ci : rows);
      p.N = (int)(order ? rows : c.ci);
      p.K = (int)c.t;
      (order ? p.brows : p.arows) = (int)lddz;
      (order ? p.arows : p.brows) = x_rows;
      p.a = order ? w.x : dl;
      p.b = order ? dl : w.x;
      p.e.scale = back;
      p.e.C = static_cast<char*>(o.dF) + (order ? row0 * o.lddf : row0) * size;
      p.e.ldc = o.lddf;
      if ((e = launch_product(c.dtype, false, false, p, ws + w.product, s)) != hipSuccess) break;
    }
    if (o.dX) {
      Product p{};
      p.A = F;
      p.lda = ldf;
      p.B = dz;
      p.ldb = lddz;
      p.M = (int)c.ci;
      p.N = (int)c.t;
      p.K = (int)rows;
      (order ? p.arows : p.aK) = f_line;
      p.bK = (int)lddz;
      p.a = fl;
      p.b = dl;
      p.e.scale = back;
      p.e.C = o.dX;
      p.e.ldc = o.lddx;
      if (w.pieces == 1) {
        if (rows == 0) p.aK = p.bK = 0;                // no terms: zeros
        e = launch_product(c.dtype, order == 0, true, p, ws + w.product, s);
      } else {
        p.splits = w.splits;
        p.part = reinterpret_cast<float*>(ws + w.dx);
        p.add = piece > 0;
        e = launch_product_part(c.dtype, order == 0, true, p, s);
        dx = p;
      }
    }
  }
  if (e == hipSuccess && o.dX && w.pieces > 1) e = launch_product_join(c.dtype, dx, s);
  return e;
}

int backward(const LossCall& c, const Wanted& o, void* ws, hipStream_t s) {
  char* p = static_cast<char*>(ws);
  const hipError_t e = c.dtype == LINEAR_F32    ? loss_backward<float>(c, o, p, s)
                       : c.dtype == LINEAR_BF16 ? loss_backward<bf16>(c, o, p, s)
                                                : loss_backward<f16>(c, o, p, s);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}

// lse .. workspace_bytes, arguments `first` on.
int check_wanted(const LossCall& c, const Wanted& o, const void* ws, int64_t bytes, int first) {
  if (!o.lse && c.t > 0) return -first;
  if (!o.g && c.t > 0) return -(first + 1);
  if (o.ginc != 0 && o.ginc != 1) return -(first + 2);
  if (o.dX && bad_ld(o.lddx, c.ci)) return -(first + 4);
  if (o.dF && bad_ld(o.lddf, c.f_order ? c.ci : c.kn)) return -(first + 6);
  const int64_t need = layout_of(c, o).bytes;
  if (!ws || ((uintptr_t)ws & 15)) return -(first + 8);
  if (bytes < need) return -(first + 9);
  return 0;
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_linear_loss_backward_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k,
                                                          int aligned) {
  using namespace linear;
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  if (k < 0 || k > LOSS_MAX_K || t * k >= kElemLimit) return -6;
  int64_t most = 0;
  // without dF X is copied only where its lines want it
  auto take = [&](Lines f, Lines x) {
    for (int df = 0; df < 2; ++df) most = std::max(most, backward_layout(dtype, kn, ci, t, f_order, k, f, x, true, df).bytes);
  };
  if (aligned) {
    take(lines_if(dtype, true, f_order ? ci : kn), lines_if(dtype, true, ci));
  } else {
    for (Lines f : kAnyLines)
      for (Lines x : kAnyLines) take(f, x);
  }
  return most;
}

extern "C" int convgemm_linear_cross_entropy_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order,
                                                      int64_t ldf, const void* X, int64_t ldx, const void* bias,
                                                      const void* labels, int itype, int64_t ignore, const float* lse,
                                                      const float* g, int ginc, void* dX, int64_t lddx, void* dF,
                                                      int64_t lddf, void* dbias, void* workspace, int64_t workspace_bytes,
                                                      hipStream_t stream) {
  using namespace linear;
  const LossCall c{dtype, kn, ci, t, F, f_order, ldf, X, ldx, bias, labels, ignore, 0, nullptr, 0, 0, nullptr, 0, 1.0, itype};
  const Wanted o{lse, g, ginc, dX, lddx, dF, lddf, dbias};
  if (int e = check_loss_layer(c)) return e;
  if (!labels && t > 0) return -11;
  if (itype != LOSS_I32 && itype != LOSS_I64) return -12;
  if (int e = check_wanted(c, o, workspace, workspace_bytes, 14)) return e;
  return backward(c, o, workspace, stream);
}

extern "C" int convgemm_linear_distill_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order,
                                                int64_t ldf, const void* X, int64_t ldx, const void* bias, int k,
                                                const void* top, int ttype, int64_t ldtop, const void* index, int itype,
                                                int64_t ldi, double temperature, const float* lse, const float* g, int ginc,
                                                void* dX, int64_t lddx, void* dF, int64_t lddf, void* dbias, void* workspace,
                                                int64_t workspace_bytes, hipStream_t stream) {
  using namespace linear;
  const LossCall c{dtype, kn, ci, t, F, f_order, ldf, X, ldx, bias, nullptr, 0, k, top, ttype, ldtop, index, ldi, temperature, itype};
  const Wanted o{lse, g, ginc, dX, lddx, dF, lddf, dbias};
  if (int e = check_loss_layer(c)) return e;
  if (int e = check_teacher(c)) return e;
  if (int e = check_wanted(c, o, workspace, workspace_bytes, 19)) return e;
  return backward(c, o, workspace, stream);
}
