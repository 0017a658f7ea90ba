// Losses over a layer's outputs, forward: Z = F X + bias is never written; each wave
// ends its tile with the maximum and the sum of exponentials of its rows, and with the
// targets' logits; a second launch joins the waves' parts of a column.
//
// Bound by the matrix cores where there are many columns (131072 classes of 4096
// features by 8192 tokens bf16: 6.3 to 6.5 ms, 1350 to 1390 TFLOP/s; what a tile's end adds to
// the product is an exponential, a maximum and three additions or products a logit, about 5 us of a
// 256 x 256 tile's 99), by one read of the weights where there are few (32000 x 4096 bf16 by
// one token: 48 us and 5 for the second launch, 5.4 TB/s; 131072 x 4096 by 16: 6.0 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "loss_common.h"

namespace linear {
namespace {

// Where maxima are infinite, exponentials are taken without one: exp(+inf) = inf and
// exp(-inf) = 0 are then what the formula says, and nothing is inf - inf.
__device__ inline float base_of(float top) { return fabsf(top) < INFINITY ? top : 0.0f; }

// The loss of one column a workgroup from partial products.
template <class T> __global__ __launch_bounds__(256) void shared_loss_kernel(LossProduct p, int splits) {
  __shared__ float sh[4];
  const int n = blockIdx.x;
  auto over = [&](float v, auto f) {
    for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return f(f(sh[0], sh[1]), f(sh[2], sh[3]));
  };
  auto most = [](float a, float b) { return fmaxf(a, b); };
  auto plus = [](float a, float b) { return a + b; };
  float top = -INFINITY, sum = 0.0f;
  for (int m = threadIdx.x * 4; m < p.M; m += 1024) {
    float z[4];
    shared_logits<T, 4>(p, splits, n, m, p.M - m, z);
    const float t = fmaxf(top, fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
    sum = top == -INFINITY ? sum : sum * expf(base_of(top) - base_of(t));
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += expf(z[i] - base_of(t));
    top = t;
  }
  const float all = over(top, most);
  sum = over(top == -INFINITY ? sum : sum * expf(base_of(top) - base_of(all)), plus);
  const float l = base_of(all) + logf(sum);
  if (threadIdx.x == 0) p.lse_out[n] = l;
  auto logit = [&](int64_t c) {
    float z[4];
    shared_logits<T, 4>(p, splits, n, (int)c, 1, z);
    return z[0];
  };
  if (p.y.label) {
    const int64_t label = label_of(p.y, n);
    if (threadIdx.x == 0) p.loss[n] = label == p.y.ignore ? 0.0f : label >= 0 && label < p.kn ? l - logit(label) : NAN;
    return;
  }
  const int count = p.y.count[n];
  float v = 0.0f;
  for (int e = threadIdx.x; e < count; e += 256) {
    const int64_t i = (int64_t)n * p.y.k + e;
    const float w = p.y.weight[i];
    v += w == 0.0f ? 0.0f : w * (logf(w) - (logit(p.y.index[i]) - l));
  }
  v = over(v, plus);
  if (threadIdx.x == 0) p.loss[n] = count < 0 ? NAN : count == 0 ? 0.0f : p.temperature2 * v;
}

// Ends a wave's tile with its columns' statistics.
struct StatsEnd {
  using P = LossProduct;
  template <class T> static hipError_t from_shares(const P& p, int splits, hipStream_t s) {
    shared_loss_kernel<T><<<dim3((unsigned)p.N), 256, 0, s>>>(p, splits);
    return hipGetLastError();
  }
  template <class T, int VA, int VB, bool STREAM, int WM, int WN>
  static __device__ void tile(const P& p, int, int m0, int n0, int lane, char* lds, f4 (&acc)[WM][WN]) {
    static_assert(VB == 1, "X's contraction is contiguous");
    constexpr int ROWS = 16 * WM, S = ROWS + 4;
    if (m0 >= p.M) return;
    const int q = lane >> 4, l16 = lane & 15;
    Entries entries[WN];
#pragma unroll
    for (int j = 0; j < WN; ++j) entries[j].find(p.y, n0 + 16 * j + l16, n0 + 16 * j + l16 < p.N, p.row0 + m0, ROWS);
#pragma unroll
    for (int j = 0; j < WN; ++j) entries[j].template first<false>(p.y, n0 + 16 * j + l16, p.row0 + m0, q);
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
    if (m0 + ROWS > p.M) {
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (m0 + row_of<VA>(i, r, q) >= p.M) {
#pragma unroll
            for (int j = 0; j < WN; ++j) acc[i][j][r] = -INFINITY;
          }
    }
#pragma unroll
    for (int j = 0; j < WN; ++j) {
      const int n = n0 + 16 * j + l16;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float base = base_of(top);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += exp_of<T>(acc[i][j][r] - base);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (q == 0 && n < p.N) p.sums[(int64_t)(m0 / ROWS) * p.N + n] = float2{top, sum};
      if (__any(entries[j].lo < entries[j].hi)) {
        // a target's logit lies in some lane's register; through LDS it is one read away
        float* st = reinterpret_cast<float*>(lds) + l16 * S;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
          if constexpr (VA == 1) {
            *reinterpret_cast<f4*>(st + 16 * i + 4 * q) = acc[i][j];
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) st[row_of<VA>(i, r, q)] = acc[i][j][r];
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        entries[j].template each<false>(p.y, n, p.row0 + m0, ROWS, 4, [&](int e, int row, float) {
          p.at[p.y.label ? (int64_t)n : (int64_t)n * p.y.k + e] = st[row];
        });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
};

// Joins the parts of C columns a workgroup, 256 / C lanes for each, in a fixed order:
//   lse = base + log sum exp(top_r - base) sum_r,
// then the loss.  Bound by latency: 18 us for 1024 parts of 8192 columns (67 MB), 4.6 for
// 500 of one; eight parts under way in each lane (one after the other: 42 us), and few
// columns a workgroup where there are few at all (300 columns of 782 parts by 4: 5.8 us; by
// 16 more than twice as long).
template <int C>
__global__ __launch_bounds__(256) void join_loss_kernel(int parts, int N, int64_t kn, const float2* __restrict__ sums,
                                                        const float* __restrict__ at, Targets y, float temperature2,
                                                        float* __restrict__ loss, float* __restrict__ lse) {
  constexpr int LANES = 256 / C, AHEAD = 8;
  __shared__ float sh[2][4][C];
  const int c = threadIdx.x % C, x = threadIdx.x / C, n = blockIdx.x * C + c, wave = threadIdx.x >> 6;
  const bool there = n < N;
  // over a column's lanes, C apart; `at` is another place in LDS than the call before
  auto over = [&](float v, int at, auto f) {
#pragma unroll
    for (int d = C; d < 64; d <<= 1) v = f(v, __shfl_xor(v, d));
    if ((threadIdx.x & 63) < C) sh[at][wave][c] = v;
    __syncthreads();
    return f(f(sh[at][0][c], sh[at][1][c]), f(sh[at][2][c], sh[at][3][c]));
  };
  // what the loss needs besides, asked for before the parts
  const int64_t label = y.label && there ? label_of(y, n) : -1;
  const int count = !y.label && there ? y.count[n] : 0;
  const int64_t entry = (int64_t)n * y.k + x;
  const float own = y.label ? (label >= 0 && label < kn ? at[n] : NAN) : x < count ? at[entry] : 0.0f;
  const float own_weight = x < count ? y.weight[entry] : 0.0f;
  const float2* s = sums + min(n, N - 1);
  float top = -INFINITY, sum = 0.0f;               // of this lane: sum is relative to top
  for (int r0 = x; r0 < parts; r0 += AHEAD * LANES) {
    float2 v[AHEAD];
    float t = top;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int r = r0 + k * LANES;
      v[k] = s[(int64_t)min(r, parts - 1) * N];
      if (r >= parts) v[k] = float2{-INFINITY, 0.0f};
      t = fmaxf(t, v[k].x);
    }
    // a part of -inf alone has the sum 0 (or NaN), whatever it is taken relative to
    sum = top == -INFINITY ? sum : sum * expf(base_of(top) - base_of(t));
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) sum += v[k].x == -INFINITY ? v[k].y : v[k].y * expf(base_of(v[k].x) - base_of(t));
    top = t;
  }
  const float all = over(top, 0, [](float a, float b) { return fmaxf(a, b); });
  sum = over(top == -INFINITY ? sum : sum * expf(base_of(top) - base_of(all)), 1, [](float a, float b) { return a + b; });
  const float l = base_of(all) + logf(sum);
  if (y.label) {
    if (!there || x > 0) return;
    lse[n] = l;
    loss[n] = label == y.ignore ? 0.0f : l - own;
    return;
  }
  float v = 0.0f, w = own_weight, z = own;
  for (int e = x; e < count; e += LANES) {
    if (e > x) {
      w = y.weight[entry + e - x];
      z = at[entry + e - x];
    }
    v += w == 0.0f ? 0.0f : w * (logf(w) - (z - l));
  }
  v = over(v, 0, [](float a, float b) { return a + b; });
  if (!there || x > 0) return;
  lse[n] = l;
  loss[n] = count < 0 ? NAN : count == 0 ? 0.0f : temperature2 * v;
}

// The teacher of one column, by one wave: its entries sorted by class (a bitonic
// network over class and place, so that equal classes keep their order), the weights
// q in fp32, and the first entry of every 128 classes, by which a wave of the product finds
// its targets with one load instead of a search.  4096 columns of 64 entries, 32000 classes:
// 17 us of 3400; 300 of 17, 50021 classes: 8.
template <class TT>
__global__ __launch_bounds__(64) void list_kernel(int64_t kn, int k, int size, const TT* __restrict__ top, int64_t ldtop,
                                                  const void* __restrict__ index, int64_t ldi, int wide, float scale, int bins,
                                                  int* __restrict__ sorted, float* __restrict__ weight,
                                                  uint16_t* __restrict__ bin, int* __restrict__ count) {
  __shared__ uint64_t key[LOSS_MAX_K];
  __shared__ float value[LOSS_MAX_K];
  const int64_t n = blockIdx.x;
  const int lane = threadIdx.x;
  float best = -INFINITY;
  bool bad = false;
  int valid = 0;
  for (int e = lane; e < size; e += 64) {
    uint64_t at = ~0ull;
    float v = -INFINITY;
    if (e < k) {
      const int64_t i = wide ? static_cast<const int64_t*>(index)[n * ldi + e] : (int64_t)static_cast<const int*>(index)[n * ldi + e];
      v = (float)top[n * ldtop + e];
      if (i >= 0 && v != -INFINITY) {
        ++valid;
        bad |= i >= kn;
        at = (uint64_t)min(i, kn) << 16 | (uint64_t)e;
        best = fmaxf(best, v);
      }
    }
    key[e] = at;
    value[e] = v;
  }
  for (int d = 32; d > 0; d >>= 1) {
    best = fmaxf(best, __shfl_xor(best, d));
    valid += __shfl_xor(valid, d);
  }
  bad = __any(bad);
  __syncthreads();
  for (int outer = 2; outer <= size; outer <<= 1)
    for (int d = outer >> 1; d > 0; d >>= 1) {
      for (int i = lane; i < size / 2; i += 64) {
        const int a = 2 * i - (i & (d - 1)), b = a + d;
        const uint64_t x = key[a], y = key[b];
        if ((x > y) == ((a & outer) == 0)) key[a] = y, key[b] = x;
      }
      __syncthreads();
    }
  float sum = 0.0f;
  for (int e = lane; e < valid; e += 64) sum += expf((value[key[e] & 0xffff] - best) * scale);
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  for (int e = lane; e < valid; e += 64) {
    sorted[n * k + e] = (int)(key[e] >> 16);
    weight[n * k + e] = expf((value[key[e] & 0xffff] - best) * scale) / sum;
  }
  uint16_t* out = bin + n * (bins + 1);
  for (int b = lane; b <= bins; b += 64) {
    int lo = 0, hi = valid;                   // the first entry of class 128 b or later
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if ((int64_t)(key[mid] >> 16) < (int64_t)b * kBin)
        lo = mid + 1;
      else
        hi = mid;
    }
    out[b] = (uint16_t)lo;
  }
  if (lane == 0) count[n] = bad ? -1 : valid;
}

struct Forward {
  LossPlan plan;
  int64_t sums, at, lists, shares, bytes;   // byte offsets; copies first
  int parts;
};

Forward forward_layout(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, Lines f, Lines x) {
  Forward w{};
  w.plan = loss_plan(dtype, f_order == 1, f, x, kn, t, ci);
  w.parts = (int)ceil_div(kn, w.plan.rows);
  if (w.plan.route.copy_a) w.sums += up256(copy_values(dtype, f_order == 1, kn, ci) * type_size(dtype));
  if (w.plan.route.copy_b) w.sums += up256(copy_values(dtype, true, t, ci) * type_size(dtype));
  const bool whole = w.plan.splits == 1;
  w.at = w.sums + (whole ? up256((int64_t)w.parts * t * 8) : 0);
  w.lists = w.at + (whole ? up256(t * std::max(k, 1) * 4) : 0);
  w.shares = w.lists + (k ? list_bytes(kn, t, k) : 0);
  w.bytes = w.shares + share_bytes(w.plan, kn, t);
  return w;
}

// Columns of one round: all of them, but for so many logits that a launch would hold more
// threads than 32 bits count, or the parts of the columns more memory than the operands.
int64_t round_columns(int64_t kn, int64_t t) {
  return kn * t <= 1ll << 33 ? t : std::max<int64_t>(4096, (1ll << 33) / kn / 256 * 256);
}

int forward_round(const LossCall& c, float* loss, float* lse, char* ws, hipStream_t s) {
  const Lines f = lines_of(c.dtype, c.F, c.ldf, c.f_order ? c.ci : c.kn), x = lines_of(c.dtype, c.X, c.ldx, c.ci);
  const Forward w = forward_layout(c.dtype, c.kn, c.ci, c.t, c.f_order, c.k, f, x);
  LossProduct p{};
  p.A = c.F;
  p.lda = c.ldf;
  p.B = c.X;
  p.ldb = c.ldx;
  p.M = (int)c.kn;
  p.N = (int)c.t;
  p.K = (int)c.ci;
  p.a = f;
  p.b = x;
  p.bias = c.bias;
  p.scale = (float)(1.0 / c.temperature);
  p.sums = reinterpret_cast<float2*>(ws + w.sums);
  p.at = reinterpret_cast<float*>(ws + w.at);
  p.shares = reinterpret_cast<float*>(ws + w.shares);
  p.kn = c.kn;
  p.temperature2 = (float)(c.temperature * c.temperature);
  p.loss = loss;
  p.lse_out = lse;
  hipError_t e = hipSuccess;
  if (c.k)
    e = launch_lists(c, ws + w.lists, p.y, s);
  else
    p.y = Targets{c.labels, c.itype == LOSS_I64, c.ignore, nullptr, nullptr, nullptr, nullptr, 0, 0};
  if (e == hipSuccess && c.kn > 0) e = launch_loss<StatsEnd>(c.dtype, c.f_order == 1, p, ws, s);
  if (e != hipSuccess) return LINEAR_ERR_HIP_BASE - (int)e;
  if (w.plan.splits > 1) return LINEAR_OK;
  auto join = [&](auto kernel, int columns) {
    kernel<<<dim3((unsigned)((c.t + columns - 1) / columns)), 256, 0, s>>>(w.parts, p.N, c.kn, p.sums, p.at, p.y, p.temperature2, loss, lse);
  };
  if (c.t >= 2048)
    join(join_loss_kernel<16>, 16);
  else if (c.t >= 64)
    join(join_loss_kernel<4>, 4);
  else
    join(join_loss_kernel<1>, 1);
  e = hipGetLastError();
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}

int loss_forward(const LossCall& all, float* loss, float* lse, char* ws, hipStream_t s) {
  const int64_t step = round_columns(all.kn, all.t), size = type_size(all.dtype), isize = all.itype == LOSS_I64 ? 8 : 4;
  auto ahead = [](const void* p, int64_t bytes) { return p ? static_cast<const void*>(static_cast<const char*>(p) + bytes) : p; };
  for (int64_t n = 0; n < all.t; n += step) {
    LossCall c = all;
    c.t = std::min(step, all.t - n);
    c.X = ahead(all.X, n * all.ldx * size);
    c.labels = ahead(all.labels, n * isize);
    c.top = ahead(all.top, all.k ? n * all.ldtop * type_size(all.ttype) : 0);
    c.index = ahead(all.index, n * all.ldi * isize);
    if (int e = forward_round(c, loss + n, lse + n, ws, s)) return e;
  }
  return LINEAR_OK;
}

// The bytes for all rounds: the last one has fewer columns, and with them another plan.
int64_t forward_bytes(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, Lines f, Lines x) {
  const int64_t step = round_columns(kn, t), last = t > step ? (t - 1) % step + 1 : step;
  return std::max(forward_layout(dtype, kn, ci, step, f_order, k, f, x).bytes, forward_layout(dtype, kn, ci, last, f_order, k, f, x).bytes);
}

// Every round's X has the first one's lines: they begin whole leading dimensions apart.
int64_t need_of(const LossCall& c) {
  return forward_bytes(c.dtype, c.kn, c.ci, c.t, c.f_order, c.k, lines_of(c.dtype, c.F, c.ldf, c.f_order ? c.ci : c.kn),
                       lines_of(c.dtype, c.X, c.ldx, c.ci));
}

}  // namespace

int check_loss_layer(const LossCall& c) {
  if (int e = check_sizes(c.dtype, c.kn, c.ci, c.t)) return e;
  const bool work = c.kn > 0 && c.ci > 0 && c.t > 0;
  if (!c.F && work) return -5;
  if (c.f_order != 0 && c.f_order != 1) return -6;
  if (bad_ld(c.ldf, c.f_order ? c.ci : c.kn)) return -7;
  if (!c.X && work) return -8;
  if (bad_ld(c.ldx, c.ci)) return -9;
  return 0;
}

int check_teacher(const LossCall& c) {
  if (c.k < 1 || c.k > LOSS_MAX_K || c.t * c.k >= kElemLimit) return -11;
  if (!c.top && c.t > 0) return -12;
  if (!is_type(c.ttype)) return -13;
  if (bad_ld(c.ldtop, c.k)) return -14;
  if (!c.index && c.t > 0) return -15;
  if (c.itype != LOSS_I32 && c.itype != LOSS_I64) return -16;
  if (bad_ld(c.ldi, c.k)) return -17;
  if (!(c.temperature > 0) || !std::isfinite((float)c.temperature) || !std::isfinite((float)(1.0 / c.temperature)) ||
      !std::isnormal((float)(c.temperature * c.temperature)))
    return -18;
  return 0;
}

int64_t list_bytes(int64_t kn, int64_t t, int k) {
  const int64_t bins = ceil_div(kn, kBin);
  return 2 * up256(t * k * 4) + up256(t * (bins + 1) * 2) + up256(t * 4);
}

hipError_t launch_lists(const LossCall& c, char* ws, Targets& y, hipStream_t s) {
  const int64_t bins = ceil_div(c.kn, kBin);
  int* sorted = reinterpret_cast<int*>(ws);
  ws += up256(c.t * c.k * 4);
  float* weight = reinterpret_cast<float*>(ws);
  ws += up256(c.t * c.k * 4);
  uint16_t* bin = reinterpret_cast<uint16_t*>(ws);
  ws += up256(c.t * (bins + 1) * 2);
  int* count = reinterpret_cast<int*>(ws);
  y = Targets{nullptr, 0, 0, sorted, weight, bin, count, c.k, (int)bins};
  int size = 2;
  while (size < c.k) size *= 2;
  auto launch = [&](auto* top) {
    list_kernel<<<dim3((unsigned)c.t), 64, 0, s>>>(c.kn, c.k, size, top, c.ldtop, c.index, c.ldi, c.itype == LOSS_I64,
                                                   (float)(1.0 / c.temperature), (int)bins, sorted, weight, bin, count);
    return hipGetLastError();
  };
  switch (c.ttype) {
    case LINEAR_F32: return launch(static_cast<const float*>(c.top));
    case LINEAR_BF16: return launch(static_cast<const bf16*>(c.top));
    default: return launch(static_cast<const f16*>(c.top));
  }
}

}  // namespace linear

extern "C" int64_t convgemm_linear_loss_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, int aligned) {
  using namespace linear;
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  if (k < 0 || k > LOSS_MAX_K || t * k >= kElemLimit) return -6;
  if (t == 0) return 0;
  if (aligned)
    return forward_bytes(dtype, kn, ci, t, f_order, k, lines_if(dtype, true, f_order ? ci : kn), lines_if(dtype, true, ci));
  int64_t most = 0;
  for (Lines f : kAnyLines)
    for (Lines x : kAnyLines) most = std::max(most, forward_bytes(dtype, kn, ci, t, f_order, k, f, x));
  return most;
}

extern "C" int convgemm_linear_cross_entropy(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order,
                                             int64_t ldf, const void* X, int64_t ldx, const void* bias, const void* labels,
                                             int itype, int64_t ignore, float* loss, float* lse, void* workspace,
                                             int64_t workspace_bytes, hipStream_t stream) {
  using namespace linear;
  const LossCall c{dtype, kn, ci, t, F, f_order, ldf, X, ldx, bias, labels, ignore, 0, nullptr, 0, 0, nullptr, 0, 1.0, itype};
  if (int e = check_loss_layer(c)) return e;
  if (!labels && t > 0) return -11;
  if (itype != LOSS_I32 && itype != LOSS_I64) return -12;
  if (!loss && t > 0) return -14;
  if (!lse && t > 0) return -15;
  if (t == 0) return LINEAR_OK;
  if (!workspace || ((uintptr_t)workspace & 15)) return -16;
  if (workspace_bytes < need_of(c)) return -17;
  return loss_forward(c, loss, lse, static_cast<char*>(workspace), stream);
}

extern "C" int convgemm_linear_distill(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                                       const void* X, int64_t ldx, const void* bias, int k, const void* top, int ttype,
                                       int64_t ldtop, const void* index, int itype, int64_t ldi, double temperature,
                                       float* loss, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  using namespace linear;
  const LossCall c{dtype, kn, ci, t, F, f_order, ldf, X, ldx, bias, nullptr, 0, k, top, ttype, ldtop, index, ldi, temperature, itype};
  if (int e = check_loss_layer(c)) return e;
  if (int e = check_teacher(c)) return e;
  if (!loss && t > 0) return -19;
  if (!lse && t > 0) return -20;
  if (t == 0) return LINEAR_OK;
  if (!workspace || ((uintptr_t)workspace & 15)) return -21;
  if (workspace_bytes < need_of(c)) return -22;
  return loss_forward(c, loss, lse, static_cast<char*>(workspace), stream);
}
