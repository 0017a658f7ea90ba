// The layer's gradients: dZ = dO act'(Z) and dbias = dZ 1 in one pass over dO
// (and Z), then dX = F^T dZ and dF = dZ X^T as two products of linear.hip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "linear_common.h"

namespace linear {
namespace {

// dZ between the two products is held in the layer's type: one rounding, as large
// as a result's own, so that a 16-bit dX or dF is off by about 1.4 roundings instead
// of one (777 tokens through 1001 x 515, GELU, fp16: 2.9e-4 of its norm instead of
// 2.1e-4; bf16: 2.3e-3 instead of 1.7e-3).  The matrix cores take both operands in
// one type, and what the rounding leaves over would have to be multiplied as well,
// twice the work.  relu's dZ is exact.
//
// fp16's range does not hold every dZ: GELU's slope reaches 1.13, so a dO from 57967
// on gives an infinite one, and a small dO times a small slope lies below the
// smallest value.  dZ is therefore held times a power of two that puts the largest
// finite |dO| between 2^14 and 2^15 (the products' sums are multiplied back in
// fp32): nothing finite overflows, and the lower end's spacing loses at most 2^-39
// of the largest |dO|.
constexpr int kPeaks = 512;

__device__ inline float wave_max(float v) {
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// The largest finite |dO| of each workgroup's part, the parts as in slope_kernel.
// One more read of dO, bound by memory and for small ones by latency: 4096 tokens of
// 16384 rows 27 us (4.9 TB/s), 777 of 1001 3.7 us.
__global__ __launch_bounds__(256) void peak_kernel(int kn, int t, int span, int cols, int parts, const f16* __restrict__ dO,
                                                   int64_t lddo, float* __restrict__ peaks) {
  constexpr int V = kVec<f16>;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  float top = 0.0f;
  auto take = [&](float d) {
    d = fabsf(d);
    top = fmaxf(top, d < INFINITY ? d : 0.0f);      // neither infinities nor NaN
  };
  for (int64_t at = blockIdx.x; at < (int64_t)cols * parts; at += gridDim.x) {
    const int part = (int)(at / cols), m = ((int)(at - (int64_t)part * cols) * 32 + x) * V;
    const int lo = part * span, hi = min(t, lo + span);
    if (m + V <= kn) {
#pragma unroll 4
      for (int n = lo + y; n < hi; n += 8) {
        float d[V];
        load_vec(dO + (int64_t)n * lddo + m, d);
#pragma unroll
        for (int i = 0; i < V; ++i) take(d[i]);
      }
    } else {
      for (int n = lo + y; n < hi; n += 8)
        for (int i = m; i < kn; ++i) take((float)dO[(int64_t)n * lddo + i]);
    }
  }
  __shared__ float sh[4];
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) peaks[blockIdx.x] = fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

// The power of two by which dZ is held, the same in every wave: each reads all
// peaks, so that no barrier stands between this and the loads that follow.
__device__ inline float scale_of(const float* peaks, int count) {
  float top = 0.0f;
#pragma unroll
  for (int k = 0; k < kPeaks / 64; ++k) {
    const int i = k * 64 + (int)(threadIdx.x & 63);
    top = fmaxf(top, peaks[min(i, count - 1)]);
  }
  top = wave_max(top);
  int e = 15;
  if (top > 0.0f) frexpf(top, &e);                  // top in [2^(e-1), 2^e)
  return ldexpf(1.0f, 15 - e);
}

// dZ (WRITE: to lines of lddz values with zeros behind the last one; ACT: dO
// times the slope at Z, else dO itself) and (SUM) the sums of its rows.  A
// workgroup owns 32 vectors (128 or 256 rows) of `span` tokens; its eight groups
// of 32 lanes take every eighth token.  The sums are of the fp32 values, before
// dZ is rounded.  With `peaks` (fp16) dZ is written times scale_of() and 1 /
// scale_of() to `back`.  Bound by memory: one read of dO and Z and
// one write of dZ (4096 rows, 8192 tokens, bf16: 15 us for dbias alone, 4.5 TB/s; 32
// with GELU, 6 TB/s).
template <class T, bool ACT, bool WRITE, bool SUM>
__global__ __launch_bounds__(256) void slope_kernel(int kn, int t, int span, const T* __restrict__ dO, int64_t lddo,
                                                    const T* __restrict__ Z, int64_t ldz, int act, T* __restrict__ dZ,
                                                    int64_t lddz, float* __restrict__ part, T* __restrict__ dbias,
                                                    const float* __restrict__ peaks, int npeaks, float* __restrict__ back) {
  constexpr int V = kVec<T>;
  float scale = 1.0f;
  if constexpr (ACT && WRITE && std::is_same_v<T, f16>) {
    if (peaks) {
      scale = scale_of(peaks, npeaks);
      if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *back = 1.0f / scale;
    }
  }
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int m = (blockIdx.x * 32 + x) * V;
  const int lo = blockIdx.y * span, hi = min(t, lo + span);
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  if (m + V <= kn) {
#pragma unroll 4
    for (int n = lo + y; n < hi; n += 8) {
      float d[V], z[V];
      load_vec(dO + (int64_t)n * lddo + m, d);
      if (ACT) {
        load_vec(Z + (int64_t)n * ldz + m, z);
        act_grads<T, V>(d, z, act);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += d[i];
      if (WRITE) {
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] *= scale;
        store_vec(dZ + (int64_t)n * lddz + m, d);
      }
    }
  } else if (m < kn) {
    for (int n = lo + y; n < hi; n += 8) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float d = 0.0f;
        if (m + i < kn) {
          d = (float)dO[(int64_t)n * lddo + m + i];
          if (ACT) {
            const float z = (float)Z[(int64_t)n * ldz + m + i];
            act_grads<T, 1>(&d, &z, act);
          }
        }
        if (WRITE && m + i < lddz) dZ[(int64_t)n * lddz + m + i] = (T)(d * scale);
        sum[i] += d;
      }
    }
  }
  if (!SUM) return;
  __shared__ float sh[8][32 * V];
#pragma unroll
  for (int i = 0; i < V; ++i) sh[y][x * V + i] = sum[i];
  __syncthreads();
  for (int r = threadIdx.x; r < 32 * V; r += 256) {
    const int k = blockIdx.x * 32 * V + r;
    if (k >= kn) break;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sh[i][r];
    if (part)
      part[(int64_t)blockIdx.y * kn + k] = s;
    else
      dbias[k] = (T)s;
  }
}

// Adds the parts of dbias in a fixed order: 32 rows of a workgroup, eight groups
// of lanes that take every eighth part.
template <class T> __global__ __launch_bounds__(256) void bias_kernel(int kn, int parts, const float* part, T* dbias) {
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, k = blockIdx.x * 32 + x;
  __shared__ float sh[8][32];
  float s = 0.0f;
  if (k < kn) {
#pragma unroll 8
    for (int i = y; i < parts; i += 8) s += part[(int64_t)i * kn + k];
  }
  sh[y][x] = s;
  __syncthreads();
  if (y > 0 || k >= kn) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += sh[i][x];
  dbias[k] = (T)s;
}

// Tokens of one workgroup of slope_kernel: about four workgroups for each
// compute unit, 256 parts at most; up to 128 tokens one part, which needs no
// second launch (80 tokens of 1000 rows: 4 us instead of 3 and 2.3).
int slope_span(int dtype, int64_t kn, int64_t t) {
  const int64_t width = 32 * 16 / type_size(dtype), cols = (kn + width - 1) / width;
  const int64_t parts = std::min<int64_t>(256, std::max<int64_t>(1, 4 * compute_units() / std::max<int64_t>(cols, 1)));
  return (int)(t <= 128 ? std::max<int64_t>(t, 1) : std::max<int64_t>(32, (t + parts - 1) / parts));
}

// The workspace, in order, for the outputs that are wanted: one that is left out
// never adds to it.
struct Layout {
  Lines f, x, d;               // how the products' operands lie; d: dZ's lines, here or dO's own
  bool own = false;            // dZ is written here: a product wants it, and there is an activation or dO's lines are not direct
  int64_t lddz = 0;            // kn rounded up to whole vectors
  int64_t part = 0;            // byte offset of the partial dbias
  int span = 0, parts = 0;
  int cols = 0;                // workgroups of slope_kernel along the rows
  int npeaks = 0;              // fp16 with a slope other than 0 and 1: the peaks,
  int64_t peaks = 0;           // their byte offset, 1 / scale behind them
  int64_t product = 0;         // byte offset of the products' workspace
  int64_t bytes = 0;
};

Layout layout(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int act, Lines f, Lines x, Lines d, bool want_dx,
              bool want_df) {
  auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
  const int64_t vec = 16 / type_size(dtype);
  Layout w;
  w.own = (want_dx || want_df) &&
          (act != LINEAR_ACT_NONE || d == Lines::kFar || (d == Lines::kRagged && dtype != LINEAR_F32));
  if (w.own) {
    w.lddz = (kn + vec - 1) / vec * vec;
    d = lines_of(dtype, nullptr, w.lddz, w.lddz);
    w.part = up(w.lddz * t * type_size(dtype));
  }
  w.f = f, w.x = x, w.d = d;
  w.span = slope_span(dtype, kn, t);
  w.parts = (int)((t + w.span - 1) / w.span);
  w.cols = (int)((kn + 32 * vec - 1) / (32 * vec));
  w.peaks = w.part + (w.parts > 1 ? up((int64_t)w.parts * kn * 4) : 0);
  if (w.own && dtype == LINEAR_F16 && act > LINEAR_ACT_RELU) w.npeaks = (int)std::min<int64_t>(kPeaks, (int64_t)w.cols * w.parts);
  w.product = w.peaks + (w.npeaks ? up((w.npeaks + 1) * 4) : 0);
  int64_t most = 0;
  if (want_dx) most = product_workspace(dtype, f_order == 0, true, f, d, ci, t, kn);
  if (want_df)
    most = std::max(most, f_order ? product_workspace(dtype, false, false, x, d, ci, kn, t)
                                  : product_workspace(dtype, false, false, d, x, kn, ci, t));
  w.bytes = w.product + most;
  return w;
}

template <class T> hipError_t launch_slope(int64_t kn, int64_t t, const Layout& w, const void* dO, int64_t lddo, const void* Z,
                                           int64_t ldz, int act, char* ws, void* dbias, hipStream_t s) {
  const dim3 grid((unsigned)w.cols, (unsigned)std::max(1, w.parts));
  float* peaks = w.npeaks ? reinterpret_cast<float*>(ws + w.peaks) : nullptr;
  if constexpr (std::is_same_v<T, f16>) {
    if (peaks) {
      peak_kernel<<<dim3((unsigned)w.npeaks), 256, 0, s>>>((int)kn, (int)t, w.span, w.cols, w.parts, static_cast<const T*>(dO), lddo,
                                                           peaks);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  auto k = act != LINEAR_ACT_NONE ? (!w.own ? slope_kernel<T, true, false, true>
                                    : dbias ? slope_kernel<T, true, true, true>
                                            : slope_kernel<T, true, true, false>)
           : !w.own ? slope_kernel<T, false, false, true>
           : dbias  ? slope_kernel<T, false, true, true>
                    : slope_kernel<T, false, true, false>;
  float* part = w.parts > 1 ? reinterpret_cast<float*>(ws + w.part) : nullptr;
  k<<<grid, 256, 0, s>>>((int)kn, (int)t, w.span, static_cast<const T*>(dO), lddo, static_cast<const T*>(Z), ldz, act,
                         reinterpret_cast<T*>(ws), w.lddz, part, static_cast<T*>(dbias), peaks, w.npeaks,
                         peaks ? peaks + w.npeaks : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dbias || !part) return e;
  bias_kernel<T><<<dim3((unsigned)((kn + 31) / 32)), 256, 0, s>>>((int)kn, w.parts, part, static_cast<T*>(dbias));
  return hipGetLastError();
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_linear_backward_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int act,
                                                     int aligned) {
  if (int e = linear::check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  if (act < LINEAR_ACT_NONE || act > LINEAR_ACT_SILU) return -6;
  using namespace linear;
  if (aligned)
    return layout(dtype, kn, ci, t, f_order, act, lines_if(dtype, true, f_order ? ci : kn), lines_if(dtype, true, ci),
                  lines_if(dtype, true, kn), true, true).bytes;
  int64_t most = 0;
  for (Lines f : kAnyLines)
    for (Lines x : kAnyLines)
      for (Lines d : kAnyLines) most = std::max(most, layout(dtype, kn, ci, t, f_order, act, f, x, d, true, true).bytes);
  return most;
}

extern "C" int convgemm_linear_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                                        const void* X, int64_t ldx, const void* dO, int64_t lddo, const void* Z, int64_t ldz,
                                        int act, void* dX, int64_t lddx, void* dF, int64_t lddf, void* dbias, void* workspace,
                                        int64_t workspace_bytes, hipStream_t stream) {
  using namespace linear;
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (!F && dX && kn > 0 && ci > 0 && t > 0) return -5;
  if (f_order != 0 && f_order != 1) return -6;
  if (dX && bad_ld(ldf, f_order ? ci : kn)) return -7;
  if (!X && dF && kn > 0 && ci > 0 && t > 0) return -8;
  if (dF && bad_ld(ldx, ci)) return -9;
  if (!dO && kn > 0 && t > 0) return -10;
  if (bad_ld(lddo, kn)) return -11;
  if (act < LINEAR_ACT_NONE || act > LINEAR_ACT_SILU) return -14;
  if (act != LINEAR_ACT_NONE && !Z && kn > 0 && t > 0) return -12;
  if (act != LINEAR_ACT_NONE && bad_ld(ldz, kn)) return -13;
  if (dX && bad_ld(lddx, ci)) return -16;
  if (dF && bad_ld(lddf, f_order ? ci : kn)) return -18;
  const Layout w = layout(dtype, kn, ci, t, f_order, act,
                          dX ? lines_of(dtype, F, ldf, f_order ? ci : kn) : Lines::kDirect,
                          dF ? lines_of(dtype, X, ldx, ci) : Lines::kDirect, lines_of(dtype, dO, lddo, kn), dX, dF);
  if (w.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))) return -20;
  if (workspace_bytes < w.bytes) return -21;
  char* ws = static_cast<char*>(workspace);
  hipError_t e = hipSuccess;
  if (kn > 0 && (dbias || (w.own && t > 0))) {
    switch (dtype) {
      case LINEAR_F32: e = launch_slope<float>(kn, t, w, dO, lddo, Z, ldz, act, ws, dbias, stream); break;
      case LINEAR_BF16: e = launch_slope<bf16>(kn, t, w, dO, lddo, Z, ldz, act, ws, dbias, stream); break;
      default: e = launch_slope<f16>(kn, t, w, dO, lddo, Z, ldz, act, ws, dbias, stream);
    }
  }
  const void* dZ = w.own ? workspace : dO;
  const int64_t lddz = w.own ? w.lddz : lddo;
  const float* back = w.npeaks ? reinterpret_cast<const float*>(ws + w.peaks) + w.npeaks : nullptr;
  const int dz_rows = (int)(w.own ? w.lddz : kn);      // as loaded: zeros follow in the library's own copy
  if (e == hipSuccess && dX) {
    Product p{};
    p.A = F;
    p.lda = ldf;
    p.B = dZ;
    p.ldb = lddz;
    p.M = (int)ci;
    p.N = (int)t;
    p.K = (int)kn;
    p.bK = dz_rows;
    p.a = w.f;
    p.b = w.d;
    p.e.scale = back;
    p.e.C = dX;
    p.e.ldc = lddx;
    e = launch_product(dtype, f_order == 0, true, p, ws + w.product, stream);
  }
  if (e == hipSuccess && dF) {
    // dF with kn fastest is dZ X^T; with ci fastest its transpose X dZ^T
    Product p{};
    p.A = f_order ? X : dZ;
    p.lda = f_order ? ldx : lddz;
    p.B = f_order ? dZ : X;
    p.ldb = f_order ? lddz : ldx;
    p.M = (int)(f_order ? ci : kn);
    p.N = (int)(f_order ? kn : ci);
    p.K = (int)t;
    (f_order ? p.brows : p.arows) = dz_rows;
    p.a = f_order ? w.x : w.d;
    p.b = f_order ? w.d : w.x;
    p.e.scale = back;
    p.e.C = dF;
    p.e.ldc = lddf;
    e = launch_product(dtype, false, false, p, ws + w.product, stream);
  }
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}
