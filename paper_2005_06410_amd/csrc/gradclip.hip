// The norm of many gradients together, and the gradients scaled to at most a
// given norm, on gfx950: one pass that sums the squares and one that scales.
//
// Squares are formed and summed in fp64: a gradient of 1e30 or 1e-30 squares
// without leaving the range, and the sum over 10^9 values keeps more digits
// than its fp32 result shows.  Every workgroup takes a contiguous run of chunks
// of the tensors laid end to end and writes one partial sum; the scaling pass
// adds the partial sums in order in each of its workgroups, so the result does
// not depend on which workgroup ends first and no third launch is needed.
//
// Bound by memory: 16-byte loads at any alignment, four in flight per thread; 400 M
// fp32 values take 283 us for the norm (5.6 TB/s) and 648 for the scaling (4.9 TB/s,
// the rate of a large copy).
// The second pass takes each workgroup's run from its end, where the first one
// left off: what is still in the last-level cache (256 MB) is not read again
// from HBM.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "linear_common.h"

namespace linear {
namespace {

constexpr int kList = 240;          // tensors of one launch: the list travels in the kernel's arguments
constexpr int64_t kTensorLimit = 1ll << 37;   // values of one tensor
constexpr int kParts = 2048;        // partial sums (workgroups of the first pass)
// Above this the scaled values are stored past the caches: what of the gradients
// is still in the last-level cache stays there for the second pass (200 bf16
// tensors, 180 MB: 99 -> 90 us).
constexpr int64_t kStream = 128ll << 20;
constexpr int kMinChunk = 4096;     // bytes that a workgroup takes at a time: one vector per thread ..
constexpr int kMaxChunk = 32768;    // .. to eight; larger ones where a list would have 2^30 chunks

struct List {
  const void* g[kList];
  void* out[kList];
  int64_t n[kList];
  int first[kList + 1];             // chunks before each tensor
  unsigned char dtype[kList];
  int count;
  int chunk;                        // bytes
};

__device__ inline double block_sum(double v) {
  __shared__ double sh[4];
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  __syncthreads();
  return v;
}

// The tensor that holds chunk c.
__device__ inline int tensor_of(const List& l, int c) {
  int lo = 0, hi = l.count;          // first[lo] <= c < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= c) lo = mid; else hi = mid;
  }
  return lo;
}

// Calls f(vectors at hand, first of them) for the n values of a chunk in groups
// of up to four 16-byte vectors per thread, and g(value) for what is left over.
template <class T, class F, class G> __device__ inline void for_values(int64_t n, F f, G g) {
  constexpr int V = kVec<T>;
  const int whole = (int)(n / V);
  int i = threadIdx.x;
  for (; i + 768 < whole; i += 1024) f(std::integral_constant<int, 4>{}, i);
  for (; i < whole; i += 256) f(std::integral_constant<int, 1>{}, i);
  const int rest = (int)(n - (int64_t)whole * V);
  if ((int)threadIdx.x < rest) g(whole * V + (int)threadIdx.x);
}

template <class T> __device__ inline double squares(const T* g, int64_t n) {
  constexpr int V = kVec<T>;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for_values<T>(
      n,
      [&](auto count, int i) {
        constexpr int C = decltype(count)::value;
        float v[C][V];
#pragma unroll
        for (int u = 0; u < C; ++u) load_vec(g + (int64_t)(i + 256 * u) * V, v[u]);
#pragma unroll
        for (int u = 0; u < C; ++u)
#pragma unroll
          for (int j = 0; j < V; ++j) s[j & 3] = fma((double)v[u][j], (double)v[u][j], s[j & 3]);
      },
      [&](int i) {
        const double x = (double)(float)g[i];
        s[0] = fma(x, x, s[0]);
      });
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// c = m 2^e: e = 0 where c is a normal fp32 value (or 0, 1 or NaN), and m in [1/2, 1)
// where it is smaller, since a large gradient times such a c is a normal value again.
struct Factor {
  float m;
  int e;
};

__device__ inline Factor factor_of(double norm, double max_norm) {
  if (norm <= max_norm) return Factor{1.0f, 0};
  const double c = max_norm / norm;                  // a NaN norm gives a NaN factor
  int e = 0;
  const double m = c > 0.0 && c < 0x1p-126 ? frexp(c, &e) : c;
  return Factor{(float)m, e};
}

template <bool STREAM, class T> __device__ inline void scale(const T* g, T* out, int64_t n, Factor c) {
  constexpr int V = kVec<T>;
  for_values<T>(
      n,
      [&](auto count, int i) {
        constexpr int C = decltype(count)::value;
        float v[C][V];
#pragma unroll
        for (int u = 0; u < C; ++u) load_vec(g + (int64_t)(i + 256 * u) * V, v[u]);
#pragma unroll
        for (int u = 0; u < C; ++u) {
#pragma unroll
          for (int j = 0; j < V; ++j) v[u][j] = ldexpf(v[u][j] * c.m, c.e);
          result_vec<T, STREAM>(out + (int64_t)(i + 256 * u) * V, v[u]);
        }
      },
      [&](int i) { out[i] = (T)ldexpf((float)g[i] * c.m, c.e); });
}

// Calls f(tensor, first value, values) for the chunks lo .. hi-1, one at a time,
// from the last one where `back` is set.
template <bool back, class F> __device__ inline void for_chunks(const List& l, int lo, int hi, F f) {
  if (lo >= hi) return;
  int i = tensor_of(l, back ? hi - 1 : lo);
  for (int k = 0; k < hi - lo; ++k) {
    const int c = back ? hi - 1 - k : lo + k;
    while (c >= l.first[i + 1]) ++i;
    while (c < l.first[i]) --i;
    const int64_t per = l.chunk / (l.dtype[i] == LINEAR_F32 ? 4 : 2);
    const int64_t at = (int64_t)(c - l.first[i]) * per;
    f(i, at, min(l.n[i] - at, per));
  }
}

__global__ __launch_bounds__(256) void norm_kernel(List l, double* part) {
  const int chunks = l.first[l.count];
  const int lo = (int)((int64_t)chunks * blockIdx.x / gridDim.x), hi = (int)((int64_t)chunks * (blockIdx.x + 1) / gridDim.x);
  double s = 0.0;
  for_chunks<false>(l, lo, hi, [&](int i, int64_t at, int64_t n) {
    if (l.dtype[i] == LINEAR_F32)
      s += squares(static_cast<const float*>(l.g[i]) + at, n);
    else if (l.dtype[i] == LINEAR_BF16)
      s += squares(static_cast<const bf16*>(l.g[i]) + at, n);
    else
      s += squares(static_cast<const f16*>(l.g[i]) + at, n);
  });
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// sqrt of the partial sums' total, the same in every workgroup.
__device__ inline double total_norm(const double* part, int parts) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
  return sqrt(block_sum(s));
}

__global__ __launch_bounds__(256) void total_kernel(const double* part, int parts, float* norm) {
  const double v = total_norm(part, parts);
  if (threadIdx.x == 0) *norm = (float)v;
}

template <bool STREAM>
__global__ __launch_bounds__(256) void scale_kernel(List l, const double* part, int parts, double max_norm, float* norm) {
  const double v = total_norm(part, parts);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  const Factor c = factor_of(v, max_norm);
  const int chunks = l.first[l.count];
  const int lo = (int)((int64_t)chunks * blockIdx.x / gridDim.x), hi = (int)((int64_t)chunks * (blockIdx.x + 1) / gridDim.x);
  for_chunks<true>(l, lo, hi, [&](int i, int64_t at, int64_t n) {
    if (c.m == 1.0f && c.e == 0 && l.out[i] == l.g[i]) return;
    if (l.dtype[i] == LINEAR_F32)
      scale<STREAM>(static_cast<const float*>(l.g[i]) + at, static_cast<float*>(l.out[i]) + at, n, c);
    else if (l.dtype[i] == LINEAR_BF16)
      scale<STREAM>(static_cast<const bf16*>(l.g[i]) + at, static_cast<bf16*>(l.out[i]) + at, n, c);
    else
      scale<STREAM>(static_cast<const f16*>(l.g[i]) + at, static_cast<f16*>(l.out[i]) + at, n, c);
  });
}

// Fills `l` with tensors from `from` on; returns the next one that did not fit.
int take(List& l, int chunk, int from, int count, const void* const* g, void* const* out, const int64_t* n, const int* dtype) {
  l.count = 0;
  l.first[0] = 0;
  l.chunk = chunk;
  for (; from < count && l.count < kList; ++from) {
    if (n[from] == 0) continue;
    const int64_t chunks = (n[from] * type_size(dtype[from]) + chunk - 1) / chunk;
    const int i = l.count++;
    l.g[i] = g[from];
    l.out[i] = out ? out[from] : nullptr;
    l.n[i] = n[from];
    l.dtype[i] = (unsigned char)dtype[from];
    l.first[i + 1] = l.first[i] + (int)chunks;
  }
  return from;
}

// Bytes of all tensors, or 2^60 where they are more (a norm may count one tensor
// any number of times).
int64_t bytes_of(int count, const int64_t* n, const int* dtype) {
  constexpr int64_t most = 1ll << 60;
  int64_t bytes = 0;
  for (int i = 0; i < count && bytes < most; ++i) bytes += n[i] * type_size(dtype[i]);
  return std::min(bytes, most);
}

// Bytes of a chunk: as large as leaves every one of the first pass's workgroups
// a chunk.  A list holds kList kTensorLimit values at most, 2^47 bytes: with chunks
// of 2^30 bytes it has fewer than 2^31 chunks in any case.
int chunk_of(int64_t bytes) {
  int chunk = kMinChunk;
  while (chunk < kMaxChunk && bytes / (2 * chunk) >= kParts) chunk *= 2;
  while (chunk < 1 << 30 && bytes / chunk >= 1ll << 30) chunk *= 2;
  return chunk;
}

unsigned workgroups(const List& l) { return (unsigned)std::min(l.first[l.count], kParts); }

int launches_of(int count) { return std::max(1, (count + kList - 1) / kList); }

int run(int count, const void* const* g, void* const* out, const int64_t* n, const int* dtype, double max_norm, float* norm,
        void* workspace, hipStream_t s) {
  double* part = static_cast<double*>(workspace);
  int parts = 0;
  List l;
  const int64_t bytes = bytes_of(count, n, dtype);
  const int chunk = chunk_of(bytes);
  for (int at = 0; at < count;) {
    at = take(l, chunk, at, count, g, out, n, dtype);
    if (l.count == 0) break;
    norm_kernel<<<dim3(workgroups(l)), 256, 0, s>>>(l, part + parts);
    parts += (int)workgroups(l);
  }
  hipError_t e = hipGetLastError();
  bool told = false;
  for (int at = 0; e == hipSuccess && out && at < count;) {
    at = take(l, chunk, at, count, g, out, n, dtype);
    if (l.count == 0) break;
    const auto k = bytes >= kStream ? scale_kernel<true> : scale_kernel<false>;
    k<<<dim3(workgroups(l)), 256, 0, s>>>(l, part, parts, max_norm, told ? nullptr : norm);
    told = true;
    e = hipGetLastError();
  }
  if (e == hipSuccess && !told) {
    total_kernel<<<1, 256, 0, s>>>(part, parts, norm);
    e = hipGetLastError();
  }
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}

// Arguments shared by the two calls, by the norm call's numbering.
int check(int count, const void* const* g, const int64_t* n, const int* dtype) {
  if (count < 0) return 1;
  if (count == 0) return 0;
  if (!g) return 2;
  if (!n) return 3;
  if (!dtype) return 4;
  for (int i = 0; i < count; ++i) {
    if (n[i] < 0 || n[i] >= kTensorLimit) return 3;
    if (!is_type(dtype[i])) return 4;
    if (n[i] > 0 && !g[i]) return 2;
  }
  return 0;
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_grad_workspace(int count) {
  if (count < 0) return -1;
  return (int64_t)linear::launches_of(count) * linear::kParts * 8;
}

extern "C" int convgemm_grad_norm(int count, const void* const* g, const int64_t* n, const int* dtype, float* norm,
                                  void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  if (int e = linear::check(count, g, n, dtype)) return -e;
  if (!norm) return -5;
  if (!workspace || ((uintptr_t)workspace & 15)) return -6;
  if (workspace_bytes < convgemm_grad_workspace(count)) return -7;
  return linear::run(count, g, nullptr, n, dtype, 0.0, norm, workspace, stream);
}

extern "C" int convgemm_grad_clip(int count, const void* const* g, void* const* out, const int64_t* n, const int* dtype,
                                  double max_norm, float* norm, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  if (int e = linear::check(count, g, n, dtype)) return e > 2 ? -(e + 1) : -e;
  if (count > 0 && !out) return -3;
  for (int i = 0; i < count; ++i)
    if (n[i] > 0 && !out[i]) return -3;
  if (!(max_norm >= 0.0)) return -6;
  if (!norm) return -7;
  if (!workspace || ((uintptr_t)workspace & 15)) return -8;
  if (workspace_bytes < convgemm_grad_workspace(count)) return -9;
  return linear::run(count, g, out, n, dtype, max_norm, norm, workspace, stream);
}
