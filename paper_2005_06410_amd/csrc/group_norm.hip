// Group norm with an activation, channels fastest, and its gradients.
//
// What a thread owns is always one 16-byte vector of channels (V = 4 or 8), at every
// `rows`-th position: neighbouring threads take neighbouring vectors, so that loads are
// whole lines, and sums by channel stay in one thread's registers until the end.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <numeric>

#include "group_norm.h"
#include "linear_common.h"
#include "ltlt_internal.h"

namespace linear {
namespace {

struct Map {
  const void* p;
  int64_t ld, ldb;
};

struct Norm {
  int c, s, groups, per;       // per: channels of a group
  int64_t b;
  Map x, d;                    // input; dO (gradients)
  const void* weight;
  const void* bias;
  int act;
  float eps;
  Map o;                       // O, or dI
  float* mean;
  float* rstd;
  // gradients: sums by channel, [parts][c] of dZ and, behind them, of dZ xhat
  float* sums;
  int parts;
  // resident kernels
  int vecs, units, unit_groups;     // vectors of a unit, units of an image, groups of a unit
  int rows, slots;                  // threads along positions of one image, images at a time
  int lanes;                        // threads that add up one group
  int blocks;                       // workgroups along the images
  // split kernels
  int chunk, chunks;                // positions of a chunk, chunks of an image
  float2* part;                     // [b][chunks][c] mean and squares around it; or [b][groups] averages
};

// cnt >= 1 values of a vector from p on as they are stored, zeros behind.
template <class T> __device__ inline Packed<T> read_vec(const T* p, int cnt) {
  constexpr int V = kVec<T>;
  if (cnt >= V) return *reinterpret_cast<const Packed<T>*>(p);
  Packed<T> q;
#pragma unroll
  for (int i = 0; i < V; ++i) q.v[i] = i < cnt ? p[i] : (T)0.0f;
  return q;
}

template <class T> __device__ inline void write_vec(T* p, int cnt, const float* v) {
  constexpr int V = kVec<T>;
  if (cnt >= V) return store_vec(p, v);
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < cnt) p[i] = (T)v[i];
}

template <class T> __device__ inline void channel_values(const void* p, int ch, int cnt, float other, float* v) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = p && i < cnt ? (float)static_cast<const T*>(p)[ch + i] : other;
}

// ---------------------------------------------------------------------------
// resident: a unit (whole groups, whole vectors) of an image in registers
// ---------------------------------------------------------------------------
// One read and one write of everything.  Thread tid has vector tid % vecs of the unit
// and the positions row, row + rows, ... (row = tid / vecs % rows) of image slot
// tid / vecs / rows: maps smaller than a workgroup share it.
template <class T, int NT> struct Resident {
  static constexpr int V = kVec<T>;
  const Norm& a;
  float* sh;                   // [slots rows][vecs V], then the sums of the groups
  int vec, row, slot, ch, cnt, base;
  int local[V];                // groups of this thread's channels, in the unit
  bool owner;

  __device__ Resident(const Norm& n, float* lds, int unit) : a(n), sh(lds) {
    const int tid = threadIdx.x;
    vec = tid % a.vecs;
    const int line = tid / a.vecs;
    slot = line / a.rows;
    row = line - slot * a.rows;
    base = unit * a.vecs * V;
    ch = base + vec * V;
    cnt = a.c - ch;
    owner = slot < a.slots && cnt > 0;
#pragma unroll
    for (int i = 0; i < V; ++i) local[i] = min((vec * V + i) / a.per, a.unit_groups - 1);
  }

  __device__ void put(const float* v) {
    if (slot < a.slots) {
      float* to = sh + (slot * a.rows + row) * a.vecs * V + vec * V;
#pragma unroll
      for (int i = 0; i < V; i += 4) *reinterpret_cast<f4*>(to + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    }
  }

  // The sum over a group and its image of one value by channel and thread; v[i]
  // becomes that of channel i's group.  Threads without values bring zeros.
  __device__ void group_sum(float* v) {
    put(v);
    __syncthreads();
    float* sums = sh + NT * V;
    const int items = a.slots * a.unit_groups, lane = threadIdx.x & (a.lanes - 1), each = a.rows * a.per;
    for (int it = threadIdx.x / a.lanes; it < (items + NT / a.lanes - 1) / (NT / a.lanes) * (NT / a.lanes); it += NT / a.lanes) {
      float s = 0.0f;
      if (it < items) {
        const int sl = it / a.unit_groups, g = it - sl * a.unit_groups;
        const float* from = sh + sl * a.rows * a.vecs * V + g * a.per;
        for (int e = lane; e < each; e += a.lanes) {
          const int r = e / a.per;
          s += from[r * a.vecs * V + e - r * a.per];
        }
      }
      for (int d = a.lanes >> 1; d > 0; d >>= 1) s += __shfl_xor(s, d);
      if (lane == 0 && it < items) sums[it] = s;
    }
    __syncthreads();
    const float* mine = sums + min(slot, a.slots - 1) * a.unit_groups;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = mine[local[i]];
  }
};

template <class T, int NT, int RV> __global__ __launch_bounds__(NT) void norm_resident_kernel(Norm a) {
  constexpr int V = kVec<T>;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int unit = blockIdx.x % a.units, block = blockIdx.x / a.units;
  Resident<T, NT> r(a, lds, unit);
  float w[V], b[V];
  channel_values<T>(a.weight, r.ch, r.cnt, 1.0f, w);
  channel_values<T>(a.bias, r.ch, r.cnt, 0.0f, b);
  const float inverse_n = 1.0f / ((float)a.per * (float)a.s);
  for (int64_t n0 = (int64_t)block * a.slots; n0 < a.b; n0 += (int64_t)a.blocks * a.slots) {
    const int64_t n = n0 + r.slot;
    const bool there = r.owner && n < a.b;
    Packed<T> x[RV];
    float mean[V], rstd[V];
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = rstd[i] = 0.0f;
    const T* from = static_cast<const T*>(a.x.p) + n * a.x.ldb + r.ch;
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      const int p = r.row + k * a.rows;
      if (there && p < a.s) x[k] = read_vec<T>(from + p * a.x.ld, r.cnt);
    }
#pragma unroll
    for (int k = 0; k < RV; ++k)
      if (there && r.row + k * a.rows < a.s) {
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] += (float)x[k].v[i];
      }
    r.group_sum(mean);
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] *= inverse_n;
#pragma unroll
    for (int k = 0; k < RV; ++k)
      if (there && r.row + k * a.rows < a.s) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = i < r.cnt ? (float)x[k].v[i] - mean[i] : 0.0f;
          rstd[i] += d * d;
        }
      }
    r.group_sum(rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] = 1.0f / sqrtf(rstd[i] * inverse_n + a.eps);
    if (there && r.row == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < r.cnt && (r.ch + i) % a.per == 0) {
          const int64_t at = n * a.groups + (r.ch + i) / a.per;
          if (a.mean) a.mean[at] = mean[i];
          if (a.rstd) a.rstd[at] = rstd[i];
        }
    }
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.ldb + r.ch;
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] *= w[i];
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      const int p = r.row + k * a.rows;
      if (there && p < a.s) {
        float z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = ((float)x[k].v[i] - mean[i]) * rstd[i] + b[i];
        act_values<T, V>(z, a.act);
        write_vec(to + p * a.o.ld, r.cnt, z);
      }
    }
    __syncthreads();
  }
}

// dZ and xhat of one vector.
template <class T> __device__ inline void slopes(const Norm& a, const Packed<T>& x, const Packed<T>& d, const float* mean,
                                                 const float* rstd, const float* w, const float* b, float* dz, float* xhat) {
  constexpr int V = kVec<T>;
  float z[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    xhat[i] = ((float)x.v[i] - mean[i]) * rstd[i];
    z[i] = xhat[i] * w[i] + b[i];
    dz[i] = (float)d.v[i];
  }
  act_grads<T, V>(dz, z, a.act);
}

template <class T, int NT, int RV, bool DX> __global__ __launch_bounds__(NT) void norm_resident_grad_kernel(Norm a) {
  constexpr int V = kVec<T>;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int unit = blockIdx.x % a.units, block = blockIdx.x / a.units;
  Resident<T, NT> r(a, lds, unit);
  float w[V], b[V], total[V], total_x[V];
  channel_values<T>(a.weight, r.ch, r.cnt, 1.0f, w);
  channel_values<T>(a.bias, r.ch, r.cnt, 0.0f, b);
#pragma unroll
  for (int i = 0; i < V; ++i) total[i] = total_x[i] = 0.0f;
  const float inverse_n = 1.0f / ((float)a.per * (float)a.s);
  for (int64_t n0 = (int64_t)block * a.slots; n0 < a.b; n0 += (int64_t)a.blocks * a.slots) {
    const int64_t n = n0 + r.slot;
    const bool there = r.owner && n < a.b;
    Packed<T> x[RV], d[RV];
    const T* from = static_cast<const T*>(a.x.p) + n * a.x.ldb + r.ch;
    const T* dfrom = static_cast<const T*>(a.d.p) + n * a.d.ldb + r.ch;
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      const int p = r.row + k * a.rows;
      if (there && p < a.s) {
        x[k] = read_vec<T>(from + p * a.x.ld, r.cnt);
        d[k] = read_vec<T>(dfrom + p * a.d.ld, r.cnt);
      }
    }
    float mean[V], rstd[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t at = n * a.groups + (r.ch + i) / a.per;
      mean[i] = there && i < r.cnt ? a.mean[at] : 0.0f;
      rstd[i] = there && i < r.cnt ? a.rstd[at] : 0.0f;
    }
    float s[V], sx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = sx[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < RV; ++k)
      if (there && r.row + k * a.rows < a.s) {
        float dz[V], xhat[V];
        slopes<T>(a, x[k], d[k], mean, rstd, w, b, dz, xhat);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s[i] += dz[i];
          sx[i] += dz[i] * xhat[i];
        }
      }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i >= r.cnt) s[i] = sx[i] = 0.0f;
      total[i] += s[i];
      total_x[i] += sx[i];
    }
    if constexpr (DX) {
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= w[i], sx[i] *= w[i];
      r.group_sum(s);
      __syncthreads();
      r.group_sum(sx);
      T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.ldb + r.ch;
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= inverse_n, sx[i] *= inverse_n;
#pragma unroll
      for (int k = 0; k < RV; ++k) {
        const int p = r.row + k * a.rows;
        if (there && p < a.s) {
          float dz[V], xhat[V];
          slopes<T>(a, x[k], d[k], mean, rstd, w, b, dz, xhat);
#pragma unroll
          for (int i = 0; i < V; ++i) dz[i] = rstd[i] * (dz[i] * w[i] - s[i] - xhat[i] * sx[i]);
          write_vec(to + p * a.o.ld, r.cnt, dz);
        }
      }
      __syncthreads();
    }
  }
  if (!a.sums) return;
  // sums by channel over this workgroup's threads
  const int lines = a.slots * a.rows, width = a.vecs * V;
  for (int which = 0; which < 2; ++which) {
    r.put(which ? total_x : total);
    __syncthreads();
    float* to = a.sums + ((int64_t)which * a.parts + block) * a.c + r.base;
    int lanes = 64;
    while (lanes > 1 && lanes * width > NT) lanes >>= 1;
    const int lane = threadIdx.x & (lanes - 1), step = NT / lanes;
    for (int i0 = 0; i0 < width; i0 += step) {
      const int i = i0 + threadIdx.x / lanes;
      float v = 0.0f;
      if (i < width)
        for (int e = lane; e < lines; e += lanes) v += lds[e * width + i];
      for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor(v, d);
      if (lane == 0 && i < width && r.base + i < a.c) to[i] = v;
    }
    __syncthreads();
  }
}

// dweight and dbias: the parts of a channel added in a fixed order, 32 channels of a
// workgroup, 32 threads each.
template <class T> __global__ __launch_bounds__(1024) void norm_sums_kernel(int c, int64_t parts, const float* __restrict__ sums,
                                                                            T* __restrict__ dweight, T* __restrict__ dbias) {
  __shared__ float sh[32][32];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, ch = blockIdx.x * 32 + x;
  for (int which = 0; which < 2; ++which) {
    T* to = which ? dweight : dbias;
    if (!to) continue;
    float s = 0.0f;
    if (ch < c) {
      const float* p = sums + which * parts * c + ch;
#pragma unroll 8
      for (int64_t i = y; i < parts; i += 32) s += p[i * c];
    }
    __syncthreads();
    sh[y][x] = s;
    __syncthreads();
    if (y == 0 && ch < c) {
#pragma unroll
      for (int i = 1; i < 32; ++i) s += sh[i][x];
      to[ch] = (T)s;
    }
  }
}

// ---------------------------------------------------------------------------
// split: chunks of an image's positions in workgroups of their own
// ---------------------------------------------------------------------------
// A first pass over the input gives sums by chunk and channel, a small launch the
// groups' statistics, and a second pass the result.
constexpr int kSplitThreads = 256;
constexpr int kAhead = 4;                          // vectors of each input that a thread has under way

struct Place {
  int ch, cnt, vec, row, rows, lo, hi;
  int64_t n, at;                                   // image; chunk among all images'
};

// Part `id` of the work: an image, a chunk and a block of up to 256 vectors; this
// thread's vector and first position.
template <class T> __device__ inline Place place_of(const Norm& a, int64_t id) {
  Place p;
  p.at = id / a.units;
  p.n = p.at / a.chunks;
  const int chunk = (int)(p.at - p.n * a.chunks), first = (int)(id - p.at * a.units) * a.vecs;
  p.rows = kSplitThreads / a.vecs;
  p.vec = threadIdx.x % a.vecs;
  p.row = threadIdx.x / a.vecs;
  p.ch = (first + p.vec) * kVec<T>;
  p.cnt = p.row < p.rows ? a.c - p.ch : 0;
  p.lo = chunk * a.chunk;
  p.hi = min(a.s, p.lo + a.chunk);
  return p;
}

__device__ inline int64_t all_parts(const Norm& a) { return a.b * a.chunks * a.units; }

// f(position, vectors) for every position of this thread; kAhead loads of each input
// are issued before the first is used, since what f stores may be the input itself.
template <class T, bool TWO, class F> __device__ inline void each_position(const Norm& a, const Place& p, F f) {
  const T* x = static_cast<const T*>(a.x.p) + p.n * a.x.ldb + p.ch;
  const T* d = TWO ? static_cast<const T*>(a.d.p) + p.n * a.d.ldb + p.ch : x;
  for (int at = p.lo + p.row; at < p.hi; at += kAhead * p.rows) {
    Packed<T> vx[kAhead], vd[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int q = at + k * p.rows;
      if (q < p.hi) {
        vx[k] = read_vec<T>(x + q * a.x.ld, p.cnt);
        if (TWO) vd[k] = read_vec<T>(d + q * a.d.ld, p.cnt);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int q = at + k * p.rows;
      if (q < p.hi) f(q, vx[k], vd[k]);
    }
  }
}

// The sums over the workgroup's rows of one value by channel and thread, in every
// thread of the channel.  sh: (kSplitThreads + 256) V floats.
template <class T> __device__ inline void over_rows(const Norm& a, const Place& p, float* sh, const float* v, float* out) {
  constexpr int V = kVec<T>;
  const int width = a.vecs * V;
  float* sums = sh + kSplitThreads * V;
  if (p.row < p.rows) {
#pragma unroll
    for (int i = 0; i < V; ++i) sh[p.row * width + p.vec * V + i] = v[i];
  }
  __syncthreads();
  int lanes = 64;
  while (lanes > 1 && lanes * width > kSplitThreads) lanes >>= 1;
  const int lane = threadIdx.x & (lanes - 1), step = kSplitThreads / lanes;
  for (int i0 = 0; i0 < width; i0 += step) {
    const int i = i0 + threadIdx.x / lanes;
    float t = 0.0f;
    if (i < width)
      for (int r = lane; r < p.rows; r += lanes) t += sh[r * width + i];
    for (int d = lanes >> 1; d > 0; d >>= 1) t += __shfl_xor(t, d);
    if (lane == 0 && i < width) sums[i] = t;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) out[i] = sums[p.vec * V + i];
  __syncthreads();
}

// Mean and squares around it of each channel over a chunk: a thread sums differences
// to its first value, then the threads are joined by their means.
template <class T> __global__ __launch_bounds__(kSplitThreads) void norm_stats_kernel(Norm a) {
  constexpr int V = kVec<T>;
  __shared__ float sh[(kSplitThreads + 256) * V];
  for (int64_t id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place p = place_of<T>(a, id);
    float first[V], s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) first[i] = s[i] = q[i] = 0.0f;
    const int start = p.lo + p.row;
    int mine = 0;
    if (p.cnt > 0 && start < p.hi) {
      mine = (p.hi - start + p.rows - 1) / p.rows;
      each_position<T, false>(a, p, [&](int at, const Packed<T>& x, const Packed<T>&) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float v = (float)x.v[i];
          if (at == start) first[i] = v;
          const float d = v - first[i];
          s[i] += d;
          q[i] += d * d;
        }
      });
    }
    const float count = (float)mine, over = mine ? 1.0f / count : 0.0f;
    float mean[V], square[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      q[i] -= s[i] * s[i] * over;
      first[i] += s[i] * over;              // this thread's mean
      s[i] = first[i] * count;
    }
    over_rows<T>(a, p, sh, s, mean);
    const float n = (float)(p.hi - p.lo);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mean[i] /= n;
      const float d = first[i] - mean[i];
      q[i] += mine ? count * d * d : 0.0f;
    }
    over_rows<T>(a, p, sh, q, square);
    if (p.row == 0 && p.cnt > 0) {
      float2* to = a.part + p.at * a.c + p.ch;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < p.cnt) to[i] = float2{mean[i], square[i]};
    }
  }
}

// A sum over 256 threads, in each of them.
__device__ inline float block_sum(float v, float* sh) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// The groups' mean and rstd from their chunks and channels.
__global__ __launch_bounds__(256) void norm_join_kernel(Norm a) {
  __shared__ float sh[4];
  for (int64_t id = blockIdx.x; id < a.b * a.groups; id += gridDim.x) {
    const int64_t n = id / a.groups;
    const float2* from = a.part + n * a.chunks * a.c + (id - n * a.groups) * a.per;
    const int64_t total = (int64_t)a.chunks * a.per;
    auto length = [&](int64_t chunk) { return (float)min(a.chunk, a.s - (int)chunk * a.chunk); };
    float s = 0.0f;
    for (int64_t e = threadIdx.x; e < total; e += 256) {
      const int64_t k = e / a.per;
      s += from[k * a.c + e - k * a.per].x * length(k);
    }
    const float all = (float)a.per * (float)a.s;
    const float m = block_sum(s, sh) / all;
    s = 0.0f;
    for (int64_t e = threadIdx.x; e < total; e += 256) {
      const int64_t k = e / a.per;
      const float2 v = from[k * a.c + e - k * a.per];
      s += v.y + length(k) * (v.x - m) * (v.x - m);
    }
    s = block_sum(s, sh);
    if (threadIdx.x == 0) {
      a.mean[id] = m;
      a.rstd[id] = 1.0f / sqrtf(s / all + a.eps);
    }
  }
}

template <class T> __device__ inline void group_values(const Norm& a, const Place& p, float* mean, float* rstd) {
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) {
    const int64_t at = p.n * a.groups + min(p.ch + i, a.c - 1) / a.per;
    mean[i] = a.mean[at];
    rstd[i] = a.rstd[at];
  }
}

// O from the statistics; from the last part back, so that what the first pass read last
// is read first, from the caches.
template <class T> __global__ __launch_bounds__(kSplitThreads) void norm_apply_kernel(Norm a) {
  constexpr int V = kVec<T>;
  for (int64_t id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place p = place_of<T>(a, all_parts(a) - 1 - id);
    if (p.cnt <= 0) continue;
    float w[V], b[V], mean[V], rstd[V];
    channel_values<T>(a.weight, p.ch, p.cnt, 1.0f, w);
    channel_values<T>(a.bias, p.ch, p.cnt, 0.0f, b);
    group_values<T>(a, p, mean, rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] *= w[i];
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + p.n * a.o.ldb + p.ch;
    each_position<T, false>(a, p, [&](int at, const Packed<T>& x, const Packed<T>&) {
      float z[V];
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = ((float)x.v[i] - mean[i]) * rstd[i] + b[i];
      act_values<T, V>(z, a.act);
      write_vec(to + at * a.o.ld, p.cnt, z);
    });
  }
}

// Sums of dZ and dZ xhat by chunk and channel.
template <class T> __global__ __launch_bounds__(kSplitThreads) void norm_slopes_kernel(Norm a) {
  constexpr int V = kVec<T>;
  __shared__ float sh[(kSplitThreads + 256) * V];
  for (int64_t id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place p = place_of<T>(a, id);
    float s[V], sx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = sx[i] = 0.0f;
    if (p.cnt > 0) {
      float w[V], b[V], mean[V], rstd[V];
      channel_values<T>(a.weight, p.ch, p.cnt, 1.0f, w);
      channel_values<T>(a.bias, p.ch, p.cnt, 0.0f, b);
      group_values<T>(a, p, mean, rstd);
      each_position<T, true>(a, p, [&](int, const Packed<T>& x, const Packed<T>& d) {
        float dz[V], xhat[V];
        slopes<T>(a, x, d, mean, rstd, w, b, dz, xhat);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s[i] += dz[i];
          sx[i] += dz[i] * xhat[i];
        }
      });
    }
    over_rows<T>(a, p, sh, s, s);
    over_rows<T>(a, p, sh, sx, sx);
    if (p.row == 0 && p.cnt > 0) {
      float* to = a.sums + p.at * a.c + p.ch;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < p.cnt) {
          to[i] = s[i];
          to[(int64_t)a.parts * a.c + i] = sx[i];
        }
    }
  }
}

// The groups' avg d and avg(d xhat).
template <class T> __global__ __launch_bounds__(256) void norm_averages_kernel(Norm a) {
  __shared__ float sh[4];
  for (int64_t id = blockIdx.x; id < a.b * a.groups; id += gridDim.x) {
    const int64_t n = id / a.groups, g = id - n * a.groups;
    const int64_t total = (int64_t)a.chunks * a.per, first = n * a.chunks * a.c + g * a.per;
    float s = 0.0f, sx = 0.0f;
    for (int64_t e = threadIdx.x; e < total; e += 256) {
      const int64_t k = e / a.per, i = e - k * a.per;
      const float w = a.weight ? (float)static_cast<const T*>(a.weight)[g * a.per + i] : 1.0f;
      s += w * a.sums[first + k * a.c + i];
      sx += w * a.sums[(int64_t)a.parts * a.c + first + k * a.c + i];
    }
    const float all = (float)a.per * (float)a.s;
    s = block_sum(s, sh) / all;
    sx = block_sum(sx, sh) / all;
    if (threadIdx.x == 0) a.part[id] = float2{s, sx};
  }
}

template <class T> __global__ __launch_bounds__(kSplitThreads) void norm_dx_kernel(Norm a) {
  constexpr int V = kVec<T>;
  for (int64_t id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place p = place_of<T>(a, all_parts(a) - 1 - id);
    if (p.cnt <= 0) continue;
    float w[V], b[V], mean[V], rstd[V], s[V], sx[V];
    channel_values<T>(a.weight, p.ch, p.cnt, 1.0f, w);
    channel_values<T>(a.bias, p.ch, p.cnt, 0.0f, b);
    group_values<T>(a, p, mean, rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 v = a.part[p.n * a.groups + min(p.ch + i, a.c - 1) / a.per];
      s[i] = v.x;
      sx[i] = v.y;
    }
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + p.n * a.o.ldb + p.ch;
    each_position<T, true>(a, p, [&](int at, const Packed<T>& x, const Packed<T>& d) {
      float dz[V], xhat[V];
      slopes<T>(a, x, d, mean, rstd, w, b, dz, xhat);
#pragma unroll
      for (int i = 0; i < V; ++i) dz[i] = rstd[i] * (dz[i] * w[i] - s[i] - xhat[i] * sx[i]);
      write_vec(to + at * a.o.ld, p.cnt, dz);
    });
  }
}

// ---------------------------------------------------------------------------
// choice and launch
// ---------------------------------------------------------------------------
int64_t up(int64_t v) { return (v + 255) / 256 * 256; }
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups for that many parts; the kernels go on from there.
dim3 grid_of(int64_t parts) { return dim3((unsigned)std::min<int64_t>(parts, 1 << 20)); }

struct NormPlan {
  bool resident;
  int threads, held;                 // resident: threads of a workgroup, vectors that a thread holds
  int vecs, units, unit_groups, rows, slots, lanes, blocks;
  int chunk, chunks;
  int64_t sums, stats, bytes;        // byte offsets: part first, then the sums, then mean and rstd
};

// Resident where a unit of whole groups and whole vectors fits a workgroup's registers;
// the unit is widened to 128 bytes of each position (a line of the caches) while it
// still fits and leaves two workgroups for every compute unit.
NormPlan plan_of(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, bool grad) {
  NormPlan p{};
  const int64_t V = 16 / type_size(dtype), per = c / groups, all = div_up(c, V), cu = compute_units();
  const int64_t unit = std::min<int64_t>(std::lcm(per, V) / V, all);
  const int most = grad ? 8 : 16;
  auto fits = [&](int64_t vecs, int threads) { return vecs <= threads && div_up(s, std::max<int64_t>(1, threads / vecs)) <= most; };
  if (fits(unit, 1024)) {
    p.resident = true;
    int64_t vecs = unit;
    while (vecs < 8 && vecs < all && fits(std::min(vecs + unit, all), 1024) && div_up(all, std::min(vecs + unit, all)) * b >= 2 * cu)
      vecs = std::min(vecs + unit, all);
    p.threads = 256;
    while (!fits(vecs, p.threads)) p.threads *= 2;
    const int64_t lines = p.threads / vecs;
    p.vecs = (int)vecs;
    p.units = (int)div_up(all, vecs);
    p.unit_groups = (int)std::max<int64_t>(1, std::min<int64_t>(groups, vecs * V / per));
    p.rows = (int)std::min(lines, std::max<int64_t>(s, 1));
    p.slots = (int)std::min<int64_t>(lines / p.rows, std::max<int64_t>(b, 1));
    const int64_t need = div_up(std::max<int64_t>(s, 1), p.rows);
    p.held = 1;
    while (p.held < need) p.held *= 2;
    p.lanes = 64;
    while (p.lanes > 1 && p.lanes * (int64_t)p.slots * p.unit_groups > p.threads) p.lanes /= 2;
    const int64_t rounds = div_up(std::max<int64_t>(b, 1), p.slots);
    p.blocks = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, 8 * cu * 256 / p.threads / p.units));
    p.sums = 0;
    p.bytes = grad ? up(2 * (int64_t)p.blocks * c * 4) : 0;
    return p;
  }
  p.vecs = (int)std::min<int64_t>(all, kSplitThreads);
  p.units = (int)div_up(all, p.vecs);
  const int64_t rows = kSplitThreads / p.vecs;
  const int64_t want = std::max<int64_t>(1, div_up(8 * cu, b * p.units));
  // 256 values at most to a thread's sum
  p.chunk = (int)(std::min<int64_t>(256, div_up(std::max(div_up(s, want), std::min(s, 16 * rows)), rows)) * rows);
  p.chunks = (int)div_up(s, p.chunk);
  p.sums = grad ? up(b * groups * 8) : up(b * p.chunks * c * 8);
  p.stats = p.sums + (grad ? up(2 * b * p.chunks * c * 4) : 0);
  p.bytes = p.stats + (grad ? 0 : 2 * up(b * groups * 4));
  return p;
}

int check_norm(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  if (!is_type(dtype)) return -1;
  if (c < 0 || c >= kSizeLimit) return -2;
  if (s < 0 || s >= kSizeLimit) return -3;
  if (b < 0 || b >= 1ll << 31 || (c * s > 0 && b >= kElemLimit / (c * s))) return -4;
  if (groups < 1 || groups > std::max<int64_t>(c, 1) || c % groups) return -5;
  return 0;
}

// ld (its argument's number `at`) and ldb behind it.
int check_map(int64_t c, int64_t s, int64_t b, int64_t ld, int64_t ldb, int at) {
  if (ld < std::max<int64_t>(c, 1) || ld >= kElemLimit) return -at;
  if (s > 1 && ld > kElemLimit / s) return -at;
  if (b > 1 && (ldb < (s - 1) * ld + c || ldb >= kElemLimit)) return -(at + 1);
  return 0;
}

template <class T, int NT, bool GRAD, bool DX> hipError_t launch_held(const NormPlan& p, const Norm& a, hipStream_t s) {
  const int lds = (NT * kVec<T> + p.slots * p.unit_groups) * 4;
  auto go = [&](auto kernel) {
    const hipError_t e = ltlt::ensure_dynamic_lds((const void*)kernel, (2 * NT * kVec<T>) * 4);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)((int64_t)p.units * p.blocks)), NT, lds, s>>>(a);
    return hipGetLastError();
  };
  if constexpr (GRAD) {
    switch (p.held) {
      case 1: return go(norm_resident_grad_kernel<T, NT, 1, DX>);
      case 2: return go(norm_resident_grad_kernel<T, NT, 2, DX>);
      case 4: return go(norm_resident_grad_kernel<T, NT, 4, DX>);
      default: return go(norm_resident_grad_kernel<T, NT, 8, DX>);
    }
  } else {
    switch (p.held) {
      case 1: return go(norm_resident_kernel<T, NT, 1>);
      case 2: return go(norm_resident_kernel<T, NT, 2>);
      case 4: return go(norm_resident_kernel<T, NT, 4>);
      case 8: return go(norm_resident_kernel<T, NT, 8>);
      default: return go(norm_resident_kernel<T, NT, 16>);
    }
  }
}

template <class T, bool GRAD, bool DX> hipError_t launch_resident(const NormPlan& p, const Norm& a, hipStream_t s) {
  switch (p.threads) {
    case 256: return launch_held<T, 256, GRAD, DX>(p, a, s);
    case 512: return launch_held<T, 512, GRAD, DX>(p, a, s);
    default: return launch_held<T, 1024, GRAD, DX>(p, a, s);
  }
}

void fill(Norm& a, const NormPlan& p, char* ws) {
  a.vecs = p.vecs, a.units = p.units, a.unit_groups = p.unit_groups, a.rows = p.rows, a.slots = p.slots, a.lanes = p.lanes;
  a.blocks = p.blocks, a.chunk = p.chunk, a.chunks = p.chunks;
  a.part = reinterpret_cast<float2*>(ws);
}

template <class T> hipError_t launch_norm(Norm a, const NormPlan& p, char* ws, hipStream_t s) {
  fill(a, p, ws);
  if (p.resident) return launch_resident<T, false, false>(p, a, s);
  const dim3 grid = grid_of(a.b * p.chunks * p.units);
  norm_stats_kernel<T><<<grid, kSplitThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!a.mean) a.mean = reinterpret_cast<float*>(ws + p.stats);
  if (!a.rstd) a.rstd = reinterpret_cast<float*>(ws + p.stats + up(a.b * a.groups * 4));
  norm_join_kernel<<<grid_of(a.b * a.groups), 256, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  norm_apply_kernel<T><<<grid, kSplitThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class T> hipError_t launch_norm_grad(Norm a, const NormPlan& p, char* ws, void* dweight, void* dbias, hipStream_t s) {
  fill(a, p, ws);
  hipError_t e;
  const bool want = dweight || dbias;
  if (p.resident) {
    a.parts = p.blocks;
    a.sums = want ? reinterpret_cast<float*>(ws + p.sums) : nullptr;
    e = a.o.p ? launch_resident<T, true, true>(p, a, s) : launch_resident<T, true, false>(p, a, s);
  } else {
    a.parts = (int)(a.b * p.chunks);
    a.sums = reinterpret_cast<float*>(ws + p.sums);
    const dim3 grid = grid_of(a.b * p.chunks * p.units);
    norm_slopes_kernel<T><<<grid, kSplitThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (e == hipSuccess && a.o.p) {
      norm_averages_kernel<T><<<grid_of(a.b * a.groups), 256, 0, s>>>(a);
      if ((e = hipGetLastError()) == hipSuccess) {
        norm_dx_kernel<T><<<grid, kSplitThreads, 0, s>>>(a);
        e = hipGetLastError();
      }
    }
  }
  if (e != hipSuccess || !want) return e;
  norm_sums_kernel<T><<<dim3((unsigned)div_up(a.c, 32)), 1024, 0, s>>>(a.c, a.parts, a.sums, static_cast<T*>(dweight), static_cast<T*>(dbias));
  return hipGetLastError();
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_group_norm_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  return c * s * b == 0 ? 0 : plan_of(dtype, c, s, b, groups, false).bytes;
}

extern "C" int64_t convgemm_group_norm_backward_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  return c * s * b == 0 ? 0 : plan_of(dtype, c, s, b, groups, true).bytes;
}

extern "C" int convgemm_group_norm(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, const void* I, int64_t ldi, int64_t ldbi,
                                   const void* weight, const void* bias, double eps, int act, void* O, int64_t ldo, int64_t ldbo,
                                   float* mean, float* rstd, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  const bool work = c * s * b > 0;
  if (!I && work) return -6;
  if (int e = check_map(c, s, b, ldi, ldbi, 7)) return e;
  if (!(eps >= 0) || !std::isfinite((float)eps)) return -11;
  if (act < LINEAR_ACT_NONE || act > LINEAR_ACT_SILU) return -12;
  if (!O && work) return -13;
  if (int e = check_map(c, s, b, ldo, ldbo, 14)) return e;
  if (!work) return LINEAR_OK;
  const NormPlan p = plan_of(dtype, c, s, b, groups, false);
  if (p.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))) return -18;
  if (workspace_bytes < p.bytes) return -19;
  Norm a{};
  a.c = (int)c, a.s = (int)s, a.groups = (int)groups, a.per = (int)(c / groups), a.b = b;
  a.x = Map{I, ldi, ldbi};
  a.o = Map{O, ldo, ldbo};
  a.weight = weight, a.bias = bias, a.act = act, a.eps = (float)eps, a.mean = mean, a.rstd = rstd;
  char* ws = static_cast<char*>(workspace);
  const hipError_t e = dtype == LINEAR_F32    ? launch_norm<float>(a, p, ws, stream)
                       : dtype == LINEAR_BF16 ? launch_norm<bf16>(a, p, ws, stream)
                                              : launch_norm<f16>(a, p, ws, stream);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}

extern "C" int convgemm_group_norm_backward(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, const void* I, int64_t ldi,
                                            int64_t ldbi, const void* dO, int64_t lddo, int64_t ldbdo, const void* weight,
                                            const void* bias, int act, const float* mean, const float* rstd, void* dI, int64_t lddi,
                                            int64_t ldbdi, void* dweight, void* dbias, void* workspace, int64_t workspace_bytes,
                                            hipStream_t stream) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  const bool work = c * s * b > 0;
  if (!I && work) return -6;
  if (int e = check_map(c, s, b, ldi, ldbi, 7)) return e;
  if (!dO && work) return -9;
  if (int e = check_map(c, s, b, lddo, ldbdo, 10)) return e;
  if (act < LINEAR_ACT_NONE || act > LINEAR_ACT_SILU) return -14;
  if (!mean && work) return -15;
  if (!rstd && work) return -16;
  if (dI) {
    if (int e = check_map(c, s, b, lddi, ldbdi, 18)) return e;
  }
  const NormPlan p = work ? plan_of(dtype, c, s, b, groups, true) : NormPlan{};
  if (p.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))) return -22;
  if (workspace_bytes < p.bytes) return -23;
  if ((!dI && !dweight && !dbias) || c == 0) return LINEAR_OK;
  Norm a{};
  a.c = (int)c, a.s = (int)s, a.groups = (int)groups, a.per = (int)(c / groups), a.b = b;
  a.x = Map{I, ldi, ldbi};
  a.d = Map{dO, lddo, ldbdo};
  a.o = Map{dI, lddi, ldbdi};
  a.weight = weight, a.bias = bias, a.act = act;
  a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
  char* ws = static_cast<char*>(workspace);
  hipError_t e = hipSuccess;
  auto go = [&](auto* none) {
    using T = std::remove_pointer_t<decltype(none)>;
    if (work) return launch_norm_grad<T>(a, p, ws, dweight, dbias, stream);
    // nothing to add up: zeros
    if (!dweight && !dbias) return hipSuccess;
    norm_sums_kernel<T><<<dim3((unsigned)div_up(c, 32)), 1024, 0, stream>>>((int)c, 0, nullptr, static_cast<T*>(dweight), static_cast<T*>(dbias));
    return hipGetLastError();
  };
  e = dtype == LINEAR_F32 ? go((float*)nullptr) : dtype == LINEAR_BF16 ? go((bf16*)nullptr) : go((f16*)nullptr);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}
