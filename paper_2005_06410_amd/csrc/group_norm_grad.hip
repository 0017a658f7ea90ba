// The gradients of group norm with an activation, channels fastest.
#include "group_norm_common.h"

namespace linear {
namespace {

// dZ of a vector and, in t, x - mean: Z = t (weight rstd) + bias.
template <class T, int ACT, int MODE>
__device__ inline void slopes(const Packed<T>& x, const Packed<T>& d, const float* mean, const float* a, const float* b, float* dz, float* t) {
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) {
    t[i] = (float)x.v[i] - mean[MODE == kOneGroup ? 0 : i];
    dz[i] = act_grad<T, ACT>((float)d.v[i], t[i] * a[i] + b[i]);
  }
}

// A power of two that x - mean is multiplied by and rstd^2 divided by, since the square of a
// large or small rstd alone would leave fp32's range (a third factor for each value, rstd twice,
// needs eight registers more: 28 x 28 x 360 x 64 fp16, 30 groups 106 us, so 100).
template <int N> __device__ inline float stretch(const float (&rstd)[N]) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, rstd[i]);
  return top > 0x1p40f ? 0x1p64f : top < 0x1p-40f ? 0x1p-64f : 1.0f;
}

template <class T, int NT, int RV, int MODE> __global__ __launch_bounds__(NT) void norm_resident_grad_kernel(Norm a) {
  constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  Resident<T, NT, MODE> r(a, lds);
  const Channels<T, MODE> c(a, r.base + r.vec * V);
  r.place(c);
  float w[V], b[V], total[V], total_x[V];
  c.values(a.weight, 1.0f, w);
  c.values(a.bias, 0.0f, b);
#pragma unroll
  for (int i = 0; i < V; ++i) total[i] = total_x[i] = 0.0f;
  const float inverse_n = 1.0f / ((float)a.per * (float)a.s);
  for (int64_t n0 = (int64_t)r.block * a.slots; n0 < a.b; n0 += (int64_t)a.blocks * a.slots) {
    const int64_t n = n0 + r.slot;
    const bool there = r.owner && n < a.b;
    Packed<T> x[RV], d[RV];
    const T* from = static_cast<const T*>(a.x.p) + n * a.x.ldb + c.ch;
    const T* dfrom = static_cast<const T*>(a.d.p) + n * a.d.ldb + c.ch;
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      const int p = r.row + k * a.rows;
      if (there && p < a.s) {
        x[k] = c.read(from + p * a.x.ld);
        d[k] = c.read(dfrom + p * a.d.ld);
      }
    }
    float mean[H], rstd[H], scale[V], s[V], sx[V];
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int64_t at = n * a.groups + r.first + r.local[i];
      mean[i] = there ? a.mean[at] : 0.0f;
      rstd[i] = there ? a.rstd[at] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      scale[i] = rstd[MODE == kOneGroup ? 0 : i] * w[i];
      s[i] = sx[i] = 0.0f;
    }
    by_act(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < RV; ++k)
        if (there && r.row + k * a.rows < a.s) {
          float dz[V], t[V];
          slopes<T, decltype(act)::value, MODE>(x[k], d[k], mean, scale, b, dz, t);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            s[i] += dz[i];
            sx[i] += dz[i] * t[i];
          }
        }
    });
    float both[2][H];
#pragma unroll
    for (int i = 0; i < H; ++i) both[0][i] = both[1][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int h = MODE == kOneGroup ? 0 : i;
      sx[i] *= rstd[h];
      total[i] += s[i];
      total_x[i] += sx[i];
      both[0][h] += s[i] * w[i];
      both[1][h] += sx[i] * w[i];
    }
    if (!a.o.p) continue;
    r.group_sums(c, both);
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.ldb + c.ch;
    // dI = dZ (weight rstd) - rstd avg d - (x - mean) rstd^2 avg(d xhat)
    const float by = stretch(rstd), inverse_by = __builtin_amdgcn_rcpf(by);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      both[0][i] *= inverse_n * rstd[i];
      both[1][i] *= inverse_n * rstd[i] * (rstd[i] * inverse_by);
    }
    by_act(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < RV; ++k) {
        const int p = r.row + k * a.rows;
        if (there && p < a.s) {
          float dz[V], t[V];
          slopes<T, decltype(act)::value, MODE>(x[k], d[k], mean, scale, b, dz, t);
#pragma unroll
          for (int i = 0; i < V; ++i) dz[i] = dz[i] * scale[i] - both[0][MODE == kOneGroup ? 0 : i] - t[i] * by * both[1][MODE == kOneGroup ? 0 : i];
          c.template write<false>(to + p * a.o.ld, dz);
        }
      }
    });
  }
  if (!a.sums) return;
  // sums by channel over this workgroup's threads
  const int lines = a.slots * a.rows, width = a.vecs * V;
  int lanes = 64;
  while (lanes > 1 && lanes * width > NT) lanes >>= 1;
  const int lane = threadIdx.x & (lanes - 1), step = NT / lanes, base = r.base;
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if (r.slot < a.slots) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c.mine(i)) lds[r.line * width + r.vec * V + i - c.skip] = which ? total_x[i] : total[i];
    }
    __syncthreads();
    float* to = a.sums + (which * a.parts + r.block) * a.c + base;
    for (int i0 = 0; i0 < width; i0 += step) {
      const int i = i0 + threadIdx.x / lanes;
      float v = 0.0f;
      if (i < width)
        for (int e = lane; e < lines; e += lanes) v += lds[e * width + i];
      for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor(v, d);
      if (lane == 0 && i < width && base + i < a.c) to[i] = v;
    }
  }
}

template <class T, int RV, bool WHOLE, int NT> __global__ __launch_bounds__(NT) void norm_feature_grad_kernel(Norm a) {
  constexpr int V = kVec<T>;
  // the sums of three waves, or the two joins of eight
  __shared__ float sh[2][NT == 512 ? 1 : 3][NT == 512 ? 8 : 64 * RV * V];
  const Feature<T, RV, WHOLE, NT> f(a);
  float w[RV][V], b[RV][V], total[RV][V], total_x[RV][V];
#pragma unroll
  for (int k = 0; k < RV; ++k) {
    f.values(a.weight, 1.0f, k, w[k]);
    f.values(a.bias, 0.0f, k, b[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) total[k][i] = total_x[k][i] = 0.0f;
  }
  const float inverse_n = 1.0f / (float)a.per;
  const int g = min(f.g, a.groups - 1);
  for (int64_t n = f.n; n < a.b; n += f.step) {
    Packed<T> x[RV], d[RV];
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      x[k] = f.read(a.x, n, k);
      d[k] = f.read(a.d, n, k);
    }
    const float mean = a.mean[n * a.groups + g], rstd = a.rstd[n * a.groups + g];
    by_act(a.act, [&](auto act) {
      float s = 0.0f, sx = 0.0f, dz[RV][V], t[RV][V];
#pragma unroll
      for (int k = 0; k < RV; ++k) {
        float scale[V];
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] = rstd * w[k][i];
        slopes<T, decltype(act)::value, kOneGroup>(x[k], d[k], &mean, scale, b[k], dz[k], t[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          t[k][i] *= rstd;                              // xhat
          const bool mine = f.any[k] && f.mine(k, i);
          total[k][i] += dz[k][i];
          total_x[k][i] += dz[k][i] * t[k][i];
          s += mine ? dz[k][i] * w[k][i] : 0.0f;
          sx += mine ? dz[k][i] * w[k][i] * t[k][i] : 0.0f;
        }
      }
      if (!a.o.p) return;
      s = f.sum(s, a.lanes, sh[0][0]) * inverse_n;
      sx = f.sum(sx, a.lanes, sh[1][0]) * inverse_n;
#pragma unroll
      for (int k = 0; k < RV; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) dz[k][i] = rstd * (dz[k][i] * w[k][i] - s - t[k][i] * sx);
        if (f.any[k]) f.write(a.o, n, k, dz[k]);
      }
    });
  }
  if (!a.sums) return;
  // four images' waves have the same channels
  const int lane = threadIdx.x & 63, wave = NT == 512 ? 0 : threadIdx.x >> 6;
  if (wave > 0) {
#pragma unroll
    for (int k = 0; k < RV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        sh[0][wave - 1][(k * V + i) * 64 + lane] = total[k][i];
        sh[1][wave - 1][(k * V + i) * 64 + lane] = total_x[k][i];
      }
  }
  __syncthreads();
  if (wave > 0) return;
  float* to = a.sums + (int64_t)(blockIdx.x / a.units) * a.c;
#pragma unroll
  for (int k = 0; k < RV; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float s = total[k][i], sx = total_x[k][i];
#pragma unroll
      for (int v = 0; v < (NT == 512 ? 0 : 3); ++v) {
        s += sh[0][v][(k * V + i) * 64 + lane];
        sx += sh[1][v][(k * V + i) * 64 + lane];
      }
      if (f.any[k] && f.mine(k, i)) {
        to[f.at[k] + i] = s;
        to[a.parts * a.c + f.at[k] + i] = sx;
      }
    }
}

// dweight and dbias: the parts of a channel added in a fixed order; a.span (8 or 64)
// channels of a workgroup, NT / span threads each, one output a workgroup (the weights' first).
template <class T, int NT> __device__ inline void channel_sums(const Norm& a, int block) {
  __shared__ float sh[NT];
  const int span = a.span, blocks = (a.c + span - 1) / span, which = block >= blocks ? 1 : 0, lines = NT / span;
  T* to = static_cast<T*>(which ? a.dbias : a.dweight);
  if (!to) return;
  const int x = threadIdx.x & (span - 1), y = threadIdx.x / span, ch = (block - which * blocks) * span + x;
  float s = 0.0f;
  if (ch < a.c) {
    const float* p = a.sums + (which ? 0 : a.parts * a.c) + ch;
    // 64 at a time, so that a thread's sum stays short
    for (int64_t lo = y; lo < a.parts; lo += 64 * lines) {
      float t = 0.0f;
#pragma unroll 8
      for (int64_t i = lo; i < min(a.parts, lo + 64 * lines); i += lines) t += p[i * a.c];
      s += t;
    }
  }
  // lanes `span` apart have the same channel
  for (int d = span; d < 64; d <<= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) < span) sh[(threadIdx.x >> 6) * span + x] = s;
  __syncthreads();
  if (y > 0 || ch >= a.c) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) s += sh[i * span + x];
  to[ch] = (T)s;
}

template <class T, int NT> __global__ __launch_bounds__(NT) void norm_sums_kernel(Norm a) { channel_sums<T, NT>(a, blockIdx.x); }

// Sums of dZ and dZ xhat by chunk and channel.
template <class T, int MODE> __global__ __launch_bounds__(kSplitThreads) void norm_slopes_kernel(Norm a) {
  constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  __shared__ float sh[(kSplitThreads + 256) * V];
  for (int id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place<T, MODE> p(a, id);
    float s[V], sx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = sx[i] = 0.0f;
    if (p.owner) {
      float scale[V], b[V], mean[H], rstd[H];
      int64_t at[H];
      p.c.values(a.weight, 1.0f, scale);
      p.c.values(a.bias, 0.0f, b);
      group_values<T, MODE>(a, p, at, mean, rstd);
#pragma unroll
      for (int i = 0; i < V; ++i) scale[i] *= rstd[MODE == kOneGroup ? 0 : i];
      by_act(a.act, [&](auto act) {
        each_position<T, MODE, true>(a, p, [&](int, const Packed<T>& x, const Packed<T>& d) {
          float dz[V], t[V];
          slopes<T, decltype(act)::value, MODE>(x, d, mean, scale, b, dz, t);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            s[i] += dz[i];
            sx[i] += dz[i] * t[i];
          }
        });
      });
#pragma unroll
      for (int i = 0; i < V; ++i) sx[i] *= rstd[MODE == kOneGroup ? 0 : i];
    }
    over_rows<T, MODE>(a, p, sh, s, s);
    over_rows<T, MODE>(a, p, sh, sx, sx);
    if (p.row == 0 && p.owner) {
      float* to = a.sums + p.at * a.c + p.c.ch;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (p.c.mine(i)) {
          to[i] = s[i];
          to[a.parts * a.c + i] = sx[i];
        }
    }
  }
}

// The chunks' sums of each channel and image, as of one chunk.
__global__ __launch_bounds__(kJoinThreads) void norm_chunks_kernel(Norm a, float* to) {
  __shared__ float sh[kJoinThreads];
  each_channel(a, [&](int64_t n, int ch, bool there, int line) {
    const float* from = a.sums + n * a.chunks * a.c + ch;
    float s = 0.0f, sx = 0.0f;
    if (there) {
#pragma unroll 4
      for (int k = line; k < a.chunks; k += kChannelLines) {
        s += from[(int64_t)k * a.c];
        sx += from[(a.parts + k) * a.c];
      }
    }
    s = channel_sum(s, sh);
    sx = channel_sum(sx, sh);
    if (there && line == 0) {
      to[n * a.c + ch] = s;
      to[(a.b + n) * a.c + ch] = sx;
    }
  });
}

// The groups' avg d and avg(d xhat) from the sums of their chunks and channels.
template <class T> __global__ __launch_bounds__(kJoinThreads) void norm_averages_kernel(Norm a) {
  __shared__ float sh[kJoinThreads / 64];
  const T* weight = static_cast<const T*>(a.weight);
  const float count = (float)a.per * (float)a.s;
  for (int64_t id = blockIdx.x; id < a.b * a.groups; id += gridDim.x) {
    const int64_t n = id / a.groups;
    const int first = (int)(id - n * a.groups) * a.per;
    const float* from = a.sums + n * a.chunks * a.c + first;
    float s = 0.0f, sx = 0.0f;
    each_entry(a, [&](int k, int i) {
      const float w = weight ? (float)weight[first + i] : 1.0f;
      s += w * from[(int64_t)k * a.c + i];
      sx += w * from[(a.parts + k) * a.c + i];
    });
    s = block_sum(s, sh) / count;
    sx = block_sum(sx, sh) / count;
    if (threadIdx.x == 0) a.part[id] = float2{s, sx};
  }
}

// The first `extra` workgroups add up dweight and dbias beside the others.
template <class T, int MODE, bool STREAM> __global__ __launch_bounds__(kSplitThreads) void norm_dx_kernel(Norm a) {
  constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  if ((int)blockIdx.x < a.extra) return channel_sums<T, kSplitThreads>(a, blockIdx.x);
  for (int id = blockIdx.x - a.extra; id < all_parts(a); id += gridDim.x - a.extra) {
    const Place<T, MODE> p(a, all_parts(a) - 1 - id);
    if (!p.owner) continue;
    float scale[V], b[V], mean[H], rstd[H], s[H], sx[H];
    int64_t at[H];
    p.c.values(a.weight, 1.0f, scale);
    p.c.values(a.bias, 0.0f, b);
    group_values<T, MODE>(a, p, at, mean, rstd);
    const float by = stretch(rstd), inverse_by = __builtin_amdgcn_rcpf(by);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float2 v = a.part[at[i]];
      s[i] = v.x * rstd[i];
      sx[i] = v.y * rstd[i] * (rstd[i] * inverse_by);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] *= rstd[MODE == kOneGroup ? 0 : i];
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + p.n * a.o.ldb + p.c.ch;
    by_act(a.act, [&](auto act) {
      each_position<T, MODE, true>(a, p, [&](int q, const Packed<T>& x, const Packed<T>& d) {
        float dz[V], t[V];
        slopes<T, decltype(act)::value, MODE>(x, d, mean, scale, b, dz, t);
#pragma unroll
        for (int i = 0; i < V; ++i) dz[i] = dz[i] * scale[i] - s[MODE == kOneGroup ? 0 : i] - t[i] * by * sx[MODE == kOneGroup ? 0 : i];
        p.c.template write<STREAM>(to + q * a.o.ld, dz);
      });
    });
  }
}

inline int sums_blocks(const Norm& a) { return 2 * (int)div_up(a.c, a.span); }

template <class T, int MODE> hipError_t launch_mode(Norm& a, const NormPlan& p, char* ws, bool want, hipStream_t s) {
  if (p.resident) {
    a.parts = p.blocks;
    a.sums = want ? reinterpret_cast<float*>(ws + p.sums) : nullptr;
    // group_sums() of two values, or the sums by channel behind the images
    const int64_t floats = std::max(2 * (p.threads * (int64_t)kHeld<T, MODE> + (int64_t)p.slots * p.unit_groups * p.shares),
                                    p.threads * (int64_t)kVec<T>);
    if constexpr (MODE == kTiny) {
      return start_resident(norm_resident_grad_kernel<T, 256, 8, MODE>, p, a, floats, s);
    } else {
      if (p.threads == 512) return start_resident(norm_resident_grad_kernel<T, 512, 8, MODE>, p, a, floats, s);
      switch (p.held) {
        case 1: return start_resident(norm_resident_grad_kernel<T, 256, 1, MODE>, p, a, floats, s);
        case 4: return start_resident(norm_resident_grad_kernel<T, 256, 4, MODE>, p, a, floats, s);
        default: return start_resident(norm_resident_grad_kernel<T, 256, 8, MODE>, p, a, floats, s);
      }
    }
  }
  a.parts = a.b * p.chunks;
  a.sums = reinterpret_cast<float*>(ws + p.sums);
  dim3 grid = grid_of(a.b * p.chunks * p.units);
  norm_slopes_kernel<T, MODE><<<grid, kSplitThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Norm join = a;
  if (p.wide) {
    join.sums = reinterpret_cast<float*>(ws + p.joined);
    join.parts = a.b, join.chunks = 1;
    norm_chunks_kernel<<<grid_of(a.b * div_up(a.c, 64)), kJoinThreads, 0, s>>>(a, join.sums);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.sums = join.sums, a.parts = join.parts;
  }
  if (!a.o.p) return e;
  norm_averages_kernel<T><<<grid_of(a.b * a.groups), join_threads((int64_t)a.per * join.chunks), 0, s>>>(join);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  a.extra = want ? sums_blocks(a) : 0;
  grid.x += a.extra;
  if (streamed<T>(a))
    norm_dx_kernel<T, MODE, true><<<grid, kSplitThreads, 0, s>>>(a);
  else
    norm_dx_kernel<T, MODE, false><<<grid, kSplitThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class T, bool WHOLE> hipError_t launch_feature(const NormPlan& p, const Norm& a, hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<dim3((unsigned)((int64_t)p.units * p.blocks)), p.threads, 0, s>>>(a);
    return hipGetLastError();
  };
  if (p.threads == 512) {
    switch (p.held) {
      case 1: return go(norm_feature_grad_kernel<T, 1, WHOLE, 512>);
      case 2: return go(norm_feature_grad_kernel<T, 2, WHOLE, 512>);
      default: return go(norm_feature_grad_kernel<T, 4, WHOLE, 512>);
    }
  }
  switch (p.held) {
    case 1: return go(norm_feature_grad_kernel<T, 1, WHOLE, 256>);
    case 2: return go(norm_feature_grad_kernel<T, 2, WHOLE, 256>);
    default: return go(norm_feature_grad_kernel<T, 4, WHOLE, 256>);
  }
}

template <class T, int NT> hipError_t launch_sums(const Norm& a, hipStream_t s) {
  norm_sums_kernel<T, NT><<<dim3((unsigned)sums_blocks(a)), NT, 0, s>>>(a);
  return hipGetLastError();
}

template <class T> hipError_t launch_norm_grad(Norm a, const NormPlan& p, char* ws, hipStream_t s) {
  fill<T>(a, p, ws);
  const bool want = a.dweight || a.dbias;
  hipError_t e;
  if (p.feature) {
    a.parts = p.blocks;
    a.sums = want ? reinterpret_cast<float*>(ws + p.sums) : nullptr;
    e = p.mode == kOneGroup ? launch_feature<T, true>(p, a, s) : launch_feature<T, false>(p, a, s);
  } else {
    e = by_mode(p.mode, [&](auto mode) { return launch_mode<T, decltype(mode)::value>(a, p, ws, want, s); });
  }
  // split gradients have added them up beside dI already; without it, in the same order
  if (e != hipSuccess || !want || a.extra) return e;
  return p.feature || p.resident ? launch_sums<T, 1024>(a, s) : launch_sums<T, kSplitThreads>(a, s);
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_group_norm_backward_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  return c * s * b == 0 ? 0 : plan_of(dtype, c, s, b, groups, true).bytes;
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
  a.weight = weight, a.bias = bias, a.dweight = dweight, a.dbias = dbias, a.act = act;
  a.span = c >= kSpanChannels ? 64 : 8;
  a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
  char* ws = static_cast<char*>(workspace);
  hipError_t e = hipSuccess;
  auto go = [&](auto* none) {
    using T = std::remove_pointer_t<decltype(none)>;
    if (work) return launch_norm_grad<T>(a, p, ws, stream);
    // nothing to add up: zeros
    if (!dweight && !dbias) return hipSuccess;
    return launch_sums<T, kSplitThreads>(a, stream);
  };
  e = dtype == LINEAR_F32 ? go((float*)nullptr) : dtype == LINEAR_BF16 ? go((bf16*)nullptr) : go((f16*)nullptr);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}
