// Group norm with an activation, channels fastest.
#include "group_norm_common.h"

namespace linear {
namespace {

template <class T, int NT, int RV, int MODE> __global__ __launch_bounds__(NT) void norm_resident_kernel(Norm a) {
  constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  Resident<T, NT, MODE> r(a, lds);
  const Channels<T, MODE> c(a, r.base + r.vec * V);
  r.place(c);
  float w[V], b[V];
  c.values(a.weight, 1.0f, w);
  c.values(a.bias, 0.0f, b);
  const Count count((float)a.per * (float)a.s);
  for (int64_t n0 = (int64_t)r.block * a.slots; n0 < a.b; n0 += (int64_t)a.blocks * a.slots) {
    const int64_t n = n0 + r.slot;
    const bool there = r.owner && n < a.b;
    Packed<T> x[RV];
    float mean[1][H], rstd[1][H];
#pragma unroll
    for (int i = 0; i < H; ++i) mean[0][i] = rstd[0][i] = 0.0f;
    const T* from = static_cast<const T*>(a.x.p) + n * a.x.ldb + c.ch;
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      const int p = r.row + k * a.rows;
      if (there && p < a.s) x[k] = c.read(from + p * a.x.ld);
    }
#pragma unroll
    for (int k = 0; k < RV; ++k)
      if (there && r.row + k * a.rows < a.s) {
#pragma unroll
        for (int i = 0; i < V; ++i) mean[0][MODE == kOneGroup ? 0 : i] += (float)x[k].v[i];
      }
    r.group_sums(c, mean);
#pragma unroll
    for (int i = 0; i < H; ++i) mean[0][i] = count.quotient(mean[0][i]);
#pragma unroll
    for (int k = 0; k < RV; ++k)
      if (there && r.row + k * a.rows < a.s) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = (float)x[k].v[i] - mean[0][MODE == kOneGroup ? 0 : i];
          rstd[0][MODE == kOneGroup ? 0 : i] += d * d;
        }
      }
    r.group_sums(c, rstd);
#pragma unroll
    for (int i = 0; i < H; ++i) rstd[0][i] = rstd_of(rstd[0][i], count, a.eps);
    if (there && r.row == 0) {
      // the threads that have a group's first channel
#pragma unroll
      for (int i = 0; i < H; ++i)
        if (c.mine(i) && r.local[i] * (int)a.run.d == (MODE == kOneGroup ? r.vec : r.vec * V + i - c.skip)) {
          const int64_t at = n * a.groups + r.first + r.local[i];
          if (a.mean) a.mean[at] = mean[0][i];
          if (a.rstd) a.rstd[at] = rstd[0][i];
        }
    }
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.ldb + c.ch;
    float scale[V];
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] = rstd[0][MODE == kOneGroup ? 0 : i] * w[i];
    by_act(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < RV; ++k) {
        const int p = r.row + k * a.rows;
        if (there && p < a.s) {
          float z[V];
#pragma unroll
          for (int i = 0; i < V; ++i)
            z[i] = act_value<T, decltype(act)::value>(((float)x[k].v[i] - mean[0][MODE == kOneGroup ? 0 : i]) * scale[i] + b[i]);
          c.template write<false>(to + p * a.o.ld, z);
        }
      }
    });
  }
}

template <class T, int RV, int IM, bool WHOLE, int NT> __global__ __launch_bounds__(NT) void norm_feature_kernel(Norm a) {
  constexpr int V = kVec<T>;
  __shared__ float sh[2][NT / 64];
  const Feature<T, RV, WHOLE, NT> f(a);
  float w[RV][V], b[RV][V];
#pragma unroll
  for (int k = 0; k < RV; ++k) {
    f.values(a.weight, 1.0f, k, w[k]);
    f.values(a.bias, 0.0f, k, b[k]);
  }
  const Count count((float)a.per);
  for (int64_t n0 = f.n; n0 < a.b; n0 += IM * f.step) {
    Packed<T> x[IM][RV];
    float mean[IM], rstd[IM];
    // images behind the last are read as the last one again and not written
#pragma unroll
    for (int m = 0; m < IM; ++m)
#pragma unroll
      for (int k = 0; k < RV; ++k) x[m][k] = f.read(a.x, min(n0 + m * f.step, a.b - 1), k);
#pragma unroll
    for (int m = 0; m < IM; ++m) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < RV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s += f.any[k] && f.mine(k, i) ? (float)x[m][k].v[i] : 0.0f;
      mean[m] = count.quotient(f.sum(s, a.lanes, sh[0]));
    }
#pragma unroll
    for (int m = 0; m < IM; ++m) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < RV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = (float)x[m][k].v[i] - mean[m];
          s += f.any[k] && f.mine(k, i) ? d * d : 0.0f;
        }
      rstd[m] = rstd_of(f.sum(s, a.lanes, sh[1]), count, a.eps);
    }
    by_act(a.act, [&](auto act) {
#pragma unroll
      for (int m = 0; m < IM; ++m) {
        const int64_t n = n0 + m * f.step;
        if (n >= a.b) break;
        if (f.any[0] && (threadIdx.x & (a.lanes - 1)) == 0) {
          if (a.mean) a.mean[n * a.groups + f.g] = mean[m];
          if (a.rstd) a.rstd[n * a.groups + f.g] = rstd[m];
        }
#pragma unroll
        for (int k = 0; k < RV; ++k) {
          float z[V];
#pragma unroll
          for (int i = 0; i < V; ++i) z[i] = act_value<T, decltype(act)::value>(((float)x[m][k].v[i] - mean[m]) * (rstd[m] * w[k][i]) + b[k][i]);
          if (f.any[k]) f.write(a.o, n, k, z);
        }
      }
    });
  }
}

// Mean and squares around it of each channel over a chunk: a thread takes its values
// relative to its first one, four at a time around the mean of those before,
//   d = x - mean,   mean += sum d / n,   squares += sum d^2 - (sum d)^2 / n,
// n with the four.  At least half of sum d^2 stays (a quarter of the first four), whatever lies
// far from the others; relative to the first value alone, a far one there left the difference of
// sums as large as all of them (a value of 10^6 before 256 of 0.1: rstd off by 3e-4).  Then the
// threads are joined by their means.
template <class T, int MODE> __global__ __launch_bounds__(kSplitThreads) void norm_stats_kernel(Norm a) {
  constexpr int V = kVec<T>;
  __shared__ float sh[(kSplitThreads + 256) * V];
  for (int id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place<T, MODE> p(a, id);
    float first[V], m[V], s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) first[i] = m[i] = q[i] = 0.0f;
    int mine = 0;
    if (p.owner)
      each_batch<T, MODE, false>(a, p, [&](int at, const Packed<T>(&x)[kAhead], const Packed<T>(&)[kAhead]) {
        if (mine == 0) {
#pragma unroll
          for (int i = 0; i < V; ++i) first[i] = (float)x[0].v[i];
        }
        // COUNT values from the k-th on
        auto take = [&](int k, auto COUNT) {
          constexpr int count = decltype(COUNT)::value;
          mine += count;
          const float over = __builtin_amdgcn_rcpf((float)mine);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float sum = 0.0f, squares = 0.0f;
#pragma unroll
            for (int j = 0; j < count; ++j) {
              const float d = (float)x[k + j].v[i] - first[i] - m[i];
              sum += d;
              squares += d * d;
            }
            const float by = sum * over;
            m[i] += by;
            q[i] += squares - by * sum;
          }
        };
        if (at + (kAhead - 1) * p.rows < p.hi) return take(0, std::integral_constant<int, kAhead>{});
#pragma unroll
        for (int k = 0; k < kAhead - 1; ++k)
          if (at + k * p.rows < p.hi) take(k, std::integral_constant<int, 1>{});
      });
    const float count = (float)mine;
    float mean[V], square[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      first[i] += m[i];                     // this thread's mean
      s[i] = first[i] * count;
    }
    over_rows<T, MODE>(a, p, sh, s, mean);
    const Count n((float)(p.hi - p.lo));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mean[i] = n.quotient(mean[i]);
      const float d = first[i] - mean[i];
      q[i] += mine ? count * d * d : 0.0f;
    }
    over_rows<T, MODE>(a, p, sh, q, square);
    if (p.row == 0 && p.owner) {
      float2* to = a.part + p.at * a.c + p.c.ch;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (p.c.mine(i)) to[i] = float2{mean[i], square[i]};
    }
  }
}

__device__ inline float chunk_length(const Norm& a, int chunk) { return (float)min(a.chunk, a.s - chunk * a.chunk); }

// Mean and squares around it of each channel and image from its chunks, as of one chunk.
__global__ __launch_bounds__(kJoinThreads) void norm_channels_kernel(Norm a, float2* to) {
  __shared__ float sh[kJoinThreads];
  each_channel(a, [&](int64_t n, int ch, bool there, int line) {
    const float2* from = a.part + n * a.chunks * a.c + ch;
    float s = 0.0f, q = 0.0f;
    if (there) {
#pragma unroll 4
      for (int k = line; k < a.chunks; k += kChannelLines) s += from[(int64_t)k * a.c].x * chunk_length(a, k);
    }
    const float m = channel_sum(s, sh) / (float)a.s;
    if (there) {
#pragma unroll 4
      for (int k = line; k < a.chunks; k += kChannelLines) {
        const float2 v = from[(int64_t)k * a.c];
        q += v.y + chunk_length(a, k) * (v.x - m) * (v.x - m);
      }
    }
    q = channel_sum(q, sh);
    if (there && line == 0) to[n * a.c + ch] = float2{m, q};
  });
}

// The groups' mean and rstd from their chunks and channels.
__global__ __launch_bounds__(kJoinThreads) void norm_groups_kernel(Norm a) {
  __shared__ float sh[kJoinThreads / 64];
  for (int64_t id = blockIdx.x; id < a.b * a.groups; id += gridDim.x) {
    const int64_t n = id / a.groups;
    const float2* from = a.part + n * a.chunks * a.c + (id - n * a.groups) * a.per;
    float s = 0.0f;
    each_entry(a, [&](int k, int i) { s += from[(int64_t)k * a.c + i].x * chunk_length(a, k); });
    const float all = (float)a.per * (float)a.s;
    const float m = block_sum(s, sh) / all;
    s = 0.0f;
    each_entry(a, [&](int k, int i) {
      const float2 v = from[(int64_t)k * a.c + i];
      s += v.y + chunk_length(a, k) * (v.x - m) * (v.x - m);
    });
    s = block_sum(s, sh);
    if (threadIdx.x == 0) {
      a.mean[id] = m;
      a.rstd[id] = rstd_of(s, Count(all), a.eps);
    }
  }
}

// O from the statistics; from the last part back, so that what the first pass read last
// is read first, from the caches.
template <class T, int MODE, bool STREAM> __global__ __launch_bounds__(kSplitThreads) void norm_apply_kernel(Norm a) {
  constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  for (int id = blockIdx.x; id < all_parts(a); id += gridDim.x) {
    const Place<T, MODE> p(a, all_parts(a) - 1 - id);
    if (!p.owner) continue;
    float scale[V], b[V], mean[H], rstd[H];
    int64_t at[H];
    p.c.values(a.weight, 1.0f, scale);
    p.c.values(a.bias, 0.0f, b);
    group_values<T, MODE>(a, p, at, mean, rstd);
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] *= rstd[MODE == kOneGroup ? 0 : i];
    T* to = static_cast<T*>(const_cast<void*>(a.o.p)) + p.n * a.o.ldb + p.c.ch;
    by_act(a.act, [&](auto act) {
      each_position<T, MODE, false>(a, p, [&](int q, const Packed<T>& x, const Packed<T>&) {
        float z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = act_value<T, decltype(act)::value>(((float)x.v[i] - mean[MODE == kOneGroup ? 0 : i]) * scale[i] + b[i]);
        p.c.template write<STREAM>(to + q * a.o.ld, z);
      });
    });
  }
}

// The mean and rstd of no values: 0 / 0.
__global__ __launch_bounds__(256) void norm_nothing_kernel(int64_t count, float* mean, float* rstd) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
    if (mean) mean[i] = NAN;
    if (rstd) rstd[i] = NAN;
  }
}

template <class T, int MODE> hipError_t launch_mode(Norm a, const NormPlan& p, char* ws, hipStream_t s) {
  if (p.resident) {
    const int64_t floats = p.threads * (int64_t)kHeld<T, MODE> + (int64_t)p.slots * p.unit_groups * p.shares;
    if constexpr (MODE == kTiny) {
      return start_resident(norm_resident_kernel<T, 256, 8, MODE>, p, a, floats, s);
    } else {
      if (p.threads == 512) return start_resident(norm_resident_kernel<T, 512, 8, MODE>, p, a, floats, s);
      switch (p.held) {
        case 1: return start_resident(norm_resident_kernel<T, 256, 1, MODE>, p, a, floats, s);
        case 4: return start_resident(norm_resident_kernel<T, 256, 4, MODE>, p, a, floats, s);
        default: return start_resident(norm_resident_kernel<T, 256, 8, MODE>, p, a, floats, s);
      }
    }
  }
  if (!a.mean) a.mean = reinterpret_cast<float*>(ws + p.stats);
  if (!a.rstd) a.rstd = reinterpret_cast<float*>(ws + p.stats + up(a.b * a.groups * 4));
  const dim3 grid = grid_of(a.b * p.chunks * p.units);
  norm_stats_kernel<T, MODE><<<grid, kSplitThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Norm join = a;
  if (p.wide) {
    join.part = reinterpret_cast<float2*>(ws + p.joined);
    join.chunks = 1, join.chunk = a.s;
    norm_channels_kernel<<<grid_of(a.b * div_up(a.c, 64)), kJoinThreads, 0, s>>>(a, join.part);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  norm_groups_kernel<<<grid_of(a.b * a.groups), join_threads((int64_t)a.per * join.chunks), 0, s>>>(join);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (streamed<T>(a))
    norm_apply_kernel<T, MODE, true><<<grid, kSplitThreads, 0, s>>>(a);
  else
    norm_apply_kernel<T, MODE, false><<<grid, kSplitThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class T, bool WHOLE> hipError_t launch_feature(const NormPlan& p, const Norm& a, hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<dim3((unsigned)((int64_t)p.units * p.blocks)), p.threads, 0, s>>>(a);
    return hipGetLastError();
  };
  if (p.threads == 512) {
    switch (p.held) {
      case 1: return go(norm_feature_kernel<T, 1, 1, WHOLE, 512>);
      case 2: return go(norm_feature_kernel<T, 2, 1, WHOLE, 512>);
      default: return go(norm_feature_kernel<T, 4, 1, WHOLE, 512>);
    }
  }
  switch (p.held) {
    case 1: return go(norm_feature_kernel<T, 1, 2, WHOLE, 256>);
    case 2: return go(norm_feature_kernel<T, 2, 2, WHOLE, 256>);
    default: return go(norm_feature_kernel<T, 4, 1, WHOLE, 256>);
  }
}

template <class T> hipError_t launch_norm(Norm a, const NormPlan& p, char* ws, hipStream_t s) {
  fill<T>(a, p, ws);
  if (p.feature) return p.mode == kOneGroup ? launch_feature<T, true>(p, a, s) : launch_feature<T, false>(p, a, s);
  return by_mode(p.mode, [&](auto mode) { return launch_mode<T, decltype(mode)::value>(a, p, ws, s); });
}

}  // namespace
}  // namespace linear

extern "C" int64_t convgemm_group_norm_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  using namespace linear;
  if (int e = check_norm(dtype, c, s, b, groups)) return e;
  return c * s * b == 0 ? 0 : plan_of(dtype, c, s, b, groups, false).bytes;
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
  if (!work) {
    if (b == 0 || (!mean && !rstd)) return LINEAR_OK;
    norm_nothing_kernel<<<grid_of(div_up(groups * b, 256)), 256, 0, stream>>>(groups * b, mean, rstd);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
  }
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

