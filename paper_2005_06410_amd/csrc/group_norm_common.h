// Shared by group norm (group_norm.hip) and its gradients (group_norm_grad.hip).
//
// What a thread owns is always one 16-byte vector of channels (V = 4 or 8), at every
// `rows`-th position: neighbouring threads take neighbouring vectors, so that loads are
// whole lines, and sums by channel stay in one thread's registers until the end.
//
// All of it is bound by memory, and by latencies where there is little (a kernel of this
// kind takes 4 to 5 us at least).  Three ways:
// * features (one position an image): a group in the lanes of a wave, no barriers.  4001
//   tokens of 1000 channels bf16, GELU: 12 us, gradients 14 (through LDS: 23 and 34).
// * resident: a unit of whole groups in a workgroup's registers, one read and one write.  27 x
//   27 x 256 x 80 fp32, 32 groups: 26 us (4.6 TB/s), gradients 40 (4.5 TB/s).
// * split, for larger maps: two reads.  256 x 256 x 128 x 16 bf16: 50 us for the statistics
//   (5.4 TB/s), 92 for the result (5.9), 102 and 138 for the gradients (5.2 and 5.8).  Rounds of
//   images that the last-level cache could hold from the first pass to the second were no
//   faster (162 us instead of 146 forward): the second read is not what bounds it, and each round adds three launches.
#pragma once

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

// x / d for x d < 2^32 by one multiplication.
struct Divider {
  uint32_t d, m;
  __device__ int operator()(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }
};

struct Norm {
  int c, s, groups, per;            // per: channels of a group
  int64_t b;
  Map x, d;                         // input; dO (gradients)
  const void* weight;
  const void* bias;
  void* dweight;
  void* dbias;
  int act;
  float eps;
  Map o;                            // O, or dI
  float* mean;
  float* rstd;
  float* sums;                      // gradients: by channel, [parts][c] of dZ and, behind them, of dZ xhat
  int64_t parts;
  // resident kernels
  int vecs, units, unit_groups;     // vectors of a unit, units of an image, groups of a unit
  int rows, slots;                  // threads along positions of one image, images at a time
  int lanes, shares;                // lanes that add up one share of a group, shares of a group
  int blocks;                       // workgroups along the images
  Divider vec, row, run, group;     // by vecs, rows, a group's values in a line, a unit's groups
  // split kernels
  int chunk, chunks;                // positions of a chunk, chunks of an image
  float2* part;                     // [b][chunks][c] mean and squares around it; or [b][groups] averages
  int extra, span;                  // gradients: workgroups that add up dweight and dbias, channels of one
};

// Channels from which a workgroup adds up 64 of them, and not 8 (the more threads for
// each): the gradients of 4096 tokens of 2048 channels fp32 38.2 us, with 8 41.0; of 1024 of 16384
// bf16 174 and 205.  1000 channels take the same either way.
constexpr int64_t kSpanChannels = 2048;

// How a thread's vector lies: its channels all in one group (per is a multiple of V), so
// that what belongs to a group is held once instead of V times; in several groups; in
// several groups and the last vector of a position not whole; or c < V.
enum Mode { kOneGroup, kWhole, kTail, kTiny };
template <class T, int MODE> constexpr int kHeld = MODE == kOneGroup ? 1 : kVec<T>;

// The channels of a thread.  The last vector of a position that is no whole one begins
// earlier, so that it ends with the last channel, and its first `skip` channels are the
// vector's before it: loads are then whole vectors everywhere (a load that may also be
// one of single values is compiled to four narrow ones: 153 channels of 143 x 59 x 26 bf16
// forward and gradients 137 instead of 392 us).
template <class T, int MODE> struct Channels {
  static constexpr int V = kVec<T>;
  int ch, skip, cnt;
  bool any;

  __device__ Channels(const Norm& a, int at) {
    any = at < a.c;
    ch = at, skip = 0, cnt = V;
    if (MODE == kTail && at > a.c - V) {
      ch = a.c - V;
      skip = at - ch;
    }
    if (MODE == kTiny) cnt = a.c;
  }
  __device__ bool mine(int i) const { return (MODE != kTail || i >= skip) && (MODE != kTiny || i < cnt); }

  __device__ Packed<T> read(const T* p) const {
    if (MODE != kTiny) return *reinterpret_cast<const Packed<T>*>(p);
    Packed<T> q;
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = p[min(i, cnt - 1)];
    return q;
  }
  template <bool STREAM> __device__ void write(T* p, const float* v) const {
    if (MODE < kTail || (MODE == kTail && skip == 0)) return result_vec<T, STREAM>(p, v);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (mine(i)) p[i] = (T)v[i];
  }
  // weight or bias, `other` without one
  __device__ void values(const void* p, float other, float* v) const {
    if (!p || !any) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = other;
    } else {
      const Packed<T> q = read(static_cast<const T*>(p) + ch);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (float)q.v[i];
    }
  }
};

// f(activation as a constant): one branch for a whole kernel.
template <class F> __device__ inline void by_act(int act, F f) {
  if (act == LINEAR_ACT_NONE) return f(std::integral_constant<int, LINEAR_ACT_NONE>{});
  with_act(act, f);
}

// sum / n rounded once, by n's inverse and what the product loses: three operations
// where a division takes ten (27 x 27 x 256 x 80 fp32, 32 groups: 25.9 us, with divisions and a
// root 28.8).  The inverse's rounding alone would be the same way in every group.
struct Count {
  float n, inverse;
  __device__ explicit Count(float v) : n(v), inverse(1.0f / v) {}
  __device__ float quotient(float sum, float* lost = nullptr) const {
    const float first = sum * inverse;
    if (!(fabsf(first) < INFINITY)) return first;        // nothing is lost of it, and inf - inf is not inf
    const float q = fmaf(fmaf(-first, n, sum), inverse, first);
    if (lost) *lost = fmaf(-q, n, sum) * inverse;
    return q;
  }
};

// 1 / sqrt(sum / n + eps), rounded about once, since what follows multiplies by it: the
// quotient and the sum with what their roundings lose, the hardware's root and one step of
// Newton's.
__device__ inline float rstd_of(float sum, const Count& n, float eps) {
  float lost = 0.0f;
  const float q = n.quotient(sum, &lost), v = q + eps, e = v - q;
  lost += (q - (v - e)) + (eps - e);
  // no sum of normal size (0 and NaN among them) has a finite root to go on from
  if (!(v >= 1.17549435e-38f && v < INFINITY)) return 1.0f / sqrtf(v);
  const float r = __builtin_amdgcn_rsqf(v), p = v * r;
  const float left = fmaf(-p, r, 1.0f) - (fmaf(v, r, -p) + lost * r) * r;   // 1 - (v + lost) r^2
  return fmaf(0.5f * r, left, r);
}

// ---------------------------------------------------------------------------
// resident: a unit (whole groups, whole vectors) of an image in registers
// ---------------------------------------------------------------------------
// One read and one write of everything.  Thread tid has vector tid % vecs of the unit
// and the positions row, row + rows, ... (row = tid / vecs % rows) of image slot
// tid / vecs / rows: maps smaller than a workgroup share it.
template <class T, int NT, int MODE> struct Resident {
  static constexpr int V = kVec<T>, H = kHeld<T, MODE>;
  const Norm& a;
  float* sh;                   // M times [lines][vecs][H], then M times the groups' shares
  int block, vec, line, row, slot, base, first;
  int local[H];                // groups of this thread's channels, in the unit
  bool owner;

  // Workgroup id -> unit and images.  Consecutive ids go to different XCDs; the units of
  // an image go to one, since they share its lines in the L2 cache.
  __device__ Resident(const Norm& n, float* lds) : a(n), sh(lds) {
    const int id = blockIdx.x, whole = (a.blocks & ~7) * a.units;
    int unit;
    if (id < whole) {
      const int j = id >> 3, q = j / a.units;
      unit = j - q * a.units;
      block = q * 8 + (id & 7);
    } else {
      const int q = (id - whole) / a.units;
      unit = id - whole - q * a.units;
      block = (a.blocks & ~7) + q;
    }
    const int tid = threadIdx.x;
    line = a.vec(tid);
    vec = tid - line * a.vecs;
    slot = a.row(line);
    row = line - slot * a.rows;
    base = unit * a.vecs * V;
    first = unit * a.unit_groups;
  }

  // run is a group's values in a line: per channels, or per / V vectors.
  __device__ void place(const Channels<T, MODE>& c) {
    owner = slot < a.slots && c.any;
#pragma unroll
    for (int i = 0; i < H; ++i)
      local[i] = min(a.run(MODE == kOneGroup ? vec : max(vec * V + i - c.skip, 0)), a.unit_groups - 1);
  }

  // The sums over a group and its image of M values by channel and thread; v[m] becomes
  // those of this thread's groups.  Threads without values bring zeros.
  template <int M> __device__ void group_sums(const Channels<T, MODE>& c, float (&v)[M][H]) {
    const int width = a.vecs * H, run = (int)a.run.d, each = a.rows * run, items = a.slots * a.unit_groups;
    if (slot < a.slots) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < H; ++i)
          if (c.mine(i)) sh[m * NT * H + line * width + vec * H + i - c.skip] = v[m][i];
    }
    __syncthreads();
    float* sums = sh + M * NT * H;
    const int lane = threadIdx.x & (a.lanes - 1), subs = items * a.shares, step = NT / a.lanes;
    for (int at = 0; at < subs; at += step) {
      const int sub = at + threadIdx.x / a.lanes, it = sub / a.shares, share = sub - it * a.shares;
      const int sl = a.group(min(it, items - 1)), g = min(it, items - 1) - sl * a.unit_groups;
      const float* from = sh + sl * a.rows * width + g * run;
      float s[M];
#pragma unroll
      for (int m = 0; m < M; ++m) s[m] = 0.0f;
      if (sub < subs)
        for (int e = share * a.lanes + lane; e < each; e += a.shares * a.lanes) {
          const int r = a.run(e);
#pragma unroll
          for (int m = 0; m < M; ++m) s[m] += from[m * NT * H + r * width + e - r * run];
        }
      for (int d = a.lanes >> 1; d > 0; d >>= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) s[m] += __shfl_xor(s[m], d);
      if (lane == 0 && sub < subs) {
#pragma unroll
        for (int m = 0; m < M; ++m) sums[m * subs + sub] = s[m];
      }
    }
    __syncthreads();
    const float* mine = sums + min(slot, a.slots - 1) * a.unit_groups * a.shares;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int i = 0; i < H; ++i) {
        float s = 0.0f;
        for (int k = 0; k < a.shares; ++k) s += mine[m * subs + local[i] * a.shares + k];
        v[m][i] = s;
      }
  }
};

// ---------------------------------------------------------------------------
// features: one position an image, a group in the lanes of a wave
// ---------------------------------------------------------------------------
// A group of `per` channels lies in `lanes` lanes of one wave, RV vectors each, so that its
// sums are a few exchanges between lanes, without LDS or barriers; 64 / lanes groups lie side
// by side.  A wave keeps its groups from image to image.  Groups too large for a wave (NT =
// 512) lie in a workgroup, which joins its waves' sums in LDS.  4096 tokens of 8192 channels
// bf16, one group: 39 us, gradients 93 (split: 277 and 533).
template <class T, int RV, bool WHOLE, int NT> struct Feature {
  static constexpr int V = kVec<T>, W = NT == 512 ? 1 : 4;   // images under way in a workgroup
  int64_t n, step;             // this wave's first image and the next one's distance
  int g, at[RV], skip[RV];     // group; first channel of each vector, and channels of it that are the one's before
  bool any[RV];

  __device__ Feature(const Norm& a) {
    const int lane = threadIdx.x & (NT / W - 1), wave = threadIdx.x / (NT / W), side = NT / W / a.lanes;
    const int sets = a.units, block = blockIdx.x / sets, set = blockIdx.x - block * sets;
    n = (int64_t)block * W + wave;
    step = (int64_t)a.blocks * W;
    g = set * side + lane / a.lanes;
    const int l = lane & (a.lanes - 1);
#pragma unroll
    for (int k = 0; k < RV; ++k) {
      int o = (l + k * a.lanes) * V;
      any[k] = g < a.groups && o < a.per;
      skip[k] = 0;
      if (!WHOLE && o > a.per - V) {
        skip[k] = o - (a.per - V);
        o = a.per - V;
      }
      at[k] = any[k] ? g * a.per + o : 0;
    }
  }
  __device__ bool mine(int k, int i) const { return WHOLE || i >= skip[k]; }
  __device__ Packed<T> read(const Map& m, int64_t image, int k) const {
    return *reinterpret_cast<const Packed<T>*>(static_cast<const T*>(m.p) + image * m.ldb + at[k]);
  }
  __device__ void write(const Map& m, int64_t image, int k, const float* v) const {
    T* p = static_cast<T*>(const_cast<void*>(m.p)) + image * m.ldb + at[k];
    if (WHOLE || skip[k] == 0) return store_vec(p, v);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i >= skip[k]) p[i] = (T)v[i];
  }
  __device__ void values(const void* p, float other, int k, float* v) const {
    Packed<T> q{};
    if (p) q = *reinterpret_cast<const Packed<T>*>(static_cast<const T*>(p) + at[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p ? (float)q.v[i] : other;
  }
  // over the group's lanes; sh: NT / 64 floats that the sum before did not use
  __device__ static float sum(float v, int lanes, float* sh) {
    for (int d = 1; d < min(lanes, 64); d <<= 1) v += __shfl_xor(v, d);
    if (NT == 512) {
      if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < NT / 64; ++i) v += sh[i];
    }
    return v;
  }
};

// ---------------------------------------------------------------------------
// split: chunks of an image's positions in workgroups of their own
// ---------------------------------------------------------------------------
// A first pass over the input gives sums by chunk and channel, a small launch the
// groups' statistics, and a second pass the result.
constexpr int kSplitThreads = 256;
constexpr int kAhead = 4;                          // vectors of each input that a thread has under way

// Part `id` of a launch: an image, a chunk and a block of up to 256 vectors; this
// thread's channels and first position.
template <class T, int MODE> struct Place {
  int vec, row, rows, lo, hi;
  int64_t n, at;                                   // image; chunk among all images
  Channels<T, MODE> c;
  bool owner;

  __device__ Place(const Norm& a, int id) : c(a, init(a, id)) { owner = row < rows && c.any; }

  __device__ int init(const Norm& a, int id) {
    const int rest = id / a.units, image = rest / a.chunks;
    n = image;
    at = rest;
    const int chunk = rest - image * a.chunks, first = (id - rest * a.units) * a.vecs;
    rows = kSplitThreads / a.vecs;
    row = threadIdx.x / a.vecs;
    vec = threadIdx.x - row * a.vecs;
    lo = chunk * a.chunk;
    hi = min(a.s, lo + a.chunk);
    return (first + vec) * kVec<T>;
  }
};

// Below 2^31: a part has thousands of values, and all of them are below 2^40.
__device__ inline int all_parts(const Norm& a) { return (int)a.b * a.chunks * a.units; }

// f(first position, vectors) for the positions of this thread, up to kAhead at a
// time, `rows` apart; all loads are issued before the first is used, since what f stores may
// be the input itself.
template <class T, int MODE, bool TWO, class F> __device__ inline void each_batch(const Norm& a, const Place<T, MODE>& p, F f) {
  const T* x = static_cast<const T*>(a.x.p) + p.n * a.x.ldb + p.c.ch;
  const T* d = TWO ? static_cast<const T*>(a.d.p) + p.n * a.d.ldb + p.c.ch : x;
  for (int at = p.lo + p.row; at < p.hi; at += kAhead * p.rows) {
    Packed<T> vx[kAhead], vd[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      // the last one again where there is none
      const int q = min(at + k * p.rows, p.hi - 1);
      vx[k] = p.c.read(x + q * a.x.ld);
      if (TWO) vd[k] = p.c.read(d + q * a.d.ld);
    }
    f(at, vx, vd);
  }
}

// f(position, vectors) for every position of this thread.
template <class T, int MODE, bool TWO, class F> __device__ inline void each_position(const Norm& a, const Place<T, MODE>& p, F f) {
  each_batch<T, MODE, TWO>(a, p, [&](int at, const Packed<T>(&vx)[kAhead], const Packed<T>(&vd)[kAhead]) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int q = at + k * p.rows;
      if (q < p.hi) f(q, vx[k], vd[k]);
    }
  });
}

// The sums over the workgroup's rows of one value by channel and thread, in every
// thread of the channel.  sh: (kSplitThreads + 256) V floats.
template <class T, int MODE> __device__ inline void over_rows(const Norm& a, const Place<T, MODE>& p, float* sh, const float* v, float* out) {
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

// Joins of a group's chunks have 1024 threads where there is that much to read, or 256 (512 x
// 100 x 100 fp32, 1 group: 133 us against 773; 60 maps of 31 x 45 x 90, 9 groups: 28.4 against 24.1).
constexpr int kJoinThreads = 1024;
inline int join_threads(int64_t entries) { return entries > 2048 ? kJoinThreads : 256; }

// A sum over all threads of a join, in each of them; sh: kJoinThreads / 64 floats.
__device__ inline float block_sum(float v, float* sh) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0f;
  for (int i = 0; i < (int)blockDim.x / 64; ++i) v += sh[i];
  return v;
}

// f(chunk, channel of the group) for a group's chunks and channels, dealt out to a
// workgroup's threads.
template <class F> __device__ inline void each_entry(const Norm& a, F f) {
  const int threads = blockDim.x;
  if (a.per >= threads) {
    for (int k = 0; k < a.chunks; ++k)
#pragma unroll 4
      for (int i = threadIdx.x; i < a.per; i += threads) f(k, i);
  } else {
    const int lines = threads / a.per, line = threadIdx.x / a.per, i = threadIdx.x - line * a.per;
    if (line < lines) {
#pragma unroll 4
      for (int k = line; k < a.chunks; k += lines) f(k, i);
    }
  }
}

template <class T, int MODE> __device__ inline void group_values(const Norm& a, const Place<T, MODE>& p, int64_t* at, float* mean, float* rstd) {
#pragma unroll
  for (int i = 0; i < kHeld<T, MODE>; ++i) {
    at[i] = p.n * a.groups + min(p.c.ch + i, a.c - 1) / a.per;
    mean[i] = a.mean[at[i]];
    rstd[i] = a.rstd[at[i]];
  }
}

// Where a group has many chunks and channels, its chunks are joined channel by channel
// first: 64 channels of an image in a workgroup, 16 threads for each of them.  2 maps of 40 x
// 40 x 2000 fp16, one group: 36 us (gradients 46) where one workgroup a group took 515 (526).  The
// limit is where the launch pays: 12800 entries (640 channels of 64 x 64, 32 groups) 23.3 us
// without it, 28.6 with it; 45000 (300 of 60 x 60, 2 groups) 32.6 and 25.2.
constexpr int kWideEntries = 16384, kChannelLines = kJoinThreads / 64;

// The sum over a channel's threads, in each of them; sh: kJoinThreads floats.
__device__ inline float channel_sum(float v, float* sh) {
  const int x = threadIdx.x & 63;
  __syncthreads();
  sh[threadIdx.x] = v;
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int i = 0; i < kChannelLines; ++i) v += sh[i * 64 + x];
  return v;
}

// f(image, channel, whether there is one, this thread's first chunk) for all of them; f
// is called by whole workgroups.
template <class F> __device__ inline void each_channel(const Norm& a, F f) {
  const int blocks = (a.c + 63) / 64;
  for (int64_t id = blockIdx.x; id < a.b * blocks; id += gridDim.x) {
    const int64_t n = id / blocks;
    const int ch = (int)(id - n * blocks) * 64 + (threadIdx.x & 63);
    f(n, ch, ch < a.c, (int)threadIdx.x >> 6);
  }
}

constexpr int kUnitVecs = 4;

// ---------------------------------------------------------------------------
// choice and launch
// ---------------------------------------------------------------------------
inline int64_t up(int64_t v) { return (v + 255) / 256 * 256; }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline Divider divider(int64_t d) { return Divider{(uint32_t)d, (uint32_t)((0x100000000ull + d - 1) / d)}; }

// Workgroups for that many parts; the kernels go on from there.
inline dim3 grid_of(int64_t parts) { return dim3((unsigned)std::min<int64_t>(parts, 1 << 20)); }

struct NormPlan {
  bool resident, feature;
  bool wide;                         // chunks are joined by channel first
  Mode mode;
  int threads, held;                 // resident and feature: threads of a workgroup, vectors that a thread holds
  int vecs, units, unit_groups, rows, slots, lanes, shares, blocks;
  int chunk, chunks;
  int64_t sums, joined, stats, bytes;   // byte offsets: part first, then the sums, those by image, mean and rstd
};

constexpr int kMostHeld = 8;                       // vectors of a thread

inline NormPlan plan_of(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, bool grad) {
  NormPlan p{};
  const int64_t V = 16 / type_size(dtype), per = c / groups, all = div_up(c, V), cu = compute_units();
  const int64_t unit = std::min<int64_t>(std::lcm(per, V) / V, all);
  p.mode = per % V == 0 ? kOneGroup : c % V == 0 ? kWhole : c > V ? kTail : kTiny;
  auto fits = [&](int64_t vecs, int threads) { return vecs <= threads && div_up(s, std::max<int64_t>(1, threads / vecs)) <= kMostHeld; };
  if (s == 1 && per >= V && per <= 512 * V * 4) {
    p.feature = true;
    const int64_t vecs = div_up(per, V), lanes = vecs > 64 * 4 ? 512 : 64;
    p.threads = lanes == 64 ? 256 : 512;
    p.lanes = 1;
    while (p.lanes < lanes && p.lanes < vecs) p.lanes *= 2;
    p.held = 1;
    while (p.held * p.lanes < vecs) p.held *= 2;
    p.units = (int)div_up(groups, lanes / p.lanes);
    const int64_t most = std::max<int64_t>(1, 2 * cu / p.units), turns = div_up(b, lanes == 64 ? 4 : 1);
    p.blocks = (int)div_up(turns, div_up(turns, most));
    p.bytes = grad ? up(2 * (int64_t)p.blocks * c * 4) : 0;
    return p;
  }
  // resident: 0.2 (0.4) ns a value of one workgroup on a compute unit, and 5 us; split: the
  // same spread over all units, and what its three launches take
  const double each = (double)unit * V * s * (grad ? 0.4e-3 : 0.2e-3), rounds = (double)div_up(div_up(all, unit) * b, cu);
  const double split = (grad ? 28.0 : 18.0) + each * div_up(all, unit) * b / cu;
  if (fits(unit, p.mode == kTiny ? 256 : 512) && 5.0 + each * rounds <= split) {
    p.resident = true;
    int64_t vecs = unit;
    // a line of the caches at each position, where workgroups enough are left
    while (vecs < kUnitVecs && vecs < all) {
      const int64_t wide = std::min(vecs + unit, all);
      if (!fits(wide, 512) || div_up(all, wide) * b < 4 * cu) break;
      vecs = wide;
    }
    p.threads = fits(vecs, 256) ? 256 : 512;
    const int64_t lines = p.threads / vecs;
    p.vecs = (int)vecs;
    p.units = (int)div_up(all, vecs);
    p.unit_groups = (int)std::max<int64_t>(1, std::min<int64_t>(groups, vecs * V / per));
    p.rows = (int)std::min(lines, std::max<int64_t>(s, 1));
    p.slots = (int)std::min<int64_t>(lines / p.rows, std::max<int64_t>(b, 1));
    const int64_t need = div_up(std::max<int64_t>(s, 1), p.rows);
    p.held = need == 1 ? 1 : need <= 4 ? 4 : 8;
    if (p.mode == kTiny) p.held = 8;
    const int64_t items = (int64_t)p.slots * p.unit_groups;
    p.lanes = 64;
    while (p.lanes > 1 && p.lanes * items > p.threads) p.lanes /= 2;
    p.shares = 1;
    while (p.lanes == 64 && 2 * p.shares * 64 * items <= p.threads) p.shares *= 2;
    // workgroups along the images, each with as many rounds of them
    const int64_t turns = div_up(std::max<int64_t>(b, 1), p.slots);
    const int64_t most = std::max<int64_t>(1, (grad ? 2 : 16) * cu * 256 / p.threads / p.units);
    p.blocks = (int)div_up(turns, div_up(turns, most));
    p.bytes = grad ? up(2 * (int64_t)p.blocks * c * 4) : 0;
    return p;
  }
  p.vecs = (int)std::min<int64_t>(all, kSplitThreads);
  p.units = (int)div_up(all, p.vecs);
  const int64_t rows = kSplitThreads / p.vecs;
  // parts of 64 KB, four to sixteen for every compute unit: below, what each part sets up
  // shows (18 KB: 25 % longer); above, too little is under way
  const int64_t parts = std::clamp<int64_t>(c * s * b * type_size(dtype) >> 16, 4 * cu, 16 * cu);
  const int64_t want = std::max<int64_t>(1, div_up(parts, b * p.units));
  // 256 values at most to a thread's sum
  p.chunk = (int)(std::min<int64_t>(256, div_up(std::max(div_up(s, want), std::min(s, kAhead * rows)), rows)) * rows);
  p.chunks = (int)div_up(s, p.chunk);
  p.sums = grad ? up(b * groups * 8) : up(b * p.chunks * c * 8);
  p.wide = p.chunks > 1 && per * p.chunks > kWideEntries;
  p.joined = p.sums + (grad ? up(2 * b * p.chunks * c * 4) : 0);
  p.stats = p.joined + (p.wide ? up(b * c * 8) : 0);
  p.bytes = p.stats + (grad ? 0 : 2 * up(b * groups * 4));
  return p;
}

inline int check_norm(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups) {
  if (!is_type(dtype)) return -1;
  if (c < 0 || c >= kSizeLimit) return -2;
  if (s < 0 || s >= kSizeLimit) return -3;
  if (b < 0 || b >= 1ll << 31 || (c * s > 0 && b >= kElemLimit / (c * s))) return -4;
  if (groups < 1 || groups > std::max<int64_t>(c, 1) || c % groups) return -5;
  return 0;
}

// ld (its argument's number `at`) and ldb behind it.
inline int check_map(int64_t c, int64_t s, int64_t b, int64_t ld, int64_t ldb, int at) {
  if (ld < std::max<int64_t>(c, 1) || ld >= kElemLimit) return -at;
  if (s > 1 && ld > kElemLimit / s) return -at;
  if (b > 1 && (ldb < (s - 1) * ld + c || ldb >= kElemLimit)) return -(at + 1);
  return 0;
}

template <class T> void fill(Norm& a, const NormPlan& p, char* ws) {
  a.vecs = p.vecs, a.units = p.units, a.unit_groups = p.unit_groups, a.rows = p.rows, a.slots = p.slots, a.lanes = p.lanes;
  a.shares = p.shares, a.blocks = p.blocks, a.chunk = p.chunk, a.chunks = p.chunks;
  a.part = reinterpret_cast<float2*>(ws);
  if (!p.resident) return;
  a.vec = divider(p.vecs);
  a.row = divider(p.rows);
  a.run = divider(p.mode == kOneGroup ? a.per / kVec<T> : a.per);
  a.group = divider(p.unit_groups);
}

// Results from here on are stored past the caches.
template <class T> bool streamed(const Norm& a) { return (double)a.c * a.s * a.b * sizeof(T) >= 64e6; }

template <class K> hipError_t start_resident(K kernel, const NormPlan& p, const Norm& a, int64_t floats, hipStream_t s) {
  const hipError_t e = ltlt::ensure_dynamic_lds((const void*)kernel, 65536);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)((int64_t)p.units * p.blocks)), p.threads, (unsigned)floats * 4, s>>>(a);
  return hipGetLastError();
}

// f(mode as a constant)
template <class F> hipError_t by_mode(Mode mode, F f) {
  switch (mode) {
    case kOneGroup: return f(std::integral_constant<int, kOneGroup>{});
    case kWhole: return f(std::integral_constant<int, kWhole>{});
    case kTail: return f(std::integral_constant<int, kTail>{});
    default: return f(std::integral_constant<int, kTiny>{});
  }
}

}  // namespace
}  // namespace linear
