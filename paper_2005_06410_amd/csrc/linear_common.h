// Shared by the layer operators (linear.hip, linear_grad.hip): element types,
// 16-byte vectors at any address, activations and the product's description.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "linear.h"

namespace linear {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16;
typedef _Float16 f16;

// Values of one 16-byte chunk.
template <class T> constexpr int kVec = 16 / (int)sizeof(T);

// kVec consecutive values as fp32, from and to any address the type allows: the
// 16-byte accesses carry no alignment promise, which global memory serves in
// hardware.
template <class T> struct __attribute__((packed, aligned(sizeof(T)))) Packed {
  T v[kVec<T>];
};

template <class T> __device__ inline void load_vec(const T* p, float* out) {
  const Packed<T> q = *reinterpret_cast<const Packed<T>*>(p);
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) out[i] = (float)q.v[i];
}

template <class T> __device__ inline void store_vec(T* p, const float* v) {
  Packed<T> q;
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) q.v[i] = (T)v[i];
  *reinterpret_cast<Packed<T>*>(p) = q;
}

constexpr float kTanhScale = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

// exp(x) and 1 / x: to fp32 accuracy for fp32 results; for the 16-bit types by
// the hardware's approximations, whose error of about 2^-22 is far below the
// result's rounding.
template <class T> __device__ inline float exp_of(float x) {
  return sizeof(T) == 4 ? expf(x) : __builtin_amdgcn_exp2f(1.4426950408889634f * x);
}
template <class T> __device__ inline float inverse(float x) { return sizeof(T) == 4 ? 1.0f / x : __builtin_amdgcn_rcpf(x); }

// Phi(z), and in `e` exp(-z^2 / 2).  Both forms keep their relative accuracy for
// negative z, where Phi falls to nothing.  fp32: erfc.  16-bit types: Phi(-|z|) =
// exp(-x^2) E(x) / 2 with x = |z| / sqrt(2) and E(x) = exp(x^2) erfc(x) as t times a
// polynomial in t = 1 / (1 + p x), a third of erfc's instructions (the epilogue of
// a large product is bound by them).  p and the five coefficients were fitted to the
// smallest largest relative error over 0 <= x <= 9.5 (z to -13.4, where exp(-x^2)
// leaves the range): 2.72e-5, a ninth of fp16's rounding.  Five coefficients with the
// smallest absolute error of erf instead are 0.16 % off at z = -5 and 1 % at -8.
template <class T> __device__ inline float normal_cdf(float z, float& e) {
  e = exp_of<T>(-0.5f * z * z);
  if constexpr (sizeof(T) == 4) return 0.5f * erfcf(-0.7071067811865476f * z);
  const float x = 0.7071067811865476f * fabsf(z);
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.531413257f * x);
  const float q = 0.5f * e * t *
                  (0.298716263f + t * (0.316155627f + t * (0.167573495f + t * (0.39991392f + t * -0.182386526f))));
  return z < 0.0f ? q : 1.0f - q;
}

// The logistic function of 2u, u = sqrt(2/pi) (z + 0.044715 z^3): (1 + tanh u) / 2
// without its cancellation for negative u.
template <class T> __device__ inline float tanh_gate(float z) {
  const float u = kTanhScale * (z + kTanhCubic * z * z * z);
  return inverse<T>(1.0f + exp_of<T>(-2.0f * u));
}

// f(std::integral_constant) of the activation: one branch for a whole vector.
template <class F> __device__ inline void with_act(int act, F f) {
  switch (act) {
    case LINEAR_ACT_RELU: return f(std::integral_constant<int, LINEAR_ACT_RELU>{});
    case LINEAR_ACT_GELU: return f(std::integral_constant<int, LINEAR_ACT_GELU>{});
    case LINEAR_ACT_GELU_TANH: return f(std::integral_constant<int, LINEAR_ACT_GELU_TANH>{});
    case LINEAR_ACT_SILU: return f(std::integral_constant<int, LINEAR_ACT_SILU>{});
  }
}

// act(z) in fp32.
template <class T, int ACT> __device__ inline float act_value(float z) {
  float e;
  if constexpr (ACT == LINEAR_ACT_RELU) return z <= 0.0f ? 0.0f : z;
  if constexpr (ACT == LINEAR_ACT_GELU) return z * normal_cdf<T>(z, e);
  if constexpr (ACT == LINEAR_ACT_GELU_TANH) return z * tanh_gate<T>(z);
  if constexpr (ACT == LINEAR_ACT_SILU) return z * inverse<T>(1.0f + exp_of<T>(-z));
  return z;
}

// d act'(z) in fp32.
template <class T, int ACT> __device__ inline float act_grad(float d, float z) {
  if constexpr (ACT == LINEAR_ACT_RELU) return z <= 0.0f ? 0.0f : d;   // zero also where d is not finite
  if constexpr (ACT == LINEAR_ACT_GELU) {
    float e;
    const float c = normal_cdf<T>(z, e);
    return d * (c + z * (0.3989422804014327f * e));
  }
  if constexpr (ACT == LINEAR_ACT_GELU_TANH) {
    // beyond 16 the slope is 0 or 1 to the last bit, and z^3 could overflow
    const float s = tanh_gate<T>(z);
    const float slope = s + 2.0f * z * s * (1.0f - s) * kTanhScale * (1.0f + 3.0f * kTanhCubic * z * z);
    return d * (z > 16.0f ? 1.0f : z < -16.0f ? 0.0f : slope);
  }
  if constexpr (ACT == LINEAR_ACT_SILU) {
    const float s = inverse<T>(1.0f + exp_of<T>(-z));
    return d * (s * (1.0f + z * (1.0f - s)));
  }
  return d;
}

template <class T, int N> __device__ inline void act_values(float* v, int act) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<T, decltype(a)::value>(v[i]);
  });
}

template <class T, int N> __device__ inline void act_grads(float* d, const float* z, int act) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = act_grad<T, decltype(a)::value>(d[i], z[i]);
  });
}

// store_vec(), past the caches with STREAM: for results so large that keeping them
// only drives out what is still read.
template <class T, bool STREAM> __device__ inline void result_vec(T* p, const float* v) {
  if constexpr (STREAM) {
    typedef uint32_t w4 __attribute__((ext_vector_type(4), aligned(2)));
    Packed<T> q;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) q.v[i] = (T)v[i];
    __builtin_nontemporal_store(__builtin_bit_cast(w4, q), reinterpret_cast<w4*>(p));
  } else {
    store_vec(p, v);
  }
}

// An operand's lines (its contiguous extents): 16-byte aligned and whole 16 bytes
// long, or not, or so far apart that a tile's offsets do not fit the direct loads.
enum class Lines { kDirect, kRagged, kFar };
constexpr Lines kAnyLines[] = {Lines::kDirect, Lines::kRagged, Lines::kFar};

// Most lines of an operand that one stage of a tile spans, and the bytes that its
// loads reach (32-bit offsets, below those that say "nowhere").
constexpr int64_t kStageLines = 256, kReach = 0xfffff000ll;

inline Lines lines_of(int dtype, const void* p, int64_t ld, int64_t len) {
  const int64_t size = dtype == LINEAR_F32 ? 4 : 2;
  if (ld * size * kStageLines > kReach) return Lines::kFar;
  return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0 && len * size % 16 == 0 ? Lines::kDirect : Lines::kRagged;
}

// The same before addresses and leading dimensions are known, of lines that may be
// next to each other.
inline Lines lines_if(int dtype, bool aligned, int64_t len) {
  const Lines l = lines_of(dtype, nullptr, len, len);
  return l == Lines::kDirect && !aligned ? Lines::kRagged : l;
}

// What follows a product: C = act(product scale + bias) + residual, Z = product
// scale + bias.
struct Epilogue {
  const void* bias;       // M values or nullptr
  const void* residual;   // M x N or nullptr
  int64_t ldr;
  void* Z;                // M x N or nullptr
  int64_t ldz;
  void* C;
  int64_t ldc;
  int act;
  const float* scale;     // 16-bit types only: one value or nullptr
};

// C (M x N, M fastest) = A (M x K) B (K x N).
struct Product {
  const void* A;
  const void* B;
  int64_t lda, ldb;
  int M, N, K;            // M, N >= 1
  int arows, aK;          // extents of the operands as they are loaded: M and K
  int brows, bK;          // (N and K), or more where zeros follow
  Lines a, b;             // the operands' lines, as the workspace was sized for
  int splits;             // workgroups that share a tile's contraction
  int mtiles, ntiles;
  float* part;            // [splits][N][M] partial products, or nullptr where the epilogue follows (splits = 1)
  bool add;               // the partial products are added to what `part` holds
  Epilogue e;
};

// The first `cnt` of kVec values from p on, all of them with WHOLE in one load; else
// the others are copies of the last one, so that the single loads are not under
// branches and none waits for another (1535 x 1001 by 2047 fp16 with bias and
// residual: 36 us value by value, 34 under branches, 29 so).
template <class T, bool WHOLE> __device__ inline void load_part(const T* p, int cnt, float* out) {
  if constexpr (WHOLE) {
    load_vec(p, out);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) out[i] = (float)p[min(i, cnt - 1)];
  }
}

template <class T, bool WHOLE, bool STREAM> __device__ inline void store_part(T* p, int cnt, const float* v) {
  if constexpr (WHOLE) {
    result_vec<T, STREAM>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
      if (i < cnt) p[i] = (T)v[i];
  }
}

// Values m .. of column n of the result, kVec of them (WHOLE) or the cnt >= 1 that
// it still has; sums(v) gives the product's fp32 sums.
template <class T, bool WHOLE, bool STREAM, class F>
__device__ inline void finish(const Epilogue& e, int m, int n, int cnt, F sums) {
  constexpr int V = kVec<T>;
  float b[V], r[V], v[V];
  if (e.bias) load_part<T, WHOLE>(static_cast<const T*>(e.bias) + m, cnt, b);
  if (e.residual) load_part<T, WHOLE>(static_cast<const T*>(e.residual) + (int64_t)n * e.ldr + m, cnt, r);
  sums(v);
  if constexpr (sizeof(T) == 2) {
    if (e.scale) {
      const float c = *e.scale;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= c;
    }
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += b[i];
  }
  if (e.Z) store_part<T, WHOLE, STREAM>(static_cast<T*>(e.Z) + (int64_t)n * e.ldz + m, cnt, v);
  act_values<T, V>(v, e.act);
  if (e.residual) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += r[i];
  }
  store_part<T, WHOLE, STREAM>(static_cast<T*>(e.C) + (int64_t)n * e.ldc + m, cnt, v);
}

// The same for one value.
template <class T> __device__ inline void finish_one(const Epilogue& e, int m, int n, float v) {
  if (sizeof(T) == 2 && e.scale) v *= *e.scale;
  if (e.bias) v += (float)static_cast<const T*>(e.bias)[m];
  if (e.Z) static_cast<T*>(e.Z)[(int64_t)n * e.ldz + m] = (T)v;
  act_values<T, 1>(&v, e.act);
  if (e.residual) v += (float)static_cast<const T*>(e.residual)[(int64_t)n * e.ldr + m];
  static_cast<T*>(e.C)[(int64_t)n * e.ldc + m] = (T)v;
}

// linear.hip.  Where A's (B's) contiguous index is the contraction, a_kc (b_kc)
// is set; its rows are then ld apart, else its contraction indices are.
int compute_units();

// Bytes of workspace for a product.
int64_t product_workspace(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K);

// p.arows, aK, brows, bK: the extents as loaded, or 0 where they are M, N and K.
hipError_t launch_product(int dtype, bool a_kc, bool b_kc, Product p, void* workspace, hipStream_t s);

// A contraction whose operands come piece by piece: the partial products of one
// piece, written to p.part or (p.add) added to it, p.splits of them (at least
// product_splits() of the largest piece); then what launch_product() does with their
// sum.  The operands' lines are kDirect, or kFar even in a padded copy.
int product_splits(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K);
hipError_t launch_product_part(int dtype, bool a_kc, bool b_kc, Product p, hipStream_t s);
hipError_t launch_product_join(int dtype, const Product& p, hipStream_t s);

// Argument checks of the C ABI.
constexpr int64_t kSizeLimit = 1ll << 24;
constexpr int64_t kElemLimit = 1ll << 40;

inline bool is_type(int dtype) { return dtype == LINEAR_F32 || dtype == LINEAR_BF16 || dtype == LINEAR_F16; }
inline int64_t type_size(int dtype) { return dtype == LINEAR_F32 ? 4 : 2; }

// 0, or minus the first invalid one of dtype, kn, ci, t (arguments 1 .. 4).
inline int check_sizes(int dtype, int64_t kn, int64_t ci, int64_t t) {
  if (!is_type(dtype)) return -1;
  if (kn < 0 || kn >= kSizeLimit) return -2;
  if (ci < 0 || ci >= kSizeLimit || kn * ci >= kElemLimit) return -3;
  if (t < 0 || t >= kSizeLimit || kn * t >= kElemLimit || ci * t >= kElemLimit) return -4;
  return 0;
}

inline bool bad_ld(int64_t ld, int64_t extent) { return ld < (extent > 1 ? extent : 1) || ld >= kSizeLimit; }

}  // namespace linear
