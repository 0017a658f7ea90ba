// The layer: its product (linear_product.h) with bias, activation and residual, and
// the products of its gradients.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "linear_common.h"
#include "linear_product.h"

namespace linear {

// Compute units of the current device, asked for once per device.
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return 256;
  }
  if (dev >= 0 && dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
    (void)hipGetLastError();
    return 256;
  }
  if (dev >= 0 && dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

namespace {

template <class R> hipError_t launch_ring(Product p, hipStream_t s) {
  p.mtiles = (p.M + R::MT - 1) / R::MT;
  p.ntiles = (p.N + R::NTILE - 1) / R::NTILE;
  const hipError_t e = ltlt::ensure_dynamic_lds((const void*)ring_kernel<R>, R::LDS);
  if (e != hipSuccess) return e;
  ring_kernel<R><<<dim3((unsigned)((int64_t)p.mtiles * p.ntiles * p.splits)), R::NT, R::LDS, s>>>(p);
  return hipGetLastError();
}

template <class T, bool AKC, bool BKC> hipError_t launch_wide(Product p, hipStream_t s) {
  p.mtiles = (p.M + 255) / 256;
  p.ntiles = (p.N + 255) / 256;
  // 4096 x 16384 by 8192 tokens and back, bf16: 1728 us with ordinary stores, 1710 past
  // the caches; 2048 x 8192 by 2048 (33 MB in between): 137 and 141
  const bool stream = (int64_t)p.M * p.N * (int)sizeof(T) >= (64ll << 20);
  auto k = stream ? wide_kernel<T, AKC, BKC, true> : wide_kernel<T, AKC, BKC, false>;
  const hipError_t e = ltlt::ensure_dynamic_lds((const void*)k, 2 * kWideBuffer);
  if (e != hipSuccess) return e;
  k<<<dim3((unsigned)((int64_t)p.mtiles * p.ntiles * p.splits)), 512, 2 * kWideBuffer, s>>>(p);
  return hipGetLastError();
}

template <class T, bool AKC, bool BKC, int W> hipError_t launch_shape(Shape shape, const Product& p, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (shape == kWide) return launch_wide<T, AKC, BKC>(p, s);
  }
  if (shape == kSquare4) return launch_ring<Ring<T, AKC, BKC, 4, 2, 2, 4, 1, 1, 4, W>>(p, s);
  if (shape == kTall) return launch_ring<Ring<T, AKC, BKC, 4, 2, 2, 2, 1, 1, 3, W>>(p, s);
  if (shape == kSmall) return launch_ring<Ring<T, AKC, BKC, 2, 2, 2, 2, 1, 1, 4, W>>(p, s);
  if (shape == kQuad64) return launch_ring<Ring<T, AKC, BKC, 2, 2, 2, 2, 2, 2, 4, W>>(p, s);
  if (shape == kBlock32) return launch_ring<Ring<T, AKC, BKC, 2, 2, 1, 1, 4, 4, 4, W>>(p, s);
  if constexpr (BKC) {
    if (shape == kNarrow32) return launch_ring<Ring<T, AKC, BKC, 4, 2, 1, 1, 4, 4, 3, W>>(p, s);
    if (shape == kNarrow16) return launch_ring<Ring<T, AKC, BKC, 4, 1, 1, 1, 4, 4, 3, W>>(p, s);
    if constexpr (sizeof(T) == 4) {
      if (shape == kSlim80) return launch_ring<Ring<T, AKC, BKC, 1, 5, 1, 1, 8, 4, 3, W>>(p, s);
      if (shape == kRow80) return launch_ring<Ring<T, AKC, BKC, 2, 5, 1, 1, 4, 2, 2, W>>(p, s);
    }
  }
  if constexpr (AKC && BKC) {
    if (shape == kThin16) return launch_ring<Ring<T, AKC, BKC, 1, 1, 1, 1, 8, 8, 4, W>>(p, s);
  }
  return launch_ring<Ring<T, AKC, BKC, 4, 4, 2, 2, 1, 1, 2, W>>(p, s);
}

template <class T, bool AKC, bool BKC> hipError_t launch_registers(const Product& p, hipStream_t s) {
  if (p.N > 64) return launch_ring<Ring<T, AKC, BKC, 4, 4, 2, 2, 1, 1, 2, 0>>(p, s);
  if constexpr (BKC) {
    if (p.N <= 16) return launch_ring<Ring<T, AKC, BKC, 4, 1, 1, 1, 4, 4, 2, 0>>(p, s);
  }
  return launch_ring<Ring<T, AKC, BKC, 4, 4, 1, 1, 4, 4, 2, 0>>(p, s);
}

template <class T, int W> hipError_t launch_ordered(bool a_kc, bool b_kc, Shape shape, const Product& p, hipStream_t s) {
  return a_kc ? launch_shape<T, true, true, W>(shape, p, s)
         : b_kc ? launch_shape<T, false, true, W>(shape, p, s)
                : launch_shape<T, false, false, W>(shape, p, s);
}

template <class T> hipError_t launch_route(const Route& r, bool a_kc, bool b_kc, Shape shape, const Product& p, hipStream_t s) {
  if (r.width == 0)
    return a_kc   ? launch_registers<T, true, true>(p, s)
           : b_kc ? launch_registers<T, false, true>(p, s)
                  : launch_registers<T, false, false>(p, s);
  if constexpr (sizeof(T) == 4) {
    if (r.width == 4) return launch_ordered<T, 4>(a_kc, b_kc, shape, p, s);
  }
  return launch_ordered<T, 16>(a_kc, b_kc, shape, p, s);
}

template <class T> hipError_t launch_join(const Product& p, hipStream_t s) {
  const int64_t vecs = (p.M / kVec<T> + p.M % kVec<T>) * (int64_t)p.N;
  join_kernel<T><<<dim3((unsigned)std::min<int64_t>((vecs + 255) / 256, 4096)), 256, 0, s>>>(p);
  return hipGetLastError();
}

template <class T> hipError_t launch_typed(int dtype, bool a_kc, bool b_kc, Product p, char* ws, hipStream_t s) {
  const Route r = route_of(dtype, a_kc, b_kc, p.a, p.b, p.M, p.N, p.K);
  hipError_t e = hipSuccess;
  Shape shape = kSquare2;
  if (r.width == 0) {
    true_extents(p);
    p.splits = register_splits(dtype, b_kc, p.M, p.N, p.K);
  } else {
    const Plan plan = plan_of(dtype, r.width, a_kc, b_kc, p.M, p.N, p.K);
    p.splits = plan.splits;
    shape = plan.shape;
    e = copy_operands<T>(dtype, r, a_kc, b_kc, p, ws, s);
  }
  p.part = p.splits > 1 ? reinterpret_cast<float*>(ws) : nullptr;
  p.add = false;
  if (e == hipSuccess) e = launch_route<T>(r, a_kc, b_kc, shape, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  return launch_join<T>(p, s);
}

// The partial products alone, with the splits, `part` and `add` that the product names.
template <class T> hipError_t launch_part_typed(int dtype, bool a_kc, bool b_kc, Product p, hipStream_t s) {
  const Route r = route_of(dtype, a_kc, b_kc, p.a, p.b, p.M, p.N, p.K);
  if (r.copy_a || r.copy_b || r.width == 4) return hipErrorInvalidValue;   // does not occur
  Shape shape = kSquare2;
  if (r.width == 0)
    true_extents(p);
  else
    shape = plan_of(dtype, r.width, a_kc, b_kc, p.M, p.N, p.K).shape;
  return launch_route<T>(r, a_kc, b_kc, shape, p, s);
}

}  // namespace

void product_choice(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K, int* out) {
  if (M <= 0 || N <= 0) {
    for (int i = 0; i < 6; ++i) out[i] = 0;
    return;
  }
  const Route r = route_of(dtype, a_kc, b_kc, a, b, M, N, K);
  if (r.width == 0) {
    const RegisterTile t = register_tile(b_kc, N);
    out[0] = 4, out[1] = t.m, out[2] = t.n, out[3] = register_splits(dtype, b_kc, M, N, K), out[4] = 0, out[5] = 0;
  } else {
    const Plan p = plan_of(dtype, r.width, a_kc, b_kc, M, N, K);
    const Tile& t = kTiles[p.shape];
    out[0] = p.shape == kWide ? 1 : r.width == 16 ? 2 : 3;
    out[1] = t.m, out[2] = t.n, out[3] = p.splits, out[4] = r.copy_a + r.copy_b, out[5] = p.shape;
  }
}

int64_t product_workspace(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K) {
  const Route r = route_of(dtype, a_kc, b_kc, a, b, M, N, K);
  int64_t bytes = 0;
  if (r.copy_a) bytes += up256(copy_values(dtype, a_kc, M, K) * type_size(dtype));
  if (r.copy_b) bytes += up256(copy_values(dtype, b_kc, N, K) * type_size(dtype));
  const int64_t splits = product_splits(dtype, a_kc, b_kc, a, b, M, N, K);
  return bytes + (splits > 1 ? splits * M * N * 4 : 0);
}

hipError_t launch_product(int dtype, bool a_kc, bool b_kc, Product p, void* workspace, hipStream_t s) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  if (a_kc && !b_kc) return hipErrorInvalidValue;   // does not occur
  set_extents(p);
  char* ws = static_cast<char*>(workspace);
  switch (dtype) {
    case LINEAR_F32: return launch_typed<float>(dtype, a_kc, b_kc, p, ws, s);
    case LINEAR_BF16: return launch_typed<bf16>(dtype, a_kc, b_kc, p, ws, s);
    default: return launch_typed<f16>(dtype, a_kc, b_kc, p, ws, s);
  }
}

int product_splits(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K) {
  const Route r = route_of(dtype, a_kc, b_kc, a, b, M, N, K);
  return r.width == 0 ? register_splits(dtype, b_kc, M, N, K) : plan_of(dtype, r.width, a_kc, b_kc, M, N, K).splits;
}

hipError_t launch_product_part(int dtype, bool a_kc, bool b_kc, Product p, hipStream_t s) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  if (a_kc && !b_kc) return hipErrorInvalidValue;   // does not occur
  set_extents(p);
  switch (dtype) {
    case LINEAR_F32: return launch_part_typed<float>(dtype, a_kc, b_kc, p, s);
    case LINEAR_BF16: return launch_part_typed<bf16>(dtype, a_kc, b_kc, p, s);
    default: return launch_part_typed<f16>(dtype, a_kc, b_kc, p, s);
  }
}

hipError_t launch_product_join(int dtype, const Product& p, hipStream_t s) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  switch (dtype) {
    case LINEAR_F32: return launch_join<float>(p, s);
    case LINEAR_BF16: return launch_join<bf16>(p, s);
    default: return launch_join<f16>(p, s);
  }
}

}  // namespace linear

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------
using linear::bad_ld;
using linear::check_sizes;

extern "C" int64_t convgemm_linear_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int aligned) {
  using namespace linear;
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  if (aligned)
    return product_workspace(dtype, f_order == 1, true, lines_if(dtype, true, f_order ? ci : kn), lines_if(dtype, true, ci), kn, t, ci);
  int64_t most = 0;
  for (Lines f : kAnyLines)
    for (Lines x : kAnyLines) most = std::max(most, product_workspace(dtype, f_order == 1, true, f, x, kn, t, ci));
  return most;
}

extern "C" int convgemm_linear_choice(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int aligned, int* out) {
  using namespace linear;
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  if (!out) return -7;
  product_choice(dtype, f_order == 1, true, lines_if(dtype, aligned, f_order ? ci : kn), lines_if(dtype, aligned, ci), kn, t, ci, out);
  return LINEAR_OK;
}

extern "C" int convgemm_linear(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                               const void* X, int64_t ldx, const void* bias, int act, const void* residual, int64_t ldr,
                               void* Z, int64_t ldz, void* O, int64_t ldo, void* workspace, int64_t workspace_bytes,
                               hipStream_t stream) {
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  const bool work = kn > 0 && t > 0;
  if (!F && work && ci > 0) return -5;
  if (f_order != 0 && f_order != 1) return -6;
  if (bad_ld(ldf, f_order ? ci : kn)) return -7;
  if (!X && work && ci > 0) return -8;
  if (bad_ld(ldx, ci)) return -9;
  if (act < LINEAR_ACT_NONE || act > LINEAR_ACT_SILU) return -11;
  if (residual && bad_ld(ldr, kn)) return -13;
  if (Z && bad_ld(ldz, kn)) return -15;
  if (!O && work) return -16;
  if (bad_ld(ldo, kn)) return -17;
  linear::Product p{};
  p.a = linear::lines_of(dtype, F, ldf, f_order ? ci : kn);
  p.b = linear::lines_of(dtype, X, ldx, ci);
  const int64_t need = linear::product_workspace(dtype, f_order == 1, true, p.a, p.b, kn, t, ci);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 15))) return -18;
  if (need > 0 && workspace_bytes < need) return -19;
  if (!work) return LINEAR_OK;
  p.A = F;
  p.lda = ldf;
  p.B = X;
  p.ldb = ldx;
  p.M = (int)kn;
  p.N = (int)t;
  p.K = (int)ci;
  p.e = linear::Epilogue{bias, residual, ldr, Z, ldz, O, ldo, act, nullptr};
  const hipError_t e = linear::launch_product(dtype, f_order == 1, true, p, workspace, stream);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}
