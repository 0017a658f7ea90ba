// The layer's matrix product on gfx950: C = act(A B + bias) + residual, both
// operands in either order, fp32, bf16 and fp16 on the matrix cores with fp32
// sums.
//
// Tiles.  A workgroup owns an MT x NT tile of C and walks the contraction in
// chunks of 128 bytes per row (32 fp32 or 64 16-bit values), two LDS buffers
// deep.  What one lane feeds the matrix cores is always a 16-byte fragment:
//   * 16-bit types: 8 contraction values of one row, one v_mfma_*_16x16x32;
//   * fp32: 4 contraction values of one row for four v_mfma_f32_16x16x4_f32
//     (lane group q = lane / 16 takes contraction values 4q .. 4q+3 of a group
//     of 16, one per instruction).
// An operand whose contraction index is contiguous ("KC") lies in LDS as rows
// of 128 bytes whose eight 16-byte chunks are permuted by the row (chunk ^ row
// & 7), so that 16 rows are read without bank conflicts.  An operand whose rows
// are contiguous ("MC") lies there as it is in memory, one line of MT values
// per contraction index: fp32 reads four rows of one contraction index at a
// time (so lane l16 holds rows 4 l16 + i, i the block), the 16-bit types read
// through the transposing ds_read_b64_tr_b16, their 32-byte blocks permuted by
// the contraction index for the same reason.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "linear_common.h"

namespace linear {

int compute_units() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      n <= 0) {
    (void)hipGetLastError();
    return 256;
  }
  return n;
}

namespace {

// ---------------------------------------------------------------------------
// one operand's tile
// ---------------------------------------------------------------------------
// LDS placement of a 16-bit MC line: permutation of its 32-byte blocks.
template <int ROWS> __device__ inline int mc_swizzle(int k) {
  return ((k & 3) | ((k >> 3) & 1) << 2) & (ROWS / 16 - 1);
}

// Staging of a tile of ROWS x 128 bytes by NT threads; thread `tid` moves the
// 16-byte chunks tid, tid + NT, ... in LDS order.
template <class T, bool KC, int ROWS, int NT, bool DMA> struct Stage {
  static constexpr int V = kVec<T>;
  static constexpr int BK = 128 / (int)sizeof(T);
  static constexpr int CHUNKS = ROWS * 8 / NT;
  static_assert(CHUNKS * NT == ROWS * 8, "whole chunks");
  const T* base;          // the tile's first row, contraction index 0
  int64_t ld;
  int rows, K;            // rows that exist from the tile's first one; contraction length
  int tid;
  uint32_t voff[DMA ? CHUNKS : 1];
  u4 reg[DMA ? 1 : CHUNKS];

  // chunk c of the tile: its row (KC) or contraction index (MC) and the first
  // value along the contiguous index
  __device__ static void place(int c, int& line, int& first) {
    if (KC) {
      line = c >> 3;
      first = ((c & 7) ^ (line & 7)) * V;
    } else {
      constexpr int CPL = ROWS / V;
      line = c / CPL;
      int q = c % CPL;
      if (sizeof(T) == 2) q ^= mc_swizzle<ROWS>(line) << 1;
      first = q * V;
    }
  }

  __device__ void init(const void* p, int64_t ld_, int row0, int nrows, int K_, int tid_) {
    ld = ld_;
    base = static_cast<const T*>(p) + (KC ? (int64_t)row0 * ld : (int64_t)row0);
    rows = nrows - row0;
    K = K_;
    tid = tid_;
    if (DMA) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        int line, first;
        place(i * NT + tid, line, first);
        voff[i] = (uint32_t)(line * (int)(ld * sizeof(T))) + (uint32_t)(first * sizeof(T));
      }
    }
  }

  // Loads chunk-tile kt: straight into LDS (DMA), or into registers.
  __device__ void load(int kt, char* lds) {
    const int k0 = kt * BK;
    const T* b = base + (KC ? (int64_t)k0 : (int64_t)k0 * ld);
    if (DMA) {
      // range: up to the operand's last value; beyond it (rows past the end of
      // a KC operand, contraction indices past the end of an MC one) the load
      // gives zero.  A KC row's chunks past the contraction's end lie inside
      // the next row and are sent out of range.
      const int64_t span = KC ? ((int64_t)(min(rows, ROWS) - 1) * ld + (K - k0)) : ((int64_t)(min(K - k0, BK) - 1) * ld + rows);
      const uint64_t bytes = (uint64_t)span * sizeof(T);
      const uint32_t range = bytes > 0xfffff000u ? 0xfffff000u : (uint32_t)bytes;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(b), (short)0, (int)range, 0x00020000);
      const int wave0 = __builtin_amdgcn_readfirstlane(tid & ~63);
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        uint32_t v = voff[i];
        if (KC && k0 + BK > K) {
          int line, first;
          place(i * NT + tid, line, first);
          if (first >= K - k0) v = 0xffffffffu;
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (i * NT + wave0) * 16), 16,
                                                 (int)v, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        int line, first;
        place(i * NT + tid, line, first);
        const int lines = KC ? rows : K - k0;
        const int left = (KC ? K - k0 : rows) - first;
        u4 w = {0, 0, 0, 0};
        if (line < lines && left > 0) {
          const T* q = b + (int64_t)line * ld + first;
          if (left >= V) {
            const Packed<T> x = *reinterpret_cast<const Packed<T>*>(q);
            w = __builtin_bit_cast(u4, x);
          } else {
            Packed<T> x = __builtin_bit_cast(Packed<T>, w);
#pragma unroll
            for (int j = 0; j < V; ++j)
              if (j < left) x.v[j] = q[j];
            w = __builtin_bit_cast(u4, x);
          }
        }
        reg[i] = w;
      }
    }
  }

  // Puts what load() left in registers into LDS.
  __device__ void store(char* lds) {
    if (!DMA) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) *reinterpret_cast<u4*>(lds + (i * NT + tid) * 16) = reg[i];
    }
  }
};

// The fragments of W 16-row blocks (from block `b0` of the tile) for fragment
// group g of a staged chunk.  fp32 MC: f[4 j + kk][i] is row 4 l16 + i of the
// 64 rows of block quad j, else f[i] belongs to row l16 of block i.
template <class T, bool KC, int ROWS, int W> __device__ inline void fragments(const char* lds, int b0, int g, int lane, u4* f) {
  const int q = lane >> 4, l16 = lane & 15;
  if (KC) {
    const char* p = lds + (b0 * 16 + l16) * 128 + (((4 * g + q) ^ (l16 & 7)) << 4);
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = *reinterpret_cast<const u4*>(p + i * 2048);
  } else if (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < W / 4; ++j)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        f[4 * j + kk] = *reinterpret_cast<const u4*>(lds + (16 * g + 4 * q + kk) * (ROWS * 4) + (b0 * 16 + 64 * j + 4 * l16) * 4);
  } else {
    const int line = 32 * g + 8 * q + (l16 >> 2);
    const int s = mc_swizzle<ROWS>(line);
    const char* p = lds + line * (ROWS * 2) + (l16 & 3) * 8;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const char* a = p + ((b0 + i) ^ s) * 32;
      typedef __attribute__((address_space(3))) s4* lp;
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(a));
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(a + 4 * ROWS * 2));
      f[i] = __builtin_bit_cast(u4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
}

__device__ inline float lane_value(const u4* f, bool kc, int i, int kk) {
  return __builtin_bit_cast(float, kc ? f[i][kk] : f[(i & ~3) + kk][i & 3]);
}

template <class T, bool AKC, bool BKC, int WM, int WN>
__device__ inline void multiply(const u4* a, const u4* b, f4 (&acc)[WM][WN]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(lane_value(a, AKC, i, kk), lane_value(b, BKC, j, kk), acc[i][j], 0, 0, 0);
  } else {
    typedef T v8 __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) {
        const v8 x = __builtin_bit_cast(v8, a[i]), y = __builtin_bit_cast(v8, b[j]);
        if constexpr (__is_same(T, bf16))
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[i][j], 0, 0, 0);
        else
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, acc[i][j], 0, 0, 0);
      }
  }
}

// ---------------------------------------------------------------------------
// the tiled product
// ---------------------------------------------------------------------------
// Workgroup id -> tile.  Consecutive ids go to different XCDs, so ids are
// dealt out such that each XCD gets a contiguous run of tiles; within a run,
// tiles go down groups of eight row tiles before the next column, so that the
// tiles of an XCD that run together share rows of A and columns of B in its L2.
__device__ inline void tile_of(int t, int mtiles, int ntiles, int& tm, int& tn) {
  const int T = mtiles * ntiles, T8 = T & ~7;
  if (t < T8) t = (t & 7) * (T8 >> 3) + (t >> 3);
  const int per = 8 * ntiles, grp = t / per, m0 = grp * 8, rows = min(8, mtiles - m0), r = t - grp * per;
  tn = r / rows;
  tm = m0 + r - tn * rows;
}

// The accumulators of a wave, through its own part of LDS, as vectors along M.
// Block column by block column: (16 WM) x 16 sums, then 16-byte results with
// neighbouring lanes next to each other along M.
template <class T, bool AKC, bool BKC, int WM, int WN>
__device__ inline void write_tile(const Product& p, int split, int m0, int n0, int lane, char* lds, f4 (&acc)[WM][WN]) {
  constexpr int S = 16 * WM + 4;               // floats from one column to the next
  float* st = reinterpret_cast<float*>(lds);
  const int q = lane >> 4, l16 = lane & 15;
#pragma unroll
  for (int j = 0; j < WN; ++j) {
    if (sizeof(T) == 4 && !AKC) {
#pragma unroll
      for (int i = 0; i < WM; i += 4)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f4*>(st + l16 * S + 16 * i + 16 * q + 4 * r) =
              f4{acc[i][j][r], acc[i + 1][j][r], acc[i + 2][j][r], acc[i + 3][j][r]};
    } else {
#pragma unroll
      for (int i = 0; i < WM; ++i) *reinterpret_cast<f4*>(st + l16 * S + 16 * i + 4 * q) = acc[i][j];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int V = kVec<T>;
    constexpr int PER = 16 * WM / V;           // vectors of a column
    for (int x = lane; x < PER * 16; x += 64) {
      const int col = x / PER, row = (x % PER) * V;
      const int n = n0 + ((sizeof(T) == 4 && !BKC) ? 64 * (j >> 2) + 4 * col + (j & 3) : 16 * j + col);
      const int m = m0 + row;
      const float* src = st + col * S + row;
      if (n >= p.N) continue;
      if (m + V <= p.M) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          const f4 w = *reinterpret_cast<const f4*>(src + i);
          v[i] = w[0], v[i + 1] = w[1], v[i + 2] = w[2], v[i + 3] = w[3];
        }
        if (p.splits > 1) {
          float* d = p.part + ((int64_t)split * p.N + n) * p.M + m;
#pragma unroll
          for (int i = 0; i < V; i += 4) store_vec(d + i, v + i);
        } else {
          finish_vec<T>(p.e, m, n, v);
        }
      } else {
        for (int i = 0; m + i < p.M; ++i) {
          if (p.splits > 1)
            p.part[((int64_t)split * p.N + n) * p.M + m + i] = src[i];
          else
            finish_one<T>(p.e, m + i, n, src[i]);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <class T, bool AKC, bool BKC, int WM, int WN, int WAVES_M, int WAVES_N, bool DMA>
__global__ __launch_bounds__(64 * WAVES_M* WAVES_N) void product_kernel(Product p) {
  constexpr int NT = 64 * WAVES_M * WAVES_N;
  constexpr int MT = 16 * WM * WAVES_M, NTILE = 16 * WN * WAVES_N;
  constexpr int BK = 128 / (int)sizeof(T);
  constexpr int ABYTES = MT * 128, BBYTES = NTILE * 128;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tiles = p.mtiles * p.ntiles;
  const int split = blockIdx.x / tiles;
  int tm, tn;
  tile_of(blockIdx.x - split * tiles, p.mtiles, p.ntiles, tm, tn);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WAVES_M, wn = wave / WAVES_M;

  f4 acc[WM][WN];
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int j = 0; j < WN; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};

  const int kts = (p.K + BK - 1) / BK;
  const int klo = (int)((int64_t)kts * split / p.splits), khi = (int)((int64_t)kts * (split + 1) / p.splits);
  Stage<T, AKC, MT, NT, DMA> sa;
  Stage<T, BKC, NTILE, NT, DMA> sb;
  sa.init(p.A, p.lda, tm * MT, p.M, p.K, tid);
  sb.init(p.B, p.ldb, tn * NTILE, p.N, p.K, tid);

  auto compute = [&](const char* buf) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      u4 a[WM], b[WN];
      fragments<T, AKC, MT, WM>(buf, wm * WM, g, lane, a);
      fragments<T, BKC, NTILE, WN>(buf + ABYTES, wn * WN, g, lane, b);
      multiply<T, AKC, BKC>(a, b, acc);
    }
  };
  if (klo < khi) {
    sa.load(klo, smem);
    sb.load(klo, smem + ABYTES);
    sa.store(smem);
    sb.store(smem + ABYTES);
    __syncthreads();
    for (int kt = klo; kt < khi; ++kt) {
      char* cur = smem + ((kt - klo) & 1) * (ABYTES + BBYTES);
      char* nxt = smem + ((kt - klo + 1) & 1) * (ABYTES + BBYTES);
      if (kt + 1 < khi) {
        sa.load(kt + 1, nxt);
        sb.load(kt + 1, nxt + ABYTES);
      }
      compute(cur);
      if (kt + 1 < khi) {
        sa.store(nxt);
        sb.store(nxt + ABYTES);
      }
      __syncthreads();
    }
  }
  write_tile<T, AKC, BKC, WM, WN>(p, split, tm * MT + wm * WM * 16, tn * NTILE + wn * WN * 16, lane,
                                  smem + wave * (16 * WM + 4) * 16 * 4, acc);
}

// Sums the partial products of a split contraction in order and finishes them.
template <class T> __global__ __launch_bounds__(256) void join_kernel(Product p) {
  constexpr int V = kVec<T>;
  const int per = (p.M + V - 1) / V;
  const int64_t total = (int64_t)per * p.N;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
    const int n = (int)(x / per), m = (int)(x - (int64_t)n * per) * V;
    const float* d = p.part + (int64_t)n * p.M + m;
    const int64_t next = (int64_t)p.N * p.M;
    if (m + V <= p.M) {
      float v[V], w[4];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = 0.0f;
      for (int s = 0; s < p.splits; ++s, d += next) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          load_vec(d + i, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i + j] += w[j];
        }
      }
      finish_vec<T>(p.e, m, n, v);
    } else {
      for (int i = 0; m + i < p.M; ++i) {
        float v = 0.0f;
        for (int s = 0; s < p.splits; ++s) v += d[s * next + i];
        finish_one<T>(p.e, m + i, n, v);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// choice and launch
// ---------------------------------------------------------------------------
constexpr int kTile = 128;

// How many workgroups share a tile's contraction: enough that the device has
// two workgroups per compute unit, with at least four chunks each.
int split_of(int dtype, int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ((M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  const int64_t kts = (K + (dtype == LINEAR_F32 ? 32 : 64) - 1) / (dtype == LINEAR_F32 ? 32 : 64);
  if (tiles == 0) return 1;
  const int64_t want = 2 * compute_units() / tiles;
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, kts / 4, 64}));
}

// Whether an operand can be staged by loads that go straight to LDS.
bool direct(int dtype, const void* p, int64_t ld, bool kc, int64_t rows, int64_t K) {
  const int64_t size = dtype == LINEAR_F32 ? 4 : 2, vec = 16 / size;
  return ((uintptr_t)p & 15) == 0 && ld % vec == 0 && (kc ? K : rows) % vec == 0 && ld * size * 256 < (1ll << 32) - 4096;
}

template <class T, bool AKC, bool BKC> hipError_t launch_typed(const Product& p, bool dma, hipStream_t s) {
  constexpr int kLds = 2 * (kTile + kTile) * 128;
  const dim3 grid((unsigned)((int64_t)p.mtiles * p.ntiles * p.splits));
  auto k = dma ? product_kernel<T, AKC, BKC, 4, 4, 2, 2, true> : product_kernel<T, AKC, BKC, 4, 4, 2, 2, false>;
  static_assert(4 * (16 * 4 + 4) * 16 * 4 <= kLds, "result staging fits");
  k<<<grid, 256, kLds, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t vecs = (int64_t)((p.M + kVec<T> - 1) / kVec<T>) * p.N;
  join_kernel<T><<<dim3((unsigned)std::min<int64_t>((vecs + 255) / 256, 4096)), 256, 0, s>>>(p);
  return hipGetLastError();
}

template <class T> hipError_t launch_ordered(bool a_kc, bool b_kc, const Product& p, bool dma, hipStream_t s) {
  if (a_kc && b_kc) return launch_typed<T, true, true>(p, dma, s);
  if (!a_kc && b_kc) return launch_typed<T, false, true>(p, dma, s);
  return launch_typed<T, false, false>(p, dma, s);   // (KC, MC) does not occur
}

}  // namespace

int64_t product_workspace(int dtype, int64_t M, int64_t N, int64_t K) {
  const int splits = split_of(dtype, M, N, K);
  return splits > 1 ? (int64_t)splits * M * N * 4 : 0;
}

hipError_t launch_product(int dtype, bool a_kc, bool b_kc, Product p, void* workspace, hipStream_t s) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  if (a_kc && !b_kc) return hipErrorInvalidValue;
  p.splits = split_of(dtype, p.M, p.N, p.K);
  p.mtiles = (p.M + kTile - 1) / kTile;
  p.ntiles = (p.N + kTile - 1) / kTile;
  p.part = static_cast<float*>(workspace);
  const bool dma = direct(dtype, p.A, p.lda, a_kc, p.M, p.K) && direct(dtype, p.B, p.ldb, b_kc, p.N, p.K);
  switch (dtype) {
    case LINEAR_F32: return launch_ordered<float>(a_kc, b_kc, p, dma, s);
    case LINEAR_BF16: return launch_ordered<bf16>(a_kc, b_kc, p, dma, s);
    default: return launch_ordered<f16>(a_kc, b_kc, p, dma, s);
  }
}

}  // namespace linear

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------
using linear::bad_ld;
using linear::check_sizes;

extern "C" int64_t convgemm_linear_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order) {
  if (int e = check_sizes(dtype, kn, ci, t)) return e;
  if (f_order != 0 && f_order != 1) return -5;
  return linear::product_workspace(dtype, kn, t, ci);
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
  const int64_t need = linear::product_workspace(dtype, kn, t, ci);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 15))) return -18;
  if (need > 0 && workspace_bytes < need) return -19;
  if (!work) return LINEAR_OK;
  linear::Product p{};
  p.A = F;
  p.lda = ldf;
  p.B = X;
  p.ldb = ldx;
  p.M = (int)kn;
  p.N = (int)t;
  p.K = (int)ci;
  p.e = linear::Epilogue{bias, residual, ldr, Z, ldz, O, ldo, act};
  const hipError_t e = linear::launch_product(dtype, f_order == 1, true, p, workspace, stream);
  return e == hipSuccess ? LINEAR_OK : LINEAR_ERR_HIP_BASE - (int)e;
}
