// The layer's matrix product on gfx950: C = act(A B + bias) + residual, both
// operands in either order, fp32, bf16 and fp16 on the matrix cores with fp32
// sums.
//
// What one lane feeds the matrix cores is always a 16-byte fragment:
//   * 16-bit types: 8 contraction values of one row, one v_mfma_*_16x16x32;
//   * fp32: 4 contraction values of one row for four v_mfma_f32_16x16x4_f32
//     (lane group q = lane / 16 takes contraction values 4q .. 4q+3 of a group
//     of 16, one per instruction).
// The contraction is walked in chunks of 128 bytes per row (32 fp32 or 64
// 16-bit values: two fragments per lane).  An operand whose contraction index
// is contiguous ("KC") lies in LDS as rows of 128 bytes whose eight 16-byte
// pieces are permuted by the row (piece ^ row & 7), so that 16 rows are read
// without bank conflicts.  An operand whose rows are contiguous ("MC") lies
// there as it is in memory, one line per contraction index: fp32 reads V = 4, 2
// or 1 neighbouring rows of one contraction index at a time (lane l16 then holds
// rows V l16 + i, i the block), the 16-bit types read through the transposing
// ds_read_b64_tr_b16, their 32-byte blocks permuted by the contraction index so
// that the four lines of a read lie in different banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "linear_common.h"
#include "ltlt_internal.h"

namespace linear {
namespace {

// ---------------------------------------------------------------------------
// one operand's tile
// ---------------------------------------------------------------------------
// LDS placement of a 16-bit MC line k of ROWS values: permutation of its 32-byte
// blocks.  A transposing read takes 32 lanes at once: four lines from 8q and four
// from 8q + 8, 32 bytes each, which this puts into the 256 bytes of the banks
// once.
template <int ROWS> __device__ inline int mc_swizzle(int k) {
  const int low = k & 3, high = (k >> 3) & 1;
  return ROWS >= 128 ? low | high << 2 : ROWS == 64 ? low >> 1 | high << 1 : ROWS == 32 ? high : 0;
}

// A range-checked load of WIDTH bytes a lane, straight to LDS: lane i's bytes go
// to `lds` + i WIDTH, zeros where the lane's offset is outside the range.  In
// assembly (it has no result register) because the compiler takes such a load to
// alias every transposing read and would wait for all loads before each; the
// kernels count the outstanding loads themselves.  The wait states are those that
// a vector memory instruction needs after a vector instruction has written one
// of its scalar registers (5) or after m0 was written (1).
typedef int i4 __attribute__((ext_vector_type(4)));
__device__ inline i4 buffer_of(const void* p, uint32_t range) {
  const uint64_t a = (uint64_t)p;
  return i4{(int)(uint32_t)a, (int)((uint32_t)(a >> 32) & 0xffffu), (int)range, 0x00020000};
}
template <int WIDTH> __device__ inline void load_to_lds(i4 r, uint32_t voff, const char* lds) {
  const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds;
  if constexpr (WIDTH == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(r) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(r) : "memory", "m0");
}

// Neighbouring rows that a lane reads at a time from an fp32 MC operand of W
// blocks.
constexpr int mc_rows(int W) { return W % 4 == 0 ? 4 : W % 2 == 0 ? 2 : 1; }

// The operand as the kernels load it: `rows` and `K` may be larger than the
// product's where the operand is a padded copy whose padding holds zeros.
template <class T> struct Operand {
  const T* p;
  int64_t ld;
  int rows, K;
};

// Staging of DEPTH chunks (ROWS x 128 bytes each) at a time by NT threads, in LDS
// order: straight to LDS, WIDTH = 16 or 4 bytes a lane and load, or through
// registers (WIDTH = 0).  4 bytes (fp32) need no more alignment than fp32 has and
// end at any value; their four times as many loads are hidden where the fp32
// matrix instructions are the bound.
template <class T, bool KC, int ROWS, int DEPTH, int NT, int WIDTH> struct Stage {
  static constexpr bool DMA = WIDTH > 0;
  static constexpr int V = kVec<T>;
  static constexpr int BK = 128 / (int)sizeof(T);
  static constexpr int LANES = WIDTH == 4 ? 4 : 1;          // lanes of a 16-byte piece
  static constexpr int PIECES = ROWS * 8 * DEPTH * LANES / NT;
  static constexpr int BYTES = ROWS * 128 * DEPTH;
  static_assert(PIECES * NT == ROWS * 8 * DEPTH * LANES, "whole pieces");
  static_assert(WIDTH == 0 || WIDTH == 16 || (WIDTH == 4 && sizeof(T) == 4), "load widths");
  static_assert(WIDTH == 0 || (KC ? ROWS : BK * DEPTH) <= kStageLines, "32-bit offsets");
  const T* at;            // the tile's first row, next contraction index
  int64_t ld;
  int64_t left;           // values from `at` to the operand's last one
  int rows;               // rows that exist from the tile's first one
  int K;                  // contraction values that are left
  int tid, wave0;
  uint32_t voff[DMA ? PIECES : 1];
  u4 reg[DMA ? 1 : PIECES];

  // what lane slot c moves: its row (KC) or contraction index (MC) and the first
  // value along the contiguous index
  __device__ static void place(int slot, int& line, int& first) {
    const int c = slot / LANES;
    const int sub = c / (ROWS * 8), w = c % (ROWS * 8);
    if (KC) {
      line = w >> 3;
      first = sub * BK + ((w & 7) ^ (line & 7)) * V;
    } else {
      constexpr int PPL = ROWS / V;
      line = w / PPL;
      int q = w % PPL;
      if (sizeof(T) == 2) q ^= mc_swizzle<ROWS>(line) << 1;
      first = q * V;
      line += sub * BK;
    }
    first += slot % LANES;
  }

  // Starts at contraction index k0; loads stop at `end`.
  __device__ void init(const Operand<T>& o, int row0, int k0, int end, int tid_) {
    ld = o.ld;
    at = o.p + (KC ? (int64_t)row0 * ld + k0 : (int64_t)k0 * ld + row0);
    rows = o.rows - row0;
    K = (DMA ? o.K : min(o.K, end)) - k0;
    left = KC ? (int64_t)(min(rows, ROWS) - 1) * ld + K : (int64_t)(K - 1) * ld + rows;
    tid = tid_;
    wave0 = __builtin_amdgcn_readfirstlane(tid & ~63) * (16 / LANES);
    if (DMA) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        int line, first;
        place(i * NT + tid, line, first);
        voff[i] = (uint32_t)line * (uint32_t)(ld * sizeof(T)) + (uint32_t)first * (uint32_t)sizeof(T);
      }
    }
  }

  // Loads the next DEPTH chunks (nothing where `more` is not set): straight
  // into LDS (DMA), or into registers.
  __device__ void load(bool more, char* lds) {
    if constexpr (DMA) {
      // range: up to the operand's last value; beyond it (rows past the end of
      // a KC operand, contraction indices past the end of an MC one) the load
      // gives zero.  A KC row's pieces past the contraction's end lie inside
      // the next row and are sent out of range.
      const int64_t bytes = left * (int)sizeof(T);
      const uint32_t range = !more || bytes <= 0 ? 0u : bytes > kReach ? (uint32_t)kReach : (uint32_t)bytes;
      const i4 r = buffer_of(at, range);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        uint32_t v = voff[i];
        if (KC) {
          int line, first;
          place(i * NT + tid, line, first);
          if (first >= K) v = 0xffffffffu;
        }
        load_to_lds<DMA ? WIDTH : 4>(r, v, lds + i * NT * (16 / LANES) + wave0);
      }
    } else if (more) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        int line, first;
        place(i * NT + tid, line, first);
        const int lines = KC ? rows : K;
        const int valid = (KC ? K : rows) - first;
        u4 w = {0, 0, 0, 0};
        if (line < lines && valid > 0) {
          const T* q = at + (int64_t)line * ld + first;
          if (valid >= V) {
            const Packed<T> x = *reinterpret_cast<const Packed<T>*>(q);
            w = __builtin_bit_cast(u4, x);
          } else {
            Packed<T> x = __builtin_bit_cast(Packed<T>, w);
#pragma unroll
            for (int j = 0; j < V; ++j)
              if (j < valid) x.v[j] = q[j];
            w = __builtin_bit_cast(u4, x);
          }
        }
        reg[i] = w;
      }
    }
    const int64_t step = KC ? (int64_t)(BK * DEPTH) : (int64_t)(BK * DEPTH) * ld;
    at += step;
    left -= step;
    K -= BK * DEPTH;
  }

  // Puts what load() left in registers into LDS.
  __device__ void store(char* lds) {
    if (!DMA) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) *reinterpret_cast<u4*>(lds + (i * NT + tid) * 16) = reg[i];
    }
  }
};

// The fragments of W 16-row blocks (from block `b0` of the tile) for fragment
// group g of a staged chunk: f[i] belongs to row l16 of block i, or, fp32 MC,
// f[4 (i / V) + kk][i % V] to row V l16 + i % V of its 16 V rows.
template <class T, bool KC, int ROWS, int W> __device__ inline void fragments(const char* lds, int b0, int g, int lane, u4* f) {
  const int q = lane >> 4, l16 = lane & 15;
  if constexpr (KC) {
    const char* p = lds + (b0 * 16 + l16) * 128 + (((4 * g + q) ^ (l16 & 7)) << 4);
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = *reinterpret_cast<const u4*>(p + i * 2048);
  } else if constexpr (sizeof(T) == 4) {
    constexpr int V = mc_rows(W);
    typedef uint32_t uv __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int j = 0; j < W / V; ++j)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const char* a = lds + (16 * g + 4 * q + kk) * (ROWS * 4) + (b0 * 16 + 16 * V * j + V * l16) * 4;
        if constexpr (V == 1) {
          f[4 * j + kk][0] = *reinterpret_cast<const uint32_t*>(a);
        } else {
          const uv x = *reinterpret_cast<const uv*>(a);
#pragma unroll
          for (int v = 0; v < V; ++v) f[4 * j + kk][v] = x[v];
        }
      }
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

template <class T, bool KC> constexpr int neighbours(int W) { return sizeof(T) == 4 && !KC ? mc_rows(W) : 1; }

// Registers that fragments() fills.
template <class T, bool KC> constexpr int frag_count(int W) { return sizeof(T) == 4 && !KC ? W / mc_rows(W) * 4 : W; }

template <bool KC, int W> __device__ inline float lane_value(const u4* f, int i, int kk) {
  constexpr int V = mc_rows(W);
  const uint32_t x = KC ? f[i][kk] : f[4 * (i / V) + kk][i % V];
  return __builtin_bit_cast(float, x);
}

template <class T> __device__ inline f4 mfma16(u4 a, u4 b, f4 c) {
  typedef T v8 __attribute__((ext_vector_type(8)));
  if constexpr (__is_same(T, bf16))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}

// Adds the products of WM x WN blocks to the sums from block (i0, j0) on.
template <class T, bool AKC, bool BKC, int WM, int WN, class Acc>
__device__ inline void multiply(const u4* a, const u4* b, Acc& acc, int i0 = 0, int j0 = 0) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
          acc[i0 + i][j0 + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
              lane_value<AKC, WM>(a, i, kk), lane_value<BKC, WN>(b, j, kk), acc[i0 + i][j0 + j], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) acc[i0 + i][j0 + j] = mfma16<T>(a[i], b[j], acc[i0 + i][j0 + j]);
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

// COLS columns of ROWS sums, staged by this wave ROWS + 4 floats apart, to the
// result: rows m0 .., columns n0, n0 + step, ...  Neighbouring lanes take
// neighbouring 16-byte results of a column.
template <class T, int ROWS, int COLS, bool STREAM>
__device__ inline void write_columns(const Product& p, int split, int m0, int n0, int step, int lane, const float* st) {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  constexpr int V = kVec<T>;
  constexpr int PER = ROWS / V;              // vectors of a column
  for (int x = lane; x < PER * COLS; x += 64) {
    const int col = x / PER, row = (x % PER) * V;
    const int n = n0 + step * col, m = m0 + row;
    const float* src = st + col * (ROWS + 4) + row;
    if (n >= p.N || m >= p.M) continue;
    const int cnt = min(V, p.M - m);
    auto sums = [&](float* v) {
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f4 w = *reinterpret_cast<const f4*>(src + i);
        v[i] = w[0], v[i + 1] = w[1], v[i + 2] = w[2], v[i + 3] = w[3];
      }
    };
    if (!p.part) {
      if (cnt == V)
        finish<T, true, STREAM>(p.e, m, n, cnt, sums);
      else
        finish<T, false, STREAM>(p.e, m, n, cnt, sums);
    } else {
      float* d = p.part + ((int64_t)split * p.N + n) * p.M + m;
      if (cnt == V) {
        float v[V];
        sums(v);
        if (p.add) {
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            float w[4];
            load_vec(d + i, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] += w[j];
          }
        }
#pragma unroll
        for (int i = 0; i < V; i += 4) store_vec(d + i, v + i);
      } else {
        for (int i = 0; i < cnt; ++i) d[i] = p.add ? d[i] + src[i] : src[i];
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The accumulators of a wave, through its own part of LDS, as vectors along M.
// Block column by block column: (16 WM) x 16 sums, then 16-byte results with
// neighbouring lanes next to each other along M.
// VA and VB neighbouring rows (columns) lie in neighbouring blocks (fp32 MC).
template <class T, int VA, int VB, bool STREAM = false, int WM, int WN>
__device__ inline void write_tile(const Product& p, int split, int m0, int n0, int lane, char* lds, f4 (&acc)[WM][WN]) {
  constexpr int S = 16 * WM + 4;               // floats from one column to the next
  float* st = reinterpret_cast<float*>(lds);
  const int q = lane >> 4, l16 = lane & 15;
#pragma unroll
  for (int j = 0; j < WN; ++j) {
    if constexpr (VA > 1) {
      typedef float fv __attribute__((ext_vector_type(VA)));
#pragma unroll
      for (int i = 0; i < WM; i += VA)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          fv x;
#pragma unroll
          for (int v = 0; v < VA; ++v) x[v] = acc[i + v][j][r];
          *reinterpret_cast<fv*>(st + l16 * S + 16 * i + VA * (4 * q + r)) = x;
        }
    } else {
#pragma unroll
      for (int i = 0; i < WM; ++i) *reinterpret_cast<f4*>(st + l16 * S + 16 * i + 4 * q) = acc[i][j];
    }
    write_columns<T, 16 * WM, 16, STREAM>(p, split, m0, n0 + 16 * VB * (j / VB) + j % VB, VB, lane, st);
  }
}

// What a kernel does with a wave's sums: the layer's results.
struct LayerEnd {
  using P = Product;
  template <class T, int VA, int VB, bool STREAM, int WM, int WN>
  static __device__ void tile(const P& p, int split, int m0, int n0, int lane, char* lds, f4 (&acc)[WM][WN]) {
    write_tile<T, VA, VB, STREAM>(p, split, m0, n0, lane, lds, acc);
  }
};

// Until at most N loads are outstanding (the counter holds 63).
template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N < 63 ? N : 63) : "memory"); }

__device__ inline void workgroup_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <class T> __device__ inline Operand<T> operand_a(const Product& p) {
  return Operand<T>{static_cast<const T*>(p.A), p.lda, p.arows, p.aK};
}
template <class T> __device__ inline Operand<T> operand_b(const Product& p) {
  return Operand<T>{static_cast<const T*>(p.B), p.ldb, p.brows, p.bK};
}

// A tile of (16 WM WAVES_M) x (16 WN WAVES_N), its contraction walked in stages
// of DEPTH chunks whose 2 DEPTH fragment groups are shared by WAVES_K groups of
// waves; the groups' sums are added in order at the end.  LDS is a ring of
// STAGES stages: the loads of stage s + STAGES - 1 are issued before stage s is
// multiplied, so STAGES - 1 stages are under way at any time.  For few tokens the
// bound is the bytes under way: 16384 x 4096 bf16 weights by 8 tokens run at 5.6 TB/s
// with 73 KB per compute unit, at 3.5 with 27; for tens to hundreds of tokens it is
// what the L2 caches deliver (8 to 9 TB/s at 80 and at 300 tokens) and a stage's own
// latencies (0.3 us).
template <class T, bool AKC, bool BKC, int WM, int WN, int WAVES_M, int WAVES_N, int WAVES_K, int DEPTH, int STAGES, int WIDTH>
struct Ring {
  static constexpr bool DMA = WIDTH > 0;
  static constexpr int GROUPS = 2 * DEPTH / WAVES_K;    // fragment groups of a stage that one wave takes
  static_assert(GROUPS * WAVES_K == 2 * DEPTH, "whole fragment groups");
  static constexpr int MT = 16 * WM * WAVES_M, NTILE = 16 * WN * WAVES_N;
  static constexpr int WAVES = WAVES_M * WAVES_N * WAVES_K, NT = 64 * WAVES;
  using SA = Stage<T, AKC, MT, DEPTH, NT, WIDTH>;
  using SB = Stage<T, BKC, NTILE, DEPTH, NT, WIDTH>;
  static constexpr int BK = SA::BK * DEPTH;
  static constexpr int STAGE_BYTES = SA::BYTES + SB::BYTES;
  static constexpr int SUM_BYTES = (WAVES_K - 1) * MT * NTILE * 4;
  static constexpr int OUT_BYTES = WAVES_M * WAVES_N * (16 * WM + 4) * 16 * 4;
  static constexpr int LDS = STAGES * STAGE_BYTES > SUM_BYTES + OUT_BYTES ? STAGES * STAGE_BYTES : SUM_BYTES + OUT_BYTES;

  template <class END> static __device__ void run(const typename END::P& p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tiles = p.mtiles * p.ntiles;
    const int split = blockIdx.x / tiles;
    int tm, tn;
    tile_of(blockIdx.x - split * tiles, p.mtiles, p.ntiles, tm, tn);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / (WAVES_M * WAVES_N), w = wave % (WAVES_M * WAVES_N);
    const int wm = w % WAVES_M, wn = w / WAVES_M;

    f4 acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    const int steps = (p.K + BK - 1) / BK;
    const int lo = (int)((int64_t)steps * split / p.splits), hi = (int)((int64_t)steps * (split + 1) / p.splits);
    SA sa;
    SB sb;
    sa.init(operand_a<T>(p), tm * MT, lo * BK, hi * BK, tid);
    sb.init(operand_b<T>(p), tn * NTILE, lo * BK, hi * BK, tid);

    // this wave's fragment groups of a stage; `between` runs while they are read
    auto compute = [&](const char* buf, auto between) {
      u4 a[GROUPS][frag_count<T, AKC>(WM)], b[GROUPS][frag_count<T, BKC>(WN)];
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const int group = kg * GROUPS + i, chunk = group >> 1;
        fragments<T, AKC, MT, WM>(buf + chunk * MT * 128, wm * WM, group & 1, lane, a[i]);
        fragments<T, BKC, NTILE, WN>(buf + SA::BYTES + chunk * NTILE * 128, wn * WN, group & 1, lane, b[i]);
      }
      between();
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) multiply<T, AKC, BKC, WM, WN>(a[i], b[i], acc);
    };
    auto load = [&](int s, char* buf) {
      sa.load(s < hi, buf);
      sb.load(s < hi, buf + SA::BYTES);
    };
    if constexpr (DMA) {
      constexpr int L = SA::PIECES + SB::PIECES;
#pragma unroll
      for (int i = 0; i < STAGES - 1; ++i) load(lo + i, smem + i * STAGE_BYTES);
      int at = 0;                                // stage s lies at `at`
      for (int s = lo; s < hi; ++s) {
        wait_loads<(STAGES - 2) * L>();
        workgroup_barrier();
        compute(smem + at * STAGE_BYTES, [&] { load(s + STAGES - 1, smem + (at == 0 ? STAGES - 1 : at - 1) * STAGE_BYTES); });
        at = at + 1 == STAGES ? 0 : at + 1;
      }
      wait_loads<0>();
      workgroup_barrier();
    } else if (lo < hi) {
      load(lo, smem);
      sa.store(smem);
      sb.store(smem + SA::BYTES);
      __syncthreads();
      for (int s = lo; s < hi; ++s) {
        char* cur = smem + ((s - lo) & 1) * STAGE_BYTES;
        char* nxt = smem + ((s - lo + 1) & 1) * STAGE_BYTES;
        if (s + 1 < hi) load(s + 1, nxt);
        compute(cur, [] {});
        if (s + 1 < hi) {
          sa.store(nxt);
          sb.store(nxt + SA::BYTES);
        }
        __syncthreads();
      }
    }
    if constexpr (WAVES_K > 1) {
      f4* sum = reinterpret_cast<f4*>(smem) + w * (WM * WN * 64) + lane;
      constexpr int next = WAVES_M * WAVES_N * WM * WN * 64;
      if (kg > 0) {
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j) sum[(kg - 1) * next + (i * WN + j) * 64] = acc[i][j];
      }
      __syncthreads();
      if (kg > 0) return;
#pragma unroll 1
      for (int k = 0; k < WAVES_K - 1; ++k)
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j) acc[i][j] += sum[k * next + (i * WN + j) * 64];
    }
    END::template tile<T, neighbours<T, AKC>(WM), neighbours<T, BKC>(WN), false>(
        p, split, tm * MT + wm * WM * 16, tn * NTILE + wn * WN * 16, lane, smem + SUM_BYTES + w * (16 * WM + 4) * 16 * 4, acc);
  }
};

// Two waves per SIMD at least: 256 registers, which keeps the sums in the
// registers that the matrix instructions and the epilogue both reach.
template <class R> __global__ __launch_bounds__(R::NT, 2) void ring_kernel(Product p) { R::template run<LayerEnd>(p); }

// ---------------------------------------------------------------------------
// the 256 x 256 product (16-bit types, both operands straight to LDS)
// ---------------------------------------------------------------------------
// Eight waves, two by four, each with a 128 x 64 part of the tile. Per chunk a
// wave's part is four quarters of 16 matrix instructions each, and
// every quarter is a phase between two workgroup barriers:
//   phase 0: rows half 0 x columns half 0    reads A0, B0
//   phase 1: rows half 0 x columns half 1    reads B1
//   phase 2: rows half 1 x columns half 1    reads A1
//   phase 3: rows half 1 x columns half 0    reads nothing
// LDS holds two chunks. A quarter of a chunk (A0, B0, B1 or A1: 16 KB) is loaded
// again as soon as every wave has read it: the four phases of chunk k start
// the loads of B1 and A1 of chunk k+1 and of A0 and B0 of chunk k+2. Loads
// return in order, so waiting until eight are outstanding (two a quarter and
// phase) always means: what the next phase reads is there, and every load has
// four phases to arrive. The upper four waves run one barrier behind the
// lower four, so that on every SIMD one wave reads while the other multiplies.
// 8192^3 bf16: 1430 TFLOP/s with the contraction contiguous in both operands, 1378
// and 1353 with one and none (the library's product in turn on the same card: 1645,
// 1407 and 1229; cards differ by 5 %); the 128 x 128 ring: 1050 at 4096^3.  Bound by
// the matrix cores at the clock that they hold; between tiles, by the results, which
// are written while no product runs.
// One operand of the wide product: sub-tiles of SR rows (64 of A, 32 of B) x
// 128 bytes, each as in Stage. Half h of the operand is the sub-tiles 2 s + h.
template <class T, bool KC, int SR> struct WideStage {
  static constexpr int PER = 512 / (SR * 8);     // sub-tiles that 512 threads load at once
  static constexpr int SIZE = (int)sizeof(T), V = kVec<T>, BK = 128 / SIZE;
  const T* base;
  int64_t ld;
  int rows, K;
  int first;                                     // KC: this lane's first contraction value in a chunk
  uint32_t voff[4];                              // [2 h + j]: part j of half h
  uint32_t to[4];                                // its place in LDS
  i4 r;
  uint32_t mask;

  __device__ void init(const Operand<T>& o, int row0, int tid) {
    ld = o.ld;
    base = o.p + (KC ? (int64_t)row0 * ld : (int64_t)row0);
    rows = o.rows - row0;
    K = o.K;
    const int c = tid % (SR * 8), group = tid / (SR * 8);
    int line, q;
    if (KC) {
      line = c >> 3;
      q = (c & 7) ^ (line & 7);
    } else {
      constexpr int CPL = SR / V;
      line = c / CPL;
      q = c % CPL;
      if (SIZE == 2) q ^= mc_swizzle<SR>(line) << 1;
    }
    first = q * V;
    const int wave0 = __builtin_amdgcn_readfirstlane(tid & ~63) % (SR * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int sub = 2 * (PER * j + group) + h;
        voff[2 * h + j] = (KC ? (uint32_t)(sub * SR + line) * (uint32_t)(ld * SIZE) : (uint32_t)line * (uint32_t)(ld * SIZE) + (uint32_t)(sub * SR * SIZE)) +
                          (uint32_t)(first * SIZE);
        to[2 * h + j] = __builtin_amdgcn_readfirstlane((sub * SR * 8 + wave0) * 16);
      }
  }

  // Makes chunk kt the one that load() takes; nothing is loaded from `end` on.
  __device__ void at(int kt, int end) {
    const int k0 = kt * BK;
    const T* b = base + (KC ? (int64_t)k0 : (int64_t)k0 * ld);
    const int64_t span = KC ? (int64_t)(min(rows, 256) - 1) * ld + (K - k0) : (int64_t)(min(K - k0, BK) - 1) * ld + rows;
    const uint64_t bytes = (uint64_t)span * SIZE;
    const uint32_t range = kt >= end ? 0u : bytes > (uint64_t)kReach ? (uint32_t)kReach : (uint32_t)bytes;
    r = buffer_of(b, range);
    mask = KC && first >= K - k0 ? 0xffffffffu : 0u;
  }

  __device__ void load(int h, char* lds) const {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      load_to_lds<16>(r, voff[2 * h + j] | mask, lds + to[2 * h + j]);
  }
};

constexpr int kWideBuffer = 65536;                 // one chunk of both operands

template <class T, bool AKC, bool BKC, bool STREAM, class END> __device__ inline void wide_run(const typename END::P& p) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tiles = p.mtiles * p.ntiles;
  const int split = blockIdx.x / tiles;
  int tm, tn;
  tile_of(blockIdx.x - split * tiles, p.mtiles, p.ntiles, tm, tn);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;

  f4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};

  constexpr int BK = 128 / (int)sizeof(T);
  const int kts = (p.K + BK - 1) / BK;
  const int klo = (int)((int64_t)kts * split / p.splits), khi = (int)((int64_t)kts * (split + 1) / p.splits);
  WideStage<T, AKC, 64> sa;
  WideStage<T, BKC, 32> sb;
  sa.init(operand_a<T>(p), tm * 256, tid);
  sb.init(operand_b<T>(p), tn * 256, tid);

  sa.at(klo, khi);
  sb.at(klo, khi);
  sa.load(0, smem);
  sb.load(0, smem + 32768);
  sb.load(1, smem + 32768);
  sa.load(1, smem);
  sa.at(klo + 1, khi);
  sb.at(klo + 1, khi);
  sa.load(0, smem + kWideBuffer);
  sb.load(0, smem + kWideBuffer + 32768);
  wait_loads<8>();
  workgroup_barrier();
  if (wm == 1) workgroup_barrier();

  for (int kt = klo; kt < khi; ++kt) {
    char* cur = smem + ((kt - klo) & 1) * kWideBuffer;
    char* nxt = smem + ((kt - klo + 1) & 1) * kWideBuffer;
    constexpr int FA = frag_count<T, AKC>(4), FB = frag_count<T, BKC>(2);
    u4 a[2][FA], b0[2][FB], b1[2][FB];
    auto read_a = [&](int h) {
#pragma unroll
      for (int g = 0; g < 2; ++g) fragments<T, AKC, 64, 4>(cur + (wm * 2 + h) * 8192, 0, g, lane, a[g]);
    };
    auto read_b = [&](int h, u4 (&b)[2][FB]) {
#pragma unroll
      for (int g = 0; g < 2; ++g) fragments<T, BKC, 32, 2>(cur + 32768 + (wn * 2 + h) * 4096, 0, g, lane, b[g]);
    };
    auto quarter = [&](int h, const u4 (&b)[2][FB], int jh) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int g = 0; g < 2; ++g) multiply<T, AKC, BKC, 4, 2>(a[g], b[g], acc, 4 * h, 2 * jh);
      __builtin_amdgcn_s_setprio(0);
    };
    read_b(0, b0);
    read_a(0);
    sb.load(1, nxt + 32768);
    wait_loads<8>();
    workgroup_barrier();
    quarter(0, b0, 0);
    workgroup_barrier();

    read_b(1, b1);
    sa.load(1, nxt);
    wait_loads<8>();
    workgroup_barrier();
    quarter(0, b1, 1);
    workgroup_barrier();

    read_a(1);
    sa.at(kt + 2, khi);
    sa.load(0, cur);
    workgroup_barrier();
    quarter(1, b1, 1);
    workgroup_barrier();

    sb.at(kt + 2, khi);
    sb.load(0, cur + 32768);
    wait_loads<8>();
    workgroup_barrier();
    quarter(1, b0, 0);
    workgroup_barrier();
  }
  if (wm == 0) workgroup_barrier();
  // the loads past the end wrote zeros; LDS is free after them
  wait_loads<0>();
  workgroup_barrier();
  END::template tile<T, neighbours<T, AKC>(4), neighbours<T, BKC>(2), STREAM>(p, split, tm * 256 + wm * 128, tn * 256 + wn * 64, lane,
                                                                      smem + wave * (16 * 8 + 4) * 16 * 4, acc);
}

template <class T, bool AKC, bool BKC, bool STREAM> __global__ __launch_bounds__(512) void wide_kernel(Product p) {
  wide_run<T, AKC, BKC, STREAM, LayerEnd>(p);
}

// Sums the partial products of a split contraction in order and finishes them:
// first every whole vector, then value by value what the columns have left over,
// so that a wave has one kind only.
template <class T> __global__ __launch_bounds__(256) void join_kernel(Product p) {
  constexpr int V = kVec<T>;
  const int per = p.M / V, rest = p.M - per * V;
  const int64_t whole = (int64_t)per * p.N, total = whole + (int64_t)rest * p.N, next = (int64_t)p.N * p.M;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
    if (x < whole) {
      const int n = (int)(x / per), m = (int)(x - (int64_t)n * per) * V;
      const float* d = p.part + (int64_t)n * p.M + m;
      finish<T, true, false>(p.e, m, n, V, [&](float* v) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
        for (int s = 0; s < p.splits; ++s, d += next) {
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            float w[4];
            load_vec(d + i, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] += w[j];
          }
        }
      });
    } else {
      const int n = (int)((x - whole) / rest), m = per * V + (int)((x - whole) % rest);
      const float* d = p.part + (int64_t)n * p.M + m;
      float v = 0.0f;
      for (int s = 0; s < p.splits; ++s) v += d[s * next];
      finish_one<T>(p.e, m, n, v);
    }
  }
}

// Padded copies of up to two operands whose lines are not 16-byte aligned or no
// multiple of 16 bytes long: lines of `len` values, `ld` apart, to lines of
// `to_ld` values with zeros behind the last one.  One extra pass over an operand
// costs a fraction of what the direct loads gain once a tile's rows are used by
// more than one column tile.
struct Copy {
  const void* from;
  void* to;
  int64_t ld, to_ld, lines;
  int len;
};

template <class T> __global__ __launch_bounds__(256) void pad_kernel(Copy a, Copy b, int a_blocks) {
  constexpr int V = kVec<T>;
  const bool second = (int)blockIdx.x >= a_blocks;
  const Copy c = second ? b : a;
  const int64_t block = second ? blockIdx.x - a_blocks : blockIdx.x, blocks = second ? gridDim.x - a_blocks : a_blocks;
  const uint32_t per = (uint32_t)(c.to_ld / V);
  const int64_t total = c.lines * per;
  for (int64_t x0 = block * 256; x0 < total; x0 += blocks * 256) {
    const int64_t line0 = x0 / per;                         // the same for the workgroup
    const uint32_t x = (uint32_t)(x0 - line0 * per) + threadIdx.x;
    const int64_t line = line0 + x / per;
    const int at = (int)(x % per) * V;
    if (line >= c.lines) continue;
    const T* q = static_cast<const T*>(c.from) + line * c.ld + at;
    Packed<T> v;
    if (at + V <= c.len) {
      v = *reinterpret_cast<const Packed<T>*>(q);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v.v[i] = at + i < c.len ? q[i] : (T)0.0f;
    }
    *reinterpret_cast<u4*>(static_cast<T*>(c.to) + line * c.to_ld + at) = __builtin_bit_cast(u4, v);
  }
}

// ---------------------------------------------------------------------------
// choice and launch
// ---------------------------------------------------------------------------
// The kernels: tile, chunks of a stage, stages, workgroups that a compute unit holds
// (by their LDS), and, for fp32 and for the 16-bit types, what their time is made
// of (microseconds): `start` for a launch and the first loads, `stage` the least
// time of a stage (its latencies), `rate` the share of kRate that the matrix
// instructions reach, `out` the result of a 64 x 64 part.
// The figures are a fit to the times of 500 random products of layers with 64 ..
// 16384 outputs and inputs and 1 .. 8192 tokens for each type, every kernel with
// 1, 2, 4 and 8 splits, operands in the caches.  On 741 (fp32) and 179 (bf16)
// other such products the choice by them is 3.1 and 1.7 % slower on average than
// the fastest kernel of each.  Without one of the kernels the fastest would be
// slower on average by (fp32 / bf16) 0.4 % for bf16 (256 x 256), 0.3 / 0.5 and 0 /
// 0.4 % (128 x 128), 0.2 / 0.1 % (128 x 64), 2.2 / 3.2 and 0.1 / 0.4 % (64 x 64),
// 0.9 / 1.6 % (32 x 32), 0.1 / 0 % (64 x 32), 2.7 / 0.1 % (64 x 16),
// 4.2 / 1.3 % (16 x 16), 0.1 % for fp32 (32 x 80 and 16 x 80, which save up to a
// quarter just below a multiple of 80 tokens); the large tiles matter where the work
// is large.  Cold operands have one constant of their own (time_of()) and no fit.
enum Shape { kWide, kSquare2, kSquare4, kTall, kSmall, kQuad64, kBlock32, kNarrow32, kNarrow16, kThin16, kRow80, kSlim80, kShapes };
struct Figures {
  float start, stage, rate, out;
};
struct Tile {
  int m, n, depth, stages, held;
  Figures f32, f16;
};
constexpr Tile kTiles[kShapes] = {
    {256, 256, 1, 2, 1,     {}, {4.90f, 0.60f, 1.02f, 0.181f}},  // eight waves in two groups that alternate (16-bit types)
    {128, 128, 1, 2, 2,     {3.34f, 0.61f, 1.22f, 0.060f}, {3.49f, 0.87f, 1.18f, 0.073f}},  // two workgroups per unit
    {128, 128, 1, 4, 1,     {2.87f, 0.44f, 1.25f, 0.187f}, {3.64f, 0.57f, 1.00f, 0.102f}},  // eight waves
    {128, 64, 1, 3, 2,      {4.60f, 1.04f, 1.20f, 0.331f}, {4.08f, 0.45f, 1.06f, 0.199f}},
    {64, 64, 1, 4, 2,       {3.85f, 0.26f, 1.07f, 0.097f}, {3.60f, 0.29f, 1.08f, 0.087f}},
    {64, 64, 2, 4, 1,       {3.94f, 0.72f, 1.11f, 0.286f}, {4.06f, 0.36f, 0.85f, 0.043f}},  // eight waves, two for each part of the tile
    {32, 32, 4, 4, 1,       {4.88f, 0.49f, 0.66f, 0.060f}, {4.10f, 0.31f, 1.01f, 0.065f}},  // four waves share the contraction
    {64, 32, 4, 3, 1,       {4.21f, 0.33f, 0.89f, 0.012f}, {4.29f, 0.39f, 0.80f, 0.000f}},  // four waves share the contraction
    {64, 16, 4, 3, 1,       {4.02f, 0.42f, 1.03f, 0.000f}, {4.02f, 0.44f, 0.78f, 0.000f}},  // four waves share the contraction
    {16, 16, 8, 4, 1,       {4.37f, 0.40f, 1.22f, 0.003f}, {4.14f, 0.27f, 0.94f, 0.002f}},  // eight waves share the contraction: one token
    {32, 80, 2, 2, 2,       {5.59f, 0.79f, 1.03f, 0.000f}, {}},                                // fp32, 65 .. 320 tokens: with the next one 9 % of random layers
    {16, 80, 4, 3, 1,       {4.42f, 0.49f, 0.82f, 0.118f}, {}},                                // the same, eight waves share the contraction
};
struct Rates {
  double mul;             // operations per microsecond and compute unit
  double load;            // bytes per microsecond into a compute unit's LDS
  double read;            // bytes per microsecond from memory
  double join, join_rate; // the launch that adds split contractions, and its bytes
};
constexpr Rates kRates32 = {0.4259e6, 51.7e3, 4.82e6, 3.23, 2.78e6}, kRates16 = {6.741e6, 69.6e3, 4.87e6, 3.39, 3.17e6};

struct Plan {
  Shape shape;
  int splits;
  double us;              // what the figures say it takes
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

double time_of(const Tile& t, bool f32, int width, int64_t M, int64_t N, int64_t K, int64_t splits, int64_t cu) {
  const int size = f32 ? 4 : 2;
  const Figures& f = f32 ? t.f32 : t.f16;
  const Rates& r = f32 ? kRates32 : kRates16;
  const int64_t deep = 128 / size * t.depth, groups = ceil_div(M, t.m) * ceil_div(N, t.n) * splits;
  const double steps = (double)ceil_div(ceil_div(K, deep), splits);
  const double load = (t.m + t.n) * 128.0 * t.depth / r.load * (width == 4 ? 4.0 : 1.0);   // four times as many loads
  const double mul = 2.0 * t.m * t.n * deep / (r.mul * f.rate);
  auto round = [&](int64_t c) {   // c workgroups per compute unit at once
    return steps * std::max<double>(f.stage, c * std::max(load, mul)) + f.out * c * (t.m * t.n / 4096.0);
  };
  const int64_t full = groups / (t.held * cu), rest = groups % (t.held * cu);
  const double work = full * round(t.held) + (rest ? round(ceil_div(rest, cu)) : 0.0);
  // what the workgroups have under way bounds the rate of reading: about 2 us for
  // a load from memory, half of that from the last-level cache
  const double bytes = (double)size * ((double)M * K + (double)K * N);
  const double way = std::min(groups, t.held * cu) * (double)(std::min<int64_t>(t.m, M) + std::min<int64_t>(t.n, N)) * 128.0 *
                     t.depth * (t.stages - 1);
  const double read = bytes / std::min(r.read, way / (bytes > 32e6 ? 2.0 : 1.0));
  double us = std::max(work, read) + 0.05 * std::min(work, read) + f.start;
  if (splits > 1) us += r.join + splits * (double)M * N * 8.0 / r.join_rate;
  return us;
}

Plan search_plan(bool f32, int width, bool a_kc, bool b_kc, bool whole, int64_t M, int64_t N, int64_t K, int64_t cu) {
  Plan best{kSquare2, 1, 0.0};
  for (int i = 0; i < kShapes; ++i) {
    const Tile& t = kTiles[i];
    // narrow tiles read the weights again for every column of tiles, from memory
    // where they are cold: four times at most
    if (i >= kNarrow32 && (!b_kc || N > 4 * t.n)) continue;
    if ((i == kThin16 && !a_kc) || ((i == kRow80 || i == kSlim80) && !f32) || (i == kWide && f32)) continue;
    const int64_t stages = ceil_div(K, (f32 ? 32 : 64) * t.depth);
    for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (splits > 1 && (whole || stages < 2 * splits || ceil_div(M, t.m) * ceil_div(N, t.n) * splits > 4 * cu)) break;
      const double us = time_of(t, f32, width, M, N, K, splits, cu);
      if (best.us == 0.0 || us < best.us) best = Plan{(Shape)i, splits, us};
    }
  }
  return best;
}

// search_plan(), remembered by its arguments: it takes microseconds, as long as
// a launch.  `whole`: no contraction may be shared by workgroups.
Plan plan_of(int dtype, int width, bool a_kc, bool b_kc, int64_t M, int64_t N, int64_t K, bool whole = false) {
  struct Entry {
    int64_t M = -1, N, K;
    int cu, kind;
    Plan plan;
  };
  static thread_local Entry known[256];
  if (M <= 0 || N <= 0) return Plan{kSquare2, 1, 0.0};
  const bool f32 = dtype == LINEAR_F32;
  const int cu = compute_units(), kind = width * 16 + whole * 8 + f32 * 4 + a_kc * 2 + b_kc;
  Entry& e = known[(uint64_t)(M * 0x9e3779b1 + N * 0x85ebca77 + K * 0xc2b2ae3d + kind) % 251];
  if (e.M != M || e.N != N || e.K != K || e.cu != cu || e.kind != kind)
    e = Entry{M, N, K, cu, kind, search_plan(f32, width, a_kc, b_kc, whole, M, N, K, cu)};
  return e.plan;
}

// The tile of the kernels that load through registers, and how often its
// contraction is split: until every compute unit has a workgroup, each with four
// stages at least; 16 times at most, but for a contraction of millions of values.
struct RegisterTile {
  int m, n, depth;
};
RegisterTile register_tile(bool b_kc, int64_t N) {
  return N > 64 ? RegisterTile{128, 128, 1} : b_kc && N <= 16 ? RegisterTile{64, 16, 4} : RegisterTile{64, 64, 4};
}

inline int register_splits(int dtype, bool b_kc, int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0) return 1;
  const RegisterTile t = register_tile(b_kc, N);
  const int64_t stages = ceil_div(K, t.depth * (dtype == LINEAR_F32 ? 32 : 64)), tiles = ceil_div(M, t.m) * ceil_div(N, t.n);
  return (int)std::max<int64_t>(1, std::min<int64_t>({compute_units() / tiles, stages / 4, K < 1 << 21 ? 16 : 256}));
}

int64_t padded(int dtype, int64_t n) { return dtype == LINEAR_F32 ? (n + 3) / 4 * 4 : (n + 7) / 8 * 8; }

// Values of an operand's padded copy.
int64_t copy_values(int dtype, bool kc, int64_t rows, int64_t K) { return kc ? rows * padded(dtype, K) : K * padded(dtype, rows); }

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// How operands reach LDS: directly where their lines are direct.  Through
// registers, with 64-bit addresses, where even a copy's lines would be too long for
// the direct loads (from 2^22 fp32 or 2^23 16-bit values on).  Else, for few
// columns of 16-bit types, through registers (a copy would triple what is read of
// an operand that is read about once); for fp32 by loads of single values, from
// any address, where the figures above say that this is faster than a padded
// copy (not without `single`: those kernels do not exist for every end); else from
// padded copies.
struct Route {
  int width;              // bytes of a direct load; 0 = through registers
  bool copy_a, copy_b;
};

Route route_of(int dtype, bool a_kc, bool b_kc, Lines a, Lines b, int64_t M, int64_t N, int64_t K, bool single = true) {
  const Route copied{16, a != Lines::kDirect, b != Lines::kDirect};
  if (!copied.copy_a && !copied.copy_b) return copied;
  auto long_lines = [&](int64_t len) { return lines_of(dtype, nullptr, padded(dtype, len), padded(dtype, len)) == Lines::kFar; };
  if (long_lines(a_kc ? K : M) || long_lines(b_kc ? K : N)) return Route{0, false, false};
  if (single && dtype == LINEAR_F32 && a != Lines::kFar && b != Lines::kFar) {
    const int64_t values = (copied.copy_a ? copy_values(dtype, a_kc, M, K) : 0) + (copied.copy_b ? copy_values(dtype, b_kc, N, K) : 0);
    const double copy = 5.0 + 2.0 * 4.0 * values / kRates32.read;
    if (plan_of(dtype, 4, a_kc, b_kc, M, N, K).us < plan_of(dtype, 16, a_kc, b_kc, M, N, K).us + copy) return Route{4, false, false};
  }
  if (b_kc && N <= 64) return Route{0, false, false};
  return copied;
}

// Puts the padded copies that the route wants at `ws` and makes them the product's
// operands; `ws` is then what follows them.
template <class T> hipError_t copy_operands(int dtype, const Route& r, bool a_kc, bool b_kc, Product& p, char*& ws, hipStream_t s) {
  if (!r.copy_a && !r.copy_b) return hipSuccess;
  Copy c[2];
  int n = 0;
  if (r.copy_a) {
    c[n++] = Copy{p.A, ws, p.lda, padded(dtype, a_kc ? p.K : p.M), a_kc ? p.M : p.K, a_kc ? p.K : p.M};
    p.A = ws;
    p.lda = c[0].to_ld;
    (a_kc ? p.aK : p.arows) = (int)p.lda;
    ws += up256(copy_values(dtype, a_kc, p.M, p.K) * (int)sizeof(T));
  }
  if (r.copy_b) {
    c[n++] = Copy{p.B, ws, p.ldb, padded(dtype, b_kc ? p.K : p.N), b_kc ? p.N : p.K, b_kc ? p.K : p.N};
    p.B = ws;
    p.ldb = c[n - 1].to_ld;
    (b_kc ? p.bK : p.brows) = (int)p.ldb;
    ws += up256(copy_values(dtype, b_kc, p.N, p.K) * (int)sizeof(T));
  }
  auto blocks = [](const Copy& x) { return (int)std::min<int64_t>((x.lines * (x.to_ld / kVec<T>) + 255) / 256, 4096); };
  const int first = blocks(c[0]), second = n > 1 ? blocks(c[1]) : 0;
  if (first + second == 0) return hipSuccess;
  pad_kernel<T><<<dim3((unsigned)(first + second)), 256, 0, s>>>(c[0], c[n - 1], first);
  return hipGetLastError();
}

// Extents of operands that are loaded as they are.
inline void set_extents(Product& p) {
  if (p.arows == 0) p.arows = p.M;
  if (p.brows == 0) p.brows = p.N;
  if (p.aK == 0) p.aK = p.K;
  if (p.bK == 0) p.bK = p.K;
}

inline void true_extents(Product& p) {
  p.arows = p.M;
  p.brows = p.N;
  p.aK = p.bK = p.K;
}

}  // namespace
}  // namespace linear
