// k_linear_tc.cuh -- matrix products of 16-bit operands on the tensor cores,
// with the linear layer's epilogue (include/pic_linear.h).
//
// C[i][j] = sum_k A(i, k) B(j, k): a CTA (CG = 1) or a pair of CTAs (CG = 2)
// computes tiles of CG x 128 rows and BN columns, one after another, in fp32
// accumulators in tensor memory.  Three kinds of warps work side by side:
//   warp 0      one thread keeps a ring of STAGES slices of A and B (64 of K)
//               filled by TMA; what lies outside the matrices reads as zero
//   warp 1      one thread issues the MMAs, 16 of K each
//   the others  the epilogue (8 warps, 4 for 64 columns): accumulators, bias, pre,
//               activation, residual, rounding, and out through shared memory: by
//               TMA where rows start and end on 16-byte boundaries, in one run
//               where narrow rows lie end to end, else by plain stores
// There are two sets of accumulators, so that a tile's epilogue runs under the
// next tile's MMAs.  A tensor core truncates when it adds to an accumulator, so one is
// taken over after 1024 additions, 16384 of K (at most 2^-13 is lost of a sum of terms of
// one sign, 6e-5 on average): over longer K the epilogue warps add what they take over to
// sums of the CTA's own in the workspace, to nearest, under the next MMAs.  An operand may be contiguous along K or along its rows
// (dz and x in dw = dz^T x): TMA then brings blocks of 64 rows x 64 of K and
// the MMA reads them transposed.  A product that has fewer tiles than the GPU
// has SMs is cut along K: each part's accumulators go to the workspace in fp32,
// and a second kernel adds the parts in order and runs the epilogue.
//
// Measured: bf16 4096 x 4096 -> 16384 GELU with pairs of CTAs and 256 columns 287 us,
// 1.92 PFLOP/s, what a plain library product does in a burst; the tensor pipe is busy
// 89 % of the time.  fp16 24 x 4096 -> 16384 28 us: 134 MB of weights at 4.8 TB/s, over
// the 128 tiles that there are.
//
// Each wait is bounded: a thread whose wait runs out raises its CTA's abort
// flag and the status word, and every role skips what is left.
#pragma once

#include "linear.cuh"
#include "linear_ptx.cuh"

namespace pic {
namespace lin {

struct TcMaps {
  CUtensorMap a, b, y, pre;
};

struct TcParams {
  Product p;             // K in elements; a and b only through the maps
  long long tiles_i, tiles_j;
  long long work;        // tiles x splits
  int splits;
  int k_blocks;          // slices of 64 in all of K
  int part_blocks;       // slices of one part
  int a_mn, b_mn;        // the operand is contiguous along its rows
  int store_tma;         // y (and pre) go out by TMA
  float* parts;          // fp32 parts, or null: the epilogue runs in the kernel
  float* carry;          // [CTAs][128][BN] sums so far, for kernels of long parts
  Waits waits;
};

constexpr int kSlice = 64;           // K of one stage
constexpr int kPanelBytes = 32 * 128;  // 32 rows x 64 columns of a 16-bit type
constexpr int kTcTakeover = 256;     // slices that stay in an accumulator
constexpr int kGroupRows = 2048;     // rows of A that neighbouring tiles share the columns of B for

// At most limit polls; false (with the flags raised) if the phase does not
// complete in time or another thread has given up.
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, volatile int* abort_flag, const Waits& w) {
  if (tc::mbar_test_wait(bar, parity)) return true;
  for (uint32_t i = 0; i < w.spin_limit; ++i) {
    if (tc::mbar_try_wait(bar, parity)) return true;
    if ((i & 63u) == 63u) {
      if (*abort_flag) return false;
      if (i > 4096) __nanosleep(64);
    }
  }
  *abort_flag = 1;
  atomicOr(w.status, 1);
  return false;
}
// After an abort: until what this CTA has started completes, for as long as a wait
// at most.  The MMAs that the calling thread has issued:
template <int CG>
__device__ __forceinline__ void drain_mmas(uint32_t bar_drain, const Waits& w) {
  tc::mma_commit_cg<CG>(bar_drain);
  for (uint32_t i = 0; i < w.spin_limit && !tc::mbar_try_wait(bar_drain, 0); ++i) {
  }
}
// TMA loads: the last of a ring of `stages`, the next of which would go to stage s
// in phase `phase` (a stage that was never filled is passed at once).
__device__ __forceinline__ void drain_loads(uint32_t bar_full, int stages, int s, uint32_t phase, const Waits& w) {
  for (int k = 0; k < stages; ++k) {
    if (--s < 0) s = stages - 1, phase ^= 1;
    for (uint32_t i = 0; i < w.spin_limit && !tc::mbar_try_wait(bar_full + 8 * s, phase); ++i) {
    }
  }
}

template <int CG, int BN>
struct TcShape {
  static constexpr int kRows = 128 * CG;
  static constexpr int kBRows = BN / CG;  // rows of B that one CTA holds
  static constexpr int kABytes = 128 * 128, kBBytes = kBRows * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  // BN = 64: two CTAs on an SM, else one
  static constexpr int kStages = BN == 256 ? 6 : BN == 128 ? 5 : 3;
  // Epilogue warps: 32 rows and BN, or half of BN, columns each.  With four, a
  // tile of 128 x 128 that also writes pre took 5 us, longer than its slices up to
  // K = 1536.
  static constexpr int kEpi = BN == 64 ? 4 : 8;
  static constexpr int kThreads = 64 + 32 * kEpi;
  static constexpr int kColumns = BN == 64 ? 64 : BN / 2;
  static constexpr int kPanels = BN == 64 ? 2 : 1;  // buffers of a warp
  static constexpr int kOffPanels = kStages * kStageBytes;
  static constexpr int kOffBars = kOffPanels + kEpi * kPanels * kPanelBytes;
  static constexpr int kBars = 2 * kStages + 4 + 1;
  static constexpr int kSmem = kOffBars + kBars * 8 + 16 + 1024;  // 1024: the base is rounded up
  static constexpr int kTmemCols = 2 * BN;
};

// Row and column tile of tile t: groups of kGroupRows rows, columns outermost
// within a group, so that the group's rows of A and one column block of B stay in L2.
template <int ROWS>
__device__ __forceinline__ void tile_place(long long t, long long tiles_i, long long tiles_j, long long& ti,
                                           long long& tj) {
  constexpr int G = kGroupRows / ROWS;
  const long long group = t / (G * tiles_j), first = group * G;
  const long long size = min(static_cast<long long>(G), tiles_i - first);
  const long long in = t - group * G * tiles_j;
  ti = first + in % size;
  tj = in / size;
}

template <typename T>
__device__ __forceinline__ uint32_t idesc_of(int M, int N, bool a_mn, bool b_mn) {
  return tc::idesc_16(M, N, !std::is_same<T, __half>::value, a_mn, b_mn);
}

// Word `i` of row r of a panel buffer.
__device__ __forceinline__ uint32_t panel_at(uint32_t buf, int r, int i) {
  return buf + r * 128 + (((i >> 2) ^ (r & 7)) * 16) + (i & 3) * 4;
}
__device__ __forceinline__ uint32_t panel_word(uint32_t buf, int r, int i) {
  uint32_t w;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(panel_at(buf, r, i)) : "memory");
  return w;
}
// Whether every row of a matrix starts on a 16-byte boundary from column col0 on.
template <typename T>
__device__ __forceinline__ bool rows_on16(const void* m, long long ld, long long col0) {
  return ((reinterpret_cast<uintptr_t>(m) + col0 * sizeof(T)) | static_cast<uintptr_t>(ld * sizeof(T))) % 16 == 0;
}

// Whether 32 rows of a matrix from a multiple of 32 on are one run of memory on a
// 16-byte boundary: narrow rows without gaps, whatever their width.
template <typename T>
__device__ __forceinline__ bool packed_rows(const void* m, long long ld, const Product& p) {
  return ld == p.J && p.J <= 128 / static_cast<int>(sizeof(T)) && reinterpret_cast<uintptr_t>(m) % 16 == 0;
}

// One warp's panel (32 rows from row0, 128 bytes of columns from col0; this
// lane's row in v) to global memory: into the panel buffer, swizzled as TMA and
// the banks like it, then one TMA store, or one word of a row per lane and row.
template <typename T>
__device__ __forceinline__ void put_panel(const uint32_t (&v)[32], uint32_t buf, int lane, long long row0, long long col0,
                                          const Product& p, void* out, long long ld, const CUtensorMap* map,
                                          bool by_tma) {
  if (!by_tma && row0 + 32 <= p.I && packed_rows<T>(out, ld, p)) {
    // as the rows lie in memory, and out in one copy
    const int n = static_cast<int>(p.J);
    const uint32_t row = buf + lane * n * sizeof(T);
    if (sizeof(T) == 4 || n % 2 == 0) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c * static_cast<int>(4 / sizeof(T)) < n) asm volatile("st.shared.b32 [%0], %1;" ::"r"(row + 4 * c), "r"(v[c]) : "memory");
    } else {
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        if (2 * c < n) asm volatile("st.shared.u16 [%0], %1;" ::"r"(row + 4 * c), "h"(static_cast<uint16_t>(v[c])) : "memory");
        if (2 * c + 1 < n)
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(row + 4 * c + 2), "h"(static_cast<uint16_t>(v[c] >> 16)) : "memory");
      }
    }
    tc::fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tc::bulk_store(static_cast<T*>(out) + row0 * n, buf, 32 * n * sizeof(T));
      tc::bulk_commit();
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 8; ++c)
    tc::sts128(buf + lane * 128 + ((c ^ (lane & 7)) * 16), v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
  if (by_tma) {
    tc::fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tc::tma_store_2d(map, static_cast<int>(col0), static_cast<int>(row0), buf);
      tc::bulk_commit();
    }
    return;
  }
  __syncwarp();
  const int n = static_cast<int>(min(static_cast<long long>(128 / sizeof(T)), p.J - col0));  // columns that exist
  const int rows = static_cast<int>(min(32LL, p.I - row0));
  T* o = static_cast<T*>(out) + row0 * ld + col0;
#pragma unroll 8
  for (int r = 0; r < rows; ++r, o += ld) {
    const uint32_t w = panel_word(buf, r, lane);
    if constexpr (sizeof(T) == 4) {
      if (lane < n) reinterpret_cast<uint32_t*>(o)[lane] = w;
    } else {
      // words of two columns where the row's words lie: columns 2 l, 2 l + 1, or
      // 2 l + 1, 2 l + 2 of a row that starts in the middle of one
      uint16_t* h = reinterpret_cast<uint16_t*>(o) + 2 * lane;
      if ((reinterpret_cast<uintptr_t>(o) & 2) == 0) {
        if (2 * lane + 1 < n)
          *reinterpret_cast<uint32_t*>(h) = w;
        else if (2 * lane < n)
          h[0] = static_cast<uint16_t>(w);
      } else {
        const uint32_t next = __shfl_down_sync(0xffffffffu, w, 1);
        if (lane == 0) h[0] = static_cast<uint16_t>(w);
        if (lane < 31 && 2 * lane + 2 < n)
          *reinterpret_cast<uint32_t*>(h + 1) = w >> 16 | next << 16;
        else if (2 * lane + 1 < n)
          h[1] = static_cast<uint16_t>(w >> 16);
      }
    }
  }
  __syncwarp();
  if (lane == 0) tc::bulk_commit();  // an empty group: every panel has one, so that waits can count them
}

// 64 columns of a warp's 32 rows of a residual of a 16-bit type, loaded before they are
// wanted: where rows lie on 16-byte boundaries each lane has its own row's; where
// the rows are one run of memory, 16 bytes here and there of it; else word `lane`
// of every row.
template <typename T>
struct Residual {
  static constexpr int kCols = 64;
  uint32_t w[32];
  int mode;  // 0: this lane's row, 1: a run, 2: a word of every row
  int n;     // columns that exist

  __device__ __forceinline__ void load(const Product& p, long long row0, long long col0, int lane) {
    n = static_cast<int>(min(static_cast<long long>(kCols), p.J - col0));
    const int rows = static_cast<int>(min(32LL, p.I - row0));
    const T* o = static_cast<const T*>(p.residual) + row0 * p.ldr + col0;
    mode = n == kCols && rows_on16<T>(p.residual, p.ldr, col0) ? 0 : rows == 32 && packed_rows<T>(p.residual, p.ldr, p) ? 1 : 2;
    if (mode == 0) {
      const uint4* v = reinterpret_cast<const uint4*>(o + lane * p.ldr);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 q = lane < rows ? v[c] : make_uint4(0, 0, 0, 0);
        w[4 * c] = q.x, w[4 * c + 1] = q.y, w[4 * c + 2] = q.z, w[4 * c + 3] = q.w;
      }
    } else if (mode == 1) {
      const uint4* v = reinterpret_cast<const uint4*>(o);
      const int count = 32 * n * static_cast<int>(sizeof(T)) / 16;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 q = c * 32 + lane < count ? v[c * 32 + lane] : make_uint4(0, 0, 0, 0);
        w[4 * c] = q.x, w[4 * c + 1] = q.y, w[4 * c + 2] = q.z, w[4 * c + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int half = 0; half < 32; half += 16) {
        uint32_t high[16];
#pragma unroll
        for (int r = 0; r < 16; ++r, o += p.ldr) {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(o) + 2 * lane;
          w[half + r] = load_if(h, half + r < rows && 2 * lane < n);
          high[r] = load_if(h + 1, half + r < rows && 2 * lane + 1 < n);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) w[half + r] |= high[r] << 16;
      }
    }
  }
  // adds this lane's row to v, through the panel buffer where it has to be turned
  __device__ __forceinline__ void add(float* v, uint32_t buf, int lane) {
    if (mode == 1) {
      __syncwarp();
#pragma unroll
      for (int c = 0; c < 8; ++c)
        tc::sts128(buf + (c * 32 + lane) * 16, w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
      __syncwarp();
      const uint32_t row = buf + lane * n * sizeof(T);
      if (n % 2 == 0) {
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          w[c] = 0;
          if (2 * c < n) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[c]) : "r"(row + 4 * c) : "memory");
        }
      } else {
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          uint16_t lo = 0, hi = 0;
          if (2 * c < n) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(lo) : "r"(row + 4 * c) : "memory");
          if (2 * c + 1 < n) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(hi) : "r"(row + 4 * c + 2) : "memory");
          w[c] = lo | static_cast<uint32_t>(hi) << 16;
        }
      }
      __syncwarp();
    } else if (mode == 2) {
      __syncwarp();
#pragma unroll
      for (int r = 0; r < 32; ++r)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(panel_at(buf, r, lane)), "r"(w[r]) : "memory");
      __syncwarp();
#pragma unroll
      for (int c = 0; c < 8; ++c)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4 * c]), "=r"(w[4 * c + 1]), "=r"(w[4 * c + 2]), "=r"(w[4 * c + 3])
                     : "r"(buf + lane * 128 + ((c ^ (lane & 7)) * 16))
                     : "memory");
      __syncwarp();
    }
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      const float2 f = unpack2_of<T>(w[c]);
      v[2 * c] += f.x;
      v[2 * c + 1] += f.y;
    }
  }
};

// Adds 64 columns (or those of them that exist) of the bias to v.
template <typename T>
__device__ __forceinline__ void add_row(float (&v)[64], const T* r, int cols) {
  if (cols >= 64 && (reinterpret_cast<uintptr_t>(r) & 15) == 0) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint4 q = *reinterpret_cast<const uint4*>(r + 8 * c);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack2_of<T>(w[e]);
        v[8 * c + 2 * e] += f.x;
        v[8 * c + 2 * e + 1] += f.y;
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < 64; ++c)
      if (c < cols) v[c] += to_f32(r[c]);
  }
}

// The fp32 epilogue of a warp's 32 rows x 64 columns of sums, a row in each lane's v:
// they are turned in shared memory (kTurnBytes), and then the lanes walk down the
// columns, so that every load and store is a run of 128 bytes whatever the strides.
// A warp or two of an SM's quarter do this for every tile, so it counts instructions:
// pointers move by a row, whole tiles ask for no row's existence, and a column of a
// residual's 32 loads are under way together.
constexpr int kTurnStride = 33;  // floats, 32 columns at a time: no bank conflicts either way
constexpr int kTurnBytes = 32 * kTurnStride * 4;

// One column (of every lane) down the rows.
template <bool WHOLE>
__device__ __forceinline__ void finish_column(const Product& p, const float* turn, int c, long long row0, long long col,
                                              int rows, const float (&q)[32]) {
  const float bias = p.bias ? static_cast<const float*>(p.bias)[col] : 0.0f;
  float* pre = p.pre ? static_cast<float*>(p.pre) + row0 * p.ldpre + col : nullptr;
  float* y = static_cast<float*>(p.y) + row0 * p.ldy + col;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += 8) {
    if (!WHOLE && r0 >= rows) break;
    float z[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) z[u] = turn[(r0 + u) * kTurnStride + c] + bias;
    if (pre) {
#pragma unroll
      for (int u = 0; u < 8; ++u, pre += p.ldpre)
        if (WHOLE || r0 + u < rows) *pre = z[u];
    }
    if (p.act == PIC_ACT_RELU) {
#pragma unroll
      for (int u = 0; u < 8; ++u) z[u] = relu_nan(z[u]);
    } else if (p.act == PIC_ACT_GELU) {
#pragma unroll
      for (int u = 0; u < 8; u += 2) {
        const float2 y = gelu2<true>(make_float2(z[u], z[u + 1]));
        z[u] = y.x, z[u + 1] = y.y;
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u, y += p.ldy)
      if (WHOLE || r0 + u < rows) *y = z[u] + q[r0 + u];
  }
}

__device__ __forceinline__ void finish_rows(const float (&v)[64], const Product& p, float* turn, int lane, long long row0,
                                            long long col0) {
  const int rows = static_cast<int>(min(32LL, p.I - row0));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (col0 + 32 * h >= p.J) break;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 32; ++c) turn[lane * kTurnStride + c] = v[32 * h + c];
    __syncwarp();
    const long long col = col0 + 32 * h + lane;
    if (col >= p.J) continue;
    float q[32] = {};
    if (p.residual) {
      const float* res = static_cast<const float*>(p.residual) + row0 * p.ldr + col;
#pragma unroll
      for (int r = 0; r < 32; ++r, res += p.ldr) q[r] = __uint_as_float(load_if(reinterpret_cast<const uint32_t*>(res), r < rows));
    }
    if (rows == 32)
      finish_column<true>(p, turn, lane, row0, col, rows, q);
    else
      finish_column<false>(p, turn, lane, row0, col, rows, q);
  }
}

// The same of a swapped product: a lane's row is a column of y, and neighbouring lanes'
// are neighbours.
__device__ __forceinline__ void finish_swapped(const float (&v)[64], const Product& p, int lane, long long row0,
                                               long long col0) {
  const long long i = row0 + lane;
  if (i >= p.I) return;
  const int cols = static_cast<int>(min(64LL, p.J - col0));
  const float bias = p.bias ? static_cast<const float*>(p.bias)[i] : 0.0f;
#pragma unroll
  for (int c0 = 0; c0 < 64; c0 += 8) {
    if (c0 >= cols) break;
    float q[8] = {};
    if (p.residual) {
      const uint32_t* res = static_cast<const uint32_t*>(p.residual) + (col0 + c0) * p.ldr + i;
#pragma unroll
      for (int u = 0; u < 8; ++u, res += p.ldr) q[u] = __uint_as_float(load_if(res, c0 + u < cols));
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (c0 + u >= cols) break;
      const long long j = col0 + c0 + u;
      const float z = v[c0 + u] + bias;
      if (p.pre) static_cast<float*>(p.pre)[j * p.ldpre + i] = z;
      static_cast<float*>(p.y)[j * p.ldy + i] = act_value<true>(z, p.act) + q[u];
    }
  }
}

// A product cut along K: a tile's parts are [rank][panel][quarter][16][32 rows][4
// columns] of fp32 each; an item is four columns of a row, and neighbouring items
// are neighbouring columns.
struct JoinItem {
  long long i, j;
  int at;  // in a part, in float4
};
template <int ROWS>
__device__ __forceinline__ JoinItem join_place(int in, int bn, long long ti, long long tj) {
  const int c4 = in & 15, row = in >> 4 & 31, quarter = in >> 9 & 3, rest = in >> 11;
  const int panel = rest % (bn / 64), rank = rest / (bn / 64);
  return {ti * ROWS + rank * 128 + quarter * 32 + row, tj * bn + panel * 64 + c4 * 4,
          rest << 11 | quarter << 9 | c4 << 5 | row};
}

// The epilogue of an item's sums.
template <typename T>
__device__ __forceinline__ void finish_item(const Product& p, const JoinItem& m, const float4& sum) {
  const float v[4] = {sum.x, sum.y, sum.z, sum.w};
  if constexpr (sizeof(T) == 4) {
    if (p.swapped) {
      const float b = p.bias ? static_cast<const float*>(p.bias)[m.i] : 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const long long j = m.j + c;
        if (j >= p.J) break;
        if (p.pre) static_cast<float*>(p.pre)[j * p.ldpre + m.i] = v[c] + b;
        float z = act_value<true>(v[c] + b, p.act);
        if (p.residual) z += static_cast<const float*>(p.residual)[j * p.ldr + m.i];
        static_cast<float*>(p.y)[j * p.ldy + m.i] = z;
      }
      return;
    }
  }
  T y[4], pre[4];
  const int cols = static_cast<int>(min(4LL, p.J - m.j));
  struct alignas(4 * sizeof(T)) Four {
    T t[4];
  };
  const T* bias = static_cast<const T*>(p.bias) + m.j;
  const T* res = static_cast<const T*>(p.residual) + m.i * p.ldr + m.j;
  Four b{}, r{};
  if (p.bias) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c < cols) b.t[c] = bias[c];
  }
  if (p.residual) {
    if (cols == 4 && reinterpret_cast<uintptr_t>(res) % sizeof(Four) == 0) {
      r = *reinterpret_cast<const Four*>(res);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < cols) r.t[c] = res[c];
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    float z = v[c];
    if (p.bias) z += to_f32(b.t[c]);
    pre[c] = from_f32<T>(z);
    z = act_value<sizeof(T) == 4>(z, p.act);
    if (p.residual) z += to_f32(r.t[c]);
    y[c] = from_f32<T>(z);
  }
  const auto put = [&](void* out, long long ld, const T (&t)[4]) {
    T* o = static_cast<T*>(out) + m.i * ld + m.j;
    if (cols == 4 && reinterpret_cast<uintptr_t>(o) % sizeof(Four) == 0) {
      *reinterpret_cast<Four*>(o) = {t[0], t[1], t[2], t[3]};
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < cols) o[c] = t[c];
    }
  };
  if (p.pre) put(p.pre, p.ldpre, pre);
  put(p.y, p.ldy, y);
}

// a[0..3], bits of floats, plus f.
__device__ __forceinline__ void add4(uint32_t* a, const float4& f) {
  a[0] = __float_as_uint(__uint_as_float(a[0]) + f.x);
  a[1] = __float_as_uint(__uint_as_float(a[1]) + f.y);
  a[2] = __float_as_uint(__uint_as_float(a[2]) + f.z);
  a[3] = __float_as_uint(__uint_as_float(a[3]) + f.w);
}

// A tile with more K than stays in an accumulator: an epilogue warp takes the
// accumulators over `n` times and sums them up in `sums` (panels of [16][32 lanes] x 4
// columns, each lane's its own); the tile's last ones it adds where they are, in tensor
// memory, for the usual path to find.  A function of its own, so that it takes no
// registers from that path; false after an abort.
struct Carry {
  float4* sums;
  uint32_t tmem, bar_acc, lead_free;
  int from, to, n, lane;
  bool withhold;
  volatile int* abort_flag;
};
template <int CG, int BN>
__device__ __noinline__ bool carry_sums(const Carry& m, const Waits& waits, int buf, uint32_t phase) {
  for (int t = 0; m.n > 0 && t <= m.n; ++t) {
    if (!__all_sync(0xffffffffu, wait_bounded(m.bar_acc + 8 * buf, phase, m.abort_flag, waits))) return false;
    tc::tc_fence_after();
    for (int c0 = m.from; c0 < m.to; c0 += 64) {
      const uint32_t at = m.tmem + buf * BN + c0;
      uint32_t r[64];
      tc::tmem_ld64_wait(at, r);
      if (t < m.n && c0 + 64 == m.to) {
        tc::tc_fence_before();
        __syncwarp();
        if (m.lane == 0 && !m.withhold) {
          if constexpr (CG == 2)
            tc::mbar_arrive_cluster(m.lead_free + 8 * buf);
          else
            tc::mbar_arrive(m.lead_free + 8 * buf);
        }
      }
      float4* o = m.sums + c0 / 64 * (128 * 16);
      if (t > 0) {
#pragma unroll
        for (int c = 0; c < 16; ++c) add4(r + 4 * c, o[c * 32]);
      }
      if (t < m.n) {
#pragma unroll
        for (int c = 0; c < 16; ++c)
          o[c * 32] = make_float4(__uint_as_float(r[4 * c]), __uint_as_float(r[4 * c + 1]), __uint_as_float(r[4 * c + 2]),
                                  __uint_as_float(r[4 * c + 3]));
      } else {
#pragma unroll
        for (int c = 0; c < 64; c += 16) tc::tmem_st16(at + c, r + c);
        tc::tmem_st_wait();
      }
    }
    if (++buf == 2) buf = 0, phase ^= 1;
  }
  return true;
}

// LONG: parts with more than kTcTakeover slices.  (In one kernel with the others, 4096 x
// 512 -> 4096 with residual took 36.8 us instead of 35.6.)
template <typename T, int CG, int BN, bool LONG>
__global__ void __launch_bounds__(TcShape<CG, BN>::kThreads, BN == 64 ? 2 : 1)
    tc_kernel(const __grid_constant__ TcParams q, const __grid_constant__ TcMaps maps) {
  using S = TcShape<CG, BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0;
  const uint32_t bars = base + S::kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * S::kStages, bar_acc = bar_empty + 8 * S::kStages,
                 bar_free = bar_acc + 16, bar_drain = bar_free + 16;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::kOffBars + 8 * S::kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kOffBars + 8 * S::kBars + 4);

  if (threadIdx.x == 0) {
    tc::prefetch_map(&maps.a);
    tc::prefetch_map(&maps.b);
    for (int s = 0; s < S::kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, 1);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(bar_acc + 8 * b, 1);
      tc::mbar_init(bar_free + 8 * b, S::kEpi * CG);
    }
    tc::mbar_init(bar_drain, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) tc::tmem_alloc_cg<CG>(tc::smem_addr(tmem_slot), S::kTmemCols);
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  auto wait = [&](uint32_t bar, uint32_t parity) { return wait_bounded(bar, parity, abort_flag, q.waits); };
  const long long first = blockIdx.x / CG, step = gridDim.x / CG;
  // slices of work item w
  auto part = [&](long long w, int& k0, int& k1) {
    k0 = static_cast<int>(w % q.splits) * q.part_blocks;
    k1 = min(q.k_blocks, k0 + q.part_blocks);
  };

  // the TMA and the MMA thread's place in the ring of stages.  elect_one picks the
  // same lane each time; asked in the branch itself, it lets the compiler know that
  // one thread is there (with a flag set before, 4096 x 4096 -> 16384 took 6 % longer)
  int s = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (warp == 0) {
    if (tc::elect_one()) {
      const uint32_t lead_full = CG == 2 ? tc::map_rank(bar_full, 0) : bar_full;
      for (long long w = first; w < q.work && ok; w += step) {
        long long ti, tj;
        tile_place<S::kRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
        const int i0 = static_cast<int>(ti * S::kRows + rank * 128), j0 = static_cast<int>(tj * BN + rank * S::kBRows);
        int k0, k1;
        part(w, k0, k1);
        for (int kb = k0; kb < k1; ++kb) {
          if (!(ok = wait(bar_empty + 8 * s, phase ^ 1))) break;
          if (rank == 0) tc::mbar_arrive_expect_tx(bar_full + 8 * s, CG * S::kStageBytes);
          const uint32_t sa = base + s * S::kStageBytes, sb = sa + S::kABytes, bar = lead_full + 8 * s;
          const int k = kb * kSlice;
          if (q.a_mn) {
#pragma unroll
            for (int c = 0; c < 2; ++c) tc::tma_load_2d<CG == 2>(sa + c * 8192, &maps.a, i0 + 64 * c, k, bar);
          } else {
            tc::tma_load_2d<CG == 2>(sa, &maps.a, k, i0, bar);
          }
          if (q.b_mn) {
#pragma unroll
            for (int c = 0; c < S::kBRows / 64; ++c)
              tc::tma_load_2d<CG == 2>(sb + c * 8192, &maps.b, j0 + 64 * c, k, bar);
          } else {
            tc::tma_load_2d<CG == 2>(sb, &maps.b, k, j0, bar);
          }
          if (++s == S::kStages) s = 0, phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && tc::elect_one()) {
      constexpr uint32_t kM = 128 * CG;
      const uint32_t idesc = idesc_of<T>(kM, BN, q.a_mn != 0, q.b_mn != 0);
      // one MMA takes 16 of K: 32 bytes of a K-major row, 16 rows of an MN-major block
      const uint32_t a_step = q.a_mn ? 2048 : 32, b_step = q.b_mn ? 2048 : 32;
      int buf = 0;
      uint32_t free_phase = 0;
      for (long long w = first; w < q.work && ok; w += step) {
        if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
        tc::tc_fence_after();
        int k0, k1;
        part(w, k0, k1);
        uint32_t d = tmem + buf * BN;
        for (int kb = k0, t1 = k0 + kTcTakeover; kb < k1; ++kb) {
          if (LONG && kb == t1) {
            tc::mma_commit_cg<CG>(bar_acc + 8 * buf);
            if (++buf == 2) buf = 0, free_phase ^= 1;
            if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
            tc::tc_fence_after();
            d = tmem + buf * BN;
            k0 = kb, t1 += kTcTakeover;
          }
          if (!(ok = wait(bar_full + 8 * s, phase))) break;
          tc::tc_fence_after();
          const uint32_t sa = base + s * S::kStageBytes, sb = sa + S::kABytes;
#pragma unroll
          for (int kk = 0; kk < kSlice / 16; ++kk)
            tc::mma_16<CG>(d, tc::smem_desc_sw128(sa + kk * a_step, 8192, 1024),
                           tc::smem_desc_sw128(sb + kk * b_step, 8192, 1024), idesc, (kb > k0 || kk > 0) ? 1u : 0u);
          tc::mma_commit_cg<CG>(bar_empty + 8 * s);
          if (++s == S::kStages) s = 0, phase ^= 1;
        }
        if (!ok) break;
        tc::mma_commit_cg<CG>(bar_acc + 8 * buf);
        if (++buf == 2) buf = 0, free_phase ^= 1;
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;  // the 32 lanes of tensor memory that this warp may read
    const Product& p = q.p;
    const int from = (warp - 2) / 4 * S::kColumns, to = from + S::kColumns;  // columns of the tile
    const uint32_t panels = base + S::kOffPanels + (warp - 2) * S::kPanels * kPanelBytes;
    const uint32_t lead_free = CG == 2 ? tc::map_rank(bar_free, 0) : bar_free;
    int buf = 0, pb = 0;
    for (long long w = first; w < q.work; w += step) {
      long long ti, tj;
      tile_place<S::kRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
      const long long row0 = ti * S::kRows + rank * 128 + quarter * 32, j0 = tj * BN;
      if constexpr (LONG) {
        int k0, k1;
        part(w, k0, k1);
        const Carry c{reinterpret_cast<float4*>(q.carry) + blockIdx.x * static_cast<long long>(128 * BN / 4) + quarter * (32 * 16) + lane,
                      tmem + (static_cast<uint32_t>(quarter * 32) << 16), bar_acc, lead_free, from, to, (k1 - k0 - 1) / kTcTakeover, lane,
                      q.waits.test_fault && w == 0 && rank == 0 && quarter == 0, abort_flag};
        if (!carry_sums<CG, BN>(c, q.waits, buf, phase)) break;
        buf += c.n;
        phase ^= buf >> 1 & 1, buf &= 1;
      }
      // tiles of 64 columns wait for memory: their residual is on its way before they
      // are summed (for larger tiles that would take registers that they need)
      Residual<T> res;
      constexpr bool kEarly = BN == 64;
      if (kEarly && p.residual && !q.parts && row0 < p.I && j0 < p.J) res.load(p, row0, j0, lane);
      if (!__all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase))) break;
      tc::tc_fence_after();
      const uint32_t d = tmem + buf * BN + (static_cast<uint32_t>(quarter * 32) << 16);
      for (int c0 = from; c0 < to; c0 += 64) {
        uint32_t raw_acc[64];
        tc::tmem_ld64_wait(d + c0, raw_acc);
        if (c0 + 64 == to) {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0 && !(q.waits.test_fault && w == 0 && rank == 0 && quarter == 0)) {
            if constexpr (CG == 2)
              tc::mbar_arrive_cluster(lead_free + 8 * buf);
            else
              tc::mbar_arrive(bar_free + 8 * buf);
          }
        }
        if (q.parts) {
          // part w, panel c0 / 64, this warp's 32 rows: [16][32 lanes][4 columns]
          float4* o = reinterpret_cast<float4*>(q.parts) +
                      ((w * CG + rank) * (BN / 64) + c0 / 64) * (128 * 16) + quarter * (32 * 16) + lane;
#pragma unroll
          for (int c = 0; c < 16; ++c)
            o[c * 32] = make_float4(__uint_as_float(raw_acc[4 * c]), __uint_as_float(raw_acc[4 * c + 1]),
                                    __uint_as_float(raw_acc[4 * c + 2]), __uint_as_float(raw_acc[4 * c + 3]));
          continue;
        }
        if (row0 >= p.I || j0 + c0 >= p.J) continue;  // nothing of this panel is inside
        float v[64];
#pragma unroll
        for (int c = 0; c < 64; ++c) v[c] = __uint_as_float(raw_acc[c]);
        const int cols = static_cast<int>(min(64LL, p.J - j0 - c0));
        if (p.bias) add_row<T>(v, static_cast<const T*>(p.bias) + j0 + c0, cols);
        uint32_t out[32];
        if (p.pre) {
#pragma unroll
          for (int c = 0; c < 32; ++c) out[c] = pack2_of<T>(v[2 * c], v[2 * c + 1]);
          if (lane == 0) tc::bulk_wait_read<S::kPanels - 1>();  // the buffer's last store has been read
          __syncwarp();
          put_panel<T>(out, panels + pb * kPanelBytes, lane, row0, j0 + c0, p, p.pre, p.ldpre, &maps.pre, q.store_tma);
          if (++pb == S::kPanels) pb = 0;
        }
        if (p.act == PIC_ACT_GELU) {
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            const float2 r = unpack2(gelu_approx2(pack2(v[c], v[c + 1])));
            v[c] = r.x;
            v[c + 1] = r.y;
          }
        } else if (p.act == PIC_ACT_RELU) {
#pragma unroll
          for (int c = 0; c < 64; ++c) v[c] = relu_nan(v[c]);
        }
        if (lane == 0) tc::bulk_wait_read<S::kPanels - 1>();
        __syncwarp();
        if (p.residual) {
          if (!kEarly) res.load(p, row0, j0 + c0, lane);
          res.add(v, panels + pb * kPanelBytes, lane);
        }
#pragma unroll
        for (int c = 0; c < 32; ++c) out[c] = pack2_of<T>(v[2 * c], v[2 * c + 1]);
        put_panel<T>(out, panels + pb * kPanelBytes, lane, row0, j0 + c0, p, p.y, p.ldy, &maps.y, q.store_tma);
        if (++pb == S::kPanels) pb = 0;
      }
      if (++buf == 2) buf = 0, phase ^= 1;
    }
    if (lane == 0) tc::bulk_wait_all();
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies and MMAs in flight use shared and tensor memory.  The other CTA of a
    // pair may have started copies that this one did not expect: it lingers for far
    // longer than a copy takes.
    if (warp == 0 && rank == 0 && tc::elect_one()) drain_loads(bar_full, S::kStages, s, phase, q.waits);
    if (warp == 1 && rank == 0 && tc::elect_one()) drain_mmas<CG>(bar_drain, q.waits);
    if (CG == 2) __nanosleep(200000);
    __syncthreads();
  }
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  if (warp == 1) tc::tmem_dealloc_cg<CG>(tmem, S::kTmemCols);
}

// A [rows][cols] matrix in boxes of 128 bytes of columns and box_rows rows,
// 128-byte swizzled; false if the driver will not make the map.
bool encode(CUtensorMap* map, const void* m, long long rows, long long cols, long long ld, int box_rows, int dtype);
// Allows a kernel `smem` bytes of shared memory, once per device; each kernel of
// these files has a slot of its own below kSmemSlots.
constexpr int kSmemSlots = 26;
int allow_smem(const void* fn, int slot, int smem);

// The kernel for tiles of bn columns: 64 and 128 by one CTA, 256 by a pair.
const void* tc_kernel_f16(int bn, bool long_parts);
const void* tc_kernel_bf16(int bn, bool long_parts);

template <typename T, bool LONG>
const void* tc_kernel_of(int bn) {
  if (bn == 256) return reinterpret_cast<const void*>(tc_kernel<T, 2, 256, LONG>);
  if (bn == 128) return reinterpret_cast<const void*>(tc_kernel<T, 1, 128, LONG>);
  return reinterpret_cast<const void*>(tc_kernel<T, 1, 64, LONG>);
}

}  // namespace lin
}  // namespace pic
