// k_linear_narrow.cu -- the whole gradient of a narrow layer (a hidden layer of a
// synthesis net, over the pixels of images) in one pass over the rows:
//
//   dz = dy act'(z),  dx = dz w,  dw += dz^T x,  db += dz
//
// Bound by memory: dy, z and x are read once and dx is written once, where
// separate products would write dz and read it twice.  A CTA stays on its SM and
// takes tiles of 128 rows.  One tile of dz in shared memory (64 columns to a row
// of 128 bytes, swizzled) is both operands: read along its rows it is A of
// dx = dz w, read across them A of dw = dz^T x.  dw stays in tensor memory from
// tile to tile; at the end each CTA writes its dw and db, and a small second kernel
// adds the CTAs' in order.  A tensor core truncates when it adds to an accumulator, so
// a CTA takes no more than kMostTiles tiles: 1024 additions, which lose at most 2^-13
// of a sum of terms of one sign (6e-5 on average), below the rounding of the output.
// From 2.5 million rows on there is more than one CTA for each SM, one after another.
//
// Up to 128 columns on each side for 16-bit types, 64 for fp32, whose values are
// cut into three bfloat16 pieces as in cut3.cuh (dw is then taken over into
// registers after every tile).
//
// Roles of the 16 warps: 0..3 dx out of tensor memory, 4 and 5 (fp32) take dw
// over, 6 issues the MMAs, 8..15 make dz and db.  Rows of 16-bit values on 16-byte
// boundaries, up to 64 of them, come by TMA (warp 7) into a ring of three tiles of
// dy, z and x, 48 KB each; x is an operand as it lands, and dz takes the place of
// dy.  Rows that lie end to end, whatever their width, are runs of memory: warp 7
// copies a tile's run of each matrix as it is, a tile or more ahead, and warps 8..15
// pick their elements out of it.  Else warps 8..15 load 4 x 16 bytes of dy, z and x per thread at a time, x of
// this tile under way while dz is computed, dy and z of the next while x is written
// to shared memory: any stride and alignment, but less in flight.
//
// Measured: fp16 393216 x 64 -> 64 ReLU 38.8 us for 201 MB, 5.2 TB/s, 78 % of the copy
// rate; fp32 65536 x 40 -> 40 GELU 29 us for 42 MB: there the chain of cutting,
// multiplying and taking over, one tile at a time, is what takes the time.
//
// An infinite or NaN value among fp32 pieces would spread (inf 0 = NaN): its tile
// is marked, and dx and dw of that tile are computed again on the FP32 cores.
#include "cut3.cuh"
#include "k_linear_tc.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kThreads = 512;
constexpr int kLoadWarp = 8, kLoaders = 256;
constexpr int kMmaWarp = 6, kTmaWarp = 7;
constexpr int kTile = 128;
constexpr int kMarks = 8;  // more tiles than the loaders can be ahead of the others
constexpr int kSms = 152;
constexpr int kMostTiles = 128;  // of a CTA, where dw stays in tensor memory

struct NarrowParams {
  NarrowGrad g;
  long long tiles;
  int vec_dy, vec_z, vec_x, store_tma;
  int raw_ring, raw_bytes;  // kRun: copies in flight, and the room of one
  int raw_z, raw_x;         // where z and x begin in it
  float* parts;  // [CTAs][N K + N]
  Waits waits;
};

// How dy, z and x arrive: through registers, by TMA, as runs of memory.
enum Source { kReg, kTma, kRun };
constexpr int kMaxRing = 4;

// T: element; WIDE: up to 128 columns (16-bit types), else 64.
template <typename T, bool WIDE, Source SRC>
struct Shape {
  static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kPer = 16 / sizeof(T);          // elements of a load
  static constexpr int kBlocks = WIDE ? 2 : 1;         // of 64 columns
  static constexpr int kCols = 64 * kBlocks;
  static constexpr int kVecs = kCols / kPer;           // loads of a row
  static constexpr int kPassRows = kLoaders / kVecs;   // rows that the loaders cover at once
  static constexpr int kUnitRows = 4 * kPassRows;      // rows of a unit: four loads of each matrix per thread
  static constexpr int kUnits = kTile / kUnitRows;
  static_assert(kUnits * kUnitRows == kTile, "whole units");
  static constexpr int kBlockBytes = kTile * 128;
  static constexpr int kPlaneBytes = kBlocks * kBlockBytes;
  static constexpr int kStageBytes = (SRC == kTma ? 3 : 2 * kPlanes) * kPlaneBytes;  // dz, x (and z)
  static constexpr int kStages = sizeof(T) == 4 ? 1 : SRC == kRun ? (WIDE ? 1 : 2) : WIDE ? 2 : SRC == kTma ? 3 : 4;
  static constexpr int kPanels = sizeof(T) == 4 && SRC == kRun ? 1 : 2;  // buffers of a dx warp
  static constexpr int kWBlock = kCols * 128, kWPlane = kBlocks * kWBlock;
  static constexpr int kOffW = kStages * kStageBytes;
  static constexpr int kOffPanels = kOffW + kPlanes * kWPlane;
  static constexpr int kOffSums = kOffPanels + 4 * kPanels * kPanelBytes;
  static constexpr int kOffBars = kOffSums + kLoaders * kPer * 4;
  // full, empty; landed, taken; dx ready, free; dw ready, free; drain
  static constexpr int kBars = 2 * kStages + 2 * kMaxRing + 4 + 4 + 1;
  static constexpr int kOffMarks = kOffBars + kBars * 8 + 8;
  static constexpr int kOffRaw = (kOffMarks + (kMarks + 1) * 4 + 127) / 128 * 128;
  static constexpr int kSmem = kOffRaw + 1024;  // 1024: the base is rounded up
  static constexpr int kTmemDw = 2 * kCols;  // columns: two buffers of dx, then dw (fp32: two)
  static constexpr int kTmemCols = WIDE ? 512 : 256;
};

template <typename T>
struct Vec16 {
  static constexpr int kPer = 16 / sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ void get(const T* p, int n, bool vec) {
    if (n >= kPer && vec) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
      return;
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = load_if(reinterpret_cast<const uint32_t*>(p) + i, i < n);
    } else {
      uint32_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = load_if(reinterpret_cast<const uint16_t*>(p) + i, i < n);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = e[2 * i] | e[2 * i + 1] << 16;
    }
  }
  // the same from an element of shared memory on
  __device__ __forceinline__ void get_shared(uint32_t at, int n) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = 0;
        if (i < n) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(at + 4 * i) : "memory");
      }
    } else {
      // the words that hold them; what they hold of others goes
      uint32_t h[5] = {};
      if (n > 0) {
#pragma unroll
        for (int i = 0; i < 5; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(h[i]) : "r"((at & ~3u) + 4 * i) : "memory");
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t v = (at & 2) ? __funnelshift_r(h[i], h[i + 1], 16) : h[i];
        w[i] = 2 * i + 1 < n ? v : 2 * i < n ? v & 0xffffu : 0u;
      }
    }
  }
  __device__ __forceinline__ void widen(float (&f)[kPer]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = __uint_as_float(w[i]);
      } else {
        const float2 v = unpack2_of<T>(w[i]);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
      }
    }
  }
};

// 16 bytes' worth of elements at (row, first column col) of a tile whose blocks of
// 64 columns are `block` bytes apart: one store, or three of half the size.
template <typename T>
__device__ __forceinline__ uint32_t put_vec(uint32_t tile, int block, int plane, int row, int col, const uint32_t (&w)[4]) {
  const uint32_t at = tile + (col >> 6) * block + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4);
  if constexpr (sizeof(T) == 4) {
    uint32_t h0, m0, l0, h1, m1, l1;
    cut3(w[0], w[1], h0, m0, l0);
    cut3(w[2], w[3], h1, m1, l1);
    const uint32_t a = at + (col & 4) * 2;
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(h0), "r"(h1) : "memory");
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a + plane), "r"(m0), "r"(m1) : "memory");
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a + 2 * plane), "r"(l0), "r"(l1) : "memory");
    return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
  } else {
    tc::sts128(at, w[0], w[1], w[2], w[3]);
    return 0;
  }
}

// d *= act'(v)
template <bool EXACT, int N>
__device__ __forceinline__ void times_act_grad(float (&d)[N], const float (&v)[N], int act) {
  if (act == PIC_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = v[e] > 0.0f ? d[e] : 0.0f;
  } else {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 r = act_grad2<EXACT>(make_float2(d[e], d[e + 1]), make_float2(v[e], v[e + 1]), PIC_ACT_GELU);
      d[e] = r.x;
      d[e + 1] = r.y;
    }
  }
}

__device__ __forceinline__ float dz_again(const NarrowGrad& g, long long i, int n) {
  const float d = static_cast<const float*>(g.dy)[i * g.lddy + n];
  return g.act == PIC_ACT_NONE ? d : act_grad<true>(d, static_cast<const float*>(g.pre)[i * g.ldpre + n], g.act);
}
// dx of a row, and a tile's part of a row of dw, on the FP32 cores (fp32 only).
__device__ __noinline__ void dx_again(float* v, const NarrowGrad& g, long long i) {
  for (int k = 0; k < 64; ++k) {
    float s = 0.0f;
    if (i < g.I && k < g.K)
      for (int n = 0; n < g.N; ++n) s = fmaf(dz_again(g, i, n), static_cast<const float*>(g.w)[n * g.ldw + k], s);
    v[k] = s;
  }
}
__device__ __noinline__ void dw_again(float* v, const NarrowGrad& g, long long i0, int n) {
  for (int k = 0; k < 64; ++k) {
    float s = 0.0f;
    if (n < g.N && k < g.K)
      for (long long i = i0; i < min(g.I, i0 + kTile); ++i)
        s = fmaf(dz_again(g, i, n), static_cast<const float*>(g.x)[i * g.ldx + k], s);
    v[k] = s;
  }
}

struct NarrowMaps {
  CUtensorMap dx, dy, z, x;
};

template <typename T, bool WIDE, Source SRC>
__global__ void __launch_bounds__(kThreads, 1)
    narrow_kernel(const __grid_constant__ NarrowParams q, const __grid_constant__ NarrowMaps maps) {
  using S = Shape<T, WIDE, SRC>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const NarrowGrad& g = q.g;
  const uint32_t bars = base + S::kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * S::kStages, bar_landed = bar_empty + 8 * S::kStages,
                 bar_taken = bar_landed + 8 * kMaxRing, bar_dx = bar_taken + 8 * kMaxRing,
                 bar_dx_free = bar_dx + 16, bar_dw = bar_dx_free + 16, bar_dw_free = bar_dw + 16, bar_drain = bar_dw_free + 16;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::kOffBars + 8 * S::kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kOffBars + 8 * S::kBars + 4);
  // mark t % kMarks holds t + 1 if this CTA's t-th tile has an infinite or NaN
  // operand; the last one is w's
  volatile int* marks = reinterpret_cast<volatile int*>(smem + S::kOffMarks);

  if (threadIdx.x == 0) {
    if (SRC == kTma) tc::prefetch_map(&maps.dy);
    for (int s = 0; s < S::kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, kLoaders / 32);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int r = 0; r < kMaxRing; ++r) {
      tc::mbar_init(bar_landed + 8 * r, 1);
      tc::mbar_init(bar_taken + 8 * r, kLoaders / 32);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(bar_dx + 8 * b, 1);
      tc::mbar_init(bar_dx_free + 8 * b, 4);
      tc::mbar_init(bar_dw + 8 * b, 1);
      tc::mbar_init(bar_dw_free + 8 * b, 2);
    }
    tc::mbar_init(bar_drain, 1);
    *abort_flag = 0;
    for (int m = 0; m <= kMarks; ++m) marks[m] = 0;
    tc::fence_mbar_init();
  }
  if (warp == kMmaWarp) tc::tmem_alloc_cg<1>(tc::smem_addr(tmem_slot), S::kTmemCols);
  __syncthreads();
  // w [N][K], zero to whole blocks
  if (g.dx) {
    uint32_t largest = 0;
    const bool vec = reinterpret_cast<uintptr_t>(g.w) % 16 == 0 && g.ldw % S::kPer == 0;
    for (int e = threadIdx.x; e < S::kCols * S::kVecs; e += kThreads) {
      const int row = e / S::kVecs, col = e % S::kVecs * S::kPer;
      Vec16<T> v;
      v.get(static_cast<const T*>(g.w) + row * g.ldw + col, row < g.N ? g.K - col : 0, vec);
      largest = max(largest, put_vec<T>(base + S::kOffW, S::kWBlock, S::kWPlane, row, col, v.w));
    }
    if (largest >= kCutLimit) marks[kMarks] = 1;
  }
  tc::fence_async_smem();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto wait = [&](uint32_t bar, uint32_t parity) { return wait_bounded(bar, parity, abort_flag, q.waits); };
  float* my_parts = q.parts + blockIdx.x * static_cast<long long>(g.N * g.K + g.N);

  // the TMA thread's place in the ring of stages
  int ring_s = 0;
  uint32_t ring_phase = 0;

  if (warp >= kLoadWarp) {
    const int tid = threadIdx.x - 32 * kLoadWarp;
    const int row = tid / S::kVecs, col = tid % S::kVecs * S::kPer;
    const T* dy = static_cast<const T*>(g.dy) + col;
    const T* z = static_cast<const T*>(g.pre) + col;
    const T* x = static_cast<const T*>(g.x) + col;
    const int n_dz = g.N - col, n_x = g.dw ? g.K - col : 0;
    const bool has_act = g.act != PIC_ACT_NONE;
    Vec16<T> vy[4], vz[4], vx[4];
    auto load_dz = [&](long long i0) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const long long i = i0 + row + u * S::kPassRows;
        vy[u].get(dy + i * g.lddy, i < g.I ? n_dz : 0, q.vec_dy);
        if (has_act) vz[u].get(z + i * g.ldpre, i < g.I ? n_dz : 0, q.vec_z);
      }
    };
    float sum[S::kPer] = {};
    int s = 0, count = 0;
    uint32_t phase = 0;
    if constexpr (SRC == kTma) {
      for (long long tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        if (!__all_sync(0xffffffffu, wait(bar_landed + 8 * s, phase))) break;
        const uint32_t sdz = base + s * S::kStageBytes, sz = sdz + 2 * S::kPlaneBytes;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = row + u * S::kPassRows;
          const uint32_t at = r * 128 + (((col >> 3) ^ (r & 7)) << 4);
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(vy[u].w[0]), "=r"(vy[u].w[1]), "=r"(vy[u].w[2]), "=r"(vy[u].w[3])
                       : "r"(sdz + at));
          if (has_act)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(vz[u].w[0]), "=r"(vz[u].w[1]), "=r"(vz[u].w[2]), "=r"(vz[u].w[3])
                         : "r"(sz + at));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float d[S::kPer], v[S::kPer];
          vy[u].widen(d);
          if (has_act) {
            vz[u].widen(v);
            times_act_grad<sizeof(T) == 4, S::kPer>(d, v, g.act);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2_of<T>(d[2 * i], d[2 * i + 1]);
            put_vec<T>(sdz, S::kBlockBytes, S::kPlaneBytes, row + u * S::kPassRows, col, w);
          }
#pragma unroll
          for (int e = 0; e < S::kPer; ++e) sum[e] += d[e];
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar_full + 8 * s);
        if (++s == S::kStages) s = 0, phase ^= 1;
      }
    } else {
    if (SRC == kReg && blockIdx.x < q.tiles) load_dz(blockIdx.x * static_cast<long long>(kTile));
    int raw = 0;
    uint32_t raw_phase = 0;
    for (long long tile = blockIdx.x; tile < q.tiles; tile += gridDim.x, ++count) {
      uint32_t largest = 0;
      bool ok = true;
      if (SRC == kRun && !__all_sync(0xffffffffu, wait(bar_landed + 8 * raw, raw_phase))) break;
#pragma unroll
      for (int unit = 0; unit < S::kUnits; ++unit) {
        const long long i0 = tile * kTile + unit * S::kUnitRows;
        if constexpr (SRC == kRun) {
          const uint32_t from = base + S::kOffRaw + raw * q.raw_bytes;
          constexpr int kElem = sizeof(T);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int r = unit * S::kUnitRows + row + u * S::kPassRows;
            const bool here = tile * kTile + r < g.I;
            vy[u].get_shared(from + (r * g.N + col) * kElem, here ? n_dz : 0);
            if (has_act) vz[u].get_shared(from + q.raw_z + (r * g.N + col) * kElem, here ? n_dz : 0);
            if (g.dw) vx[u].get_shared(from + q.raw_x + (r * g.K + col) * kElem, here ? n_x : 0);
          }
          if (unit + 1 == S::kUnits) {
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar_taken + 8 * raw);
            if (++raw == q.raw_ring) raw = 0, raw_phase ^= 1;
          }
        } else if (n_x > 0) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const long long i = i0 + row + u * S::kPassRows;
            vx[u].get(x + i * g.ldx, i < g.I ? n_x : 0, q.vec_x);
          }
        }
        // dz in the place of dy
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float d[S::kPer], v[S::kPer];
          vy[u].widen(d);
          if (has_act) {
            vz[u].widen(v);
            times_act_grad<sizeof(T) == 4, S::kPer>(d, v, g.act);
          }
#pragma unroll
          for (int e = 0; e < S::kPer; ++e) sum[e] += d[e];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4)
              vy[u].w[i] = __float_as_uint(d[i]);
            else
              vy[u].w[i] = pack2_of<T>(d[2 * i], d[2 * i + 1]);
          }
        }
        if (unit == 0) ok = __all_sync(0xffffffffu, wait(bar_empty + 8 * s, phase ^ 1));
        if (!ok) break;
        const uint32_t sdz = base + s * S::kStageBytes, sx = sdz + S::kPlanes * S::kPlaneBytes;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          largest = max(largest, put_vec<T>(sdz, S::kBlockBytes, S::kPlaneBytes, unit * S::kUnitRows + row + u * S::kPassRows, col, vy[u].w));
        if (SRC == kRun) {
        } else if (unit + 1 < S::kUnits)
          load_dz(i0 + S::kUnitRows);
        else if (tile + gridDim.x < q.tiles)
          load_dz((tile + gridDim.x) * kTile);
        if (g.dw) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (n_x <= 0) vx[u].w[0] = vx[u].w[1] = vx[u].w[2] = vx[u].w[3] = 0;
            largest = max(largest, put_vec<T>(sx, S::kBlockBytes, S::kPlaneBytes, unit * S::kUnitRows + row + u * S::kPassRows, col, vx[u].w));
          }
        }
      }
      if (!ok) break;
      if (largest >= kCutLimit) marks[count % kMarks] = count + 1;
      tc::fence_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar_full + 8 * s);
      if (++s == S::kStages) s = 0, phase ^= 1;
    }
    }
    // db: the threads of a column
    __syncwarp();
    if (g.db) {
      float* sums = reinterpret_cast<float*>(smem + S::kOffSums);
#pragma unroll
      for (int e = 0; e < S::kPer; ++e) sums[row * S::kCols + col + e] = sum[e];
      tc::named_bar(1, kLoaders);
      if (tid < g.N) {
        float t = 0.0f;
        for (int r = 0; r < S::kPassRows; ++r) t += sums[r * S::kCols + tid];
        my_parts[g.N * g.K + tid] = t;
      }
    }
  } else if (warp == kMmaWarp) {
    if (tc::elect_one()) {
      const int k_pad = (g.K + 15) / 16 * 16, n_steps = (g.N + 15) / 16;
      const uint32_t idesc_dx = idesc_of<T>(128, k_pad, false, true), idesc_dw = idesc_of<T>(128, k_pad, true, true);
      // of a dz of one block the MMA's rows 64..127 are rows 0..63 again, not looked at
      const uint32_t dz_lbo = WIDE && g.N > 64 ? S::kBlockBytes : 0;
      int s = 0, buf = 0;
      uint32_t phase = 0, free_phase = 0;
      bool ok = true, first = true;
      for (long long tile = blockIdx.x; tile < q.tiles && ok; tile += gridDim.x) {
        if (!(ok = wait(bar_full + 8 * s, phase) && (SRC != kTma || wait(bar_landed + 8 * s, phase)))) break;
        tc::tc_fence_after();
        const uint32_t sdz = base + s * S::kStageBytes, sx = sdz + S::kPlanes * S::kPlaneBytes, sw = base + S::kOffW;
        constexpr int kProducts = S::kPlanes == 3 ? 6 : 1;
        if (g.dx) {
          if (!(ok = wait(bar_dx_free + 8 * buf, free_phase ^ 1))) break;
          tc::tc_fence_after();
#pragma unroll
          for (int t = 0; t < kProducts; ++t) {
            const int pa = kProducts == 6 ? cut_a(t) : 0, pb = kProducts == 6 ? cut_b(t) : 0;
            for (int kk = 0; kk < n_steps; ++kk)
              tc::mma_16<1>(tmem + buf * S::kCols,
                            tc::smem_desc_sw128(sdz + pa * S::kPlaneBytes + (kk >> 2) * S::kBlockBytes + (kk & 3) * 32, 8192, 1024),
                            tc::smem_desc_sw128(sw + pb * S::kWPlane + kk * 2048, S::kWBlock, 1024), idesc_dx,
                            (t > 0 || kk > 0) ? 1u : 0u);
          }
          tc::mma_commit(bar_dx + 8 * buf);
        }
        if (g.dw) {
          const uint32_t d = tmem + S::kTmemDw + (S::kPlanes == 3 ? buf * S::kCols : 0);
          if (S::kPlanes == 3) {
            if (!(ok = wait(bar_dw_free + 8 * buf, free_phase ^ 1))) break;
            tc::tc_fence_after();
          }
#pragma unroll
          for (int t = 0; t < kProducts; ++t) {
            const int pa = kProducts == 6 ? cut_a(t) : 0, pb = kProducts == 6 ? cut_b(t) : 0;
#pragma unroll
            for (int kk = 0; kk < kTile / 16; ++kk)
              tc::mma_16<1>(d, tc::smem_desc_sw128(sdz + pa * S::kPlaneBytes + kk * 2048, dz_lbo, 1024),
                            tc::smem_desc_sw128(sx + pb * S::kPlaneBytes + kk * 2048, S::kBlockBytes, 1024), idesc_dw,
                            ((S::kPlanes == 1 && !first) || t > 0 || kk > 0) ? 1u : 0u);
          }
          if (S::kPlanes == 3) tc::mma_commit(bar_dw + 8 * buf);
          first = false;
        }
        tc::mma_commit(bar_empty + 8 * s);
        if (++s == S::kStages) s = 0, phase ^= 1;
        if (++buf == 2) buf = 0, free_phase ^= 1;
      }
      if (ok && S::kPlanes == 1 && g.dw) tc::mma_commit(bar_dw);
    }
    __syncwarp();
  } else if (SRC == kRun && warp == kTmaWarp) {
    if (tc::elect_one()) {
      constexpr long long kElem = sizeof(T);
      for (long long tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        if (!wait(bar_taken + 8 * ring_s, ring_phase ^ 1)) break;
        const uint32_t at = base + S::kOffRaw + ring_s * q.raw_bytes, bar = bar_landed + 8 * ring_s;
        const long long rows = min(static_cast<long long>(kTile), g.I - tile * kTile);
        uint32_t bytes = 0;
        // whole 16 bytes by an asynchronous copy; the last tile's last few by themselves
        const auto copy = [&](const void* m, long long cols, uint32_t to, bool go) {
          const char* from = static_cast<const char*>(m) + tile * kTile * cols * kElem;
          const int all = static_cast<int>(rows * cols * kElem), whole = all / 16 * 16;
          if (!go) {
            bytes += whole;
            for (int e = whole; e < all; e += 2) {
              const uint16_t v = *reinterpret_cast<const uint16_t*>(from + e);
              asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + e), "h"(v) : "memory");
            }
          } else if (whole > 0) {
            tc::bulk_load(to, from, whole, bar);
          }
        };
        for (int go = 0; go < 2; ++go) {
          copy(g.dy, g.N, at, go);
          if (g.act != PIC_ACT_NONE) copy(g.pre, g.N, at + q.raw_z, go);
          if (g.dw) copy(g.x, g.K, at + q.raw_x, go);
          if (!go) tc::mbar_arrive_expect_tx(bar, bytes);
        }
        if (++ring_s == q.raw_ring) ring_s = 0, ring_phase ^= 1;
      }
    }
    __syncwarp();
  } else if (SRC == kTma && warp == kTmaWarp) {
    if (tc::elect_one()) {
      const bool has_z = g.act != PIC_ACT_NONE;
      const uint32_t bytes = S::kPlaneBytes * (1 + (g.dw ? 1 : 0) + (has_z ? 1 : 0));
      for (long long tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        if (!wait(bar_empty + 8 * ring_s, ring_phase ^ 1)) break;
        const uint32_t at = base + ring_s * S::kStageBytes, bar = bar_landed + 8 * ring_s;
        const int i = static_cast<int>(tile * kTile);
        tc::mbar_arrive_expect_tx(bar, bytes);
        tc::tma_load_2d<false>(at, &maps.dy, 0, i, bar);
        if (has_z) tc::tma_load_2d<false>(at + 2 * S::kPlaneBytes, &maps.z, 0, i, bar);
        if (g.dw) tc::tma_load_2d<false>(at + S::kPlaneBytes, &maps.x, 0, i, bar);
        if (++ring_s == S::kStages) ring_s = 0, ring_phase ^= 1;
      }
    }
    __syncwarp();
  } else if (warp < 4) {
    const uint32_t panels = base + S::kOffPanels + warp * S::kPanels * kPanelBytes;
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    Product p{};  // what put_panel looks at
    p.I = g.I, p.J = g.K;
    int buf = 0, pb = 0, count = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (long long tile = blockIdx.x; g.dx && tile < q.tiles; tile += gridDim.x, ++count) {
      ok = __all_sync(0xffffffffu, wait(bar_dx + 8 * buf, phase));
      if (!ok) break;
      tc::tc_fence_after();
      const long long row0 = tile * kTile + warp * 32;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) {
        uint32_t r[64];
        if (64 * b < g.K) tc::tmem_ld64_wait(tmem + buf * S::kCols + 64 * b + lanes, r);
        if (b + 1 == S::kBlocks) {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0 && !(q.waits.test_fault && tile == 0 && warp == 0)) tc::mbar_arrive(bar_dx_free + 8 * buf);
        }
        if (64 * b >= g.K || row0 >= g.I) continue;
        if constexpr (sizeof(T) == 4) {
          if (marks[count % kMarks] == count + 1 || marks[kMarks]) {
            float v[64];
            dx_again(v, g, row0 + lane);
#pragma unroll
            for (int c = 0; c < 64; ++c) r[c] = __float_as_uint(v[c]);
          }
        }
        constexpr int kPanels = sizeof(T) == 4 ? 2 : 1;
#pragma unroll
        for (int h = 0; h < kPanels; ++h) {
          if (64 * b + 32 * h * (kPanels - 1) >= g.K) break;
          uint32_t out[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if constexpr (sizeof(T) == 4)
              out[c] = r[32 * h + c];
            else
              out[c] = pack2_of<T>(__uint_as_float(r[2 * c]), __uint_as_float(r[2 * c + 1]));
          }
          if (lane == 0) tc::bulk_wait_read<S::kPanels - 1>();
          __syncwarp();
          put_panel<T>(out, panels + pb * kPanelBytes, lane, row0, 64 * b + 32 * h, p, g.dx, g.lddx, &maps.dx, q.store_tma);
          if (++pb == S::kPanels) pb = 0;
        }
      }
      if (++buf == 2) buf = 0, phase ^= 1;
    }
    if (lane == 0) tc::bulk_wait_all();
    __syncwarp();
    if (S::kPlanes == 1 && g.dw && ok && __all_sync(0xffffffffu, wait(bar_dw, 0))) {
      tc::tc_fence_after();
      const int n = warp * 32 + lane;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) {
        if (64 * b >= g.K || warp * 32 >= g.N) break;
        uint32_t r[64];
        tc::tmem_ld64_wait(tmem + S::kTmemDw + 64 * b + lanes, r);
        if (n < g.N)
#pragma unroll
          for (int c = 0; c < 64; ++c)
            if (64 * b + c < g.K) my_parts[n * g.K + 64 * b + c] = __uint_as_float(r[c]);
      }
    }
    __syncwarp();
  } else if (S::kPlanes == 3 && warp < 6 && g.dw) {
    const int n = (warp - 4) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp - 4) * 32) << 16;
    float v[64] = {};
    int buf = 0, count = 0;
    uint32_t phase = 0;
    for (long long tile = blockIdx.x; tile < q.tiles; tile += gridDim.x, ++count) {
      if (!__all_sync(0xffffffffu, wait(bar_dw + 8 * buf, phase))) break;
      tc::tc_fence_after();
      if (marks[count % kMarks] == count + 1) {
        float u[64];
        dw_again(u, g, tile * kTile, n);
#pragma unroll
        for (int c = 0; c < 64; ++c) v[c] += u[c];
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t r[32];
          tc::tmem_ld32_wait(tmem + S::kTmemDw + buf * S::kCols + 32 * h + lanes, r);
#pragma unroll
          for (int c = 0; c < 32; ++c) v[32 * h + c] += __uint_as_float(r[c]);
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar_dw_free + 8 * buf);
      if (++buf == 2) buf = 0, phase ^= 1;
    }
    if (n < g.N)
#pragma unroll
      for (int c = 0; c < 64; ++c)
        if (c < g.K) my_parts[n * g.K + c] = v[c];
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // copies and MMAs in flight use shared and tensor memory
    if (SRC != kReg && warp == kTmaWarp && tc::elect_one())
      drain_loads(bar_landed, SRC == kRun ? q.raw_ring : S::kStages, ring_s, ring_phase, q.waits);
    if (warp == kMmaWarp && tc::elect_one()) drain_mmas<1>(bar_drain, q.waits);
    __syncthreads();
  }
  tc::tc_fence_after();
  if (warp == kMmaWarp) tc::tmem_dealloc_cg<1>(tmem, S::kTmemCols);
}

// dw and db from the CTAs' parts: a block finishes 32 values, its warps add every
// 32nd part, the first warp the warps' sums.
template <typename T>
__global__ void __launch_bounds__(1024) add_parts_kernel(const float* parts, int n_parts, const NarrowGrad g) {
  constexpr int kAtOnce = (kSms + 31) / 32;  // loads of a thread under way together
  __shared__ float sums[32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nk = g.N * g.K, per = nk + g.N;
  const int e = blockIdx.x * 32 + lane;
  float v = 0.0f;
  if (e < per) {
    for (int s0 = warp; s0 < n_parts; s0 += 32 * kAtOnce) {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int s = s0 + 32 * i;
        if (s < n_parts) v += __ldcg(parts + s * static_cast<long long>(per) + e);
      }
    }
  }
  sums[warp][lane] = v;
  __syncthreads();
  if (warp > 0 || e >= per) return;
#pragma unroll
  for (int w = 1; w < 32; ++w) v += sums[w][lane];
  if (e >= nk) {
    if (g.db) static_cast<T*>(g.db)[e - nk] = from_f32<T>(v);
  } else if (g.dw) {
    static_cast<T*>(g.dw)[e / g.K * g.lddw + e % g.K] = from_f32<T>(v);
  }
}

// As many CTAs as SMs, or a multiple of that (fp32 takes dw over after every tile).
int ctas(const NarrowGrad& g, int dtype) {
  const long long tiles = (g.I + kTile - 1) / kTile, each = dtype == PIC_DTYPE_F32 ? tiles : kMostTiles;
  const long long most = kSms * ((tiles + kSms * each - 1) / (kSms * each));
  return static_cast<int>(tiles < most ? tiles : most);
}

// The run mode's room for copies: a tile's dy, z and x, each on a 16-byte boundary
// with some bytes to read past its end; as many tiles as fit, false if none does.
template <typename T, bool WIDE>
bool plan_runs(NarrowParams& q) {
  const NarrowGrad& g = q.g;
  const int dz = (kTile * g.N * static_cast<int>(sizeof(T)) + 47) / 16 * 16;
  const int x = (kTile * g.K * static_cast<int>(sizeof(T)) + 47) / 16 * 16;
  q.raw_z = dz;
  q.raw_x = g.act != PIC_ACT_NONE ? 2 * dz : dz;
  q.raw_bytes = (q.raw_x + (g.dw ? x : 0) + 127) / 128 * 128;
  q.raw_ring = (227 * 1024 - Shape<T, WIDE, kRun>::kSmem) / q.raw_bytes;
  if (q.raw_ring > kMaxRing) q.raw_ring = kMaxRing;
  return q.raw_ring > 0;
}

template <typename T, bool WIDE, Source SRC>
int run(const NarrowGrad& g, NarrowParams& q, NarrowMaps& maps, int grid, int slot, cudaStream_t s) {
  const void* fn = reinterpret_cast<const void*>(narrow_kernel<T, WIDE, SRC>);
  const int fixed = Shape<T, WIDE, SRC>::kSmem;
  const int smem = SRC == kRun ? 227 * 1024 : fixed;  // the attribute is set once, for runs of any width
  static_assert(Shape<T, WIDE, SRC>::kSmem <= 227 * 1024, "shared memory of an SM");
  if (allow_smem(fn, slot, smem) != PIC_OK) return PIC_ERR_CUDA;
  void* args[] = {&q, &maps};
  if (cudaLaunchKernel(fn, dim3(grid), dim3(kThreads), args, smem, s) != cudaSuccess) return PIC_ERR_CUDA;
  if (g.dw || g.db) {
    const int per = g.N * g.K + g.N;
    add_parts_kernel<T><<<(per + 31) / 32, 1024, 0, s>>>(q.parts, grid, g);
  }
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace

bool narrow_takes(const NarrowGrad& g, int dtype) {
  const int most = dtype == PIC_DTYPE_F32 ? 64 : 128;
  return (g.dx || g.dw) && g.N <= most && g.K <= most && g.I >= 1024;
}

long long narrow_workspace(const NarrowGrad& g, int dtype) {
  return ctas(g, dtype) * static_cast<long long>(g.N * g.K + g.N) * 4;
}

int narrow_grad(const NarrowGrad& g, int dtype, void* ws, const Waits& waits, cudaStream_t s) {
  NarrowParams q{};
  const int elem = dtype == PIC_DTYPE_F32 ? 4 : 2, grid = ctas(g, dtype);
  const auto on16 = [&](const void* m, long long ld) { return reinterpret_cast<uintptr_t>(m) % 16 == 0 && ld * elem % 16 == 0; };
  q.g = g;
  q.tiles = (g.I + kTile - 1) / kTile;
  q.vec_dy = on16(g.dy, g.lddy), q.vec_z = on16(g.pre, g.ldpre), q.vec_x = on16(g.x, g.ldx);
  q.store_tma = g.dx && g.K * elem % 16 == 0 && on16(g.dx, g.lddx) && g.lddx * elem < (1LL << 40);
  q.parts = static_cast<float*>(ws);
  q.waits = waits;
  NarrowMaps maps{};
  const auto far = [&](long long ld) { return ld * elem >= (1LL << 40); };
  if (q.store_tma && !encode(&maps.dx, g.dx, g.I, g.K, g.lddx, 32, dtype)) return PIC_ERR_CUDA;
  const bool wide = g.N > 64 || g.K > 64, has_z = g.act != PIC_ACT_NONE;
  const bool tma = dtype != PIC_DTYPE_F32 && !wide && q.vec_dy && !far(g.lddy) && (!has_z || (q.vec_z && !far(g.ldpre))) &&
                   (!g.dw || (q.vec_x && !far(g.ldx)));
  if (tma && !(encode(&maps.dy, g.dy, g.I, g.N, g.lddy, kTile, dtype) &&
               (!has_z || encode(&maps.z, g.pre, g.I, g.N, g.ldpre, kTile, dtype)) &&
               (!g.dw || encode(&maps.x, g.x, g.I, g.K, g.ldx, kTile, dtype))))
    return PIC_ERR_CUDA;
  // rows end to end, from a 16-byte boundary on
  const auto packed = [](const void* m, long long ld, int cols) { return ld == cols && reinterpret_cast<uintptr_t>(m) % 16 == 0; };
  const bool runs = !tma && packed(g.dy, g.lddy, g.N) && (!has_z || packed(g.pre, g.ldpre, g.N)) && (!g.dw || packed(g.x, g.ldx, g.K));
  if (dtype == PIC_DTYPE_F32)
    return runs && plan_runs<float, false>(q) ? run<float, false, kRun>(g, q, maps, grid, 15, s) : run<float, false, kReg>(g, q, maps, grid, 8, s);
  if (dtype == PIC_DTYPE_F16) {
    if (tma) return run<__half, false, kTma>(g, q, maps, grid, 10, s);
    if (wide) return runs && plan_runs<__half, true>(q) ? run<__half, true, kRun>(g, q, maps, grid, 16, s) : run<__half, true, kReg>(g, q, maps, grid, 9, s);
    return runs && plan_runs<__half, false>(q) ? run<__half, false, kRun>(g, q, maps, grid, 17, s) : run<__half, false, kReg>(g, q, maps, grid, 11, s);
  }
  using B = __nv_bfloat16;
  if (tma) return run<B, false, kTma>(g, q, maps, grid, 13, s);
  if (wide) return runs && plan_runs<B, true>(q) ? run<B, true, kRun>(g, q, maps, grid, 18, s) : run<B, true, kReg>(g, q, maps, grid, 12, s);
  return runs && plan_runs<B, false>(q) ? run<B, false, kRun>(g, q, maps, grid, 19, s) : run<B, false, kReg>(g, q, maps, grid, 14, s);
}

}  // namespace lin
}  // namespace pic
