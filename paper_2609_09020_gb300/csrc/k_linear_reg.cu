// k_linear_reg.cu -- matrix products of fp32 matrices on the tensor cores, cut
// into bfloat16 pieces (cut3.cuh) on their way through registers.  Tiles are 128 x
// 64; the cuts along K are those of k_linear_tc.cuh.
//
// An infinite or NaN value would meet the zero pieces of others (inf 0 = NaN), so
// a loader that sees one marks the takeover (two slices) it belongs to, and the
// epilogue computes that takeover's sums again with FP32 FMAs from global memory:
// right, and only then slow; no wait is longer than a few such sums, however long K is.
//
// Roles: warps 0..3 epilogue (32 rows each), warps 4..11 load slices of A and B (16
// bytes per lane and load where they may), cut them and write them to shared memory
// as the MMA wants them, warp 12 issues the MMAs.  What bounds it is the loaders'
// work, some 40 operations for four values, so a thread's quads are whole rows
// apart and share their addresses.  The loads of the next slice are under way while
// this one is written.  Measured: 1.7 us for a slice of 64 of K, 92 TFLOP/s over all
// SMs; 100 x 4096 -> 2048 34 us, 128 x 2048 -> 8192 59.
#include "cut3.cuh"
#include "k_linear_reg.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kEpiWarps = 4, kLoadWarps = 8, kMmaWarp = kEpiWarps + kLoadWarps;
constexpr int kThreads = 32 * (kMmaWarp + 1), kLoaders = 32 * kLoadWarps;
constexpr unsigned kMarks = 16;  // more than the takeovers that the loaders can be ahead of the epilogue (5)
constexpr int kChunk = 2;  // slices of 64 between two takeovers of the accumulators

constexpr int kAPlane = kRegRows * 128, kBPlane = kRegCols * 128;  // bytes
constexpr int kStageBytes = kPieces * (kAPlane + kBPlane);
constexpr int kStages = 2;
constexpr int kOffPanels = kStages * kStageBytes;
constexpr int kOffBars = kOffPanels + kEpiWarps * kTurnBytes;
constexpr int kBufs = 4;  // accumulators
constexpr int kBars = 2 * kStages + 2 * kBufs + 1;
constexpr int kOffMarks = kOffBars + kBars * 8 + 8;
constexpr int kSmem = kOffMarks + kMarks * 4 + 8 + 1024;  // 1024: the base is rounded up
constexpr int kTmemCols = kBufs * kRegCols;

struct Quad {
  uint32_t w[4];
};

__device__ __forceinline__ void sts64(uint32_t saddr, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(saddr), "r"(a), "r"(b) : "memory");
}

// One slice of an operand: ROWS rows x 64 of K, stored as rows of 64 (along K), or as
// 64 rows (of K) of ROWS, which are one or two blocks of 64.  A loader thread has
// kTurns quads of it, whole turns of rows apart.
template <int ROWS>
struct Slice {
  static constexpr int kTurns = ROWS * 64 / 4 / kLoaders;
  Quad q[kTurns];

  // rows [r0, rows), columns [c0, cols) of the stored matrix exist
  __device__ __forceinline__ void load(const float* m, long long ld, bool mn, bool vec, long long r0, long long rows,
                                       long long c0, long long cols, int tid) {
    const int across = mn ? ROWS / 4 : 16, row = tid / across, col = tid % across * 4, turn = kLoaders / across;
    const int n = static_cast<int>(max(0LL, min(4LL, cols - c0 - col)));
    const int left = static_cast<int>(min(static_cast<long long>(ROWS), rows - r0)) - row;
    const float* p = m + (r0 + row) * ld + c0 + col;
    if (vec && n == 4) {
#pragma unroll
      for (int u = 0; u < kTurns; ++u, p += turn * ld) {
        uint4 f = make_uint4(0, 0, 0, 0);
        if (u * turn < left) f = __ldg(reinterpret_cast<const uint4*>(p));
        q[u].w[0] = f.x, q[u].w[1] = f.y, q[u].w[2] = f.z, q[u].w[3] = f.w;
      }
    } else {
#pragma unroll
      for (int u = 0; u < kTurns; ++u, p += turn * ld)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          q[u].w[i] = load_if(reinterpret_cast<const uint32_t*>(p) + i, u * turn < left && i < n);
    }
  }
  // true if a value is infinite or NaN (or from kCutLimit on).  Of the rows that do not exist (from
  // `rows` on) nothing is written: what the MMA makes of them is not looked at.
  __device__ __forceinline__ bool store(uint32_t s, bool mn, long long rows, int tid) const {
    constexpr int kPlane = ROWS * 128;
    const int across = mn ? ROWS / 4 : 16, row = tid / across, col = tid % across * 4, turn = kLoaders / across;
    const uint32_t at = s + (col >> 6) * 8192 + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4) + (col & 4) * 2;
    uint32_t largest = 0;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      if ((mn ? col : row + u * turn) >= rows) break;
      uint32_t h0, m0, l0, h1, m1, l1;
#pragma unroll
      for (int i = 0; i < 4; ++i) largest = max(largest, q[u].w[i] & 0x7fffffffu);
      cut3(q[u].w[0], q[u].w[1], h0, m0, l0);
      cut3(q[u].w[2], q[u].w[3], h1, m1, l1);
      sts64(at + u * turn * 128, h0, h1);
      sts64(at + u * turn * 128 + kPlane, m0, m1);
      sts64(at + u * turn * 128 + 2 * kPlane, l0, l1);
    }
    return largest >= kCutLimit;
  }
};

// The epilogue's takeovers from slice c0 to the tile's end, where the first is marked: those
// that are, added to v from memory again.  A function of its own, so that it takes no
// registers from the usual path.
struct TakeMarked {
  long long row, col0;
  int c0, k1, lane;
  uint32_t tmem, bar_acc, bar_free;
  bool withhold;
  volatile int* abort_flag;
  volatile unsigned* marks;
};
__device__ __noinline__ bool take_marked(float* sums, const TcParams& q, const RegOperands& o, const TakeMarked& m, int buf,
                                         uint32_t phase, unsigned takeover) {
  float v[64];
#pragma unroll
  for (int c = 0; c < 64; ++c) v[c] = sums[c];
  for (int c0 = m.c0; c0 < m.k1; c0 += kChunk, ++takeover) {
    if (!__all_sync(0xffffffffu, wait_bounded(m.bar_acc + 8 * buf, phase, m.abort_flag, q.waits))) return false;
    tc::tc_fence_after();
    if (m.marks[takeover % kMarks] == takeover + 1) {
      sum_again(v, static_cast<const float*>(o.a), q.a_mn ? 1 : o.lda, q.a_mn ? o.lda : 1, static_cast<const float*>(o.b),
                q.b_mn ? 1 : o.ldb, q.b_mn ? o.ldb : 1, m.row, q.p.I, m.col0, q.p.J, c0 * 64LL,
                min(q.p.K, min(m.k1, c0 + kChunk) * 64LL));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t r[32];
        tc::tmem_ld32_wait(m.tmem + buf * kRegCols + 32 * h, r);
#pragma unroll
        for (int c = 0; c < 32; ++c) v[32 * h + c] += __uint_as_float(r[c]);
      }
    }
    tc::tc_fence_before();
    __syncwarp();
    if (m.lane == 0 && !m.withhold) tc::mbar_arrive(m.bar_free + 8 * buf);
    if (++buf == kBufs) buf = 0, phase ^= 1;
  }
#pragma unroll
  for (int c = 0; c < 64; ++c) sums[c] = v[c];
  return true;
}

__global__ void __launch_bounds__(kThreads, 1)
    reg_kernel(const __grid_constant__ TcParams q, const __grid_constant__ TcMaps maps, const __grid_constant__ RegOperands o) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bars = base + kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * kStages, bar_acc = bar_empty + 8 * kStages,
                 bar_free = bar_acc + 8 * kBufs, bar_drain = bar_free + 8 * kBufs;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffBars + 8 * kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + 8 * kBars + 4);
  // mark t % kMarks holds t + 1 if this CTA's t-th takeover has an infinite or NaN operand
  volatile unsigned* marks = reinterpret_cast<volatile unsigned*>(smem + kOffMarks);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, kLoadWarps);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      tc::mbar_init(bar_acc + 8 * b, 1);
      tc::mbar_init(bar_free + 8 * b, kEpiWarps);
    }
    tc::mbar_init(bar_drain, 1);
    *abort_flag = 0;
    for (unsigned m = 0; m < kMarks; ++m) marks[m] = 0;
    tc::fence_mbar_init();
  }
  if (warp == kMmaWarp) tc::tmem_alloc_cg<1>(tc::smem_addr(tmem_slot), kTmemCols);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Product& p = q.p;
  const float* ma = static_cast<const float*>(o.a);
  const float* mb = static_cast<const float*>(o.b);
  auto wait = [&](uint32_t bar, uint32_t parity) { return wait_bounded(bar, parity, abort_flag, q.waits); };
  auto part = [&](long long w, int& k0, int& k1) {
    k0 = static_cast<int>(w % q.splits) * q.part_blocks;
    k1 = min(q.k_blocks, k0 + q.part_blocks);
  };
  

  if (warp >= kEpiWarps && warp < kMmaWarp) {
    const int tid = threadIdx.x - 32 * kEpiWarps;
    Slice<kRegRows> a;
    Slice<kRegCols> b;
    // a place in the CTA's sequence of slices; loads are one slice ahead of stores
    struct Cursor {
      long long w, ti, tj;
      int k0, kb, k1;
      unsigned takeover;
    };
    auto enter = [&](Cursor& c) {
      if (c.w >= q.work) return;
      part(c.w, c.k0, c.k1);
      tile_place<kRegRows>(c.w / q.splits, q.tiles_i, q.tiles_j, c.ti, c.tj);
      c.kb = c.k0;
    };
    auto advance = [&](Cursor& c) {
      ++c.kb;
      if (c.kb == c.k1 || (c.kb - c.k0) % kChunk == 0) ++c.takeover;
      if (c.kb < c.k1) return;
      c.w += gridDim.x;
      enter(c);
    };
    auto load_a = [&](Slice<kRegRows>& x, const Cursor& c) {
      if (c.w >= q.work) return;
      if (q.a_mn)
        x.load(ma, o.lda, true, o.vec_a, c.kb * 64LL, p.K, c.ti * kRegRows, p.I, tid);
      else
        x.load(ma, o.lda, false, o.vec_a, c.ti * kRegRows, p.I, c.kb * 64LL, p.K, tid);
    };
    auto load_b = [&](Slice<kRegCols>& x, const Cursor& c) {
      if (c.w >= q.work) return;
      if (q.b_mn)
        x.load(mb, o.ldb, true, o.vec_b, c.kb * 64LL, p.K, c.tj * kRegCols, p.J, tid);
      else
        x.load(mb, o.ldb, false, o.vec_b, c.tj * kRegCols, p.J, c.kb * 64LL, p.K, tid);
    };
    // a B that is the same for all tiles is written to every stage once
    const bool fixed_b = q.tiles_j == 1 && q.k_blocks == 1;
    Cursor put{blockIdx.x, 0, 0, 0, 0, 0, 0};
    enter(put);
    Cursor get = put;
    load_a(a, get);
    load_b(b, get);
    if (get.w < q.work) advance(get);
    uint32_t phase = 0;
    int filled = 0;
    bool bad_b = false;
    // stage i's slice; false at the end
    auto step = [&](int i) -> bool {
      if (put.w >= q.work) return false;
      if (!__all_sync(0xffffffffu, wait(bar_empty + 8 * i, phase ^ 1))) return false;
      const uint32_t sa = base + i * kStageBytes;
      const bool bad = a.store(sa, q.a_mn, p.I - put.ti * kRegRows, tid);
      load_a(a, get);
      if (!fixed_b || filled < kStages) bad_b |= b.store(sa + kPieces * kAPlane, q.b_mn, p.J - put.tj * kRegCols, tid);
      ++filled;
      if (!fixed_b) load_b(b, get);
      if (bad || bad_b) marks[put.takeover % kMarks] = put.takeover + 1;
      if (!fixed_b) bad_b = false;
      if (get.w < q.work) advance(get);
      advance(put);
      tc::fence_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar_full + 8 * i);
      return true;
    };
    int s = 0;
    while (step(s))
      if (++s == kStages) s = 0, phase ^= 1;
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (tc::elect_one()) {
      const uint32_t a_step = q.a_mn ? 2048 : 32, b_step = q.b_mn ? 2048 : 32;
      int s = 0, buf = 0;
      uint32_t phase = 0, free_phase = 0;
      bool ok = true;
      for (long long w = blockIdx.x; w < q.work && ok; w += gridDim.x) {
        long long ti, tj;
        tile_place<kRegRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
        // as many columns as exist, in sixteens
        const int n = static_cast<int>(min(static_cast<long long>(kRegCols), (p.J - tj * kRegCols + 15) / 16 * 16));
        const uint32_t idesc = tc::idesc_16(128, n, true, q.a_mn != 0, q.b_mn != 0);
        int k0, k1;
        part(w, k0, k1);
        for (int c0 = k0; c0 < k1 && ok; c0 += kChunk) {
          if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * kRegCols;
          const int c1 = min(k1, c0 + kChunk);
          for (int kb = c0; kb < c1; ++kb) {
            if (!(ok = wait(bar_full + 8 * s, phase))) break;
            tc::tc_fence_after();
            const uint32_t sa = base + s * kStageBytes, sb = sa + kPieces * kAPlane;
            const int steps = static_cast<int>(min(4LL, (p.K - kb * 64LL + 15) / 16));
#pragma unroll
            for (int t = 0; t < 6; ++t)
              for (int kk = 0; kk < steps; ++kk)
                tc::mma_16<1>(d, tc::smem_desc_sw128(sa + cut_a(t) * kAPlane + kk * a_step, 8192, 1024),
                              tc::smem_desc_sw128(sb + cut_b(t) * kBPlane + kk * b_step, 8192, 1024), idesc,
                              (kb > c0 || t > 0 || kk > 0) ? 1u : 0u);
            tc::mma_commit(bar_empty + 8 * s);
            if (++s == kStages) s = 0, phase ^= 1;
          }
          if (!ok) break;
          tc::mma_commit(bar_acc + 8 * buf);
          if (++buf == kBufs) buf = 0, free_phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp;
    float* turn = reinterpret_cast<float*>(smem + kOffPanels + warp * kTurnBytes);
    int buf = 0;
    unsigned takeover = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (long long w = blockIdx.x; w < q.work && ok; w += gridDim.x) {
      long long ti, tj;
      tile_place<kRegRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
      const long long row0 = ti * kRegRows + quarter * 32, col0 = tj * kRegCols;
      int k0, k1;
      part(w, k0, k1);
      float v[64];
      for (int c0 = k0; c0 < k1; c0 += kChunk, ++takeover) {
        ok = __all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase));
        if (!ok) break;
        tc::tc_fence_after();
        if (marks[takeover % kMarks] == takeover + 1) {  // the rest of the tile's
          float u[64];
#pragma unroll
          for (int c = 0; c < 64; ++c) u[c] = c0 == k0 ? 0.0f : v[c];
          const TakeMarked m{row0 + lane, col0, c0, k1, lane, tmem + (static_cast<uint32_t>(quarter * 32) << 16), bar_acc,
                             bar_free, q.waits.test_fault && w == 0 && quarter == 0, abort_flag, marks};
          ok = take_marked(u, q, o, m, buf, phase, takeover);
#pragma unroll
          for (int c = 0; c < 64; ++c) v[c] = u[c];
          const int n = (k1 - c0 + kChunk - 1) / kChunk;
          takeover += n - 1, buf += n;
          phase ^= buf / kBufs & 1, buf %= kBufs;
          c0 = k1;
          if (!ok) break;
          continue;
        }
        const uint32_t d = tmem + buf * kRegCols + (static_cast<uint32_t>(quarter * 32) << 16);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t r[32];
          tc::tmem_ld32_wait(d + 32 * h, r);
#pragma unroll
          for (int c = 0; c < 32; ++c)
            v[32 * h + c] = c0 == k0 ? __uint_as_float(r[c]) : v[32 * h + c] + __uint_as_float(r[c]);
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0 && !(q.waits.test_fault && w == 0 && quarter == 0)) tc::mbar_arrive(bar_free + 8 * buf);
        if (++buf == kBufs) buf = 0, phase ^= 1;
      }
      if (!ok) break;
      if (q.parts) {
        float4* out = reinterpret_cast<float4*>(q.parts) + w * (128 * 16) + quarter * (32 * 16) + lane;
#pragma unroll
        for (int c = 0; c < 16; ++c) out[c * 32] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        continue;
      }
      if (row0 >= p.I) continue;
      if (p.swapped)
        finish_swapped(v, p, lane, row0, col0);
      else
        finish_rows(v, p, turn, lane, row0, col0);
    }
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // MMAs in flight still read shared memory
    if (warp == kMmaWarp && tc::elect_one()) drain_mmas<1>(bar_drain, q.waits);
    __syncthreads();
  }
  tc::tc_fence_after();
  if (warp == kMmaWarp) tc::tmem_dealloc_cg<1>(tmem, kTmemCols);
}

}  // namespace

RegKernel reg_kernel_info() { return {reinterpret_cast<const void*>(reg_kernel), kThreads, kSmem}; }

}  // namespace lin
}  // namespace pic
