// k_linear_planes.cu -- large products of fp32 matrices on the tensor cores.  A
// first kernel cuts each matrix into three planes of bfloat16 pieces (cut3.cuh),
// once, in the workspace; the product then is the one of k_linear_tc.cuh for a
// pair of CTAs, with three planes of each operand in a stage and six MMAs for
// every 16 of K.  (k_linear_reg.cu cuts on the way into shared memory instead,
// again for every tile: better where a matrix is used by one tile or two.)
//
// A stage is 32 of K, half a slice: five stages of 36 KB keep more loads under way
// than two of 64 of K did.  With four accumulators instead of two, whose way to the
// epilogue and back is hidden, 2048 x 1024 -> 4096 takes 85 us where it took 98: 202
// TFLOP/s of fp32, 1.2 PFLOP/s of bfloat16 products.
//
// Roles: warp 0 TMA, warp 1 MMAs, warps 2..9 epilogue: 32 rows x 64 columns
// each, which takes the accumulators over after every kTakeover slices.
//
// An infinite or NaN value would meet the zero pieces of others (inf 0 = NaN), so
// the first kernel marks the blocks of 128 x 128 that have one, and an epilogue warp
// computes the sums of a takeover's K, where its rows or columns are marked there,
// again with FP32 FMAs: no wait is longer than a few such sums, however long K is.
#include "cut3.cuh"
#include "k_linear_planes.cuh"

namespace pic {
namespace lin {
namespace {

constexpr int kEpi = 8;
constexpr int kThreads = 64 + 32 * kEpi;
constexpr int kTakeover = 2;
constexpr int kHalf = 32;  // K of a stage, half a slice
constexpr int kABytes = 128 * 2 * kHalf, kBBytes = kPlCols / 2 * 2 * kHalf;  // one plane of one CTA
constexpr int kBlock = kHalf * 128;  // 64 rows of an operand that lies along them
constexpr int kStageBytes = kPieces * (kABytes + kBBytes);
constexpr int kStages = 5;
constexpr int kOffPanels = kStages * kStageBytes;
constexpr int kOffBars = kOffPanels + kEpi * kTurnBytes;
constexpr int kBufs = 4;  // accumulators: their way to the epilogue and back is longer than a slice's MMAs
constexpr int kBars = 2 * kStages + 2 * kBufs + 1;
constexpr int kSmem = kOffBars + kBars * 8 + 16 + 1024;
constexpr int kTmemCols = kBufs * kPlCols;

struct CutPair {
  CutMatrix m[2];
  unsigned blocks0;  // blocks of the first matrix
};

__global__ void __launch_bounds__(256) cut_kernel(const CutPair q) {
  const int which = blockIdx.x < q.blocks0 ? 0 : 1;
  const unsigned block = which ? blockIdx.x - q.blocks0 : blockIdx.x;
  const float* m = q.m[which].m;
  const long long ld = q.m[which].ld, rows = q.m[which].rows, cols = q.m[which].cols, ld_out = q.m[which].ld_out;
  uint16_t* planes = static_cast<uint16_t*>(q.m[which].planes);
  const unsigned col_blocks = static_cast<unsigned>((cols + kPlBlock - 1) / kPlBlock);
  const long long r0 = block / col_blocks * static_cast<long long>(kPlBlock);
  const long long c0 = block % col_blocks * static_cast<long long>(kPlBlock);
  const long long plane = rows * ld_out;
  // 16 quads of four columns for each thread: a warp takes a row's 128 columns
  const long long col = c0 + threadIdx.x % 32 * 4;
  const bool vec = reinterpret_cast<uintptr_t>(m) % 16 == 0 && ld % 4 == 0;
  uint32_t largest = 0;
#pragma unroll 4
  for (int u = 0; u < kPlBlock / 8; ++u) {
    const long long r = r0 + threadIdx.x / 32 + u * 8;
    if (r >= rows || col >= cols) continue;
    uint32_t w[4];
    const float* p = m + r * ld + col;
    if (vec && col + 4 <= cols) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = col + i < cols ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) largest = max(largest, w[i] & 0x7fffffffu);
    uint32_t h0, m0, l0, h1, m1, l1;
    cut3(w[0], w[1], h0, m0, l0);
    cut3(w[2], w[3], h1, m1, l1);
    // rows are a multiple of eight places: the four are there
    uint16_t* o = planes + r * ld_out + col;
    *reinterpret_cast<uint2*>(o) = make_uint2(h0, h1);
    *reinterpret_cast<uint2*>(o + plane) = make_uint2(m0, m1);
    *reinterpret_cast<uint2*>(o + 2 * plane) = make_uint2(l0, l1);
  }
  const int bad = __syncthreads_or(largest >= kCutLimit);
  if (threadIdx.x == 0) q.m[which].marks[block] = bad;
}

// Whether a block of the 128 rows (or columns of B) `group` and of slices
// [k0, k1) of K is marked.
__device__ __forceinline__ bool marked(const PlOperand& o, bool mn, long long group, long long groups, int k0, int k1,
                                       int lane) {
  if (group >= groups) return false;
  bool bad = false;
  for (int b = k0 / 2 + lane; b <= (k1 - 1) / 2; b += 32)
    bad |= o.marks[mn ? b * static_cast<long long>(o.col_blocks) + group : group * o.col_blocks + b] != 0;
  return __any_sync(0xffffffffu, bad);
}
__device__ __forceinline__ bool marked_in(const PlOperands& o, const TcParams& q, long long a_group, long long b_group,
                                          int k0, int k1, int lane) {
  return marked(o.a, q.a_mn, a_group, (q.p.I + 127) / 128, k0, k1, lane) ||
         marked(o.b, q.b_mn, b_group, (q.p.J + 127) / 128, k0, k1, lane);
}

// The epilogue's takeovers of slices [k0, k1) where some are marked: those from memory
// again.  A function of its own, so that it takes no registers from the usual path
// (inlined, 2048 x 1024 -> 4096 took 92 us instead of 84).
struct TakeMarked {
  long long a_group, b_group, row, col0;
  int k0, k1, lane;
  uint32_t tmem, bar_acc, lead_free;
  bool withhold;
  volatile int* abort_flag;
};
__device__ __noinline__ bool take_marked(float* out, const TcParams& q, const PlOperands& o, const TakeMarked& m, int buf,
                                         uint32_t phase) {
  float v[64] = {};
  for (int c0 = m.k0; c0 < m.k1; c0 += kTakeover) {
    if (!__all_sync(0xffffffffu, wait_bounded(m.bar_acc + 8 * buf, phase, m.abort_flag, q.waits))) return false;
    tc::tc_fence_after();
    const int c1 = min(m.k1, c0 + kTakeover);
    if (marked_in(o, q, m.a_group, m.b_group, c0, c1, m.lane)) {
      sum_again(v, o.a.m, q.a_mn ? 1 : o.a.ld, q.a_mn ? o.a.ld : 1, o.b.m, q.b_mn ? 1 : o.b.ld, q.b_mn ? o.b.ld : 1,
                m.row, q.p.I, m.col0, q.p.J, c0 * 64LL, min(q.p.K, c1 * 64LL));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t r[32];
        tc::tmem_ld32_wait(m.tmem + buf * kPlCols + 32 * h, r);
#pragma unroll
        for (int c = 0; c < 32; ++c)
          v[32 * h + c] += __uint_as_float(r[c]);
      }
    }
    tc::tc_fence_before();
    __syncwarp();
    if (m.lane == 0 && !m.withhold) tc::mbar_arrive_cluster(m.lead_free + 8 * buf);
    if (++buf == kBufs) buf = 0, phase ^= 1;
  }
#pragma unroll
  for (int c = 0; c < 64; ++c) out[c] = v[c];
  return true;
}

__global__ void __launch_bounds__(kThreads, 1)
    planes_kernel(const __grid_constant__ TcParams q, const __grid_constant__ TcMaps maps,
                  const __grid_constant__ PlOperands o) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const uint32_t bars = base + kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * kStages, bar_acc = bar_empty + 8 * kStages,
                 bar_free = bar_acc + 8 * kBufs, bar_drain = bar_free + 8 * kBufs;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffBars + 8 * kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + 8 * kBars + 4);

  if (threadIdx.x == 0) {
    tc::prefetch_map(&maps.a);
    tc::prefetch_map(&maps.b);
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, 1);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      tc::mbar_init(bar_acc + 8 * b, 1);
      tc::mbar_init(bar_free + 8 * b, kEpi * 2);
    }
    tc::mbar_init(bar_drain, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) tc::tmem_alloc_cg<2>(tc::smem_addr(tmem_slot), kTmemCols);
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Product& p = q.p;
  auto wait = [&](uint32_t bar, uint32_t parity) { return wait_bounded(bar, parity, abort_flag, q.waits); };
  const long long first = blockIdx.x / 2, step = gridDim.x / 2;
  auto part = [&](long long w, int& k0, int& k1) {
    k0 = static_cast<int>(w % q.splits) * q.part_blocks;
    k1 = min(q.k_blocks, k0 + q.part_blocks);
  };
  // one plane is kABytes (kBBytes) of rows along K (64 bytes each); of an operand
  // along its rows each block of 64 rows has its three planes of kBlock bytes
  const int a_plane = q.a_mn ? kBlock : kABytes, b_plane = q.b_mn ? kBlock : kBBytes;

  // the TMA and the MMA thread's place in the ring of stages (elect_one picks the
  // same lane each time)
  int s = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (warp == 0) {
    if (tc::elect_one()) {
      const uint32_t lead_full = tc::map_rank(bar_full, 0);
      for (long long w = first; w < q.work && ok; w += step) {
        long long ti, tj;
        tile_place<kPlRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
        const int i0 = static_cast<int>(ti * kPlRows + rank * 128), j0 = static_cast<int>(tj * kPlCols + rank * 64);
        int k0, k1;
        part(w, k0, k1);
        for (int kh = 2 * k0; kh < 2 * k1; ++kh) {
          if (!(ok = wait(bar_empty + 8 * s, phase ^ 1))) break;
          if (rank == 0) tc::mbar_arrive_expect_tx(bar_full + 8 * s, 2 * kStageBytes);
          const uint32_t sa = base + s * kStageBytes, sb = sa + kPieces * kABytes, bar = lead_full + 8 * s;
          const int k = kh * kHalf;
          if (q.a_mn) {
            tc::tma_load_planes_pair(sa, &maps.a, i0, k, bar);
            tc::tma_load_planes_pair(sa + kPieces * kBlock, &maps.a, i0 + 64, k, bar);
          } else {
            tc::tma_load_planes_pair(sa, &maps.a, k, i0, bar);
          }
          if (q.b_mn)
            tc::tma_load_planes_pair(sb, &maps.b, j0, k, bar);
          else
            tc::tma_load_planes_pair(sb, &maps.b, k, j0, bar);
          if (++s == kStages) s = 0, phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && tc::elect_one()) {
      const uint32_t idesc = tc::idesc_16(256, kPlCols, true, q.a_mn != 0, q.b_mn != 0);
      const uint32_t a_step = q.a_mn ? 2048 : 32, b_step = q.b_mn ? 2048 : 32;
      int buf = 0;
      uint32_t free_phase = 0;
      for (long long w = first; w < q.work && ok; w += step) {
        int k0, k1;
        part(w, k0, k1);
        for (int c0 = k0; c0 < k1 && ok; c0 += kTakeover) {
          if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * kPlCols;
          const int h0 = 2 * c0, h1 = 2 * min(k1, c0 + kTakeover);
          for (int kh = h0; kh < h1 && ok; kh += 2) {
            // a slice's two stages: the products of small pieces of both, then hi hi of both
            const int s2 = s + 1 == kStages ? 0 : s + 1;
            const uint32_t phase2 = s2 == 0 ? phase ^ 1 : phase;
            const auto products = [&](int stage, int t0, int t1, bool first) {
              const uint32_t sa = base + stage * kStageBytes, sb = sa + kPieces * kABytes;
#pragma unroll
              for (int t = t0; t < t1; ++t)
#pragma unroll
                for (int kk = 0; kk < kHalf / 16; ++kk) {
                  const uint32_t a = sa + cut_a(t) * a_plane + kk * a_step, b = sb + cut_b(t) * b_plane + kk * b_step;
                  tc::mma_16<2>(d, q.a_mn ? tc::smem_desc_sw128(a, kPieces * kBlock, 1024) : tc::smem_desc_sw64(a),
                                q.b_mn ? tc::smem_desc_sw128(b, kPieces * kBlock, 1024) : tc::smem_desc_sw64(b), idesc,
                                (!first || t > t0 || kk > 0) ? 1u : 0u);
                }
            };
            if (!(ok = wait(bar_full + 8 * s, phase))) break;
            tc::tc_fence_after();
            products(s, 0, 5, kh == h0);
            if (!(ok = wait(bar_full + 8 * s2, phase2))) break;
            tc::tc_fence_after();
            products(s2, 0, 5, false);
            products(s, 5, 6, false);
            tc::mma_commit_cg<2>(bar_empty + 8 * s);
            products(s2, 5, 6, false);
            tc::mma_commit_cg<2>(bar_empty + 8 * s2);
            s = s2 + 1, phase = phase2;
            if (s == kStages) s = 0, phase ^= 1;
          }
          if (!ok) break;
          tc::mma_commit_cg<2>(bar_acc + 8 * buf);
          if (++buf == kBufs) buf = 0, free_phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    float* turn = reinterpret_cast<float*>(smem + kOffPanels + (warp - 2) * kTurnBytes);
    const uint32_t lead_free = tc::map_rank(bar_free, 0);
    int buf = 0;
    for (long long w = first; w < q.work && ok; w += step) {
      long long ti, tj;
      tile_place<kPlRows>(w / q.splits, q.tiles_i, q.tiles_j, ti, tj);
      const long long row0 = ti * kPlRows + rank * 128 + quarter * 32, col0 = tj * kPlCols + half * 64;
      int k0, k1;
      part(w, k0, k1);
      float v[64];
      const bool withhold = q.waits.test_fault && w == 0 && rank == 0 && warp == 2;
      if (!marked_in(o, q, ti * 2 + rank, tj, k0, k1, lane)) {
        for (int c0 = k0; c0 < k1; c0 += kTakeover) {
          ok = __all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase));
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * kPlCols + half * 64 + (static_cast<uint32_t>(quarter * 32) << 16);
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
          if (lane == 0 && !withhold) tc::mbar_arrive_cluster(lead_free + 8 * buf);
          if (++buf == kBufs) buf = 0, phase ^= 1;
        }
      } else {
        float u[64];
        const TakeMarked m{ti * 2 + rank, tj, row0 + lane, col0, k0, k1, lane,
                           tmem + half * 64 + (static_cast<uint32_t>(quarter * 32) << 16), bar_acc, lead_free, withhold,
                           abort_flag};
        ok = take_marked(u, q, o, m, buf, phase);
        buf += (k1 - k0 + kTakeover - 1) / kTakeover;
        phase ^= buf / kBufs & 1, buf %= kBufs;
#pragma unroll
        for (int c = 0; c < 64; ++c) v[c] = u[c];
      }
      if (!ok) break;
      if (q.parts) {
        float4* out = reinterpret_cast<float4*>(q.parts) + ((w * 2 + rank) * 2 + half) * (128 * 16) + quarter * (32 * 16) + lane;
#pragma unroll
        for (int c = 0; c < 16; ++c) out[c * 32] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        continue;
      }
      if (row0 >= p.I || col0 >= p.J) continue;
      finish_rows(v, p, turn, lane, row0, col0);
    }
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // as in k_linear_tc.cuh
    if (warp == 0 && rank == 0 && tc::elect_one()) drain_loads(bar_full, kStages, s, phase, q.waits);
    if (warp == 1 && rank == 0 && tc::elect_one()) drain_mmas<2>(bar_drain, q.waits);
    __nanosleep(200000);
    __syncthreads();
  }
  tc::cluster_sync();
  tc::tc_fence_after();
  if (warp == 1) tc::tmem_dealloc_cg<2>(tmem, kTmemCols);
}

}  // namespace

PlKernel planes_kernel_info() { return {reinterpret_cast<const void*>(planes_kernel), kThreads, kSmem}; }

int cut_planes(const CutMatrix (&m)[2], cudaStream_t s) {
  const auto blocks = [](const CutMatrix& c) {
    return static_cast<unsigned>((c.rows + kPlBlock - 1) / kPlBlock * ((c.cols + kPlBlock - 1) / kPlBlock));
  };
  const CutPair q{{m[0], m[1]}, blocks(m[0])};
  cut_kernel<<<q.blocks0 + blocks(m[1]), 256, 0, s>>>(q);
  return cudaGetLastError() == cudaSuccess ? PIC_OK : PIC_ERR_CUDA;
}

}  // namespace lin
}  // namespace pic
