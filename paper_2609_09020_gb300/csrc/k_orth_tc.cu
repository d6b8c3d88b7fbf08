// k_orth_tc.cu -- the products of orthogonalised updates on the tensor cores,
// organised as k_linear_tc.cuh's (a ring of stages filled by TMA, one thread that
// issues the MMAs, two sets of accumulators in tensor memory, the epilogue in the other
// warps): all matrices of a list in one launch, each with tensor maps of its own.
//
// Operands are halves of kScale v.  Where values are held in two, a product is three
// products of halves, lo hi, hi lo and hi hi.  At 256 columns each is a run along K of its
// own in the same accumulators, the small ones first: their operands are loaded three
// times, and the loads, 64 bytes a clock into an SM, keep up with the MMAs.  At fewer columns they would
// not (1024 x 1024 fp32, a call: 245 us): both halves of a slice are loaded together, and
// the small products have accumulators of their own.  There an epilogue warp has one panel,
// and takes the sums over into registers every few slices (Job::take), where they are added
// to nearest; at 256 columns it has two, for which there are not enough.
//
// A = X X^T and A^2 are symmetric: tiles on and below the diagonal are computed and
// kept.  Where an operand's slice would lie above it, its mirror image is loaded, which
// lies along the other dimension, and the MMA is told so.  An epilogue reads the old
// X (or A) of its panel, and writes the new one, by TMA through the panel's buffers: the next
// panel is on its way while its sums are awaited.  (By lanes, a row each, the update of four
// 2048 x 2048 and two 2048 x 8192 matrices took 200 us; from and to a copy of its own in fp32
// 175.)  A product with few tiles is cut along K: each part's
// sums go to the workspace, and the warp that is the last to bring its part of a panel
// adds all parts of it in order and finishes it, so that the result does not depend on
// which is last.
//
// Measured, five steps: bf16 four 2048 x 2048 and two 2048 x 8192 matrices 1.31 ms, 1.4 PFLOP/s of
// the operations that there are with symmetry (a step's products 69, 42 and 140 us); fp32 1024 x
// 1024 193 us, some 12 us for each of 15 products that wait on one another.
#include "k_linear_tc.cuh"
#include "orth.cuh"

namespace pic {
namespace orth {
namespace {

using lin::kSlice;

// BOTH: a stage has both halves of its slices.
template <int CG, int BN, bool BOTH>
struct Shape {
  static constexpr int kABytes = 128 * 128, kBRows = BN / CG, kBBytes = kBRows * 128;
  static constexpr int kHalves = BOTH ? 2 : 1;
  static constexpr int kStageBytes = kHalves * (kABytes + kBBytes);
  static constexpr int kCtas = BN == 64 && !BOTH ? 2 : 1;
  static constexpr int kStages = BOTH ? (BN == 64 ? 4 : CG == 2 ? 3 : 2) : BN == 64 ? 3 : 5;
  static constexpr int kEpi = BN == 64 ? 4 : 8;
  static constexpr int kThreads = 64 + 32 * kEpi;
  static constexpr int kColumns = BN == 64 ? 64 : BN / 2;
  static constexpr int kOffPanels = kStages * kStageBytes;  // two halves of each warp
  static constexpr int kOffBars = kOffPanels + kEpi * 2 * lin::kPanelBytes;
  static constexpr int kBars = 2 * kStages + 4 + 1 + kEpi;
  static constexpr int kSmem = kOffBars + kBars * 8 + 16 + 1024;  // 1024: the base is rounded up
  static constexpr int kBufCols = kHalves * BN;  // BOTH: the sums, and those of the small products
  static constexpr int kTmemCols = 2 * kBufCols;
};

template <bool PAIR>
__device__ __forceinline__ void load_3d(uint32_t dst, const void* tmap, int x, int y, int z, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void store_3d(const void* tmap, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}

// Before the use of a tensor map in global memory (made on the host, and copied there).
__device__ __forceinline__ void acquire_map(const void* tmap) {
  asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" ::"l"(reinterpret_cast<uint64_t>(tmap)) : "memory");
}

// 64 halves of a lane's row from a panel's buffer: v += f times them.
__device__ __forceinline__ void add_panel(float (&v)[64], float f, uint32_t buf, int lane) {
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(buf + lane * 128 + ((c ^ (lane & 7)) * 16))
                 : "memory");
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = lin::unpack2_of<__half>(w[e]);
      v[8 * c + 2 * e] = fmaf(f, x.x, v[8 * c + 2 * e]);
      v[8 * c + 2 * e + 1] = fmaf(f, x.y, v[8 * c + 2 * e + 1]);
    }
  }
}
// A panel (32 rows, a lane's row in v, of 64 halves) to its buffer, as TMA takes it.
__device__ __forceinline__ void fill_panel(const uint32_t (&v)[32], uint32_t buf, int lane) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    tc::sts128(buf + lane * 128 + ((c ^ (lane & 7)) * 16), v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
}

// 32 rows x 64 columns of sums to a matrix of type T, turned in the panel buffer so that a
// row's columns leave together.
template <typename T>
__device__ __forceinline__ void put_out(const float (&v)[64], float* turn, int lane, T* out, long long ld, int rows, int cols) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (32 * h >= cols) break;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 32; ++c) turn[lane * 32 + (c ^ lane)] = v[32 * h + c];
    __syncwarp();
    if (32 * h + lane < cols) {
      T* o = out + 32 * h + lane;
#pragma unroll 8
      for (int r = 0; r < rows; ++r) o[r * ld] = lin::from_f32<T>(turn[r * 32 + (lane ^ r)]);
    }
  }
}

template <Stage STAGE, int CG, int BN, bool BOTH>
__global__ void __launch_bounds__(Shape<CG, BN, BOTH>::kThreads, Shape<CG, BN, BOTH>::kCtas)
    stage_kernel(const __grid_constant__ StageParams q) {
  using S = Shape<CG, BN, BOTH>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0;
  const uint32_t bars = base + S::kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * S::kStages, bar_acc = bar_empty + 8 * S::kStages,
                 bar_free = bar_acc + 16, bar_drain = bar_free + 16, bar_in = bar_drain + 8;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::kOffBars + 8 * S::kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kOffBars + 8 * S::kBars + 4);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      tc::mbar_init(bar_full + 8 * s, 1);
      tc::mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(bar_acc + 8 * b, 1);
      tc::mbar_init(bar_free + 8 * b, S::kEpi * CG);
    }
    tc::mbar_init(bar_drain, 1);
    for (int e = 0; e < S::kEpi; ++e) tc::mbar_init(bar_in + 8 * e, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) tc::tmem_alloc_cg<CG>(tc::smem_addr(tmem_slot), S::kTmemCols);
  if (q.n_maps <= kAcquiredFirst)
    for (int i = threadIdx.x; i < q.n_maps; i += blockDim.x) acquire_map(q.maps + i);
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  wait_for_earlier();
  // (a fence takes half a microsecond)
  const bool acquired = q.n_maps <= kAcquiredFirst;

  // Whether slice k of an operand lies along i (j): by itself, or, of a symmetric matrix, as
  // the mirror image of one above the diagonal.
  constexpr int kBlock = 128 * CG;
  const auto lies_along = [](int mn, int half, int at, int k) { return mn != 0 || (half != 0 && k / kBlock > at / kBlock); };
  auto wait = [&](uint32_t bar, uint32_t parity) { return lin::wait_bounded(bar, parity, abort_flag, q.waits); };
  const int first = blockIdx.x / CG, step = gridDim.x / CG;

  int s = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (warp == 0) {
    if (tc::elect_one()) {
      const uint32_t lead_full = CG == 2 ? tc::map_rank(bar_full, 0) : bar_full;
      const CUtensorMap* known[2] = {nullptr, nullptr};
      for (int w = first; w < q.n && ok; w += step) {
        const Job job = q.jobs[w];
        const int i0 = job.i + rank * 128, j0 = job.j + rank * S::kBRows;
        const CUtensorMap* maps = q.maps + static_cast<long long>(job.matrix) * kMaps;
        const auto map_of = [&](int which) { return maps + (which == kMapX ? q.from : which); };
        const CUtensorMap *mp = map_of(job.p_map), *mq = map_of(job.q_map);
        if (!acquired && mp != known[0]) acquire_map(mp);
        if (!acquired && mq != known[1]) acquire_map(mq);
        known[0] = mp, known[1] = mq;
        const int k0 = job.k0, k1 = job.k1;
        for (int term = !BOTH && job.halves == 2 ? 0 : 2; term < 3 && ok; ++term) {
          const int zp = term == 0, zq = term == 1, halves = BOTH ? job.halves : 1;
          for (int kb = k0; kb < k1; ++kb) {
            if (!(ok = wait(bar_empty + 8 * s, phase ^ 1))) break;
            if (rank == 0) tc::mbar_arrive_expect_tx(bar_full + 8 * s, CG * halves * (S::kABytes + S::kBBytes));
            const uint32_t bar = lead_full + 8 * s;
            const int k = kb * kSlice;
            const bool p_mn = lies_along(job.p_mn, job.p_half, job.i, k), q_mn = lies_along(job.q_mn, job.q_half, job.j, k);
            // boxes of 64 x 64 either way
            for (int h = 0; h < halves; ++h) {
              const uint32_t sa = base + s * S::kStageBytes + h * S::kABytes,
                             sb = base + s * S::kStageBytes + S::kHalves * S::kABytes + h * S::kBBytes;
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                if (p_mn)
                  load_3d<CG == 2>(sa + c * 8192, mp, i0 + 64 * c, k, zp + h, bar);
                else
                  load_3d<CG == 2>(sa + c * 8192, mp, k, i0 + 64 * c, zp + h, bar);
              }
#pragma unroll
              for (int c = 0; c < S::kBRows / 64; ++c) {
                if (q_mn)
                  load_3d<CG == 2>(sb + c * 8192, mq, j0 + 64 * c, k, zq + h, bar);
                else
                  load_3d<CG == 2>(sb + c * 8192, mq, k, j0 + 64 * c, zq + h, bar);
              }
            }
            if (++s == S::kStages) s = 0, phase ^= 1;
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && tc::elect_one()) {
      int buf = 0;
      uint32_t free_phase = 0;
      for (int w = first; w < q.n && ok; w += step) {
        const Job job = q.jobs[w];  // (a copy: through memory each slice would read it again)
        const bool two = BOTH && job.halves == 2;
        const int k0 = job.k0, k1 = job.k1, slices = (k1 - k0) * (!BOTH && job.halves == 2 ? 3 : 1), each = two ? job.take : slices;
        for (int n0 = 0, kb = k0; n0 < slices && ok; n0 += each) {
          if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * S::kBufCols;
          for (int n = n0; n < min(slices, n0 + each); ++n) {
            const bool p_mn = lies_along(job.p_mn, job.p_half, job.i, kb * kSlice),
                       q_mn = lies_along(job.q_mn, job.q_half, job.j, kb * kSlice);
            if (++kb == k1) kb = k0;
            const uint32_t idesc = tc::idesc_16(128 * CG, BN, false, p_mn, q_mn);
            // one MMA takes 16 of K: 32 bytes of a K-major row, 16 rows of an MN-major block
            const uint32_t a_step = p_mn ? 2048 : 32, b_step = q_mn ? 2048 : 32;
            if (!(ok = wait(bar_full + 8 * s, phase))) break;
            tc::tc_fence_after();
            const uint32_t sa = base + s * S::kStageBytes, sb = sa + S::kHalves * S::kABytes;
            const auto multiply = [&](uint32_t to, uint32_t a, uint32_t b, bool begin) {
#pragma unroll
              for (int kk = 0; kk < kSlice / 16; ++kk)
                tc::mma_16<CG>(to, tc::smem_desc_sw128(a + kk * a_step, 8192, 1024),
                               tc::smem_desc_sw128(b + kk * b_step, 8192, 1024), idesc, (!begin || kk > 0) ? 1u : 0u);
            };
            if (two) {
              multiply(d + BN, sa + S::kABytes, sb, n == n0);
              multiply(d + BN, sa, sb + S::kBBytes, false);
            }
            multiply(d, sa, sb, n == n0);
            tc::mma_commit_cg<CG>(bar_empty + 8 * s);
            if (++s == S::kStages) s = 0, phase ^= 1;
          }
          if (!ok) break;
          tc::mma_commit_cg<CG>(bar_acc + 8 * buf);
          if (++buf == 2) buf = 0, free_phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;  // the 32 lanes of tensor memory that this warp may read
    const int from = (warp - 2) / 4 * S::kColumns, to = from + S::kColumns;
    uint8_t* buffers = smem + S::kOffPanels + (warp - 2) * 2 * lin::kPanelBytes;
    const uint32_t buffer = tc::smem_addr(buffers), here = bar_in + 8 * (warp - 2);
    const uint32_t lead_free = CG == 2 ? tc::map_rank(bar_free, 0) : bar_free;
    const int below = rank * 128 + quarter * 32;  // rows of the tile above this warp's
    int buf = 0;
    uint32_t in_phase = 0;
    bool coming = false;  // the old values of the panel that is next
    const CUtensorMap *read = nullptr, *written = nullptr;
    const auto inside = [&](const Job& job, const Matrix& m, int c0) {
      return job.i + below < (STAGE == kUpdate ? m.rows : m.m) && job.j + c0 < (STAGE == kUpdate ? m.cols : m.m);
    };
    // sends for the old values of a panel: X, or A
    const auto fetch = [&](const Job& job, const Matrix& m, int c0) {
      coming = true;
      if (lane != 0) return;
      const CUtensorMap* map = q.maps + static_cast<long long>(job.matrix) * kMaps + kMapPanel + (STAGE == kUpdate ? q.from : kMapA);
      if (!acquired && map != read) acquire_map(map);
      read = map;
      const int n = STAGE == kUpdate ? (m.halves == 2 || q.lo_from ? 2 : 1) : m.halves;
      tc::bulk_wait_read<0>();  // the buffers' last stores have been read
      tc::mbar_arrive_expect_tx(here, n * lin::kPanelBytes);
      for (int z = 0; z < n; ++z) load_3d<false>(buffer + z * lin::kPanelBytes, map, job.j + c0, job.i + below, z, here);
    };
    // whether a panel's old values can be sent for before its sums are there
    const auto ahead = [&](const Job& job, const Matrix& m, int c0) {
      return STAGE != kGram && job.parts == 1 && inside(job, m, c0);
    };
    if (first < q.n) {
      const Job& job = q.jobs[first];
      const Matrix& m = q.matrices[job.matrix];
      if (ahead(job, m, from)) fetch(job, m, from);
    }
    for (int w = first; w < q.n; w += step) {
      const Job& job = q.jobs[w];
      const Matrix& m = q.matrices[job.matrix];
      const int I = STAGE == kUpdate ? m.rows : m.m, J = STAGE == kUpdate ? m.cols : m.m;
      const int row0 = job.i + below, parts = job.parts;
      const bool two_halves = BOTH && job.halves == 2;
      const int k0 = job.k0, k1 = job.k1, each = two_halves ? job.take : k1 - k0;
      static_assert(!BOTH || S::kColumns == 64, "a warp's sums stay in its registers");
      for (int c0 = from; c0 < to && ok; c0 += 64) {
        float v[64];
        for (int k = k0; k < k1; k += each) {
          if (c0 == from) {
            ok = __all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase));
            if (!ok) break;
            tc::tc_fence_after();
          }
          const uint32_t d = tmem + buf * S::kBufCols + (static_cast<uint32_t>(quarter * 32) << 16) + c0;
          if (k == k0) {
            uint32_t sums[64];
            tc::tmem_ld64_wait(d, sums);
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] = __uint_as_float(sums[c]);
          } else {
#pragma unroll
            for (int h = 0; h < 64; h += 32) {
              uint32_t sums[32];
              tc::tmem_ld32_wait(d + h, sums);
#pragma unroll
              for (int c = 0; c < 32; ++c) v[h + c] += __uint_as_float(sums[c]);
            }
          }
          if (two_halves) {
#pragma unroll
            for (int h = 0; h < 64; h += 32) {
              uint32_t small[32];
              tc::tmem_ld32_wait(d + BN + h, small);
#pragma unroll
              for (int c = 0; c < 32; ++c) v[h + c] += __uint_as_float(small[c]);
            }
          }
          if (c0 + 64 == to) {
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0 && !(q.waits.test_fault && w == 0 && rank == 0 && quarter == 0)) {
              if constexpr (CG == 2)
                tc::mbar_arrive_cluster(lead_free + 8 * buf);
              else
                tc::mbar_arrive(bar_free + 8 * buf);
            }
            if (++buf == 2) buf = 0, phase ^= 1;
          }
        }
        if (!ok) break;
        const int col0 = job.j + c0, cols = min(64, J - col0);
        bool mine = inside(job, m, c0);
        if (mine && parts > 1) {
          // [part][rank][panel][quarter][16][32 lanes][4 columns]
          constexpr int kPanels = CG * (BN / 64) * 4;  // warps' panels of a tile
          const int panel = (rank * (BN / 64) + c0 / 64) * 4 + quarter;
          float4* o = q.parts + (static_cast<long long>(job.slot + job.part) * kPanels + panel) * 512 + lane;
#pragma unroll
          for (int c = 0; c < 16; ++c) __stcg(o + c * 32, make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]));
          __threadfence();
          __syncwarp();
          unsigned* counter = q.counters + static_cast<long long>(job.slot) * kPanels + panel;
          unsigned before = 0;
          if (lane == 0) before = atomicAdd(counter, 1);
          before = __shfl_sync(0xffffffffu, before, 0);
          mine = before + 1 == static_cast<unsigned>(parts);  // else others bring theirs later
          if (mine) {
            if (STAGE != kGram) fetch(job, m, c0);
            __threadfence();
            if (lane == 0) *counter = 0;  // for the next launch
            const float4* all = q.parts + (static_cast<long long>(job.slot) * kPanels + panel) * 512 + lane;
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] = 0.0f;
            for (int p = 0; p < parts; ++p, all += kPanels * 512) {
#pragma unroll
              for (int c = 0; c < 16; ++c) {
                const float4 f = __ldcg(all + c * 32);
                v[4 * c] += f.x, v[4 * c + 1] += f.y, v[4 * c + 2] += f.z, v[4 * c + 3] += f.w;
              }
            }
          }
        }
        if (mine) {
          const bool two = m.halves == 2 || (STAGE == kUpdate && q.lo_to), two_old = m.halves == 2 || (STAGE == kUpdate && q.lo_from);
          // X is the first one's times `rest`
          const float rest = STAGE != kPolynomial && q.first ? *m.rest : 1.0f;
          const float f = (STAGE == kPolynomial ? q.co.c : STAGE == kGram ? rest * rest : rest) / kScale;
#pragma unroll
          for (int c = 0; c < 64; ++c) v[c] *= f;
          if constexpr (STAGE != kGram) {
            if (!__all_sync(0xffffffffu, wait(here, in_phase))) {
              ok = false;
              break;
            }
            in_phase ^= 1;
            coming = false;
            const float o = STAGE == kPolynomial ? q.co.b : q.co.a * rest;
            if (two_old) add_panel(v, o, buffer + lin::kPanelBytes, lane);
            add_panel(v, o, buffer, lane);
          } else {
            if (lane == 0) tc::bulk_wait_read<0>();
          }
          __syncwarp();
          if (STAGE == kUpdate && q.last) {
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] *= 1.0f / kScale;
            const int rows = min(32, I - row0);
            const long long at = row0 * m.ld_out + col0;
            float* turn = reinterpret_cast<float*>(buffers);
            if (m.dtype == PIC_DTYPE_F32)
              put_out(v, turn, lane, static_cast<float*>(m.out) + at, m.ld_out, rows, cols);
            else if (m.dtype == PIC_DTYPE_F16)
              put_out(v, turn, lane, static_cast<__half*>(m.out) + at, m.ld_out, rows, cols);
            else
              put_out(v, turn, lane, static_cast<__nv_bfloat16*>(m.out) + at, m.ld_out, rows, cols);
            tc::fence_async_smem();
            __syncwarp();
          } else {
            uint32_t half[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) half[c] = lin::pack2_of<__half>(v[2 * c], v[2 * c + 1]);
            fill_panel(half, buffer, lane);
            if (two) {
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                const float2 h = lin::unpack2_of<__half>(half[c]);
                half[c] = lin::pack2_of<__half>(v[2 * c] - h.x, v[2 * c + 1] - h.y);
              }
              fill_panel(half, buffer + lin::kPanelBytes, lane);
            }
            tc::fence_async_smem();
            __syncwarp();
            if (lane == 0) {
              const CUtensorMap* map = q.maps + static_cast<long long>(job.matrix) * kMaps + kMapPanel +
                                       (STAGE == kUpdate ? q.from ^ 1 : STAGE == kGram ? kMapA : kMapB);
              if (!acquired && map != written) acquire_map(map);
              written = map;
              store_3d(map, col0, row0, 0, buffer);
              if (two) store_3d(map, col0, row0, 1, buffer + lin::kPanelBytes);
              tc::bulk_commit();
            }
          }
        }
        if (c0 + 64 < to) {
          if (ahead(job, m, c0 + 64)) fetch(job, m, c0 + 64);
        } else if (w + step < q.n) {
          const Job& next = q.jobs[w + step];
          const Matrix& nm = q.matrices[next.matrix];
          if (ahead(next, nm, from)) fetch(next, nm, from);
        }
      }
      if (!ok) break;
    }
    if (lane == 0) {
      tc::bulk_wait_all();
      // after an abort: what has been sent for and not awaited
      for (uint32_t i = 0; coming && i < q.waits.spin_limit && !tc::mbar_try_wait(here, in_phase); ++i) {
      }
    }
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies and MMAs in flight use shared and tensor memory.  The other CTA of a
    // pair may have started copies that this one did not expect: it lingers for far
    // longer than a copy takes.
    if (warp == 0 && rank == 0 && tc::elect_one()) lin::drain_loads(bar_full, S::kStages, s, phase, q.waits);
    if (warp == 1 && rank == 0 && tc::elect_one()) lin::drain_mmas<CG>(bar_drain, q.waits);
    if (CG == 2) __nanosleep(200000);
    __syncthreads();
  }
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  if (warp == 1) tc::tmem_dealloc_cg<CG>(tmem, S::kTmemCols);
}

template <Stage STAGE, int CG, int BN, bool BOTH>
int launch(const StageParams& q, int slot, lin::Chain& s) {
  using S = Shape<CG, BN, BOTH>;
  static_assert((S::kSmem + 1024) * S::kCtas <= 228 * 1024, "shared memory of an SM");
  const void* fn = reinterpret_cast<const void*>(stage_kernel<STAGE, CG, BN, BOTH>);
  if (lin::allow_smem(fn, slot, S::kSmem) != PIC_OK) return PIC_ERR_CUDA;
  const long long want = static_cast<long long>(q.n) * CG, most = 152 * S::kCtas;
  void* args[] = {const_cast<StageParams*>(&q)};
  return s.launch(fn, dim3(static_cast<unsigned>(want < most ? want : most)), S::kThreads, S::kSmem, CG, args);
}

template <Stage STAGE>
int launch_shape(TileShape shape, bool both, const StageParams& q, lin::Chain& s) {
  if (shape == k64) return both ? launch<STAGE, 1, 64, true>(q, 64 + STAGE, s) : launch<STAGE, 1, 64, false>(q, 44 + STAGE, s);
  if (shape == k128) return both ? launch<STAGE, 1, 128, true>(q, 67 + STAGE, s) : launch<STAGE, 1, 128, false>(q, 47 + STAGE, s);
  if constexpr (STAGE != kUpdate)
    if (shape == kPair128) return launch<STAGE, 2, 128, true>(q, 75 + STAGE, s);
  return launch<STAGE, 2, 256, false>(q, 50 + STAGE, s);
}

}  // namespace

int launch_stage(Stage stage, TileShape shape, bool both, const StageParams& q, lin::Chain& s) {
  if (q.n == 0) return PIC_OK;
  if (stage == kGram) return launch_shape<kGram>(shape, both, q, s);
  if (stage == kPolynomial) return launch_shape<kPolynomial>(shape, both, q, s);
  return launch_shape<kUpdate>(shape, both, q, s);
}

}  // namespace orth
}  // namespace pic
