// k_group_tc.cuh -- grouped matrix products of 16-bit operands on the tensor cores,
// organised as k_linear_tc.cuh's: a ring of stages (64 of K) that one thread fills by
// TMA, one thread that issues the MMAs, two sets of accumulators in tensor memory, and
// the epilogue in the other warps under the next tile's MMAs.  What groups change:
//
//   kRows   C[i][j] = sum_k A(i, k) B_g(j, k): a tile is 128 or 256 rows of one group.
//           Rows behind the group's are loaded with it (rows of a product do not meet)
//           and not stored: panels of 32 rows that end inside go out by plain stores.
//   kSums   C_g[i][j] = sum over the group's rows of A(k, i) B(k, j): each group has
//           tensor maps of its own, which end with it, so that what is behind its last
//           row reads as zero in both operands.  Groups of more than `chunk` rows are
//           cut: parts in fp32, joined in order by a second kernel.
//   kTurned kRows with few rows in a group: the weights are the operand with 128
//           rows, the group's rows the one with BN, so that next to nothing but the
//           weights is loaded.  An epilogue lane has a column of y.
//
// Every CTA makes the table of groups from the offsets in shared memory, so that a call
// is one launch and needs no order of its CTAs.
//
// Measured: bf16 8192 x 4096 -> 4096 GELU in 8 uneven groups 184 us, 1.5 PFLOP/s (of 576 tiles
// of 256 x 256, an eighth are groups' last ones, and 76 pairs take eight rounds of them; with six
// stages, for which the table leaves no room, 181); the sums 171 us; 64 groups, half of them
// with 96 rows together, 2048 -> 4096 80 us, 6.3 TB/s of weights; fp16 1000000 x 64 -> 64 keeping
// z 67 us, 5.7 TB/s.
#pragma once

#include "group.cuh"
#include "k_linear_tc.cuh"

namespace pic {
namespace grp {

using lin::kSlice;

enum TcMode { kRows = 0, kSums = 1, kTurned = 2 };

struct GtMaps {
  CUtensorMap a, b, y, pre;  // kSums: a and b as the groups' maps begin
};

struct GtParams {
  long long rows;     // of all groups, and around them
  long long I, J, K;  // kSums: I; else K
  long long tiles_i, tiles_j;  // kTurned: columns of y are tiles_i; kSums: of one group
  int groups;
  const long long* offsets;
  int b_mn;           // kRows: the weights lie along j; kTurned: the same, they are A
  int chunk;          // kSums: rows of a part, a multiple of 64
  int store_tma;
  const CUtensorMap* maps;  // kSums: [groups][2]
  float* parts;       // kSums
  const void* bias;
  long long bias_group;
  void* y;
  long long ldy, y_group;
  void* pre;
  long long ldpre;
  int act;
  Waits waits;
};

// As lin::TcShape, with room for the table of groups.
template <int CG, int BN, TcMode MODE>
struct GtShape {
  static constexpr bool kTurn = MODE == kTurned;
  static constexpr int kRowsOfTile = 128 * CG;
  static constexpr int kBRows = BN / CG;
  static constexpr int kABytes = 128 * 128, kBBytes = kBRows * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kCtas = BN <= 64 ? 2 : 1;
  static constexpr int kStages = kTurn ? (BN == 64 ? 4 : 5) : BN == 64 ? 3 : 5;
  static constexpr int kEpi = BN <= 64 ? 4 : 8;
  static constexpr int kThreads = 64 + 32 * kEpi;
  static constexpr int kColumns = BN <= 64 ? BN : BN / 2;
  static constexpr int kPanelBytes = kTurn ? 0 : lin::kPanelBytes;
  static constexpr int kOffPanels = kStages * kStageBytes;
  static constexpr int kOffTable = kOffPanels + kEpi * kPanelBytes;
  static constexpr int kOffBars = (kOffTable + static_cast<int>(sizeof(GroupTable)) + 15) / 16 * 16;
  static constexpr int kBars = 2 * kStages + 4 + 1;
  static constexpr int kSmem = kOffBars + kBars * 8 + 16 + 1024;  // 1024: the base is rounded up
  static constexpr int kBufCols = BN < 32 ? 32 : BN;              // of an accumulator
  static constexpr int kTmemCols = 2 * kBufCols;
};

template <bool PAIR>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int x, int y, int z, uint32_t bar) {
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
__device__ __forceinline__ void tma_store_3d(const void* tmap, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}
// Before the use of a tensor map in global memory that an earlier kernel wrote.
__device__ __forceinline__ void acquire_map(const void* tmap) {
  asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(reinterpret_cast<uint64_t>(tmap)) : "memory");
}

// One warp's panel (32 rows, 128 bytes of columns from col0; this lane's row in v)
// through the panel buffer: by TMA (two or three coordinates), or, of `rows` rows from
// `out` on, one word of a row per lane and row.
template <typename T, bool THREE>
__device__ __forceinline__ void put_rows(const uint32_t (&v)[32], uint32_t buf, int lane, T* out, long long ld, int rows,
                                         int cols, const CUtensorMap* map, int x, int y, int z, bool by_tma) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    tc::sts128(buf + lane * 128 + ((c ^ (lane & 7)) * 16), v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
  if (by_tma) {
    tc::fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      if constexpr (THREE)
        tma_store_3d(map, x, y, z, buf);
      else
        tc::tma_store_2d(map, x, y, buf);
      tc::bulk_commit();
    }
    return;
  }
  __syncwarp();
#pragma unroll 8
  for (int r = 0; r < rows; ++r, out += ld) {
    const uint32_t w = lin::panel_word(buf, r, lane);
    // words of two columns where the row's words lie: columns 2 l, 2 l + 1, or
    // 2 l + 1, 2 l + 2 of a row that starts in the middle of one
    uint16_t* h = reinterpret_cast<uint16_t*>(out) + 2 * lane;
    if ((reinterpret_cast<uintptr_t>(out) & 2) == 0) {
      if (2 * lane + 1 < cols)
        *reinterpret_cast<uint32_t*>(h) = w;
      else if (2 * lane < cols)
        h[0] = static_cast<uint16_t>(w);
    } else {
      const uint32_t next = __shfl_down_sync(0xffffffffu, w, 1);
      if (lane == 0) h[0] = static_cast<uint16_t>(w);
      if (lane < 31 && 2 * lane + 2 < cols)
        *reinterpret_cast<uint32_t*>(h + 1) = w >> 16 | next << 16;
      else if (2 * lane + 1 < cols)
        h[1] = static_cast<uint16_t>(w >> 16);
    }
  }
  __syncwarp();
  if (lane == 0) tc::bulk_commit();  // an empty group: every panel has one, so that waits can count them
}

// What a work item is.
struct GtItem {
  int g, first, len;    // the group, its first row and its rows
  long long ti, tj;
  int k0, k1;           // slices
  int item;             // kSums: the group's part
  bool whole;           // kSums: the group's only one
};

template <int CG, int BN, TcMode MODE>
__device__ __forceinline__ long long work_of(const GtParams& q, const GroupTable& t) {
  if constexpr (MODE == kRows) return t.tiles[q.groups] * q.tiles_j;
  if constexpr (MODE == kTurned) return t.tiles[q.groups] * q.tiles_i;
  return t.tiles[q.groups] * (q.tiles_i * q.tiles_j);
}
template <int CG, int BN, TcMode MODE>
__device__ __forceinline__ GtItem item_of(const GtParams& q, const GroupTable& t, long long w) {
  GtItem m;
  if constexpr (MODE == kSums) {
    const long long per = q.tiles_i * q.tiles_j;
    m.item = static_cast<int>(w / per);
    m.g = t.find(m.item, q.groups);
    lin::tile_place<128 * CG>(w % per, q.tiles_i, q.tiles_j, m.ti, m.tj);
    const int part = m.item - t.tiles[m.g];
    m.first = t.start[m.g], m.len = t.rows(m.g);
    m.whole = m.len <= q.chunk;
    m.k0 = part * (q.chunk / kSlice);
    m.k1 = min((m.len + kSlice - 1) / kSlice, m.k0 + q.chunk / kSlice);
  } else {
    long long rt;
    if constexpr (MODE == kRows) {
      lin::tile_place<128 * CG>(w, t.tiles[q.groups], q.tiles_j, rt, m.tj);
    } else {
      rt = w / q.tiles_i;
      m.ti = w % q.tiles_i;
    }
    m.g = t.find(static_cast<int>(rt), q.groups);
    (MODE == kRows ? m.ti : m.tj) = rt - t.tiles[m.g];
    m.first = t.start[m.g], m.len = t.rows(m.g);
    m.k0 = 0, m.k1 = static_cast<int>((q.K + kSlice - 1) / kSlice);
  }
  return m;
}

template <typename T, int CG, int BN, TcMode MODE>
__global__ void __launch_bounds__(GtShape<CG, BN, MODE>::kThreads, GtShape<CG, BN, MODE>::kCtas)
    group_kernel(const __grid_constant__ GtParams q, const __grid_constant__ GtMaps maps) {
  using S = GtShape<CG, BN, MODE>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_addr(smem_raw);
  uint8_t* smem = smem_raw + ((1024 - (raw & 1023)) & 1023);
  const uint32_t base = tc::smem_addr(smem);
  GroupTable& table = *reinterpret_cast<GroupTable*>(smem + S::kOffTable);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0;
  const uint32_t bars = base + S::kOffBars;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * S::kStages, bar_acc = bar_empty + 8 * S::kStages,
                 bar_free = bar_acc + 16, bar_drain = bar_free + 16;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::kOffBars + 8 * S::kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kOffBars + 8 * S::kBars + 4);

  if (threadIdx.x == 0) {
    if (MODE != kSums) {
      tc::prefetch_map(&maps.a);
      tc::prefetch_map(&maps.b);
    }
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
  make_table(table, q.offsets, q.groups, q.rows, MODE == kSums ? q.chunk : MODE == kTurned ? BN : 128 * CG,
             MODE == kSums ? 1 : 0, q.waits.status);
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  wait_for_earlier();

  auto wait = [&](uint32_t bar, uint32_t parity) { return lin::wait_bounded(bar, parity, abort_flag, q.waits); };
  const long long first = blockIdx.x / CG, step = gridDim.x / CG, work = work_of<CG, BN, MODE>(q, table);

  int s = 0;
  uint32_t phase = 0;
  bool ok = true;
  if (warp == 0) {
    if (tc::elect_one()) {
      const uint32_t lead_full = CG == 2 ? tc::map_rank(bar_full, 0) : bar_full;
      int known = -1;  // kSums: the group whose maps have been acquired
      for (long long w = first; w < work && ok; w += step) {
        const GtItem m = item_of<CG, BN, MODE>(q, table, w);
        const CUtensorMap *ma = &maps.a, *mb = &maps.b;
        int i0 = static_cast<int>(m.ti * S::kRowsOfTile + rank * 128), j0 = static_cast<int>(m.tj * BN + rank * S::kBRows);
        if constexpr (MODE == kRows) i0 += m.first;
        if constexpr (MODE == kTurned) j0 += m.first;
        if constexpr (MODE == kSums) {
          ma = q.maps + 2 * m.g, mb = ma + 1;
          if (known != m.g && m.k0 < m.k1) {
            acquire_map(ma);
            acquire_map(mb);
            known = m.g;
          }
        }
        for (int kb = m.k0; kb < m.k1; ++kb) {
          if (!(ok = wait(bar_empty + 8 * s, phase ^ 1))) break;
          if (rank == 0) tc::mbar_arrive_expect_tx(bar_full + 8 * s, CG * S::kStageBytes);
          const uint32_t sa = base + s * S::kStageBytes, sb = sa + S::kABytes, bar = lead_full + 8 * s;
          const int k = kb * kSlice;
          if constexpr (MODE == kSums) {
#pragma unroll
            for (int c = 0; c < 2; ++c) tc::tma_load_2d<CG == 2>(sa + c * 8192, ma, i0 + 64 * c, m.first + k, bar);
#pragma unroll
            for (int c = 0; c < S::kBRows / 64; ++c)
              tc::tma_load_2d<CG == 2>(sb + c * 8192, mb, j0 + 64 * c, m.first + k, bar);
          } else if constexpr (MODE == kRows) {
            tc::tma_load_2d<CG == 2>(sa, ma, k, i0, bar);
            if (q.b_mn) {
#pragma unroll
              for (int c = 0; c < S::kBRows / 64; ++c)
                tma_load_3d<CG == 2>(sb + c * 8192, mb, j0 + 64 * c, k, m.g, bar);
            } else {
              tma_load_3d<CG == 2>(sb, mb, k, j0, m.g, bar);
            }
          } else {
            if (q.b_mn) {
#pragma unroll
              for (int c = 0; c < 2; ++c) tma_load_3d<false>(sa + c * 8192, ma, i0 + 64 * c, k, m.g, bar);
            } else {
              tma_load_3d<false>(sa, ma, k, i0, m.g, bar);
            }
            tc::tma_load_2d<false>(sb, mb, k, j0, bar);
          }
          if (++s == S::kStages) s = 0, phase ^= 1;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && tc::elect_one()) {
      const bool a_mn = MODE == kSums || (MODE == kTurned && q.b_mn), b_mn = MODE == kSums || (MODE == kRows && q.b_mn);
      const uint32_t idesc = lin::idesc_of<T>(128 * CG, BN, a_mn, b_mn);
      // one MMA takes 16 of K: 32 bytes of a K-major row, 16 rows of an MN-major block
      const uint32_t a_step = a_mn ? 2048 : 32, b_step = b_mn ? 2048 : 32;
      int buf = 0;
      uint32_t free_phase = 0;
      for (long long w = first; w < work && ok; w += step) {
        const GtItem m = item_of<CG, BN, MODE>(q, table, w);
        if (m.k0 >= m.k1) continue;
        if (!(ok = wait(bar_free + 8 * buf, free_phase ^ 1))) break;
        tc::tc_fence_after();
        const uint32_t d = tmem + buf * S::kBufCols;
        for (int kb = m.k0; kb < m.k1; ++kb) {
          if (!(ok = wait(bar_full + 8 * s, phase))) break;
          tc::tc_fence_after();
          const uint32_t sa = base + s * S::kStageBytes, sb = sa + S::kABytes;
#pragma unroll
          for (int kk = 0; kk < kSlice / 16; ++kk)
            tc::mma_16<CG>(d, tc::smem_desc_sw128(sa + kk * a_step, 8192, 1024),
                           tc::smem_desc_sw128(sb + kk * b_step, 8192, 1024), idesc, (kb > m.k0 || kk > 0) ? 1u : 0u);
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
    const int from = (warp - 2) / 4 * S::kColumns, to = from + S::kColumns;
    const uint32_t panel = base + S::kOffPanels + (warp - 2) * S::kPanelBytes;
    const uint32_t lead_free = CG == 2 ? tc::map_rank(bar_free, 0) : bar_free;
    int buf = 0;
    for (long long w = first; w < work; w += step) {
      const GtItem m = item_of<CG, BN, MODE>(q, table, w);
      const bool empty = m.k0 >= m.k1;  // kSums: a group without rows
      if (!empty) {
        if (!__all_sync(0xffffffffu, wait(bar_acc + 8 * buf, phase))) break;
        tc::tc_fence_after();
      }
      const uint32_t d = tmem + buf * S::kBufCols + (static_cast<uint32_t>(quarter * 32) << 16);
      const auto release = [&] {
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0 && !(q.waits.test_fault && w == 0 && rank == 0 && quarter == 0)) {
          if constexpr (CG == 2)
            tc::mbar_arrive_cluster(lead_free + 8 * buf);
          else
            tc::mbar_arrive(bar_free + 8 * buf);
        }
      };
      if constexpr (MODE == kTurned) {
        float v[BN];
        if constexpr (BN == 16) {
          uint32_t r[16];
          tc::tmem_ld16(d, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < BN; ++c) v[c] = __uint_as_float(r[c]);
        } else {
#pragma unroll
          for (int c0 = 0; c0 < BN; c0 += 32) {
            uint32_t r[32];
            tc::tmem_ld32_wait(d + c0, r);
#pragma unroll
            for (int c = 0; c < 32; ++c) v[c0 + c] = __uint_as_float(r[c]);
          }
        }
        release();
        const long long col = m.ti * 128 + quarter * 32 + lane;  // of y
        const int rows = min(BN, m.len - static_cast<int>(m.tj) * BN);
        const long long row = m.first + m.tj * BN;
        if (col < q.J) {
          const float bias = q.bias ? lin::to_f32(static_cast<const T*>(q.bias)[m.g * q.bias_group + col]) : 0.0f;
          T* y = static_cast<T*>(q.y) + row * q.ldy + col;
          T* pre = q.pre ? static_cast<T*>(q.pre) + row * q.ldpre + col : nullptr;
#pragma unroll
          for (int c = 0; c < BN; ++c) {
            if (c >= rows) break;
            const float z = v[c] + bias;
            if (pre) pre[c * q.ldpre] = lin::from_f32<T>(z);
            y[c * q.ldy] = lin::from_f32<T>(lin::act_value<false>(z, q.act));
          }
        }
      } else {
        const long long row0 = m.ti * S::kRowsOfTile + rank * 128 + quarter * 32, j0 = m.tj * BN;
        const int limit = MODE == kRows ? m.len : static_cast<int>(q.I);
        const int rows = static_cast<int>(min(32LL, limit - row0));
        // a TMA store leaves out what is outside the matrix, not what is outside the group
        const bool by_tma = q.store_tma && (MODE == kSums || rows == 32);
        for (int c0 = from; c0 < to; c0 += 64) {
          uint32_t raw_acc[64];
          if (empty) {
#pragma unroll
            for (int c = 0; c < 64; ++c) raw_acc[c] = 0;
          } else {
            tc::tmem_ld64_wait(d + c0, raw_acc);
            if (c0 + 64 == to) release();
          }
          if constexpr (MODE == kSums) {
            if (!m.whole) {
              // the group's part, this tile, panel c0 / 64, this warp's 32 rows: [16][32 lanes][4 columns]
              float4* o = reinterpret_cast<float4*>(q.parts) +
                          (((part_slot(table, m.g, m.item, q.chunk, lane) * q.tiles_i + m.ti) * q.tiles_j + m.tj) * CG + rank) * (BN / 64) * (128 * 16) +
                          c0 / 64 * (128 * 16) + quarter * (32 * 16) + lane;
#pragma unroll
              for (int c = 0; c < 16; ++c)
                o[c * 32] = make_float4(__uint_as_float(raw_acc[4 * c]), __uint_as_float(raw_acc[4 * c + 1]),
                                        __uint_as_float(raw_acc[4 * c + 2]), __uint_as_float(raw_acc[4 * c + 3]));
              continue;
            }
          }
          if (rows <= 0 || j0 + c0 >= q.J) continue;  // nothing of this panel is inside
          float v[64];
#pragma unroll
          for (int c = 0; c < 64; ++c) v[c] = __uint_as_float(raw_acc[c]);
          const int cols = static_cast<int>(min(64LL, q.J - j0 - c0));
          if (q.bias) lin::add_row<T>(v, static_cast<const T*>(q.bias) + m.g * q.bias_group + j0 + c0, cols);
          const long long row = MODE == kRows ? m.first + row0 : row0;
          uint32_t out[32];
          if (q.pre) {
#pragma unroll
            for (int c = 0; c < 32; ++c) out[c] = lin::pack2_of<T>(v[2 * c], v[2 * c + 1]);
            if (lane == 0) tc::bulk_wait_read<0>();  // the buffer's last store has been read
            __syncwarp();
            put_rows<T, false>(out, panel, lane, static_cast<T*>(q.pre) + row * q.ldpre + j0 + c0, q.ldpre, rows, cols,
                               &maps.pre, static_cast<int>(j0 + c0), static_cast<int>(row), 0, by_tma);
          }
          if (q.act == PIC_ACT_GELU) {
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
              const float2 r = unpack2(gelu_approx2(pack2(v[c], v[c + 1])));
              v[c] = r.x;
              v[c + 1] = r.y;
            }
          } else if (q.act == PIC_ACT_RELU) {
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] = relu_nan(v[c]);
          }
#pragma unroll
          for (int c = 0; c < 32; ++c) out[c] = lin::pack2_of<T>(v[2 * c], v[2 * c + 1]);
          if (lane == 0) tc::bulk_wait_read<0>();
          __syncwarp();
          T* y = static_cast<T*>(q.y) + (MODE == kSums ? m.g * q.y_group : 0) + row * q.ldy + j0 + c0;
          put_rows<T, MODE == kSums>(out, panel, lane, y, q.ldy, rows, cols, &maps.y, static_cast<int>(j0 + c0),
                                     static_cast<int>(row), m.g, by_tma);
        }
      }
      if (!empty && ++buf == 2) buf = 0, phase ^= 1;
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
    if (warp == 0 && rank == 0 && tc::elect_one()) lin::drain_loads(bar_full, S::kStages, s, phase, q.waits);
    if (warp == 1 && rank == 0 && tc::elect_one()) lin::drain_mmas<CG>(bar_drain, q.waits);
    if (CG == 2) __nanosleep(200000);
    __syncthreads();
  }
  if constexpr (CG == 2) tc::cluster_sync();
  tc::tc_fence_after();
  if (warp == 1) tc::tmem_dealloc_cg<CG>(tmem, S::kTmemCols);
}

// The kernel for tiles of bn columns (kTurned: rows of a group), and what it is launched with.
struct GtKernel {
  const void* fn;
  int threads, smem, cg, ctas, slot;
};
GtKernel group_kernel_f16(TcMode mode, int bn);
GtKernel group_kernel_bf16(TcMode mode, int bn);

template <typename T, int CG, int BN, TcMode MODE>
GtKernel group_kernel_info(int slot) {
  using S = GtShape<CG, BN, MODE>;
  static_assert(S::kSmem * S::kCtas + 1024 * S::kCtas <= 228 * 1024 && S::kSmem <= 227 * 1024, "shared memory of an SM");
  return {reinterpret_cast<const void*>(group_kernel<T, CG, BN, MODE>), S::kThreads, S::kSmem, CG, S::kCtas, slot};
}
template <typename T>
GtKernel group_kernel_of(TcMode mode, int bn, int slot0) {
  if (mode == kTurned) {
    if (bn == 16) return group_kernel_info<T, 1, 16, kTurned>(slot0);
    if (bn == 32) return group_kernel_info<T, 1, 32, kTurned>(slot0 + 1);
    return group_kernel_info<T, 1, 64, kTurned>(slot0 + 2);
  }
  if (mode == kSums) {
    if (bn == 64) return group_kernel_info<T, 1, 64, kSums>(slot0 + 3);
    if (bn == 128) return group_kernel_info<T, 1, 128, kSums>(slot0 + 4);
    return group_kernel_info<T, 2, 256, kSums>(slot0 + 5);
  }
  if (bn == 64) return group_kernel_info<T, 1, 64, kRows>(slot0 + 6);
  if (bn == 128) return group_kernel_info<T, 1, 128, kRows>(slot0 + 7);
  return group_kernel_info<T, 2, 256, kRows>(slot0 + 8);
}

}  // namespace grp
}  // namespace pic
